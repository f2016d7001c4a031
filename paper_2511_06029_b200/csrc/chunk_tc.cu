// lethe_chunk_attend, the attention itself, on the fifth-generation tensor cores (bf16 and byte caches).
//
// S = Q K^T and O += P V with tcgen05.mma: the 128 x 128 fp32 logits and the 128 x D outputs live in tensor memory, the softmax
// threads read a row each, write the probabilities back as bf16 over the logits they came from, and those are the A operand of the
// second product where they lie.  A CTA holds two row tiles (two softmax groups of four warps) and each has a warp of its own that
// issues its products, so one group's exponentials run under the other's products and neither waits for the other's hand-offs.
// A job is 64 keys of one group, half a tile, and a group's logits have two buffers: the logits of job n + 1 are there before job
// n's probabilities are done, so a group's softmax does not wait for its products.  (A product with 64 columns takes as long as one
// with 128, it is bound by reading Q; with one 128-column buffer the softmax stood still for the products and the two hand-offs,
// 1700 of a tile's 4900 clocks.)  Row maxima are followed lazily: the outputs are rescaled only when a maximum has grown by more
// than 2^8 since the last time, which a row's first few tiles settle; the sums stay far inside fp32.
//
// What the two groups work on depends on the unit:
//   pair  two row tiles: a group each, the same keys
//   alt   one row tile: the groups take alternate key tiles and merge at the end
//   quad  at most 16 rows (single tokens, drafted tokens): the rows are put into the tile four times, once per 32 lanes of tensor
//         memory, and each of a group's four warps takes every fourth run of 16 keys (its probabilities of the others' keys are
//         zero): all eight warps work instead of two, and the eight parts merge at the end
//
// Roles: warps 0-7 softmax; warps 8 and 9 issue the MMAs; warp 10 fetches the query tiles; warp 11 K and V tiles by TMA (one thread)
// or, for byte caches and odd page sizes, warps 11-14 read, convert and store them (exact: e4m3 and e5m2 are bf16 values).  K and V
// tiles alternate in a ring.  Negative scales flip the sign of Q inside the MMA.
//
// Measured (bf16, 32 query over 8 KV heads of 128): an 8192-token prompt in 525 us, 1.05 PFLOP/s on the two products, 0.64 of a large
// GEMM's rate; 512 tokens behind 1024 of 8 sequences 105 us.  A step of a pair takes about 3950 clocks: 2950 are the tensor pipe's (the
// 64-column products bound by reading Q), the rest is where both groups' exponentials (1000 of a 64-column job) and hand-offs do
// not fit under it.  (A quarter of the exponentials on the FMA pipes, as in the relevance kernel, gained nothing
// here and cost code.)
//
// Roundings: the probabilities to bf16 (the products' operands share a type; half a step is 2^-8 of a weight, and the sum l is taken
// before, in fp32), the outputs to bf16 last.
#include <string.h>

#include "chunk_tc.cuh"

namespace lethe {
namespace {

constexpr int kSoftWarps = 8;
constexpr int kMmaWarp = 8;      // and 9: one per group
constexpr int kQWarp = 10;
constexpr int kLoadWarp = 11;    // TMA
constexpr int kGatherWarp = 11;  // four warps
constexpr int kMaxStages = 8;
constexpr int kQuadRows = kChunkQuadRows;
constexpr float kLazy = 8.f;  // log2 of the growth of a row maximum that is left standing

template <bool TMA>
__host__ __device__ constexpr int tc_threads() { return (TMA ? kLoadWarp + 1 : kGatherWarp + 4) * 32; }
template <int D>
__host__ __device__ constexpr int stages() { return D == 128 ? 4 : 8; }
template <int D>
constexpr size_t smem_bytes() { return 1024 + (size_t)(2 + stages<D>()) * tile_bytes<D>(); }

template <int MOD>
struct Shared {
    unsigned long long full[kMaxStages], empty[kMaxStages];
    unsigned long long q_full, q_done, q_soft, merge, merge_all;
    unsigned long long s_full[2][2], p_full[2][2], o_full[2][2];  // [group][buffer]: logits, probabilities, output product
    unsigned long long drained[2];
    uint32_t tmem_base;
    int abort;
    int loaded, q_loaded, issued[2];  // ring entries, query loads and MMAs started (for the drain after a timeout)
    float2 merge_ml[kTile];
    alignas(16) int kpos[MOD ? kSoftWarps : 1][kTile];     // positions of the tile's keys, one copy per warp
    alignas(16) float kposf[MOD ? kSoftWarps : 1][kTile];  // the same relative to the unit's first query
    alignas(16) unsigned char turn[kSoftWarps][32][80];     // 32 columns of a warp's output rows on their way out (rows 16 bytes apart in the banks)
};

template <int N>
struct Width {
    static constexpr int value = N;
};

// A CTA's piece of a unit, as every role derives it from the plan.
struct Piece {
    ChunkItem it;
    int idx;         // item of the call
    int tok0, toks;  // tokens of the unit
    int tile0, nt;   // key tiles
    int hi;          // slots from here on are hidden from the whole unit
    bool alt;        // one row tile, the groups take alternate key tiles (quad included)
    bool quad;       // at most 16 rows
    bool head, tail; // begins / ends here
};

__device__ __forceinline__ Piece piece_of(const ChunkArgs& a, int u, int at, int stop, int s0, int s1) {
    Piece p;
    p.idx = u / a.QT;
    p.tok0 = (u - p.idx * a.QT) * a.TU;
    p.it = chunk_item(a, p.idx);
    p.toks = min(p.it.T - p.tok0, a.TU);
    p.hi = a.u_hi ? a.u_hi[u] : (a.append ? p.it.n_old + p.tok0 + p.toks : p.it.n_old);
    const int before = tiles_before(a, p.toks, s0, at);
    p.tile0 = (a.u_lo ? a.u_lo[u] : 0) + before;
    p.nt = tiles_before(a, p.toks, s0, stop) - before;
    p.alt = p.toks <= a.TT;
    p.quad = p.toks * a.G <= kQuadRows;
    p.head = before == 0;
    p.tail = stop == s1;
    return p;
}

// A piece's tiles are taken last first: the nearest keys of a causal row, which a distance bias favours, set its maximum at once
// (first to last, steep slopes made it grow, and the outputs be rescaled, with every job: 7000 clocks of each).  Job n of a group is
// half 1 - (n & 1) of its (n / 2)-th tile; jobs run from first_job to job_end.
__device__ __forceinline__ int seq_tile(const Piece& p, int s) { return p.tile0 + p.nt - 1 - s; }
// Where the piece's last tile has nothing to see in its second half, that job is left out.
__device__ __forceinline__ int first_job(const Piece& p, int g) { return (!p.alt || g == 0) && p.hi - (p.tile0 + p.nt - 1) * kTile <= 64; }
__device__ __forceinline__ int job_end(const Piece& p, int g) { return p.alt ? 2 * ((p.nt - g + 1) >> 1) : 2 * p.nt; }
__device__ __forceinline__ int job_seq(const Piece& p, int g, int n) { return p.alt ? 2 * (n >> 1) + g : n >> 1; }

// Ring entries of a piece's tiles, by their place in that order.  A pair goes through K and V of one tile at a time; with alternate tiles both groups' K come first
// (a group needs its next K before the other has let its V go: in the ring's order K0 V0 K1 V1 four slots would lock up).
__device__ __forceinline__ int k_entry(const Piece& p, int t) { return p.alt ? 4 * (t >> 1) + (t & 1) : 2 * t; }
__device__ __forceinline__ int v_entry(const Piece& p, int t) { return p.alt ? 4 * (t >> 1) + min(2, p.nt - (t & ~1)) + (t & 1) : 2 * t + 1; }
__device__ __forceinline__ int entry_tile(const Piece& p, int e, bool& is_v) {
    if (!p.alt) {
        is_v = e & 1;
        return e >> 1;
    }
    const int both = min(2, p.nt - 2 * (e >> 2)), rem = e & 3;
    is_v = rem >= both;
    return 2 * (e >> 2) + (is_v ? rem - both : rem);
}

// A wait for a ring entry looks at one bit of the slot's phase, so the waiter has to know that the slot's entry before has landed:
// it has used that one itself, or a piece lies between.  The V of a last tile without a partner is the exception, it follows a K
// of the other group; whoever waits for it first sees that the loader has got to it (which it does only once that K is used).
__device__ __forceinline__ bool lone_v(const Piece& p, int t) { return p.alt && t + 1 == p.nt && !(t & 1); }
__device__ __forceinline__ bool wait_issued(volatile int* loaded, int e, volatile int* abort_flag, int limit) {
    bool ok = *loaded > e;
    for (int it = 1; !ok && it < limit && !*abort_flag; ++it) ok = *loaded > e;
    if (!ok) *abort_flag = 1;
    return __all_sync(0xffffffffu, ok);
}

// Calls f(piece) for each piece of this CTA, in order; f returns false to stop.
template <typename F>
__device__ __forceinline__ void for_pieces(const ChunkArgs& a, F f) {
    const int total = a.plan->total, per = a.plan->per;
    const int begin = min(total, (int)blockIdx.x * per), end = min(total, begin + per);
    if (begin >= end) return;
    int u = a.cta_unit[blockIdx.x], s0 = a.u_start[u];
    for (int at = begin; at < end; ++u) {
        const int s1 = a.u_start[u + 1];
        if (s1 > at) {
            const int stop = min(end, s1);
            const Piece p = piece_of(a, u, at, stop, s0, s1);
            if (p.nt > 0 && !f(p)) return;
            at = stop;
        }
        s0 = s1;
    }
}

template <int D, bool TMA, int MOD>
__global__ void __launch_bounds__(tc_threads<TMA>(), 1) chunk_tc_attend(const __grid_constant__ ChunkArgs a, const __grid_constant__ ChunkMaps maps) {
    constexpr int TILE = tile_bytes<D>(), NS = stages<D>(), KS = D / 16;
    constexpr int kOCol = 256;  // tensor memory: S0 | S1 | O0 | O1, 128 columns each (two buffers of logits each, P over its logits)
    extern __shared__ unsigned char dyn_raw[];
    __shared__ Shared<MOD> sh;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t q_tile = (smem_u32(dyn_raw) + 1023u) & ~1023u;
    const uint32_t ring = q_tile + 2 * TILE;
    unsigned char* const q_generic = dyn_raw + (q_tile - smem_u32(dyn_raw));
    volatile int* abort_flag = &sh.abort;
    const int limit = a.wait_limit > 0 ? a.wait_limit : kChunkWaitLimit;
    const int used = a.TT * a.G;

    if (tid == 0) {
        for (int i = 0; i < NS; ++i) {
            bar_init(&sh.full[i], TMA ? 1 : 4);
            bar_init(&sh.empty[i], 2);
        }
        bar_init(&sh.q_full, 1);
        bar_init(&sh.q_done, 2);
        bar_init(&sh.q_soft, kSoftWarps);
        bar_init(&sh.merge, 4);
        bar_init(&sh.merge_all, kSoftWarps);
        for (int g = 0; g < 2; ++g) {
            for (int hf = 0; hf < 2; ++hf) {
                bar_init(&sh.s_full[g][hf], 1);
                bar_init(&sh.p_full[g][hf], 4);
                bar_init(&sh.o_full[g][hf], 1);
            }
            bar_init(&sh.drained[g], 1);
        }
        sh.abort = sh.loaded = sh.q_loaded = sh.issued[0] = sh.issued[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    dependency_wait();
    dependency_release();
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = sh.tmem_base;

    if (warp >= kLoadWarp) {
        // ------------------------------------------------------------------ K and V tiles
        int e = 0;
        if (TMA) {
            TileLoader<D> loader;
            int item = -1;
            for_pieces(a, [&](const Piece& p) {
                if (p.it.item != item) loader.reset();
                item = p.it.item;
                for (int t = 0; t < 2 * p.nt; ++t, ++e) {
                    const int s = e % NS;
                    if (e >= NS && !warp_wait(&sh.empty[s], e / NS - 1, abort_flag, limit)) return false;
                    if (lane == 0) {
                        bar_expect_tx(&sh.full[s], TILE);
                        *(volatile int*)&sh.loaded = e + 1;
                    }
                    __syncwarp();
                    bool is_v;
                    const int tile = seq_tile(p, entry_tile(p, t, is_v));
                    loader.load(a, is_v ? &maps.v : &maps.k, p.it.item, p.it.n, tile * kTile, ring + s * TILE, &sh.full[s]);
                }
                if (loader.bad) record_error(a.status, LETHE_ERR_PAGE, p.it.item);
                loader.bad = false;
                return true;
            });
        } else {
            bool bad = false;
            // bf16 tiles take two register tiles; the next one's loads are under way while this one waits for its slot
            const int gt = tid - kGatherWarp * 32, halves = a.dtype == LETHE_BF16 ? 2 : 1;
            for_pieces(a, [&](const Piece& p) {
                Gather<D, 128> now, next;
                auto load = [&](Gather<D, 128>& x, int i) {  // i-th register tile of the piece
                    bool is_v;
                    const int tile = seq_tile(p, entry_tile(p, i / halves, is_v));
                    x.load(a, is_v ? a.v : a.k, p.it.item, p.hi, tile * kTile, gt, i % halves, &bad);
                };
                load(now, 0);
                for (int i = 0; i < 2 * p.nt * halves; ++i) {
                    if (i + 1 < 2 * p.nt * halves) load(next, i + 1);
                    const int s = e % NS;
                    if (i % halves == 0) {
                        if (e >= NS && !warp_wait(&sh.empty[s], e / NS - 1, abort_flag, limit)) return false;
                        if (gt == 0) *(volatile int*)&sh.loaded = e + 1;
                    }
                    now.store(a, ring + s * TILE, gt, i % halves);
                    if ((i + 1) % halves == 0) {
                        proxy_fence();
                        __syncwarp();
                        if (lane == 0) bar_arrive(&sh.full[s]);
                        ++e;
                    }
                    now = next;
                }
                if (bad) record_error(a.status, LETHE_ERR_PAGE, p.it.item);
                bad = false;
                return true;
            });
        }
    } else if (warp == kQWarp) {
        // ------------------------------------------------------------------ query tiles
        if (lane == 0) {
            int k = 0;
            for_pieces(a, [&](const Piece& p) {
                // the previous unit's products have read the tiles, and its softmax groups are done with them as merge space
                if (k > 0 && (!bar_wait(&sh.q_done, k - 1, abort_flag, limit) || !bar_wait(&sh.q_soft, k - 1, abort_flag, limit))) return false;
                const int copies = p.quad ? 4 : p.alt ? 1 : 2;
                const CUtensorMap* map = p.quad ? &maps.q16 : &maps.q;
                bar_expect_tx(&sh.q_full, (unsigned)(copies * (p.quad ? kQuadRows / a.G * a.G : used) * D * 2));
                sh.q_loaded = k + 1;
                for (int c = 0; c < copies; ++c)
#pragma unroll
                    for (int hf = 0; hf < D / 64; ++hf)
                        tma_4d(q_tile + (p.quad ? c * 32 * 128 : c * TILE) + hf * kHalfBytes, map, 64 * hf, p.it.hkv * a.G, p.it.first + p.tok0 + (p.quad ? 0 : c * a.TT), p.it.li, &sh.q_full);
                ++k;
                return true;
            });
        }
        __syncwarp();
    } else if (warp >= kMmaWarp) {
        // ------------------------------------------------------------------ MMA issue: the warp waits as one, one lane issues
        const int g = warp - kMmaWarp;
        const uint32_t pv_desc = mma_idesc(D, true, false);
        const uint64_t q_desc = smem_desc(q_tile, 16), k_desc = smem_desc(ring, 16), v_desc = smem_desc(ring, kHalfBytes);
        const uint32_t st = tmem + g * 128, ot = tmem + kOCol + g * 128;
        int k = 0, base = 0;           // pieces done, first ring entry of the piece
        unsigned np0 = 0, np1 = 0;     // probabilities consumed so far, per buffer
        for_pieces(a, [&](const Piece& p) {
            const uint32_t qk_desc = mma_idesc(64, false, a.scale[p.it.l] < 0.f);
            const uint64_t qd = q_desc + (uint64_t)((p.alt ? 0 : g) * (TILE >> 4));
            const int n0 = first_job(p, g), end = job_end(p, g);
            if (!warp_wait(&sh.q_full, k, abort_flag, limit)) return false;
            // a tile's ring entry is let go by both groups, or twice by the one that uses it
            auto let_go = [&](int slot) {
                tc_commit(&sh.empty[slot]);
                if (p.alt) tc_commit(&sh.empty[slot]);
            };
            auto qk = [&](int n) -> bool {
                const int buf = n & 1, e = base + k_entry(p, job_seq(p, g, n)), slot = e % NS;
                if (!warp_wait(&sh.full[slot], e / NS, abort_flag, limit)) return false;
                tc_after();
                if (elect_one()) {
                    const uint64_t kd = k_desc + (uint64_t)(slot * (TILE >> 4) + (1 - buf) * (64 * 128 >> 4));
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        constexpr int half16 = kHalfBytes >> 4;
                        mma_ss(st + buf * 64, qd + (ks >> 2) * half16 + (ks & 3) * 2, kd + (ks >> 2) * half16 + (ks & 3) * 2, qk_desc, ks > 0);
                    }
                    sh.issued[g] = 1;
                    tc_commit(&sh.s_full[g][buf]);
                    if (buf == 1) let_go(slot);
                    if (n + 1 == end) tc_commit(&sh.q_done);
                }
                __syncwarp();
                return true;
            };
            if (n0 < end && !qk(n0)) return false;
            if (n0 + 1 < end && !qk(n0 + 1)) return false;
            if (n0 >= end && elect_one()) tc_commit(&sh.q_done);
            __syncwarp();
            for (int n = n0; n < end; ++n) {
                const int buf = n & 1, half = 1 - buf, t = job_seq(p, g, n), e = base + v_entry(p, t), slot = e % NS;
                if (buf == 0 || n == n0) {
                    if (lone_v(p, t) && !wait_issued(&sh.loaded, e, abort_flag, limit)) return false;
                    if (!warp_wait(&sh.full[slot], e / NS, abort_flag, limit)) return false;
                }
                const int steps = max(1, (min(64, p.hi - seq_tile(p, t) * kTile - 64 * half) + 15) / 16);
                const uint64_t vd = v_desc + (uint64_t)(slot * (TILE >> 4) + half * (64 * 128 >> 4));
                if (!warp_wait(&sh.p_full[g][buf], buf ? np1++ : np0++, abort_flag, limit)) return false;
                tc_after();
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        if (ks < steps) mma_ts(ot, st + 64 * buf + ks * 8, vd + (uint64_t)(ks * (2048 >> 4)), pv_desc, n > n0 || ks > 0);
                    tc_commit(&sh.o_full[g][buf]);
                    if (buf == 1) let_go(slot);
                }
                __syncwarp();
                if (n + 2 < end && !qk(n + 2)) return false;
            }
            base += 2 * p.nt;
            ++k;
            return true;
        });
    } else {
        // ------------------------------------------------------------------ softmax
        const int g = warp >> 2, quarter = warp & 3;
        const uint32_t s_addr = tmem + ((uint32_t)(quarter * 32) << 16) + g * 128;
        const uint32_t o_addr = s_addr + kOCol;
        constexpr bool sloped = MOD == kSloped;
        const bool cap = MOD == kCapped || (sloped && a.softcap > 0.f);
        const bool by_pos = MOD && (sloped || a.window > 0 || a.doc_start || a.prefix_len);
        const bool mask_pos = MOD && (a.window > 0 || a.doc_start || a.prefix_len);
        float* const merge_o = reinterpret_cast<float*>(q_generic);  // parts to merge, where the query tiles were
        unsigned s0 = 0, s1 = 0, o0 = 0, o1 = 0;  // logits taken and products asked for so far, per buffer
        int n_v = 0, k = 0, n_m = 0, n_q = 0;     // ring entries so far; pieces, merged pieces, quad pieces
        for_pieces(a, [&](const Piece& p) {
            const int r = p.quad ? lane : quarter * 32 + lane;  // row of the tile
            const int tile_rows = p.quad ? p.toks * a.G : min(used, p.toks * a.G - (p.alt ? 0 : g * used));
            const bool valid_row = r < tile_rows;
            const bool busy = p.quad || quarter * 32 < tile_rows;  // the warp has rows at all
            const int tok = p.tok0 + (p.alt ? 0 : g * a.TT) + min(r, tile_rows - 1) / a.G, h = r % a.G;
            // a scale of zero is a very small one here, so that a hidden key's -inf stays one
            const float scale = fabsf(a.scale[p.it.l]) * a.k_scale[p.it.l], sl2 = fmaxf(scale * 1.4426950408889634f, 1e-36f);
            // rows that are not there count as seeing everything: they never ask for a mask
            const int lim = valid_row && a.append ? p.it.n_old + tok + 1 : INT32_MAX;
            int lo = INT32_MIN, pos0 = 0, prefix = INT32_MIN;
            float slope = 0.f, qf = 0.f, cap_in = 0.f, cap2 = 0.f;
            if (MOD) {
                int qpos = 0;
                if (a.token_pos) {
                    qpos = a.token_pos[p.it.first + tok];
                    pos0 = a.token_pos[p.it.first + p.tok0];
                    qf = (float)((long long)qpos - pos0);
                }
                if (valid_row) lo = chunk_lo(a, p.it.first + tok, qpos);
                if (a.prefix_len) prefix = a.prefix_len[p.it.b];
                if (sloped) slope = a.slopes[p.it.hkv * a.G + h] * 1.4426950408889634f;
                if (cap) {
                    cap_in = fminf(scale / a.softcap, 1e15f);  // its square has to stay finite
                    cap2 = a.softcap * 1.4426950408889634f;
                }
            }
            // what a logit has to be multiplied by, once shaped, to be in log2 units
            const float ml = cap || sloped ? 1.f : sl2;
            float m = -INFINITY, l = 0.f;
            const int n0 = first_job(p, g), end = job_end(p, g);
            int kp_min, from = 0, to = 0;  // masks by position, per tile
            bool clean = true, run = true;
            int kp_next[4];  // positions of the next tile's keys, fetched a tile ahead
            auto fetch_pos = [&](int t) {
                const int j0 = seq_tile(p, t) * kTile;
                const int32_t* pos = a.pos + (size_t)p.it.item * a.cap_tokens + j0;
#pragma unroll
                for (int c = 0; c < 4; ++c) kp_next[c] = j0 + c * 32 + lane < p.it.n ? pos[c * 32 + lane] : INT32_MAX;
            };
            // A group without a job here (one key tile, alternate tiles) would see nothing of the piece before its merge, and after a pair,
            // whose end it does not wait for either, q_done's phase before the piece's could still be open: its wait would pass at
            // once, and the group's arrivals on merge and q_soft would count for a piece too early.  The queries come after both.
            if (n0 >= end && !warp_wait(&sh.q_full, k, abort_flag, limit)) return false;
            if (MOD && by_pos && busy && n0 < end) fetch_pos(job_seq(p, g, n0));
            for (int n = n0; n < end; ++n) {
                const int buf = n & 1, half = 1 - buf, t = job_seq(p, g, n), j0 = seq_tile(p, t) * kTile;
                if (MOD && by_pos && busy && (buf == 0 || n == n0)) {  // while the product runs
                    kp_min = INT32_MAX;
                    __syncwarp();
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int kp = kp_next[c];
                        sh.kpos[warp][c * 32 + lane] = kp;
                        sh.kposf[warp][c * 32 + lane] = (float)((long long)kp - pos0);
                        kp_min = min(kp_min, kp);
                    }
                    __syncwarp();
                    const int ahead = (n | 1) + 1;
                    if (ahead < end) fetch_pos(job_seq(p, g, ahead));
                    if (mask_pos) {
                        kp_min = __reduce_min_sync(0xffffffffu, kp_min);
                        const int nn = p.it.n - j0;
                        clean = __all_sync(0xffffffffu, kp_min >= lo && lim - j0 >= kTile && nn >= kTile);
                        if (!clean) {
                            // Positions that grow with the slot (any cache that was only appended to and pruned): what a row sees of
                            // the tile is a run of columns [from, to), found by halving.  Else every key is tested by itself.
                            bool up = true;
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                const int x = c * 32 + lane;
                                up = up && (x + 1 >= kTile || sh.kpos[warp][x] <= sh.kpos[warp][x + 1]);
                            }
                            run = __all_sync(0xffffffffu, up);
                            from = 0;
                            int opened = 0;  // keys before the prefix's end
#pragma unroll
                            for (int by = kTile / 2; by >= 1; by >>= 1) {
                                if (sh.kpos[warp][from + by - 1] < lo) from += by;
                                if (sh.kpos[warp][opened + by - 1] < prefix) opened += by;
                            }
                            from += sh.kpos[warp][from] < lo;
                            opened += sh.kpos[warp][opened] < prefix;
                            to = lim == INT32_MAX ? nn : max(lim - j0, min(opened, nn));
                        }
                    }
                }
                if (!warp_wait(&sh.s_full[g][buf], buf ? s1++ : s0++, abort_flag, limit)) return false;
                tc_after();
                const int seen = p.hi - j0 - 64 * half;  // keys of this half that the unit sees at all
                if (seen < 64 && (seen <= 0 || (seen & 15))) {
                    // Rows behind the last slot may hold anything, and 0 x NaN is NaN: clear those the product's last step takes in.
                    // Not before the logits are there: they show that the product two jobs back, and with it the ring slot's last
                    // entry, is done (a wait that is a whole turn of the ring early would take the last entry's phase for this one's).
                    const int e = n_v + v_entry(p, t), r0 = 64 * half + max(seen, 0), rows = 64 * half + max(16, (seen + 15) & ~15) - r0;
                    if (lone_v(p, t) && !wait_issued(&sh.loaded, e, abort_flag, limit)) return false;
                    if (!warp_wait(&sh.full[e % NS], e / NS, abort_flag, limit)) return false;
                    for (int x = quarter * 32 + lane; x < rows * (D / 8); x += kTile) st_shared_16(chunk_addr(ring + (e % NS) * TILE, r0 + x / (D / 8), x % (D / 8)), make_uint4(0, 0, 0, 0));
                    proxy_fence();
                }
                // NC logits of the thread's row from column c0 of the tile: the whole half, or a quad warp's share of it
                auto job = [&](auto width) -> bool {
                    constexpr int NC = decltype(width)::value;
                    const int c0 = 64 * half + (NC == 64 ? 0 : NC * quarter);
                    const uint32_t s_buf = s_addr + 64 * buf;
                    uint32_t v[NC], pk[32];
                    if (MOD) {
                        // Scores are shaped sixteen columns at a time and put back: unrolled over the whole row the code outgrows the
                        // instruction cache (a job took 8000 clocks instead of 2500).
                        const float in = cap ? 1.f : sl2;
                        const int nv = min(lim, p.it.n) - j0;
                        const bool masked = mask_pos ? !clean : __any_sync(0xffffffffu, nv < c0 + NC);
                        if ((masked && mask_pos && !run) || cap || sloped) {
#pragma unroll 1
                            for (int c = 0; c < NC; c += 16) {
                                const uint32_t at = s_buf + (NC == 64 ? c : NC * quarter);
                                uint32_t w[16];
                                tmem_ld16(at, w);
                                tmem_ld_wait();
                                if (cap) cap_scores<16>(w, cap_in, cap2, valid_row);
                                if (sloped) {
#pragma unroll
                                    for (int y = 0; y < 16; y += 4) {
                                        const float4 kf = *reinterpret_cast<const float4*>(&sh.kposf[warp][c0 + c + y]);
                                        w[y] = __float_as_uint(fmaf(-slope, fabsf(qf - kf.x), __uint_as_float(w[y]) * in));
                                        w[y + 1] = __float_as_uint(fmaf(-slope, fabsf(qf - kf.y), __uint_as_float(w[y + 1]) * in));
                                        w[y + 2] = __float_as_uint(fmaf(-slope, fabsf(qf - kf.z), __uint_as_float(w[y + 2]) * in));
                                        w[y + 3] = __float_as_uint(fmaf(-slope, fabsf(qf - kf.w), __uint_as_float(w[y + 3]) * in));
                                    }
                                }
                                if (masked) {
                                    if (!mask_pos || run) {
                                        const int y0 = (mask_pos ? from : 0) - c0 - c, y1 = (mask_pos ? to : nv) - c0 - c;
#pragma unroll
                                        for (int y = 0; y < 16; ++y)
                                            if (y < y0 || y >= y1) w[y] = 0xff800000u;
                                    } else {
                                        const int nn = p.it.n - j0 - c0 - c, nl = lim == INT32_MAX ? nn : lim - j0 - c0 - c;
#pragma unroll
                                        for (int y = 0; y < 16; ++y) {
                                            const int kp = sh.kpos[warp][c0 + c + y];
                                            if (!((y < nl || (kp < prefix && y < nn)) && kp >= lo)) w[y] = 0xff800000u;
                                        }
                                    }
                                }
                                tmem_st16(at, w);
                            }
                            tmem_st_wait();
                        }
                    }
                    if (NC == 64) {
                        tmem_ld32(s_buf, v);
                        tmem_ld32(s_buf + 32, v + (NC == 64 ? 32 : 0));
                    } else tmem_ld16(s_buf + NC * quarter, v);
                    tmem_ld_wait();
                    if (!MOD) {
                        const int nv = min(lim, p.it.n) - j0 - c0;  // of these keys the row sees so many
                        if (__any_sync(0xffffffffu, nv < NC)) {
#pragma unroll
                            for (int c = 0; c < NC; ++c)
                                if (c >= nv) v[c] = 0xff800000u;
                        }
                    } else if (mask_pos && !clean && run && !(cap || sloped)) {  // a run, and nothing else to shape
                        const int y0 = from - c0, y1 = to - c0;
                        if (__any_sync(0xffffffffu, y0 > 0 || y1 < NC)) {
#pragma unroll
                            for (int c = 0; c < NC; ++c)
                                if (c < y0 || c >= y1) v[c] = 0xff800000u;
                        }
                    }
                    if (NC == 16 && a.park && valid_row) {
                        float4* d = reinterpret_cast<float4*>(a.park + ((size_t)p.idx * a.park_rows + r) * a.park_pitch + j0 + c0);
#pragma unroll
                        for (int y = 0; y < 16; y += 4)
                            d[y / 4] = make_float4(__uint_as_float(v[y]) * ml, __uint_as_float(v[y + 1]) * ml, __uint_as_float(v[y + 2]) * ml, __uint_as_float(v[y + 3]) * ml);
                    }
                    float m0 = __uint_as_float(v[0]), m1 = __uint_as_float(v[1]);
#pragma unroll
                    for (int c = 2; c + 3 < NC; c += 4) {
                        m0 = max3(m0, __uint_as_float(v[c]), __uint_as_float(v[c + 1]));
                        m1 = max3(m1, __uint_as_float(v[c + 2]), __uint_as_float(v[c + 3]));
                    }
                    const float mt = max3(max3(m0, m1, m1), __uint_as_float(v[NC - 2]), __uint_as_float(v[NC - 1])) * ml;
                    const bool grow = valid_row && !(mt <= m + kLazy);  // true from -inf, and for a NaN, which the row then keeps
                    if (__any_sync(0xffffffffu, grow)) {
                        const float w = grow ? exp2_diff(m, mt) : 1.f;
                        if (grow) m = mt;
                        l *= w;
                        if (n > n0) {  // the product of the job before may still be adding
                            if (!warp_wait(&sh.o_full[g][buf ^ 1], (buf ? o0 : o1) - 1, abort_flag, limit)) return false;
                            tc_after();
#pragma unroll 1
                            for (int c = 0; c < D; c += 32) {
                                tmem_ld32(o_addr + c, pk);
                                tmem_ld_wait();
#pragma unroll
                                for (int y = 0; y < 32; ++y) pk[y] = __float_as_uint(__uint_as_float(pk[y]) * w);
                                tmem_st32(o_addr + c, pk);
                            }
                        }
                    }
                    const uint64_t ml2 = two(ml, ml), nm2 = m == -INFINITY ? 0 : two(-m, -m);
                    uint64_t la = 0, lb = 0;
#pragma unroll
                    for (int y = 0; y < NC; y += 8) {
                        float p[8];
#pragma unroll
                        for (int z = 0; z < 8; z += 2) {
                            const float2 x = apart(fma2(two(__uint_as_float(v[y + z]), __uint_as_float(v[y + z + 1])), ml2, nm2));
                            p[z] = fast_exp2(x.x);
                            p[z + 1] = fast_exp2(x.y);
                        }
                        la = add2(add2(la, two(p[0], p[1])), two(p[4], p[5]));
                        lb = add2(add2(lb, two(p[2], p[3])), two(p[6], p[7]));
#pragma unroll
                        for (int z = 0; z < 8; z += 2) pk[(y + z) / 2] = pack_bf16(p[z], p[z + 1]);
                    }
                    const float2 sum = apart(add2(la, lb));
                    l += sum.x + sum.y;
                    if (NC == 64) tmem_st32(s_buf, pk);
                    else {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            uint32_t z[8];
#pragma unroll
                            for (int y = 0; y < 8; ++y) z[y] = q == quarter ? pk[y] : 0u;
                            tmem_st8(s_buf + 8 * q, z);
                        }
                    }
                    tmem_st_wait();
                    return true;
                };
                if (p.quad) {
                    if (!job(Width<16>())) return false;
                } else if (busy) {
                    if (!job(Width<64>())) return false;
                }
                if (buf) ++o1;
                else ++o0;
                tc_before();
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.p_full[g][buf]);
            }
            n_v += 2 * p.nt;
            // ---- the piece's outputs
            const bool worked = n0 < end;
            if (worked && !warp_wait(&sh.o_full[g][1], o1 - 1, abort_flag, limit)) return false;  // the last job is a first half, buffer 1
            tc_after();
            const bool whole = p.head && p.tail;
            const size_t part = ((size_t)blockIdx.x * 2 + (p.head ? 1 : 0)) * 2 + (p.alt ? 0 : g);
            __nv_bfloat16* const out0 = (__nv_bfloat16*)a.out + (((size_t)p.it.li * a.n_tokens + p.it.first) * a.Hq + p.it.hkv * a.G) * D;
            auto row_stats = [&](int token, int head, int row, float mr, float lr) {
                if (!whole) a.part_ml[part * kChunkPartRows + row] = make_float2(mr, lr);
                else {
                    const float lse2 = lr == 0.f ? -INFINITY : mr + log2f(lr);
                    if (a.lse) a.lse[((size_t)p.it.li * a.n_tokens + p.it.first + token) * a.Hq + p.it.hkv * a.G + head] = lse2 * 0.6931471805599453f;
                    a.nlse2[(((size_t)p.it.li * a.Hkv + p.it.hkv) * a.n_tokens + p.it.first + token) * a.G + head] = lr == 0.f ? -INFINITY : -lse2;
                }
            };
            if (p.quad) {
                // eight parts [warp][D][16 rows]; then every warp finishes D / 8 columns of all rows
                if (!warp_wait(&sh.q_done, k, abort_flag, limit)) return false;
                if (lane < kQuadRows) sh.merge_ml[warp * kQuadRows + lane] = make_float2(m, l);
                if (worked) {
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        uint32_t o[32];
                        tmem_ld32(o_addr + c, o);
                        tmem_ld_wait();
                        if (lane < kQuadRows)
#pragma unroll
                            for (int y = 0; y < 32; ++y) merge_o[(warp * D + c + y) * kQuadRows + lane] = __uint_as_float(o[y]);
                    }
                }
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.merge_all);
                if (!warp_wait(&sh.merge_all, n_q++, abort_flag, limit)) return false;
                constexpr int NE = D / 16;
                const int row = lane & (kQuadRows - 1), d0 = warp * (D / 8) + (lane >> 4) * NE;
                if (row < tile_rows) {
                    float mx = -INFINITY, lt = 0.f, acc[NE] = {};
#pragma unroll
                    for (int i = 0; i < kSoftWarps; ++i) mx = fmaxf(mx, sh.merge_ml[i * kQuadRows + row].x);
#pragma unroll
                    for (int i = 0; i < kSoftWarps; ++i) {
                        const float2 part_i = sh.merge_ml[i * kQuadRows + row];
                        const float w = exp2_diff(part_i.x, mx);
                        lt += part_i.y * w;
                        if (w != 0.f)
#pragma unroll
                            for (int e = 0; e < NE; ++e) acc[e] = fmaf(merge_o[(i * D + d0 + e) * kQuadRows + row], w, acc[e]);
                    }
                    const int token = p.tok0 + row / a.G, head = row % a.G;
                    if (whole) {
                        const float inv = lt == 0.f ? 0.f : a.v_scale[p.it.l] / lt;
                        uint32_t w[NE / 2];
#pragma unroll
                        for (int e = 0; e < NE; e += 2) w[e / 2] = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
                        __nv_bfloat16* d = out0 + ((size_t)token * a.Hq + head) * D + d0;
                        if (NE == 8) *reinterpret_cast<uint4*>(d) = make_uint4(w[0], w[1], w[NE / 2 - 2], w[NE / 2 - 1]);
                        else *reinterpret_cast<uint2*>(d) = make_uint2(w[0], w[1]);
                    } else {
#pragma unroll
                        for (int e = 0; e < NE; ++e) a.part_o[(part * D + d0 + e) * kChunkPartRows + row] = acc[e];
                    }
                    if (d0 == 0) row_stats(token, head, row, mx, lt);
                }
            } else {
                if (p.alt) {
                    if (g == 1) {
                        if (!warp_wait(&sh.q_done, k, abort_flag, limit)) return false;
                        if (busy) {
                            sh.merge_ml[r] = make_float2(m, l);
                            if (worked) {
#pragma unroll 1
                                for (int c = 0; c < D; c += 32) {
                                    uint32_t o[32];
                                    tmem_ld32(o_addr + c, o);
                                    tmem_ld_wait();
#pragma unroll
                                    for (int y = 0; y < 32; ++y) merge_o[(c + y) * kTile + r] = __uint_as_float(o[y]);
                                }
                            }
                        }
                        __syncwarp();
                        if (lane == 0) bar_arrive(&sh.merge);
                    } else if (!warp_wait(&sh.merge, n_m, abort_flag, limit)) return false;
                    ++n_m;
                }
                if (busy && !(p.alt && g == 1)) {
                    float w0 = 1.f, w1 = 0.f;
                    if (p.alt) {
                        const float2 other = sh.merge_ml[r];
                        const float mx = fmaxf(m, other.x);
                        w0 = exp2_diff(m, mx);
                        w1 = exp2_diff(other.x, mx);
                        l = l * w0 + other.y * w1;
                        m = mx;
                    }
                    const float mul = !whole ? 1.f : (l == 0.f ? 0.f : a.v_scale[p.it.l] / l);
                    const float mine = l == 0.f ? 0.f : w0 * mul, others = l == 0.f ? 0.f : w1 * mul;
                    __nv_bfloat16* dst[4];  // where the rows go that this lane writes a piece of
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const int row = quarter * 32 + y * 8 + (lane >> 2), tk = p.tok0 + (p.alt ? 0 : g * a.TT) + row / a.G;
                        dst[y] = row < tile_rows ? out0 + ((size_t)tk * a.Hq + row % a.G) * D + (lane & 3) * 8 : nullptr;
                    }
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        uint32_t o[32];
                        tmem_ld32(o_addr + c, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int y = 0; y < 32; ++y) {
                            // what nothing was added to may hold anything
                            o[y] = mine == 0.f ? 0u : __float_as_uint(__uint_as_float(o[y]) * mine);
                        }
                        if (p.alt && others != 0.f)
#pragma unroll
                            for (int y = 0; y < 32; ++y) o[y] = __float_as_uint(fmaf(merge_o[(c + y) * kTile + r], others, __uint_as_float(o[y])));
                        if (!whole) {
                            if (valid_row)
#pragma unroll
                                for (int y = 0; y < 32; ++y) a.part_o[(part * D + c + y) * kChunkPartRows + r] = __uint_as_float(o[y]);
                            continue;
                        }
                        // rows are turned through shared memory: four lanes then write 64 bytes of a row together
                        __syncwarp();
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const uint32_t* f = o + 8 * y;
                            *reinterpret_cast<uint4*>(&sh.turn[warp][lane][16 * y]) =
                                make_uint4(pack_bf16(__uint_as_float(f[0]), __uint_as_float(f[1])), pack_bf16(__uint_as_float(f[2]), __uint_as_float(f[3])),
                                           pack_bf16(__uint_as_float(f[4]), __uint_as_float(f[5])), pack_bf16(__uint_as_float(f[6]), __uint_as_float(f[7])));
                        }
                        __syncwarp();
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            if (dst[y]) *reinterpret_cast<uint4*>(dst[y] + c) = *reinterpret_cast<const uint4*>(&sh.turn[warp][y * 8 + (lane >> 2)][16 * (lane & 3)]);
                    }
                    if (valid_row) row_stats(tok, h, r, m, l);
                }
            }
            tc_before();   // O has been read: the next unit's first product may overwrite it (ordered by p_full)
            proxy_fence(); // the merge space goes back to the query loads
            __syncwarp();
            if (lane == 0) bar_arrive(&sh.q_soft);
            ++k;
            return true;
        });
    }

    tc_before();
    __syncthreads();
    tc_after();
    if (sh.abort) {  // uniform for the CTA: see everything this CTA has started end
        if (tid == 0) record_error(a.status, LETHE_ERR_TIMEOUT, blockIdx.x);
        if ((warp == kMmaWarp || warp == kMmaWarp + 1) && sh.issued[warp - kMmaWarp] && elect_one()) {  // the lane that issued them: a commit follows one's own MMAs
            tc_commit(&sh.drained[warp - kMmaWarp]);
            bar_drain(&sh.drained[warp - kMmaWarp], 0);
        }
        if (TMA && warp == kLoadWarp && lane == 0)
            for (int e = max(0, sh.loaded - NS); e < sh.loaded; ++e) bar_drain(&sh.full[e % NS], e / NS);
        if (warp == kQWarp && lane == 0 && sh.q_loaded > 0) bar_drain(&sh.q_full, sh.q_loaded - 1);
        tc_before();
        __syncthreads();
        tc_after();
    }
    if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

template <int D, bool TMA, int MOD>
cudaError_t launch_t(const ChunkArgs& a, const ChunkMaps& maps, cudaStream_t stream) {
    cudaError_t e = prepare_kernel((const void*)chunk_tc_attend<D, TMA, MOD>, smem_bytes<D>());
    if (e != cudaSuccess) return e;
    if (e == cudaSuccess) e = launch_dependent(chunk_tc_attend<D, TMA, MOD>, dim3(a.n_cta), tc_threads<TMA>(), smem_bytes<D>(), stream, a, maps);
    return e;
}

template <int D, bool TMA>
cudaError_t launch_m(const ChunkArgs& a, const ChunkMaps& maps, cudaStream_t stream) {
    switch (score_kind(a)) {
        case kPlain: return launch_t<D, TMA, kPlain>(a, maps, stream);
        case kMasked: return launch_t<D, TMA, kMasked>(a, maps, stream);
        case kCapped: return launch_t<D, TMA, kCapped>(a, maps, stream);
        default: return launch_t<D, TMA, kSloped>(a, maps, stream);
    }
}

}  // namespace

bool build_chunk_maps(void* encode, const ChunkArgs& a, int n_layers, ChunkMaps* maps) {
    typedef CUresult (*encode_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    encode_fn fn = reinterpret_cast<encode_fn>(encode);
    memset(maps, 0, sizeof(*maps));
    const cuuint32_t es[4] = {1, 1, 1, 1};
    const cuuint64_t D = a.D;
    const cuuint64_t qd[4] = {D, (cuuint64_t)a.Hq, (cuuint64_t)a.n_tokens, (cuuint64_t)a.nl};
    const cuuint64_t qs[3] = {D * 2, a.Hq * D * 2, (cuuint64_t)a.n_tokens * a.Hq * D * 2};
    const cuuint32_t qb[4] = {64, (cuuint32_t)a.G, (cuuint32_t)a.TT, 1};
    if (fn(&maps->q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(a.q), qd, qs, qb, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return false;
    const cuuint32_t qb16[4] = {64, (cuuint32_t)a.G, (cuuint32_t)(kQuadRows / a.G), 1};
    if (fn(&maps->q16, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(a.q), qd, qs, qb16, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return false;
    if (!tma_can_tile(a)) return true;
    const cuuint64_t rows = a.paged ? (cuuint64_t)a.page_tokens : (cuuint64_t)a.capacity;
    const cuuint64_t kd[3] = {D, rows, a.paged ? (cuuint64_t)a.n_pages : (cuuint64_t)n_layers * a.B * a.Hkv};
    const cuuint64_t ks[2] = {D * 2, rows * D * 2};
    const cuuint32_t kb[3] = {64, a.paged ? (cuuint32_t)a.page_tokens : (cuuint32_t)kTile, 1};
    for (int i = 0; i < 2; ++i)
        if (fn(i ? &maps->v : &maps->k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(i ? a.v : a.k), kd, ks, kb, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return false;
    return true;
}

cudaError_t launch_chunk_tc(const ChunkArgs& a, const ChunkMaps& maps, cudaStream_t stream) {
    if (tma_can_tile(a)) return a.D == 128 ? launch_m<128, true>(a, maps, stream) : launch_m<64, true>(a, maps, stream);
    return a.D == 128 ? launch_m<128, false>(a, maps, stream) : launch_m<64, false>(a, maps, stream);
}

}  // namespace lethe
