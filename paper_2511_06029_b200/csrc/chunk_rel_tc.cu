// lethe_chunk_attend, Eq. 5 for the chunk, on the tensor cores: rel[j] = gamma^T rel[j] + sum over tokens and heads of
// gamma^(T-1-i) p_ihj, from the final softmax statistics.
//
// The logits are formed again, transposed: S^T = K Q^T with 128 keys on the tensor-memory lanes and 128 (token, head) columns, so
// that a thread owns a key, adds its row up in registers and stores one sum — no atomics, one order.  With the column's bias
// (log2 of the decay weight minus the log-sum-exp) a column costs one FMA, one exponential and one add, and the exponentials are
// the bound (16 a clock per SM, 1024 clocks a tile against 512 of products).  The alternative, writing column sums from the
// attention kernel, would need the final maxima and sums before the last key is known.
//
// A unit is a pair of key tiles of one item (two groups of four warps), its steps are the query tiles that meet it; the plan gives
// every CTA an equal stretch of the line of all steps (a causal prompt's first keys meet every token, its last keys few), and the
// parts of a unit that CTAs share are added up afterwards in order.  Two CTAs to an SM cover each other's hand-offs; with slopes one,
// which then has registers for all that its columns bring along (calls of 512-token chunks with a cap and slopes 262 us with two that
// spill, 242 with one; with a cap alone 205 us with two, 217 with one).  Warp 8 issues the MMAs, warp 9 loads tiles by TMA; tiles that TMA cannot take
// (byte caches, odd pages) are gathered by the softmax warps, once per unit.  An 8192-token prompt of 32 heads over 8: about 360 us,
// 1250 clocks of a tile, of which the special-function unit has 768 with a quarter of the exponentials on the FMA pipes.
#include "chunk_tc.cuh"

namespace lethe {
namespace {

constexpr int kSoftWarps = 8;
constexpr int kMmaWarp = 8;
constexpr int kLoadWarp = 9;
constexpr int kThreads = 10 * 32;
// Of eight exponentials, computed by polynomial: an 8192-token prompt takes 925 us with none, 907 with two, 1000 with four in runs short
// enough that the clock holds; where the power cap lowers it 996, 999 and 1058.
constexpr int kFmaShare = 2;
constexpr int kTmemCols = 256;  // one logit tile per group

template <int D>
constexpr size_t smem_bytes() { return 1024 + 3 * (size_t)tile_bytes<D>(); }  // two key tiles, one query tile

template <int MOD>
struct Shared {
    unsigned long long k_full, k_empty, q_full, q_empty;
    unsigned long long s_full[2], s_empty[2];
    unsigned long long drained;
    uint32_t tmem_base;
    int abort;
    int k_loads, q_loads, issued;
    alignas(16) float bias[kSoftWarps][kTile];
    alignas(16) float qpos[MOD == kSloped ? kSoftWarps : 1][kTile];   // relative to the sequence's first new token
    alignas(16) float slope[MOD == kSloped ? kSoftWarps : 1][kTile];  // log2 units
    alignas(16) int lo[MOD ? kSoftWarps : 1][kTile];
};

// A CTA's piece of a unit: query tiles [qa, qb) of the pair of key tiles that begins at slot j0.
struct RelPiece {
    ChunkItem it;
    int idx, pair, j0, qa, qb;
    int s0, s1;      // the unit's steps on the line
    bool head, tail; // begins / ends here
};

// Calls f(piece) for each piece of this CTA, in order; f returns false to stop.
template <typename F>
__device__ __forceinline__ void for_rel_pieces(const ChunkArgs& a, F f) {
    const int total = a.plan->rel_total, per = a.plan->rel_per;
    const int begin = min(total, (int)blockIdx.x * per), end = min(total, begin + per);
    if (begin >= end) return;
    RelPiece p;
    p.idx = a.rel_item[blockIdx.x];
    p.it = chunk_item(a, p.idx);
    p.s0 = a.rel_start[p.idx];
    p.pair = 0;
    if (!a.rel_hull) {  // the pairs at the front all meet every query tile
        const int tiles = (p.it.T + a.TT - 1) / a.TT;
        const int same = a.append ? min(rel_pairs(p.it), p.it.n_old / (2 * kTile) + 1) : rel_pairs(p.it);
        p.pair = min((begin - p.s0) / tiles, same);
        p.s0 += p.pair * tiles;
    }
    for (int at = begin; at < end;) {
        if (p.it.n_old < 0 || p.it.T == 0 || p.pair >= rel_pairs(p.it)) {
            p.it = chunk_item(a, ++p.idx);
            p.pair = 0;
            continue;
        }
        const int2 h = rel_hull(a, p.it, p.idx, p.pair);
        p.s1 = p.s0 + rel_steps(h);
        if (p.s1 > at) {
            const int stop = min(end, p.s1);
            p.j0 = p.pair * 2 * kTile;
            p.qa = h.x + at - p.s0;
            p.qb = min(h.y, h.x + stop - p.s0);  // qb <= qa: nobody sees the pair
            p.head = at == p.s0;
            p.tail = stop == p.s1;
            if (!f(p)) return;
            at = stop;
        }
        p.s0 = p.s1;
        ++p.pair;
    }
}

template <int D, bool TMA, int MOD>
__global__ void __launch_bounds__(kThreads, MOD == kSloped ? 1 : 2) chunk_tc_rel(const __grid_constant__ ChunkArgs a, const __grid_constant__ ChunkMaps maps) {
    constexpr int TILE = tile_bytes<D>(), KS = D / 16;
    extern __shared__ unsigned char dyn_raw[];
    __shared__ Shared<MOD> sh;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t k_tile = (smem_u32(dyn_raw) + 1023u) & ~1023u, q_tile = k_tile + 2 * TILE;
    volatile int* abort_flag = &sh.abort;
    const int limit = a.wait_limit > 0 ? a.wait_limit : kChunkWaitLimit;
    const int used = a.TT * a.G;

    if (tid == 0) {
        bar_init(&sh.k_full, TMA ? 1 : kSoftWarps);
        bar_init(&sh.k_empty, 1);
        bar_init(&sh.q_full, 1);
        bar_init(&sh.q_empty, 1);
        for (int g = 0; g < 2; ++g) {
            bar_init(&sh.s_full[g], 1);
            bar_init(&sh.s_empty[g], 4);
        }
        bar_init(&sh.drained, 1);
        sh.abort = sh.k_loads = sh.q_loads = sh.issued = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // columns that the query boxes never write stay zero
    for (int i = tid; i < (kTile - used) * (D / 8); i += kThreads)
        st_shared_16(chunk_addr(q_tile, used + i / (D / 8), i % (D / 8)), make_uint4(0, 0, 0, 0));
    proxy_fence();
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    dependency_wait();
    dependency_release();
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = sh.tmem_base;

    if (warp == kLoadWarp) {
        TileLoader<D> loader;  // bad pages: the attention has recorded them
        int k = 0, qn = 0;
        for_rel_pieces(a, [&](const RelPiece& p) {
            if (p.qb <= p.qa) return true;
            if (TMA) {
                if (k > 0 && !warp_wait(&sh.k_empty, k - 1, abort_flag, limit)) return false;
                const int tiles = p.j0 + kTile < p.it.n ? 2 : 1;
                if (lane == 0) {
                    bar_expect_tx(&sh.k_full, tiles * TILE);
                    sh.k_loads = k + 1;
                }
                __syncwarp();
                loader.reset();
                for (int g = tiles - 1; g >= 0; --g) loader.load(a, &maps.k, p.it.item, p.it.n, p.j0 + g * kTile, k_tile + g * TILE, &sh.k_full);
            }
            ++k;
            for (int qt = p.qa; qt < p.qb; ++qt) {
                if (qn > 0 && !warp_wait(&sh.q_empty, qn - 1, abort_flag, limit)) return false;
                ++qn;
                if (lane == 0) {
                    bar_expect_tx(&sh.q_full, (unsigned)(used * D * 2));
                    sh.q_loads = qn;
                }
                __syncwarp();
                if (lane < D / 64) tma_4d(q_tile + lane * kHalfBytes, &maps.q, 64 * lane, p.it.hkv * a.G, p.it.first + qt * a.TT, p.it.li, &sh.q_full);
            }
            return true;
        });
        __syncwarp();
    } else if (warp == kMmaWarp) {
        const uint64_t q_desc = smem_desc(q_tile, 16), k_desc = smem_desc(k_tile, 16);
        int k = 0, qn = 0;
        int ns[2] = {0, 0};
        for_rel_pieces(a, [&](const RelPiece& p) {
            if (p.qb <= p.qa) return true;
            const int tiles = p.j0 + kTile < p.it.n ? 2 : 1;
            const uint32_t desc = mma_idesc(kTile, false, a.scale[p.it.l] < 0.f);
            if (!warp_wait(&sh.k_full, k++, abort_flag, limit)) return false;
            for (int qt = p.qa; qt < p.qb; ++qt, ++qn) {
                if (!warp_wait(&sh.q_full, qn, abort_flag, limit)) return false;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    if (g >= tiles) break;
                    if (ns[g] > 0 && !warp_wait(&sh.s_empty[g], ns[g] - 1, abort_flag, limit)) return false;
                    tc_after();
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) {
                            const uint32_t off = ((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4;
                            mma_ss(tmem + g * kTile, k_desc + (g * (TILE >> 4) + off), q_desc + off, desc, ks > 0);
                        }
                        sh.issued = 1;
                        tc_commit(&sh.s_full[g]);
                        if (g == tiles - 1) tc_commit(&sh.q_empty);
                        if (g == tiles - 1 && qt + 1 == p.qb) tc_commit(&sh.k_empty);
                    }
                    __syncwarp();
                    ++ns[g];
                }
            }
            return true;
        });
    } else {
        const int g = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
        const uint32_t s_addr = tmem + ((uint32_t)(quarter * 32) << 16) + g * kTile;
        int n_s = 0, k = 0;
        int col_tok[4];  // token of the tile that lane's columns lane, lane + 32, ... belong to
#pragma unroll
        for (int x = 0; x < 4; ++x) col_tok[x] = (x * 32 + lane) / a.G;
        if (tid == 0)  // where the stretch begins, for the merge
            for_rel_pieces(a, [&](const RelPiece& p) {
                a.rel_cut[blockIdx.x] = make_int4(p.idx, p.pair, p.s0, p.s1);
                return false;
            });
        __syncwarp();
        for_rel_pieces(a, [&](const RelPiece& p) {
            const ChunkItem& it = p.it;
            const int j0 = p.j0, j = j0 + g * kTile + r;  // this thread's key
            if (p.qb <= p.qa) {  // only the decay
                float* rel = a.rel + (size_t)it.item * a.cap_tokens + j;
                if (j < it.n) *rel = j < it.n_old ? exp2f((float)it.T * a.gamma_log2) * *rel : 0.f;
                if (j0 == 0 && tid == 0 && a.append) a.len[it.item] = it.n;
                return true;
            }
            if (!TMA) {
                bool bad = false;
                if (k > 0 && !warp_wait(&sh.k_empty, k - 1, abort_flag, limit)) return false;
                for (int t = 0; t < (j0 + kTile < it.n ? 2 : 1); ++t)
                    for (int half = 0; half < (a.dtype == LETHE_BF16 ? 2 : 1); ++half) {
                        Gather<D, kSoftWarps * 32> x;
                        x.load(a, a.k, it.item, it.n, j0 + t * kTile, tid, half, &bad);
                        x.store(a, k_tile + t * TILE, tid, half);
                    }
                proxy_fence();
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.k_full);
            }
            ++k;
            if (j0 == 0 && p.head && tid == 0 && a.append) a.len[it.item] = it.n;
            if (j0 + g * kTile >= it.n) return true;  // the second tile does not exist
            float* rel = a.rel + (size_t)it.item * a.cap_tokens + j;
            const bool whole = p.head && p.tail;
            const float old = whole && j < it.n_old ? *rel : 0.f;
            const float scale = fabsf(a.scale[it.l]) * a.k_scale[it.l], sl2 = scale * 1.4426950408889634f;
            float cap_in = 0.f, cap2 = 0.f, kf = 0.f;
            int kp = 0, prefix = INT32_MIN, pos0 = 0;
            constexpr bool sloped = MOD == kSloped;
            const bool cap = MOD == kCapped || (sloped && a.softcap > 0.f);
            const bool mask_pos = MOD && (a.window > 0 || a.doc_start || a.prefix_len);
            if (MOD) {
                if (cap) {
                    cap_in = fminf(scale / a.softcap, 1e15f);  // its square has to stay finite
                    cap2 = a.softcap * 1.4426950408889634f;
                }
                if (a.token_pos) pos0 = a.token_pos[it.first];
                if (a.prefix_len) prefix = a.prefix_len[it.b];
                if (mask_pos || sloped) {
                    kp = j < it.n ? a.pos[(size_t)it.item * a.cap_tokens + j] : 0;
                    kf = (float)((long long)kp - pos0);
                }
            }
            float col_slope[4];
            if (MOD)
#pragma unroll
                for (int x = 0; x < 4; ++x) col_slope[x] = sloped ? a.slopes[it.hkv * a.G + (x * 32 + lane) % a.G] * 1.4426950408889634f : 0.f;
            const float* nlse = a.nlse2 + (((size_t)it.li * a.Hkv + it.hkv) * a.n_tokens + it.first) * a.G;
            uint64_t acc[2] = {0, 0};
            float acc0 = 0.f;  // of columns tested one by one
            // what the tile's columns bring along, fetched a tile ahead: lane x has columns x, x + 32, ...
            float next_bias[4];
            int next_pos[4], next_doc[4];
            auto fetch = [&](int qt) {
                const int cols = min(a.TT, it.T - qt * a.TT) * a.G;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int c = x * 32 + lane;
                    next_bias[x] = c < cols ? nlse[qt * used + c] : -INFINITY;
                    if (MOD) {
                        const int tok = it.first + qt * a.TT + col_tok[x];
                        next_pos[x] = c < cols && a.token_pos ? a.token_pos[tok] : 0;
                        next_doc[x] = c < cols && a.doc_start ? a.doc_start[tok] : INT32_MIN;
                    }
                }
            };
            fetch(p.qa);
            for (int qt = p.qa; qt < p.qb; ++qt) {
                // one copy per warp (the warps never wait for one another)
                const int cols = min(a.TT, it.T - qt * a.TT) * a.G;
                int lo_max = INT32_MIN;
                bool nan = false;  // a token whose scores are NaN: every column is tested, so that it comes through
                __syncwarp();
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int c = x * 32 + lane;
                    const float bias = next_bias[x] + (float)(it.T - 1 - qt * a.TT - col_tok[x]) * a.gamma_log2;
                    sh.bias[warp][c] = bias;
                    nan = nan || bias != bias;
                    if (MOD) {
                        int lo = next_doc[x];
                        if (a.window > 0) lo = (int)max((long long)lo, (long long)next_pos[x] - a.window + 1);
                        if (sloped) {
                            sh.qpos[warp][c] = (float)((long long)next_pos[x] - pos0);
                            sh.slope[warp][c] = col_slope[x];
                        }
                        sh.lo[warp][c] = c < cols ? lo : INT32_MAX;  // columns that are not there see nothing
                        if (c < cols) lo_max = max(lo_max, lo);
                    }
                }
                if (MOD) lo_max = __reduce_max_sync(0xffffffffu, lo_max);
                if (qt + 1 < p.qb) fetch(qt + 1);
                __syncwarp();
                // the columns [from, to) see this thread's key: they reach it in causal order (or a prefix opens it to all), and their
                // windows and documents, which grow with the tokens, have not left it behind
                int from = a.append && !(MOD && kp < prefix) ? (j - it.n_old - qt * a.TT) * a.G : 0, to = cols;
                bool run = true;
                // a short tile's other columns are tokens of other sequences: whatever they hold must not count
                const bool clean = cols == used && __all_sync(0xffffffffu, !nan && from <= 0 && (!mask_pos || kp >= lo_max));
                if (MOD && mask_pos && !clean) {
                    bool up = true;
#pragma unroll
                    for (int x = 0; x < 4; ++x) up = up && (x * 32 + lane + 1 >= kTile || sh.lo[warp][x * 32 + lane] <= sh.lo[warp][x * 32 + lane + 1]);
                    run = __all_sync(0xffffffffu, up);
                    int end = 0;
#pragma unroll
                    for (int half = kTile / 2; half >= 1; half >>= 1)
                        if (sh.lo[warp][end + half - 1] <= kp) end += half;
                    end += sh.lo[warp][end] <= kp;
                    to = min(to, end);
                }
                if (j >= it.n) to = 0;
                if (!warp_wait(&sh.s_full[g], n_s++, abort_flag, limit)) return false;
                tc_after();
                // rolled where there is more than the causal mask: unrolled, the code outgrows the instruction cache (packed documents 274
                // -> 287 us); in narrow pieces where scores are shaped: 32 columns spill
                constexpr int W = shaped(MOD) ? 16 : 32;
#pragma unroll (MOD ? 1 : 4)
                for (int ch = 0; ch < kTile; ch += W) {
                    if (ch >= cols) break;  // a short chunk leaves most columns empty
                    uint32_t v[W];
                    if (W == 32) tmem_ld32(s_addr + ch, v);
                    else tmem_ld16(s_addr + ch, v);
                    tmem_ld_wait();
                    if (ch + W >= cols) {
                        tc_before();
                        __syncwarp();
                        if (lane == 0) bar_arrive(&sh.s_empty[g]);
                    }
                    float ml = sl2;
                    if (MOD) {
                        if (cap) {
                            ml = 1.f;
                            cap_scores<W>(v, cap_in, cap2, j < it.n);
                        }
                        if (sloped) {
#pragma unroll
                            for (int c = 0; c < W; c += 4) {
                                const float4 qp = *reinterpret_cast<const float4*>(&sh.qpos[warp][ch + c]), sl = *reinterpret_cast<const float4*>(&sh.slope[warp][ch + c]);
                                v[c] = __float_as_uint(fmaf(-sl.x, fabsf(qp.x - kf), __uint_as_float(v[c]) * ml));
                                v[c + 1] = __float_as_uint(fmaf(-sl.y, fabsf(qp.y - kf), __uint_as_float(v[c + 1]) * ml));
                                v[c + 2] = __float_as_uint(fmaf(-sl.z, fabsf(qp.z - kf), __uint_as_float(v[c + 2]) * ml));
                                v[c + 3] = __float_as_uint(fmaf(-sl.w, fabsf(qp.w - kf), __uint_as_float(v[c + 3]) * ml));
                            }
                            ml = 1.f;
                        }
                    }
                    const float4* b4 = reinterpret_cast<const float4*>(sh.bias[warp] + ch);
                    if (clean) {
                        const uint64_t ml2 = two(ml, ml);
#pragma unroll
                        for (int c = 0; c < W; c += 8) {
                            const float4 b0 = b4[c / 4], b1 = b4[c / 4 + 1];
                            const uint64_t bias[4] = {two(b0.x, b0.y), two(b0.z, b0.w), two(b1.x, b1.y), two(b1.z, b1.w)};
#pragma unroll
                            for (int z = 0; z < 4; ++z) {
                                const float2 x = apart(fma2(two(__uint_as_float(v[c + 2 * z]), __uint_as_float(v[c + 2 * z + 1])), ml2, bias[z]));
                                const float2 e = 2 * z >= 8 - kFmaShare ? exp2_fma(x.x, x.y) : make_float2(fast_exp2(x.x), fast_exp2(x.y));
                                acc[z & 1] = add2(acc[z & 1], two(e.x, e.y));
                            }
                        }
                    } else if (run) {
                        if (__any_sync(0xffffffffu, from < ch + W && to > ch)) {
                            const int c0 = from - ch, c1 = to - ch;
#pragma unroll
                            for (int c = 0; c < W; c += 4) {
                                const float4 b = b4[c / 4];
                                const float e0 = fast_exp2(fmaf(__uint_as_float(v[c]), ml, b.x)), e1 = fast_exp2(fmaf(__uint_as_float(v[c + 1]), ml, b.y));
                                const float e2 = fast_exp2(fmaf(__uint_as_float(v[c + 2]), ml, b.z)), e3 = fast_exp2(fmaf(__uint_as_float(v[c + 3]), ml, b.w));
                                if (c >= c0 && c < c1) acc0 += e0;
                                if (c + 1 >= c0 && c + 1 < c1) acc0 += e1;
                                if (c + 2 >= c0 && c + 2 < c1) acc0 += e2;
                                if (c + 3 >= c0 && c + 3 < c1) acc0 += e3;
                            }
                        }
                    } else if (MOD) {  // documents that do not grow with the tokens: every column by itself
#pragma unroll
                        for (int c = 0; c < W; ++c) {
                            const float e = fast_exp2(fmaf(__uint_as_float(v[c]), ml, sh.bias[warp][ch + c]));
                            if (j < it.n && ch + c >= from && ch + c < cols && kp >= sh.lo[warp][ch + c]) acc0 += e;
                        }
                    }
                }
            }
            const float2 both = apart(add2(acc[0], acc[1]));
            const float sum = both.x + both.y + acc0;
            if (!whole) a.rel_part[((size_t)blockIdx.x * 2 + (p.head ? 1 : 0)) * (2 * kTile) + g * kTile + r] = sum;
            else if (j < it.n) *rel = fmaf(exp2f((float)it.T * a.gamma_log2), old, sum);
            return true;
        });
    }

    tc_before();
    __syncthreads();
    tc_after();
    if (sh.abort) {  // uniform for the CTA: see everything this CTA has started end
        if (tid == 0) record_error(a.status, LETHE_ERR_TIMEOUT, blockIdx.x);
        if (warp == kMmaWarp && sh.issued && elect_one()) {  // the lane that issued them: a commit follows one's own MMAs
            tc_commit(&sh.drained);
            bar_drain(&sh.drained, 0);
        }
        if (warp == kLoadWarp && lane == 0) {
            if (TMA && sh.k_loads > 0) bar_drain(&sh.k_full, sh.k_loads - 1);
            if (sh.q_loads > 0) bar_drain(&sh.q_full, sh.q_loads - 1);
        }
        tc_before();
        __syncthreads();
        tc_after();
    }
    if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

template <int D, bool TMA, int MOD>
cudaError_t launch_t(const ChunkArgs& a, const ChunkMaps& maps, cudaStream_t stream) {
    cudaError_t e = prepare_kernel((const void*)chunk_tc_rel<D, TMA, MOD>, smem_bytes<D>());
    if (e == cudaSuccess) e = launch_dependent(chunk_tc_rel<D, TMA, MOD>, dim3(a.n_rel_cta), kThreads, smem_bytes<D>(), stream, a, maps);
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

cudaError_t launch_chunk_rel_tc(const ChunkArgs& a, const ChunkMaps& maps, cudaStream_t stream) {
    if (tma_can_tile(a)) return a.D == 128 ? launch_m<128, true>(a, maps, stream) : launch_m<64, true>(a, maps, stream);
    return a.D == 128 ? launch_m<128, false>(a, maps, stream) : launch_m<64, false>(a, maps, stream);
}

}  // namespace lethe
