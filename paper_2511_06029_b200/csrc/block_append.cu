// lethe_block_append and lethe_block_read: filling a cache in 8 bits with a scale for each block of tokens, and reading it back.
// Measured (Llama-8B heads): a prompt of 8205 tokens, 184 MB, 45 us for the append = 4.1 TB/s; with the queries in a launch of their own 29 + 30
// us, since filling blocks is a chain of short steps (rows, angles, magnitude, codes, range) that a few resident blocks of threads go
// through at 1.7 TB/s: now the queries' stream runs beside it.  Single tokens of 8 sequences and 32 layers: 5 us, 22 where one of them fills
// blocks.  Reading 34 MB of rows back 9 us, 13 where the codes come from memory.
#include "block.cuh"

namespace lethe {
cudaError_t launch_append_len(const int32_t* chunk_start, int32_t* len, int B, int Hkv, int layer_begin, int n_items, int n_tokens, int max_chunk,
                              int cap_tokens, cudaStream_t stream);
namespace {

using bf16 = __nv_bfloat16;
constexpr int kQueryRows = 16, kManyQueryRows = 32, kQueryTokens = 2;
// Blocks to fill for each SM from which two heads share their angles.  Both sides at D = 128 (us, a head each first): 5.1 for each (752 in all)
// 21.5 and 23.7 with queries, 16.0 and 16.7 without; 8.2 35.2 and 34.3, 20.8 and 19.1; 13.9 54 and 51, 30 and 24; 27 98 and 90, 56 and 45.
constexpr int kPlenty = 8;
// Single tokens of this many items and more have a warp to an item, others a block of threads.  A warp's row is the cheaper one, a
// sequence that fills blocks the dearer one, since its heads' warps lie together.  On average over the steps of sequences in blocks of 32:
// 64 items 7 us with warps and 4.5 with blocks, 2048 items 10.4 and 10.2, 16384 items 42 and 54 (without a full block 6.7 and 9.4 of 2048
// items, with one sequence's 23 and 13).  Two and more tokens: 2048 items 9.4 to 31 us with warps, 10.2 to 16 with blocks.
constexpr int kManyItems = 2048;

// Magnitudes of two bf16 are two 16-bit whole numbers in the same order; from kNotFinite on they are infinities and NaN.
constexpr unsigned kNotFinite = 0x7f80;
__device__ __forceinline__ uint32_t top_of(const uint4& w, uint32_t top) {
    top = __vmaxu2(top, w.x & 0x7fff7fffu);
    top = __vmaxu2(top, w.y & 0x7fff7fffu);
    top = __vmaxu2(top, w.z & 0x7fff7fffu);
    return __vmaxu2(top, w.w & 0x7fff7fffu);
}
// The same without those that are not finite.
__device__ __noinline__ uint32_t finite_top_of(uint4 w, uint32_t top) {
    auto finite = [](uint32_t x) {
        x &= 0x7fff7fffu;
        return ((x & 0xffffu) >= kNotFinite ? 0u : x & 0xffffu) | (x >= kNotFinite << 16 ? 0u : x & 0xffff0000u);
    };
    return __vmaxu2(__vmaxu2(__vmaxu2(top, finite(w.x)), finite(w.y)), __vmaxu2(finite(w.z), finite(w.w)));
}
// Codes of eight values of at most the largest magnitude: 1.5 x 2^23 added to a product rounds it to the nearest whole number (ties to
// even), which the sum's lowest byte holds.
__device__ __forceinline__ uint2 codes8(const uint4& w, float inv) {
    float f[8];
    Piece<bf16>::unpack(w, f);
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = __float_as_uint(__fadd_rn(__fmul_rn(f[i], inv), 12582912.f));
    auto four = [](uint32_t a, uint32_t b, uint32_t x, uint32_t y) { return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(x, y, 0x0040), 0x5410); };
    return make_uint2(four(c[0], c[1], c[2], c[3]), four(c[4], c[5], c[6], c[7]));
}
// Of any eight: limited to -127 .. 127, NaN 0.
__device__ __noinline__ uint2 any_codes8(uint4 w, float inv) {
    float f[8];
    Piece<bf16>::unpack(w, f);
    uint32_t c[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i / 4] |= ((uint32_t)min(max(__float2int_rn(f[i] * inv), -127), 127) & 0xffu) << (8 * (i & 3));
    return make_uint2(c[0], c[1]);
}

// What a call does to an item.
struct Filled {
    int li, h, item;
    int s0, n0, n1;  // first new token; tokens before and after; n1 = 0: no tokens, -1: no room for them
};
__device__ __forceinline__ Filled filled(const BlockView& c, const NewRows& in, int idx) {
    const BlockItem it = block_item(c.layer_begin, c.B, c.Hkv, idx);
    Filled f = {it.li, it.h, it.item, in.chunk_start[it.b], 0, 0};
    const int n_new = max(in.chunk_start[it.b + 1] - f.s0, 0);  // before chunk_start has been looked over: it may hold anything
    f.n0 = block_len(c, it.item);
    if (n_new > 0 && f.n0 + (long long)n_new <= c.cap_tokens) f.n1 = f.n0 + n_new;
    else if (n_new > 0) f.n1 = -1;
    return f;
}

// Blocks of threads: first those of the items.
// FEW (calls of one token to a sequence, of many items): one to as many items as it has warps, since mostly a row goes to an open block, a
// warp's work; items that fill a block then have all warps, one after the other.
// Else: `units` to `heads` (1 .. 8) KV heads of a sequence, which share the cosines and sines of their tokens (where they have the same length, as
// they mostly do).  Unit u quantises the u-th of the blocks that the call fills; unit 0 also moves what is left over to the open block (it
// has read the rows that were there by then).
// The rest of the blocks rotate queries: kQueryRows rows of a token each (FEW), or kManyQueryRows of kQueryTokens tokens.  They lie between the
// others, one of those to every `stride` blocks: the queries' stream goes on while the others wait for one load after the other.
// Bound by memory: rows are read once and kept packed in registers between the search for the largest magnitude and the rounding.
template <int D, int TPT, bool VEC, bool FEW>  // TPT: tasks of 16 elements per thread, of K and of V
__global__ void __launch_bounds__(256, TPT == 1 ? 4 : TPT == 2 ? 3 : 2) block_append_kernel(const __grid_constant__ BlockView c, const __grid_constant__ NewRows in, int units, int heads, unsigned kv_blocks, unsigned stride) {
    extern __shared__ __align__(16) unsigned char tile[];  // [T][D] key codes; then cosines [T][D / 2] and sines of a block's new tokens
    float* cos_at = reinterpret_cast<float*>(tile + c.T * D);
    float* sin_at = cos_at + c.T * (D / 2);
    __shared__ __align__(16) float cs[FEW ? 8 : kQueryTokens][64], sn[FEW ? 8 : kQueryTokens][64];  // of the queries' tokens, or of a warp's row
    __shared__ unsigned tops[2][8];
    __shared__ uint32_t least[8][32], greatest[8][32];
    __shared__ Filled some[8];
    dependency_wait();
    dependency_release();
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, w = tid >> 5;
    constexpr int kPerRow = D / 16;
    const int half = in.rot_dim / 2;
    // the items of the block, one to a warp (FEW) or one after the other; their lengths are asked for together with chunk_start
    const unsigned turn_no = blockIdx.x / stride;
    const bool is_kv = turn_no * stride == blockIdx.x && turn_no < kv_blocks;
    const int groups = (c.Hkv + heads - 1) / heads, g = turn_no / units, u = turn_no - g * units;
    if (is_kv) {
        const int i = FEW ? w : tid;
        const int idx = FEW ? turn_no * (nt / 32) + i : g / groups * c.Hkv + g % groups * heads + i;
        if (FEW ? lane == 0 : i < heads) {
            some[i] = Filled{0, 0, 0, 0, 0, 0};
            if (FEW ? idx < c.n_items : g % groups * heads + i < c.Hkv) some[i] = filled(c, in, idx);
        }
    }
    if (!starts_ok(in.chunk_start, c.B, in.n_tokens, in.max_chunk, nullptr)) {
        if (blockIdx.x == 0 && tid == 0) record_error(c.status, LETHE_ERR_INVALID_ARG, 0);
        return;
    }
    // the pieces of a row's task; rotated by a row of cosines and sines
    auto load_row = [&](const bf16* src, int task, bool rotated, const float* co_row, const float* si_row, int& at0, int& at1, uint4& x, uint4& y) {
        if (VEC || !rotated) {
            bool turned;
            piece_pair<bf16>(in, task, rotated, at0, at1, turned);
            x = *reinterpret_cast<const uint4*>(src + at0);
            y = *reinterpret_cast<const uint4*>(src + at1);
        } else {
            load_by_element<bf16>(in, src, task, [&](int p, float& co, float& si) { co = co_row[p], si = si_row[p]; }, at0, at1, x, y);
        }
    };
    auto turn_row = [&](int task, const float* co_row, const float* si_row, uint4& x, uint4& y) {
        int at0, at1;
        bool turned;
        piece_pair<bf16>(in, task, true, at0, at1, turned);
        if (turned) {
            float co[8], si[8];
            look_up(co_row + first_pair(in, at0), co);
            look_up(si_row + first_pair(in, at0), si);
            turn_pieces<bf16>(in, x, y, co, si);
        }
    };
    if (!is_kv) {
        constexpr int TQ = FEW ? 1 : kQueryTokens, kRows = FEW ? kQueryRows : kManyQueryRows;
        const int rows_total = c.nl * c.Hq, per_tok = (rows_total + kRows - 1) / kRows;
        const int qb = blockIdx.x - min(turn_no + 1, kv_blocks), tok0 = qb / per_tok * TQ, r0 = qb % per_tok * kRows;
        const int first = in.chunk_start[0], last = in.chunk_start[c.B];
        for (int i = tid; i < TQ * 64; i += nt) {
            const int p = i & 63, ti = i >> 6;
            if (p < half && tok0 + ti < in.n_tokens) turn_by(turn_of(in, p), in.axis_pos[(size_t)axis_of(in, p) * in.n_tokens + tok0 + ti], cs[ti][p], sn[ti][p]);
        }
        const int tasks = min(rows_total - r0, kRows) * kPerRow;
        for (int t0 = 0; t0 < tasks; t0 += nt) {  // uniform for the block
            const int t = t0 + tid, r = r0 + t / kPerRow, li = r / c.Hq, task = t % kPerRow;
            const size_t off = (((size_t)li * in.n_tokens + tok0) * c.Hq + r - li * c.Hq) * D, pitch = (size_t)c.Hq * D;
            int at0 = 0, at1 = 0;
            uint4 x[TQ], y[TQ];
            bool there[TQ];
#pragma unroll
            for (int k = 0; k < TQ; ++k) {
                there[k] = t < tasks && tok0 + k >= first && tok0 + k < last;
                if (VEC && there[k]) load_row((const bf16*)in.q + off + k * pitch, task, true, nullptr, nullptr, at0, at1, x[k], y[k]);
            }
            if (t0 == 0) __syncthreads();  // the angles
#pragma unroll
            for (int k = 0; k < TQ; ++k)
                if (there[k]) {
                    if (VEC) turn_row(task, cs[k], sn[k], x[k], y[k]);
                    else load_row((const bf16*)in.q + off + k * pitch, task, true, cs[k], sn[k], at0, at1, x[k], y[k]);
                }
            if (!VEC) __syncwarp();  // q_out may be q: a row's tasks lie in one warp, all have read before one writes
#pragma unroll
            for (int k = 0; k < TQ; ++k)
                if (there[k]) {
                    bf16* to = (bf16*)in.q_out + off + k * pitch;
                    *reinterpret_cast<uint4*>(to + at0) = x[k];
                    *reinterpret_cast<uint4*>(to + at1) = y[k];
                }
        }
        return;
    }
    const bool rotated = in.axis_pos != nullptr;
    auto row_of = [&](const Filled& f, int slot) { return (((size_t)f.li * in.n_tokens + f.s0 + slot - f.n0) * c.Hkv + f.h) * D; };
    auto put = [&](const Filled& f, int slot, int at0, int at1, const uint4& kx, const uint4& ky, const uint4& vx, const uint4& vy) {
        const size_t off = ((size_t)f.item * c.T + (slot & (c.T - 1))) * D;
        *reinterpret_cast<uint4*>(c.k_open + off + at0) = kx;
        *reinterpret_cast<uint4*>(c.k_open + off + at1) = ky;
        *reinterpret_cast<uint4*>(c.v_open + off + at0) = vx;
        *reinterpret_cast<uint4*>(c.v_open + off + at1) = vy;
    };
    unsigned long long per_pos = 0;  // of pair tid % 64
    size_t axis_at = 0;
    if (rotated && (tid & 63) < half) {
        per_pos = turn_of(in, tid & 63);
        axis_at = (size_t)axis_of(in, tid & 63) * in.n_tokens;
    }
    // cosines and sines of the new tokens of slots s_first .. s_end - 1 of a block
    auto angles = [&](const Filled& f, int s_first, int s_end) {
        const int p = tid & 63, step = nt >> 6;
        if (p >= half) return;
        const int32_t* pos = in.axis_pos + axis_at + f.s0 - f.n0;
        int at = s_first + (tid >> 6) < s_end ? pos[s_first + (tid >> 6)] : 0;
#pragma unroll 1
        for (int slot = s_first + (tid >> 6); slot < s_end; slot += step) {
            const int next = slot + step < s_end ? pos[slot + step] : 0;
            const int to = (slot & (c.T - 1)) * (D / 2) + p;
            turn_by(per_pos, at, cos_at[to], sin_at[to]);
            at = next;
        }
    };
    // new rows from slot s_first on to the item's open block, by all threads
    auto to_open = [&](const Filled& f, int s_first) {
        if (s_first >= f.n1) return;
        if (rotated) {
            __syncthreads();
            angles(f, s_first, f.n1);
            __syncthreads();
        }
        for (int t = tid; t < (f.n1 - s_first) * kPerRow; t += nt) {
            const int slot = s_first + t / kPerRow, task = t % kPerRow, row = (slot & (c.T - 1)) * (D / 2);
            int at0, at1;
            uint4 kx, ky;
            load_row((const bf16*)in.k + row_of(f, slot), task, rotated, cos_at + row, sin_at + row, at0, at1, kx, ky);
            const bf16* v = (const bf16*)in.v + row_of(f, slot);
            const uint4 vx = *reinterpret_cast<const uint4*>(v + at0), vy = *reinterpret_cast<const uint4*>(v + at1);
            if (VEC && rotated) turn_row(task, cos_at + row, sin_at + row, kx, ky);
            put(f, slot, at0, at1, kx, ky, vx, vy);
        }
    };
    // a block that the call fills, by all threads; `known`: the angles of its new tokens are there already
    auto to_block = [&](const Filled& f, int blk, bool known) {
        const size_t open = (size_t)f.item * c.T;
        const int slot0 = blk << c.t_shift;
        uint4 kx[TPT], ky[TPT], vx[TPT], vy[TPT];
        auto fetch = [&]() {
#pragma unroll
            for (int i = 0; i < TPT; ++i) {
                const int t = tid + i * nt, r = t / kPerRow, task = t % kPerRow, slot = slot0 + r;
                int at0, at1;
                const bool old = slot < f.n0;
                const bf16* k = old ? c.k_open + (open + r) * D : (const bf16*)in.k + row_of(f, slot);
                const bf16* v = old ? c.v_open + (open + r) * D : (const bf16*)in.v + row_of(f, slot);
                if (VEC || !rotated || !old) {
                    load_row(k, task, rotated, cos_at + r * (D / 2), sin_at + r * (D / 2), at0, at1, kx[i], ky[i]);
                } else {  // the pieces as load_by_element takes them
                    at0 = 16 * task;
                    at1 = at0 + 8;
                    kx[i] = *reinterpret_cast<const uint4*>(k + at0);
                    ky[i] = *reinterpret_cast<const uint4*>(k + at1);
                }
                vx[i] = *reinterpret_cast<const uint4*>(v + at0);
                vy[i] = *reinterpret_cast<const uint4*>(v + at1);
            }
        };
        if (VEC || !rotated) fetch();
        __syncthreads();  // the tables of the block before have been read
        if (rotated && !known) {
            angles(f, max(slot0, f.n0), slot0 + c.T);
            __syncthreads();
        }
        if (!VEC && rotated) fetch();
        uint32_t packed_k = 0, packed_v = 0;
#pragma unroll
        for (int i = 0; i < TPT; ++i) {
            const int t = tid + i * nt, r = t / kPerRow;
            if (VEC && rotated && slot0 + r >= f.n0) turn_row(t % kPerRow, cos_at + r * (D / 2), sin_at + r * (D / 2), kx[i], ky[i]);
            packed_k = top_of(ky[i], top_of(kx[i], packed_k));
            packed_v = top_of(vy[i], top_of(vx[i], packed_v));
        }
        const long long page = block_page(c, f.item, blk);
        unsigned bits_k, bits_v;  // the largest magnitudes, as bf16
        auto over_block = [&]() {
            bits_k = __reduce_max_sync(0xffffffffu, max(packed_k & 0xffffu, packed_k >> 16));
            bits_v = __reduce_max_sync(0xffffffffu, max(packed_v & 0xffffu, packed_v >> 16));
            if (lane == 0) {
                tops[0][w] = bits_k;
                tops[1][w] = bits_v;
            }
            __syncthreads();
            for (int i = 0; i < nt / 32; ++i) {
                bits_k = max(bits_k, tops[0][i]);
                bits_v = max(bits_v, tops[1][i]);
            }
        };
        over_block();
        const bool any = max(bits_k, bits_v) >= kNotFinite;  // the same in all threads
        if (any) {
            packed_k = packed_v = 0;
#pragma unroll
            for (int i = 0; i < TPT; ++i) {
                packed_k = finite_top_of(ky[i], finite_top_of(kx[i], packed_k));
                packed_v = finite_top_of(vy[i], finite_top_of(vx[i], packed_v));
            }
            __syncthreads();  // the table has been read
            over_block();
        }
        const float top_k = __uint_as_float(bits_k << 16), top_v = __uint_as_float(bits_v << 16);
        if (page < 0) {
            if (tid == 0) record_error(c.status, LETHE_ERR_PAGE, f.item);
            return;
        }
        const float inv_k = top_k >= kBlockTiny ? __fdiv_rn(127.f, top_k) : 0.f, inv_v = top_v >= kBlockTiny ? __fdiv_rn(127.f, top_v) : 0.f;
        int8_t* kd = c.k + (size_t)page * c.T * D;
        int8_t* vd = c.v + (size_t)page * c.T * D;
#pragma unroll
        for (int i = 0; i < TPT; ++i) {
            const int t = tid + i * nt, r = t / kPerRow;
            int at0, at1;
            bool turned;
            piece_pair<bf16>(in, t % kPerRow, VEC && rotated, at0, at1, turned);
            uint2 a, b, x, y;
            if (any) {
                a = any_codes8(kx[i], inv_k), b = any_codes8(ky[i], inv_k);
                x = any_codes8(vx[i], inv_v), y = any_codes8(vy[i], inv_v);
            } else {
                a = codes8(kx[i], inv_k), b = codes8(ky[i], inv_k);
                x = codes8(vx[i], inv_v), y = codes8(vy[i], inv_v);
            }
            *reinterpret_cast<uint2*>(kd + r * D + at0) = a;
            *reinterpret_cast<uint2*>(kd + r * D + at1) = b;
            *reinterpret_cast<uint2*>(tile + r * D + at0) = a;
            *reinterpret_cast<uint2*>(tile + r * D + at1) = b;
            *reinterpret_cast<uint2*>(vd + r * D + at0) = x;
            *reinterpret_cast<uint2*>(vd + r * D + at1) = y;
        }
        if (tid == 0) {
            c.k_scale[page] = top_k >= kBlockTiny ? __fdiv_rn(top_k, 127.f) : 0.f;
            c.v_scale[page] = top_v >= kBlockTiny ? __fdiv_rn(top_v, 127.f) : 0.f;
        }
        if (!c.k_range) return;
        // four elements to a thread, the rows in turn among the groups of threads
        constexpr int W = D / 4;
        const int groups = nt / W, x4 = tid % W, gr = tid / W;
        __syncthreads();
        uint32_t lo = 0x7f7f7f7fu, hi = 0x81818181u;
        for (int r = gr; r < c.T; r += groups) {
            const uint32_t x = *reinterpret_cast<const uint32_t*>(tile + r * D + 4 * x4);
            lo = __vmins4(lo, x);
            hi = __vmaxs4(hi, x);
        }
        if (W == 16) {  // D = 64: two groups in a warp
            lo = __vmins4(lo, __shfl_xor_sync(0xffffffffu, lo, 16));
            hi = __vmaxs4(hi, __shfl_xor_sync(0xffffffffu, hi, 16));
        }
        least[w][lane] = lo;
        greatest[w][lane] = hi;
        __syncthreads();
        if (tid < W) {
            for (int g = 1; g < nt / 32; ++g) {
                lo = __vmins4(lo, least[g][x4]);
                hi = __vmaxs4(hi, greatest[g][x4]);
            }
            uint32_t* range = reinterpret_cast<uint32_t*>(c.k_range + (size_t)page * 2 * D);
            range[x4] = lo;
            range[W + x4] = hi;
        }
    };

    if constexpr (!FEW) {
        int known = -1;  // the length before the call of the item that the angles were made for
        for (int i = 0; i < heads; ++i) {
            const Filled f = some[i];
            const int b0 = f.n0 >> c.t_shift, b1 = f.n1 >> c.t_shift;
            if (f.n1 < 0 && u == 0 && tid == 0) record_error(c.status, LETHE_ERR_CAPACITY, f.item);
            if (f.n1 <= 0 || (u > 0 && b0 + u >= b1)) continue;
            if (b0 + u < b1) {
                to_block(f, b0 + u, known == f.n0);
                known = f.n0;
            }
            if (u == 0) {
                __syncthreads();  // the open rows have been read
                const int s_first = b1 > b0 ? b1 << c.t_shift : f.n0;
                if (s_first < f.n1) known = -1;
                to_open(f, s_first);
                if (units == 1 && tid == 0) c.len[f.item] = f.n1;  // no other block needs the item's old length
            }
        }
    } else {
        const Filled f = some[w];
        const bool fills = f.n1 > 0 && f.n1 >> c.t_shift > f.n0 >> c.t_shift;
        if (f.n1 < 0 && lane == 0) record_error(c.status, LETHE_ERR_CAPACITY, f.item);
        if (f.n1 > 0 && !fills) {
            if (rotated) {
                for (int p = lane; p < half; p += 32) turn_by(turn_of(in, p), in.axis_pos[(size_t)axis_of(in, p) * in.n_tokens + f.s0], cs[w][p], sn[w][p]);
                __syncwarp();
            }
            if (lane < kPerRow) {
                int at0, at1;
                uint4 kx, ky;
                load_row((const bf16*)in.k + row_of(f, f.n0), lane, rotated, cs[w], sn[w], at0, at1, kx, ky);
                const bf16* v = (const bf16*)in.v + row_of(f, f.n0);
                const uint4 vx = *reinterpret_cast<const uint4*>(v + at0), vy = *reinterpret_cast<const uint4*>(v + at1);
                if (VEC && rotated) turn_row(lane, cs[w], sn[w], kx, ky);
                put(f, f.n0, at0, at1, kx, ky, vx, vy);
            }
        }
        if (__syncthreads_or(fills))
            for (int i = 0; i < nt / 32; ++i) {
                const Filled o = some[i];
                if (o.n1 > 0 && o.n1 >> c.t_shift > o.n0 >> c.t_shift) to_block(o, o.n0 >> c.t_shift, false);  // its last token: nothing stays open
            }
        if (lane == 0 && f.n1 > 0) c.len[f.item] = f.n1;
    }
}

// A thread takes 8 elements, of K and of V, of kReadRows slots that lie a block of threads apart.
constexpr int kReadRows = 2;
template <int D>
__global__ void __launch_bounds__(256) block_read_kernel(const __grid_constant__ BlockView c, const int32_t* slot_begin, int n_slots, int per_item, bf16* k_out, bf16* v_out) {
    dependency_wait();
    dependency_release();
    constexpr int kPieces = D / 8, kApart = 256 / kPieces;
    const int idx = blockIdx.x / per_item, chunk = blockIdx.x - idx * per_item;
    const BlockItem it = block_item(c.layer_begin, c.B, c.Hkv, idx);
    const int n = block_len(c, it.item);
    const long long begin = slot_begin ? slot_begin[it.b] : 0;
    const int d = (threadIdx.x % kPieces) * 8, i0 = chunk * kReadRows * kApart + threadIdx.x / kPieces;
    long long page[kReadRows];
    uint4 x[kReadRows], y[kReadRows];
    float ks[kReadRows], vs[kReadRows];
#pragma unroll
    for (int u = 0; u < kReadRows; ++u) {
        const int i = i0 + u * kApart;
        const long long slot = begin + i;
        page[u] = -1;
        if (i < n_slots && slot >= 0 && slot < n >> c.t_shift << c.t_shift) {
            page[u] = block_page(c, it.item, (int)slot >> c.t_shift);
            if (page[u] < 0 && d == 0 && (i == 0 || ((int)slot & (c.T - 1)) == 0)) record_error(c.status, LETHE_ERR_PAGE, it.item);
        }
    }
#pragma unroll
    for (int u = 0; u < kReadRows; ++u) {
        const int i = i0 + u * kApart;
        const long long slot = begin + i;
        const int r = (int)slot & (c.T - 1);
        x[u] = y[u] = make_uint4(0, 0, 0, 0);
        if (page[u] >= 0) {
            const size_t off = ((size_t)page[u] * c.T + r) * D + d;
            const uint2 a = *reinterpret_cast<const uint2*>(c.k + off), b = *reinterpret_cast<const uint2*>(c.v + off);
            x[u].x = a.x, x[u].y = a.y, y[u].x = b.x, y[u].y = b.y;
            ks[u] = c.k_scale[page[u]];
            vs[u] = c.v_scale[page[u]];
        } else if (i < n_slots && slot >= n >> c.t_shift << c.t_shift && slot < n) {
            const size_t off = ((size_t)it.item * c.T + r) * D + d;
            x[u] = *reinterpret_cast<const uint4*>(c.k_open + off);
            y[u] = *reinterpret_cast<const uint4*>(c.v_open + off);
        }
    }
#pragma unroll
    for (int u = 0; u < kReadRows; ++u) {
        const int i = i0 + u * kApart;
        if (i >= n_slots) continue;
        if (page[u] >= 0) {
            float f[8], g[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t wa = e < 4 ? x[u].x : x[u].y, wb = e < 4 ? y[u].x : y[u].y;
                f[e] = (float)(int8_t)(wa >> (8 * (e & 3))) * ks[u];
                g[e] = (float)(int8_t)(wb >> (8 * (e & 3))) * vs[u];
            }
            x[u] = Piece<bf16>::pack(f);
            y[u] = Piece<bf16>::pack(g);
        }
        const size_t to = ((size_t)idx * n_slots + i) * D + d;
        *reinterpret_cast<uint4*>(k_out + to) = x[u];
        *reinterpret_cast<uint4*>(v_out + to) = y[u];
    }
}

struct Shape {
    int units, heads, threads;
    unsigned kv_blocks, grid, stride;
    bool few;
};
template <int D, int TPT>
cudaError_t launch_d(const BlockView& c, const NewRows& in, const Shape& sh, cudaStream_t stream) {
    const bool vec = !in.axis_pos || rotation_in_pieces<bf16>(in);
    const size_t smem = (size_t)c.T * D * (in.axis_pos ? 5 : 1);
    auto go = [&](auto kern) {
        const cudaError_t e = prepare_kernel((const void*)kern, smem);
        return e != cudaSuccess ? e : launch_dependent(kern, dim3(sh.grid), sh.threads, smem, stream, c, in, sh.units, sh.heads, sh.kv_blocks, sh.stride);
    };
    if (sh.few) return vec ? go(block_append_kernel<D, TPT, true, true>) : go(block_append_kernel<D, TPT, false, true>);
    return vec ? go(block_append_kernel<D, TPT, true, false>) : go(block_append_kernel<D, TPT, false, false>);
}

}  // namespace

cudaError_t launch_block_append(const BlockView& c, const NewRows& in, cudaStream_t stream) {
    const int tasks = c.T * c.D / 16, threads = min(256, tasks), per = tasks / threads, group = threads / 32;
    Shape sh;
    sh.threads = threads;
    sh.few = in.max_chunk == 1 && c.n_items >= kManyItems;
    // blocks that a sequence's tokens can fill: all but a last one that the call leaves open
    sh.units = max(1, (int)(((long long)in.max_chunk + c.T - 1) / c.T));
    const long long to_fill = (long long)c.nl * c.Hkv * (in.n_tokens / c.T + c.B);
    sh.heads = to_fill >= (long long)kPlenty * c.sm_count ? 2 : 1;
    sh.kv_blocks = sh.few ? (unsigned)((c.n_items + group - 1) / group) : (unsigned)c.nl * c.B * ((c.Hkv + sh.heads - 1) / sh.heads) * sh.units;
    const int q_tok = sh.few ? 1 : kQueryTokens, q_rows = sh.few ? kQueryRows : kManyQueryRows;
    sh.grid = sh.kv_blocks + (in.q ? (unsigned)((in.n_tokens + q_tok - 1) / q_tok) * (unsigned)((c.nl * c.Hq + q_rows - 1) / q_rows) : 0);
    sh.stride = sh.grid / sh.kv_blocks;
    cudaError_t e;
    if (c.D == 128) e = per == 1 ? launch_d<128, 1>(c, in, sh, stream) : per == 2 ? launch_d<128, 2>(c, in, sh, stream) : launch_d<128, 4>(c, in, sh, stream);
    else e = per == 1 ? launch_d<64, 1>(c, in, sh, stream) : launch_d<64, 2>(c, in, sh, stream);
    if (e == cudaSuccess && !sh.few && sh.units > 1)
        e = launch_append_len(in.chunk_start, c.len, c.B, c.Hkv, c.layer_begin, c.n_items, in.n_tokens, in.max_chunk, c.cap_tokens, stream);
    return e;
}

cudaError_t launch_block_read(const BlockView& c, const int32_t* slot_begin, int n_slots, void* k_out, void* v_out, cudaStream_t stream) {
    const int rows = kReadRows * 256 / (c.D / 8), per_item = (n_slots + rows - 1) / rows;
    const unsigned grid = (unsigned)c.n_items * per_item;
    return c.D == 128 ? launch_dependent(block_read_kernel<128>, dim3(grid), 256, 0, stream, c, slot_begin, n_slots, per_item, (bf16*)k_out, (bf16*)v_out)
                      : launch_dependent(block_read_kernel<64>, dim3(grid), 256, 0, stream, c, slot_begin, n_slots, per_item, (bf16*)k_out, (bf16*)v_out);
}

}  // namespace lethe
