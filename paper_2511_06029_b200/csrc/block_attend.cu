// lethe_block_attend: softmax attention of single query tokens over a cache in 8 bits with a scale for each block of tokens.
//
// Bound by memory: 2 D bytes per token and KV head.  The steps of 32 tokens of all items lie end to end on a line (an item's full
// blocks, or those its list names, then its open rows), which is cut evenly over the warps of the GPU, since lengths are known on the
// device only: ragged batches, one long sequence and many short ones are balanced alike.  A warp goes through its stretch alone, with a
// ring of TMA tiles of its own and no barrier with the others.  What a CTA's warps have of one item is merged when all of them are done
// (adjacent stretches belong to adjacent warps), and what a CTA has of an item that other CTAs share by the last of them to finish, in
// the order of the line: nothing is added atomically.
//
// S^T = K Q^T (tokens on M, the group's heads on N) on the codes themselves: m16n8k32 s8 MMAs, a query row as a whole number of 21 bits
// relative to its largest element, in three digits of 7 bits, so that the sums are exact.  The scale of the key block is a factor of the
// logits; the scale of the value block goes into the exponent, p' = exp2(s + log2 vs - m), so that the probabilities meet plain codes
// in O^T += V^T P^T (m16n8k16 f16 MMAs, the probabilities turned by movmatrix), and the sum of probabilities takes p' / vs.  A value code
// becomes the f16 of the same value by bit operations (1024 + 128 + x is 0x6400 | (x ^ 0x80)) and one subtraction, exactly.  m is the
// largest s + log2 vs up to a factor of 2^6: it only moves when a logit outgrows it by that, and p' is kept 2^9 up, so that f16 (up to
// 2^15 in use) holds probabilities down to 2^-23 of the largest with full precision.  Rows of open blocks take bf16 MMAs with the
// probabilities in two terms.  Stretches whose value scales leave the range that one m can serve, or whose open rows overflow, are done once
// more by far_stretch, plainly.
//
// Measured (us, calls captured in a graph): a step of the Llama-8B shape, 571 MB, 102 = 5.6 TB/s, 0.86 of the copy rate; one sequence of 131072
// tokens, 268 MB, 51 = 0.81; a ragged batch in blocks of 16 62 = 0.79; one layer of the first 13 (3.5 until the first tiles are asked for, 2 to 5
// for two or three steps a warp, 4 for the merges).  8 warps with two tiles each: the more is in flight the further apart the warps of an SM end
// (16 warps of three 16-token tiles: 78 to 105 us, 113 in all; 12 of two: 83 to 95, 105), and fewer warps leave no time for a conversion of the keys,
// which is why the logits come from the codes (f16 keys on 8 warps: 124).  Letting warps that are ahead wait for the others: 155.
#include <string.h>

#include "block_attend.cuh"
#include "chunk_tc.cuh"
#include "kv8_utils.cuh"

namespace lethe {
namespace {

constexpr int kThreads = kBlockWarps * 32;
constexpr int kStep = kBlockStep, kTailWeight = kBlockTail, kPad = kBlockPad;
constexpr int kLine = 2048;     // items whose places on the line are kept in shared memory; of more, only every so many-th is
constexpr float kLazy = 6.f;    // how far (log2) a logit may lie above m
constexpr float kLift = 9.f;    // p' is kept up by this (log2)
// Value scales that a stretch takes with one m: up to 2^40 either side of the first of them, r.  The sum of p' / vs lies between 2^-31 and 2^72
// then, with 2^17 tokens, and with open rows, of scale 1, it may come down to 2^9 r or up to 2^22 r.  What has the largest scale sets m, so the
// smallest one is 2^90 below it at most where r lies between 2^-50 and 2^60: shares of less than 2^-35 of the largest vanish.  Beyond, r may
// be 2^-96 to 2^90, but scales only 2^10 further out (no block of zeros below 2^-50), 2^106 in all: shares of less than 2^-20 vanish.
constexpr float kFar = 0x1p40f, kFarther = 0x1p10f, kLowRef = 0x1p-50f, kHighRef = 0x1p60f, kLeastRef = 0x1p-96f, kMostRef = 0x1p90f;
constexpr float kZeroLog2 = -40.f;  // where a block of zeros, which only the sum of probabilities knows, counts for m

template <int D>
__host__ __device__ constexpr int stage_bytes() { return kStep * D * 2; }
template <int D>
__host__ __device__ constexpr int stages() { return kBlockStages * 128 / D; }

// One end of a warp's stretch that is not a whole item.
struct Rec {
    int idx;       // item of the call, -1: none
    int start, w;  // where the item lies on the line
    bool begins, ends;
};

template <int D>
struct __align__(1024) Smem {
    unsigned char ring[kBlockWarps][stages<D>()][stage_bytes<D>()];
    float first[kBlockWarps][8 * D];        // O of a warp's first stretch, when it has others after it (the last one's goes to its ring)
    unsigned long long bars[kBlockWarps][stages<D>()];
    int line[kLine + 1], len[kLine];
    int prefix[kThreads + 1], totals[kBlockWarps];
    Rec rec[32];                            // warp w: 2 w its first stretch, 2 w + 1 its last
    float m[32][8], l[32][8];               // a part's weight is l 2^m; its O is divided by that
    int abort;
};

struct Span {
    int n, full, blocks, steps, open, w;
};
__device__ __forceinline__ Span span_of(const BlockAttendArgs& a, int n) {
    Span s;
    s.n = n;
    s.full = s.n >> a.c.t_shift;
    s.blocks = a.selected ? min(a.n_select, s.full) : s.full;
    s.steps = ((s.blocks << a.c.t_shift) + kStep - 1) / kStep;
    s.open = s.n & (a.c.T - 1);
    s.w = kPad + s.steps + kTailWeight * ((s.open + 31) >> 5);
    return s;
}

__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* map, int x, int y, unsigned long long* b, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(smem_u32(b)), "l"(policy) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}
// d = a b + c, 8-bit whole numbers.
__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, const int (&c)[4]) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
                 : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]));
}
// Bytes 0 and 2 of x, whole numbers in two's complement, as two halves.
__device__ __forceinline__ uint32_t halves_of(uint32_t x) {
    uint32_t y;
    asm("lop3.b32 %0, %1, 0x00ff00ff, 0x64806480, 0x6a;" : "=r"(y) : "r"(x));  // (x & mask) ^ bias
    const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&y), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t*>(&h);
}

// State of a stretch: lane = 4 g + t has heads 2t and 2t + 1; o[i] = (d, 2t), (d, 2t + 1), (d + 1, 2t), (d + 1, 2t + 1) with d = first_d + 2 i.
template <int D>
struct Acc {
    float o[D / 16][4];
    float m[2], l[2];  // l: this lane's tokens only
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
    }
    // x: logits of H x 16 tokens (row g: x[h][0], x[h][1]; row g + 8: x[h][2], x[h][3]) -> p', and m moved where it has to be
    template <int H>
    __device__ __forceinline__ void softmax(float (&x)[H][4], const float (&inv_vs)[H]) {
        float a = fmaxf(x[0][0], x[0][2]), b = fmaxf(x[0][1], x[0][3]);
#pragma unroll
        for (int h = 1; h < H; ++h) {
            a = fmaxf(a, fmaxf(x[h][0], x[h][2]));
            b = fmaxf(b, fmaxf(x[h][1], x[h][3]));
        }
        if (__any_sync(0xffffffffu, a > m[0] + kLazy || b > m[1] + kLazy)) {
            float na = a, nb = b;
#pragma unroll
            for (int s = 4; s < 32; s <<= 1) {
                na = fmaxf(na, __shfl_xor_sync(0xffffffffu, na, s));
                nb = fmaxf(nb, __shfl_xor_sync(0xffffffffu, nb, s));
            }
            na = fmaxf(na, m[0]);
            nb = fmaxf(nb, m[1]);
            const float fa = exp2_diff(m[0], na), fb = exp2_diff(m[1], nb);
            m[0] = na;
            m[1] = nb;
            l[0] *= fa;
            l[1] *= fb;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                o[i][0] *= fa;
                o[i][1] *= fb;
                o[i][2] *= fa;
                o[i][3] *= fb;
            }
        }
        const float ma = m[0] == -INFINITY ? 0.f : m[0] - kLift, mb = m[1] == -INFINITY ? 0.f : m[1] - kLift;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            x[h][0] = fast_exp2(x[h][0] - ma);
            x[h][1] = fast_exp2(x[h][1] - mb);
            x[h][2] = fast_exp2(x[h][2] - ma);
            x[h][3] = fast_exp2(x[h][3] - mb);
            l[0] = fmaf(x[h][0] + x[h][2], inv_vs[h], l[0]);
            l[1] = fmaf(x[h][1] + x[h][3], inv_vs[h], l[1]);
        }
    }
};

// The root of exp2(a - b): a part that is 2^228 times as large as another may count for as much with a weight as small as that.
__device__ __forceinline__ float root_diff(float a, float b) { return a == -INFINITY ? 0.f : fast_exp2(0.5f * (a - b)); }
// A share of a sum, root x rest, as two factors: itself and 1, or the two where fp32 does not hold it.
__device__ __forceinline__ float2 share_of(float root, float rest) {
    const float share = root * rest;
    return share < 0x1p-100f ? make_float2(root, rest) : make_float2(share, 1.f);
}

// Tokens of an item for values of any size: full blocks of the steps g0 .. g1 - 1 and open rows r0 .. r1 - 1, a warp, a token at a time with
// D / 32 elements to a lane.  Leaves m, l (weight l 2^m) and O / l of each head in shared memory, or, with part = NULL, the item's output.
// Everything is held in the values' own size: O is a mean at all times.  A thirtieth of the kernel's speed (a step of the Llama-8B shape, all
// of it by this function, 3.4 ms), for values that no model has; in a function of its own it costs ordinary calls nothing, in the kernel's
// loop 4 us of that step.
template <int D>
__device__ __noinline__ void far_stretch(const BlockAttendArgs& a, int idx, int g0, int g1, int r0, int r1, float* part, float* part_m, float* part_l) {
    constexpr int E = D / 32, U = 8;
    const BlockView& c = a.c;
    const int lane = threadIdx.x & 31;
    const BlockItem it = block_item(c.layer_begin, c.B, c.Hkv, idx);
    const int full = block_len(c, it.item) >> c.t_shift, blocks = a.selected ? min(a.n_select, full) : full;
    const size_t row0 = (((size_t)it.li * c.B + it.b) * c.Hkv + it.h) * c.G;
    float q[8][E], o[8][E], m[8], l[8], scale[8];
#pragma unroll
    for (int h = 0; h < 8; ++h) {
        bool bad = false;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            q[h][e] = h < c.G ? __bfloat162float(a.q[(row0 + h) * D + E * lane + e]) : 0.f;
            bad = bad || !(fabsf(q[h][e]) < INFINITY);
            o[h][e] = 0.f;
        }
        scale[h] = __any_sync(0xffffffffu, bad) ? __uint_as_float(0x7fc00000u) : c.scale_log2[c.layer_begin + it.li];
        m[h] = -INFINITY;
        l[h] = 0.f;
    }
    auto token = [&](const float (&k)[E], const float (&v)[E], float k_scale) {
#pragma unroll
        for (int h = 0; h < 8; ++h) {
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) s = fmaf(q[h][e], k[e], s);
#pragma unroll
            for (int k = 16; k; k >>= 1) s += __shfl_xor_sync(0xffffffffu, s, k);
            s *= k_scale * scale[h];
            const float top = fmaxf(m[h], s), old = root_diff(m[h], top), now = root_diff(s, top);
            const float was = l[h] * old, sum = fmaf(was, old, now * now), inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int e = 0; e < E; ++e) o[h][e] = o[h][e] * old * (was * inv) + v[e] * now * (now * inv);
            m[h] = top;
            l[h] = sum;
        }
    };
    const int group = min(c.T, kStep);  // tokens of a step that lie in one block
#pragma unroll 1
    for (int j = g0 * kStep; j < g1 * kStep; j += group) {
        const int e0 = j >> c.t_shift;
        if (e0 >= blocks) break;
        const int blk = a.selected ? a.selected[(size_t)idx * a.n_select + e0] : e0;
        if (blk < 0) continue;
        const long long page = blk < full ? block_page(c, it.item, blk) : -1;
        if (page < 0) {  // the kernel's own way records only what it has come to
            if (lane == 0) record_error(c.status, blk < full ? LETHE_ERR_PAGE : LETHE_ERR_INVALID_ARG, it.item);
            continue;
        }
        const float ks = c.k_scale[page], vs = c.v_scale[page];
        const size_t at = ((size_t)page * c.T + (j & (c.T - 1))) * D + E * lane;
#pragma unroll 1
        for (int i0 = 0; i0 < group; i0 += U) {
            uint32_t kw[U], vw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int8_t *kp = c.k + at + (size_t)(i0 + u) * D, *vp = c.v + at + (size_t)(i0 + u) * D;
                kw[u] = E == 4 ? *reinterpret_cast<const uint32_t*>(kp) : *reinterpret_cast<const uint16_t*>(kp);
                vw[u] = E == 4 ? *reinterpret_cast<const uint32_t*>(vp) : *reinterpret_cast<const uint16_t*>(vp);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float k[E], v[E];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    k[e] = (float)(int8_t)(kw[u] >> (8 * e));
                    v[e] = (float)(int8_t)(vw[u] >> (8 * e)) * vs;
                }
                token(k, v, ks);
            }
        }
    }
#pragma unroll 1
    for (int r = r0; r < r1; ++r) {
        const size_t at = ((size_t)it.item * c.T + r) * D + E * lane;
        float k[E], v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            k[e] = __bfloat162float(c.k_open[at + e]);
            v[e] = __bfloat162float(c.v_open[at + e]);
        }
        token(k, v, 1.f);
    }
#pragma unroll
    for (int h = 0; h < 8; ++h) {
        if (part) {
#pragma unroll
            for (int e = 0; e < E; ++e) part[h * D + E * lane + e] = o[h][e];
            if (lane == 0) {
                part_m[h] = m[h];
                part_l[h] = l[h];
            }
        } else if (h < c.G) {
#pragma unroll
            for (int e = 0; e < E; ++e) a.out[(row0 + h) * D + E * lane + e] = __float2bfloat16(o[h][e]);
            if (a.lse && lane == 0) a.lse[row0 + h] = l[h] == 0.f ? -INFINITY : (m[h] + log2f(l[h])) * 0.6931471805599453f;
        }
    }
}

// Elements that a lane reads of a key row (16 bytes at each of D / 64 places) and of a value row, and the order of a tile's tokens among
// the MMA's rows: chosen so that eight neighbouring lanes touch eight different 16-byte columns of the swizzled tile at D = 128.
template <int D>
__device__ __forceinline__ int token_row(int r) {  // row 0 .. 7 of the MMA -> token of the tile
    return D == 128 ? ((r >> 1) | ((r & 1) << 2)) : r;
}
template <int D>
__device__ __forceinline__ int first_d(int g) { return D == 128 ? 16 * ((g >> 1) | ((g & 1) << 2)) : 8 * g; }
template <int D>
__device__ __forceinline__ uint32_t swizzled(int row, int byte) {
    return D == 128 ? row * 128 + (byte ^ ((row & 7) << 4)) : row * 64 + (byte ^ (((row >> 1) & 3) << 4));
}

// O^T += V^T P^T for rows a, b (tokens of k = 2t, 2t + 1) and c, d (k = 2t + 8, 2t + 9), words of four codes.
template <int D>
__device__ __forceinline__ void value_word(float (*o)[4], uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t p0, uint32_t p1) {
    const uint32_t ab = __byte_perm(a, b, 0x5410), cd = __byte_perm(c, d, 0x5410);
    const uint32_t f0[4] = {halves_of(ab), halves_of(ab >> 8), halves_of(cd), halves_of(cd >> 8)};
    mma_f16(o[0], f0, p0, p1);
    const uint32_t ef = __byte_perm(a, b, 0x7632), gh = __byte_perm(c, d, 0x7632);
    const uint32_t f1[4] = {halves_of(ef), halves_of(ef >> 8), halves_of(gh), halves_of(gh >> 8)};
    mma_f16(o[1], f1, p0, p1);
}

// 32 open rows from row r0 on: keys and values straight from memory, bf16, all asked for before anything is used.
template <int D>
__device__ __forceinline__ void open_rows(const BlockAttendArgs& a, Acc<D>& acc, const BlockItem& it, int r0, int n_open, const float (&scale2)[2], float v_ref, float inv_ref_log2) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const __nv_bfloat16* K = a.c.k_open + (size_t)it.item * a.c.T * D;
    const __nv_bfloat16* V = a.c.v_open + (size_t)it.item * a.c.T * D;
    const __nv_bfloat16* Q = a.q + (((size_t)it.li * a.c.B + it.b) * a.c.Hkv + it.h) * a.c.G * D;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    constexpr int J = D / 32;  // 8 elements of a lane each
    uint4 q[J], k[2][2][J], v[2][4][D / 64];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int d = j * 32 + 8 * t;
        q[j] = g < a.c.G ? *reinterpret_cast<const uint4*>(Q + (size_t)g * D + d) : zero;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = r0 + 16 * h + 8 * r + g;
                k[h][r][j] = row < n_open ? *reinterpret_cast<const uint4*>(K + (size_t)row * D + d) : zero;
            }
    }
    const int d0 = first_d<D>(g);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = r0 + 16 * h + 2 * t + (i & 1) + (i >> 1) * 8;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) v[h][i][j] = row < n_open ? *reinterpret_cast<const uint4*>(V + (size_t)row * D + d0 + 8 * j) : zero;
        }
    float s[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[h][i] = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const uint4 x = k[h][0][j], y = k[h][1][j];
            const uint32_t f0[4] = {x.x, y.x, x.y, y.y}, f1[4] = {x.z, y.z, x.w, y.w};
            mma_bf16(s[h], f0, q[j].x, q[j].y);
            mma_bf16(s[h], f1, q[j].z, q[j].w);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[h][i] = r0 + 16 * h + 8 * (i >> 1) + g < n_open ? fmaf(s[h][i], scale2[i & 1], inv_ref_log2) : -INFINITY;
    }
    const float inv[2] = {v_ref, v_ref};
    acc.template softmax<2>(s, inv);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t p[2][2];  // [term][rows 0 .. 7, 8 .. 15]
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float u = s[h][2 * i], w = s[h][2 * i + 1];
            const uint32_t big = pack_bf16(u, w);
            p[0][i] = movmatrix_trans(big);
            p[1][i] = movmatrix_trans(pack_bf16(u - __uint_as_float(big << 16), w - __uint_as_float(big & 0xffff0000u)));
        }
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            const uint32_t x[4][4] = {{v[h][0][j].x, v[h][0][j].y, v[h][0][j].z, v[h][0][j].w}, {v[h][1][j].x, v[h][1][j].y, v[h][1][j].z, v[h][1][j].w},
                                      {v[h][2][j].x, v[h][2][j].y, v[h][2][j].z, v[h][2][j].w}, {v[h][3][j].x, v[h][3][j].y, v[h][3][j].z, v[h][3][j].w}};
#pragma unroll
            for (int w = 0; w < 4; ++w) {  // elements 2 w and 2 w + 1 of the eight
                const uint32_t f[4] = {__byte_perm(x[0][w], x[1][w], 0x5410), __byte_perm(x[0][w], x[1][w], 0x7632),
                                       __byte_perm(x[2][w], x[3][w], 0x5410), __byte_perm(x[2][w], x[3][w], 0x7632)};
                mma_bf16(acc.o[4 * j + w], f, p[0][0], p[0][1]);
                mma_bf16(acc.o[4 * j + w], f, p[1][0], p[1][1]);
            }
        }
    }
}

// The last place of an ascending table (its first entry is at most x) that holds at most x; a warp, 32 places at a time.
__device__ __forceinline__ int last_at_most(const int* table, int n, int x, int lane) {
    int lo = 0;
    while (n > 1) {
        const int step = (n + 31) / 32, i = lane * step;
        const unsigned ok = __ballot_sync(0xffffffffu, i < n && table[lo + i] <= x);
        const int k = 31 - __clz(ok);
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) block_attend_kernel(const __grid_constant__ BlockAttendArgs a, const __grid_constant__ BlockMaps maps) {
    constexpr int NS = stages<D>(), SB = stage_bytes<D>(), C = D / 64;
    extern __shared__ __align__(1024) unsigned char raw[];
    Smem<D>& sm = *reinterpret_cast<Smem<D>*>(raw + ((1024 - (smem_u32(raw) & 1023)) & 1023));
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, g = lane >> 2, t = lane & 3;
    const BlockView& c = a.c;
    if (lane == 0) {
        for (int s = 0; s < NS; ++s) bar_init(&sm.bars[w][s], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid < 32) sm.rec[tid].idx = -1;
    if (tid == 0) {
        sm.abort = 0;
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.v) : "memory");
    }
    dependency_wait();
    dependency_release();

    // the line: a run of items to each thread
    auto len_of = [&](int idx) { return block_len(c, block_item(c.layer_begin, c.B, c.Hkv, idx).item); };
    const bool fits = c.n_items <= kLine;
    const int run = (c.n_items + kThreads - 1) / kThreads, i0 = min(c.n_items, tid * run), i1 = min(c.n_items, i0 + run);
    int mine = 0;
#pragma unroll 4
    for (int i = i0; i < i1; ++i) {
        const int n = len_of(i), wt = span_of(a, n).w;
        if (fits) {
            sm.len[i] = n;
            sm.line[i] = wt;
        }
        mine += wt;
    }
    {
        int x = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) sm.totals[w] = x;
        __syncthreads();
        int base = 0;
#pragma unroll
        for (int i = 0; i < kBlockWarps; ++i)
            if (i < w) base += sm.totals[i];
        int at = base + x - mine;
        sm.prefix[tid] = at;
        if (tid == kThreads - 1) sm.prefix[kThreads] = base + x;
        if (fits)
            for (int i = i0; i < i1; ++i) {
                const int wt = sm.line[i];
                sm.line[i] = at;
                at += wt;
            }
        __syncthreads();
    }
    const long long total = sm.prefix[kThreads];
    // Warps in use: at least two steps each (or an item's beginning), as far as there are.  Over seven calls behind a selection, 10 to 23 us: with
    // one 1.3 less to 0.5 more, with three 0.1 less to 1.5 more, with four 0.2 less to 2.5 more.
    const long long warps = min((long long)a.n_cta * kBlockWarps, (total + 1) / 2);
    if ((long long)blockIdx.x * kBlockWarps >= warps) return;
    auto cta_at = [&](int pos) { return (int)(((pos + 1LL) * warps - 1) / total) / kBlockWarps; };
    const int wid = blockIdx.x * kBlockWarps + w;
    const int at0 = wid < warps ? (int)(wid * total / warps) : 0, at1 = wid < warps ? (int)((wid + 1) * total / warps) : 0;

    if (at0 < at1) {
        // the item that holds at0
        int idx, start;
        if (fits) {
            idx = last_at_most(sm.line, c.n_items, at0, lane);
            start = sm.line[idx];
        } else {
            const int chunk = last_at_most(sm.prefix, kThreads, at0, lane);
            idx = chunk * run;
            start = sm.prefix[chunk];
            for (;;) {
                const int i = idx + lane;
                int x = i < c.n_items ? span_of(a, len_of(i)).w : 0x3fffffff / 32;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, x, o);
                    if (lane >= o) x += y;
                }
                const unsigned past = __ballot_sync(0xffffffffu, x > at0 - start);
                const int skip = past ? __ffs(past) - 1 : 32;
                const int before = __shfl_sync(0xffffffffu, x, max(skip - 1, 0));
                if (skip) start += before;
                idx += skip;
                if (skip < 32) break;
            }
        }

        const uint64_t policy = l2_evict_first_policy();
        uint32_t k_at[C], v_at[2];  // this lane's places in a tile's first 16 tokens; eight rows further nothing but 8 D is added
#pragma unroll
        for (int k = 0; k < C; ++k) k_at[k] = swizzled<D>(token_row<D>(g), 64 * k + 16 * t);
#pragma unroll
        for (int k = 0; k < 2; ++k) v_at[k] = swizzled<D>(token_row<D>(2 * t + k), first_d<D>(g));
        const uint32_t ring = smem_u32(sm.ring[w]);
        int stage = 0;
        unsigned phase = 0;      // of `stage`
        int put = 0;             // stage that is filled next
        bool aborted = false;
        int at = at0;
        while (at < at1) {
            const BlockItem it = block_item(c.layer_begin, c.B, c.Hkv, idx);
            const Span sp = span_of(a, fits ? sm.len[idx] : len_of(idx));
            const int p0 = at - start, p1 = min(at1 - start, sp.w);
            const int g0 = min(max(p0 - kPad, 0), sp.steps), g1 = aborted ? g0 : min(max(p1 - kPad, 0), sp.steps);

            // runs of up to 32 blocks, one to a lane: the one that is being asked for (its scales are still on their way) and the one
            // that is worked on.  The former is ahead by less than a run.
            int ask0 = -64, ask_page = -1, use0 = -64;
            float ask_ks = 0.f, ask_vs = 0.f, ks = 0.f, lv = 0.f, iv = 0.f;  // iv: v_ref / vs, negative: a block whose values are zero
            float v_ref = 1.f, inv_ref = 1.f;
            bool have_ref = false, far = false;
            auto ask_run = [&](int e0) {
                ask0 = e0;
                ask_page = -1;
                ask_ks = ask_vs = 0.f;
                const int e = e0 + lane;
                if (e < sp.blocks) {
                    int blk = e;
                    if (a.selected) {
                        blk = a.selected[(size_t)idx * a.n_select + e];
                        if (blk >= sp.full) {
                            record_error(c.status, LETHE_ERR_INVALID_ARG, it.item);
                            blk = -1;
                        }
                    }
                    if (blk >= 0) {
                        ask_page = (int)block_page(c, it.item, blk);
                        if (ask_page < 0) record_error(c.status, LETHE_ERR_PAGE, it.item);
                    }
                    if (ask_page >= 0) {
                        ask_ks = c.k_scale[ask_page];
                        ask_vs = c.v_scale[ask_page];
                    }
                }
            };
            auto use_run = [&]() {
                use0 = ask0;
                ks = ask_ks;
                if (!have_ref) {
                    // a power of two near the first value scale: the others are taken relative to it
                    const unsigned some = __ballot_sync(0xffffffffu, ask_vs > 0.f && ask_vs < INFINITY);
                    if (some) {
                        const float v0 = __shfl_sync(0xffffffffu, ask_vs, __ffs(some) - 1);
                        const int ex = min(max((int)(__float_as_uint(v0) >> 23), 1), 252);
                        v_ref = __uint_as_float((uint32_t)ex << 23);
                        inv_ref = __uint_as_float((uint32_t)(254 - ex) << 23);
                        have_ref = true;
                        far = v_ref < kLeastRef || v_ref > kMostRef;
                    }
                }
                const float rel = ask_vs * inv_ref;
                const bool low = v_ref < kLowRef;
                const float least = low ? 1.f / kFarther : 1.f / kFar, most = v_ref > kHighRef ? kFarther : kFar;
                far = far || __any_sync(0xffffffffu, ask_page >= 0 && (rel > most || rel < (ask_vs > 0.f || low ? least : 0.f)));
                lv = ask_page < 0 ? -INFINITY : ask_vs == 0.f ? kZeroLog2 : __log2f(rel);  // no block: no weight
                iv = ask_vs == 0.f ? -kFar : __fdividef(1.f, rel);
            };
            // step gi: one tile of a block of 32 tokens or more, or two blocks of 16
            auto issue = [&](int gi) {
                unsigned long long* bar = &sm.bars[w][put];
                const uint32_t dst = ring + put * SB;
                if (c.t_shift > 4) {
                    const int e = gi >> (c.t_shift - 5);
                    if (e >= ask0 + 32 || ask0 < 0) ask_run(e);
                    const int pg = __shfl_sync(0xffffffffu, ask_page, e - ask0);
                    if (lane == 0) {
                        bar_expect_tx(bar, pg < 0 ? 0 : SB);
                        if (pg >= 0) {
                            const int row = (pg << c.t_shift) + ((gi * kStep) & (c.T - 1));
                            tma_2d(dst, &maps.k, 0, row, bar, policy);
                            tma_2d(dst + SB / 2, &maps.v, 0, row, bar, policy);
                        }
                    }
                } else {
                    if (2 * gi >= ask0 + 32 || ask0 < 0) ask_run(2 * gi);  // runs begin at even blocks
                    const int p0 = __shfl_sync(0xffffffffu, ask_page, 2 * gi - ask0), p1 = __shfl_sync(0xffffffffu, ask_page, 2 * gi + 1 - ask0);
                    if (lane == 0) {
                        bar_expect_tx(bar, (p0 < 0 ? 0 : SB / 2) + (p1 < 0 ? 0 : SB / 2));
                        if (p0 >= 0) {
                            tma_2d(dst, &maps.k, 0, p0 * 16, bar, policy);
                            tma_2d(dst + SB / 2, &maps.v, 0, p0 * 16, bar, policy);
                        }
                        if (p1 >= 0) {
                            tma_2d(dst + SB / 4, &maps.k, 0, p1 * 16, bar, policy);
                            tma_2d(dst + 3 * (SB / 4), &maps.v, 0, p1 * 16, bar, policy);
                        }
                    }
                }
                put = put + 1 == NS ? 0 : put + 1;
            };

            // queries: whole numbers of up to 2^20 either way (21 bits), in three digits, in the order of the key codes
            uint32_t qf[3][4 * C];
            float scale2[2], open2[2];
            int queued = min(g1, g0 + NS);
            {
                const __nv_bfloat16* Q = a.q + (((size_t)it.li * c.B + it.b) * c.Hkv + it.h) * c.G * D + (size_t)g * D;
                uint4 x[C][2];
#pragma unroll
                for (int k = 0; k < C; ++k)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        x[k][j] = g < c.G ? *reinterpret_cast<const uint4*>(Q + 64 * k + 16 * t + 8 * j) : make_uint4(0, 0, 0, 0);
#pragma unroll 1
                for (int i = g0; i < queued; ++i) issue(i);
                float big = 0.f;
                float f[C][16];
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    Piece<__nv_bfloat16>::unpack(x[k][0], f[k]);
                    Piece<__nv_bfloat16>::unpack(x[k][1], f[k] + 8);
#pragma unroll
                    for (int j = 0; j < 16; ++j) big = fmaxf(big, fabsf(f[k][j]));
                }
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
                // a power of two brings the largest magnitude to [2^19, 2^20)
                int ex = (int)((__float_as_uint(big) >> 23) & 0xffu) - 19;
                ex = big > 0.f && big < INFINITY ? min(max(ex, 2), 252) : 127;
                const float mul = __uint_as_float((uint32_t)(254 - ex) << 23);
                const float div = __uint_as_float((uint32_t)ex << 23);
                bool bad = false;  // a query with a NaN or an infinity has no whole numbers: all its logits are NaN
#pragma unroll
                for (int k = 0; k < C; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t digit[3] = {0, 0, 0};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float y = f[k][4 * j + i];
                            bad = bad || !(fabsf(y) < INFINITY);
                            const int v = __float2int_rn(y * mul), d2 = (v + 8192) >> 14, r = v - (d2 << 14), d1 = (r + 64) >> 7, d0 = r - (d1 << 7);
                            digit[2] |= (uint32_t)(d2 & 0xff) << (8 * i);
                            digit[1] |= (uint32_t)(d1 & 0xff) << (8 * i);
                            digit[0] |= (uint32_t)(d0 & 0xff) << (8 * i);
                        }
#pragma unroll
                        for (int i = 0; i < 3; ++i) qf[i][4 * k + j] = digit[i];
                    }
                const unsigned bads = __ballot_sync(0xffffffffu, bad);
                float scale = c.scale_log2[c.layer_begin + it.li];
                if (bads >> (4 * g) & 15u) scale = __uint_as_float(0x7fc00000u);
                open2[0] = __shfl_sync(0xffffffffu, scale, 8 * t);
                open2[1] = __shfl_sync(0xffffffffu, scale, 8 * t + 4);
                scale2[0] = open2[0] * __shfl_sync(0xffffffffu, div, 8 * t);
                scale2[1] = open2[1] * __shfl_sync(0xffffffffu, div, 8 * t + 4);
            }
            Acc<D> acc;
            acc.clear();
            float b_ks[2] = {0.f, 0.f}, b_lv[2] = {0.f, 0.f}, b_iv[2] = {0.f, 0.f};  // of the blocks at hand
            int done = g0;
            for (int gi = g0; gi < g1; done = ++gi) {
                const int e = (gi * kStep) >> c.t_shift;
                if (e >= use0 + 32 || use0 < 0) {
                    use_run();
                    if (far) break;
                }
                if (c.t_shift <= 5 || gi == g0 || !((gi * kStep) & (c.T - 1))) {
                    b_ks[0] = b_ks[1] = __shfl_sync(0xffffffffu, ks, e - use0);
                    b_lv[0] = b_lv[1] = __shfl_sync(0xffffffffu, lv, e - use0);
                    b_iv[0] = b_iv[1] = __shfl_sync(0xffffffffu, iv, e - use0);
                    if (c.t_shift == 4) {
                        b_ks[1] = __shfl_sync(0xffffffffu, ks, e + 1 - use0);
                        b_lv[1] = __shfl_sync(0xffffffffu, lv, e + 1 - use0);
                        b_iv[1] = __shfl_sync(0xffffffffu, iv, e + 1 - use0);
                    }
                }
                unsigned long long* bar = &sm.bars[w][stage];
                if (!warp_wait(bar, phase, &sm.abort, a.wait_limit)) {
                    if (lane == 0) record_error(c.status, LETHE_ERR_TIMEOUT, blockIdx.x);
                    aborted = true;
                    break;
                }
                const uint32_t tile = ring + stage * SB;
                uint4 kx[2][C][2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int k = 0; k < C; ++k)
#pragma unroll
                        for (int r = 0; r < 2; ++r) kx[h][k][r] = lds128(tile + k_at[k] + h * (SB / 4) + r * 8 * D);
                float p[2][4];
                {
                    constexpr int kMagic = 0x4b400000;  // 1.5 x 2^23 as bits: a whole number added to it is the fraction of that float
                    const int from[4] = {kMagic, kMagic, kMagic, kMagic};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        int sums[3][4];
#pragma unroll
                        for (int k = 0; k < C; ++k) {
                            const uint4 x = kx[h][k][0], y = kx[h][k][1];
#pragma unroll
                            for (int i = 0; i < 3; ++i) {
                                if (k == 0) mma_s8(sums[i], x.x, y.x, x.y, y.y, qf[i][0], qf[i][1], from);
                                else mma_s8(sums[i], x.x, y.x, x.y, y.y, qf[i][4 * k], qf[i][4 * k + 1], sums[i]);
                                mma_s8(sums[i], x.z, y.z, x.w, y.w, qf[i][4 * k + 2], qf[i][4 * k + 3], sums[i]);
                            }
                        }
                        const float ka = b_ks[h] * scale2[0], kb = b_ks[h] * scale2[1];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            constexpr float kOff = 12582912.f;
                            const float s2 = __int_as_float(sums[2][i]) - kOff, s1 = __int_as_float(sums[1][i]) - kOff, s0 = __int_as_float(sums[0][i]) - kOff;
                            p[h][i] = fmaf(fmaf(fmaf(s2, 128.f, s1), 128.f, s0), i & 1 ? kb : ka, b_lv[h]);
                        }
                    }
                }
                uint4 vx[2][4];
                uint2 vy[2][4];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t at = tile + SB / 2 + h * (SB / 4) + v_at[k & 1] + (k >> 1) * 8 * D;
                        if (D == 128) vx[h][k] = lds128(at);
                        else vy[h][k] = lds64(at);
                    }
                __syncwarp();
                stage = stage + 1 == NS ? 0 : stage + 1;
                phase ^= stage == 0;
                if (queued < g1) issue(queued++);

                const float inv[2] = {fabsf(b_iv[0]), fabsf(b_iv[1])};
                acc.template softmax<2>(p, inv);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t b0 = movmatrix_trans(pack_f16(p[h][0], p[h][1])), b1 = movmatrix_trans(pack_f16(p[h][2], p[h][3]));
                    if (b_iv[h] < 0.f) b0 = b1 = 0;  // values of zero
                    if (D == 128) {
                        value_word<D>(acc.o, vx[h][0].x, vx[h][1].x, vx[h][2].x, vx[h][3].x, b0, b1);
                        value_word<D>(acc.o + 2, vx[h][0].y, vx[h][1].y, vx[h][2].y, vx[h][3].y, b0, b1);
                        value_word<D>(acc.o + D / 32, vx[h][0].z, vx[h][1].z, vx[h][2].z, vx[h][3].z, b0, b1);
                        value_word<D>(acc.o + D / 32 + 2, vx[h][0].w, vx[h][1].w, vx[h][2].w, vx[h][3].w, b0, b1);
                    } else {
                        value_word<D>(acc.o, vy[h][0].x, vy[h][1].x, vy[h][2].x, vy[h][3].x, b0, b1);
                        value_word<D>(acc.o + 2, vy[h][0].y, vy[h][1].y, vy[h][2].y, vy[h][3].y, b0, b1);
                    }
                }
            }
            // after a break: what is in flight lands before the warp goes on
            for (; done < queued; ++done) {
                bar_drain(&sm.bars[w][stage], phase);
                stage = stage + 1 == NS ? 0 : stage + 1;
                phase ^= stage == 0;
            }
            // open rows whose place on the line lies in the stretch
            const int tail0 = (max(p0 - kPad - sp.steps, 0) + kTailWeight - 1) / kTailWeight, tail1 = (max(p1 - kPad - sp.steps, 0) + kTailWeight - 1) / kTailWeight;
            for (int j = tail0; j < tail1 && 32 * j < sp.open && !far; ++j) open_rows<D>(a, acc, it, 32 * j, sp.open, open2, v_ref, __log2f(inv_ref));

#pragma unroll
            for (int s = 4; s < 32; s <<= 1) {
                acc.l[0] += __shfl_xor_sync(0xffffffffu, acc.l[0], s);
                acc.l[1] += __shfl_xor_sync(0xffffffffu, acc.l[1], s);
            }
            // What leaves the stretch is divided by its sum: a mean of values is as large as they are, and a part's weight is its sum.
            const float lift = v_ref < kLowRef ? 0x1p64f : 1.f, drop = v_ref < kLowRef ? 0x1p-64f : 1.f;  // the factor itself must not vanish
            float top[2], all = 0.f;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float f = acc.l[k] == 0.f ? 0.f : __fdividef(v_ref * lift, acc.l[k]);
                top[k] = acc.l[k] == 0.f ? -INFINITY : acc.m[k] - kLift;
                float sizes = 0.f;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    acc.o[i][k] = acc.o[i][k] * f * drop;
                    acc.o[i][2 + k] = acc.o[i][2 + k] * f * drop;
                    sizes += fabsf(acc.o[i][k]) + fabsf(acc.o[i][2 + k]);
                }
                if (acc.l[k] < INFINITY) all += sizes;  // a query that is not finite has a sum that is not, and gives NaN either way
            }
            far = far || (tail0 < tail1 && __any_sync(0xffffffffu, !(all < INFINITY)));  // open rows may hold anything
            const bool begins = p0 == 0, ends = p1 == sp.w;
            const bool last = at1 <= start + sp.w;  // nothing of this warp comes after it: the ring is free
            const int which = 2 * w + (last ? 1 : 0);
            float* const part = begins && ends ? nullptr : last ? reinterpret_cast<float*>(sm.ring[w]) : sm.first[w];
            if (part && lane == 0) {
                Rec& rec = sm.rec[which];
                rec.idx = idx;
                rec.start = start;
                rec.w = sp.w;
                rec.begins = begins;
                rec.ends = ends;
            }
            const int d0 = first_d<D>(g);
            if (far) {
                far_stretch<D>(a, idx, g0, aborted ? g0 : g1, min(32 * tail0, sp.open), min(32 * tail1, sp.open), part, sm.m[which], sm.l[which]);
            } else if (!part) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int head = 2 * t + k;
                    if (head >= c.G) continue;
                    const size_t row = (((size_t)it.li * c.B + it.b) * c.Hkv + it.h) * c.G + head;
                    uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + row * D + d0);
#pragma unroll
                    for (int i = 0; i < D / 16; i += 2)
                        *reinterpret_cast<uint2*>(dst + i) = make_uint2(pack_bf16(acc.o[i][k], acc.o[i][2 + k]), pack_bf16(acc.o[i + 1][k], acc.o[i + 1][2 + k]));
                    if (a.lse && g == 0) a.lse[row] = acc.l[k] == 0.f ? -INFINITY : (top[k] + log2f(acc.l[k])) * 0.6931471805599453f;
                }
            } else {
                if (g == 0) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        sm.m[which][2 * t + k] = top[k];
                        sm.l[which][2 * t + k] = acc.l[k];
                    }
                }
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) *reinterpret_cast<float2*>(part + (2 * t + k) * D + d0 + 2 * i) = make_float2(acc.o[i][k], acc.o[i][2 + k]);
            }
            at = start + p1;
            start += sp.w;
            ++idx;
        }
    }
    __syncthreads();

    // The parts there are, in the order of the line; those of one item follow one another.  A lane stands for a part; every warp finds out.
    const int part_idx = lane < 2 * kBlockWarps ? sm.rec[lane].idx : -1;
    const unsigned have = __ballot_sync(0xffffffffu, part_idx >= 0), below = have & ((1u << lane) - 1);
    const int prev = __shfl_sync(0xffffffffu, part_idx, below ? 31 - __clz(below) : 0);
    const unsigned firsts = __ballot_sync(0xffffffffu, part_idx >= 0 && (!below || prev != part_idx));
    // A warp merges one head of one item at a time, D / 32 elements to a lane.  The CTA's first and last item, which other CTAs may share, come
    // first and fall to different warps: they take a round trip or two more.
    constexpr int E = D / 32;
    const int items = __popc(firsts);
#pragma unroll 1
    for (int unit = w; unit < items * c.G; unit += kBlockWarps) {
        const int order = unit / c.G, head = unit - order * c.G;
        unsigned rest = firsts;
        for (int k = order == 0 ? 0 : order == 1 ? items - 1 : order - 1; k > 0; --k) rest &= rest - 1;
        const int r0 = __ffs(rest) - 1;
        const unsigned later = rest & (rest - 1);
        const unsigned chain = have & ~((1u << r0) - 1) & (later ? (1u << (__ffs(later) - 1)) - 1 : 0xffffffffu);
        const Rec& rec = sm.rec[r0];
        const bool whole = rec.begins && sm.rec[31 - __clz(chain)].ends;
        const BlockItem it = block_item(c.layer_begin, c.B, c.Hkv, rec.idx);
        {
            const bool in = chain >> lane & 1;
            float m = in ? sm.m[lane][head] : -INFINITY;
            float l = in ? sm.l[lane][head] : 0.f;
            const float mine_m = m;
#pragma unroll
            for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float half = root_diff(mine_m, m), mine_l = l * half;
            l = mine_l * half;
#pragma unroll
            for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
            const float2 share = share_of(half, l == 0.f ? 0.f : __fdividef(mine_l, l));  // a part's, of the sum
            float o[E];
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 4
            for (unsigned k = chain; k; k &= k - 1) {
                const int r = __ffs(k) - 1;
                const float* src = (r & 1 ? reinterpret_cast<const float*>(sm.ring[r >> 1]) : sm.first[r >> 1]) + head * D + E * lane;
                const float sx = __shfl_sync(0xffffffffu, share.x, r), sy = __shfl_sync(0xffffffffu, share.y, r);
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = fmaf(src[e] * sx, sy, o[e]);
            }
            if (!whole) {
                // the item goes on in other CTAs: the last of them to come here merges
                float* part = a.cta_part + (((size_t)blockIdx.x * 2 + (rec.begins ? 1 : 0)) * 8 + head) * kBlockPart;
#pragma unroll
                for (int e = 0; e < E; ++e) part[4 + E * lane + e] = o[e];
                if (lane == 0) *reinterpret_cast<float2*>(part) = make_float2(m, l);
                __syncwarp();
                const int c0 = cta_at(rec.start), c1 = cta_at(rec.start + rec.w - 1);
                int seen = 0;
                if (lane == 0) {
                    int* counter = a.counters + (size_t)rec.idx * 8 + head;
                    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(seen) : "l"(counter) : "memory");  // the warp's part lies before
                    if (seen == c1 - c0) *counter = 0;
                }
                if (__shfl_sync(0xffffffffu, seen, 0) != c1 - c0) continue;
                __syncwarp();  // lane 0 has seen the other CTAs' parts; a shuffle alone would not order the other lanes' loads behind that
                m = -INFINITY;
                l = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 1
                for (int base = c0; base <= c1; base += 32) {  // the statistics of 32 parts at once, then their O
                    auto part_of = [&](int cta) { return a.cta_part + (((size_t)cta * 2 + (cta == c0 ? 1 : 0)) * 8 + head) * kBlockPart; };
                    const int n = min(32, c1 - base + 1);
                    constexpr int U = 8;  // parts that are asked for together, the first of them with the statistics
                    float x[U][E];
                    auto ask = [&](int k0) {
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            if (k0 + u >= n) continue;
                            const float* src = part_of(base + k0 + u) + 4 + E * lane;
                            if constexpr (E == 4) {
                                const float4 v = __ldcg(reinterpret_cast<const float4*>(src));
                                x[u][0] = v.x, x[u][1] = v.y, x[u][2] = v.z, x[u][3] = v.w;
                            } else {
                                const float2 v = __ldcg(reinterpret_cast<const float2*>(src));
                                x[u][0] = v.x, x[u][1] = v.y;
                            }
                        }
                    };
                    const float2 ml = lane < n ? __ldcg(reinterpret_cast<const float2*>(part_of(base + lane))) : make_float2(-INFINITY, 0.f);
                    ask(0);
                    float nm = ml.x;
#pragma unroll
                    for (int k = 16; k; k >>= 1) nm = fmaxf(nm, __shfl_xor_sync(0xffffffffu, nm, k));
                    nm = fmaxf(nm, m);
                    const float old_half = root_diff(m, nm), old = l * old_half, half = root_diff(ml.x, nm), mine = ml.y * half;
                    float sum = mine * half;
#pragma unroll
                    for (int k = 16; k; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
                    l = fmaf(old, old_half, sum);
                    m = nm;
                    const float2 was = share_of(old_half, l == 0.f ? 0.f : __fdividef(old, l)), is = share_of(half, l == 0.f ? 0.f : __fdividef(mine, l));
#pragma unroll
                    for (int e = 0; e < E; ++e) o[e] = o[e] * was.x * was.y;
#pragma unroll 1
                    for (int k0 = 0; k0 < n; k0 += U) {
                        if (k0) ask(k0);
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            const float sx = __shfl_sync(0xffffffffu, is.x, (k0 + u) & 31), sy = __shfl_sync(0xffffffffu, is.y, (k0 + u) & 31);
                            if (k0 + u >= n) continue;
#pragma unroll
                            for (int e = 0; e < E; ++e) o[e] = fmaf(x[u][e] * sx, sy, o[e]);
                        }
                    }
                }
            }
            const size_t row = (((size_t)it.li * c.B + it.b) * c.Hkv + it.h) * c.G + head;
            uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + row * D) + E / 2 * lane;
            if constexpr (E == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
            else *dst = pack_bf16(o[0], o[1]);
            if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        }
    }
}

template <int D>
cudaError_t launch_d(const BlockAttendArgs& a, const BlockMaps& maps, cudaStream_t stream) {
    const size_t smem = sizeof(Smem<D>) + 1024;
    cudaError_t e = prepare_kernel((const void*)block_attend_kernel<D>, smem);
    return e != cudaSuccess ? e : launch_dependent(block_attend_kernel<D>, dim3(a.n_cta), kThreads, smem, stream, a, maps);
}

}  // namespace

bool build_block_maps(void* encode, const BlockView& c, BlockMaps* maps) {
    typedef CUresult (*encode_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    encode_fn fn = reinterpret_cast<encode_fn>(encode);
    const cuuint64_t dims[2] = {(cuuint64_t)c.D, (cuuint64_t)c.n_pages * c.T};
    const cuuint64_t pitch[1] = {(cuuint64_t)c.D};
    const cuuint32_t box[2] = {(cuuint32_t)c.D, (cuuint32_t)(c.T < kStep ? c.T : kStep)}, es[2] = {1, 1};
    const CUtensorMapSwizzle swizzle = c.D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
    for (int i = 0; i < 2; ++i)
        if (fn(i ? &maps->v : &maps->k, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, i ? c.v : c.k, dims, pitch, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return false;
    return true;
}

cudaError_t launch_block_attend(const BlockAttendArgs& a, const BlockMaps& maps, cudaStream_t stream) {
    return a.c.D == 128 ? launch_d<128>(a, maps, stream) : launch_d<64>(a, maps, stream);
}

}  // namespace lethe
