// PTX wrappers and operand layouts shared by the tensor-core kernels of lethe_chunk_attend (tcgen05, TMA, mbarriers).
#pragma once
#include <cuda.h>

#include "chunk.cuh"
#include "mma_utils.cuh"

namespace lethe {

// Tensor maps: K and V as [items or pages][rows][D], Q as [nl][n_tokens][Hq][D]; 64-element (128-byte) inner boxes, 128-byte swizzle.
struct alignas(64) ChunkMaps {
    CUtensorMap k, v, q, q16;  // q: a whole row tile; q16: at most 16 rows of it
};

namespace {

constexpr int kTile = kChunkTile;          // rows of every operand tile
constexpr int kHalfBytes = kTile * 128;    // 64 elements of each of a tile's rows: one swizzled region
constexpr int kChunkWaitLimit = 400000;

template <int D>
__host__ __device__ constexpr int tile_bytes() { return kTile * D * 2; }

__device__ __forceinline__ void bar_init(unsigned long long* b, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(unsigned long long* b) {
    asm volatile("{ .reg .b64 st; mbarrier.arrive.shared::cta.b64 st, [%0]; }" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void bar_expect_tx(unsigned long long* b, unsigned bytes) {
    asm volatile("{ .reg .b64 st; mbarrier.arrive.expect_tx.shared::cta.b64 st, [%0], %1; }" ::"r"(smem_u32(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(unsigned long long* b, unsigned parity) {
    unsigned ok;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(ok) : "r"(smem_u32(b)), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool bar_test(unsigned long long* b, unsigned parity) {
    unsigned ok;
    asm volatile("{ .reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(ok) : "r"(smem_u32(b)), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded wait for the completion of phase `phase` (0, 1, 2, ...); false = gave up, or another thread already did.  The first look
// never blocks.
__device__ __forceinline__ bool bar_wait(unsigned long long* b, unsigned phase, volatile int* abort_flag, int limit) {
    const unsigned parity = phase & 1;
    if (bar_test(b, parity)) return true;
    for (int it = 1; it < limit; ++it) {
        if (bar_try(b, parity)) return true;
        if (*abort_flag) return false;
        if (it > 64) __nanosleep(64);
    }
    *abort_flag = 1;
    return false;
}
// The same for a whole warp, which goes on or gives up as one (collective instructions follow).
__device__ __forceinline__ bool warp_wait(unsigned long long* b, unsigned phase, volatile int* abort_flag, int limit) {
    return __all_sync(0xffffffffu, bar_wait(b, phase, abort_flag, limit));
}
// The same with the built-in limit and no abort flag: for what a CTA has started itself and must see end before it returns.
__device__ __forceinline__ void bar_drain(unsigned long long* b, unsigned phase) {
    for (int it = 0; it < kChunkWaitLimit; ++it) {
        if (bar_try(b, phase & 1)) return;
        if (it > 64) __nanosleep(64);
    }
}

// One lane of a converged warp: what it issues stays on the uniform datapath, where the MMA takes its descriptors from.
__device__ __forceinline__ bool elect_one() {
    unsigned ok;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(ok));
    return ok != 0;
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(unsigned long long* b) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, unsigned long long* b) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void tma_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, unsigned long long* b) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(b)) : "memory");
}

// Shared-memory descriptor of a tile kept as rows of 128 bytes with the 128-byte swizzle, 8-row groups 1024 bytes apart.
// K-major (the row is the M or N axis): the leading offset is unused.  MN-major (the row is the contraction axis, 64 elements of
// the other axis along it): the leading offset leads to the next 64 elements, one region further.
__device__ __forceinline__ uint64_t smem_desc(uint32_t saddr, uint32_t leading) {
    uint64_t d = 0;
    d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(leading >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
// tcgen05.mma.kind::f16, bf16 x bf16 -> fp32, M = 128, N columns; B K-major or MN-major, A optionally negated.
__device__ __forceinline__ uint32_t mma_idesc(int N, bool b_mn_major, bool negate_a) {
    uint32_t d = 0;
    d |= 1u << 4;
    d |= 1u << 7;
    d |= 1u << 10;
    d |= (negate_a ? 1u : 0u) << 13;
    d |= (b_mn_major ? 1u : 0u) << 16;
    d |= (uint32_t)(N >> 3) << 17;
    d |= (uint32_t)(kTile >> 4) << 24;
    return d;
}
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }"
        ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}

// 32 consecutive columns of this thread's TMEM lane (asynchronous: ld_wait before the registers are used).
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
          "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
          "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
          "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]),
          "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]),
          "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
          "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t two(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 apart(uint64_t x) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(x));
    return f;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// A NaN among them comes through.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// 2^x of two values on the FMA pipes, for a share of the exponentials that the special-function unit (16 a clock per SM) is the bound
// of: x = n + r with n the nearest whole number (the low bits of x + 1.5 * 2^23) and r in [-1/2, 1/2], 2^r by a polynomial fitted
// to the relative error (2.1e-7 in fp32), n added to the exponent.  x is at most 127 here; below
// -126 the result is 0 (for a NaN too: the callers look for those).
__device__ __forceinline__ float2 exp2_fma(float lo, float hi) {
    constexpr float c[6] = {1.0000000716545048f, 0.6931469670591965f, 0.2402211972442394f, 0.05550713282584675f, 0.009675541310994419f, 0.0013276469054922968f};
    const uint64_t x = two(fmaxf(lo, -126.f), fmaxf(hi, -126.f));
    const uint64_t t = add2(x, two(12582912.f, 12582912.f));
    const uint64_t r = fma2(add2(t, two(-12582912.f, -12582912.f)), two(-1.f, -1.f), x);
    uint64_t p = two(c[5], c[5]);
#pragma unroll
    for (int i = 4; i >= 0; --i) p = fma2(p, r, two(c[i], c[i]));
    const float2 pf = apart(p), tf = apart(t);
    const float a = __int_as_float(__float_as_int(pf.x) + (__float_as_int(tf.x) << 23)), b = __int_as_float(__float_as_int(pf.y) + (__float_as_int(tf.y) << 23));
    return make_float2(lo >= -126.f ? a : 0.f, hi >= -126.f ? b : 0.f);
}

// What the kernels are compiled for: code that a call does not need would only fill the instruction cache (packed documents, whose
// masks alone go by position, took 376 us before the code that shapes scores was compiled apart and 287 after; 274 today).
constexpr int kPlain = 0;   // causal only
constexpr int kMasked = 1;  // masks by position
constexpr int kCapped = 2;  // a cap, with or without masks
constexpr int kSloped = 3;  // slopes, with or without a cap and masks
__host__ __device__ constexpr bool shaped(int kind) { return kind >= kCapped; }
inline int score_kind(const ChunkArgs& a) {
    if (a.slopes) return kSloped;
    if (a.softcap > 0.f) return kCapped;
    return a.window > 0 || a.doc_start || a.prefix_len ? kMasked : kPlain;
}

__device__ __forceinline__ float fast_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// softcap * tanh(t) in log2 units (cap2 = softcap * log2(e)) of NC logits, t = v * cap_in: v times a polynomial in t^2 (five
// coefficients: 1.4e-7 of tanh in fp32) while |t| <= 0.55, else 1 - 2 / (1 + 2^(2 t log2 e)), which alone has an absolute error of an
// ulp of one: at small t that times the cap would cost a score its low bits, and so each logit takes its own form, whatever its
// neighbours are.  The second form is computed for a piece of sixteen columns that has a larger one, and chosen without a branch
// (512-token chunks with a cap and slopes 243 us; 234 when the whole piece took it).
// `care`: what this lane holds counts (rows that are not there may hold anything, which must not send the warp down the longer path).
template <int NC>
__device__ __forceinline__ void cap_scores(uint32_t* v, float cap_in, float cap2, bool care) {
    const float k = cap2 * cap_in, far = 0.55f / cap_in;
    const uint64_t far2 = two(2.8853900817779268f * cap_in, 2.8853900817779268f * cap_in);
    const uint64_t sq = two(cap_in * cap_in, cap_in * cap_in);
    const uint64_t c0 = two(0.9999999676367849f * k, 0.9999999676367849f * k), c1 = two(-0.3333279501836578f * k, -0.3333279501836578f * k);
    const uint64_t c2 = two(0.13318876828366036f * k, 0.13318876828366036f * k), c3 = two(-0.052589315256801286f * k, -0.052589315256801286f * k);
    const uint64_t c4 = two(0.01631543615226489f * k, 0.01631543615226489f * k);
#pragma unroll
    for (int c = 0; c < NC; c += 16) {
        float big = 0.f;
        uint64_t x[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) {
            big = max3(big, fabsf(__uint_as_float(v[c + 2 * y])), fabsf(__uint_as_float(v[c + 2 * y + 1])));
            x[y] = two(__uint_as_float(v[c + 2 * y]), __uint_as_float(v[c + 2 * y + 1]));
            const uint64_t u = mul2(mul2(x[y], x[y]), sq);
            const float2 r = apart(mul2(x[y], fma2(u, fma2(u, fma2(u, fma2(u, c4, c3), c2), c1), c0)));
            v[c + 2 * y] = __float_as_uint(r.x);
            v[c + 2 * y + 1] = __float_as_uint(r.y);
        }
        if (__any_sync(0xffffffffu, care && !(big <= far))) {  // some are outside the polynomial's range (or NaN)
#pragma unroll
            for (int y = 0; y < 8; ++y) {
                const float2 raw = apart(x[y]), t = apart(mul2(x[y], far2));
                const float2 e = apart(add2(two(fast_exp2(t.x), fast_exp2(t.y)), two(1.f, 1.f)));
                const float2 r = apart(fma2(two(fast_rcp(e.x), fast_rcp(e.y)), two(-2.f * cap2, -2.f * cap2), two(cap2, cap2)));
                if (!(fabsf(raw.x) <= far)) v[c + 2 * y] = __float_as_uint(r.x);
                if (!(fabsf(raw.y) <= far)) v[c + 2 * y + 1] = __float_as_uint(r.y);
            }
        }
    }
}

__device__ __forceinline__ void st_shared_16(uint32_t addr, const uint4& x) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}
// 16-byte chunk c of row r of a tile: halves of 64 elements are separate regions, chunks are swizzled by the row.
__device__ __forceinline__ uint32_t chunk_addr(uint32_t tile, int r, int c) {
    return tile + (c >> 3) * kHalfBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4);
}

// K or V rows [j0, j0 + 128) by TMA, issued by a converged warp: a contiguous item in one box per 64 elements, a paged one page by
// page, each lane its own.  Rows past the item's capacity, pages past its last slot and ids outside the pool read as zeros
// (coordinates outside the map).
template <int D>
struct TileLoader {
    int window = INT32_MIN, pages;        // page ids of 32 consecutive table entries, one per lane
    int ahead_at = INT32_MIN, ahead;      // and of the 32 before them, where a piece goes on
    bool bad = false;

    __device__ __forceinline__ int fetch(const ChunkArgs& a, int item, int n, int at) {
        const int i = at + (threadIdx.x & 31);
        if (i < 0 || (long long)i * a.page_tokens >= n) return (int)a.n_pages;  // outside the map: zeros
        const int page = a.page_table[(size_t)item * a.capacity + i];
        if (page >= 0 && page < a.n_pages) return page;
        bad = true;
        return (int)a.n_pages;
    }
    // a new item: nothing kept is of use
    __device__ __forceinline__ void reset() { window = ahead_at = INT32_MIN; }
    __device__ __forceinline__ void load(const ChunkArgs& a, const CUtensorMap* map, int item, int n, int j0, uint32_t dst, unsigned long long* bar) {
        const int lane = threadIdx.x & 31;
        if (!a.paged) {
            if (lane < D / 64) tma_3d(dst + lane * kHalfBytes, map, 64 * lane, j0, item, bar);
            return;
        }
        const int pt = a.page_tokens, per_tile = kTile / pt;  // pt is 8 .. 128 and divides 128: 1 .. 16 pages
        const int first = j0 / pt, want = first & ~31;        // tiles do not lie across windows
        if (want != window) {
            if (want == ahead_at) pages = ahead;
            else pages = fetch(a, item, n, want);
            window = want;
            ahead_at = want - 32;                             // tiles come last first
            ahead = fetch(a, item, n, ahead_at);
        }
        const int page = __shfl_sync(0xffffffffu, pages, (first & 31) + (lane & (per_tile - 1)));
        if (lane < per_tile)
#pragma unroll
            for (int hf = 0; hf < D / 64; ++hf) tma_3d(dst + hf * kHalfBytes + lane * pt * 128, map, 64 * hf, 0, page, bar);
    }
};

// Eight stored 8-bit floats as bf16 (exact).  The bits go where bf16 has them, sign on top and the exponent's and mantissa's bits
// joined below, and a multiplication by a power of two moves the exponent's bias over; zeros and subnormals come out right.  That
// takes five full-rate instructions for two elements; conversion instructions (through f16 and fp32) are fewer but run at a
// fraction of the rate.  Not for NaN and e5m2's infinities, whose exponent does not fit: `expand8_any`.
__device__ __forceinline__ uint4 expand8(uint2 w, bool e5m2) {
    const uint32_t mul = e5m2 ? 0x77807780u : 0x7b807b80u;  // 2^112, 2^120
    const uint32_t keep = e5m2 ? 0x0fe00fe0u : 0x07f007f0u;
    const int shift = e5m2 ? 3 : 4;
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t v = __byte_perm(i < 2 ? w.x : w.y, 0u, i & 1 ? 0x3424 : 0x1404);  // each byte on top of its 16 bits
        const uint32_t x = (v & 0x80008000u) | ((v >> shift) & keep);
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(o[i]) : "r"(x), "r"(mul));
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}
// Nonzero where a byte of w has the largest exponent (e4m3: is NaN).
__device__ __forceinline__ uint32_t special_bytes(uint32_t w, bool e5m2) { return ((w & 0x7f7f7f7fu) + (e5m2 ? 0x04040404u : 0x01010101u)) & 0x80808080u; }
__device__ __noinline__ uint4 expand8_any(uint2 w, bool e5m2) {
    uint32_t h[4], o[4];
    if (e5m2) {  // an e5m2 byte is the upper byte of the half of the same value
        h[0] = __byte_perm(w.x, 0u, 0x1404); h[1] = __byte_perm(w.x, 0u, 0x3424);
        h[2] = __byte_perm(w.y, 0u, 0x1404); h[3] = __byte_perm(w.y, 0u, 0x3424);
    } else {
        asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %2; cvt.rn.f16x2.e4m3x2 %0, lo; cvt.rn.f16x2.e4m3x2 %1, hi; }" : "=r"(h[0]), "=r"(h[1]) : "r"(w.x));
        asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %2; cvt.rn.f16x2.e4m3x2 %0, lo; cvt.rn.f16x2.e4m3x2 %1, hi; }" : "=r"(h[2]), "=r"(h[3]) : "r"(w.y));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; cvt.f32.f16 %0, l; cvt.f32.f16 %1, h; }" : "=f"(lo), "=f"(hi) : "r"(h[i]));
        o[i] = pack_bf16(lo, hi);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

// The same tile by NT threads with plain loads: any page size, any storage type.  A thread holds its 16-byte pieces of a stored tile in
// registers between `load` and `store`, so that the next tile's loads run under this one's conversion and the wait for its slot.
// Rows at or beyond `end` are zeros.
template <int D, int NT>
struct Gather {
    static constexpr int kByteLoads = kTile * D / 16 / NT;  // 16 bytes: 16 elements of a byte cache, 8 of a bf16 one (two loads then)
    uint4 x[kByteLoads];

    // half: which half of the columns (bf16: a register tile is half a tile wide)
    __device__ __forceinline__ void load(const ChunkArgs& a, const void* base, int item, int end, int j0, unsigned tid, int half, bool* bad) {
        const bool bytes = a.dtype != LETHE_BF16;
        constexpr unsigned C = D / 16;       // 16-byte pieces of a row of bytes, or of half a bf16 row
        constexpr unsigned kStep = NT / C;   // rows from one piece of a thread to its next
        const unsigned r0 = tid / C, c = tid % C;
        const size_t row_bytes = bytes ? D : 2 * D;
        const char* col = (const char*)base + (bytes ? c : half * C + c) * 16;
        const int left = end - j0 - (int)r0;  // rows of the tile from this thread's first on that there are
        if (!a.paged) {
            const char* src = col + ((size_t)item * a.capacity + j0 + r0) * row_bytes;
#pragma unroll
            for (int u = 0; u < kByteLoads; ++u)
                x[u] = (int)(u * kStep) < left ? *reinterpret_cast<const uint4*>(src + u * kStep * row_bytes) : make_uint4(0, 0, 0, 0);
            return;
        }
#pragma unroll
        for (int u = 0; u < kByteLoads; ++u) {
            x[u] = make_uint4(0, 0, 0, 0);
            if ((int)(u * kStep) < left) {
                long long at;
                if (bytes) {  // 16-token pages
                    const unsigned slot = j0 + r0 + u * kStep;
                    const int page = a.page_table[(size_t)item * a.capacity + (slot >> 4)];
                    at = page < 0 || page >= a.n_pages ? -1 : (long long)page * 16 + (slot & 15);
                } else at = chunk_row(a, item, j0 + r0 + u * kStep);
                if (at < 0) *bad = true;
                else x[u] = *reinterpret_cast<const uint4*>(col + (size_t)at * row_bytes);
            }
        }
    }
    __device__ __forceinline__ void store(const ChunkArgs& a, uint32_t dst, unsigned tid, int half) const {
        constexpr unsigned C = D / 16;
        const bool e5m2 = a.dtype == LETHE_FP8_E5M2;
        if (a.dtype == LETHE_BF16) {
#pragma unroll
            for (int u = 0; u < kByteLoads; ++u) {
                st_shared_16(chunk_addr(dst, tid / C + u * (NT / C), half * C + tid % C), x[u]);
            }
            return;
        }
        uint32_t special = 0;
#pragma unroll
        for (int u = 0; u < kByteLoads; ++u) special |= special_bytes(x[u].x, e5m2) | special_bytes(x[u].y, e5m2) | special_bytes(x[u].z, e5m2) | special_bytes(x[u].w, e5m2);
        if (!special) {
#pragma unroll
            for (int u = 0; u < kByteLoads; ++u) {
                const unsigned r = tid / C + u * (NT / C), c = tid % C;
                st_shared_16(chunk_addr(dst, r, 2 * c), expand8(make_uint2(x[u].x, x[u].y), e5m2));
                st_shared_16(chunk_addr(dst, r, 2 * c + 1), expand8(make_uint2(x[u].z, x[u].w), e5m2));
            }
        } else {
#pragma unroll
            for (int u = 0; u < kByteLoads; ++u) {
                const unsigned r = tid / C + u * (NT / C), c = tid % C;
                st_shared_16(chunk_addr(dst, r, 2 * c), expand8_any(make_uint2(x[u].x, x[u].y), e5m2));
                st_shared_16(chunk_addr(dst, r, 2 * c + 1), expand8_any(make_uint2(x[u].z, x[u].w), e5m2));
            }
        }
    }
};

// Whether K and V tiles can come by TMA: bf16 rows, and pages that tile the 128 rows in whole swizzle groups.
inline bool tma_can_tile(const ChunkArgs& a) {
    if (a.dtype != LETHE_BF16) return false;
    return !a.paged || (a.page_tokens >= 8 && kTile % a.page_tokens == 0 && a.n_pages <= 0x7ffffffeLL);
}

}  // namespace

// encode: cuTensorMapEncodeTiled; false = a map could not be made.
bool build_chunk_maps(void* encode, const ChunkArgs& a, int n_layers, ChunkMaps* maps);
cudaError_t launch_chunk_tc(const ChunkArgs& a, const ChunkMaps& maps, cudaStream_t stream);
cudaError_t launch_chunk_rel_tc(const ChunkArgs& a, const ChunkMaps& maps, cudaStream_t stream);

}  // namespace lethe
