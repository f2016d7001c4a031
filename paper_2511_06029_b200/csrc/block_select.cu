// lethe_block_select: the blocks that a query may profit from, by an upper bound of what their keys can reach.
//
// The bound of one element is max(qx * least, qx * greatest): the greatest for qx >= 0, the least otherwise.  Summed over the G heads of
// a group it is  sum_d greatest_d * up_d + least_d * down_d  with up_d / down_d the sums of the heads' positive / negative codes, so a
// block costs 2 D multiplications whatever G is.  Whole numbers: |up|, |down| <= 8 * 127 fit 16 bits, the sum stays below 2^24.
// Bound by memory: 2 D bytes for each block.  The blocks of an item are split over several thread blocks; the last of them to finish
// selects: the n-th greatest key by histograms over a narrowing range, then one ordered pass.
// Measured: 64 items of 1024 blocks, 17 MB, 11 us (13.5 with inputs that come from memory), of which 4 until the scores are there, 1 for the
// arrival and 4 for choosing 64 of them (three ranges, five barriers each): a launch's chain of latencies, not the bytes (2.6 us).  Four
// blocks of a lane in flight instead of two take 73 registers and with them a second wave: 2.5 us more.
#include "block.cuh"

namespace lethe {
namespace {

constexpr int kThreads = 256;
constexpr int kKeep = 8192;  // scores that the selection keeps in shared memory; beyond, it reads them again

// Order-preserving map of a finite float to 32 bits.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int dp2a(int a16, int b8, int c, bool high) {
    return high ? __dp2a_hi(a16, b8, c) : __dp2a_lo(a16, b8, c);
}

// Sum of v over the block, and what comes before this thread.
__device__ __forceinline__ int block_scan(int v, int* table, int& before) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) table[w] = x;
    __syncthreads();
    int base = 0, total = 0;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) {
        if (i < w) base += table[i];
        total += table[i];
    }
    before = base + x - v;
    return total;
}

template <int D>
__global__ void __launch_bounds__(kThreads) block_select_kernel(const __grid_constant__ BlockView c, const __nv_bfloat16* q, int n_select, int sink, int recent,
                                                                float* scores, int* counters, int splits, int32_t* selected) {
    __shared__ uint32_t keep[kKeep];
    __shared__ int hist[256];
    __shared__ int table[kThreads / 32];
    __shared__ float tops[kThreads / 32];
    __shared__ __align__(16) int16_t up[128], down[128];
    __shared__ int found[2], last;
    dependency_wait();
    dependency_release();
    const int tid = threadIdx.x, lane = tid & 31;
    const int idx = blockIdx.x / splits, split = blockIdx.x - idx * splits;
    const BlockItem it = block_item(c.layer_begin, c.B, c.Hkv, idx);
    const int full = block_len(c, it.item) >> c.t_shift;
    int32_t* list = selected + (size_t)idx * n_select;
    if (full <= n_select) {
        if (split == 0)
            for (int i = tid; i < n_select; i += kThreads) list[i] = i < full ? i : -1;
        return;
    }
    const int per = (full + splits - 1) / splits, blk0 = split * per, blk1 = min(full, blk0 + per);

    // D / 16 lanes to a block, each with 16 elements of both bounds; U blocks of a lane in flight, the first of them before the queries
    constexpr int kLanes = D / 16, kTeams = kThreads / kLanes, U = 2;
    const int part = tid % kLanes, team = tid / kLanes;
    long long page[U];
    uint4 down_to[U], up_to[U];
    float ks[U];
    auto ask = [&](int base) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int blk = base + k * kTeams + team;
            page[k] = blk < blk1 ? block_page(c, it.item, blk) : -1;
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            down_to[k] = up_to[k] = make_uint4(0, 0, 0, 0);
            ks[k] = 0.f;
            if (page[k] >= 0) {
                const uint4* r = reinterpret_cast<const uint4*>(c.k_range + (size_t)page[k] * 2 * D) + part;
                // not the read-only path: this grid may be alive while the append before it still writes them
                down_to[k] = __ldcg(r);
                up_to[k] = __ldcg(r + D / 16);
                ks[k] = __ldcg(c.k_scale + page[k]);
            }
        }
    };
    ask(blk0);

    // the group's queries as codes, summed over the heads by sign
    const __nv_bfloat16* qi = q + (((size_t)it.li * c.B + it.b) * c.Hkv + it.h) * c.G * D;
    float top = 0.f;
    for (int i = tid; i < c.G * D; i += kThreads) {
        const float m = fabsf(__bfloat162float(qi[i]));
        if (m < INFINITY) top = fmaxf(top, m);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) tops[tid >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) top = fmaxf(top, tops[w]);
    const float inv = top >= kBlockTiny ? __fdiv_rn(127.f, top) : 0.f;
    if (tid < D) {
        int u = 0, d = 0;
        for (int g = 0; g < c.G; ++g) {
            const int x = min(max(__float2int_rn(__bfloat162float(qi[g * D + tid]) * inv), -127), 127);
            u += max(x, 0);
            d += min(x, 0);
        }
        up[tid] = (int16_t)u;
        down[tid] = (int16_t)d;
    }
    __syncthreads();

    int cu[8], cd[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        cu[i] = reinterpret_cast<const int*>(up)[part * 8 + i];
        cd[i] = reinterpret_cast<const int*>(down)[part * 8 + i];
    }
    float* mine = scores + (size_t)idx * c.capacity;
#pragma unroll 1
    for (int base = blk0; base < blk1; base += U * kTeams) {
        if (base > blk0) ask(base);
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const uint32_t h[4] = {up_to[k].x, up_to[k].y, up_to[k].z, up_to[k].w}, l[4] = {down_to[k].x, down_to[k].y, down_to[k].z, down_to[k].w};
            int sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum = dp2a(cu[i], (int)h[i / 2], sum, i & 1);
                sum = dp2a(cd[i], (int)l[i / 2], sum, i & 1);
            }
#pragma unroll
            for (int o = 1; o < kLanes; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const int blk = base + k * kTeams + team;
            if (part == 0 && blk < blk1) {
                mine[blk] = __fmul_rn(ks[k], (float)sum) + 0.f;  // no negative zero
                if (page[k] < 0) record_error(c.status, LETHE_ERR_PAGE, it.item);
            }
        }
    }
    if (splits > 1) {
        __syncthreads();
        if (tid == 0) {
            int seen;
            asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(seen) : "l"(counters + idx) : "memory");  // the block's scores lie before
            last = seen == splits - 1;
            if (last) counters[idx] = 0;
        }
        __syncthreads();
        if (!last) return;
    } else {
        __syncthreads();
    }

    // candidates lie between the blocks that are always chosen; fewer than all of them are wanted
    const int first = sink, end = full - recent;
    const int wanted = n_select - sink - recent;
    const bool kept = end - first <= kKeep;
    uint32_t least = 0xffffffffu, greatest = 0;
    for (int i = first + tid; i < end; i += kThreads) {
        const uint32_t k = key_of(__ldcg(mine + i));
        if (kept) keep[i - first] = k;
        least = min(least, k);
        greatest = max(greatest, k);
    }
    least = __reduce_min_sync(0xffffffffu, least);
    greatest = __reduce_max_sync(0xffffffffu, greatest);
    if (tid == 0) found[0] = -1, found[1] = 0;
    __syncthreads();
    if (lane == 0) {
        atomicMin(reinterpret_cast<unsigned*>(&found[0]), least);
        atomicMax(reinterpret_cast<unsigned*>(&found[1]), greatest);
    }
    __syncthreads();
    uint32_t lo = (uint32_t)found[0], hi = (uint32_t)found[1];
    auto key_at = [&](int i) { return kept ? keep[i - first] : key_of(__ldcg(mine + i)); };
    // keys above hi are chosen, `need` more come from [lo, hi]
    int need = wanted;
    while (need > 0 && lo < hi) {
        const int shift = max(0, 24 - __clz(hi - lo));  // at most 256 buckets
        hist[tid] = 0;
        __syncthreads();
        for (int i = first + tid; i < end; i += kThreads) {
            const uint32_t k = key_at(i);
            if (k >= lo && k <= hi) atomicAdd(&hist[(k - lo) >> shift], 1);
        }
        __syncthreads();
        const int bucket = 255 - tid, count = hist[bucket];  // from the top
        int before;
        block_scan(count, table, before);
        if (before < need && before + count >= need) {
            found[0] = bucket;
            found[1] = before;
        }
        __syncthreads();
        const uint32_t new_lo = lo + ((uint32_t)found[0] << shift);
        const uint32_t width = (shift ? (1u << shift) : 1u) - 1u;
        need -= found[1];
        const bool whole = hist[found[0]] == need;  // all of the bucket
        hi = min(hi - new_lo, width) + new_lo;
        lo = new_lo;
        __syncthreads();  // found and hist are written again
        if (whole) break;
    }
    // in [lo, hi]: either all are chosen (need of them), or lo == hi and the first `need`
    const int run = (end - first + kThreads - 1) / kThreads, i0 = min(end, first + tid * run), i1 = min(end, i0 + run);
    int above = 0, equal = 0;
    for (int i = i0; i < i1; ++i) {
        const uint32_t k = key_at(i);
        if (k > hi) ++above;
        else if (k >= lo) ++equal;
    }
    int above_before, equal_before;
    block_scan(above, table, above_before);
    block_scan(equal, table, equal_before);
    int at = sink + above_before + min(equal_before, need);
    for (int i = i0; i < i1; ++i) {
        const uint32_t k = key_at(i);
        const bool in_range = k >= lo && k <= hi;
        if (k > hi || (in_range && equal_before < need)) list[at++] = i;
        equal_before += in_range;
    }
    for (int i = tid; i < sink; i += kThreads) list[i] = i;
    for (int i = tid; i < recent; i += kThreads) list[n_select - recent + i] = end + i;
}

}  // namespace

cudaError_t launch_block_select(const BlockView& c, const void* q, int n_select, int sink, int recent, float* scores, int* counters, int splits,
                                int32_t* selected, cudaStream_t stream) {
    const dim3 grid((unsigned)c.n_items * splits);
    return c.D == 128 ? launch_dependent(block_select_kernel<128>, grid, kThreads, 0, stream, c, (const __nv_bfloat16*)q, n_select, sink, recent, scores, counters, splits, selected)
                      : launch_dependent(block_select_kernel<64>, grid, kThreads, 0, stream, c, (const __nv_bfloat16*)q, n_select, sink, recent, scores, counters, splits, selected);
}

}  // namespace lethe
