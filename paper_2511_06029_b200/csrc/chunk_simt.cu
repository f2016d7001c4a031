// lethe_chunk_attend on fp32 caches: CUDA-core kernels (the tensor cores have no full fp32 product).  Both are bound by the fp32
// FMA rate: 64 query rows by 32 keys per step, operands in shared memory, 4 x 2 logits and 4 x D / 16 outputs per thread, so that
// a 16-byte shared-memory read feeds 5 to 8 FMAs per operand.  A chunk of 33 tokens behind 512 (8 heads over 2 of 64): 46 us for the
// call, the launches' latency and a handful of steps; 58 with 64 keys per step and copies through registers.
#include "chunk.cuh"
#include "mma_utils.cuh"

namespace lethe {
namespace {

constexpr int kSimtThreads = 256;
constexpr int kRows = 64;   // query rows of a unit
constexpr int kKeys = 32;   // keys per step
constexpr int kPad = 4;     // row padding of the staged tiles: rows start in different banks

// Rows [j0, j0 + count) of K or V of an item on their way into shared memory, missing rows (at or beyond `end`, or on a page outside
// the pool) as zeros.
template <int D>
__device__ __forceinline__ void stage_rows(const ChunkArgs& a, const void* base, int item, int j0, int end, int count, float* dst, bool* bad) {
    for (int i = threadIdx.x; i < count * (D / 4); i += kSimtThreads) {
        const int r = i / (D / 4), c = i % (D / 4);
        long long at = -1;
        if (j0 + r < end) {
            at = chunk_row(a, item, j0 + r);
            if (at < 0) *bad = true;
        }
        cp_async16(smem_u32(dst + r * (D + kPad) + c * 4), (const float*)base + (size_t)max(at, 0LL) * D + c * 4, at >= 0 ? 16 : 0);
    }
}
// The same of query rows [r0, r0 + count) of a sequence's packed tokens, from token `tok`.
template <int D>
__device__ __forceinline__ void stage_queries(const ChunkArgs& a, const ChunkItem& it, int tok, int r0, int rows, int count, float* dst) {
    for (int i = threadIdx.x; i < count * (D / 4); i += kSimtThreads) {
        const int r = r0 + i / (D / 4), c = i % (D / 4), rr = min(r, rows - 1);
        const float* src = (const float*)a.q + (((size_t)it.li * a.n_tokens + it.first + tok + rr / a.G) * a.Hq + it.hkv * a.G + rr % a.G) * D + c * 4;
        cp_async16(smem_u32(dst + (i / (D / 4)) * (D + kPad) + c * 4), src, r < rows ? 16 : 0);
    }
}

// The logit of a visible key in log2 units, -inf for a hidden one.
__device__ __forceinline__ float shaped_logit(const ChunkArgs& a, const ChunkRow& row, float s, int j, int n, int kpos, float scale, int prefix) {
    if (!((j < row.lim || (kpos < prefix && j < n)) && kpos >= row.lo)) return -INFINITY;
    float x = s * scale;
    if (a.softcap > 0.f) x = a.softcap * capped(x / a.softcap);
    x *= 1.4426950408889634f;
    if (a.slopes) x -= row.slope * fabsf((float)((long long)row.qpos - kpos));
    return x;
}

template <int D>
__global__ void __launch_bounds__(kSimtThreads) chunk_simt_attend(const __grid_constant__ ChunkArgs a) {
    extern __shared__ __align__(16) float smem[];
    float* sq = smem;                        // [kRows][D + kPad]
    float* skv = sq + kRows * (D + kPad);    // two stages of K [kKeys][D + kPad] and V
    float* sp = skv + 4 * kKeys * (D + kPad);  // [kRows][kKeys + 1] probabilities
    dependency_wait();
    dependency_release();
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;  // thread: rows 4 ty .. + 3; keys tx, tx + 16; elements 4 tx + 64 i
    const int total = a.plan->total, per = a.plan->per;
    const int begin = min(total, (int)blockIdx.x * per), end = min(total, begin + per);
    if (begin >= end) return;
    bool bad = false;
    for (int u = a.cta_unit[blockIdx.x], at = begin; at < end; ++u) {
        const int s0 = a.u_start[u], s1 = a.u_start[u + 1];
        if (s1 <= at) continue;
        const int stop = min(end, s1);
        const int idx = u / a.QT, tok0 = (u - idx * a.QT) * a.TU;
        const ChunkItem it = chunk_item(a, idx);
        const int rows = min(it.T - tok0, a.TU) * a.G;
        const int base_tile = (a.u_lo ? a.u_lo[u] : 0) - s0;
        const float scale = a.scale[it.l];
        const int prefix = a.prefix_len ? a.prefix_len[it.b] : INT32_MIN;
        const int32_t* pos = a.pos + (size_t)it.item * a.cap_tokens;
        const bool by_pos = a.slopes || a.window || a.doc_start || a.prefix_len;
        __syncthreads();  // the previous unit's readers are done
        stage_queries<D>(a, it, tok0, 0, rows, kRows, sq);
        ChunkRow row[4];
        float m[4], l[4], o[4][D / 16];
        int slot_end = 0;  // slots from here on are hidden from the whole unit
        slot_end = a.u_hi ? a.u_hi[u] : (a.append ? it.n_old + min(it.T, tok0 + a.TU) : it.n_old);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = ty * 4 + i, tok = tok0 + min(r, rows - 1) / a.G;
            row[i].lim = r < rows ? it.n_old + (a.append ? tok + 1 : 0) : INT32_MIN;
            row[i].qpos = a.token_pos ? a.token_pos[it.first + tok] : 0;
            row[i].lo = r < rows ? chunk_lo(a, it.first + tok, row[i].qpos) : INT32_MAX;
            row[i].slope = a.slopes ? a.slopes[it.hkv * a.G + r % a.G] * 1.4426950408889634f : 0.f;
            m[i] = -INFINITY;
            l[i] = 0.f;
#pragma unroll
            for (int e = 0; e < D / 16; ++e) o[i][e] = 0.f;
        }
        // steps of kKeys keys, the next one's rows under way while this one is worked on
        const int j_begin = (base_tile + at) * a.tile, j_end = min((base_tile + stop) * a.tile, slot_end);
        auto stage = [&](int j0, int buf) {
            float* sk = skv + buf * 2 * kKeys * (D + kPad);
            stage_rows<D>(a, a.k, it.item, j0, slot_end, kKeys, sk, &bad);
            stage_rows<D>(a, a.v, it.item, j0, slot_end, kKeys, sk + kKeys * (D + kPad), &bad);
        };
        if (j_begin < j_end) stage(j_begin, 0);
        cp_async_commit();
        {
            int buf = 0;
            for (int j0 = j_begin; j0 < j_end; j0 += kKeys, buf ^= 1) {
                cp_async_wait<0>();
                __syncthreads();
                if (j0 + kKeys < j_end) stage(j0 + kKeys, buf ^ 1);
                cp_async_commit();
                const float* sk = skv + buf * 2 * kKeys * (D + kPad);
                const float* sv = sk + kKeys * (D + kPad);
                float s[4][2] = {};
#pragma unroll 4
                for (int d = 0; d < D; d += 4) {
                    const float4 k0 = *reinterpret_cast<const float4*>(sk + tx * (D + kPad) + d);
                    const float4 k1 = *reinterpret_cast<const float4*>(sk + (tx + 16) * (D + kPad) + d);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float4 x = *reinterpret_cast<const float4*>(sq + (ty * 4 + i) * (D + kPad) + d);
                        s[i][0] = fmaf(x.x, k0.x, fmaf(x.y, k0.y, fmaf(x.z, k0.z, fmaf(x.w, k0.w, s[i][0]))));
                        s[i][1] = fmaf(x.x, k1.x, fmaf(x.y, k1.y, fmaf(x.z, k1.z, fmaf(x.w, k1.w, s[i][1]))));
                    }
                }
                int kp[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) kp[h] = by_pos && j0 + tx + 16 * h < slot_end ? pos[j0 + tx + 16 * h] : 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int j = j0 + tx + 16 * h;
                        s[i][h] = j < slot_end ? shaped_logit(a, row[i], s[i][h], j, it.n, kp[h], scale, prefix) : -INFINITY;
                    }
                    float mx = fmaxf(s[i][0], s[i][1]);
#pragma unroll
                    for (int off = 8; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
                    mx = fmaxf(mx, m[i]);
                    const float ref = mx == -INFINITY ? 0.f : mx;
                    const float w = exp2_diff(m[i], ref), p0 = fast_exp2(s[i][0] - ref), p1 = fast_exp2(s[i][1] - ref);
                    m[i] = mx;
                    l[i] = l[i] * w + p0 + p1;  // this thread's share of the row sum
#pragma unroll
                    for (int e = 0; e < D / 16; ++e) o[i][e] *= w;
                    sp[(ty * 4 + i) * (kKeys + 1) + tx] = p0;
                    sp[(ty * 4 + i) * (kKeys + 1) + tx + 16] = p1;
                }
                __syncwarp();  // a row's sixteen threads are in one warp
#pragma unroll 4
                for (int j = 0; j < kKeys; ++j) {
                    float p[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[i] = sp[(ty * 4 + i) * (kKeys + 1) + j];
#pragma unroll
                    for (int e = 0; e < D / 64; ++e) {
                        const float4 v = *reinterpret_cast<const float4*>(sv + j * (D + kPad) + tx * 4 + 64 * e);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            o[i][4 * e] = fmaf(p[i], v.x, o[i][4 * e]);
                            o[i][4 * e + 1] = fmaf(p[i], v.y, o[i][4 * e + 1]);
                            o[i][4 * e + 2] = fmaf(p[i], v.z, o[i][4 * e + 2]);
                            o[i][4 * e + 3] = fmaf(p[i], v.w, o[i][4 * e + 3]);
                        }
                    }
                }
                __syncwarp();
            }
            cp_async_wait<0>();
        }
        const bool whole = at == s0 && stop == s1;
        const size_t part = ((size_t)blockIdx.x * 2 + (at == s0 ? 1 : 0)) * 2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], off);
            const int r = ty * 4 + i;
            if (r >= rows) continue;
            const int tok = tok0 + r / a.G, h = r % a.G;
            const size_t orow = ((size_t)it.li * a.n_tokens + it.first + tok) * a.Hq + it.hkv * a.G + h;
            const float mul = !whole ? 1.f : (l[i] == 0.f ? 0.f : 1.f / l[i]);
#pragma unroll
            for (int e = 0; e < D / 64; ++e) {
                if (whole) *reinterpret_cast<float4*>((float*)a.out + orow * D + tx * 4 + 64 * e) = make_float4(o[i][4 * e] * mul, o[i][4 * e + 1] * mul, o[i][4 * e + 2] * mul, o[i][4 * e + 3] * mul);
                else
#pragma unroll
                    for (int x = 0; x < 4; ++x) a.part_o[(part * D + tx * 4 + 64 * e + x) * kChunkPartRows + r] = o[i][4 * e + x];
            }
            if (tx == 0) {
                if (!whole) a.part_ml[part * kChunkPartRows + r] = make_float2(m[i], l[i]);
                else {
                    const float lse2 = l[i] == 0.f ? -INFINITY : m[i] + log2f(l[i]);
                    if (a.lse) a.lse[orow] = lse2 * 0.6931471805599453f;
                    a.nlse2[(((size_t)it.li * a.Hkv + it.hkv) * a.n_tokens + it.first + tok) * a.G + h] = l[i] == 0.f ? -INFINITY : -lse2;
                }
            }
        }
        if (bad) record_error(a.status, LETHE_ERR_PAGE, it.item);
        bad = false;
        at = stop;
    }
}

// Eq. 5 for the chunk: one block per (item, 32 keys); threads own 2 keys x 4 of 64 query rows per step and add up
// exp2(logit - lse + log2 of the row's decay weight).  The last launch that reads len: block 0 of an item stores the new one.
template <int D>
__global__ void __launch_bounds__(kSimtThreads) chunk_simt_rel(const __grid_constant__ ChunkArgs a) {
    extern __shared__ __align__(16) float smem[];
    float* sk = smem;                        // [kKeys][D + kPad]
    float* sqs = sk + kKeys * (D + kPad);    // two stages of [kRows][D + kPad]
    dependency_wait();
    const int per_item = (a.cap_tokens + kKeys - 1) / kKeys;
    const int idx = blockIdx.x / per_item, block = blockIdx.x - idx * per_item;
    const ChunkItem it = chunk_item(a, idx);
    if (it.n_old < 0 || it.T == 0) return;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;  // thread: keys ty, ty + 16; rows tx + 16 i
    if (block == 0 && tid == 0 && a.append) a.len[it.item] = it.n;
    const int j0 = block * kKeys;
    if (j0 >= it.n) return;
    bool bad = false;  // the attention has recorded bad pages
    stage_rows<D>(a, a.k, it.item, j0, it.n, kKeys, sk, &bad);
    const int rows = it.T * a.G;
    // rows before the first that reaches key j0 in causal order see nothing here, unless a prefix opens it to all
    const int first = a.append && !a.prefix_len ? max(0, j0 - it.n_old) * a.G & ~(kRows - 1) : 0;
    if (first < rows) stage_queries<D>(a, it, 0, first, rows, kRows, sqs);
    cp_async_commit();
    const float scale = a.scale[it.l];
    const int prefix = a.prefix_len ? a.prefix_len[it.b] : INT32_MIN;
    const bool by_pos = a.slopes || a.window || a.doc_start || a.prefix_len;
    int kp[2];
    float acc[2] = {}, old[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int j = j0 + ty + 16 * k;
        kp[k] = by_pos && j < it.n ? a.pos[(size_t)it.item * a.cap_tokens + j] : 0;
        old[k] = j < it.n_old ? a.rel[(size_t)it.item * a.cap_tokens + j] : 0.f;
    }
    int buf = 0;
    for (int r0 = first; r0 < rows; r0 += kRows, buf ^= 1) {
        cp_async_wait<0>();
        __syncthreads();
        if (r0 + kRows < rows) stage_queries<D>(a, it, 0, r0 + kRows, rows, kRows, sqs + (buf ^ 1) * kRows * (D + kPad));
        cp_async_commit();
        const float* sq = sqs + buf * kRows * (D + kPad);
        ChunkRow row[4];
        float bias[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = min(r0 + tx + 16 * i, rows - 1), tok = r / a.G;
            row[i].lim = r0 + tx + 16 * i < rows ? it.n_old + (a.append ? tok + 1 : 0) : INT32_MIN;
            row[i].qpos = a.token_pos ? a.token_pos[it.first + tok] : 0;
            row[i].lo = r0 + tx + 16 * i < rows ? chunk_lo(a, it.first + tok, row[i].qpos) : INT32_MAX;
            row[i].slope = a.slopes ? a.slopes[it.hkv * a.G + r % a.G] * 1.4426950408889634f : 0.f;
            bias[i] = a.nlse2[(((size_t)it.li * a.Hkv + it.hkv) * a.n_tokens + it.first) * a.G + r] + (float)(it.T - 1 - tok) * a.gamma_log2;
        }
        float s[2][4] = {};
#pragma unroll 4
        for (int d = 0; d < D; d += 4) {
            const float4 k0 = *reinterpret_cast<const float4*>(sk + ty * (D + kPad) + d);
            const float4 k1 = *reinterpret_cast<const float4*>(sk + (ty + 16) * (D + kPad) + d);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 x = *reinterpret_cast<const float4*>(sq + (tx + 16 * i) * (D + kPad) + d);
                s[0][i] = fmaf(x.x, k0.x, fmaf(x.y, k0.y, fmaf(x.z, k0.z, fmaf(x.w, k0.w, s[0][i]))));
                s[1][i] = fmaf(x.x, k1.x, fmaf(x.y, k1.y, fmaf(x.z, k1.z, fmaf(x.w, k1.w, s[1][i]))));
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = shaped_logit(a, row[i], s[k][i], j0 + ty + 16 * k, it.n, kp[k], scale, prefix);
                if (x != -INFINITY) acc[k] += fast_exp2(x + bias[i]);
            }
    }
    cp_async_wait<0>();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) acc[k] += __shfl_xor_sync(0xffffffffu, acc[k], off);
        const int j = j0 + ty + 16 * k;
        if (tx == 0 && j < it.n) a.rel[(size_t)it.item * a.cap_tokens + j] = fmaf(exp2f((float)it.T * a.gamma_log2), old[k], acc[k]);
    }
}

template <int D>
cudaError_t launch_t(const ChunkArgs& a, cudaStream_t stream) {
    const size_t smem = ((size_t)(kRows + 4 * kKeys) * (D + kPad) + kRows * (kKeys + 1)) * sizeof(float);
    const size_t smem_rel = (size_t)(kKeys + 2 * kRows) * (D + kPad) * sizeof(float);
    cudaError_t e = prepare_kernel((const void*)chunk_simt_attend<D>, smem);
    if (e == cudaSuccess) e = prepare_kernel((const void*)chunk_simt_rel<D>, smem_rel);
    if (e == cudaSuccess) e = launch_dependent(chunk_simt_attend<D>, dim3(a.n_cta), kSimtThreads, smem, stream, a);
    if (e == cudaSuccess) e = launch_chunk_combine(a, stream);
    if (e == cudaSuccess) e = launch_dependent(chunk_simt_rel<D>, dim3((a.cap_tokens + kKeys - 1) / kKeys * a.n_items), kSimtThreads, smem_rel, stream, a);
    return e;
}

}  // namespace

cudaError_t launch_chunk_simt(const ChunkArgs& a, cudaStream_t stream) {
    return a.D == 128 ? launch_t<128>(a, stream) : launch_t<64>(a, stream);
}

}  // namespace lethe
