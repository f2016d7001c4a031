// lethe_rotate: rotary positions with several axes, applied to the queries and keys of a step.
//
// Bound by memory: every element is read and written once.  A block takes one token and a run of its rows (heads of all layers,
// queries first, then keys), so the cosines and sines of the token's pairs are computed once per block, while the rows it has
// already asked for are on their way.  Angles: position x frequency is formed in turns as a 64-bit fraction, where the integer
// product's overflow is the reduction modulo one turn; the fraction is rounded to fp32 last.
// Measured: 8192 tokens of 32 + 8 heads of 128 in bf16, 168 MB both ways, 31 us = 5.4 TB/s, 0.83 of the copy rate (46 us with 16 rows
// per block and one task per thread); eight tokens 2.6 us on the device, 8 for a call.
#include "common.cuh"
#include "rotate.cuh"

namespace lethe {
namespace {

constexpr int kRotThreads = 160;
constexpr int kFewRows = 16;  // rows per block where there are few tokens
constexpr int kManyRows = 40; // otherwise: 320 tasks of bf16 rows of 128, two per thread
constexpr int kTasks = 2;

template <typename T>
struct Pack;  // 16 bytes of a row as floats
template <>
struct Pack<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void unpack(const uint4& w, float* f) {
        f[0] = __uint_as_float(w.x); f[1] = __uint_as_float(w.y); f[2] = __uint_as_float(w.z); f[3] = __uint_as_float(w.w);
    }
    static __device__ __forceinline__ uint4 pack(const float* f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};
template <>
struct Pack<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void two(uint32_t w, float* f) {
        f[0] = __uint_as_float(w << 16);
        f[1] = __uint_as_float(w & 0xffff0000u);
    }
    static __device__ __forceinline__ uint32_t one(float a, float b) {
        __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<uint32_t*>(&v);
    }
    static __device__ __forceinline__ void unpack(const uint4& w, float* f) { two(w.x, f); two(w.y, f + 2); two(w.z, f + 4); two(w.w, f + 6); }
    static __device__ __forceinline__ uint4 pack(const float* f) {
        return make_uint4(one(f[0], f[1]), one(f[2], f[3]), one(f[4], f[5]), one(f[6], f[7]));
    }
};

// Row r of token `tok`: rows 0 .. nl Hq - 1 are queries (layer-major), the rest keys.
template <typename T>
__device__ __forceinline__ void row_at(const RotateArgs& a, int tok, int r, const T*& src, T*& dst) {
    const int nq = a.nl * a.Hq;
    const bool key = r >= nq;
    const int H = key ? a.Hkv : a.Hq, rr = key ? r - nq : r;
    const size_t off = (((size_t)(rr / H) * a.n_tokens + tok) * H + rr % H) * a.D;
    src = (const T*)(key ? a.k : a.q) + off;
    dst = (T*)(key ? a.k_out : a.q_out) + off;
}

// VEC: pairs come in whole 16-byte pieces (HALVES: two pieces half a rotation apart; PAIRS: one piece holds whole pairs).
template <typename T, bool VEC, int U>
__global__ void __launch_bounds__(kRotThreads) rotate_kernel(const __grid_constant__ RotateArgs a) {
    using P = Pack<T>;
    __shared__ float cs[64], sn[64];
    dependency_wait();
    dependency_release();
    const int tid = threadIdx.x;
    const int blocks = (a.rows + a.rows_per_block - 1) / a.rows_per_block;  // per token
    const int tok = blockIdx.x / blocks, r0 = (blockIdx.x - tok * blocks) * a.rows_per_block;
    const int rows = min(a.rows - r0, a.rows_per_block);
    const int half = a.rot_dim / 2;
    auto angles = [&]() {
        if (tid < half) {
            const int pos = a.axis_pos[(size_t)a.axis[tid] * a.n_tokens + tok];
            const unsigned long long turn = (unsigned long long)(long long)pos * a.turn[tid];
            const int top = (int)((turn + 0x80000000ull) >> 32);  // the nearest 2^-32 turn, as a signed fraction
            float s, c;
            sincospif((float)top * 4.656612873077393e-10f, &s, &c);  // 2^-31: half turns
            cs[tid] = c;
            sn[tid] = a.inverse ? -s : s;
        }
        __syncthreads();
    };
    if (VEC) {
        // a task is one 16-byte piece (PAIRS), or the two pieces of as many pairs (HALVES), or a piece to copy; U tasks of a thread have
        // their loads in flight together
        const int rot_tasks = (a.halves ? half : a.rot_dim) / P::N;
        const int per_row = rot_tasks + (a.D - a.rot_dim) / P::N;
        const int tasks = rows * per_row;
        bool ready = false;
        for (int t0 = 0; t0 < tasks; t0 += U * kRotThreads) {  // uniform for the block
            uint4 x[U], y[U];
            T* dst[U];
            int at[U];
            bool copy[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int t = t0 + u * kRotThreads + tid;
                dst[u] = nullptr;
                if (t < tasks) {
                    const int r = t / per_row, c = t - r * per_row;
                    const T* src;
                    row_at<T>(a, tok, r0 + r, src, dst[u]);
                    copy[u] = c >= rot_tasks;
                    at[u] = copy[u] ? a.rot_dim + (c - rot_tasks) * P::N : c * P::N;
                    x[u] = *reinterpret_cast<const uint4*>(src + at[u]);
                    if (a.halves && !copy[u]) y[u] = *reinterpret_cast<const uint4*>(src + at[u] + half);
                }
            }
            if (!ready) angles();
            ready = true;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!dst[u]) continue;
                if (!copy[u]) {
                    float f[P::N], g[P::N];
                    P::unpack(x[u], f);
                    if (a.halves) {
                        P::unpack(y[u], g);
#pragma unroll
                        for (int i = 0; i < P::N; ++i) {
                            const float c = cs[at[u] + i], s = sn[at[u] + i], v = f[i], w = g[i];
                            f[i] = v * c - w * s;
                            g[i] = v * s + w * c;
                        }
                        *reinterpret_cast<uint4*>(dst[u] + at[u] + half) = P::pack(g);
                    } else {
#pragma unroll
                        for (int i = 0; i < P::N; i += 2) {
                            const float c = cs[(at[u] + i) / 2], s = sn[(at[u] + i) / 2], v = f[i], w = f[i + 1];
                            f[i] = v * c - w * s;
                            f[i + 1] = v * s + w * c;
                        }
                    }
                    x[u] = P::pack(f);
                }
                *reinterpret_cast<uint4*>(dst[u] + at[u]) = x[u];
            }
        }
    } else {
        angles();
        const int per_row = half + (a.D - a.rot_dim);  // pairs, then elements to copy
        for (int t = tid; t < rows * per_row; t += kRotThreads) {
            const int r = t / per_row, c = t - r * per_row;
            const T* src;
            T* dst;
            row_at<T>(a, tok, r0 + r, src, dst);
            if (c >= half) {
                dst[a.rot_dim + c - half] = src[a.rot_dim + c - half];
                continue;
            }
            const int i0 = a.halves ? c : 2 * c, i1 = a.halves ? c + half : 2 * c + 1;
            const float u = to_float<T>(src[i0]), w = to_float<T>(src[i1]);
            dst[i0] = from_float<T>(u * cs[c] - w * sn[c]);
            dst[i1] = from_float<T>(u * sn[c] + w * cs[c]);
        }
    }
}

template <typename T>
cudaError_t launch_t(const RotateArgs& a, cudaStream_t stream) {
    // whole 16-byte pieces: pairs that lie half a rotation apart need the half to be a multiple of a piece, neighbours the whole
    const bool vec = (a.halves ? a.rot_dim / 2 : a.rot_dim) % Pack<T>::N == 0;
    const unsigned grid = (unsigned)a.n_tokens * (unsigned)((a.rows + a.rows_per_block - 1) / a.rows_per_block);
    if (!vec) return launch_dependent(rotate_kernel<T, false, 1>, dim3(grid), kRotThreads, 0, stream, a);
    return a.rows_per_block > kFewRows ? launch_dependent(rotate_kernel<T, true, kTasks>, dim3(grid), kRotThreads, 0, stream, a)
                                       : launch_dependent(rotate_kernel<T, true, 1>, dim3(grid), kRotThreads, 0, stream, a);
}

}  // namespace

cudaError_t launch_rotate(const RotateArgs& args, bool f32, cudaStream_t stream) {
    RotateArgs a = args;
    // Few tokens: many small blocks, for the latency.  Many: more bytes in flight per thread and the angles once per token (8192
    // tokens of 32 + 8 heads of 128: 31 us = 5.4 TB/s, against 46 us with 16 rows and one task, 36 us with 24 or 48 rows).  The bound
    // between the two lies somewhere between 8 and 8192 tokens, where they were measured.  A block has one token's rows only, so a
    // model of few or narrow heads leaves some of its threads idle.
    a.rows_per_block = a.n_tokens < 1024 ? kFewRows : kManyRows;
    return f32 ? launch_t<float>(a, stream) : launch_t<__nv_bfloat16>(a, stream);
}

}  // namespace lethe
