// lethe_append: new rows into a cache, keys (and the same tokens' queries) rotated on the way.
//
// Bound by memory: each new row is read and written once.  A block takes one token and a run of its rows, K and V of the (layer, KV
// head) pairs first, then the queries, so the cosines and sines of the token's pairs are computed once per block, while the rows and the
// short chain of loads that says where a row goes (sequence, length, page) are on their way.
#include "block.cuh"
#include "kv8_utils.cuh"

namespace lethe {
namespace {

constexpr int kAppendThreads = 192;
constexpr int kFewRows = 16;   // rows per block where there are few tokens; even: K and V of an item stay together
constexpr int kManyRows = 48;  // otherwise: 384 tasks of bf16 rows of 128, two per thread

enum { kSame = 0, kE4m3 = 1, kE5m2 = 2 };

template <bool E5M2>
__device__ __forceinline__ uint2 to_bytes8(const uint4& w, float scale) {
    float f[8];
    Piece<__nv_bfloat16>::unpack(w, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __fdiv_rn(f[i], scale);
    return make_uint2(f32x2_to_fp8x2<E5M2>(f[0], f[1]) | (f32x2_to_fp8x2<E5M2>(f[2], f[3]) << 16),
                      f32x2_to_fp8x2<E5M2>(f[4], f[5]) | (f32x2_to_fp8x2<E5M2>(f[6], f[7]) << 16));
}

// What becomes of a row.
struct Row {
    char* dst;    // NULL: dropped
    float scale;  // byte caches
};

template <typename T, int KV, bool VEC, int U>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const __grid_constant__ AppendArgs a, int rows_total, int rows_per_block) {
    using P = Piece<T>;
    __shared__ float cs[64], sn[64];
    __shared__ Row rows[kManyRows];
    dependency_wait();
    dependency_release();
    const int tid = threadIdx.x;
    const int blocks = (rows_total + rows_per_block - 1) / rows_per_block;  // per token
    const int tok = blockIdx.x / blocks, r0 = (blockIdx.x - tok * blocks) * rows_per_block;
    const int n_rows = min(rows_total - r0, rows_per_block);
    const int kv_rows = 2 * a.nl * a.Hkv;
    const int per_row = a.D / (2 * P::N), shift = 31 - __clz(per_row);
    const int tasks = n_rows << shift;
    auto source = [&](int r, bool& rotated) -> const T* {
        if (r < kv_rows) {
            rotated = !(r & 1) && a.in.axis_pos;
            const int lh = r >> 1, li = lh / a.Hkv;
            return (const T*)(r & 1 ? a.in.v : a.in.k) + (((size_t)li * a.in.n_tokens + tok) * a.Hkv + lh - li * a.Hkv) * a.D;
        }
        rotated = true;
        const int rq = r - kv_rows, li = rq / a.Hq;
        return (const T*)a.in.q + (((size_t)li * a.in.n_tokens + tok) * a.Hq + rq - li * a.Hq) * a.D;
    };
    auto look = [&](int p, float& c, float& s) { c = cs[p], s = sn[p]; };

    // where the rows go; the angles
    int new_len = -1, len_item = 0;
    auto place = [&]() {
        if (a.in.axis_pos && tid < a.in.rot_dim / 2) pair_turn(a.in, tid, a.in.axis_pos[(size_t)a.in.axis[tid] * a.in.n_tokens + tok], cs[tid], sn[tid]);
        if (tid < n_rows) {
            const int r = r0 + tid;
            Row row = {nullptr, 1.f};
            const int first = a.in.chunk_start[0], last = a.in.chunk_start[a.B];
            if (tok >= first && tok < last) {
                if (r >= kv_rows) {
                    const int rq = r - kv_rows, li = rq / a.Hq;
                    row.dst = (char*)a.in.q_out + (((size_t)li * a.in.n_tokens + tok) * a.Hq + rq - li * a.Hq) * a.D * sizeof(T);
                } else {
                    int b = 0, hi = a.B;  // last b with chunk_start[b] <= tok: the sequence of this token (empty ones before it are passed over)
                    while (hi - b > 1) {
                        const int mid = (b + hi) >> 1;
                        if (a.in.chunk_start[mid] <= tok) b = mid;
                        else hi = mid;
                    }
                    const int s0 = a.in.chunk_start[b], n_new = a.in.chunk_start[b + 1] - s0;
                    const int lh = r >> 1, li = lh / a.Hkv, l = a.layer_begin + li;
                    const int item = (l * a.B + b) * a.Hkv + lh - li * a.Hkv;
                    const int n_old = min(max(a.len[item], 0), a.cap_tokens);
                    const bool key = !(r & 1);
                    if (n_new < 0 || n_old + (long long)n_new > a.cap_tokens) {
                        if (key && tok == s0) record_error(a.status, LETHE_ERR_CAPACITY, item);
                    } else {
                        const int slot = n_old + tok - s0;
                        long long at = (long long)item * a.capacity + slot;
                        if (a.paged) {
                            const int page = a.page_table[(size_t)item * a.capacity + slot / a.page_tokens];
                            at = page < 0 || page >= a.n_pages ? -1 : (long long)page * a.page_tokens + slot % a.page_tokens;
                        }
                        const size_t row_bytes = (size_t)a.D * (KV == kSame ? sizeof(T) : 1);
                        if (at >= 0) row.dst = (char*)(key ? a.k : a.v) + (size_t)at * row_bytes;
                        else if (key) record_error(a.status, LETHE_ERR_PAGE, item);
                        row.scale = key ? a.k_scale[l] : a.v_scale[l];
                        if (key) {
                            const size_t entry = (size_t)item * a.cap_tokens + slot;
                            a.pos[entry] = a.token_pos[tok];
                            a.rel[entry] = 0.f;
                            new_len = n_old + n_new;
                            len_item = item;
                        }
                    }
                }
            }
            rows[tid] = row;
        }
    };

    auto store = [&](int t, int at0, int at1, const uint4& x, const uint4& y) {
        const int i = t >> shift;
        const Row row = rows[i];
        if (!row.dst) return;
        if (KV == kSame || r0 + i >= kv_rows) {
            *reinterpret_cast<uint4*>(row.dst + at0 * sizeof(T)) = x;
            *reinterpret_cast<uint4*>(row.dst + at1 * sizeof(T)) = y;
        } else {
            *reinterpret_cast<uint2*>(row.dst + at0) = to_bytes8<KV == kE5m2>(x, row.scale);
            *reinterpret_cast<uint2*>(row.dst + at1) = to_bytes8<KV == kE5m2>(y, row.scale);
        }
    };
    bool ready = false;
    for (int t0 = 0; t0 < tasks; t0 += U * kAppendThreads) {  // uniform for the block
        uint4 x[U], y[U];
        int at0[U], at1[U];
        bool turned[U];
        if (VEC) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int t = t0 + u * kAppendThreads + tid;
                if (t < tasks) {
                    bool rotated;
                    const T* src = source(r0 + (t >> shift), rotated);
                    piece_pair<T>(a.in, t & (per_row - 1), rotated, at0[u], at1[u], turned[u]);
                    x[u] = *reinterpret_cast<const uint4*>(src + at0[u]);
                    y[u] = *reinterpret_cast<const uint4*>(src + at1[u]);
                }
            }
        }
        if (!ready) {
            if (!starts_ok(a.in.chunk_start, a.B, a.in.n_tokens, a.in.max_chunk)) {
                if (blockIdx.x == 0 && tid == 0) record_error(a.status, LETHE_ERR_INVALID_ARG, 0);
                return;
            }
            place();
            __syncthreads();
            // the item's one new token is this block's: every reader of its length is done
            if (a.in.max_chunk == 1 && new_len >= 0) a.len[len_item] = new_len;
            ready = true;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = t0 + u * kAppendThreads + tid;
            if (t < tasks) {
                if (VEC) {
                    if (turned[u]) turn_pieces<T>(a.in, at0[u], x[u], y[u], look);
                } else {
                    bool rotated;
                    const T* src = source(r0 + (t >> shift), rotated);
                    load_task<T, false>(a.in, src, t & (per_row - 1), rotated, look, at0[u], at1[u], x[u], y[u]);
                }
            }
            if (!VEC) __syncwarp();  // q_out may be q: a row's tasks lie in one warp, all have read before one writes
            if (t < tasks) store(t, at0[u], at1[u], x[u], y[u]);
        }
    }
}

// len of every item that took its tokens.
__global__ void __launch_bounds__(256) append_len_kernel(const int32_t* chunk_start, int32_t* len, int B, int Hkv, int layer_begin, int n_items, int n_tokens,
                                                         int max_chunk, int cap_tokens) {
    dependency_wait();
    dependency_release();
    if (!starts_ok(chunk_start, B, n_tokens, max_chunk)) return;
    const int idx = blockIdx.x * 256 + threadIdx.x;
    if (idx >= n_items) return;
    const BlockItem it = block_item(layer_begin, B, Hkv, idx);
    const int n_new = chunk_start[it.b + 1] - chunk_start[it.b], n_old = min(max(len[it.item], 0), cap_tokens);
    if (n_new > 0 && n_old + (long long)n_new <= cap_tokens) len[it.item] = n_old + n_new;
}

template <typename T, int KV>
cudaError_t launch_t(const AppendArgs& a, cudaStream_t stream) {
    const int rows = a.nl * (2 * a.Hkv + (a.in.q ? a.Hq : 0));
    // as in lethe_rotate: small blocks for the latency of few tokens, else the angles once per token
    const int per_block = a.in.n_tokens < 1024 ? kFewRows : kManyRows;
    const unsigned grid = (unsigned)a.in.n_tokens * (unsigned)((rows + per_block - 1) / per_block);
    const bool vec = !a.in.axis_pos || rotation_in_pieces<T>(a.in);
    if (!vec) return launch_dependent(append_kernel<T, KV, false, 1>, dim3(grid), kAppendThreads, 0, stream, a, rows, per_block);
    if (per_block > kFewRows) return launch_dependent(append_kernel<T, KV, true, 2>, dim3(grid), kAppendThreads, 0, stream, a, rows, per_block);
    return launch_dependent(append_kernel<T, KV, true, 1>, dim3(grid), kAppendThreads, 0, stream, a, rows, per_block);
}

}  // namespace

cudaError_t launch_append_len(const int32_t* chunk_start, int32_t* len, int B, int Hkv, int layer_begin, int n_items, int n_tokens, int max_chunk,
                              int cap_tokens, cudaStream_t stream) {
    return launch_dependent(append_len_kernel, dim3((n_items + 255) / 256), 256, 0, stream, chunk_start, len, B, Hkv, layer_begin, n_items, n_tokens, max_chunk,
                            cap_tokens);
}

cudaError_t launch_append(const AppendArgs& a, cudaStream_t stream) {
    cudaError_t e;
    switch (a.dtype) {
        case LETHE_F32: e = launch_t<float, kSame>(a, stream); break;
        case LETHE_BF16: e = launch_t<__nv_bfloat16, kSame>(a, stream); break;
        case LETHE_FP8_E4M3: e = launch_t<__nv_bfloat16, kE4m3>(a, stream); break;
        default: e = launch_t<__nv_bfloat16, kE5m2>(a, stream);
    }
    // with more than one token to a sequence several blocks need the old length
    if (e == cudaSuccess && a.in.max_chunk > 1)
        e = launch_append_len(a.in.chunk_start, a.len, a.B, a.Hkv, a.layer_begin, a.nl * a.B * a.Hkv, a.in.n_tokens, a.in.max_chunk, a.cap_tokens, stream);
    return e;
}

}  // namespace lethe
