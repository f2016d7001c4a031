// lethe_append: new rows into a cache, keys (and the same tokens' queries) rotated on the way.
//
// Bound by memory: each new row is read and written once.  A block takes a few tokens and a run of their rows, K and V of the (layer, KV
// head) pairs first, then the queries, so the cosines and sines of a token's pairs are computed once per block, while the rows and the
// chain of loads that says where a row goes (sequence, length, page) are on their way.
// Measured: 8192 tokens of 32 + 8 + 8 heads of 128 in bf16, 202 MB both ways, 40 us = 5.1 TB/s, 0.77 of the copy rate (one token to a block
// 45, four 43, 384 threads 49; a block lives about 7 us, of which 2 until it knows where its rows go); single tokens of 8 sequences and 32
// layers 4.4 us on the device.
#include "block.cuh"
#include "kv8_utils.cuh"

namespace lethe {
namespace {

constexpr int kAppendThreads = 192;
constexpr int kFewRows = 16;   // rows per block of one token; even: K and V of an item stay together
constexpr int kManyRows = 48;  // rows per block of kManyTokens tokens
constexpr int kManyTokens = 2;
// Small blocks of one token, for the latency, up to this many of them; else what a block does once, the chain of loads above all, serves
// two tokens.  Both sides (us, one token first): 768 blocks 5.8 and 6.4, 1536 blocks 8.5 and 7.1, 2304 blocks 10.6 and 8.0; single tokens of 8
// sequences and 32 layers (768) 5.1 and 5.8, of 16 (1536) 8.0 and 6.1.
constexpr int kManyBlocks = 1024;

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
    bool cached;  // K or V, else a query
};

// TK tokens and rows_per_block rows of each to a block; a task is 2 x 16 bytes of a row, those of the TK tokens in flight together.
template <typename T, int KV, bool VEC, int TK>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const __grid_constant__ AppendArgs a, int rows_total, int rows_per_block, bool sets_len) {
    using P = Piece<T>;
    constexpr int kRows = TK > 1 ? kManyRows : kFewRows;
    __shared__ __align__(16) float cs[TK][64], sn[TK][64];
    __shared__ Row rows[TK * kRows];
    __shared__ int starts[kStartsKept];
    dependency_wait();
    dependency_release();
    const int tid = threadIdx.x;
    const int blocks = (rows_total + rows_per_block - 1) / rows_per_block;  // per group of tokens
    const int group = blockIdx.x / blocks, r0 = (blockIdx.x - group * blocks) * rows_per_block, tok0 = group * TK;
    const int n_rows = min(rows_total - r0, rows_per_block), n_tok = min(a.in.n_tokens - tok0, TK);
    const int kv_rows = 2 * a.nl * a.Hkv;
    const int per_row = a.D / (2 * P::N), shift = 31 - __clz(per_row);
    const int tasks = n_rows << shift;
    // a row of the first token, and how far those of the next tokens lie apart
    auto source = [&](int r, size_t& pitch, bool& rotated) -> const T* {
        if (r < kv_rows) {
            rotated = !(r & 1) && a.in.axis_pos;
            const int lh = r >> 1, li = lh / a.Hkv;
            pitch = (size_t)a.Hkv * a.D;
            return (const T*)(r & 1 ? a.in.v : a.in.k) + (((size_t)li * a.in.n_tokens + tok0) * a.Hkv + lh - li * a.Hkv) * a.D;
        }
        rotated = true;
        const int rq = r - kv_rows, li = rq / a.Hq;
        pitch = (size_t)a.Hq * a.D;
        return (const T*)a.in.q + (((size_t)li * a.in.n_tokens + tok0) * a.Hq + rq - li * a.Hq) * a.D;
    };

    // where the rows go; the angles
    int new_len = -1, len_item = 0;
    auto place = [&]() {
        static_assert(kAppendThreads % 64 == 0, "a thread's angles are all of one pair");
        const int p = tid & 63;
        if (a.in.axis_pos && p < a.in.rot_dim / 2) {
            const int32_t* pos = a.in.axis_pos + (size_t)axis_of(a.in, p) * a.in.n_tokens + tok0;
            const unsigned long long per_pos = turn_of(a.in, p);
            for (int ti = tid >> 6; ti < n_tok; ti += kAppendThreads / 64) turn_by(per_pos, pos[ti], cs[ti][p], sn[ti][p]);
        }
        const int32_t* start = a.B < kStartsKept ? starts : a.in.chunk_start;
        for (int v = tid; v < n_rows * TK; v += kAppendThreads) {
            const int ti = v % TK, i = v / TK, r = r0 + i, tok = tok0 + ti;
            Row row = {nullptr, 1.f, false};
            if (ti < n_tok && tok >= start[0] && tok < start[a.B]) {
                if (r >= kv_rows) {
                    const int rq = r - kv_rows, li = rq / a.Hq;
                    row.dst = (char*)a.in.q_out + (((size_t)li * a.in.n_tokens + tok) * a.Hq + rq - li * a.Hq) * a.D * sizeof(T);
                } else {
                    const int b = sequence_of(start, a.B, tok), s0 = start[b], n_new = start[b + 1] - s0;
                    const int lh = r >> 1, li = lh / a.Hkv, l = a.layer_begin + li;
                    const int item = (l * a.B + b) * a.Hkv + lh - li * a.Hkv;
                    const int n_old = min(max(a.len[item], 0), a.cap_tokens);
                    const bool key = !(r & 1);
                    if (n_old + (long long)n_new > a.cap_tokens) {
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
                        row.cached = true;
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
            rows[v] = row;
        }
    };
    auto store = [&](const Row& row, int at0, int at1, const uint4& x, const uint4& y) {
        if (!row.dst) return;
        if (KV == kSame || !row.cached) {
            *reinterpret_cast<uint4*>(row.dst + at0 * sizeof(T)) = x;
            *reinterpret_cast<uint4*>(row.dst + at1 * sizeof(T)) = y;
        } else {
            *reinterpret_cast<uint2*>(row.dst + at0) = to_bytes8<KV == kE5m2>(x, row.scale);
            *reinterpret_cast<uint2*>(row.dst + at1) = to_bytes8<KV == kE5m2>(y, row.scale);
        }
    };
    bool ready = false;
    for (int t0 = 0; t0 < tasks; t0 += kAppendThreads) {  // uniform for the block
        const int t = t0 + tid, i = t >> shift;
        const bool there = t < tasks;
        uint4 x[TK], y[TK];
        int at0 = 0, at1 = 0;
        bool rotated = false, turned = false;
        size_t pitch = 0;
        const T* src = there ? source(r0 + i, pitch, rotated) : nullptr;
        if (VEC && there) {
            piece_pair<T>(a.in, t & (per_row - 1), rotated, at0, at1, turned);
#pragma unroll
            for (int u = 0; u < TK; ++u)
                if (u < n_tok) {
                    x[u] = *reinterpret_cast<const uint4*>(src + u * pitch + at0);
                    y[u] = *reinterpret_cast<const uint4*>(src + u * pitch + at1);
                }
        }
        if (!ready) {
            if (!starts_ok(a.in.chunk_start, a.B, a.in.n_tokens, a.in.max_chunk, starts)) {
                if (blockIdx.x == 0 && tid == 0) record_error(a.status, LETHE_ERR_INVALID_ARG, 0);
                return;
            }
            place();
            __syncthreads();
            // the item's one new token is this block's: every reader of its length is done
            if (sets_len && new_len >= 0) a.len[len_item] = new_len;
            ready = true;
        }
#pragma unroll
        for (int u = 0; u < TK; ++u) {
            const bool now = there && u < n_tok;
            if (VEC) {
                if (now && turned) {
                    float c[P::N], s[P::N];
                    const int p0 = first_pair(a.in, at0);
                    look_up(cs[u] + p0, c);
                    look_up(sn[u] + p0, s);
                    turn_pieces<T>(a.in, x[u], y[u], c, s);
                }
            } else {
                if (now) {
                    if (rotated) {
                        load_by_element<T>(a.in, src + u * pitch, t & (per_row - 1), [&](int p, float& c, float& s) { c = cs[u][p], s = sn[u][p]; }, at0, at1, x[u], y[u]);
                    } else {
                        piece_pair<T>(a.in, t & (per_row - 1), false, at0, at1, turned);
                        x[u] = *reinterpret_cast<const uint4*>(src + u * pitch + at0);
                        y[u] = *reinterpret_cast<const uint4*>(src + u * pitch + at1);
                    }
                }
                __syncwarp();  // q_out may be q: a row's tasks lie in one warp, all have read before one writes
            }
            if (now) store(rows[i * TK + u], at0, at1, x[u], y[u]);
        }
    }
}

// len of every item that took its tokens.
__global__ void __launch_bounds__(256) append_len_kernel(const int32_t* chunk_start, int32_t* len, int B, int Hkv, int layer_begin, int n_items, int n_tokens,
                                                         int max_chunk, int cap_tokens) {
    dependency_wait();
    dependency_release();
    if (!starts_ok(chunk_start, B, n_tokens, max_chunk, nullptr)) return;
    const int idx = blockIdx.x * 256 + threadIdx.x;
    if (idx >= n_items) return;
    const BlockItem it = block_item(layer_begin, B, Hkv, idx);
    const int n_new = chunk_start[it.b + 1] - chunk_start[it.b], n_old = min(max(len[it.item], 0), cap_tokens);
    if (n_new > 0 && n_old + (long long)n_new <= cap_tokens) len[it.item] = n_old + n_new;
}

// One token to a sequence at most: nobody else needs an item's old length.  (A thread has at most one row to place.)
static_assert(kManyRows * kManyTokens <= kAppendThreads && kFewRows <= kAppendThreads, "");
bool sets_len(const AppendArgs& a) { return a.in.max_chunk == 1; }

template <typename T, int KV>
cudaError_t launch_t(const AppendArgs& a, cudaStream_t stream) {
    const int rows = a.nl * (2 * a.Hkv + (a.in.q ? a.Hq : 0));
    const bool vec = !a.in.axis_pos || rotation_in_pieces<T>(a.in);
    const long long small = (long long)a.in.n_tokens * ((rows + kFewRows - 1) / kFewRows);
    if (small >= kManyBlocks && vec) {
        const int blocks = (rows + kManyRows - 1) / kManyRows, per_block = ((rows + blocks - 1) / blocks + 1) & ~1;  // even
        const unsigned grid = (unsigned)((a.in.n_tokens + kManyTokens - 1) / kManyTokens) * (unsigned)((rows + per_block - 1) / per_block);
        return launch_dependent(append_kernel<T, KV, true, kManyTokens>, dim3(grid), kAppendThreads, 0, stream, a, rows, per_block, sets_len(a));
    }
    const unsigned grid = (unsigned)small;
    return vec ? launch_dependent(append_kernel<T, KV, true, 1>, dim3(grid), kAppendThreads, 0, stream, a, rows, kFewRows, sets_len(a))
               : launch_dependent(append_kernel<T, KV, false, 1>, dim3(grid), kAppendThreads, 0, stream, a, rows, kFewRows, sets_len(a));
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
    if (e == cudaSuccess && !sets_len(a))
        e = launch_append_len(a.in.chunk_start, a.len, a.B, a.Hkv, a.layer_begin, a.nl * a.B * a.Hkv, a.in.n_tokens, a.in.max_chunk, a.cap_tokens, stream);
    return e;
}

}  // namespace lethe
