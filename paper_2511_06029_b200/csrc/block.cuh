// Arguments and device helpers of the kernels around lethe_append and lethe_block_cache.
#pragma once
#include "chunk.cuh"
#include "rotate.cuh"

namespace lethe {

// New rows of a call: packed tokens of all sequences, and how they are rotated.
struct NewRows {
    const int32_t* chunk_start;
    const void* q;       // NULL: no queries to rotate
    void* q_out;
    const void* k;
    const void* v;
    const int32_t* axis_pos;  // NULL: keys come rotated
    int n_tokens, max_chunk;
    int rot_dim, halves;
    unsigned long long turn[64];  // turns per position, a fraction of 2^64
    unsigned char axis[64];
};

// lethe_append: the cache as it is addressed by rows.
struct AppendArgs {
    NewRows in;
    void* k;
    void* v;
    float* rel;
    int32_t* pos;
    int32_t* len;
    const int32_t* page_table;
    const int32_t* token_pos;
    int32_t* status;
    long long n_pages;
    int dtype, D, B, Hq, Hkv, capacity, cap_tokens, page_tokens, paged;
    int layer_begin, nl;
    float k_scale[kMaxLayers];
    float v_scale[kMaxLayers];
};

// A block cache and the layers of a call.
struct BlockView {
    int8_t* k;
    int8_t* v;
    float* k_scale;
    float* v_scale;
    int8_t* k_range;
    __nv_bfloat16* k_open;
    __nv_bfloat16* v_open;
    int32_t* len;
    const int32_t* page_table;  // NULL: contiguous
    int32_t* status;
    long long n_pages;          // blocks that exist: pages, or items * capacity
    int B, Hq, Hkv, G, D, T, t_shift, capacity, cap_tokens;
    int layer_begin, nl, n_items, sm_count;
    float scale_log2[kMaxLayers];  // lethe_block_attend: softmax scale per absolute layer, in log2 units
};

constexpr float kBlockTiny = 7.8886090522101181e-31f;  // 2^-100: a block with nothing as large is stored as zeros

cudaError_t launch_append(const AppendArgs& a, cudaStream_t stream);
cudaError_t launch_block_append(const BlockView& c, const NewRows& in, cudaStream_t stream);
cudaError_t launch_block_read(const BlockView& c, const int32_t* slot_begin, int n_slots, void* k_out, void* v_out, cudaStream_t stream);
cudaError_t launch_block_select(const BlockView& c, const void* q, int n_select, int sink, int recent, float* scores, int* counters,
                                int splits, int32_t* selected, cudaStream_t stream);

// An item of a call's layers: index within the call -> sequence, absolute item.
struct BlockItem {
    int li, b, h, item;
};
__device__ __forceinline__ BlockItem block_item(int layer_begin, int B, int Hkv, int idx) {
    BlockItem it;
    it.h = idx % Hkv;
    const int lb = idx / Hkv;
    it.b = lb % B;
    it.li = lb / B;
    it.item = ((layer_begin + it.li) * B + it.b) * Hkv + it.h;
    return it;
}

// The page of block `blk` of an absolute item; -1 for a page id outside the pool.
__device__ __forceinline__ long long block_page(const BlockView& c, int item, int blk) {
    if (!c.page_table) return (long long)item * c.capacity + blk;
    const int page = c.page_table[(size_t)item * c.capacity + blk];
    return page < 0 || page >= c.n_pages ? -1 : page;
}
__device__ __forceinline__ int block_len(const BlockView& c, int item) { return min(max(c.len[item], 0), c.cap_tokens); }

// Whether chunk_start is well-formed (the same answer in every thread of the block; a barrier).  `kept`: a table of kStartsKept entries in
// shared memory that takes it, where there are fewer sequences than that.
constexpr int kStartsKept = 512;
__device__ __forceinline__ bool starts_ok(const int32_t* start, int B, int n_tokens, int max_chunk, int* kept) {
    bool ok = true;
    for (int b = threadIdx.x; b < B; b += blockDim.x) {
        const int s0 = start[b], s1 = start[b + 1];
        ok = ok && s0 >= 0 && s1 >= s0 && s1 <= n_tokens && s1 - s0 <= max_chunk;
        if (kept && B < kStartsKept) {
            kept[b] = s0;
            if (b == B - 1) kept[B] = s1;
        }
    }
    return __syncthreads_and(ok);
}
// The sequence of a token: the last b with start[b] <= tok (empty ones before it are passed over).
__device__ __forceinline__ int sequence_of(const int32_t* start, int B, int tok) {
    int b = 0, hi = B;
    while (hi - b > 1) {
        const int mid = (b + hi) >> 1;
        if (start[mid] <= tok) b = mid;
        else hi = mid;
    }
    return b;
}

// cos and sin of one pair's angle, position x frequency taken in turns as a 64-bit fraction (whose overflow is the reduction).  The nearest
// quarter turn is taken off exactly; on the eighth of a turn either side that is left, z = -1 .. 1, sin(pi z / 4) / z and
// (cos(pi z / 4) - 1) / z^2 are cubics in z^2 fitted for the smallest largest error (2.4e-9 and 1.9e-10): about 25 instructions, largest error
// with all roundings 1.02e-7 (2^-23 is 1.19e-7), 2e-8 on average; an angle rounded to fp32 before its reduction has three times that.
__device__ __forceinline__ void turn_by(unsigned long long per_pos, int pos, float& c, float& s) {
    const unsigned long long turn = (unsigned long long)(long long)pos * per_pos;
    const unsigned top = (unsigned)((turn + 0x80000000ull) >> 32) + 0x20000000u;  // the nearest 2^-32 turn, an eighth of a turn on
    const float z = (float)((int)(top & 0x3fffffffu) - 0x20000000) * 1.862645149230957e-9f;  // 2^-29
    const float u = z * z;
    const float si = z * fmaf(fmaf(fmaf(-3.595450834836811e-05f, u, 0.002490007085725665f), u, -0.08074543625116348f), u, 0.7853981852531433f);
    const float co = fmaf(fmaf(fmaf(fmaf(3.5419668620306766e-06f, u, -0.00032596138771623373f), u, 0.01585433818399906f), u, -0.3084251284599304f), u, 1.f);
    const unsigned quarter = top >> 30;
    c = quarter & 1 ? si : co;
    s = quarter & 1 ? co : si;
    if ((quarter + 1) & 2) c = -c;
    if (quarter & 2) s = -s;
}

// A pair's frequency and axis, which are among the kernel's parameters.  Lanes that read different parameters through the constant cache are
// served one after the other (2 us at the head of every block); by their address they are read like other memory.
__device__ __forceinline__ unsigned long long turn_of(const NewRows& in, int pair) {
    unsigned long long v;
    asm("ld.u64 %0, [%1];" : "=l"(v) : "l"(in.turn + pair));
    return v;
}
__device__ __forceinline__ int axis_of(const NewRows& in, int pair) {
    unsigned v;
    asm("ld.u8 %0, [%1];" : "=r"(v) : "l"(in.axis + pair));
    return (int)v;
}

// 16 bytes of a row as floats, and back.
template <typename T>
struct Piece;
template <>
struct Piece<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void unpack(const uint4& w, float* f) {
        f[0] = __uint_as_float(w.x); f[1] = __uint_as_float(w.y); f[2] = __uint_as_float(w.z); f[3] = __uint_as_float(w.w);
    }
    static __device__ __forceinline__ uint4 pack(const float* f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};
template <>
struct Piece<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ uint32_t one(float a, float b) {
        __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<uint32_t*>(&v);
    }
    static __device__ __forceinline__ void two(uint32_t w, float* f) {
        f[0] = __uint_as_float(w << 16);
        f[1] = __uint_as_float(w & 0xffff0000u);
    }
    static __device__ __forceinline__ void unpack(const uint4& w, float* f) { two(w.x, f); two(w.y, f + 2); two(w.z, f + 4); two(w.w, f + 6); }
    static __device__ __forceinline__ uint4 pack(const float* f) {
        return make_uint4(one(f[0], f[1]), one(f[2], f[3]), one(f[4], f[5]), one(f[6], f[7]));
    }
};

// A row of D elements is taken as D / (2 N) tasks of two 16-byte pieces, which hold both halves of their pairs: with pairs half a
// rotation apart, pieces (c, c + half / N); with neighbouring pairs, (2c, 2c + 1); behind the rotated part, (2c, 2c + 1).
// `turned` says whether the task's pieces are rotated.  `vec`: the style's pieces are whole (rotation_in_pieces).
template <typename T>
__device__ __forceinline__ void piece_pair(const NewRows& in, int task, bool rotated_row, int& at0, int& at1, bool& turned) {
    constexpr int N = Piece<T>::N;
    const int hp = in.rot_dim / (2 * N);  // pieces of half the rotated part
    if (in.halves && rotated_row && task < hp) {
        at0 = task * N;
        at1 = at0 + hp * N;
        turned = true;
    } else {
        at0 = 2 * task * N;
        at1 = at0 + N;
        turned = rotated_row && at0 < in.rot_dim;
    }
}
// Whether the pairs of a row come in whole tasks of piece_pair.
template <typename T>
inline bool rotation_in_pieces(const NewRows& in) {
    return in.rot_dim % (2 * Piece<T>::N) == 0;
}

// The first of the N pairs of a rotated task.
__device__ __forceinline__ int first_pair(const NewRows& in, int at0) { return in.halves ? at0 : at0 / 2; }

// Rotates the two pieces of a task by the cosines and sines of its N pairs.
template <typename T>
__device__ __forceinline__ void turn_pieces(const NewRows& in, uint4& x, uint4& y, const float (&c)[Piece<T>::N], const float (&s)[Piece<T>::N]) {
    using P = Piece<T>;
    constexpr int N = P::N;
    float f[N], g[N];
    P::unpack(x, f);
    P::unpack(y, g);
    if (in.halves) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float v = f[i], w = g[i];
            f[i] = v * c[i] - w * s[i];
            g[i] = v * s[i] + w * c[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            float v = f[i], w = f[i + 1];
            f[i] = v * c[i / 2] - w * s[i / 2];
            f[i + 1] = v * s[i / 2] + w * c[i / 2];
            v = g[i], w = g[i + 1];
            g[i] = v * c[N / 2 + i / 2] - w * s[N / 2 + i / 2];
            g[i + 1] = v * s[N / 2 + i / 2] + w * c[N / 2 + i / 2];
        }
    }
    x = P::pack(f);
    y = P::pack(g);
}
// N cosines or sines from a table in shared memory (16-byte aligned, as the task's first pair is).
template <int N>
__device__ __forceinline__ void look_up(const float* table, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const float4 x = *reinterpret_cast<const float4*>(table + i);
        v[i] = x.x, v[i + 1] = x.y, v[i + 2] = x.z, v[i + 3] = x.w;
    }
}

// One element of a rotated row, from memory (rotations whose pairs do not come in whole pieces).
template <typename T, typename Look>
__device__ __forceinline__ float turned_element(const NewRows& in, const T* src, int d, Look look) {
    if (d >= in.rot_dim) return to_float<T>(src[d]);
    const int half = in.rot_dim / 2;
    const int p = in.halves ? (d < half ? d : d - half) : d / 2;
    const int i0 = in.halves ? p : 2 * p, i1 = in.halves ? p + half : 2 * p + 1;
    const float v = to_float<T>(src[i0]), w = to_float<T>(src[i1]);
    float c, s;
    look(p, c, s);
    // one product rounded, the other fused with the sum: as the compiler forms it where both elements are made at once
    return d == i0 ? fmaf(v, c, -__fmul_rn(w, s)) : fmaf(v, s, __fmul_rn(w, c));
}
// The two pieces of a task of a row whose pairs do not come in whole pieces.
template <typename T, typename Look>
__device__ __forceinline__ void load_by_element(const NewRows& in, const T* src, int task, Look look, int& at0, int& at1, uint4& x, uint4& y) {
    constexpr int N = Piece<T>::N;
    at0 = 2 * task * N;
    at1 = at0 + N;
    float f[N], g[N];
#pragma unroll 1
    for (int i = 0; i < N; ++i) {
        f[i] = turned_element<T>(in, src, at0 + i, look);
        g[i] = turned_element<T>(in, src, at1 + i, look);
    }
    x = Piece<T>::pack(f);
    y = Piece<T>::pack(g);
}

}  // namespace lethe
