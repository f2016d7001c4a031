// lethe_block_append and lethe_block_read: filling a cache in 8 bits with a scale for each block of tokens, and reading it back.
#include "block.cuh"

namespace lethe {
cudaError_t launch_append_len(const int32_t* chunk_start, int32_t* len, int B, int Hkv, int layer_begin, int n_items, int n_tokens, int max_chunk,
                              int cap_tokens, cudaStream_t stream);
namespace {

using bf16 = __nv_bfloat16;
constexpr int kQueryRows = 16;

__device__ __forceinline__ float finite_top(const uint4& w, float top) {
    float f[8];
    Piece<bf16>::unpack(w, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float m = fabsf(f[i]);
        if (m < INFINITY) top = fmaxf(top, m);  // false for NaN too
    }
    return top;
}
__device__ __forceinline__ uint32_t code(float x, float inv) {
    return (uint32_t)min(max(__float2int_rn(x * inv), -127), 127) & 0xffu;  // NaN converts to 0
}
__device__ __forceinline__ uint2 codes8(const uint4& w, float inv) {
    float f[8];
    Piece<bf16>::unpack(w, f);
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = code(f[i], inv);
    return make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
}

// The first n_items * units blocks: unit u of an item quantises the u-th of the blocks that the call fills; unit 0 also moves what is
// left over to the open block (it has read the rows that were there by then).  The rest rotate queries, kQueryRows rows of a token each.
// Bound by memory: rows are read once and kept packed in registers between the search for the largest magnitude and the rounding.
template <int D, int TPT, bool VEC>  // TPT: tasks of 16 elements per thread, of K and of V
__global__ void __launch_bounds__(256) block_append_kernel(const __grid_constant__ BlockView c, const __grid_constant__ NewRows in, int units) {
    extern __shared__ __align__(16) unsigned char tile[];  // [T][D] key codes
    __shared__ unsigned long long turn[64];
    __shared__ unsigned char axis[64];
    __shared__ float cs[64], sn[64];
    __shared__ float tops[2][8];
    __shared__ uint32_t least[8][32], greatest[8][32];
    dependency_wait();
    dependency_release();
    const int tid = threadIdx.x, nt = blockDim.x;
    constexpr int kPerRow = D / 16;
    const int half = in.rot_dim / 2;
    const bool ok = starts_ok(in.chunk_start, c.B, in.n_tokens, in.max_chunk);
    if (!ok) {
        if (blockIdx.x == 0 && tid == 0) record_error(c.status, LETHE_ERR_INVALID_ARG, 0);
        return;
    }
    const unsigned kv_blocks = (unsigned)c.n_items * units;
    if (blockIdx.x >= kv_blocks) {
        const int rows_total = c.nl * c.Hq, per_tok = (rows_total + kQueryRows - 1) / kQueryRows;
        const int qb = blockIdx.x - kv_blocks, tok = qb / per_tok, r0 = (qb - tok * per_tok) * kQueryRows;
        if (tok < in.chunk_start[0] || tok >= in.chunk_start[c.B]) return;
        for (int p = tid; p < half; p += nt) pair_turn(in, p, in.axis_pos[(size_t)in.axis[p] * in.n_tokens + tok], cs[p], sn[p]);
        __syncthreads();
        const int tasks = min(rows_total - r0, kQueryRows) * kPerRow;
        for (int t0 = 0; t0 < tasks; t0 += nt) {  // uniform for the block
            const int t = t0 + tid, r = r0 + t / kPerRow, li = r / c.Hq;
            const size_t off = (((size_t)li * in.n_tokens + tok) * c.Hq + r - li * c.Hq) * D;
            int at0, at1;
            uint4 x, y;
            if (t < tasks)
                load_task<bf16, VEC>(in, (const bf16*)in.q + off, t % kPerRow, true, [&](int p, float& co, float& si) { co = cs[p], si = sn[p]; }, at0, at1, x, y);
            if (!VEC) __syncwarp();  // q_out may be q: a row's tasks lie in one warp, all have read before one writes
            if (t < tasks) {
                *reinterpret_cast<uint4*>((bf16*)in.q_out + off + at0) = x;
                *reinterpret_cast<uint4*>((bf16*)in.q_out + off + at1) = y;
            }
        }
        return;
    }
    const int idx = blockIdx.x / units, u = blockIdx.x - idx * units;
    const BlockItem it = block_item(c.layer_begin, c.B, c.Hkv, idx);
    const int s0 = in.chunk_start[it.b], n_new = in.chunk_start[it.b + 1] - s0;
    if (n_new == 0) return;
    const int n0 = block_len(c, it.item);
    if (n0 + (long long)n_new > c.cap_tokens) {
        if (u == 0 && tid == 0) record_error(c.status, LETHE_ERR_CAPACITY, it.item);
        return;
    }
    const int n1 = n0 + n_new, b0 = n0 >> c.t_shift, b1 = n1 >> c.t_shift;
    if (u > 0 && b0 + u >= b1) return;
    if (in.axis_pos) {
        for (int p = tid; p < half; p += nt) {
            turn[p] = in.turn[p];
            axis[p] = in.axis[p];
        }
        __syncthreads();
    }
    const size_t open = (size_t)it.item * c.T;
    const bf16* new_k = (const bf16*)in.k + ((size_t)it.li * in.n_tokens * c.Hkv + it.h) * D;
    const bf16* new_v = (const bf16*)in.v + ((size_t)it.li * in.n_tokens * c.Hkv + it.h) * D;
    const size_t tok_pitch = (size_t)c.Hkv * D;
    auto load_new = [&](int tok, int task, int& at0, int& at1, uint4& kx, uint4& ky, uint4& vx, uint4& vy) {
        auto look = [&](int p, float& co, float& si) {
            const int pos = in.axis_pos[(size_t)axis[p] * in.n_tokens + tok];
            const unsigned long long full = (unsigned long long)(long long)pos * turn[p];
            sincospif((float)(int)((full + 0x80000000ull) >> 32) * 4.656612873077393e-10f, &si, &co);  // as pair_turn
        };
        load_task<bf16, VEC>(in, new_k + tok * tok_pitch, task, in.axis_pos != nullptr, look, at0, at1, kx, ky);
        const bf16* v = new_v + tok * tok_pitch;
        vx = *reinterpret_cast<const uint4*>(v + at0);
        vy = *reinterpret_cast<const uint4*>(v + at1);
    };
    if (b0 + u < b1) {
        const int blk = b0 + u;
        uint4 kx[TPT], ky[TPT], vx[TPT], vy[TPT];
        float top_k = 0.f, top_v = 0.f;
#pragma unroll
        for (int i = 0; i < TPT; ++i) {
            const int t = tid + i * nt, r = t / kPerRow, slot = (blk << c.t_shift) + r;
            int at0, at1;
            if (slot < n0) {
                bool turned;
                piece_pair<bf16>(in, t % kPerRow, VEC && in.axis_pos, at0, at1, turned);
                const size_t off = (open + r) * D;
                kx[i] = *reinterpret_cast<const uint4*>(c.k_open + off + at0);
                ky[i] = *reinterpret_cast<const uint4*>(c.k_open + off + at1);
                vx[i] = *reinterpret_cast<const uint4*>(c.v_open + off + at0);
                vy[i] = *reinterpret_cast<const uint4*>(c.v_open + off + at1);
            } else {
                load_new(s0 + slot - n0, t % kPerRow, at0, at1, kx[i], ky[i], vx[i], vy[i]);
            }
            top_k = finite_top(ky[i], finite_top(kx[i], top_k));
            top_v = finite_top(vy[i], finite_top(vx[i], top_v));
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            top_k = fmaxf(top_k, __shfl_xor_sync(0xffffffffu, top_k, o));
            top_v = fmaxf(top_v, __shfl_xor_sync(0xffffffffu, top_v, o));
        }
        if ((tid & 31) == 0) {
            tops[0][tid >> 5] = top_k;
            tops[1][tid >> 5] = top_v;
        }
        __syncthreads();
        for (int w = 0; w < nt / 32; ++w) {
            top_k = fmaxf(top_k, tops[0][w]);
            top_v = fmaxf(top_v, tops[1][w]);
        }
        const float inv_k = top_k >= kBlockTiny ? __fdiv_rn(127.f, top_k) : 0.f, inv_v = top_v >= kBlockTiny ? __fdiv_rn(127.f, top_v) : 0.f;
        const long long page = block_page(c, it.item, blk);
        if (page < 0) {
            if (tid == 0) record_error(c.status, LETHE_ERR_PAGE, it.item);
        } else {
            int8_t* kd = c.k + (size_t)page * c.T * D;
            int8_t* vd = c.v + (size_t)page * c.T * D;
#pragma unroll
            for (int i = 0; i < TPT; ++i) {
                const int t = tid + i * nt, r = t / kPerRow;
                int at0, at1;
                bool turned;
                piece_pair<bf16>(in, t % kPerRow, VEC && in.axis_pos, at0, at1, turned);
                const uint2 a = codes8(kx[i], inv_k), b = codes8(ky[i], inv_k);
                *reinterpret_cast<uint2*>(kd + r * D + at0) = a;
                *reinterpret_cast<uint2*>(kd + r * D + at1) = b;
                *reinterpret_cast<uint2*>(tile + r * D + at0) = a;
                *reinterpret_cast<uint2*>(tile + r * D + at1) = b;
                *reinterpret_cast<uint2*>(vd + r * D + at0) = codes8(vx[i], inv_v);
                *reinterpret_cast<uint2*>(vd + r * D + at1) = codes8(vy[i], inv_v);
            }
            if (tid == 0) {
                c.k_scale[page] = top_k >= kBlockTiny ? __fdiv_rn(top_k, 127.f) : 0.f;
                c.v_scale[page] = top_v >= kBlockTiny ? __fdiv_rn(top_v, 127.f) : 0.f;
            }
            if (c.k_range) {
                // four elements to a thread, the rows in turn among the groups of threads
                constexpr int W = D / 4;
                const int groups = nt / W, w = tid % W, gr = tid / W;
                __syncthreads();
                uint32_t lo = 0x7f7f7f7fu, hi = 0x81818181u;
                for (int r = gr; r < c.T; r += groups) {
                    const uint32_t x = *reinterpret_cast<const uint32_t*>(tile + r * D + 4 * w);
                    lo = __vmins4(lo, x);
                    hi = __vmaxs4(hi, x);
                }
                // at D = 64 there may be more groups than rows of the table: they fold by shuffles (W = 16 lanes apart)
                if (W == 16) {
                    lo = __vmins4(lo, __shfl_xor_sync(0xffffffffu, lo, 16));
                    hi = __vmaxs4(hi, __shfl_xor_sync(0xffffffffu, hi, 16));
                }
                least[tid >> 5][tid & 31] = lo;
                greatest[tid >> 5][tid & 31] = hi;
                __syncthreads();
                if (tid < W) {
                    for (int g = 1; g < nt / 32; ++g) {
                        lo = __vmins4(lo, least[g][w]);
                        hi = __vmaxs4(hi, greatest[g][w]);
                    }
                    uint32_t* range = reinterpret_cast<uint32_t*>(c.k_range + (size_t)page * 2 * D);
                    range[w] = lo;
                    range[W + w] = hi;
                }
            }
        }
    }
    if (u == 0) {
        // what is left over; all reads of open rows lie before the barrier
        __syncthreads();
        const int s_first = b1 > b0 ? b1 << c.t_shift : n0;
        for (int t = tid; t < (n1 - s_first) * kPerRow; t += nt) {
            const int slot = s_first + t / kPerRow;
            int at0, at1;
            uint4 kx, ky, vx, vy;
            load_new(s0 + slot - n0, t % kPerRow, at0, at1, kx, ky, vx, vy);
            const size_t off = (open + (slot & (c.T - 1))) * D;
            *reinterpret_cast<uint4*>(c.k_open + off + at0) = kx;
            *reinterpret_cast<uint4*>(c.k_open + off + at1) = ky;
            *reinterpret_cast<uint4*>(c.v_open + off + at0) = vx;
            *reinterpret_cast<uint4*>(c.v_open + off + at1) = vy;
        }
        if (units == 1 && tid == 0) c.len[it.item] = n1;  // no other block needs the item's old length
    }
}

// A thread takes 8 elements of a slot, of K and of V.
template <int D>
__global__ void __launch_bounds__(256) block_read_kernel(const __grid_constant__ BlockView c, const int32_t* slot_begin, int n_slots, bf16* k_out, bf16* v_out, unsigned total) {
    dependency_wait();
    dependency_release();
    const unsigned t = blockIdx.x * 256u + threadIdx.x;
    if (t >= total) return;
    constexpr int kPieces = D / 8;
    const unsigned row = t / kPieces;
    const int d = (t % kPieces) * 8;
    const int idx = row / n_slots, i = row - (unsigned)idx * n_slots;
    const BlockItem it = block_item(c.layer_begin, c.B, c.Hkv, idx);
    const int n = block_len(c, it.item);
    const long long slot = (slot_begin ? (long long)slot_begin[it.b] : 0) + i;
    uint4 x = make_uint4(0, 0, 0, 0), y = x;
    if (slot >= 0 && slot < n) {
        const int r = (int)slot & (c.T - 1), blk = (int)slot >> c.t_shift;
        if (blk == n >> c.t_shift) {
            const size_t off = ((size_t)it.item * c.T + r) * D + d;
            x = *reinterpret_cast<const uint4*>(c.k_open + off);
            y = *reinterpret_cast<const uint4*>(c.v_open + off);
        } else {
            const long long page = block_page(c, it.item, blk);
            if (page < 0) {
                if (d == 0 && r == 0) record_error(c.status, LETHE_ERR_PAGE, it.item);
            } else {
                const size_t off = ((size_t)page * c.T + r) * D + d;
                const uint2 a = *reinterpret_cast<const uint2*>(c.k + off), b = *reinterpret_cast<const uint2*>(c.v + off);
                const float ks = c.k_scale[page], vs = c.v_scale[page];
                float f[8], g[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t wa = e < 4 ? a.x : a.y, wb = e < 4 ? b.x : b.y;
                    f[e] = (float)(int8_t)(wa >> (8 * (e & 3))) * ks;
                    g[e] = (float)(int8_t)(wb >> (8 * (e & 3))) * vs;
                }
                x = Piece<bf16>::pack(f);
                y = Piece<bf16>::pack(g);
            }
        }
    }
    reinterpret_cast<uint4*>(k_out)[t] = x;
    reinterpret_cast<uint4*>(v_out)[t] = y;
}

template <int D, int TPT>
cudaError_t launch_d(const BlockView& c, const NewRows& in, int units, unsigned grid, int threads, cudaStream_t stream) {
    const bool vec = !in.axis_pos || rotation_in_pieces<bf16>(in);
    return vec ? launch_dependent(block_append_kernel<D, TPT, true>, dim3(grid), threads, (size_t)c.T * D, stream, c, in, units)
               : launch_dependent(block_append_kernel<D, TPT, false>, dim3(grid), threads, (size_t)c.T * D, stream, c, in, units);
}

}  // namespace

cudaError_t launch_block_append(const BlockView& c, const NewRows& in, cudaStream_t stream) {
    // blocks that a sequence's tokens can fill: all but a last one that the call leaves open
    const int units = max(1, (int)(((long long)in.max_chunk + c.T - 1) / c.T));
    const unsigned q_blocks = in.q ? (unsigned)in.n_tokens * (unsigned)((c.nl * c.Hq + kQueryRows - 1) / kQueryRows) : 0;
    const unsigned grid = (unsigned)c.n_items * units + q_blocks;
    const int tasks = c.T * c.D / 16, threads = min(256, tasks), per = tasks / threads;
    cudaError_t e;
    if (c.D == 128) e = per == 1 ? launch_d<128, 1>(c, in, units, grid, threads, stream) : per == 2 ? launch_d<128, 2>(c, in, units, grid, threads, stream)
                                                                                                   : launch_d<128, 4>(c, in, units, grid, threads, stream);
    else e = per == 1 ? launch_d<64, 1>(c, in, units, grid, threads, stream) : launch_d<64, 2>(c, in, units, grid, threads, stream);
    if (e == cudaSuccess && units > 1)
        e = launch_append_len(in.chunk_start, c.len, c.B, c.Hkv, c.layer_begin, c.n_items, in.n_tokens, in.max_chunk, c.cap_tokens, stream);
    return e;
}

cudaError_t launch_block_read(const BlockView& c, const int32_t* slot_begin, int n_slots, void* k_out, void* v_out, cudaStream_t stream) {
    const unsigned total = (unsigned)c.n_items * n_slots * (c.D / 8);
    const unsigned grid = (total + 255) / 256;
    return c.D == 128 ? launch_dependent(block_read_kernel<128>, dim3(grid), 256, 0, stream, c, slot_begin, n_slots, (bf16*)k_out, (bf16*)v_out, total)
                      : launch_dependent(block_read_kernel<64>, dim3(grid), 256, 0, stream, c, slot_begin, n_slots, (bf16*)k_out, (bf16*)v_out, total);
}

}  // namespace lethe
