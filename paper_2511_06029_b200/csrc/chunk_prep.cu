// lethe_chunk_attend: append of the new rows, the plan that cuts the attention evenly, and the merge of its parts.
#include "chunk.cuh"

namespace lethe {
namespace {

constexpr int kPrepThreads = 256;
constexpr int kPrepWarps = kPrepThreads / 32;
constexpr int kRangeThreads = 1024;  // one block per item: its tiles, units and pairs are gone through by warps
constexpr int kRangeWarps = kRangeThreads / 32;
constexpr int kSeqShared = 1024;  // chunk_start entries kept in shared memory (longer batches read it from global memory)

// Whether chunk_start never decreases, stays inside [0, n_tokens] and has no sequence above max_chunk; uniform for the block.
__device__ bool chunk_start_ok(const ChunkArgs& a) {
    bool ok = true;
    for (int b = threadIdx.x; b < a.B; b += kPrepThreads) {
        const int s0 = a.chunk_start[b], s1 = a.chunk_start[b + 1];
        ok = ok && s0 >= 0 && s0 <= s1 && s1 <= a.n_tokens && s1 - s0 <= a.max_chunk;
    }
    return __syncthreads_and(ok);
}

__device__ __forceinline__ int unit_cost(const ChunkArgs& a, int u) {
    const int idx = u / a.QT, qt = u - idx * a.QT;
    const int n_old = a.n_old[idx];
    if (n_old < 0) return 0;
    const int b = (idx / a.Hkv) % a.B;
    const int T = a.chunk_start[b + 1] - a.chunk_start[b], tok0 = qt * a.TU;
    if (tok0 >= T) return 0;
    if (a.u_hi) return unit_pad(a, T - tok0) + max(1, (a.u_hi[u] + a.tile - 1) / a.tile - a.u_lo[u]);
    const int hi = a.append ? n_old + min(T, tok0 + a.TU) : n_old;
    return unit_pad(a, T - tok0) + max(1, (hi + a.tile - 1) / a.tile);  // rows that see nothing still have to be written
}

// Exclusive prefix sum over the block's threads; `total` is the sum.
__device__ int block_scan(int mine, int* total) {
    __shared__ int sums[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    int x = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
    }
    __syncthreads();  // the last call's readers are done
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    const int of_warp = lane < warps ? sums[lane] : 0;
    *total = __reduce_add_sync(0xffffffffu, of_warp);
    return __reduce_add_sync(0xffffffffu, lane < warp ? of_warp : 0) + x - mine;
}

// Lays `n` costs end to end: starts, the whole, equal stretches for `n_cta` CTAs, and for each CTA the entry that its stretch begins in.
// The whole launch waits for this one block: every cost is computed once, the loads of neighbouring threads side by side, and the
// loops stay rolled, because code that runs once is paid for by fetching it.
template <typename Cost>
__device__ void lay_line(int n, int n_cta, int min_per, int* start, int* cta_entry, int* total_out, int* per_out, Cost cost) {
    constexpr int kShared = 2048;
    __shared__ int few[kShared];
    int* costs = n <= kShared ? few : start;  // long lines keep them where the starts go
    const int tid = threadIdx.x;
    __syncthreads();  // the last line's readers are done
#pragma unroll 1
    for (int i = tid; i < n; i += (int)blockDim.x) costs[i] = cost(i);
    __syncthreads();
    const int seg = (n + (int)blockDim.x - 1) / (int)blockDim.x;
    const int i0 = min(n, tid * seg), i1 = min(n, i0 + seg);
    int mine = 0, total;
#pragma unroll 1
    for (int i = i0; i < i1; ++i) mine += costs[i];
    int at = block_scan(mine, &total);
    const int per = max(min_per, (total + n_cta - 1) / n_cta);
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
        const int next = at + costs[i];
        start[i] = at;
#pragma unroll 1
        for (int k = (at + per - 1) / per; k * per < next; ++k) cta_entry[k] = i;
        at = next;
    }
    if (tid == 0) {
        start[n] = total;
        *total_out = total;
        *per_out = per;
    }
}

// The plan: the units' line for the attention, the items' line for the relevance.  One block.
__device__ void make_plan(const ChunkArgs& a) {
    lay_line(a.n_units, a.n_cta, a.min_per, a.u_start, a.cta_unit, &a.plan->total, &a.plan->per, [&](int u) { return unit_cost(a, u); });
    if (!a.rel_start) return;
    lay_line(a.n_items, a.n_rel_cta, 1, a.rel_start, a.rel_item, &a.plan->rel_total, &a.plan->rel_per, [&](int idx) -> int {
        const ChunkItem it = chunk_item(a, idx);
        if (it.n_old < 0 || it.T == 0) return 0;
        if (a.rel_cost) return a.rel_cost[idx];
        const int pairs = rel_pairs(it), tiles = (it.T + a.TT - 1) / a.TT;
        int pr = a.append ? min(pairs, it.n_old / (2 * kChunkTile) + 1) : pairs;  // these meet every query tile
        int sum = pr * tiles;
#pragma unroll 1
        for (; pr < pairs; ++pr) sum += rel_steps(rel_hull(a, it, idx, pr));
        return sum;
    });
}

// Two fp32 values -> two bytes of an 8-bit float, saturating (the low byte is the first).
__device__ __forceinline__ uint32_t to_bytes(float lo, float hi, bool e5m2) {
    uint32_t y;
    if (e5m2) asm("{ .reg .b16 r; cvt.rn.satfinite.e5m2x2.f32 r, %2, %1; cvt.u32.u16 %0, r; }" : "=r"(y) : "f"(lo), "f"(hi));
    else asm("{ .reg .b16 r; cvt.rn.satfinite.e4m3x2.f32 r, %2, %1; cvt.u32.u16 %0, r; }" : "=r"(y) : "f"(lo), "f"(hi));
    return y;
}
__device__ __forceinline__ uint32_t quantise4(uint32_t ab, uint32_t cd, float scale, bool e5m2) {
    const float a = __uint_as_float(ab << 16) / scale, b = __uint_as_float(ab & 0xffff0000u) / scale;
    const float c = __uint_as_float(cd << 16) / scale, d = __uint_as_float(cd & 0xffff0000u) / scale;
    return to_bytes(a, b, e5m2) | (to_bytes(c, d, e5m2) << 16);
}

// Blocks 1.. : the (layer, token, KV head) rows.  Memory-bound: each new row is read and written once with 16-byte accesses (8192
// tokens with 8 KV heads of 128 in bf16, 67 MB both ways: 16 us; 24 with rows counted in 64 bits).  Block 0 writes n_old, clears the
// call's counters and, when no mask goes by position, the plan; small calls wait for it (4 us with the launch).
__global__ void __launch_bounds__(kPrepThreads) chunk_append_kernel(const __grid_constant__ ChunkArgs a) {
    __shared__ int cs[kSeqShared + 1];
    dependency_wait();
    dependency_release();
    const int tid = threadIdx.x, lane = tid & 31;
    const bool ok = chunk_start_ok(a);
    if (blockIdx.x == 0) {
        if (tid == 0) {
            a.plan->refused = !ok;
            a.plan->done = 0;
            if (!ok) record_error(a.status, LETHE_ERR_INVALID_ARG, 0);
        }
        for (int idx = tid; idx < a.n_items; idx += kPrepThreads) {
            int n_old = -1;
            if (ok) {
                const int b = (idx / a.Hkv) % a.B, l = a.layer_begin + idx / (a.Hkv * a.B);
                const int item = (l * a.B + b) * a.Hkv + idx % a.Hkv;
                const int T = a.chunk_start[b + 1] - a.chunk_start[b];
                n_old = min(max(a.len[item], 0), a.cap_tokens);
                if (a.append && n_old + (long long)T > a.cap_tokens) {
                    n_old = -1;
                    record_error(a.status, LETHE_ERR_CAPACITY, item);
                }
            }
            a.n_old[idx] = n_old;
        }
        __syncthreads();
        if (!a.u_hi) make_plan(a);
        return;
    }
    if (!ok) return;
    const bool in_shared = a.B <= kSeqShared;
    if (in_shared)
        for (int b = tid; b <= a.B; b += kPrepThreads) cs[b] = a.chunk_start[b];
    __syncthreads();
    const int* start = in_shared ? cs : a.chunk_start;

    const bool bytes = a.dtype == LETHE_FP8_E4M3 || a.dtype == LETHE_FP8_E5M2, e5m2 = a.dtype == LETHE_FP8_E5M2;
    const int act = a.dtype == LETHE_F32 ? 4 : 2;
    const int src_row = a.D * act, dst_row = bytes ? a.D : src_row;
    const int chunks = src_row / 16;  // 16-byte pieces of a new row: 8 .. 32
    // A half-warp takes a row at a time, first its K, then its V, U of each in flight: where a row goes is a short chain of
    // dependent loads (length, page), so a warp works on 2 U rows at once.  Rows are counted in 32 bits: the divisions of a
    // 64-bit count took longer than the copy.
    constexpr int U = 2;
    const unsigned rows = (unsigned)a.nl * a.n_tokens * a.Hkv, hkvs = a.Hkv, tokens = a.n_tokens;
    const unsigned half = lane >> 4, hl = lane & 15;
    const unsigned step = (gridDim.x - 1) * kPrepWarps * 2 * U;
    const int first = start[0], last = start[a.B];
    for (unsigned r0 = ((blockIdx.x - 1) * kPrepWarps + (tid >> 5)) * 2 * U; r0 < rows; r0 += step) {
        int item[U], slot[U], lay[U];
        unsigned tok[U], lt[U];
        long long at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned r = r0 + 2 * u + half;
            item[u] = -1;
            at[u] = -1;
            if (r >= rows) continue;
            lt[u] = r / hkvs;
            const unsigned hkv = r - lt[u] * hkvs, li = lt[u] / tokens;
            tok[u] = lt[u] - li * tokens;
            if ((int)tok[u] < first || (int)tok[u] >= last) continue;
            int lo = 0, hi = a.B;  // last b with start[b] <= tok: the sequence of this token (empty ones before it are passed over)
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (start[mid] <= (int)tok[u]) lo = mid;
                else hi = mid;
            }
            const int T = start[lo + 1] - start[lo];
            lay[u] = a.layer_begin + li;
            item[u] = (lay[u] * a.B + lo) * a.Hkv + hkv;
            const int n_old = min(max(a.len[item[u]], 0), a.cap_tokens);
            slot[u] = n_old + (long long)T > a.cap_tokens ? -1 : n_old + (int)tok[u] - start[lo];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (item[u] < 0) continue;
            if (slot[u] < 0) {  // refused: nothing of the item changes, its outputs are zero
                const unsigned head = (r0 + 2 * u + half - lt[u] * hkvs) * a.G;
                char* o = (char*)a.out + ((size_t)lt[u] * a.Hq + head) * src_row;
                for (int i = hl; i < a.G * chunks; i += 16) reinterpret_cast<uint4*>(o)[i] = make_uint4(0, 0, 0, 0);
                if (a.lse && hl < a.G) a.lse[(size_t)lt[u] * a.Hq + head + hl] = -INFINITY;
                continue;
            }
            if (hl == 0) a.pos[(size_t)item[u] * a.cap_tokens + slot[u]] = a.token_pos[tok[u]];
            at[u] = chunk_row(a, item[u], slot[u]);
            if (at[u] < 0 && hl == 0) record_error(a.status, LETHE_ERR_PAGE, item[u]);
        }
        for (int c = hl; c < chunks; c += 16) {
            uint4 x[U][2];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (at[u] >= 0) {
                    const size_t src = (size_t)(r0 + 2 * u + half) * src_row;
                    x[u][0] = reinterpret_cast<const uint4*>((const char*)a.k_new + src)[c];
                    x[u][1] = reinterpret_cast<const uint4*>((const char*)a.v_new + src)[c];
                }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (at[u] >= 0) {
                    char* kd = (char*)const_cast<void*>(a.k) + (size_t)at[u] * dst_row;
                    char* vd = (char*)const_cast<void*>(a.v) + (size_t)at[u] * dst_row;
                    if (!bytes) {
                        reinterpret_cast<uint4*>(kd)[c] = x[u][0];
                        reinterpret_cast<uint4*>(vd)[c] = x[u][1];
                    } else {
                        const float ks = a.k_scale[lay[u]], vs = a.v_scale[lay[u]];
                        reinterpret_cast<uint2*>(kd)[c] = make_uint2(quantise4(x[u][0].x, x[u][0].y, ks, e5m2), quantise4(x[u][0].z, x[u][0].w, ks, e5m2));
                        reinterpret_cast<uint2*>(vd)[c] = make_uint2(quantise4(x[u][1].x, x[u][1].y, vs, e5m2), quantise4(x[u][1].z, x[u][1].w, vs, e5m2));
                    }
                }
        }
    }
}

// Masks by position.  A block takes one item: the smallest and largest position of each of its key tiles, then for each unit the
// first tile with a key that its farthest-reaching token may still see and the end of what the prefix opens.  Conservative
// whatever the order of the positions is; the attention tests every key that is left.  The last block to finish plans.  Bound by
// latency (256 items of about 2000 slots: 8 us, most of it the plan and the code's first fetch); 32 warps to an item because a long
// prompt has one item per KV head only (8 warps: packed documents of 4096 tokens 298 us instead of 274).
__global__ void __launch_bounds__(kRangeThreads) chunk_range_kernel(const __grid_constant__ ChunkArgs a) {
    __shared__ int last;
    dependency_wait();
    dependency_release();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const ChunkItem it = chunk_item(a, blockIdx.x);
    if (it.n_old >= 0 && it.T > 0) {
        const int tiles = (it.n + a.tile - 1) / a.tile;
        int2* bounds = a.bounds + (size_t)blockIdx.x * a.cap_tiles;
        const int32_t* pos = a.pos + (size_t)it.item * a.cap_tokens;
        for (int t = warp; t < tiles; t += kRangeWarps) {
            int mn = INT32_MAX, mx = INT32_MIN;
#pragma unroll
            for (int i = 0; i < kChunkTile / 32; ++i) {
                const int j = t * a.tile + i * 32 + lane;
                if (j < it.n && i * 32 < a.tile) {
                    const int p = pos[j];
                    mn = min(mn, p);
                    mx = max(mx, p);
                }
            }
            mn = __reduce_min_sync(0xffffffffu, mn);
            mx = __reduce_max_sync(0xffffffffu, mx);
            if (lane == 0) bounds[t] = make_int2(mn, mx);
        }
        __syncthreads();
        const int units = (it.T + a.TU - 1) / a.TU;
        for (int qt = warp; qt < units; qt += kRangeWarps) {
            const int tok0 = qt * a.TU, tok1 = min(it.T, tok0 + a.TU);
            int lo = INT32_MAX;
            for (int i = tok0 + lane; i < tok1; i += 32) lo = min(lo, chunk_lo(a, it.first + i, a.window > 0 ? a.token_pos[it.first + i] : 0));
            lo = __reduce_min_sync(0xffffffffu, lo);
            int hi = a.append ? it.n_old + tok1 : it.n_old;
            int t_lo = 0;
            bool found = false;
            for (int t0 = 0; t0 < tiles && !found; t0 += 32) {
                const unsigned hit = __ballot_sync(0xffffffffu, t0 + lane < tiles && bounds[t0 + lane].y >= lo);
                if (hit) {
                    t_lo = t0 + __ffs(hit) - 1;
                    found = true;
                }
            }
            if (a.prefix_len) {
                const int prefix = a.prefix_len[it.b];
                for (int t0 = (tiles - 1) & ~31; t0 >= 0; t0 -= 32) {
                    const unsigned hit = __ballot_sync(0xffffffffu, t0 + lane < tiles && bounds[t0 + lane].x < prefix);
                    if (hit) {
                        hi = max(hi, min(it.n, (t0 + 32 - __clz(hit)) * a.tile));
                        break;
                    }
                }
            }
            if (!found || t_lo * a.tile >= hi) t_lo = 0, hi = 0;
            if (lane == 0) {
                a.u_lo[blockIdx.x * a.QT + qt] = t_lo;
                a.u_hi[blockIdx.x * a.QT + qt] = hi;
            }
        }
    }
    __syncthreads();  // the item's u_lo and u_hi are there
    if (it.n_old >= 0 && it.T > 0 && a.rel_hull) {
        // query tiles that each pair of key tiles meets, from the ranges of their units
        __shared__ int cost;
        if (tid == 0) cost = 0;
        __syncthreads();
        const int pairs = rel_pairs(it), tiles = (it.T + a.TT - 1) / a.TT;
        int mine = 0;
        for (int pr = warp; pr < pairs; pr += kRangeWarps) {
            const int j0 = pr * 2 * kChunkTile;
            int first = INT32_MAX, end = 0;
            for (int qt = lane; qt < tiles; qt += 32) {
                const int u = blockIdx.x * a.QT + qt * a.TT / a.TU;
                if (a.u_hi[u] > j0 && a.u_lo[u] * kChunkTile < j0 + 2 * kChunkTile) {
                    first = min(first, qt);
                    end = max(end, qt + 1);
                }
            }
            first = __reduce_min_sync(0xffffffffu, first);
            end = __reduce_max_sync(0xffffffffu, end);
            if (end == 0) first = 0;  // nobody sees the pair
            if (lane == 0) a.rel_hull[(size_t)blockIdx.x * ((a.cap_tiles + 1) / 2) + pr] = make_int2(first, end);
            mine += rel_steps(make_int2(first, end));
        }
        if (lane == 0) atomicAdd(&cost, mine);  // whole numbers: any order
        __syncthreads();
        if (tid == 0) a.rel_cost[blockIdx.x] = cost;
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(&a.plan->done, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    make_plan(a);
}

// Merges the parts of each unit that more than one CTA worked on.  A block takes 32 rows of the unit that lies across the beginning
// of CTA c's stretch (the first such c of the unit speaks for it): thread (x, y) of 32 x 8 adds up elements y, y + 8, ... of row x
// over the parts, in the order of the keys they cover, and the rows are turned in shared memory so that reads and writes are both
// whole lines.  Bound by memory, 512 bytes per row and part: at most two parts per CTA, 38 MB (one block to a unit took 86 us behind
// eight 512-token chunks, blocks of 32 rows at the boundaries about 10).
constexpr int kCombineRows = 32;
__global__ void __launch_bounds__(kPrepThreads) chunk_combine_kernel(const __grid_constant__ ChunkArgs a, int row_blocks) {
    __shared__ float tile[kCombineRows][128 + 1];
    dependency_wait();
    dependency_release();
    const int c_mid = 1 + blockIdx.x / row_blocks, row0 = (blockIdx.x % row_blocks) * kCombineRows;
    const int per = a.plan->per;
    if ((long long)c_mid * per >= a.plan->total) return;
    const int u = a.cta_unit[c_mid];
    const int s0 = a.u_start[u], s1 = a.u_start[u + 1];
    const int c0 = s0 / per, c1 = (s1 - 1) / per;
    if (c0 != c_mid - 1) return;  // begins here (nothing to merge) or was begun before CTA c_mid - 1
    const int idx = u / a.QT, tok0 = (u - idx * a.QT) * a.TU;
    const ChunkItem it = chunk_item(a, idx);
    const int toks = min(it.T - tok0, a.TU), rows = toks * a.G;
    const int cf = (s0 + unit_pad(a, toks)) / per;  // the first CTA that has some of its tiles; all after it have
    if (cf == c1) return;                            // one CTA had all of its tiles and has written the outputs
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    // row blocks do not lie across row tiles: a tile has TT * G <= 128 rows, four blocks
    const int tile_idx = row0 / kChunkPartRows, r = row0 % kChunkPartRows + x;
    const int row = tile_idx * a.TT * a.G + r;
    const bool ok = r < a.TT * a.G && row < rows;
    constexpr int E = 16;  // elements per thread at D = 128
    float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    if (ok) {
#pragma unroll 1
        for (int c = cf; c <= c1; ++c) {  // rolled: code that runs once is paid for by fetching it
            const size_t p = (size_t)(c * 2 + (c == cf ? 1 : 0)) * 2 + tile_idx;  // begun in cf, earlier in the rest
            const float2 ml = a.part_ml[p * kChunkPartRows + r];
            const float* src = a.part_o + (p * a.D + y) * kChunkPartRows + r;
            float v[E];
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = y + 8 * e < a.D ? src[(size_t)e * 8 * kChunkPartRows] : 0.f;
            if (ml.x == -INFINITY && ml.y == 0.f) continue;  // the part saw nothing of this row
            const float mx = fmaxf(m, ml.x);
            const float w_old = exp2_diff(m, mx), w = fast_exp2(ml.x - mx);
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = o[e] * w_old + v[e] * w;
            l = l * w_old + ml.y * w;
            m = mx;
        }
        const float inv = l == 0.f ? 0.f : a.v_scale[it.l] / l;  // nothing seen: zero; a NaN stays one
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (y + 8 * e < a.D) tile[x][y + 8 * e] = o[e] * inv;
        if (y == 0) {
            const int tok = it.first + tok0 + row / a.G, h = row % a.G;
            const float lse2 = l == 0.f ? -INFINITY : m + log2f(l);
            if (a.lse) a.lse[((size_t)it.li * a.n_tokens + tok) * a.Hq + it.hkv * a.G + h] = lse2 * 0.6931471805599453f;
            a.nlse2[(((size_t)it.li * a.Hkv + it.hkv) * a.n_tokens + tok) * a.G + h] = l == 0.f ? -INFINITY : -lse2;
        }
    }
    __syncthreads();
    for (int rr = y; rr < kCombineRows; rr += 8) {
        const int r2 = row0 % kChunkPartRows + rr, row2 = tile_idx * a.TT * a.G + r2;
        if (r2 >= a.TT * a.G || row2 >= rows) break;
        const size_t orow = ((size_t)it.li * a.n_tokens + it.first + tok0 + row2 / a.G) * a.Hq + it.hkv * a.G + row2 % a.G;
        for (int d = 2 * x; d < a.D; d += 64) {
            if (a.dtype == LETHE_F32) *reinterpret_cast<float2*>((float*)a.out + orow * a.D + d) = make_float2(tile[rr][d], tile[rr][d + 1]);
            else *reinterpret_cast<__nv_bfloat162*>((__nv_bfloat16*)a.out + orow * a.D + d) = __floats2bfloat162_rn(tile[rr][d], tile[rr][d + 1]);
        }
    }
}

// Eq. 5 from parked logits: a thread takes four keys, adds up exp2(logit - lse + log2 of the row's decay weight) over the chunk's rows.
// Bound by memory: 4 bytes per row and key read, against 2 D of the key itself for the transposed product.  Chunks of up to 16 rows
// take it: single tokens of 32 sequences with a window and a cap 79 us for the call, 107 with the transposed product; four drafted
// tokens of 8 sequences 39 against 48.
constexpr int kParkKeys = 4 * kPrepThreads;
__global__ void __launch_bounds__(kPrepThreads) chunk_rel_parked_kernel(const __grid_constant__ ChunkArgs a) {
    __shared__ float bias[kChunkQuadRows];
    dependency_wait();
    dependency_release();
    const int per_item = (a.cap_tokens + kParkKeys - 1) / kParkKeys;
    const int idx = blockIdx.x / per_item, block = blockIdx.x - idx * per_item;
    const ChunkItem it = chunk_item(a, idx);
    if (it.n_old < 0 || it.T == 0 || block * kParkKeys >= it.n) return;
    const int tid = threadIdx.x, rows = it.T * a.G;
    if (block == 0 && tid == 0 && a.append) a.len[it.item] = it.n;
    if (tid < rows) bias[tid] = a.nlse2[(((size_t)it.li * a.Hkv + it.hkv) * a.n_tokens + it.first) * a.G + tid] + (float)(it.T - 1 - tid / a.G) * a.gamma_log2;
    // what the attention has gone through, and so written: one unit per item
    const int lo = a.u_hi ? a.u_lo[idx] * kChunkTile : 0, hi = a.u_hi ? a.u_hi[idx] : it.n;
    const int j0 = block * kParkKeys + 4 * tid;
    float* rel = a.rel + (size_t)it.item * a.cap_tokens + j0;
    float old[4], sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k) old[k] = j0 + k < it.n_old ? rel[k] : 0.f;
    __syncthreads();
    if (j0 < hi && j0 + 4 > lo) {  // lo is a multiple of four; keys from hi on are -inf or left out below
        const float* src = a.park + (size_t)idx * a.park_rows * a.park_pitch + j0;
#pragma unroll 4
        for (int r = 0; r < rows; ++r) {
            const float4 x = *reinterpret_cast<const float4*>(src + (size_t)r * a.park_pitch);
            const float b = bias[r];
            if (x.x != -INFINITY) sum[0] += fast_exp2(x.x + b);
            if (x.y != -INFINITY) sum[1] += fast_exp2(x.y + b);
            if (x.z != -INFINITY) sum[2] += fast_exp2(x.z + b);
            if (x.w != -INFINITY) sum[3] += fast_exp2(x.w + b);
        }
    }
    const float decay = exp2f((float)it.T * a.gamma_log2);
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (j0 + k < it.n) rel[k] = fmaf(decay, old[k], j0 + k < hi ? sum[k] : 0.f);
}

// Pairs of key tiles that more than one CTA of the relevance kernel worked on: the parts are added in the order of their tokens.
// One block per CTA whose stretch begins inside a pair, the pair's first such CTA speaks for it.  A launch's latency, 3 us.
__global__ void __launch_bounds__(kPrepThreads) chunk_rel_finish_kernel(const __grid_constant__ ChunkArgs a) {
    dependency_wait();
    dependency_release();
    const int c = 1 + blockIdx.x, per = a.plan->rel_per;
    if ((long long)c * per >= a.plan->rel_total) return;
    const int4 cut = a.rel_cut[c];  // item, pair, first step, end
    const int c0 = cut.z / per, c1 = (cut.w - 1) / per;
    if (c0 != c - 1 || cut.z == c * per) return;
    const ChunkItem it = chunk_item(a, cut.x);
    const int j = cut.y * 2 * kChunkTile + threadIdx.x;
    if (j >= it.n) return;
    float sum = 0.f;
    for (int k = c0; k <= c1; ++k) sum += a.rel_part[((size_t)k * 2 + (k == c0 ? 1 : 0)) * (2 * kChunkTile) + threadIdx.x];
    float* rel = a.rel + (size_t)it.item * a.cap_tokens + j;
    *rel = fmaf(exp2f((float)it.T * a.gamma_log2), j < it.n_old ? *rel : 0.f, sum);
}

}  // namespace

cudaError_t launch_chunk_rel_parked(const ChunkArgs& a, cudaStream_t stream) {
    const int per_item = (a.cap_tokens + kParkKeys - 1) / kParkKeys;
    return launch_dependent(chunk_rel_parked_kernel, dim3(per_item * a.n_items), kPrepThreads, 0, stream, a);
}

cudaError_t launch_chunk_rel_finish(const ChunkArgs& a, cudaStream_t stream) {
    static_assert(kPrepThreads == 2 * kChunkTile, "one thread per key of a pair");
    return launch_dependent(chunk_rel_finish_kernel, dim3(a.n_rel_cta - 1), kPrepThreads, 0, stream, a);
}

cudaError_t launch_chunk_append(const ChunkArgs& a, cudaStream_t stream) {
    // at most two waves of blocks
    const long long rows = a.append ? (long long)a.nl * a.n_tokens * a.Hkv : 0;
    const long long want = (rows + 4 * kPrepWarps - 1) / (4 * kPrepWarps);
    const int blocks = 1 + (int)(want < 2368 ? want : 2368);
    cudaError_t e = launch_dependent(chunk_append_kernel, dim3(blocks), kPrepThreads, 0, stream, a);
    if (e == cudaSuccess && a.u_hi) e = launch_dependent(chunk_range_kernel, dim3(a.n_items), kRangeThreads, 0, stream, a);
    return e;
}

cudaError_t launch_chunk_combine(const ChunkArgs& a, cudaStream_t stream) {
    if (a.n_cta < 2) return cudaSuccess;
    // rows of a unit in the parts: one or two row tiles, each padded to whole blocks
    const int tile_rows = min(a.TT, a.max_chunk) * a.G;
    const int row_blocks = a.max_chunk > a.TT && a.TU > a.TT ? 2 * kChunkPartRows / kCombineRows : (tile_rows + kCombineRows - 1) / kCombineRows;
    return launch_dependent(chunk_combine_kernel, dim3((a.n_cta - 1) * row_blocks), kPrepThreads, 0, stream, a, row_blocks);
}

}  // namespace lethe
