// Arguments and device helpers shared by the kernels of lethe_chunk_attend.
//
// A call is a short chain of launches, each a programmatic dependent of the one before:
//   append   new rows into the cache, pos; block 0 writes the plan
//   range    only for masks by position: the tiles each unit can see, then the plan
//   attend   softmax attention of the chunk, split evenly over the GPU by the plan
//   combine  merges what the split left in parts
//   rel      Eq. 5 for the chunk from the final softmax statistics; len.  Chunks of at most 16 rows (single tokens, drafted tokens):
//            from the logits that `attend` has parked; longer ones: from a second, transposed product
//
// A unit is a block of TU consecutive tokens of one sequence with the G query heads of one KV head (for the tensor-core
// kernel two tiles of up to 128 rows).  Its cost is the number of 128-key tiles it can see.  The plan lays all units end to
// end on a line of tiles and gives every CTA an equal stretch: lengths are only known on the device, and an even cut keeps
// ragged batches, single long sequences and causal triangles balanced alike.  A stretch may begin or end inside a unit; such
// a unit leaves one part per CTA, joined by `combine` in CTA order (deterministic: nothing is added atomically).
#pragma once
#include "common.cuh"

namespace lethe {

constexpr int kChunkTile = 128;    // keys per tile of the tensor-core kernels
constexpr int kChunkParts = 4;     // parts a CTA can leave: (unit begun earlier, unit begun here and continued later) x two row tiles
constexpr int kChunkPartRows = 128;
constexpr int kChunkQuadRows = 16; // rows of a short chunk that all softmax warps work on together

struct ChunkPlan {  // head of the call's scratch
    int total;      // tiles of all units
    int per;        // tiles per CTA
    int refused;    // chunk_start is malformed: nothing is done
    int done;       // blocks of the range kernel that have finished
    int rel_total;  // steps of the relevance kernel
    int rel_per;    // steps per CTA
};

struct ChunkArgs {
    const void* k;
    const void* v;
    float* rel;
    int32_t* pos;
    int32_t* len;
    const int32_t* page_table;
    const void* q;
    const void* k_new;
    const void* v_new;
    const int32_t* token_pos;
    const int32_t* chunk_start;
    void* out;
    float* lse;
    int32_t* status;
    // scratch
    ChunkPlan* plan;
    int* n_old;      // [items] retained tokens before the call; -1: the item is left alone
    int* u_start;    // [n_units + 1] where each unit begins on the line: its pad, then its tiles
    int* u_lo;       // [n_units] first key tile of the unit (masks by position only, else NULL)
    int* u_hi;       // [n_units] slots the unit can see end here (masks by position only, else NULL)
    int* cta_unit;   // [n_cta] the unit that holds the first tile of each CTA's stretch
    // the relevance kernel's line (tensor-core kernels, else NULL): (pair of key tiles, query tile) steps, item by item
    int* rel_start;  // [n_items + 1] first step of each item
    int* rel_item;   // [n_rel_cta] the item that holds the first step of each CTA's stretch
    int2* rel_hull;  // [n_items][ceil(cap_tiles / 2)] query tiles that meet a pair: first and end (masks by position only, else NULL)
    int* rel_cost;   // [n_items] steps of an item (masks by position only)
    int4* rel_cut;   // [n_rel_cta] where a CTA's stretch begins: item, pair, first step of the pair, end of it
    float* rel_part; // [n_rel_cta][2][256] sums of a pair begun earlier, and of one begun here and continued later
    int n_rel_cta;
    int2* bounds;    // [items][cap_tiles] smallest and largest pos of a key tile (masks by position only, else NULL)
    float* park;     // [n_items][park_rows][park_pitch] shaped logits in log2 units, -inf where masked (short chunks, else NULL)
    int park_rows, park_pitch;
    float* nlse2;    // [nl][Hkv][n_tokens][G] minus the log-sum-exp, in log2 units; -inf for a row that sees nothing
    float* part_o;   // [n_cta][kChunkParts][D][kChunkPartRows]: a thread that owns a row writes beside its neighbours
    float2* part_ml; // [n_cta][kChunkParts][kChunkPartRows] (max in log2 units, sum)
    long long n_pages;
    int dtype, D;
    int B, Hq, Hkv, G, capacity, cap_tokens, page_tokens, paged;
    int layer_begin, nl, n_items, n_tokens, max_chunk;
    int TT;          // tokens per row tile
    int TU;          // tokens per unit
    int QT;          // units per item
    int tile;        // keys per tile of the plan: 128 for the tensor cores, fewer for the CUDA cores
    int n_units, n_cta, cap_tiles, min_per;
    int pad;         // tiles' worth of time that beginning and ending a unit takes (unit_pad), laid on the line before its tiles
    int append;
    float gamma_log2;
    int wait_limit;
    // score modification
    float softcap;
    int window;
    const float* slopes;
    const int32_t* doc_start;
    const int32_t* prefix_len;
    float scale[kMaxLayers];    // softmax scale, by absolute layer
    float k_scale[kMaxLayers];
    float v_scale[kMaxLayers];
};

struct ChunkItem {
    int li, l, b, hkv, item;  // item: absolute flat item
    int first, T;             // first packed token and number of tokens of the sequence
    int n_old, n;             // slots before and after the call; n_old = -1: left alone
};

// One sequence's stretch of the packed tokens is taken as chunk_start says: the append kernel has checked it (plan->refused).
__device__ __forceinline__ ChunkItem chunk_item(const ChunkArgs& a, int idx) {
    ChunkItem c;
    c.hkv = idx % a.Hkv;
    c.b = (idx / a.Hkv) % a.B;
    c.li = idx / (a.Hkv * a.B);
    c.l = a.layer_begin + c.li;
    c.item = (c.l * a.B + c.b) * a.Hkv + c.hkv;
    c.first = a.chunk_start[c.b];
    c.T = a.chunk_start[c.b + 1] - c.first;
    c.n_old = a.n_old[idx];
    c.n = c.n_old + (a.append ? c.T : 0);
    return c;
}

// Byte offset of row `slot` of an item, in rows; -1 for a page id outside the pool.
__device__ __forceinline__ long long chunk_row(const ChunkArgs& a, int item, int slot) {
    if (!a.paged) return (long long)item * a.capacity + slot;
    const int page = a.page_table[(size_t)item * a.capacity + slot / a.page_tokens];
    if (page < 0 || page >= a.n_pages) return -1;
    return (long long)page * a.page_tokens + slot % a.page_tokens;
}

// What a query row needs to know to test a key.
struct ChunkRow {
    int lim;     // slots below lim are in causal order
    int qpos;    // original position
    int lo;      // keys with a smaller position are hidden (window, document)
    float slope; // distance bias, log2 units
};

__device__ __forceinline__ int chunk_lo(const ChunkArgs& a, int tok, int qpos) {
    int lo = INT32_MIN;
    if (a.window > 0) {
        const long long w = (long long)qpos - a.window + 1;
        lo = w < INT32_MIN ? INT32_MIN : (int)w;
    }
    if (a.doc_start) lo = max(lo, a.doc_start[tok]);
    return lo;
}

// softcap * tanh(x / softcap) in log2 units: t = x / softcap, cap2 = softcap * log2(e).  An odd polynomial (fitted to tanh(t) / t
// on t^2 <= 0.55^2; largest error 1e-9 before rounding) where scores usually are, 1 - 2 / (1 + e^2|t|) beyond: that form alone
// has an absolute error of an ulp of one at small t, which times the cap would cost a score its low bits.
__device__ __forceinline__ float capped_small(float t) {
    const float u = t * t;
    float p = fmaf(u, -0.006235556820094805f, 0.021039673409724794f);
    p = fmaf(u, p, -0.05384270671952741f);
    p = fmaf(u, p, 0.13332460742850846f);
    p = fmaf(u, p, -0.33333310957894996f);
    p = fmaf(u, p, 0.9999999990645916f);
    return t * p;
}
__device__ __forceinline__ float capped_large(float t) {
    const float e = fast_exp2(fabsf(t) * 2.885390081777927f);
    const float r = copysignf(1.f - __fdividef(2.f, 1.f + fminf(e, 1e30f)), t);
    return t == t ? r : t;  // the minimum would turn a NaN into a cap
}
__device__ __forceinline__ float capped(float t) { return fabsf(t) <= 0.55f ? capped_small(t) : capped_large(t); }

// Tiles' worth of time that beginning and ending a unit of `toks` tokens takes (a unit with two row tiles of outputs).
__device__ __forceinline__ int unit_pad(const ChunkArgs& a, int toks) { return toks > a.TT ? a.pad : 0; }
// Tiles of a unit that begins at s0 on the line which lie before point x of the line.
__device__ __forceinline__ int tiles_before(const ChunkArgs& a, int toks, int s0, int x) { return max(0, x - s0 - unit_pad(a, toks)); }

// Query tiles that a pair of key tiles (its first slot j0) meets: [lo, hi); none where masks hide it from all.
__device__ __forceinline__ int2 rel_hull(const ChunkArgs& a, const ChunkItem& it, int idx, int pair) {
    if (a.rel_hull) return a.rel_hull[(size_t)idx * ((a.cap_tiles + 1) / 2) + pair];
    const int lo = a.append ? max(0, pair * 2 * kChunkTile - it.n_old) / a.TT : 0;  // earlier tokens do not reach the pair
    return make_int2(lo, (it.T + a.TT - 1) / a.TT);
}
__device__ __forceinline__ int rel_steps(int2 hull) { return max(1, hull.y - hull.x); }  // a pair that nobody sees still decays
__device__ __forceinline__ int rel_pairs(const ChunkItem& it) { return (it.n + 2 * kChunkTile - 1) / (2 * kChunkTile); }

cudaError_t launch_chunk_append(const ChunkArgs& a, cudaStream_t stream);
cudaError_t launch_chunk_combine(const ChunkArgs& a, cudaStream_t stream);
cudaError_t launch_chunk_rel_parked(const ChunkArgs& a, cudaStream_t stream);
cudaError_t launch_chunk_rel_finish(const ChunkArgs& a, cudaStream_t stream);
cudaError_t launch_chunk_simt(const ChunkArgs& a, cudaStream_t stream);

// Launch with the programmatic dependency attribute: the kernel may start while the one before it is still finishing and waits
// (griddepcontrol.wait) before it touches global memory.
template <typename... KArgs, typename... Args>
inline cudaError_t launch_dependent(void (*kern)(KArgs...), dim3 grid, int threads, size_t smem, cudaStream_t stream, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, KArgs(args)...);
}
__device__ __forceinline__ void dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void dependency_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace lethe
