// Arguments of lethe_block_attend's kernel.
#pragma once
#include <cuda.h>

#include "block.cuh"

namespace lethe {

constexpr int kBlockWarps = 16;  // warps of a CTA, each with a ring of its own; one CTA per SM

struct alignas(64) BlockMaps {
    CUtensorMap k, v;  // [blocks * block_tokens][D] bytes, boxes of 16 rows
};

struct BlockAttendArgs {
    BlockView c;
    const __nv_bfloat16* q;
    const int32_t* selected;  // NULL: all blocks
    __nv_bfloat16* out;
    float* lse;
    float* warp_part;         // [CTAs][kBlockWarps][kBlockPart]: a warp's first stretch, when it has others after it
    float* cta_part;          // [CTAs][2][kBlockPart]: items that begin before / go on behind the CTA
    int* counters;            // [items] CTAs that have left a part, zero between launches
    int n_select, n_cta, wait_limit;
};
constexpr int kBlockPart = 16 + 8 * 128;  // 8 x (max, sum), then O by head

bool build_block_maps(void* encode, const BlockView& c, BlockMaps* maps);
cudaError_t launch_block_attend(const BlockAttendArgs& a, const BlockMaps& maps, cudaStream_t stream);

}  // namespace lethe
