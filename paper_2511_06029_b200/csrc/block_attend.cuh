// Arguments of lethe_block_attend's kernel.
#pragma once
#include <cuda.h>

#include "block.cuh"

namespace lethe {

constexpr int kBlockWarps = 8;  // warps of a CTA, each with a ring of its own; one CTA per SM
constexpr int kBlockStep = 32;  // tokens of a step
constexpr int kBlockTail = 3;   // length on the line of 32 open rows, which are fetched without a ring
constexpr int kBlockPad = 3;    // and of an item's beginning: its length, first pages, queries and first tile come one after the other
constexpr int kBlockStages = 2;  // steps in a ring at D = 128

struct alignas(64) BlockMaps {
    CUtensorMap k, v;  // [blocks * block_tokens][D] bytes, boxes of a step's rows, or of a block's where those are fewer
};

struct BlockAttendArgs {
    BlockView c;
    const __nv_bfloat16* q;
    const int32_t* selected;  // NULL: all blocks
    __nv_bfloat16* out;
    float* lse;
    float* cta_part;          // [CTAs][2][8 heads][kBlockPart]: items that begin before / go on behind the CTA
    int* counters;            // [items][8 heads] CTAs that have left a part, zero between launches
    int n_select, n_cta, wait_limit;
};
constexpr int kBlockPart = 4 + 128;  // m, l (the part's weight is l 2^m), two unused, then O divided by the weight

bool build_block_maps(void* encode, const BlockView& c, BlockMaps* maps);
cudaError_t launch_block_attend(const BlockAttendArgs& a, const BlockMaps& maps, cudaStream_t stream);

}  // namespace lethe
