// Arguments of lethe_rotate's kernel, also used by lethe_chunk_attend for queries and keys that come unrotated.
#pragma once
#include "chunk.cuh"

namespace lethe {

struct RotateArgs {
    const void* q;
    const void* k;
    void* q_out;
    void* k_out;
    const int32_t* axis_pos;
    int nl, n_tokens, Hq, Hkv, D, rot_dim, halves, inverse;
    int rows;            // nl * (Hq + Hkv); Hkv = 0 without keys
    int rows_per_block;
    unsigned long long turn[64];  // turns per position, a fraction of 2^64
    unsigned char axis[64];
};

cudaError_t launch_rotate(const RotateArgs& a, bool f32, cudaStream_t stream);

}  // namespace lethe
