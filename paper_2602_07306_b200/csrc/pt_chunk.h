// Attention of a ragged chunk of new tokens per sequence over the paged KV cache (pt_chunk.cu).
#pragma once
#include "pt_internal.h"

namespace pt {

struct ChunkP {
    const __nv_bfloat16* q;        // [T][M][nq*dh], the rows of sequence b behind those of sequence b - 1
    const __nv_bfloat16* pool_l;   // KV slab of one layer, track 0
    int64_t pool_tstride;
    __nv_bfloat16* o;              // [T][M][nq*dh]
    const int32_t* bt; int maxp;
    const int32_t* qlen;           // [B] new tokens
    const int32_t* kvlen;          // [B] keys cached, the new tokens' included
    int T, B, M, nq, nkv, ps, num_pages;
    float scale_log2;              // log2(e) / sqrt(dh)
    int* status;
};

size_t chunk_scratch_bytes(int T, int B, int nq, int dh);
// simple: the plain kernel (one warp per row and head), which takes any head_dim and page size and serves what the other does not
pt_status launch_chunk_attn(const ChunkP& p, int dh, void* scratch, bool simple, cudaStream_t st);
// pt_chunk_tc.cu: the tensor-memory kernel (head_dim 64 or 128, pages of a multiple of 16 tokens)
size_t chunk_tc_scratch_bytes(int dh);
pt_status launch_chunk_attn_tc(const ChunkP& p, int dh, void* scratch, cudaStream_t st);
// the attention of one layer of a pt_extend call
pt_status launch_chunk_attn_call(Call& k, const __nv_bfloat16* q, const __nv_bfloat16* pool_l, __nv_bfloat16* o);

}  // namespace pt
