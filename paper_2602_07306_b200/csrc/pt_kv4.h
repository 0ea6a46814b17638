// The 4-bit storage format of the KV cache (pt_kv_dtype PT_KV_E2M1): write, read back, attention from the codes.
#pragma once
#include "pt_internal.h"

namespace pt {

// A page is [kv_head][slot / 16] blocks of 16 tokens: K codes, K scales, V codes, V scales (pt.h has the order inside).
__host__ __device__ constexpr int kv4_codes(int dh) { return 8 * dh; }                 // bytes of 16 tokens' K (or V) codes
__host__ __device__ constexpr int kv4_scales(int dh) { return 16 * (dh / 32); }        // and of their scales
__host__ __device__ constexpr int kv4_block(int dh) { return 2 * (kv4_codes(dh) + kv4_scales(dh)); }
inline bool kv4_supported(int dh, int ps) { return (dh == 64 || dh == 128) && ps % 16 == 0 && ps >= 16 && ps <= 64; }

struct Kv4Slab {                      // one layer
    char* pool_l; int64_t tstride;    // track 0; bytes between tracks
    int nkv, ps, num_pages;
};

// whether two stretches of memory share a byte
inline bool kv4_meet(const void* a, double bytes_a, const void* b, double bytes_b) {
    const double x = (double)(uintptr_t)a, y = (double)(uintptr_t)b;                // below 2^53 where an address is one
    return x < y + bytes_b && y < x + bytes_a;
}

struct Kv4WriteP {
    const __nv_bfloat16* k; const __nv_bfloat16* v;   // vector of (track, row, head) at t*tstride + row*row_stride + head*head_stride
    int64_t tstride, row_stride, head_stride;
    Kv4Slab slab;
    const int64_t* slots;             // [M] page * ps + slot, negative: the row is not cached
    __nv_bfloat16* k_out; __nv_bfloat16* v_out;       // [T][M][nkv*dh] the rounded values, may be null
    int T, M;
    int* status;
};
pt_status launch_kv4_write(const Kv4WriteP& p, int dh, cudaStream_t st);

struct Kv4ReadP {
    Kv4Slab slab;
    const int32_t* bt; int maxp;
    const int32_t* kvlen;             // [B]
    __nv_bfloat16* out_l; int64_t out_tstride;        // pages [K|V][kv_head][out_ps][dh]; elements between tracks
    const int32_t* obt; int omaxp; int ops, opages;
    int T, B;
    int* status;
};
pt_status launch_kv4_read(const Kv4ReadP& p, int dh, cudaStream_t st);

struct Kv4AttnP {
    const __nv_bfloat16* q;           // [T][M][nq*dh], the rows of sequence b behind those of sequence b - 1
    __nv_bfloat16* o;
    Kv4Slab slab;
    const int32_t* bt; int maxp;
    const int32_t* qlen;              // [B] new tokens; null: one each
    const int32_t* kvlen;             // [B] keys cached, the new tokens' included
    int T, B, M, nq;
    float scale_log2;                 // log2(e) / sqrt(dh)
    int tiles;                        // row tiles a pass, 1 .. 3
    int* status;
};
int kv4_mean_tiles(int64_t rows, int B);                           // for `rows` (token, head) rows of a KV head whose lengths are not known
size_t kv4_attn_scratch_bytes(int dh);
pt_status launch_kv4_attn(const Kv4AttnP& p, int dh, void* scratch, cudaStream_t st);


// one layer of a forward call on an E2M1 cache
pt_status launch_kv4_write_call(Call& k, int layer);
pt_status launch_kv4_read_call(Call& k, int layer);               // all of the call's keys into the bf16 copy
pt_status launch_kv4_attn_call(Call& k, const __nv_bfloat16* q, int layer, __nv_bfloat16* o);
// How a call with n_new[b] new tokens on sequences that then have lens[b] keys attends: straight to the codes with `tiles` row tiles
// a pass (1 .. 3), or (0) to a bf16 copy.  G: query heads per KV head.
int kv4_plan(const int32_t* lens, const int32_t* n_new, int B, int G);

}  // namespace pt
