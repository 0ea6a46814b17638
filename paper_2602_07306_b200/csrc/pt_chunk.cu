// Attention of a ragged chunk of new tokens over the paged KV cache: sequence b brings qlen[b] rows (none is allowed)
// that sit at the last qlen[b] of its kvlen[b] cached positions; row s sees the keys 0 .. kvlen - qlen + s.
#include "pt_chunk.h"
#include "pt_kernels.h"
#include "pt_ptx.cuh"

namespace pt {

namespace {

// The sequence of packed row m (-1 behind the last one) and its first row; a warp calls it with all lanes.  False where
// any length is out of range (reported, and the caller writes nothing).
__device__ __forceinline__ bool find_sequence(const ChunkP& p, int m, int& b, int& first) {
    const int lane = threadIdx.x & 31;
    int64_t run = 0;
    bool bad = false;
    b = -1; first = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
        const bool in = b0 + lane < p.B;
        const int ql = in ? p.qlen[b0 + lane] : 0, kl = in ? p.kvlen[b0 + lane] : 0;
        bad |= ql < 0 || kl < ql || (int64_t)kl > (int64_t)p.maxp * p.ps;
        int64_t incl = ql;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int64_t u = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += u; }
        const bool mine = in && m >= run + incl - ql && m < run + incl;
        const unsigned who = __ballot_sync(0xffffffffu, mine);
        if (who) {
            b = b0 + __ffs(who) - 1;
            first = (int)__shfl_sync(0xffffffffu, run + incl - ql, __ffs(who) - 1);
        }
        run += __shfl_sync(0xffffffffu, incl, 31);
    }
    bad = __any_sync(0xffffffffu, bad) || run > p.M;
    if (bad && lane == 0) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_CHUNK_LEN);
    return !bad;
}

// One warp per (row, query head, track): online softmax over the visible keys, everything in fp32.
template <int DH>
__global__ void __launch_bounds__(128)
k_chunk_simple(const ChunkP p) {
    constexpr int PER = DH / 32;
    const int64_t id = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31, t = blockIdx.y;
    if (id >= (int64_t)p.M * p.nq) return;
    const int m = (int)(id / p.nq), head = (int)(id % p.nq), kvh = head / (p.nq / p.nkv);
    int b, first;
    if (!find_sequence(p, m, b, first) || b < 0) return;
    const int pos = p.kvlen[b] - p.qlen[b] + (m - first);
    const size_t row = ((size_t)t * p.M + m) * (size_t)(p.nq * DH) + (size_t)head * DH;
    float qv[PER], acc[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) { qv[i] = __bfloat162float(p.q[row + lane + 32 * i]) * p.scale_log2; acc[i] = 0.f; }
    float mx = -INFINITY, den = 0.f;
    const __nv_bfloat16* slab = p.pool_l + (size_t)t * p.pool_tstride;
    for (int j = 0; j <= pos; ++j) {
        const int page = p.bt[(size_t)b * p.maxp + j / p.ps];
        if (page < 0 || page >= p.num_pages) { if (lane == 0) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_CHUNK_PAGE); return; }
        const __nv_bfloat16* kp = slab + (((size_t)page * 2) * p.nkv + kvh) * p.ps * DH + (size_t)(j % p.ps) * DH;
        const __nv_bfloat16* vp = kp + (size_t)p.nkv * p.ps * DH;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) s += qv[i] * __bfloat162float(kp[lane + 32 * i]);
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        const float nm = fmaxf(mx, s);
        const float corr = exp2f(mx - nm), w = exp2f(s - nm);
        den = den * corr + w;
#pragma unroll
        for (int i = 0; i < PER; ++i) acc[i] = acc[i] * corr + w * __bfloat162float(vp[lane + 32 * i]);
        mx = nm;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) p.o[row + lane + 32 * i] = __float2bfloat16_rn(acc[i] / den);
}

}  // namespace

static bool chunk_tc_supported(int dh, int ps) { return (dh == 64 || dh == 128) && ps % 16 == 0; }

// The same whatever the batch: the tensor-memory kernel cuts its work once per block, not once per sequence.
size_t chunk_scratch_bytes(int T, int B, int nq, int dh) { return dh == 32 ? 256 : chunk_tc_scratch_bytes(dh); }

pt_status launch_chunk_attn(const ChunkP& p, int dh, void* scratch, bool simple, cudaStream_t st) {
    if (!simple && chunk_tc_supported(dh, p.ps)) return launch_chunk_attn_tc(p, dh, scratch, st);
    const int64_t blocks = ((int64_t)p.M * p.nq + 3) / 4;
    if (blocks > 0x7fffffff || p.T > 65535) { set_error("chunk attention grid too large"); return PT_ERR_INVALID_ARG; }
    const dim3 grid((unsigned)blocks, p.T);
    if (dh == 32) k_chunk_simple<32><<<grid, 128, 0, st>>>(p);
    else if (dh == 64) k_chunk_simple<64><<<grid, 128, 0, st>>>(p);
    else k_chunk_simple<128><<<grid, 128, 0, st>>>(p);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) { set_error("k_chunk_simple launch: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return PT_OK;
}

pt_status launch_chunk_attn_call(Call& k, const __nv_bfloat16* q, const __nv_bfloat16* pool_l, __nv_bfloat16* o) {
    const pt_model* m = k.m;
    const pt_config& g = m->cfg;
    ChunkP p{};
    p.q = q; p.o = o; p.qlen = k.w.meta.qlen; p.kvlen = k.w.meta.kvlen;
    p.T = g.T; p.B = k.B; p.M = k.M; p.nq = g.heads; p.nkv = g.kv_heads;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)m->dh);
    p.status = m->status();
    if (k.c->coded()) {                     // over the bf16 copy of code * scale, as a prefill
        p.pool_l = (const __nv_bfloat16*)k.w.attn_kv; p.pool_tstride = (int64_t)k.w.meta.attn_pages * 2 * m->KVD * 16;
        p.bt = k.w.meta.bt_attn; p.maxp = k.w.meta.maxp_attn; p.ps = 16; p.num_pages = k.w.meta.attn_pages;
    } else {
        p.pool_l = pool_l; p.pool_tstride = (int64_t)g.L * k.c->slab_elems;
        p.bt = k.w.meta.bt; p.maxp = k.w.meta.maxp; p.ps = k.c->ps; p.num_pages = k.c->num_pages;
    }
    return launch_chunk_attn(p, m->dh, k.w.chunk, false, k.st);
}

}  // namespace pt

using namespace pt;

extern "C" pt_status pt_kernel_chunk_attn_scratch_bytes(int32_t T, int32_t B, int32_t nq, int32_t dh, size_t* bytes) {
    if (!bytes || T < 1 || B < 1 || nq < 1 || dh < 1) { set_error("bad argument"); return PT_ERR_INVALID_ARG; }
    *bytes = chunk_scratch_bytes(T, B, nq, dh);
    return PT_OK;
}

extern "C" pt_status pt_kernel_chunk_attn(const void* q, const void* pool_l, int64_t pool_track_stride,
                                          const int32_t* block_table, int32_t maxp, const int32_t* q_len, const int32_t* kv_len,
                                          int32_t T, int32_t B, int32_t M, int32_t nq, int32_t nkv, int32_t dh, int32_t ps,
                                          int32_t num_pages, void* out, int32_t impl, void* scratch, size_t scratch_bytes,
                                          void* status, void* stream) {
    if (!q || !pool_l || !block_table || !q_len || !kv_len || !out || !scratch || !status) { set_error("null argument"); return PT_ERR_INVALID_ARG; }
    if (T < 1 || B < 1 || M < 1 || M > (1 << 30) || nq < 1 || nkv < 1 || nq % nkv || maxp < 1 || num_pages < 1 || pool_track_stride < 0) { set_error("bad sizes"); return PT_ERR_INVALID_ARG; }
    if (nq / nkv > 8) { set_error("more than 8 query heads per KV head"); return PT_ERR_UNSUPPORTED; }
    if (dh != 32 && dh != 64 && dh != 128) { set_error("head_dim %d not in {32, 64, 128}", dh); return PT_ERR_UNSUPPORTED; }
    if (ps < 8 || ps > 64 || ps % 8) { set_error("page size must be a multiple of 8 in [8, 64]"); return PT_ERR_INVALID_ARG; }
    if ((int64_t)maxp * ps > 0x7fffffff - 127) { set_error("a block table of more than 2^31 - 128 keys"); return PT_ERR_UNSUPPORTED; }   // rounded up to tiles in 32 bits
    if (impl != 0 && impl != 1) { set_error("impl must be 0 or 1"); return PT_ERR_INVALID_ARG; }
    if (impl == 0 && !chunk_tc_supported(dh, ps)) { set_error("impl 0 needs head_dim 64 or 128 and pages of a multiple of 16 tokens"); return PT_ERR_UNSUPPORTED; }
    if ((uintptr_t)q % 16 || (uintptr_t)pool_l % 16 || pool_track_stride % 8 || (uintptr_t)out % 32 || (uintptr_t)scratch % 256) {
        set_error("q and the pool must be 16-byte aligned (its track stride a multiple of 8 elements), out 32-byte, scratch 256-byte"); return PT_ERR_MISALIGNED;
    }
    if (((uintptr_t)block_table | (uintptr_t)q_len | (uintptr_t)kv_len | (uintptr_t)status) % 4) { set_error("block_table, q_len, kv_len and status must be 4-byte aligned"); return PT_ERR_MISALIGNED; }
    const size_t need = chunk_scratch_bytes(T, B, nq, dh);
    if (scratch_bytes < need) { set_error("scratch: %zu < %zu bytes", scratch_bytes, need); return PT_ERR_BUFFER_TOO_SMALL; }
    ChunkP p{};
    p.q = (const __nv_bfloat16*)q; p.pool_l = (const __nv_bfloat16*)pool_l; p.pool_tstride = pool_track_stride; p.o = (__nv_bfloat16*)out;
    p.bt = block_table; p.maxp = maxp; p.qlen = q_len; p.kvlen = kv_len;
    p.T = T; p.B = B; p.M = M; p.nq = nq; p.nkv = nkv; p.ps = ps; p.num_pages = num_pages;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)dh);
    p.status = (int*)status;
    return launch_chunk_attn(p, dh, scratch, impl == 1, (cudaStream_t)stream);
}
