// Attention of one or a few new tokens per sequence straight from a 4-bit cache (pt_kv_dtype PT_KV_E2M1).
// A warp per row and head, one key at a time.
#include "pt_kv4.cuh"
#include "pt_tc.h"
#include "pt_ptx.cuh"

namespace pt {

namespace {

template <int DH>
__global__ void __launch_bounds__(128) k_kv4_attn(const Kv4AttnP p) {
    grid_dep_wait();
    grid_dep_launch();
    constexpr int PER = DH / 32;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31, t = blockIdx.y, nkv = p.slab.nkv, ps = p.slab.ps;
    if (w >= (int64_t)p.M * p.nq) return;
    const int r = (int)(w / p.nq), head = (int)(w % p.nq), kvh = head / (p.nq / nkv);
    int b = -1, pos = 0;
    int64_t row0 = 0;
    bool bad = false;
    for (int i = 0; i < p.B; ++i) {
        const int ql = p.qlen ? p.qlen[i] : 1, kl = p.kvlen[i];
        if (ql < 0 || kl < ql || kl > (int64_t)p.maxp * ps) bad = true;
        if (b < 0 && r < row0 + ql) { b = i; pos = kl - ql + (int)(r - row0); }
        row0 += ql;
    }
    if (bad || row0 > p.M) { if (lane == 0) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_KV4_LEN); return; }
    if (b < 0) return;
    const size_t at = ((size_t)t * p.M + r) * p.nq * DH + (size_t)head * DH;
    float qv[PER], acc[PER] = {}, m = -INFINITY, l = 0.f;
    for (int i = 0; i < PER; ++i) qv[i] = __bfloat162float(p.q[at + lane + 32 * i]) * p.scale_log2;
    for (int j = 0; j <= pos; ++j) {
        const int page = p.bt[(size_t)b * p.maxp + j / ps];
        if (page < 0 || page >= p.slab.num_pages) { if (lane == 0) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_KV4_PAGE); return; }
        const int sl = j % 16;
        const char* kc = p.slab.pool_l + (size_t)t * p.slab.tstride + (((int64_t)page * nkv + kvh) * (ps / 16) + j % ps / 16) * kv4_block(DH);
        const char* vc = kc + kv4_codes(DH) + kv4_scales(DH);
        float s = 0.f, v[PER];
        for (int i = 0; i < PER; ++i) {                      // dim 32 i + lane
            uint32_t h[4];
            kv4_codes8(*(const uint32_t*)(kc + kv4_k_word(DH, sl, i, lane >> 3)) >> (4 * (lane & 7)), h);
            s += qv[i] * __low2float(*(const __half2*)h) * kv4_scale((uint8_t)kc[kv4_codes(DH) + kv4_k_scale(DH, sl, i)]);
            kv4_codes8((uint32_t) * (const uint16_t*)(vc + kv4_v_half(DH, sl, i, lane >> 2)) >> (4 * (lane & 3)), h);
            v[i] = __low2float(*(const __half2*)h) * kv4_scale((uint8_t)vc[kv4_codes(DH) + kv4_v_scale(DH, sl, i)]);
        }
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        const float nm = fmaxf(m, s), corr = exp2f(m - nm), wgt = exp2f(s - nm);
        l = l * corr + wgt;
        for (int i = 0; i < PER; ++i) acc[i] = acc[i] * corr + wgt * v[i];
        m = nm;
    }
    for (int i = 0; i < PER; ++i) p.o[at + lane + 32 * i] = __float2bfloat16_rn(acc[i] / l);
}

}  // namespace

size_t kv4_attn_scratch_bytes(int dh) { return (size_t)160 * 2 * 16 * (dh + 2) * 4; }

pt_status launch_kv4_attn(const Kv4AttnP& p, int dh, void* scratch, cudaStream_t st) {
    (void)scratch;
    const dim3 grid((unsigned)(((int64_t)p.M * p.nq + 3) / 4), p.T);
    const cudaError_t e = launch_dependent(dh == 64 ? k_kv4_attn<64> : k_kv4_attn<128>, grid, dim3(128), (size_t)0, st, p);
    if (e != cudaSuccess) { set_error("k_kv4_attn launch: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return PT_OK;
}

}  // namespace pt
