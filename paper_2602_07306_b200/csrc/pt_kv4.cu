// The 4-bit storage format of the KV cache (pt_kv_dtype PT_KV_E2M1): new tokens' K and V into its pages, and sequences back out.
//   k_kv4_write   a thread has eight consecutive values of a vector, four threads a group of 32: the group's maximum takes two
//                 shuffles, its scale is the smallest E5M3 number s with max <= 6 s, and eight codes are one word of K or two
//                 half words of V
//   k_kv4_read    a warp has one head's K and V of 16 tokens, in the order in which they lie: 16 bytes a lane and load
// Both move bytes and compute little.
#include <algorithm>

#include "pt_kv4.cuh"
#include "pt_tc.h"
#include "pt_ptx.cuh"

namespace pt {

namespace {

constexpr int kThreads = 256;

// The code of v / s for the group's scale s, given r = 1 / s rounded: ties between codes have to be met exactly.  v has 8
// significant bits and a tie times s has 7, so v / s is either a tie or at least 2^-8 of it away; v * r is off by 2^-23, and
// rounding it to 12 bits returns to the tie.
__device__ __forceinline__ float kv4_quotient(float v, float r) { return __uint_as_float((__float_as_uint(v * r) + 0x800u) & ~0xfffu); }
__device__ __forceinline__ uint32_t kv4_encode8(const float* y) {
    uint32_t w;
    asm("{\n .reg .b8 a, b, c, d;\n cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n mov.b32 %0, {a, b, c, d};\n}"
        : "=r"(w) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
    return w;
}

template <int DH>
__global__ void __launch_bounds__(kThreads) k_kv4_write(const Kv4WriteP p) {
    constexpr int PER = DH / 8;                                    // threads of a vector
    grid_dep_wait();
    grid_dep_launch();
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int oct = (int)(i % PER), group = oct >> 2, q = oct & 3;
    const int64_t vec = i / PER;                                   // (row, head, K|V)
    const int t = blockIdx.y, nkv = p.slab.nkv;
    const int64_t heads = (int64_t)2 * nkv;
    const bool live = vec < p.M * heads;                           // every lane takes part in the shuffles
    const int64_t row = live ? vec / heads : 0;
    const int kvh = (int)(vec - row * heads), head = live ? kvh % nkv : 0;
    const bool is_v = kvh >= nkv;
    const __nv_bfloat16* src = (is_v ? p.v : p.k) + (size_t)t * p.tstride + row * p.row_stride + head * p.head_stride + oct * 8;
    const uint4 raw = live ? *reinterpret_cast<const uint4*>(src) : make_uint4(0, 0, 0, 0);
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    // magnitudes as whole numbers: a NaN is above infinity, which is above the rest
    uint32_t top = 0;
#pragma unroll
    for (int a = 0; a < 4; ++a) top = __vmaxu2(top, w[a] & 0x7fff7fffu);
    top = max(top & 0xffffu, top >> 16);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const bool bad = top >= 0x7f80u;
    const float amax = bad ? 0.f : __uint_as_float(top << 16);
    // amax / 6 cut to 4 significant bits, or the next number where that is too small (the product is exact)
    uint32_t byte = (uint32_t)__half_as_ushort(__float2half_rz(fminf(amax * (1.0f / 6.0f), 61440.f))) >> 7;
    if (byte < 247 && 6.0f * kv4_scale(byte) < amax) ++byte;
    const float s = kv4_scale(byte), r = s > 0.f ? 1.0f / s : 0.f;
    float y[8];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        y[2 * a] = kv4_quotient(__uint_as_float(w[a] << 16), r);
        y[2 * a + 1] = kv4_quotient(__uint_as_float(w[a] & 0xffff0000u), r);
    }
    const uint32_t code = bad ? 0u : kv4_encode8(y);
    if (bad) byte = 255;
    if (!live) return;
    __nv_bfloat16* val = is_v ? p.v_out : p.k_out;
    if (val) {
        uint32_t h[4];
        kv4_codes8(code, h);
        const float sv = kv4_scale(byte);
        *reinterpret_cast<uint4*>(val + (((size_t)t * p.M + row) * nkv + head) * DH + oct * 8) =
            make_uint4(kv4_value2(h[0], sv), kv4_value2(h[1], sv), kv4_value2(h[2], sv), kv4_value2(h[3], sv));
    }
    const int64_t slot = p.slots[row];
    if (slot < 0) return;
    if (slot >= (int64_t)p.slab.num_pages * p.slab.ps) { report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_KV4_PAGE); return; }
    const int64_t page = slot / p.slab.ps;
    const int in = (int)(slot - page * p.slab.ps), sl = in & 15;
    char* blk = p.slab.pool_l + (size_t)t * p.slab.tstride + ((page * nkv + head) * (p.slab.ps / 16) + in / 16) * kv4_block(DH);
    if (is_v) {
        blk += kv4_codes(DH) + kv4_scales(DH);
        *reinterpret_cast<uint16_t*>(blk + kv4_v_half(DH, sl, group, 2 * q)) = (uint16_t)code;
        *reinterpret_cast<uint16_t*>(blk + kv4_v_half(DH, sl, group, 2 * q + 1)) = (uint16_t)(code >> 16);
        if (q == 0) blk[kv4_codes(DH) + kv4_v_scale(DH, sl, group)] = (char)byte;
    } else {
        *reinterpret_cast<uint32_t*>(blk + kv4_k_word(DH, sl, group, q)) = code;
        if (q == 0) blk[kv4_codes(DH) + kv4_k_scale(DH, sl, group)] = (char)byte;
    }
}

template <int DH>
__global__ void __launch_bounds__(kThreads) k_kv4_read(const Kv4ReadP p, const int per) {
    constexpr int NG = DH / 32;
    __shared__ long long pre[kThreads + 1];
    grid_dep_wait();
    grid_dep_launch();
    const int lane = threadIdx.x & 31, nkv = p.slab.nkv, ps = p.slab.ps;
    bool bad = false;
    kv4_scan(p.B, per, pre, [&](int b) {
        const int n = p.kvlen[b];
        if (n < 0 || n > (int64_t)p.maxp * ps || n > (int64_t)p.omaxp * p.ops) { bad = true; return 0; }
        return (n + 15) >> 4;
    });
    if (__syncthreads_or(bad)) { if (bad) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_KV4_LEN); return; }
    // units: (track, 16-token block of the call, head), heads fastest; a warp has a run of them
    const long long blocks = pre[kThreads], units = blocks * nkv * p.T;
    const long long warps = (long long)gridDim.x * (kThreads / 32), w = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    long long u = units * w / warps;
    const long long end = units * (w + 1) / warps;
    if (u >= end) return;
    int t = (int)(u / (blocks * nkv)), head = (int)(u % nkv);
    long long blk = u / nkv - (long long)t * blocks;
    int b = 0, n = 0, at = 0;                              // sequence, its keys, its block
    auto seek = [&]() {
        const int i = kv4_find(pre, kThreads, blk);
        long long rest = blk - pre[i];
        for (b = i * per;; ++b) {
            n = p.kvlen[b];
            const int have = (n + 15) >> 4;
            if (rest < have) break;
            rest -= have;
        }
        at = (int)rest;
    };
    seek();
    for (; u < end; ++u) {
        const int page = p.bt[(size_t)b * p.maxp + at * 16 / ps];
        // lane l < 16: where token l of the block goes (elements from the track's slab, K; -1: nowhere)
        int64_t to = -1;
        if (lane < 16 && at * 16 + lane < n) {
            const int pos = at * 16 + lane, opage = p.obt[(size_t)b * p.omaxp + pos / p.ops];
            if (opage < 0 || opage >= p.opages) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_KV4_PAGE);
            else to = (((int64_t)opage * 2 * nkv + head) * p.ops + pos % p.ops) * DH;
        }
        if (page < 0 || page >= p.slab.num_pages) {
            if (lane == 0) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_KV4_PAGE);
        } else {
            const char* src = p.slab.pool_l + (size_t)t * p.slab.tstride + (((int64_t)page * nkv + head) * (ps / 16) + at * 16 % ps / 16) * kv4_block(DH);
            __nv_bfloat16* out = p.out_l + (size_t)t * p.out_tstride;
            const int64_t v_off = (int64_t)nkv * p.ops * DH;
            const char* ksc = src + kv4_codes(DH);
            const char* vcodes = ksc + kv4_scales(DH);
            const char* vsc = vcodes + kv4_codes(DH);
            const int g = lane >> 2, q = lane & 3;
#pragma unroll
            for (int i = 0; i < 2; ++i) {                  // K: tokens 2 g and 2 g + 1
                const int tok = 2 * g + i;
                const int64_t dst = __shfl_sync(0xffffffffu, to, tok);
                uint32_t c[NG];
#pragma unroll
                for (int j = 0; j < NG; ++j) c[j] = *reinterpret_cast<const uint32_t*>(src + kv4_k_word(DH, tok, j, q));
                if (dst < 0) continue;
#pragma unroll
                for (int j = 0; j < NG; ++j) {
                    const float s = kv4_scale((uint8_t)ksc[kv4_k_scale(DH, tok, j)]);
                    uint32_t h[4];
                    kv4_codes8(c[j], h);
                    *reinterpret_cast<uint4*>(out + dst + 32 * j + 8 * q) = make_uint4(kv4_value2(h[0], s), kv4_value2(h[1], s), kv4_value2(h[2], s), kv4_value2(h[3], s));
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {                  // V: tokens 4 q .. 4 q + 3
                const int tok = 4 * q + i;
                const int64_t dst = __shfl_sync(0xffffffffu, to, tok);
                uint32_t c[NG / 2];
#pragma unroll
                for (int j = 0; j < NG / 2; ++j) c[j] = *reinterpret_cast<const uint32_t*>(vcodes + kv4_v_half(DH, tok, 2 * j, g));
                if (dst < 0) continue;
#pragma unroll
                for (int j = 0; j < NG; ++j) {
                    const float s = kv4_scale((uint8_t)vsc[kv4_v_scale(DH, tok, j)]);
                    uint32_t h[2];
                    kv4_codes4(j & 1 ? c[j / 2] >> 16 : c[j / 2], h);
                    *reinterpret_cast<uint2*>(out + dst + v_off + 32 * j + 4 * g) = make_uint2(kv4_value2(h[0], s), kv4_value2(h[1], s));
                }
            }
        }
        if (++head == nkv) {
            head = 0;
            ++at; ++blk;
            if (at * 16 >= n && u + 1 < end) {
                if (blk == blocks) { blk = 0; ++t; }
                seek();
            }
        }
    }
}

int sm_count() {
    static int sms_[kMaxDevices] = {};
    int& sms = sms_[current_device()];
    if (!sms && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, current_device()) != cudaSuccess) sms = 148;
    return sms;
}

}  // namespace

pt_status launch_kv4_write(const Kv4WriteP& p, int dh, cudaStream_t st) {
    const int64_t blocks = ((int64_t)p.M * 2 * p.slab.nkv * (dh / 8) + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffff || p.T > 65535) { set_error("too many rows or tracks for one call"); return PT_ERR_UNSUPPORTED; }
    const cudaError_t e = launch_dependent(dh == 64 ? k_kv4_write<64> : k_kv4_write<128>, dim3((unsigned)blocks, p.T), dim3(kThreads), (size_t)0, st, p);
    if (e != cudaSuccess) { set_error("k_kv4_write launch: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return PT_OK;
}

pt_status launch_kv4_read(const Kv4ReadP& p, int dh, cudaStream_t st) {
    const int64_t most = ((int64_t)p.T * p.B * (((int64_t)p.maxp * p.slab.ps + 15) / 16) * p.slab.nkv + kThreads / 32 - 1) / (kThreads / 32);
    const int blocks = (int)std::min<int64_t>(most, (int64_t)sm_count() * 8);
    const cudaError_t e = launch_dependent(dh == 64 ? k_kv4_read<64> : k_kv4_read<128>, dim3(blocks), dim3(kThreads), (size_t)0, st, p, (p.B + kThreads - 1) / kThreads);
    if (e != cudaSuccess) { set_error("k_kv4_read launch: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return PT_OK;
}

static Kv4Slab slab_of(const Call& k, int layer) {
    const pt_kv_cache* c = k.c;
    const pt_config& g = k.m->cfg;
    return {c->pool + (size_t)layer * c->slab_elems, (int64_t)g.L * c->slab_elems, g.kv_heads, c->ps, c->num_pages};
}

pt_status launch_kv4_write_call(Call& k, int layer) {
    const pt_model* m = k.m;
    const pt_config& g = m->cfg;
    Kv4WriteP p{};
    p.k = (const __nv_bfloat16*)k.w.kv_stage; p.v = p.k + (int64_t)m->KVD * k.M;      // [T][K|V][kv_head][M][dh]
    p.tstride = (int64_t)2 * m->KVD * k.M; p.head_stride = (int64_t)k.M * m->dh; p.row_stride = m->dh;
    p.slab = slab_of(k, layer);
    p.slots = k.w.meta.row_kvoff; p.T = g.T; p.M = k.M; p.status = m->status();
    return launch_kv4_write(p, m->dh, k.st);
}

pt_status launch_kv4_read_call(Call& k, int layer) {
    const pt_model* m = k.m;
    Kv4ReadP p{};
    p.slab = slab_of(k, layer);
    p.bt = k.w.meta.bt; p.maxp = k.w.meta.maxp; p.kvlen = k.w.meta.kvlen;
    p.out_l = (__nv_bfloat16*)k.w.attn_kv; p.out_tstride = (int64_t)k.w.meta.attn_pages * 2 * m->KVD * 16;
    p.obt = k.w.meta.bt_attn; p.omaxp = k.w.meta.maxp_attn; p.ops = 16; p.opages = k.w.meta.attn_pages;
    p.T = m->cfg.T; p.B = k.B; p.status = m->status();
    return launch_kv4_read(p, m->dh, k.st);
}

pt_status launch_kv4_attn_call(Call& k, const __nv_bfloat16* q, int layer, __nv_bfloat16* o) {
    const pt_model* m = k.m;
    Kv4AttnP p{};
    p.q = q; p.o = o; p.slab = slab_of(k, layer);
    p.bt = k.w.meta.bt; p.maxp = k.w.meta.maxp; p.qlen = k.decode ? nullptr : k.w.meta.qlen; p.kvlen = k.w.meta.kvlen;
    p.T = m->cfg.T; p.B = k.B; p.M = k.M; p.nq = m->cfg.heads;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)m->dh);
    p.status = m->status();
    return launch_kv4_attn(p, m->dh, k.w.attn4, k.st);
}

// The attention from the codes reads a sequence's keys once for every 24 (token, head) rows; the other way writes the bf16 copy
// and reads it, at the cost of about three such passes.
bool kv4_direct(const int32_t* lens, const int32_t* n_new, int B, int G) {
    double passes = 0, once = 0;
    for (int b = 0; b < B; ++b) {
        passes += (double)lens[b] * (((int64_t)n_new[b] * G + 23) / 24);
        once += lens[b];
    }
    return passes <= 3 * once;
}

}  // namespace pt

#include "pt_kernels.h"

using namespace pt;

static pt_status check_shape(const void* pool_l, int64_t stride, int32_t T, int32_t nkv, int32_t dh, int32_t ps, int32_t num_pages) {
    if (T < 1 || nkv < 1 || num_pages < 1 || stride < 0 || nkv > 65535) { set_error("bad sizes"); return PT_ERR_INVALID_ARG; }
    if (dh != 64 && dh != 128) { set_error("an E2M1 cache needs head_dim 64 or 128"); return PT_ERR_UNSUPPORTED; }
    if (ps < 16 || ps > 64 || ps % 16) { set_error("an E2M1 cache needs pages of a multiple of 16 tokens, 64 at most"); return PT_ERR_UNSUPPORTED; }
    if ((uintptr_t)pool_l % 16 || stride % 16) { set_error("the pool must be 16-byte aligned, its track stride a multiple of 16 bytes"); return PT_ERR_MISALIGNED; }
    return PT_OK;
}
static bool table_too_long(int32_t maxp, int32_t ps) { return (int64_t)maxp * ps > 0x7fffffff - 127; }   // positions are rounded up to tiles in 32 bits

extern "C" pt_status pt_kernel_kv_write_e2m1(const void* k, const void* v, int64_t track_stride, int64_t row_stride, int32_t T, int32_t M,
                                             int32_t nkv, int32_t dh, int32_t ps, int32_t num_pages, void* pool_l, int64_t pool_track_stride,
                                             const int64_t* slots, void* k_out, void* v_out, void* status, void* stream) {
    if (!k || !v || !pool_l || !slots || !status || !k_out != !v_out) { set_error("null argument (k_out and v_out come together)"); return PT_ERR_INVALID_ARG; }
    if (M < 1 || M > (1 << 30) || track_stride < 0 || row_stride < 0) { set_error("bad sizes"); return PT_ERR_INVALID_ARG; }
    pt_status s = check_shape(pool_l, pool_track_stride, T, nkv, dh, ps, num_pages);
    if (s != PT_OK) return s;
    if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)k_out | (uintptr_t)v_out) % 16 || track_stride % 8 || row_stride % 8) {
        set_error("k, v, k_out and v_out must be 16-byte aligned, strides a multiple of 8 elements"); return PT_ERR_MISALIGNED;
    }
    if ((uintptr_t)slots % 8 || (uintptr_t)status % 4) { set_error("slots must be 8-byte, status 4-byte aligned"); return PT_ERR_MISALIGNED; }
    Kv4WriteP p{};
    p.k = (const __nv_bfloat16*)k; p.v = (const __nv_bfloat16*)v; p.tstride = track_stride; p.row_stride = row_stride; p.head_stride = dh;
    p.slab = {(char*)pool_l, pool_track_stride, nkv, ps, num_pages};
    p.slots = slots; p.k_out = (__nv_bfloat16*)k_out; p.v_out = (__nv_bfloat16*)v_out; p.T = T; p.M = M; p.status = (int*)status;
    return launch_kv4_write(p, dh, (cudaStream_t)stream);
}

extern "C" pt_status pt_kernel_kv_read_e2m1(const void* pool_l, int64_t pool_track_stride, const int32_t* block_table, int32_t maxp, const int32_t* kv_len,
                                            int32_t T, int32_t B, int32_t nkv, int32_t dh, int32_t ps, int32_t num_pages,
                                            void* out_l, int64_t out_track_stride, const int32_t* out_table, int32_t out_maxp, int32_t out_ps, int32_t out_pages,
                                            void* status, void* stream) {
    if (!pool_l || !block_table || !kv_len || !out_l || !out_table || !status) { set_error("null argument"); return PT_ERR_INVALID_ARG; }
    if (B < 1 || maxp < 1 || out_maxp < 1 || out_pages < 1 || out_track_stride < 0) { set_error("bad sizes"); return PT_ERR_INVALID_ARG; }
    if (out_ps < 8 || out_ps > 64 || out_ps % 8) { set_error("out_ps must be a multiple of 8 in [8, 64]"); return PT_ERR_INVALID_ARG; }
    pt_status s = check_shape(pool_l, pool_track_stride, T, nkv, dh, ps, num_pages);
    if (s != PT_OK) return s;
    if (table_too_long(maxp, ps) || table_too_long(out_maxp, out_ps)) { set_error("a block table of more than 2^31 - 128 keys"); return PT_ERR_UNSUPPORTED; }
    if ((uintptr_t)out_l % 16 || out_track_stride % 8) { set_error("out must be 16-byte aligned, its track stride a multiple of 8 elements"); return PT_ERR_MISALIGNED; }
    if (((uintptr_t)block_table | (uintptr_t)kv_len | (uintptr_t)out_table | (uintptr_t)status) % 4) { set_error("tables, kv_len and status must be 4-byte aligned"); return PT_ERR_MISALIGNED; }
    Kv4ReadP p{};
    p.slab = {(char*)pool_l, pool_track_stride, nkv, ps, num_pages};
    p.bt = block_table; p.maxp = maxp; p.kvlen = kv_len; p.out_l = (__nv_bfloat16*)out_l; p.out_tstride = out_track_stride;
    p.obt = out_table; p.omaxp = out_maxp; p.ops = out_ps; p.opages = out_pages; p.T = T; p.B = B; p.status = (int*)status;
    return launch_kv4_read(p, dh, (cudaStream_t)stream);
}

extern "C" pt_status pt_kernel_attn_e2m1_scratch_bytes(int32_t T, int32_t nq, int32_t nkv, int32_t dh, size_t* bytes) {
    if (!bytes || T < 1 || nq < 1 || nkv < 1 || (dh != 64 && dh != 128)) { set_error("bad argument"); return PT_ERR_INVALID_ARG; }
    *bytes = kv4_attn_scratch_bytes(dh);
    return PT_OK;
}

extern "C" pt_status pt_kernel_attn_e2m1(const void* q, const void* pool_l, int64_t pool_track_stride, const int32_t* block_table, int32_t maxp,
                                         const int32_t* q_len, const int32_t* kv_len, int32_t T, int32_t B, int32_t M, int32_t nq, int32_t nkv, int32_t dh,
                                         int32_t ps, int32_t num_pages, void* out, void* scratch, size_t scratch_bytes, void* status, void* stream) {
    if (!q || !pool_l || !block_table || !kv_len || !out || !scratch || !status) { set_error("null argument"); return PT_ERR_INVALID_ARG; }
    if (B < 1 || M < 1 || M > (1 << 26) || nq < 1 || nkv < 1 || nq % nkv || maxp < 1 || (!q_len && M != B)) { set_error("bad sizes"); return PT_ERR_INVALID_ARG; }
    pt_status s = check_shape(pool_l, pool_track_stride, T, nkv, dh, ps, num_pages);
    if (s != PT_OK) return s;
    if (nq / nkv > 8) { set_error("more than 8 query heads per KV head"); return PT_ERR_UNSUPPORTED; }
    if (table_too_long(maxp, ps)) { set_error("a block table of more than 2^31 - 128 keys"); return PT_ERR_UNSUPPORTED; }
    if (((uintptr_t)q | (uintptr_t)out) % 16 || (uintptr_t)scratch % 256) { set_error("q and out must be 16-byte, scratch 256-byte aligned"); return PT_ERR_MISALIGNED; }
    if (((uintptr_t)block_table | (uintptr_t)q_len | (uintptr_t)kv_len | (uintptr_t)status) % 4) { set_error("block_table, q_len, kv_len and status must be 4-byte aligned"); return PT_ERR_MISALIGNED; }
    const size_t need = kv4_attn_scratch_bytes(dh);
    if (scratch_bytes < need) { set_error("scratch: %zu < %zu bytes", scratch_bytes, need); return PT_ERR_BUFFER_TOO_SMALL; }
    Kv4AttnP p{};
    p.q = (const __nv_bfloat16*)q; p.o = (__nv_bfloat16*)out;
    p.slab = {(char*)pool_l, pool_track_stride, nkv, ps, num_pages};
    p.bt = block_table; p.maxp = maxp; p.qlen = q_len; p.kvlen = kv_len; p.T = T; p.B = B; p.M = M; p.nq = nq;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)dh);
    p.status = (int*)status;
    return launch_kv4_attn(p, dh, scratch, (cudaStream_t)stream);
}
