// The 4-bit storage format of the KV cache (pt_kv_dtype PT_KV_E2M1): new tokens' K and V into its pages, and sequences back out.
//   k_kv4_write   a thread has sixteen consecutive values of a vector, two threads a group of 32
//   k_kv4_read    a warp has one head's K and V of 16 tokens, in the order in which they lie: 16 bytes a lane and load
// Both are bound by the bytes they move.  Measured (a plain copy: 6.4 TB/s): 8192 tokens of 8 tracks and 8 KV heads of 128 with their
// values out 99 us (608 MB, 6.1 TB/s; 105-107 for passes in a row on warmer boxes; with eight values a thread and codes written where they fell 184), contexts of 28 sequences of
// 0.8-4k keys read back 105 us (638 MB, 6.1 TB/s).
#include <algorithm>
#include <type_traits>

#include "pt_kv4.cuh"
#include "pt_tc.h"
#include "pt_ptx.cuh"

namespace pt {

namespace {

constexpr int kThreads = 256;

// The code of v / s for the group's scale s, given r = 1 / s rounded: ties between codes have to be met exactly.  v has 8
// significant bits and a tie times s has 7, so v / s is either a tie (0.25 .. 5) or at least 2^-8 of it away; v * r is off by
// 2^-22 of it, and a sum with 1.5 * 2^10 rounds it to multiples of 2^-13, which returns to the tie.  The sign stays, of zeros too.
__device__ __forceinline__ float kv4_divided(float v, float r) {
    constexpr float kRound = 1536.f;
    return __uint_as_float(__float_as_uint(fmaf(v, r, kRound) - kRound) | (__float_as_uint(v) & 0x80000000u));
}
__device__ __forceinline__ uint32_t kv4_encode8(const float* y) {
    uint32_t w;
    asm("{\n .reg .b8 a, b, c, d;\n cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n mov.b32 %0, {a, b, c, d};\n}"
        : "=r"(w) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
    return w;
}

// Sixteen values of a vector, half of a group (its other half is the lane's neighbour's): their codes in two words (the
// lowest value's lowest), and the byte of the group's scale.
__device__ __forceinline__ uint2 kv4_encode(const uint4* raw, uint32_t& byte) {
    const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
    // magnitudes as whole numbers: a NaN is above infinity, which is above the rest
    uint32_t top = 0;
#pragma unroll
    for (int a = 0; a < 8; ++a) top = __vmaxu2(top, w[a] & 0x7fff7fffu);
    top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top & 0xffffu, top >> 16);
    const bool bad = top >= 0x7f80u;
    const float amax = bad ? 0.f : __uint_as_float(top << 16);
    // amax / 6 cut to 4 significant bits, or the next number where that is too small (the product is exact)
    byte = (uint32_t)__half_as_ushort(__float2half_rz(fminf(amax * (1.0f / 6.0f), 61440.f))) >> 7;
    if (byte < 247 && 6.0f * kv4_scale(byte) < amax) ++byte;
    const float s = kv4_scale(byte);
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));           // off by 2^-23: see kv4_divided
    if (byte == 0) r = 0.f;
    float y[16];
#pragma unroll
    for (int a = 0; a < 8; ++a) {
        y[2 * a] = kv4_divided(__uint_as_float(w[a] << 16), r);
        y[2 * a + 1] = kv4_divided(__uint_as_float(w[a] & 0xffff0000u), r);
    }
    if (bad) { byte = 255; return make_uint2(0u, 0u); }
    return make_uint2(kv4_encode8(y), kv4_encode8(y + 8));
}

// A block has 16 rows of one track and head.  Tokens that follow one another lie side by side in a block of the cache, but
// each in pieces of 8 bytes (V) and 16 (K): the rows' codes meet in shared memory and go out piece by piece in the order of
// the cache, as if row 0's slot were followed by the others.  Where it is not, the same pieces go to the same places less
// well together.
template <int DH>
__global__ void __launch_bounds__(DH) k_kv4_write(const Kv4WriteP p) {
    constexpr int PER = DH / 16, THREADS = DH, NG = DH / 32;       // threads of a vector; 16 vectors
    constexpr int KP = DH / 8, VP = DH / 16;                       // bytes of a piece
    __shared__ __align__(16) uint8_t img[2][16][DH / 2];           // K, V: a token's pieces in order
    __shared__ __align__(16) uint8_t scales[2][16][NG];
    __shared__ int64_t where[16];                                  // byte of the token's cache block in the track's slab, -1: nowhere
    __shared__ int slot_in[16];                                    // its slot in that block
    grid_dep_wait();
    grid_dep_launch();
    const int tid = threadIdx.x, r = tid / PER, part = tid % PER, group = part >> 1, half = part & 1;
    const int head = blockIdx.y, t = blockIdx.z, nkv = p.slab.nkv;
    const int64_t row = (int64_t)blockIdx.x * 16 + r;
    const bool live = row < p.M;                                   // every lane takes part in the shuffles
    uint4 raw[2][2] = {};
    if (live) {
        const size_t at = (size_t)t * p.tstride + row * p.row_stride + head * p.head_stride + part * 16;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint4* src = reinterpret_cast<const uint4*>((x ? p.v : p.k) + at);
            raw[x][0] = src[0]; raw[x][1] = src[1];
        }
    }
    const size_t out_at = (((size_t)t * p.M + row) * nkv + head) * DH + part * 16;
    if (tid < 16) {
        const int64_t row_t = (int64_t)blockIdx.x * 16 + tid, slot = row_t < p.M ? p.slots[row_t] : -1;
        int64_t to = -1;
        int in = tid;
        if (slot >= (int64_t)p.slab.num_pages * p.slab.ps) {
            report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_KV4_PAGE);
        } else if (slot >= 0) {
            const int64_t page = slot / p.slab.ps;
            in = (int)(slot - page * p.slab.ps);
            to = ((page * nkv + head) * (p.slab.ps / 16) + in / 16) * kv4_block(DH);
        }
        where[tid] = to;
        slot_in[tid] = in & 15;
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        uint32_t byte;
        const uint2 code = kv4_encode(raw[x], byte);
        if (p.k_out && live) {
            const float s = kv4_scale(byte);
            uint4* val = reinterpret_cast<uint4*>((x ? p.v_out : p.k_out) + out_at);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t h[4];
                kv4_codes8(i ? code.y : code.x, h);
                val[i] = make_uint4(kv4_value2(h[0], s), kv4_value2(h[1], s), kv4_value2(h[2], s), kv4_value2(h[3], s));
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t c = i ? code.y : code.x;
            if (x == 0) {
                *reinterpret_cast<uint32_t*>(&img[0][r][(2 * half + i) * KP + group * 4]) = c;
            } else {
                *reinterpret_cast<uint16_t*>(&img[1][r][(4 * half + 2 * i) * VP + group * 2]) = (uint16_t)c;
                *reinterpret_cast<uint16_t*>(&img[1][r][(4 * half + 2 * i + 1) * VP + group * 2]) = (uint16_t)(c >> 16);
            }
        }
        if (half == 0) scales[x][r][group] = (uint8_t)byte;
    }
    __syncthreads();
    char* const slab = p.slab.pool_l + (size_t)t * p.slab.tstride;
    const int first = slot_in[0];
    auto row_of = [&](int s) { return (s - first) & 15; };         // the row that has slot s if they follow row 0
    for (int i = tid; i < 128 + 64 + 16 * NG + 16; i += THREADS) {
        if (i < 128) {                                             // V codes
            const int s = DH == 128 ? 4 * (i / 2 % 4) + 2 * (i / 64) + i % 2 : 4 * (i / 4 % 4) + i % 4, g = DH == 128 ? i / 8 % 8 : i / 16;
            const int w = row_of(s);
            if (where[w] < 0) continue;
            char* dst = slab + where[w] + kv4_codes(DH) + kv4_scales(DH) + kv4_v_half(DH, slot_in[w], 0, g);
            if constexpr (DH == 128) *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(&img[1][w][g * VP]);
            else *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(&img[1][w][g * VP]);
        } else if (i < 192) {                                      // K codes
            const int x = i - 128, at = x / 4, w = row_of(at % 8 * 2 + at / 8);
            if (where[w] < 0) continue;
            char* dst = slab + where[w] + kv4_k_word(DH, slot_in[w], 0, x % 4);
            if constexpr (DH == 128) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(&img[0][w][x % 4 * KP]);
            else *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(&img[0][w][x % 4 * KP]);
        } else if (i < 192 + 16 * NG) {                            // V scales, a byte each
            const int x = i - 192, s = x / (4 * NG) * 4 + x % 4, j = x / 4 % NG, w = row_of(s);
            if (where[w] < 0) continue;
            slab[where[w] + 2 * kv4_codes(DH) + kv4_scales(DH) + kv4_v_scale(DH, slot_in[w], j)] = (char)scales[1][w][j];
        } else {                                                   // K scales, a token's together
            const int w = row_of(i - 192 - 16 * NG);
            if (where[w] < 0) continue;
            char* dst = slab + where[w] + kv4_codes(DH) + kv4_k_scale(DH, slot_in[w], 0);
            if constexpr (DH == 128) *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(scales[0][w]);
            else *reinterpret_cast<uint16_t*>(dst) = *reinterpret_cast<const uint16_t*>(scales[0][w]);
        }
    }
}

template <int N> struct alignas(N * 4) Words { uint32_t w[N]; };

// A warp has a run of units (track, 16-token block of the call, head), heads fastest; it finds the start of its run by itself.
template <int DH>
__global__ void __launch_bounds__(kThreads) k_kv4_read(const Kv4ReadP p) {
    constexpr int NG = DH / 32;
    using Code = std::conditional_t<NG == 4, uint4, uint2>;        // a lane's codes of a token of K
    grid_dep_wait();
    grid_dep_launch();
    const int lane = threadIdx.x & 31, nkv = p.slab.nkv, ps = p.slab.ps, g = lane >> 2, q = lane & 3;
    const int per = (p.B + 31) / 32;
    bool bad = false;
    int mine = 0, n = 0;
    for (int b = lane * per; b < min(p.B, (lane + 1) * per); ++b) {
        n = p.kvlen[b];
        if (n < 0 || n > (int64_t)p.maxp * ps || n > (int64_t)p.omaxp * p.ops) { bad = true; break; }
        mine += (n + 15) >> 4;
    }
    if (__any_sync(0xffffffffu, bad)) { if (bad && blockIdx.x == 0) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_KV4_LEN); return; }
    const int up = kv4_scan(mine), blocks = __shfl_sync(0xffffffffu, up, 31);
    const long long per_track = (long long)blocks * nkv, units = per_track * p.T;
    const long long warps = (long long)gridDim.x * (kThreads / 32), w = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const long long share = kv4_quotient(units, warps), more = units - share * warps;
    long long left = share + (w < more);
    if (left == 0) return;
    const long long u = share * w + min(w, more);
    int t = (int)kv4_quotient(u, per_track);
    const long long in = u - t * per_track;
    int blk = (int)kv4_quotient(in, nkv), head = (int)(in - (long long)blk * nkv);
    int b, at;                                                     // sequence, its block
    {
        const int l = __popc(__ballot_sync(0xffffffffu, up <= blk));
        at = blk - __shfl_sync(0xffffffffu, up - mine, l);
        b = l * per;
        n = per > 1 ? p.kvlen[b] : __shfl_sync(0xffffffffu, n, l);
        while (at >= (n + 15) >> 4) { at -= (n + 15) >> 4; n = p.kvlen[++b]; }
    }
    // lane l < 16 has where token l of the block goes: elements from the track's slab (head 0, K); -1: nowhere
    int page;
    int64_t to;
    auto look = [&]() {
        page = p.bt[(size_t)b * p.maxp + at * 16 / ps];
        to = -1;
        if (lane < 16 && at * 16 + lane < n) {
            const int pos = at * 16 + lane, opage = p.obt[(size_t)b * p.omaxp + pos / p.ops];
            if ((uint32_t)opage >= (uint32_t)p.opages) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_KV4_PAGE);
            else to = ((int64_t)opage * 2 * nkv * p.ops + pos % p.ops) * DH;
        }
        if ((uint32_t)page >= (uint32_t)p.slab.num_pages) {
            if (lane == 0) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_KV4_PAGE);
            page = 0; to = -1;
        }
    };
    look();
    for (;;) {
        const char* src = p.slab.pool_l + (size_t)t * p.slab.tstride + (((int64_t)page * nkv + head) * (ps / 16) + at * 16 % ps / 16) * kv4_block(DH);
        const char* vsrc = src + kv4_codes(DH) + kv4_scales(DH);
        // K: tokens 2 g and 2 g + 1, V: tokens 4 q .. 4 q + 3; all loads first
        Words<NG> kc[2];
        Words<4> vc[NG / 2];                                       // dh 128: of two tokens each; dh 64: of four
        Words<NG / 2> ks;
        Words<NG> vs;
#pragma unroll
        for (int i = 0; i < 2; ++i) *reinterpret_cast<Code*>(&kc[i]) = __ldcs(reinterpret_cast<const Code*>(src + kv4_k_word(DH, 2 * g + i, 0, q)));
        if constexpr (NG == 4) {
            *reinterpret_cast<uint4*>(&vc[0]) = __ldcs(reinterpret_cast<const uint4*>(vsrc + lane * 16));
            *reinterpret_cast<uint4*>(&vc[1]) = __ldcs(reinterpret_cast<const uint4*>(vsrc + 512 + lane * 16));
            *reinterpret_cast<uint2*>(&ks) = *reinterpret_cast<const uint2*>(src + kv4_codes(DH) + g * 8);
            *reinterpret_cast<uint4*>(&vs) = *reinterpret_cast<const uint4*>(vsrc + kv4_codes(DH) + q * 16);
        } else {
            *reinterpret_cast<uint4*>(&vc[0]) = __ldcs(reinterpret_cast<const uint4*>(vsrc + lane * 16));
            ks.w[0] = *reinterpret_cast<const uint32_t*>(src + kv4_codes(DH) + g * 4);
            *reinterpret_cast<uint2*>(&vs) = *reinterpret_cast<const uint2*>(vsrc + kv4_codes(DH) + q * 8);
        }
        __nv_bfloat16* out = p.out_l + (size_t)t * p.out_tstride + (size_t)head * p.ops * DH;
        const int64_t v_off = (int64_t)nkv * p.ops * DH;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t dst = __shfl_sync(0xffffffffu, to, 2 * g + i);
            if (dst >= 0) {
#pragma unroll
                for (int j = 0; j < NG; ++j) {
                    const int x = i * NG + j;
                    const float s = kv4_scale((ks.w[x / 4] >> (x % 4 * 8)) & 0xffu);
                    uint32_t h[4];
                    kv4_codes8(kc[i].w[j], h);
                    *reinterpret_cast<uint4*>(out + dst + 32 * j + 8 * q) = make_uint4(kv4_value2(h[0], s), kv4_value2(h[1], s), kv4_value2(h[2], s), kv4_value2(h[3], s));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t dst = __shfl_sync(0xffffffffu, to, 4 * q + i);
            if (dst >= 0) {
#pragma unroll
                for (int j = 0; j < NG; ++j) {
                    const uint32_t c = NG == 4 ? vc[i / 2 % (NG / 2)].w[i % 2 * 2 + j / 2] : vc[0].w[i];
                    const float s = kv4_scale((vs.w[j] >> (8 * i)) & 0xffu);
                    uint32_t h[2];
                    kv4_codes4(j & 1 ? c >> 16 : c, h);
                    *reinterpret_cast<uint2*>(out + dst + v_off + 32 * j + 4 * g) = make_uint2(kv4_value2(h[0], s), kv4_value2(h[1], s));
                }
            }
        }
        if (--left == 0) break;
        if (++head == nkv) {
            head = 0;
            ++at;
            if (++blk == blocks) { blk = 0; ++t; b = -1; at = n = 0; }
            while (at * 16 >= n) { n = p.kvlen[++b]; at = 0; }
            look();
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
    const cudaError_t e = launch_dependent(dh == 64 ? k_kv4_write<64> : k_kv4_write<128>, dim3((p.M + 15) / 16, p.slab.nkv, p.T), dim3(dh), (size_t)0, st, p);
    if (e != cudaSuccess) { set_error("k_kv4_write launch: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return PT_OK;
}

pt_status launch_kv4_read(const Kv4ReadP& p, int dh, cudaStream_t st) {
    const double blocks_most = (double)p.B * ((double)p.maxp * p.slab.ps / 16 + 1);      // of one track: counted in 32 bits
    if (blocks_most > 2e9) { set_error("too many sequences or pages for one call"); return PT_ERR_UNSUPPORTED; }
    if (p.T > 1 && p.out_tstride < (int64_t)p.opages * 2 * p.slab.nkv * p.ops * dh) { set_error("the tracks of the output overlap"); return PT_ERR_INVALID_ARG; }
    // Short runs: warps that run side by side then read and write side by side.  (Four contexts of 9-16k keys, 8 tracks, 4 KV heads:
    // 195 us with a run for each of 64 warps an SM, 173 us with 512.)
    const double warps = std::min(blocks_most * p.T * p.slab.nkv, (double)sm_count() * 512);
    const int blocks = ((int)warps + kThreads / 32 - 1) / (kThreads / 32);
    const cudaError_t e = launch_dependent(dh == 64 ? k_kv4_read<64> : k_kv4_read<128>, dim3(blocks), dim3(kThreads), (size_t)0, st, p);
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
    p.T = m->cfg.T; p.B = k.B; p.M = k.M; p.nq = m->cfg.heads; p.tiles = k.direct;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)m->dh);
    p.status = m->status();
    return launch_kv4_attn(p, m->dh, k.w.attn4, k.st);
}

// The attention from the codes reads a sequence's keys once a pass of 8, 16 or 24 (token, head) rows, which takes a time of 1, 1.6 or
// 2 (four sequences of 20k keys, 4 tracks, 4 KV heads: 34, 54 and 67 us a pass beside a start of 10); the call has one of the three,
// the one that is best over all of its sequences.  The other way writes the bf16 copy and reads it: a time of 6, at 64 rows and a
// little more that of three passes of 24.
int kv4_plan(const int32_t* lens, const int32_t* n_new, int B, int G) {
    constexpr double kPass[3] = {1.0, 1.6, 2.0}, kCopy = 6.0;
    double passes[3] = {}, once = 0;
    for (int b = 0; b < B; ++b) {
        const int64_t eights = ((int64_t)n_new[b] * G + 7) / 8;
        for (int i = 0; i < 3; ++i) passes[i] += (double)lens[b] * (double)((eights + i) / (i + 1));
        once += lens[b];
    }
    int best = 0;
    for (int i = 1; i < 3; ++i)
        if (passes[i] * kPass[i] < passes[best] * kPass[best]) best = i;
    return passes[best] * kPass[best] <= kCopy * once ? best + 1 : 0;
}

}  // namespace pt

#include "pt_kernels.h"

using namespace pt;

static pt_status check_shape(const void* pool_l, int64_t stride, int32_t T, int32_t nkv, int32_t dh, int32_t ps, int32_t num_pages) {
    if (T < 1 || nkv < 1 || num_pages < 1 || stride < 0) { set_error("bad sizes"); return PT_ERR_INVALID_ARG; }
    if (T > 65535 || nkv > 65535 || (int64_t)T * nkv > 1 << 24) { set_error("more than 2^24 heads of all tracks, or 65535 tracks or heads"); return PT_ERR_UNSUPPORTED; }
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
    if (T > 1 && pool_track_stride < (int64_t)num_pages * nkv * (ps / 16) * kv4_block(dh)) { set_error("the pool's tracks overlap"); return PT_ERR_INVALID_ARG; }
    if (k_out) {
        const int64_t row = (int64_t)nkv * dh;
        const double in = ((double)(T - 1) * track_stride + (double)(M - 1) * row_stride + row) * 2, out = (double)T * M * row * 2;
        const bool alike = (M == 1 || row_stride == row) && (T == 1 || track_stride == M * row);
        for (const void* from : {k, v})
            for (const void* to : {(const void*)k_out, (const void*)v_out})
                if (kv4_meet(from, in, to, out) && !(from == to && alike)) { set_error("k_out and v_out are k and v, alike in their strides, or apart from them"); return PT_ERR_INVALID_ARG; }
        if (kv4_meet(k_out, out, v_out, out)) { set_error("k_out and v_out overlap"); return PT_ERR_INVALID_ARG; }
    }
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
    if (q == out) { set_error("out must not overlap q"); return PT_ERR_INVALID_ARG; }
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
    p.tiles = q_len ? kv4_mean_tiles((int64_t)M * (nq / nkv), B) : 1;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)dh);
    p.status = (int*)status;
    return launch_kv4_attn(p, dh, scratch, (cudaStream_t)stream);
}
