// Device helpers of the 4-bit cache format that its kernels share.
#pragma once
#include "pt_kv4.h"

namespace pt {

// Order of a block of 16 tokens (pt.h): places in bytes from the start of the K codes, of the V codes, of the scales.
__device__ __forceinline__ int kv4_k_word(int dh, int slot, int group, int q) { return ((slot & 1) * 8 + (slot >> 1)) * (dh / 2) + q * (dh / 8) + group * 4; }
__device__ __forceinline__ int kv4_v_half(int dh, int slot, int group, int g) {
    const int q = slot >> 2, i = slot & 3;
    return (dh == 128 ? (i >> 1) * 512 + (4 * g + q) * 16 + (i & 1) * 8 : (4 * g + q) * 16 + i * 4) + group * 2;
}
__device__ __forceinline__ int kv4_k_scale(int dh, int slot, int group) { return slot * (dh / 32) + group; }
__device__ __forceinline__ int kv4_v_scale(int dh, int slot, int group) { return (slot >> 2) * (dh / 8) + group * 4 + (slot & 3); }

// A scale byte is the upper half of a positive fp16 without its sign: 5 exponent bits, 3 mantissa bits.
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __half2float(__ushort_as_half((unsigned short)(byte << 7))); }
// eight codes (low four bits first) -> four f16 pairs
__device__ __forceinline__ void kv4_codes8(uint32_t w, uint32_t* h) {
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
        " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}" : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// four codes
__device__ __forceinline__ void kv4_codes4(uint32_t w, uint32_t* h) {
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %2;\n cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n}" : "=r"(h[0]), "=r"(h[1]) : "r"(w));
}
__device__ __forceinline__ uint32_t kv4_bf16(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// an f16 pair of code values times a scale, as a bf16 pair: exact (two significant bits times four)
__device__ __forceinline__ uint32_t kv4_value2(uint32_t h, float s) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    return kv4_bf16(f.x * s, f.y * s);
}

// Running sums over the lanes of a warp, the lane's own included.
template <typename N> __device__ __forceinline__ N kv4_scan(N x) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const N y = __shfl_up_sync(0xffffffffu, x, o);
        if ((int)(threadIdx.x & 31) >= o) x += y;
    }
    return x;
}
// a / b for positive numbers: in 32 bits where they fit
__device__ __forceinline__ long long kv4_quotient(long long a, long long b) {
    return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}

}  // namespace pt
