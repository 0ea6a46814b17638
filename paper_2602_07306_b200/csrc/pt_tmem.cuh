// The wait for loads from tensor memory, for every kernel that makes them.
#pragma once

namespace pt {

// Keeps arithmetic on v behind the volatile statement before it.
template <int N>
__device__ __forceinline__ void tm_pin(float* v) {
#pragma unroll
    for (int i = 0; i < N; i += 8)
        asm volatile("" : "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]), "+f"(v[i + 6]), "+f"(v[i + 7]) :: "memory");
}
// Waits for this thread's tensor-memory loads, which write the N registers of v (and of w).  To the compiler a load has written
// them where it stands: naming them behind the wait keeps arithmetic on them from being moved in front of it.
template <int N>
__device__ __forceinline__ void tm_wait_ld(float* v) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    tm_pin<N>(v);
}
template <int N>
__device__ __forceinline__ void tm_wait_ld(float* v, float* w) {
    tm_wait_ld<N>(v);
    tm_pin<N>(w);
}

}  // namespace pt
