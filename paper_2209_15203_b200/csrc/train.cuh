// Shared device-side pieces of the training operators (layer norm, cross entropy, AdamW):
// element types, conversions, warp and group reductions.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace tk {

typedef unsigned int u32;
typedef unsigned long long u64;
typedef __nv_bfloat16 bf16;

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float v) { return __float2bfloat16_rn(v); }

// One value of a tensor whose type (fp32 or bf16) is known at run time only; used for vectors of
// `dim` values that stay in cache, where a uniform branch costs nothing that can be measured.
__device__ __forceinline__ float load_any(const void* p, int64_t i, bool is_bf16) {
    return is_bf16 ? to_float(((const bf16*)p)[i]) : ((const float*)p)[i];
}
__device__ __forceinline__ void store_any(void* p, int64_t i, float v, bool is_bf16) {
    if (is_bf16)
        ((bf16*)p)[i] = from_float<bf16>(v);
    else
        ((float*)p)[i] = v;
}

// First thing of a kernel that is launched with programmatic stream serialization: its launch overlaps the end of the kernel
// before, which it waits for here.  (Letting its CTAs start while the one before still runs, by griddepcontrol.launch_dependents,
// made the chain of the loss slower: 40 us instead of 22 for 61 tokens x 50257 x 768; without any overlap 27 us.)
__device__ __forceinline__ void wait_for_predecessor() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Two fp32 values per instruction; each operation rounds as its scalar form does.
struct Pair {
    u64 v;
};
__device__ __forceinline__ Pair pair(float a, float b) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ Pair both(float a) { return pair(a, a); }
__device__ __forceinline__ void split(Pair p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.v)); }
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

}  // namespace tk
