// Two binary32 values in a 64-bit register pair: sums and products of both in one instruction, rounded as two would be.
#pragma once
#include <cstdint>

namespace cerar {
namespace packed {

__device__ __forceinline__ uint64_t two_of(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void parts(uint64_t r, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(r)); }
__device__ __forceinline__ uint64_t all(float x) { return two_of(x, x); }
__device__ __forceinline__ uint64_t mul2(uint64_t x, uint64_t y) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t x, uint64_t y) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ uint64_t mad2(uint64_t x, uint64_t y, uint64_t z) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
    return r;
}
__device__ __forceinline__ uint64_t swapped(uint64_t x) { return x >> 32 | x << 32; }
// two neighbouring bfloat16 values
__device__ __forceinline__ uint64_t of_bf16(uint32_t q) { return (uint64_t)(q & 0xFFFF0000u) << 32 | (q << 16); }

}  // namespace packed
}  // namespace cerar
