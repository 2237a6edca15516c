// What kernels with matrix instructions share: operands' types, the instruction for
// bf16 and float16, and 4-bit codes as its operands.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace hl {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <class T>
__device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (std::is_same<T, __bf16>::value)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                  0);
}

// Ends a row of matrix instructions: the instructions after it may write the
// operands of those before. On gfx950 a product has come out wrong now and then
// when the instruction right after it wrote one of its operand registers; the
// compiler places no wait states there, and five are enough.
__device__ inline void products_end() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 4");
  __builtin_amdgcn_sched_barrier(0);
}

// 16 + code as operands. The mask is in a scalar register and the exponents in a
// vector one, so that one instruction takes both.
template <class T>
struct Codes {
  static constexpr bool BF = std::is_same<T, __bf16>::value;
  static constexpr uint32_t LESS = BF ? 0xC1C0C1C0u : 0xCE00CE00u;  // two of -24: 16, and the 8 that a code has too much
  uint32_t mask, one;
  __device__ Codes() {
    mask = BF ? 0x00780078u : 0x03C003C0u, one = BF ? 0x41804180u : 0x4C004C00u;
    asm volatile("" : "+s"(mask), "+v"(one));
  }
  // of the codes at bit AT of two halves
  template <int AT>
  __device__ uint32_t pair(uint32_t w) const {
    constexpr int up = (BF ? 3 : 6) - AT;
    return ((up > 0 ? w << (up > 0 ? up : 0) : w >> (up > 0 ? 0 : -up)) & mask) | one;
  }
};

// f(0) .. f(N - 1), with the number known to the compiler.
template <int N, class F>
__device__ inline void each(F f) {
  if constexpr (N > 0) {
    each<N - 1>(f);
    f(std::integral_constant<int, N - 1>());
  }
}

}  // namespace hl
