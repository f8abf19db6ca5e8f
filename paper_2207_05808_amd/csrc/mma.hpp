// Matrix-core building blocks shared by the output layer's kernels
// (w4_matmul.hip, linear_xent.hip): bf16 products with 32-bit sums, and exact
// splits of wider types into bf16 parts.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mdn {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Element types of the matrices (MADDNESS_F32 / BF16 / F16).
struct Bf16 { uint16_t bits; };
struct F16 { uint16_t bits; };

// Any value of these types is the exact sum of kParts bf16 numbers (8, 11 and
// 24 significant bits, 8 a part), so a product with bf16 weights is exact in
// the 32-bit sum for each part.
template <class T> struct Parts;
template <> struct Parts<Bf16> { static constexpr int n = 1; };
template <> struct Parts<F16> { static constexpr int n = 2; };
template <> struct Parts<float> { static constexpr int n = 3; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(Bf16 v) { return __uint_as_float((uint32_t)v.bits << 16); }
__device__ __forceinline__ float to_float(F16 v) { return (float)__builtin_bit_cast(_Float16, v.bits); }
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ Bf16 from_float<Bf16>(float v) { return {__builtin_bit_cast(uint16_t, (__bf16)v)}; }
template <> __device__ __forceinline__ F16 from_float<F16>(float v) { return {__builtin_bit_cast(uint16_t, (_Float16)v)}; }

// Two values as their bf16 parts, out[p] part p (0 the leading one) of both:
// each part is what the ones before leave, rounded to 8 bits, so three hold 24
// bits exactly and the parts fall by 2^-8.  A part is kept below the largest
// bf16 but for the last, which so carries an infinity or a NaN alone.
template <int P>
__device__ __forceinline__ void split2(float a, float b, uint32_t (&out)[P]) {
  constexpr float kMost = 3.38953138925153547590e38f;   // largest bf16
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const bool last = p == P - 1;
    const f32x2 v = last ? (f32x2){a, b} : (f32x2){__builtin_amdgcn_fmed3f(a, -kMost, kMost), __builtin_amdgcn_fmed3f(b, -kMost, kMost)};
    out[p] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    if (!last) {
      a -= __uint_as_float(out[p] << 16);
      b -= __uint_as_float(out[p] & 0xffff0000u);
    }
  }
}

// 16 bytes at any element alignment (the hardware takes unaligned addresses)
struct __attribute__((packed, aligned(2))) Bytes16 { uint32_t w[4]; };
__device__ __forceinline__ u32x4 load16(const void* p) {
  const Bytes16 v = *static_cast<const Bytes16*>(p);
  return (u32x4){v.w[0], v.w[1], v.w[2], v.w[3]};
}

__device__ __forceinline__ void store16(void* p, u32x4 v) { *static_cast<Bytes16*>(p) = Bytes16{{v[0], v[1], v[2], v[3]}}; }

// LDS by byte address
template <class V> using LdsPtr = __attribute__((address_space(3))) V*;
template <class V> __device__ __forceinline__ LdsPtr<V> lds_at(uint32_t byte) { return (LdsPtr<V>)(uintptr_t)byte; }
__device__ __forceinline__ uint32_t lds_address(const void* p) {   // (uniform)
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(LdsPtr<const char>)p);
}

// A barrier that orders LDS only: global loads stay in flight across it.
__device__ __forceinline__ void lds_only_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

}  // namespace mdn
