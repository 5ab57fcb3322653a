// Device helpers of the serving operators (ftprompt.hip, ftcache.hip), gfx950 / CDNA4 only.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ftserve {

typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint16_t ushort2v __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef short short2v __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f;
constexpr int64_t MOST_GROUPS = (1ll << 24) - 1;      // workgroups of 256 threads: a launch has fewer than 2^32 threads in a dimension

__device__ __forceinline__ float as_f(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_u(float f) { return __builtin_bit_cast(uint32_t, f); }
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }

// two values of a 16-bit type in a word (BF: bf16, else fp16), and back; rounded to nearest, ties to even
template <bool BF> __device__ __forceinline__ uint32_t pack2(float a, float b) {
  const float2v x = {a, b};
  if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf2v));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, half2v));
}
template <bool BF> __device__ __forceinline__ float low_of(uint32_t u) {
  if constexpr (BF) return as_f(u << 16);
  else return (float)__builtin_bit_cast(half2v, u)[0];
}
template <bool BF> __device__ __forceinline__ float high_of(uint32_t u) {
  if constexpr (BF) return as_f(u & 0xFFFF0000u);
  else return (float)__builtin_bit_cast(half2v, u)[1];
}
template <bool BF> __device__ __forceinline__ uint32_t largest_finite_plus_one() { return BF ? 0x7F80u : 0x7C00u; }

// The sequence that packed unit `x` belongs to: the last b with at(b) <= x, where at does not fall and at(0) <= x.
// 64 probes a step, one per lane: one step for 64 sequences, two for 4096.
template <class F> __device__ __forceinline__ int sequence_of(int batch, int64_t x, F at) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = batch;
  while (n > 1) {
    const int step = (n + 63) >> 6, i = lane * step;
    const bool below = i < n && at(lo + i) <= x;
    const int last = __popcll(__ballot(below)) - 1, first = last < 0 ? 0 : last * step;
    lo += first;
    n = n - first < step ? n - first : step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ int clamped(int x, int hi) { return x < 0 ? 0 : x > hi ? hi : x; }

}  // namespace ftserve
