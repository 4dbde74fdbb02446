// What the operators around the attention share: host checks, loads and stores of eight elements at any alignment, sums over lanes.
#pragma once
#include <cstring>

#include "device_common.hpp"

namespace chunk_attn {

// Keeps the error's text for chunk_attn_strerror; returns CHUNK_ATTN_HIP_ERROR (api.hip).
int report_hip(hipError_t e, const char* what);

// By the bits: the compiler is told that there are no NaN (-fno-honor-nans), which would make a comparison of one anything.
inline bool finite_number(double x) {
  uint64_t b;
  std::memcpy(&b, &x, 8);
  return (b >> 52 & 0x7ff) != 0x7ff;
}
inline bool finite_number(float x) {
  uint32_t b;
  std::memcpy(&b, &x, 4);
  return (b >> 23 & 0xff) != 0xff;
}

// Eight elements from any address that suits their type: the hardware takes 16-byte accesses at any address of global memory (aligned ones are faster).
struct __attribute__((packed, aligned(2))) Loose8 {
  __bf16 e[8];
};
struct __attribute__((packed, aligned(4))) LooseFloat8 {
  float e[8];
};
template <class T>
struct LooseOf {
  using type = Loose8;
};
template <>
struct LooseOf<float> {
  using type = LooseFloat8;
};
// The first n (at most 8) elements at p as floats, zeros behind them.
template <class T>
__device__ __forceinline__ void load_up_to_8(const T* p, int n, float* x) {
  if (n >= 8) {
    const typename LooseOf<T>::type v = *reinterpret_cast<const typename LooseOf<T>::type*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v.e[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < n ? (float)p[e] : 0.f;
  }
}
template <class T>
__device__ __forceinline__ void store_up_to_8(T* p, int n, const float* x) {
  if (n >= 8) {
    typename LooseOf<T>::type v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v.e[e] = (T)x[e];
    *reinterpret_cast<typename LooseOf<T>::type*>(p) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = (T)x[e];
  }
}

// Sum over groups of `LANES` neighbouring lanes; every lane gets it.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int o = LANES / 2; o >= 1; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

}  // namespace chunk_attn
