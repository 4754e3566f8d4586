// seq_rows.hpp -- rows of any width, alignment and stride in packs of elements, and the
// functions of one number that several kernels of libqdseq.so share.
#pragma once

#include <type_traits>

#include "seq_common.hpp"

namespace seq {

template <class T> __device__ inline float to_f32(T x) { return (float)x; }
template <class T> __device__ inline T from_f32(float x) { return (T)x; }

// VEC consecutive elements, 16 bytes in the norms and 4 to 32 elsewhere, at any alignment: rows of odd
// widths start anywhere.  Where VEC does not divide the width (TAIL), a row's last lane takes its
// last VEC elements, some of which its neighbour has as well: both store the same
// values, and only the neighbour counts them in sums.  That leaves no branch around
// the accesses (a branch per element at the row's end let each load wait for the
// one before: 32000 x 1024 then took 141 us in place of 95).
template <class T, int VEC> struct Pack { T v[VEC]; };

template <class T, int VEC> __device__ inline void load(float* out, const T* p) {
  Pack<T, VEC> e;
  __builtin_memcpy(&e, p, sizeof(e));
#pragma unroll
  for (int i = 0; i < VEC; ++i) out[i] = to_f32(e.v[i]);
}
template <class T, int VEC> __device__ inline void store(T* p, const float* in) {
  Pack<T, VEC> e;
#pragma unroll
  for (int i = 0; i < VEC; ++i) e.v[i] = from_f32<T>(in[i]);
  __builtin_memcpy(p, &e, sizeof(e));
}
// The weight is fp32 or of the tensors' type.
template <class T, int VEC> __device__ inline void load_weight(float* out, const void* w, bool w32, int col) {
  if (w32) {
    const float* p = (const float*)w + col;
    if constexpr (VEC == 8) {
      load<float, 4>(out, p);
      load<float, 4>(out + 4, p + 4);
    } else {
      load<float, VEC>(out, p);
    }
  } else {
    load<T, VEC>(out, (const T*)w + col);
  }
}
// Where the pack of a lane at column `col` (inside the row) starts.
template <int VEC, bool TAIL> __device__ inline int pack_at(int col, int width) {
  return TAIL ? min(col, width - VEC) : col;
}

template <int V> using Int = std::integral_constant<int, V>;

// 1 / (1 + e^-x) with the hardware's exponential and reciprocal (an ulp each): infinite
// arguments and exponentials give 0 or 1.
__device__ inline float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + fast_exp2(-kLog2e * x)); }
// The derivative of x sigmoid(x), from s = sigmoid(x).
__device__ inline float silu_slope(float x, float s) { return s * fmaf(x, 1.0f - s, 1.0f); }

}  // namespace seq
