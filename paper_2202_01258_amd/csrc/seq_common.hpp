// seq_common.hpp -- types, conversions, matrix instructions and lane exchanges
// shared by the kernels of libqdseq.so (gfx950, 64 lanes per wave).
//
// Lane layouts of the matrix instructions used here (checked on the device):
//   32x32x16: A: lane holds row l % 32, k = 8 (l / 32) + 0..7;  B: column l % 32, the same k;
//             C: lane holds column l % 32, register i is row i % 4 + 8 (i / 4) + 4 (l / 32).
//   16x16x32: A: row l % 16, k = 8 (l / 16) + 0..7;  B: column l % 16, the same k;
//             C: column l % 16, register i is row 4 (l / 16) + i.
// A product's k index may be permuted as long as both operands agree.  That lets
// a C tile be the B operand of the next product without leaving its registers:
// its rows are then k, in the order that the lane already holds them, and the A
// operand is read in the same order.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/qd_seq.h"

namespace seq {

typedef __bf16 bf16;
typedef _Float16 half;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef half half2v __attribute__((ext_vector_type(2)));
typedef half half4v __attribute__((ext_vector_type(4)));
typedef half half8v __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T> struct Vec;
template <> struct Vec<bf16> { using x2 = bf16x2; using x4 = bf16x4; using x8 = bf16x8; };
template <> struct Vec<half> { using x2 = half2v; using x4 = half4v; using x8 = half8v; };
template <class T> using x2 = typename Vec<T>::x2;
template <class T> using x4 = typename Vec<T>::x4;
template <class T> using x8 = typename Vec<T>::x8;

__device__ inline f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mfma32(half8v a, half8v b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mfma16(half8v a, half8v b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Two floats to two 16-bit values, to nearest even.
template <class T> __device__ inline x2<T> pack2(float a, float b) {
  return __builtin_convertvector(f32x2{a, b}, x2<T>);
}
template <class T> __device__ inline x8<T> pack8(const float* p) {
  x2<T> r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = pack2<T>(p[2 * i], p[2 * i + 1]);
  return __builtin_shufflevector(__builtin_shufflevector(r[0], r[1], 0, 1, 2, 3),
                                 __builtin_shufflevector(r[2], r[3], 0, 1, 2, 3), 0, 1, 2, 3, 4, 5,
                                 6, 7);
}
template <class T> __device__ inline x4<T> pack4(float a, float b, float c, float d) {
  return __builtin_shufflevector(pack2<T>(a, b), pack2<T>(c, d), 0, 1, 2, 3);
}
template <class T> __device__ inline x8<T> join8(x4<T> a, x4<T> b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <class T> __device__ inline x8<T> zero8() {
  return __builtin_bit_cast(x8<T>, u32x4{0, 0, 0, 0});
}

__device__ inline float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float fast_log2(float x) { return __builtin_amdgcn_logf(x); }

// The value of lane l ^ 32, combined with this lane's.
__device__ inline float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <class T> __device__ inline T shfl_xor(T v, int mask) { return __shfl_xor(v, mask, 64); }

__device__ inline float wave_sum(float x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) x += shfl_xor(x, m);
  return x;
}
__device__ inline float wave_max(float x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) x = fmaxf(x, shfl_xor(x, m));
  return x;
}

using lds_s16x4 = __attribute__((address_space(3))) s16x4;

// Four rows of 16 columns, transposed.  In each group of 16 lanes, lane i gives
// the address of columns 4 (i % 4) .. + 3 of row i / 4 and receives column i,
// rows 0..3.
template <class T> __device__ inline x4<T> lds_read_transposed(const T* p) {
  return __builtin_bit_cast(
      x4<T>, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(const_cast<T*>(p))));
}

// Tiles in LDS: rows of DP 16-bit values in chunks of 8 (16 bytes), chunk c of
// row r at place c ^ swizzle(r), so that lanes that read the same chunk of
// consecutive rows spread over all banks (256 bytes: two rows of 64 values, or
// one of 128).
template <int DP> __device__ inline int swizzle(int row) {
  return DP == 64 ? (row >> 1) & 7 : row & 15;
}
template <int DP> __device__ inline int tile_at(int row, int chunk) {
  return row * DP + ((chunk ^ swizzle<DP>(row)) << 3);
}

// Shared memory that is read in pieces of 16 bytes.
#define SEQ_SHARED __shared__ __attribute__((aligned(16)))

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

struct View {
  char* p;
  int64_t b, t, h;     // strides in elements
};
template <class T> __device__ inline T* at(const View& v, int64_t b, int64_t t, int64_t h) {
  return (T*)v.p + b * v.b + t * v.t + h * v.h;
}
inline View view(const qds_view& v) { return View{(char*)v.data, v.stride[0], v.stride[1], v.stride[2]}; }

// Rows of a view are read and written in pieces of 16 bytes.
inline bool usable(const qds_view& v, bool rows = true) {
  return v.data && aligned16(v.data) && v.stride[0] % 8 == 0 && v.stride[2] % 8 == 0 &&
         (!rows || v.stride[1] % 8 == 0);
}

// 64 rows of a tensor in the registers of a workgroup of BLOCK threads (to be
// written to LDS): rows from `end` on and columns from `dim` on are zero and
// are not read.
template <class T, int DP, int BLOCK> struct Staged {
  static constexpr int N = 64 * DP / 8 / BLOCK;
  u32x4 r[N];
  __device__ void load(const T* p, int64_t stride, int row0, int end, int dim) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x + i * BLOCK, row = id / (DP / 8), c = id % (DP / 8);
      r[i] = u32x4{0, 0, 0, 0};
      if (row0 + row < end && c * 8 < dim)
        r[i] = *reinterpret_cast<const u32x4*>(p + (int64_t)(row0 + row) * stride + c * 8);
    }
  }
  __device__ void store(T* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x + i * BLOCK, row = id / (DP / 8), c = id % (DP / 8);
      *reinterpret_cast<u32x4*>(lds + tile_at<DP>(row, c)) = r[i];
    }
  }
};

// Rows row0 + l % 32 of a tile, the s-th 16 columns.
template <class T, int DP> __device__ inline x8<T> tile_rows(const T* lds, int row0, int s) {
  const int l = threadIdx.x & 63;
  return __builtin_bit_cast(x8<T>, *reinterpret_cast<const u32x4*>(lds + tile_at<DP>(row0 + (l & 31), s * 2 + (l >> 5))));
}
// Columns dt * 32 + l % 32 of a tile as rows of an operand whose k are the
// tile's rows row0 + 8 (e / 4) + 4 (l / 32) + e % 4, e = 0..7: the order in
// which a C tile holds its rows.
template <class T, int DP> __device__ inline x8<T> tile_columns(const T* lds, int row0, int dt) {
  const int l = threadIdx.x & 63;
  const int row = row0 + 4 * (l >> 5) + ((l & 15) >> 2);
  const int col = dt * 32 + ((l >> 4) & 1) * 16 + (l & 3) * 4;
  const x4<T> a = lds_read_transposed(lds + tile_at<DP>(row, col >> 3) + (col & 7));
  const x4<T> b = lds_read_transposed(lds + tile_at<DP>(row + 8, col >> 3) + (col & 7));
  return join8<T>(a, b);
}
// Row of register i of a 32x32 C tile.
__device__ inline int c_row(int i) { return (i & 3) + 8 * (i >> 2) + 4 * ((threadIdx.x & 63) >> 5); }

// A C tile whose columns are a tensor's rows: register 4 b + 0..3 are four
// neighbouring elements of the row.
template <class T> __device__ inline void store_column(T* row, int dt, const f32x16& c, float factor, int dim) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int d = dt * 32 + 8 * b + 4 * half;
    if (d < dim)
      *reinterpret_cast<u32x2*>(row + d) = __builtin_bit_cast(
          u32x2, pack4<T>(c[4 * b] * factor, c[4 * b + 1] * factor, c[4 * b + 2] * factor, c[4 * b + 3] * factor));
  }
}

// Workgroups that follow each other go round the card's eight XCDs, each with
// an L2 cache of its own.  This gives each XCD a contiguous piece of the work
// items, so that items that read the same keys share a cache.
constexpr int kXcds = 8;
__device__ inline int xcd_order(int id, int count) {
  const int per = count / kXcds, rest = count % kXcds;
  const int x = id % kXcds, y = id / kXcds;
  return x * per + min(x, rest) + y;
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

constexpr int kFill = 512;       // workgroups that fill the card: two per compute unit

inline qds_status launch_status() {
  return hipGetLastError() == hipSuccess ? QDS_OK : QDS_ERR_HIP;
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline uint64_t align_up(uint64_t x) { return (x + 255) / 256 * 256; }

}  // namespace seq
