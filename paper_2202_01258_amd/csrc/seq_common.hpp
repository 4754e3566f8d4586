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
#include "seq_plan.hpp"

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
// row r at place c ^ swizzle(r).  LDS has 64 banks (256 bytes): 16 lanes that read
// one chunk of consecutive rows, an operand's rows, are to meet 16 different places,
// and 32 lanes that read four neighbouring chunks of four rows, a transposed read,
// four different quarters.  (Counted: with r itself for the swizzle half of all LDS
// cycles were conflicts of the transposed reads.)
template <int DP> __device__ inline int swizzle(int row) {
  return DP == 64 ? ((row & 2) << 1) | ((row >> 2) & 3) : ((row & 3) << 2) | ((row >> 2) & 3);
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
// Tiles of 64 rows are addressed with 31 bits from their first row.  A single row's stride
// means nothing; it is set to 0.
inline bool near_rows(qds_view& v, int length) {
  if (length < 2) v.stride[1] = 0;
  return v.stride[1] < (1 << 23) && v.stride[1] > -(1 << 23);
}

// ROWS rows of a tensor in the registers of a workgroup of BLOCK threads (to be
// written to LDS): rows from `end` on and columns from `dim` on are zero and
// are not read.  Buffer loads: the address is a scalar base per tile, a lane's
// offset that never changes and a scalar offset per load, and an offset past the
// buffer's size loads zero, so a load costs two vector instructions and no branch.
constexpr uint32_t kBufferSize = 0x7fffffffu, kOutside = 0x80000000u;
constexpr int kBufferFlags = 0x00027000;           // raw buffer of 32-bit data
template <class T, int DP, int BLOCK, int ROWS = 64> struct Staged {
  static constexpr int N = ROWS * DP / 8 / BLOCK, STEP = BLOCK / (DP / 8);   // loads; rows between two of a thread's
  u32x4 r[N];
  const T* base;
  int64_t stride;
  uint32_t offset, step;       // bytes: of the thread's first piece in a tile, and from one to the next
  int place;                   // its row, or one that no tensor has for columns that are not real
  // A stride below 0 counts the tile's rows from its last one.
  __device__ void init(const T* p, int64_t row_stride, int dim) {
    base = p;
    stride = row_stride;
    const int c = threadIdx.x % (DP / 8), row = threadIdx.x / (DP / 8);
    const uint32_t bytes = (uint32_t)(stride < 0 ? -stride : stride) * 2;
    step = STEP * bytes;
    offset = (stride < 0 ? ROWS - 1 - row : row) * bytes + c * 16;
    place = c * 8 < dim ? row : 1 << 30;
  }
  __device__ void load(int row0, int end) {
    const T* first = base + (int64_t)(stride < 0 ? row0 + ROWS - 1 : row0) * stride;
    const auto buffer = __builtin_amdgcn_make_buffer_rsrc((void*)first, 0, kBufferSize, kBufferFlags);
    const uint32_t down = stride < 0 ? step : 0, up = stride < 0 ? 0 : step;
    const int rows = end - row0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t at = place < rows - i * STEP ? offset - i * down : kOutside;
      r[i] = __builtin_amdgcn_raw_buffer_load_b128(buffer, at, i * up, 0);
    }
  }
  __device__ void store(T* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      *reinterpret_cast<u32x4*>(lds + tile_at<DP>(threadIdx.x / (DP / 8) + i * STEP, threadIdx.x % (DP / 8))) = r[i];
  }
};

// Where a lane reads a tile's operands: byte offsets for the tile's first piece.  The
// other pieces are at these with some of the bits 4..7 (the place of a chunk) flipped
// and a multiple of 8 rows added, both known at compile time.
template <int DP> struct Lanes {
  static constexpr int ROW = DP * 2;
  uint32_t rows, columns, straight, ordered;
  __device__ Lanes() {
    const int l = threadIdx.x & 63, half = l >> 5, r = l & 31, quad = (l & 15) >> 2;
    // of a transposed read: 16 columns for each group of 16 lanes, in pieces of 4
    const int piece = l & 3, turned = (piece >> 1) | ((piece & 1) << 1), group = ((l >> 4) & 1) * 2;
    rows = r * ROW + ((half ^ swizzle<DP>(r)) << 4);
    columns = (4 * half + quad) * ROW + (((group + (piece >> 1)) ^ swizzle<DP>(4 * half + quad)) << 4) + (piece & 1) * 8;
    straight = (8 * half + quad) * ROW + (((group + (piece >> 1)) ^ swizzle<DP>(8 * half + quad)) << 4) + (piece & 1) * 8;
    ordered = (8 * half + quad) * ROW + (((group + (turned >> 1)) ^ swizzle<DP>(8 * half + quad)) << 4) + (turned & 1) * 8;
  }
  // Makes the compiler form the other pieces' offsets again (an instruction each)
  // where it would otherwise keep them all in registers that a kernel lacks.
  __device__ void forget() { asm volatile("" : "+v"(rows), "+v"(columns), "+v"(straight), "+v"(ordered)); }
};
template <class T> __device__ inline const T* tile_byte(const T* lds, uint32_t offset) {
  return (const T*)((const char*)lds + offset);
}

// Rows row0 + l % 32 of a tile, the s-th 16 columns (row0: a multiple of 32).
template <class T, int DP> __device__ inline x8<T> tile_rows(const T* lds, const Lanes<DP>& at, int row0, int s) {
  return __builtin_bit_cast(x8<T>, *reinterpret_cast<const u32x4*>(tile_byte(lds, (at.rows ^ (s << 5)) + row0 * DP * 2)));
}
// Columns dt * 32 + l % 32 of a tile as rows (or columns) of an operand whose k are the
// tile's rows row0 + 8 (e / 4) + 4 (l / 32) + e % 4, e = 0..7: the order in
// which a C tile holds its rows (row0: a multiple of 16).
template <class T, int DP> __device__ inline x8<T> tile_columns(const T* lds, const Lanes<DP>& at, int row0, int dt) {
  const uint32_t first = at.columns ^ (dt << 6), second = first ^ 32;       // swizzle(r + 8)
  const x4<T> a = lds_read_transposed(tile_byte(lds, first + row0 * DP * 2));
  const x4<T> b = lds_read_transposed(tile_byte(lds, second + (row0 + 8) * DP * 2));
  return join8<T>(a, b);
}
// The same with k the tile's rows row0 + 8 (l / 32) + e.
template <class T, int DP> __device__ inline x8<T> tile_columns_straight(const T* lds, uint32_t lane_at, int row0, int dt) {
  const uint32_t first = lane_at ^ (dt << 6), second = first ^ 16;      // swizzle(r + 4)
  const x4<T> a = lds_read_transposed(tile_byte(lds, first + row0 * DP * 2));
  const x4<T> b = lds_read_transposed(tile_byte(lds, second + (row0 + 4) * DP * 2));
  return join8<T>(a, b);
}
// Asks the compiler to keep LDS reads AHEAD products in front of the N products
// that use them (READS reads each) in the code before it, up to the last branch.
// Left alone it reads each operand right before its product, and every product
// then waits for LDS (some 100 cycles against 32).
template <int N, int READS, int AHEAD> __device__ inline void reads_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, READS * AHEAD, 0);
#pragma unroll
  for (int i = 0; i < N - AHEAD; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
}

// The wave's number in its workgroup, as a scalar (so that what depends on it branches for the whole wave).
__device__ inline int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
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

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A launch has fewer than 2^32 threads in a dimension: HIP takes a larger grid without an
// error and leaves workgroups out.
constexpr uint32_t most_blocks(int threads) { return 0xffffffffu / (uint32_t)threads; }

inline qds_status launch_status() {
  return hipGetLastError() == hipSuccess ? QDS_OK : QDS_ERR_HIP;
}

inline uint64_t align_up(uint64_t x) { return (x + 255) / 256 * 256; }

}  // namespace seq
