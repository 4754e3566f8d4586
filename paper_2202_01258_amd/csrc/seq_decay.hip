// seq_decay.hip -- linear attention with a decay for each head: by chunks
// (forward and backward) and the recurrent single-token step.  The C ABI is in
// include/qd_seq.h.
//
// One recurrence serves every direction.  With rows x, y of DK and z of DV elements,
//   M_i = a M_{i-1} + f y_i^T z_i,   out_i = g x_i M_i:
//   o:  (x, y, z) = (q, k, v),   M the state S,                  f = 1, g = scale;
//   dq: (do, v, k),              M = S^T,                        f = 1, g = scale;
//   dv: (k, q, do), rows reversed, M = R = scale sum a^(t-s) q_t^T do_t + the state's gradient, f = scale, g = 1;
//   dk: (v, do, q), rows reversed, M = R^T,                      f = scale, g = 1.
// A chunk of 64 rows is
//   out = f g ((x y^T) . a^(i-j) [j <= i]) z + g a^(i+1) x M,   M <- a^64 M + f y^T (a^(63-j) z),
// all products on the matrix cores, the state in registers.  By its bytes (each
// row read and written once) the recurrence is bound by memory.
#include "seq_common.hpp"

namespace seq {
namespace {

constexpr int kChunk = 64;
constexpr int kEarly = 128;

// a^n for lambda = log2(a).  `lambda` is kept finite (decay_rate), so that a^0 is 1
// for a = 0, too; below the bound a^1 is 0 already.  Not-a-number stays (fmaxf would
// make it the bound).
__device__ inline float decay_power(float lambda, float n) { return fast_exp2(lambda * n); }
__device__ inline float decay_rate(const float* log_decay, int h) {
  const float lambda = log_decay[h] * kLog2e;
  return lambda < -1.0e4f ? -1.0e4f : lambda;
}

// One direction of the recurrence.
struct Role {
  View x, y, z, out;
  const float* init;     // the state before the first row [b][h][dim_k][dim_v] of the caller's sides, or null
  float* last;           // the state after the last row, or null
  float* states;         // [b][h][segment][DK][DV]: each segment's own sum, then the state before it
  float sums, outputs;   // the factors f of what is summed and g of the outputs
  bool reversed;         // rows from the last to the first
  bool swapped;          // init and last are [dim_z][dim_x] (the transpose of M)
};

struct DecayArgs {
  Role role[3];
  const int32_t* lengths;
  const float* log_decay;
  int32_t batch, length, heads, dim_x, dim_z;
  int32_t segments, segment_rows;     // segment_rows: a multiple of 64
};

__device__ inline int rows_of(const DecayArgs& a, int b) {
  if (!a.lengths) return a.length;
  return min(max(a.lengths[b], 0), a.length);
}

// N tiles of 32 rows of the state, 32 columns; the first is tile `first` of all.
// In memory [rows][cols], or transposed.  The left operand of the products that
// form it has its rows in an order (`ordered` reads) that puts 8 neighbouring rows
// of the state into registers 8 u .. 8 u + 7 of a tile, so that they are an operand
// of the output's product against plain rows of x.
template <int N> struct State {
  f32x16 m[N];
  int first;
  __device__ int row_of(int t, int i) const {
    return (first + t) * 32 + 16 * (i >> 3) + 8 * ((threadIdx.x & 63) >> 5) + (i & 7);
  }
  __device__ void zero() {
#pragma unroll
    for (int t = 0; t < N; ++t) m[t] = f32x16{};
  }
  // Buffer loads, all under way at once: an element outside is read as 0, without a branch
  // (with one, each load was waited for by itself).
  __device__ void load(const float* p, int rows, int cols, int col, bool swapped) {
    const auto buffer = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, kBufferSize, kBufferFlags);
    const uint32_t step = swapped ? 4 : 4 * cols, base = swapped ? col * 4 * rows : col * 4;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = row_of(t, i);
        const uint32_t at = row < rows && col < cols ? base + row * step : kOutside;
        m[t][i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buffer, at, 0, 0));
      }
  }
  __device__ void store(float* p, int rows, int cols, int col, bool swapped, float factor) const {
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = row_of(t, i);
        if (row < rows && col < cols) p[swapped ? col * rows + row : row * cols + col] = factor * m[t][i];
      }
  }
};

// How many numbers of 16 bits carry an fp32 one: the state is fp32, so its
// summands f a^(63-j) y_j z_j keep 24 bits in bfloat16, 22 in float16 (y is exact;
// f z a^(63-j) is split).  Of a float16 y below its normal range the matrix instruction's sums
// keep 2^-24 of what 2^-14 would have given: for y = 2^-24 the relative error is 5e-5.
template <class T> struct Terms;
template <> struct Terms<bf16> { static constexpr int n = 3; };
template <> struct Terms<half> { static constexpr int n = 2; };

// float16 ends at 65504 and in steps of 2^-24.  What it carries for an fp32 sum is first
// brought to its upper end by a power of two that takes the largest of the numbers that
// share it to 2^14 .. 2^15; its inverse takes the products back.  Numbers below 2^-29 of
// that largest keep fewer bits, those below 2^-40 none.  bfloat16 has fp32's range.
// LEAST bounds the power to 2^(141 - LEAST).
template <class T> constexpr bool kScaled = std::is_same<T, half>::value;
template <uint32_t LEAST = 15> __device__ inline float to_upper_end(float largest) {
  const uint32_t e = min(max(__float_as_uint(largest) >> 23, LEAST), 254u);      // the power and its inverse are normal numbers
  return __uint_as_float((268 - e) << 23);
}
__device__ inline float inverse(float power) { return __uint_as_float(0x7f000000u - __float_as_uint(power)); }

// Waves per 32 columns of the state.  With 128 columns four waves have a column
// block each, with all rows.  With 64 columns two waves share a block: each holds
// half of the state's rows and forms the outputs of half of the chunk's rows, and
// they show each other their halves of the state (rounded, as the product wants
// them) through LDS.  That halves the time that a chunk takes a workgroup, which
// is what bounds few heads: chunks follow each other.
template <int DV> constexpr int kShare = DV == 64 ? 2 : 1;
template <int DV> constexpr int kDecayBlock = 2 * DV * kShare<DV>;

// A workgroup has one batch element and head, and one segment of its rows.  Where
// there are too few heads to fill the card, a sequence is cut into segments: with
// OUT false a segment only forms its own sum, k_decay_scan turns the sums into the
// states before the segments, and a second launch with OUT true starts from those.
// Few heads are bound by their chunks' sequence: 32 x 1000 rows, 8 heads of 64 take 38 us
// forward and 71 us back (float16, with its powers of two, 49 and 84; 47 and 97 with two
// waves on a SIMD in place of three).  131072 rows, 16 heads of 128, in segments: 273 to
// 293 us for the sums, 561 to 589 us for the outputs, at 3.7 to 3.9 TB/s.
template <class T, int DK, int DV, bool OUT>
__global__ __launch_bounds__(kDecayBlock<DV>, kScaled<T> && DK + DV <= kEarly ? 3 : 2) void k_decay_chunks(DecayArgs a) {
  constexpr int SHARE = kShare<DV>, BLOCK = kDecayBlock<DV>, WAVES = BLOCK / 64, SLICES = DV / 32;
  constexpr int TILES = DK / 32, OWN = TILES / SHARE;
  SEQ_SHARED T sx[OUT ? kChunk * DK : 8], sy[kChunk * DK], sz[kChunk * DV];
  SEQ_SHARED T sp[OUT ? kChunk * kChunk : 8];
  SEQ_SHARED T sm[OUT && SHARE == 2 ? WAVES * OWN * 2 * 64 * 8 : 8];
  SEQ_SHARED float s_age[kChunk];            // f a^(rows - 1 - j) of the chunk's rows
  // what takes products with the state back (each share's columns), and the powers of products of rows (each row's halves)
  SEQ_SHARED float s_state[OUT && kScaled<T> ? SHARE * DV : 4], s_rows[OUT && kScaled<T> ? 2 * kChunk : 4];
  const Role& role = a.role[blockIdx.z];
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int slice = wave % SLICES, part = wave / SLICES;
  const int b = blockIdx.x / a.heads, h = blockIdx.x % a.heads;
  const int n = rows_of(a, b);
  const int first = blockIdx.y * a.segment_rows, end = min(first + a.segment_rows, n);
  const float lambda = decay_rate(a.log_decay, h);
  const int64_t list = (int64_t)b * a.heads + h;
  const int64_t turn = role.reversed ? n - 1 : 0, sign = role.reversed ? -1 : 1;
  const int col = slice * 32 + (lane & 31);

  Lanes<DK> at_k;
  Lanes<DV> at_v;
  Lanes<64> at_p;
  State<OWN> st;
  st.first = part * OWN;
  float* mine = role.states + (list * a.segments + blockIdx.y) * (DK * DV);
  if (OUT && a.segments > 1)
    st.load(mine, DK, DV, col, false);
  else if (OUT && role.init)
    st.load(role.init + list * a.dim_x * a.dim_z, a.dim_x, a.dim_z, col, role.swapped);
  else
    st.zero();

  if (first < end) {
    Staged<T, DK, BLOCK> rx, ry;
    Staged<T, DV, BLOCK> rz;
    if (OUT) rx.init(at<T>(role.x, b, turn, h), sign * role.x.t, a.dim_x);
    ry.init(at<T>(role.y, b, turn, h), sign * role.y.t, a.dim_x);
    rz.init(at<T>(role.z, b, turn, h), sign * role.z.t, a.dim_z);
    // f g a^(i-j) of a wave's products of rows, 0 for j > i: the same in every chunk
    const float both = role.sums * role.outputs;
    float fade[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int gap = (wave == 1 ? 32 : 0) + (lane & 31) - c_row(r);
      fade[r] = gap >= 0 ? both * decay_power(lambda, gap) : 0.0f;
    }
    auto fetch = [&](int row0) {
      if (row0 >= end) return;
      if (OUT) rx.load(row0, end);
      ry.load(row0, end);
      rz.load(row0, end);
    };
    fetch(first);
    for (int row0 = first; row0 < end; row0 += kChunk) {
      const int count = min(kChunk, end - row0);
      if (DK == 128) at_k.forget();
      // the gradient of the last state meets the last row without a decay
      const int less = role.reversed && row0 == 0 ? 1 : 0;
      if (OUT) rx.store(sx);
      ry.store(sy);
      rz.store(sz);
      if (threadIdx.x < kChunk)
        s_age[threadIdx.x] = (int)threadIdx.x < count ? role.sums * decay_power(lambda, count - 1 - threadIdx.x) : 0.0f;
      // The products of rows and the state are rounded to the tensors' type for the
      // output's products: as much as the output's own rounding.  Float16 also brings each
      // column of the state, and each row of a quarter of the products of rows, to its
      // upper end: states grow beyond 65504 and gradients are small where outputs are neither.
      x8<T> packed[OUT ? OWN : 1][2];
      if constexpr (OUT) {
        float up = 1.0f;
        if constexpr (kScaled<T>) {
          float top = 0.0f;
#pragma unroll
          for (int t = 0; t < OWN; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, fabsf(st.m[t][r]));
          up = to_upper_end(max_halves(top));
          if (lane < 32) s_state[part * DV + col] = inverse(up);
        }
#pragma unroll
        for (int t = 0; t < OWN; ++t)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            float m[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) m[e] = kScaled<T> ? st.m[t][8 * u + e] * up : st.m[t][8 * u + e];
            packed[t][u] = pack8<T>(m);
            if (SHARE == 2)
              *reinterpret_cast<x8<T>*>(sm + (((wave * OWN + t) * 2 + u) * 64 + lane) * 8) = packed[t][u];
          }
      }
      __syncthreads();
      if (DK + DV <= kEarly) fetch(row0 + kChunk);
      if constexpr (OUT) {
        // Quarters (0, 0), (1, 0), (1, 1) of the products of rows, transposed (columns are i), a wave each.
        if (wave < 3) {
          const int ib = wave > 0, jb = wave > 1;
          f32x16 s = f32x16{};
#pragma unroll
          for (int ks = 0; ks < DK / 16; ++ks)
            s = mfma32(tile_rows<T, DK>(sy, at_k, jb * 32, ks), tile_rows<T, DK>(sx, at_k, ib * 32, ks), s);
          const int i = ib * 32 + (lane & 31);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] *= fade[r];
          if constexpr (kScaled<T>) {
            // up to 2^40: below that, products are nothing in a float16 output, and the output in
            // fp32 is multiplied with the power, too
            float top = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, fabsf(s[r]));
            const float up = to_upper_end<101>(max_halves(top));
            if (lane < 32) s_rows[jb * kChunk + i] = up;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] *= up;
          }
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4) {
            const int j = jb * 32 + 8 * r4 + 4 * (lane >> 5);
            *reinterpret_cast<u32x2*>(sp + tile_at<64>(i, j >> 3) + (j & 7)) =
                __builtin_bit_cast(u32x2, pack4<T>(s[4 * r4], s[4 * r4 + 1], s[4 * r4 + 2], s[4 * r4 + 3]));
          }
        }
        __syncthreads();
      }
      x8<T> z[4];
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) z[ks] = tile_columns_straight<T, DV>(sz, at_v.straight, 16 * ks, slice);
      if constexpr (OUT) {
        auto state_of = [&](int t, int u) {
          if (SHARE == 1) return packed[t % OWN][u];
          const int holder = slice + SLICES * (t / OWN);
          return *reinterpret_cast<const x8<T>*>(sm + (((holder * OWN + t % OWN) * 2 + u) * 64 + lane) * 8);
        };
        auto output = [&](int ib) {
          const int i = ib * 32 + (lane & 31);
          const float reach = role.outputs * decay_power(lambda, i + 1 - less);
          f32x16 o = f32x16{};
          if constexpr (kScaled<T>) {
            // Each share and each half has powers of its own.
#pragma unroll
            for (int q = 0; q < SHARE; ++q) {
              f32x16 sum = f32x16{};
#pragma unroll
              for (int t = q * OWN; t < (q + 1) * OWN; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) sum = mfma32(state_of(t, u), tile_rows<T, DK>(sx, at_k, ib * 32, 2 * t + u), sum);
#pragma unroll
              for (int r4 = 0; r4 < 4; ++r4) {
                const f32x4 down = *reinterpret_cast<const f32x4*>(s_state + q * DV + slice * 32 + 8 * r4 + 4 * (lane >> 5));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float part_sum = sum[4 * r4 + e] * (down[e] * reach);
                  o[4 * r4 + e] = q == 0 ? part_sum : o[4 * r4 + e] + part_sum;
                }
              }
            }
#pragma unroll
            for (int jb = 0; jb < 2; ++jb) {
              if (jb > ib) break;
              const float up = s_rows[jb * kChunk + i];
              o *= up;
#pragma unroll
              for (int ks = 2 * jb; ks < 2 * jb + 2; ++ks) o = mfma32(z[ks], tile_rows<T, 64>(sp, at_p, ib * 32, ks), o);
              o *= inverse(up);
            }
          } else {
            // the halves in one order for both waves, so that sums do not depend on the wave
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
              for (int u = 0; u < 2; ++u) o = mfma32(state_of(t, u), tile_rows<T, DK>(sx, at_k, ib * 32, 2 * t + u), o);
            o *= reach;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              if (ks < 2 * (ib + 1)) o = mfma32(z[ks], tile_rows<T, 64>(sp, at_p, ib * 32, ks), o);
          }
          if (i < count) {
            const int64_t row = turn + sign * (row0 + i);
            store_column<T>(at<T>(role.out, b, row, h), slice, o, 1.0f, a.dim_z);
          }
        };
        if (SHARE == 2) {
          output(part);
        } else {
          output(0);
          if (kScaled<T>) __builtin_amdgcn_sched_barrier(0);       // both at once would not fit the registers
          output(1);
        }
      }
      // The next rows' loads are under way during the state's products alone: with the
      // output's in between as well, the registers that they fill would not fit.
      if (DK + DV > kEarly) {
        __builtin_amdgcn_sched_barrier(0);
        fetch(row0 + kChunk);
      }
      const float age = decay_power(lambda, count - less);
#pragma unroll
      for (int t = 0; t < OWN; ++t) st.m[t] *= age;
      // f z a^(63-j) of a lane's 8 rows in step ks
      auto summand = [&](int ks, float* v) {
        const int j = 16 * ks + 8 * (lane >> 5);
        const f32x4 w0 = *reinterpret_cast<const f32x4*>(s_age + j), w1 = *reinterpret_cast<const f32x4*>(s_age + j + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)z[ks][e] * (e < 4 ? w0[e & 3] : w1[e & 3]);
      };
      auto split = [&](x8<T>* term, float* v) {
#pragma unroll
        for (int p = 0; p < Terms<T>::n; ++p) {
          term[p] = pack8<T>(v);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] -= (float)term[p][e];
        }
      };
      if constexpr (kScaled<T>) {
        // a power of two for each of the state's columns, which is a column of z: in the lane and lane ^ 32
        float top = 0.0f, v[8];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          summand(ks, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
        }
        const float up = to_upper_end(max_halves(top)), down = inverse(up);
        x8<T> term[4][Terms<T>::n];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          summand(ks, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= up;
          split(term[ks], v);
        }
#pragma unroll
        for (int t = 0; t < OWN; ++t) {
          f32x16 sum = f32x16{};
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {
            const x8<T> y = tile_columns_straight<T, DK>(sy, at_k.ordered, 16 * ks, st.first + t);
#pragma unroll
            for (int p = Terms<T>::n - 1; p >= 0; --p) sum = mfma32(y, term[ks][p], sum);
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) st.m[t][r] = fmaf(sum[r], down, st.m[t][r]);
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          x8<T> term[Terms<T>::n];
          float v[8];
          summand(ks, v);
          split(term, v);
#pragma unroll
          for (int t = 0; t < OWN; ++t) {
            const x8<T> y = tile_columns_straight<T, DK>(sy, at_k.ordered, 16 * ks, st.first + t);
#pragma unroll
            for (int p = Terms<T>::n - 1; p >= 0; --p) st.m[t] = mfma32(y, term[p], st.m[t]);
          }
        }
      }
      __syncthreads();
    }
  }
  if (!OUT) {
    st.store(mine, DK, DV, col, false, 1.0f);
    return;
  }
  if (a.segments == 1 && role.last) {
    const float f = role.reversed && n > 0 ? decay_power(lambda, 1) : 1.0f;
    st.store(role.last + list * a.dim_x * a.dim_z, a.dim_x, a.dim_z, col, role.swapped, f);
  }
  // rows past the end
  const int stop = min(first + a.segment_rows, a.length);
  const int packs = a.dim_z / 8;
  for (int64_t x = threadIdx.x; x < (int64_t)(stop - max(first, n)) * packs; x += BLOCK) {
    T* row = at<T>(role.out, b, max(first, n) + x / packs, h);
    *reinterpret_cast<u32x4*>(row + x % packs * 8) = u32x4{0, 0, 0, 0};
  }
}

// From each segment's own sum to the state before it.  A thread has one element of M and
// one of PARTS parts of the segments: it adds their sums, the parts' sums give where each
// part starts, and it goes through its segments again from there (one part starts at
// once).  All sums are in a fixed order.
// Eight parts where there are more than 64 segments: a thread's chain of 505 took 63 of
// 106 us (129161 rows, one head of 64 x 128), in parts the call takes 76; 64 segments of
// 8 heads of 128 x 128 take 57 in one part, 61 in eight.
template <int DK, int DV, int PARTS> __global__ __launch_bounds__(256) void k_decay_scan(DecayArgs a) {
  constexpr int M = DK * DV, ELEMENTS = 256 / PARTS, BLOCKS = M / ELEMENTS, AHEAD = 8;
  __shared__ float sums[PARTS][ELEMENTS];
  const Role& role = a.role[blockIdx.z];
  const int64_t list = blockIdx.x / BLOCKS;
  const int part = threadIdx.x / ELEMENTS, lane = threadIdx.x % ELEMENTS;
  const int e = blockIdx.x % BLOCKS * ELEMENTS + lane, row = e / DV, col = e % DV;
  const int b = (int)(list / a.heads), h = (int)(list % a.heads);
  const int n = rows_of(a, b);
  const float lambda = decay_rate(a.log_decay, h);
  const bool real = row < a.dim_x && col < a.dim_z;
  const int64_t outer = list * a.dim_x * a.dim_z + (role.swapped ? col * a.dim_x + row : row * a.dim_z + col);
  float m = role.init && real ? role.init[outer] : 0.0f;
  const int per = (a.segments + PARTS - 1) / PARTS;
  // rows of segments s .. s + many - 1; one less where the first of reversed rows is among them
  auto fade = [&](int s, int many) {
    const int64_t left = (int64_t)n - (int64_t)s * a.segment_rows, all = (int64_t)many * a.segment_rows;
    const int count = left <= 0 ? 0 : (int)(left < all ? left : all);
    return decay_power(lambda, count - (role.reversed && s == 0 && count > 0 ? 1 : 0));
  };
  const int first = min(part * per, a.segments), end = min(first + per, a.segments);
  float* p = role.states + (list * a.segments) * M + e;
  if constexpr (PARTS > 1) {
    float sum = 0.0f;
#pragma unroll 8
    for (int s = first; s < end; ++s) sum = fmaf(sum, fade(s, 1), p[(int64_t)s * M]);
    sums[part][lane] = sum;
    __syncthreads();
    for (int q = 0; q < part; ++q) {
      const int from = min(q * per, a.segments);
      m = fmaf(m, fade(from, min(from + per, a.segments) - from), sums[q][lane]);
    }
  }
  for (int s0 = first; s0 < end; s0 += AHEAD) {
    float own[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) own[i] = s0 + i < end ? p[(int64_t)(s0 + i) * M] : 0.0f;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (s0 + i >= end) break;
      p[(int64_t)(s0 + i) * M] = m;
      m = fmaf(m, fade(s0 + i, 1), own[i]);
    }
  }
  if (role.last && real && part == PARTS - 1)
    role.last[outer] = m * (role.reversed && n > 0 ? decay_power(lambda, 1) : 1.0f);
}

// ---------------------------------------------------------------------------
// Single-token step
// ---------------------------------------------------------------------------
struct StepArgs {
  View q, k, v, o;
  const float *log_decay, *state_in;
  float* state_out;
  int32_t heads, dim_k, dim_v;
  float scale;
};

// Bound by reading and writing the states.  A workgroup has one state; a thread
// has four columns of every (1024 / DV)-th row, so a wave's loads are contiguous.
// 16384 states of 64 x 64: 98 us, 5.5 TB/s.
template <class T, int DK, int DV> __global__ __launch_bounds__(256) void k_decay_step(StepArgs a) {
  constexpr int LANES = DV / 4, ROWS = 256 / LANES, N = DK / ROWS;
  SEQ_SHARED float part[ROWS][DV];
  const int col = threadIdx.x % LANES * 4, sub = threadIdx.x / LANES;
  const int b = blockIdx.x / a.heads, h = blockIdx.x % a.heads;
  const int64_t base = (int64_t)blockIdx.x * a.dim_k * a.dim_v;
  const T *q = at<T>(a.q, b, 0, h), *k = at<T>(a.k, b, 0, h), *v = at<T>(a.v, b, 0, h);
  const bool in_col = col < a.dim_v;
  f32x4 s[N];
  float qr[N], kr[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int row = i * ROWS + sub;
    const bool real = row < a.dim_k && in_col;
    s[i] = real ? *reinterpret_cast<const f32x4*>(a.state_in + base + (int64_t)row * a.dim_v + col) : f32x4{};
    qr[i] = real ? (float)q[row] : 0.0f;
    kr[i] = real ? (float)k[row] : 0.0f;
  }
  f32x4 vv = f32x4{};
  if (in_col) {
    const x4<T> raw = __builtin_bit_cast(x4<T>, *reinterpret_cast<const u32x2*>(v + col));
#pragma unroll
    for (int e = 0; e < 4; ++e) vv[e] = (float)raw[e];
  }
  const float decay = decay_power(decay_rate(a.log_decay, h), 1.0f);
  f32x4 o = f32x4{};
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int row = i * ROWS + sub;
    s[i] = s[i] * decay + vv * kr[i];
    o += s[i] * qr[i];
    if (row < a.dim_k && in_col) *reinterpret_cast<f32x4*>(a.state_out + base + (int64_t)row * a.dim_v + col) = s[i];
  }
  *reinterpret_cast<f32x4*>(&part[sub][col]) = o;
  __syncthreads();
  if ((int)threadIdx.x < a.dim_v) {
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) sum += part[r][threadIdx.x];
    at<T>(a.o, b, 0, h)[threadIdx.x] = (T)(sum * a.scale);
  }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
qds_status validate(const qds_decay_config* c) {
  if (!c || c->abi_version != QDS_ABI_VERSION) return QDS_ERR_INVALID_ARG;
  if (c->dtype != QDS_BF16 && c->dtype != QDS_F16)
    return c->dtype == QDS_F32 ? QDS_ERR_UNSUPPORTED : QDS_ERR_INVALID_ARG;
  if (c->batch < 0 || c->length < 0 || c->length >= (1 << 30) || c->heads < 1) return QDS_ERR_INVALID_ARG;
  if (c->dim_k < 1 || c->dim_v < 1) return QDS_ERR_INVALID_ARG;
  if (c->dim_k % 8 || c->dim_v % 8 || c->dim_k > 128 || c->dim_v > 128) return QDS_ERR_UNSUPPORTED;
  if (!(c->scale > 0.0f) || c->scale > 3.0e38f) return QDS_ERR_INVALID_ARG;
  if ((int64_t)c->batch * c->heads > most_blocks(256)) return QDS_ERR_UNSUPPORTED;      // workgroups of 256 threads
  return QDS_OK;
}

int pad(int dim) { return dim <= 64 ? 64 : 128; }

struct SegmentPlan {
  int32_t segments, rows;
};
// Segments only where there are too few states for half of the compute units: cutting
// reads y and z twice and moves 4 DK DV bytes of state per segment four times.  Forward, us,
// whole | cut: 80 states of 64, 8000 rows 201 | 118;  120 states of 64, 8000 rows 204 | 184;
// 192 states of 64, 8000 rows 205 | 292;  240 of 128, 1000 rows 72 | 121.
// Short sequences stay whole, as two more launches cost more than eight chunks of 64 columns or
// four of 128: 32 states of 64, 512 rows 18.5 | 22.  A segment has two chunks or more: 32 states
// of 64 x 128, 819 rows 26 us with 128 rows, 29 with 256, 28 with 64.
SegmentPlan segment_plan(const qds_decay_config* c, int roles) {
  const int64_t lists = (int64_t)c->batch * c->heads * roles;
  int64_t want = lists > 0 && lists < kFill / 4 ? ceil_div(kFill, lists) : 1;
  const int64_t columns = pad(c->dim_k > c->dim_v ? c->dim_k : c->dim_v);
  const int64_t most = c->length * columns <= 1 << 15 ? 1 : ceil_div(c->length, 2 * kChunk);
  if (want > most) want = most;
  if (want < 1) want = 1;
  SegmentPlan p;
  p.rows = (int32_t)(ceil_div(ceil_div(c->length, want), kChunk) * kChunk);
  if (p.rows < kChunk) p.rows = kChunk;
  p.segments = (int32_t)ceil_div(c->length, p.rows);
  if (p.segments < 1) p.segments = 1;
  return p;
}
uint64_t state_bytes(const qds_decay_config* c, int segments) {
  if (segments == 1) return 0;
  return align_up((uint64_t)c->batch * c->heads * segments * pad(c->dim_k) * pad(c->dim_v) * sizeof(float));
}

template <class T, int DK, int DV> void run_roles(const DecayArgs& a, int roles, hipStream_t s) {
  const uint32_t lists = (uint32_t)a.batch * a.heads;
  if (a.segments > 1) {
    k_decay_chunks<T, DK, DV, false><<<dim3(lists, a.segments, roles), kDecayBlock<DV>, 0, s>>>(a);
    if (a.segments <= 64)
      k_decay_scan<DK, DV, 1><<<dim3(lists * (DK * DV / 256), 1, roles), 256, 0, s>>>(a);
    else
      k_decay_scan<DK, DV, 8><<<dim3(lists * (DK * DV / 32), 1, roles), 256, 0, s>>>(a);
  }
  k_decay_chunks<T, DK, DV, true><<<dim3(lists, a.segments, roles), kDecayBlock<DV>, 0, s>>>(a);
}
template <class T> void run_dims(const DecayArgs& a, int roles, hipStream_t s) {
  const int dk = pad(a.dim_x), dv = pad(a.dim_z);
  if (dk == 64 && dv == 64) run_roles<T, 64, 64>(a, roles, s);
  else if (dk == 64) run_roles<T, 64, 128>(a, roles, s);
  else if (dv == 64) run_roles<T, 128, 64>(a, roles, s);
  else run_roles<T, 128, 128>(a, roles, s);
}
void run(const qds_decay_config* c, const DecayArgs& a, int roles, void* stream) {
  if (c->dtype == QDS_BF16) run_dims<bf16>(a, roles, (hipStream_t)stream);
  else run_dims<half>(a, roles, (hipStream_t)stream);
}

DecayArgs decay_args(const qds_decay_config* c, const SegmentPlan& p, const int32_t* lengths, const float* log_decay) {
  DecayArgs a{};
  a.lengths = lengths;
  a.log_decay = log_decay;
  a.batch = c->batch;
  a.length = c->length;
  a.heads = c->heads;
  a.dim_x = c->dim_k;
  a.dim_z = c->dim_v;
  a.segments = p.segments;
  a.segment_rows = p.rows;
  return a;
}

}  // namespace
}  // namespace seq

using namespace seq;

extern "C" qds_status qds_decay_forward_workspace(const qds_decay_config* c, uint64_t* bytes) {
  const qds_status st = validate(c);
  if (st != QDS_OK) return st;
  if (!bytes) return QDS_ERR_INVALID_ARG;
  *bytes = state_bytes(c, segment_plan(c, 1).segments);
  return QDS_OK;
}

extern "C" qds_status qds_decay_forward(const qds_decay_config* c, qds_view q, qds_view k, qds_view v,
                                        const float* log_decay, const float* state_in,
                                        const int32_t* lengths, qds_view o, float* state_out,
                                        void* workspace, uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  const qds_status st = qds_decay_forward_workspace(c, &need);
  if (st != QDS_OK) return st;
  if (c->batch == 0) return QDS_OK;
  if (!log_decay) return QDS_ERR_INVALID_ARG;
  if (c->length > 0 && (!usable(q) || !usable(k) || !usable(v) || !usable(o))) return QDS_ERR_INVALID_ARG;
  if (need && (!workspace || ((uintptr_t)workspace & 255))) return QDS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return QDS_ERR_WORKSPACE_TOO_SMALL;
  if (c->length > 0 && (!near_rows(q, c->length) || !near_rows(k, c->length) || !near_rows(v, c->length))) return QDS_ERR_UNSUPPORTED;
  DecayArgs a = decay_args(c, segment_plan(c, 1), lengths, log_decay);
  a.role[0] = Role{view(q), view(k), view(v), view(o), state_in, state_out, (float*)workspace, 1.0f, c->scale, false, false};
  run(c, a, 1, stream);
  return launch_status();
}

extern "C" qds_status qds_decay_backward_workspace(const qds_decay_config* c, uint64_t* bytes) {
  const qds_status st = validate(c);
  if (st != QDS_OK) return st;
  if (!bytes) return QDS_ERR_INVALID_ARG;
  *bytes = 3 * state_bytes(c, segment_plan(c, 3).segments);
  return QDS_OK;
}

extern "C" qds_status qds_decay_backward(const qds_decay_config* c, qds_view dout, qds_view q, qds_view k,
                                         qds_view v, const float* log_decay, const float* state_in,
                                         const float* dstate_out, const int32_t* lengths, qds_view dq,
                                         qds_view dk, qds_view dv, float* dstate_in, void* workspace,
                                         uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  const qds_status st = qds_decay_backward_workspace(c, &need);
  if (st != QDS_OK) return st;
  if (c->batch == 0) return QDS_OK;
  if (!log_decay) return QDS_ERR_INVALID_ARG;
  if (c->length > 0 && (!usable(dout) || !usable(q) || !usable(k) || !usable(v) || !usable(dq) ||
                        !usable(dk) || !usable(dv)))
    return QDS_ERR_INVALID_ARG;
  if (need && (!workspace || ((uintptr_t)workspace & 255))) return QDS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return QDS_ERR_WORKSPACE_TOO_SMALL;
  if (c->length > 0 && (!near_rows(dout, c->length) || !near_rows(q, c->length) || !near_rows(k, c->length) || !near_rows(v, c->length))) return QDS_ERR_UNSUPPORTED;
  const SegmentPlan p = segment_plan(c, 3);
  const uint64_t each = state_bytes(c, p.segments) / sizeof(float);
  float* ws = (float*)workspace;
  const Role rq{view(dout), view(v), view(k), view(dq), state_in, nullptr, ws, 1.0f, c->scale, false, true};
  const Role rk{view(v), view(dout), view(q), view(dk), dstate_out, nullptr, ws + each, c->scale, 1.0f, true, true};
  const Role rv{view(k), view(q), view(dout), view(dv), dstate_out, dstate_in, ws + 2 * each, c->scale, 1.0f, true, false};
  DecayArgs a = decay_args(c, p, lengths, log_decay);
  if (c->dim_k == c->dim_v) {
    a.role[0] = rq, a.role[1] = rk, a.role[2] = rv;
    run(c, a, 3, stream);
  } else {
    a.role[0] = rv;
    run(c, a, 1, stream);
    a.dim_x = c->dim_v, a.dim_z = c->dim_k;
    a.role[0] = rq, a.role[1] = rk;
    run(c, a, 2, stream);
  }
  return launch_status();
}

extern "C" qds_status qds_decay_step(const qds_decay_config* c, qds_view q, qds_view k, qds_view v,
                                     const float* log_decay, const float* state_in, qds_view o,
                                     float* state_out, void* stream) {
  const qds_status st = validate(c);
  if (st != QDS_OK) return st;
  if (c->batch == 0) return QDS_OK;
  if (!usable(q, false) || !usable(k, false) || !usable(v, false) || !usable(o, false) || !log_decay ||
      !state_in || !state_out || !aligned16(state_in) || !aligned16(state_out))
    return QDS_ERR_INVALID_ARG;
  const StepArgs a{view(q), view(k), view(v), view(o), log_decay, state_in, state_out, c->heads, c->dim_k, c->dim_v, c->scale};
  const uint32_t grid = (uint32_t)c->batch * c->heads;
  hipStream_t s = (hipStream_t)stream;
  const int dk = pad(c->dim_k), dv = pad(c->dim_v);
  auto go = [&](auto t) {
    using T = decltype(t);
    if (dk == 64 && dv == 64) k_decay_step<T, 64, 64><<<grid, 256, 0, s>>>(a);
    else if (dk == 64) k_decay_step<T, 64, 128><<<grid, 256, 0, s>>>(a);
    else if (dv == 64) k_decay_step<T, 128, 64><<<grid, 256, 0, s>>>(a);
    else k_decay_step<T, 128, 128><<<grid, 256, 0, s>>>(a);
  };
  if (c->dtype == QDS_BF16) go(bf16{});
  else go(half{});
  return launch_status();
}
