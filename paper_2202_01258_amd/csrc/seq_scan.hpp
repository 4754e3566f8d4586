// seq_scan.hpp -- what the forward and backward kernels of the selective scan share.
//
// A column's states are split among the four lanes of a quad, S each, so a wave has 16
// columns.  Rows are taken K at a time: lane q of a quad does what is done once for a row
// and column (step size, products, gate) for rows q, q + 4, ..., and gives it to the
// others by lane moves; rows of b and c, which all columns share, come through LDS.  An
// episode may be cut into segments that run side by side: a first pass forms what each
// segment leaves behind when it starts from zero, and the main pass starts each segment from
// its true state, which follows from what all segments in front of it left (the main pass
// works that out where they are few, a scan between the two where they are many).
#pragma once

#include <algorithm>

#include "seq_common.hpp"
#include "seq_rows.hpp"

namespace seq {

constexpr int kScanStates = 32;                  // at most

// Rows that the backward pass has at a time: it starts from the state in front of them ("mark"),
// which the forward pass leaves, and keeps their states in registers.  With 16 rows the marks take half
// the memory, but neither decays nor b and c fit beside the states.
constexpr int kScanRows = 8;
struct Rows {
  char* p;
  int64_t b, t;                                  // strides in elements
};
inline Rows rows(const qds_rows& r) { return Rows{(char*)r.data, r.stride[0], r.stride[1]}; }
template <class T> __device__ inline T* row_of(const Rows& r, int64_t b, int64_t t) {
  return (T*)r.p + b * r.b + t * r.t;
}

struct ScanArgs {
  Rows u, delta, b, c, gate, dout;
  void *o, *du, *ddelta, *dgate, *db, *dc;       // contiguous
  const float *a, *skip, *bias, *first, *dlast;
  float *last, *dfirst, *da, *dskip, *dbias;
  float* marks;                                  // [batch][blocks][width][4 S]
  float* left_state;                             // [batch][pieces][width][4 S]: left behind by a piece; after a scan, what it starts from
  float* left_time;                              // [batch][pieces][width]: sum of a piece's steps
  float* rows_part;                              // [batch][length][column blocks][2][4 S]: shares of db and dc
  float* cols_part;                              // [shares][width][4 S]: of da
  float* ends_part;                              // [shares][2][width]: of dskip and dbias
  float* saved;                                  // [threads of the main pass][2 S + 2]: of a block that is done again
  const int32_t* lengths;
  int32_t batch, length, width, states, blocks, col_blocks, shares;
  int32_t seg, segs;                             // rows of a segment of the main pass; segments
  int32_t piece, pieces, ratio;                  // rows of a piece of the first pass; pieces; pieces of a segment
  bool joined;                                   // a scan has run
};
// A kernel's arguments, its only ones, read anew: what is needed once for an episode's part is
// not kept in scalar registers.  Those are short: the backward pass kept 121 numbers in vector
// registers' lanes, and took them out within its rows (32 x 1000 x 512 with 16 states, forward and
// backward: 397 us so, 388 without).
__device__ inline const ScanArgs& read_args() {
  auto p = (const __attribute__((address_space(4))) ScanArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const ScanArgs*)p;
}
__device__ inline int rows_in(const ScanArgs& a, int64_t b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.length) : a.length;
}

// Episodes' parts in the order in which workgroups start: all episodes' first ones, then all
// second ones, another episode first each time.  Short episodes lack the late parts: dealt
// episode by episode, a compute unit had the same part of all its episodes (a ragged training
// pass of 32 x 1000 x 512: 1% more).
struct Item {
  int64_t b;
  int part;
  __device__ Item(uint32_t item, int batch)
      : b((item + item / (uint32_t)batch) % (uint32_t)batch), part((int)(item / (uint32_t)batch)) {}
};

// The value of lane J of this lane's quad, of lane q ^ 1, of lane q ^ 2.
template <int CTRL> __device__ inline float lane_move(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// A moved number is used by S instructions: kept from being merged into each of them, where it
// would make each take the time of a move (4.4 cycles against 2.7).
template <int J> __device__ inline float quad_lane(float v) {
  float r = lane_move<J * 0x55>(v);
  asm("" : "+v"(r));
  return r;
}
__device__ inline float quad_sum(float v) {
  v += lane_move<0xB1>(v);
  return v + lane_move<0x4E>(v);
}
// a where the mask's bits are set, b elsewhere; a select by a mask in scalar registers takes longer.
__device__ inline float pick(uint32_t mask, float a, float b) {
  return __uint_as_float(__builtin_amdgcn_bitop3_b32(mask, __float_as_uint(a), __float_as_uint(b), 0xca));
}
// Four rows' values in four lanes: lane q gets row q's sum over the quad.  odd and high: all bits
// set where bit 0 and bit 1 of q are.
struct Quad {
  uint32_t odd, high;
  __device__ explicit Quad(int q) : odd(q & 1 ? ~0u : 0), high(q & 2 ? ~0u : 0) {}
};
__device__ inline float quad_rows(const float* v, Quad m) {
  const float a = pick(m.odd, v[1], v[0]) + lane_move<0xB1>(pick(m.odd, v[0], v[1]));
  const float b = pick(m.odd, v[3], v[2]) + lane_move<0xB1>(pick(m.odd, v[2], v[3]));
  return pick(m.high, b, a) + lane_move<0x4E>(pick(m.high, a, b));
}

// log(1 + e^x): log(1 + e) is formed as log(w) e / (w - 1) with w = 1 + e as rounded, which takes w's rounding
// back where e is small; that leaves an error below 6 2^-24.  The exponent's own rounding adds |x| 2^-24 (10 2^-24 in
// all for steps of 0.001, 65 at e^-87, below which e is 0).  float32 takes that back as well; beside
// 16-bit numbers that would cost 1 x 65536 x 1024 504 us in place of 492 (32 x 1000 x 512, training: 390 and 385).
constexpr float kLog2eRest = (float)(1.4426950408889634 - (double)kLog2e);
struct Step {
  float dt, slope;                               // and its derivative, sigmoid(x)
};
template <class T> __device__ inline Step softplus(float x) {
  const float top = -kLog2e * fabsf(x);
  float e = fast_exp2(top);
  if constexpr (sizeof(T) == 4) {
    const float lost = fmaf(-kLog2eRest, fabsf(x), fmaf(-kLog2e, fabsf(x), -top));
    e = fmaf(e * __builtin_amdgcn_fmed3f(lost, -1.0f, 1.0f), kLn2, e);     // of an infinite x it is no number, and e is 0
  }
  const float w = 1.0f + e, back = w - 1.0f;
  const float log1 = back == 0.0f ? e : kLn2 * fast_log2(w) * e * __builtin_amdgcn_rcpf(back);
  const float r = __builtin_amdgcn_rcpf(w);
  return Step{(x > 0.0f ? x : 0.0f) + log1, x > 0.0f ? r : e * r};
}

// a in units of log 2, finite: rows behind an episode have dt = 0 and must leave the state alone.
__device__ inline float rate(float a) {
  const float x = a * kLog2e;
  return x < -0x1.fffffep127f ? -0x1.fffffep127f : x > 0x1.fffffep127f ? 0x1.fffffep127f : x;
}

// S neighbouring floats, aligned to them all where S allows.
template <int S> struct alignas(S * 4 > 16 ? 16 : S * 4) Floats { float v[S]; };
template <int S> __device__ inline void load_floats(float* out, const float* p) {
  const Floats<S> f = *reinterpret_cast<const Floats<S>*>(p);
#pragma unroll
  for (int s = 0; s < S; ++s) out[s] = f.v[s];
}
template <int S> __device__ inline void store_floats(float* p, const float* in) {
  Floats<S> f;
#pragma unroll
  for (int s = 0; s < S; ++s) f.v[s] = in[s];
  *reinterpret_cast<Floats<S>*>(p) = f;
}
// One number by a buffer access: a scalar base, the lane's offset and a scalar offset in bytes.
// From kOutside on a load gives 0 and a store does nothing.
template <class T> __device__ inline uint32_t get_bits(const char* base, uint32_t lane_at, uint32_t at) {
  const auto buffer = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, kBufferSize, kBufferFlags);
  if constexpr (sizeof(T) == 4) return __builtin_amdgcn_raw_buffer_load_b32(buffer, lane_at, at, 0);
  else return __builtin_amdgcn_raw_buffer_load_b16(buffer, lane_at, at, 0);
}
// The number that was loaded, a register each until here: left to itself the compiler joins two
// 16-bit numbers in one register as soon as they are loaded, and so waits for memory there.
template <class T> __device__ inline float number(uint32_t bits) {
  asm volatile("" : "+v"(bits));
  if constexpr (sizeof(T) == 4) return __uint_as_float(bits);
  else return to_f32(__builtin_bit_cast(T, (uint16_t)bits));
}
template <class T> __device__ inline void put(char* base, uint32_t lane_at, uint32_t at, T v) {
  const auto buffer = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, kBufferSize, kBufferFlags);
  if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), buffer, lane_at, at, 0);
  else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), buffer, lane_at, at, 0);
}

// The lane's states of column `at` in a tensor of the caller's, [..][width][states]; `p` is the
// same for the wave.
template <int S> __device__ inline void load_states(float* out, const float* p, int at, int q, int states) {
#pragma unroll
  for (int s = 0; s < S; ++s)
    out[s] = __uint_as_float(get_bits<float>((const char*)p, p && q * S + s < states ? (at * states + q * S) * 4u : kOutside, s * 4));
}
template <int S> __device__ inline void store_states(float* p, int at, int q, int states, bool in, const float* v) {
#pragma unroll
  for (int s = 0; s < S; ++s) put<float>((char*)p, in && q * S + s < states ? (at * states + q * S) * 4u : kOutside, s * 4, v[s]);
}

// Four lanes may hold more states than there are.  Those that are not there are 0 wherever states meet
// (their rate is -1, so that no step makes them anything else); b and c are 0 for them, which is
// not enough beside an infinite input or gradient.  Kernels for such counts (TAIL) look for one in
// each block of rows (13 states, 16 x 1000 x 1024: 395 us for a training pass, 385 without; outputs of 1 x
// 16384 x 1024: 137 and 134); masks on each state would be some 8 of a row's 97 instructions.
template <int S> struct Held {
  int count;                                     // of the lane's states
  __device__ Held(int q, int states) : count(states - q * S) {}
  __device__ float keep(int s, float v) const { return s < count ? v : 0.0f; }
  __device__ void keep_all(float* v) const {
#pragma unroll
    for (int s = 0; s < S; ++s) v[s] = keep(s, v[s]);
  }
};
template <int S> __device__ inline void load_rates(float* out, const ScanArgs& a, int at, int q) {
  load_states<S>(out, a.a, at, q, a.states);
  const Held<S> held(q, a.states);
#pragma unroll
  for (int s = 0; s < S; ++s) out[s] = s < held.count ? rate(out[s]) : -1.0f;
}
// Whether one of a wave's numbers is 2^EXPONENT or more, or not a number.
template <int EXPONENT, class... F> __device__ inline bool any_from(F... v) {
  uint32_t top = 0;
  ((top = max(top, __float_as_uint(v) & 0x7fffffffu)), ...);
  return __builtin_amdgcn_ballot_w64(top >= (EXPONENT + 127u) << 23) != 0;
}

// Which of a block's rows q, q + 4, ... an episode still has: rows left, less one, counted from a
// lane's first.  Below 0 from a row on, where the sign bit makes an offset kOutside.
struct Left {
  int x;
  __device__ int at(int i) const { return x - 4 * i; }
  __device__ float keep(int i, float v) const { return __uint_as_float(__float_as_uint(v) & ~(uint32_t)(at(i) >> 31)); }
  __device__ uint32_t offset(int i, uint32_t lane_at) const { return lane_at | ((uint32_t)at(i) & kOutside); }
};

// A tensor's rows t + q, t + 4 + q, ... at a lane's column, t a scalar that goes up or down: an
// access costs one vector instruction beside it and no 64-bit arithmetic.  Rows are from 0 to
// less than 2^23 elements apart.  Columns that are not real are outside.
template <class T> struct Track {
  char* p;                                       // of row t
  uint32_t step, lane_at;                        // bytes: from row to row, and the lane's
  __device__ Track(const void* base, int64_t batch_stride, int64_t row_stride, int64_t b, int t, int q, int at, bool real) {
    step = (uint32_t)row_stride * sizeof(T);
    p = (char*)base + b * batch_stride * (int64_t)sizeof(T) + (int64_t)t * step;
    lane_at = real ? q * step + at * (uint32_t)sizeof(T) : kOutside;
  }
  __device__ Track(const Rows& r, int64_t b, int t, int q, int at, bool real) : Track(r.p, r.b, r.t, b, t, q, at, real) {}
  __device__ void move(int rows) { p += (int64_t)rows * step; }
  // a multiple of the step, formed where it is needed: scalar registers are short, too
  __device__ uint32_t ahead(int i) const {
    uint32_t s = step;
    if (i > 0) asm volatile("" : "+s"(s));
    return 4 * i * s;
  }
  __device__ uint32_t load(int i, Left left) const { return get_bits<T>(p, left.offset(i, lane_at), ahead(i)); }
  __device__ void store(int i, Left left, float v) const { put<T>(p, left.offset(i, lane_at), ahead(i), from_f32<T>(v)); }
};

// K rows of b and c on their way to LDS: [K][2][4 S], what is behind the episode or the states is 0.
// A wave has rows of b or of c, not of both, so that its base is a scalar.
template <class T, int S, int K, int BLOCK> struct StagedRows {
  static constexpr int N = 4 * S, PART = (K * N + 63) / 64 * 64, EACH = (2 * PART + BLOCK - 1) / BLOCK;
  const char* p[EACH];
  uint32_t step[EACH], lane_at[EACH];
  uint32_t v[EACH];
  __device__ StagedRows(const ScanArgs& a, int64_t b, int t) {
    const int wave = wave_index() * 64;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int k = (threadIdx.x + i * BLOCK) % PART;
      const bool first = wave + i * BLOCK < PART;
      const int64_t stride = first ? a.b.t : a.c.t, batch = first ? a.b.b : a.c.b;
      step[i] = (uint32_t)stride * sizeof(T);
      p[i] = (first ? a.b.p : a.c.p) + b * batch * (int64_t)sizeof(T) + (int64_t)t * step[i];
      lane_at[i] = k < K * N && k % N < a.states ? k / N * step[i] + k % N * (uint32_t)sizeof(T) : kOutside;
    }
  }
  __device__ void load(int rows) {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      int k = (threadIdx.x + i * BLOCK) % PART;
      asm volatile("" : "+v"(k));                // its row is not kept
      v[i] = get_bits<T>(p[i], lane_at[i] | ((uint32_t)(rows - 1 - k / N) & kOutside), 0);
    }
  }
  __device__ void move(int rows) {
#pragma unroll
    for (int i = 0; i < EACH; ++i) p[i] += (int64_t)rows * step[i];
  }
  __device__ void store(float* lds) const {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int id = threadIdx.x + i * BLOCK, k = id % PART;
      if (id < 2 * PART && k < K * N) lds[(k / N * 2 + id / PART) * N + k % N] = number<T>(v[i]);
    }
  }
};

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
inline qds_status validate_scan(const qds_scan_config* c, bool step) {
  if (!c || c->abi_version != QDS_ABI_VERSION) return QDS_ERR_INVALID_ARG;
  if (c->dtype < QDS_F32 || c->dtype > QDS_F16) return QDS_ERR_INVALID_ARG;
  if (c->batch < 0 || (!step && (c->length < 0 || c->length >= (1 << 30)))) return QDS_ERR_INVALID_ARG;
  if (c->width < 1 || c->width > (1 << 20) || c->states < 1) return QDS_ERR_INVALID_ARG;
  if (c->states > kScanStates) return QDS_ERR_UNSUPPORTED;
  return QDS_OK;
}
// Rows that a scan reads are from 0 to less than 2^23 elements apart (a single row's stride
// means nothing and is set to 0).
inline bool near_rows(qds_rows& r, int length) {
  if (length < 2) r.stride[1] = 0;
  return !r.data || (r.stride[1] >= 0 && r.stride[1] < (1 << 23));
}
inline int lane_states(const qds_scan_config* c) { return c->states <= 4 ? 1 : c->states <= 8 ? 2 : c->states <= 16 ? 4 : 8; }
inline int mark_count(const qds_scan_config* c) { return (int)ceil_div(c->length, kScanRows); }

// The root of what rows with a sum of steps `time` multiply a state by: all of it need not be a float, and
// what is 0 or infinite stays so.  Limited to where neither half is infinite or 0: beyond, a number
// comes to infinity by 2^254, or to less than 2^-124 by 2^-252.  No rows: 1, whatever the rate.
__device__ inline float half_decay(float time, float rate) {
  const float half = fast_exp2(__builtin_amdgcn_fmed3f(0.5f * time * rate, -126.0f, 127.0f));
  return time == 0.0f ? 1.0f : half;
}

// What all pieces before `until` leave together when the first starts from x (the pieces in their
// order, or from the last one backwards).
template <int S, bool BACK> __device__ inline void follow(float* x, const ScanArgs& a, const float* rates, int64_t b, int until, int at, int q) {
  constexpr int N = 4 * S;
  const int first = BACK ? a.pieces - 1 : 0, count = BACK ? a.pieces - until : until;
  const float* state = a.left_state + (b * a.pieces + first) * a.width * N + (uint32_t)(at * N + q * S);
  const float* time = a.left_time + (b * a.pieces + first) * a.width + at;
#pragma unroll 4
  for (int i = 0; i < count; ++i) {
    const int64_t to = (int64_t)(BACK ? -i : i) * a.width;
    float left[S];
    load_floats<S>(left, state + to * N);
    const float t = time[to];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const float half = half_decay(t, rates[s]);
      x[s] = fmaf(x[s] * half, half, left[s]);
    }
  }
}

// The same for many pieces: puts what each starts from in its place.  Sixteen states per workgroup, whose
// pieces are dealt to sixteen groups of threads: each forms what its share does to any x, then, from
// what the groups before it do, what its own pieces start from.
constexpr int kScanJoin = 256;
template <int N, bool BACK> __global__ __launch_bounds__(kScanJoin) void k_scan_join(ScanArgs a) {
  __shared__ float shares[2][16][16];
  const int i = threadIdx.x & 15, group = threadIdx.x >> 4;
  const int64_t id = (int64_t)blockIdx.x * 16 + i, column = id / N, all = (int64_t)a.batch * a.width;
  const int n = (int)(id % N);
  const bool real = column < all, in = real && n < a.states;
  const int64_t b = real ? column / a.width : 0;
  const int at = real ? (int)(column % a.width) : 0;
  const float r = in ? rate(a.a[(int64_t)at * a.states + n]) : -1.0f;
  // pieces with something left behind, in their order; one more starts behind the last
  const int count = BACK ? a.pieces - a.ratio : a.pieces - 1, share = (count + 15) / 16;
  const int from = min(group * share, count), to = min(from + share, count);
  auto place = [&](int k) { return (b * a.pieces + (BACK ? a.pieces - 1 - k : k)) * a.width + at; };
  float time = 0.0f, left = 0.0f;
  if (real) {
#pragma unroll 4
    for (int k = from; k < to; ++k) {
      const int64_t where = place(k);
      const float t = a.left_time[where], half = half_decay(t, r);
      left = fmaf(left * half, half, a.left_state[where * N + n]);
      time += t;
    }
  }
  shares[0][group][i] = time;
  shares[1][group][i] = left;
  __syncthreads();
  if (!real) return;
  const float* first = BACK ? a.dlast : a.first;
  float x = in && first ? first[column * a.states + n] : 0.0f;
  for (int g = 0; g < group; ++g) {
    const float half = half_decay(shares[0][g][i], r);
    x = fmaf(x * half, half, shares[1][g][i]);
  }
#pragma unroll 4
  for (int k = from; k < to; ++k) {
    const int64_t where = place(k);
    const float gone = a.left_state[where * N + n], half = half_decay(a.left_time[where], r);
    a.left_state[where * N + n] = x;
    x = fmaf(x * half, half, gone);
  }
  if (to == count && (from < to || group == 0)) a.left_state[place(count) * N + n] = x;
}

// Waves of a pass over whole episodes.
inline int64_t whole_waves(const qds_scan_config* c) { return std::max<int64_t>(1, (int64_t)c->batch * ceil_div(c->width, 16)); }

// Rows of a segment and their number, for a kernel that wants `waves` waves.
struct Cut {
  int seg, segs;
};
inline Cut cut(const qds_scan_config* c, int64_t waves, int least, int unit) {
  const int64_t want = std::max<int64_t>(1, waves / whole_waves(c));
  int64_t seg = std::max<int64_t>(least, ceil_div(c->length, want));
  seg = ceil_div(seg, unit) * unit;
  return Cut{(int)seg, (int)std::max<int64_t>(1, ceil_div(c->length, seg))};
}
constexpr int kFewPieces = 32;                   // so many are followed by the main pass itself
// Whether the launch that joins more of them can be made: only few columns are cut so far.
inline bool joinable(const qds_scan_config* c, int pieces) {
  return pieces <= kFewPieces || ceil_div((int64_t)c->batch * c->width * 4 * lane_states(c), 16) <= most_blocks(kScanJoin);
}

template <class F> void scan_instance(const qds_scan_config* c, F&& f) {
  auto with_tail = [&](auto type, auto S) {
    if (c->states == 4 * decltype(S)::value) f(type, S, std::false_type{});
    else f(type, S, std::true_type{});
  };
  auto with_type = [&](auto S) {
    if (c->dtype == QDS_F32) with_tail(float(), S);
    else if (c->dtype == QDS_BF16) with_tail(bf16(), S);
    else with_tail(half(), S);
  };
  switch (lane_states(c)) {
    case 1: return with_type(Int<1>{});
    case 2: return with_type(Int<2>{});
    case 4: return with_type(Int<4>{});
    default: return with_type(Int<8>{});
  }
}

inline ScanArgs scan_args(const qds_scan_config* c) {
  ScanArgs a{};
  a.batch = c->batch;
  a.length = c->length;
  a.width = c->width;
  a.states = c->states;
  a.blocks = mark_count(c);
  return a;
}

}  // namespace seq
