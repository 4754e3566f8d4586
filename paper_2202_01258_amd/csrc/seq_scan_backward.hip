// seq_scan_backward.hip -- gradients of the selective state space scan.  The C ABI is in
// include/qd_seq.h, the layout of the work in seq_scan.hpp.
//
// Bound by the vector units: 97 vector instructions for a row of 16 columns and 16 states.  In 32 episodes of up
// to 1000 rows x 512 bfloat16 (184 us under the tracer) they are issued in 88% of the time in which a SIMD has its two
// waves, and in 73% of the kernel's: episodes that end leave places that are not filled.  Two waves a SIMD is what
// the states in registers leave; three, with fewer of them kept, took 1.07 of the time.
#include <algorithm>

#include "seq_scan.hpp"

namespace seq {
namespace {

constexpr int kJoinBlock = 256;

// With m_t = e^(dt_{t+1} a) dh_{t+1}, what reaches row t from the rows behind it:
//   dh = m_t + dy_t c_t;  m_{t-1} = e^(dt_t a) dh.
// One piece of 64 columns from its last row to its first, from zero: what it leaves to the
// piece before, and the sum of its steps.
template <class T, int S, bool GATE> __global__ __launch_bounds__(256) void k_scan_back(ScanArgs a) {
  constexpr int K = S <= 4 ? 16 : 8, N = 4 * S, QUADS = K / 4, BLOCK = 256;
  SEQ_SHARED float bc[2][K * 2 * N];
  const int q = threadIdx.x & 3, blocks = (a.width + 63) / 64;
  const uint32_t item = blockIdx.x / (uint32_t)blocks;
  const int col = (blockIdx.x % (uint32_t)blocks) * 64 + (threadIdx.x >> 2);
  const bool real = col < a.width;
  const int at = real ? col : a.width - 1;
  const Item which(item, a.batch);
  const int64_t b = which.b;
  const int piece = a.ratio + which.part;                         // no segment asks what the first one's pieces leave
  const int n = rows_in(a, b), begin = piece * a.piece, end = min(begin + a.piece, a.length), live = min(end, n);
  float rates[S], m[S], time = 0.0f;
  load_rates<S>(rates, a, at, q);
#pragma unroll
  for (int s = 0; s < S; ++s) m[s] = 0.0f;
  const float bias = a.bias ? a.bias[at] : 0.0f;
  if (begin < live) {
    uint32_t d[QUADS], g[QUADS], z[QUADS];
    const int last = begin + (live - 1 - begin) / K * K;
    Track<T> td(a.delta, b, last, q, at, real), tg(a.dout, b, last, q, at, real), tz(a.gate, b, last, q, at, real);
    StagedRows<T, S, K, BLOCK> rows(a, b, last);
    auto fetch = [&](int t) {
      const Left left{live - t - q - 1};
#pragma unroll
      for (int i = 0; i < QUADS; ++i) {
        d[i] = td.load(i, left);
        g[i] = tg.load(i, left);
        if (GATE) z[i] = tz.load(i, left);
      }
      rows.load(live - t);
      td.move(-K);
      tg.move(-K);
      if (GATE) tz.move(-K);
      rows.move(-K);
    };
    fetch(last);
    rows.store(bc[0]);
    __syncthreads();
    int buffer = 0;
    for (int t = last; t >= begin; t -= K) {
      const Left left{live - t - q - 1};
      float dt[QUADS], dy[QUADS];
#pragma unroll
      for (int i = 0; i < QUADS; ++i) {
        dt[i] = left.keep(i, softplus<T>(number<T>(d[i]) + bias).dt);
        dy[i] = number<T>(g[i]);
        if (GATE) {
          const float zz = number<T>(z[i]);
          dy[i] *= zz * sigmoid(zz);
        }
        time += dt[i];
      }
      const bool more = t > begin;
      if (more) fetch(t - K);
      const float* lds = bc[buffer] + N + q * S;
#pragma unroll
      for (int i = QUADS - 1; i >= 0; --i) {
        auto row = [&](auto J) {
          constexpr int j = decltype(J)::value;
          const float dtj = quad_lane<j>(dt[i]), dyj = quad_lane<j>(dy[i]);
          float cv[S];
          load_floats<S>(cv, lds + (4 * i + j) * 2 * N);
#pragma unroll
          for (int s = 0; s < S; ++s) m[s] = fast_exp2(dtj * rates[s]) * fmaf(dyj, cv[s], m[s]);
        };
        row(Int<3>{});
        row(Int<2>{});
        row(Int<1>{});
        row(Int<0>{});
        __builtin_amdgcn_sched_barrier(0);
      }
      if (more) {
        rows.store(bc[buffer ^ 1]);
        __syncthreads();
        buffer ^= 1;
      }
    }
  }
  time = quad_sum(time);
  Held<S>(q, a.states).keep_all(m);
  if (real) store_floats<S>(a.left_state + ((b * a.pieces + piece) * a.width + at) * N + q * S, m);
  if (real && q == 0) a.left_time[(b * a.pieces + piece) * a.width + at] = time;
}

// Sums over a wave's 16 columns of four rows' terms of db and dc, through LDS: each lane leaves
// its S terms of a row where they are read by two lanes for each (row, b or c, states of a lane),
// eight columns each.  Added in registers, by moves between lanes, they took 87 cycles of a
// wave's row; here it is two writes, two reads and ten additions.
template <int S> struct ColumnSums {
  static constexpr int N = 4 * S;
  static constexpr int PAD = 68 * S;             // 64 lanes, and as much as sets the rows' reads in other banks
  float* own;                                    // [4 rows][2][68][S]
  __device__ explicit ColumnSums(float* lds) : own(lds) {}
  __device__ void leave(int row, int which, const float* v) const {
    store_floats<S>(own + (row * 2 + which) * PAD + (threadIdx.x & 63) * S, v);
  }
  // The reads of a join, to be waited for as late as possible; then the sums, to part[row][2][4 S].
  struct Reads {
    float v[8][S];
    int to;
  };
  __device__ Reads read() const {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    int l = threadIdx.x & 63;
    asm volatile("" : "+v"(l));                  // what follows from it is not kept from call to call
    const int half = l & 1, q = (l >> 1) & 3, which = (l >> 3) & 1, row = l >> 4;
    const int from = (row * 2 + which) * PAD + (half * 32 + q) * S;
    Reads r;
    r.to = row * 2 * N + which * N + q * S;
#pragma unroll
    for (int i = 0; i < 8; ++i) load_floats<S>(r.v[i], own + from + i * 4 * S);
    return r;
  }
  __device__ static void join(const Reads& r, float* part) {
    float sum[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      sum[s] = ((r.v[0][s] + r.v[1][s]) + (r.v[2][s] + r.v[3][s])) + ((r.v[4][s] + r.v[5][s]) + (r.v[6][s] + r.v[7][s]));
      sum[s] += lane_move<0xB1>(sum[s]);
    }
    if ((threadIdx.x & 1) == 0) store_floats<S>(part + r.to, sum);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
};

// A thread's column and quarter of its states, formed anew at each call: offsets that only the
// ends of an episode need are not kept in registers throughout.
struct Place {
  int q, at;
  bool real;
  __device__ Place(int width, int first) {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    q = t & 3;
    at = first + (t >> 2);
    real = at < width;
    at = real ? at : width - 1;
  }
};

// The largest magnitude of three; a number that is none does not count.
__device__ inline float largest(float a, float b, float c) {
  asm("v_max3_f32 %0, |%1|, |%2|, |%0|" : "+v"(a) : "v"(b), "v"(c));
  return a;
}

// A place in memory for what a thread has of a block that is done again: gradients from behind, sums.
using Saved = __attribute__((address_space(1))) float;
template <int S> __device__ inline Saved* saved_at() {
  Saved* p = (Saved*)read_args().saved + ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * (2 * S + 2);
  asm volatile("" : "+v"(p));                    // what is saved is not kept in registers as well
  return p;
}

// Whether a block's states and gradients may reach 2^127, its steps and inputs being below 2^16; states
// whose rate is above 0 may.
template <int S> __device__ inline bool may_overflow(const float* first, const float* m, const float* rates, const float* lds) {
  constexpr int N = 4 * S;
  bool odd = false;
#pragma unroll
  for (int s = 0; s < S; ++s) odd |= any_from<50>(first[s], m[s]) || any_from<16>(rates[s] > 0.0f ? __builtin_inff() : 0.0f);
#pragma unroll 1
  for (int k = 0; k < kScanRows; ++k) {
    float b[S];
    load_floats<S>(b, lds + k * 2 * N);
#pragma unroll
    for (int s = 0; s < S; ++s) odd |= any_from<16>(b[s]);
  }
  return odd;
}

// A block's rows, from t on, a row at a time and only what is there, for numbers that need not be finite.
// Slow (each row forms all states in front of it), and short: it takes no registers from the usual way.
template <class T, int S, bool GATE> __device__ inline void by_rows(uint32_t item, int t, int first_col, const float* lds,
                                                                    const float* rates, float bias, float skip, float* m,
                                                                    float* da, float& dskip, float& dbias,
                                                                    const ColumnSums<S>& sums, float* part) {
  constexpr int K = kScanRows, N = 4 * S;
  const ScanArgs& a = read_args();
  const int64_t b = Item(item, a.batch).b;
  const Place place(a.width, first_col);
  const int q = place.q, at = place.at, rows = place.real ? rows_in(a, b) - t : 0;
  const Held<S> held(q, a.states);
  const float* first = a.marks + (b * a.blocks + t / K) * a.width * N + (uint32_t)(at * N + q * S);
#pragma unroll 1
  for (int k = K - 1; k >= 0; --k) {
    float before[S], after[S], bv[S], cv[S], tb[S], tc[S], u = 0.0f;
    Step step{0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < S; ++s) after[s] = place.real ? first[s] : 0.0f;
#pragma unroll 1
    for (int r = 0; r <= k; ++r) {
      u = r < rows ? to_f32(row_of<T>(a.u, b, t + r)[at]) : 0.0f;
      step = softplus<T>(r < rows ? to_f32(row_of<T>(a.delta, b, t + r)[at]) + bias : 0.0f);
      if (r >= rows) step.dt = 0.0f;
      load_floats<S>(bv, lds + r * 2 * N);
#pragma unroll
      for (int s = 0; s < S; ++s) {
        before[s] = after[s];
        after[s] = held.keep(s, fmaf(fast_exp2(step.dt * rates[s]), after[s], step.dt * u * bv[s]));
      }
    }
    const bool in = k < rows;
    const float g = in ? to_f32(row_of<T>(a.dout, b, t + k)[at]) : 0.0f;
    const float z = GATE && in ? to_f32(row_of<T>(a.gate, b, t + k)[at]) : 0.0f;
    const float dy = GATE ? g * (z * sigmoid(z)) : g;
    float along = 0.0f, te = 0.0f, y = 0.0f;
    load_floats<S>(cv, lds + k * 2 * N + N);
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const float dh = held.keep(s, fmaf(dy, cv[s], m[s]));
      tb[s] = dh * (step.dt * u);
      tc[s] = dy * after[s];
      along = fmaf(dh, bv[s], along);
      y = fmaf(after[s], cv[s], y);
      m[s] = dh * fast_exp2(step.dt * rates[s]);
      const float f = m[s] * before[s];
      da[s] = in ? fmaf(f, step.dt, da[s]) : da[s];
      te = fmaf(f, rates[s], te);
    }
    sums.leave(k & 3, 0, tb);
    sums.leave(k & 3, 1, tc);
    along = quad_sum(along);
    te = quad_sum(te);
    y = fmaf(skip, u, quad_sum(y));
    if (in && q == (k & 3)) {
      const int64_t to = (b * a.length + t + k) * a.width + at;
      const float raw = fmaf(along, u, te * kLn2) * step.slope;
      dskip = fmaf(dy, u, dskip);
      dbias += raw;
      ((T*)a.du)[to] = from_f32<T>(fmaf(along, step.dt, skip * dy));
      ((T*)a.ddelta)[to] = from_f32<T>(raw);
      if (GATE) ((T*)a.dgate)[to] = from_f32<T>(g * y * silu_slope(z, sigmoid(z)));
    }
    if ((k & 3) == 0) sums.join(sums.read(), part + k * 2 * N);
  }
}

// All gradients.  A workgroup has COLS columns and goes through every `shares`-th segment, each
// from its last block of rows to its first: a block's states and decays are formed again from
// its mark and kept in registers for the way back.
template <class T, int S, int COLS, bool GATE, bool TAIL> __global__ __launch_bounds__(COLS * 4, 2) void k_scan_backward(ScanArgs args) {
  constexpr int K = kScanRows, N = 4 * S, QUADS = K / 4, BLOCK = COLS * 4, WAVES = BLOCK / 64;
  constexpr bool KEEP = S <= 4;                                     // decays for the way back; else they are formed again
  SEQ_SHARED float bc[2][K * 2 * N];
  // one place only where LDS is short: a barrier more keeps its readers and writers apart
  constexpr int PARTS = S <= 4 ? 2 : 1;
  SEQ_SHARED float part[PARTS][WAVES][K * 2 * N];
  SEQ_SHARED float terms[WAVES][4 * 2 * ColumnSums<S>::PAD];
  const int wave = wave_index();
  const ColumnSums<S> sums(terms[wave]);
  const int block = blockIdx.x % (uint32_t)args.col_blocks;
  const uint32_t share = blockIdx.x / (uint32_t)args.col_blocks;
  const Place place(args.width, block * COLS);
  const int q = place.q, at = place.at;
  const bool real = place.real;
  const Quad quad(q);
  float rates[S], da[S], dskip = 0.0f, dbias = 0.0f;
  load_rates<S>(rates, args, at, q);
#pragma unroll
  for (int s = 0; s < S; ++s) da[s] = 0.0f;
  const float bias = args.bias ? args.bias[at] : 0.0f, skip = args.skip ? args.skip[at] : 0.0f;
  int buffer = 0;
  uint32_t item = share;
  while (true) {
    const ScanArgs& a = read_args();
    if (item >= (uint32_t)(a.batch * a.segs)) break;
    const Item which(item, a.batch);
    const int64_t b = which.b;
    const int seg = which.part;
    const int n = rows_in(a, b), begin = seg * a.seg, end = min(begin + a.seg, a.length), live = min(end, n);
    float m[S];
    auto enter = [&] {
      const Place entry(a.width, block * COLS);
      const int behind = min((seg + 1) * a.ratio, a.pieces);          // the first piece behind this segment
      if (a.joined) {
        load_floats<S>(m, a.left_state + (b * a.pieces + behind - 1) * a.width * N + (uint32_t)(entry.at * N + entry.q * S));
      } else {
        load_states<S>(m, a.dlast ? a.dlast + b * a.width * a.states : nullptr, entry.at, entry.q, a.states);
        follow<S, true>(m, a, rates, b, behind, entry.at, entry.q);
      }
#pragma unroll
      for (int s = 0; s < S; ++s) m[s] = real ? m[s] : 0.0f;         // columns that are not real add nothing to db and dc
    };
    if (begin >= live) {
      if (seg == 0) enter();                                          // an episode without rows hands its gradient through
    } else {
      uint32_t u[QUADS], d[QUADS], z[QUADS], g[QUADS];
      float first[S];
      const int last = begin + (live - 1 - begin) / K * K;
      Track<T> tu(a.u, b, last, q, at, real), td(a.delta, b, last, q, at, real), tg(a.dout, b, last, q, at, real),
          tz(a.gate, b, last, q, at, real);
      StagedRows<T, S, K, BLOCK> rows(a, b, last);
      const float* mark = a.marks + (b * a.blocks + last / K) * a.width * N;
      auto fetch = [&](int t) {
        const Left left{live - t - q - 1};
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
          u[i] = tu.load(i, left);
          d[i] = td.load(i, left);
          g[i] = tg.load(i, left);
          if (GATE) z[i] = tz.load(i, left);
        }
        load_floats<S>(first, mark + (uint32_t)(at * N + q * S));
        rows.load(live - t);
        tu.move(-K);
        td.move(-K);
        tg.move(-K);
        if (GATE) tz.move(-K);
        rows.move(-K);
        mark -= (int64_t)a.width * N;
      };
      const int64_t whole = (int64_t)a.length * a.width;
      Track<T> du(a.du, whole, a.width, b, last, q, at, real);          // ddelta and dgate lie alike
      char *ddelta = (char*)a.ddelta + (du.p - (char*)a.du), *dgate = (char*)a.dgate + (du.p - (char*)a.du);
      float* to = a.rows_part + ((b * a.length + last) * a.col_blocks + block) * 2 * N;
      // The waves' sums of a block from t on, in their order, and on to the block before.
      auto end_block = [&](int t) {
#pragma unroll
        for (int i = 0; i < (K * 2 * N + BLOCK - 1) / BLOCK; ++i) {
          const int k = threadIdx.x + i * BLOCK, r = t + k / (2 * N);
          if (k < K * 2 * N && r < live) {
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sum += part[buffer % PARTS][w][k];
            to[(int64_t)(k / (2 * N)) * a.col_blocks * 2 * N + k % (2 * N)] = sum;
          }
        }
        du.move(-K);
        ddelta -= (int64_t)K * du.step;
        dgate -= (int64_t)K * du.step;
        to -= (int64_t)K * a.col_blocks * 2 * N;
      };
      fetch(last);
      enter();                                   // while the first block is on its way
      rows.store(bc[buffer]);
      __syncthreads();
      int t = last;
      // Rows behind the episode, which only the last block has, take part with steps of 0: not where a
      // state or a gradient may be infinite.  (In front of the blocks: with the choice among them, the usual
      // way took 1.02 to 1.11 of its time.  16 x 1000 x 1024: 16 states 385 us as without, 32 states 728 and 716.)
      bool odd_end = false;
      if (t + K > live) {
        odd_end = may_overflow<S>(first, m, rates, bc[buffer] + q * S) ||
                  any_from<16>(number<T>(u[0]), number<T>(u[1]), number<T>(d[0]) + bias, number<T>(d[1]) + bias);
        terms[wave][0] = odd_end ? 1.0f : 0.0f;             // the waves go the same way
        __syncthreads();
        float any = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) any += terms[w][0];
        odd_end = __builtin_amdgcn_readfirstlane(any > 0.0f);
        __syncthreads();
      }
      if (odd_end) {
        by_rows<T, S, GATE>(item, t, block * COLS, bc[buffer] + q * S, rates, bias, skip, m, da, dskip, dbias, sums,
                            part[buffer % PARTS][wave]);
        if (t > begin) {
          fetch(t - K);
          rows.store(bc[buffer ^ 1]);
        }
        __syncthreads();
        end_block(t);
        __syncthreads();
        buffer ^= 1;
        t -= K;
      }
      for (; t >= begin; t -= K) {
        const Left left{live - t - q - 1};
        const float* lds = bc[buffer] + q * S;
        // States that are not there take part with factors of 0, which is not enough beside infinities: a
        // block that may come to any is done again, a row at a time.
        float gd[QUADS], gu[QUADS], gg[QUADS], gz[QUADS];           // the numbers as they were read
        bool odd = false;
        if (TAIL) {
          float top = bias;
#pragma unroll
          for (int i = 0; i < QUADS; ++i) {
            gd[i] = number<T>(d[i]);
            gu[i] = number<T>(u[i]);
            gg[i] = number<T>(g[i]);
            gz[i] = GATE ? number<T>(z[i]) : 0.0f;
            top = largest(largest(top, gd[i], gu[i]), gg[i], gz[i]);
          }
          odd = __builtin_amdgcn_ballot_w64(top >= 0x1p60f) != 0;
        }
        if (__builtin_expect(odd, 0)) {
          Saved* p = saved_at<S>();
#pragma unroll
          for (int s = 0; s < S; ++s) {
            p[s] = m[s];
            p[S + s] = da[s];
          }
          p[2 * S] = dskip;
          p[2 * S + 1] = dbias;
        }
        float h[K + 1][S], e[KEEP ? K : 1][S];                      // h[r]: in front of row r; e[r]: its decay
        float dt[QUADS], slope[QUADS], uu[QUADS], dy[QUADS];
        float kb[KEEP ? K : 1][S], kc[KEEP ? K : 1][S];             // the block's b and c, where registers allow
        if (KEEP) {
#pragma unroll
          for (int k = 0; k < K; ++k) {
            load_floats<S>(kb[k], lds + k * 2 * N);
            load_floats<S>(kc[k], lds + k * 2 * N + N);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int s = 0; s < S; ++s) h[0][s] = real ? first[s] : 0.0f;
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
          if (!TAIL) gd[i] = number<T>(d[i]);
          const Step step = softplus<T>(gd[i] + bias);
          dt[i] = left.keep(i, real ? step.dt : 0.0f);
          slope[i] = step.slope;
          uu[i] = TAIL ? gu[i] : number<T>(u[i]);
          const float x = dt[i] * uu[i];
          float y[4];
          auto row = [&](auto J) {
            constexpr int j = decltype(J)::value;
            const int k = 4 * i + j;
            const float dtj = quad_lane<j>(dt[i]), xj = quad_lane<j>(x);
            float bv[S], cv[S];
            if (!KEEP) load_floats<S>(bv, lds + k * 2 * N);
            if (!KEEP && GATE) load_floats<S>(cv, lds + k * 2 * N + N);
#pragma unroll
            for (int s = 0; KEEP && s < S; ++s) {
              bv[s] = kb[k][s];
              cv[s] = kc[k][s];
            }
#pragma unroll
            for (int s = 0; s < S; ++s) {
              const float decay = fast_exp2(dtj * rates[s]);
              if (KEEP) e[4 * i + j][s] = decay;
              h[4 * i + j + 1][s] = fmaf(decay, h[4 * i + j][s], xj * bv[s]);
              if (GATE) y[j] = s == 0 ? h[4 * i + j + 1][s] * cv[s] : fmaf(h[4 * i + j + 1][s], cv[s], y[j]);
            }
          };
          row(Int<0>{});
          row(Int<1>{});
          row(Int<2>{});
          row(Int<3>{});
          const float out = TAIL ? gg[i] : number<T>(g[i]);
          dy[i] = out;
          if (GATE) {
            const float zz = TAIL ? gz[i] : number<T>(z[i]), s = sigmoid(zz);
            dy[i] = out * (zz * s);
            const float yy = fmaf(skip, uu[i], quad_rows(y, quad));
            put<T>(dgate, left.offset(i, du.lane_at), du.ahead(i), from_f32<T>(out * yy * silu_slope(zz, s)));
          }
          asm volatile("" : "+v"(slope[i]));     // now, not where it is used: its parts take more registers
          __builtin_amdgcn_sched_barrier(0);     // no reads of later rows before these are done
        }
        const bool more = t > begin;
        if (KEEP && more) fetch(t - K);
        // b and c are read and steps are moved again: kept from above they would take as many
        // registers as the states
        int again = q * S;
        asm volatile("" : "+v"(again));
        lds = bc[buffer] + again;
#pragma unroll
        for (int i = 0; i < QUADS; ++i) asm volatile("" : "+v"(dt[i]));
        Left rest = left;
        asm volatile("" : "+v"(rest.x));
#pragma unroll
        for (int i = QUADS - 1; i >= 0; --i) {
          const float x = dt[i] * uu[i];
          float along[4], te[4];
          auto row = [&](auto J) {
            constexpr int j = decltype(J)::value;
            const float dtj = quad_lane<j>(dt[i]), xj = quad_lane<j>(x), dyj = quad_lane<j>(dy[i]);
            const int k = 4 * i + j;
            float bv[S], cv[S], tb[S], tc[S];
            if (!KEEP) load_floats<S>(bv, lds + k * 2 * N);
            if (!KEEP) load_floats<S>(cv, lds + k * 2 * N + N);
#pragma unroll
            for (int s = 0; KEEP && s < S; ++s) {
              bv[s] = kb[k][s];
              cv[s] = kc[k][s];
            }
#pragma unroll
            for (int s = 0; s < S; ++s) {
              const float dh = fmaf(dyj, cv[s], m[s]);
              tb[s] = dh * xj;
              tc[s] = dyj * h[k + 1][s];
              along[j] = s == 0 ? dh * bv[s] : fmaf(dh, bv[s], along[j]);
              m[s] = dh * (KEEP ? e[k][s] : fast_exp2(dtj * rates[s]));
              const float f = m[s] * h[k][s];
              da[s] = fmaf(f, dtj, da[s]);
              te[j] = s == 0 ? f * rates[s] : fmaf(f, rates[s], te[j]);
            }
            sums.leave(j, 0, tb);
            sums.leave(j, 1, tc);
          };
          row(Int<3>{});
          row(Int<2>{});
          row(Int<1>{});
          row(Int<0>{});
          __builtin_amdgcn_sched_barrier(0);
          const auto reads = sums.read();
          const float db = quad_rows(along, quad), dtime = quad_rows(te, quad) * kLn2;
          const float raw = rest.keep(i, fmaf(db, uu[i], dtime) * slope[i]);
          dskip = fmaf(dy[i], uu[i], dskip);               // both are 0 behind the episode
          dbias += raw;
          du.store(i, rest, fmaf(db, dt[i], skip * dy[i]));
          put<T>(ddelta, rest.offset(i, du.lane_at), du.ahead(i), from_f32<T>(raw));
          sums.join(reads, part[buffer % PARTS][wave] + 4 * i * 2 * N);
          if (!KEEP && i == QUADS / 2 && more) fetch(t - K);          // where some states are no longer needed
          __builtin_amdgcn_sched_barrier(0);
        }
        if (__builtin_expect(odd, 0)) {
          const Saved* p = saved_at<S>();
#pragma unroll
          for (int s = 0; s < S; ++s) {
            m[s] = p[s];
            da[s] = p[S + s];
          }
          dskip = p[2 * S];
          dbias = p[2 * S + 1];
          by_rows<T, S, GATE>(item, t, block * COLS, lds, rates, bias, skip, m, da, dskip, dbias, sums, part[buffer % PARTS][wave]);
        }
        if (more) rows.store(bc[buffer ^ 1]);
        __syncthreads();
        end_block(t);
        if (PARTS == 1) __syncthreads();
        buffer ^= 1;
      }
    }
    const ScanArgs& z = read_args();
    item += z.shares;
    const Place exit(z.width, block * COLS);
    if (seg == 0 && z.dfirst) store_states<S>(z.dfirst + b * z.width * z.states, exit.at, exit.q, z.states, exit.real, m);
    Track<T> dead(z.du, (int64_t)z.length * z.width, z.width, b, max(begin, live), exit.q, exit.at, exit.real);
    for (int t = max(begin, live); t < end; t += 4) {
      const Left left{end - t - exit.q - 1};
      const int64_t here = dead.p - (char*)z.du;
      dead.store(0, left, 0.0f);
      put<T>((char*)z.ddelta + here, left.offset(0, dead.lane_at), 0, from_f32<T>(0.0f));
      if (GATE) put<T>((char*)z.dgate + here, left.offset(0, dead.lane_at), 0, from_f32<T>(0.0f));
      dead.move(4);
    }
  }
  const ScanArgs& a = read_args();
  dskip = quad_sum(dskip);
  dbias = quad_sum(dbias);
  const Place end(a.width, block * COLS);
  if (!end.real) return;
  store_floats<S>(a.cols_part + ((int64_t)share * a.width + end.at) * N + end.q * S, da);
  if (end.q == 0) {
    a.ends_part[(int64_t)share * 2 * a.width + end.at] = dskip;
    a.ends_part[((int64_t)share * 2 + 1) * a.width + end.at] = dbias;
  }
}

// The shares' sums, always in the same order: db and dc, a number a thread, in the first
// `row_groups` workgroups; da, dskip and dbias in the others, 16 numbers each, whose shares are
// dealt to 16 groups of threads.
template <class T, int N> __global__ __launch_bounds__(kJoinBlock) void k_scan_sums(ScanArgs a, uint32_t row_groups) {
  __shared__ float part[16][16];
  if (blockIdx.x < row_groups) {
    const int64_t id = (int64_t)blockIdx.x * kJoinBlock + threadIdx.x, row = id / (2 * N);
    const int k = (int)(id % (2 * N)), n = k % N;
    if (row >= (int64_t)a.batch * a.length || n >= a.states) return;
    const int64_t b = row / a.length;
    float sum = 0.0f;
    if ((int)(row % a.length) < rows_in(a, b)) {
#pragma unroll 4
      for (int i = 0; i < a.col_blocks; ++i) sum += a.rows_part[(row * a.col_blocks + i) * 2 * N + k];
    }
    ((T*)(k < N ? a.db : a.dc))[row * a.states + n] = from_f32<T>(sum);
    return;
  }
  const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
  const int64_t id = (int64_t)(blockIdx.x - row_groups) * 16 + lane, numbers = (int64_t)a.width * N, ends = (int64_t)a.width * 2;
  const float* from = nullptr;
  int64_t step = 0;
  if (id < numbers) {
    from = a.cols_part + id;
    step = numbers;
  } else if (id < numbers + ends) {
    from = a.ends_part + (id - numbers);
    step = ends;
  }
  float sum = 0.0f;
  if (from) {
#pragma unroll 8
    for (int i = group; i < a.shares; i += 16) sum += from[i * step];
  }
  part[group][lane] = sum;
  __syncthreads();
  if (group != 0 || !from) return;
  sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum += part[i][lane];
  if (id < numbers) {
    const int n = (int)(id % N);
    if (n < a.states) a.da[id / N * a.states + n] = sum;
  } else {
    const int64_t k = id - numbers;
    if (k < a.width) {
      if (a.dskip) a.dskip[k] = sum;
    } else if (a.dbias) {
      a.dbias[k - a.width] = sum;
    }
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// The main pass holds two waves on each SIMD; the pieces of the first pass are shorter than its segments.
constexpr int64_t kPieceWaves = 8192, kWaves = 2048;
constexpr int kLeastRows = 32;
constexpr int64_t kWorkgroups = 1024;       // each leaves a share of da
// Episodes of different lengths leave places: segments that are cut anyway are then shorter, down to
// 128 rows, for four times the workgroups, which start where others have ended (forward and backward,
// without and with: 32 episodes of up to 1000 rows x 512 348 and 325 us, 24 of up to 1500 x 384 375 and 331).
// The host does not know the lengths, only that there are some.  Where all are alike it may lose
// (32 x 1000 x 512 385 and 411, 16 x 1000 x 1024 385 and 413) or gain (24 x 1500 x 384 398 and 367): a program whose
// episodes are of one length gives none.
constexpr int kRaggedRows = 128, kRaggedRounds = 4;
constexpr int kCols = 64;

constexpr int64_t kMostRows = 1 << 25;      // of all episodes: k_scan_sums takes a workgroup for four of them at 32 states

struct Plan {
  Cut pieces, parts;
  int col_blocks, shares;
  uint64_t left_state, left_time, rows_part, cols_part, ends_part, saved, bytes;
};
Plan plan_of(const qds_scan_config* c, bool ragged) {
  Plan p;
  const int64_t n = 4 * lane_states(c), rows = (int64_t)c->batch * c->length;
  p.pieces = cut(c, kPieceWaves, kLeastRows, kScanRows);
  p.parts = cut(c, kWaves, p.pieces.seg, p.pieces.seg);
  const int rounds = ragged && p.parts.segs > 1 ? kRaggedRounds : 1;
  if (rounds > 1) p.parts = cut(c, rounds * kWaves, std::min(p.parts.seg, std::max(p.pieces.seg, kRaggedRows)), p.pieces.seg);
  p.col_blocks = (int)ceil_div(c->width, kCols);
  const int64_t items = (int64_t)c->batch * p.parts.segs;
  p.shares = (int)std::max<int64_t>(1, std::min(items, std::max<int64_t>(1, rounds * kWorkgroups / p.col_blocks)));
  uint64_t at = 0;
  auto take = [&](uint64_t floats) {
    const uint64_t here = at;
    at += align_up(floats * sizeof(float));
    return here;
  };
  const uint64_t left = p.parts.segs > 1 ? (uint64_t)c->batch * p.pieces.segs * c->width : 0;
  p.left_state = take(left * n);
  p.left_time = take(left);
  p.rows_part = take((uint64_t)rows * p.col_blocks * 2 * n);
  p.cols_part = take((uint64_t)p.shares * c->width * n);
  p.ends_part = take((uint64_t)p.shares * c->width * 2);
  p.saved = take(c->states == n ? 0 : (uint64_t)p.shares * p.col_blocks * kCols * 4 * (2 * lane_states(c) + 2));
  p.bytes = at;
  return p;
}
bool fits(const qds_scan_config* c) {
  const Plan p = plan_of(c, false);
  const int64_t most = most_blocks(kJoinBlock);
  return (int64_t)c->batch <= most / (ceil_div(c->width, 64) * p.pieces.segs) && joinable(c, p.pieces.segs) &&
         (int64_t)c->batch * c->length <= kMostRows;
}

}  // namespace
}  // namespace seq

using namespace seq;

extern "C" qds_status qds_selective_scan_backward_workspace(const qds_scan_config* c, uint64_t* bytes) {
  const qds_status st = validate_scan(c, false);
  if (st != QDS_OK) return st;
  if (!bytes) return QDS_ERR_INVALID_ARG;
  if (!fits(c)) return QDS_ERR_UNSUPPORTED;
  *bytes = std::max(plan_of(c, false).bytes, plan_of(c, true).bytes);      // whether there are lengths is not known here
  return QDS_OK;
}

extern "C" qds_status qds_selective_scan_backward(const qds_scan_config* c, qds_rows dout, qds_rows u, qds_rows delta,
                                                  const float* a_, qds_rows b, qds_rows cc, const float* skip,
                                                  qds_rows gate, const float* bias, const void* marks,
                                                  const float* dstate_out, const int32_t* lengths, void* du,
                                                  void* ddelta, float* da, void* db, void* dc, float* dskip,
                                                  void* dgate, float* dbias, float* dstate_in, void* workspace,
                                                  uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  const qds_status st = qds_selective_scan_backward_workspace(c, &need);
  if (st != QDS_OK) return st;
  if (!a_ || !da || !workspace || ((uintptr_t)workspace & 255)) return QDS_ERR_INVALID_ARG;
  if (c->batch > 0 && c->length > 0 &&
      (!dout.data || !u.data || !delta.data || !b.data || !cc.data || !marks || !du || !ddelta || !db || !dc ||
       (gate.data && !dgate) || ((uintptr_t)marks & 255)))
    return QDS_ERR_INVALID_ARG;
  if (dstate_in && dstate_in == dstate_out) return QDS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return QDS_ERR_WORKSPACE_TOO_SMALL;
  for (qds_rows* r : {&dout, &u, &delta, &b, &cc, &gate})
    if (!near_rows(*r, c->length)) return QDS_ERR_UNSUPPORTED;
  for (const void* to : {du, ddelta, dgate})                                // blocks may be gone through again
    for (const qds_rows& from : {dout, u, delta, gate})
      if (to && to == from.data) return QDS_ERR_INVALID_ARG;
  const Plan p = plan_of(c, lengths != nullptr);
  ScanArgs a = scan_args(c);
  a.u = rows(u);
  a.delta = rows(delta);
  a.b = rows(b);
  a.c = rows(cc);
  a.gate = rows(gate);
  a.dout = rows(dout);
  a.du = du;
  a.ddelta = ddelta;
  a.db = db;
  a.dc = dc;
  a.dgate = dgate;
  a.a = a_;
  a.skip = skip;
  a.bias = bias;
  a.dlast = dstate_out;
  a.dfirst = dstate_in;
  a.da = da;
  a.dskip = dskip;
  a.dbias = dbias;
  a.lengths = lengths;
  a.marks = (float*)marks;
  a.seg = p.parts.seg;
  a.segs = p.parts.segs;
  a.piece = p.pieces.seg;
  a.pieces = p.pieces.segs;
  a.ratio = p.parts.seg / p.pieces.seg;
  a.joined = a.segs > 1 && a.pieces > kFewPieces;
  if (a.segs == 1) a.ratio = a.pieces;
  a.col_blocks = p.col_blocks;
  a.shares = c->batch > 0 ? p.shares : 0;
  char* ws = (char*)workspace;
  a.left_state = (float*)(ws + p.left_state);
  a.left_time = (float*)(ws + p.left_time);
  a.rows_part = (float*)(ws + p.rows_part);
  a.cols_part = (float*)(ws + p.cols_part);
  a.ends_part = (float*)(ws + p.ends_part);
  a.saved = (float*)(ws + p.saved);
  hipStream_t s = (hipStream_t)stream;
  scan_instance(c, [&](auto type, auto S, auto TAIL) {
    using T = decltype(type);
    constexpr int L = decltype(S)::value, N = 4 * L;
    constexpr bool tail = decltype(TAIL)::value;
    if (c->batch > 0) {
      if (a.segs > 1) {
        const uint32_t grid = (uint32_t)(c->batch * ceil_div(c->width, 64) * (a.pieces - a.ratio));
        if (gate.data) k_scan_back<T, L, true><<<grid, 256, 0, s>>>(a);
        else k_scan_back<T, L, false><<<grid, 256, 0, s>>>(a);
        if (a.joined) k_scan_join<N, true><<<(uint32_t)ceil_div((int64_t)c->batch * c->width * N, 16), kScanJoin, 0, s>>>(a);
      }
      const uint32_t grid = (uint32_t)(a.col_blocks * a.shares);
      if (gate.data) k_scan_backward<T, L, kCols, true, tail><<<grid, kCols * 4, 0, s>>>(a);
      else k_scan_backward<T, L, kCols, false, tail><<<grid, kCols * 4, 0, s>>>(a);
    }
    const uint32_t row_groups = (uint32_t)ceil_div((int64_t)c->batch * c->length * 2 * N, kJoinBlock);
    const uint32_t col_groups = (uint32_t)ceil_div((int64_t)c->width * (N + 2), 16);
    k_scan_sums<T, N><<<row_groups + col_groups, kJoinBlock, 0, s>>>(a, row_groups);
  });
  return launch_status();
}
