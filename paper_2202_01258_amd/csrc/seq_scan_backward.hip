// seq_scan_backward.hip -- gradients of the selective state space scan.  The C ABI is in
// include/qd_seq.h, the layout of the work in seq_scan.hpp.
#include <algorithm>

#include "seq_scan.hpp"

namespace seq {
namespace {

constexpr int kJoinBlock = 256;

// With m_t = e^(dt_{t+1} a) dh_{t+1}, what reaches row t from the rows behind it:
//   dh = m_t + dy_t c_t;  m_{t-1} = e^(dt_t a) dh.
// One segment of 64 columns from its last row to its first, from zero: what it leaves to
// the segment before, and the sum of its steps.
template <class T, int S> __global__ __launch_bounds__(256) void k_scan_back(ScanArgs a) {
  constexpr int K = kScanRows<S>, N = 4 * S, QUADS = K / 4, BLOCK = 256;
  SEQ_SHARED float bc[2][K * 2 * N];
  const int q = threadIdx.x & 3, blocks = (a.width + 63) / 64;
  const uint32_t item = blockIdx.x / (uint32_t)blocks;
  const int col = (blockIdx.x % (uint32_t)blocks) * 64 + (threadIdx.x >> 2);
  const bool real = col < a.width;
  const int at = real ? col : a.width - 1;
  const int64_t b = item / (uint32_t)(a.segs - 1);
  const int seg = 1 + (int)(item % (uint32_t)(a.segs - 1));       // nothing comes before the first segment
  const int n = rows_in(a, b), begin = seg * a.seg, end = min(begin + a.seg, a.length), live = min(end, n);
  float rates[S], m[S], time = 0.0f;
  load_states<S>(rates, a.a, at, q, a.states);
#pragma unroll
  for (int s = 0; s < S; ++s) {
    rates[s] = rate(rates[s]);
    m[s] = 0.0f;
  }
  const float bias = a.bias ? a.bias[at] : 0.0f;
  if (begin < live) {
    T d[QUADS], g[QUADS], z[QUADS];
    Track<T> td, tg, tz;
    td.init(a.delta, b, q, at);
    tg.init(a.dout, b, q, at);
    tz.init(a.gate, b, q, at);
    StagedRows<T, S, BLOCK> rows;
    auto fetch = [&](int t) {
#pragma unroll
      for (int i = 0; i < QUADS; ++i) {
        const bool in = t + 4 * i + q < live;
        d[i] = td.load(t, i, in);
        g[i] = tg.load(t, i, in);
        if (a.gate.p) z[i] = tz.load(t, i, in);
      }
      rows.load(a, b, t, live);
    };
    const int last = begin + (live - 1 - begin) / K * K;
    fetch(last);
    rows.store(bc[0]);
    __syncthreads();
    int buffer = 0;
    for (int t = last; t >= begin; t -= K) {
      float dt[QUADS], dy[QUADS];
#pragma unroll
      for (int i = 0; i < QUADS; ++i) {
        const bool in = t + 4 * i + q < live;
        dt[i] = in ? softplus(to_f32(d[i]) + bias).dt : 0.0f;
        dy[i] = to_f32(g[i]);
        if (a.gate.p) dy[i] *= to_f32(z[i]) * sigmoid(to_f32(z[i]));
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
      }
      if (more) {
        rows.store(bc[buffer ^ 1]);
        __syncthreads();
        buffer ^= 1;
      }
    }
  }
  time = quad_sum(time);
  if (real) store_floats<S>(a.seg_state + ((b * a.segs + seg) * a.width + at) * N + q * S, m);
  if (real && q == 0) a.seg_time[(b * a.segs + seg) * a.width + at] = time;
}

// What reaches each segment's last row from behind.
template <int N> __global__ __launch_bounds__(kJoinBlock) void k_scan_back_join(ScanArgs a) {
  const int64_t id = (int64_t)blockIdx.x * kJoinBlock + threadIdx.x, column = id / N;
  const int n = (int)(id % N);
  if (column >= (int64_t)a.batch * a.width) return;
  const int64_t b = column / a.width;
  const int at = (int)(column % a.width);
  const bool in = n < a.states;
  float x = in && a.dlast ? a.dlast[column * a.states + n] : 0.0f;
  const float r = in ? rate(a.a[(int64_t)at * a.states + n]) : 0.0f;
#pragma unroll 4
  for (int seg = a.segs - 1; seg > 0; --seg) {
    const int64_t where = (b * a.segs + seg) * a.width + at;
    const float left = a.seg_state[where * N + n], time = a.seg_time[where];
    a.seg_state[where * N + n] = x;
    x = fmaf(fast_exp2(r * time), x, left);
  }
  a.seg_state[(b * a.segs * a.width + at) * N + n] = x;
}

// Sums of 16 values over the wave's 16 columns (lane bits 2 to 5): halves of the values go to
// halves of the lanes, so each step adds half as many numbers as the one before.  The lane
// gets the sum of value 8 bit5 + 4 bit4 + 2 bit3 + bit2.
__device__ inline float sum_columns(const float* v) {
  float w[8], z[4], p[2];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 8]), false, false);
    w[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(w[i]), __float_as_uint(w[i + 4]), false, false);
    z[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  const bool three = threadIdx.x & 8, two = threadIdx.x & 4;
#pragma unroll
  for (int i = 0; i < 2; ++i) p[i] = (three ? z[i + 2] : z[i]) + lane_move<0x128>(three ? z[i] : z[i + 2]);   // lane ^ 8
  return (two ? p[1] : p[0]) + lane_move<0x1B>(lane_move<0x141>(two ? p[0] : p[1]));                          // lane ^ 4 = (lane ^ 7) ^ 3
}

// All gradients.  A workgroup has COLS columns and goes through every `shares`-th segment, each
// from its last block of rows to its first: a block's states and decays are formed again from
// its mark and kept in registers for the way back.
template <class T, int S, int COLS> __global__ __launch_bounds__(COLS * 4) void k_scan_backward(ScanArgs a) {
  constexpr int K = kScanRows<S>, N = 4 * S, QUADS = K / 4, BLOCK = COLS * 4, WAVES = BLOCK / 64;
  constexpr bool KEEP = S <= 4;                                     // decays for the way back; else they are formed again
  constexpr int GROUP = 8 / S;                                      // rows whose sums over columns are formed together
  SEQ_SHARED float bc[2][K * 2 * N];
  SEQ_SHARED float part[2][WAVES][K * 2 * N];
  const int q = threadIdx.x & 3, wave = wave_index();
  const int block = blockIdx.x % (uint32_t)a.col_blocks;
  const uint32_t share = blockIdx.x / (uint32_t)a.col_blocks;
  const int col = block * COLS + (threadIdx.x >> 2);
  const bool real = col < a.width;
  const int at = real ? col : a.width - 1;
  float rates[S], da[S], dskip = 0.0f, dbias = 0.0f;
  load_states<S>(rates, a.a, at, q, a.states);
#pragma unroll
  for (int s = 0; s < S; ++s) {
    rates[s] = rate(rates[s]);
    da[s] = 0.0f;
  }
  const float bias = a.bias ? a.bias[at] : 0.0f, skip = a.skip ? a.skip[at] : 0.0f;
  // where this lane's sums over columns go: value (row, b or c, state) of a group of rows
  const int value = ((threadIdx.x >> 5) & 1) * 8 + ((threadIdx.x >> 4) & 1) * 4 + ((threadIdx.x >> 3) & 1) * 2 + ((threadIdx.x >> 2) & 1);
  const int target = value / (2 * S) * 2 * N + (value / S % 2) * N + q * S + value % S;
  int buffer = 0;
  const uint32_t items = (uint32_t)(a.batch * a.segs);
  for (uint32_t item = share; item < items; item += a.shares) {
    const int64_t b = item / (uint32_t)a.segs;
    const int seg = (int)(item % (uint32_t)a.segs);
    const int n = rows_in(a, b), begin = seg * a.seg, end = min(begin + a.seg, a.length), live = min(end, n);
    Track<T> tu, td, tz, tg, tdu, tdd, tdz;
    tu.init(a.u, b, q, at);
    td.init(a.delta, b, q, at);
    tg.init(a.dout, b, q, at);
    tdu.init(a.du, b, q, at);
    tdd.init(a.ddelta, b, q, at);
    tz.init(a.gate, b, q, at);
    tdz.init(a.dgate, b, q, at);
    float m[S];
    if (a.segs > 1) load_floats<S>(m, a.seg_state + (b * a.segs + seg) * a.width * N + (uint32_t)(at * N + q * S));
    else load_states<S>(m, a.dlast ? a.dlast + b * a.width * a.states : nullptr, at, q, a.states);
#pragma unroll
    for (int s = 0; s < S; ++s) m[s] = real ? m[s] : 0.0f;           // columns that are not real add nothing to db and dc
    if (begin < live) {
      T u[QUADS], d[QUADS], z[QUADS], g[QUADS];
      float first[S];
      StagedRows<T, S, BLOCK> rows;
      auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
          const bool in = real && t + 4 * i + q < live;
          u[i] = tu.load(t, i, in);
          d[i] = td.load(t, i, in);
          g[i] = tg.load(t, i, in);
          if (a.gate.p) z[i] = tz.load(t, i, in);
        }
        load_floats<S>(first, a.marks + (b * a.blocks + t / K) * a.width * N + (uint32_t)(at * N + q * S));
        rows.load(a, b, t, live);
      };
      const int last = begin + (live - 1 - begin) / K * K;
      fetch(last);
      rows.store(bc[buffer]);
      __syncthreads();
      for (int t = last; t >= begin; t -= K) {
        const float* lds = bc[buffer] + q * S;
        float h[K + 1][S], e[KEEP ? K : 1][S];                      // h[r]: in front of row r; e[r]: its decay
        float dt[QUADS], slope[QUADS], uu[QUADS], dy[QUADS];
#pragma unroll
        for (int s = 0; s < S; ++s) h[0][s] = real ? first[s] : 0.0f;
#pragma unroll
        for (int i = 0; i < QUADS; ++i) {
          const int r = t + 4 * i + q;
          const bool in = real && r < live;
          const Step step = softplus(to_f32(d[i]) + bias);
          dt[i] = in ? step.dt : 0.0f;
          slope[i] = step.slope;
          uu[i] = to_f32(u[i]);
          const float x = dt[i] * uu[i];
          float y[4];
          auto row = [&](auto J) {
            constexpr int j = decltype(J)::value, k = j;
            const float dtj = quad_lane<j>(dt[i]), xj = quad_lane<j>(x);
            float bv[S], cv[S];
            load_floats<S>(bv, lds + (4 * i + k) * 2 * N);
            load_floats<S>(cv, lds + (4 * i + k) * 2 * N + N);
            y[j] = 0.0f;
#pragma unroll
            for (int s = 0; s < S; ++s) {
              const float decay = fast_exp2(dtj * rates[s]);
              if (KEEP) e[4 * i + j][s] = decay;
              h[4 * i + j + 1][s] = fmaf(decay, h[4 * i + j][s], xj * bv[s]);
              y[j] = fmaf(h[4 * i + j + 1][s], cv[s], y[j]);
            }
          };
          row(Int<0>{});
          row(Int<1>{});
          row(Int<2>{});
          row(Int<3>{});
          const float out = to_f32(g[i]);
          dy[i] = out;
          if (a.gate.p) {
            const float zz = to_f32(z[i]), s = sigmoid(zz);
            dy[i] = out * (zz * s);
            const float yy = fmaf(skip, uu[i], quad_rows(y, q));
            tdz.store(t, i, in, out * yy * silu_slope(zz, s));
          }
          __builtin_amdgcn_sched_barrier(0);     // no reads of later rows before these are done: registers are short
        }
        const bool more = t > begin;
        float sums[16];
        // b and c are read and steps are moved again: kept from above they would take as many
        // registers as the states
        int again = q * S;
        asm volatile("" : "+v"(again));
        lds = bc[buffer] + again;
#pragma unroll
        for (int i = 0; i < QUADS; ++i) asm volatile("" : "+v"(dt[i]));
#pragma unroll
        for (int i = QUADS - 1; i >= 0; --i) {
          const float x = dt[i] * uu[i];
          float along[4], te[4];
          auto row = [&](auto J) {
            constexpr int j = decltype(J)::value;
            const float dtj = quad_lane<j>(dt[i]), xj = quad_lane<j>(x), dyj = quad_lane<j>(dy[i]);
            const int k = 4 * i + j;
            float bv[S], cv[S];
            load_floats<S>(bv, lds + k * 2 * N);
            load_floats<S>(cv, lds + k * 2 * N + N);
            along[j] = te[j] = 0.0f;
#pragma unroll
            for (int s = 0; s < S; ++s) {
              const float dh = fmaf(dyj, cv[s], m[s]);
              sums[k % GROUP * 2 * S + s] = dh * xj;
              sums[k % GROUP * 2 * S + S + s] = dyj * h[k + 1][s];
              along[j] = fmaf(dh, bv[s], along[j]);
              m[s] = dh * (KEEP ? e[k][s] : fast_exp2(dtj * rates[s]));
              const float f = m[s] * h[k][s];
              da[s] = fmaf(f, dtj, da[s]);
              te[j] = fmaf(f, rates[s], te[j]);
            }
            if (k % GROUP == 0) part[buffer][wave][k * 2 * N + target] = sum_columns(sums);
          };
          row(Int<3>{});
          row(Int<2>{});
          row(Int<1>{});
          row(Int<0>{});
          const float db = quad_rows(along, q), dtime = quad_rows(te, q) * kLn2;
          const int r = t + 4 * i + q;
          const float ddelta = fmaf(db, uu[i], dtime) * slope[i];
          const bool in = real && r < live;
          dskip = fmaf(dy[i], uu[i], dskip);               // both are 0 behind the episode
          dbias += in ? ddelta : 0.0f;
          tdu.store(t, i, in, fmaf(db, dt[i], skip * dy[i]));
          tdd.store(t, i, in, ddelta);
          // the next block's loads, where half of this one's states are no longer needed
          if (i == QUADS / 2 && more) fetch(t - K);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (more) rows.store(bc[buffer ^ 1]);
        __syncthreads();
        // the waves' sums, in their order
#pragma unroll
        for (int i = 0; i < (K * 2 * N + BLOCK - 1) / BLOCK; ++i) {
          const int k = threadIdx.x + i * BLOCK, r = t + k / (2 * N);
          if (k < K * 2 * N && r < live) {
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sum += part[buffer][w][k];
            a.rows_part[((b * a.length + r) * a.col_blocks + block) * 2 * N + k % (2 * N)] = sum;
          }
        }
        buffer ^= 1;
      }
    }
    if (seg == 0 && a.dfirst) store_states<S>(a.dfirst + b * a.width * a.states, at, q, a.states, real, m);
    for (int t = max(begin, live); t < end; t += 4) {
      const bool in = real && t + q < end;
      tdu.store(t, 0, in, 0.0f);
      tdd.store(t, 0, in, 0.0f);
      if (a.gate.p) tdz.store(t, 0, in, 0.0f);
    }
  }
  if (!real) return;
  store_floats<S>(a.cols_part + ((int64_t)share * a.width + at) * N + q * S, da);
  dskip = quad_sum(dskip);
  dbias = quad_sum(dbias);
  if (q == 0) {
    a.ends_part[((int64_t)share * 2) * a.width + at] = dskip;
    a.ends_part[((int64_t)share * 2 + 1) * a.width + at] = dbias;
  }
}

// db and dc: each row's shares of the column blocks.
template <class T, int N> __global__ __launch_bounds__(kJoinBlock) void k_scan_rows_join(ScanArgs a) {
  const int64_t id = (int64_t)blockIdx.x * kJoinBlock + threadIdx.x, row = id / (2 * N);
  const int k = (int)(id % (2 * N)), n = k % N;
  if (row >= (int64_t)a.batch * a.length || n >= a.states) return;
  const int64_t b = row / a.length;
  const int t = (int)(row % a.length);
  float sum = 0.0f;
  if (t < rows_in(a, b)) {
#pragma unroll 4
    for (int i = 0; i < a.col_blocks; ++i) sum += a.rows_part[(row * a.col_blocks + i) * 2 * N + k];
  }
  (k < N ? row_of<T>(a.db, b, t) : row_of<T>(a.dc, b, t))[n] = from_f32<T>(sum);
}

// da, dskip and dbias: 64 numbers per workgroup, sixteen waves each add every sixteenth share.
constexpr int kJoinWaves = 16;
template <int N> __global__ __launch_bounds__(64 * kJoinWaves) void k_scan_columns_join(ScanArgs a) {
  __shared__ float part[64 * kJoinWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t id = (int64_t)blockIdx.x * 64 + lane, numbers = (int64_t)a.width * N, ends = (int64_t)a.width * 2;
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
    for (int i = wave; i < a.shares; i += kJoinWaves) sum += from[i * step];
  }
  part[threadIdx.x] = sum;
  __syncthreads();
  if (wave != 0 || !from) return;
  sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kJoinWaves; ++i) sum += part[i * 64 + lane];
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
constexpr int64_t kWaves = 2048;
constexpr int kLeastRows = 64;
constexpr int64_t kWorkgroups = 1024;       // each leaves a share of da
constexpr int kCols = 128;

struct Plan {
  Cut parts;
  int col_blocks, shares;
  uint64_t seg_state, seg_time, rows_part, cols_part, ends_part, bytes;
};
Plan plan_of(const qds_scan_config* c) {
  Plan p;
  const int64_t n = 4 * lane_states(c), rows = (int64_t)c->batch * c->length;
  p.parts = cut(c, kWaves, kLeastRows);
  p.col_blocks = (int)ceil_div(c->width, kCols);
  const int64_t items = (int64_t)c->batch * p.parts.segs;
  p.shares = (int)std::max<int64_t>(1, std::min(items, std::max<int64_t>(1, kWorkgroups / p.col_blocks)));
  uint64_t at = 0;
  auto take = [&](uint64_t floats) {
    const uint64_t here = at;
    at += align_up(floats * sizeof(float));
    return here;
  };
  const uint64_t segments = p.parts.segs > 1 ? (uint64_t)items * c->width : 0;
  p.seg_state = take(segments * n);
  p.seg_time = take(segments);
  p.rows_part = take((uint64_t)rows * p.col_blocks * 2 * n);
  p.cols_part = take((uint64_t)p.shares * c->width * n);
  p.ends_part = take((uint64_t)p.shares * c->width * 2);
  p.bytes = at;
  return p;
}
bool fits(const qds_scan_config* c) {
  const Plan p = plan_of(c);
  const int64_t most = most_blocks(kJoinBlock);
  return (int64_t)c->batch <= most / (ceil_div(c->width, 64) * p.parts.segs) && (int64_t)c->batch * c->width <= most * 8 &&
         (int64_t)c->batch * c->length <= most * 4;
}

}  // namespace
}  // namespace seq

using namespace seq;

extern "C" qds_status qds_selective_scan_backward_workspace(const qds_scan_config* c, uint64_t* bytes) {
  const qds_status st = validate_scan(c, false);
  if (st != QDS_OK) return st;
  if (!bytes) return QDS_ERR_INVALID_ARG;
  if (!fits(c)) return QDS_ERR_UNSUPPORTED;
  *bytes = plan_of(c).bytes;
  return QDS_OK;
}

extern "C" qds_status qds_selective_scan_backward(const qds_scan_config* c, qds_rows dout, qds_rows u, qds_rows delta,
                                                  const float* a_, qds_rows b, qds_rows cc, const float* skip,
                                                  qds_rows gate, const float* bias, const void* marks,
                                                  const float* dstate_out, const int32_t* lengths, qds_rows du,
                                                  qds_rows ddelta, float* da, qds_rows db, qds_rows dc, float* dskip,
                                                  qds_rows dgate, float* dbias, float* dstate_in, void* workspace,
                                                  uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  const qds_status st = qds_selective_scan_backward_workspace(c, &need);
  if (st != QDS_OK) return st;
  if (!a_ || !da || !workspace || ((uintptr_t)workspace & 255)) return QDS_ERR_INVALID_ARG;
  if (c->batch > 0 && c->length > 0 &&
      (!dout.data || !u.data || !delta.data || !b.data || !cc.data || !marks || !du.data || !ddelta.data || !db.data ||
       !dc.data || (gate.data && !dgate.data) || ((uintptr_t)marks & 255)))
    return QDS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return QDS_ERR_WORKSPACE_TOO_SMALL;
  for (qds_rows* r : {&dout, &u, &delta, &b, &cc, &gate, &du, &ddelta, &db, &dc, &dgate})
    if (!near_rows(*r, c->length)) return QDS_ERR_UNSUPPORTED;
  const Plan p = plan_of(c);
  ScanArgs a = scan_args(c);
  a.u = rows(u);
  a.delta = rows(delta);
  a.b = rows(b);
  a.c = rows(cc);
  a.gate = rows(gate);
  a.dout = rows(dout);
  a.du = rows(du);
  a.ddelta = rows(ddelta);
  a.db = rows(db);
  a.dc = rows(dc);
  a.dgate = rows(dgate);
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
  a.col_blocks = p.col_blocks;
  a.shares = c->batch > 0 ? p.shares : 0;
  char* ws = (char*)workspace;
  a.seg_state = (float*)(ws + p.seg_state);
  a.seg_time = (float*)(ws + p.seg_time);
  a.rows_part = (float*)(ws + p.rows_part);
  a.cols_part = (float*)(ws + p.cols_part);
  a.ends_part = (float*)(ws + p.ends_part);
  hipStream_t s = (hipStream_t)stream;
  scan_instance(c, [&](auto type, auto S) {
    using T = decltype(type);
    constexpr int L = decltype(S)::value, N = 4 * L;
    if (c->batch > 0) {
      if (a.segs > 1) {
        k_scan_back<T, L><<<(uint32_t)(c->batch * ceil_div(c->width, 64) * (a.segs - 1)), 256, 0, s>>>(a);
        k_scan_back_join<N><<<(uint32_t)ceil_div((int64_t)c->batch * c->width * N, kJoinBlock), kJoinBlock, 0, s>>>(a);
      }
      k_scan_backward<T, L, kCols><<<(uint32_t)(a.col_blocks * a.shares), kCols * 4, 0, s>>>(a);
      if (c->length > 0)
        k_scan_rows_join<T, N><<<(uint32_t)ceil_div((int64_t)c->batch * c->length * 2 * N, kJoinBlock), kJoinBlock, 0, s>>>(a);
    }
    k_scan_columns_join<N><<<(uint32_t)ceil_div((int64_t)c->width * (N + 2), 64), 64 * kJoinWaves, 0, s>>>(a);
  });
  return launch_status();
}
