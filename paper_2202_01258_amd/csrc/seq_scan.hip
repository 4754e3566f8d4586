// seq_scan.hip -- selective state space scan: forward and one row.  The C ABI is in
// include/qd_seq.h, the layout of the work in seq_scan.hpp.
#include <algorithm>

#include "seq_scan.hpp"

namespace seq {
namespace {

constexpr int kBlock = 256, kColumns = kBlock / 4;

// One segment of 64 columns.  LOCAL: what the segment leaves behind when it starts from
// zero, and the sum of its steps; otherwise outputs, marks and the last state.
template <class T, int S, bool LOCAL> __global__ __launch_bounds__(kBlock) void k_scan(ScanArgs a) {
  constexpr int K = kScanRows<S>, N = 4 * S, QUADS = K / 4;
  SEQ_SHARED float bc[2][K * 2 * N];
  const int q = threadIdx.x & 3;
  const uint32_t item = blockIdx.x / (uint32_t)a.col_blocks;
  const int col = (blockIdx.x % (uint32_t)a.col_blocks) * kColumns + (threadIdx.x >> 2);
  const bool real = col < a.width;
  const int at = real ? col : a.width - 1;
  const int runs = LOCAL ? a.segs - 1 : a.segs;            // nothing comes behind the last segment
  const int64_t b = item / (uint32_t)runs;
  const int seg = (int)(item % (uint32_t)runs);
  const int n = rows_in(a, b), begin = seg * a.seg, end = min(begin + a.seg, a.length), live = min(end, n);
  float rates[S], h[S];
  load_states<S>(rates, a.a, at, q, a.states);
#pragma unroll
  for (int s = 0; s < S; ++s) rates[s] = rate(rates[s]);
  const float bias = a.bias ? a.bias[at] : 0.0f, skip = a.skip ? a.skip[at] : 0.0f;
  const int64_t place = ((b * a.segs + seg) * a.width + at) * N + q * S;
  if (LOCAL) {
#pragma unroll
    for (int s = 0; s < S; ++s) h[s] = 0.0f;
  } else if (a.segs > 1) {
    load_floats<S>(h, a.seg_state + place);
  } else {
    load_states<S>(h, a.first ? a.first + b * a.width * a.states : nullptr, at, q, a.states);
  }
  float time = 0.0f;
  if (begin < live) {
    T u[QUADS], d[QUADS], z[QUADS];
    Track<T> tu, td, tz, to;
    tu.init(a.u, b, q, at);
    td.init(a.delta, b, q, at);
    if (!LOCAL) {
      tz.init(a.gate, b, q, at);
      to.init(a.o, b, q, at);
    }
    StagedRows<T, S, kBlock> rows;
    auto fetch = [&](int t) {
#pragma unroll
      for (int i = 0; i < QUADS; ++i) {
        const bool in = t + 4 * i + q < live;
        u[i] = tu.load(t, i, in);
        d[i] = td.load(t, i, in);
        if (!LOCAL && a.gate.p) z[i] = tz.load(t, i, in);
      }
      rows.load(a, b, t, live);
    };
    fetch(begin);
    rows.store(bc[0]);
    __syncthreads();
    int buffer = 0;
    for (int t = begin; t < live; t += K) {
      float dt[QUADS], uu[QUADS], zz[QUADS];
#pragma unroll
      for (int i = 0; i < QUADS; ++i) {
        const bool in = t + 4 * i + q < live;
        dt[i] = in ? softplus(to_f32(d[i]) + bias).dt : 0.0f;
        uu[i] = to_f32(u[i]);
        if (!LOCAL && a.gate.p) zz[i] = to_f32(z[i]);
      }
      const bool more = t + K < live;
      if (more) fetch(t + K);
      if (!LOCAL && a.marks && real) store_floats<S>(a.marks + ((b * a.blocks + t / K) * a.width + at) * N + q * S, h);
      const float* lds = bc[buffer] + q * S;
#pragma unroll
      for (int i = 0; i < QUADS; ++i) {
        const float x = dt[i] * uu[i];
        float y[4];
        auto row = [&](auto J) {
          constexpr int j = decltype(J)::value;
          const float dtj = quad_lane<j>(dt[i]), xj = quad_lane<j>(x);
          float bv[S], cv[S];
          load_floats<S>(bv, lds + (4 * i + j) * 2 * N);
          if (!LOCAL) load_floats<S>(cv, lds + (4 * i + j) * 2 * N + N);
          y[j] = 0.0f;
#pragma unroll
          for (int s = 0; s < S; ++s) {
            h[s] = fmaf(fast_exp2(dtj * rates[s]), h[s], xj * bv[s]);
            if (!LOCAL) y[j] = fmaf(h[s], cv[s], y[j]);
          }
        };
        row(Int<0>{});
        row(Int<1>{});
        row(Int<2>{});
        row(Int<3>{});
        if (LOCAL) {
          time += dt[i];
        } else {
          float o = fmaf(skip, uu[i], quad_rows(y, q));
          if (a.gate.p) o *= zz[i] * sigmoid(zz[i]);
          to.store(t, i, real && t + 4 * i + q < live, o);
        }
      }
      if (more) {
        rows.store(bc[buffer ^ 1]);
        __syncthreads();
        buffer ^= 1;
      }
    }
  }
  if (LOCAL) {
    time = quad_sum(time);
    if (real) store_floats<S>(a.seg_state + place, h);
    if (real && q == 0) a.seg_time[(b * a.segs + seg) * a.width + at] = time;
  } else {
    Track<T> to;
    to.init(a.o, b, q, at);
    for (int t = max(begin, live); t < end; t += 4) to.store(t, 0, real && t + q < end, 0.0f);
    if (seg == a.segs - 1 && a.last) store_states<S>(a.last + b * a.width * a.states, at, q, a.states, real, h);
  }
}

// What each segment starts from: x = e^(a time) x + what the segment before left behind.
template <int N> __global__ __launch_bounds__(kBlock) void k_scan_join(ScanArgs a) {
  const int64_t id = (int64_t)blockIdx.x * kBlock + threadIdx.x, column = id / N;
  const int n = (int)(id % N);
  if (column >= (int64_t)a.batch * a.width) return;
  const int64_t b = column / a.width;
  const int at = (int)(column % a.width);
  const bool in = n < a.states;
  float x = in && a.first ? a.first[column * a.states + n] : 0.0f;
  const float r = in ? rate(a.a[(int64_t)at * a.states + n]) : 0.0f;
#pragma unroll 4
  for (int seg = 0; seg < a.segs - 1; ++seg) {
    const int64_t where = (b * a.segs + seg) * a.width + at;
    const float left = a.seg_state[where * N + n], time = a.seg_time[where];
    a.seg_state[where * N + n] = x;
    x = fmaf(fast_exp2(r * time), x, left);
  }
  a.seg_state[((b * a.segs + a.segs - 1) * a.width + at) * N + n] = x;
}

// One row: the state is what is read and written.
template <class T, int S> __global__ __launch_bounds__(kBlock) void k_scan_step(ScanArgs a) {
  const uint32_t id = blockIdx.x * kBlock + threadIdx.x, column = id >> 2;
  if (column >= (uint32_t)(a.batch * a.width)) return;
  const int q = threadIdx.x & 3;
  const int64_t b = column / (uint32_t)a.width;
  const int at = (int)(column % (uint32_t)a.width);
  float r[S], h[S], y = 0.0f;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int n = q * S + s;
    h[s] = n < a.states ? a.first[(int64_t)column * a.states + n] : 0.0f;
    r[s] = n < a.states ? a.a[(int64_t)at * a.states + n] : 0.0f;
  }
  const float u = to_f32(row_of<T>(a.u, b, 0)[at]);
  const float dt = softplus(to_f32(row_of<T>(a.delta, b, 0)[at]) + (a.bias ? a.bias[at] : 0.0f)).dt;
  const T *bp = row_of<T>(a.b, b, 0), *cp = row_of<T>(a.c, b, 0);
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int n = q * S + s;
    if (n < a.states) {
      h[s] = fmaf(fast_exp2(dt * rate(r[s])), h[s], dt * u * to_f32(bp[n]));
      y = fmaf(h[s], to_f32(cp[n]), y);
    }
  }
#pragma unroll
  for (int s = 0; s < S; ++s)
    if (q * S + s < a.states) a.last[(int64_t)column * a.states + q * S + s] = h[s];
  y = quad_sum(y);
  if (q == 0) {
    float o = fmaf(a.skip ? a.skip[at] : 0.0f, u, y);
    if (a.gate.p) {
      const float z = to_f32(row_of<T>(a.gate, b, 0)[at]);
      o *= z * sigmoid(z);
    }
    row_of<T>(a.o, b, 0)[at] = from_f32<T>(o);
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
constexpr int64_t kWaves = 2048;
constexpr int kLeastRows = 64;

Cut forward_cut(const qds_scan_config* c) { return cut(c, kWaves, kLeastRows); }
uint64_t state_bytes(const qds_scan_config* c, int segs) {
  return align_up((uint64_t)c->batch * segs * c->width * 4 * lane_states(c) * sizeof(float));
}
bool fits(const qds_scan_config* c) {
  const int64_t workgroups = ceil_div(c->width, kColumns) * forward_cut(c).segs;
  return (int64_t)c->batch <= (int64_t)most_blocks(kBlock) / workgroups &&
         (int64_t)c->batch * c->width <= (int64_t)most_blocks(kBlock) * 8;
}

}  // namespace
}  // namespace seq

using namespace seq;

extern "C" qds_status qds_selective_scan_marks(const qds_scan_config* c, uint64_t* bytes) {
  const qds_status st = validate_scan(c, false);
  if (st != QDS_OK) return st;
  if (!bytes) return QDS_ERR_INVALID_ARG;
  *bytes = state_bytes(c, block_count(c));
  return QDS_OK;
}

extern "C" qds_status qds_selective_scan_workspace(const qds_scan_config* c, uint64_t* bytes) {
  const qds_status st = validate_scan(c, false);
  if (st != QDS_OK) return st;
  if (!bytes) return QDS_ERR_INVALID_ARG;
  if (!fits(c)) return QDS_ERR_UNSUPPORTED;
  const int segs = forward_cut(c).segs;
  *bytes = segs > 1 ? state_bytes(c, segs) + align_up((uint64_t)c->batch * segs * c->width * sizeof(float)) : 0;
  return QDS_OK;
}

extern "C" qds_status qds_selective_scan(const qds_scan_config* c, qds_rows u, qds_rows delta, const float* a_,
                                         qds_rows b, qds_rows cc, const float* skip, qds_rows gate, const float* bias,
                                         const float* state_in, const int32_t* lengths, qds_rows o, float* state_out,
                                         void* marks, void* workspace, uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  const qds_status st = qds_selective_scan_workspace(c, &need);
  if (st != QDS_OK) return st;
  if (c->batch == 0) return QDS_OK;
  if (!a_ || (c->length > 0 && (!u.data || !delta.data || !b.data || !cc.data || !o.data))) return QDS_ERR_INVALID_ARG;
  for (qds_rows* r : {&u, &delta, &b, &cc, &gate, &o})
    if (!near_rows(*r, c->length)) return QDS_ERR_UNSUPPORTED;
  if (((uintptr_t)marks & 255) || (need > 0 && (!workspace || ((uintptr_t)workspace & 255)))) return QDS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return QDS_ERR_WORKSPACE_TOO_SMALL;
  ScanArgs a = scan_args(c);
  const Cut parts = forward_cut(c);
  a.u = rows(u);
  a.delta = rows(delta);
  a.b = rows(b);
  a.c = rows(cc);
  a.gate = rows(gate);
  a.o = rows(o);
  a.a = a_;
  a.skip = skip;
  a.bias = bias;
  a.first = state_in;
  a.last = state_out;
  a.lengths = lengths;
  a.marks = (float*)marks;
  a.seg = parts.seg;
  a.segs = parts.segs;
  a.col_blocks = (int)ceil_div(c->width, kColumns);
  if (a.segs > 1) {
    a.seg_state = (float*)workspace;
    a.seg_time = (float*)((char*)workspace + state_bytes(c, a.segs));
  }
  hipStream_t s = (hipStream_t)stream;
  scan_instance(c, [&](auto type, auto S) {
    using T = decltype(type);
    constexpr int L = decltype(S)::value;
    const uint32_t across = (uint32_t)(a.batch * a.col_blocks);
    if (a.segs > 1) {
      k_scan<T, L, true><<<across * (a.segs - 1), kBlock, 0, s>>>(a);
      k_scan_join<4 * L><<<(uint32_t)ceil_div((int64_t)a.batch * a.width * 4 * L, kBlock), kBlock, 0, s>>>(a);
    }
    k_scan<T, L, false><<<across * a.segs, kBlock, 0, s>>>(a);
  });
  return launch_status();
}

extern "C" qds_status qds_selective_scan_step(const qds_scan_config* c, qds_rows u, qds_rows delta, const float* a_,
                                              qds_rows b, qds_rows cc, const float* skip, qds_rows gate,
                                              const float* bias, const float* state_in, qds_rows o, float* state_out,
                                              void* stream) {
  const qds_status st = validate_scan(c, true);
  if (st != QDS_OK) return st;
  if (c->batch == 0) return QDS_OK;
  if (!a_ || !u.data || !delta.data || !b.data || !cc.data || !o.data || !state_in || !state_out) return QDS_ERR_INVALID_ARG;
  const int64_t columns = (int64_t)c->batch * c->width;
  if (columns >= (1 << 30)) return QDS_ERR_UNSUPPORTED;
  ScanArgs a = scan_args(c);
  a.u = rows(u);
  a.delta = rows(delta);
  a.b = rows(b);
  a.c = rows(cc);
  a.gate = rows(gate);
  a.o = rows(o);
  a.a = a_;
  a.skip = skip;
  a.bias = bias;
  a.first = state_in;
  a.last = state_out;
  hipStream_t s = (hipStream_t)stream;
  scan_instance(c, [&](auto type, auto S) {
    k_scan_step<decltype(type), decltype(S)::value><<<(uint32_t)ceil_div(columns, kColumns), kBlock, 0, s>>>(a);
  });
  return launch_status();
}
