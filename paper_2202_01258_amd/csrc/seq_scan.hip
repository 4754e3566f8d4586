// seq_scan.hip -- selective state space scan: forward and one row.  The C ABI is in
// include/qd_seq.h, the layout of the work in seq_scan.hpp.
//
// Bound by the vector units.  A state of a row takes an exponential (8.2 cycles of a wave on a
// SIMD), two products and an fma (2.7 each), its output another fma: at 16 states 65 cycles for 16
// columns of a piece's row and 76 of an output's.  With lane moves, transposes, softplus, gate, LDS reads and
// accesses they take 143 and 176.  1 x 65536 x 1024 bfloat16: 490 us, where the bytes take 111; under the tracer, which
// lengthens it to 556, 243 us for the pieces, 13 to join them and 300 for the outputs.
#include <algorithm>

#include "seq_scan.hpp"

namespace seq {
namespace {

constexpr int kBlock = 256, kColumns = kBlock / 4;

// One segment of 64 columns.  LOCAL: what the segment leaves behind when it starts from
// zero, and the sum of its steps; otherwise outputs, marks and the last state.
template <class T, int S, bool LOCAL, bool GATE, bool TAIL> __global__ __launch_bounds__(kBlock) void k_scan(ScanArgs a) {
  constexpr int K = kScanRows, N = 4 * S, QUADS = K / 4;
  SEQ_SHARED float bc[2][K * 2 * N];
  const int q = threadIdx.x & 3;
  const Quad quad(q);
  const uint32_t item = blockIdx.x / (uint32_t)a.col_blocks;
  const int col = (blockIdx.x % (uint32_t)a.col_blocks) * kColumns + (threadIdx.x >> 2);
  const bool real = col < a.width;
  const int at = real ? col : a.width - 1;
  const Item which(item, a.batch);                         // of LOCAL all but the last segments: nothing comes behind those
  const int64_t b = which.b;
  const int seg = which.part;
  const int n = rows_in(a, b), begin = seg * a.seg, end = min(begin + a.seg, a.length), live = min(end, n);
  float rates[S], h[S];
  load_rates<S>(rates, a, at, q);
  const Held<S> held(q, a.states);
  const float bias = a.bias ? a.bias[at] : 0.0f, skip = a.skip ? a.skip[at] : 0.0f;
  const int64_t place = ((b * a.segs + seg) * a.width + at) * N + q * S;
  if (LOCAL) {
#pragma unroll
    for (int s = 0; s < S; ++s) h[s] = 0.0f;
  } else if (a.joined) {
    load_floats<S>(h, a.left_state + place);
  } else {
    load_states<S>(h, a.first ? a.first + b * a.width * a.states : nullptr, at, q, a.states);
    follow<S, false>(h, a, rates, b, seg, at, q);
  }
  float time = 0.0f;
  Track<T> out(a.o, (int64_t)a.length * a.width, a.width, b, begin, q, at, real);
  if (begin < live) {
    uint32_t u[QUADS], d[QUADS], z[QUADS];
    Track<T> tu(a.u, b, begin, q, at, real), td(a.delta, b, begin, q, at, real), tz(a.gate, b, begin, q, at, real);
    StagedRows<T, S, K, kBlock> rows(a, b, begin);
    float* marks = a.marks + (b * a.blocks + begin / K) * a.width * N;
    auto fetch = [&](int t) {
      const Left left{live - t - q - 1};
#pragma unroll
      for (int i = 0; i < QUADS; ++i) {
        u[i] = tu.load(i, left);
        d[i] = td.load(i, left);
        if (GATE) z[i] = tz.load(i, left);
      }
      rows.load(live - t);
      tu.move(K);
      td.move(K);
      if (GATE) tz.move(K);
      rows.move(K);
    };
    fetch(begin);
    rows.store(bc[0]);
    __syncthreads();
    int buffer = 0;
    for (int t = begin; t < live; t += K) {
      const Left left{live - t - q - 1};
      float dt[QUADS], uu[QUADS], zz[QUADS];
#pragma unroll
      for (int i = 0; i < QUADS; ++i) {
        dt[i] = left.keep(i, softplus<T>(number<T>(d[i]) + bias).dt);
        uu[i] = number<T>(u[i]);
        if (GATE) zz[i] = number<T>(z[i]);
      }
      const bool more = t + K < live;
      if (more) fetch(t + K);
      if (!LOCAL && a.marks) {
        if (real) store_floats<S>(marks + (uint32_t)(at * N + q * S), h);
        marks += (int64_t)a.width * N;
      }
      const float* lds = bc[buffer] + q * S;
      auto form = [&](auto CAREFUL) {
        constexpr bool careful = decltype(CAREFUL)::value;
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
#pragma unroll
            for (int s = 0; s < S; ++s) {
              h[s] = fmaf(fast_exp2(dtj * rates[s]), h[s], xj * bv[s]);
              if (careful) h[s] = held.keep(s, h[s]);
              if (!LOCAL) y[j] = s == 0 ? h[s] * cv[s] : fmaf(h[s], cv[s], y[j]);
            }
          };
          row(Int<0>{});
          row(Int<1>{});
          row(Int<2>{});
          row(Int<3>{});
          if (LOCAL) {
            time += dt[i];
          } else {
            float o = fmaf(skip, uu[i], quad_rows(y, quad));
            if (GATE) o *= zz[i] * sigmoid(zz[i]);
            out.store(i, left, o);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      if (TAIL && !LOCAL && any_from<128>(dt[0] * uu[0], dt[1] * uu[1])) form(std::true_type{});
      else form(std::false_type{});
      if (!LOCAL) out.move(K);
      if (more) {
        rows.store(bc[buffer ^ 1]);
        __syncthreads();
        buffer ^= 1;
      }
    }
  }
  if (LOCAL) {
    time = quad_sum(time);
    held.keep_all(h);
    if (real) store_floats<S>(a.left_state + place, h);
    if (real && q == 0) a.left_time[(b * a.segs + seg) * a.width + at] = time;
  } else {
    out = Track<T>(a.o, (int64_t)a.length * a.width, a.width, b, max(begin, live), q, at, real);
    for (int t = max(begin, live); t < end; t += 4) {
      out.store(0, Left{end - t - q - 1}, 0.0f);
      out.move(4);
    }
    if (seg == a.segs - 1 && a.last) store_states<S>(a.last + b * a.width * a.states, at, q, a.states, real, h);
  }
}

// One row: the state is what is read and written, a lane's share in one access at any alignment
// (one by one, 8192 x 512 columns of 16 states took 281 us, now 118, 4.8 TB/s).  Where four
// lanes hold more states than there are (TAIL), the last lanes take the last S, some of which a
// neighbour in the wave has as well: both write the same, and only the neighbour counts them.
template <class T, int S, bool TAIL> __global__ __launch_bounds__(kBlock) void k_scan_step(ScanArgs a) {
  const uint32_t id = blockIdx.x * kBlock + threadIdx.x, column = id >> 2;
  if (column >= (uint32_t)(a.batch * a.width)) return;
  const int q = threadIdx.x & 3, n = pack_at<S, TAIL>(q * S, a.states);
  const int64_t b = column / (uint32_t)a.width;
  const int at = (int)(column % (uint32_t)a.width);
  float r[S], h[S], bv[S], cv[S], y = 0.0f;
  load<float, S>(h, a.first + (int64_t)column * a.states + n);
  load<float, S>(r, a.a + (int64_t)at * a.states + n);
  load<T, S>(bv, (const T*)row_of<T>(a.b, b, 0) + n);
  load<T, S>(cv, (const T*)row_of<T>(a.c, b, 0) + n);
  const float u = to_f32(row_of<T>(a.u, b, 0)[at]);
  const float dt = softplus<T>(to_f32(row_of<T>(a.delta, b, 0)[at]) + (a.bias ? a.bias[at] : 0.0f)).dt;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    h[s] = fmaf(fast_exp2(dt * rate(r[s])), h[s], dt * u * bv[s]);
    y = TAIL && n + s < q * S ? y : fmaf(h[s], cv[s], y);
  }
  store<float, S>(a.last + (int64_t)column * a.states + n, h);
  y = quad_sum(y);
  if (q == 0) {
    float o = fmaf(a.skip ? a.skip[at] : 0.0f, u, y);
    if (a.gate.p) {
      const float z = to_f32(row_of<T>(a.gate, b, 0)[at]);
      o *= z * sigmoid(z);
    }
    ((T*)a.o)[column] = from_f32<T>(o);
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// Two waves on each SIMD do without cuts; fewer are cut to eight (a pass over the pieces costs what 0.65 to
// 0.8 of the main pass does).  Outputs of rows by 1000, bfloat16, whole and cut, in us, by waves:
//   16 states  1024: 121, 121   1536: 163, 172   1792: 164, 199   2048: 165, 214   2304: 220, 246   4096: 280, 378
//    4 states  1024:  89,  69   1536: 105, 100   1792: 111, 116   2048: 121, 131   2304: 151, 156   4096: 197, 245
// so that 16 states could do without from 1536 on.  1 x 65536 x 1024: 634 us cut for two waves, 522 for eight.  (The
// last two before b and c were staged by eight rows, which took 0.95 of that.)
constexpr int64_t kWhole = 2048, kWaves = 8192;
constexpr int kLeastRows = 32;

Cut forward_cut(const qds_scan_config* c) { return cut(c, whole_waves(c) >= kWhole ? 1 : kWaves, kLeastRows, kScanRows); }
uint64_t state_bytes(const qds_scan_config* c, int segs) {
  return align_up((uint64_t)c->batch * segs * c->width * 4 * lane_states(c) * sizeof(float));
}
bool fits(const qds_scan_config* c) {
  const int segs = forward_cut(c).segs;
  return (int64_t)c->batch <= (int64_t)most_blocks(kBlock) / (ceil_div(c->width, kColumns) * segs) && joinable(c, segs);
}

}  // namespace
}  // namespace seq

using namespace seq;

extern "C" qds_status qds_selective_scan_marks(const qds_scan_config* c, uint64_t* bytes) {
  const qds_status st = validate_scan(c, false);
  if (st != QDS_OK) return st;
  if (!bytes) return QDS_ERR_INVALID_ARG;
  *bytes = state_bytes(c, mark_count(c));
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
                                         const float* state_in, const int32_t* lengths, void* o, float* state_out,
                                         void* marks, void* workspace, uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  const qds_status st = qds_selective_scan_workspace(c, &need);
  if (st != QDS_OK) return st;
  if (c->batch == 0) return QDS_OK;
  if (!a_ || (c->length > 0 && (!u.data || !delta.data || !b.data || !cc.data || !o))) return QDS_ERR_INVALID_ARG;
  for (qds_rows* r : {&u, &delta, &b, &cc, &gate})
    if (!near_rows(*r, c->length)) return QDS_ERR_UNSUPPORTED;
  if (state_out && state_out == state_in) return QDS_ERR_INVALID_ARG;      // all segments read one, the last writes the other
  if (((uintptr_t)marks & 255) || (need > 0 && (!workspace || ((uintptr_t)workspace & 255)))) return QDS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return QDS_ERR_WORKSPACE_TOO_SMALL;
  ScanArgs a = scan_args(c);
  const Cut parts = forward_cut(c);
  a.u = rows(u);
  a.delta = rows(delta);
  a.b = rows(b);
  a.c = rows(cc);
  a.gate = rows(gate);
  a.o = o;
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
  a.piece = a.seg;
  a.pieces = a.segs;
  a.ratio = 1;
  a.joined = a.pieces > kFewPieces;
  if (a.segs > 1) {
    a.left_state = (float*)workspace;
    a.left_time = (float*)((char*)workspace + state_bytes(c, a.segs));
  }
  hipStream_t s = (hipStream_t)stream;
  scan_instance(c, [&](auto type, auto S, auto TAIL) {
    using T = decltype(type);
    constexpr int L = decltype(S)::value;
    constexpr bool tail = decltype(TAIL)::value;
    const uint32_t across = (uint32_t)(a.batch * a.col_blocks);
    if (a.segs > 1) {
      k_scan<T, L, true, false, false><<<across * (a.segs - 1), kBlock, 0, s>>>(a);
      if (a.joined) k_scan_join<4 * L, false><<<(uint32_t)ceil_div((int64_t)a.batch * a.width * 4 * L, 16), kScanJoin, 0, s>>>(a);
    }
    if (gate.data) k_scan<T, L, false, true, tail><<<across * a.segs, kBlock, 0, s>>>(a);
    else k_scan<T, L, false, false, tail><<<across * a.segs, kBlock, 0, s>>>(a);
  });
  return launch_status();
}

extern "C" qds_status qds_selective_scan_step(const qds_scan_config* c, qds_rows u, qds_rows delta, const float* a_,
                                              qds_rows b, qds_rows cc, const float* skip, qds_rows gate,
                                              const float* bias, const float* state_in, void* o, float* state_out,
                                              void* stream) {
  const qds_status st = validate_scan(c, true);
  if (st != QDS_OK) return st;
  if (c->batch == 0) return QDS_OK;
  if (!a_ || !u.data || !delta.data || !b.data || !cc.data || !o || !state_in || !state_out) return QDS_ERR_INVALID_ARG;
  const int64_t columns = (int64_t)c->batch * c->width;
  if (ceil_div(columns, kColumns) > most_blocks(kBlock)) return QDS_ERR_UNSUPPORTED;
  ScanArgs a = scan_args(c);
  a.u = rows(u);
  a.delta = rows(delta);
  a.b = rows(b);
  a.c = rows(cc);
  a.gate = rows(gate);
  a.o = o;
  a.a = a_;
  a.skip = skip;
  a.bias = bias;
  a.first = state_in;
  a.last = state_out;
  hipStream_t s = (hipStream_t)stream;
  scan_instance(c, [&](auto type, auto S, auto TAIL) {
    const uint32_t grid = (uint32_t)ceil_div(columns, kColumns);
    k_scan_step<decltype(type), decltype(S)::value, decltype(TAIL)::value><<<grid, kBlock, 0, s>>>(a);
  });
  return launch_status();
}
