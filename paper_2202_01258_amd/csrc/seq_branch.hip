// seq_branch.hip -- the norms before and after a block's branch, with the branch's gate and the
// residual's scale: forward and backward.  The C ABI is in include/qd_seq.h.
//
// Bound by memory: with a gate, five rows move forward and eight backward, against some 20 and
// 50 operations per element.  A row is read once and stays in registers: the two sums over
// it follow each other (the second norm is of what the first one scales).  32000 x 1024 bfloat16:
// forward 59 us (5.5 TB/s), backward 115 us (4.6 TB/s); 9973 x 777 float32: 27 and 52 us.
#include <algorithm>

#include "seq_common.hpp"
#include "seq_rows.hpp"

namespace seq {
namespace {

constexpr int kBlock = 256;
constexpr int kBackwardBlocks = 512;      // two workgroups per compute unit, each with its own shares of dweight

struct BranchArgs {
  const void *x, *g, *r, *w1, *w2, *dy, *dh;
  void *y, *h, *dx, *dg, *dr, *dw1, *dw2;
  float *rstds;             // [2][rows]: of x, of h
  float *partial;           // [blocks][2][width]
  int64_t x_stride, g_stride, r_stride, dy_stride, dh_stride, rows, first;
  int32_t width, blocks;
  float eps, scale;
  bool w32;
};

// Sum over the lanes that share a row: part of a wave, a wave, or the workgroup.  `part` has a
// place per wave; two calls that follow each other use different ones.
template <int TPR> __device__ inline float row_sum(float x, float* part) {
#pragma unroll
  for (int m = 1; m < TPR && m < 64; m <<= 1) x += shfl_xor(x, m);
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) x += part[w];
  }
  return x;
}
template <int TPR> constexpr int kThreads = TPR > kBlock ? TPR : kBlock;

template <class T, int VEC, int NV, int TPR, bool TAIL> __global__ __launch_bounds__(kThreads<TPR>) void k_branch(BranchArgs a) {
  __shared__ float part[2][TPR > 64 ? TPR / 64 : 1];
  constexpr int ROWS = kThreads<TPR> / TPR;
  const int lane = threadIdx.x % TPR;
  const int64_t row = a.first + (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  if (TPR <= 64 && row >= a.rows) return;        // no barrier below for rows that waves hold
  const T *x = (const T*)a.x + row * a.x_stride, *r = (const T*)a.r + row * a.r_stride;
  const T* g = a.g ? (const T*)a.g + row * a.g_stride : nullptr;
  float n[NV][VEC], h[NV][VEC], z[NV][VEC], sum = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (j * TPR + lane) * VEC, at = pack_at<VEC, TAIL>(col, a.width);
#pragma unroll
    for (int i = 0; i < VEC; ++i) n[j][i] = h[j][i] = z[j][i] = 0.0f;
    if (col < a.width) {
      load<T, VEC>(n[j], x + at);
      load<T, VEC>(h[j], r + at);
      if (g) load<T, VEC>(z[j], g + at);
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (j * TPR + lane) * VEC, at = pack_at<VEC, TAIL>(col, a.width);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const float own = TAIL && at + i < col ? 0.0f : n[j][i];
      sum = fmaf(own, own, sum);
    }
  }
  const float rx = rsqrtf(row_sum<TPR>(sum, part[0]) / (float)a.width + a.eps);
  sum = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (j * TPR + lane) * VEC, at = pack_at<VEC, TAIL>(col, a.width);
    if (col < a.width) {
      float w[VEC];
      load_weight<T, VEC>(w, a.w1, a.w32, at);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float p = n[j][i] * rx * w[i], open = g ? z[j][i] * sigmoid(z[j][i]) : 1.0f;
        h[j][i] = fmaf(open, p, a.scale * h[j][i]);
        const float own = TAIL && at + i < col ? 0.0f : h[j][i];
        sum = fmaf(own, own, sum);
      }
      store<T, VEC>((T*)a.h + row * a.width + at, h[j]);
    }
  }
  const float rh = rsqrtf(row_sum<TPR>(sum, part[1]) / (float)a.width + a.eps);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (j * TPR + lane) * VEC, at = pack_at<VEC, TAIL>(col, a.width);
    if (col < a.width) {
      float w[VEC];
      load_weight<T, VEC>(w, a.w2, a.w32, at);
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[j][i] = h[j][i] * rh * w[i];
      store<T, VEC>((T*)a.y + row * a.width + at, h[j]);
    }
  }
  if (lane == 0) {
    a.rstds[row] = rx;
    a.rstds[a.rows + row] = rh;
  }
}

// A pack as it lies in memory: 16-bit numbers take half the registers until they are used
// (a training pass, bfloat16: 32000 x 1024 195 us with floats, 182 so; 130000 x 128 108 and 94).
template <class T, int VEC> __device__ inline void fetch(Pack<T, VEC>& e, const T* p) { __builtin_memcpy(&e, p, sizeof(e)); }

// With n = x rx, p = n w1, m = h rh:  e = dy w2;  gh = dh + rh (e - m mean(e m));  dw2 = sum of dy m;
// dr = scale gh;  dgate = gh p silu'(gate);  f = gh silu(gate) w1;  dx = rx (f - n mean(f n));  dw1 = sum of gh silu(gate) n.
// h is formed again from its terms, as the stored one is rounded.  A workgroup takes rows
// blockIdx.x, + gridDim.x, ... and keeps its shares of dw1 and dw2 in registers.
template <class T, int VEC, int NV, int TPR, bool TAIL> __global__ __launch_bounds__(kThreads<TPR>) void k_branch_backward(BranchArgs a) {
  __shared__ float part[2][2][TPR > 64 ? TPR / 64 : 1];
  constexpr int ROWS = kThreads<TPR> / TPR;
  __shared__ float shares[ROWS > 1 ? (ROWS - 1) * TPR * VEC * NV * 2 : 1];
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  // The weights are read again for each row (from the caches): kept, they would take the
  // registers of another wave.
  float dw1[NV][VEC], dw2[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) dw1[j][i] = dw2[j][i] = 0.0f;
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += (int64_t)gridDim.x * ROWS) {
    const int64_t row = first + sub;
    if (TPR <= 64 && row >= a.rows) break;       // no barrier inside the loop for rows that waves hold
    const float rx = a.rstds[row], rh = a.rstds[a.rows + row];
    Pack<T, VEC> x[NV], z[NV], e[NV], d[NV], r[NV];
    float m[NV][VEC], dot = 0.0f;              // m; from the second sum on f
    // all of the row's loads are under way before the first is used
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (j * TPR + lane) * VEC, at = pack_at<VEC, TAIL>(col, a.width);
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[j].v[i] = z[j].v[i] = e[j].v[i] = d[j].v[i] = r[j].v[i] = (T)0.0f;
      if (col < a.width) {
        fetch(x[j], (const T*)a.x + row * a.x_stride + at);
        fetch(r[j], (const T*)a.r + row * a.r_stride + at);
        if (a.g) fetch(z[j], (const T*)a.g + row * a.g_stride + at);
        fetch(e[j], (const T*)a.dy + row * a.dy_stride + at);
        if (a.dh) fetch(d[j], (const T*)a.dh + row * a.dh_stride + at);
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (j * TPR + lane) * VEC, at = pack_at<VEC, TAIL>(col, a.width);
      float w1[VEC] = {}, w2[VEC] = {};
      if (col < a.width) {
        load_weight<T, VEC>(w1, a.w1, a.w32, at);
        load_weight<T, VEC>(w2, a.w2, a.w32, at);
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float zz = to_f32(z[j].v[i]), dy = to_f32(e[j].v[i]), open = a.g ? zz * sigmoid(zz) : 1.0f;
        m[j][i] = fmaf(open, to_f32(x[j].v[i]) * rx * w1[i], a.scale * to_f32(r[j].v[i])) * rh;
        dw2[j][i] = fmaf(dy, m[j][i], dw2[j][i]);
        dot = fmaf(TAIL && at + i < col ? 0.0f : dy * w2[i], m[j][i], dot);
      }
    }
    dot = row_sum<TPR>(dot, part[turn][0]) / (float)a.width;
    float dot2 = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (j * TPR + lane) * VEC, at = pack_at<VEC, TAIL>(col, a.width);
      float v[VEC], gh[VEC], w1[VEC] = {}, w2[VEC] = {};
      if (col < a.width) {
        load_weight<T, VEC>(w1, a.w1, a.w32, at);
        load_weight<T, VEC>(w2, a.w2, a.w32, at);
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        gh[i] = to_f32(d[j].v[i]) + rh * (to_f32(e[j].v[i]) * w2[i] - m[j][i] * dot);
        v[i] = a.scale * gh[i];
      }
      if (col < a.width) store<T, VEC>((T*)a.dr + row * a.width + at, v);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float zz = to_f32(z[j].v[i]), s = sigmoid(zz), open = a.g ? zz * s : 1.0f, n = to_f32(x[j].v[i]) * rx;
        v[i] = gh[i] * (n * w1[i]) * silu_slope(zz, s);
        const float f = gh[i] * open;
        dw1[j][i] = fmaf(f, n, dw1[j][i]);
        m[j][i] = f * w1[i];
        dot2 = fmaf(TAIL && at + i < col ? 0.0f : m[j][i], n, dot2);
      }
      if (a.g && col < a.width) store<T, VEC>((T*)a.dg + row * a.width + at, v);
    }
    dot2 = row_sum<TPR>(dot2, part[turn][1]) / (float)a.width;
    turn ^= 1;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (j * TPR + lane) * VEC;
      if (col >= a.width) continue;
      float v[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = rx * (m[j][i] - to_f32(x[j].v[i]) * rx * dot2);
      store<T, VEC>((T*)a.dx + row * a.width + pack_at<VEC, TAIL>(col, a.width), v);
    }
  }
  if constexpr (ROWS > 1) {
    // the shares of the lanes that hold the same columns, added in their order
    constexpr int SUMS = NV * VEC;
    if (sub > 0) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          shares[((sub - 1) * 2 * SUMS + j * VEC + i) * TPR + lane] = dw1[j][i];
          shares[((sub - 1) * 2 * SUMS + SUMS + j * VEC + i) * TPR + lane] = dw2[j][i];
        }
    }
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int s = 0; s < ROWS - 1; ++s)
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          dw1[j][i] += shares[(s * 2 * SUMS + j * VEC + i) * TPR + lane];
          dw2[j][i] += shares[(s * 2 * SUMS + SUMS + j * VEC + i) * TPR + lane];
        }
  }
  float* mine = a.partial + (int64_t)blockIdx.x * 2 * a.width;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (j * TPR + lane) * VEC, at = pack_at<VEC, TAIL>(col, a.width);
    if (col >= a.width) continue;
    store<float, VEC>(mine + at, dw1[j]);
    store<float, VEC>(mine + a.width + at, dw2[j]);
  }
}

// Rows of any width, read again for each use (from the caches): a workgroup per row.
template <class T> struct AnyRow {
  const BranchArgs& a;
  int64_t row;
  __device__ float x(int c) const { return to_f32(((const T*)a.x)[row * a.x_stride + c]); }
  __device__ float gate(int c) const { return to_f32(((const T*)a.g)[row * a.g_stride + c]); }
  __device__ float weight(const void* w, int c) const {
    float v;
    load_weight<T, 1>(&v, w, a.w32, c);
    return v;
  }
  __device__ float open(int c) const { return a.g ? gate(c) * sigmoid(gate(c)) : 1.0f; }
  __device__ float h(int c, float rx) const {
    return fmaf(open(c), x(c) * rx * weight(a.w1, c), a.scale * to_f32(((const T*)a.r)[row * a.r_stride + c]));
  }
};
template <class T> __global__ __launch_bounds__(kBlock) void k_branch_any(BranchArgs a) {
  __shared__ float part[2][kBlock / 64];
  const AnyRow<T> r{a, a.first + blockIdx.x};
  float sum = 0.0f;
  for (int c = threadIdx.x; c < a.width; c += kBlock) sum = fmaf(r.x(c), r.x(c), sum);
  const float rx = rsqrtf(row_sum<kBlock>(sum, part[0]) / (float)a.width + a.eps);
  sum = 0.0f;
  for (int c = threadIdx.x; c < a.width; c += kBlock) {
    const float h = r.h(c, rx);
    sum = fmaf(h, h, sum);
  }
  const float rh = rsqrtf(row_sum<kBlock>(sum, part[1]) / (float)a.width + a.eps);
  for (int c = threadIdx.x; c < a.width; c += kBlock) {
    const float h = r.h(c, rx);
    ((T*)a.h)[r.row * a.width + c] = from_f32<T>(h);
    ((T*)a.y)[r.row * a.width + c] = from_f32<T>(h * rh * r.weight(a.w2, c));
  }
  if (threadIdx.x == 0) {
    a.rstds[r.row] = rx;
    a.rstds[a.rows + r.row] = rh;
  }
}
template <class T> __global__ __launch_bounds__(kBlock) void k_branch_backward_any(BranchArgs a) {
  __shared__ float part[2][2][kBlock / 64];
  float *dw1 = a.partial + (int64_t)blockIdx.x * 2 * a.width, *dw2 = dw1 + a.width;
  for (int c = threadIdx.x; c < a.width; c += kBlock) dw1[c] = dw2[c] = 0.0f;     // only this thread's columns
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const AnyRow<T> r{a, row};
    const float rx = a.rstds[row], rh = a.rstds[a.rows + row];
    const T* dy = (const T*)a.dy + row * a.dy_stride;
    float dot = 0.0f, dot2 = 0.0f;
    for (int c = threadIdx.x; c < a.width; c += kBlock) {
      const float d = to_f32(dy[c]), m = r.h(c, rx) * rh;
      dw2[c] = fmaf(d, m, dw2[c]);
      dot = fmaf(d * r.weight(a.w2, c), m, dot);
    }
    dot = row_sum<kBlock>(dot, part[turn][0]) / (float)a.width;
    auto gh = [&](int c) {
      const float d = a.dh ? to_f32(((const T*)a.dh)[row * a.dh_stride + c]) : 0.0f;
      return d + rh * (to_f32(dy[c]) * r.weight(a.w2, c) - r.h(c, rx) * rh * dot);
    };
    for (int c = threadIdx.x; c < a.width; c += kBlock) {
      const float d = gh(c), n = r.x(c) * rx, w = r.weight(a.w1, c), f = d * r.open(c);
      ((T*)a.dr)[row * a.width + c] = from_f32<T>(a.scale * d);
      if (a.g) ((T*)a.dg)[row * a.width + c] = from_f32<T>(d * (n * w) * silu_slope(r.gate(c), sigmoid(r.gate(c))));
      dw1[c] = fmaf(f, n, dw1[c]);
      dot2 = fmaf(f * w, n, dot2);
    }
    dot2 = row_sum<kBlock>(dot2, part[turn][1]) / (float)a.width;
    turn ^= 1;
    for (int c = threadIdx.x; c < a.width; c += kBlock)
      ((T*)a.dx)[row * a.width + c] = from_f32<T>(rx * (gh(c) * r.open(c) * r.weight(a.w1, c) - r.x(c) * rx * dot2));
  }
}

// 64 columns per workgroup: sixteen waves each add every sixteenth share.
constexpr int kJoinWaves = 16;
template <class T> __global__ __launch_bounds__(64 * kJoinWaves) void k_branch_dweight(BranchArgs a) {
  __shared__ float part[64 * kJoinWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, which = blockIdx.y;
  const int col = blockIdx.x * 64 + lane;
  float sum = 0.0f;
  if (col < a.width) {
#pragma unroll 8
    for (int b = wave; b < a.blocks; b += kJoinWaves) sum += a.partial[((int64_t)b * 2 + which) * a.width + col];
  }
  part[threadIdx.x] = sum;
  __syncthreads();
  if (wave == 0 && col < a.width) {
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) sum += part[w * 64 + lane];
    void* to = which ? a.dw2 : a.dw1;
    if (a.w32)
      ((float*)to)[col] = sum;
    else
      ((T*)to)[col] = from_f32<T>(sum);
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
qds_status validate(const qds_branch_config* c) {
  if (!c || c->abi_version != QDS_ABI_VERSION) return QDS_ERR_INVALID_ARG;
  if (c->dtype < QDS_F32 || c->dtype > QDS_F16) return QDS_ERR_INVALID_ARG;
  if (c->weight_dtype != QDS_F32 && c->weight_dtype != c->dtype) return QDS_ERR_INVALID_ARG;
  if (c->width < 1 || c->width > (1 << 20)) return QDS_ERR_INVALID_ARG;
  if (c->rows < 0 || c->rows > 0x7fffffff) return QDS_ERR_INVALID_ARG;
  if (!(c->eps >= 0.0f) || !(c->residual_scale - c->residual_scale == 0.0f)) return QDS_ERR_INVALID_ARG;
  return QDS_OK;
}

// Calls f(VEC, NV, TPR, TAIL) as compile-time values for the least that holds a row in
// registers, up to 16 elements a lane; returns false where nothing does.
template <class T, bool TAIL, class F> bool with_lanes(int width, F&& f) {
  constexpr int V = 16 / sizeof(T), M = 16 / V;          // elements of a pack; packs a lane may have
  const Int<TAIL> tail{};
  if (width < V) return false;
  if (width <= 16 * V) f(Int<V>{}, Int<1>{}, Int<16>{}, tail);
  else if (width <= 32 * V) f(Int<V>{}, Int<1>{}, Int<32>{}, tail);
  else if (width <= 64 * V) f(Int<V>{}, Int<1>{}, Int<64>{}, tail);
  else if (width <= 128 * V) f(Int<V>{}, Int<2>{}, Int<64>{}, tail);
  else if (V == 4 && width <= 256 * V) f(Int<V>{}, Int<M>{}, Int<64>{}, tail);
  else if (width <= 256 * V) f(Int<V>{}, Int<1>{}, Int<256>{}, tail);
  else if (width <= 512 * V) f(Int<V>{}, Int<2>{}, Int<256>{}, tail);
  else if (V == 4 && width <= 1024 * V) f(Int<V>{}, Int<M>{}, Int<256>{}, tail);
  else if (width <= 512 * M * V) f(Int<V>{}, Int<M>{}, Int<512>{}, tail);
  else return false;
  return true;
}
template <class T, class F> bool with_shape(int width, F&& f) {
  return width % (16 / sizeof(T)) ? with_lanes<T, true>(width, f) : with_lanes<T, false>(width, f);
}
template <class F> void with_type(const qds_branch_config* c, F&& f) {
  if (c->dtype == QDS_F32) f(float());
  else if (c->dtype == QDS_BF16) f(bf16());
  else f(half());
}

// One launch for as many rows as one takes workgroups for, another for what is left.
template <class F> void over_rows(BranchArgs a, int threads, int rows_per_block, F&& launch) {
  const int64_t step = (int64_t)most_blocks(threads) * rows_per_block;
  for (a.first = 0; a.first < a.rows; a.first += step)
    launch(a, (uint32_t)ceil_div(std::min(a.rows - a.first, step), rows_per_block));
}

int backward_blocks(const qds_branch_config* c) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(c->rows, kBackwardBlocks));
}

BranchArgs args_of(const qds_branch_config* c) {
  BranchArgs a{};
  a.rows = c->rows;
  a.width = c->width;
  a.eps = c->eps;
  a.scale = c->residual_scale;
  a.w32 = c->weight_dtype == QDS_F32;
  return a;
}

}  // namespace
}  // namespace seq

using namespace seq;

extern "C" qds_status qds_branch_norm(const qds_branch_config* c, const void* x, int64_t x_stride, const void* gate,
                                      int64_t gate_stride, const void* residual, int64_t residual_stride,
                                      const void* branch_weight, const void* weight, void* y, void* h, float* rstds,
                                      void* stream) {
  const qds_status st = validate(c);
  if (st != QDS_OK) return st;
  if (c->rows == 0) return QDS_OK;
  if (!x || !residual || !branch_weight || !weight || !y || !h || !rstds) return QDS_ERR_INVALID_ARG;
  BranchArgs args = args_of(c);
  args.x = x;
  args.x_stride = x_stride;
  args.g = gate;
  args.g_stride = gate_stride;
  args.r = residual;
  args.r_stride = residual_stride;
  args.w1 = branch_weight;
  args.w2 = weight;
  args.y = y;
  args.h = h;
  args.rstds = rstds;
  hipStream_t s = (hipStream_t)stream;
  with_type(c, [&](auto type) {
    using T = decltype(type);
    const bool held = with_shape<T>(c->width, [&](auto V, auto NV, auto TPR, auto TAIL) {
      constexpr int tpr = decltype(TPR)::value, threads = kThreads<tpr>;
      over_rows(args, threads, threads / tpr, [&](const BranchArgs& a, uint32_t grid) {
        k_branch<T, decltype(V)::value, decltype(NV)::value, tpr, decltype(TAIL)::value><<<grid, threads, 0, s>>>(a);
      });
    });
    if (!held) over_rows(args, kBlock, 1, [&](const BranchArgs& a, uint32_t grid) { k_branch_any<T><<<grid, kBlock, 0, s>>>(a); });
  });
  return launch_status();
}

extern "C" qds_status qds_branch_norm_backward_workspace(const qds_branch_config* c, uint64_t* bytes) {
  const qds_status st = validate(c);
  if (st != QDS_OK) return st;
  if (!bytes) return QDS_ERR_INVALID_ARG;
  *bytes = align_up((uint64_t)backward_blocks(c) * 2 * c->width * sizeof(float));
  return QDS_OK;
}

extern "C" qds_status qds_branch_norm_backward(const qds_branch_config* c, const void* dy, int64_t dy_stride,
                                               const void* dh, int64_t dh_stride, const void* x, int64_t x_stride,
                                               const void* gate, int64_t gate_stride, const void* residual,
                                               int64_t residual_stride, const float* rstds, const void* branch_weight,
                                               const void* weight, void* dx, void* dgate, void* dresidual,
                                               void* dbranch_weight, void* dweight, void* workspace,
                                               uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  const qds_status st = qds_branch_norm_backward_workspace(c, &need);
  if (st != QDS_OK) return st;
  if (!branch_weight || !weight || !dbranch_weight || !dweight || !workspace || ((uintptr_t)workspace & 255))
    return QDS_ERR_INVALID_ARG;
  if (c->rows > 0 && (!dy || !x || !residual || !rstds || !dx || !dresidual || (gate && !dgate))) return QDS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return QDS_ERR_WORKSPACE_TOO_SMALL;
  BranchArgs a = args_of(c);
  a.dy = dy;
  a.dy_stride = dy_stride;
  a.dh = dh;
  a.dh_stride = dh_stride;
  a.x = x;
  a.x_stride = x_stride;
  a.g = gate;
  a.g_stride = gate_stride;
  a.r = residual;
  a.r_stride = residual_stride;
  a.rstds = const_cast<float*>(rstds);
  a.w1 = branch_weight;
  a.w2 = weight;
  a.dx = dx;
  a.dg = dgate;
  a.dr = dresidual;
  a.dw1 = dbranch_weight;
  a.dw2 = dweight;
  a.partial = (float*)workspace;
  a.blocks = c->rows > 0 ? backward_blocks(c) : 0;
  hipStream_t s = (hipStream_t)stream;
  with_type(c, [&](auto type) {
    using T = decltype(type);
    if (a.rows > 0) {
      const bool held = with_shape<T>(c->width, [&](auto V, auto NV, auto TPR, auto TAIL) {
        constexpr int tpr = decltype(TPR)::value, threads = kThreads<tpr>;
        a.blocks = (int)std::min<int64_t>(a.blocks, ceil_div(a.rows, threads / tpr));
        k_branch_backward<T, decltype(V)::value, decltype(NV)::value, tpr, decltype(TAIL)::value><<<a.blocks, threads, 0, s>>>(a);
      });
      if (!held) k_branch_backward_any<T><<<a.blocks, kBlock, 0, s>>>(a);
    }
    k_branch_dweight<T><<<dim3((uint32_t)ceil_div(a.width, 64), 2), 64 * kJoinWaves, 0, s>>>(a);
  });
  return launch_status();
}
