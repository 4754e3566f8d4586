// seq_norm.hip -- root-mean-square norm with the residual's addition: forward,
// forward with an 8-bit output, backward.  The C ABI is in include/qd_seq.h.
//
// All three are bound by memory: 8 bytes (16-bit types) move per element
// forward and again backward, against some ten operations.  A row is read once
// and stays in registers between its sum and its use: one wave holds a row of up
// to 64 lanes * 32 elements, four waves one of up to four times that.
#include <algorithm>

#include "seq_common.hpp"
#include "seq_rows.hpp"

namespace seq {
namespace {

constexpr int kBlock = 256;
constexpr float kFp8Max = 448.0f;
constexpr float kFp8Floor = 0x1p-100f;   // a smaller maximum would make 448 / maximum overflow
constexpr int kBackwardBlocks = 512;     // two workgroups per compute unit, each with its own dweight

// Sum over the lanes that share a row: part of a wave, a wave, or the workgroup.
// `part` has a place per wave; two calls that follow each other use different ones.
template <int TPR> __device__ inline float row_sum(float x, float* part) {
#pragma unroll
  for (int m = 1; m < TPR && m < 64; m <<= 1) x += shfl_xor(x, m);
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = (part[0] + part[1]) + (part[2] + part[3]);
  }
  return x;
}
template <int TPR> __device__ inline float row_max(float x, float* part) {
#pragma unroll
  for (int m = 1; m < TPR && m < 64; m <<= 1) x = fmaxf(x, shfl_xor(x, m));
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  }
  return x;
}

__device__ inline float fp8_scale(float top) {
  return top == 0.0f ? 1.0f : fmaxf(top, kFp8Floor) * (1.0f / kFp8Max);
}
// Clamped to the largest e4m3 number (what is beyond it by rounding would turn
// into not-a-number); not-a-number stays.
__device__ inline float fp8_clamp(float x) {
  x = x > kFp8Max ? kFp8Max : x;
  return x < -kFp8Max ? -kFp8Max : x;
}
__device__ inline uint32_t fp8_pack4(const float* v) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(fp8_clamp(v[0]), fp8_clamp(v[1]), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(fp8_clamp(v[2]), fp8_clamp(v[3]), r, true);
}
__device__ inline uint8_t fp8_one(float v) {
  return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(fp8_clamp(v), 0.0f, 0, false);
}

template <int VEC> __device__ inline void fp8_store(uint8_t* q, const float* v) {
  uint32_t e[VEC / 4];
#pragma unroll
  for (int i = 0; i < VEC / 4; ++i) e[i] = fp8_pack4(v + 4 * i);
  __builtin_memcpy(q, e, VEC);
}

struct ForwardArgs {
  const void *x, *r, *w;
  void *y, *h;
  float* rstd;      // or the scales of an 8-bit output
  int64_t x_stride, r_stride, rows;
  int32_t width;
  float eps;
  bool w32;
  int64_t first;    // the launch's first row
};

enum { kPlain = 0, kFp8Row = 1, kFp8Group = 2 };

// One pass.  TPR lanes hold a row, each NV packs of VEC elements, pack j at
// column (j TPR + lane) VEC: every load of a wave is one contiguous piece.
// 32000 x 1024 bfloat16: 49 us, 5.3 TB/s.  131072 x 4096 with a scale per 128: 638 us,
// 5.9 TB/s.  79133 rows of 73 halves, whose packs overlap: 17 us, 2.3 TB/s.
template <class T, int VEC, int NV, int TPR, bool TAIL, int MODE>
__global__ __launch_bounds__(kBlock) void k_norm(ForwardArgs a) {
  __shared__ float part[8];
  constexpr int ROWS = kBlock / TPR;
  const int lane = threadIdx.x % TPR;
  const int64_t row = a.first + (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  if (TPR <= 64 && row >= a.rows) return;      // no barrier below for rows that waves hold
  const T* x = (const T*)a.x + row * a.x_stride;
  const T* r = a.r ? (const T*)a.r + row * a.r_stride : nullptr;
  float h[NV][VEC];
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (j * TPR + lane) * VEC;
#pragma unroll
    for (int i = 0; i < VEC; ++i) h[j][i] = 0.0f;
    const int at = pack_at<VEC, TAIL>(col, a.width);
    if (col < a.width) {
      load<T, VEC>(h[j], x + at);
      if (r) {
        float t[VEC];
        load<T, VEC>(t, r + at);
#pragma unroll
        for (int i = 0; i < VEC; ++i) h[j][i] += t[i];
      }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const float own = TAIL && at + i < col ? 0.0f : h[j][i];
      sum = fmaf(own, own, sum);
    }
  }
  sum = row_sum<TPR>(sum, part);
  const float rstd = rsqrtf(sum / (float)a.width + a.eps);
  float top = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (j * TPR + lane) * VEC;
    if (col < a.width) {
      const int at = pack_at<VEC, TAIL>(col, a.width);
      store<T, VEC>((T*)a.h + row * a.width + at, h[j]);
      float w[VEC];
      load_weight<T, VEC>(w, a.w, a.w32, at);
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[j][i] = h[j][i] * rstd * w[i];
      if constexpr (MODE == kPlain) store<T, VEC>((T*)a.y + row * a.width + at, h[j]);
      if constexpr (MODE == kFp8Row) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) top = fmaxf(top, fabsf(h[j][i]));
      }
    }
  }
  if constexpr (MODE == kPlain) {
    if (lane == 0) a.rstd[row] = rstd;
  } else if constexpr (MODE == kFp8Row) {
    top = row_max<TPR>(top, part + 4);
    const float scale = fp8_scale(top), inv = 1.0f / scale;
    if (lane == 0) a.rstd[row] = scale;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (j * TPR + lane) * VEC;
      if (col >= a.width) continue;
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[j][i] *= inv;
      fp8_store<VEC>((uint8_t*)a.y + row * a.width + pack_at<VEC, TAIL>(col, a.width), h[j]);
    }
  } else {
    // 128 columns are 128 / VEC neighbouring lanes (all of them real, as 128 divides the width).
    static_assert(MODE == kPlain || TPR >= 128 / VEC, "a group is within a row's lanes");
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (j * TPR + lane) * VEC;
      float t = 0.0f;
#pragma unroll
      for (int i = 0; i < VEC; ++i) t = fmaxf(t, fabsf(h[j][i]));
#pragma unroll
      for (int m = 1; m < 128 / VEC; m <<= 1) t = fmaxf(t, shfl_xor(t, m));
      if (col >= a.width) continue;
      const float scale = fp8_scale(t), inv = 1.0f / scale;
      if (lane % (128 / VEC) == 0) a.rstd[row * (a.width / 128) + col / 128] = scale;
      uint8_t* q = (uint8_t*)a.y + row * a.width + col;
#pragma unroll
      for (int i = 0; i < VEC; ++i) h[j][i] *= inv;
      fp8_store<VEC>(q, h[j]);
    }
  }
}

// Rows of any width and alignment, read again for each use (from the caches): a
// workgroup per row.
template <class T, int MODE>
__global__ __launch_bounds__(kBlock) void k_norm_any(ForwardArgs a) {
  __shared__ float part[8];
  const int64_t row = a.first + blockIdx.x;
  const T* x = (const T*)a.x + row * a.x_stride;
  const T* r = a.r ? (const T*)a.r + row * a.r_stride : nullptr;
  auto at = [&](int c) { return to_f32(x[c]) + (r ? to_f32(r[c]) : 0.0f); };
  float sum = 0.0f;
  for (int c = threadIdx.x; c < a.width; c += kBlock) {
    const float h = at(c);
    sum = fmaf(h, h, sum);
  }
  sum = row_sum<kBlock>(sum, part);
  const float rstd = rsqrtf(sum / (float)a.width + a.eps);
  auto out = [&](int c, float h) {
    float w;
    load_weight<T, 1>(&w, a.w, a.w32, c);
    return h * rstd * w;
  };
  if constexpr (MODE == kPlain) {
    if (threadIdx.x == 0) a.rstd[row] = rstd;
    for (int c = threadIdx.x; c < a.width; c += kBlock) {
      const float h = at(c);
      ((T*)a.h)[row * a.width + c] = from_f32<T>(h);
      ((T*)a.y)[row * a.width + c] = from_f32<T>(out(c, h));
    }
  } else if constexpr (MODE == kFp8Row) {
    float top = 0.0f;
    for (int c = threadIdx.x; c < a.width; c += kBlock) {
      const float h = at(c);
      ((T*)a.h)[row * a.width + c] = from_f32<T>(h);
      top = fmaxf(top, fabsf(out(c, h)));
    }
    top = row_max<kBlock>(top, part + 4);
    const float scale = fp8_scale(top), inv = 1.0f / scale;
    if (threadIdx.x == 0) a.rstd[row] = scale;
    for (int c = threadIdx.x; c < a.width; c += kBlock)
      ((uint8_t*)a.y)[row * a.width + c] = fp8_one(out(c, at(c)) * inv);
  } else {
    const int lane = threadIdx.x & 63;
    for (int g = threadIdx.x >> 6; g < a.width / 128; g += kBlock / 64) {
      const int c = g * 128 + lane;
      const float h0 = at(c), h1 = at(c + 64);
      ((T*)a.h)[row * a.width + c] = from_f32<T>(h0);
      ((T*)a.h)[row * a.width + c + 64] = from_f32<T>(h1);
      const float y0 = out(c, h0), y1 = out(c + 64, h1);
      const float scale = fp8_scale(wave_max(fmaxf(fabsf(y0), fabsf(y1)))), inv = 1.0f / scale;
      if (lane == 0) a.rstd[row * (a.width / 128) + g] = scale;
      ((uint8_t*)a.y)[row * a.width + c] = fp8_one(y0 * inv);
      ((uint8_t*)a.y)[row * a.width + c + 64] = fp8_one(y1 * inv);
    }
  }
}

struct BackwardArgs {
  const void *dy, *dh, *h, *w;
  const float* rstd;
  void *dx, *dw;
  float* partial;   // [blocks][width]
  int64_t dy_stride, dh_stride, h_stride, rows;
  int32_t width, blocks;
  bool w32;
};

// g = dy w;  dx = dh + rstd (g - h rstd^2 mean(g h));  dw = sum over rows of dy h rstd.
// A workgroup takes rows blockIdx.x, + gridDim.x, ... (four at a time where a
// wave holds a row) and keeps its share of dw in registers; k_norm_dweight adds
// the workgroups' shares in a fixed order.  32000 x 1024 bfloat16: 48 us, 5.4 TB/s.
// dw is formed from h as stored, so it carries h's rounding.
template <class T, int VEC, int NV, int TPR, bool TAIL>
__global__ __launch_bounds__(kBlock) void k_norm_backward(BackwardArgs a) {
  __shared__ float part[8];
  constexpr int ROWS = kBlock / TPR;
  __shared__ float shares[ROWS > 1 ? (ROWS - 1) * TPR * VEC * NV : 1];
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float dw[NV][VEC], w[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (j * TPR + lane) * VEC;
#pragma unroll
    for (int i = 0; i < VEC; ++i) dw[j][i] = w[j][i] = 0.0f;
    if (col < a.width) load_weight<T, VEC>(w[j], a.w, a.w32, pack_at<VEC, TAIL>(col, a.width));
  }
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += (int64_t)gridDim.x * ROWS) {
    const int64_t row = first + sub;
    if (TPR <= 64 && row >= a.rows) break;     // no barrier inside the loop for rows that waves hold
    const float rstd = a.rstd[row];
    float g[NV][VEC], h[NV][VEC], d[NV][VEC];
    float dot = 0.0f;
    // all of the row's loads are under way before the first is used
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (j * TPR + lane) * VEC;
#pragma unroll
      for (int i = 0; i < VEC; ++i) g[j][i] = h[j][i] = d[j][i] = 0.0f;
      const int at = pack_at<VEC, TAIL>(col, a.width);
      if (col < a.width) {
        load<T, VEC>(g[j], (const T*)a.dy + row * a.dy_stride + at);
        load<T, VEC>(h[j], (const T*)a.h + row * a.h_stride + at);
        if (a.dh) load<T, VEC>(d[j], (const T*)a.dh + row * a.dh_stride + at);
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (j * TPR + lane) * VEC, at = pack_at<VEC, TAIL>(col, a.width);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        h[j][i] *= rstd;
        dw[j][i] = fmaf(g[j][i], h[j][i], dw[j][i]);
        g[j][i] *= w[j][i];
        dot = fmaf(TAIL && at + i < col ? 0.0f : g[j][i], h[j][i], dot);
      }
    }
    dot = row_sum<TPR>(dot, part + 4 * (turn & 1)) / (float)a.width;
    turn ^= 1;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (j * TPR + lane) * VEC;
      if (col >= a.width) continue;
#pragma unroll
      for (int i = 0; i < VEC; ++i) d[j][i] += rstd * (g[j][i] - h[j][i] * dot);
      store<T, VEC>((T*)a.dx + row * a.width + pack_at<VEC, TAIL>(col, a.width), d[j]);
    }
  }
  if constexpr (ROWS > 1) {
    // the shares of the lanes that hold the same columns, added in their order
    if (sub > 0) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) shares[((sub - 1) * NV * VEC + j * VEC + i) * TPR + lane] = dw[j][i];
    }
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int s = 0; s < ROWS - 1; ++s)
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) dw[j][i] += shares[(s * NV * VEC + j * VEC + i) * TPR + lane];
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (j * TPR + lane) * VEC;
    if (col >= a.width) continue;
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      a.partial[(int64_t)blockIdx.x * a.width + pack_at<VEC, TAIL>(col, a.width) + i] = dw[j][i];
  }
}

// Rows of any width, read again for each use; dw goes through memory that only
// this thread touches.
template <class T> __global__ __launch_bounds__(kBlock) void k_norm_backward_any(BackwardArgs a) {
  __shared__ float part[8];
  float* mine = a.partial + (int64_t)blockIdx.x * a.width;
  for (int c = threadIdx.x; c < a.width; c += kBlock) mine[c] = 0.0f;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float rstd = a.rstd[row];
    const T* dy = (const T*)a.dy + row * a.dy_stride;
    const T* hp = (const T*)a.h + row * a.h_stride;
    float dot = 0.0f;
    for (int c = threadIdx.x; c < a.width; c += kBlock) {
      const float d = to_f32(dy[c]), h = to_f32(hp[c]) * rstd;
      float w;
      load_weight<T, 1>(&w, a.w, a.w32, c);
      mine[c] = fmaf(d, h, mine[c]);
      dot = fmaf(d * w, h, dot);
    }
    dot = row_sum<kBlock>(dot, part + 4 * (turn & 1)) / (float)a.width;
    turn ^= 1;
    for (int c = threadIdx.x; c < a.width; c += kBlock) {
      float w;
      load_weight<T, 1>(&w, a.w, a.w32, c);
      float d = a.dh ? to_f32(((const T*)a.dh)[row * a.dh_stride + c]) : 0.0f;
      d += rstd * (to_f32(dy[c]) * w - to_f32(hp[c]) * rstd * dot);
      ((T*)a.dx)[row * a.width + c] = from_f32<T>(d);
    }
  }
}

// 64 columns per workgroup: sixteen waves each add every sixteenth share (a column's
// chain of loads is what takes the time: 777 columns of fp32 take 7.9 us with four
// waves, 3.9 with sixteen).
constexpr int kJoinWaves = 16;
template <class T> __global__ __launch_bounds__(64 * kJoinWaves) void k_norm_dweight(BackwardArgs a) {
  __shared__ float part[64 * kJoinWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + lane;
  float sum = 0.0f;
  if (col < a.width) {
#pragma unroll 8
    for (int b = wave; b < a.blocks; b += kJoinWaves) sum += a.partial[(int64_t)b * a.width + col];
  }
  part[threadIdx.x] = sum;
  __syncthreads();
  if (wave == 0 && col < a.width) {
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) sum += part[w * 64 + lane];
    if (a.w32)
      ((float*)a.dw)[col] = sum;
    else
      ((T*)a.dw)[col] = from_f32<T>(sum);
  }
}

qds_status validate(const qds_norm_config* c) {
  if (!c || c->abi_version != QDS_ABI_VERSION) return QDS_ERR_INVALID_ARG;
  if (c->dtype < QDS_F32 || c->dtype > QDS_F16) return QDS_ERR_INVALID_ARG;
  if (c->weight_dtype != QDS_F32 && c->weight_dtype != c->dtype) return QDS_ERR_INVALID_ARG;
  if (c->width < 1 || c->width > (1 << 20)) return QDS_ERR_INVALID_ARG;
  if (c->rows < 0 || c->rows > 0x7fffffff) return QDS_ERR_INVALID_ARG;
  if (!(c->eps >= 0.0f)) return QDS_ERR_INVALID_ARG;
  if (c->group != 0 && (c->group != 128 || c->width % 128 != 0)) return QDS_ERR_INVALID_ARG;
  return QDS_OK;
}

// Calls f(VEC, NV, TPR) as compile-time values for the least that holds a row
// in registers; returns false where nothing does.  Up to 32 elements a lane, so that
// loads of a whole row are in flight at once.  Few lanes for narrow rows: with a wave
// for each, 127238 rows of 128 took 47 us; with 16 lanes, 20 us.
// fp32 rows beyond 4096 take eight packs of four: 9947 x 4697 forward and backward
// 299 us, read again for each use 668.
template <class T, bool TAIL, class F> bool with_lanes(int width, F&& f) {
  constexpr int V = 16 / sizeof(T);
  const Int<TAIL> tail{};
  if (width < V) return false;
  if (width <= 16 * V) f(Int<V>{}, Int<1>{}, Int<16>{}, tail);
  else if (width <= 32 * V) f(Int<V>{}, Int<1>{}, Int<32>{}, tail);
  else if (width <= 64 * V) f(Int<V>{}, Int<1>{}, Int<64>{}, tail);
  else if (width <= 128 * V) f(Int<V>{}, Int<2>{}, Int<64>{}, tail);
  else if (width <= 256 * V) f(Int<V>{}, Int<4>{}, Int<64>{}, tail);
  else if (width <= 512 * V) f(Int<V>{}, Int<2>{}, Int<256>{}, tail);
  else if (width <= 1024 * V) f(Int<V>{}, Int<4>{}, Int<256>{}, tail);
  else if (V == 4 && width <= 2048 * V) f(Int<V>{}, Int<V == 4 ? 8 : 4>{}, Int<256>{}, tail);
  else return false;
  return true;
}
template <class T, class F> bool with_shape(int width, F&& f) {
  return width % (16 / sizeof(T)) ? with_lanes<T, true>(width, f) : with_lanes<T, false>(width, f);
}

// One launch for as many rows as one takes workgroups for, another for what is left.
template <class F> void over_rows(ForwardArgs a, int rows_per_block, F&& launch) {
  const int64_t step = (int64_t)most_blocks(kBlock) * rows_per_block;
  for (a.first = 0; a.first < a.rows; a.first += step)
    launch(a, (uint32_t)ceil_div(std::min(a.rows - a.first, step), rows_per_block));
}

template <class T, int MODE> void forward(const ForwardArgs& args, hipStream_t s) {
  auto any = [&] {
    over_rows(args, 1, [&](const ForwardArgs& a, uint32_t grid) { k_norm_any<T, MODE><<<grid, kBlock, 0, s>>>(a); });
  };
  const bool held = with_shape<T>(args.width, [&](auto V, auto NV, auto TPR, auto TAIL) {
    constexpr int v = decltype(V)::value, nv = decltype(NV)::value, tpr = decltype(TPR)::value;
    constexpr bool tail = decltype(TAIL)::value;
    if constexpr (MODE != kFp8Group || (tpr >= 128 / v && !tail))
      over_rows(args, kBlock / tpr, [&](const ForwardArgs& a, uint32_t grid) {
        k_norm<T, v, nv, tpr, tail, MODE><<<grid, kBlock, 0, s>>>(a);
      });
    else
      any();
  });
  if (!held) any();
}

template <int MODE> qds_status run_forward(const qds_norm_config* c, const ForwardArgs& a, void* stream) {
  if (c->rows == 0) return QDS_OK;
  hipStream_t s = (hipStream_t)stream;
  if (c->dtype == QDS_F32) forward<float, MODE>(a, s);
  else if (c->dtype == QDS_BF16) forward<bf16, MODE>(a, s);
  else forward<half, MODE>(a, s);
  return launch_status();
}

// Workgroups of the backward pass: enough to fill the card, no more than rows.
int backward_blocks(const qds_norm_config* c) {
  return (int)(c->rows < kBackwardBlocks ? (c->rows > 0 ? c->rows : 1) : kBackwardBlocks);
}

template <class T> void backward(BackwardArgs a, hipStream_t s) {
  if (a.rows > 0) {
    const bool held = with_shape<T>(a.width, [&](auto V, auto NV, auto TPR, auto TAIL) {
      constexpr int v = decltype(V)::value, nv = decltype(NV)::value, tpr = decltype(TPR)::value;
    constexpr bool tail = decltype(TAIL)::value;
      const int64_t most = ceil_div(a.rows, kBlock / tpr);
      if (a.blocks > most) a.blocks = (int)most;
      k_norm_backward<T, v, nv, tpr, tail><<<a.blocks, kBlock, 0, s>>>(a);
    });
    if (!held) k_norm_backward_any<T><<<a.blocks, kBlock, 0, s>>>(a);
  } else {
    a.blocks = 0;
  }
  k_norm_dweight<T><<<ceil_div(a.width, 64), 64 * kJoinWaves, 0, s>>>(a);
}

}  // namespace
}  // namespace seq

using namespace seq;

extern "C" qds_status qds_residual_norm(const qds_norm_config* c, const void* x, int64_t x_stride,
                                        const void* residual, int64_t residual_stride,
                                        const void* weight, void* y, void* h, float* rstd,
                                        void* stream) {
  const qds_status st = validate(c);
  if (st != QDS_OK) return st;
  if (c->group != 0) return QDS_ERR_INVALID_ARG;
  if (c->rows > 0 && (!x || !weight || !y || !h || !rstd)) return QDS_ERR_INVALID_ARG;
  const ForwardArgs a{x, residual, weight, y, h, rstd, x_stride, residual_stride, c->rows,
                      c->width, c->eps, c->weight_dtype == QDS_F32, 0};
  return run_forward<kPlain>(c, a, stream);
}

extern "C" qds_status qds_residual_norm_fp8(const qds_norm_config* c, const void* x,
                                            int64_t x_stride, const void* residual,
                                            int64_t residual_stride, const void* weight, void* q,
                                            float* scale, void* h, void* stream) {
  const qds_status st = validate(c);
  if (st != QDS_OK) return st;
  if (c->rows > 0 && (!x || !weight || !q || !scale || !h)) return QDS_ERR_INVALID_ARG;
  const ForwardArgs a{x, residual, weight, q, h, scale, x_stride, residual_stride, c->rows,
                      c->width, c->eps, c->weight_dtype == QDS_F32, 0};
  return c->group ? run_forward<kFp8Group>(c, a, stream) : run_forward<kFp8Row>(c, a, stream);
}

extern "C" qds_status qds_residual_norm_backward_workspace(const qds_norm_config* c, uint64_t* bytes) {
  const qds_status st = validate(c);
  if (st != QDS_OK) return st;
  if (!bytes) return QDS_ERR_INVALID_ARG;
  *bytes = align_up((uint64_t)backward_blocks(c) * c->width * sizeof(float));
  return QDS_OK;
}

extern "C" qds_status qds_residual_norm_backward(const qds_norm_config* c, const void* dy,
                                                 int64_t dy_stride, const void* dh,
                                                 int64_t dh_stride, const void* h, int64_t h_stride,
                                                 const float* rstd, const void* weight, void* dx,
                                                 void* dweight, void* workspace,
                                                 uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  const qds_status st = qds_residual_norm_backward_workspace(c, &need);
  if (st != QDS_OK) return st;
  if (c->group != 0 || !dweight || !workspace || !weight || ((uintptr_t)workspace & 255))
    return QDS_ERR_INVALID_ARG;
  if (c->rows > 0 && (!dy || !h || !rstd || !dx)) return QDS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return QDS_ERR_WORKSPACE_TOO_SMALL;
  const BackwardArgs a{dy, dh, h, weight, rstd, dx, dweight, (float*)workspace, dy_stride, dh_stride,
                       h_stride, c->rows, c->width, backward_blocks(c), c->weight_dtype == QDS_F32};
  hipStream_t s = (hipStream_t)stream;
  if (c->dtype == QDS_F32) backward<float>(a, s);
  else if (c->dtype == QDS_BF16) backward<bf16>(a, s);
  else backward<half>(a, s);
  return launch_status();
}

extern "C" const char* qds_status_str(qds_status status) {
  switch (status) {
    case QDS_OK: return "ok";
    case QDS_ERR_INVALID_ARG: return "invalid argument";
    case QDS_ERR_WORKSPACE_TOO_SMALL: return "workspace too small";
    case QDS_ERR_UNSUPPORTED: return "unsupported configuration";
    case QDS_ERR_HIP: return "HIP runtime or launch error";
  }
  return "unknown status";
}
