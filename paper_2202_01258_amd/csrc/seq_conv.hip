// seq_conv.hip -- short causal convolution over the rows of an episode, each column by
// itself: forward, backward, one row.  The C ABI is in include/qd_seq.h.
//
// All are bound by memory: forward moves two elements per element, backward three,
// against some 20 and 40 vector instructions.  A thread holds a pack of columns, whose
// weights stay in registers, and goes down a chunk of rows with the last taps - 1 of
// them in registers too; a chunk reads the rows in front of it once more.  131072 x 2048 float16,
// forward: 204 us (5.3 TB/s); 32 episodes of up to 1000 rows x 1024 bfloat16: forward 25 us, backward 41.
#include <algorithm>

#include "seq_common.hpp"
#include "seq_rows.hpp"

namespace seq {
namespace {

constexpr int kBlock = 256;
// Columns a thread holds, and rows whose loads are under way together: few columns leave registers
// for many waves.  16 bits, 32 x 1000 x 1024, forward and backward: two columns and eight rows
// 88 us, four and four 98; fp32, 16 x 1000 x 777: 78 and 70.
template <class T> constexpr int kVec = sizeof(T) == 2 ? 2 : 4;
template <int VEC> constexpr int kRowsAhead = VEC == 2 ? 8 : 4;

struct Rows {
  char* p;
  int64_t b, t;                          // strides in elements
};
Rows rows(const qds_rows& r) { return Rows{(char*)r.data, r.stride[0], r.stride[1]}; }
template <class T> __device__ inline T* row_of(const Rows& r, int64_t b, int64_t t) {
  return (T*)r.p + b * r.b + t * r.t;
}

struct ConvArgs {
  Rows x, y, dy, dx;
  const void *w, *bias, *first, *dlast;  // states before the first row, gradient of those behind the last
  void *last, *dw, *dbias, *dfirst;
  const int32_t* lengths;
  float* partial;                        // [shares][taps + 1][width]: each workgroup's share of dweight and dbias
  int32_t batch, length, width, chunk, chunks, packs, shares, lanes;
  bool w32, silu;
};
__device__ inline int rows_of(const ConvArgs& a, int64_t b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.length) : a.length;
}

// Row t of an episode; rows before its first are the state's.
template <class T, int VEC, int TAPS> __device__ inline void load_row(float* out, const ConvArgs& a, int64_t b, int t, int at) {
  if (t >= 0) {
    load<T, VEC>(out, row_of<T>(a.x, b, t) + at);
  } else if (a.first) {
    load<T, VEC>(out, (const T*)a.first + (b * (TAPS - 1) + (t + TAPS - 1)) * a.width + at);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) out[i] = 0.0f;
  }
}
template <class T, int VEC, int TAPS> __device__ inline void load_weights(float (*w)[VEC], float* bias, const ConvArgs& a, int at) {
#pragma unroll
  for (int k = 0; k < TAPS; ++k) load_weight<T, VEC>(w[k], a.w32 ? (const void*)((const float*)a.w + (int64_t)k * a.width) : (const void*)((const T*)a.w + (int64_t)k * a.width), a.w32, at);
#pragma unroll
  for (int i = 0; i < VEC; ++i) bias[i] = 0.0f;
  if (a.bias) load_weight<T, VEC>(bias, a.bias, a.w32, at);
}

// A thread has a pack of columns of a chunk of rows.
template <class T, int VEC, int TAPS, bool TAIL> __global__ __launch_bounds__(kBlock) void k_conv(ConvArgs a) {
  const uint32_t id = blockIdx.x * kBlock + threadIdx.x;
  const uint32_t item = id / (uint32_t)a.packs, pack = id % (uint32_t)a.packs;
  if (item >= (uint32_t)(a.batch * a.chunks)) return;
  const int64_t b = item / (uint32_t)a.chunks;
  const int chunk = (int)(item % (uint32_t)a.chunks);
  const int at = pack_at<VEC, TAIL>((int)pack * VEC, a.width);
  const int n = rows_of(a, b);
  const int begin = chunk * a.chunk, end = min(begin + a.chunk, a.length), live = min(end, n);
  if (chunk == 0 && a.last) {
#pragma unroll
    for (int i = 0; i < TAPS - 1; ++i) {
      float v[VEC];
      load_row<T, VEC, TAPS>(v, a, b, n - (TAPS - 1) + i, at);
      store<T, VEC>((T*)a.last + (b * (TAPS - 1) + i) * a.width + at, v);
    }
  }
  float w[TAPS][VEC], bias[VEC];
  load_weights<T, VEC, TAPS>(w, bias, a, at);
  constexpr int AHEAD = kRowsAhead<VEC>;
  // rows t - TAPS + 1 .. t + AHEAD - 1
  float x[TAPS - 1 + AHEAD][VEC];
  if (begin < live) {
#pragma unroll
    for (int i = 0; i < TAPS - 1; ++i) load_row<T, VEC, TAPS>(x[i], a, b, begin - (TAPS - 1) + i, at);
  }
  for (int t = begin; t < live; t += AHEAD) {
    // a chunk's last rows may be fewer: those behind are read again as the last, and not stored
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load<T, VEC>(x[TAPS - 1 + i], row_of<T>(a.x, b, min(t + i, live - 1)) + at);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      float y[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float p = bias[e];
#pragma unroll
        for (int k = 0; k < TAPS; ++k) p = fmaf(w[k][e], x[i + k][e], p);
        y[e] = a.silu ? p * sigmoid(p) : p;
      }
      if (t + i < live) store<T, VEC>(row_of<T>(a.y, b, t + i) + at, y);
    }
#pragma unroll
    for (int i = 0; i < TAPS - 1; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[i][e] = x[i + AHEAD][e];
  }
  const float zero[VEC] = {};
  for (int t = max(begin, live); t < end; ++t) store<T, VEC>(row_of<T>(a.y, b, t) + at, zero);
}

// g_t = dy_t act'(p_t);  dx_s = sum_k weight[k] g_{s + taps - 1 - k};  dweight[k] = sum_t g_t x_{t - taps + 1 + k}.
// A thread goes down its chunk and the taps - 1 rows behind it, whose g its last rows need.
// A workgroup's threads hold `lanes` packs of columns, times kBlock / lanes chunks at a time;
// it adds its threads' shares of dweight and leaves their sum for k_conv_dweight.
template <class T, int VEC, int TAPS, bool TAIL, bool SILU> __global__ __launch_bounds__(kBlock) void k_conv_backward(ConvArgs a) {
  constexpr int SUMS = (TAPS + 1) * VEC, AHEAD = kRowsAhead<VEC>;
  __shared__ float shares[kBlock / 2 * SUMS];
  const int lane = threadIdx.x & (a.lanes - 1), sub = threadIdx.x / (uint32_t)a.lanes, subs = kBlock / a.lanes;
  const int pack = blockIdx.x * a.lanes + lane;
  const bool real = pack < a.packs;
  const int col = pack * VEC, at = real ? pack_at<VEC, TAIL>(col, a.width) : 0;
  float w[TAPS][VEC], bias[VEC], sum[TAPS + 1][VEC];
  load_weights<T, VEC, TAPS>(w, bias, a, at);
#pragma unroll
  for (int k = 0; k <= TAPS; ++k)
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum[k][e] = 0.0f;
  const uint32_t items = real ? (uint32_t)(a.batch * a.chunks) : 0;
  for (uint32_t item = blockIdx.y * subs + sub; item < items; item += gridDim.y * subs) {
    const int64_t b = item / (uint32_t)a.chunks;
    const int chunk = (int)(item % (uint32_t)a.chunks);
    const int n = rows_of(a, b);
    const int begin = chunk * a.chunk, end = min(begin + a.chunk, a.length), live = min(end, n);
    // dx of the state's rows comes from the first chunk (also of an episode without rows)
    const int from = chunk == 0 ? -(TAPS - 1) : begin;
    auto out = [&](int s, float* v) {
      const int i = s - n + (TAPS - 1);              // the row's place in the last state
      if (a.dlast && i >= 0) {
        float d[VEC];
        load<T, VEC>(d, (const T*)a.dlast + (b * (TAPS - 1) + i) * a.width + at);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] += d[e];
      }
      if (s >= 0)
        store<T, VEC>(row_of<T>(a.dx, b, s) + at, v);
      else if (a.dfirst)
        store<T, VEC>((T*)a.dfirst + (b * (TAPS - 1) + s + TAPS - 1) * a.width + at, v);
    };
    if (from < live) {
      const int stop = live + TAPS - 1;                // rows t up to here: dx of row t - TAPS + 1
      float x[TAPS][VEC], g[TAPS][VEC];                // rows t - TAPS + 1 .. t
#pragma unroll
      for (int i = 0; i < TAPS; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) g[i][e] = 0.0f;
#pragma unroll
      for (int i = 1; i < TAPS; ++i) load_row<T, VEC, TAPS>(x[i], a, b, begin - TAPS + i, at);
      Pack<T, VEC> nx[AHEAD], ny[AHEAD];
      auto fetch = [&](int t0) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          const int t = max(min(t0 + i, n - 1), 0);
          __builtin_memcpy(&nx[i], row_of<T>(a.x, b, t) + at, sizeof(nx[i]));
          __builtin_memcpy(&ny[i], row_of<T>(a.dy, b, t) + at, sizeof(ny[i]));
        }
      };
      // INNER: all of the rows are the chunk's own
      auto advance = [&](int t0, auto INNER) {
        constexpr bool inner = decltype(INNER)::value;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          const int t = t0 + i;
          if (!inner && t >= stop) break;
          const bool in = inner || t < n, own = inner || t < live;
          float v[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
#pragma unroll
            for (int k = 0; k < TAPS - 1; ++k) {
              x[k][e] = x[k + 1][e];
              g[k][e] = g[k + 1][e];
            }
            x[TAPS - 1][e] = in ? to_f32(nx[i].v[e]) : 0.0f;
            float d = in ? to_f32(ny[i].v[e]) : 0.0f;
            if (SILU) {
              float p = bias[e];
#pragma unroll
              for (int k = 0; k < TAPS; ++k) p = fmaf(w[k][e], x[k][e], p);
              d = in ? d * silu_slope(p, sigmoid(p)) : 0.0f;
            }
            g[TAPS - 1][e] = d;
#pragma unroll
            for (int k = 0; k < TAPS; ++k) sum[k][e] = own ? fmaf(d, x[k][e], sum[k][e]) : sum[k][e];
            sum[TAPS][e] += own ? d : 0.0f;
            v[e] = w[0][e] * d;
#pragma unroll
            for (int k = 1; k < TAPS; ++k) v[e] = fmaf(w[k][e], g[TAPS - 1 - k][e], v[e]);
          }
          const int s = t - TAPS + 1;
          if (s >= from) {
            if (!inner || s < 0) out(s, v);
            else store<T, VEC>(row_of<T>(a.dx, b, s) + at, v);      // no row of the last state yet
          }
        }
      };
      int t0 = begin;
      if (n > 0) fetch(t0);
      while (t0 + AHEAD <= live) {
        advance(t0, std::true_type{});
        t0 += AHEAD;
        fetch(t0);
      }
      while (t0 < stop) {
        advance(t0, std::false_type{});
        t0 += AHEAD;
        if (n > 0 && t0 < stop) fetch(t0);
      }
    }
    const float zero[VEC] = {};
    for (int t = max(begin, live); t < end; ++t) store<T, VEC>(row_of<T>(a.dx, b, t) + at, zero);
  }
  // halves of the chunks' threads, added pairwise in their order
  for (int half = subs / 2; half > 0; half /= 2) {
    __syncthreads();
    if (sub >= half && sub < 2 * half) {
#pragma unroll
      for (int k = 0; k <= TAPS; ++k)
#pragma unroll
        for (int e = 0; e < VEC; ++e) shares[((sub - half) * SUMS + k * VEC + e) * a.lanes + lane] = sum[k][e];
    }
    __syncthreads();
    if (sub < half) {
#pragma unroll
      for (int k = 0; k <= TAPS; ++k)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[k][e] += shares[(sub * SUMS + k * VEC + e) * a.lanes + lane];
    }
  }
  if (sub == 0 && real) {
#pragma unroll
    for (int k = 0; k <= TAPS; ++k)
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        a.partial[((int64_t)blockIdx.y * (TAPS + 1) + k) * a.width + at + e] = sum[k][e];
  }
}

// 64 columns of one tap per workgroup: sixteen waves each add every sixteenth share.
constexpr int kJoinWaves = 16;
template <class T> __global__ __launch_bounds__(64 * kJoinWaves) void k_conv_dweight(ConvArgs a, int taps) {
  __shared__ float part[64 * kJoinWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, k = blockIdx.y;
  const int col = blockIdx.x * 64 + lane;
  float sum = 0.0f;
  if (col < a.width) {
#pragma unroll 8
    for (int s = wave; s < a.shares; s += kJoinWaves) sum += a.partial[((int64_t)s * (taps + 1) + k) * a.width + col];
  }
  part[threadIdx.x] = sum;
  __syncthreads();
  void* to = k < taps ? a.dw : a.dbias;
  if (wave == 0 && col < a.width && to) {
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kJoinWaves; ++i) sum += part[i * 64 + lane];
    const int64_t place = (k < taps ? (int64_t)k * a.width : 0) + col;
    if (a.w32)
      ((float*)to)[place] = sum;
    else
      ((T*)to)[place] = from_f32<T>(sum);
  }
}

template <class T, int VEC, int TAPS, bool TAIL> __global__ __launch_bounds__(kBlock) void k_conv_step(ConvArgs a) {
  const uint32_t id = blockIdx.x * kBlock + threadIdx.x, pack = id % (uint32_t)a.packs;
  const int64_t b = id / (uint32_t)a.packs;
  if (b >= a.batch) return;
  const int at = pack_at<VEC, TAIL>((int)pack * VEC, a.width);
  // The state may be written where it is read: columns that a neighbour has as well are
  // the neighbour's to store.
  const int skip = TAIL ? (int)pack * VEC - at : 0;
  auto put = [&](T* to, const float* v) {
    if (!TAIL || skip == 0) {
      store<T, VEC>(to, v);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (e >= skip) to[e] = from_f32<T>(v[e]);
    }
  };
  float w[TAPS][VEC], p[VEC], x[TAPS][VEC];
  load_weights<T, VEC, TAPS>(w, p, a, at);
#pragma unroll
  for (int i = 0; i < TAPS - 1; ++i) load_row<T, VEC, TAPS>(x[i], a, b, i - (TAPS - 1), at);
  load<T, VEC>(x[TAPS - 1], row_of<T>(a.x, b, 0) + at);
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
#pragma unroll
    for (int k = 0; k < TAPS; ++k) p[e] = fmaf(w[k][e], x[k][e], p[e]);
    p[e] = a.silu ? p[e] * sigmoid(p[e]) : p[e];
  }
  put(row_of<T>(a.y, b, 0) + at, p);
#pragma unroll
  for (int i = 0; i < TAPS - 1; ++i) put((T*)a.last + (b * (TAPS - 1) + i) * a.width + at, x[i + 1]);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
constexpr int kShares = 2048;            // workgroups of the backward pass, each with a share of dweight

qds_status validate(const qds_conv_config* c, bool step) {
  if (!c || c->abi_version != QDS_ABI_VERSION) return QDS_ERR_INVALID_ARG;
  if (c->dtype < QDS_F32 || c->dtype > QDS_F16) return QDS_ERR_INVALID_ARG;
  if (c->weight_dtype != QDS_F32 && c->weight_dtype != c->dtype) return QDS_ERR_INVALID_ARG;
  if (c->batch < 0 || (!step && (c->length < 0 || c->length >= (1 << 30)))) return QDS_ERR_INVALID_ARG;
  if (c->width < 1 || c->width > (1 << 20) || c->taps < 1 || c->taps > 8) return QDS_ERR_INVALID_ARG;
  if (c->silu != 0 && c->silu != 1) return QDS_ERR_INVALID_ARG;
  return QDS_OK;
}

int vec_of(const qds_conv_config* c) { return c->dtype == QDS_F32 ? kVec<float> : kVec<bf16>; }
int pack_width(const qds_conv_config* c) { return c->width < vec_of(c) ? 1 : vec_of(c); }
int packs_of(const qds_conv_config* c) { return (int)ceil_div(c->width, pack_width(c)); }

template <class T, int TAPS, class F> void with_pack(const qds_conv_config* c, F&& f) {
  constexpr int V = kVec<T>;
  if (c->width < V) f(Int<1>{}, Int<TAPS>{}, std::false_type{});
  else if (c->width % V) f(Int<V>{}, Int<TAPS>{}, std::true_type{});
  else f(Int<V>{}, Int<TAPS>{}, std::false_type{});
}
template <class T, class F> void with_taps(const qds_conv_config* c, F&& f) {
  switch (c->taps) {
    case 1: return with_pack<T, 1>(c, f);
    case 2: return with_pack<T, 2>(c, f);
    case 3: return with_pack<T, 3>(c, f);
    case 4: return with_pack<T, 4>(c, f);
    case 5: return with_pack<T, 5>(c, f);
    case 6: return with_pack<T, 6>(c, f);
    case 7: return with_pack<T, 7>(c, f);
    default: return with_pack<T, 8>(c, f);
  }
}
template <class F> void with_type(const qds_conv_config* c, F&& f) {
  if (c->dtype == QDS_F32) f(float());
  else if (c->dtype == QDS_BF16) f(bf16());
  else f(half());
}

// Rows per chunk, 8 to 64: as many as leave some 2^18 columns' chunks (a chunk reads taps - 1 rows
// twice, and its loads wait for each other).
int chunk_rows(const qds_conv_config* c) {
  const int64_t cells = (int64_t)c->batch * c->length * c->width;
  int rows = 64;
  while (rows > 8 && cells / rows < (1 << 18)) rows /= 2;
  return rows;
}
// Chunks there are; one for the state of an episode without rows.
int64_t chunk_count(const qds_conv_config* c) { return std::max<int64_t>(1, ceil_div(c->length, chunk_rows(c))); }
// Places of threads are numbered with 32 bits.
bool numbered(const qds_conv_config* c) { return (int64_t)c->batch * chunk_count(c) <= (int64_t)0x7fffffff / packs_of(c); }
// Packs side by side in a workgroup of the backward pass, and workgroups over the chunks.
int lane_count(const qds_conv_config* c) {
  int lanes = 1;
  while (lanes < 64 && lanes < packs_of(c)) lanes *= 2;
  return lanes;
}
int share_count(const qds_conv_config* c) {
  const int64_t items = (int64_t)c->batch * chunk_count(c), lanes = lane_count(c);
  const int64_t most = std::max<int64_t>(1, kShares / ceil_div(packs_of(c), lanes));
  return (int)std::min(most, std::max<int64_t>(1, ceil_div(items, kBlock / lanes)));
}

ConvArgs args_of(const qds_conv_config* c) {
  ConvArgs a{};
  a.batch = c->batch;
  a.length = c->length;
  a.width = c->width;
  a.packs = packs_of(c);
  a.lanes = lane_count(c);
  a.w32 = c->weight_dtype == QDS_F32;
  a.silu = c->silu != 0;
  return a;
}

}  // namespace
}  // namespace seq

using namespace seq;

extern "C" qds_status qds_causal_conv(const qds_conv_config* c, qds_rows x, const void* weight, const void* bias,
                                      const void* state_in, const int32_t* lengths, qds_rows y, void* state_out,
                                      void* stream) {
  const qds_status st = validate(c, false);
  if (st != QDS_OK) return st;
  if (!numbered(c)) return QDS_ERR_UNSUPPORTED;
  if (c->batch == 0) return QDS_OK;
  if (!weight || (c->length > 0 && (!x.data || !y.data))) return QDS_ERR_INVALID_ARG;
  if ((state_out && state_out == state_in) || (c->length > 0 && x.data == y.data)) return QDS_ERR_INVALID_ARG;
  ConvArgs a = args_of(c);
  a.x = rows(x);
  a.y = rows(y);
  a.w = weight;
  a.bias = bias;
  a.first = state_in;
  a.last = c->taps > 1 ? state_out : nullptr;
  a.lengths = lengths;
  a.chunk = chunk_rows(c);
  a.chunks = (int)chunk_count(c);
  const int64_t blocks = ceil_div((int64_t)c->batch * a.chunks * a.packs, kBlock);
  hipStream_t s = (hipStream_t)stream;
  with_type(c, [&](auto type) {
    with_taps<decltype(type)>(c, [&](auto V, auto K, auto TAIL) {
      k_conv<decltype(type), decltype(V)::value, decltype(K)::value, decltype(TAIL)::value><<<(uint32_t)blocks, kBlock, 0, s>>>(a);
    });
  });
  return launch_status();
}

extern "C" qds_status qds_causal_conv_backward_workspace(const qds_conv_config* c, uint64_t* bytes) {
  const qds_status st = validate(c, false);
  if (st != QDS_OK) return st;
  if (!bytes) return QDS_ERR_INVALID_ARG;
  if (!numbered(c)) return QDS_ERR_UNSUPPORTED;
  *bytes = align_up((uint64_t)share_count(c) * (c->taps + 1) * c->width * sizeof(float));
  return QDS_OK;
}

extern "C" qds_status qds_causal_conv_backward(const qds_conv_config* c, qds_rows dy, qds_rows x, const void* weight,
                                               const void* bias, const void* state_in, const void* dstate_out,
                                               const int32_t* lengths, qds_rows dx, void* dweight, void* dbias,
                                               void* dstate_in, void* workspace, uint64_t workspace_bytes,
                                               void* stream) {
  uint64_t need = 0;
  const qds_status st = qds_causal_conv_backward_workspace(c, &need);
  if (st != QDS_OK) return st;
  if (!weight || !dweight || !workspace || ((uintptr_t)workspace & 255)) return QDS_ERR_INVALID_ARG;
  if (c->batch > 0 && c->length > 0 && (!dy.data || !x.data || !dx.data)) return QDS_ERR_INVALID_ARG;
  if (dstate_in && dstate_in == dstate_out) return QDS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return QDS_ERR_WORKSPACE_TOO_SMALL;
  // a chunk reads rows of the next one
  if (dx.data && (dx.data == dy.data || dx.data == x.data)) return QDS_ERR_INVALID_ARG;
  ConvArgs a = args_of(c);
  a.x = rows(x);
  a.dy = rows(dy);
  a.dx = rows(dx);
  a.w = weight;
  a.bias = bias;
  a.first = state_in;
  a.dlast = c->taps > 1 ? dstate_out : nullptr;
  a.dfirst = c->taps > 1 ? dstate_in : nullptr;
  a.lengths = lengths;
  a.dw = dweight;
  a.dbias = dbias;
  a.partial = (float*)workspace;
  a.chunk = chunk_rows(c);
  a.chunks = (int)chunk_count(c);
  a.shares = share_count(c);
  hipStream_t s = (hipStream_t)stream;
  const dim3 grid((uint32_t)ceil_div(a.packs, a.lanes), (uint32_t)a.shares);
  const dim3 join((uint32_t)ceil_div(a.width, 64), (uint32_t)(c->taps + 1));
  with_type(c, [&](auto type) {
    using T = decltype(type);
    with_taps<T>(c, [&](auto V, auto K, auto TAIL) {
      constexpr int v = decltype(V)::value, taps = decltype(K)::value;
      constexpr bool tail = decltype(TAIL)::value;
      if (c->silu) k_conv_backward<T, v, taps, tail, true><<<grid, kBlock, 0, s>>>(a);
      else k_conv_backward<T, v, taps, tail, false><<<grid, kBlock, 0, s>>>(a);
    });
    k_conv_dweight<T><<<join, 64 * kJoinWaves, 0, s>>>(a, c->taps);
  });
  return launch_status();
}

extern "C" qds_status qds_causal_conv_step(const qds_conv_config* c, qds_rows x, const void* weight, const void* bias,
                                           const void* state_in, qds_rows y, void* state_out, void* stream) {
  const qds_status st = validate(c, true);
  if (st != QDS_OK) return st;
  if (c->batch == 0) return QDS_OK;
  if (!weight || !x.data || !y.data || (c->taps > 1 && (!state_in || !state_out))) return QDS_ERR_INVALID_ARG;
  ConvArgs a = args_of(c);
  a.x = rows(x);
  a.y = rows(y);
  a.w = weight;
  a.bias = bias;
  a.first = state_in;
  a.last = state_out;
  if (c->batch > 0x7fffffff / a.packs) return QDS_ERR_UNSUPPORTED;
  const int64_t blocks = ceil_div((int64_t)c->batch * a.packs, kBlock);
  hipStream_t s = (hipStream_t)stream;
  with_type(c, [&](auto type) {
    with_taps<decltype(type)>(c, [&](auto V, auto K, auto TAIL) {
      k_conv_step<decltype(type), decltype(V)::value, decltype(K)::value, decltype(TAIL)::value><<<(uint32_t)blocks, kBlock, 0, s>>>(a);
    });
  });
  return launch_status();
}
