// seq_window.hip -- attention over a sliding window whose first tokens stay
// visible: forward, backward, the single-token step over a ring cache, and the
// cache's filling from a prompt.  The C ABI is in include/qd_seq.h.
//
// Row i of an episode of n rows sees j <= i < n with i - j < window or j < sinks.
// Scores are kept in units of log 2: p = 2^(c s - m) with c = scale log2(e).
#include <algorithm>

#include "seq_common.hpp"

namespace seq {
namespace {

constexpr int kBlock = 256;
constexpr int kWaves = 4;
constexpr float kNoMax = -3.0e38f;     // below every score; finite, so that differences are no not-a-number
struct WindowArgs {
  View q, k, v, o, dout, dq, dk, dv;
  const int32_t* lengths;
  float *lse, *delta;
  int32_t batch, length, heads, kv_heads, dim, window, sinks;
  float scale;
  bool spread;                        // see spread()
  int32_t share;                      // log2 of the query heads of a group that a workgroup has; see shared_heads()
};

// The item of this workgroup where each list (one batch element's key head) has per_list.
__device__ inline int item_of(const WindowArgs& a, int per_list) {
  return item_order(a.spread, blockIdx.x, gridDim.x, per_list);
}

__device__ inline int rows_of(const WindowArgs& a, int b) {
  if (!a.lengths) return a.length;
  return min(max(a.lengths[b], 0), a.length);
}

// Tiles in LDS have rows of 64 or 128 columns; products are formed of the first DC of
// them: 32, 64, 96 or 128, the least that holds the head.
constexpr int padded(int columns) { return columns <= 64 ? 64 : 128; }

// One row per lane l % 32 as an operand of the 32x32x16 product (k along the row).
template <class T, int DC> __device__ inline void load_rows(x8<T>* f, const T* row, bool valid, int dim) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int s = 0; s < DC / 16; ++s) {
    const int c = s * 2 + half;
    f[s] = zero8<T>();
    if (valid && c * 8 < dim) f[s] = __builtin_bit_cast(x8<T>, *reinterpret_cast<const u32x4*>(row + c * 8));
  }
}
// The tiles of 64 keys that rows i0 .. i0 + rows - 1 can see: those of the first
// tokens that are not in the band, then the band's.
struct KeyTiles {
  int first, band, count;   // tiles of first tokens; first tile of the band; all
  __device__ KeyTiles(const WindowArgs& a, int i0, int rows, int n) {
    const int lo = max(0, i0 - a.window + 1) / 64, hi = min(i0 + rows, n) - 1;
    band = lo;
    first = min((a.sinks + 63) / 64, lo);
    count = first + hi / 64 - lo + 1;
  }
  __device__ int row(int t) const { return (t < first ? t : band + t - first) * 64; }
};

// How far back key j is seen.  Row i sees it where i - j, taken as unsigned, is below
// this: one comparison, without the branches that && and || would make of every element.
__device__ inline uint32_t reach_of(int window, int sinks, int j) { return j < sinks ? 0x40000000u : (uint32_t)window; }

// Hides what row i does not see of a tile of scores (keys j0 .. j0 + 31 as its rows).
// Most masked tiles need one side of the band only: two or three instructions an
// element, where both at once take five.
__device__ inline void hide(f32x16& s, int i, int j0, int window, int sinks, bool later, bool earlier) {
  const int half = 4 * ((threadIdx.x & 63) >> 5);
  if (later) {               // j <= i
    const int last = i - j0 - half;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = (r & 3) + 8 * (r >> 2) <= last ? s[r] : -INFINITY;
  }
  if (earlier) {             // hidden: sinks <= j <= i - window
    const int from = sinks - j0 - half;
    const uint32_t count = (uint32_t)max(i - window - sinks + 1, 0);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = (uint32_t)((r & 3) + 8 * (r >> 2) - from) >= count ? s[r] : -INFINITY;
  }
}

// ---------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------
// A workgroup has 128 query rows (of one head, or 64 or 32 rows of heads of a group), a
// wave 32 of them.  Scores are formed transposed (keys are rows of the C tile, queries
// its columns), so a query's maximum and sum are over a lane's own registers and one exchange with
// lane l ^ 32, and the weights are the B operand of o^T = v^T p^T as they are.
// Bound by the issue of matrix and vector instructions together: 32768 rows, 16 heads
// of 128 over 4 key heads, window 4096, bfloat16 take 1.09 to 1.19 ms between cards, 890 to 970 TFLOP/s (after an
// idle stretch the first launches take up to 1.48 and the twelfth 1.18: 1.23 to 1.28 in the middle).  The next
// tile's scores beside this tile's weights do not fit the registers of two waves on a
// SIMD (292 spills), and with one wave took 2.11 ms beside 1.07.
constexpr int kForwardRows = 32 * kWaves;

template <class T, int DC>
__global__ __launch_bounds__(kBlock, 2) void k_window_forward(WindowArgs a, int q_blocks) {
  constexpr int DP = padded(DC);
  SEQ_SHARED T sk[2][64 * DP], sv[2][64 * DP];
  const int lane = threadIdx.x & 63, wave = wave_index();
  Lanes<DP> place;
  const int group = a.heads / a.kv_heads;
  const int per_block = group >> a.share;
  int id = item_of(a, per_block * q_blocks);
  const int g = ((id % per_block) << a.share) + (wave & ((1 << a.share) - 1));
  id /= per_block;
  // late blocks first: they have the most keys where the window is long
  const int block = q_blocks - 1 - id % q_blocks;
  id /= q_blocks;
  const int hk = id % a.kv_heads, b = id / a.kv_heads;
  const int h = hk * group + g;
  const int n = rows_of(a, b), window = a.window, sinks = a.sinks;
  const int rows = kForwardRows >> a.share, i0 = block * rows, w0 = i0 + 32 * (wave >> a.share);
  const int i = w0 + (lane & 31);
  T* o_row = at<T>(a.o, b, i, h);
  float* lse = a.lse + ((int64_t)b * a.heads + h) * a.length + i;

  f32x16 o[DC / 32];
#pragma unroll
  for (int d = 0; d < DC / 32; ++d) o[d] = f32x16{};
  if (i0 < n) {
    const float c = a.scale * kLog2e;
    x8<T> q[DC / 16];
    load_rows<T, DC>(q, at<T>(a.q, b, i, h), i < n, a.dim);
    const KeyTiles tiles(a, i0, rows, n);
    Staged<T, DP, kBlock> rk, rv;
    rk.init(at<T>(a.k, b, 0, hk), a.k.t, a.dim);
    rv.init(at<T>(a.v, b, 0, hk), a.v.t, a.dim);
    rk.load(tiles.row(0), n);
    rv.load(tiles.row(0), n);
    rk.store(sk[0]);
    rv.store(sv[0]);
    float m = kNoMax, sum = 0.0f;
    for (int t = 0; t < tiles.count; ++t) {
      __syncthreads();
      const int j0 = tiles.row(t);
      const bool more = t + 1 < tiles.count;
      if (more) {
        rk.load(tiles.row(t + 1), n);
        rv.load(tiles.row(t + 1), n);
      }
      const T *tk = sk[t & 1], *tv = sv[t & 1];
      if (DP == 128) place.forget();
      // Keys in steps of 32 for narrow heads, whose products are short against their
      // weights: a step that no row of the wave sees is skipped (the half of a tile behind
      // the diagonal, before the band, or behind the first tokens).  Wide heads take 64.
      constexpr int STEP = DP == 64 ? 1 : 2;
#pragma unroll
      for (int first = 0; first < 2; first += STEP) {
        const int from = j0 + 32 * first, to = from + 32 * STEP - 1;
        if (from > w0 + 31 || (w0 - to >= window && from >= sinks)) continue;
        f32x16 s[STEP];
#pragma unroll
        for (int x = 0; x < STEP; ++x) {
          s[x] = f32x16{};
#pragma unroll
          for (int ks = 0; ks < DC / 16; ++ks)
            s[x] = mfma32(tile_rows<T, DP>(tk, place, (first + x) * 32, ks), q[ks], s[x]);
        }
        if (STEP == 2) reads_ahead<DC / 8, 1, 4>();
        const bool later = to > w0, earlier = w0 + 31 - from >= window && to >= sinks;
#pragma unroll
        for (int x = 0; x < STEP; ++x) hide(s[x], i, from + x * 32, window, sinks, later, earlier);
        float top = kNoMax;
#pragma unroll
        for (int x = 0; x < STEP; ++x)
#pragma unroll
          for (int r = 0; r < 16; ++r) top = fmaxf(top, s[x][r]);
        top = max_halves(top) * c;
        // The maximum is moved only where a weight would pass 2^8: any reference
        // gives the same quotient, and most tiles then need no rescaling.
        if (__any(top > m + 8.0f)) {
          const float to_m = fmaxf(m, top), alpha = fast_exp2(m - to_m);
          m = to_m;
          sum *= alpha;
#pragma unroll
          for (int d = 0; d < DC / 32; ++d) o[d] *= alpha;
        }
#pragma unroll
        for (int x = 0; x < STEP; ++x) {
          float p[16];
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            p[r] = fast_exp2(fmaf(s[x][r], c, -m));
            sum += p[r];
          }
          // The weights are rounded to the tensors' type for the matrix product
          // (their sum is not): 2^-9 or 2^-12 of each, less than o's own rounding.
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const x8<T> pb = pack8<T>(p + 8 * u);
#pragma unroll
            for (int d = 0; d < DC / 32; ++d)
              o[d] = mfma32(tile_columns<T, DP>(tv, place, (first + x) * 32 + 16 * u, d), pb, o[d]);
          }
        }
      }
      if (more) {
        rk.store(sk[(t + 1) & 1]);
        rv.store(sv[(t + 1) & 1]);
      }
    }
    sum = sum_halves(sum);
    if (i < n) {
      const float inv = 1.0f / sum;
#pragma unroll
      for (int d = 0; d < DC / 32; ++d) store_column<T>(o_row, d, o[d], inv, a.dim);
      if (lane < 32) *lse = (m + fast_log2(sum)) * kLn2;
    }
  }
  if (i >= n && i < a.length) {
#pragma unroll
    for (int d = 0; d < DC / 32; ++d) store_column<T>(o_row, d, f32x16{}, 0.0f, a.dim);
    if (lane < 32) *lse = -INFINITY;
  }
}

// ---------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------
// With p = 2^(c s - lse), delta_i = do_i . o_i, ds = p (do v^T - delta):
//   dq = scale ds k,  dk = scale ds^T q,  dv = p^T do.
// Two kernels, one over queries and one over keys, each forming p again; sums
// are then over a workgroup's own loop, in a fixed order.

// dq of the same rows as the forward pass has; also writes delta.  2 x 8192 rows,
// 16 heads of 128, window 1024, bfloat16: 251 to 264 us between cards (the forward pass takes 190 to 199).
//
// delta is formed from o as stored, so it carries o's rounding; the score gradients
// are rounded to the tensors' type for their product, relative to each of them.  In
// float16 those below 2^-24 vanish and those beyond 65504 are infinite: a loss is scaled there
// as for any float16 gradient.
template <class T, int DC>
__global__ __launch_bounds__(kBlock, 2) void k_window_dq(WindowArgs a, int q_blocks) {
  constexpr int DP = padded(DC);
  SEQ_SHARED T sk[2][64 * DP], sv[2][64 * DP];
  const int lane = threadIdx.x & 63, wave = wave_index();
  Lanes<DP> place;
  const int group = a.heads / a.kv_heads;
  const int per_block = group >> a.share;
  int id = item_of(a, per_block * q_blocks);
  const int g = ((id % per_block) << a.share) + (wave & ((1 << a.share) - 1));
  id /= per_block;
  const int block = q_blocks - 1 - id % q_blocks;
  id /= q_blocks;
  const int hk = id % a.kv_heads, b = id / a.kv_heads;
  const int h = hk * group + g;
  const int n = rows_of(a, b), window = a.window, sinks = a.sinks;
  const int rows = kForwardRows >> a.share, i0 = block * rows, w0 = i0 + 32 * (wave >> a.share);
  const int i = w0 + (lane & 31);
  const int64_t flat = ((int64_t)b * a.heads + h) * a.length + i;

  f32x16 dq[DC / 32];
#pragma unroll
  for (int d = 0; d < DC / 32; ++d) dq[d] = f32x16{};
  if (i0 < n) {
    const float c = a.scale * kLog2e;
    x8<T> q[DC / 16], go[DC / 16];
    load_rows<T, DC>(q, at<T>(a.q, b, i, h), i < n, a.dim);
    load_rows<T, DC>(go, at<T>(a.dout, b, i, h), i < n, a.dim);
    float delta = 0.0f;
    {
      x8<T> o[DC / 16];
      load_rows<T, DC>(o, at<T>(a.o, b, i, h), i < n, a.dim);
#pragma unroll
      for (int s = 0; s < DC / 16; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) delta = fmaf((float)o[s][e], (float)go[s][e], delta);
    }
    delta = sum_halves(delta);
    if (lane < 32 && i < n) a.delta[flat] = delta;
    const float lse = i < n ? a.lse[flat] * kLog2e : INFINITY;   // rows past the end: p = 0
    const KeyTiles tiles(a, i0, rows, n);
    Staged<T, DP, kBlock> rk, rv;
    rk.init(at<T>(a.k, b, 0, hk), a.k.t, a.dim);
    rv.init(at<T>(a.v, b, 0, hk), a.v.t, a.dim);
    rk.load(tiles.row(0), n);
    rv.load(tiles.row(0), n);
    rk.store(sk[0]);
    rv.store(sv[0]);
    for (int t = 0; t < tiles.count; ++t) {
      __syncthreads();
      const int j0 = tiles.row(t);
      const bool more = t + 1 < tiles.count;
      if (more) {
        rk.load(tiles.row(t + 1), n);
        rv.load(tiles.row(t + 1), n);
      }
      const T *tk = sk[t & 1], *tv = sv[t & 1];
      if (DP == 128) place.forget();
      {
#pragma unroll
        for (int jb = 0; jb < 2; ++jb) {
          const int from = j0 + 32 * jb;
          if (from > w0 + 31 || (w0 - (from + 31) >= window && from >= sinks)) continue;
          const bool later = from + 31 > w0, earlier = w0 + 31 - from >= window && from + 31 >= sinks;
          __builtin_amdgcn_sched_barrier(0);       // one half's products at a time: both would not fit the registers
          f32x16 s = f32x16{}, dp = f32x16{};
#pragma unroll
          for (int ks = 0; ks < DC / 16; ++ks) s = mfma32(tile_rows<T, DP>(tk, place, jb * 32, ks), q[ks], s);
#pragma unroll
          for (int ks = 0; ks < DC / 16; ++ks) dp = mfma32(tile_rows<T, DP>(tv, place, jb * 32, ks), go[ks], dp);
          hide(s, i, j0 + jb * 32, window, sinks, later, earlier);
          float ds[16];
#pragma unroll
          for (int r = 0; r < 16; ++r) ds[r] = fast_exp2(fmaf(s[r], c, -lse)) * (dp[r] - delta);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const x8<T> db = pack8<T>(ds + 8 * u);
#pragma unroll
            for (int d = 0; d < DC / 32; ++d)
              dq[d] = mfma32(tile_columns<T, DP>(tk, place, jb * 32 + 16 * u, d), db, dq[d]);
          }
        }
      }
      if (more) {
        rk.store(sk[(t + 1) & 1]);
        rv.store(sv[(t + 1) & 1]);
      }
    }
  }
  if (i < a.length) {
    T* row = at<T>(a.dq, b, i, h);
#pragma unroll
    for (int d = 0; d < DC / 32; ++d) store_column<T>(row, d, dq[d], i < n ? a.scale : 0.0f, a.dim);
  }
}

// A wave has 32 keys, a unit is 32 query rows of one head.  Scores have queries as
// rows and keys as columns of the C tile, so that both the weights and the score
// gradients are operands of the sums over queries as they are.  Keys stay in
// registers; values do for 64 columns, and are read from LDS for 128, where the
// registers that two waves on a SIMD leave each other are 160 for keys and sums.
// Two waves with values in LDS take 400 us where one with all in registers takes 490
// (2 x 8192 rows, 16 heads of 128, window 1024, bfloat16; 386 to 404 now, between cards).  For heads of up to 64
// no other unit has been timed: 32 ragged episodes of 1000 rows, 8 heads of 64 over 2, window 250, float16 take 64 us, of
// which waves wait 45% and the matrix units work 15%.  The weights and the score gradients are rounded as in the other two
// kernels.
template <class T, int DC>
__global__ __launch_bounds__(kBlock, 2) void k_window_dkdv(WindowArgs a, KeyPlan plan, float* parts) {
  constexpr int DP = padded(DC);
  constexpr int QT = kUnitRows;
  constexpr bool V_LDS = DP == 128;
  SEQ_SHARED T sq[2][QT * DP], sg[2][QT * DP], sv[V_LDS ? kKeyRows * DP : 8];
  SEQ_SHARED float s_lse[2][QT], s_delta[2][QT];
  const int lane = threadIdx.x & 63, wave = wave_index();
  Lanes<DP> place;
  const int group = a.heads / a.kv_heads;
  const KeyWork work = key_work(plan, a.spread, blockIdx.x, gridDim.x);
  const int head = work.list;                 // b * kv_heads + hk
  const KeyItem item = key_item(plan, work.x);
  const int hk = head % a.kv_heads, b = head / a.kv_heads;
  const int n = rows_of(a, b), window = a.window, sinks = a.sinks;
  const int j0 = item.block * kKeyRows, w0 = j0 + 32 * wave;
  const int j = w0 + (lane & 31);
  const float c = a.scale * kLog2e;
  const uint32_t reach = reach_of(window, sinks, j);

  f32x16 dk[DC / 32], dv[DC / 32];
#pragma unroll
  for (int d = 0; d < DC / 32; ++d) dk[d] = dv[d] = f32x16{};
  const KeyUnits units = key_units(item, window, sinks, n, group);
  const int per_head = units.per_head, stop = units.end;
  int unit = units.begin;
  if (unit < stop) {
    x8<T> k[DC / 16], v[V_LDS ? 1 : DC / 16];
    load_rows<T, DC>(k, at<T>(a.k, b, j, hk), j < n, a.dim);
    if constexpr (V_LDS) {
      Staged<T, DP, kBlock> rv;
      rv.init(at<T>(a.v, b, 0, hk), a.v.t, a.dim);
#pragma unroll
      for (int half = 0; half < kKeyRows / 64; ++half) {
        rv.load(j0 + half * 64, n);
        rv.store(sv + half * 64 * DP);
      }
    } else {
      load_rows<T, DC>(v, at<T>(a.v, b, j, hk), j < n, a.dim);
    }
    Staged<T, DP, kBlock, QT> rq, rg;
    rq.init(nullptr, a.q.t, a.dim);
    rg.init(nullptr, a.dout.t, a.dim);
    float r_lse = 0.0f, r_delta = 0.0f;
    int u_head = unit / per_head, u_row = unit % per_head;        // of the unit that is fetched next
    int row_fetched = 0;
    auto fetch = [&] {
      const int h = hk * group + u_head;
      row_fetched = j0 + u_row * QT;
      rq.base = at<T>(a.q, b, 0, h);
      rg.base = at<T>(a.dout, b, 0, h);
      rq.load(row_fetched, n);
      rg.load(row_fetched, n);
      if (wave == 0) {
        const int64_t flat = ((int64_t)b * a.heads + h) * a.length + min(row_fetched + (lane & 31), n - 1);
        r_lse = a.lse[flat];
        r_delta = a.delta[flat];
      }
      if (++u_row == per_head) u_row = 0, ++u_head;
    };
    auto put = [&](int buf) {
      rq.store(sq[buf]);
      rg.store(sg[buf]);
      if (threadIdx.x < QT) {
        // rows past the end: p = 0
        s_lse[buf][threadIdx.x] = row_fetched + (int)threadIdx.x < n ? r_lse * kLog2e : INFINITY;
        s_delta[buf][threadIdx.x] = r_delta;
      }
    };
    fetch();
    put(0);
    for (int buf = 0; unit < stop; ++unit, buf ^= 1) {
      __syncthreads();
      const int r0 = row_fetched;
      if (unit + 1 < stop) fetch();
      const bool none = r0 + 31 < w0 || (r0 - (w0 + 31) >= window && w0 >= sinks);
      const bool all = r0 >= w0 + 31 && (r0 + 31 - w0 < window || w0 + 31 < sinks);
      const T *tq = sq[buf], *tg = sg[buf];
      if (DP == 128) place.forget();
      if (!none) {
        f32x16 s = f32x16{}, dp = f32x16{};
#pragma unroll
        for (int ks = 0; ks < DC / 16; ++ks) s = mfma32(tile_rows<T, DP>(tq, place, 0, ks), k[ks], s);
#pragma unroll
        for (int ks = 0; ks < DC / 16; ++ks) {
          const x8<T> vf = V_LDS ? tile_rows<T, DP>(sv + 32 * DP * wave, place, 0, ks) : v[V_LDS ? 0 : ks];
          dp = mfma32(tile_rows<T, DP>(tg, place, 0, ks), vf, dp);
        }
        reads_ahead<DC / 16, 1, 4>();
        if (!all) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = (uint32_t)(r0 + c_row(r) - j) < reach ? s[r] : -INFINITY;
        }
        float p[16], ds[16];
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          const int at4 = 8 * r4 + 4 * (lane >> 5);
          const f32x4 lse = *reinterpret_cast<const f32x4*>(&s_lse[buf][at4]);
          const f32x4 delta = *reinterpret_cast<const f32x4*>(&s_delta[buf][at4]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 4 * r4 + e;
            p[r] = fast_exp2(fmaf(s[r], c, -lse[e]));
            ds[r] = p[r] * (dp[r] - delta[e]);
          }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const x8<T> pb = pack8<T>(p + 8 * u), db = pack8<T>(ds + 8 * u);
#pragma unroll
          for (int d = 0; d < DC / 32; ++d) {
            dv[d] = mfma32(tile_columns<T, DP>(tg, place, 16 * u, d), pb, dv[d]);
            dk[d] = mfma32(tile_columns<T, DP>(tq, place, 16 * u, d), db, dk[d]);
          }
        }
      }
      if (unit + 1 < stop) put(buf ^ 1);
    }
  }
  if (item.cut == 1) {
    if (j < a.length) {
      T* rk = at<T>(a.dk, b, j, hk);
      T* rv = at<T>(a.dv, b, j, hk);
#pragma unroll
      for (int d = 0; d < DC / 32; ++d) {
        store_column<T>(rk, d, dk[d], a.scale, a.dim);
        store_column<T>(rv, d, dv[d], 1.0f, a.dim);
      }
    }
  } else {
    // [list][sum][dk, dv][row][DP]
    float* to = parts + ((int64_t)head * plan.sums + item.sum) * (2 * kKeyRows * DP) + (wave * 32 + (lane & 31)) * DP;
#pragma unroll
    for (int d = 0; d < DC / 32; ++d)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int col = d * 32 + 8 * r4 + 4 * (lane >> 5);
        *reinterpret_cast<f32x4*>(to + col) =
            f32x4{dk[d][4 * r4], dk[d][4 * r4 + 1], dk[d][4 * r4 + 2], dk[d][4 * r4 + 3]};
        *reinterpret_cast<f32x4*>(to + kKeyRows * DP + col) =
            f32x4{dv[d][4 * r4], dv[d][4 * r4 + 1], dv[d][4 * r4 + 2], dv[d][4 * r4 + 3]};
      }
  }
}

// Adds the pieces of cut blocks: a thread has four columns of a row of dk and of dv.
// 7.3 us for 2 x 16 heads of 128 with 16 first tokens each.
template <class T, int DP>
__global__ __launch_bounds__(kBlock) void k_window_dkdv_join(WindowArgs a, KeyPlan plan, int per_head, const float* parts) {
  constexpr int ROWS = kBlock * 4 / DP;
  const int head = blockIdx.x / per_head, x = blockIdx.x % per_head;
  const int hk = head % a.kv_heads, b = head / a.kv_heads;
  const int block = cut_from(plan) + x / (kKeyRows / ROWS);
  const int row = (x % (kKeyRows / ROWS)) * ROWS + threadIdx.x / (DP / 4);
  const int col = threadIdx.x % (DP / 4) * 4;
  const int j = block * kKeyRows + row;
  if (j >= a.length || col >= a.dim) return;
  const int cut = block < plan.first ? plan.first_cut : plan.band_cut;
  const float* p = parts + ((int64_t)head * plan.sums + key_sums(plan, block)) * (2 * kKeyRows * DP) + row * DP + col;
  f32x4 dk = f32x4{}, dv = f32x4{};
#pragma unroll 4
  for (int s = 0; s < cut; ++s) {
    dk += *reinterpret_cast<const f32x4*>(p);
    dv += *reinterpret_cast<const f32x4*>(p + kKeyRows * DP);
    p += 2 * kKeyRows * DP;
  }
  dk *= a.scale;
  *reinterpret_cast<u32x2*>(at<T>(a.dk, b, j, hk) + col) = __builtin_bit_cast(u32x2, pack4<T>(dk[0], dk[1], dk[2], dk[3]));
  *reinterpret_cast<u32x2*>(at<T>(a.dv, b, j, hk) + col) = __builtin_bit_cast(u32x2, pack4<T>(dv[0], dv[1], dv[2], dv[3]));
}

// ---------------------------------------------------------------------------
// Single-token step
// ---------------------------------------------------------------------------
// Bound by reading the cache once.  Up to 16 query heads that share a key head
// are the columns of one matrix product, so that its keys and values are read
// once for all of them.  A workgroup has a range of slots, its waves take strips
// of 32 slots in turn and keep running maxima and sums of their own; ranges and
// waves are joined at the end.  Keys and values are loaded as whole rows and go
// through LDS (8 KB a wave for 64 columns, 16 KB for 128), which turns them.
// 8 policies of 4 key heads of 128 over 65552 slots, float16: 164 us, 5.5 TB/s; 256
// policies of 8 heads of 64 over 251 slots: 19.6 us.
constexpr int kStrip = 32;

struct StepArgs {
  View q, k, v, o;
  void *k_cache, *v_cache;
  const int32_t* pos;
  float* parts;            // [item][16]: maxima, then sums, then o [item][16][DP]
  int32_t batch, heads, kv_heads, dim, window, sinks, tiles, cut, range;
  float scale;
};

__device__ inline int slot_of(int p, int window, int sinks) { return p < sinks ? p : sinks + (p - sinks) % window; }

template <class T, int DP>
__global__ __launch_bounds__(kBlock, 2) void k_window_step(StepArgs a) {
  constexpr int OUT = DP + 4;                       // padded, so that 16 heads spread over the banks
  constexpr int kStage = 2 * kWaves * kStrip * DP * 2, kOut = kWaves * 16 * OUT * 4;
  SEQ_SHARED char lds[kStage > kOut ? kStage : kOut];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int group = a.heads / a.kv_heads, slots = a.window + a.sinks;
  // One list further from range to range: the ranges of a long cache go round the XCDs,
  // whose shares of the memory's bandwidth would else differ as the positions do (2
  // policies of 4 key heads of 128, 65536 slots: 48 us on the lists' own XCDs, 34 so).
  const int unit = (int)((blockIdx.x + blockIdx.y) % gridDim.x), tile = unit % a.tiles, head = unit / a.tiles;
  const int hk = head % a.kv_heads, b = head / a.kv_heads;
  const int pos = a.pos[b];
  const int seen = pos < 0 ? 0 : min(pos, slots - 1) + 1;
  const int fresh = pos < 0 ? -1 : slot_of(pos, a.window, a.sinks);
  const int begin = blockIdx.y * a.range, end = min(begin + a.range, seen);
  T* kc = (T*)a.k_cache + (int64_t)head * slots * a.dim;
  T* vc = (T*)a.v_cache + (int64_t)head * slots * a.dim;
  const T* k_new = at<T>(a.k, b, 0, hk);
  const T* v_new = at<T>(a.v, b, 0, hk);

  // The new row is read from k and v wherever it is needed, and written by one workgroup.
  if (tile == 0 && fresh >= begin && fresh < end && threadIdx.x < DP / 8 && threadIdx.x * 8 < a.dim) {
    const int c = threadIdx.x * 8;
    *reinterpret_cast<u32x4*>(kc + (int64_t)fresh * a.dim + c) = *reinterpret_cast<const u32x4*>(k_new + c);
    *reinterpret_cast<u32x4*>(vc + (int64_t)fresh * a.dim + c) = *reinterpret_cast<const u32x4*>(v_new + c);
  }

  const float c = a.scale * kLog2e;
  const int g = tile * 16 + (lane & 15), quad = lane >> 4;
  x8<T> q[DP / 32];
#pragma unroll
  for (int s = 0; s < DP / 32; ++s) {
    const int col = (s * 4 + quad) * 8;
    q[s] = zero8<T>();
    if (g < group && col < a.dim)
      q[s] = __builtin_bit_cast(x8<T>, *reinterpret_cast<const u32x4*>(at<T>(a.q, b, 0, hk * group + g) + col));
  }

  // Whole rows a load: a wave's lanes cover contiguous memory.
  constexpr int NV = kStrip * DP / 8 / 64;
  u32x4 rk[NV], rv[NV];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int id = lane + 64 * i, slot = s0 + id / (DP / 8), col = id % (DP / 8) * 8;
      const T* kr = slot == fresh ? k_new : kc + (int64_t)slot * a.dim;
      const T* vr = slot == fresh ? v_new : vc + (int64_t)slot * a.dim;
      rk[i] = rv[i] = u32x4{0, 0, 0, 0};
      if (slot < end && col < a.dim) {
        rk[i] = *reinterpret_cast<const u32x4*>(kr + col);
        rv[i] = *reinterpret_cast<const u32x4*>(vr + col);
      }
    }
  };

  f32x4 o[DP / 16];
#pragma unroll
  for (int d = 0; d < DP / 16; ++d) o[d] = f32x4{};
  float m = kNoMax, sum = 0.0f;
  T* stage = (T*)lds + wave * kStrip * DP;
  T* stage_k = (T*)lds + (kWaves + wave) * kStrip * DP;
  int s0 = begin + wave * kStrip;
  if (s0 < end) fetch(s0);
  for (; s0 < end; s0 += kWaves * kStrip) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int id = lane + 64 * i, place = tile_at<DP>(id / (DP / 8), id % (DP / 8));
      *reinterpret_cast<u32x4*>(stage_k + place) = rk[i];
      *reinterpret_cast<u32x4*>(stage + place) = rv[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // the wave's own writes to its stages
    __builtin_amdgcn_wave_barrier();
    if (s0 + kWaves * kStrip < end) fetch(s0 + kWaves * kStrip);
    f32x4 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = f32x4{};
#pragma unroll
      for (int ks = 0; ks < DP / 32; ++ks) {
        const x8<T> kf = __builtin_bit_cast(
            x8<T>, *reinterpret_cast<const u32x4*>(stage_k + tile_at<DP>(16 * t + (lane & 15), ks * 4 + quad)));
        s[t] = mfma16(kf, q[ks], s[t]);
      }
    }
    float top = kNoMax;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int slot = s0 + 16 * t + 4 * quad + r;
        s[t][r] = slot < end ? s[t][r] * c : -INFINITY;
        top = fmaxf(top, s[t][r]);
      }
    top = fmaxf(top, shfl_xor(top, 16));
    top = fmaxf(top, shfl_xor(top, 32));
    if (__any(top > m)) {
      const float to = fmaxf(m, top), alpha = fast_exp2(m - to);
      m = to;
      sum *= alpha;
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) o[d] *= alpha;
    }
    float p[8];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[4 * t + r] = fast_exp2(s[t][r] - m);
        sum += p[4 * t + r];
      }
    const x8<T> pb = pack8<T>(p);
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) {
      const int row = 4 * quad + ((lane & 15) >> 2), col = d * 16 + (lane & 3) * 4;
      const x4<T> lo = lds_read_transposed(stage + tile_at<DP>(row, col >> 3) + (col & 7));
      const x4<T> hi = lds_read_transposed(stage + tile_at<DP>(row + 16, col >> 3) + (col & 7));
      o[d] = mfma16(join8<T>(lo, hi), pb, o[d]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  sum += shfl_xor(sum, 16);
  sum += shfl_xor(sum, 32);

  // The waves' shares, added in their order.
  __syncthreads();
  float* out = (float*)lds;
  if (lane < 16) {
    s_m[wave][lane] = m;
    s_l[wave][lane] = sum;
  }
#pragma unroll
  for (int d = 0; d < DP / 16; ++d)
    *reinterpret_cast<f32x4*>(out + (wave * 16 + (lane & 15)) * OUT + d * 16 + 4 * quad) = o[d];
  __syncthreads();
  const int heads_here = min(16, group - tile * 16);
  const int64_t item = (int64_t)unit * a.cut + blockIdx.y, items = (int64_t)gridDim.x * a.cut;
  for (int x = threadIdx.x; x < heads_here * (DP / 4); x += kBlock) {
    const int hh = x / (DP / 4), d = x % (DP / 4) * 4;
    float top = s_m[0][hh];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][hh]);
    f32x4 r = f32x4{};
    float l = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = fast_exp2(s_m[w][hh] - top);
      l = fmaf(s_l[w][hh], f, l);
      r += *reinterpret_cast<const f32x4*>(out + (w * 16 + hh) * OUT + d) * f;
    }
    if (a.cut == 1) {
      const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);
      if (d < a.dim)
        *reinterpret_cast<u32x2*>(at<T>(a.o, b, 0, hk * group + tile * 16 + hh) + d) =
            __builtin_bit_cast(u32x2, pack4<T>(r[0] * inv, r[1] * inv, r[2] * inv, r[3] * inv));
    } else {
      if (d == 0) {
        a.parts[item * 16 + hh] = top;
        a.parts[(items + item) * 16 + hh] = l;
      }
      *reinterpret_cast<f32x4*>(a.parts + items * 32 + (item * 16 + hh) * DP + d) = r;
    }
  }
}

// Joins the ranges of one head: DP / 64 columns a lane, every eighth range a wave, as
// a range's sum waits for its loads.  One key head over 65536 slots, 128 ranges: a call takes
// 18 us, with one wave 27; 8 policies of 32 heads, 16 ranges: 4.8 us beside the step's 164.
constexpr int kStepJoinWaves = 8;
template <class T, int DP>
__global__ __launch_bounds__(64 * kStepJoinWaves) void k_window_step_join(StepArgs a) {
  __shared__ float s_top[kStepJoinWaves], s_l[kStepJoinWaves], s_r[kStepJoinWaves][DP];
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int b = blockIdx.x / a.heads, h = blockIdx.x % a.heads, group = a.heads / a.kv_heads;
  const int g = h % group;
  const int64_t first = (((int64_t)b * a.kv_heads + h / group) * a.tiles + g / 16) * a.cut;
  const int64_t items = (int64_t)a.batch * a.kv_heads * a.tiles * a.cut;
  float top = kNoMax;
  for (int s = threadIdx.x; s < a.cut; s += 64 * kStepJoinWaves) top = fmaxf(top, a.parts[(first + s) * 16 + g % 16]);
  top = wave_max(top);
  if (lane == 0) s_top[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kStepJoinWaves; ++w) top = fmaxf(top, s_top[w]);
  float l = 0.0f, r[DP / 64];
#pragma unroll
  for (int d = 0; d < DP / 64; ++d) r[d] = 0.0f;
#pragma unroll 4
  for (int s = wave; s < a.cut; s += kStepJoinWaves) {
    const int64_t at16 = (first + s) * 16 + g % 16;
    const float f = fast_exp2(a.parts[at16] - top);
    l = fmaf(a.parts[items * 16 + at16], f, l);
#pragma unroll
    for (int d = 0; d < DP / 64; ++d) r[d] = fmaf(a.parts[items * 32 + at16 * DP + d * 64 + lane], f, r[d]);
  }
  if (lane == 0) s_l[wave] = l;
#pragma unroll
  for (int d = 0; d < DP / 64; ++d) s_r[wave][d * 64 + lane] = r[d];
  __syncthreads();
  if (threadIdx.x >= a.dim) return;
  l = 0.0f;
  float sum = 0.0f;
#pragma unroll
  for (int w = 0; w < kStepJoinWaves; ++w) {
    l += s_l[w];
    sum += s_r[w][threadIdx.x];
  }
  const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);
  at<T>(a.o, b, 0, h)[threadIdx.x] = (T)(sum * inv);
}

// Slot by slot: the latest position below n that belongs in it.
template <class T>
__global__ __launch_bounds__(kBlock) void k_window_fill(WindowArgs a, T* k_cache, T* v_cache) {
  const int64_t slots = (int64_t)a.window + a.sinks, packs = a.dim / 8;
  const int64_t all = slots * packs * a.kv_heads * a.batch;
  for (int64_t x = (int64_t)blockIdx.x * kBlock + threadIdx.x; x < all; x += (int64_t)gridDim.x * kBlock) {
    const int col = (int)(x % packs) * 8;
    const int slot = (int)(x / packs % slots);
    const int64_t list = x / packs / slots;
    const int hk = (int)(list % a.kv_heads), b = (int)(list / a.kv_heads);
    const int last = rows_of(a, b) - 1;
    if (last < slot) continue;                 // nothing has come this far
    const int p = slot < a.sinks ? slot : last - (last - slot) % a.window;
    *reinterpret_cast<u32x4*>(k_cache + x * 8) = *reinterpret_cast<const u32x4*>(at<T>(a.k, b, p, hk) + col);
    *reinterpret_cast<u32x4*>(v_cache + x * 8) = *reinterpret_cast<const u32x4*>(at<T>(a.v, b, p, hk) + col);
  }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
qds_status validate(const qds_window_config* c) {
  if (!c || c->abi_version != QDS_ABI_VERSION) return QDS_ERR_INVALID_ARG;
  if (c->dtype != QDS_BF16 && c->dtype != QDS_F16)
    return c->dtype == QDS_F32 ? QDS_ERR_UNSUPPORTED : QDS_ERR_INVALID_ARG;
  if (c->batch < 0 || c->length < 0 || c->heads < 1 || c->kv_heads < 1 || c->heads % c->kv_heads)
    return QDS_ERR_INVALID_ARG;
  if (c->dim < 1) return QDS_ERR_INVALID_ARG;
  if (c->dim % 8 || c->dim > 128) return QDS_ERR_UNSUPPORTED;
  if (c->window < 1 || c->sinks < 0 || (int64_t)c->window + c->sinks >= (1 << 30) || c->length >= (1 << 30))
    return QDS_ERR_INVALID_ARG;
  if (!(c->scale > 0.0f) || c->scale > 3.0e38f) return QDS_ERR_INVALID_ARG;
  if ((int64_t)c->batch * c->heads > most_blocks(kBlock)) return QDS_ERR_UNSUPPORTED;      // the step's grid
  return QDS_OK;
}

// Whether a list's items go to all XCDs, in place of one.  One XCD reads a list's keys
// once into its own L2, but the XCDs then end apart where their work differs: lists with
// lengths, a number of them that does not divide evenly, or early rows that see less
// than a window in a large part of a list (of the stretch that an XCD has, for fewer
// than four lists; of half a list else, whose long blocks begin late in the last lists).
// Spread, the lists' keys and values share every L2: up to 64 MiB of them that costs less
// than it gains, and with two lists for each XCD or fewer it does at any size.
// Forward and backward, us, one XCD each | spread:
//   with lengths  64 lists x 1000 rows of 64, window 250       173 | 151
//                 8 x 16384 of 128, 1024                       790 | 577
//                 24 x 2048 of 64, 2048                        232 | 181
//                 96 x 4096 of 64, 1024 (96 MiB)               844 | 912
//                 64 x 8192 of 64, 512 (128 MiB)              1580 | 1754
//   without       128 x 1024 of 64, 1024                       176 | 139
//                 16 x 16384 of 64, 4096                      4750 | 5270
//                 4 x 65536 of 128, 2048                      1418 | 1503
bool spread(const qds_window_config* c, const int32_t* lengths) {
  const int64_t lists = (int64_t)c->batch * c->kv_heads;
  const bool deals_evenly = lists % kXcds == 0 || kXcds % lists == 0;
  const bool even = !lengths && deals_evenly && c->window < c->length * std::min<int64_t>(lists, 4) / 8;
  return !even && (lists <= 2 * kXcds || lists * c->length * c->dim * 4 <= 64 << 20);
}

// How many query heads of a group share a workgroup of the kernels over queries, whose four
// waves then have 32 or 64 rows of several heads in place of 128 of one: the same keys are
// loaded for as many products, but fewer tiles of them by rows that others cannot see.  Two
// or four where that divides the group.  Forward, us, one head | four: 4 x 3994 rows of 128,
// 32 heads over 4, window 113: 134 | 125;  15 x 1374 of 64, 64 over 8, window 37: 152 | 132;
// 13 x 776 of 80, 32 over 4, 104: 80 | 65;  long windows the same.
int shared_heads(const qds_window_config* c) {
  const int group = c->heads / c->kv_heads;
  return group % 4 == 0 ? 2 : group % 2 == 0 ? 1 : 0;
}

// Workgroups of the kernels over queries.
int64_t query_grid(const qds_window_config* c) {
  const int share = shared_heads(c);
  return (int64_t)c->batch * (c->heads >> share) * ceil_div(c->length, kForwardRows >> share);
}

WindowArgs window_args(const qds_window_config* c, const int32_t* lengths) {
  WindowArgs a{};
  a.lengths = lengths;
  a.batch = c->batch;
  a.length = c->length;
  a.heads = c->heads;
  a.kv_heads = c->kv_heads;
  a.dim = c->dim;
  a.window = c->window;
  a.sinks = c->sinks;
  a.scale = c->scale;
  a.spread = spread(c, lengths);
  a.share = shared_heads(c);
  return a;
}

// Calls f with the tensors' type and the columns of the head that products are formed of.
// Forward and backward, us, with products of all 64 or 128 columns | so: 10514 rows, 32 heads
// of 80 over 8, window 3652: 2490 | 2090;  4 x 4096, 8 of 96 over 2, 2000: 558 | 480;
// 2 x 2355, 32 of 32 over 8, 289: 132 | 96.
template <class T, class F> void with_columns(int dim, F&& f) {
  if (dim <= 32) f(T{}, std::integral_constant<int, 32>{});
  else if (dim <= 64) f(T{}, std::integral_constant<int, 64>{});
  else if (dim <= 96) f(T{}, std::integral_constant<int, 96>{});
  else f(T{}, std::integral_constant<int, 128>{});
}
template <class F> void with_type(int dtype, int dim, F&& f) {
  if (dtype == QDS_BF16) with_columns<bf16>(dim, f);
  else with_columns<half>(dim, f);
}

struct StepPlan {
  int32_t tiles, cut, range;
};
// Slots are cut into ranges where there are fewer heads than workgroups that fill the
// card; a range has at least four strips for each wave (with one strip, a key head over
// 65536 slots takes as long: 18.8 us, and 18.4 with four).  Short caches stay whole, as
// a second launch costs more than a longer range: 4 policies of 8 key heads of 64, 516 and
// 1016 slots, whole 6.8 and 9.4 us on the card, 12.2 and 12.1 a call; cut in two 8.0 and
// 8.9, 16.2 and 15.7 a call.  At 2016 slots whole takes 15.8, cut 9.0.
StepPlan step_plan(const qds_window_config* c) {
  StepPlan p{};
  p.tiles = (int32_t)ceil_div(c->heads / c->kv_heads, 16);
  const int64_t lists = (int64_t)c->batch * c->kv_heads * p.tiles, slots = (int64_t)c->window + c->sinks;
  constexpr int64_t strip = kWaves * kStrip;
  int64_t cut = lists > 0 ? ceil_div(kFill, lists) : 1;
  const int64_t most = ceil_div(slots, 4 * strip);
  if (cut > most) cut = most;
  if (slots * (c->dim <= 64 ? 64 : 128) <= 80 << 10) cut = 1;
  p.range = (int32_t)(ceil_div(ceil_div(slots, cut), strip) * strip);
  p.cut = (int32_t)ceil_div(slots, p.range);
  return p;
}

}  // namespace
}  // namespace seq

using namespace seq;

extern "C" qds_status qds_window_forward(const qds_window_config* c, qds_view q, qds_view k,
                                         qds_view v, const int32_t* lengths, qds_view o, float* lse,
                                         void* stream) {
  const qds_status st = validate(c);
  if (st != QDS_OK) return st;
  if (c->batch == 0 || c->length == 0) return QDS_OK;
  if (query_grid(c) > most_blocks(kBlock)) return QDS_ERR_UNSUPPORTED;
  if (!usable(q) || !usable(k) || !usable(v) || !usable(o) || !lse) return QDS_ERR_INVALID_ARG;
  if (!near_rows(k, c->length) || !near_rows(v, c->length)) return QDS_ERR_UNSUPPORTED;
  WindowArgs a = window_args(c, lengths);
  a.q = view(q), a.k = view(k), a.v = view(v), a.o = view(o), a.lse = lse;
  const int blocks = (int)ceil_div(c->length, kForwardRows >> a.share);
  const uint32_t grid = (uint32_t)query_grid(c);
  with_type(c->dtype, c->dim, [&](auto t, auto d) {
    k_window_forward<decltype(t), decltype(d)::value><<<grid, kBlock, 0, (hipStream_t)stream>>>(a, blocks);
  });
  return launch_status();
}

extern "C" qds_status qds_window_backward_workspace(const qds_window_config* c, uint64_t* bytes) {
  const qds_status st = validate(c);
  if (st != QDS_OK) return st;
  if (!bytes) return QDS_ERR_INVALID_ARG;
  const KeyPlan p = key_plan(c);
  const int64_t lists = (int64_t)c->batch * c->kv_heads;
  const int64_t joined = cut_to(p) - cut_from(p);
  if (query_grid(c) > most_blocks(kBlock) || lists * p.items > most_blocks(kBlock) ||
      lists * joined * (kKeyRows / 8) > most_blocks(kBlock))         // the join: 8 rows or more a workgroup
    return QDS_ERR_UNSUPPORTED;
  const uint64_t delta = align_up((uint64_t)c->batch * c->heads * c->length * sizeof(float));
  *bytes = delta + align_up(key_sums_bytes(c, p));
  return QDS_OK;
}

extern "C" qds_status qds_window_backward(const qds_window_config* c, qds_view dout, qds_view q,
                                          qds_view k, qds_view v, qds_view o, const float* lse,
                                          const int32_t* lengths, qds_view dq, qds_view dk,
                                          qds_view dv, void* workspace, uint64_t workspace_bytes,
                                          void* stream) {
  uint64_t need = 0;
  const qds_status st = qds_window_backward_workspace(c, &need);
  if (st != QDS_OK) return st;
  if (c->batch == 0 || c->length == 0) return QDS_OK;
  if (!usable(dout) || !usable(q) || !usable(k) || !usable(v) || !usable(o) || !usable(dq) ||
      !usable(dk) || !usable(dv) || !lse || !workspace || ((uintptr_t)workspace & 255))
    return QDS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return QDS_ERR_WORKSPACE_TOO_SMALL;
  if (!near_rows(q, c->length) || !near_rows(k, c->length) || !near_rows(v, c->length) || !near_rows(dout, c->length)) return QDS_ERR_UNSUPPORTED;
  WindowArgs a = window_args(c, lengths);
  a.q = view(q), a.k = view(k), a.v = view(v), a.o = view(o), a.dout = view(dout);
  a.dq = view(dq), a.dk = view(dk), a.dv = view(dv), a.lse = const_cast<float*>(lse);
  a.delta = (float*)workspace;
  float* parts = (float*)((char*)workspace + align_up((uint64_t)c->batch * c->heads * c->length * sizeof(float)));
  const KeyPlan plan = key_plan(c);
  const int blocks = (int)ceil_div(c->length, kForwardRows >> a.share);
  const int lists = c->batch * c->kv_heads;
  hipStream_t s = (hipStream_t)stream;
  with_type(c->dtype, c->dim, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int DC = decltype(d)::value, DP = padded(DC);
    k_window_dq<T, DC><<<(uint32_t)query_grid(c), kBlock, 0, s>>>(a, blocks);
    k_window_dkdv<T, DC><<<lists * plan.items, kBlock, 0, s>>>(a, plan, parts);
    if (cut_to(plan) > cut_from(plan)) {
      const int per_head = (cut_to(plan) - cut_from(plan)) * (kKeyRows / (kBlock * 4 / DP));
      k_window_dkdv_join<T, DP><<<(uint32_t)lists * per_head, kBlock, 0, s>>>(a, plan, per_head, parts);
    }
  });
  return launch_status();
}

extern "C" qds_status qds_window_step_workspace(const qds_window_config* c, uint64_t* bytes) {
  const qds_status st = validate(c);
  if (st != QDS_OK) return st;
  if (!bytes) return QDS_ERR_INVALID_ARG;
  const StepPlan p = step_plan(c);
  const uint64_t items = (uint64_t)c->batch * c->kv_heads * p.tiles * p.cut, dp = c->dim <= 64 ? 64 : 128;
  *bytes = p.cut == 1 ? 0 : align_up(items * 16 * (2 + dp) * sizeof(float));
  return QDS_OK;
}

extern "C" qds_status qds_window_step(const qds_window_config* c, qds_view q, qds_view k, qds_view v,
                                      void* k_cache, void* v_cache, const int32_t* pos, qds_view o,
                                      void* workspace, uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  const qds_status st = qds_window_step_workspace(c, &need);
  if (st != QDS_OK) return st;
  if (c->batch == 0) return QDS_OK;
  if (!usable(q, false) || !usable(k, false) || !usable(v, false) || !usable(o, false) || !k_cache ||
      !v_cache || !aligned16(k_cache) || !aligned16(v_cache) || !pos)
    return QDS_ERR_INVALID_ARG;
  if (need && (!workspace || ((uintptr_t)workspace & 255))) return QDS_ERR_INVALID_ARG;
  if (workspace_bytes < need) return QDS_ERR_WORKSPACE_TOO_SMALL;
  const StepPlan p = step_plan(c);
  StepArgs a{view(q), view(k), view(v), view(o), k_cache, v_cache, pos, (float*)workspace,
             c->batch, c->heads, c->kv_heads, c->dim, c->window, c->sinks, p.tiles, p.cut, p.range, c->scale};
  hipStream_t s = (hipStream_t)stream;
  with_type(c->dtype, c->dim, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int DP = padded(decltype(d)::value);
    k_window_step<T, DP><<<dim3(c->batch * c->kv_heads * p.tiles, p.cut), kBlock, 0, s>>>(a);
    if (p.cut > 1) k_window_step_join<T, DP><<<c->batch * c->heads, 64 * kStepJoinWaves, 0, s>>>(a);
  });
  return launch_status();
}

extern "C" qds_status qds_window_cache_fill(const qds_window_config* c, qds_view k, qds_view v,
                                            const int32_t* lengths, void* k_cache, void* v_cache,
                                            void* stream) {
  const qds_status st = validate(c);
  if (st != QDS_OK) return st;
  if (c->batch == 0 || c->length == 0) return QDS_OK;
  if (!usable(k) || !usable(v) || !k_cache || !v_cache || !aligned16(k_cache) || !aligned16(v_cache))
    return QDS_ERR_INVALID_ARG;
  WindowArgs a = window_args(c, lengths);
  a.k = view(k), a.v = view(v);
  const int64_t packs = ((int64_t)c->window + c->sinks) * (c->dim / 8) * c->kv_heads * c->batch;
  const int64_t most = 8 * kFill, blocks = ceil_div(packs, kBlock);
  const uint32_t grid = (uint32_t)(blocks < most ? blocks : most);
  hipStream_t s = (hipStream_t)stream;
  if (c->dtype == QDS_BF16) k_window_fill<bf16><<<grid, kBlock, 0, s>>>(a, (bf16*)k_cache, (bf16*)v_cache);
  else k_window_fill<half><<<grid, kBlock, 0, s>>>(a, (half*)k_cache, (half*)v_cache);
  return launch_status();
}
