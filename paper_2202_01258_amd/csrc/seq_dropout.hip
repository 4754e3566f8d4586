// seq_dropout.hip -- dropout from a counter, with the residual's addition.  The C ABI is in
// include/qd_seq.h.
//
// A mask is never stored: whether an element is kept follows from the seed, the step, the place
// in the program and the element's number, so the backward pass draws the same again.  Eight
// elements share a Philox4x32-10 block (Salmon et al., "Parallel random numbers: as easy as 1, 2,
// 3", SC 2011), 16 bits each: with 32 bits each, four elements would carry the block's ten
// rounds, as many vector instructions as memory leaves time for.  32000 x 1024 bfloat16: 30 us
// (131 MB, 4.4 TB/s).
#include "seq_common.hpp"
#include "seq_rows.hpp"

namespace seq {
namespace {

constexpr int kBlock = 256, kGroup = 8;

struct DropoutArgs {
  const void *x, *r;
  void* y;
  const int64_t* rng;
  int64_t elements;
  uint32_t threshold, site;
  float up;
};

struct Words {
  uint32_t x[4];
};
__device__ inline Words philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    const uint32_t n0 = (uint32_t)(b >> 32) ^ c1 ^ k0, n2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)b;
    c3 = (uint32_t)a;
    c0 = n0;
    c2 = n2;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return Words{{c0, c1, c2, c3}};
}

template <class T> __global__ __launch_bounds__(kBlock) void k_dropout(DropoutArgs a) {
  const uint32_t group = blockIdx.x * kBlock + threadIdx.x;
  const int64_t at = (int64_t)group * kGroup;
  if (at >= a.elements) return;
  const uint64_t seed = (uint64_t)a.rng[0], step = (uint64_t)a.rng[1];
  const int count = (int)(a.elements - at < kGroup ? a.elements - at : kGroup);
  float x[kGroup], r[kGroup];
#pragma unroll
  for (int i = 0; i < kGroup; ++i) r[i] = 0.0f;
  const T *xp = (const T*)a.x + at, *rp = (const T*)a.r + at;
  if (count == kGroup) {
    load<T, kGroup>(x, xp);
    if (a.r) load<T, kGroup>(r, rp);
  } else {
#pragma unroll
    for (int i = 0; i < kGroup; ++i) {
      x[i] = i < count ? to_f32(xp[i]) : 0.0f;
      if (a.r && i < count) r[i] = to_f32(rp[i]);
    }
  }
  const Words w = philox(group, a.site, (uint32_t)step, (uint32_t)(step >> 32), (uint32_t)seed, (uint32_t)(seed >> 32));
#pragma unroll
  for (int i = 0; i < kGroup; ++i) {
    const uint32_t draw = i & 1 ? w.x[i / 2] >> 16 : w.x[i / 2] & 0xffffu;
    const float kept = x[i] * a.up;
    r[i] += draw >= a.threshold ? kept : 0.0f;
  }
  T* yp = (T*)a.y + at;
  if (count == kGroup) {
    store<T, kGroup>(yp, r);
  } else {
#pragma unroll
    for (int i = 0; i < kGroup; ++i)
      if (i < count) yp[i] = from_f32<T>(r[i]);
  }
}

}  // namespace
}  // namespace seq

using namespace seq;

extern "C" qds_status qds_dropout(const qds_dropout_config* c, const void* x, const void* residual,
                                  const int64_t* rng, void* y, void* stream) {
  if (!c || c->abi_version != QDS_ABI_VERSION) return QDS_ERR_INVALID_ARG;
  if (c->dtype < QDS_F32 || c->dtype > QDS_F16) return QDS_ERR_INVALID_ARG;
  if (c->elements < 0 || c->elements > ((int64_t)1 << 34) || c->threshold > 65535) return QDS_ERR_INVALID_ARG;
  if (c->elements == 0) return QDS_OK;
  if (!x || !rng || !y) return QDS_ERR_INVALID_ARG;
  const DropoutArgs a{x, residual, y, rng, c->elements, c->threshold, c->site, 65536.0f / (float)(65536 - c->threshold)};
  const uint32_t grid = (uint32_t)ceil_div(ceil_div(c->elements, kGroup), kBlock);
  hipStream_t s = (hipStream_t)stream;
  if (c->dtype == QDS_F32) k_dropout<float><<<grid, kBlock, 0, s>>>(a);
  else if (c->dtype == QDS_BF16) k_dropout<bf16><<<grid, kBlock, 0, s>>>(a);
  else k_dropout<half><<<grid, kBlock, 0, s>>>(a);
  return launch_status();
}
