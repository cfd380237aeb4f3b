// Dropout: y = keep x / (1 - p) + res, the mask from a counter-based generator and never stored; the backward is the same
// without res. Philox4x32-10 (Salmon et al., Parallel random numbers: as easy as 1, 2, 3; 2011): ten rounds of two 32 x 32 -> 64
// products give 128 bits for a counter, 16 of them to each of eight elements.
// Bound by memory (x, res, y once each) as long as the generator hides behind it: its products are quarter rate, so a counter's
// bits are shared by eight elements; 32 bits to each would cost as much time as the memory does. 61440 x 1024 bf16 with a residual, forward
// and backward, 114 us (5.5 TB/s); 61440 x 512 fp32 51 us (4.9 TB/s); 7680 x 200 fp32 4.3 us a launch.
#include "../../../include/stacklstm_layers.h"
#include "../head/head.h"

namespace {

struct DropArgs {
  int64_t rows, first, period;                         // first: the launch's first row
  int width, groups;                                   // groups of eight elements to a row
  uint32_t cut;
  float scale;
  const void *x, *res;
  void* y;
  int64_t ldx, ldr, ldy;
  const int64_t* seed;
};

__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
    const uint32_t n0 = (uint32_t)(b >> 32) ^ c[1] ^ k0, n2 = (uint32_t)(a >> 32) ^ c[3] ^ k1;
    c[1] = (uint32_t)b, c[3] = (uint32_t)a;
    c[0] = n0, c[2] = n2;
    k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
  }
}

}  // namespace

// A thread to a group of eight elements of a row.
template <typename T>
__global__ void __launch_bounds__(256) k_dropout(DropArgs a) {
  constexpr int V = vec<T>::N, Q = 8 / V;
  // (a workgroup's first group by one division of scalars; a thread is a few rows behind it at most)
  const int64_t g0 = (int64_t)blockIdx.x * 256;
  const int64_t r0 = g0 / a.groups;
  const uint32_t at = (uint32_t)(g0 - r0 * a.groups) + threadIdx.x;
  const int64_t row = r0 + at / (uint32_t)a.groups;
  const int g = (int)(at % (uint32_t)a.groups);
  if (row >= a.rows) return;
  const int64_t all = a.first + row;
  const uint32_t mrow = a.period ? (uint32_t)all % (uint32_t)a.period : (uint32_t)all;
  const uint64_t key = (uint64_t)a.seed[0], step = (uint64_t)a.seed[1];
  uint32_t c[4] = {(uint32_t)g, mrow, (uint32_t)step, (uint32_t)(step >> 32)};
  const T* x = (const T*)a.x + row * a.ldx;
  const T* res = (const T*)a.res + (a.res ? row * a.ldr : 0);
  T* y = (T*)a.y + row * a.ldy;
  u32x4 raw[Q], add[Q];
#pragma unroll
  for (int i = 0; i < Q; ++i) {
    const bool in = (Q * g + i) * V < a.width;
    raw[i] = in ? load_vec(x, Q * g + i, a.width) : u32x4{0u, 0u, 0u, 0u};
    add[i] = a.res && in ? load_vec(res, Q * g + i, a.width) : u32x4{0u, 0u, 0u, 0u};
  }
  philox(c, (uint32_t)key, (uint32_t)(key >> 32));
#pragma unroll
  for (int i = 0; i < Q; ++i) {
    float v[V], w[V];
    vec<T>::unpack(raw[i], v);
    vec<T>::unpack(add[i], w);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int e = i * V + k;
      const uint32_t bits = e & 1 ? c[e / 2] >> 16 : c[e / 2] & 0xffffu;
      v[k] = bits >= a.cut ? v[k] * a.scale : 0.f;
      if (a.res) v[k] += w[k];
    }
    if ((Q * g + i) * V < a.width) store_vec(y, Q * g + i, a.width, v);
  }
}

namespace {

bool dropout_ok(const slstm_dropout_dims* d) {
  return d && d->rows >= 0 && d->rows <= 0x7fffffff && d->width >= 1 && d->width <= (1 << 24) &&
         (d->type == SLSTM_F32 || d->type == SLSTM_BF16) && d->p >= 0.f && d->p <= 1.f && d->period >= 0 &&
         d->period <= 0x7fffffff && stride_ok(d->ld_x, d->width) && stride_ok(d->ld_res, d->width) &&
         stride_ok(d->ld_y, d->width);
}

int dropout_run(const slstm_dropout_dims* d, const void* x, const void* res, const int64_t* seed, void* y, hipStream_t st) {
  if (!x || !seed || !y) return SLSTM_EINVAL;
  DropArgs a = {};
  a.width = d->width, a.groups = (d->width + 7) / 8, a.period = d->period, a.seed = seed;
  a.cut = (uint32_t)floor((double)d->p * 65536.0 + 0.5);
  a.scale = a.cut < 65536u ? (float)(65536.0 / (65536.0 - a.cut)) : 0.f;
  a.ldx = row_stride(d->ld_x, d->width), a.ldr = row_stride(d->ld_res, d->width), a.ldy = row_stride(d->ld_y, d->width);
  if ((y == x && a.ldx != a.ldy) || (y == res && a.ldr != a.ldy)) return SLSTM_EINVAL;
  auto run = [&](auto t) {
    typedef decltype(t) T;
    const int64_t most = kMostGroups * 256 / a.groups > 1 ? kMostGroups * 256 / a.groups : 1;
    in_pieces(d->rows, most, [&](int64_t r0, int64_t n) {
      DropArgs p = a;
      p.rows = n, p.first = r0;
      p.x = (const T*)x + r0 * a.ldx, p.res = offset((const T*)res, r0 * a.ldr), p.y = (T*)y + r0 * a.ldy;
      hipLaunchKernelGGL(k_dropout<T>, dim3((unsigned)((n * a.groups + 255) / 256)), dim3(256), 0, st, p);
    });
  };
  if (d->type == SLSTM_F32) run(float());
  else run(bf16_t());
  return hipGetLastError() == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
}

}  // namespace

extern "C" int stacklstm_dropout_fwd(const slstm_dropout_dims* d, const void* x, const void* res, const int64_t* seed, void* y,
                                     void* stream) {
  if (!dropout_ok(d)) return SLSTM_EINVAL;
  if (d->rows == 0) return SLSTM_OK;
  return dropout_run(d, x, res, seed, y, as_stream(stream));
}

extern "C" int stacklstm_dropout_bwd(const slstm_dropout_dims* d, const void* dy, const int64_t* seed, void* dx, void* stream) {
  if (!dropout_ok(d)) return SLSTM_EINVAL;
  if (d->rows == 0) return SLSTM_OK;
  return dropout_run(d, dy, nullptr, seed, dx, as_stream(stream));
}
