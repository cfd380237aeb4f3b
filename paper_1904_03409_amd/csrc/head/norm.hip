// Layer norm of rows, forward and backward.
//   s = x + res, mu = mean(s), rstd = 1 / sqrt(mean((s - mu)^2) + eps), y = (s - mu) rstd gamma + beta
//   dx = rstd (g - mean(g) - xh mean(g xh)) + dsum, g = dy gamma, xh = (s - mu) rstd
//   dgamma = sum over rows of dy xh, dbeta = sum over rows of dy
// Bound by memory: a forward reads x (and res) and writes y (and the sum) once, a backward reads s, dy
// (and dsum) and writes dx once. A row stays in registers between its loads and its stores, in the
// fewest lanes that hold it in one or two vectors each (a wave then carries several narrow rows);
// the variance is summed from differences to the mean, in 32 bits. 61440 x 1024 bf16 with a residual: forward 92 us
// (5.5 TB/s), backward 113 us (4.6 TB/s) and 6 us for the columns' sums; 22912 x 200 f32: 10.2 us (3.6 TB/s), 13.7 and 3.9 us.
#include <algorithm>

#include "../../../include/stacklstm_head.h"
#include "head.h"

namespace {

struct NormArgs {
  int rows, W, parts, strips;                          // of a backward: workgroups that take rows, and columns
  float eps;
  const void *x, *res, *dy, *dsum;
  int64_t ldx, ldr, ldd;
  const float *gamma, *beta;
  void *sum, *y, *dx;
  float *mean, *rstd, *dgamma, *dbeta, *part;
};

// threads of a workgroup with TPR lanes (or threads) to a row, and its rows
constexpr int norm_threads(int tpr) { return tpr <= 64 ? 256 : tpr; }
constexpr int norm_rows(int tpr) { return tpr <= 64 ? 256 / tpr : 1; }

}  // namespace

template <typename T, int TPR, int NV>
__global__ void __launch_bounds__(norm_threads(TPR)) k_norm_fwd(NormArgs a) {
  constexpr int V = vec<T>::N;
  __shared__ float red[2][16];
  const int t = threadIdx.x & (TPR - 1), W = a.W;
  const int64_t row = (int64_t)blockIdx.x * norm_rows(TPR) + threadIdx.x / TPR;
  const bool here = row < a.rows;
  const T* x = (const T*)a.x + row * a.ldx;
  const T* res = (const T*)a.res + row * a.ldr;
  float v[NV][V];
  u32x4 rx[NV], rr[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * TPR;
    const bool in = here && c * V < W;
    rx[i] = in ? load_vec(x, c, W) : u32x4{0u, 0u, 0u, 0u};
    rr[i] = in && a.res ? load_vec(res, c, W) : u32x4{0u, 0u, 0u, 0u};
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    vec<T>::unpack(rx[i], v[i]);
    if (a.res) {
      float r[V];
      vec<T>::unpack(rr[i], r);
#pragma unroll
      for (int k = 0; k < V; ++k) v[i][k] += r[k];
    }
#pragma unroll
    for (int k = 0; k < V; ++k) s += v[i][k];
  }
  if (a.sum && here) {
    T* o = (T*)a.sum + row * W;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if ((t + i * TPR) * V < W) store_vec(o, t + i * TPR, W, v[i]);
  }
  const float mu = group_reduce<TPR>(s, op_sum(), red[0]) / (float)W;
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float d = v[i][k] - mu;
      if ((t + i * TPR) * V + k < W) q += d * d;
    }
  const float rstd = rsqrtf(group_reduce<TPR>(q, op_sum(), red[1]) / (float)W + a.eps);
  if (!here) return;
  if (t == 0) {
    if (a.mean) a.mean[row] = mu;
    if (a.rstd) a.rstd[row] = rstd;
  }
  T* y = (T*)a.y + row * W;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * TPR;
    if (c * V >= W) continue;
    float o[V];
#pragma unroll
    for (int h = 0; h < V; h += 4) {
      float g[4] = {1.f, 1.f, 1.f, 1.f}, b[4] = {0.f, 0.f, 0.f, 0.f};
      if (a.gamma) vec<float>::unpack(load_vec(a.gamma, (c * V + h) / 4, W), g);
      if (a.beta) vec<float>::unpack(load_vec(a.beta, (c * V + h) / 4, W), b);
#pragma unroll
      for (int k = 0; k < 4; ++k) o[h + k] = (v[i][h + k] - mu) * rstd * g[k] + b[k];
    }
    store_vec(y, c, W, o);
  }
}

// dgamma | dbeta of a strip of 16 vectors of columns over all rows, for few rows: NT / 16 rows at a time.
template <typename T, int NT>
__device__ __forceinline__ void norm_strip(const NormArgs& a, int strip) {
  constexpr int V = vec<T>::N, NW = NT / 64;
  __shared__ float red[NW][2][16 * V];
  const int c = strip * 16 + (threadIdx.x & 15), W = a.W;
  float sg[V], sb[V];
#pragma unroll
  for (int k = 0; k < V; ++k) sg[k] = sb[k] = 0.f;
  if (c * V < W) {
#pragma unroll 4
    for (int row = threadIdx.x >> 4; row < a.rows; row += NT / 16) {
      float x[V], d[V];
      vec<T>::unpack(load_vec((const T*)a.x + row * a.ldx, c, W), x);
      vec<T>::unpack(load_vec((const T*)a.dy + row * a.ldd, c, W), d);
      const float mu = a.mean[row], rstd = a.rstd[row];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        sg[k] += d[k] * ((x[k] - mu) * rstd);
        sb[k] += d[k];
      }
    }
  }
#pragma unroll
  for (int k = 0; k < V; ++k) {
    sg[k] = across<16>(sg[k], op_sum());
    sb[k] = across<16>(sb[k], op_sum());
  }
  if ((threadIdx.x & 63) < 16) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      red[threadIdx.x >> 6][0][threadIdx.x % 16 * V + k] = sg[k];
      red[threadIdx.x >> 6][1][threadIdx.x % 16 * V + k] = sb[k];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * V; i += NT) {
    const int which = i / (16 * V), n = strip * 16 * V + i % (16 * V);
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) v += red[w][which][i % (16 * V)];
    float* o = which ? a.dbeta : a.dgamma;
    if (o && n < W) o[n] = v;
  }
}

// Rows in turn; a thread keeps the sums of its columns over the rows that its workgroup takes, and the
// workgroups' sums are added by k_norm_cols in a fixed order (no atomics: equal runs are equal bit for bit).
// Few rows have workgroups of their own for the columns' sums instead, which read the rows again (from L2: a launch costs
// more).
template <typename T, int TPR, int NV>
__global__ void __launch_bounds__(norm_threads(TPR)) k_norm_bwd(NormArgs a) {
  constexpr int V = vec<T>::N, RPB = norm_rows(TPR);
  if ((int)blockIdx.x >= a.parts) return norm_strip<T, norm_threads(TPR)>(a, (int)blockIdx.x - a.parts);
  __shared__ float red[2][2][16];
  extern __shared__ float cols[];                      // TPR <= 64: [2][W]
  const int t = threadIdx.x & (TPR - 1), W = a.W;
  float sg[NV][V], sb[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int k = 0; k < V; ++k) sg[i][k] = sb[i][k] = 0.f;
  const float inv = 1.f / (float)W;
  int flip = 0;
  // the next row's loads are on their way while this one is computed
  u32x4 nx[NV], nd[NV], ns[NV];
  float nmu, nrstd;
  auto fetch = [&](int64_t row) {
    const bool here = row < a.rows;
    const T* x = (const T*)a.x + row * a.ldx;
    const T* dy = (const T*)a.dy + row * a.ldd;
    const T* ds = (const T*)a.dsum + row * W;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * TPR;
      const bool in = here && c * V < W;
      nx[i] = in ? load_vec(x, c, W) : u32x4{0u, 0u, 0u, 0u};
      nd[i] = in ? load_vec(dy, c, W) : u32x4{0u, 0u, 0u, 0u};
      ns[i] = in && a.dsum ? load_vec(ds, c, W) : u32x4{0u, 0u, 0u, 0u};
    }
    nmu = here ? a.mean[row] : 0.f;
    nrstd = here ? a.rstd[row] : 0.f;
  };
  const int64_t step = (int64_t)a.parts * RPB;
  fetch((int64_t)blockIdx.x * RPB + threadIdx.x / TPR);
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += step, flip ^= 1) {
    const int64_t row = r0 + threadIdx.x / TPR;
    const bool here = row < a.rows;
    u32x4 rx[NV], rd[NV], rs[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) rx[i] = nx[i], rd[i] = nd[i], rs[i] = ns[i];
    const float mu = nmu, rstd = nrstd;
    if (r0 + step < a.rows) fetch(row + step);
    float xh[NV][V], g[NV][V], m1 = 0.f, m2 = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * TPR;
      vec<T>::unpack(rx[i], xh[i]);
      vec<T>::unpack(rd[i], g[i]);
#pragma unroll
      for (int h = 0; h < V; h += 4) {
        float w[4] = {1.f, 1.f, 1.f, 1.f};
        if (a.gamma && c * V + h < W) vec<float>::unpack(load_vec(a.gamma, (c * V + h) / 4, W), w);
#pragma unroll
        for (int k = h; k < h + 4; ++k) {
          // (past the row's end dy is 0, but (0 - mu) rstd may be past fp32's range, and 0 times that is NaN)
          xh[i][k] = c * V + k < W ? (xh[i][k] - mu) * rstd : 0.f;
          sg[i][k] += g[i][k] * xh[i][k];
          sb[i][k] += g[i][k];
          g[i][k] *= w[k - h];
          m1 += g[i][k];
          m2 += g[i][k] * xh[i][k];
        }
      }
    }
    m1 = group_reduce<TPR>(m1, op_sum(), red[flip][0]) * inv;
    m2 = group_reduce<TPR>(m2, op_sum(), red[flip][1]) * inv;
    if (!here) continue;
    T* dx = (T*)a.dx + row * W;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = t + i * TPR;
      if (c * V >= W) continue;
      float o[V], d[V];
      vec<T>::unpack(rs[i], d);
#pragma unroll
      for (int k = 0; k < V; ++k) o[k] = rstd * (g[i][k] - m1 - xh[i][k] * m2) + d[k];
      store_vec(dx, c, W, o);
    }
  }
  if (a.strips || (!a.dgamma && !a.dbeta)) return;
  float* pg = a.parts == 1 ? a.dgamma : a.part + (size_t)blockIdx.x * 2 * W;
  float* pb = a.parts == 1 ? a.dbeta : a.part + (size_t)blockIdx.x * 2 * W + W;
  if constexpr (TPR <= 64) {
    // rows of a wave, then the waves one after the other
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        sg[i][k] = across<TPR>(sg[i][k], op_sum());
        sb[i][k] = across<TPR>(sb[i][k], op_sum());
      }
    for (int w = 0; w < 4; ++w) {
      if ((int)(threadIdx.x >> 6) == w && (threadIdx.x & 63) < TPR) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int k = 0; k < V; ++k) {
            const int n = (t + i * TPR) * V + k;
            if (n >= W) continue;
            cols[n] = w ? cols[n] + sg[i][k] : sg[i][k];
            cols[W + n] = w ? cols[W + n] + sb[i][k] : sb[i][k];
          }
      }
      __syncthreads();
    }
    for (int n = threadIdx.x; n < W; n += 256) {
      if (pg) pg[n] = cols[n];
      if (pb) pb[n] = cols[W + n];
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int n = (t + i * TPR) * V + k;
        if (n >= W) continue;
        if (pg) pg[n] = sg[i][k];
        if (pb) pb[n] = sb[i][k];
      }
  }
}

// dgamma | dbeta: the sums of P workgroups.
__global__ void __launch_bounds__(1024) k_norm_cols(const float* part, int P, int W, float* dgamma, float* dbeta) {
  __shared__ float red[16][8];
  const float v = column_sum(part, P, 2 * W, red);
  const int n = blockIdx.x * 8 + threadIdx.x;
  if (threadIdx.x >= 8 || n >= 2 * W) return;
  float* o = n < W ? dgamma : dbeta;
  if (o) o[n < W ? n : n - W] = v;
}

namespace {

constexpr int kNormMaxParts = 768;                     // workgroups of a backward, three to a CU
constexpr int kNormMaxWidth = 8192;

bool norm_ok(const slstm_norm_dims* d) {
  return d && d->rows >= 0 && d->rows <= 0x7fffffff && d->width >= 1 && d->width <= kNormMaxWidth &&
         (d->type == SLSTM_F32 || d->type == SLSTM_BF16) && d->eps >= 0.f && stride_ok(d->ld_x, d->width) &&
         stride_ok(d->ld_res, d->width) && stride_ok(d->ld_dy, d->width);
}
// Lanes to a row: the fewest that hold it in one vector each, up to a wave (with half the lanes and two vectors, 30000 x 512 bf16
// took 28.4 and 29.7 us, forward and backward, instead of 25.8 and 27.7; 22912 x 100 f32 9.3 and 13.0 instead of 8.5 and 9.7),
// of two in a whole wave, then a workgroup (two barriers a row, but the sums of a thread's columns stay in registers: four
// vectors a lane of 16-bit rows take 234 of them).
int norm_vec(const slstm_norm_dims* d) { return d->type == SLSTM_F32 ? 4 : 8; }
int norm_tpr(const slstm_norm_dims* d) {
  const int n = (d->width + norm_vec(d) - 1) / norm_vec(d);
  return n <= 8 ? 8 : n <= 16 ? 16 : n <= 32 ? 32 : n <= 128 ? 64 : n <= 512 ? 256 : n <= 1024 ? 512 : 1024;
}
int norm_nv(const slstm_norm_dims* d, int tpr) {
  const int n = (d->width + norm_vec(d) - 1) / norm_vec(d), q = (n + tpr - 1) / tpr;
  return q <= 1 ? 1 : 2;
}
int norm_parts(const slstm_norm_dims* d) {
  // (all with as many rows, but for the last)
  const int64_t rpb = norm_rows(norm_tpr(d)), groups = std::max<int64_t>(1, (d->rows + rpb - 1) / rpb);
  const int64_t rounds = (groups + kNormMaxParts - 1) / kNormMaxParts;
  return (int)((groups + rounds - 1) / rounds);
}

template <typename F>
bool norm_dispatch(const slstm_norm_dims* d, F f) {
  const int tpr = norm_tpr(d), nv = norm_nv(d, tpr);
#define NORM_CASE(T_, TPR_, NV_) \
  if (tpr == TPR_ && nv == NV_) return f(T_(), std::integral_constant<int, TPR_>(), std::integral_constant<int, NV_>()), true;
#define NORM_TYPE(T_) \
  NORM_CASE(T_, 8, 1) NORM_CASE(T_, 16, 1) NORM_CASE(T_, 32, 1) NORM_CASE(T_, 64, 1) NORM_CASE(T_, 64, 2) \
  NORM_CASE(T_, 256, 1) NORM_CASE(T_, 256, 2) NORM_CASE(T_, 512, 2)
  if (d->type == SLSTM_F32) {
    NORM_TYPE(float)
    NORM_CASE(float, 1024, 2)
  } else {
    NORM_TYPE(bf16_t)
  }
#undef NORM_TYPE
#undef NORM_CASE
  return false;
}

}  // namespace

extern "C" size_t stacklstm_norm_workspace_bytes(const slstm_norm_dims* d) {
  if (!norm_ok(d)) return 0;
  const int P = norm_parts(d);
  return P > 1 ? (size_t)P * 2 * d->width * 4 : 4;
}

extern "C" int stacklstm_norm_fwd(const slstm_norm_dims* d, const void* x, const void* res, const float* gamma,
                                  const float* beta, void* sum, void* y, float* mean, float* rstd, void* stream) {
  if (!norm_ok(d)) return SLSTM_EINVAL;
  if (d->rows == 0) return SLSTM_OK;
  if (!x || !y || (sum && !res)) return SLSTM_EINVAL;
  NormArgs a = {};
  a.rows = (int)d->rows, a.W = d->width, a.eps = d->eps;
  a.x = x, a.res = res, a.gamma = gamma, a.beta = beta, a.sum = sum, a.y = y, a.mean = mean, a.rstd = rstd;
  a.ldx = row_stride(d->ld_x, d->width), a.ldr = row_stride(d->ld_res, d->width);
  const bool ok = norm_dispatch(d, [&](auto t, auto tpr, auto nv) {
    typedef decltype(t) T;
    constexpr int TPR = decltype(tpr)::value, RPB = norm_rows(TPR);
    in_pieces(d->rows, kMostGroups * RPB, [&](int64_t r0, int64_t n) {
      NormArgs p = a;
      p.rows = (int)n;
      p.x = offset((const T*)x, r0 * a.ldx), p.res = offset((const T*)res, r0 * a.ldr);
      p.sum = offset((T*)sum, r0 * a.W), p.y = offset((T*)y, r0 * a.W);
      p.mean = offset(mean, r0), p.rstd = offset(rstd, r0);
      hipLaunchKernelGGL((k_norm_fwd<T, TPR, decltype(nv)::value>), dim3((unsigned)((n + RPB - 1) / RPB)), dim3(norm_threads(TPR)),
                         0, as_stream(stream), p);
    });
  });
  if (!ok) return SLSTM_EINVAL;
  return hipGetLastError() == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
}

extern "C" int stacklstm_norm_bwd(const slstm_norm_dims* d, const void* x, const float* gamma, const float* mean,
                                  const float* rstd, const void* dy, const void* dsum, void* dx, float* dgamma, float* dbeta,
                                  void* workspace, size_t ws_bytes, void* stream) {
  if (!norm_ok(d)) return SLSTM_EINVAL;
  if (d->rows > 0 && (!x || !mean || !rstd || !dy || !dx)) return SLSTM_EINVAL;
  const int P = norm_parts(d);
  const bool cols = dgamma || dbeta;
  if (cols && P > 1) {
    if (!workspace || ((uintptr_t)workspace & 3u)) return SLSTM_EINVAL;
    if (ws_bytes < stacklstm_norm_workspace_bytes(d)) return SLSTM_EWORKSPACE;
  }
  NormArgs a = {};
  a.rows = (int)d->rows, a.W = d->width, a.eps = d->eps;
  a.x = x, a.dy = dy, a.dsum = dsum, a.gamma = gamma, a.dx = dx;
  a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd), a.dgamma = dgamma, a.dbeta = dbeta;
  a.part = (float*)workspace;
  a.ldx = row_stride(d->ld_x, d->width), a.ldd = row_stride(d->ld_dy, d->width);
  // up to 256 rows: strips of columns (17 rows of 1072: 17.9 us a training pass with a launch for the columns)
  a.parts = P;
  a.strips = cols && P > 1 && d->rows <= 256 ? (d->width + 16 * norm_vec(d) - 1) / (16 * norm_vec(d)) : 0;
  const bool ok = norm_dispatch(d, [&](auto t, auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value;
    const size_t lds = TPR <= 64 && cols && !a.strips ? (size_t)2 * d->width * 4 : 0;
    hipLaunchKernelGGL((k_norm_bwd<decltype(t), TPR, decltype(nv)::value>), dim3(P + a.strips), dim3(norm_threads(TPR)), lds,
                       as_stream(stream), a);
  });
  if (!ok) return SLSTM_EINVAL;
  if (cols && P > 1 && !a.strips)
    hipLaunchKernelGGL(k_norm_cols, dim3((2 * d->width + 7) / 8), dim3(1024), 0, as_stream(stream), a.part, P, d->width, dgamma,
                       dbeta);
  return hipGetLastError() == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
}
