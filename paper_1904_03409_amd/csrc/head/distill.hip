// Distillation loss of logits against a teacher's stored top logits, with a label's cross entropy.
//   p = softmax(value / tau) over the entries that are there, q_t = softmax(x / tau), q_1 = softmax(x)
//   loss = alpha tau^2 sum p (log p - log q_t[index]) - (1 - alpha) log q_1[label]
//   dx = a q_t + b q_1 - a sum_j p_j onehot(index_j) - b onehot(label), a = grad alpha tau, b = grad (1 - alpha)
// Bound by memory: the logits are read once and their gradient is written once. A row waits in registers
// (of a few lanes up to a workgroup of 512 threads) between its sums and its gradient, in its own type.
// The teacher's entries change a few elements of a row: they go out in a second store to those elements,
// behind the first ones' acknowledgement, instead of a search for every element.
// Rows that are too long for that, or too few of them to fill the chip, are cut into chunks: k_distill_part leaves
// each chunk's maximum and sums (and the logits at the entries), k_distill_chunk joins them. Loss and gradient: 4096 x 32000
// bf16 119 us (4.6 TB/s); 7680 x 83 f32 6.9 us; 16 x 131071 f32 in chunks 4.1 + 7.8 us (waits for memory, one after the other).
#include <algorithm>

#include "../../../include/stacklstm_head.h"
#include "head.h"

namespace {

constexpr int kEntries = 256;                          // most entries of a row
constexpr int kChunkVecs = 4;                          // vectors a thread in a chunk of 256 threads

struct DistillArgs {
  int rows, V, K, chunks;
  float tau, alpha;
  const void* x;
  void* dx;                                            // NULL: no gradient
  int64_t ldx, ldd;
  const int32_t *index, *label;
  const float *value, *grad, *stats_in;                // stats_in: m and the logs of the sums are known
  float *loss, *stats;                                 // each may be NULL
  float *part, *ent;                                   // chunks: [rows][chunks][3]; [rows][K + 1]
};

constexpr int distill_threads(int tpr) { return tpr <= 64 ? 256 : tpr; }
constexpr int distill_rows(int tpr) { return tpr <= 64 ? 256 / tpr : 1; }

// What the teacher and the label say about a row, from N threads (t of N) of which every one calls. Entry j's
// place and probability go to idx[j], p[j] (place -1: not there).
struct RowTargets {
  bool some;                                           // entries are there
  int label;                                           // -1: none
};
template <int N>
__device__ __forceinline__ RowTargets row_targets(const DistillArgs& a, int64_t row, bool here, int t, int* idx, float* p,
                                                  float* red) {
  float top = -INFINITY;
  for (int j = t; j < a.K; j += N) {
    int i = here ? a.index[row * a.K + j] : -1;
    const float w = here ? a.value[row * a.K + j] : 0.f;           // (with the index, not behind it)
    if (i < 0 || i >= a.V) i = -1;
    const float v = i >= 0 ? w : -INFINITY;
    idx[j] = i;
    p[j] = v;
    top = (v > top || v != v) ? v : top;               // (a NaN stays: the row's loss is NaN)
  }
  // lanes<>'s maximum drops NaN: carry it as a flag in the sum below (exp of it is NaN)
  top = group_reduce<N>(top, op_max(), red);
  float s = 0.f;
  for (int j = t; j < a.K; j += N) {
    const float v = p[j];
    if (idx[j] >= 0 && (top > -INFINITY || v != v)) {
      // (the difference first: values of the type's lowest are alike, over whatever tau)
      const float e = expf((v - top) / a.tau);
      p[j] = e;
      s += e;
    } else {
      p[j] = 0.f;
    }
  }
  s = group_reduce<N>(s, op_sum(), red + 16);
  RowTargets r;
  r.some = s > 0.f || s != s;
  const float inv = r.some ? 1.f / s : 0.f;
  for (int j = t; j < a.K; j += N) p[j] *= inv;
  r.label = here && a.label ? a.label[row] : -1;
  if (r.label < 0 || r.label >= a.V) r.label = -1;
  return r;
}

// Loss of a row: u[j] the logit at entry j, u[K] at the label, m the row's maximum.
template <int N>
__device__ __forceinline__ float row_loss(const DistillArgs& a, const RowTargets& r, int t, const int* idx, const float* p,
                                          const float* u, float m, float logst, float logs1, float* red) {
  const float it = 1.f / a.tau;
  float kl = 0.f;
  for (int j = t; j < a.K; j += N)
    if (p[j] > 0.f || p[j] != p[j]) kl += p[j] * (logf(p[j]) - ((u[j] - m) * it - logst));
  kl = group_reduce<N>(kl, op_sum(), red);
  float loss = r.some && a.alpha > 0.f ? a.alpha * a.tau * a.tau * kl : 0.f;
  if (r.label >= 0 && a.alpha < 1.f) loss += (1.f - a.alpha) * (logs1 - (u[a.K] - m));
  return loss;
}

// How the two exponentials of an element are made: tau = 1 needs one, tau = 2 a square, any other tau both. (An exponential
// is four times as dear as a product. Loss and gradient of 4096 rows of 32000, in one run: tau 1 and 2 122 us, 4 128, 1.5 143.)
enum { ONE = 0, SQUARE = 1, BOTH = 2 };
__device__ __forceinline__ int expo_mode(float tau, bool second) { return tau == 1.f || !second ? ONE : tau == 2.f ? SQUARE : BOTH; }

// The gradient of a row's elements.
struct RowGrad {
  Expo et, e1;
  float a, b, ct, c1;
  bool zero;
  int mode;
  template <int MODE>
  __device__ __forceinline__ float at(float x) const {
    if (MODE == ONE) return ct * et(x);
    if (MODE == SQUARE) {
      const float e = et(x);
      return e * (ct + c1 * e);
    }
    return ct * et(x) + c1 * e1(x);
  }
  __device__ __forceinline__ float operator()(float x) const {
    return mode == ONE ? at<ONE>(x) : mode == SQUARE ? at<SQUARE>(x) : at<BOTH>(x);
  }
};
__device__ __forceinline__ RowGrad row_grad(const DistillArgs& a, const RowTargets& r, int64_t row, float m, float logst,
                                            float logs1) {
  RowGrad g;
  const float gr = a.grad ? a.grad[row] : 1.f;
  g.et = Expo(m, kLog2e / a.tau);
  g.e1 = Expo(m, kLog2e);
  g.a = r.some ? gr * a.alpha * a.tau : 0.f;
  g.b = r.label >= 0 ? gr * (1.f - a.alpha) : 0.f;
  g.zero = g.a == 0.f && g.b == 0.f;
  // a over the sum of the et, b over that of the e1
  g.ct = g.a == 0.f ? 0.f : g.a * __builtin_amdgcn_exp2f(-logst * kLog2e - g.et.off);
  g.c1 = g.b == 0.f ? 0.f : g.b * __builtin_amdgcn_exp2f(-logs1 * kLog2e - g.e1.off);
  g.mode = expo_mode(a.tau, g.b != 0.f);
  if (a.tau == 1.f) g.ct += g.c1;
  if (g.mode == SQUARE) g.c1 = g.b * __builtin_amdgcn_exp2f(-logs1 * kLog2e - 2.f * g.et.off);
  return g;
}
// put(f) with the function of a row's elements, one of few kinds.
template <typename Put>
__device__ __forceinline__ void each_grad(const RowGrad& g, Put put) {
  if (g.zero) put([](float) { return 0.f; });
  else if (g.mode == ONE) put([&](float x) { return g.at<ONE>(x); });
  else if (g.mode == SQUARE) put([&](float x) { return g.at<SQUARE>(x); });
  else put([&](float x) { return g.at<BOTH>(x); });
}
// The element at entry j (j = K: the label's) with what the teacher and the label take from it.
__device__ __forceinline__ float entry_grad(const DistillArgs& a, const RowGrad& g, const RowTargets& r, int place, float x,
                                            const int* idx, const float* p) {
  float s = 0.f;
#pragma unroll 8
  for (int j = 0; j < a.K; ++j) s += idx[j] == place ? p[j] : 0.f;
  float v = g(x) - g.a * s;
  if (place == r.label) v -= g.b;
  return v;
}

}  // namespace

// Whole rows, TPR threads to each, NV vectors in a thread.
template <typename T, int TPR, int NV>
__global__ void __launch_bounds__(distill_threads(TPR)) k_distill_rows(DistillArgs a) {
  constexpr int V = vec<T>::N, RPB = distill_rows(TPR);
  __shared__ float red[6][16];
  extern __shared__ int lds[];                         // [RPB][3][K + 1]: places, probabilities, logits
  const int t = threadIdx.x & (TPR - 1), sub = RPB > 1 ? threadIdx.x / TPR : 0, n = a.K + 1;
  const int64_t row = (int64_t)blockIdx.x * RPB + sub;
  const bool here = row < a.rows;
  int* idx = lds + sub * 3 * n;
  float *p = (float*)(idx + n), *u = p + n;
  const T* x = (const T*)a.x + row * a.ldx;
  u32x4 raw[NV];
  const int W = here ? a.V : 0;
  load_row<TPR>(raw, x, t, W);
  const float end = row_end(x, t, W);
  const RowTargets r = row_targets<TPR>(a, row, here, t, idx, p, red[0]);
  for (int j = t; j <= a.K; j += TPR) {
    const int i = j < a.K ? idx[j] : r.label;
    u[j] = i >= 0 ? to_f32(x[i]) : 0.f;
  }
  float m, logst, logs1;
  if (a.stats_in) {
    m = here ? a.stats_in[row * 3] : 0.f;
    logst = here ? a.stats_in[row * 3 + 1] : 0.f;
    logs1 = here ? a.stats_in[row * 3 + 2] : 0.f;
  } else {
    m = end;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float v[V];
      vec<T>::unpack(raw[i], v);
#pragma unroll
      for (int k = 0; k < V; ++k) m = fmaxf(m, v[k]);
    }
    m = group_reduce<TPR>(m, op_max(), red[2]);
#pragma unroll
    for (int i = 0; i < NV; ++i) opaque_vec(raw[i]);
    const bool second = a.tau != 1.f && (a.stats || a.alpha < 1.f);
    const Expo et(m, kLog2e / a.tau), e1(m, kLog2e);
    float st = 0.f, s1 = 0.f;
    auto sums = [&](auto mode) {
      constexpr int MODE = decltype(mode)::value;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float v[V];
        vec<T>::unpack(raw[i], v);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float e = et(v[k]);
          st += e;
          if (MODE == SQUARE) s1 = __builtin_fmaf(e, e, s1);
          if (MODE == BOTH) s1 += e1(v[k]);
        }
        __builtin_amdgcn_sched_barrier(0);             // (one vector unpacked at a time)
      }
      const float e = et(end);
      st += e;
      if (MODE == SQUARE) s1 = __builtin_fmaf(e, e, s1);
      if (MODE == BOTH) s1 += e1(end);
    };
    const int mode = expo_mode(a.tau, second);
    if (mode == ONE) sums(std::integral_constant<int, ONE>());
    else if (mode == SQUARE) sums(std::integral_constant<int, SQUARE>());
    else sums(std::integral_constant<int, BOTH>());
    logst = et.log_sum(group_reduce<TPR>(st, op_sum(), red[3]));
    logs1 = logst;
    if (a.tau != 1.f) {
      logs1 = 0.f;
      if (second) {
        s1 = group_reduce<TPR>(s1, op_sum(), red[4]);
        logs1 = mode == SQUARE ? logf(s1) - 2.f * et.off * 0.6931471805599453f : e1.log_sum(s1);
      }
    }
    if (a.stats && here && t == 0) {
      a.stats[row * 3] = m;
      a.stats[row * 3 + 1] = logst;
      a.stats[row * 3 + 2] = logs1;
    }
  }
  if (a.loss) {
    const float loss = row_loss<TPR>(a, r, t, idx, p, u, m, logst, logs1, red[5]);
    // (the label's logit is in the LDS of the thread that fetched it)
    if (here && t == a.K % TPR) a.loss[row] = loss;
  }
  if (!a.dx) return;
  T* dx = (T*)a.dx + row * a.ldd;
  RowGrad g = {};
  g.zero = true;
  if (here) g = row_grad(a, r, row, m, logst, logs1);
#pragma unroll
  for (int i = 0; i < NV; ++i) opaque_vec(raw[i]);
  // (dx may be x: every logit that is fetched by its place has been)
  if constexpr (TPR > 64) __syncthreads();
  if (here)
    each_grad(g, [&](auto f) {
      store_row<TPR, T, NV>(dx, t, a.V, [&](int i, float (&v)[V]) {
        vec<T>::unpack(raw[i], v);
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = f(v[k]);
      });
      if (has_end<T>(t, a.V)) from_f32(dx[end_place<T>(t, a.V)], f(end));
    });
  // the elements that the teacher's entries and the label change, behind the stores above
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if constexpr (TPR > 64) __syncthreads();
  else wave_lds();
  if (!here || g.zero) return;
  for (int j = t; j <= a.K; j += TPR) {
    const int i = j < a.K ? idx[j] : r.label;
    if (i >= 0) from_f32(dx[i], entry_grad(a, g, r, i, u[j], idx, p));
  }
}

// A chunk's maximum and sums, and the logits at the entries that lie in it.
template <typename T>
__global__ void __launch_bounds__(256) k_distill_part(DistillArgs a) {
  constexpr int V = vec<T>::N;
  __shared__ float red[3][4];
  const int64_t row = blockIdx.x / a.chunks;
  const int ch = blockIdx.x % a.chunks, t = threadIdx.x, lo = ch * kChunkVecs * 256 * V;
  const T* x = (const T*)a.x + row * a.ldx;
  u32x4 raw[kChunkVecs];
  load_row<256>(raw, x, ch * kChunkVecs * 256 + t, a.V);
  const float end = row_end(x, t, ch + 1 == a.chunks ? a.V : 0);
  for (int j = t; j <= a.K; j += 256) {
    const int i = j < a.K ? a.index[row * a.K + j] : a.label ? a.label[row] : -1;
    if (i >= lo && i < a.V && i < lo + kChunkVecs * 256 * V) a.ent[row * (a.K + 1) + j] = to_f32(x[i]);
  }
  float m = end;
#pragma unroll
  for (int i = 0; i < kChunkVecs; ++i) {
    float v[V];
    vec<T>::unpack(raw[i], v);
#pragma unroll
    for (int k = 0; k < V; ++k) m = fmaxf(m, v[k]);
  }
  m = group_reduce<256>(m, op_max(), red[0]);
  float st = 0.f, s1 = 0.f;
  // (a chunk of -inf alone has the sums 0; one whose maximum is +inf, or with NaN, NaN)
  const float m0 = m > -INFINITY ? m : 0.f;
  const Expo et(m0, kLog2e / a.tau), e1(m0, kLog2e);
#pragma unroll
  for (int i = 0; i < kChunkVecs; ++i) {
    float v[V];
    vec<T>::unpack(raw[i], v);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      st += et(v[k]);
      if (a.tau != 1.f) s1 += e1(v[k]);
    }
  }
  st += et(end);
  if (a.tau != 1.f) s1 += e1(end);
  st = group_reduce<256>(st, op_sum(), red[1]) * __builtin_amdgcn_exp2f(-et.off);
  s1 = a.tau == 1.f ? st : group_reduce<256>(s1, op_sum(), red[2]) * __builtin_amdgcn_exp2f(-e1.off);
  if (t == 0) {
    float* o = a.part + (size_t)blockIdx.x * 3;
    o[0] = m;
    o[1] = st;
    o[2] = s1;
  }
}

// The gradient of a chunk, with the row's sums from its chunks (or from stats_in); the first chunk's workgroup
// writes the loss and the statistics. Logits at entries come from `ent` where there is one (another chunk's gradient
// may already stand in their place), else from the chunk itself.
template <typename T>
__global__ void __launch_bounds__(256) k_distill_chunk(DistillArgs a) {
  constexpr int V = vec<T>::N;
  __shared__ float red[3][16];
  __shared__ int idx[kEntries + 1];
  __shared__ float p[kEntries + 1], u[kEntries + 1];
  // without a gradient there is one workgroup to a row
  const int per = a.dx ? a.chunks : 1;
  const int64_t row = blockIdx.x / per;
  const int ch = blockIdx.x % per, t = threadIdx.x, lo = ch * kChunkVecs * 256 * V, hi = lo + kChunkVecs * 256 * V;
  const T* x = (const T*)a.x + row * a.ldx;
  u32x4 raw[kChunkVecs];
  float end = 0.f;
  if (a.dx) {
    load_row<256>(raw, x, ch * kChunkVecs * 256 + t, a.V);
    end = row_end(x, t, ch + 1 == a.chunks ? a.V : 0);
  }
  // the chunks' sums joined by every wave for itself, 64 at a time; the first loads go out ahead of the barriers below
  const float* q = a.part + (size_t)row * a.chunks * 3;
  const int l = t & 63;
  float m, logst, logs1, q0[3] = {-INFINITY, 0.f, 0.f};
  if (a.stats_in) {
    m = a.stats_in[row * 3];
    logst = a.stats_in[row * 3 + 1];
    logs1 = a.stats_in[row * 3 + 2];
  } else if (l < a.chunks) {
    q0[0] = q[3 * l], q0[1] = q[3 * l + 1], q0[2] = q[3 * l + 2];
  }
  const RowTargets r = row_targets<256>(a, row, true, t, idx, p, red[0]);
  if (!a.stats_in) {
    m = fmaxf(-INFINITY, q0[0]);                       // (of a chunk of NaN alone: -inf)
    for (int i = l + 64; i < a.chunks; i += 64) m = fmaxf(m, q[3 * i]);
    m = lanes<64>(m, op_max());
    float st = 0.f, s1 = 0.f;
    for (int i = l; i < a.chunks; i += 64) {
      const float mi = i == l ? q0[0] : q[3 * i], vt = i == l ? q0[1] : q[3 * i + 1], v1 = i == l ? q0[2] : q[3 * i + 2];
      // (nothing to take from a chunk of -inf, unless it holds NaN or all chunks are like it)
      if (mi == -INFINITY && m > -INFINITY) {
        st += vt;
        s1 += v1;
        continue;
      }
      st += vt * __builtin_amdgcn_exp2f((mi - m) * (kLog2e / a.tau));
      s1 += v1 * __builtin_amdgcn_exp2f((mi - m) * kLog2e);
    }
    logst = logf(lanes<64>(st, op_sum()));
    logs1 = logf(lanes<64>(s1, op_sum()));
  }
  for (int j = t; j <= a.K; j += 256) {
    const int i = j < a.K ? idx[j] : r.label;
    u[j] = i < 0 ? 0.f : a.ent ? a.ent[row * (a.K + 1) + j] : i >= lo && i < hi ? to_f32(x[i]) : 0.f;
  }
  auto row_out = [&] {
    if (ch != 0) return;
    if (a.stats && t == 0) {
      a.stats[row * 3] = m;
      a.stats[row * 3 + 1] = logst;
      a.stats[row * 3 + 2] = logs1;
    }
    if (a.loss) {
      const float loss = row_loss<256>(a, r, t, idx, p, u, m, logst, logs1, red[2]);
      if (t == a.K % 256) a.loss[row] = loss;
    }
  };
  if (!a.dx) return row_out();
  T* dx = (T*)a.dx + row * a.ldd;
  const RowGrad g = row_grad(a, r, row, m, logst, logs1);
  __syncthreads();                                     // (every element of the chunk that is fetched by place has been)
  each_grad(g, [&](auto f) {
    store_row<256, T, kChunkVecs>(dx, ch * kChunkVecs * 256 + t, a.V, [&](int i, float (&v)[V]) {
      vec<T>::unpack(raw[i], v);
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = f(v[k]);
    });
    if (ch + 1 == a.chunks && has_end<T>(t, a.V)) from_f32(dx[end_place<T>(t, a.V)], f(end));
  });
  row_out();
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (g.zero) return;
  for (int j = t; j <= a.K; j += 256) {
    const int i = j < a.K ? idx[j] : r.label;
    if (i >= lo && i < hi) from_f32(dx[i], entry_grad(a, g, r, i, u[j], idx, p));
  }
}

namespace {

int distill_vecs(const slstm_distill_dims* d) { return d->type == SLSTM_F32 ? (d->V + 3) / 4 : (d->V + 7) / 8; }
int distill_chunks(const slstm_distill_dims* d) { return (distill_vecs(d) + kChunkVecs * 256 - 1) / (kChunkVecs * 256); }
bool distill_ok(const slstm_distill_dims* d) {
  return d && d->rows >= 0 && d->rows <= 0x7fffffff && d->V >= 1 && d->V <= (1 << 22) && d->K >= 1 && d->K <= kEntries &&
         (d->type == SLSTM_F32 || d->type == SLSTM_BF16) && d->tau >= 1e-6f && d->tau <= 1e6f && d->alpha >= 0.f &&
         d->alpha <= 1.f && stride_ok(d->ld_logits, d->V) && stride_ok(d->ld_dlogits, d->V);
}
// Whole rows in registers hold up to 8192 vectors; rows of four chunks or more are cut where there are not two
// of them for every compute unit.
bool distill_cut(const slstm_distill_dims* d) {
  return distill_vecs(d) > 8192 || (distill_chunks(d) >= 4 && d->rows < 512);
}

template <typename F>
void distill_dispatch(const slstm_distill_dims* d, F f) {
  // (many entries: at most eight rows' to a workgroup's LDS)
  const int n = d->K > 64 ? std::max(distill_vecs(d), 32) : distill_vecs(d);
#define DISTILL_CASE(T_, MOST_, TPR_, NV_) \
  if (n <= MOST_) return f(T_(), std::integral_constant<int, TPR_>(), std::integral_constant<int, NV_>());
#define DISTILL_TYPE(T_) \
  DISTILL_CASE(T_, 8, 8, 1) DISTILL_CASE(T_, 16, 16, 1) DISTILL_CASE(T_, 32, 32, 1) DISTILL_CASE(T_, 64, 64, 1) \
  DISTILL_CASE(T_, 128, 64, 2) DISTILL_CASE(T_, 256, 64, 4) DISTILL_CASE(T_, 1024, 256, 4) DISTILL_CASE(T_, 2048, 256, 8) \
  DISTILL_CASE(T_, 4096, 256, 16) DISTILL_CASE(T_, 8192, 512, 16)
  if (d->type == SLSTM_F32) {
    DISTILL_TYPE(float)
  } else {
    DISTILL_TYPE(bf16_t)
  }
#undef DISTILL_TYPE
#undef DISTILL_CASE
}

size_t distill_part_bytes(const slstm_distill_dims* d) { return ((size_t)d->rows * distill_chunks(d) * 12 + 255) & ~(size_t)255; }

int distill_run(const slstm_distill_dims* d, DistillArgs a, void* workspace, size_t ws_bytes, hipStream_t st) {
  a.rows = (int)d->rows, a.V = d->V, a.K = d->K, a.tau = d->tau, a.alpha = d->alpha;
  a.ldx = row_stride(d->ld_logits, d->V), a.ldd = row_stride(d->ld_dlogits, d->V);
  a.chunks = distill_chunks(d);
  if (a.dx == a.x && a.ldx != a.ldd) return SLSTM_EINVAL;
  const bool cut = distill_cut(d);
  if (cut && !a.stats_in) {
    if (!workspace || ((uintptr_t)workspace & 3u)) return SLSTM_EINVAL;
    if (ws_bytes < stacklstm_distill_workspace_bytes(d)) return SLSTM_EWORKSPACE;
    a.part = (float*)workspace;
    a.ent = (float*)((char*)workspace + distill_part_bytes(d));
  }
  // rows r0 .. r0 + n
  auto rows = [&](auto t, int64_t r0, int64_t n) {
    typedef decltype(t) T;
    DistillArgs p = a;
    p.rows = (int)n;
    p.x = offset((const T*)a.x, r0 * a.ldx), p.dx = offset((T*)a.dx, r0 * a.ldd);
    p.index = a.index + r0 * a.K, p.value = a.value + r0 * a.K, p.label = offset(a.label, r0);
    p.grad = offset(a.grad, r0), p.stats_in = offset(a.stats_in, r0 * 3);
    p.loss = offset(a.loss, r0), p.stats = offset(a.stats, r0 * 3);
    p.part = offset(a.part, r0 * a.chunks * 3), p.ent = offset(a.ent, r0 * (a.K + 1));
    return p;
  };
  if (!cut) {
    distill_dispatch(d, [&](auto t, auto tpr, auto nv) {
      constexpr int TPR = decltype(tpr)::value, RPB = distill_rows(TPR);
      in_pieces(d->rows, kMostGroups * RPB, [&](int64_t r0, int64_t n) {
        hipLaunchKernelGGL((k_distill_rows<decltype(t), TPR, decltype(nv)::value>), dim3((unsigned)((n + RPB - 1) / RPB)),
                           dim3(distill_threads(TPR)), (size_t)RPB * 3 * (d->K + 1) * 4, st, rows(t, r0, n));
      });
    });
  } else {
    auto run = [&](auto t) {
      typedef decltype(t) T;
      in_pieces(d->rows, kMostGroups / a.chunks, [&](int64_t r0, int64_t n) {
        const dim3 all((unsigned)(n * a.chunks));
        const DistillArgs p = rows(t, r0, n);
        if (!a.stats_in) hipLaunchKernelGGL(k_distill_part<T>, all, dim3(256), 0, st, p);
        hipLaunchKernelGGL(k_distill_chunk<T>, a.dx ? all : dim3((unsigned)n), dim3(256), 0, st, p);
      });
    };
    if (d->type == SLSTM_F32) run(float());
    else run(bf16_t());
  }
  return hipGetLastError() == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
}

}  // namespace

extern "C" size_t stacklstm_distill_workspace_bytes(const slstm_distill_dims* d) {
  if (!distill_ok(d)) return 0;
  return distill_cut(d) && d->rows ? distill_part_bytes(d) + (size_t)d->rows * (d->K + 1) * 4 : 4;
}

extern "C" int stacklstm_distill_fwd(const slstm_distill_dims* d, const void* logits, const int32_t* index, const float* value,
                                     const int32_t* label, float* loss, float* stats, void* workspace, size_t ws_bytes,
                                     void* stream) {
  if (!distill_ok(d)) return SLSTM_EINVAL;
  if (d->rows == 0) return SLSTM_OK;
  if (!logits || !index || !value || !loss) return SLSTM_EINVAL;
  DistillArgs a = {};
  a.x = logits, a.index = index, a.value = value, a.label = label, a.loss = loss, a.stats = stats;
  return distill_run(d, a, workspace, ws_bytes, as_stream(stream));
}

extern "C" int stacklstm_distill_bwd(const slstm_distill_dims* d, const void* logits, const int32_t* index, const float* value,
                                     const int32_t* label, const float* stats, const float* grad, void* dlogits, void* stream) {
  if (!distill_ok(d)) return SLSTM_EINVAL;
  if (d->rows == 0) return SLSTM_OK;
  if (!logits || !index || !value || !stats || !dlogits) return SLSTM_EINVAL;
  DistillArgs a = {};
  a.x = logits, a.index = index, a.value = value, a.label = label, a.stats_in = stats, a.grad = grad, a.dx = dlogits;
  return distill_run(d, a, nullptr, 0, as_stream(stream));
}

extern "C" int stacklstm_distill_step(const slstm_distill_dims* d, const void* logits, const int32_t* index, const float* value,
                                      const int32_t* label, const float* grad, float* loss, void* dlogits, void* workspace,
                                      size_t ws_bytes, void* stream) {
  if (!distill_ok(d)) return SLSTM_EINVAL;
  if (d->rows == 0) return SLSTM_OK;
  if (!logits || !index || !value || !loss || !dlogits) return SLSTM_EINVAL;
  DistillArgs a = {};
  a.x = logits, a.index = index, a.value = value, a.label = label, a.grad = grad, a.loss = loss, a.dx = dlogits;
  return distill_run(d, a, workspace, ws_bytes, as_stream(stream));
}
