// Log probabilities of given tokens, entropy and best tokens of rows of logits, and their gradient.
//   t = x - m,  s = sum e^t,  logp = t[token] - log s,  H = log s - sum(e^t t) / s
//   dx = sum_g a_g onehot(token_g) - q (A + dH (t - (log s - H))),  q = e^t / s, A the sum of the a_g that count
// Bound by memory: the logits are read once and their gradient is written once. A row waits in registers (of a few lanes up to
// a workgroup of 512 threads) between its sums, its best tokens and its gradient, in its own type. The given tokens change a few
// elements: they go out in a second store to those elements, behind the first ones' acknowledgement.
// Best tokens: every thread has its largest logit from the maximum of the row; the N-th largest of those is a bound that at least N
// tokens reach and few others do. It is found bit by bit with ballots (its low bits are left away: a lower bound is one too).
// What reaches it goes to a list in LDS and is ranked there by whole keys (ordered bits of the logit, then the lower token); where
// equal logits make the list too long, the N best are taken one after the other.
// Rows that are too long for that, or too few of them to fill the chip, are cut into chunks: k_logprob_part leaves each chunk's
// maximum, sums and best tokens, k_logprob_join joins them, k_logprob_chunk writes a chunk's gradient.
// 4096 x 32000 bf16 with the gradient 101 us (5.2 TB/s); 1024 x 64001 bf16 with the 64 best 50 us (2.6 TB/s: load, sums and selection of a
// row follow one another, two rows to a compute unit); 512 x 83 fp32 with the 8 best 4.7; 4 x 131071 fp32 with the 10 best, in chunks,
// 6.0 + 4.2 us (waits, one after the other).
#include <algorithm>

#include "../../../include/stacklstm_layers.h"
#include "../head/head.h"

namespace {

typedef unsigned long long u64;
constexpr int kMost = 64;                              // given and best tokens of a row at most
constexpr int kChunkVecs = 4;                          // vectors a thread in a chunk of 256 threads

struct LogArgs {
  int rows, V, G, N, chunks;
  const void* x;
  void* dx;                                            // NULL: no gradient
  int64_t ldx, ldd;
  const uint8_t* legal;
  const int32_t* token;
  const float *dlogp, *dent, *stats_in;                // each may be NULL; stats_in: m, log s and H are known
  float *logp, *entropy, *value, *stats;               // each may be NULL
  int32_t* index;
  float* part;                                         // chunks: [rows][chunks][3]
  u64* cand;                                           // chunks: [rows][chunks][N]
};

constexpr int row_threads(int tpr) { return tpr <= 64 ? 256 : tpr; }
constexpr int row_count(int tpr) { return tpr <= 64 ? 256 / tpr : 1; }

// Bits in the order of the floats (-0 as 0), and back.
__device__ __forceinline__ uint32_t order_bits(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_order(uint32_t o) {
  return __uint_as_float(o ^ ((uint32_t)~((int32_t)o >> 31) | 0x80000000u));
}
// 0: none (-inf and NaN)
__device__ __forceinline__ u64 make_key(float x, uint32_t place) {
  return x > -INFINITY ? (u64)order_bits(x) << 32 | (0xffffffffu - place) : 0;
}
__device__ __forceinline__ float key_value(u64 k) { return from_order((uint32_t)(k >> 32)); }
__device__ __forceinline__ int key_place(u64 k) { return (int)(0xffffffffu - (uint32_t)k); }

// Vector i of a row (its whole vectors only) with -inf where a token is not allowed.
template <typename T>
__device__ __forceinline__ u32x4 allow(u32x4 raw, const uint8_t* legal, int i) {
  constexpr int V = vec<T>::N;
  typedef uint32_t u32_any __attribute__((aligned(1)));
#pragma unroll
  for (int q = 0; q < V / 4; ++q) {
    const uint32_t w = *(const u32_any*)(legal + i * V + 4 * q);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool ok = (w >> (8 * k)) & 0xffu;
      if constexpr (V == 4) {
        raw[k] = ok ? raw[k] : 0xff800000u;
      } else {
        const int at = 2 * q + k / 2;
        raw[at] = ok ? raw[at] : k & 1 ? (raw[at] & 0xffffu) | 0xff800000u : (raw[at] & 0xffff0000u) | 0xff80u;
      }
    }
  }
  return raw;
}
// load_row and row_end of a row's logits from vector c0 on; last: the row's end is the caller's too.
template <int STEP, typename T, int NV>
__device__ __forceinline__ void load_logits(u32x4 (&raw)[NV], float& end, const T* x, const uint8_t* legal, int c0, int t, int W, bool last) {
  load_row<STEP>(raw, x, c0, W);
  const int we = last ? W : 0;
  end = row_end(x, t, we);
  if (!legal) return;
  if (has_end<T>(t, we) && !legal[end_place<T>(t, we)]) end = -INFINITY;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (c0 + i * STEP < W / vec<T>::N) raw[i] = allow<T>(raw[i], legal, c0 + i * STEP);
    __builtin_amdgcn_sched_barrier(0);                 // (one vector's bytes at a time, as below)
  }
}

// A product that is 0 where a factor is, whatever the other (an infinity or NaN): v_mul_legacy_f32.
extern "C" __device__ float slstm_mul_zero(float a, float b) __asm("llvm.amdgcn.fmul.legacy");
__device__ __forceinline__ float mul_zero(float a, float b) { return slstm_mul_zero(a, b); }
// Sums of e^t and e^t t, t = x - m first: the largest logit's e is 1 and a lone token's logp 0 (with x k - m k in one step, k log2 e,
// it is 2^-25 off), and no m is too far from 0. The product of a vanished e is 0 whatever t is.
struct Sums {
  float s, q;
  __device__ __forceinline__ void add(float m, float x) {
    const float t = x - m, e = __builtin_amdgcn_exp2f(t * kLog2e);
    s += e;
    q += mul_zero(e, t);
  }
};

// ----- given tokens

// Token g of a row: its place, kAbsent where it is not there, kBarred where it is not allowed.
enum { kAbsent = -1, kBarred = -2 };
__device__ __forceinline__ int given(const LogArgs& a, int64_t row, int g) {
  const int i = a.token[row * a.G + g];
  if (i < 0 || i >= a.V) return kAbsent;
  return a.legal && !a.legal[row * a.V + i] ? kBarred : i;
}
__device__ __forceinline__ float log_prob(int place, float x, float m, float logs) {
  // (a logit of -inf in a row with NaN or +inf: NaN, as its others are)
  const bool none = place == kBarred || (x == -INFINITY && logs == logs);
  return place == kAbsent ? 0.f : none ? -INFINITY : (x - m) - logs;
}
// Gradient of a row's elements: -e (c1 + c2 t), and what its tokens add.
struct RowGrad {
  float m, c1, c2;
  bool zero;
  __device__ __forceinline__ float operator()(float x) const {
    const float t = x - m;
    return -mul_zero(__builtin_amdgcn_exp2f(t * kLog2e), __builtin_fmaf(c2, t, c1));
  }
};
// A: the sum of the tokens' weights that count, any: whether one of them is not 0.
__device__ __forceinline__ RowGrad row_grad(float dent, float A, bool any, float m, float logs, float H) {
  RowGrad g;
  g.zero = !any && dent == 0.f;
  g.m = m > -INFINITY ? m : 0.f;
  const float c = __builtin_amdgcn_exp2f(-logs * kLog2e);
  g.c1 = c * (A - dent * (logs - H));
  g.c2 = c * dent;
  return g;
}

// ----- best tokens, by NT threads (64: a wave)

template <int NT>
struct TopLds {
  static constexpr int kList = NT == 64 ? 512 : 1024;
  u64 list[kList], red[NT / 64];
  uint32_t mine[NT];
  int count;
};
template <int NT>
__device__ __forceinline__ void meet() {
  if constexpr (NT > 64) __syncthreads();
  else wave_lds();
}
// A value that the N-th largest of the threads' reaches (0: fewer are not 0), the same in every thread. Starts the list.
template <int NT>
__device__ __forceinline__ uint32_t top_bound(uint32_t mine, int N, int t, TopLds<NT>& s) {
  constexpr int M = NT / 64;
  uint32_t v[M];
  if (t == 0) s.count = 0;
  v[0] = mine;
  if constexpr (M > 1) s.mine[t] = mine;
  meet<NT>();
  if constexpr (M > 1) {
#pragma unroll
    for (int i = 0; i < M; ++i) v[i] = s.mine[64 * i + (t & 63)];
  }
  uint32_t b = 0;
  for (uint32_t bit = 0x80000000u; bit >= 0x400u; bit >>= 1) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) n += __popcll(__ballot(v[i] >= (b | bit)));
    if (n >= N) b |= bit;
  }
  return b;
}
template <int NT>
__device__ __forceinline__ void top_put(u64 key, TopLds<NT>& s) {
  const int i = atomicAdd(&s.count, 1);
  if (i < TopLds<NT>::kList) s.list[i] = key;
}
// emit(n, key) for the N best of the listed keys (all different), n their rank, and key 0 for the places past them, each by some
// thread. each(f): calls f with every key of this thread, listed or not, for lists that did not fit.
template <int NT, typename Each, typename Emit>
__device__ __forceinline__ void top_rank(int N, int t, TopLds<NT>& s, Each each, Emit emit) {
  meet<NT>();
  const int n = s.count;
  if (n <= TopLds<NT>::kList) {
    for (int i = t; i < n; i += NT) {
      const u64 k = s.list[i];
      int above = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) above += s.list[j] > k;
      if (above < N) emit(above, k);
    }
    for (int i = n + t; i < N; i += NT) emit(i, (u64)0);
    return;
  }
  u64 last = ~(u64)0;
  for (int r = 0; r < N; ++r) {
    u64 best = 0;
    each([&](u64 k) {
      if (k < last && k > best) best = k;
    });
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const u64 o = __shfl_xor(best, d);
      best = o > best ? o : best;
    }
    if constexpr (NT > 64) {
      if ((t & 63) == 0) s.red[t >> 6] = best;
      __syncthreads();
      for (int w = 0; w < NT / 64; ++w) best = s.red[w] > best ? s.red[w] : best;
      __syncthreads();
    }
    if (t == 0) emit(r, best);
    last = best;                                       // (every thread has the same; 0: none is left)
  }
}
// The keys of a thread's vectors c0, c0 + NT, .. and of its share of the row's end that reach the bound, and their ranks.
template <typename T, int NT, int NV, typename Emit>
__device__ __forceinline__ void top_row(u32x4 (&raw)[NV], float end, float mine, const T* x, const uint8_t* legal, int c0, int t, int W,
                                        int N, TopLds<NT>& s, Emit emit) {
  constexpr int V = vec<T>::N;
  const uint32_t b = top_bound<NT>(mine > -INFINITY ? order_bits(mine) : 0u, N, t, s);
  // (at or below the order of -inf: every number)
  const float xb = b > 0x007fffffu ? from_order(b) : -INFINITY;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    opaque_vec(raw[i]);
    float v[V];
    vec<T>::unpack(raw[i], v);
    float most = v[0];
#pragma unroll
    for (int k = 1; k < V; ++k) most = fmaxf(most, v[k]);
    if (most >= xb) {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (v[k] >= xb && v[k] > -INFINITY) top_put<NT>(make_key(v[k], (c0 + i * NT) * V + k), s);
    }
    __builtin_amdgcn_sched_barrier(0);                 // (one vector unpacked at a time)
  }
  if (end >= xb && end > -INFINITY) top_put<NT>(make_key(end, end_place<T>(t, W)), s);
  top_rank<NT>(N, t, s, [&](auto f) {
    f(make_key(end, end_place<T>(t, W)));
#pragma unroll 1
    for (int i = 0; i < NV; ++i) {
      // (read again: a loop over registers would take them all at once)
      u32x4 w[1];
      float v[V], e;
      load_logits<NT, T>(w, e, x, legal, c0 + i * NT, t, W, false);
      vec<T>::unpack(w[0], v);
#pragma unroll
      for (int k = 0; k < V; ++k) f(make_key(v[k], (c0 + i * NT) * V + k));
    }
  }, emit);
}
// What place n of a row's best tokens holds.
__device__ __forceinline__ void top_out(const LogArgs& a, int64_t row, int n, u64 key, float m, float logs) {
  a.index[row * a.N + n] = key ? key_place(key) : -1;
  a.value[row * a.N + n] = key ? (key_value(key) - m) - logs : -INFINITY;
}

}  // namespace

// Whole rows, TPR threads to each, NV vectors in a thread. TOP: best tokens are asked for (then TPR >= 64).
template <typename T, int TPR, int NV, bool TOP>
__global__ void __launch_bounds__(row_threads(TPR), NV == 16 ? 4 : 1) k_logprob_rows(LogArgs a) {
  constexpr int V = vec<T>::N, RPB = row_count(TPR), NT = TPR < 64 ? 64 : TPR;
  __shared__ float red[5][16];
  __shared__ TopLds<NT> top[TOP ? RPB : 1];
  extern __shared__ int lds[];                         // [RPB][3][G]: places, logits, weights of the given tokens
  const int t = threadIdx.x & (TPR - 1), sub = RPB > 1 ? threadIdx.x / TPR : 0;
  const int64_t row = (int64_t)blockIdx.x * RPB + sub;
  const bool here = row < a.rows;
  const T* x = (const T*)a.x + row * a.ldx;
  const uint8_t* legal = a.legal ? a.legal + row * a.V : nullptr;
  int* idx = lds + sub * 3 * a.G;
  float *u = (float*)(idx + a.G), *wt = u + a.G;
  const int W = here ? a.V : 0;
  u32x4 raw[NV];
  float end;
  load_logits<TPR, T>(raw, end, x, legal, t, t, W, true);
  float A = 0.f, some = 0.f;
  for (int g = t; g < a.G; g += TPR) {
    float v = 0.f, w = 0.f;
    const int i = here ? given(a, row, g) : kAbsent;
    if (i >= 0) {
      v = to_f32(x[i]);
      if (a.dx && a.dlogp) w = a.dlogp[row * a.G + g];
    }
    idx[g] = i, u[g] = v, wt[g] = w;
    A += w;
    some = fmaxf(some, w != w ? 1.f : fabsf(w));
  }
  float m, logs, H;
  if (a.stats_in) {
    m = here ? a.stats_in[row * 3] : 0.f;
    logs = here ? a.stats_in[row * 3 + 1] : 0.f;
    H = here ? a.stats_in[row * 3 + 2] : 0.f;
  } else {
    float mine = end;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float v[V];
      opaque_vec(raw[i]);
      vec<T>::unpack(raw[i], v);
#pragma unroll
      for (int k = 0; k < V; ++k) mine = fmaxf(mine, v[k]);
      __builtin_amdgcn_sched_barrier(0);
    }
    m = group_reduce<TPR>(mine, op_max(), red[0]);
    const float m0 = m > -INFINITY ? m : 0.f;
    Sums z = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float v[V];
      opaque_vec(raw[i]);                              // (here, not ahead of the loop: unpacked before, all of them take 100 registers more)
      vec<T>::unpack(raw[i], v);
#pragma unroll
      for (int k = 0; k < V; ++k) z.add(m0, v[k]);
      // (added up here: the compiler kept all of the second sum's terms for behind the first one's barrier)
      asm volatile("" : "+v"(z.q));
      __builtin_amdgcn_sched_barrier(0);               // (one vector unpacked at a time)
    }
    z.add(m0, end);
    const float s = group_reduce<TPR>(z.s, op_sum(), red[1]), q = group_reduce<TPR>(z.q, op_sum(), red[2]);
    logs = logf(s);
    H = s == 0.f ? 0.f : logs - q / s;
    if (here && t == 0) {
      if (a.entropy) a.entropy[row] = H;
      if (a.stats) a.stats[row * 3] = m, a.stats[row * 3 + 1] = logs, a.stats[row * 3 + 2] = H;
    }
    // (a token's place and logit are in the LDS of the thread that fetched them)
    if (here && a.logp)
      for (int g = t; g < a.G; g += TPR) a.logp[row * a.G + g] = log_prob(idx[g], u[g], m, logs);
    if constexpr (TOP) {
      if (here) top_row<T, NT, NV>(raw, end, mine, x, legal, t, t, W, a.N, top[sub], [&](int n, u64 key) { top_out(a, row, n, key, m, logs); });
    }
  }
  if (!a.dx) return;
  A = group_reduce<TPR>(A, op_sum(), red[3]);
  some = group_reduce<TPR>(some, op_max(), red[4]);
  T* dx = (T*)a.dx + row * a.ldd;
  const RowGrad g = row_grad(here && a.dent ? a.dent[row] : 0.f, A, some != 0.f, m, logs, H);
  // (dx may be x: every logit that is fetched by its place, or again, has been)
  if constexpr (TPR > 64) __syncthreads();
  if (here) {
    auto put = [&](auto f) {
      store_row<TPR, T, NV>(dx, t, a.V, [&](int i, float (&v)[V]) {
        opaque_vec(raw[i]);
        vec<T>::unpack(raw[i], v);
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = f(v[k]);
      });
      if (has_end<T>(t, a.V)) from_f32(dx[end_place<T>(t, a.V)], f(end));
    };
    if (g.zero) put([](float) { return 0.f; });
    else put(g);
  }
  // the elements that the given tokens change, behind the stores above
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if constexpr (TPR > 64) __syncthreads();
  else wave_lds();
  if (!here || g.zero) return;
  for (int j = t; j < a.G; j += TPR) {
    const int i = idx[j];
    if (i < 0) continue;
    float v = 0.f;
    for (int k = 0; k < a.G; ++k) v += idx[k] == i ? wt[k] : 0.f;
    from_f32(dx[i], v + g(u[j]));
  }
}

// A chunk's maximum and sums (m, sum e^(x - m), sum e^(x - m) (x - m)), and its best tokens.
template <typename T, bool TOP>
__global__ void __launch_bounds__(256) k_logprob_part(LogArgs a) {
  constexpr int V = vec<T>::N;
  __shared__ float red[3][16];
  __shared__ TopLds<256> top;
  const int64_t row = blockIdx.x / a.chunks;
  const int ch = blockIdx.x % a.chunks, t = threadIdx.x, c0 = ch * kChunkVecs * 256 + t;
  const T* x = (const T*)a.x + row * a.ldx;
  const uint8_t* legal = a.legal ? a.legal + row * a.V : nullptr;
  u32x4 raw[kChunkVecs];
  float end;
  load_logits<256, T>(raw, end, x, legal, c0, t, a.V, ch + 1 == a.chunks);
  float mine = end;
#pragma unroll
  for (int i = 0; i < kChunkVecs; ++i) {
    float v[V];
    vec<T>::unpack(raw[i], v);
#pragma unroll
    for (int k = 0; k < V; ++k) mine = fmaxf(mine, v[k]);
  }
  const float m = group_reduce<256>(mine, op_max(), red[0]);
  const float m0 = m > -INFINITY ? m : 0.f;
  Sums z = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kChunkVecs; ++i) {
    float v[V];
    vec<T>::unpack(raw[i], v);
#pragma unroll
    for (int k = 0; k < V; ++k) z.add(m0, v[k]);
  }
  z.add(m0, end);
  const float s = group_reduce<256>(z.s, op_sum(), red[1]), q = group_reduce<256>(z.q, op_sum(), red[2]);
  if (t == 0) {
    float* o = a.part + (size_t)blockIdx.x * 3;
    o[0] = m;
    o[1] = s;
    o[2] = q;
  }
  if constexpr (TOP)
    top_row<T, 256, kChunkVecs>(raw, end, mine, x, legal, c0, t, a.V, a.N, top, [&](int n, u64 key) { a.cand[(size_t)blockIdx.x * a.N + n] = key; });
}

// A row's outputs from its chunks' parts.
template <typename T>
__global__ void __launch_bounds__(256) k_logprob_join(LogArgs a) {
  __shared__ TopLds<256> top;
  const int64_t row = blockIdx.x;
  const int t = threadIdx.x, l = t & 63;
  const T* x = (const T*)a.x + row * a.ldx;
  // by every wave for itself, 64 chunks at a time
  const float* p = a.part + (size_t)row * a.chunks * 3;
  float m = -INFINITY, s = 0.f, w = 0.f;
  for (int i = l; i < a.chunks; i += 64) m = fmaxf(m, p[3 * i]);
  m = lanes<64>(m, op_max());
  for (int i = l; i < a.chunks; i += 64) {
    const float mi = p[3 * i], si = p[3 * i + 1], wi = p[3 * i + 2];
    // (nothing to take from a chunk of -inf, unless it holds NaN)
    if (mi == -INFINITY) {
      s += si;
      continue;
    }
    const float d = mi - m, f = __builtin_amdgcn_exp2f(d * kLog2e);
    s += si * f;
    w += mul_zero(f, wi + si * d);
  }
  s = lanes<64>(s, op_sum());
  w = lanes<64>(w, op_sum());
  const float logs = logf(s), H = s == 0.f ? 0.f : logs - w / s;
  if (t == 0) {
    if (a.entropy) a.entropy[row] = H;
    if (a.stats) a.stats[row * 3] = m, a.stats[row * 3 + 1] = logs, a.stats[row * 3 + 2] = H;
  }
  if (a.logp && t < a.G) {
    const int i = given(a, row, t);
    a.logp[row * a.G + t] = log_prob(i, i >= 0 ? to_f32(x[i]) : 0.f, m, logs);
  }
  if (a.N == 0) return;
  const int n = a.chunks * a.N;
  const u64* cand = a.cand + (size_t)row * n;
  uint32_t mine = 0;
  for (int i = t; i < n; i += 256) mine = max(mine, (uint32_t)(cand[i] >> 32));
  const uint32_t b = top_bound<256>(mine, a.N, t, top);
  for (int i = t; i < n; i += 256) {
    const u64 k = cand[i];
    if (k && (uint32_t)(k >> 32) >= b) top_put<256>(k, top);
  }
  top_rank<256>(a.N, t, top, [&](auto f) {
    for (int i = t; i < n; i += 256) f(cand[i]);
  }, [&](int r, u64 key) { top_out(a, row, r, key, m, logs); });
}

// The gradient of a chunk, with the row's statistics known.
template <typename T>
__global__ void __launch_bounds__(256) k_logprob_chunk(LogArgs a) {
  constexpr int V = vec<T>::N;
  __shared__ int idx[kMost];
  __shared__ float u[kMost], wt[kMost];
  const int64_t row = blockIdx.x / a.chunks;
  const int ch = blockIdx.x % a.chunks, t = threadIdx.x, lo = ch * kChunkVecs * 256 * V, hi = lo + kChunkVecs * 256 * V;
  const T* x = (const T*)a.x + row * a.ldx;
  const uint8_t* legal = a.legal ? a.legal + row * a.V : nullptr;
  u32x4 raw[kChunkVecs];
  float end;
  load_logits<256, T>(raw, end, x, legal, ch * kChunkVecs * 256 + t, t, a.V, ch + 1 == a.chunks);
  const float m = a.stats_in[row * 3], logs = a.stats_in[row * 3 + 1], H = a.stats_in[row * 3 + 2];
  if (t < a.G) {
    const int i = given(a, row, t);
    idx[t] = i;
    wt[t] = i >= 0 && a.dlogp ? a.dlogp[row * a.G + t] : 0.f;
    u[t] = i >= lo && i < hi ? to_f32(x[i]) : 0.f;
  }
  __syncthreads();
  float A = 0.f;
  bool any = false;
  for (int g = 0; g < a.G; ++g) {
    A += wt[g];
    any |= wt[g] != 0.f;
  }
  T* dx = (T*)a.dx + row * a.ldd;
  const RowGrad g = row_grad(a.dent ? a.dent[row] : 0.f, A, any, m, logs, H);
  auto put = [&](auto f) {
    store_row<256, T, kChunkVecs>(dx, ch * kChunkVecs * 256 + t, a.V, [&](int i, float (&v)[V]) {
      vec<T>::unpack(raw[i], v);
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = f(v[k]);
    });
    if (ch + 1 == a.chunks && has_end<T>(t, a.V)) from_f32(dx[end_place<T>(t, a.V)], f(end));
  };
  if (g.zero) put([](float) { return 0.f; });
  else put(g);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (g.zero || t >= a.G) return;
  const int i = idx[t];
  if (i < lo || i >= hi) return;
  float v = 0.f;
  for (int k = 0; k < a.G; ++k) v += idx[k] == i ? wt[k] : 0.f;
  from_f32(dx[i], v + g(u[t]));
}

namespace {

int row_vecs(const slstm_logprob_dims* d) { return d->type == SLSTM_F32 ? (d->V + 3) / 4 : (d->V + 7) / 8; }
int row_chunks(const slstm_logprob_dims* d) { return (row_vecs(d) + kChunkVecs * 256 - 1) / (kChunkVecs * 256); }
bool logprob_ok(const slstm_logprob_dims* d) {
  return d && d->rows >= 0 && d->rows <= 0x7fffffff && d->V >= 1 && d->V <= (1 << 22) && d->G >= 0 && d->G <= kMost && d->N >= 0 &&
         d->N <= kMost && (d->type == SLSTM_F32 || d->type == SLSTM_BF16) && stride_ok(d->ld_logits, d->V) &&
         stride_ok(d->ld_dlogits, d->V);
}
// Whole rows in registers hold up to 8192 vectors. Shorter ones are cut where they are long, 16-bit (twice the work to a vector) and few. A call's
// us, cut and whole; outputs alone, with the 16 best, with the gradient: 64 x 64001 bf16 9.8, 9.4; 12.8, 16.4; 13.1, 15.5; of 200 rows 9.8, 9.7;
// 17.3, 16.7; 20.5, 17.2; of 400 13.4, 15.4; 24.6, 22.7; 32.6, 27.0. 64 x 32000 fp32 10.0, 7.2; 11.2, 9.9; 13.1, 8.2; of 400 rows 11.9, 11.0; 21.1, 16.9;
// 29.1, 17.8. 64 x 32000 bf16 10.1, 7.1; 11.5, 10.5; 13.3, 9.0.
bool logprob_cut(const slstm_logprob_dims* d) {
  return row_vecs(d) > 8192 || (d->type == SLSTM_BF16 && row_vecs(d) > 4096 && d->rows < 128);
}

template <typename F>
void logprob_dispatch(const slstm_logprob_dims* d, bool top, F f) {
  // (many given tokens: at most eight rows' to a workgroup's LDS; best tokens: a wave to a row at least)
  const int n = top ? std::max(row_vecs(d), 33) : d->G > 16 ? std::max(row_vecs(d), 17) : row_vecs(d);
#define LOGPROB_CASE(T_, MOST_, TPR_, NV_, TOP_) \
  if (n <= MOST_ && top == TOP_) \
    return f(T_(), std::integral_constant<int, TPR_>(), std::integral_constant<int, NV_>(), std::integral_constant<bool, TOP_>());
#define LOGPROB_WIDE(T_, TOP_) \
  LOGPROB_CASE(T_, 64, 64, 1, TOP_) LOGPROB_CASE(T_, 128, 64, 2, TOP_) LOGPROB_CASE(T_, 256, 64, 4, TOP_) \
  LOGPROB_CASE(T_, 1024, 256, 4, TOP_) LOGPROB_CASE(T_, 2048, 256, 8, TOP_) LOGPROB_CASE(T_, 4096, 256, 16, TOP_) \
  LOGPROB_CASE(T_, 8192, 512, 16, TOP_)
#define LOGPROB_TYPE(T_) \
  LOGPROB_CASE(T_, 8, 8, 1, false) LOGPROB_CASE(T_, 16, 16, 1, false) LOGPROB_CASE(T_, 32, 32, 1, false) \
  LOGPROB_WIDE(T_, false) LOGPROB_WIDE(T_, true)
  if (d->type == SLSTM_F32) {
    LOGPROB_TYPE(float)
  } else {
    LOGPROB_TYPE(bf16_t)
  }
#undef LOGPROB_TYPE
#undef LOGPROB_WIDE
#undef LOGPROB_CASE
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
size_t part_bytes(const slstm_logprob_dims* d) { return up256((size_t)d->rows * row_chunks(d) * 12); }
size_t stats_bytes(const slstm_logprob_dims* d) { return up256((size_t)d->rows * 12); }

int logprob_run(const slstm_logprob_dims* d, LogArgs a, void* workspace, size_t ws_bytes, hipStream_t st) {
  a.rows = (int)d->rows, a.V = d->V, a.G = d->G, a.N = a.stats_in ? 0 : d->N;
  a.ldx = row_stride(d->ld_logits, d->V), a.ldd = row_stride(d->ld_dlogits, d->V);
  a.chunks = row_chunks(d);
  if (a.dx == a.x && a.ldx != a.ldd) return SLSTM_EINVAL;
  const bool cut = logprob_cut(d), sums = !a.stats_in;
  if (cut && sums) {
    if (!workspace || ((uintptr_t)workspace & 15u)) return SLSTM_EINVAL;
    if (ws_bytes < stacklstm_logprob_workspace_bytes(d)) return SLSTM_EWORKSPACE;
    a.part = (float*)workspace;
    if (!a.stats) a.stats = (float*)((char*)workspace + part_bytes(d));
    a.cand = (u64*)((char*)workspace + part_bytes(d) + stats_bytes(d));
  }
  // rows r0 .. r0 + n
  auto rows = [&](auto t, int64_t r0, int64_t n) {
    typedef decltype(t) T;
    LogArgs p = a;
    p.rows = (int)n;
    p.x = offset((const T*)a.x, r0 * a.ldx), p.dx = offset((T*)a.dx, r0 * a.ldd);
    p.legal = offset(a.legal, r0 * a.V), p.token = offset(a.token, r0 * a.G);
    p.dlogp = offset(a.dlogp, r0 * a.G), p.dent = offset(a.dent, r0), p.stats_in = offset(a.stats_in, r0 * 3);
    p.logp = offset(a.logp, r0 * a.G), p.entropy = offset(a.entropy, r0), p.stats = offset(a.stats, r0 * 3);
    p.index = offset(a.index, r0 * a.N), p.value = offset(a.value, r0 * a.N);
    p.part = offset(a.part, r0 * a.chunks * 3), p.cand = offset(a.cand, r0 * a.chunks * a.N);
    return p;
  };
  if (!cut) {
    logprob_dispatch(d, a.N > 0, [&](auto t, auto tpr, auto nv, auto top) {
      constexpr int TPR = decltype(tpr)::value, RPB = row_count(TPR);
      in_pieces(d->rows, kMostGroups * RPB, [&](int64_t r0, int64_t n) {
        hipLaunchKernelGGL((k_logprob_rows<decltype(t), TPR, decltype(nv)::value, decltype(top)::value>),
                           dim3((unsigned)((n + RPB - 1) / RPB)), dim3(row_threads(TPR)), (size_t)RPB * 3 * d->G * 4, st, rows(t, r0, n));
      });
    });
  } else {
    auto run = [&](auto t) {
      typedef decltype(t) T;
      in_pieces(d->rows, kMostGroups / a.chunks, [&](int64_t r0, int64_t n) {
        const dim3 all((unsigned)(n * a.chunks));
        LogArgs p = rows(t, r0, n);
        if (sums) {
          if (a.N) hipLaunchKernelGGL((k_logprob_part<T, true>), all, dim3(256), 0, st, p);
          else hipLaunchKernelGGL((k_logprob_part<T, false>), all, dim3(256), 0, st, p);
          hipLaunchKernelGGL(k_logprob_join<T>, dim3((unsigned)n), dim3(256), 0, st, p);
          p.stats_in = p.stats;
        }
        if (a.dx) hipLaunchKernelGGL(k_logprob_chunk<T>, all, dim3(256), 0, st, p);
      });
    };
    if (d->type == SLSTM_F32) run(float());
    else run(bf16_t());
  }
  return hipGetLastError() == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
}
bool outputs_ok(const slstm_logprob_dims* d, const void* token, const void* logp, const void* index, const void* value) {
  return (d->G == 0 || (token && logp)) && (d->N == 0 || (index && value));
}

}  // namespace

extern "C" size_t stacklstm_logprob_workspace_bytes(const slstm_logprob_dims* d) {
  if (!logprob_ok(d)) return 0;
  if (!logprob_cut(d) || d->rows == 0) return 16;
  return part_bytes(d) + stats_bytes(d) + (size_t)d->rows * row_chunks(d) * d->N * 8;
}

extern "C" int stacklstm_logprob_fwd(const slstm_logprob_dims* d, const void* logits, const uint8_t* legal, const int32_t* token,
                                     float* logp, float* entropy, int32_t* index, float* value, float* stats, void* workspace,
                                     size_t ws_bytes, void* stream) {
  if (!logprob_ok(d)) return SLSTM_EINVAL;
  if (d->rows == 0) return SLSTM_OK;
  if (!logits || !outputs_ok(d, token, logp, index, value)) return SLSTM_EINVAL;
  LogArgs a = {};
  a.x = logits, a.legal = legal, a.token = token, a.logp = logp, a.entropy = entropy, a.index = index, a.value = value;
  a.stats = stats;
  return logprob_run(d, a, workspace, ws_bytes, as_stream(stream));
}

extern "C" int stacklstm_logprob_bwd(const slstm_logprob_dims* d, const void* logits, const uint8_t* legal, const int32_t* token,
                                     const float* stats, const float* dlogp, const float* dentropy, void* dlogits, void* stream) {
  if (!logprob_ok(d)) return SLSTM_EINVAL;
  if (d->rows == 0) return SLSTM_OK;
  if (!logits || (d->G && !token) || !stats || !dlogits) return SLSTM_EINVAL;
  LogArgs a = {};
  a.x = logits, a.legal = legal, a.token = token, a.stats_in = stats, a.dlogp = dlogp, a.dent = dentropy, a.dx = dlogits;
  return logprob_run(d, a, nullptr, 0, as_stream(stream));
}

extern "C" int stacklstm_logprob_step(const slstm_logprob_dims* d, const void* logits, const uint8_t* legal, const int32_t* token,
                                      const float* dlogp, const float* dentropy, float* logp, float* entropy, int32_t* index,
                                      float* value, void* dlogits, void* workspace, size_t ws_bytes, void* stream) {
  if (!logprob_ok(d)) return SLSTM_EINVAL;
  if (d->rows == 0) return SLSTM_OK;
  if (!logits || !outputs_ok(d, token, logp, index, value) || !dlogits) return SLSTM_EINVAL;
  LogArgs a = {};
  a.x = logits, a.legal = legal, a.token = token, a.dlogp = dlogp, a.dent = dentropy, a.logp = logp, a.entropy = entropy;
  a.index = index, a.value = value, a.dx = dlogits;
  return logprob_run(d, a, workspace, ws_bytes, as_stream(stream));
}
