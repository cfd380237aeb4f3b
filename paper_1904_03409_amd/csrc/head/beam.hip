// One step of a beam search: the K best of K x V continuations of every search, then the stacks of states
// copied to the beams that go on.
//   total = (x - lse(x)) + score, falling; ties to the lower place k V + v
// Selection is bound by one read of the logits. A row (beam) waits in registers between its softmax sums and its
// selection. What is chosen has to be exact, ties included, so totals are compared as whole keys (ordered bits of
// the total, then the place). To touch few elements with them: the row's threads form 64 groups; the K-th largest of
// the groups' largest elements is a bound that at least K elements reach and few others do. Those go to a list
// in LDS and are ranked there. Where equal logits or their layout make the list too long, the K best are
// taken one after the other.
// Rows that are too long for registers, or too few to fill the chip, are cut into chunks with a pass for the
// sums before (k_beam_part). Small vocabularies take one workgroup to a search (k_beam_small).
// 64 searches of 16 x 64001 bf16: rows 41 us (3.2 TB/s; vector units 43% busy, a quarter of the wave slots taken), k_beam_merge 4.8; 64
// of 8 x 83 f32 6.1; one of 4 x 131072 f32 in chunks 3.2 + 4.8 + 3.5 us. With more than 48 beams the bound is near the least group's
// largest and the list overflows on ordinary logits: k_beam_merge of 4 searches of 64 x 131072 takes 8 ms, the
// whole selection of 32 beams 0.16.
#include <algorithm>

#include "../../../include/stacklstm_head.h"
#include "head.h"

namespace {

typedef unsigned long long u64;
constexpr int kMaxBeams = 64, kList = 1024;
constexpr float kFar = -0x1p29f;                       // base-2 exponents below it are none of a row's sum
constexpr int kPartVecs = 4;                           // vectors a thread in a chunk of 256 threads
constexpr int kSmall = 8192;                           // totals of a search that fit one workgroup's LDS

struct BeamArgs {
  int B, K, V, eos, chunks;
  const void* x;
  int64_t ldx;
  const uint8_t *legal, *done;
  const float* score;
  float* part;                                         // [rows][chunks][2]: maximum, sum
  u64* cand;                                           // [rows][chunks][K] keys, place = token
  float* score_next;
  int32_t *parent, *token;
  uint8_t* done_next;
};

// Bits in the order of the floats (-0 as 0), and back.
__device__ __forceinline__ uint32_t order_bits(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_order(uint32_t o) {
  return __uint_as_float(o ^ ((uint32_t)~((int32_t)o >> 31) | 0x80000000u));
}
// 0: no continuation (-inf and NaN)
__device__ __forceinline__ u64 make_key(float total, uint32_t place) {
  return total > -INFINITY ? (u64)order_bits(total) << 32 | (0xffffffffu - place) : 0;
}
__device__ __forceinline__ float key_total(u64 k) { return from_order((uint32_t)(k >> 32)); }
__device__ __forceinline__ uint32_t key_place(u64 k) { return 0xffffffffu - (uint32_t)k; }

template <int N>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
  auto move = [](uint32_t v, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xf, 0xf, true);
  };
  if constexpr (N >= 2) v = max(v, move(v, std::integral_constant<int, 0xb1>()));
  if constexpr (N >= 4) v = max(v, move(v, std::integral_constant<int, 0x4e>()));
  if constexpr (N >= 8) v = max(v, move(v, std::integral_constant<int, 0x141>()));
  if constexpr (N >= 16) v = max(v, move(v, std::integral_constant<int, 0x140>()));
  if constexpr (N >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(r[0], r[1]);
  }
  if constexpr (N >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max(r[0], r[1]);
  }
  return v;
}

struct TopkLds {
  u64 list[kList], red[16];
  uint32_t grp[64];
  int count;
};

// The largest values of 64 groups of NT threads' (mine: this thread's, in order bits; 0: none), to LDS. A barrier follows.
template <int NT>
__device__ __forceinline__ void topk_groups(uint32_t mine, TopkLds& s) {
  constexpr int G = NT / 64;                           // threads of a group
  mine = lanes_max<G>(mine);
  const int t = threadIdx.x;
  if (t % G == 0) s.grp[t / G] = mine;
  if (t == 0) s.count = 0;
}
// The largest value that K of the groups reach (0: they have fewer), by every wave for itself.
__device__ __forceinline__ uint32_t topk_bound(int K, const TopkLds& s) {
  const uint32_t v = s.grp[threadIdx.x & 63];
  int reach = 0;
#pragma unroll
  for (int j = 0; j < 64; ++j) reach += (uint32_t)__builtin_amdgcn_readlane((int)v, j) >= v;
  return lanes_max<64>(reach >= K ? v : 0u);
}
__device__ __forceinline__ void topk_put(u64 key, TopkLds& s) {
  const int i = atomicAdd(&s.count, 1);
  if (i < kList) s.list[i] = key;
}
// emit(n, key) for the K best of the listed keys (all different), n their rank, and key 0 for the places past them, each by some
// thread. each(f): calls f with every key of this thread, listed or not, for lists that did not fit.
template <int NT, typename Each, typename Emit>
__device__ __forceinline__ void topk_rank(int K, TopkLds& s, Each each, Emit emit) {
  __syncthreads();
  const int n = s.count, t = threadIdx.x;
  if (n <= kList) {
    for (int i = t; i < n; i += NT) {
      const u64 k = s.list[i];
      int above = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) above += s.list[j] > k;
      if (above < K) emit(above, k);
    }
    for (int i = n + t; i < K; i += NT) emit(i, (u64)0);
    return;
  }
  u64 last = ~(u64)0;
  for (int r = 0; r < K; ++r) {
    u64 best = 0;
    each([&](u64 k) {
      if (k < last && k > best) best = k;
    });
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const u64 o = __shfl_xor(best, d);
      best = o > best ? o : best;
    }
    if ((t & 63) == 0) s.red[t >> 6] = best;
    __syncthreads();
    for (int w = 0; w < NT / 64; ++w) best = s.red[w] > best ? s.red[w] : best;
    __syncthreads();
    if (t == 0) emit(r, best);
    last = best;                                       // (every thread has the same; 0: none is left)
  }
}

// Where place n of a search's K goes.
__device__ __forceinline__ void beam_out(const BeamArgs& a, int b, int n, u64 key) {
  const int64_t o = (int64_t)b * a.K + n;
  int parent = n, token = -1;
  bool done = true;
  float total = -INFINITY;
  if (key) {
    const uint32_t place = key_place(key);
    total = key_total(key);
    parent = (int)(place / (uint32_t)a.V);
    const bool was = a.done && a.done[(int64_t)b * a.K + parent];
    if (!was) {
      token = (int)(place % (uint32_t)a.V);
      done = token == a.eos;
    }
  }
  a.score_next[o] = total;
  a.parent[o] = parent;
  a.token[o] = token;
  a.done_next[o] = done;
}

// load_row of a beam's logits, -inf where a token is not allowed; end: row_end likewise (where `last`: the row's last chunk).
template <int STEP, typename T, int NV>
__device__ __forceinline__ void load_logits(const BeamArgs& a, int64_t row, int c0, u32x4 (&raw)[NV], bool last, float& end) {
  constexpr int V = vec<T>::N, Q = V / 4;
  constexpr uint32_t low = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  const T* x = (const T*)a.x + row * a.ldx;
  load_row<STEP>(raw, x, c0, a.V);
  const int t = threadIdx.x;
  end = row_end(x, t, last ? a.V : 0);
  if (!a.legal) return;
  typedef uint32_t u32_any __attribute__((aligned(1)));
  const uint8_t* l = a.legal + row * a.V;
  if (last && has_end<T>(t, a.V) && !l[end_place<T>(t, a.V)]) end = -INFINITY;
  uint32_t w[NV][Q];                                   // a byte to an element
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      w[i][q] = 0u;
      if (c0 + i * STEP < a.V / V) w[i][q] = *(const u32_any*)(l + (c0 + i * STEP) * V + 4 * q);
    }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const bool ok = (w[i][k / 4] >> (8 * (k & 3))) & 0xffu;
      if constexpr (V == 4) {
        raw[i][k] = ok ? raw[i][k] : low;
      } else {
        const uint32_t keep = k & 1 ? 0x0000ffffu : 0xffff0000u;
        raw[i][k / 2] = ok ? raw[i][k / 2] : (raw[i][k / 2] & keep) | (low & ~keep);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Whether a beam goes on with tokens; if not, its chunk's keys are written (a finished beam's one).
__device__ __forceinline__ bool beam_runs(const BeamArgs& a, int64_t row, int ch, float score) {
  const bool done = a.done && a.done[row];
  if (!done && score > -INFINITY) return true;
  u64* out = a.cand + ((size_t)row * a.chunks + ch) * a.K;
  for (int j = threadIdx.x; j < a.K; j += blockDim.x) out[j] = done && ch == 0 && j == 0 ? make_key(score, 0) : 0;
  return false;
}

}  // namespace

// A row, or with JOIN a chunk of one: the best K continuations by it.
template <typename T, int NT, int NV, bool JOIN>
__global__ void __launch_bounds__(NT) k_beam_rows(BeamArgs a) {
  constexpr int V = vec<T>::N;
  __shared__ TopkLds s;
  __shared__ float red[3][16];
  const int64_t row = JOIN ? blockIdx.x / a.chunks : blockIdx.x;
  const int ch = JOIN ? blockIdx.x % a.chunks : 0, t = threadIdx.x, c0 = ch * NT * NV + t;
  const float score = a.score[row];
  if (!beam_runs(a, row, ch, score)) return;
  u32x4 raw[NV];
  float most[NV], mine = -INFINITY;                    // largest of a vector, of all
  // sum of 2^(x k - ref) of this thread, ref the largest x k so far, from kFar on (whose rounding keeps the sum in range): the
  // exponentials run while later vectors arrive (1024 rows of 64001 in 41 us; 43.4 with a pass for the maximum before)
  float ref = kFar, sum = 0.f;
  const bool tail = !JOIN || ch + 1 == a.chunks;
  float end;
  load_logits<NT, T>(a, row, c0, raw, tail, end);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float v[V];
    vec<T>::unpack(raw[i], v);
    most[i] = v[0];
#pragma unroll
    for (int k = 1; k < V; ++k) most[i] = fmaxf(most[i], v[k]);
    mine = fmaxf(mine, most[i]);
    if constexpr (!JOIN) {
      const float up = fmaxf(ref, most[i] * kLog2e);
      sum *= __builtin_amdgcn_exp2f(ref - up);
      ref = up;
      opaque_vec(raw[i]);
      vec<T>::unpack(raw[i], v);
#pragma unroll
      for (int k = 0; k < V; ++k) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(v[k], kLog2e, -ref));
    }
    __builtin_amdgcn_sched_barrier(0);                 // (one vector unpacked at a time, here and below)
  }
  mine = fmaxf(mine, end);
  if constexpr (!JOIN) {
    const float up = fmaxf(ref, end * kLog2e);
    sum = sum * __builtin_amdgcn_exp2f(ref - up) + __builtin_amdgcn_exp2f(__builtin_fmaf(end, kLog2e, -up));
    ref = up;
  }
  topk_groups<NT>(mine > -INFINITY ? order_bits(mine) : 0u, s);
  float m, lse;
  if constexpr (JOIN) {
    // (every wave for itself: 64 chunks at a time)
    const float* q = a.part + (size_t)row * a.chunks * 2;
    m = -INFINITY;
    for (int i = t & 63; i < a.chunks; i += 64) m = fmaxf(m, q[2 * i]);
    m = lanes<64>(m, op_max());
    for (int i = t & 63; i < a.chunks; i += 64) {
      // (a chunk of -inf alone has the sum 0 and no share)
      const float mi = q[2 * i], si = q[2 * i + 1];
      sum += mi == -INFINITY ? si : si * __builtin_amdgcn_exp2f((mi - m) * kLog2e);
    }
    lse = m + logf(lanes<64>(sum, op_sum()));
    __syncthreads();
  } else {
    // maxima, reference and sums of the waves with one barrier
    constexpr int W = NT / 64;
    const int w = t >> 6, l = t & (W - 1);
    const float wref = lanes<64>(ref, op_max());
    const float wmax = lanes<64>(mine, op_max()), wsum = lanes<64>(sum * __builtin_amdgcn_exp2f(ref - wref), op_sum());
    if ((t & 63) == 0) red[0][w] = wmax, red[1][w] = wref, red[2][w] = wsum;
    __syncthreads();
    m = lanes<W>(red[0][l], op_max());
    const float top = lanes<W>(red[1][l], op_max());
    sum = lanes<W>(red[2][l] * __builtin_amdgcn_exp2f(red[1][l] - top), op_sum());
    const Expo ex(m, kLog2e);                          // (its mk is top)
    if (!(fabsf(m) < -0.5f * kFar)) {                  // out of ref's range (masked rows, infinities): once more, from memory
      sum = 0.f;
#pragma unroll 1
      for (int i = 0; i < NV; ++i) {
        float v[V], e;
        u32x4 u[1];
        load_logits<NT, T>(a, row, c0 + i * NT, u, false, e);
        vec<T>::unpack(u[0], v);
#pragma unroll
        for (int k = 0; k < V; ++k) sum += ex(v[k]);
      }
      sum += ex(end);
      __syncthreads();
      sum = group_reduce<NT>(sum, op_sum(), red[0]);
    }
    lse = m + ex.log_sum(sum);
  }
  const uint32_t bound = topk_bound(a.K, s);
  // Totals rise with x, but two different x may have one total, where the lower place wins: elements a few
  // roundings below the bound are looked at as well.
  const float xb = bound ? from_order(bound) : -INFINITY;
  const float tb = bound ? (xb - lse) + score : -INFINITY;
  const float lo = bound ? xb - 1e-6f * (fabsf(xb) + fabsf(lse) + fabsf(score)) : -INFINITY;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    opaque_vec(raw[i]);
    if (most[i] >= lo) {
      float v[V];
      vec<T>::unpack(raw[i], v);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float total = (v[k] - lse) + score;
        if (total >= tb && total > -INFINITY) topk_put(make_key(total, (c0 + i * NT) * V + k), s);
      }
    }
  }
  if (end >= lo) {
    const float total = (end - lse) + score;
    if (total >= tb && total > -INFINITY) topk_put(make_key(total, end_place<T>(t, a.V)), s);
  }
  topk_rank<NT>(a.K, s, [&](auto f) {
    f(make_key((end - lse) + score, end_place<T>(t, a.V)));
#pragma unroll 1
    for (int i = 0; i < NV; ++i) {
      // (read again: a loop over registers would take them all at once)
      u32x4 w[1];
      float v[V], e;
      load_logits<NT, T>(a, row, c0 + i * NT, w, false, e);
      vec<T>::unpack(w[0], v);
#pragma unroll
      for (int k = 0; k < V; ++k) f(make_key((v[k] - lse) + score, (c0 + i * NT) * V + k));
    }
  }, [&](int n, u64 key) { a.cand[((size_t)row * a.chunks + ch) * a.K + n] = key; });
}

// A chunk's maximum and sum.
template <typename T>
__global__ void __launch_bounds__(256) k_beam_part(BeamArgs a) {
  constexpr int V = vec<T>::N;
  __shared__ float red[2][4];
  const int64_t row = blockIdx.x / a.chunks;
  const int ch = blockIdx.x % a.chunks, t = threadIdx.x, c0 = ch * 256 * kPartVecs + t;
  if ((a.done && a.done[row]) || !(a.score[row] > -INFINITY)) return;
  u32x4 raw[kPartVecs];
  float m = -INFINITY, sum = 0.f;
  float end;
  load_logits<256, T>(a, row, c0, raw, ch + 1 == a.chunks, end);
  m = end;
#pragma unroll
  for (int i = 0; i < kPartVecs; ++i) {
    float v[V];
    vec<T>::unpack(raw[i], v);
#pragma unroll
    for (int k = 0; k < V; ++k) m = fmaxf(m, v[k]);
  }
  m = group_reduce<256>(m, op_max(), red[0]);
  const Expo ex(m > -INFINITY ? m : 0.f, kLog2e);
#pragma unroll
  for (int i = 0; i < kPartVecs; ++i) {
    float v[V];
    vec<T>::unpack(raw[i], v);
#pragma unroll
    for (int k = 0; k < V; ++k) sum += ex(v[k]);
  }
  sum += ex(end);
  sum = group_reduce<256>(sum, op_sum(), red[1]) * __builtin_amdgcn_exp2f(-ex.off);
  if (t == 0) {
    a.part[(size_t)blockIdx.x * 2] = m;
    a.part[(size_t)blockIdx.x * 2 + 1] = sum;
  }
}

// The K best of a search's candidates.
__global__ void __launch_bounds__(256) k_beam_merge(BeamArgs a) {
  __shared__ TopkLds s;
  const int b = blockIdx.x, t = threadIdx.x, per = a.chunks * a.K;
  const int64_t n = (int64_t)a.K * per;
  const u64* cand = a.cand + (size_t)b * n;
  auto get = [&](int64_t i) -> u64 {
    const u64 k = cand[i];
    // the place in the search: the same total, K V continuations
    return k ? (k & 0xffffffff00000000ull) | (0xffffffffu - (key_place(k) + (uint32_t)(i / per) * (uint32_t)a.V)) : 0;
  };
  uint32_t mine = 0;
  for (int64_t i = t; i < n; i += 256) mine = max(mine, (uint32_t)(cand[i] >> 32));
  topk_groups<256>(mine, s);
  __syncthreads();
  const uint32_t bound = topk_bound(a.K, s);
  for (int64_t i = t; i < n; i += 256) {
    const u64 k = get(i);
    if (k && (uint32_t)(k >> 32) >= bound) topk_put(k, s);
  }
  topk_rank<256>(a.K, s, [&](auto f) {
    for (int64_t i = t; i < n; i += 256) f(get(i));
  }, [&](int place, u64 key) { beam_out(a, b, place, key); });
}

// A whole search of at most kSmall continuations: a wave to a row for the softmax sums, totals in LDS.
template <typename T>
__global__ void __launch_bounds__(512) k_beam_small(BeamArgs a) {
  __shared__ TopkLds s;
  __shared__ float tot[kSmall];
  const int b = blockIdx.x, t = threadIdx.x, lane = t & 63, n = a.K * a.V;
  for (int k = t >> 6; k < a.K; k += 8) {
    const int64_t row = (int64_t)b * a.K + k;
    const T* x = (const T*)a.x + row * a.ldx;
    const uint8_t* legal = a.legal ? a.legal + row * a.V : nullptr;
    float* to = tot + k * a.V;
    const float score = a.score[row];
    const bool done = a.done && a.done[row];
    float m = -INFINITY, sum = 0.f;
#pragma unroll 4
    for (int v = lane; v < a.V; v += 64) {
      const float x1 = to_f32(x[v]);
      const bool ok = !legal || legal[v];
      const float e = ok ? x1 : -INFINITY;
      to[v] = e;
      m = fmaxf(m, e);
    }
    m = lanes<64>(m, op_max());
    const Expo ex(m, kLog2e);
#pragma unroll 4
    for (int v = lane; v < a.V; v += 64) sum += ex(to[v]);
    const float lse = m + ex.log_sum(lanes<64>(sum, op_sum()));
#pragma unroll 4
    for (int v = lane; v < a.V; v += 64) to[v] = done ? (v ? -INFINITY : score) : (to[v] - lse) + score;
  }
  __syncthreads();
  uint32_t mine = 0;
#pragma unroll 4
  for (int i = t; i < n; i += 512) {
    const float v = tot[i];
    if (v > -INFINITY) mine = max(mine, order_bits(v));
  }
  topk_groups<512>(mine, s);
  __syncthreads();
  const uint32_t bound = topk_bound(a.K, s);
#pragma unroll 4
  for (int i = t; i < n; i += 512) {
    const u64 k = make_key(tot[i], i);
    if (k && (uint32_t)(k >> 32) >= bound) topk_put(k, s);
  }
  topk_rank<512>(a.K, s, [&](auto f) {
    for (int i = t; i < n; i += 512) f(make_key(tot[i], i));
  }, [&](int place, u64 key) { beam_out(a, b, place, key); });
}

namespace {

// Rows of state: 16 KB pieces to a workgroup, or for short rows 16 lanes to a row.
constexpr int kPiece = 16384, kShort = 256;
constexpr int64_t kMostBytes = (int64_t)1 << 31;       // of a row of state
struct CopyState {
  const char* src;
  char* dst;
  const int32_t* live;
  int64_t slot_bytes;
  int32_t slots, pieces;                               // pieces 0: short rows, 16 to a workgroup
  uint32_t first;                                      // first workgroup
};
struct ReorderArgs {
  int K, count;
  int64_t rows;
  const int32_t* parent;
  CopyState st[SLSTM_BEAM_MAX_STATES];
};
typedef u32x4 u32x4_byte __attribute__((aligned(1)));

}  // namespace

// Bound by memory: the live slots of the parents are read and written once (512 beams, up to 121 slots of two states of 1 KB:
// 31 us, 4.1 TB/s).
__global__ void __launch_bounds__(256) k_beam_reorder(ReorderArgs a) {
  int q = 0;
  while (q + 1 < a.count && blockIdx.x >= a.st[q + 1].first) ++q;
  const CopyState& st = a.st[q];
  const uint32_t id = blockIdx.x - st.first;
  const bool wide = st.pieces > 0;
  const int64_t row = wide ? id / st.pieces : (int64_t)id * 16 + (threadIdx.x >> 4);
  if (row >= a.rows) return;
  const int p = a.parent[row];
  if (p < 0 || p >= a.K) return;
  const int64_t from = row / a.K * a.K + p;
  int live = st.slots;
  if (st.live) live = min(max(st.live[from], 0), st.slots);
  const int64_t bytes = live * st.slot_bytes, pitch = st.slots * st.slot_bytes;
  const int64_t lo = wide ? (int64_t)(id % st.pieces) * kPiece : 0, hi = wide ? min(bytes, lo + kPiece) : bytes;
  const char* s = st.src + from * pitch + lo;
  char* d = st.dst + row * pitch + lo;
  const int n = (int)max((int64_t)0, hi - lo), t = wide ? threadIdx.x : threadIdx.x & 15, nt = wide ? 256 : 16;
  // (a thread's loads all go out before its stores: a piece of 16 KB; short rows have no more)
  u32x4 v[kPiece / 4096];
#pragma unroll
  for (int i = 0; i < kPiece / 4096; ++i)
    if ((i * nt + t) * 16 + 16 <= n) v[i] = *(const u32x4_byte*)(s + (i * nt + t) * 16);
#pragma unroll
  for (int i = 0; i < kPiece / 4096; ++i)
    if ((i * nt + t) * 16 + 16 <= n) *(u32x4_byte*)(d + (i * nt + t) * 16) = v[i];
  const int tail = (n & ~15) + t;
  if (t < 16 && tail < n) d[tail] = s[tail];
}

namespace {

int beam_vecs(const slstm_beam_dims* d) { return d->type == SLSTM_F32 ? (d->V + 3) / 4 : (d->V + 7) / 8; }
int beam_chunks(const slstm_beam_dims* d) { return (beam_vecs(d) + 256 * kPartVecs - 1) / (256 * kPartVecs); }
bool beam_ok(const slstm_beam_dims* d) {
  return d && d->B >= 0 && d->K >= 1 && d->K <= kMaxBeams && d->V >= 1 && d->V <= (1 << 22) &&
         (d->type == SLSTM_F32 || d->type == SLSTM_BF16) && d->eos >= -1 && stride_ok(d->ld_logits, d->V) &&
         (int64_t)d->B * d->K <= 0x7fffffff;
}
// (a wave goes through its row 64 tokens at a time: one of 7360 took 20 us)
bool beam_small(const slstm_beam_dims* d) { return (int64_t)d->K * d->V <= kSmall && d->V <= 2048; }
// As the rows of a loss: 8192 vectors in registers; rows of four chunks or more are cut where there is not one of
// them for every compute unit.
bool beam_cut(const slstm_beam_dims* d) {
  return beam_vecs(d) > 8192 || (beam_chunks(d) >= 4 && (int64_t)d->B * d->K < 256);
}
size_t beam_part_bytes(const slstm_beam_dims* d) { return ((size_t)d->B * d->K * beam_chunks(d) * 8 + 255) & ~(size_t)255; }

template <typename T>
void beam_rows(const slstm_beam_dims* d, const BeamArgs& a, unsigned rows, bool cut, hipStream_t st) {
  const int n = beam_vecs(d);
  if (cut) {
    hipLaunchKernelGGL(k_beam_part<T>, dim3(rows * a.chunks), dim3(256), 0, st, a);
    hipLaunchKernelGGL((k_beam_rows<T, 256, kPartVecs, true>), dim3(rows * a.chunks), dim3(256), 0, st, a);
  } else if (n <= 1024) {
    hipLaunchKernelGGL((k_beam_rows<T, 256, 4, false>), dim3(rows), dim3(256), 0, st, a);
  } else if (n <= 2048) {
    hipLaunchKernelGGL((k_beam_rows<T, 256, 8, false>), dim3(rows), dim3(256), 0, st, a);
  } else if (n <= 4096) {
    hipLaunchKernelGGL((k_beam_rows<T, 256, 16, false>), dim3(rows), dim3(256), 0, st, a);
  } else {
    hipLaunchKernelGGL((k_beam_rows<T, 512, 16, false>), dim3(rows), dim3(512), 0, st, a);
  }
}

// Workgroups of a state's copy, and of a launch at most (of 256 threads).
int64_t reorder_groups(const CopyState& c, int64_t rows) { return c.pieces ? c.pieces * rows : (rows + 15) / 16; }
constexpr int64_t kMostReorder = 4 * kMostGroups;

}  // namespace

extern "C" size_t stacklstm_beam_workspace_bytes(const slstm_beam_dims* d) {
  if (!beam_ok(d)) return 0;
  if (beam_small(d) || d->B == 0) return 4;
  const bool cut = beam_cut(d);
  return (cut ? beam_part_bytes(d) : 0) + (size_t)d->B * d->K * (cut ? beam_chunks(d) : 1) * d->K * 8;
}

extern "C" int stacklstm_beam_select(const slstm_beam_dims* d, const void* logits, const uint8_t* legal, const float* score,
                                     const uint8_t* done, float* score_next, int32_t* parent, int32_t* token,
                                     uint8_t* done_next, void* workspace, size_t ws_bytes, void* stream) {
  if (!beam_ok(d)) return SLSTM_EINVAL;
  if (d->B == 0) return SLSTM_OK;
  if (!logits || !score || !score_next || !parent || !token || !done_next) return SLSTM_EINVAL;
  BeamArgs a = {};
  a.B = d->B, a.K = d->K, a.V = d->V, a.eos = d->eos;
  a.x = logits, a.ldx = row_stride(d->ld_logits, d->V), a.legal = legal, a.done = done, a.score = score;
  a.score_next = score_next, a.parent = parent, a.token = token, a.done_next = done_next;
  const hipStream_t st = as_stream(stream);
  const bool small = beam_small(d), cut = !small && beam_cut(d);
  if (!small) {
    if (!workspace || ((uintptr_t)workspace & 7u)) return SLSTM_EINVAL;
    if (ws_bytes < stacklstm_beam_workspace_bytes(d)) return SLSTM_EWORKSPACE;
    a.chunks = cut ? beam_chunks(d) : 1;
    a.part = (float*)workspace;
    a.cand = (u64*)((char*)workspace + (cut ? beam_part_bytes(d) : 0));
  }
  auto run = [&](auto t) {
    typedef decltype(t) T;
    // (at most 64 beams of 1024 chunks)
    in_pieces(d->B, small ? kMostGroups : kMostGroups / (a.K * a.chunks), [&](int64_t b0, int64_t n) {
      const int64_t r0 = b0 * a.K, r = n * a.K;
      BeamArgs p = a;
      p.B = (int)n;
      p.x = offset((const T*)logits, r0 * a.ldx), p.legal = offset(legal, r0 * a.V), p.score = score + r0, p.done = offset(done, r0);
      p.part = offset(a.part, r0 * a.chunks * 2), p.cand = offset(a.cand, r0 * a.chunks * a.K);
      p.score_next = score_next + r0, p.parent = parent + r0, p.token = token + r0, p.done_next = done_next + r0;
      if (small) {
        hipLaunchKernelGGL(k_beam_small<T>, dim3((unsigned)n), dim3(512), 0, st, p);
      } else {
        beam_rows<T>(d, p, (unsigned)r, cut, st);
        hipLaunchKernelGGL(k_beam_merge, dim3((unsigned)n), dim3(256), 0, st, p);
      }
    });
  };
  if (d->type == SLSTM_F32) run(float());
  else run(bf16_t());
  return hipGetLastError() == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
}

extern "C" int stacklstm_beam_reorder(const slstm_beam_dims* d, const int32_t* parent, const slstm_beam_state* states,
                                      int32_t count, void* stream) {
  if (!d || d->B < 0 || d->K < 1 || d->K > kMaxBeams || (int64_t)d->B * d->K > 0x7fffffff) return SLSTM_EINVAL;
  if (count < 0 || count > SLSTM_BEAM_MAX_STATES) return SLSTM_EINVAL;
  if (count == 0 || d->B == 0) return SLSTM_OK;
  if (!parent || !states) return SLSTM_EINVAL;
  const int64_t rows = (int64_t)d->B * d->K;
  ReorderArgs a = {};
  a.K = d->K, a.count = count, a.rows = rows, a.parent = parent;
  int64_t blocks = 0;
  for (int i = 0; i < count; ++i) {
    const slstm_beam_state& s = states[i];
    if (!s.src || !s.dst || s.slot_bytes < 1 || s.slots < 1 || s.reserved || s.slot_bytes > kMostBytes / s.slots)
      return SLSTM_EINVAL;
    const int64_t pitch = s.slot_bytes * s.slots;
    const char* d0 = (const char*)s.dst;
    // nothing is read from where a state is written, and no other state is written there
    auto meets = [&](const void* p, int64_t bytes) {
      const char* s0 = (const char*)p;
      return p && d0 < s0 + bytes && s0 < d0 + pitch * rows;
    };
    if (meets(parent, rows * 4)) return SLSTM_EINVAL;
    for (int j = 0; j < count; ++j) {
      const slstm_beam_state& o = states[j];
      if (o.slots < 1 || o.slot_bytes < 1 || o.slot_bytes > kMostBytes / o.slots) return SLSTM_EINVAL;
      if (meets(o.src, o.slot_bytes * o.slots * rows) || meets(o.live, rows * 4)) return SLSTM_EINVAL;
      if (j != i && meets(o.dst, o.slot_bytes * o.slots * rows)) return SLSTM_EINVAL;
    }
    CopyState& c = a.st[i];
    c.src = (const char*)s.src, c.dst = (char*)s.dst, c.live = s.live, c.slot_bytes = s.slot_bytes, c.slots = s.slots;
    c.pieces = pitch <= kShort ? 0 : (int32_t)((pitch + kPiece - 1) / kPiece);
    c.first = (uint32_t)blocks;                        // (of a call of one launch)
    blocks += reorder_groups(c, rows);
  }
  const hipStream_t st = as_stream(stream);
  if (blocks <= kMostReorder) {
    hipLaunchKernelGGL(k_beam_reorder, dim3((unsigned)blocks), dim3(256), 0, st, a);
  } else {
    // state by state, as many searches as one launch takes (one search of one state has up to 64 rows of 2^17 pieces)
    for (int i = 0; i < count; ++i) {
      const CopyState& c = a.st[i];
      const int64_t pitch = c.slot_bytes * c.slots;
      in_pieces(d->B, std::max<int64_t>(1, kMostReorder / (std::max(c.pieces, 1) * (int64_t)d->K)), [&](int64_t b0, int64_t n) {
        const int64_t r0 = b0 * d->K;
        ReorderArgs p = a;
        p.count = 1, p.rows = n * d->K, p.parent = parent + r0;
        p.st[0] = c;
        p.st[0].src = c.src + r0 * pitch, p.st[0].dst = c.dst + r0 * pitch, p.st[0].live = offset(c.live, r0), p.st[0].first = 0;
        hipLaunchKernelGGL(k_beam_reorder, dim3((unsigned)reorder_groups(c, p.rows)), dim3(256), 0, st, p);
      });
    }
  }
  return hipGetLastError() == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
}
