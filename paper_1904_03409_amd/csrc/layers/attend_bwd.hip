// Attention, backward. The scores are computed again from q and k, in two kernels that need no atomics:
//   k_attend_dq: a workgroup's queries over all keys.  delta = dy . y,  dp = dy . v,  s = p (dp - delta),  dq = scale sum s k
//   k_attend_dkv: a workgroup's keys over all queries of the heads that share them.  dv = sum p dy,  dk = scale sum s q
// with p = 2^(x - m) / l from the forward's m and l. Seven products where five would do if dq were added up across workgroups
// in whatever order they come; these give the same bits every time.
#include <algorithm>

#include "attend.h"

#pragma clang fp contract(off)

namespace {

template <typename T, int DP>
struct Bwd {
  typedef Head<T, DP> H;
  // rows of a tile in LDS: two tiles of 32 KB at most together with what is kept in registers; 16 own rows to a wave at 256
  static constexpr int R = H::BYTES <= 256 ? 64 : H::BYTES <= 512 ? 32 : 16, NU = R / H::UNIT;
  static constexpr int TILE = R * H::ROW, LDS = 2 * TILE + 3 * R * 4;
  static constexpr int QT = DP <= 128 ? 2 : 1, OWN = 64 * QT;            // own rows of a wave / 16, of a workgroup
};

}  // namespace

template <typename T, int DP>
__global__ void __launch_bounds__(256) k_attend_dq(AttendArgs a) {
  typedef Head<T, DP> H;
  typedef Bwd<T, DP> F;
  typedef frag_t<T> frag;
  constexpr int QT = F::QT;
  extern __shared__ __align__(16) unsigned char sm[];
  unsigned char *kt = sm, *vt = sm + F::TILE;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), l16 = lane & 15, lq = lane >> 4;
  const Place pl = place_of(a);
  const int b = uni(pl.bh / a.Hk), hk = uni(pl.bh % a.Hk), rows = a.Tq * a.G;
  const int qlen = clamp_len(a.q_len, b, a.Tq), klen = clamp_len(a.k_len, b, a.Tk);
  const int kend = pl.tile * F::OWN / a.G < qlen ? klen : 0;
  int qt_[QT], qh_[QT];
  bool here[QT], used[QT];
  frag q[QT][H::STEPS], g[QT][H::STEPS];
  float m[QT], inv[QT], delta[QT];
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    const int r = pl.tile * F::OWN + 16 * (QT * wave + j) + l16;
    qt_[j] = r / a.G;
    qh_[j] = hk * a.G + r % a.G;
    here[j] = r < rows;
    used[j] = here[j] && qt_[j] < qlen;
    load_own<T, DP>((const T*)a.q + (int64_t)b * a.sq.b + (int64_t)qt_[j] * a.sq.t + (int64_t)qh_[j] * a.sq.h, used[j], a.D, lq, q[j]);
    load_own<T, DP>((const T*)a.dy + (int64_t)b * a.sdy.b + (int64_t)qt_[j] * a.sdy.t + (int64_t)qh_[j] * a.sdy.h, used[j], a.D, lq, g[j]);
    frag y[H::STEPS];
    load_own<T, DP>((const T*)a.y + (int64_t)b * a.sy.b + (int64_t)qt_[j] * a.sy.t + (int64_t)qh_[j] * a.sy.h, used[j], a.D, lq, y);
    float d = 0.f;
#pragma unroll
    for (int s = 0; s < H::STEPS; ++s)
#pragma unroll
      for (int e = 0; e < H::V; ++e) d += (float)g[j][s][e] * (float)y[s][e];
    const int64_t at = ((int64_t)b * a.Hq + qh_[j]) * a.Tq + qt_[j];
    m[j] = used[j] ? a.stats_in[2 * at] : INFINITY;
    inv[j] = used[j] ? a.stats_in[2 * at + 1] : 0.f;
    // (a query without keys: nothing, whatever dy holds)
    used[j] = inv[j] != 0.f;
    delta[j] = used[j] ? rows_sum(d) : 0.f;
    if (here[j] && lq == 0) a.delta[at] = delta[j];
  }
  const T* kp = (const T*)a.k + (int64_t)b * a.sk.b + (int64_t)hk * a.sk.h;
  const T* vp = (const T*)a.v + (int64_t)b * a.sv.b + (int64_t)hk * a.sv.h;
  const uint8_t* mask = a.mask ? a.mask + (int64_t)b * a.Tk : nullptr;
  Stage<T, DP, F::R> sk, sv;
  auto load = [&](int k0) {
    auto ok = [&](int r) { return k0 + r < kend && (!mask || mask[k0 + r]); };
    sk.load(kp + (int64_t)k0 * a.sk.t, a.sk.t, a.D, ok);
    sv.load(vp + (int64_t)k0 * a.sv.t, a.sv.t, a.D, ok);
  };
  f32x4 o[QT][H::DT];
#pragma unroll
  for (int j = 0; j < QT; ++j)
#pragma unroll
    for (int dt = 0; dt < H::DT; ++dt) o[j][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (kend > 0) load(0);
  for (int k0 = 0; k0 < kend; k0 += F::R) {
    sk.store(kt);
    sv.store(vt);
    const unsigned long long there = __ballot(lane < F::R && k0 + lane < kend && (!mask || mask[k0 + lane]));
    __syncthreads();
    if (k0 + F::R < kend) load(k0 + F::R);
#pragma unroll
    for (int u = 0; u < F::NU; ++u) {
      f32x4 s[H::SUB][QT], dp[H::SUB][QT];
#pragma unroll
      for (int i = 0; i < H::SUB; ++i) {
#pragma unroll
        for (int j = 0; j < QT; ++j) s[i][j] = dp[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        scores<T, DP, QT>(s[i], kt, u * H::UNIT, i, l16, lq, q);
        scores<T, DP, QT>(dp[i], vt, u * H::UNIT, i, l16, lq, g);
      }
      frag w[QT];
#pragma unroll
      for (int j = 0; j < QT; ++j) {
        f32x4 ds[H::SUB];
#pragma unroll
        for (int i = 0; i < H::SUB; ++i) {
          const uint32_t bits = (uint32_t)(there >> (u * H::UNIT + row_of<T>(i, 4 * lq)));
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float x = bits >> r & 1 ? s[i][j][r] * a.c : -INFINITY;
            const float p = __builtin_amdgcn_exp2f(x - m[j]) * inv[j];
            ds[i][r] = p * (dp[i][j][r] - delta[j]);
          }
        }
        w[j] = weights<T, H::SUB>(ds);
      }
      sums<T, DP, QT>(o, kt, u * H::UNIT, l16, lq, w);
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    if (!here[j]) continue;
    T* dq = (T*)a.dq + (int64_t)b * a.sdq.b + (int64_t)qt_[j] * a.sdq.t + (int64_t)qh_[j] * a.sdq.h;
#pragma unroll
    for (int dt = 0; dt < H::DT; ++dt)
      if (16 * dt + 4 * lq < a.D) store4(dq, 16 * dt + 4 * lq, a.D, used[j] ? o[j][dt] * a.scale : f32x4{0.f, 0.f, 0.f, 0.f});
  }
}

template <typename T, int DP>
__global__ void __launch_bounds__(256) k_attend_dkv(AttendArgs a) {
  typedef Head<T, DP> H;
  typedef Bwd<T, DP> F;
  typedef frag_t<T> frag;
  constexpr int KN = F::QT;
  extern __shared__ __align__(16) unsigned char sm[];
  unsigned char *qt = sm, *gt = sm + F::TILE;
  float* st = (float*)(sm + 2 * F::TILE);              // [3][R]: m, 1 / l, delta
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), l16 = lane & 15, lq = lane >> 4;
  const Place pl = place_of(a);
  const int b = uni(pl.bh / a.Hk), hk = uni(pl.bh % a.Hk);
  const int qlen = clamp_len(a.q_len, b, a.Tq), klen = clamp_len(a.k_len, b, a.Tk);
  // (no key of the tile is there: no queries)
  const int qend = pl.tile * F::OWN < klen ? qlen : 0;
  int key[KN];
  bool there[KN];
  frag k[KN][H::STEPS], v[KN][H::STEPS];
#pragma unroll
  for (int j = 0; j < KN; ++j) {
    key[j] = pl.tile * F::OWN + 16 * (KN * wave + j) + l16;
    there[j] = key[j] < klen && (!a.mask || a.mask[(int64_t)b * a.Tk + key[j]]);
    load_own<T, DP>((const T*)a.k + (int64_t)b * a.sk.b + (int64_t)key[j] * a.sk.t + (int64_t)hk * a.sk.h, there[j], a.D, lq, k[j]);
    load_own<T, DP>((const T*)a.v + (int64_t)b * a.sv.b + (int64_t)key[j] * a.sv.t + (int64_t)hk * a.sv.h, there[j], a.D, lq, v[j]);
  }
  f32x4 dk[KN][H::DT], dv[KN][H::DT];
#pragma unroll
  for (int j = 0; j < KN; ++j)
#pragma unroll
    for (int dt = 0; dt < H::DT; ++dt) dk[j][dt] = dv[j][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  Stage<T, DP, F::R> sq, sg;
  float sm_ = 0.f, si_ = 0.f, sd_ = 0.f;
  // tiles of the first head's queries, then of the next one's
  const int tiles = (qend + F::R - 1) / F::R, all = tiles * a.G;
  auto load = [&](int n) {
    const int h = hk * a.G + n / tiles, t0 = n % tiles * F::R;
    auto ok = [&](int r) { return t0 + r < qend; };
    sq.load((const T*)a.q + (int64_t)b * a.sq.b + (int64_t)t0 * a.sq.t + (int64_t)h * a.sq.h, a.sq.t, a.D, ok);
    sg.load((const T*)a.dy + (int64_t)b * a.sdy.b + (int64_t)t0 * a.sdy.t + (int64_t)h * a.sdy.h, a.sdy.t, a.D, ok);
    if (tid < F::R) {
      sm_ = INFINITY, si_ = sd_ = 0.f;
      if (t0 + tid < qend) {
        const int64_t at = ((int64_t)b * a.Hq + h) * a.Tq + t0 + tid;
        sm_ = a.stats_in[2 * at], si_ = a.stats_in[2 * at + 1], sd_ = a.delta[at];
      }
    }
  };
  if (all) load(0);
  for (int n = 0; n < all; ++n) {
    sq.store(qt);
    sg.store(gt);
    if (tid < F::R) st[tid] = sm_, st[F::R + tid] = si_, st[2 * F::R + tid] = sd_;
    __syncthreads();
    if (n + 1 < all) load(n + 1);
#pragma unroll
    for (int u = 0; u < F::NU; ++u) {
      f32x4 s[H::SUB][KN], dp[H::SUB][KN];
#pragma unroll
      for (int i = 0; i < H::SUB; ++i) {
#pragma unroll
        for (int j = 0; j < KN; ++j) s[i][j] = dp[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        scores<T, DP, KN>(s[i], qt, u * H::UNIT, i, l16, lq, k);
        scores<T, DP, KN>(dp[i], gt, u * H::UNIT, i, l16, lq, v);
      }
      frag wp[KN], ws[KN];
#pragma unroll
      for (int j = 0; j < KN; ++j) {
        f32x4 p[H::SUB], ds[H::SUB];
#pragma unroll
        for (int i = 0; i < H::SUB; ++i) {
          const int at = u * H::UNIT + row_of<T>(i, 4 * lq);
          const f32x4 m = *(const f32x4*)(st + at), inv = *(const f32x4*)(st + F::R + at), delta = *(const f32x4*)(st + 2 * F::R + at);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float x = there[j] ? s[i][j][r] * a.c : -INFINITY;
            p[i][r] = __builtin_amdgcn_exp2f(x - m[r]) * inv[r];
            ds[i][r] = p[i][r] * (dp[i][j][r] - delta[r]);
          }
        }
        wp[j] = weights<T, H::SUB>(p);
        ws[j] = weights<T, H::SUB>(ds);
      }
      sums<T, DP, KN>(dv, gt, u * H::UNIT, l16, lq, wp);
      sums<T, DP, KN>(dk, qt, u * H::UNIT, l16, lq, ws);
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < KN; ++j) {
    if (key[j] >= a.Tk) continue;
    T* ok = (T*)a.dk + (int64_t)b * a.sdk.b + (int64_t)key[j] * a.sdk.t + (int64_t)hk * a.sdk.h;
    T* ov = (T*)a.dv + (int64_t)b * a.sdv.b + (int64_t)key[j] * a.sdv.t + (int64_t)hk * a.sdv.h;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < H::DT; ++dt) {
      if (16 * dt + 4 * lq >= a.D) continue;
      store4(ok, 16 * dt + 4 * lq, a.D, there[j] ? dk[j][dt] * a.scale : zero);
      store4(ov, 16 * dt + 4 * lq, a.D, there[j] ? dv[j][dt] : zero);
    }
  }
}

extern "C" size_t stacklstm_attend_bwd_workspace_bytes(const slstm_attend_dims* d) {
  if (!attend_ok(d)) return 0;
  return (size_t)d->B * d->Tq * d->Hq * 4 + 16;
}

extern "C" int stacklstm_attend_bwd(const slstm_attend_dims* d, const void* q, const void* k, const void* v, const int32_t* q_len,
                                    const int32_t* k_len, const uint8_t* mask, const void* y, const float* stats, const void* dy,
                                    void* dq, void* dk, void* dv, void* workspace, size_t ws_bytes, void* stream) {
  if (!attend_ok(d)) return SLSTM_EINVAL;
  if (d->B == 0 || (d->Tq == 0 && d->Tk == 0)) return SLSTM_OK;
  if ((d->Tq && (!q || !y || !stats || !dy || !dq)) || (d->Tk && (!k || !v || !dk || !dv))) return SLSTM_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 15u)) return SLSTM_EINVAL;
  if (ws_bytes < stacklstm_attend_bwd_workspace_bytes(d)) return SLSTM_EWORKSPACE;
  const void* in[] = {q, k, v, y, dy};
  void* out[] = {dq, dk, dv};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 5; ++j)
      if (out[i] && out[i] == in[j]) return SLSTM_EINVAL;
    if (out[i] && out[i] == out[(i + 1) % 3]) return SLSTM_EINVAL;
  }
  AttendArgs a = attend_args(d);
  a.q = q, a.k = k, a.v = v, a.q_len = q_len, a.k_len = k_len, a.mask = mask, a.y = y, a.stats_in = stats, a.dy = dy;
  a.dq = dq, a.dk = dk, a.dv = dv, a.delta = (float*)workspace;
  const hipStream_t st = as_stream(stream);
  return attend_dispatch(d, [&](auto t, auto dp) {
    typedef decltype(t) T;
    constexpr int DP = decltype(dp)::value;
    typedef Bwd<T, DP> F;
    static std::atomic<uint64_t> dev[2];
    hipError_t e = hipSuccess;
    if (d->Tq) {
      a.tiles = (int)(((int64_t)d->Tq * a.G + F::OWN - 1) / F::OWN);
      e = attend_launch(k_attend_dq<T, DP>, a, (int64_t)a.tiles * d->B * d->Hk, F::LDS, dev[0], st);
    }
    if (e == hipSuccess && d->Tk) {
      a.tiles = (d->Tk + F::OWN - 1) / F::OWN;
      e = attend_launch(k_attend_dkv<T, DP>, a, (int64_t)a.tiles * d->B * d->Hk, F::LDS, dev[1], st);
    }
    return e == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
  });
}
