// Attention, backward. The scores are computed again from q and k, without atomics:
//   k_attend_dq: a workgroup's queries over all keys.  delta = dy . y,  dp = dy . v,  s = p (dp - delta),  dq = scale sum s k
//   k_attend_dkv: a workgroup's keys over all queries of the heads that share them.  dv = sum p dy,  dk = scale sum s q
// with p = 2^(x - m) / l from the forward's m and l. Seven products where five would do if dq were added up across workgroups
// in whatever order they come; these give the same bits every time. Up to 128 keys (of heads up to 64) are a workgroup's at once:
// k_attend_short does the five products, and reads q and dy once.
// Bound by the matrix and vector units together where keys are many (2 sequences of 4096 queries and 4000 keys, 16 heads of 128 over 4,
// bf16: dq 360 to 380 us, 850 TFLOP/s of its three products; dk and dv 510 to 530, 800 of its four, and 23 for joining their splits); fp32
// 4 x 1024 x 1000, 8 heads of 64: 133 and 165 us, 95 and 102 TFLOP/s of the 154 of a large product. Of few keys by a workgroup's
// start and the waits between its phases: 256 x 240 x 120, 8 heads of 64, bf16 111 us (2.8 TB/s; two kernels took 76 + 64), 64 x 119 x
// 60, 4 heads of 50, fp32 29 us (20 + 31).
#include <algorithm>

#include "attend.h"

#pragma clang fp contract(off)

namespace {

// Units of a tile whose sums are taken in one call: fp32 has an addition for each call (sums), which takes the place of products.
// 2 x 1024 x 1000, 8 heads, dq and dk and dv, by ones and by twos: of 64 74, 90 and 71, 87 us; of 128 151, 318 and 140, 289.
template <typename T, int NU>
constexpr int kPair = sizeof(T) == 4 && NU > 1 ? 2 : 1;

template <typename T, int DP, bool DMA, bool DQ, bool FEW>
struct Bwd {
  typedef Head<T, DP> H;
  // rows of a tile in LDS: two tiles of 32 KB at most together with what is kept in registers; 16 own rows to a wave at 256. FEW: sums over
  // up to kChain rows in fp32 heads of 256, in one chain and tiles of 16; other sums take 32 rows to a tile, but for dk and dv by way of registers,
  // which spill (2 x 1024 x 1000, 8 heads, 16 and 32 rows: dq 257, 232 us, by way of registers 329, 306, dk and dv 362, 300).
  static constexpr bool WIDE = H::BYTES > 512;
  static_assert(!FEW || WIDE, "fp32 heads of 256");
  static constexpr int R = H::BYTES <= 256 ? 64 : FEW || (WIDE && !DMA && !DQ) ? 16 : 32, NU = R / H::UNIT, UP = kPair<T, NU>;
  static constexpr int TILE = R * H::BYTES, LDS = 4 * TILE + 2 * 3 * R * 4;
  // own rows of a wave / 16, of a workgroup (fp32 heads of 128 by way of registers: two would not fit)
  static constexpr int QT = DP <= 64 || (DP == 128 && (DMA || sizeof(T) == 2)) ? 2 : 1, OWN = 64 * QT;
  // waves on a SIMD that the registers are to leave room for: two hide each other's waits (bf16, dq: 237 registers of heads of 128, 253 of 256;
  // 4 x 2048 x 2000, 8 heads of 256: 257 us, with one wave 553)
  static constexpr int WDQ = H::BYTES <= 128 || (DMA && sizeof(T) == 2) ? 2 : 1;
  static constexpr int WDKV = H::BYTES <= 128 ? 2 : 1;
};

// A workgroup of k_attend_dkv. BIG: eight waves with 32 keys each, whose values stay in LDS (their registers leave room for two
// waves on a SIMD that way: bf16 heads of 128; with everything in registers one wave has 337).
template <typename T, int DP, bool DMA, bool BIG, bool FEW>
struct Keys {
  typedef Bwd<T, DP, DMA, false, FEW> F;
  static constexpr int NT = BIG ? 512 : 256, N = BIG ? 2 : F::QT, ALL = NT / 4 * N, WAVES = BIG ? 2 : F::WDKV;
  static constexpr int LDS = F::LDS + (BIG ? ALL * F::H::BYTES : 0);
};

// A workgroup of k_attend_short: NW waves with 16 KN keys each, query tiles of 64 (fp32: 32).
template <typename T, int DP, int NW, int KN>
struct Short {
  typedef Head<T, DP> H;
  static constexpr int ALL = 16 * NW * KN, R = sizeof(T) == 2 ? 64 : 32, NU = R / H::UNIT, TILE = R * H::BYTES, KTILE = ALL * H::BYTES;
  static constexpr int SROW = R * (int)sizeof(T), STILE = ALL * SROW;
  static constexpr int LDS = 4 * TILE + KTILE + STILE + (4 + NW) * R * 4;
};

}  // namespace

template <typename T, int DP, bool DMA, bool FEW>
__global__ void __launch_bounds__(256, (Bwd<T, DP, DMA, true, FEW>::WDQ)) k_attend_dq(AttendArgs a) {
  typedef Head<T, DP> H;
  typedef Bwd<T, DP, DMA, true, FEW> F;
  typedef frag_t<T> frag;
  constexpr int QT = F::QT;
  extern __shared__ __align__(16) unsigned char sm[];
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), l16 = lane & 15, lq = lane >> 4;
  const Place pl = place_of(a);
  const int b = uni(pl.bh / a.Hk), hk = uni(pl.bh % a.Hk), rows = a.Tq * a.G;
  const int qlen = clamp_len(a.q_len, b, a.Tq), klen = clamp_len(a.k_len, b, a.Tk);
  const int kbeg = a.splits > 1 ? pl.split * a.chunk : 0;
  const int kend = pl.tile * F::OWN / a.G < qlen ? (a.splits > 1 ? min(klen, kbeg + a.chunk) : klen) : kbeg;
  int qt_[QT], qh_[QT];
  bool here[QT], used[QT];
  u32x4 qr[QT][H::STEPS], gr[QT][H::STEPS], yr[QT][H::STEPS];
  uint32_t lost[sizeof(T) == 2 ? QT : 1][H::STEPS][2];                   // what y's rounding took off
  float m[QT], inv[QT], delta[QT];
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    const int r = pl.tile * F::OWN + 16 * (QT * wave + j) + l16;
    here[j] = r < rows;
    const int in = min(r, rows - 1);
    qt_[j] = in / a.G;
    qh_[j] = hk * a.G + in % a.G;
    used[j] = here[j] && qt_[j] < qlen;
    fetch_own<T, DP>((const T*)a.q + (int64_t)b * a.sq.b + (int64_t)qt_[j] * a.sq.t + (int64_t)qh_[j] * a.sq.h, used[j], a.D, lq, qr[j]);
    fetch_own<T, DP>((const T*)a.dy + (int64_t)b * a.sdy.b + (int64_t)qt_[j] * a.sdy.t + (int64_t)qh_[j] * a.sdy.h, used[j], a.D, lq, gr[j]);
    fetch_own<T, DP>((const T*)a.y + (int64_t)b * a.sy.b + (int64_t)qt_[j] * a.sy.t + (int64_t)qh_[j] * a.sy.h, used[j], a.D, lq, yr[j]);
    m[j] = INFINITY, inv[j] = 0.f;
    if (used[j]) {
      const float* st = stats_row(a, (float*)a.stats_in, b, qh_[j], qt_[j]);
      m[j] = st[0], inv[j] = st[1];
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int s = 0; s < H::STEPS; ++s)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int w = 2 * (4 * s + lq) + i;
            lost[j][s][i] = 4 * w < a.D ? ((const uint32_t*)st)[2 + w] : 0u;
          }
      }
    }
  }
  const T* kp = (const T*)a.k + (int64_t)b * a.sk.b + (int64_t)hk * a.sk.h;
  const T* vp = (const T*)a.v + (int64_t)b * a.sv.b + (int64_t)hk * a.sv.h;
  const uint8_t* mask = a.mask ? a.mask + (int64_t)b * a.Tk : nullptr;
  Mover<T, DP, F::R, DMA> mk, mv;
  mk.start(a.sk.t, a.D);
  mv.start(a.sv.t, a.D);
  auto stage = [&](int n) { return sm + (n & 1) * 2 * F::TILE; };
  auto go = [&](int k0, int n) {
    const uint8_t* there = mask ? mask + k0 : nullptr;
    mk.go(kp + (int64_t)k0 * a.sk.t, a.sk.t, a.D, kend - k0, there, stage(n));
    mv.go(vp + (int64_t)k0 * a.sv.t, a.sv.t, a.D, kend - k0, there, stage(n) + F::TILE);
  };
  f32x4 o[QT][H::DT];
#pragma unroll
  for (int j = 0; j < QT; ++j)
#pragma unroll
    for (int dt = 0; dt < H::DT; ++dt) o[j][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (kbeg < kend) go(kbeg, 0);
  frag q[QT][H::STEPS], g[QT][H::STEPS];
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    place_own<T, DP>(qr[j], a.D, lq, q[j]);
    place_own<T, DP>(gr[j], a.D, lq, g[j]);
    frag y[H::STEPS];
    place_own<T, DP>(yr[j], a.D, lq, y);
    float d = 0.f;
#pragma unroll
    for (int s = 0; s < H::STEPS; ++s)
#pragma unroll
      for (int e = 0; e < H::V; ++e) {
        float v = (float)y[s][e];
        if constexpr (sizeof(T) == 2) v += used[j] ? lost_value(v, lost[j][s][e >> 2] >> (8 * (e & 3))) : 0.f;
        d += (float)g[j][s][e] * v;
      }
    // (a query without keys: nothing, whatever dy holds)
    used[j] = inv[j] != 0.f;
    delta[j] = used[j] ? rows_sum(d) : 0.f;
  }
  auto put_delta = [&] {
#pragma unroll
    for (int j = 0; j < QT; ++j)
      if (here[j] && lq == 0) {
        float* to = a.delta + (((int64_t)b * a.Hq + qh_[j]) * a.Tq + qt_[j]) * 3;
        to[0] = m[j], to[1] = inv[j], to[2] = delta[j];
      }
  };
  const bool one = a.splits == 1 && kend <= F::R;      // all keys in one tile
  if (pl.split == 0 && (!one || kend <= 0)) put_delta();
  for (int k0 = kbeg, n = 0; k0 < kend; k0 += F::R, ++n) {
    const unsigned char *kt = stage(n), *vt = kt + F::TILE;
    const unsigned long long there = __ballot(lane < F::R && k0 + lane < kend && (!mask || mask[k0 + lane]));
    if constexpr (DMA) wait_vm<0>();
    else mk.land(a.D, stage(n)), mv.land(a.D, stage(n) + F::TILE);
    __syncthreads();
    if (k0 + F::R < kend) go(k0 + F::R, n + 1);
    // p and dp of score tile i of unit u
    auto probs = [&](int u, int i, f32x4 (&p)[QT], f32x4 (&dp)[QT]) {
#pragma unroll
      for (int j = 0; j < QT; ++j) p[j] = dp[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      scores<T, DP, QT>(p, kt, u * H::UNIT, i, l16, lq, q);
      scores<T, DP, QT>(dp, vt, u * H::UNIT, i, l16, lq, g);
      const uint32_t bits = (uint32_t)(there >> (u * H::UNIT + row_of<T>(i, 4 * lq)));
#pragma unroll
      for (int j = 0; j < QT; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float x = bits >> r & 1 ? p[j][r] * a.c : -INFINITY;
          p[j][r] = __builtin_amdgcn_exp2f(x - m[j]) * inv[j];
        }
    };
    if (one) {
      // delta from the same p and dp that it is taken from: with one key their difference is 0, with few as exact as they are
      float part[QT];
#pragma unroll
      for (int j = 0; j < QT; ++j) part[j] = 0.f;
#pragma unroll 1
      for (int u = 0; u < F::NU; ++u)
#pragma unroll
        for (int i = 0; i < H::SUB; ++i) {
          f32x4 p[QT], dp[QT];
          probs(u, i, p, dp);
#pragma unroll
          for (int j = 0; j < QT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) part[j] += p[j][r] * dp[j][r];
        }
#pragma unroll
      for (int j = 0; j < QT; ++j) {
        part[j] = rows_sum(part[j]);
        delta[j] = used[j] ? part[j] : 0.f;
      }
      put_delta();
    }
#pragma unroll
    for (int u0 = 0; u0 < F::NU; u0 += F::UP) {
      frag w[F::UP][QT];
#pragma unroll
      for (int u = 0; u < F::UP; ++u)
#pragma unroll
        for (int i = 0; i < H::SUB; ++i) {
          f32x4 p[QT], dp[QT];
          probs(u0 + u, i, p, dp);
#pragma unroll
          for (int j = 0; j < QT; ++j) {
            f32x4 ds;
#pragma unroll
            for (int r = 0; r < 4; ++r) ds[r] = p[j][r] * (dp[j][r] - delta[j]);
            put_weights(w[u][j], i, ds);
          }
        }
      sums<T, DP, QT, F::UP, FEW>(o, kt, u0 * H::UNIT, l16, lq, w);
    }
  }
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    if (!here[j]) continue;
    auto v = [&](int dt) { return used[j] ? o[j][dt] * a.scale : f32x4{0.f, 0.f, 0.f, 0.f}; };
    if (a.splits > 1) {
      const int64_t row = (((int64_t)pl.split * a.B + b) * a.Hq + qh_[j]) * a.Tq + qt_[j];
      store_cols<float, DP>(a.part + row * a.D, lq, a.D, v);
    } else {
      store_cols<T, DP>((T*)a.dq + (int64_t)b * a.sdq.b + (int64_t)qt_[j] * a.sdq.t + (int64_t)qh_[j] * a.sdq.h, lq, a.D, v);
    }
  }
}

template <typename T, int DP, bool DMA, bool BIG, bool FEW>
__global__ void __launch_bounds__((Keys<T, DP, DMA, BIG, FEW>::NT), (Keys<T, DP, DMA, BIG, FEW>::WAVES)) k_attend_dkv(AttendArgs a) {
  typedef Head<T, DP> H;
  typedef Bwd<T, DP, DMA, false, FEW> F;
  typedef frag_t<T> frag;
  typedef Keys<T, DP, DMA, BIG, FEW> K;
  constexpr int KN = K::N;
  extern __shared__ __align__(16) unsigned char sm[];
  float* stats = (float*)(sm + 4 * F::TILE);           // two stages of [3][R]: m, 1 / l, delta
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), l16 = lane & 15, lq = lane >> 4;
  const Place pl = place_of(a);
  const int b = uni(pl.bh / a.Hk), hk = uni(pl.bh % a.Hk);
  const int qlen = clamp_len(a.q_len, b, a.Tq), klen = clamp_len(a.k_len, b, a.Tk);
  // (no key of the tile is there: no queries)
  const int qend = pl.tile * K::ALL < klen ? qlen : 0;
  int key[KN];
  bool there[KN];
  u32x4 kr[KN][H::STEPS], vr[KN][H::STEPS];
  unsigned char* own = sm + F::LDS + wave * 16 * KN * H::BYTES;          // BIG: the wave's values
#pragma unroll
  for (int j = 0; j < KN; ++j) {
    key[j] = pl.tile * K::ALL + 16 * (KN * wave + j) + l16;
    there[j] = key[j] < klen && (!a.mask || a.mask[(int64_t)b * a.Tk + key[j]]);
    const int in = min(key[j], a.Tk - 1);
    fetch_own<T, DP>((const T*)a.k + (int64_t)b * a.sk.b + (int64_t)in * a.sk.t + (int64_t)hk * a.sk.h, there[j], a.D, lq, kr[j]);
    fetch_own<T, DP>((const T*)a.v + (int64_t)b * a.sv.b + (int64_t)in * a.sv.t + (int64_t)hk * a.sv.h, there[j], a.D, lq, vr[j]);
  }
  f32x4 dk[KN][H::DT], dv[KN][H::DT];
#pragma unroll
  for (int j = 0; j < KN; ++j)
#pragma unroll
    for (int dt = 0; dt < H::DT; ++dt) dk[j][dt] = dv[j][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  Mover<T, DP, F::R, DMA, K::NT> mq, mg;
  mq.start(a.sq.t, a.D);
  mg.start(a.sdy.t, a.D);
  float tm = 0.f, ti = 0.f, td = 0.f;
  // tiles of the first head's queries, then of the next one's
  const int tiles = (qend + F::R - 1) / F::R;
  int n0 = 0, all = tiles * a.G;
  int h = hk * a.G, t0 = 0;                            // of the next tile to go
  if (a.splits > 1 && all > 0) {
    const int each = all / a.splits, more = all - each * a.splits;
    n0 = uni(each * pl.split + min(pl.split, more));
    all = uni(n0 + each + (pl.split < more ? 1 : 0));
    h += uni(n0 / tiles);
    t0 = uni(n0 % tiles) * F::R;
  }
  auto stage = [&](int n) { return sm + (n & 1) * 2 * F::TILE; };
  // (pointers go on by steps: products of 64 bits for each tile took as long as its first matrix products)
  const T *qp = (const T*)a.q + (int64_t)b * a.sq.b + (int64_t)t0 * a.sq.t + (int64_t)h * a.sq.h;
  const T *gp = (const T*)a.dy + (int64_t)b * a.sdy.b + (int64_t)t0 * a.sdy.t + (int64_t)h * a.sdy.h;
  const float* sp = a.delta + (((int64_t)b * a.Hq + h) * a.Tq + t0) * 3;
  const int64_t qstep = F::R * a.sq.t, gstep = F::R * a.sdy.t;
  auto go = [&](int n) {
    // (ahead of the DMAs: before it writes a register that a load may be in flight for, the compiler waits for all that is)
    if (tid < F::R) {
      tm = INFINITY, ti = td = 0.f;
      if (t0 + tid < qend) tm = sp[3 * tid], ti = sp[3 * tid + 1], td = sp[3 * tid + 2];
    }
    mq.go(qp, a.sq.t, a.D, qend - t0, nullptr, stage(n));
    mg.go(gp, a.sdy.t, a.D, qend - t0, nullptr, stage(n) + F::TILE);
    t0 += F::R, qp += qstep, gp += gstep, sp += 3 * F::R;
    if (t0 >= qend) {
      qp += a.sq.h - tiles * qstep, gp += a.sdy.h - tiles * gstep, sp += 3 * (a.Tq - tiles * F::R);
      t0 = 0;
    }
  };
  if (n0 < all) go(n0);
  frag k[KN][H::STEPS], v[BIG ? 1 : KN][H::STEPS];
#pragma unroll
  for (int j = 0; j < KN; ++j) {
    place_own<T, DP>(kr[j], a.D, lq, k[j]);
    place_own<T, DP>(vr[j], a.D, lq, v[BIG ? 0 : j]);
    if constexpr (BIG) {
#pragma unroll
      for (int s = 0; s < H::STEPS; ++s)
        *(frag*)(own + (16 * j + l16) * H::BYTES + ((4 * s + lq) ^ own_swz<H::GPR>(l16)) * 16) = v[0][s];
    }
  }
  for (int n = n0; n < all; ++n) {
    const unsigned char *qt = stage(n), *gt = qt + F::TILE;
    float* st = stats + (n & 1) * 3 * F::R;
    if constexpr (DMA) wait_vm<0>();
    else mq.land(a.D, stage(n)), mg.land(a.D, stage(n) + F::TILE);
    if (tid < F::R) st[tid] = tm, st[F::R + tid] = ti, st[2 * F::R + tid] = td;
    __syncthreads();
    if (n + 1 < all) go(n + 1);
#pragma unroll
    for (int u0 = 0; u0 < F::NU; u0 += F::UP) {
      frag wp[F::UP][KN], ws[F::UP][KN];
#pragma unroll
      for (int u = 0; u < F::UP; ++u)
#pragma unroll
        for (int i = 0; i < H::SUB; ++i) {
          const int unit = (u0 + u) * H::UNIT;
          f32x4 s[KN], dp[KN];
#pragma unroll
          for (int j = 0; j < KN; ++j) s[j] = dp[j] = f32x4{0.f, 0.f, 0.f, 0.f};
          scores<T, DP, KN>(s, qt, unit, i, l16, lq, k);
          if constexpr (BIG) scores_lds<T, DP, KN>(dp, gt, unit, i, l16, lq, own);
          else scores<T, DP, KN>(dp, gt, unit, i, l16, lq, v);
          const int at = unit + row_of<T>(i, 4 * lq);
          const f32x4 m = *(const f32x4*)(st + at), inv = *(const f32x4*)(st + F::R + at), delta = *(const f32x4*)(st + 2 * F::R + at);
#pragma unroll
          for (int j = 0; j < KN; ++j) {
            f32x4 p, ds;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float x = there[j] ? s[j][r] * a.c : -INFINITY;
              p[r] = __builtin_amdgcn_exp2f(x - m[r]) * inv[r];
              ds[r] = p[r] * (dp[j][r] - delta[r]);
            }
            put_weights(wp[u][j], i, p);
            put_weights(ws[u][j], i, ds);
          }
        }
      sums<T, DP, KN, F::UP, FEW>(dv, gt, u0 * H::UNIT, l16, lq, wp);
      sums<T, DP, KN, F::UP, FEW>(dk, qt, u0 * H::UNIT, l16, lq, ws);
    }
  }
#pragma unroll
  for (int j = 0; j < KN; ++j) {
    if (key[j] >= a.Tk) continue;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    auto vk = [&](int dt) { return there[j] ? dk[j][dt] * a.scale : zero; };
    auto vv = [&](int dt) { return there[j] ? dv[j][dt] : zero; };
    if (a.splits > 1) {
      const int64_t all = (int64_t)a.B * a.Hk * a.Tk * a.D;
      float* p = a.part + (int64_t)pl.split * 2 * all + ((int64_t)pl.bh * a.Tk + key[j]) * a.D;
      store_cols<float, DP>(p, lq, a.D, vk);
      store_cols<float, DP>(p + all, lq, a.D, vv);
    } else {
      store_cols<T, DP>((T*)a.dk + (int64_t)b * a.sdk.b + (int64_t)key[j] * a.sdk.t + (int64_t)hk * a.sdk.h, lq, a.D, vk);
      store_cols<T, DP>((T*)a.dv + (int64_t)b * a.sdv.b + (int64_t)key[j] * a.sdv.t + (int64_t)hk * a.sdv.h, lq, a.D, vv);
    }
  }
}

// All keys of a (sequence, key head) in one workgroup, up to 128: the five products of a query tile at once, q and dy read once, and y
// not at all: delta = sum p dp over the keys that are here. The waves share 32 or 16 keys each for the scores and the sums of dk and
// dv; their s go through LDS, where dq's product takes a query tile to a wave, over all keys.
template <typename T, int DP, bool DMA, int NW, int KN>
__global__ void __launch_bounds__(64 * NW, 2) k_attend_short(AttendArgs a) {
  typedef Head<T, DP> H;
  typedef Short<T, DP, NW, KN> F;
  typedef frag_t<T> frag;
  constexpr int R = F::R, QN = R / 16, DN = H::DT * QN / NW;              // column tiles of dq that a wave has of its query tile
  extern __shared__ __align__(16) unsigned char sm[];
  unsigned char *kt = sm + 4 * F::TILE, *ds_ = kt + F::KTILE;            // keys; s: [key][query]
  float *stats = (float*)(ds_ + F::STILE), *parts = stats + 4 * R;       // two stages of [2][R]: m, 1 / l; [NW][R]: the waves' sums of p dp
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), l16 = lane & 15, lq = lane >> 4;
  const Place pl = place_of(a);
  const int b = uni(pl.bh / a.Hk), hk = uni(pl.bh % a.Hk);
  const int qend = clamp_len(a.q_len, b, a.Tq), klen = clamp_len(a.k_len, b, a.Tk);
  int key[KN];
  bool there[KN];
  u32x4 kr[KN][H::STEPS], vr[KN][H::STEPS];
#pragma unroll
  for (int j = 0; j < KN; ++j) {
    key[j] = 16 * (KN * wave + j) + l16;
    there[j] = key[j] < klen && (!a.mask || a.mask[(int64_t)b * a.Tk + key[j]]);
    const int in = min(key[j], a.Tk - 1);
    fetch_own<T, DP>((const T*)a.k + (int64_t)b * a.sk.b + (int64_t)in * a.sk.t + (int64_t)hk * a.sk.h, there[j], a.D, lq, kr[j]);
    fetch_own<T, DP>((const T*)a.v + (int64_t)b * a.sv.b + (int64_t)in * a.sv.t + (int64_t)hk * a.sv.h, there[j], a.D, lq, vr[j]);
  }
  f32x4 dk[KN][H::DT], dv[KN][H::DT];
#pragma unroll
  for (int j = 0; j < KN; ++j)
#pragma unroll
    for (int dt = 0; dt < H::DT; ++dt) dk[j][dt] = dv[j][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  Mover<T, DP, R, DMA, 64 * NW> mq, mg;
  mq.start(a.sq.t, a.D);
  mg.start(a.sdy.t, a.D);
  float tm = 0.f, ti = 0.f;
  // tiles of the first head's queries, then of the next one's; those behind the last query are there for dq's zeros
  const int tiles = (a.Tq + R - 1) / R;
  int n0 = 0, all = tiles * a.G;
  int h = hk * a.G, t0 = 0;                            // of the next tile to go
  if (a.splits > 1) {
    const int each = all / a.splits, more = all - each * a.splits;
    n0 = uni(each * pl.split + min(pl.split, more));
    all = uni(n0 + each + (pl.split < more ? 1 : 0));
    h += uni(n0 / tiles);
    t0 = uni(n0 % tiles) * R;
  }
  auto stage = [&](int n) { return sm + (n & 1) * 2 * F::TILE; };
  // (pointers go on by steps: products of 64 bits for each tile took as long as its first matrix products)
  const T *qp = (const T*)a.q + (int64_t)b * a.sq.b + (int64_t)t0 * a.sq.t + (int64_t)h * a.sq.h;
  const T *gp = (const T*)a.dy + (int64_t)b * a.sdy.b + (int64_t)t0 * a.sdy.t + (int64_t)h * a.sdy.h;
  const float* sp = a.stats_in + 2 * (((int64_t)b * a.Hq + h) * a.Tq + t0);
  const int64_t qstep = R * a.sq.t, gstep = R * a.sdy.t;
  auto go = [&](int n) {
    if (t0 < qend) {
      // (ahead of the DMAs: before it writes a register that a load may be in flight for, the compiler waits for all that is)
      if (tid < R) {
        tm = INFINITY, ti = 0.f;
        if (t0 + tid < qend) tm = sp[2 * tid], ti = sp[2 * tid + 1];
      }
      mq.go(qp, a.sq.t, a.D, qend - t0, nullptr, stage(n));
      mg.go(gp, a.sdy.t, a.D, qend - t0, nullptr, stage(n) + F::TILE);
    }
    t0 += R, qp += qstep, gp += gstep, sp += 2 * R;
    if (t0 >= a.Tq) {
      qp += a.sq.h - tiles * qstep, gp += a.sdy.h - tiles * gstep, sp += 2 * (a.Tq - tiles * R);
      t0 = 0;
    }
  };
  int oh = h, ot = t0;                                 // of the tile at hand
  if (n0 < all) go(n0);
  frag k[KN][H::STEPS], v[KN][H::STEPS];
#pragma unroll
  for (int j = 0; j < KN; ++j) {
    place_own<T, DP>(kr[j], a.D, lq, k[j]);
    place_own<T, DP>(vr[j], a.D, lq, v[j]);
#pragma unroll
    for (int s = 0; s < H::STEPS; ++s) *(frag*)(kt + key[j] * H::BYTES + ((4 * s + lq) ^ swz<T, H::GPR>(key[j])) * 16) = k[j][s];
  }
  uint32_t keep[KN], low[KN];
#pragma unroll
  for (int j = 0; j < KN; ++j) keep[j] = there[j] ? 0xffffffffu : 0u, low[j] = there[j] ? 0u : 0xff800000u;
  for (int n = n0; n < all; ++n) {
    const unsigned char *qt = stage(n), *gt = qt + F::TILE;
    float* st = stats + (n & 1) * 2 * R;
    // this wave's query tile of dq, and its columns
    const int qn = wave % QN, d0 = wave / QN * DN, row = ot + 16 * qn + l16;
    f32x4 o[DN];
#pragma unroll
    for (int dt = 0; dt < DN; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bool live = ot < qend;
    if (live) {
      if constexpr (DMA) wait_vm<0>();
      else mq.land(a.D, stage(n)), mg.land(a.D, stage(n) + F::TILE);
      if (tid < R) st[tid] = tm, st[R + tid] = ti;
    }
    __syncthreads();
    if (n + 1 < all) go(n + 1);
    if (live) {
      f32x4 p[F::NU][H::SUB][KN], dp[F::NU][H::SUB][KN];
#pragma unroll
      for (int u = 0; u < F::NU; ++u)
#pragma unroll
        for (int i = 0; i < H::SUB; ++i) {
#pragma unroll
          for (int j = 0; j < KN; ++j) p[u][i][j] = dp[u][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
          scores<T, DP, KN>(p[u][i], qt, u * H::UNIT, i, l16, lq, k);
          scores<T, DP, KN>(dp[u][i], gt, u * H::UNIT, i, l16, lq, v);
          const int at = u * H::UNIT + row_of<T>(i, 4 * lq);
          const f32x4 m = *(const f32x4*)(st + at), inv = *(const f32x4*)(st + R + at);
          f32x4 part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < KN; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              // (-inf where the key is not there, without a branch: its p is 0)
              const float x = __uint_as_float((__float_as_uint(p[u][i][j][r] * a.c) & keep[j]) | low[j]);
              p[u][i][j][r] = __builtin_amdgcn_exp2f(x - m[r]) * inv[r];
              part[r] = __builtin_fmaf(p[u][i][j][r], dp[u][i][j][r], part[r]);
            }
#pragma unroll
          for (int r = 0; r < 4; ++r) part[r] = lanes<16>(part[r], op_sum());
          if (l16 == 0) *(f32x4*)(parts + wave * R + at) = part;
        }
      __syncthreads();
      constexpr int UP = kPair<T, F::NU>;
#pragma unroll
      for (int u0 = 0; u0 < F::NU; u0 += UP) {
        frag wp[UP][KN], ws[UP][KN];
#pragma unroll
        for (int half = 0; half < UP; ++half) {
          const int u = u0 + half;
#pragma unroll
          for (int i = 0; i < H::SUB; ++i) {
            const int at = u * H::UNIT + row_of<T>(i, 4 * lq);
            f32x4 delta = *(const f32x4*)(parts + at);
#pragma unroll
            for (int w = 1; w < NW; ++w) delta += *(const f32x4*)(parts + w * R + at);
#pragma unroll
            for (int j = 0; j < KN; ++j) {
              f32x4 ds;
#pragma unroll
              for (int r = 0; r < 4; ++r) ds[r] = p[u][i][j][r] * (dp[u][i][j][r] - delta[r]);
              put_weights(wp[half][j], i, p[u][i][j]);
              put_weights(ws[half][j], i, ds);
            }
          }
          // (a lane's weights are neighbours in a key's row of s: one granule)
#pragma unroll
          for (int j = 0; j < KN; ++j) *(frag*)(ds_ + key[j] * F::SROW + ((4 * u + lq) ^ swz<T, F::SROW / 16>(key[j])) * 16) = ws[half][j];
        }
        sums<T, DP, KN, UP, false>(dv, gt, u0 * H::UNIT, l16, lq, wp);
        sums<T, DP, KN, UP, false>(dk, qt, u0 * H::UNIT, l16, lq, ws);
      }
      __syncthreads();
#pragma unroll
      for (int ku = 0; ku < F::ALL / H::UNIT; ++ku) {
        const frag w = column<T, F::SROW / 16>(ds_, ku * H::UNIT, qn, l16, lq);
#pragma unroll
        for (int dt = 0; dt < DN; ++dt) o[dt] = product<T>(column<T, H::GPR>(kt, ku * H::UNIT, d0 + dt, l16, lq), w, o[dt]);
      }
    }
    if (row < a.Tq) {
      // (a query without keys has 1 / l = 0: nothing, whatever dy holds)
      const bool used = live && row < qend && st[R + 16 * qn + l16] != 0.f;
      T* dq = (T*)a.dq + (int64_t)b * a.sdq.b + (int64_t)row * a.sdq.t + (int64_t)oh * a.sdq.h;
      store_some<T, DN>(dq, 16 * d0, lq, a.D, [&](int dt) { return used ? o[dt] * a.scale : f32x4{0.f, 0.f, 0.f, 0.f}; });
    }
    ot += R;
    if (ot >= a.Tq) ot = 0, ++oh;
  }
#pragma unroll
  for (int j = 0; j < KN; ++j) {
    if (key[j] >= a.Tk) continue;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    auto vk = [&](int dt) { return there[j] ? dk[j][dt] * a.scale : zero; };
    auto vv = [&](int dt) { return there[j] ? dv[j][dt] : zero; };
    if (a.splits > 1) {
      const int64_t every = (int64_t)a.B * a.Hk * a.Tk * a.D;
      float* p = a.part + (int64_t)pl.split * 2 * every + ((int64_t)pl.bh * a.Tk + key[j]) * a.D;
      store_cols<float, DP>(p, lq, a.D, vk);
      store_cols<float, DP>(p + every, lq, a.D, vv);
    } else {
      store_cols<T, DP>((T*)a.dk + (int64_t)b * a.sdk.b + (int64_t)key[j] * a.sdk.t + (int64_t)hk * a.sdk.h, lq, a.D, vk);
      store_cols<T, DP>((T*)a.dv + (int64_t)b * a.sdv.b + (int64_t)key[j] * a.sdv.t + (int64_t)hk * a.sdv.h, lq, a.D, vv);
    }
  }
}

// Gradients from their splits: four elements of a head to a thread. part: [splits][arrays][B, H, T, D], blockIdx.y the array.
template <typename T>
__global__ void __launch_bounds__(256) k_attend_sum(const float* part, int splits, int64_t first, int B, int H, int len, int D,
                                                    T* to0, slstm_strides s0, T* to1, slstm_strides s1) {
  const int per = (D + 3) / 4;
  const int64_t id = (first + blockIdx.x) * 256 + threadIdx.x, row = id / per, rows = (int64_t)B * H * len;
  if (row >= rows) return;
  const int n = (int)(id - row * per) * 4, bh = (int)(row / len), t = (int)(row - (int64_t)bh * len), left = D - n;
  const float* p = part + ((int64_t)blockIdx.y * rows + row) * D;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int i = 0; i < splits; ++i) {
    float v[4];
    vec<float>::unpack(load_vec(p + (int64_t)i * gridDim.y * rows * D, n / 4, D), v);
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] += v[k];
  }
  const slstm_strides st = blockIdx.y ? s1 : s0;
  T* to = (blockIdx.y ? to1 : to0) + (int64_t)(bh / H) * st.b + (int64_t)t * st.t + (int64_t)(bh % H) * st.h;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < left) from_f32(to[n + k], s[k]);
}

namespace {

// Keys of a workgroup of k_attend_dkv, and splits of its queries. 256 keys with eight waves (Keys) where they are there;
// queries are split, 64 of them at least to each part, until there are two workgroups to a compute unit, where there is not one to each (backward
// us: 1 x 500 x 500, 4 heads of 100, fp32 97, 118 from 128 queries on, 199 whole; 1 x 3000 x 300, 2 heads of 64, fp32 72, 75 with up to 16 parts, 85
// with up to 64, but one head over 16384 queries of 4 and 100 keys 430, 235 with up to 64; 2 x 4096 x 1000, 4 heads of 64, bf16 65, 67 for one workgroup
// to a compute unit, 75 for four)
// (2 sequences of 4096 x 4000, 4 key heads of 128, of unequal lengths: eight waves and four parts 541 + 23 us; four waves with
// everything in registers and no parts 872, eight with 16 keys each 742).
struct KeyPlan {
  bool one, big;                                       // one: k_attend_short
  int tiles, splits;
  int qsplits, qchunk;                                 // k_attend_dq: splits of the keys
};
KeyPlan key_plan(const slstm_attend_dims* d) {
  KeyPlan p;
  p.one = attend_few_keys(d);
  p.big = d->type == SLSTM_BF16 && d->D > 64 && d->D <= 128 && d->Tk > 128;
  const int keys = p.one ? 128 : p.big ? 256 : d->D > 128 || (d->D > 64 && d->type == SLSTM_F32) ? 64 : 128;
  p.tiles = (d->Tk + keys - 1) / keys;
  const int64_t groups = std::max<int64_t>(1, (int64_t)p.tiles * d->B * d->Hk), most = (int64_t)d->Tq * (d->Hq / d->Hk) / 64;
  p.splits = (int)std::max<int64_t>(1, groups < 256 ? std::min<int64_t>(std::min<int64_t>(512 / groups, most), 32) : 1);
  // few row tiles, many keys: splits of 128 keys at least, likewise (backward us: 1 x 300 queries over 4000 keys, one head of 128, fp32
  // 109, 878 whole, 101 from 64 keys on, 132 from 256; 1 x 9 over 16000, 4 heads of 64, 82, and 99 with up to 32 or 128 splits; 1 x 64 over 16000,
  // 4 heads of 64 over one, bf16, 60, 55 with up to 32, 78 with up to 128)
  const int own = d->D <= 128 ? 128 : 64;
  const int64_t rows = (int64_t)d->Tq * (d->Hq / d->Hk), qgroups = std::max<int64_t>(1, (rows + own - 1) / own * d->B * d->Hk);
  // (where one of a workgroup's four waves has all the rows, twice as many workgroups. Backward us with 512, 1024 and 2048: 42 x 2 queries, 4168
  // keys, 8 heads of 48, fp32 1306, 1036, 1037, bf16 331, 293, 297; of 128 2711, 2154, 2175 and 639, 608, 613; 12 x 8, 14953 keys, 4 heads of 51 823, 838,
  // 853 and 255, 258, 264; 32 x 4, 4000 keys, 16 heads over 4, of 200, fp32 2025, 2039, 2078, of 256, bf16 779, 799, 839)
  const int64_t goal = rows <= own / 4 ? 1024 : 512;
  int64_t parts = qgroups < goal / 2 && !p.one ? std::min<int64_t>(std::min<int64_t>(goal / qgroups, d->Tk / 128), 64) : 1;
  if (parts < 1) parts = 1;
  p.qchunk = (int)(((d->Tk + parts - 1) / parts + 63) / 64 * 64);
  p.qsplits = parts > 1 ? (d->Tk + p.qchunk - 1) / p.qchunk : 1;
  return p;
}
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

extern "C" size_t stacklstm_attend_bwd_workspace_bytes(const slstm_attend_dims* d) {
  if (!attend_ok(d)) return 0;
  const KeyPlan p = key_plan(d);
  const size_t delta = up256((size_t)d->B * d->Tq * d->Hq * 12 + 16);
  // (dq's parts have been summed before dk's and dv's are written)
  const size_t dkv = p.splits > 1 ? (size_t)p.splits * 2 * d->B * d->Hk * d->Tk * d->D * 4 : 0;
  const size_t dq = p.qsplits > 1 ? (size_t)p.qsplits * d->B * d->Hq * d->Tq * d->D * 4 : 0;
  return delta + std::max(dkv, dq);
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
  a.part = (float*)((char*)workspace + up256((size_t)d->B * d->Tq * d->Hq * 12 + 16));
  const KeyPlan plan = key_plan(d);
  const hipStream_t st = as_stream(stream);
  return attend_dispatch(d, [&](auto t, auto dp) {
    typedef decltype(t) T;
    constexpr int DP = decltype(dp)::value;
    hipError_t e = hipSuccess;
    a.splits = plan.splits;
    if (plan.one) {
      if constexpr (DP <= 64) {
        a.tiles = 1;
        auto run = [&](auto dma, auto nw, auto kn) {
          constexpr int NW = decltype(nw)::value, KN = decltype(kn)::value;
          static std::atomic<uint64_t> dev;
          return attend_launch(k_attend_short<T, DP, decltype(dma)::value, NW, KN>, a, (int64_t)d->B * d->Hk * a.splits,
                               Short<T, DP, NW, KN>::LDS, dev, st, 64 * NW);
        };
        auto keys = [&](auto dma) {
          constexpr std::integral_constant<int, 4> four;
          constexpr std::integral_constant<int, DP == 64 && sizeof(T) == 4 ? 8 : 4> waves;
          if (d->Tk <= 64) return run(dma, four, std::integral_constant<int, 1>());
          return run(dma, waves, std::integral_constant<int, 8 / decltype(waves)::value>());
        };
        e = dma_ok(d, q, a.sq) && dma_ok(d, dy, a.sdy) ? keys(std::true_type()) : keys(std::false_type());
      }
    }
    // gradients from their splits
    auto sum = [&](int arrays, int H, int len, T* to0, const slstm_strides& s0, T* to1, const slstm_strides& s1) {
      const int64_t blocks = ((int64_t)d->B * H * len * ((d->D + 3) / 4) + 255) / 256;
      in_pieces(blocks, kMostGroups, [&](int64_t b0, int64_t n) {
        hipLaunchKernelGGL(k_attend_sum<T>, dim3((unsigned)n, arrays), dim3(256), 0, st, a.part, a.splits, b0, d->B, H, len, d->D, to0, s0,
                           to1, s1);
      });
      return hipGetLastError();
    };
    if (!plan.one && d->Tq) {
      a.splits = plan.qsplits, a.chunk = plan.qchunk;
      auto go = [&](auto kern, int own, int lds, std::atomic<uint64_t>& dev) {
        a.tiles = (int)(((int64_t)d->Tq * a.G + own - 1) / own);
        return attend_launch(kern, a, (int64_t)a.tiles * d->B * d->Hk * a.splits, lds, dev, st);
      };
      auto run = [&](auto dma) {
        constexpr bool DMA = decltype(dma)::value;
        if constexpr (sizeof(T) * DP > 512) {
          if (std::min(a.chunk, d->Tk) <= kChain) {
            typedef Bwd<T, DP, DMA, true, true> F;
            static std::atomic<uint64_t> dev;
            return go(k_attend_dq<T, DP, DMA, true>, F::OWN, F::LDS, dev);
          }
        }
        typedef Bwd<T, DP, DMA, true, false> F;
        static std::atomic<uint64_t> dev;
        return go(k_attend_dq<T, DP, DMA, false>, F::OWN, F::LDS, dev);
      };
      e = dma_ok(d, k, a.sk) && dma_ok(d, v, a.sv) ? run(std::true_type()) : run(std::false_type());
      if (e == hipSuccess && a.splits > 1) e = sum(1, d->Hq, d->Tq, (T*)dq, a.sdq, (T*)dq, a.sdq);
    }
    if (e == hipSuccess && !plan.one && d->Tk) {
      a.splits = plan.splits;
      auto go = [&](auto kern, int keys, int threads, int lds, std::atomic<uint64_t>& dev) {
        a.tiles = (d->Tk + keys - 1) / keys;
        return attend_launch(kern, a, (int64_t)a.tiles * d->B * d->Hk * a.splits, lds, dev, st, threads);
      };
      auto run = [&](auto dma) {
        constexpr bool DMA = decltype(dma)::value;
        if constexpr (DMA && sizeof(T) == 2 && DP == 128) {
          if (plan.big) {
            typedef Keys<T, DP, DMA, true, false> K;
            static std::atomic<uint64_t> dev;
            return go(k_attend_dkv<T, DP, DMA, true, false>, K::ALL, K::NT, K::LDS, dev);
          }
        }
        if constexpr (sizeof(T) * DP > 512) {
          if ((int64_t)d->Tq * a.G <= (int64_t)kChain * a.splits) {
            typedef Keys<T, DP, DMA, false, true> K;
            static std::atomic<uint64_t> dev;
            return go(k_attend_dkv<T, DP, DMA, false, true>, K::ALL, K::NT, K::LDS, dev);
          }
        }
        typedef Keys<T, DP, DMA, false, false> K;
        static std::atomic<uint64_t> dev;
        return go(k_attend_dkv<T, DP, DMA, false, false>, K::ALL, K::NT, K::LDS, dev);
      };
      e = dma_ok(d, q, a.sq) && dma_ok(d, dy, a.sdy) ? run(std::true_type()) : run(std::false_type());
    }
    if (e == hipSuccess && d->Tk && plan.splits > 1) e = sum(2, d->Hk, d->Tk, (T*)dk, a.sdk, (T*)dv, a.sdv);
    return e == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
  });
}
