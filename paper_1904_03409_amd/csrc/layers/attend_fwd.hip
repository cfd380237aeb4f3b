// Attention, forward: one pass over the keys with the running reference and sum of the softmax.
//   x = c q . k (base 2),  l = sum 2^(x - m),  o = sum 2^(x - m) v,  y = o / l
// The reference m of a row need not be its largest x: one that is up to 8 below serves as well (weights then reach 2^8), and o and l are
// only brought to a new one when a row's largest has risen by more than 8 (rarely behind the first tiles).
// A wave has 16 QT queries (query and head of those that share a key's head) and all of a key tile, or, where there are few
// queries, a quarter of the tile (WK = 4), whose parts are joined through LDS. Where the row tiles do not fill the chip the
// keys are split over workgroups and k_attend_join joins their sums.
// Bound by the matrix and vector units together where queries are many (2 sequences of 4096 x 4000, 16 heads of 128 over 4, bf16: 275 us,
// 760 TFLOP/s, matrix units 30% and vector units 40% busy; fp32 4 x 1024 x 1000, 8 heads of 64: 88 us, 95 TFLOP/s), by the keys' bytes
// where they are few (8 beams of 8 sequences over up to 16384 keys, 16 heads of 128 over 4: 38 us, 5.5 TB/s, and 4.6 for the join), by a
// workgroup's start and waits where both are (256 x 240 x 120, 8 heads of 64, bf16: 51 us, 3.1 TB/s).
// With register staging, padded rows and one wave to a SIMD the first of these took 610 us.
#include <algorithm>

#include "attend.h"

#pragma clang fp contract(off)

namespace {

template <typename T, int DP, int WK, bool DMA>
struct Fwd {
  typedef Head<T, DP> H;
  // keys of a tile: 16 KB of keys and of values, twice, at most; with four waves along the keys a unit to each
  static constexpr int KT = WK == 4 ? 4 * H::UNIT : H::BYTES <= 256 ? 64 : H::BYTES <= 512 ? 32 : 16;
  static constexpr int KW = KT / WK, NU = KW / H::UNIT;                  // keys and units of a wave
  static constexpr int TILE = KT * H::BYTES;
  // waves on a SIMD that the registers are to leave room for: two hide each other's waits and run products beside exponentials
  static constexpr int WAVES = H::BYTES <= 128 || (DMA && (H::BYTES <= 256 || WK == 1)) ? 2 : 1;
  static constexpr int JOIN = WK == 4 ? 4 * 16 * (DP + 4) * 4 + 4 * 2 * 16 * 4 : 0;
  static constexpr int STAGES = 4 * TILE <= 160 * 1024 ? 2 : 1;
  static constexpr int LDS = 2 * STAGES * TILE > JOIN ? 2 * STAGES * TILE : JOIN;
};

// A row's outputs: o its sums (columns 16 dt + 4 lq ..), of reference m and sum l.
template <typename T, int DP>
__device__ __forceinline__ void fwd_row(const AttendArgs& a, int b, int t, int h, int lq, const f32x4 (&o)[DP / 16], float m, float l) {
  // (l: 0 where no key is there; NaN stays)
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* y = (T*)a.out + (int64_t)b * a.sy.b + (int64_t)t * a.sy.t + (int64_t)h * a.sy.h;
  store_cols<T, DP>(y, lq, a.D, [&](int dt) { return l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o[dt] * inv; });
  if (!a.stats) return;
  float* s = stats_row(a, a.stats, b, h, t);
  if (lq == 0) s[0] = l == 0.f ? INFINITY : m, s[1] = inv;
  if constexpr (sizeof(T) == 2) {
    if (a.width == 2) return;
#pragma unroll
    for (int dt = 0; dt < DP / 16; ++dt) {
      if (16 * dt + 4 * lq >= a.D) continue;
      uint32_t w = 0;
#pragma unroll
      for (int r = 0; r < 4; ++r) w |= (l == 0.f ? 0u : lost_byte(o[dt][r] * inv)) << (8 * r);
      ((uint32_t*)s)[2 + 4 * dt + lq] = w;
    }
  }
}

}  // namespace

// LOOP: keys of two tiles at most, which stay in LDS while the workgroup goes through a.reps row tiles, the next one's queries on their
// way during this one's products: a row tile then costs neither a start nor a wait for its keys.
// FEW: sums over up to kChain keys of a wave.
template <typename T, int DP, int QT, int WK, bool DMA, bool LOOP, bool FEW>
__global__ void __launch_bounds__(256, (Fwd<T, DP, WK, DMA>::WAVES)) k_attend_fwd(AttendArgs a) {
  typedef Head<T, DP> H;
  typedef Fwd<T, DP, WK, DMA> F;
  typedef typename H::frag frag;
  extern __shared__ __align__(16) unsigned char sm[];
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), l16 = lane & 15, lq = lane >> 4;
  const int wk = WK == 4 ? wave : 0, wq = WK == 4 ? 0 : wave;
  const Place pl = place_of(a);
  const int b = uni(pl.bh / a.Hk), hk = uni(pl.bh % a.Hk), rows = a.Tq * a.G;
  constexpr int ROWS = 16 * QT * (4 / WK);
  const int qlen = clamp_len(a.q_len, b, a.Tq), klen = clamp_len(a.k_len, b, a.Tk);
  const int kbeg = pl.split * a.chunk;
  int tile = LOOP ? pl.tile * a.reps : pl.tile;
  const int tend = LOOP ? min(tile + a.reps, (rows - 1) / ROWS + 1) : tile + 1;        // (rows: up to 2^31 - 1)
  // (no query of the tile is there: no keys)
  auto keys_end = [&] { return uni(tile * ROWS / a.G < qlen ? min(klen, kbeg + a.chunk) : kbeg); };
  int kend = keys_end();
  // place, head and row of the array of a lane's queries
  int qt_[QT], qh_[QT];
  bool here[QT];
  auto find = [&](int tile) {
#pragma unroll
    for (int j = 0; j < QT; ++j) {
      const int r = tile * ROWS + 16 * (QT * wq + j) + l16;
      here[j] = r < rows;
      const int in = min(r, rows - 1);
      qt_[j] = in / a.G;
      qh_[j] = hk * a.G + in % a.G;
    }
  };
  u32x4 qr[QT][H::STEPS];
  auto fetch = [&] {
#pragma unroll
    for (int j = 0; j < QT; ++j)
      fetch_own<T, DP>((const T*)a.q + (int64_t)b * a.sq.b + (int64_t)qt_[j] * a.sq.t + (int64_t)qh_[j] * a.sq.h,
                       here[j] && qt_[j] < qlen, a.D, lq, qr[j]);
  };
  find(tile);
  fetch();
  const T* kp = (const T*)a.k + (int64_t)b * a.sk.b + (int64_t)hk * a.sk.h;
  const T* vp = (const T*)a.v + (int64_t)b * a.sv.b + (int64_t)hk * a.sv.h;
  const uint8_t* mask = a.mask ? a.mask + (int64_t)b * a.Tk : nullptr;
  Mover<T, DP, F::KT, DMA> mk, mv;
  mk.start(a.sk.t, a.D);
  mv.start(a.sv.t, a.D);
  auto stage = [&](int n) { return sm + (F::STAGES == 2 ? (n & 1) * 2 * F::TILE : 0); };
  auto go = [&](int k0, int n) {
    const uint8_t* there = mask ? mask + k0 : nullptr;
    mk.go(kp + (int64_t)k0 * a.sk.t, a.sk.t, a.D, kend - k0, there, stage(n));
    mv.go(vp + (int64_t)k0 * a.sv.t, a.sv.t, a.D, kend - k0, there, stage(n) + F::TILE);
  };
  if (kbeg < kend) go(kbeg, 0);
  for (bool again = false; tile < tend; ++tile, again = true) {
  if (again) kend = keys_end();
  f32x4 o[QT][H::DT];
  float m[QT], l[QT];
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    m[j] = -INFINITY, l[j] = 0.f;
#pragma unroll
    for (int dt = 0; dt < H::DT; ++dt) o[j][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  frag q[QT][H::STEPS];
#pragma unroll
  for (int j = 0; j < QT; ++j) place_own<T, DP>(qr[j], a.D, lq, q[j]);
  if (LOOP && tile + 1 < tend) {
    find(tile + 1);
    fetch();
  }
  for (int k0 = kbeg, n = 0; k0 < kend; k0 += F::KT, ++n) {
    const unsigned char *kt = stage(n), *vt = kt + F::TILE;
    const int first = k0 + wk * F::KW;
    const unsigned long long there = __ballot(lane < F::KW && first + lane < kend && (!mask || mask[first + lane]));
    if (!LOOP || !again) {
      if constexpr (DMA) wait_vm<0>();
      else mk.land(a.D, stage(n)), mv.land(a.D, stage(n) + F::TILE);
      __syncthreads();
      if (F::STAGES == 2 && k0 + F::KT < kend) go(k0 + F::KT, n + 1);
    }
    if (there) {
      f32x4 s[F::NU][H::SUB][QT];
#pragma unroll
      for (int u = 0; u < F::NU; ++u)
#pragma unroll
        for (int i = 0; i < H::SUB; ++i) {
#pragma unroll
          for (int j = 0; j < QT; ++j) s[u][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
          scores<T, DP, QT>(s[u][i], kt, wk * F::KW + u * H::UNIT, i, l16, lq, q);
        }
      // x = c s: where all keys are there and no row's largest is far from 0, c goes into the exponent's own step (a reference of up
      // to 2^20 is rounded by 2^-4 at most, the same for all of a row's terms); else the products stand in the scores' place
      float top[QT], c = a.c;
      bool plain = there == (F::KW == 64 ? ~0ull : (1ull << (F::KW & 63)) - 1) && a.c > 0.f;
      if (plain) {
        bool far = false;
#pragma unroll
        for (int j = 0; j < QT; ++j) {
          top[j] = -INFINITY;
#pragma unroll
          for (int u = 0; u < F::NU; ++u)
#pragma unroll
            for (int i = 0; i < H::SUB; ++i)
#pragma unroll
              for (int r = 0; r < 4; ++r) top[j] = fmaxf(top[j], s[u][i][j][r]);
          top[j] *= a.c;
          far |= !(fabsf(top[j]) < 0x1p20f);
        }
        plain = !__any(far);
      }
      if (!plain) {
        c = 1.f;
#pragma unroll
        for (int j = 0; j < QT; ++j) top[j] = -INFINITY;
#pragma unroll
        for (int u = 0; u < F::NU; ++u)
#pragma unroll
          for (int i = 0; i < H::SUB; ++i) {
            const uint32_t bits = (uint32_t)(there >> (u * H::UNIT + row_of<T>(i, 4 * lq)));
#pragma unroll
            for (int j = 0; j < QT; ++j)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float x = bits >> r & 1 ? s[u][i][j][r] * a.c : -INFINITY;
                s[u][i][j][r] = x;
                top[j] = fmaxf(top[j], x);
              }
          }
      }
      bool rise = false;
#pragma unroll
      for (int j = 0; j < QT; ++j) {
        top[j] = rows_max(top[j]);
        rise |= top[j] > m[j] + 8.f;
      }
      if (__any(rise)) {
#pragma unroll
        for (int j = 0; j < QT; ++j) {
          const float to = top[j] > m[j] + 8.f ? top[j] : m[j];
          // (-inf: nothing has come yet)
          const float f = m[j] == to ? 1.f : __builtin_amdgcn_exp2f(m[j] - to);
          m[j] = to;
          l[j] *= f;
#pragma unroll
          for (int dt = 0; dt < H::DT; ++dt) o[j][dt] *= f;
        }
      }
      frag w[F::NU][QT];
#pragma unroll
      for (int j = 0; j < QT; ++j) {
        const float ref = m[j] == -INFINITY ? 0.f : m[j];
        float sum = 0.f;                               // (a tile's, so that l has a rounding for a tile)
#pragma unroll
        for (int u = 0; u < F::NU; ++u) {
#pragma unroll
          for (int i = 0; i < H::SUB; ++i) {
            f32x4 p;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i][j][r], c, -ref));
              sum += p[r];
            }
            put_weights(w[u][j], i, p);
          }
        }
        l[j] += sum;
      }
      sums<T, DP, QT, F::NU, FEW>(o, vt, wk * F::KW, l16, lq, w);
    }
    if constexpr (F::STAGES == 1) {
      __syncthreads();
      if (k0 + F::KT < kend) go(k0 + F::KT, n + 1);
    }
  }
#pragma unroll
  for (int j = 0; j < QT; ++j) l[j] = rows_sum(l[j]);
  if constexpr (WK == 4) {
    __syncthreads();                                   // (every wave has read its last tile)
    // the waves' parts, [wave][16][DP + 4], and their references and sums, [wave][2][16], in the tiles' place
    float *po = (float*)sm, *pm = po + 4 * 16 * (DP + 4);
    float* mine = po + (wave * 16 + l16) * (DP + 4) + 4 * lq;
#pragma unroll
    for (int dt = 0; dt < H::DT; ++dt) *(f32x4*)(mine + 16 * dt) = o[0][dt];
    if (lq == 0) pm[wave * 32 + l16] = m[0], pm[wave * 32 + 16 + l16] = l[0];
    __syncthreads();
    // the first wave has a place for every result (few queries: their sums are small)
    if (wave) return;
    m[0] = -INFINITY, l[0] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) m[0] = fmaxf(m[0], pm[w * 32 + l16]);
#pragma unroll
    for (int dt = 0; dt < H::DT; ++dt) o[0][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float mw = pm[w * 32 + l16], f = mw == m[0] ? 1.f : __builtin_amdgcn_exp2f(mw - m[0]);
      l[0] += pm[w * 32 + 16 + l16] * f;
      const float* part = po + (w * 16 + l16) * (DP + 4) + 4 * lq;
#pragma unroll
      for (int dt = 0; dt < H::DT; ++dt) o[0][dt] += *(const f32x4*)(part + 16 * dt) * f;
    }
  }
  if (LOOP) find(tile);
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    if (!here[j]) continue;
    // (behind its sequence's last query)
    if (qt_[j] >= qlen) m[j] = -INFINITY, l[j] = 0.f;
    if (a.splits == 1) {
      fwd_row<T, DP>(a, b, qt_[j], qh_[j], lq, o[j], m[j], l[j]);
    } else {
      const int64_t r = ((int64_t)pl.split * a.B * a.Hk + pl.bh) * rows + qt_[j] * a.G + qh_[j] - hk * a.G;
      store_cols<float, DP>(a.part + r * a.D, lq, a.D, [&](int dt) { return o[j][dt]; });
      if (lq == 0) a.ml[2 * r] = m[j], a.ml[2 * r + 1] = l[j];
    }
  }
  }
}

// Rows' splits joined: four columns to a thread, 2^cs threads to a row's columns, its splits shared by 2^gs groups of those. (The parts come
// from other XCDs' workgroups, 2 us away: one thread for a row's columns took 8 us for 16 splits and 25 for 64.)
template <typename T>
__global__ void __launch_bounds__(256) k_attend_join(AttendArgs a, int cs, int gs) {
  __shared__ f32x4 sv[256];
  __shared__ float sml[2][256];
  const int rows = a.Tq * a.G, all = rows * a.B * a.Hk, t = threadIdx.x;
  const int64_t row = ((a.first + blockIdx.x) << (8 - cs - gs)) + (t >> (cs + gs));
  const int n = (t & ((1 << cs) - 1)) * 4, g = t >> cs & ((1 << gs) - 1);
  const bool here = row < all && n < a.D;
  float m = -INFINITY, l = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = g; s0 < a.splits; s0 += 4 << gs) {
    float ms[4], ls[4];
    u32x4 p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = here && s0 + (i << gs) < a.splits;
      const int64_t at = in ? (int64_t)(s0 + (i << gs)) * all + row : 0;
      ms[i] = in ? a.ml[2 * at] : -INFINITY, ls[i] = in ? a.ml[2 * at + 1] : 0.f;
      p[i] = in ? load_vec(a.part + at * a.D, n / 4, a.D) : u32x4{0u, 0u, 0u, 0u};
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, ms[i]);
    const float back = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
    m = top, l *= back;
    v *= back;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = ms[i] == m ? 1.f : __builtin_amdgcn_exp2f(ms[i] - m);
      float x[4];
      vec<float>::unpack(p[i], x);
      l += ls[i] * f;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += x[k] * f;
    }
  }
  if (gs) {
    sv[t] = v, sml[0][t] = m, sml[1][t] = l;
    __syncthreads();
    if (g) return;
    const float m0 = m;
    for (int i = 1; i < 1 << gs; ++i) m = fmaxf(m, sml[0][t + (i << cs)]);
    const float f0 = m0 == m ? 1.f : __builtin_amdgcn_exp2f(m0 - m);
    v *= f0, l *= f0;
    for (int i = 1; i < 1 << gs; ++i) {
      const int o = t + (i << cs);
      const float f = sml[0][o] == m ? 1.f : __builtin_amdgcn_exp2f(sml[0][o] - m);
      v += sv[o] * f, l += sml[1][o] * f;
    }
  }
  if (!here) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int bh = (int)row / rows, r = (int)row - bh * rows, b = bh / a.Hk, place = r / a.G, h = (bh - b * a.Hk) * a.G + r % a.G;
  T* y = (T*)a.out + (int64_t)b * a.sy.b + (int64_t)place * a.sy.t + (int64_t)h * a.sy.h;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (n + k < a.D) from_f32(y[n + k], l == 0.f ? 0.f : v[k] * inv);
  if (!a.stats) return;
  float* s = stats_row(a, a.stats, b, h, place);
  if (n == 0) s[0] = l == 0.f ? INFINITY : m, s[1] = inv;
  if (sizeof(T) == 2 && a.width > 2) {
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) w |= (l == 0.f || n + k >= a.D ? 0u : lost_byte(v[k] * inv)) << (8 * k);
    ((uint32_t*)s)[2 + n / 4] = w;
  }
}

namespace {

// Row tiles and splits. Up to 16 rows (queries times heads of a key) share their keys in a tile (64 x 16 x 2000, 4 heads of 64, fp32 47 us, a
// wave to them 90; 16 x 16 x 1000, 8 of 64, bf16 11.9, 12.4); more rows go 16 or, bf16 and more than 64, 32 to a wave (64 x 64 x 1000, 8 of 64 25, 30; 64 x 96
// x 1000 33, 30; 64 x 128 x 1000, 8 of 128 76, 55).
constexpr int kLoopKeys = 128;                         // two tiles of heads of up to 64
struct FwdPlan {
  int qt, wk, rows, tiles, splits, chunk, reps;
};
FwdPlan fwd_plan(const slstm_attend_dims* d) {
  FwdPlan p;
  const int64_t R = (int64_t)d->Tq * (d->Hq / d->Hk);
  // (heads of 256: 32 rows to a wave need more registers than there are)
  const bool wide = d->D > 128;
  if (R <= 16) p.qt = 1, p.wk = 4;
  else if (R <= 64 || wide || d->type == SLSTM_F32) p.qt = 1, p.wk = 1;
  else p.qt = 2, p.wk = 1;
  p.rows = 16 * p.qt * (4 / p.wk);
  p.tiles = (int)((R + p.rows - 1) / p.rows);
  // splits of 128 keys at least, until there are two workgroups to a compute unit, where there is not one to each (us of a call: a query over
  // 4096 keys, 8 heads of 64, bf16 9.7, 11.1 from 64 keys on, 10.0 from 256, 28 whole; 300 queries over 4000 keys, one head of 128, fp32 23, 26, 31,
  // 333; 8 x 8 queries over up to 16384 keys, 16 heads of 128 over 4, bf16 41, 59 for one workgroup to a compute unit, 48 for four; but a query of 32
  // heads over 8, 16384 keys, 26, 20 for one)
  const int64_t groups = (int64_t)p.tiles * d->B * d->Hk;
  const int64_t want = groups > 0 && groups < 256 ? 512 / groups : 1, most = ((int64_t)d->Tk + 127) / 128;
  p.splits = (int)std::max<int64_t>(1, std::min(want, most));
  p.chunk = (((d->Tk + p.splits - 1) / p.splits) + 127) / 128 * 128;
  if (p.chunk < 128) p.chunk = 128;
  p.splits = std::max(1, (d->Tk + p.chunk - 1) / p.chunk);
  // few keys, many row tiles: several of them to a workgroup as long as there are three workgroups to a compute unit (with it and without: 256 x
  // 240 x 60, 8 heads of 64, fp32 107, 132 us; 512 x 240 x 60, 8 of 50 268, 345; bf16 256 x 240 x 120, 8 of 64 48, 50; 64 x 500 x 100 28.8, 27.2; 400 x 130 x
  // 100, 4 of 32 26.0, 24.8; as long as there are one to six 0 to 5% either way)
  p.reps = 1;
  if (p.wk == 1 && R > 64 && d->Tk <= kLoopKeys && d->D <= 64 && p.splits == 1) {
    p.reps = (int)std::max<int64_t>(1, std::min<int64_t>(p.tiles, groups / 768));
    p.tiles = (p.tiles + p.reps - 1) / p.reps;
  }
  return p;
}
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

extern "C" int32_t stacklstm_attend_stats_width(const slstm_attend_dims* d) { return attend_ok(d) ? attend_stats_width(d) : 0; }

extern "C" size_t stacklstm_attend_fwd_workspace_bytes(const slstm_attend_dims* d) {
  if (!attend_ok(d)) return 0;
  const FwdPlan p = fwd_plan(d);
  if (p.splits == 1) return 16;
  const size_t rows = (size_t)p.splits * d->B * d->Tq * d->Hq;
  return up256(rows * d->D * 4) + rows * 8;
}

extern "C" int stacklstm_attend_fwd(const slstm_attend_dims* d, const void* q, const void* k, const void* v, const int32_t* q_len,
                                    const int32_t* k_len, const uint8_t* mask, void* y, float* stats, void* workspace, size_t ws_bytes,
                                    void* stream) {
  if (!attend_ok(d)) return SLSTM_EINVAL;
  if (d->B == 0 || d->Tq == 0) return SLSTM_OK;
  if (!q || !y || (d->Tk && (!k || !v))) return SLSTM_EINVAL;
  if (y == q || (d->Tk && (y == k || y == v))) return SLSTM_EINVAL;
  AttendArgs a = attend_args(d);
  a.q = q, a.k = k, a.v = v, a.q_len = q_len, a.k_len = k_len, a.mask = mask, a.out = y, a.stats = stats;
  const FwdPlan p = fwd_plan(d);
  a.tiles = p.tiles, a.splits = p.splits, a.chunk = p.chunk, a.reps = p.reps;
  if (p.splits > 1) {
    if (!workspace || ((uintptr_t)workspace & 15u)) return SLSTM_EINVAL;
    if (ws_bytes < stacklstm_attend_fwd_workspace_bytes(d)) return SLSTM_EWORKSPACE;
    a.part = (float*)workspace;
    a.ml = (float*)((char*)workspace + up256((size_t)p.splits * d->B * d->Tq * d->Hq * d->D * 4));
  }
  const hipStream_t st = as_stream(stream);
  const int64_t groups = (int64_t)p.tiles * d->B * d->Hk * p.splits;
  return attend_dispatch(d, [&](auto t, auto dp) {
    typedef decltype(t) T;
    constexpr int DP = decltype(dp)::value;
    auto run = [&](auto dma) {
      constexpr bool DMA = decltype(dma)::value;
      // (fp32 heads of 256 by way of registers: four waves' keys would not fit; the one tile of rows is one either way)
      if constexpr (DMA || sizeof(T) * DP <= 512) {
        if (p.wk == 4) {
          static std::atomic<uint64_t> dev;
          return attend_launch(k_attend_fwd<T, DP, 1, 4, DMA, false, false>, a, groups, Fwd<T, DP, 4, DMA>::LDS, dev, st);
        }
      }
      if constexpr (DP <= 64) {
        static_assert(2 * Fwd<T, DP, 1, DMA>::KT >= kLoopKeys && Fwd<T, DP, 1, DMA>::STAGES == 2, "all keys stay");
        if (p.reps > 1) {
          static std::atomic<uint64_t> dev;
          return attend_launch(k_attend_fwd<T, DP, (sizeof(T) == 4 ? 1 : 2), 1, DMA, true, false>, a, groups, Fwd<T, DP, 1, DMA>::LDS, dev, st);
        }
      }
      if constexpr (sizeof(T) * DP > 512) {
        if (std::min(p.chunk, d->Tk) <= kChain) {
          static std::atomic<uint64_t> dev;
          return attend_launch(k_attend_fwd<T, DP, 1, 1, DMA, false, true>, a, groups, Fwd<T, DP, 1, DMA>::LDS, dev, st);
        }
      }
      if (DP > 128 || p.qt == 1) {
        static std::atomic<uint64_t> dev;
        return attend_launch(k_attend_fwd<T, DP, 1, 1, DMA, false, false>, a, groups, Fwd<T, DP, 1, DMA>::LDS, dev, st);
      }
      static std::atomic<uint64_t> dev;
      return attend_launch(k_attend_fwd<T, DP, (DP > 128 || sizeof(T) == 4 ? 1 : 2), 1, DMA, false, false>, a, groups, Fwd<T, DP, 1, DMA>::LDS, dev, st);
    };
    hipError_t e = dma_ok(d, k, a.sk) && dma_ok(d, v, a.sv) ? run(std::true_type()) : run(std::false_type());
    if (e == hipSuccess && p.splits > 1) {
      int cs = 0, gs = 0;
      while (4 << cs < d->D) ++cs;
      while (cs + gs < 8 && 1 << gs < p.splits) ++gs;
      in_pieces((((int64_t)d->B * d->Tq * d->Hq << (cs + gs)) + 255) / 256, kMostGroups, [&](int64_t b0, int64_t n) {
        a.first = b0;
        hipLaunchKernelGGL(k_attend_join<T>, dim3((unsigned)n), dim3(256), 0, st, a, cs, gs);
      });
      e = hipGetLastError();
    }
    return e == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
  });
}
