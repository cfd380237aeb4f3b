// What the attention kernels share: tiles of rows in LDS, fragments of the matrix instructions, work-space layout.
//
// Every product is a 16x16 matrix instruction (bf16: k of 32; fp32: the fp32 instruction, k of 4) of two kinds:
//   scores: rows of a tile in LDS times rows that a wave keeps in registers, over the width of a head. The result of a lane is
//     four rows of the tile (4 lq ..) for one of its own rows (l16), so softmax values need no exchange but with three lanes.
//   sums: (the tile's columns)^T times such results, over the rows of the tile. Which tile row a result belongs to is free:
//     rows are taken in an order that makes a lane's results, as they are, the fragment that the second product wants (bf16: eight
//     neighbouring rows of a unit of 32; fp32: one of four).
// l16 = lane % 16, lq = lane / 16.
#pragma once
#include <atomic>

#include "../../../include/stacklstm_layers.h"
#include "../head/head.h"

namespace {

struct AttendArgs {
  int B, Tq, Tk, Hq, Hk, G, D;                         // G: query heads to a key's
  float c, scale;                                      // c: scale log2 e
  const void *q, *k, *v, *y, *dy;
  slstm_strides sq, sk, sv, sy, sdy, sdq, sdk, sdv;
  const int32_t *q_len, *k_len;
  const uint8_t* mask;
  void *out, *dq, *dk, *dv;
  // [B, Hq, Tq, width]: reference of a row's exponents (base 2), 1 / sum, and (width > 2) what y's rounding took off, a byte to an element
  float* stats;
  const float* stats_in;
  int width;
  float *delta;                                        // [B, Hq, Tq, 3]: what k_attend_dkv reads of a row: reference, 1 / sum, dy . y
  // splits: [splits][B Hk][rows][D] sums, [splits][B Hk][rows][2] references and sums; of dk and dv [splits][2][B Hk][Tk][D]
  float *part, *ml;
  int tiles, splits, chunk, reps;                      // workgroups of a (sequence, key head) and split; keys of a split; row tiles of a workgroup
  int64_t first;                                       // a launch's first workgroup
  int64_t piece, full;                                 // neighbours on an XCD; how many are dealt out that way
};

template <typename T> struct frag_of { typedef f32x4 type; };
template <> struct frag_of<bf16_t> { typedef bf16x8 type; };
template <typename T> using frag_t = typename frag_of<T>::type;

// A head's width padded to DP elements.
template <typename T, int DP>
struct Head {
  typedef typename frag_of<T>::type frag;
  static constexpr int V = vec<T>::N;
  static constexpr int BYTES = DP * (int)sizeof(T), GPR = BYTES / 16, STEPS = GPR / 4, DT = DP / 16;
  static constexpr int SUB = sizeof(T) == 2 ? 2 : 1, UNIT = 16 * SUB;      // tiles of 16 rows, and rows, of a unit
};

// Rows of a tile lie densely in LDS; 16-byte granule c of row r is at place c ^ swz(r) of its row, so that neither the 16 rows of a
// score's fragment nor the rows of a transposed one meet in a bank. A 16-byte read is served in four parts: lanes 0 .. 3, 12 .. 15,
// 20 .. 23, 24 .. 27 are one of them (with parts of 16 neighbours in mind a read took 8 cycles instead of 4). bf16: fragments take
// rows 0 .. 3, 8 .. 11, 16 .. 19, 24 .. 27 (+ 4) of a unit; a transposed read takes pairs of granules of eight of them. fp32: rows 0 .. 15;
// every fourth row, four granules.
template <typename T, int GPR>
__device__ __forceinline__ int swz(int r) {
  if constexpr (sizeof(T) == 4) return GPR >= 16 ? r & 15 : (r >> 1) & 7;
  else if constexpr (GPR >= 16) return (r & 3) << 1 | (r & 8);
  else if constexpr (GPR == 8) return (r & 2) | (r >> 1 & 4);
  else return r >> 2 & 2;
}

// The same for rows that are read 16 neighbours at a time.
template <int GPR>
__device__ __forceinline__ int own_swz(int r) { return GPR >= 16 ? r & 15 : GPR == 8 ? (r >> 1) & 7 : (r >> 2) & 3; }

// Tile row (of a unit) that row i of score tile `sub` is; the four rows of a lane's result are row_of(sub, 4 lq) + 0 .. 3.
template <typename T>
__device__ __forceinline__ int row_of(int sub, int i) {
  return sizeof(T) == 2 ? 8 * (i >> 2) + 4 * sub + (i & 3) : i;
}

// Granule c of a row of D elements, in two parts as load_vec's: the load (in bounds whatever c is) and the granule's place, zeros
// past the row's end. No load waits for a branch.
template <typename T>
__device__ __forceinline__ u32x4 fetch_granule(const T* row, int c, int D) {
  if (D < vec<T>::N) return c == 0 ? load_vec(row, 0, D) : u32x4{0u, 0u, 0u, 0u};
  return *(const u32x4_any*)(row + min(c * vec<T>::N, D - vec<T>::N));
}
template <typename T>
__device__ __forceinline__ u32x4 place_granule(u32x4 v, int c, int D, bool there) {
  constexpr int V = vec<T>::N;
  const u32x4 zero = {0u, 0u, 0u, 0u};
  if (D % V == 0 || D < V) return there && c * V < D ? v : zero;
  v = shift_vec<T>(v, min(c * V - min(c * V, D - V), V));
  return there ? v : zero;
}
// Fragments of a wave's own row: 16 bytes of every 64, zeros where it is not there (what is padding is not read). In two parts:
// all of a workgroup's first loads are on their way before the first of them is waited for.
template <typename T, int DP>
__device__ __forceinline__ void fetch_own(const T* row, bool there, int D, int lq, u32x4 (&r)[Head<T, DP>::STEPS]) {
#pragma unroll
  for (int s = 0; s < Head<T, DP>::STEPS; ++s) r[s] = u32x4{0u, 0u, 0u, 0u};
  if (there) {
#pragma unroll
    for (int s = 0; s < Head<T, DP>::STEPS; ++s) r[s] = fetch_granule(row, 4 * s + lq, D);
  }
}
template <typename T, int DP>
__device__ __forceinline__ void place_own(const u32x4 (&r)[Head<T, DP>::STEPS], int D, int lq, frag_t<T> (&f)[Head<T, DP>::STEPS]) {
#pragma unroll
  for (int s = 0; s < Head<T, DP>::STEPS; ++s) f[s] = __builtin_bit_cast(frag_t<T>, place_granule<T>(r[s], 4 * s + lq, D, true));
}

// acc += tile rows (of unit row `base`, a multiple of the unit, score tile sub) times own rows.
template <typename T, int DP, int N>
__device__ __forceinline__ void scores(f32x4 (&acc)[N], const unsigned char* tile, int base, int sub, int l16, int lq,
                                       const frag_t<T> (&own)[N][Head<T, DP>::STEPS]) {
  typedef Head<T, DP> H;
  const int row = row_of<T>(sub, l16), f = swz<T, H::GPR>(row);
  auto step = [&](int s) { return *(const typename H::frag*)(tile + (base + row) * H::BYTES + ((4 * s + lq) ^ f) * 16); };
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int s = 0; s < H::STEPS; ++s) {
      const typename H::frag a = step(s);
#pragma unroll
      for (int j = 0; j < N; ++j) acc[j] = mfma_bf16_16x16x32(a, own[j][s], acc[j]);
    }
  } else {
    // (the next step's 16 bytes on their way during this one's products, as in sums below)
    typename H::frag a = step(0);
#pragma unroll
    for (int s = 0; s < H::STEPS; ++s) {
      typename H::frag next = a;
      if (s + 1 < H::STEPS) next = step(s + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], own[j][s][e], acc[j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      a = next;
    }
  }
}

// The same with own rows in LDS too (16 j + l16 of `own`).
template <typename T, int DP, int N>
__device__ __forceinline__ void scores_lds(f32x4 (&acc)[N], const unsigned char* tile, int base, int sub, int l16, int lq,
                                           const unsigned char* own) {
  typedef Head<T, DP> H;
  const int row = row_of<T>(sub, l16);
  own += opaque(l16 * H::BYTES);                       // (read for every tile: the compiler would keep them in registers)
#pragma unroll
  for (int s = 0; s < H::STEPS; ++s) {
    const typename H::frag a = *(const typename H::frag*)(tile + (base + row) * H::BYTES + ((4 * s + lq) ^ swz<T, H::GPR>(row)) * 16);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const typename H::frag b = *(const typename H::frag*)(own + 16 * j * H::BYTES + ((4 * s + lq) ^ own_swz<H::GPR>(l16)) * 16);
      acc[j] = mfma_bf16_16x16x32(a, b, acc[j]);
    }
  }
}

// A unit's results as the second product's fragment: score tile `sub` of it.
__device__ __forceinline__ void put_weights(bf16x8& w, int sub, const f32x4& p) {
#pragma unroll
  for (int r = 0; r < 4; ++r) w[4 * sub + r] = static_cast<__bf16>(p[r]);
}
__device__ __forceinline__ void put_weights(f32x4& w, int, const f32x4& p) { w = p; }
// Columns 16 dt .. of a unit (from row `base` on) as a fragment: a lane has column l16, and the unit's rows as the weights have them.
template <typename T, int GPR>
__device__ __forceinline__ frag_t<T> column(const unsigned char* tile, int base, int dt, int l16, int lq) {
  if constexpr (sizeof(T) == 2) {
    // transposed: the lane gives the address of unit row 8 lq + l16 / 4 and columns 4 (l16 % 4) of the tile, and gets column
    // l16, four rows
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    const int row = 8 * lq + (l16 >> 2);
    const unsigned char* q = tile + (base + row) * GPR * 16 + ((2 * dt + (l16 >> 1 & 1)) ^ swz<T, GPR>(row)) * 16 + (l16 & 1) * 8;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(q));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(q + 4 * GPR * 16));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = 4 * lq + e;
      if constexpr (GPR >= 16) {
        // (4 dt + l16 / 4) ^ (4 lq + e) taken apart, so that eight numbers and constants make all of a unit's addresses
        static_assert(GPR % 16 == 0, "whole fours of columns");
        const unsigned char* q = tile + row * GPR * 16 + ((l16 >> 2) ^ e) * 16 + (l16 & 3) * 4;
        v[e] = *(const float*)(q + ((dt & 3) ^ lq) * 64 + (base * GPR * 16 + (dt >> 2) * 256));
      } else {
        v[e] = *(const float*)(tile + (base + row) * GPR * 16 + ((4 * dt + (l16 >> 2)) ^ swz<T, GPR>(base + row)) * 16 + (l16 & 3) * 4);
      }
    }
    return v;
  }
}
template <typename T>
__device__ __forceinline__ f32x4 product(const frag_t<T>& a, const frag_t<T>& b, f32x4 c) {
  if constexpr (sizeof(T) == 2) {
    return mfma_bf16_16x16x32(a, b, c);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
}
// acc[j][dt] += (columns 16 dt .. of the NU units from row `base` on)^T times the weights w[u][j].
// fp32 takes a call's products from 0 on and adds what they come to, so that acc has a rounding for 16 NU rows and not for each: a chain of
// n roundings is off by 2.5e-8 sqrt(n / 2) of a sum of random signs (16384 keys: 2.3e-6, where its terms are good to 3e-7). The additions' cost:
// 4 x 1024 x 1000, 8 heads of 64, forward and backward 77 + 255 -> 78 + 265 us; 2 x 2048 x 2000, 8 heads of 256, 552 + 1917 -> 565 + 2045, of
// 201 872 + 2440 -> 981 + 2902. CHAIN: one chain all the same, for sums of few rows (kChain).
constexpr int kChain = 256;
template <typename T, int DP, int N, int NU, bool CHAIN>
__device__ __forceinline__ void sums(f32x4 (&acc)[N][DP / 16], const unsigned char* tile, int base, int l16, int lq, const frag_t<T> (&w)[NU][N]) {
  typedef Head<T, DP> H;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int dt = 0; dt < H::DT; ++dt) {
        const frag_t<T> a = column<T, H::GPR>(tile, base + u * H::UNIT, dt, l16, lq);
#pragma unroll
        for (int j = 0; j < N; ++j) acc[j][dt] = mfma_bf16_16x16x32(a, w[u][j], acc[j][dt]);
      }
  } else {
    // (the next columns are on their way during these ones' products: left to itself the compiler read one number, waited, read the
    // next. 2 x 2048 x 2000, 8 heads of 256, forward, dq, dk and dv: 804, 1076, 1260 us; 673, 856, 1056 this way, here and in scores)
    frag_t<T> a = column<T, H::GPR>(tile, base, 0, l16, lq);
    f32x4 t[2][N];
#pragma unroll
    for (int dt = 0; dt < H::DT; ++dt) {
#pragma unroll
      for (int j = 0; j < N; ++j) t[dt & 1][j] = CHAIN ? acc[j][dt] : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        frag_t<T> next = a;
        if (u + 1 < NU) next = column<T, H::GPR>(tile, base + (u + 1) * H::UNIT, dt, l16, lq);
        else if (dt + 1 < H::DT) next = column<T, H::GPR>(tile, base, dt + 1, l16, lq);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < N; ++j) t[dt & 1][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], w[u][j][e], t[dt & 1][j], 0, 0, 0);
        // (the columns before these: their products have ended)
        if (u == 0 && dt > 0) {
#pragma unroll
          for (int j = 0; j < N; ++j) acc[j][dt - 1] = CHAIN ? t[(dt - 1) & 1][j] : acc[j][dt - 1] + t[(dt - 1) & 1][j];
        }
        __builtin_amdgcn_sched_barrier(0);
        a = next;
      }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j][H::DT - 1] = CHAIN ? t[(H::DT - 1) & 1][j] : acc[j][H::DT - 1] + t[(H::DT - 1) & 1][j];
  }
}

// ROWS rows on their way from memory to LDS: zeros where a row is not there and past a head's end. With DMA straight to LDS (rows
// of whole, aligned granules), else through registers: go() starts a tile, land() puts it in place.
template <typename T, int DP, int ROWS, bool DMA, int NT = 256>
struct Mover {
  typedef Head<T, DP> H;
  static constexpr int ALL = ROWS * H::GPR, I = (ALL + NT - 1) / NT;
  static_assert(!DMA || ALL % NT == 0, "whole waves");
  u32x4 r[DMA ? 1 : I];
  uint32_t there[DMA ? 1 : I];                         // mask bytes
  int rows;
  uint32_t off[DMA ? I : 1];
  static __device__ __forceinline__ void place(int i, int& row, int& c) {
    const int L = i * NT + threadIdx.x;
    row = L / H::GPR;
    c = (L % H::GPR) ^ swz<T, H::GPR>(row);
  }
  __device__ __forceinline__ void start(int64_t stride, int D) {
    if constexpr (DMA) {
#pragma unroll
      for (int i = 0; i < I; ++i) {
        int row, c;
        place(i, row, c);
        off[i] = c * H::V < D ? (uint32_t)(row * stride + c * H::V) * (uint32_t)sizeof(T) : kOOB;
      }
    }
  }
  // rows 0 .. n of base (more than 0), those with mask byte 0 (mask not NULL) left out
  __device__ __forceinline__ void go(const T* base, int64_t stride, int D, int n, const uint8_t* mask, unsigned char* tile) {
    n = uni(min(n, ROWS));                             // (descriptors are scalar registers)
    if constexpr (DMA) {
      const rsrc_t rs = make_rsrc(base, (size_t)((n - 1) * stride + D) * sizeof(T));
      const int wave = uni(threadIdx.x >> 6);
#pragma unroll
      for (int i = 0; i < I; ++i) {
        uint32_t o = off[i];
        if (mask) {
          int row, c;
          place(i, row, c);
          if (row >= n || !mask[row]) o = kOOB;
        }
        bdma16(rs, o, 0, lds_addr(tile + (i * (NT / 64) + wave) * 1024));
      }
    } else {
      rows = n;
#pragma unroll
      for (int i = 0; i < I; ++i) {
        int row, c;
        place(i, row, c);
        row = min(row, n - 1);
        r[i] = fetch_granule(base + row * stride, c, D);
        there[i] = mask ? mask[row] : 1u;
      }
    }
  }
  __device__ __forceinline__ void land(int D, unsigned char* tile) const {
    if constexpr (!DMA) {
#pragma unroll
      for (int i = 0; i < I; ++i) {
        int row, c;
        place(i, row, c);
        const int L = i * NT + threadIdx.x;
        if (ALL % NT == 0 || L < ALL) *(u32x4*)(tile + L * 16) = place_granule<T>(r[i], c, D, row < rows && there[i]);
      }
    }
  }
};

template <typename T>
__device__ __forceinline__ void store4(T* to, const f32x4& v) {
  if constexpr (sizeof(T) == 4) {
    *(u32x4_any*)to = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  } else {
    typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
    *(u32x2_any*)to = u32x2_any{(uint32_t)f32_to_bf16_bits(v[0]) | (uint32_t)f32_to_bf16_bits(v[1]) << 16,
                                (uint32_t)f32_to_bf16_bits(v[2]) | (uint32_t)f32_to_bf16_bits(v[3]) << 16};
  }
}
// A row's columns n0 + 16 dt + 4 lq .., dt < DN, f(dt) their values.
template <typename T, int DN, typename F>
__device__ __forceinline__ void store_some(T* row, int n0, int lq, int D, F f) {
  n0 += 4 * lq;
  if (D % 4 == 0) {
#pragma unroll
    for (int dt = 0; dt < DN; ++dt)
      if (n0 + 16 * dt < D) store4(row + n0 + 16 * dt, f(dt));
  } else {
#pragma unroll
    for (int dt = 0; dt < DN; ++dt) {
      const f32x4 v = f(dt);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (n0 + 16 * dt + r < D) from_f32(row[n0 + 16 * dt + r], v[r]);
    }
  }
}
template <typename T, int DP, typename F>
__device__ __forceinline__ void store_cols(T* row, int lq, int D, F f) { store_some<T, DP / 16>(row, 0, lq, D, f); }

// What a 16-bit y loses, in 1/254 of the last place of the rounded value: delta = dy . y of a backward takes it back. Without it delta is
// off by 2^-9 of its terms, and where one key outweighs the others p (dp - delta) is small beside them: gradients of 4 keys were 0.0036
// off, twice the rounding of their outputs. (Keys of one tile alone: k_attend_dq sums p dp instead.)
__device__ __forceinline__ float last_place(uint32_t bits) {             // of a bfloat16; 0 for zeros and what is below 2^-119
  const int e = (int)(bits >> 7 & 0xffu) - 7;
  return e > 0 ? __uint_as_float((uint32_t)e << 23) : 0.f;
}
__device__ __forceinline__ uint32_t lost_byte(float v) {
  const uint32_t b = f32_to_bf16_bits(v);
  const float place = last_place(b), off = v - bf16_bits_to_f32((bf16_t)b);
  // (a power of two: 1 / place by its exponent)
  const float q = place > 0.f && fabsf(off) <= place ? off * __uint_as_float(0x7f000000u - __float_as_uint(place)) * 254.f : 0.f;
  return (uint32_t)(int)__builtin_rintf(q) & 0xffu;
}
__device__ __forceinline__ float lost_value(float y, uint32_t byte) {
  return (float)(int8_t)byte * (last_place(__float_as_uint(y) >> 16) * (1.f / 254.f));
}
// A row's statistics: l = 0: no key.
__device__ __forceinline__ float* stats_row(const AttendArgs& a, float* stats, int b, int h, int t) {
  return stats + (((int64_t)b * a.Hq + h) * a.Tq + t) * a.width;
}
__device__ __forceinline__ int clamp_len(const int32_t* len, int b, int most) {
  return len ? max(0, min(len[b], most)) : most;
}
// Over the lanes that hold the same own row.
__device__ __forceinline__ float rows_max(float v) { return half_swap(row_swap(v, op_max()), op_max()); }
__device__ __forceinline__ float rows_sum(float v) { return half_swap(row_swap(v, op_sum()), op_sum()); }

// Workgroup -> (sequence and key head, split, row tile). Workgroups go to the 8 XCDs in turn; an XCD takes every eighth run of
// `piece` of them, so that row tiles that share keys find them in its L2, and sequences of other lengths are spread over the XCDs.
struct Place {
  int bh, split, tile;
};
__device__ __forceinline__ Place place_of(const AttendArgs& a) {
  // (32 bits: 64-bit divisions took 4 us of every workgroup's start)
  uint32_t id = (uint32_t)a.first + blockIdx.x;
  const uint32_t piece = (uint32_t)a.piece, run = (id >> 3) / piece;
  if (id < (uint32_t)a.full) id = (run * 8 + (id & 7)) * piece + ((id >> 3) - run * piece);
  Place p;
  const uint32_t per = (uint32_t)a.tiles * (uint32_t)a.splits, bh = id / per, rest = id - bh * per;
  p.bh = (int)bh;
  p.split = a.splits == 1 ? 0 : (int)(rest / (uint32_t)a.tiles);
  p.tile = (int)(rest - (uint32_t)p.split * (uint32_t)a.tiles);
  return p;
}

// ----------------------------------------------------------------------------- host

inline bool strides_zero(const slstm_strides& s) { return s.b == 0 && s.t == 0 && s.h == 0; }
inline slstm_strides strides_of(const slstm_strides& s, int T, int H, int D) {
  if (!strides_zero(s)) return s;
  return slstm_strides{(int64_t)T * H * D, (int64_t)H * D, D};
}
inline bool stride_range(const slstm_strides& s) {
  const int64_t most = (int64_t)1 << 40;
  return s.b >= 0 && s.t >= 0 && s.h >= 0 && s.b < most && s.t < most && s.h < most;
}
// No two elements of an output at one place: in the order of the strides each step passes all that lies within it.
inline bool strides_apart(const slstm_strides& s, int B, int T, int H, int D) {
  int64_t st[3] = {s.b, s.t, s.h}, n[3] = {B, T, H};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (st[j] < st[i]) {
        int64_t x = st[i]; st[i] = st[j]; st[j] = x;
        x = n[i]; n[i] = n[j]; n[j] = x;
      }
  __int128 extent = D;
  for (int i = 0; i < 3; ++i) {
    if (n[i] < 2) continue;
    if (st[i] < extent) return false;
    extent += (__int128)st[i] * (n[i] - 1);
  }
  return extent < (__int128)1 << 60;
}
inline bool attend_ok(const slstm_attend_dims* d) {
  if (!d || d->B < 0 || d->Tq < 0 || d->Tk < 0 || d->Tq > (1 << 24) || d->Tk > (1 << 24) || d->Hq < 1 || d->Hk < 1 ||
      d->Hq > (1 << 16) || d->Hk > (1 << 16) || d->Hq % d->Hk || d->D < 1 || d->D > 256)
    return false;
  if (d->type != SLSTM_F32 && d->type != SLSTM_BF16) return false;
  if (!(fabsf(d->scale) <= 0x1p127f)) return false;    // (scale log2 e is finite too)
  if ((int64_t)d->Tq * d->Hq > 0x7fffffff || (int64_t)d->Tk * d->Hk > 0x7fffffff) return false;
  if ((int64_t)d->Tq * d->Hq * d->B > 0x7fffffff || (int64_t)d->Tk * d->Hk * d->B > 0x7fffffff) return false;
  const slstm_strides* s[8] = {&d->q, &d->k, &d->v, &d->dy, &d->y, &d->dq, &d->dk, &d->dv};
  for (int i = 0; i < 8; ++i) {
    if (!stride_range(*s[i])) return false;
    const bool keys = i == 1 || i == 2 || i >= 6;
    if (i >= 4 && !strides_zero(*s[i]) && !strides_apart(*s[i], d->B, keys ? d->Tk : d->Tq, keys ? d->Hk : d->Hq, d->D)) return false;
  }
  return true;
}
// Whether a backward takes all keys at once (k_attend_short), which needs no y.
inline bool attend_few_keys(const slstm_attend_dims* d) { return d->Tk >= 1 && d->Tk <= 128 && d->D <= 64; }
inline int attend_stats_width(const slstm_attend_dims* d) {
  return d->type == SLSTM_BF16 && !attend_few_keys(d) ? 2 + (d->D + 3) / 4 : 2;
}
inline AttendArgs attend_args(const slstm_attend_dims* d) {
  AttendArgs a = {};
  a.B = d->B, a.Tq = d->Tq, a.Tk = d->Tk, a.Hq = d->Hq, a.Hk = d->Hk, a.G = d->Hq / d->Hk, a.D = d->D;
  a.scale = d->scale, a.c = (float)((double)d->scale * 1.4426950408889634);
  const int Tq = d->Tq, Tk = d->Tk, Hq = d->Hq, Hk = d->Hk, D = d->D;
  a.sq = strides_of(d->q, Tq, Hq, D), a.sy = strides_of(d->y, Tq, Hq, D), a.sdy = strides_of(d->dy, Tq, Hq, D);
  a.sdq = strides_of(d->dq, Tq, Hq, D), a.sk = strides_of(d->k, Tk, Hk, D), a.sv = strides_of(d->v, Tk, Hk, D);
  a.sdk = strides_of(d->dk, Tk, Hk, D), a.sdv = strides_of(d->dv, Tk, Hk, D);
  a.splits = 1, a.width = attend_stats_width(d);
  return a;
}
// f(type, width): the kernels' variants.
template <typename F>
int attend_dispatch(const slstm_attend_dims* d, F f) {
  auto width = [&](auto t) {
    if (d->D <= 32) return f(t, std::integral_constant<int, 32>());
    if (d->D <= 64) return f(t, std::integral_constant<int, 64>());
    if (d->D <= 128) return f(t, std::integral_constant<int, 128>());
    return f(t, std::integral_constant<int, 256>());
  };
  return d->type == SLSTM_F32 ? width(float()) : width(bf16_t());
}
// A kernel's LDS limit is raised once to a device, not at every call.
inline hipError_t allow_lds(const void* kern, int lds, std::atomic<uint64_t>& devices) {
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
  if (bit && (devices.load(std::memory_order_relaxed) & bit)) return hipSuccess;
  const hipError_t s = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (s == hipSuccess) devices.fetch_or(bit, std::memory_order_relaxed);
  return s;
}
// Whether rows may go by DMA: whole granules of 16 bytes at aligned places, rows that do not overlap (a row behind the last is then
// past the descriptor's end), a tile of at most 64 (of few queries 128) rows within 2^31 bytes.
inline bool dma_ok(const slstm_attend_dims* d, const void* p, const slstm_strides& s) {
  const int e = d->type == SLSTM_F32 ? 4 : 2, V = 16 / e;
  return d->D % V == 0 && ((uintptr_t)p & 15u) == 0 && s.b % V == 0 && s.t % V == 0 && s.h % V == 0 && s.t >= d->D &&
         s.t * 128 * e < ((int64_t)1 << 31);
}
// All workgroups of a kernel, in as many launches as they need.
template <typename K>
hipError_t attend_launch(K kern, AttendArgs a, int64_t groups, int lds, std::atomic<uint64_t>& devices, hipStream_t st, int threads = 256) {
  if (lds > 65536) {
    const hipError_t e = allow_lds((const void*)kern, lds, devices);
    if (e != hipSuccess) return e;
  }
  // about eight runs to an XCD: of whole sequences (whose heads lie in the same cache lines) where there are 8 of them, of parts of a head's
  // tiles where there are few heads. Forward + backward us, like this, undealt, and in eight whole runs: 2 x 1000 x 1000, 64 heads of 64, bf16
  // 54 + 143, 64 + 149, 57 + 154; 64 x 240 x 240, 8 of 64, fp32 78 + 251, 82 + 253, 76 + 248; 2 x 4096 x 4000, 16 of 128 over 4, bf16 244 + 818, 240 + 815,
  // 276 + 925; 256 x 240 x 120, 8 of 64, bf16 48 + 109, 49 + 111, 48 + 107 (lengths ragged)
  const int64_t per = (int64_t)a.tiles * a.splits, heads = (int64_t)a.B * a.Hk;
  a.piece = a.B >= 8 ? per * a.Hk * (a.B >= 128 ? a.B / 64 : 1) : heads >= 64 ? per * (heads / 64) : (per + 64 / heads - 1) / (64 / heads);
  a.full = groups / (8 * a.piece) * (8 * a.piece);
  in_pieces(groups, kMostGroups, [&](int64_t g0, int64_t n) {
    a.first = g0;
    hipLaunchKernelGGL(kern, dim3((unsigned)n), dim3(threads), (size_t)lds, st, a);
  });
  return hipGetLastError();
}

}  // namespace
