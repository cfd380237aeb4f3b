// Linear layer with its epilogue, and its backward:
//   z = x W + b, y = act(z) + res;  dz = dy act'(z), dx = dz W^T, dW = x^T dz, db = sum over rows of dz
// All three products are C(m, n) = sum_k A(m, k) B(n, k) on the matrix units, 16x16 tiles (bf16: k of 32; fp32: the
// fp32 instruction, k of 4), fp32 sums. An operand lies in memory either by rows of k ("flat": x and dz of y and dx,
// W of dx) or with k as the row ("tall": W of y, both operands of dW). A flat operand's slice is kept in LDS by rows
// of 128 bytes and read 16 bytes a lane; a tall one's by its rows of k, and is read transposed (16-bit) or element by
// element (fp32). 16-byte granules are permuted within a row so that fragment reads spread over the banks.
// Slices reach LDS by DMA, a few slices ahead. That takes operands of whole 16-byte granules: those at odd places or
// of odd widths are first copied to padded rows in the work space (k_linear_pad; dz is written there anyhow). For few rows,
// where a copy of W would cost more than it gives, slices go through registers, with the rows' ends cut off there.
// Where the tiles do not fill the chip the sum over k is split, and k_linear_join adds the parts and applies the
// epilogue. Bound by the matrix units where rows are many: 61440 x 1024 x 4096 bf16 forward 691 us (746 TFLOP/s with gelu, z and
// residual, 2.3 GB past L2), dx 431 (1196), dW 436 (1182); 7680 x 500 x 333 f32 forward 37 us (69 TFLOP/s), dx and dW 64 (80); by W's
// bytes where they are few: 64 x 1024 x 32000 bf16 14.2 us (5.0 TB/s).
#include <algorithm>
#include <atomic>

#include "../../../include/stacklstm_head.h"
#include "head.h"

namespace {

struct GemmArgs {
  int M, N, K, splits, chunk;                          // chunk: k of a split, a whole number of slices
  const void *A, *B;
  int64_t lda, ldb;
  const void *bias, *res;
  void *y, *z;
  int64_t ldy, ldr;
  int act;
  float* part;                                         // [splits][M][N], NULL: none
  const void* dz;                                      // k_linear_any: z, where the operand that is dz is given as dy
  int64_t lddz;
  int dzact;
  const float* dbpart;                                 // dW: blocks of rows summed by workgroups behind the tiles, [dbrows][N]
  int tiles, dbrows;
  void* db;
};

// sigma(2 sqrt(2/pi) (z + 0.044715 z^3)): 1 / (1 + 2^(z (k + k3 z^2)))
__device__ __forceinline__ float gelu_gate(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * (z * z * -0.10294324f - 2.3022082f)));
}
// (1 - e) / (1 + e), e = 2^(-2 |z| log2 e), with z's sign; near 0, where 1 - e keeps few of z's bits, the series up to z^9 (the
// next term is 9e-9 of z at 0.25). Within 3e-7 of the value itself.
__device__ __forceinline__ float tanh_exp(float z) { return __builtin_amdgcn_exp2f(-2.8853900817779268f * fabsf(z)); }
__device__ __forceinline__ float tanh_act(float z) {
  const float e = tanh_exp(z), q = z * z;
  const float p = __builtin_fmaf(q, __builtin_fmaf(q, __builtin_fmaf(q, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f);
  const float far = copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), z);
  return fabsf(z) < 0.25f ? __builtin_fmaf(z * q, p, z) : far;
}
// (one branch for a vector)
template <int V>
__device__ __forceinline__ void act_fwd(float (&z)[V], int act) {
  auto each = [&](auto f) {
#pragma unroll
    for (int k = 0; k < V; ++k) z[k] = f(z[k]);
  };
  switch (act) {
    case SLSTM_ACT_RELU: each([](float v) { return v > 0.f ? v : v != v ? v : 0.f; }); break;
    case SLSTM_ACT_TANH: each([](float v) { return tanh_act(v); }); break;
    case SLSTM_ACT_SILU: each([](float v) { return v * sigmoidf_(v); }); break;
    case SLSTM_ACT_GELU: each([](float v) { return v * gelu_gate(v); }); break;
  }
}
// (tanh' = 1 / cosh^2; z/2 (1 + tanh u) = z sigma(2u); derivative of z sigma(2u): s + z s (1 - s) 2u')
template <int V>
__device__ __forceinline__ void act_bwd(float (&d)[V], const float (&z)[V], int act) {
  auto each = [&](auto f) {
#pragma unroll
    for (int k = 0; k < V; ++k) d[k] *= f(z[k]);
  };
  switch (act) {
    case SLSTM_ACT_RELU: each([](float v) { return v > 0.f ? 1.f : v != v ? v : 0.f; }); break;
    case SLSTM_ACT_TANH:
      each([](float v) {
        const float e = tanh_exp(v), r = __builtin_amdgcn_rcpf(1.f + e);
        return 4.f * e * r * r;
      });
      break;
    case SLSTM_ACT_SILU:
      each([](float v) {
        const float s = sigmoidf_(v);
        return s * (1.f + v * (1.f - s));
      });
      break;
    case SLSTM_ACT_GELU:
      each([](float v) {
        const float s = gelu_gate(v);
        // (s (1 - s) is 0 long before |z| = 64: the square of a large z stays finite beside it)
        return s + v * s * (1.f - s) * (1.5957691216057308f + 0.21406445f * fminf(v * v, 4096.f));
      });
      break;
  }
}

// 16 bytes of a row from its first element on; with ALL they are all there, else `left` elements are.
template <bool ALL, typename T>
__device__ __forceinline__ void put(T* row, int left, const float (&v)[vec<T>::N]) {
  if (ALL) *(u32x4_any*)row = vec<T>::pack(v);
  else store_vec(row, 0, left, v);
}
// One row piece of the epilogue: v[] at column n of row m, with its bias and residual.
template <bool ALL, typename T>
__device__ __forceinline__ void finish(const GemmArgs& g, int64_t m, int n, float (&v)[vec<T>::N], const float (&b)[vec<T>::N],
                                       u32x4 res) {
  constexpr int V = vec<T>::N;
  const int left = g.N - n;
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] += b[k];
  if (g.z) put<ALL>((T*)g.z + m * g.N + n, left, v);
  act_fwd(v, g.act);
  if (g.res) {
    float r[V];
    vec<T>::unpack(res, r);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] += r[k];
  }
  put<ALL>((T*)g.y + m * g.ldy + n, left, v);
}
template <typename T>
__device__ __forceinline__ void load_bias(const GemmArgs& g, int n, float (&b)[vec<T>::N]) {
  vec<T>::unpack(g.bias && n < g.N ? load_vec((const T*)g.bias + n, 0, g.N - n) : u32x4{0u, 0u, 0u, 0u}, b);
}
template <bool ALL, typename T>
__device__ __forceinline__ u32x4 load_res(const GemmArgs& g, int64_t m, int n) {
  const T* r = (const T*)g.res + m * g.ldr + n;
  return ALL ? *(const u32x4_any*)r : load_vec(r, 0, g.N - n);
}

// Sizes of a block tile. A slice of k is 128 bytes of each flat row, whole cache lines (64 bytes at a time took twice the
// requests: the product below at 1150 TFLOP/s instead of 1212); a step of it 64 bytes (32 k of 16 bits, 16 of fp32): one
// (four) matrix instructions of a pair of fragments.
constexpr int kSteps = 2;
template <typename T, int BM, int BN>
struct Tile {
  static constexpr int BK = 128 / (int)sizeof(T);
  static constexpr int NT = BM == 256 ? 512 : 256, WN = BM == 256 ? 4 : 2, WM = NT / 64 / WN;
  static constexpr int MI = BM / WM / 16, NJ = BN / WN / 16;
  static constexpr int ABYTES = BM * 128, BBYTES = BN * 128;
  static constexpr int IA = ABYTES / 16 / NT, IB = BBYTES / 16 / NT;       // granules of a thread
};

// Place of granule c of a slice's row r (flat: r a row of the operand, tall: r a k).
template <typename T, bool TALL, int ROWS>
__device__ __forceinline__ int swz(int r) {
  if constexpr (!TALL) return r & 7;
  else if constexpr (sizeof(T) == 4) return 4 * ((r >> 2) & 3);
  else if constexpr (ROWS >= 128) return 2 * ((r & 3) | (((r >> 3) & 1) << 2));
  else return 2 * (((r >> 1) & 1) | (((r >> 3) & 1) << 1));
}
// Row and granule (in memory) that thread position L of a slice holds.
template <typename T, bool TALL, int ROWS>
__device__ __forceinline__ void place(int L, int& r, int& c) {
  constexpr int G = TALL ? ROWS * (int)sizeof(T) / 16 : 8;
  r = L / G;
  c = (L % G) ^ swz<T, TALL, ROWS>(r);
}

// A lane's 16 bytes of k of one 16-row tile and step.
template <typename T> struct frag_of { typedef f32x4 type; };
template <> struct frag_of<bf16_t> { typedef bf16x8 type; };
template <typename T, bool TALL, int ROWS>
__device__ __forceinline__ typename frag_of<T>::type load_frag(const unsigned char* p, int tile, int step, int l16, int lq) {
  const int r = 16 * tile + l16;
  if constexpr (!TALL) {
    return *(const typename frag_of<T>::type*)(p + (r * 8 + ((4 * step + lq) ^ swz<T, TALL, ROWS>(r))) * 16);
  } else if constexpr (sizeof(T) == 2) {
    // transposed: the lane gives the address of k row 8 lq + l16 / 4 and columns 4 (l16 % 4) of the tile, and gets
    // column l16, four k
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    constexpr int G = ROWS / 8;
    const int k = 8 * lq + (l16 >> 2);
    const unsigned char* q = p + (step * 32 + k) * G * 16 + ((2 * tile + ((l16 & 3) >> 1)) ^ swz<T, TALL, ROWS>(k)) * 16 + (l16 & 1) * 8;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(q));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(q + 4 * G * 16));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    f32x4 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int k = 16 * step + 4 * lq + q;
      v[q] = *(const float*)(p + (k * (ROWS / 4) + ((r >> 2) ^ swz<T, TALL, ROWS>(k))) * 16 + (r & 3) * 4);
    }
    return v;
  }
}
// The products of row tile i of a step. C^T = B^T A^T: a lane holds row l16 and columns 4 lq .. 4 lq + 3 of a tile. (fp32:
// a lane's four k go to four instructions, for both operands alike.)
template <typename T, int NJ>
__device__ __forceinline__ void mma(const typename frag_of<T>::type& a, const typename frag_of<T>::type (&b)[NJ], f32x4 (&acc)[NJ]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[j] = mfma_bf16_16x16x32(b[j], a, acc[j]);
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[j][q], a[q], acc[j], 0, 0, 0);
  }
}

// Which tile and which part of k a workgroup has.
struct Where {
  int split, m0, n0, kbeg, kend, nr, nc;
};
template <int BM, int BN>
__device__ __forceinline__ Where where(const GemmArgs& g, int lid) {
  Where w;
  const int NTL = (g.N + BN - 1) / BN, MTL = (g.M + BM - 1) / BM, tiles = NTL * MTL, all = tiles * g.splits;
  // workgroups go to the 8 XCDs in turn: each XCD takes a contiguous run of tiles, in groups of 8 row tiles to a
  // column tile, so that what its L2 holds is used again
  const int full = all & ~7;
  if (lid < full) lid = (lid & 7) * (full >> 3) + (lid >> 3);
  w.split = uni(lid / tiles);
  lid -= w.split * tiles;
  constexpr int GM = 8;
  const int gi = lid / (GM * NTL), gm = min(GM, MTL - gi * GM), rem = lid - gi * GM * NTL;
  w.m0 = uni((gi * GM + rem % gm) * BM);               // (scalar registers: descriptors are made of them)
  w.n0 = uni((rem / gm) * BN);
  w.kbeg = min(g.K, w.split * g.chunk);
  w.kend = min(g.K, w.kbeg + g.chunk);
  w.nr = min(BM, g.M - w.m0);
  w.nc = min(BN, g.N - w.n0);
  return w;
}

// db: columns 32 b .. of the sums of P blocks of rows, by NT threads with NT floats of LDS.
template <typename T, int NT>
__device__ __forceinline__ void db_cols(const float* part, int P, int N, T* db, int b, float* red) {
  const int n = b * 32 + (threadIdx.x & 31), r = threadIdx.x >> 5;
  float s = 0.f;
  if (n < N) {
#pragma unroll 8
    for (int p = r; p < P; p += NT / 32) s += part[(int64_t)p * N + n];
  }
  red[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x >= 32 || n >= N) return;
  float v = 0.f;
#pragma unroll
  for (int k = 0; k < NT / 32; ++k) v += red[32 * k + threadIdx.x];
  from_f32(db[n], v);
}

// Results of a tile from the accumulators. A lane holds four columns (4 lq ..) of row l16 of every 16x16 tile: 16 bytes of an
// fp32 output; for a 16-bit one neighbouring column tiles exchange rows of lanes, so that a lane has eight columns of one of
// them. Either way an instruction writes 64 bytes of 16 rows. The residual's loads all go out first: one after the other they
// took half the time of a tile (61440 x 1024 x 4096, gelu, z, residual: 913 us, then 754; 690 without a way through LDS).
template <bool ALL, typename T, int MI, int NJ>
__device__ __forceinline__ void results(const GemmArgs& g, const Where& w, f32x4 (&acc)[MI][NJ], int wm, int wn, int l16, int lq) {
  constexpr int V = vec<T>::N, P = V == 4 ? NJ : NJ / 2;         // pieces of a row tile
  int n[P];
  float bias[P][V];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    n[p] = w.n0 + 16 * NJ * wn + (V == 4 ? 16 * p + 4 * lq : 16 * (2 * p + (lq & 1)) + 8 * (lq >> 1));
    load_bias<T>(g, n[p], bias[p]);
  }
  auto in = [&](int i, int p) { return ALL || (16 * (MI * wm + i) + l16 < w.nr && n[p] < g.N); };
  u32x4 res[MI][P];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int p = 0; p < P; ++p)
      res[i][p] = g.res && in(i, p) ? load_res<ALL, T>(g, w.m0 + 16 * (MI * wm + i) + l16, n[p]) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < MI; ++i) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      float v[V];
      if constexpr (V == 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = acc[i][p][k];
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][2 * p][k]), __float_as_uint(acc[i][2 * p + 1][k]), false, false);
          v[k] = __uint_as_float(s[0]);
          v[k + 4] = __uint_as_float(s[1]);
        }
      }
      if (in(i, p)) finish<ALL, T>(g, w.m0 + 16 * (MI * wm + i) + l16, n[p], v, bias[p], res[i][p]);
    }
  }
}
template <typename T, int MI, int NJ, int BM, int BN>
__device__ __forceinline__ void epilogue(const GemmArgs& g, const Where& w, f32x4 (&acc)[MI][NJ], int wm, int wn, int l16, int lq) {
  if (g.part) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int m = 16 * (MI * wm + i) + l16, n = w.n0 + 16 * (NJ * wn + j) + 4 * lq;
        const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
        if (m < w.nr && n < g.N) store_vec(g.part + ((int64_t)w.split * g.M + w.m0 + m) * g.N + n, 0, g.N - n, v);
      }
  } else if (w.nr == BM && w.nc == BN) {
    results<true, T, MI, NJ>(g, w, acc, wm, wn, l16, lq);
  } else {
    results<false, T, MI, NJ>(g, w, acc, wm, wn, l16, lq);
  }
}

// The DMA of an operand's slices: a lane's offsets are the same in every slice. Flat: the slice's start goes into the scalar
// offset, and a lane past the end of k reads nothing; tall: into the descriptor's base, whose end stops rows past it.
template <typename T, bool TALL, int ROWS, int NT, int I>
struct Mover {
  uint32_t off[I];
  int col[I];                                          // flat: first k of the lane's granule
  const T* base;
  int64_t ld;
  rsrc_t rs;
  int n;
  __device__ __forceinline__ void start(const T* p, int64_t ld_, int n_, int k, int wave, int lane) {
    constexpr int V = vec<T>::N;
    base = p, ld = ld_, n = n_;
#pragma unroll
    for (int i = 0; i < I; ++i) {
      int r, c;
      place<T, TALL, ROWS>((i * (NT / 64) + wave) * 64 + lane, r, c);
      col[i] = c * V;
      off[i] = (TALL ? c * V < n : r < n) ? (uint32_t)(r * (int)ld + c * V) * (uint32_t)sizeof(T) : kOOB;
    }
    // (rows are whole granules in memory: a padded one's last is there)
    if (!TALL) rs = make_rsrc(base, (size_t)((n - 1) * ld + (k + V - 1) / V * V) * sizeof(T));
  }
  // slice at k0 of a k that ends at kend
  __device__ __forceinline__ void slice(int k0, int kend) {
    constexpr int V = vec<T>::N, BK = 128 / (int)sizeof(T);
    if (TALL) {
      const int rows = uni(max(0, min(BK, kend - k0)));
      // (no row: a descriptor of no bytes)
      rs = make_rsrc(base + (int64_t)k0 * ld, (size_t)(rows * ld - (rows > 0 ? ld - (n + V - 1) / V * V : 0)) * sizeof(T));
    }
  }
  __device__ __forceinline__ void go(int i, int k0, int kend, unsigned char* to, int wave) {
    uint32_t o = off[i], so = 0;
    if (!TALL) {
      o = k0 + col[i] < kend ? o : kOOB;
      so = __builtin_amdgcn_readfirstlane((uint32_t)k0 * (uint32_t)sizeof(T));
      asm volatile("" : "+s"(so));                     // (in a register: the instruction takes no literal there)
    }
    bdma16(rs, o, so, lds_addr(to + (i * (NT / 64) + wave) * 1024));
  }
};

}  // namespace

// Operands of whole granules, by DMA into SA and SB stages of LDS. A row tile's fragment of the next step is read as soon as
// its products of this step are issued, so reads from LDS go along with the products; the columns' fragments have two sets.
// In a slice's last step the waves meet: the next slice has landed, everybody has read what it needs of this one, and its
// stages take later slices. The operand that comes from memory (the other one is read again and again from L2) is further
// ahead: three stages of it and two of the other fill a CU's LDS at 256 x 256.
// dx of 61440 x 1024 x 4096, bf16, random values: 1196 TFLOP/s (the best launch 1250); with fragments read at the start of each
// slice and two stages of either operand 1090.
template <typename T, bool AT, bool BT, int BM, int BN, int SA, int SB>
__device__ __forceinline__ void dma_tile(const GemmArgs& g, int lid) {
  typedef Tile<T, BM, BN> S;
  typedef typename frag_of<T>::type frag;
  constexpr int BK = S::BK, NT = S::NT, MI = S::MI, NJ = S::NJ, MEET = MI >= 4 ? 1 : 0;
  static_assert(SA - SB <= 1 && SB - SA <= 1 && SA >= 2 && SB >= 2, "stages");
  extern __shared__ __align__(16) unsigned char sm[];
  if constexpr (AT)
    if (lid >= g.tiles) return db_cols<T, NT>(g.dbpart, g.dbrows, g.N, (T*)g.db, lid - g.tiles, (float*)sm);
  const Where w = where<BM, BN>(g, lid);
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN, l16 = lane & 15, lq = lane >> 4;
  Mover<T, AT, BM, NT, S::IA> ma;
  Mover<T, BT, BN, NT, S::IB> mb;
  ma.start((const T*)g.A + (AT ? w.m0 : (int64_t)w.m0 * g.lda), g.lda, w.nr, g.K, wave, lane);
  mb.start((const T*)g.B + (BT ? w.n0 : (int64_t)w.n0 * g.ldb), g.ldb, w.nc, g.K, wave, lane);
  auto stage_a = [&](int i) { return sm + i * S::ABYTES; };
  auto stage_b = [&](int i) { return sm + SA * S::ABYTES + i * S::BBYTES; };
  auto move_a = [&](int i, int k0, int buf) { ma.go(i, k0, w.kend, stage_a(buf), wave); };
  auto move_b = [&](int i, int k0, int buf) { mb.go(i, k0, w.kend, stage_b(buf), wave); };
  f32x4 acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < (SA > SB ? SA : SB); ++s) {
    const int k = w.kbeg + s * BK;
    if (s < SA) {
      ma.slice(k, w.kend);
#pragma unroll
      for (int i = 0; i < S::IA; ++i) move_a(i, k, s);
    }
    if (s < SB) {
      mb.slice(k, w.kend);
#pragma unroll
      for (int i = 0; i < S::IB; ++i) move_b(i, k, s);
    }
  }
  frag a[MI], b[2][NJ];
  auto read_a = [&](const unsigned char* st, int step, int i) { a[i] = load_frag<T, AT, BM>(st, MI * wm + i, step, l16, lq); };
  auto read_b = [&](const unsigned char* st, int step, frag (&f)[NJ]) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) f[j] = load_frag<T, BT, BN>(st, NJ * wn + j, step, l16, lq);
  };
  wait_vm<(SA - 1) * S::IA + (SB - 1) * S::IB>();
  __syncthreads();                                     // the first slice landed
  // (in the loop's order: a wait at its head holds for both ways in)
  __builtin_amdgcn_s_waitcnt(0xc07f);
  read_b(stage_b(0), 0, b[0]);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    read_a(stage_a(0), 0, i);
    __builtin_amdgcn_sched_barrier(0);
  }
  int ia = 0, ib = 0;                                  // stages of the slice at k0
  for (int k0 = w.kbeg; k0 < w.kend; k0 += BK) {
    const int na = ia + 1 == SA ? 0 : ia + 1, nb = ib + 1 == SB ? 0 : ib + 1;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const bool last = s + 1 == kSteps;
      const unsigned char *pa = stage_a(last ? na : ia), *pb = stage_b(last ? nb : ib);
      const int step = last ? 0 : s + 1;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        mma<T, NJ>(a[i], b[s & 1], acc[i]);
        if (i == MEET) {
          if (last) {
            wait_vm<(SA - 2) * S::IA + (SB - 2) * S::IB>();
            __syncthreads();
            ma.slice(k0 + SA * BK, w.kend);
            mb.slice(k0 + SB * BK, w.kend);
          }
          read_b(pb, step, b[(s & 1) ^ 1]);
#pragma unroll
          for (int h = 0; h <= MEET; ++h) read_a(pa, step, h);
        } else if (i > MEET) {
          read_a(pa, step, i);
        }
        // DMAs, a few behind each row tile: the nearer slice's first
        if (last && i >= MEET) {
          constexpr int PER = S::IA + S::IB, PARTS = MI - MEET;
          const int p0 = (i - MEET) * PER / PARTS, p1 = (i - MEET + 1) * PER / PARTS;
#pragma unroll
          for (int p = 0; p < PER; ++p) {
            if (p < p0 || p >= p1) continue;
            if (SA >= SB) {
              if (p < S::IB) move_b(p, k0 + SB * BK, ib);
              else move_a(p - S::IB, k0 + SA * BK, ia);
            } else {
              if (p < S::IA) move_a(p, k0 + SA * BK, ia);
              else move_b(p - S::IA, k0 + SB * BK, ib);
            }
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    ia = na;
    ib = nb;
  }
  wait_vm<0>();                                        // (DMAs past the end of k write zeros to LDS: all are done before it is given up)
  epilogue<T, MI, NJ, BM, BN>(g, w, acc, wm, wn, l16, lq);
}

template <typename T, bool AT, bool BT, int BM, int BN, int SA, int SB>
__global__ void __launch_bounds__((Tile<T, BM, BN>::NT), 2) k_linear(GemmArgs g) {
  dma_tile<T, AT, BT, BM, BN, SA, SB>(g, (int)blockIdx.x);
}
// dx and dW (and db) in one launch: the first x.tiles workgroups take dx.
template <typename T, int TILE, int SA, int SB>
__global__ void __launch_bounds__((Tile<T, TILE, TILE>::NT), 2) k_linear_both(GemmArgs x, GemmArgs w) {
  const int b = (int)blockIdx.x;
  if (b < x.tiles) dma_tile<T, false, false, TILE, TILE, SA, SB>(x, b);
  else dma_tile<T, true, true, TILE, TILE, SA, SB>(w, b - x.tiles);
}

// Operands at any place, through registers, one slice ahead; two stages. A slice's loads all go out before the first is
// waited for; rows are cut to their ends, and zeros put behind them, on the way to LDS. With DZ an operand is dy act'(z),
// made on that way too (rounded to T, as a stored one is): A of dx, B of dW.
template <typename T, bool AT, bool BT, int BM, int BN, bool DZ>
__device__ __forceinline__ void any_tile(const GemmArgs& g, int lid) {
  typedef Tile<T, BM, BN> S;
  typedef typename frag_of<T>::type frag;
  constexpr int BK = S::BK, NT = S::NT, MI = S::MI, NJ = S::NJ;
  constexpr bool DA = DZ && !BT, DB = DZ && AT;
  extern __shared__ __align__(16) unsigned char sm[];
  const Where w = where<BM, BN>(g, lid);
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN, l16 = lane & 15, lq = lane >> 4;
  const T* A = (const T*)g.A + (AT ? w.m0 : (int64_t)w.m0 * g.lda);
  const T* B = (const T*)g.B + (BT ? w.n0 : (int64_t)w.n0 * g.ldb);
  [[maybe_unused]] const T* Z = (const T*)g.dz + (!BT ? (int64_t)w.m0 * g.lddz : w.n0);
  u32x4 ra[S::IA], rb[S::IB], rz[DA ? S::IA : DB ? S::IB : 1];
  // f(i, row, granule): granule i of the thread; rows past the last are the last one (their results are not stored, or they
  // are taken out of the slice)
  auto each = [&](auto tall, auto rows, auto n, auto f) {
    constexpr bool TALL = decltype(tall)::value;
#pragma unroll
    for (int i = 0; i < decltype(n)::value; ++i) {
      int r, c;
      place<T, TALL, decltype(rows)::value>(i * NT + tid, r, c);
      f(i, r, c);
    }
  };
  typedef std::bool_constant<AT> at;
  typedef std::bool_constant<BT> bt;
  typedef std::integral_constant<int, BM> bm;
  typedef std::integral_constant<int, BN> bn;
  typedef std::integral_constant<int, S::IA> na;
  typedef std::integral_constant<int, S::IB> nb;
  // A granule's row, and the row's elements from the slice (flat) or the tile (tall) on.
  auto spot = [&](auto tall, const T* p, int64_t ld, int k0, int rows, int r) {
    const int left = w.kend - k0, rr = min(r, (decltype(tall)::value ? left : rows) - 1);
    return p + (decltype(tall)::value ? (int64_t)(k0 + rr) * ld : (int64_t)rr * ld + k0);
  };
  auto fetch = [&](int k0) {
    const int left = w.kend - k0;
    each(at(), bm(), na(), [&](int i, int r, int c) {
      ra[i] = fetch_vec(spot(at(), A, g.lda, k0, w.nr, r), c, AT ? w.nr : left);
      if constexpr (DA)
        if (g.dz) rz[i] = fetch_vec(spot(at(), Z, g.lddz, k0, w.nr, r), c, left);
    });
    each(bt(), bn(), nb(), [&](int i, int r, int c) {
      rb[i] = fetch_vec(spot(bt(), B, g.ldb, k0, w.nc, r), c, BT ? w.nc : left);
      if constexpr (DB)
        if (g.dz) rz[i] = fetch_vec(spot(bt(), Z, g.lddz, k0, w.nc, r), c, w.nc);
    });
  };
  auto through = [&](u32x4& dy, u32x4 z) {
    float d[vec<T>::N], v[vec<T>::N];
    vec<T>::unpack(dy, d);
    vec<T>::unpack(z, v);
    act_bwd(d, v, g.dzact);
    dy = vec<T>::pack(d);
  };
  f32x4 acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (w.kbeg < w.kend) fetch(w.kbeg);
  int buf = 0;
  for (int k0 = w.kbeg; k0 < w.kend; k0 += BK, buf ^= 1) {
    unsigned char* st = sm + buf * (S::ABYTES + S::BBYTES);
    const int left = w.kend - k0;
    const bool cut_a = left < BK || w.nr < BM, cut_b = left < BK || w.nc < BN;
    each(at(), bm(), na(), [&](int i, int r, int c) {
      u32x4 v = ra[i];
      if (cut_a) v = place_vec<T>(v, c, AT ? w.nr : left);
      if constexpr (DA)
        if (g.dz) through(v, cut_a ? place_vec<T>(rz[i], c, left) : rz[i]);
      if (AT && r >= left) v = u32x4{0u, 0u, 0u, 0u};
      *(u32x4*)(st + (i * NT + tid) * 16) = v;
    });
    each(bt(), bn(), nb(), [&](int i, int r, int c) {
      u32x4 v = rb[i];
      if (cut_b) v = place_vec<T>(v, c, BT ? w.nc : left);
      if constexpr (DB)
        if (g.dz) through(v, cut_b ? place_vec<T>(rz[i], c, w.nc) : rz[i]);
      if (BT && r >= left) v = u32x4{0u, 0u, 0u, 0u};
      *(u32x4*)(st + S::ABYTES + (i * NT + tid) * 16) = v;
    });
    __syncthreads();
    if (k0 + BK < w.kend) fetch(k0 + BK);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      frag a[MI], b[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) b[j] = load_frag<T, BT, BN>(st + S::ABYTES, NJ * wn + j, s, l16, lq);
#pragma unroll
      for (int i = 0; i < MI; ++i) a[i] = load_frag<T, AT, BM>(st, MI * wm + i, s, l16, lq);
#pragma unroll
      for (int i = 0; i < MI; ++i) mma<T, NJ>(a[i], b, acc[i]);
    }
  }
  epilogue<T, MI, NJ, BM, BN>(g, w, acc, wm, wn, l16, lq);
}
template <typename T, bool AT, bool BT, int BM, int BN>
__global__ void __launch_bounds__((Tile<T, BM, BN>::NT), 2) k_linear_any(GemmArgs g) {
  extern __shared__ __align__(16) unsigned char sm[];
  if constexpr (AT)
    if ((int)blockIdx.x >= g.tiles)
      return db_cols<T, Tile<T, BM, BN>::NT>(g.dbpart, g.dbrows, g.N, (T*)g.db, (int)blockIdx.x - g.tiles, (float*)sm);
  any_tile<T, AT, BT, BM, BN, false>(g, (int)blockIdx.x);
}

// The parts of a split product, and the epilogue: 64 vectors to a workgroup, each wave adds every fourth part, the first one the
// waves' sums, always in the same order (dW of 26751 x 176 x 416 bf16: 6.9 us; with all parts added by one wave 18).
template <typename T>
__global__ void __launch_bounds__(256) k_linear_join(GemmArgs g, int64_t first) {
  constexpr int V = vec<T>::N;
  __shared__ float red[3][V][64];
  const int nv = (g.N + V - 1) / V, q = threadIdx.x >> 6, l = threadIdx.x & 63;
  const int64_t all = (int64_t)g.M * nv, at = first + (int64_t)blockIdx.x * 64 + l, i = min(at, all - 1), m = i / nv;
  const int n = (int)(i - m * nv) * V;
  float b[V], v[V];
  u32x4 res = {0u, 0u, 0u, 0u};
  if (q == 0) {
    load_bias<T>(g, n, b);
    if (g.res) res = load_res<false, T>(g, m, n);
  }
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = 0.f;
#pragma unroll 8
  for (int s = q; s < g.splits; s += 4) {
    const float* p = g.part + ((int64_t)s * g.M + m) * g.N + n;
#pragma unroll
    for (int k = 0; k < V; k += 4) {
      float w[4];
      vec<float>::unpack(load_vec(p, k / 4, g.N - n), w);
#pragma unroll
      for (int h = 0; h < 4; ++h) v[k + h] += w[h];
    }
  }
  if (q) {
#pragma unroll
    for (int k = 0; k < V; ++k) red[q - 1][k][l] = v[k];
  }
  __syncthreads();
  if (q || at >= all) return;
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] += red[0][k][l] + red[1][k][l] + red[2][k][l];
  finish<false, T>(g, m, n, v, b, res);
}

namespace {
struct DzArgs {
  int M, N, act, rows;                                 // rows of a workgroup
  const void *dy, *z;
  int64_t ldd, ldz;
  void *dz, *lo;                                       // dz NULL: dy serves; lo: what rounding took off dz, or NULL
  float* part;                                         // [row blocks][N], NULL: no sums, or
  void* db;                                            // one block of rows: the sums themselves
};
// CV column vectors (strip bx) of a block of rows (by), 256 / CV rows at a time and the loads of four such steps together: a row
// after the other, each with a wait, 128 rows of 520 took 23 us.
template <typename T, int CV>
__device__ __forceinline__ void dz_strip(const DzArgs& a, int bx, int by) {
  constexpr int V = vec<T>::N, R = 256 / CV, U = 4;
  __shared__ float red[R][CV * V + 4];
  const int t = threadIdx.x % CV, c = bx * CV + t, r = threadIdx.x / CV;
  const int64_t lo = (int64_t)by * a.rows, hi = min((int64_t)a.M, lo + a.rows);
  float s[V];
#pragma unroll
  for (int k = 0; k < V; ++k) s[k] = 0.f;
  if (c * V < a.N) {
    for (int64_t m = lo + r; m < hi; m += U * R) {
      u32x4 rd[U], rz[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t n = min(m + u * R, hi - 1);
        rd[u] = fetch_vec((const T*)a.dy + n * a.ldd, c, a.N);
        if (a.z) rz[u] = fetch_vec((const T*)a.z + n * a.N, c, a.N);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t n = m + u * R;
        if (n >= hi) break;
        float d[V];
        vec<T>::unpack(place_vec<T>(rd[u], c, a.N), d);
        if (a.z) {
          float z[V];
          vec<T>::unpack(place_vec<T>(rz[u], c, a.N), z);
          act_bwd(d, z, a.act);
        }
#pragma unroll
        for (int k = 0; k < V; ++k) s[k] += d[k];
        if (a.dz) store_vec((T*)a.dz + n * a.ldz, c, (int)a.ldz, d);     // (zeros to the end of the padded row)
        if (a.lo) {
          float hi[V];
          vec<T>::unpack(vec<T>::pack(d), hi);
#pragma unroll
          for (int k = 0; k < V; ++k) d[k] = fabsf(hi[k]) < INFINITY ? d[k] - hi[k] : 0.f;
          store_vec((T*)a.lo + n * a.ldz, c, (int)a.ldz, d);
        }
      }
    }
  }
  if (!a.part && !a.db) return;
#pragma unroll
  for (int k = 0; k < V; ++k) red[r][t * V + k] = s[k];
  __syncthreads();
  for (int i = threadIdx.x; i < CV * V; i += 256) {
    const int n = bx * CV * V + i;
    if (n >= a.N) continue;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < R; ++k) v += red[k][i];
    if (a.db) from_f32(((T*)a.db)[n], v);
    else a.part[(int64_t)by * a.N + n] = v;
  }
}

struct PadArgs {
  struct {
    const void* src;
    void* dst;
    int64_t rows, ld;
    int cols;
  } op[2];
  uint32_t first;                                      // first workgroup of the second
};
// Rows copied to rows of whole granules, zeros behind their ends; kPad granules to a workgroup, whatever rows they lie in (16
// rows to one: 3035 x 395 x 26869 f32 with a residual 728 us instead of 609).
constexpr int kPad = 1024;
template <typename T>
__device__ __forceinline__ void pad_rows(const PadArgs& a, uint32_t b) {
  constexpr int V = vec<T>::N, U = kPad / 256;
  const bool second = b >= a.first;
  const auto& o = a.op[second];
  const uint32_t nv = (o.cols + V - 1) / V;
  const int64_t i0 = (int64_t)(b - (second ? a.first : 0)) * kPad, r0 = i0 / nv;
  const uint32_t c0 = (uint32_t)(i0 - r0 * nv), n = (uint32_t)min((int64_t)kPad, o.rows * nv - i0);
  u32x4 v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t j = c0 + min(threadIdx.x + 256 * u, n - 1);
    v[u] = fetch_vec((const T*)o.src + (r0 + j / nv) * o.ld, (int)(j % nv), o.cols);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t i = threadIdx.x + 256 * u;
    if (i < n) *(u32x4*)((T*)o.dst + (i0 + i) * V) = place_vec<T>(v[u], (int)((c0 + i) % nv), o.cols);
  }
}
}  // namespace

// dz = dy act'(z), and the sums of its columns over a block of rows, by the first nd workgroups; copies by the others.
template <typename T, int CV>
__global__ void __launch_bounds__(256) k_linear_dz(DzArgs a, int strips, int nd, PadArgs p) {
  const int b = (int)blockIdx.x;
  if (b < nd) dz_strip<T, CV>(a, b % strips, b / strips);
  else pad_rows<T>(p, (uint32_t)(b - nd));
}
template <typename T>
__global__ void __launch_bounds__(256) k_linear_pad(PadArgs a) {
  pad_rows<T>(a, blockIdx.x);
}

// A whole backward of few rows in one launch: nx tiles of dx, nw of dW, then strips of db; dz is made where it is read.
template <typename T>
__global__ void __launch_bounds__(256, 2) k_linear_few(GemmArgs x, GemmArgs w, DzArgs a, int nx, int nw) {
  const int b = (int)blockIdx.x;
  if (b < nx) any_tile<T, false, false, 64, 64, true>(x, b);
  else if (b < nx + nw) any_tile<T, true, true, 64, 64, true>(w, b - nx);
  else dz_strip<T, 8>(a, b - nx - nw, 0);
}

// db where no dW is asked for.
template <typename T>
__global__ void __launch_bounds__(256) k_linear_db(const float* part, int P, int N, T* db) {
  __shared__ float red[256];
  db_cols<T, 256>(part, P, N, db, (int)blockIdx.x, red);
}

namespace {

bool al16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
// How a product runs: block tile, parts of k.
struct Plan {
  int tile, splits, chunk;
  double us;                                           // estimated
};
// A CU's TFLOP/s with as many workgroups of a tile as it holds, and the us of a slice where there are few.
struct TileCost {
  double rate, latency;
  int held;
};
TileCost tile_cost(bool f32, int t) {
  return {f32 ? (t == 128 ? 0.56 : 0.52) : t == 256 ? 4.2 : t == 128 ? 3.0 : 2.2, f32 ? 0.45 : 0.35, t == 256 ? 1 : t == 128 ? 2 : 3};
}
double join_us(int64_t M, int64_t N, int64_t s) { return s > 1 ? 5 + (s + 1) * (double)M * N * 4 / 7e6 : 0; }
// The tile and the split with the least estimated time, in us: a CU's share of the products at the tile's rate (TFLOP/s of a
// CU with as many workgroups as it holds: a smaller tile reads more operands to a product), or a workgroup's slices at
// the latency of one where there are few; split parts are written, read once more and take a launch. Over 99 products
// (rows 16 to 61440, k and columns 48 to 32000) the choice takes 1.03 times the best of 64, 128, 256 and splits of 1 to 64
// in the geometric mean, 1.28 times at most.
Plan gemm_plan(int64_t M, int64_t N, int64_t K, int type, bool wide) {
  const bool f32 = type == SLSTM_F32;
  const int BK = f32 ? 32 : 64;
  const int64_t slices = std::max<int64_t>(1, (K + BK - 1) / BK);
  Plan best = {64, 1, (int)(slices * BK), 1e300};
  for (int t = wide && !f32 ? 256 : 128; t >= 64; t /= 2) {
    const TileCost c = tile_cost(f32, t);
    const int64_t tiles = ((M + t - 1) / t) * ((N + t - 1) / t);
    for (int64_t s = 1; s <= 64 && (s == 1 || (slices / s >= 4 && tiles * s <= 2048)); ++s) {
      const int64_t per = (slices + s - 1) / s, n = tiles * s;
      if ((slices + per - 1) / per != s) continue;
      const double us = 2 + std::max(((n + 255) / 256) * (2e-6 * t * t * per * BK / c.rate), ((n + 256 * c.held - 1) / (256 * c.held)) * per * c.latency) +
                        join_us(M, N, s);
      if (us < best.us) best = {t, (int)s, (int)(per * BK), us};
    }
  }
  return best;
}
// dx [M, K] and dW [K, N] in one launch: tile and dW's split (us 1e300: not to be). Their workgroups share the CUs, so the whole
// rounds and the last one's waits of two launches become one sum of work.
Plan both_plan(int64_t M, int64_t K, int64_t N, int type) {
  const bool f32 = type == SLSTM_F32;
  const int BK = f32 ? 32 : 64;
  const int64_t sx = (N + BK - 1) / BK, sw = std::max<int64_t>(1, (M + BK - 1) / BK);
  Plan best = {64, 1, (int)(sw * BK), 1e300};
  for (int t = 128; t >= 64; t /= 2) {
    const TileCost c = tile_cost(f32, t);
    const int64_t tx = ((M + t - 1) / t) * ((K + t - 1) / t), tw = ((K + t - 1) / t) * ((N + t - 1) / t);
    if (tx + tw > 1 << 20) continue;
    for (int64_t s = 1; s <= 64 && (s == 1 || (sw / s >= 4 && tw * s <= 2048)); ++s) {
      const int64_t per = (sw + s - 1) / s;
      if ((sw + per - 1) / per != s) continue;
      const double slice = 2e-6 * t * t * BK / c.rate;
      const double share = std::min<double>(c.held, (tx + tw * s + 255) / 256);      // workgroups that a CU holds together
      const double us = 2 + std::max((tx * sx + tw * s * per) * slice / 256 + 0.5 * per * slice, std::max(sx, per) * std::max(c.latency, share * slice)) +
                        join_us(K, N, s);
      if (us < best.us) best = {t, (int)s, (int)(per * BK), us};
    }
  }
  return best;
}
size_t part_bytes(const Plan& p, int64_t M, int64_t N) {
  return p.splits > 1 ? ((size_t)p.splits * M * N * 4 + 255) & ~(size_t)255 : 0;
}
// Either way of staging: the work space does not depend on the arrays' alignment.
size_t gemm_bytes(int64_t M, int64_t N, int64_t K, int type) {
  const size_t a = part_bytes(gemm_plan(M, N, K, type, false), M, N);
  return type == SLSTM_F32 ? a : std::max(a, part_bytes(gemm_plan(M, N, K, type, true), M, N));
}
// The parts of a product with dz in two planes.
size_t wide_bytes(int64_t M, int64_t N, int64_t K, int type) {
  const int splits = std::max(gemm_plan(M, N, K, type, false).splits, gemm_plan(M, N, K, type, true).splits);
  return (size_t)2 * splits * M * N * 4;
}

// A kernel's LDS limit is raised once to a device, not at every call.
hipError_t allow_lds(const void* kern, int lds, std::atomic<uint64_t>& devices) {
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
  if (bit && (devices.load(std::memory_order_relaxed) & bit)) return hipSuccess;
  const hipError_t s = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (s == hipSuccess) devices.fetch_or(bit, std::memory_order_relaxed);
  return s;
}
// T the operands' type, AT: whether A has k as the row. Products with more tiles than a launch may have workgroups are not split
// over k; they go out in several launches of whole rows of tiles.
template <typename T, bool AT>
hipError_t tile_launch(const void* kern, const GemmArgs& g, int tile, int threads, int lds, std::atomic<uint64_t>& devices, hipStream_t st) {
  if (lds > 65536) {
    const hipError_t e = allow_lds(kern, lds, devices);
    if (e != hipSuccess) return e;
  }
  const int64_t across = ((int64_t)g.N + tile - 1) / tile * g.splits;
  hipError_t e = hipSuccess;
  in_pieces(g.M, tile * std::max<int64_t>(1, kMostGroups / across), [&](int64_t m0, int64_t m) {
    GemmArgs a = g;
    a.M = (int)m;
    a.tiles = (int)((m + tile - 1) / tile * across);
    a.A = (const T*)g.A + (AT ? m0 : m0 * g.lda);
    a.y = offset((T*)g.y, m0 * g.ldy), a.z = offset((T*)g.z, m0 * g.N), a.res = offset((const T*)g.res, m0 * g.ldr);
    a.part = offset(g.part, m0 * g.N);                 // (of one split, where m0 is not 0)
    if (m0) a.dbpart = nullptr;
    void* args[] = {&a};
    if (e == hipSuccess)
      e = hipLaunchKernel(kern, dim3((unsigned)(a.tiles + (a.dbpart ? (g.N + 31) / 32 : 0))), dim3(threads), args, lds, st);
  });
  return e;
}
template <typename T, bool AT, bool BT, int TILE, int SA, int SB>
hipError_t launch_dma(const GemmArgs& g, hipStream_t st) {
  typedef Tile<T, TILE, TILE> S;
  static std::atomic<uint64_t> devices;
  return tile_launch<T, AT>((const void*)k_linear<T, AT, BT, TILE, TILE, SA, SB>, g, TILE, S::NT, S::ABYTES * SA + S::BBYTES * SB, devices, st);
}
template <typename T, bool AT, bool BT, int TILE>
hipError_t launch_any(const GemmArgs& g, hipStream_t st) {
  typedef Tile<T, TILE, TILE> S;
  static std::atomic<uint64_t> devices;
  return tile_launch<T, AT>((const void*)k_linear_any<T, AT, BT, TILE, TILE>, g, TILE, S::NT, (S::ABYTES + S::BBYTES) * 2, devices, st);
}

// A matrix of rows as a product reads it. whole: its rows are whole granules at aligned places, in reach of a
// descriptor's 32-bit offsets (in a padded copy: with zeros behind the row's end).
struct Operand {
  const void* p;
  int64_t ld;
  bool whole;
};
int granule(int type) { return type == SLSTM_F32 ? 4 : 8; }
size_t esize(int type) { return type == SLSTM_F32 ? 4 : 2; }
int64_t padded(int64_t cols, int type) { return (cols + granule(type) - 1) / granule(type) * granule(type); }
constexpr int64_t kReach = 1 << 21;
bool dims_whole(int64_t cols, int64_t ld, int type) { return cols % granule(type) == 0 && ld % granule(type) == 0 && ld <= kReach; }
Operand as_is(const void* p, int64_t cols, int64_t ld, int type) { return {p, ld, al16(p) && dims_whole(cols, ld, type)}; }
// Whether matrices at odd places are copied for this many rows of x, and a copy's bytes (by the dims alone). Copied, and through
// registers as they are, a training pass of 300 x 333 x 83 f32 37.4 and 46.8 us, 700 x 777 x 1001 bf16 37.8 and 53.4, 129 x 85
// x 46 f32 25.2 and 26.6; 4000 x 333 x 777 f32 121 and 179.
bool copies(int64_t M) { return M > 128; }
bool needs_copy(int64_t M, int64_t cols, int64_t ld, int type) {
  return copies(M) && !dims_whole(cols, ld, type) && padded(cols, type) <= kReach;
}
// A backward in one launch (k_linear_few): up to 128 rows, and a sum of dx over N of at most 8 slices, which take the latency
// of a load and of act' each. (A training pass of 3 x 16 x 16: 22.6 us with a launch for each of dz, dx and dW, 13.7 in one. 128
// x 512 in, gelu: 256 out in one 17.6 us, 260 out in three 5.0 + 9.4 + 5.9; 380 out in one 24.7.)
bool few_rows(const slstm_linear_dims* d) {
  return d->M > 0 && d->M <= 128 && d->N <= (d->type == SLSTM_F32 ? 256 : 512);
}
size_t copy_bytes(int64_t rows, int64_t cols, int type) { return ((size_t)rows * padded(cols, type) * esize(type) + 255) & ~(size_t)255; }

// Copies of up to two matrices in one launch.
struct Copies {
  PadArgs a = {};
  int n = 0;
  int64_t blocks = 0;
  Operand add(const void* src, int64_t rows, int64_t cols, int64_t ld, void* dst, int type) {
    a.op[n].src = src, a.op[n].dst = dst, a.op[n].rows = rows, a.op[n].ld = ld, a.op[n].cols = (int)cols;
    if (n == 0) a.first = 0xffffffffu;
    else a.first = (uint32_t)blocks;
    ++n;
    blocks += (rows * (padded(cols, type) / granule(type)) + kPad - 1) / kPad;
    return {dst, padded(cols, type), true};
  }
  hipError_t run(int type, hipStream_t st) const {
    if (blocks == 0) return hipSuccess;
    if (type == SLSTM_F32) hipLaunchKernelGGL(k_linear_pad<float>, dim3((unsigned)blocks), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(k_linear_pad<bf16_t>, dim3((unsigned)blocks), dim3(256), 0, st, a);
    return hipGetLastError();
  }
};

hipError_t join_launch(const GemmArgs& g, int type, hipStream_t st) {
  const int V = granule(type);
  const int64_t n = (int64_t)g.M * ((g.N + V - 1) / V);
  in_pieces(n, 64 * kMostGroups, [&](int64_t first, int64_t m) {
    const dim3 grid((unsigned)((m + 63) / 64));
    if (type == SLSTM_F32) hipLaunchKernelGGL(k_linear_join<float>, grid, dim3(256), 0, st, g, first);
    else hipLaunchKernelGGL(k_linear_join<bf16_t>, grid, dim3(256), 0, st, g, first);
  });
  return hipGetLastError();
}
template <typename T, int TILE, int SA, int SB>
hipError_t launch_both(GemmArgs x, GemmArgs w, hipStream_t st) {
  typedef Tile<T, TILE, TILE> S;
  constexpr int lds = S::ABYTES * SA + S::BBYTES * SB;
  static std::atomic<uint64_t> devices;
  const void* kern = (const void*)k_linear_both<T, TILE, SA, SB>;
  if (lds > 65536) {
    const hipError_t e = allow_lds(kern, lds, devices);
    if (e != hipSuccess) return e;
  }
  auto tiles = [](const GemmArgs& g) { return ((g.M + TILE - 1) / TILE) * ((g.N + TILE - 1) / TILE) * g.splits; };
  x.tiles = tiles(x), w.tiles = tiles(w);
  void* args[] = {&x, &w};
  return hipLaunchKernel(kern, dim3(x.tiles + w.tiles + (w.dbpart ? (w.N + 31) / 32 : 0)), dim3(S::NT), args, lds, st);
}

// The tiles of a product by a plan.
template <bool AT, bool BT>
hipError_t gemm_tiles(GemmArgs g, const Operand& A, const Operand& B, const Plan& p, int type, hipStream_t st) {
  g.A = A.p, g.lda = A.ld, g.B = B.p, g.ldb = B.ld, g.splits = p.splits, g.chunk = p.chunk;
  const bool dma = A.whole && B.whole, big = p.tile == 128;
  if (type == SLSTM_F32) {
    if (dma) return big ? launch_dma<float, AT, BT, 128, 3, 2>(g, st) : launch_dma<float, AT, BT, 64, 3, 3>(g, st);
    return big ? launch_any<float, AT, BT, 128>(g, st) : launch_any<float, AT, BT, 64>(g, st);
  }
  if (!dma) return big ? launch_any<bf16_t, AT, BT, 128>(g, st) : launch_any<bf16_t, AT, BT, 64>(g, st);
  if (p.tile == 256) return launch_dma<bf16_t, AT, BT, 256, 3, 2>(g, st);
  return big ? launch_dma<bf16_t, AT, BT, 128, 3, 2>(g, st) : launch_dma<bf16_t, AT, BT, 64, 3, 3>(g, st);
}
// One product with its epilogue; g has the sizes and the outputs.
template <bool AT, bool BT>
hipError_t gemm(GemmArgs g, const Operand& A, const Operand& B, int type, float* part, hipStream_t st) {
  const Plan p = gemm_plan(g.M, g.N, g.K, type, A.whole && B.whole);
  if (p.splits > 1) g.part = part;
  const hipError_t e = gemm_tiles<AT, BT>(g, A, B, p, type, st);
  g.splits = p.splits;
  return e != hipSuccess || p.splits == 1 ? e : join_launch(g, type, st);
}
// The same with dz (A, or with AT B) in two planes, `lo` the second: two products whose parts are added together. 16-bit matrix
// units take dz with 8 significant bits, as the caller gives dy; that is the choice unless a caller asks for this one: dx and dW of
// 61440 x 1024 x 4096 are then 0.0024 off of their size, where their own rounding alone is 0.0017, and the backward takes 1220 us
// instead of 2340 (6000 x 176 x 416: 23 and 54).
template <bool AT, bool BT>
hipError_t gemm_wide(GemmArgs g, const Operand& A, const Operand& B, const Operand& lo, int type, float* part, hipStream_t st) {
  const Plan p = gemm_plan(g.M, g.N, g.K, type, A.whole && B.whole);
  g.part = part;
  hipError_t e = gemm_tiles<AT, BT>(g, A, B, p, type, st);
  g.part = part + (int64_t)p.splits * g.M * g.N;
  g.dbpart = nullptr;
  if (e == hipSuccess) e = gemm_tiles<AT, BT>(g, AT ? A : lo, AT ? lo : B, p, type, st);
  g.part = part;
  g.splits = 2 * p.splits;
  return e != hipSuccess ? e : join_launch(g, type, st);
}
// Both products of a backward, dW's split in p.
hipError_t gemm_both(GemmArgs x, GemmArgs w, const Operand& dz, const Operand& W, const Operand& X, const Plan& p, int type, float* part,
                     hipStream_t st) {
  x.A = dz.p, x.lda = dz.ld, x.B = W.p, x.ldb = W.ld, x.splits = 1, x.chunk = x.K;
  w.A = X.p, w.lda = X.ld, w.B = dz.p, w.ldb = dz.ld, w.splits = p.splits, w.chunk = p.chunk;
  w.part = p.splits > 1 ? part : nullptr;
  hipError_t e;
  if (type == SLSTM_F32) e = p.tile == 128 ? launch_both<float, 128, 3, 2>(x, w, st) : launch_both<float, 64, 3, 3>(x, w, st);
  else e = p.tile == 128 ? launch_both<bf16_t, 128, 3, 2>(x, w, st) : launch_both<bf16_t, 64, 3, 3>(x, w, st);
  return e != hipSuccess || p.splits == 1 ? e : join_launch(w, type, st);
}
// Whether one launch is estimated to take less than two and the gap between them (fp32's two are a fifth slower than estimated:
// a last round's workgroups have a CU to themselves). One and two launches, us of dx and dW: 6000 x 176 x 416 bf16 16.5 and 24.3,
// f32 27.9 and 38.7; 7680 x 512 x 512 f32 77.8 and 82.6; two where chains of slices are long: 512 x 1024 x 8000 f32 177 and 147,
// 128 x 1024 x 32000 583 and 165.
bool both_pays(const slstm_linear_dims* d, const Plan& b) {
  const double two = gemm_plan(d->M, d->K, d->N, d->type, true).us + gemm_plan(d->K, d->N, d->M, d->type, true).us + 1;
  return d->M > 0 && b.us * (d->type == SLSTM_F32 ? 0.8 : 1.) < two;
}

int act_of(const slstm_linear_dims* d) { return d->act & ~SLSTM_LINEAR_WIDE_DZ; }
bool wide_dz(const slstm_linear_dims* d) {
  return d->type == SLSTM_BF16 && act_of(d) != SLSTM_ACT_NONE && (d->act & SLSTM_LINEAR_WIDE_DZ);
}
bool linear_ok(const slstm_linear_dims* d) {
  if (!d || d->M < 0 || d->M > (1 << 30) || d->K < 1 || d->K > (1 << 24) || d->N < 1 || d->N > (1 << 24)) return false;
  if (d->type != SLSTM_F32 && d->type != SLSTM_BF16) return false;
  if (act_of(d) < SLSTM_ACT_NONE || act_of(d) > SLSTM_ACT_GELU) return false;
  if (!stride_ok(d->ld_x, d->K) || !stride_ok(d->ld_w, d->N) || !stride_ok(d->ld_res, d->N) || !stride_ok(d->ld_y, d->N) ||
      !stride_ok(d->ld_dy, d->N))
    return false;
  // tiles of 64 of each output, and 2^19 workgroups for db, in 31 bits
  auto tiles = [](int64_t m, int64_t n) { return ((m + 63) / 64) * ((n + 63) / 64); };
  const int64_t most = 0x7fffffff - (1 << 19);
  return tiles(d->M, d->N) <= most && tiles(d->M, d->K) <= most && tiles(d->K, d->N) <= most;
}
// Strips of columns and blocks of rows of k_linear_dz: about 2048 workgroups, none for fewer than 64 rows, one block for up to
// 128 (it writes db itself). Up to 2048 rows strips of 8 vectors (128 bytes of a row), more workgroups; 32 above.
struct DzPlan {
  bool narrow;
  int strips, blocks, rows;
};
DzPlan dz_plan(const slstm_linear_dims* d) {
  DzPlan p;
  p.narrow = d->M <= 2048;
  const int cols = (p.narrow ? 8 : 32) * granule(d->type);
  p.strips = (d->N + cols - 1) / cols;
  const int64_t want = d->M <= 128 ? 1 : std::max<int64_t>(1, std::min<int64_t>({(d->M + 63) / 64, 2048 / p.strips, 256}));
  p.rows = (int)(((d->M + want - 1) / want + 7) / 8 * 8);
  p.blocks = (int)std::max<int64_t>(1, (d->M + std::max(1, p.rows) - 1) / std::max(1, p.rows));
  return p;
}
// Work space of a forward: copies of x and W, parts; of a backward: dz (or a copy of dy), copies of W and x, sums of
// columns, parts.
struct Spaces {
  size_t dz, lo, x, W, db, part, total;
};
Spaces fwd_spaces(const slstm_linear_dims* d) {
  Spaces s = {};
  s.x = 0;
  s.W = s.x + (needs_copy(d->M, d->K, row_stride(d->ld_x, d->K), d->type) ? copy_bytes(d->M, d->K, d->type) : 0);
  s.part = s.W + (needs_copy(d->M, d->N, row_stride(d->ld_w, d->N), d->type) ? copy_bytes(d->K, d->N, d->type) : 0);
  s.total = s.part + gemm_bytes(d->M, d->N, d->K, d->type);
  return s;
}
Spaces bwd_spaces(const slstm_linear_dims* d) {
  Spaces s = {};
  const bool dz = act_of(d) != SLSTM_ACT_NONE || needs_copy(d->M, d->N, row_stride(d->ld_dy, d->N), d->type);
  s.lo = dz ? copy_bytes(d->M, d->N, d->type) : 0;
  s.x = s.lo + (wide_dz(d) ? copy_bytes(d->M, d->N, d->type) : 0);
  s.W = s.x + (needs_copy(d->M, d->K, row_stride(d->ld_x, d->K), d->type) ? copy_bytes(d->M, d->K, d->type) : 0);
  s.db = s.W + (needs_copy(d->M, d->N, row_stride(d->ld_w, d->N), d->type) ? copy_bytes(d->K, d->N, d->type) : 0);
  s.part = s.db + (((size_t)dz_plan(d).blocks * d->N * 4 + 255) & ~(size_t)255);
  if (wide_dz(d)) {
    s.total = s.part + std::max(wide_bytes(d->M, d->K, d->N, d->type), wide_bytes(d->K, d->N, d->M, d->type));
    return s;
  }
  s.total = s.part + std::max({gemm_bytes(d->M, d->K, d->N, d->type), gemm_bytes(d->K, d->N, d->M, d->type),
                               part_bytes(both_plan(d->M, d->K, d->N, d->type), d->K, d->N)});
  return s;
}

}  // namespace

extern "C" size_t stacklstm_linear_fwd_workspace_bytes(const slstm_linear_dims* d) {
  return linear_ok(d) ? std::max<size_t>(4, fwd_spaces(d).total) : 0;
}
extern "C" size_t stacklstm_linear_bwd_workspace_bytes(const slstm_linear_dims* d) {
  return linear_ok(d) ? std::max<size_t>(4, bwd_spaces(d).total) : 0;
}

extern "C" int stacklstm_linear_fwd(const slstm_linear_dims* d, const void* x, const void* W, const void* b, const void* res,
                                    void* y, void* z, void* workspace, size_t ws_bytes, void* stream) {
  if (!linear_ok(d)) return SLSTM_EINVAL;
  if (d->M == 0) return SLSTM_OK;
  if (!x || !W || !y || !workspace || !al16(workspace)) return SLSTM_EINVAL;
  if (res == y && row_stride(d->ld_res, d->N) != row_stride(d->ld_y, d->N)) return SLSTM_EINVAL;
  const Spaces s = fwd_spaces(d);
  if (ws_bytes < s.total) return SLSTM_EWORKSPACE;
  const hipStream_t st = as_stream(stream);
  char* ws = (char*)workspace;
  const int64_t ldx = row_stride(d->ld_x, d->K), ldw = row_stride(d->ld_w, d->N);
  Copies cp;
  const Operand ox = s.W > s.x ? cp.add(x, d->M, d->K, ldx, ws + s.x, d->type) : as_is(x, d->K, ldx, d->type);
  const Operand ow = s.part > s.W ? cp.add(W, d->K, d->N, ldw, ws + s.W, d->type) : as_is(W, d->N, ldw, d->type);
  hipError_t e = cp.run(d->type, st);
  GemmArgs g = {};
  g.M = (int)d->M, g.N = d->N, g.K = d->K;
  g.bias = b, g.res = res, g.y = y, g.z = z, g.act = act_of(d);
  g.ldy = row_stride(d->ld_y, d->N), g.ldr = row_stride(d->ld_res, d->N);
  if (e == hipSuccess) e = gemm<false, true>(g, ox, ow, d->type, (float*)(ws + s.part), st);
  return e == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
}

extern "C" int stacklstm_linear_bwd(const slstm_linear_dims* d, const void* x, const void* W, const void* z, const void* dy,
                                    void* dx, void* dW, void* db, void* workspace, size_t ws_bytes, void* stream) {
  if (!linear_ok(d)) return SLSTM_EINVAL;
  const bool act = act_of(d) != SLSTM_ACT_NONE, wide = wide_dz(d);
  if (!workspace || !al16(workspace)) return SLSTM_EINVAL;
  if (d->M > 0 && (!dy || (act && !z) || (dW && !x) || (dx && !W))) return SLSTM_EINVAL;
  const Spaces s = bwd_spaces(d);
  if (ws_bytes < s.total) return SLSTM_EWORKSPACE;
  if (d->M == 0) dx = nullptr;
  const hipStream_t st = as_stream(stream);
  char* ws = (char*)workspace;
  const int64_t ldx = row_stride(d->ld_x, d->K), ldw = row_stride(d->ld_w, d->N), ldd = row_stride(d->ld_dy, d->N);
  const bool product = dx || dW, own = s.lo > s.dz && product && d->M > 0;
  if (few_rows(d) && !wide) {
    auto tiles = [](int64_t m, int64_t n) { return (int)(((m + 63) / 64) * ((n + 63) / 64)); };
    GemmArgs gx = {}, gw = {};
    gx.M = (int)d->M, gx.N = d->K, gx.K = d->N, gx.A = dy, gx.lda = ldd, gx.B = W, gx.ldb = ldw, gx.y = dx, gx.ldy = d->K;
    gw.M = d->K, gw.N = d->N, gw.K = (int)d->M, gw.A = x, gw.lda = ldx, gw.B = dy, gw.ldb = ldd, gw.y = dW, gw.ldy = d->N;
    gx.splits = gw.splits = 1, gx.chunk = gx.K, gw.chunk = gw.K;
    if (act) gx.dz = gw.dz = z, gx.lddz = gw.lddz = d->N, gx.dzact = gw.dzact = act_of(d);
    DzArgs a = {};
    a.M = (int)d->M, a.N = d->N, a.act = act_of(d), a.rows = (int)d->M, a.dy = dy, a.z = act ? z : nullptr, a.ldd = ldd, a.db = db;
    const int nx = dx ? tiles(d->M, d->K) : 0, nw = dW ? tiles(d->K, d->N) : 0, nb = db ? dz_plan(d).strips : 0;
    if (nx + nw + nb == 0) return SLSTM_OK;
    const dim3 grid(nx + nw + nb);
    constexpr int lds = 2 * (Tile<float, 64, 64>::ABYTES + Tile<float, 64, 64>::BBYTES);
    if (d->type == SLSTM_F32) hipLaunchKernelGGL(k_linear_few<float>, grid, dim3(256), lds, st, gx, gw, a, nx, nw);
    else hipLaunchKernelGGL(k_linear_few<bf16_t>, grid, dim3(256), lds, st, gx, gw, a, nx, nw);
    return hipGetLastError() == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
  }
  Operand oz = as_is(dy, d->N, ldd, d->type);
  if (own) oz = {ws + s.dz, padded(d->N, d->type), padded(d->N, d->type) <= kReach};
  Copies cp;
  Operand ox = {}, ow = {};
  if (dW) ox = s.W > s.x ? cp.add(x, d->M, d->K, ldx, ws + s.x, d->type) : as_is(x, d->K, ldx, d->type);
  if (dx) ow = s.db > s.W ? cp.add(W, d->K, d->N, ldw, ws + s.W, d->type) : as_is(W, d->N, ldw, d->type);
  const DzPlan p = dz_plan(d);
  const int nd = db || own ? p.strips * p.blocks : 0;
  hipError_t e = hipSuccess;
  if (nd + cp.blocks > 0) {
    DzArgs a = {};
    a.M = (int)d->M, a.N = d->N, a.act = act_of(d), a.rows = p.rows, a.dy = dy, a.z = act ? z : nullptr;
    a.ldd = ldd, a.ldz = padded(d->N, d->type), a.dz = own ? ws + s.dz : nullptr, a.lo = own && wide ? ws + s.lo : nullptr, a.part = db && p.blocks > 1 ? (float*)(ws + s.db) : nullptr;
    a.db = db && p.blocks == 1 ? db : nullptr;
    const dim3 grid((unsigned)(nd + cp.blocks));
    auto run = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a, p.strips, nd, cp.a); };
    if (d->type == SLSTM_F32) run(p.narrow ? k_linear_dz<float, 8> : k_linear_dz<float, 32>);
    else run(p.narrow ? k_linear_dz<bf16_t, 8> : k_linear_dz<bf16_t, 32>);
    if (a.part && !dW) {
      const dim3 cols((d->N + 31) / 32);
      if (d->type == SLSTM_F32) hipLaunchKernelGGL(k_linear_db<float>, cols, dim3(256), 0, st, a.part, p.blocks, d->N, (float*)db);
      else hipLaunchKernelGGL(k_linear_db<bf16_t>, cols, dim3(256), 0, st, a.part, p.blocks, d->N, (bf16_t*)db);
    }
    e = hipGetLastError();
  }
  float* part = (float*)(ws + s.part);
  GemmArgs gx = {}, gw = {};
  gx.M = (int)d->M, gx.N = d->K, gx.K = d->N, gx.y = dx, gx.ldy = d->K;
  gw.M = d->K, gw.N = d->N, gw.K = (int)d->M, gw.y = dW, gw.ldy = d->N;
  if (db && p.blocks > 1) gw.dbpart = (const float*)(ws + s.db), gw.dbrows = p.blocks, gw.db = db;
  if (wide && own) {
    const Operand lo = {ws + s.lo, oz.ld, oz.whole};
    if (e == hipSuccess && dx) e = gemm_wide<false, false>(gx, oz, ow, lo, d->type, part, st);
    if (e == hipSuccess && dW) e = gemm_wide<true, true>(gw, ox, oz, lo, d->type, part, st);
    return e == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
  }
  if (dx && dW && ox.whole && ow.whole && oz.whole) {
    const Plan b = both_plan(d->M, d->K, d->N, d->type);
    if (both_pays(d, b)) {
      if (e == hipSuccess) e = gemm_both(gx, gw, oz, ow, ox, b, d->type, part, st);
      return e == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
    }
  }
  if (e == hipSuccess && dx) e = gemm<false, false>(gx, oz, ow, d->type, part, st);
  if (e == hipSuccess && dW) e = gemm<true, true>(gw, ox, oz, d->type, part, st);
  return e == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
}
