// Linear layer with its epilogue, and its backward:
//   z = x W + b, y = act(z) + res;  dz = dy act'(z), dx = dz W^T, dW = x^T dz, db = sum over rows of dz
// All three products are C(m, n) = sum_k A(m, k) B(n, k) on the matrix units, 16x16 tiles (bf16: k of 32; fp32: the
// fp32 instruction, k of 4), fp32 sums. An operand lies in memory either by rows of k ("flat": x and dz of y and dx,
// W of dx) or with k as the row ("tall": W of y, both operands of dW). A flat operand's slice is kept in LDS by rows
// of 128 bytes and read 16 bytes a lane; a tall one's by its rows of k, and is read transposed (16-bit) or element by
// element (fp32). 16-byte granules are permuted within a row so that fragment reads spread over the banks.
// Slices reach LDS by DMA where every operand is 16-bit and aligned, a few slices ahead; otherwise through
// registers, one slice ahead, with the rows' ends cut off there.
// Where the tiles do not fill the chip the sum over k is split, and k_linear_join adds the parts and applies the
// epilogue.
#include <algorithm>

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
};

__device__ __forceinline__ float act_fwd(float z, int act) {
  switch (act) {
    case SLSTM_ACT_RELU: return z > 0.f ? z : z != z ? z : 0.f;
    case SLSTM_ACT_TANH: return tanhf_(z);
    case SLSTM_ACT_SILU: return z * sigmoidf_(z);
    case SLSTM_ACT_GELU: return z * sigmoidf_(1.5957691216057308f * (z + 0.044715f * z * z * z));
    default: return z;
  }
}
// (z/2 (1 + tanh u) = z sigma(2u); derivative of z sigma(2u): s + z s (1 - s) 2u')
__device__ __forceinline__ float act_bwd(float z, int act) {
  switch (act) {
    case SLSTM_ACT_RELU: return z > 0.f ? 1.f : z != z ? z : 0.f;
    case SLSTM_ACT_TANH: {
      const float a = tanhf_(z);
      return 1.f - a * a;
    }
    case SLSTM_ACT_SILU: {
      const float s = sigmoidf_(z);
      return s * (1.f + z * (1.f - s));
    }
    case SLSTM_ACT_GELU: {
      const float s = sigmoidf_(1.5957691216057308f * (z + 0.044715f * z * z * z));
      return s + z * s * (1.f - s) * 1.5957691216057308f * (1.f + 0.134145f * z * z);
    }
    default: return 1.f;
  }
}

// One row piece of the epilogue: v[] at column n of row m.
template <typename T>
__device__ __forceinline__ void finish(const GemmArgs& g, int64_t m, int n, float (&v)[vec<T>::N]) {
  constexpr int V = vec<T>::N;
  const int left = g.N - n;
  if (g.bias) {
    float b[V];
    vec<T>::unpack(load_vec((const T*)g.bias + n, 0, left), b);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] += b[k];
  }
  if (g.z) store_vec((T*)g.z + m * g.N + n, 0, left, v);
  if (g.act != SLSTM_ACT_NONE) {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = act_fwd(v[k], g.act);
  }
  if (g.res) {
    float r[V];
    vec<T>::unpack(load_vec((const T*)g.res + m * g.ldr + n, 0, left), r);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] += r[k];
  }
  store_vec((T*)g.y + m * g.ldy + n, 0, left, v);
}

// Sizes of a block tile. A slice is 128 bytes of k: 64 (16-bit) or 32 (fp32).
template <typename T, int BM, int BN>
struct Tile {
  static constexpr int BK = 128 / (int)sizeof(T), NT = BM == 256 ? 512 : 256, WN = BM == 256 ? 4 : 2, WM = NT / 64 / WN;
  static constexpr int MI = BM / WM / 16, NJ = BN / WN / 16;
  static constexpr int ABYTES = BM * 128, BBYTES = BN * 128, STAGE = ABYTES + BBYTES;
  static constexpr int IA = BM * 8 / NT, IB = BN * 8 / NT;       // granules of a thread
};
constexpr int gemm_lds(int stage, int stages) { return stage * stages; }

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

}  // namespace

template <typename T, bool AT, bool BT, int BM, int BN, bool DMA, int NS>
__global__ void __launch_bounds__((Tile<T, BM, BN>::NT), 2) k_linear(GemmArgs g) {
  typedef Tile<T, BM, BN> S;
  constexpr int V = vec<T>::N, BK = S::BK, NT = S::NT, MI = S::MI, NJ = S::NJ;
  static_assert(!DMA || sizeof(T) == 2, "DMA of 16-bit operands");
  extern __shared__ __align__(16) unsigned char sm[];
  const int NTL = (g.N + BN - 1) / BN, MTL = (g.M + BM - 1) / BM, tiles = NTL * MTL, all = tiles * g.splits;
  int lid = (int)blockIdx.x;
  // workgroups go to the 8 XCDs in turn: each XCD takes a contiguous run of tiles, in groups of 8 row tiles to a
  // column tile, so that what its L2 holds is used again
  {
    const int full = all & ~7;
    if (lid < full) lid = (lid & 7) * (full >> 3) + (lid >> 3);
  }
  const int zs = lid / tiles;
  lid -= zs * tiles;
  constexpr int GM = 8;
  const int gi = lid / (GM * NTL), gm = min(GM, MTL - gi * GM), rem = lid - gi * GM * NTL;
  const int m0 = (gi * GM + rem % gm) * BM, n0 = (rem / gm) * BN;
  const int kbeg = min(g.K, zs * g.chunk), kend = min(g.K, kbeg + g.chunk);
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN, l16 = lane & 15, lq = lane >> 4;
  const int nr = min(BM, g.M - m0), nc = min(BN, g.N - n0);
  const T* A = (const T*)g.A + (AT ? m0 : (int64_t)m0 * g.lda);
  const T* B = (const T*)g.B + (BT ? n0 : (int64_t)n0 * g.ldb);

  // DMA of the slice at k0 (past kend: nothing is read; the count of a wave's DMAs stays the same)
  [[maybe_unused]] auto dma = [&](int k0, int buf, int part, int parts) {
    unsigned char* st = sm + buf * S::STAGE;
    auto one = [&](auto tall, auto rows, const T* p, int64_t ld, int n, unsigned char* to, int i) {
      constexpr bool TALL = decltype(tall)::value;
      constexpr int ROWS = decltype(rows)::value;
      int r, c;
      place<T, TALL, ROWS>((i * (NT / 64) + wave) * 64 + lane, r, c);
      const int left = kend - k0;
      const bool in = TALL ? r < left && c * V < n : r < n && c * V < left;
      const T* base = TALL ? p + (int64_t)k0 * ld : p + k0;
      const rsrc_t rs = make_rsrc(base, left > 0 ? (size_t)((TALL ? min(BK, left) - 1 : n - 1) * ld + (TALL ? n : min(BK, left))) * 2 : 0);
      bdma16(rs, in ? (uint32_t)(r * (int)ld + c * V) * 2u : kOOB, 0u, lds_addr(to + (i * (NT / 64) + wave) * 1024));
    };
#pragma unroll
    for (int i = 0; i < S::IA; ++i)
      if (i % parts == part) one(std::integral_constant<bool, AT>(), std::integral_constant<int, BM>(), A, g.lda, nr, st, i);
#pragma unroll
    for (int i = 0; i < S::IB; ++i)
      if ((S::IA + i) % parts == part)
        one(std::integral_constant<bool, BT>(), std::integral_constant<int, BN>(), B, g.ldb, nc, st + S::ABYTES, i);
  };
  // the same through registers
  [[maybe_unused]] u32x4 ra[S::IA], rb[S::IB];
  [[maybe_unused]] auto fetch = [&](int k0) {
    const int left = kend - k0;
#pragma unroll
    for (int i = 0; i < S::IA; ++i) {
      int r, c;
      place<T, AT, BM>(i * NT + tid, r, c);
      const bool in = left > 0 && r < (AT ? left : nr);
      ra[i] = in ? load_vec(A + (AT ? (int64_t)(k0 + r) * g.lda : (int64_t)r * g.lda + k0), c, AT ? nr : left) : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int i = 0; i < S::IB; ++i) {
      int r, c;
      place<T, BT, BN>(i * NT + tid, r, c);
      const bool in = left > 0 && r < (BT ? left : nc);
      rb[i] = in ? load_vec(B + (BT ? (int64_t)(k0 + r) * g.ldb : (int64_t)r * g.ldb + k0), c, BT ? nc : left) : u32x4{0u, 0u, 0u, 0u};
    }
  };
  [[maybe_unused]] auto put = [&](int buf) {
    unsigned char* st = sm + buf * S::STAGE;
#pragma unroll
    for (int i = 0; i < S::IA; ++i) *(u32x4*)(st + (i * NT + tid) * 16) = ra[i];
#pragma unroll
    for (int i = 0; i < S::IB; ++i) *(u32x4*)(st + S::ABYTES + (i * NT + tid) * 16) = rb[i];
  };

  f32x4 acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  // products of a staged slice; between(i): behind those of row tile i of the first half
  auto products = [&](const unsigned char* st, auto between) {
    if constexpr (sizeof(T) == 2) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      // a lane's 8 k of tile `tile`: from one row, or transposed: the lane gives the address of k row
      // 8 lq + l16 / 4 and columns 4 (l16 % 4) of the tile, and gets column l16, four k
      auto frag = [&](auto tall, auto rows, const unsigned char* p, int tile, int kc) {
        constexpr bool TALL = decltype(tall)::value;
        constexpr int ROWS = decltype(rows)::value;
        if constexpr (!TALL) {
          const int r = 16 * tile + l16;
          return *(const bf16x8*)(p + (r * 8 + ((4 * kc + lq) ^ swz<T, TALL, ROWS>(r))) * 16);
        } else {
          constexpr int G = ROWS / 8;
          const int k = 8 * lq + (l16 >> 2);
          const unsigned char* q = p + (kc * 32 + k) * G * 16 + ((2 * tile + ((l16 & 3) >> 1)) ^ swz<T, TALL, ROWS>(k)) * 16 + (l16 & 1) * 8;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(q));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(q + 4 * G * 16));
          return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
      };
#pragma unroll
      for (int kc = 0; kc < 2; ++kc) {
        bf16x8 a[MI], b[NJ];
#pragma unroll
        for (int i = 0; i < MI; ++i) a[i] = frag(std::integral_constant<bool, AT>(), std::integral_constant<int, BM>(), st, MI * wm + i, kc);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          b[j] = frag(std::integral_constant<bool, BT>(), std::integral_constant<int, BN>(), st + S::ABYTES, NJ * wn + j, kc);
#pragma unroll
        for (int i = 0; i < MI; ++i) {
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[i][j] = mfma_bf16_16x16x32(b[j], a[i], acc[i][j]);
          if (kc == 0) between(i);
        }
      }
    } else {
      // a lane's four k (4 lq .. 4 lq + 3 of 16) go to four instructions, for both operands alike
      auto frag = [&](auto tall, auto rows, const unsigned char* p, int tile, int kc) {
        constexpr bool TALL = decltype(tall)::value;
        constexpr int ROWS = decltype(rows)::value;
        const int r = 16 * tile + l16;
        if constexpr (!TALL) {
          return *(const f32x4*)(p + (r * 8 + ((4 * kc + lq) ^ swz<T, TALL, ROWS>(r))) * 16);
        } else {
          f32x4 v;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int k = 16 * kc + 4 * lq + q;
            v[q] = *(const float*)(p + (k * (ROWS / 4) + ((r >> 2) ^ swz<T, TALL, ROWS>(k))) * 16 + (r & 3) * 4);
          }
          return v;
        }
      };
#pragma unroll
      for (int kc = 0; kc < 2; ++kc) {
        f32x4 a[MI], b[NJ];
#pragma unroll
        for (int i = 0; i < MI; ++i) a[i] = frag(std::integral_constant<bool, AT>(), std::integral_constant<int, BM>(), st, MI * wm + i, kc);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          b[j] = frag(std::integral_constant<bool, BT>(), std::integral_constant<int, BN>(), st + S::ABYTES, NJ * wn + j, kc);
#pragma unroll
        for (int i = 0; i < MI; ++i) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[j][q], a[i][q], acc[i][j], 0, 0, 0);
          if (kc == 0) between(i);
        }
      }
    }
  };

  if constexpr (DMA) {
    constexpr int PER = S::IA + S::IB;
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) dma(kbeg + s * BK, s, 0, 1);
    int buf = 0;
    for (int k0 = kbeg; k0 < kend; k0 += BK) {
      wait_vm<(NS - 2) * PER>();
      __syncthreads();                                 // this slice landed, the stage before it is free
      const int next = buf == 0 ? NS - 1 : buf - 1;
      products(sm + buf * S::STAGE, [&](int i) { dma(k0 + (NS - 1) * BK, next, i, MI); });
      buf = buf + 1 == NS ? 0 : buf + 1;
    }
    wait_vm<0>();
  } else {
    static_assert(NS == 2, "two stages");
    fetch(kbeg);
    int buf = 0;
    for (int k0 = kbeg; k0 < kend; k0 += BK, buf ^= 1) {
      put(buf);
      __syncthreads();
      if (k0 + BK < kend) fetch(k0 + BK);
      products(sm + buf * S::STAGE, [](int) {});
    }
  }
  __syncthreads();                                     // the stages are free

  // a wave turns 16 rows of its tile at a time into row pieces of 16 bytes a lane
  constexpr int CW = 16 * NJ, LD = CW + 4, VR = 64 * V / CW;
  float* ws = reinterpret_cast<float*>(sm) + wave * (16 * LD);
#pragma unroll
  for (int i = 0; i < MI; ++i) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) *(f32x4*)&ws[l16 * LD + j * 16 + 4 * lq] = acc[i][j];
    wave_lds();
#pragma unroll
    for (int e = 0; e < 16 / VR; ++e) {
      const int r = e * VR + lane / (CW / V), c = (lane % (CW / V)) * V;
      const int m = 16 * (MI * wm + i) + r, n = n0 + CW * wn + c;
      if (m >= nr || n >= g.N) continue;
      float v[V];
#pragma unroll
      for (int k = 0; k < V; k += 4) {
        const f32x4 q = *(const f32x4*)&ws[r * LD + c + k];
#pragma unroll
        for (int h = 0; h < 4; ++h) v[k + h] = q[h];
      }
      if (g.part) {
        float* o = g.part + ((int64_t)zs * g.M + m0 + m) * g.N + n;
#pragma unroll
        for (int k = 0; k < V; k += 4) {
          const float w[4] = {v[k], v[k + 1], v[k + 2], v[k + 3]};
          store_vec(o, k / 4, g.N - n, w);
        }
      } else {
        finish<T>(g, m0 + m, n, v);
      }
    }
    wave_lds();
  }
}

// The parts of a split product added in order, and the epilogue.
template <typename T>
__global__ void __launch_bounds__(256) k_linear_join(GemmArgs g) {
  constexpr int V = vec<T>::N;
  const int nv = (g.N + V - 1) / V;
  const int64_t all = (int64_t)g.M * nv;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / nv;
    const int n = (int)(i - m * nv) * V;
    float v[V];
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = 0.f;
    for (int s = 0; s < g.splits; ++s) {
      const float* p = g.part + ((int64_t)s * g.M + m) * g.N + n;
#pragma unroll
      for (int k = 0; k < V; k += 4) {
        float w[4];
        vec<float>::unpack(load_vec(p, k / 4, g.N - n), w);
#pragma unroll
        for (int h = 0; h < 4; ++h) v[k + h] += w[h];
      }
    }
    finish<T>(g, m, n, v);
  }
}

namespace {
struct DzArgs {
  int M, N, act, rows;                                 // rows of a workgroup
  const void *dy, *z;
  int64_t ldd, ldz;
  void* dz;                                            // NULL: dy serves
  float* part;                                         // [row blocks][N], NULL: no db
};
}  // namespace

// dz = dy act'(z), and the sums of its columns over a block of rows: 32 column vectors, 8 rows at a time.
template <typename T>
__global__ void __launch_bounds__(256) k_linear_dz(DzArgs a) {
  constexpr int V = vec<T>::N;
  __shared__ float red[8][32 * V + 4];
  const int c = (int)blockIdx.x * 32 + (threadIdx.x & 31), r8 = threadIdx.x >> 5;
  const int64_t lo = (int64_t)blockIdx.y * a.rows, hi = min((int64_t)a.M, lo + a.rows);
  float s[V];
#pragma unroll
  for (int k = 0; k < V; ++k) s[k] = 0.f;
  if (c * V < a.N) {
#pragma unroll 4
    for (int64_t m = lo + r8; m < hi; m += 8) {
      float d[V];
      vec<T>::unpack(load_vec((const T*)a.dy + m * a.ldd, c, a.N), d);
      if (a.z) {
        float z[V];
        vec<T>::unpack(load_vec((const T*)a.z + m * a.N, c, a.N), z);
#pragma unroll
        for (int k = 0; k < V; ++k) d[k] *= act_bwd(z[k], a.act);
      }
#pragma unroll
      for (int k = 0; k < V; ++k) s[k] += d[k];
      if (a.dz) store_vec((T*)a.dz + m * a.ldz, c, a.N, d);
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int k = 0; k < V; ++k) red[r8][(threadIdx.x & 31) * V + k] = s[k];
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * V; i += 256) {
    const int n = (int)blockIdx.x * 32 * V + i;
    if (n >= a.N) continue;
    float v = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) v += red[r][i];
    a.part[(int64_t)blockIdx.y * a.N + n] = v;
  }
}

// db: the sums of P blocks of rows, 8 columns and 32 parts of the P to a workgroup.
template <typename T>
__global__ void __launch_bounds__(256) k_linear_db(const float* part, int P, int N, T* db) {
  __shared__ float red[32][9];
  const int n = blockIdx.x * 8 + (threadIdx.x & 7), p0 = threadIdx.x >> 3;
  float s = 0.f;
  if (n < N)
    for (int p = p0; p < P; p += 32) s += part[(int64_t)p * N + n];
  red[p0][threadIdx.x & 7] = s;
  __syncthreads();
  if (threadIdx.x >= 8 || n >= N) return;
  float v = 0.f;
#pragma unroll
  for (int p = 0; p < 32; ++p) v += red[p][threadIdx.x];
  from_f32(db[n], v);
}

namespace {

bool al16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
// How a product runs: block tile, parts of k, and whether its operands go to LDS by DMA.
struct Plan {
  int tile, splits, chunk;
  bool dma;
};
// The largest tile that fills three quarters of the 256 CUs, k split where that helps (a part takes at least
// eight slices); 256 x 256 only by DMA, and no tile of which more than half would be past the end.
Plan gemm_plan(int64_t M, int64_t N, int64_t K, int type, bool dma) {
  const int BK = type == SLSTM_F32 ? 32 : 64;
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(64, K / (8 * BK)));
  Plan p = {64, 1, 0, dma};
  int64_t tiles = 0;
  for (int t = dma ? 256 : 128; t >= 64; t /= 2) {
    tiles = ((M + t - 1) / t) * ((N + t - 1) / t);
    p.tile = t;
    if (std::min(M, N) > t / 2 && tiles * most >= 192) break;
  }
  const int64_t want = p.tile == 256 ? 256 : 512;
  if (tiles * 2 <= want) p.splits = (int)std::max<int64_t>(1, std::min(most, want / std::max<int64_t>(1, tiles)));
  const int64_t slices = (K + BK - 1) / BK, per = (slices + p.splits - 1) / p.splits;
  p.chunk = (int)(std::max<int64_t>(1, per) * BK);
  p.splits = (int)std::max<int64_t>(1, (slices + per - 1) / std::max<int64_t>(1, per));
  return p;
}
size_t part_bytes(const Plan& p, int64_t M, int64_t N) {
  return p.splits > 1 ? ((size_t)p.splits * M * N * 4 + 255) & ~(size_t)255 : 0;
}
// Either way of staging: the work space does not depend on the arrays' alignment.
size_t gemm_bytes(int64_t M, int64_t N, int64_t K, int type) {
  const size_t a = part_bytes(gemm_plan(M, N, K, type, false), M, N);
  return type == SLSTM_F32 ? a : std::max(a, part_bytes(gemm_plan(M, N, K, type, true), M, N));
}

template <typename T, bool AT, bool BT, int TILE, bool DMA, int NS>
hipError_t gemm_launch(const GemmArgs& g, hipStream_t st) {
  auto kern = k_linear<T, AT, BT, TILE, TILE, DMA, NS>;
  typedef Tile<T, TILE, TILE> S;
  constexpr int lds = gemm_lds(S::STAGE, NS);
  const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  const int64_t tiles = (((int64_t)g.M + TILE - 1) / TILE) * (((int64_t)g.N + TILE - 1) / TILE) * g.splits;
  hipLaunchKernelGGL(kern, dim3((unsigned)tiles), dim3(S::NT), lds, st, g);
  return hipGetLastError();
}
// One product with its epilogue; g has the operands, the sizes and the outputs.
template <bool AT, bool BT>
hipError_t gemm(GemmArgs g, int type, float* part, hipStream_t st) {
  // DMA: 16-bit operands whose rows are whole granules at aligned places
  const bool dma = type == SLSTM_BF16 && al16(g.A) && al16(g.B) && g.lda % 8 == 0 && g.ldb % 8 == 0 &&
                   (AT ? g.M : g.K) % 8 == 0 && (BT ? g.N : g.K) % 8 == 0 && g.lda <= (1 << 22) && g.ldb <= (1 << 22);
  const Plan p = gemm_plan(g.M, g.N, g.K, type, dma);
  g.splits = p.splits;
  g.chunk = p.chunk;
  g.part = p.splits > 1 ? part : nullptr;
  hipError_t e;
  if (type == SLSTM_F32)
    e = p.tile == 128 ? gemm_launch<float, AT, BT, 128, false, 2>(g, st) : gemm_launch<float, AT, BT, 64, false, 2>(g, st);
  else if (!dma)
    e = p.tile == 128 ? gemm_launch<bf16_t, AT, BT, 128, false, 2>(g, st) : gemm_launch<bf16_t, AT, BT, 64, false, 2>(g, st);
  else if (p.tile == 256)
    e = gemm_launch<bf16_t, AT, BT, 256, true, 2>(g, st);
  else
    e = p.tile == 128 ? gemm_launch<bf16_t, AT, BT, 128, true, 2>(g, st) : gemm_launch<bf16_t, AT, BT, 64, true, 4>(g, st);
  if (e != hipSuccess || p.splits == 1) return e;
  const int V = type == SLSTM_F32 ? 4 : 8;
  const int64_t n = (int64_t)g.M * ((g.N + V - 1) / V);
  const dim3 grid((unsigned)std::min<int64_t>((n + 255) / 256, 4096));
  if (type == SLSTM_F32) hipLaunchKernelGGL(k_linear_join<float>, grid, dim3(256), 0, st, g);
  else hipLaunchKernelGGL(k_linear_join<bf16_t>, grid, dim3(256), 0, st, g);
  return hipGetLastError();
}

bool linear_ok(const slstm_linear_dims* d) {
  if (!d || d->M < 0 || d->M > (1 << 30) || d->K < 1 || d->K > (1 << 24) || d->N < 1 || d->N > (1 << 24)) return false;
  if (d->type != SLSTM_F32 && d->type != SLSTM_BF16) return false;
  if (d->act < SLSTM_ACT_NONE || d->act > SLSTM_ACT_GELU) return false;
  if (!stride_ok(d->ld_x, d->K) || !stride_ok(d->ld_w, d->N) || !stride_ok(d->ld_res, d->N) || !stride_ok(d->ld_y, d->N) ||
      !stride_ok(d->ld_dy, d->N))
    return false;
  // tiles of 64 of each output, in 31 bits
  auto tiles = [](int64_t m, int64_t n) { return ((m + 63) / 64) * ((n + 63) / 64); };
  const int64_t most = 0x7fffffff;
  return tiles(d->M, d->N) <= most && tiles(d->M, d->K) <= most && tiles(d->K, d->N) <= most;
}
int esize(const slstm_linear_dims* d) { return d->type == SLSTM_F32 ? 4 : 2; }
// Blocks of rows of k_linear_dz: about 2048 workgroups, none for fewer than 64 rows.
struct DzPlan {
  int strips, blocks, rows;
};
DzPlan dz_plan(const slstm_linear_dims* d) {
  DzPlan p;
  const int V = 16 / esize(d);
  p.strips = (d->N + 32 * V - 1) / (32 * V);
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>({(d->M + 63) / 64, 2048 / p.strips, 256}));
  p.rows = (int)(((d->M + want - 1) / want + 7) / 8 * 8);
  p.blocks = (int)std::max<int64_t>(1, (d->M + std::max(1, p.rows) - 1) / std::max(1, p.rows));
  return p;
}
size_t dz_stride(const slstm_linear_dims* d) { return ((size_t)d->N + 7) / 8 * 8; }
size_t dz_bytes(const slstm_linear_dims* d) {
  return d->act == SLSTM_ACT_NONE ? 0 : ((size_t)d->M * dz_stride(d) * esize(d) + 255) & ~(size_t)255;
}
size_t db_bytes(const slstm_linear_dims* d) { return ((size_t)dz_plan(d).blocks * d->N * 4 + 255) & ~(size_t)255; }

}  // namespace

extern "C" size_t stacklstm_linear_fwd_workspace_bytes(const slstm_linear_dims* d) {
  if (!linear_ok(d)) return 0;
  return std::max<size_t>(4, gemm_bytes(d->M, d->N, d->K, d->type));
}
extern "C" size_t stacklstm_linear_bwd_workspace_bytes(const slstm_linear_dims* d) {
  if (!linear_ok(d)) return 0;
  return dz_bytes(d) + db_bytes(d) + std::max(gemm_bytes(d->M, d->K, d->N, d->type), gemm_bytes(d->K, d->N, d->M, d->type));
}

extern "C" int stacklstm_linear_fwd(const slstm_linear_dims* d, const void* x, const void* W, const void* b, const void* res,
                                    void* y, void* z, void* workspace, size_t ws_bytes, void* stream) {
  if (!linear_ok(d)) return SLSTM_EINVAL;
  if (d->M == 0) return SLSTM_OK;
  if (!x || !W || !y || !workspace || !al16(workspace)) return SLSTM_EINVAL;
  if (res == y && row_stride(d->ld_res, d->N) != row_stride(d->ld_y, d->N)) return SLSTM_EINVAL;
  if (ws_bytes < stacklstm_linear_fwd_workspace_bytes(d)) return SLSTM_EWORKSPACE;
  GemmArgs g = {};
  g.M = (int)d->M, g.N = d->N, g.K = d->K, g.A = x, g.B = W;
  g.lda = row_stride(d->ld_x, d->K), g.ldb = row_stride(d->ld_w, d->N);
  g.bias = b, g.res = res, g.y = y, g.z = z, g.act = d->act;
  g.ldy = row_stride(d->ld_y, d->N), g.ldr = row_stride(d->ld_res, d->N);
  return gemm<false, true>(g, d->type, (float*)workspace, as_stream(stream)) == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
}

extern "C" int stacklstm_linear_bwd(const slstm_linear_dims* d, const void* x, const void* W, const void* z, const void* dy,
                                    void* dx, void* dW, void* db, void* workspace, size_t ws_bytes, void* stream) {
  if (!linear_ok(d)) return SLSTM_EINVAL;
  const bool act = d->act != SLSTM_ACT_NONE;
  if (!workspace || !al16(workspace)) return SLSTM_EINVAL;
  if (d->M > 0 && (!dy || (act && !z) || (dW && !x) || (dx && !W))) return SLSTM_EINVAL;
  if (ws_bytes < stacklstm_linear_bwd_workspace_bytes(d)) return SLSTM_EWORKSPACE;
  const hipStream_t st = as_stream(stream);
  char* ws = (char*)workspace;
  float* dbp = (float*)(ws + dz_bytes(d));
  float* part = (float*)(ws + dz_bytes(d) + db_bytes(d));
  const void* dz = act ? ws : dy;
  const int64_t ldz = act ? (int64_t)dz_stride(d) : row_stride(d->ld_dy, d->N);
  hipError_t e = hipSuccess;
  if (db || (act && (dx || dW) && d->M > 0)) {
    const DzPlan p = dz_plan(d);
    DzArgs a = {};
    a.M = (int)d->M, a.N = d->N, a.act = d->act, a.rows = p.rows, a.dy = dy, a.z = act ? z : nullptr;
    a.ldd = row_stride(d->ld_dy, d->N), a.ldz = ldz, a.dz = act && (dx || dW) ? ws : nullptr, a.part = db ? dbp : nullptr;
    const dim3 grid(p.strips, p.blocks);
    if (d->type == SLSTM_F32) hipLaunchKernelGGL(k_linear_dz<float>, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(k_linear_dz<bf16_t>, grid, dim3(256), 0, st, a);
    if (db) {
      const dim3 cols((d->N + 7) / 8);
      if (d->type == SLSTM_F32) hipLaunchKernelGGL(k_linear_db<float>, cols, dim3(256), 0, st, dbp, p.blocks, d->N, (float*)db);
      else hipLaunchKernelGGL(k_linear_db<bf16_t>, cols, dim3(256), 0, st, dbp, p.blocks, d->N, (bf16_t*)db);
    }
    e = hipGetLastError();
  }
  if (e == hipSuccess && dx && d->M > 0) {
    GemmArgs g = {};
    g.M = (int)d->M, g.N = d->K, g.K = d->N, g.A = dz, g.B = W, g.lda = ldz, g.ldb = row_stride(d->ld_w, d->N);
    g.y = dx, g.ldy = d->K;
    e = gemm<false, false>(g, d->type, part, st);
  }
  if (e == hipSuccess && dW) {
    GemmArgs g = {};
    g.M = d->K, g.N = d->N, g.K = (int)d->M, g.A = x, g.B = dz, g.lda = row_stride(d->ld_x, d->K), g.ldb = ldz;
    g.y = dW, g.ldy = d->N;
    e = gemm<true, true>(g, d->type, part, st);
  }
  return e == hipSuccess ? SLSTM_OK : SLSTM_EDEVICE;
}
