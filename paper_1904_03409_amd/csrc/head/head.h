// Shared device helpers of the operators behind the recurrence (include/stacklstm_head.h).
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../common.h"

// Rows are read and written in vectors of 16 bytes from the row's first element on, whatever the
// row's alignment (global memory instructions need none on gfx950); the last vector of a row whose
// width is no whole number of vectors goes element by element.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));

template <typename T> struct vec;
template <> struct vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(u32x4 r, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
  }
  static __device__ __forceinline__ u32x4 pack(const float (&v)[4]) {
    return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
};
template <> struct vec<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(u32x4 r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(r[i] << 16);
      v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  }
  // nearest even, the one rounding of a 16-bit output
  static __device__ __forceinline__ u32x4 pack(const float (&v)[8]) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r[i] = (uint32_t)f32_to_bf16_bits(v[2 * i]) | (uint32_t)f32_to_bf16_bits(v[2 * i + 1]) << 16;
    return r;
  }
};
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16_t v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ void from_f32(float& d, float v) { d = v; }
__device__ __forceinline__ void from_f32(bf16_t& d, float v) { d = f32_to_bf16_bits(v); }

// v with its first s elements taken away, zeros behind the others.
template <typename T>
__device__ __forceinline__ u32x4 shift_vec(u32x4 v, int s) {
  if constexpr (sizeof(T) == 2) {
    const u32x4 w = {__builtin_amdgcn_alignbit(v[1], v[0], 16), __builtin_amdgcn_alignbit(v[2], v[1], 16),
                     __builtin_amdgcn_alignbit(v[3], v[2], 16), v[3] >> 16};
    v = s & 1 ? w : v;
    s >>= 1;
  }
  v = s & 1 ? u32x4{v[1], v[2], v[3], 0u} : v;
  v = s & 2 ? u32x4{v[2], v[3], 0u, 0u} : v;
  return s >= 4 ? u32x4{0u, 0u, 0u, 0u} : v;
}
// Vector i of a row of W elements, zeros past the row's end, in two parts: the load, of the row's last 16 bytes where the row
// ends in the vector or before it (no branch waits for a value), and the shift to the vector's place.
template <typename T>
__device__ __forceinline__ u32x4 fetch_vec(const T* row, int i, int W) {
  constexpr int V = vec<T>::N;
  if (W >= V) return *(const u32x4_any*)(row + min(i * V, W - V));
  u32x4 r = {0u, 0u, 0u, 0u};
  if constexpr (V == 4) {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (i * V + k < W) r[k] = __float_as_uint(row[i * V + k]);
  } else {
#pragma unroll
    for (int k = 0; k < 7; ++k)
      if (i * V + k < W) r[k / 2] |= (uint32_t)row[i * V + k] << (16 * (k & 1));
  }
  return r;
}
template <typename T>
__device__ __forceinline__ u32x4 place_vec(u32x4 v, int i, int W) {
  constexpr int V = vec<T>::N;
  if (W < V) return v;
  const int s = i * V - min(i * V, W - V);
  if (W % V != 0) return shift_vec<T>(v, s);
  return s ? u32x4{0u, 0u, 0u, 0u} : v;
}
template <typename T>
__device__ __forceinline__ u32x4 load_vec(const T* row, int i, int W) { return place_vec<T>(fetch_vec(row, i, W), i, W); }
template <typename T>
__device__ __forceinline__ void store_vec(T* row, int i, int W, const float (&v)[vec<T>::N]) {
  constexpr int V = vec<T>::N;
  if ((i + 1) * V <= W) {
    *(u32x4_any*)(row + i * V) = vec<T>::pack(v);
    return;
  }
#pragma unroll
  for (int k = 0; k < V - 1; ++k)
    if (i * V + k < W) from_f32(row[i * V + k], v[k]);
}

// The whole vectors c0, c0 + STEP, .. of a row, -inf behind them (no share in maximum and sums), and with row_end the element
// behind the last whole one that lane t takes of the fewer than a vector that are left: -inf for most. (Partial vectors
// put together element by element cost a branch to each vector and the registers of its other outcome.)
template <int STEP, typename T, int NV>
__device__ __forceinline__ void load_row(u32x4 (&raw)[NV], const T* row, int c0, int W) {
  constexpr uint32_t low = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    raw[i] = u32x4{low, low, low, low};
    if (c0 + i * STEP < W / vec<T>::N) raw[i] = *(const u32x4_any*)(row + (c0 + i * STEP) * vec<T>::N);
  }
}
template <typename T>
__device__ __forceinline__ bool has_end(int t, int W) { return t < W % vec<T>::N; }
template <typename T>
__device__ __forceinline__ int end_place(int t, int W) { return W / vec<T>::N * vec<T>::N + t; }
template <typename T>
__device__ __forceinline__ float row_end(const T* row, int t, int W) {
  return has_end<T>(t, W) ? to_f32(row[end_place<T>(t, W)]) : -INFINITY;
}
// f(i, v): the values of whole vector c0 + i STEP, written to the row.
template <int STEP, typename T, int NV, typename F>
__device__ __forceinline__ void store_row(T* row, int c0, int W, F f) {
  constexpr int V = vec<T>::N;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (c0 + i * STEP < W / V) {
      float v[V];
      f(i, v);
      *(u32x4_any*)(row + (c0 + i * STEP) * V) = vec<T>::pack(v);
    }
    __builtin_amdgcn_sched_barrier(0);                 // (one vector unpacked at a time)
  }
}

// Packed values that are unpacked again behind this point, instead of being kept unpacked in registers.
__device__ __forceinline__ void opaque_vec(u32x4& v) { asm volatile("" : "+v"(v)); }
// Order between a wave's LDS stores and its other lanes' loads of them.
__device__ __forceinline__ void wave_lds() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Reductions over groups of N neighbouring lanes (N a power of two up to 64), the result in every
// lane: DPP moves inside a row of 16 lanes, row and half swaps above it; no LDS.
struct op_sum { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct op_max { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };
template <int CTRL>
__device__ __forceinline__ float dpp_move(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <typename Op>
__device__ __forceinline__ float row_swap(float v, Op op) {        // lane ^ 16
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <typename Op>
__device__ __forceinline__ float half_swap(float v, Op op) {       // lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <int N, typename Op>
__device__ __forceinline__ float lanes(float v, Op op) {
  asm("" : "+v"(v));                                   // (a product stays rounded: fused into the first sum it gives every lane another result)
  if constexpr (N >= 2) v = op(v, dpp_move<0xb1>(v));              // quad_perm 1, 0, 3, 2
  if constexpr (N >= 4) v = op(v, dpp_move<0x4e>(v));              // quad_perm 2, 3, 0, 1
  if constexpr (N >= 8) v = op(v, dpp_move<0x141>(v));             // row_half_mirror
  if constexpr (N >= 16) v = op(v, dpp_move<0x140>(v));            // row_mirror
  if constexpr (N >= 32) v = row_swap(v, op);
  if constexpr (N >= 64) v = half_swap(v, op);
  return v;
}
// The other way round: over the lanes that have the same place in their group of N, the groups of a wave joined.
template <int N, typename Op>
__device__ __forceinline__ float across(float v, Op op) {
  asm("" : "+v"(v));
  if constexpr (N <= 8) v = op(v, __shfl_xor(v, 8));
  if constexpr (N <= 16) v = row_swap(v, op);
  if constexpr (N <= 32) v = half_swap(v, op);
  return v;
}
// Over a workgroup of NT threads (N <= 64: over the lane's group of N), the result in every thread. `red`:
// NT / 64 floats of LDS that no other reduction in flight uses; one barrier.
template <int NT, typename Op>
__device__ __forceinline__ float group_reduce(float v, Op op, float* red) {
  v = lanes<(NT < 64 ? NT : 64)>(v, op);
  if constexpr (NT > 64) {
    constexpr int W = NT / 64;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lanes<W>(red[threadIdx.x & (W - 1)], op);
  }
  return v;
}

// Sum over P rows of N columns, 8 columns to a workgroup of 1024 threads: column blockIdx.x * 8 + threadIdx.x in the first 8. A
// column's 128 threads take a row each in turn (768 rows of 400 columns: 3.8 us where 32 threads to a column took 4.4).
__device__ __forceinline__ float column_sum(const float* part, int P, int N, float (&red)[16][8]) {
  const int n = blockIdx.x * 8 + (threadIdx.x & 7);
  float s = 0.f;
  if (n < N) {
#pragma unroll 4
    for (int p = threadIdx.x >> 3; p < P; p += 128) s += part[(int64_t)p * N + n];
  }
  s = across<8>(s, op_sum());
  if ((threadIdx.x & 63) < 8) red[threadIdx.x >> 6][threadIdx.x & 7] = s;
  __syncthreads();
  float v = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) v += red[w][threadIdx.x & 7];
  return v;
}

constexpr float kLog2e = 1.4426950408889634f;
// exp((x - m) k ln 2) as 2^(x k - mk) in one fused step, m the largest x of a row. mk is m k rounded: every term of a row is
// off by the one factor 2^off, which its sum and its gradient take out again. off is up to half a rounding step of mk, 32 where
// |mk| is below 2^30; past that the factor (or its square) would leave fp32's range, but no value there is within 64 of m k but m
// itself: an element is the maximum or nothing (2^-64), and is told from it by any k that is no smaller. A power of two makes
// m k exact and off 0.
struct Expo {
  float k, mk, off;
  __device__ __forceinline__ Expo() {}
  __device__ __forceinline__ Expo(float m, float k_) : k(k_), mk(m * k_) {
    if (!(fabsf(mk) < 0x1p30f) && fabsf(m) < INFINITY) {
      // (past fp32's range a smaller power does: neighbours of such an m are 2^81 apart and more, and k is at most 2^21)
      k = fabsf(mk) < 1e38f ? __uint_as_float((__float_as_uint(k) + 0x7fffffu) & 0x7f800000u) : 0x1p-60f;
      mk = m * k;
    }
    off = __builtin_fmaf(m, k, -mk);
  }
  __device__ __forceinline__ float operator()(float x) const { return __builtin_amdgcn_exp2f(__builtin_fmaf(x, k, -mk)); }
  __device__ __forceinline__ float log_sum(float s) const { return logf(s) - off * 0.6931471805599453f; }
};

// Host side: a row stride as given (0: dense), and whether one may be.
static inline int64_t row_stride(int64_t ld, int64_t width) { return ld ? ld : width; }
static inline bool stride_ok(int64_t ld, int64_t width) { return ld == 0 || (ld >= width && ld <= ((int64_t)1 << 40)); }
// Workgroups of a launch at most: HIP refuses a grid of 2^32 threads and more, and a workgroup here has up to 1024. Calls with more
// are cut into several launches, of whole rows (or searches) that need nothing of each other.
constexpr int64_t kMostGroups = 1 << 21;
// f(first, n) for pieces of `all` that are `most` long.
template <typename F>
static inline void in_pieces(int64_t all, int64_t most, F f) {
  for (int64_t i = 0; i < all; i += most) f(i, all - i < most ? all - i : most);
}
template <typename T>
static inline T* offset(T* p, int64_t n) { return p ? p + n : nullptr; }
static inline hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }
