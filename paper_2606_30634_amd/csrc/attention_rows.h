// Tiles of 32 rows of a head on v_mfma_f32_32x32x2_f32: operands from global memory, products, the sum of a
// block's waves and the rows it writes.  Shared by the fp32 attention kernels (attention.hip, attention_ranges.hip).
#pragma once
#include "common.h"

namespace {

constexpr int TR = 32;  // rows of a block and of a tile
constexpr int NW = 4;   // waves of a block

__device__ __forceinline__ f32x16 mfma2(float a, float b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

// Orders one lane's LDS accesses before another lane's of the same wave
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Four consecutive elements as fp32 (rows start on 4 elements: head_dim and every width are
// multiples of 32)
__device__ __forceinline__ f32x4 ld4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ __forceinline__ f32x4 ld4(const bf16* p) {
  const bf16x4 v = *reinterpret_cast<const bf16x4*>(p);
  return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
}
__device__ __forceinline__ void st4(float* p, const f32x4& v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ void st4(bf16* p, const f32x4& v) {
  *reinterpret_cast<bf16x4*>(p) = bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
}

// Row operand: this lane's half of row `row` (stride ld) for a contraction over the head dimension:
// group q holds elements 8 q + 4 (lane / 32) .. + 3, so that step (q, j) pairs 8 q + j with 8 q + 4 + j.
template <int HD>
struct RowFrag {
  f32x4 v[HD / 8];
  template <typename T>
  __device__ __forceinline__ void load(const T* p, int64_t row, int ld) {
    const T* r = p + row * ld + 4 * (threadIdx.x % 64 / 32);
#pragma unroll
    for (int q = 0; q < HD / 8; ++q) v[q] = ld4(r + 8 * q);
  }
  // whether every value of the wave's rows is finite (the sum stays 0 as long as they are)
  __device__ __forceinline__ bool finite() const {
    float z = 0.f;
#pragma unroll
    for (int q = 0; q < HD / 8; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) z = __builtin_fmaf(v[q][j], 0.f, z);
    return __all(z == 0.f);
  }
};
// S (+)= A B^T over the head dimension: accumulator rows are A's rows, columns B's
template <int HD>
__device__ __forceinline__ f32x16 rows_product(const RowFrag<HD>& a, const RowFrag<HD>& b) {
  f32x16 s;
#pragma unroll
  for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
  for (int q = 0; q < HD / 8; ++q)
#pragma unroll
    for (int j = 0; j < 4; ++j) s = mfma2(a.v[q][j], b.v[q][j], s);
  return s;
}

// acc[dt] (rows 32 dt .. of X^T, columns the block's rows) += X^T W over the 32 tile rows of X, whose
// weights w sit in an accumulator (rows: tile rows).  Tile row r is row min(row0 + r, last) of X.
template <int HD>
struct ColFrag {
  float f[HD / 32][16];
  template <typename T>
  __device__ __forceinline__ void load(const T* x, int row0, int last, int ld) {
    const int lane = threadIdx.x % 64;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const T* r = x + (int64_t)min(row0 + 8 * (e / 4) + 4 * (lane / 32) + e % 4, last) * ld + lane % 32;
#pragma unroll
      for (int dt = 0; dt < HD / 32; ++dt) f[dt][e] = to_f32(r[32 * dt]);
    }
  }
  __device__ __forceinline__ void product(f32x16 (&acc)[HD / 32], const f32x16& w) const {
#pragma unroll
    for (int e = 0; e < 16; ++e)
#pragma unroll
      for (int dt = 0; dt < HD / 32; ++dt) acc[dt] = mfma2(f[dt][e], w[e], acc[dt]);
  }
};
template <int HD, typename T>
__device__ __forceinline__ void cols_product(f32x16 (&acc)[HD / 32], const T* x, int row0, int last, int ld,
                                             const f32x16& w) {
  ColFrag<HD> f;
  f.load(x, row0, last, ld);
  f.product(acc, w);
}

// The same sum where some column does not see every tile row and a row holds an infinity or a NaN: its
// weights there are 0, and 0 times such a value would be a NaN.  Row by row, each column the rows that
// it sees (seen(r) for this lane's); tile: 32 x 32 floats of this wave's LDS.
template <int HD, typename T, typename F>
__device__ __forceinline__ void cols_product_seen(f32x16 (&acc)[HD / 32], const T* x, int row0, int ld,
                                                  const f32x16& w, float* tile, F&& seen) {
  const int lane = threadIdx.x % 64;
#pragma unroll
  for (int e = 0; e < 16; ++e) tile[(8 * (e / 4) + 4 * (lane / 32) + e % 4) * TR + lane % 32] = w[e];
  wave_fence();
#pragma unroll
  for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll 1
    for (int r = 0; r < TR; ++r) {
      if (!seen(r)) continue;
      const float wr = tile[r * TR + lane % 32];
      const T* xr = x + (int64_t)(row0 + r) * ld + 32 * dt + 4 * (lane / 32);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 v = ld4(xr + 8 * q);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[dt][4 * q + j] += wr * v[j];
      }
    }
  wave_fence();
}

// LDS of one wave (floats): its partial sums, [dt][e][lane]
template <int HD>
constexpr int WAVE_LDS = (HD / 32) * 16 * 64;

// Sum of the waves' accumulators over red ([wave][dt][e][lane]), in wave order.
template <int HD>
__device__ __forceinline__ void put_partial(float* red, const f32x16 (&acc)[HD / 32], float scale) {
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
#pragma unroll
  for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) red[((wave * (HD / 32) + dt) * 16 + e) * 64 + lane] = acc[dt][e] * scale;
}
template <int HD>
__device__ __forceinline__ float get_sum(const float* red, int dt, int e) {
  const int lane = threadIdx.x % 64;
  float v = red[(dt * 16 + e) * 64 + lane];
#pragma unroll
  for (int w = 1; w < NW; ++w) v += red[((w * (HD / 32) + dt) * 16 + e) * 64 + lane];
  return v;
}

// The summed rows leave as rows of out (row row0 + lane mod 32, elements 32 dt + 8 (e / 4) + 4 (lane /
// 32) ..+ 3: 16-byte chunks): wave w writes the chunks e / 4 = w.  With RoPE tables the rows are
// rotated back by -angle(position) first: element c < hd/2 pairs with c + hd/2, which the same lane
// holds (another dt, or for head dimension 32 e + 8).
template <int HD, typename T>
__device__ __forceinline__ void store_rows(const float* red, float scale, T* out, int ld, int row0, int S,
                                           const float* cos_t, const float* sin_t, float* out32 = nullptr) {
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int row = row0 + lane % 32;
#pragma unroll
  for (int dt = 0; dt < HD / 32; ++dt) {
    const int c = 32 * dt + 8 * wave + 4 * (lane / 32);
    f32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = get_sum<HD>(red, dt, 4 * wave + j) * scale;
    if (cos_t) {
      constexpr int HH = HD / 2;
      const bool first = c < HH;
      const int pd = HD == 32 ? dt : (first ? dt + HD / 64 : dt - HD / 64), pe = HD == 32 ? (4 * wave) ^ 8 : 4 * wave;
      const int64_t t = (int64_t)min(row, S - 1) * HH + c % HH;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = get_sum<HD>(red, pd, pe + j) * scale, cs = cos_t[t + j], sn = sin_t[t + j];
        v[j] = first ? v[j] * cs + p * sn : v[j] * cs - p * sn;
      }
    }
    if (row < S) {
      st4(out + (int64_t)row * ld + c, v);
      if (out32) st4(out32 + (int64_t)row * ld + c, v);
    }
  }
}

__device__ __forceinline__ float pair_max(float v) { return fmaxf(v, __shfl_xor(v, 32, WAVE)); }
__device__ __forceinline__ float pair_sum(float v) { return v + __shfl_xor(v, 32, WAVE); }

// Waves per SIMD the kernels are built for: within these bounds the accumulators stay in vector registers
// and nothing spills.  Left to itself the compiler keeps them in accumulator registers, copies them for the
// row-by-row sums of a tile with non-finite rows, and fits one wave less (16 sequences of 512, 8 heads of
// 64: forward 122 us against 99, backward 469 against 423).
constexpr int fwd_waves(int hd) { return hd == 128 ? 1 : hd == 64 ? 3 : 4; }
constexpr int bwd_waves(int hd) { return hd == 128 ? 1 : 2; }

}  // namespace
