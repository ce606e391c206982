// Dropout whose mask is a function of the element's place, added to a residual.
//
//   out = resid + [u(e) >= t] x 65536 / (65536 - t),  t = round(65536 p),  e = row cols + col
// u(e) is the 16-bit number e mod 8 of Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as
// easy as 1, 2, 3", 2011) of the counter (e / 8, offset) under the key seed, so that the backward makes the
// same mask again and nothing is stored.  A thread takes the 8 elements of a counter: with 16-byte loads HBM
// bounds it (8192 x 4096 bf16 with its residual: 201 MB in 37 us, 5.4 TB/s; the generator's 20 wide products a counter
// fit beside that).
#include "common.h"
#include "kernels.h"
#include <algorithm>

namespace {

__device__ __forceinline__ u32x4 philox(uint64_t g, uint64_t offset, uint64_t seed) {
  uint32_t x0 = (uint32_t)g, x1 = (uint32_t)(g >> 32), x2 = (uint32_t)offset, x3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)x0 * 0xD2511F53u, b = (uint64_t)x2 * 0xCD9E8D57u;
    x0 = (uint32_t)(b >> 32) ^ x1 ^ k0;
    x2 = (uint32_t)(a >> 32) ^ x3 ^ k1;
    x1 = (uint32_t)b;
    x3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{x0, x1, x2, x3};
}

template <typename T>
struct Vec8 {
  T v[8];
};

// VEC: the 8 elements of a counter are contiguous and aligned in every array (row: the counters of a row, or
// 0 where the arrays have no gaps); else they are taken one by one.  From counter g0 on.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dropout(DropoutArgs a, int64_t row, int64_t n, int64_t g0) {
  const int64_t g = g0 + (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (8 * g >= n) return;
  u32x4 w = {0, 0, 0, 0};
  if (a.threshold) w = philox((uint64_t)g, a.offset, a.seed);
  const float scale = 65536.0f / (float)(65536u - a.threshold);
  auto one = [&](int j, float x) {
    const uint32_t u = j % 2 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu;
    return u >= a.threshold ? x * scale : 0.f;
  };
  const T *x = (const T*)a.x, *r = (const T*)a.resid;
  T* o = (T*)a.out;
  if constexpr (VEC) {
    const int64_t i = row ? g / row : 0, c = 8 * (row ? g % row : g);
    if (row || 8 * g + 8 <= n) {
      const Vec8<T> xv = *reinterpret_cast<const Vec8<T>*>(__builtin_assume_aligned(x + i * a.ldx + c, 16));
      Vec8<T> ov;
      if (r) {
        const Vec8<T> rv = *reinterpret_cast<const Vec8<T>*>(__builtin_assume_aligned(r + i * a.ldr + c, 16));
#pragma unroll
        for (int j = 0; j < 8; ++j) ov.v[j] = from_f32<T>(one(j, to_f32(xv.v[j])) + to_f32(rv.v[j]));
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) ov.v[j] = from_f32<T>(one(j, to_f32(xv.v[j])));
      }
      *reinterpret_cast<Vec8<T>*>(__builtin_assume_aligned(o + i * a.ldo + c, 16)) = ov;
      return;
    }
  }
  int64_t i = 8 * g / a.cols, c = 8 * g % a.cols;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (8 * g + j >= n) break;
    float v = one(j, to_f32(x[i * a.ldx + c]));
    if (r) v += to_f32(r[i * a.ldr + c]);
    o[i * a.ldo + c] = from_f32<T>(v);
    if (++c == a.cols) {
      c = 0;
      ++i;
    }
  }
}

}  // namespace

void launch_dropout(bool bf, const DropoutArgs& a, hipStream_t st) {
  const int64_t n = a.rows * a.cols;
  const int per = bf ? 8 : 4;  // elements of 16 bytes
  auto fits = [&](const void* p, int64_t ld) { return !p || ((uintptr_t)p % 16 == 0 && ld % per == 0); };
  const bool flat = a.rows == 1 || (a.ldx == a.cols && (!a.resid || a.ldr == a.cols) && a.ldo == a.cols);
  const bool vec = flat ? fits(a.x, 0) && fits(a.resid, 0) && fits(a.out, 0)
                        : a.cols % 8 == 0 && fits(a.x, a.ldx) && fits(a.resid, a.ldr) && fits(a.out, a.ldo);
  const int64_t row = flat ? 0 : a.cols / 8;
  // a launch takes fewer than 2^32 threads: 2^35 elements
  for (int64_t g0 = 0; 8 * g0 < n; g0 += 256 * MAX_BLOCKS_256) {
    const unsigned blocks = (unsigned)std::min(cdiv(cdiv(n - 8 * g0, 8), 256), MAX_BLOCKS_256);
    if (bf && vec) dropout<bf16, true><<<blocks, 256, 0, st>>>(a, row, n, g0);
    else if (bf) dropout<bf16, false><<<blocks, 256, 0, st>>>(a, row, n, g0);
    else if (vec) dropout<float, true><<<blocks, 256, 0, st>>>(a, row, n, g0);
    else dropout<float, false><<<blocks, 256, 0, st>>>(a, row, n, g0);
  }
}
