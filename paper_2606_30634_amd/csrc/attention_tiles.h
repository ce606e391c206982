// Tiles of a head on v_mfma_f32_32x32x16_bf16: streamed to LDS, read as operands, and the rows written from
// accumulators.  Shared by the bf16 attention kernels (attention_mfma.hip, which has the layout's description,
// and attention_ranges_mfma.hip).
#pragma once
#include "common.h"

namespace {

constexpr int QB = 128;   // queries (forward, dQ) or keys (dK/dV) per workgroup
constexpr int KB = 64;    // rows per streamed tile
constexpr int NT = 256;   // 4 waves
constexpr float LOG2E = 1.4426950408889634f;


typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// two floats -> two RNE bf16 in one dword (a in the low half): one v_cvt_pk_bf16_f32
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const bf16x2 v = __builtin_convertvector((f32x2){a, b}, bf16x2);
  uint32_t u;
  __builtin_memcpy(&u, &v, 4);
  return u;
}

// Chunk permutation of tile row r (HD/8 chunks of 16 bytes per row):
//   HD = 128 (a row spans the 64 banks): swz = 4 (r mod 4) + (r / 4 mod 4), a bijection on any 16
//     consecutive rows (16-byte row reads) that sends 4 consecutive rows (k0 a multiple of 4) to 4
//     different 4-chunk groups (transposing reads of 4 rows x 32 columns);
//   HD = 64 (two rows per 64 banks): swz = 4 (r / 2 mod 2) + (r / 4 mod 4), the same two properties
//     over the rows of one parity;
//   HD = 32 (four rows per 64 banks): swz = r / 4 mod 4: 16 consecutive rows read 16 different chunks, and 4
//     consecutive rows of 32 columns are all the chunks of 4 rows.
template <int HD>
__device__ __forceinline__ int swz(int r) {
  if constexpr (HD == 128) return 4 * (r & 3) + ((r >> 2) & 3);
  else if constexpr (HD == 64) return 4 * ((r >> 1) & 1) + ((r >> 2) & 3);
  else return (r >> 2) & 3;
}
// element index of (row r, column c) in a swizzled [row][HD] tile
template <int HD>
__device__ __forceinline__ int tidx(int r, int c) {
  return r * HD + ((((c >> 3) ^ swz<HD>(r))) << 3) + (c & 7);
}

// fragment of a [row][k] tile: row r0 + lane mod 32, k = k0 + 8 (lane / 32) .. +7
template <int HD>
__device__ __forceinline__ bf16x8 frag_rows(const bf16* T, int r0, int k0) {
  const int l = threadIdx.x % 64;
  return *reinterpret_cast<const bf16x8*>(T + tidx<HD>(r0 + l % 32, k0 + 8 * (l / 32)));
}

// fragment of the transpose of a [k][col] tile: col c0 + lane mod 32, k = k0 + 8 (lane / 32) .. +7,
// from two transposing reads (each 16-lane group reads 4 rows x 16 columns; lane j gets column j)
template <int HD>
__device__ __forceinline__ bf16x8 frag_cols(const bf16* T, int c0, int k0) {
  const int l = threadIdx.x % 64, g = l / 16, i = l % 16;
  const int c = c0 + 16 * (g & 1) + 4 * (i & 3);
  const int k = k0 + 8 * (g >> 1) + (i >> 2);
  typedef __attribute__((address_space(3))) v4i16_t lds_v4i16;
  const v4i16_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(T + tidx<HD>(k, c)));
  const v4i16_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(T + tidx<HD>(k + 4, c)));
  bf16x8 f;
  __builtin_memcpy(&f, &lo, 8);
  __builtin_memcpy(reinterpret_cast<char*>(&f) + 8, &hi, 8);
  return f;
}

// gfx950 v_permlane32_swap(X, Y) exchanges lanes 32..63 of X with lanes 0..31 of Y (no LDS trip).
__device__ __forceinline__ void swap32(uint32_t& x, uint32_t& y) {
  const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
  x = r[0];
  y = r[1];
}
// v combined with the value of lane l ^ 32: after swap32(a, a) the two results are v and the
// partner's value in some order, so a commutative op of the two gives the same value on both lanes
__device__ __forceinline__ float pair_max(float v) {
  uint32_t a = __float_as_uint(v), b = a;
  swap32(a, b);
  return fmaxf(__uint_as_float(a), __uint_as_float(b));
}
__device__ __forceinline__ float pair_sum(float v) {
  uint32_t a = __float_as_uint(v), b = a;
  swap32(a, b);
  return __uint_as_float(a) + __uint_as_float(b);
}

// B operand (8 consecutive k at column lane mod 32) from a 32x32 accumulator whose rows are the k
// index, for the 16-row group starting at accumulator index ib (0 or 8).  Lane half h holds rows
// ib+4h..ib+4h+3 of the group; the operand wants rows 8h..8h+7: half 0 needs its own rows ib..ib+3
// then its partner's, half 1 its partner's rows ib+4..ib+7 then its own.  Swapping the packed lower
// pair (lanes 32..63) with the packed upper pair (lanes 0..31) leaves exactly that in every lane:
// the first word of each swap is the operand's first half, the second word its second half.
template <int IB>
__device__ __forceinline__ bf16x8 acc_rows_to_b(const f32x16& s) {
  uint32_t lo0 = pack2(s[IB + 0], s[IB + 1]), lo1 = pack2(s[IB + 2], s[IB + 3]);
  uint32_t hi0 = pack2(s[IB + 4], s[IB + 5]), hi1 = pack2(s[IB + 6], s[IB + 7]);
  swap32(lo0, hi0);
  swap32(lo1, hi1);
  const uint32_t pw[4] = {lo0, lo1, hi0, hi1};
  bf16x8 r;
  __builtin_memcpy(&r, pw, 16);
  return r;
}

// The same operand from an accumulator split in two: hi = bf16(s) and lo = bf16(s - hi), so that
// a product with hi and one with lo add up to the product with s to about 2^-17 relative (s - hi is
// exact in fp32).
template <int IB>
__device__ __forceinline__ void acc_rows_to_b_split(const f32x16& s, bf16x8& hi, bf16x8& lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float a = s[IB + 2 * q], b = s[IB + 2 * q + 1];
    h[q] = pack2(a, b);
    l[q] = pack2(a - __uint_as_float(h[q] << 16), b - __uint_as_float(h[q] & 0xffff0000u));
  }
  swap32(h[0], h[2]);
  swap32(h[1], h[3]);
  swap32(l[0], l[2]);
  swap32(l[1], l[3]);
  __builtin_memcpy(&hi, h, 16);
  __builtin_memcpy(&lo, l, 16);
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Streamed tiles: KB rows x HD of a head (row stride ld) land in a swizzled [KB][HD] LDS tile by
// direct-to-LDS loads.  Load q of a wave writes 1 KB (16 bytes per lane, in lane order), so LDS
// chunk p = (q * 4 + wave) * 64 + lane of the tile holds row p / (HD/8), data chunk
// (p mod HD/8) ^ swz(row): the layout tidx reads.  Rows at or beyond the tile's valid rows repeat
// its last valid row (finite data whose probabilities the causal mask makes exactly zero).
template <int HD>
struct DmaRowTile {
  static constexpr int CPR = HD / 8;
  static constexpr int PER = KB * CPR / NT;  // loads per thread and tile
  static_assert(PER * NT == KB * CPR, "tile does not split evenly over the threads");
  // byte offset, from the tile's first row in global memory, of this thread's q-th load
  __device__ static uint32_t voff(int q, int ld, int rows) {
    const int p = (q * (NT / 64) + (int)threadIdx.x / 64) * 64 + (int)threadIdx.x % 64;
    const int r = p / CPR, kc = (p % CPR) ^ swz<HD>(r);
    return 2u * (uint32_t)(min(r, rows - 1) * ld + kc * 8);
  }
  // the tile's rows [row0, row0 + KB) of g (rows below S valid) into the LDS tile at lds
  __device__ static void issue(const bf16* g, int ld, int row0, int S, uint32_t lds) {
    const bf16* t = g + (int64_t)row0 * ld;
    const uint32_t w = (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x / 64) * 1024u;
#pragma unroll
    for (int q = 0; q < PER; ++q) dma16(t, voff(q, ld, S - row0), lds + w + (uint32_t)q * (NT / 64) * 1024u);
  }
  // This thread's q-th load with a range that ends with the head's last row (rows past it arrive as
  // zeros); lds: the tile's address plus 1 KB per wave.
  __device__ static void issue_range(u32x4 range, int q, int ld, uint32_t lds) {
    dma16_range(range, voff(q, ld, KB), lds + (uint32_t)q * (NT / 64) * 1024u);
  }
};

// stages of the streamed-tile ring: a tile's loads are issued NS - 1 iterations before it is used
template <int HD>
constexpr int ring_stages() { return HD == 128 ? 2 : 3; }

// Waits until this thread's loads of the current iteration's stage are in LDS: issued after them
// are the loads of the next NS - 2 iterations, those that exist (`more` = the next iteration does)
template <int NS, int PER_STAGE>
__device__ __forceinline__ void ring_wait(bool more) {
  if constexpr (NS >= 3) {
    if (more) wait_vm_lds<(NS - 2) * PER_STAGE>();
    else wait_vm_lds<0>();
  } else {
    wait_vm_lds<0>();
  }
}

// Writes a wave's 32 columns of X^T (accumulators: rows d, column = the wave's 32 rows) as rows of
// out (row stride ldo) through the LDS staging area, scaled.  Ends with all staging reads done.
// With rope tables the rows are gradients w.r.t. RoPE-rotated vectors and leave rotated back by
// -angle(position, i) (position = row within the sequence): the gradient w.r.t. the unrotated ones.
template <int HD>
__device__ __forceinline__ void stage_rows_from_t(float* __restrict__ stage, const f32x16* acc, float scale) {
  constexpr int OP = HD + 4;  // fp32 staging pitch
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, half = lane / 32, col = lane % 32;
#pragma unroll
  for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e)
      stage[(wave * 32 + col) * OP + dt * 32 + 8 * (e / 4) + 4 * half + (e % 4)] = acc[dt][e] * scale;
  __syncthreads();
}
template <int HD>
__device__ __forceinline__ void store_rows_from_t(float* __restrict__ stage, const f32x16* acc, float scale,
                                                  bf16* __restrict__ out, int ldo, int row0_wg, int S,
                                                  const float* rope_cos = nullptr,
                                                  const float* rope_sin = nullptr,
                                                  float* __restrict__ out32 = nullptr) {
  constexpr int OP = HD + 4;
  stage_rows_from_t<HD>(stage, acc, scale);
  for (int c = threadIdx.x; c < QB * HD / 8; c += NT) {
    const int r = c / (HD / 8), d = (c % (HD / 8)) * 8;
    const int row = row0_wg + r;
    if (row >= S) continue;
    const float* sr = stage + r * OP;
    bf16x8 ov;
    if (rope_cos) {
      constexpr int HH = HD / 2;
      const bool first = d < HH;
      const int i0 = d % HH;
      const float* xp = sr + (first ? d + HH : d - HH);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float cs = rope_cos[row * HH + i0 + q], sn = rope_sin[row * HH + i0 + q];
        ov[q] = (bf16)(first ? sr[d + q] * cs + xp[q] * sn : sr[d + q] * cs - xp[q] * sn);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q) ov[q] = (bf16)sr[d + q];
      if (out32) {  // the fp32 rows too (same layout)
        float* o32 = out32 + (int64_t)row * ldo + d;
        *reinterpret_cast<f32x4*>(o32) = f32x4{sr[d], sr[d + 1], sr[d + 2], sr[d + 3]};
        *reinterpret_cast<f32x4*>(o32 + 4) = f32x4{sr[d + 4], sr[d + 5], sr[d + 6], sr[d + 7]};
      }
    }
    *reinterpret_cast<bf16x8*>(out + (int64_t)row * ldo + d) = ov;
  }
  __syncthreads();
}

// The same rows in fp32, unscaled (partial sums of a split dK/dV item)
template <int HD>
__device__ __forceinline__ void store_partial_from_t(float* __restrict__ stage, const f32x16* acc,
                                                     float* __restrict__ out, int ldo, int row0_wg, int S) {
  stage_rows_from_t<HD>(stage, acc, 1.0f);
  for (int c = threadIdx.x; c < QB * HD / 4; c += NT) {
    const int r = c / (HD / 4), d = (c % (HD / 4)) * 4, row = row0_wg + r;
    if (row < S)
      *reinterpret_cast<f32x4*>(out + (int64_t)row * ldo + d) = *reinterpret_cast<const f32x4*>(stage + r * (HD + 4) + d);
  }
  __syncthreads();
}

// Work item of block L in a 1-D grid of N blocks made of units of per_unit items (a unit: the blocks of
// one head, which stream the same K/V or Q/dO rows), a unit's heavier items first.  All units' heaviest
// items come first, then their second heaviest, so that the launch ends on light ones everywhere: unit
// after unit it ended on the last units' whole descents, with 1.4 of 2 waves per SIMD busy on average
// (forward of 8 x 1024 tokens, 12 heads of 64: 50 -> 38 us; 2 x 4096, 32 of 128: 513 -> 462 us; their
// backwards 105 -> 84 and 1040 -> 968 us).  The hardware places block L on XCD L mod 8: when 8 divides
// the units, XCD x gets the units x U/8 .. of the U, whose blocks (and query heads of one key/value head)
// share its L2.
__device__ __forceinline__ void xcd_item(int L, int N, int per_unit, int& unit, int& idx) {
  const int units = N / per_unit;
  if (units % 8 == 0) {
    const int u8 = units / 8, r = L / 8;
    unit = (L % 8) * u8 + r % u8;
    idx = r / u8;
  } else {
    unit = L % units;
    idx = L / units;
  }
}

template <int HD>
struct Lds {
  static constexpr int NS = ring_stages<HD>();
  static constexpr int TSZ = KB * HD;  // elements of one [KB][HD] tile
  static constexpr size_t out_bytes = (size_t)QB * (HD + 4) * 4;  // fp32 output staging
  // forward and dQ: a stage holds a K and a V tile; dK/dV: a Q and a dO tile, then the lse and
  // delta values of the tile's rows
  static constexpr size_t kv_stage = (size_t)2 * TSZ * 2;
  static constexpr size_t qd_stage = (size_t)2 * TSZ * 2 + 2 * KB * 4;
  static constexpr size_t mx(size_t x, size_t y) { return x > y ? x : y; }
  static constexpr size_t fwd_bytes() { return mx(NS * kv_stage, out_bytes); }
  static constexpr size_t dq_bytes() { return fwd_bytes(); }
  static constexpr size_t dkv_bytes() { return mx(NS * qd_stage, out_bytes); }
};

// acc += A B with the accumulator kept in accumulator registers (this file's builtin MFMAs keep theirs
// in vector registers, which 128 more would overflow).  The compiler does not know the instruction, so
// its distances are kept here: in the loop operands come from LDS reads (waited for) or vector
// instructions several MFMAs back, and one accumulator's products are 16 MFMAs apart; COPIED (outside
// the loop, where the compiler moves accumulators between registers) waits between such a move and the
// product; and acc_settled() stands between the last products and any other read.
template <bool COPIED>
__device__ __forceinline__ void mfma_acc(f32x16& acc, const bf16x8& a, const bf16x8& b) {
  if constexpr (COPIED) asm volatile("s_nop 4\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
  else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
__device__ __forceinline__ void acc_settled(f32x16 (&x)[4], f32x16 (&y)[4]) {
  asm volatile("s_nop 15\n\ts_nop 15"
               : "+a"(x[0]), "+a"(x[1]), "+a"(x[2]), "+a"(x[3]), "+a"(y[0]), "+a"(y[1]), "+a"(y[2]), "+a"(y[3]));
}
// keeps the computation of two values ahead of this point of the schedule
__device__ __forceinline__ void pin(float& x, float& y) { asm volatile("" : "+v"(x), "+v"(y)); }

}  // namespace
