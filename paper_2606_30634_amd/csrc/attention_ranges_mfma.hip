// Attention over key ranges (the formulas are in attention_ranges.hip) for bf16, on the bf16 matrix cores, with the
// tiles, operand layouts and rings of attention_mfma.hip.
//
// What differs from the causal kernels there: tiles start at the first key that a query of the block sees and end
// with the last, so nothing else is loaded; every lane owns one query (one key in dK/dV) and keeps its range, and
// only tiles that some row does not see whole are masked; rows come from strided tensors; a forward block
// may hold the query heads of one key/value head (`pack` rows per query) and a share of the keys.
// A block whose result is not finite (a value that one of its rows does not see may be an infinity or a NaN, and 0
// times it is a NaN) computes the rows in question again, key by key over what they see.
//
// What bounds them: long rows the matrix cores and the vector work beside them, which one SIMD's two waves (one in
// dK/dV of 128) overlap only in part; short documents also a block's start and end and the part of its tiles that no row
// sees; a few queries on long caches HBM (16 x 32768 keys, 8 heads of 128: 5.6 TB/s).  One causal row block of 4096 tokens
// (2 sequences, 32 heads of 128 on 8), by the flops of the pairs seen: forward 336-347 us, 0.79-0.82 PFLOP/s (o kept in fp32,
// so three times the P V products: 495 us; scores capped: 385-392 us), backward 1004 us, 0.68 PFLOP/s (capped 1267, and
// 1859 with every tile past the polynomial).
#include "attention_ranges.h"
#include "attention_tiles.h"
#include <algorithm>
#include <atomic>

namespace {

// Scores in log2 units from the products x = q.k of a 32 x 32 accumulator: c (x scale), or c cap tanh(x scale / cap)
struct CapScale {
  float sl2;    // scale log2(e)
  float y_of;   // scale / cap
  float out;    // cap log2(e)
  float small;  // |x| up to which |y| <= SMALL
  static constexpr float SMALL = 0.4f;
  __device__ explicit CapScale(const RangeArgs& a) {
    sl2 = a.scale * LOG2E;
    y_of = a.cap > 0.f ? a.scale / a.cap : 0.f;
    out = a.cap * LOG2E;
    small = SMALL / y_of;
  }
};

template <int N>
__device__ __forceinline__ float largest(const f32x16 (&s)[N]) {
  float big = 0.f;
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) big = fmaxf(big, fabsf(s[t][e]));
  return big;
}

// tanh(y) up to CapScale::SMALL: y + y^3 P(y^2) with the minimax P of degree 2 (relative error 2^-23, below the rounding
// of the products)
__device__ __forceinline__ float tanh_small(float y) {
  const float z = y * y;
  float p = __builtin_fmaf(z, -0.0477941558f, 0.1327762753f);
  p = __builtin_fmaf(z, p, -0.3333188295f);
  return y * __builtin_fmaf(z, p, 1.0f);
}

// tanh(scale x / cap) of a wave's products, `big` their largest |x| in the lane.  One branch for the wave: where no
// |y| passes CapScale::SMALL (most tiles) the polynomial alone.
__device__ __forceinline__ void tanh_scores(f32x16 (&s)[2], const CapScale& c, float big) {
  if (__all(big <= c.small)) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[t][e] = tanh_small(s[t][e] * c.y_of);
  } else {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float g;
        s[t][e] = tanh_and_slope(s[t][e] * c.y_of, g);
      }
  }
}

// One score of the row-by-row path, in log2 units, and the derivative of its cap
__device__ __forceinline__ float score2(float x, const RangeArgs& a, const CapScale& c, float slope2, float far, float& g) {
  g = 1.f;
  x = a.cap > 0.f ? c.out * tanh_and_slope(x * c.y_of, g) : x * c.sl2;
  return a.slopes ? __builtin_fmaf(-slope2, fabsf(far), x) : x;
}

// Whether every element of a row held by a wave is a NaN, which nothing added to it changes
template <int N>
__device__ __forceinline__ bool all_nan(const float (&x)[N]) {
  bool nan = true;
#pragma unroll
  for (int k = 0; k < N; ++k) nan &= x[k] != x[k];
  return __all(nan);
}

// The elements of a row that a wave holds: lane, lane + 64, .. of a head (32: the upper lanes repeat the lower ones)
template <int HD>
constexpr int PER_LANE = (HD + 63) / 64;
template <int HD>
__device__ __forceinline__ int row_lane() { return threadIdx.x % (HD < 64 ? HD : 64); }

// x.y of two rows of a head
template <int HD>
__device__ __forceinline__ float row_dot(const bf16* x, const bf16* y) {
  float s = 0.f;
  for (int c = 0; c < HD; c += 8) {
    const bf16x8 u = *reinterpret_cast<const bf16x8*>(x + c), v = *reinterpret_cast<const bf16x8*>(y + c);
#pragma unroll
    for (int j = 0; j < 8; ++j) s += (float)u[j] * (float)v[j];
  }
  return s;
}

// ------------------------------------------------------------------------------------------ forward
// Rows of a forward block: row r of unit (sequence b, heads h0 .. h0 + pack - 1) is query r / pack of head
// h0 + r mod pack.
struct Rows {
  int pack, n, h0, b;
  __device__ int query(int r) const { return pack == 1 ? r : r / pack; }
  __device__ int head(int r) const { return pack == 1 ? h0 : h0 + r % pack; }
};

// o of one row again, touching only what it sees: a key per lane for the weights, columns per lane for the sum
template <int HD>
__device__ __forceinline__ void row_again(const RangeArgs& a, const Rows& rows, int r, float base, float inv, int k_lo,
                                                    int k_hi, float* part) {
  const int lane = threadIdx.x % 64, el = row_lane<HD>(), i = rows.query(r), h = rows.head(r), kvh = h / (a.Hq / a.Hkv);
  const bf16* q = rows_of<bf16>(a.q, rows.b, h) + (int64_t)i * a.q.row;
  const bf16* k = rows_of<bf16>(a.k, rows.b, kvh);
  const bf16* v = rows_of<bf16>(a.v, rows.b, kvh);
  const CapScale c(a);
  const float slope2 = a.slopes ? a.slopes[h] * LOG2E : 0.f;
  const int64_t pos = position(a, rows.b, i);
  float o[PER_LANE<HD>];
#pragma unroll
  for (int d = 0; d < PER_LANE<HD>; ++d) o[d] = 0.f;
  for (int j0 = k_lo; j0 < k_hi && !all_nan(o); j0 += 64) {
    const int n = min(64, k_hi - j0), j = j0 + min(lane, n - 1);
    float g;
    const float p = fast_exp2(score2(row_dot<HD>(q, k + (int64_t)j * a.k.row), a, c, slope2, (float)(pos - j), g) - base);
    for (int t = 0; t < n; ++t) {
      const float w = __shfl(p, t, 64);
#pragma unroll
      for (int d = 0; d < PER_LANE<HD>; ++d) o[d] += w * (float)v[(int64_t)(j0 + t) * a.v.row + 64 * d + el];
    }
  }
  const int64_t row = ((int64_t)rows.b * a.Sq + i) * a.Hq + h;
#pragma unroll
  for (int d = 0; d < PER_LANE<HD>; ++d) {
    if (part) part[row * HD + 64 * d + el] = o[d];
    else {
      ((bf16*)a.o)[row * HD + 64 * d + el] = (bf16)(o[d] * inv);
      if (a.o32) a.o32[row * HD + 64 * d + el] = o[d] * inv;
    }
  }
}

// The operand of acc_rows_to_b in three parts, each the bf16 nearest to what the ones before it leave: 24 bits, so
// that their products with V add up to those of the fp32 value.
template <int IB>
__device__ __forceinline__ void acc_rows_to_b_parts(const f32x16& s, bf16x8 (&part)[3]) {
  uint32_t w[3][4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float a = s[IB + 2 * q], b = s[IB + 2 * q + 1];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      w[k][q] = pack2(a, b);
      a -= __uint_as_float(w[k][q] << 16);
      b -= __uint_as_float(w[k][q] & 0xffff0000u);
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    swap32(w[k][0], w[k][2]);
    swap32(w[k][1], w[k][3]);
    __builtin_memcpy(&part[k], w[k], 16);
  }
}

// EXACT (o kept in fp32): P enters the P V product in three bf16 parts, 24 bits, so that the o in fp32 is one.  With
// two parts (16 bits) 4 x 2048 packed tokens, 16 heads of 128, take 61 us instead of 65.  Else P is rounded to bf16, as
// in the causal kernels (error of o 2.0e-3 of its norm; its own rounding alone 1.7e-3): long rows would pay for two products
// more (one causal row of 4096 tokens: 340 -> 495 us), few queries on ragged caches for the chain of the one wave that
// has their rows (16 x 1 query on up to 32768 keys: 227 us, 240 with two parts, 265 with three).
template <int HD, bool EXACT, bool CAP, bool BIAS>
__global__ void __launch_bounds__(NT, 2) range_flash_fwd(RangeArgs a, int pack) {
  using L = Lds<HD>;
  using TT = DmaRowTile<HD>;
  constexpr int KS = HD / 16, DT = HD / 32, NS = L::NS;
  extern __shared__ __align__(16) unsigned char smem[];
  bf16* ring = reinterpret_cast<bf16*>(smem);  // [NS][K tile | V tile], swizzled
  Rows rows;
  rows.pack = pack;
  rows.n = a.Sq * pack;
  const int nb = (rows.n + QB - 1) / QB, heads = a.Hq / pack;
  int unit, idx;  // unit: (sequence, query head or key/value head); last query blocks first
  if (a.nsplit == 1) {
    xcd_item(blockIdx.x, nb * heads * a.B, nb, unit, idx);
  } else {
    // shares of long caches share nothing in an L2, and sequences of different lengths must not fall to one XCD
    // each: every XCD takes some of all (16 answers of 1 .. 32768 keys, 8 key/value heads: 251 -> 233 us)
    unit = blockIdx.x % (heads * a.B);
    idx = blockIdx.x / (heads * a.B);
  }
  const int rb = nb - 1 - idx / a.nsplit, split = idx % a.nsplit;
  rows.h0 = unit % heads * pack;
  rows.b = unit / heads;
  const int b = rows.b, kvh = rows.h0 / (a.Hq / a.Hkv);
  const bf16* kbase = rows_of<bf16>(a.k, b, kvh);
  const bf16* vbase = rows_of<bf16>(a.v, b, kvh);
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, half = lane / 32, col = lane % 32;
  const int r0 = rb * QB + wave * 32, myr = r0 + col;
  const bool valid = myr < rows.n;
  const int i = rows.query(min(myr, rows.n - 1)), h = rows.head(min(myr, rows.n - 1));
  bf16x8 qf[KS];  // loaded first: the ranges and the first tiles' loads do not wait for them
  {
    const bf16* q = rows_of<bf16>(a.q, b, h) + (int64_t)i * a.q.row + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (valid) qf[ks] = *reinterpret_cast<const bf16x8*>(q + ks * 16);
      else for (int j = 0; j < 8; ++j) qf[ks][j] = (bf16)0.f;
    }
  }
  const int2 mask = seen_keys(a, b, i);
  const WaveKeys wk(mask, valid);
  // the block's keys, and this share's tiles of them
  int blo, bhi;
  {
    const int x = rb * QB + lane, y = x + 64;
    const int2 sx = x < rows.n ? seen_keys(a, b, rows.query(x)) : make_int2(0, 0);
    const int2 sy = y < rows.n ? seen_keys(a, b, rows.query(y)) : make_int2(0, 0);
    bhi = wave_max_i(max(sx.y, sy.y));
    blo = wave_min_i(min(sx.y > 0 ? sx.x : INT32_MAX, sy.y > 0 ? sy.x : INT32_MAX));
    if (bhi == 0) blo = 0;
  }
  const int ntile = (bhi - blo + KB - 1) / KB;
  const int t0 = __builtin_amdgcn_readfirstlane((int)((int64_t)ntile * split / a.nsplit));
  const int t1 = __builtin_amdgcn_readfirstlane((int)((int64_t)ntile * (split + 1) / a.nsplit));
  auto issue = [&](int t) {
    bf16* st = ring + (t % NS) * 2 * L::TSZ;
    TT::issue(kbase, a.k.row, blo + t * KB, bhi, lds_addr(st));
    TT::issue(vbase, a.v.row, blo + t * KB, bhi, lds_addr(st + L::TSZ));
  };
  const CapScale cs(a);
  float slope2 = 0.f;
  int64_t pos = 0;
  if constexpr (BIAS) {
    slope2 = a.slopes[h] * LOG2E;
    pos = position(a, b, i);
  }
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (t0 + s < t1) issue(t0 + s);
  // the register loads and the first tiles together, so that the wait the compiler needs for the former is not placed
  // inside the loop (where it would drain the ring)
  wait_vm_lds<0>();
  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
  float m = -INFINITY, lsum = 0.f;

  for (int kt = t0; kt < t1; ++kt) {
    ring_wait<NS, 2 * TT::PER>(kt + 1 < t1);
    block_barrier();
    if (kt + NS - 1 < t1) issue(kt + NS - 1);
    const bf16* Ks = ring + (kt % NS) * 2 * L::TSZ;
    const bf16* Vs = Ks + L::TSZ;
    const int key0 = blo + kt * KB;
    if (key0 < wk.hi && key0 + KB > wk.lo) {
      f32x16 s[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
      bf16x8 fk[2][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) fk[0][t] = frag_rows<HD>(Ks, t * 32, 0);
      static_for<KS>([&](auto KSI) {
        constexpr int ks = KSI, c = ks & 1;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (ks + 1 < KS) {
#pragma unroll
          for (int t = 0; t < 2; ++t) fk[c ^ 1][t] = frag_rows<HD>(Ks, t * 32, (ks + 1) * 16);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
          s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[c][t], qf[ks], s[t], 0, 0, 0);
        if constexpr (ks + 1 < KS) {
          static_for<2>([&](auto) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // one MFMA
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // one LDS read
          });
        }
        __builtin_amdgcn_sched_barrier(0);
      });
      // P V in four steps of 16 keys, the weights, their parts and the V fragments of the next step between this step's
      // MFMAs: a wave issues in order, and a tile's vector work ahead of all its MFMAs runs beside nothing.
      constexpr int NP = EXACT ? 3 : 1;
      const float to_log2 = CAP ? cs.out : cs.sl2;  // of a product, or with CAP its tanh
      bf16x8 part[2][NP], vf[2][DT];
      float rs[2] = {0.f, 0.f}, base;
      auto weights = [&](auto KK) {
        constexpr int kk = KK, t = kk / 2, IB = kk % 2 * 8;
#pragma unroll
        for (int e = IB; e < IB + 8; ++e) {
          const float p = fast_exp2(BIAS ? s[t][e] - base : __builtin_fmaf(s[t][e], to_log2, -base));
          s[t][e] = p;
          rs[e % 2] += p;
        }
        if constexpr (EXACT) acc_rows_to_b_parts<IB>(s[t], part[kk % 2]);
        else part[kk % 2][0] = acc_rows_to_b<IB>(s[t]);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vf[kk % 2][dt] = frag_cols<HD>(Vs, dt * 32, kk * 16);
      };
      const bool whole = wk.whole(key0, key0 + KB);
      float big = 0.f;
      if constexpr (CAP) {
        big = largest(s);
        tanh_scores(s, cs, big);
      }
      if constexpr (BIAS) {
        const float pos_far = (float)(pos - key0 - 4 * half);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float far = fabsf(pos_far - (float)(t * 32 + 8 * (e / 4) + e % 4));
            s[t][e] = __builtin_fmaf(-slope2, far, s[t][e] * to_log2);
          }
      }
      if (!whole) {
        const uint32_t first = (uint32_t)(key0 + 4 * half - mask.x), len = (uint32_t)(mask.y - mask.x);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (first + (uint32_t)(t * 32 + 8 * (e / 4) + e % 4) >= len) s[t][e] = -INFINITY;
      }
      // the lazy maximum of flash_fwd; a row that sees nothing yet has base 0 and weights of 0.  A capped score is at
      // most its |x| scale, whose maximum is at hand: it mostly says that no row's maximum moves.
      base = m;
      if (!CAP || BIAS || !__all(pair_max(big) * cs.sl2 <= m + 8.0f)) {
        float bm = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) bm = fmaxf(bm, s[t][e]);
        bm = pair_max(bm);
        if constexpr (!BIAS) bm *= to_log2;  // with it s is in log2 units already
        const bool move = bm > m + 8.0f;
        const float mn = move ? bm : m;
        const float corr = (m == -INFINITY) ? 0.f : fast_exp2(m - mn);
        base = weight_base(mn);
        m = mn;
        lsum *= corr;
        if (__any(move)) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[dt][e] *= corr;
        }
      }
      weights(std::integral_constant<int, 0>{});
      static_for<4>([&](auto KK) {
        constexpr int kk = KK;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kk + 1 < 4) weights(std::integral_constant<int, kk + 1>{});
#pragma unroll
        for (int k = NP - 1; k >= 0; --k)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[kk % 2][dt], part[kk % 2][k], o[dt], 0, 0, 0);
        if constexpr (kk + 1 < 4) {
          static_for<NP * DT>([&](auto I) {
            constexpr int i = I;
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // one MFMA
            if constexpr (i < DT) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);  // a fragment's LDS reads
            __builtin_amdgcn_sched_group_barrier(0x002, EXACT ? 10 : 18, 0);  // vector work
          });
        }
        __builtin_amdgcn_sched_barrier(0);
      });
      lsum += pair_sum(rs[0] + rs[1]);
    }
  }
  block_barrier();  // every wave is done with the last tile: the ring becomes the output staging
  const float inv = a.nsplit > 1 ? 1.0f : lsum == 0.f ? 0.f : 1.0f / lsum;
  const int64_t n = (int64_t)a.B * a.Sq * a.Hq;
  if (half == 0 && valid) {
    if (a.nsplit > 1) a.part_ml[n * split + ((int64_t)b * a.Sq + i) * a.Hq + h] = make_float2(m, lsum);
    else a.lse[((int64_t)b * a.Hq + h) * a.Sq + i] = (weight_base(m) + log2f(lsum)) * 0.6931471805599453f;
  }
  float z = 0.f;  // stays 0 as long as every value is finite
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) z = __builtin_fmaf(o[dt][e], 0.f, z);
  float* stage = reinterpret_cast<float*>(smem);
  stage_rows_from_t<HD>(stage, o, 1.0f);
  // the rows leave scaled: the factor of row r is in lane r mod 32 of wave r / 32
  float* scales = stage + QB * (HD + 4);
  if (half == 0) scales[wave * 32 + col] = inv;
  __syncthreads();
  float* part = a.nsplit > 1 ? a.part + n * split * HD : nullptr;
  for (int c = threadIdx.x; c < QB * HD / 8; c += NT) {
    const int r = rb * QB + c / (HD / 8), d = (c % (HD / 8)) * 8;
    if (r >= rows.n) continue;
    const float* sr = stage + c / (HD / 8) * (HD + 4) + d;
    const float f = scales[c / (HD / 8)];
    const f32x4 lo = *reinterpret_cast<const f32x4*>(sr) * f, hi = *reinterpret_cast<const f32x4*>(sr + 4) * f;
    const int64_t at = (((int64_t)b * a.Sq + rows.query(r)) * a.Hq + rows.head(r)) * HD + d;
    float* f32 = part ? part : EXACT ? a.o32 : nullptr;
    if (f32) {
      *reinterpret_cast<f32x4*>(f32 + at) = lo;
      *reinterpret_cast<f32x4*>(f32 + at + 4) = hi;
    }
    if (!part) {
      bf16x8 ov;
#pragma unroll
      for (int q = 0; q < 4; ++q) { ov[q] = (bf16)lo[q]; ov[q + 4] = (bf16)hi[q]; }
      *reinterpret_cast<bf16x8*>((bf16*)a.o + at) = ov;
    }
  }
  uint64_t bad = __ballot(valid && !(z == 0.f));
  if (__syncthreads_or(bad != 0)) {  // behind every wave's stores of these rows
    bad = (bad | bad >> 32) & 0xffffffffu;
    while (bad) {
      const int c = __builtin_ctzll(bad);
      bad &= bad - 1;
      row_again<HD>(a, rows, r0 + c, weight_base(__shfl(m, c, 64)), __shfl(inv, c, 64),
                    max(__shfl(mask.x, c, 64), blo + t0 * KB), min(__shfl(mask.y, c, 64), blo + t1 * KB), part);
    }
  }
}

// ------------------------------------------------------------------------------------------ backward
// P and dS are rounded to bf16 for their products, as in the causal kernels: the gradients are 2.4e-3 of their norm off, of
// which their own rounding is 1.7e-3.  In two parts each they would take three products more to the seven there are, in
// kernels that the matrix cores and the vector work between them bound.
// The tanh of a tile's products ahead of a softmax of the backward.  Behind the polynomial its slope is 1 - t^2, an
// instruction of the softmax.  A t near 1 has lost it (at y = 8 it would be 6 % off, from y = 10 on 0), so in the other branch the
// slope comes from e = exp(-2 |y|), as 4 e / (1 + e)^2, and is put where the softmax finds it for nothing more:
//   dK/dV  into dp = (dp - delta) slope, of which the softmax subtracts keep delta = 0 and takes clamp(one - t^2) = 1
//   dQ     into the score: ds alone is wanted, so s becomes t + log(slope) / cap, and the softmax's slope is at least 1
// (a pair that is not seen has s = -inf or its ds replaced).
struct FarTanh {
  float t, a, e, r;  // tanh(y), log2(e), e, 1 / (1 + e)
  __device__ FarTanh(float x, const CapScale& c) {
    asm volatile("" : "+v"(x));  // apart from the other branch: what both compute would be kept for the whole tile ahead of them
    const float y = x * c.y_of;
    a = fabsf(y) * -2.8853900817779268f;
    e = fast_exp2(a);
    r = __builtin_amdgcn_rcpf(1.0f + e);
    const float far = copysignf(__builtin_fmaf(-2.0f * e, r, 1.0f), y);
    t = fabsf(y) < TANH_SMALL ? __builtin_fmaf(y, tanh_excess(y * y), y) : far;
  }
  __device__ float slope() const { return 4.0f * e * r * r; }
  __device__ float log2_slope() const { return __builtin_fmaf(2.0f, __builtin_amdgcn_logf(r), a + 2.0f); }
};
struct CapSlope {
  float keep = 1.f, one = 1.f;
  __device__ float operator()(float t) const { return __builtin_amdgcn_fmed3f(__builtin_fmaf(-t, t, one), 0.f, 1.f); }
  __device__ float less(float dp, float delta) const { return __builtin_fmaf(-keep, delta, dp); }
};
// delta: of the lane's accumulator rows, four at a time 8 apart
__device__ __forceinline__ CapSlope tanh_ahead(f32x16& s, f32x16& dp, const CapScale& c, const float* delta) {
  CapSlope r;
  if (__all(largest(reinterpret_cast<const f32x16(&)[1]>(s)) <= c.small)) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = tanh_small(s[e] * c.y_of);
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const FarTanh f(s[e], c);
      dp[e] = (dp[e] - delta[8 * (e / 4) + e % 4]) * f.slope();
      s[e] = f.t;  // last, as in the other branch: the compiler joins the branches' last stores, and a choice between s
    }              // and dp there would put both into scratch memory
    r.keep = 0.f;
    r.one = 2.f;
  }
  return r;
}
// gives the least slope
__device__ __forceinline__ float tanh_ahead_dq(f32x16 (&s)[2], const CapScale& c) {
  if (__all(largest(s) <= c.small)) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[t][e] = tanh_small(s[t][e] * c.y_of);
    return 0.f;
  }
  const float per = 1.0f / c.out;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const FarTanh f(s[t][e], c);
      s[t][e] = __builtin_fmaf(f.log2_slope(), per, f.t);
      __builtin_amdgcn_sched_barrier(0);
    }
  return 1.f;
}

// P of one pair, from s = q.k or with CAP its tanh
template <bool CAP, bool BIAS>
__device__ __forceinline__ float weight(float s, float nlse2, const CapScale& c, float slope2, float far) {
  float x = __builtin_fmaf(s, CAP ? c.out : c.sl2, nlse2);
  if constexpr (BIAS) x = __builtin_fmaf(-slope2, fabsf(far), x);
  return fast_exp2(x);
}
template <int N>
__device__ __forceinline__ bool all_finite(const f32x16 (&x)[N]) {
  float z = 0.f;  // stays 0 as long as every value is finite
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) z = __builtin_fmaf(x[t][e], 0.f, z);
  return z == 0.f;
}

// x rotated back by the angle of row `row` (as store_rows_from_t): lane l holds elements l, l + 64, ..
template <int HD>
__device__ __forceinline__ void unrotate(float (&x)[PER_LANE<HD>], const RangeArgs& a, int row) {
  constexpr int HH = HD / 2;
  const int lane = row_lane<HD>();
  if (!a.rope_cos) return;
  const int64_t t = (int64_t)row * HH + lane % HH;
  const float cs = a.rope_cos[t], sn = a.rope_sin[t];
  if constexpr (HD == 128) {
    const float u = x[0], v = x[1];
    x[0] = u * cs + v * sn;
    x[1] = v * cs - u * sn;
  } else {
    const float other = __shfl_xor(x[0], HH, 64);
    x[0] = lane < HH ? x[0] * cs + other * sn : x[0] * cs - other * sn;
  }
}

// dq of query i again, touching only the keys it sees in [k_lo, k_hi)
template <int HD>
__device__ __forceinline__ void dq_row_again(const RangeArgs& a, int split, int b, int h, int i, int k_lo, int k_hi) {
  const int lane = threadIdx.x % 64, el = row_lane<HD>(), kvh = h / (a.Hq / a.Hkv);
  int2 keys = seen_keys_kept(a, (int64_t)b * a.Sq + i);
  keys.x = max(keys.x, k_lo);
  keys.y = min(keys.y, k_hi);
  const bf16* q = rows_of<bf16>(a.q, b, h) + (int64_t)i * a.q.row;
  const bf16* d = rows_of<bf16>(a.dout, b, h) + (int64_t)i * a.dout.row;
  const bf16* k = rows_of<bf16>(a.k, b, kvh);
  const bf16* v = rows_of<bf16>(a.v, b, kvh);
  const CapScale c(a);
  const float slope2 = a.slopes ? a.slopes[h] * LOG2E : 0.f;
  const int64_t pos = position(a, b, i), sidx = ((int64_t)b * a.Hq + h) * a.Sq + i;
  const float nl = a.nlse[sidx], dl = a.delta[sidx];
  float acc[PER_LANE<HD>];
#pragma unroll
  for (int x = 0; x < PER_LANE<HD>; ++x) acc[x] = 0.f;
  for (int j0 = keys.x; j0 < keys.y && !all_nan(acc); j0 += 64) {
    const int n = min(64, keys.y - j0), j = j0 + min(lane, n - 1);
    float g;
    const float p = fast_exp2(score2(row_dot<HD>(q, k + (int64_t)j * a.k.row), a, c, slope2, (float)(pos - j), g) + nl);
    const float ds = p * (row_dot<HD>(d, v + (int64_t)j * a.v.row) - dl) * g;
    for (int t = 0; t < n; ++t) {
      const float w = __shfl(ds, t, 64);
#pragma unroll
      for (int x = 0; x < PER_LANE<HD>; ++x) acc[x] += w * (float)k[(int64_t)(j0 + t) * a.k.row + 64 * x + el];
    }
  }
  if (a.qsplit > 1) {
    float* part = dq_part<HD>(a, split, b, h) + (int64_t)i * a.Hq * HD;
#pragma unroll
    for (int x = 0; x < PER_LANE<HD>; ++x) part[64 * x + el] = acc[x];
    return;
  }
#pragma unroll
  for (int x = 0; x < PER_LANE<HD>; ++x) acc[x] *= a.scale;
  unrotate<HD>(acc, a, i);
  bf16* out = rows_out<bf16>(a.dq, b, h) + (int64_t)i * a.dq.row;
#pragma unroll
  for (int x = 0; x < PER_LANE<HD>; ++x) out[64 * x + el] = (bf16)acc[x];
}

// What a dK/dV item covers: keys of block kb, 64-query tiles of the queries [by.x, by.y) that see one of them, of
// every query head of the group: iterations [it0, nit) of tiles x group (its share of nsplit)
struct KeyItem {
  int kb, kvh, b, split, tiles, it0, nit, qlo, qhi;
  __device__ KeyItem(const RangeArgs& a, int kb_, int split_, int kvh_, int b_) : kb(kb_), kvh(kvh_), b(b_), split(split_) {
    const int2 by = a.sees[(int64_t)b * ((a.Sk + QB - 1) / QB) + kb];
    qlo = __builtin_amdgcn_readfirstlane(by.x);
    qhi = __builtin_amdgcn_readfirstlane(by.y);
    tiles = (qhi - qlo + KB - 1) / KB;
    const int64_t all = (int64_t)(a.Hq / a.Hkv) * tiles;
    it0 = __builtin_amdgcn_readfirstlane((int)(all * split / a.nsplit));
    nit = __builtin_amdgcn_readfirstlane((int)(all * (split + 1) / a.nsplit));
  }
};

// Where partial sums of split items lie: dk (0) or dv (1) of `split`, rows of Hkv HD
template <int HD>
__device__ __forceinline__ float* dkv_part(const RangeArgs& a, int split, int which, int b, int kvh) {
  return a.part + (((int64_t)split * 2 + which) * a.B + b) * a.Sk * a.Hkv * HD + kvh * HD;
}

// dk and dv of one key again over the item's iterations, touching only the queries that see it
template <int HD>
__device__ __forceinline__ void dkv_row_again(const RangeArgs& a, const KeyItem& it_, int key) {
  const int lane = threadIdx.x % 64, el = row_lane<HD>(), group = a.Hq / a.Hkv, b = it_.b;
  const bf16* k = rows_of<bf16>(a.k, b, it_.kvh) + (int64_t)key * a.k.row;
  const bf16* v = rows_of<bf16>(a.v, b, it_.kvh) + (int64_t)key * a.v.row;
  const CapScale c(a);
  float dk[PER_LANE<HD>], dv[PER_LANE<HD>];
#pragma unroll
  for (int x = 0; x < PER_LANE<HD>; ++x) dk[x] = dv[x] = 0.f;
  for (int it = it_.it0; it < it_.nit && !(all_nan(dk) && all_nan(dv)); ++it) {
    const int h = it_.kvh * group + it / it_.tiles, q0 = it_.qlo + it % it_.tiles * KB;
    const int i = min(q0 + lane, it_.qhi - 1);
    const bool on = q0 + lane < it_.qhi && sees(seen_keys_kept(a, (int64_t)b * a.Sq + i), key);
    const bf16* q = rows_of<bf16>(a.q, b, h);
    const bf16* d = rows_of<bf16>(a.dout, b, h);
    const int64_t sidx = ((int64_t)b * a.Hq + h) * a.Sq + i;
    const float slope2 = a.slopes ? a.slopes[h] * LOG2E : 0.f;
    float g;
    const float p = fast_exp2(score2(row_dot<HD>(q + (int64_t)i * a.q.row, k), a, c, slope2, (float)(position(a, b, i) - key), g) +
                              a.nlse[sidx]);
    const float ds = p * (row_dot<HD>(d + (int64_t)i * a.dout.row, v) - a.delta[sidx]) * g;
    for (uint64_t left = __ballot(on); left; left &= left - 1) {
      const int t = __builtin_ctzll(left);
      const float wp = __shfl(p, t, 64), wd = __shfl(ds, t, 64);
#pragma unroll
      for (int x = 0; x < PER_LANE<HD>; ++x) {
        dv[x] += wp * (float)d[(int64_t)(q0 + t) * a.dout.row + 64 * x + el];
        dk[x] += wd * (float)q[(int64_t)(q0 + t) * a.q.row + 64 * x + el];
      }
    }
  }
  if (a.nsplit > 1) {
    const int64_t row = (int64_t)key * a.Hkv * HD;
#pragma unroll
    for (int x = 0; x < PER_LANE<HD>; ++x) {
      dkv_part<HD>(a, it_.split, 0, b, it_.kvh)[row + 64 * x + el] = dk[x];
      dkv_part<HD>(a, it_.split, 1, b, it_.kvh)[row + 64 * x + el] = dv[x];
    }
    return;
  }
#pragma unroll
  for (int x = 0; x < PER_LANE<HD>; ++x) dk[x] *= a.scale;
  unrotate<HD>(dk, a, key);
#pragma unroll
  for (int x = 0; x < PER_LANE<HD>; ++x) {
    (rows_out<bf16>(a.dk, b, it_.kvh) + (int64_t)key * a.dk.row)[64 * x + el] = (bf16)dk[x];
    (rows_out<bf16>(a.dv, b, it_.kvh) + (int64_t)key * a.dv.row)[64 * x + el] = (bf16)dv[x];
  }
}

// The item's dk and dv leave, and the keys whose sums are not finite are computed again
template <int HD>
__device__ __forceinline__ void dkv_store(const RangeArgs& a, const KeyItem& item, const f32x16 (&dk)[HD / 32],
                                          const f32x16 (&dv)[HD / 32], float* stage) {
  const int wave = threadIdx.x / 64, key0 = item.kb * QB + wave * 32;
  uint64_t bad = __ballot(key0 + (int)(threadIdx.x % 32) < a.Sk && !(all_finite(dk) && all_finite(dv)));
  if (a.nsplit > 1) {
    store_partial_from_t<HD>(stage, dk, dkv_part<HD>(a, item.split, 0, item.b, item.kvh), a.Hkv * HD, item.kb * QB, a.Sk);
    store_partial_from_t<HD>(stage, dv, dkv_part<HD>(a, item.split, 1, item.b, item.kvh), a.Hkv * HD, item.kb * QB, a.Sk);
  } else {
    store_rows_from_t<HD>(stage, dk, a.scale, rows_out<bf16>(a.dk, item.b, item.kvh), a.dk.row, item.kb * QB, a.Sk,
                          a.rope_cos, a.rope_sin);
    store_rows_from_t<HD>(stage, dv, 1.0f, rows_out<bf16>(a.dv, item.b, item.kvh), a.dv.row, item.kb * QB, a.Sk);
  }
  if (__syncthreads_or(bad != 0)) {  // behind every wave's stores of these rows
    bad = (bad | bad >> 32) & 0xffffffffu;
    for (; bad; bad &= bad - 1) dkv_row_again<HD>(a, item, key0 + __builtin_ctzll(bad));
  }
}

// frag_rows and frag_cols of a given lane
template <int HD>
__device__ __forceinline__ bf16x8 frag_rows_of(const bf16* T, int r0, int k0, int l) {
  return *reinterpret_cast<const bf16x8*>(T + tidx<HD>(r0 + l % 32, k0 + 8 * (l / 32)));
}
template <int HD>
__device__ __forceinline__ bf16x8 frag_cols_of(const bf16* T, int c0, int k0, int l) {
  const int g = l / 16, i = l % 16, c = c0 + 16 * (g & 1) + 4 * (i & 3), k = k0 + 8 * (g >> 1) + (i >> 2);
  typedef __attribute__((address_space(3))) v4i16_t lds_v4i16;
  const v4i16_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(T + tidx<HD>(k, c)));
  const v4i16_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(T + tidx<HD>(k + 4, c)));
  bf16x8 f;
  __builtin_memcpy(&f, &lo, 8);
  __builtin_memcpy(reinterpret_cast<char*>(&f) + 8, &hi, 8);
  return f;
}

template <int HD, bool CAP, bool BIAS>
__device__ __forceinline__ void range_dq_block(const RangeArgs& a, int qb, int split, int h, int b,
                                               unsigned char* __restrict__ smem) {
  using L = Lds<HD>;
  using TT = DmaRowTile<HD>;
  constexpr int KS = HD / 16, DT = HD / 32, NS = L::NS;
  bf16* ring = reinterpret_cast<bf16*>(smem);  // [NS][K tile | V tile], swizzled
  const int kvh = h / (a.Hq / a.Hkv);
  const bf16* kbase = rows_of<bf16>(a.k, b, kvh);
  const bf16* vbase = rows_of<bf16>(a.v, b, kvh);
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, half = lane / 32, col = lane % 32;
  const int myq = qb * QB + wave * 32 + col, i = min(myq, a.Sq - 1);
  const bool valid = myq < a.Sq;
  const int64_t row0 = (int64_t)b * a.Sq;
  bf16x8 qf[KS], df[KS];
  {
    const bf16* q = rows_of<bf16>(a.q, b, h) + (int64_t)i * a.q.row + 8 * half;
    const bf16* d = rows_of<bf16>(a.dout, b, h) + (int64_t)i * a.dout.row + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[ks] = *reinterpret_cast<const bf16x8*>(q + ks * 16);
      df[ks] = *reinterpret_cast<const bf16x8*>(d + ks * 16);
    }
  }
  const int64_t sidx = ((int64_t)b * a.Hq + h) * a.Sq + i;
  const float nl = a.nlse[sidx], dl = a.delta[sidx];
  const int2 mask = seen_keys_kept(a, row0 + i);
  const WaveKeys wk(mask, valid);
  int blo, bhi;  // the block's keys
  {
    const int x = qb * QB + lane, y = x + 64;
    const int2 sx = x < a.Sq ? seen_keys_kept(a, row0 + x) : make_int2(0, 0);
    const int2 sy = y < a.Sq ? seen_keys_kept(a, row0 + y) : make_int2(0, 0);
    bhi = wave_max_i(max(sx.y, sy.y));
    blo = wave_min_i(min(sx.y > 0 ? sx.x : INT32_MAX, sy.y > 0 ? sy.x : INT32_MAX));
    if (bhi == 0) blo = 0;
  }
  const int tiles = (bhi - blo + KB - 1) / KB;  // of which this share takes [kt0, ntile)
  const int kt0 = __builtin_amdgcn_readfirstlane((int)((int64_t)tiles * split / a.qsplit));
  const int ntile = __builtin_amdgcn_readfirstlane((int)((int64_t)tiles * (split + 1) / a.qsplit));
  auto issue = [&](int t) {
    bf16* st = ring + (t % NS) * 2 * L::TSZ;
    TT::issue(kbase, a.k.row, blo + t * KB, bhi, lds_addr(st));
    TT::issue(vbase, a.v.row, blo + t * KB, bhi, lds_addr(st + L::TSZ));
  };
  const CapScale cs(a);
  float slope2 = 0.f;
  int64_t pos = 0;
  if constexpr (BIAS) {
    slope2 = a.slopes[h] * LOG2E;
    pos = position(a, b, i);
  }
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (kt0 + s < ntile) issue(kt0 + s);
  wait_vm_lds<0>();  // as in the forward
  f32x16 dq[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) dq[dt][e] = 0.f;
  for (int kt = kt0; kt < ntile; ++kt) {
    ring_wait<NS, 2 * TT::PER>(kt + 1 < ntile);
    block_barrier();
    if (kt + NS - 1 < ntile) issue(kt + NS - 1);
    const bf16* Ks = ring + (kt % NS) * 2 * L::TSZ;
    const bf16* Vs = Ks + L::TSZ;
    const int key0 = blo + kt * KB;
    if (key0 < wk.hi && key0 + KB > wk.lo) {
      // frag_rows and frag_cols; with CAP at 128 their addresses are formed here, tile by tile: kept across the loop they
      // push other registers out to memory (2 x 4096 tokens, 32 heads on 8: dQ 800 us, 512 so)
      int at = lane;
      if constexpr (CAP && HD == 128) asm volatile("" : "+v"(at));
      auto rows_at = [&](const bf16* T, int r, int k) { return frag_rows_of<HD>(T, r, k, at); };
      auto cols_at = [&](const bf16* T, int c, int k) { return frag_cols_of<HD>(T, c, k, at); };
      // as in attention_mfma.hip: S and dP of both 32-key sub-tiles, then the softmax and the dQ products of each
      f32x16 s[2], dp[2];
      if constexpr (HD == 128) {
        bf16x8 fk[2][2], fv[2][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          fk[0][t] = rows_at(Ks, t * 32, 0);
          fv[0][t] = rows_at(Vs, t * 32, 0);
        }
        static_for<KS>([&](auto KSI) {
          constexpr int ks = KSI, c = ks & 1;
          __builtin_amdgcn_sched_barrier(0);
          if constexpr (ks + 1 < KS) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              fk[c ^ 1][t] = rows_at(Ks, t * 32, (ks + 1) * 16);
              fv[c ^ 1][t] = rows_at(Vs, t * 32, (ks + 1) * 16);
            }
          }
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[c][t], qf[ks], ks ? s[t] : f32x16{}, 0, 0, 0);
            dp[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv[c][t], df[ks], ks ? dp[t] : f32x16{}, 0, 0, 0);
          }
          if constexpr (ks + 1 < KS) {
            static_for<4>([&](auto) {
              __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // one MFMA
              __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // one LDS read
            });
          }
          __builtin_amdgcn_sched_barrier(0);
        });
      } else {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows_at(Ks, t * 32, ks * 16), qf[ks], ks ? s[t] : f32x16{}, 0, 0, 0);
            dp[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows_at(Vs, t * 32, ks * 16), df[ks], ks ? dp[t] : f32x16{}, 0, 0, 0);
          }
      }
      float least = 0.f;
      if constexpr (CAP) least = tanh_ahead_dq(s, cs);
      const float base_far = BIAS ? (float)(pos - key0 - 4 * half) : 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        constexpr int NC = 2 * DT, RA = 3;
        bf16x8 fc[RA + 1];
        if constexpr (HD == 128) {
          static_for<RA>([&](auto QI) {
            constexpr int q = QI;
            fc[q] = cols_at(Ks, (q % DT) * 32, t * 32 + (q / DT) * 16);
          });
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float far = base_far - (float)(t * 32 + 8 * (e / 4) + e % 4);
          dp[t][e] = weight<CAP, BIAS>(s[t][e], nl, cs, slope2, far) * (dp[t][e] - dl);
          if constexpr (CAP) dp[t][e] *= __builtin_amdgcn_fmed3f(__builtin_fmaf(-s[t][e], s[t][e], 1.0f), least, 1.f);
        }
        if (!wk.whole(key0 + t * 32, key0 + t * 32 + 32)) {
          const uint32_t first = (uint32_t)(key0 + t * 32 + 4 * half - mask.x), len = (uint32_t)(mask.y - mask.x);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (first + (uint32_t)(8 * (e / 4) + e % 4) >= len) dp[t][e] = 0.f;
        }
        if constexpr (HD == 128) {
          const bf16x8 b0 = acc_rows_to_b<0>(dp[t]), b1 = acc_rows_to_b<8>(dp[t]);
          static_for<NC>([&](auto QI) {
            constexpr int q = QI, g2 = q / DT, dt = q % DT;
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (q + RA < NC)
              fc[(q + RA) % (RA + 1)] = cols_at(Ks, ((q + RA) % DT) * 32, t * 32 + ((q + RA) / DT) * 16);
            dq[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fc[q % (RA + 1)], g2 ? b1 : b0, dq[dt], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
          });
        } else {
#pragma unroll
          for (int g2 = 0; g2 < 2; ++g2) {
            const bf16x8 bop = g2 ? acc_rows_to_b<8>(dp[t]) : acc_rows_to_b<0>(dp[t]);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
              dq[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cols_at(Ks, dt * 32, t * 32 + g2 * 16), bop, dq[dt], 0, 0, 0);
          }
        }
      }
    }
  }
  block_barrier();  // every wave is done with the last tile: the ring becomes the output staging
  uint64_t bad = __ballot(valid && !all_finite(dq));
  float* stage = reinterpret_cast<float*>(smem);
  if (a.qsplit > 1) store_partial_from_t<HD>(stage, dq, dq_part<HD>(a, split, b, h), a.Hq * HD, qb * QB, a.Sq);
  else store_rows_from_t<HD>(stage, dq, a.scale, rows_out<bf16>(a.dq, b, h), a.dq.row, qb * QB, a.Sq, a.rope_cos, a.rope_sin);
  if (__syncthreads_or(bad != 0)) {
    bad = (bad | bad >> 32) & 0xffffffffu;
    for (; bad; bad &= bad - 1)
      dq_row_again<HD>(a, split, b, h, qb * QB + wave * 32 + __builtin_ctzll(bad), blo + kt0 * KB, blo + ntile * KB);
  }
}

// A stage of streamed query rows: Q and dO tiles, then nlse2, delta, seen_lo and seen_len of the rows
template <int HD>
struct QueryStage {
  static constexpr int TSZ = KB * HD, SZ = 2 * TSZ + 8 * KB;  // bf16 elements
  static constexpr size_t bytes(int stages) { return std::max((size_t)stages * SZ * 2, Lds<HD>::out_bytes); }
};

// Scores of the queries [r0, r0 + 32) of a stage that do not see this lane's key become -inf; nothing where all of
// them see all keys of the wave.  (A lane's keys are those of lanes 0 .. 31 of its wave, in order.)
template <int HD>
__device__ __forceinline__ void mask_unseen(f32x16& s, const bf16* stage, int r0, int mykey) {
  const uint32_t* lo = reinterpret_cast<const uint32_t*>(stage + 2 * QueryStage<HD>::TSZ) + 2 * KB + r0;
  const uint32_t* n = lo + KB;
  const int lane = threadIdx.x % 64, row = lane % 32, half = lane / 32;
  // lane l looks at row l mod 32, for the wave's first key or its last
  const uint32_t key = (uint32_t)(mykey - row) + 31u * half;
  if (__all(key - lo[row] < n[row])) return;
#pragma unroll
  for (int e4 = 0; e4 < 4; ++e4) {
    const u32x4 lo4 = *reinterpret_cast<const u32x4*>(lo + 8 * e4 + 4 * half), n4 = *reinterpret_cast<const u32x4*>(n + 8 * e4 + 4 * half);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if ((uint32_t)mykey - lo4[j] >= n4[j]) s[4 * e4 + j] = -INFINITY;
  }
}

// dK and dV of head dimensions 32 and 64
template <int HD, bool CAP, bool BIAS>
__device__ __forceinline__ void range_dkv_block(const RangeArgs& a, const KeyItem& item, unsigned char* __restrict__ smem) {
  using TT = DmaRowTile<HD>;
  using Q = QueryStage<HD>;
  constexpr int KS = HD / 16, DT = HD / 32, NS = ring_stages<HD>();
  bf16* ring = reinterpret_cast<bf16*>(smem);
  const int group = a.Hq / a.Hkv, b = item.b;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, half = lane / 32, col = lane % 32;
  const int k0 = item.kb * QB + wave * 32, mykey = k0 + col, kc = min(mykey, a.Sk - 1);
  const int wu = __builtin_amdgcn_readfirstlane(wave);
  // each wave loads one row vector per stage
  auto issue = [&](int it) {
    const int h = item.kvh * group + it / item.tiles, q0 = item.qlo + it % item.tiles * KB;
    bf16* st = ring + (it % NS) * Q::SZ;
    TT::issue(rows_of<bf16>(a.q, b, h), a.q.row, q0, item.qhi, lds_addr(st));
    TT::issue(rows_of<bf16>(a.dout, b, h), a.dout.row, q0, item.qhi, lds_addr(st + Q::TSZ));
    const void* v = wu == 0 ? (const void*)(a.nlse + ((int64_t)b * a.Hq + h) * a.Sq)
                  : wu == 1 ? (const void*)(a.delta + ((int64_t)b * a.Hq + h) * a.Sq)
                  : wu == 2 ? (const void*)(a.seen_lo + (int64_t)b * a.Sq) : (const void*)(a.seen_len + (int64_t)b * a.Sq);
    // rows past the last query repeat it (TT::issue), but see no key: their seen_len is 0
    const float* row = (const float*)v + q0;
    dma4_range(buffer_range(row, (const float*)v + item.qhi), 4u * (uint32_t)lane, lds_addr(st + 2 * Q::TSZ) + (uint32_t)wu * KB * 4u);
  };
  bf16x8 kf[KS], vf[KS];
  {
    const bf16* k = rows_of<bf16>(a.k, b, item.kvh) + (int64_t)kc * a.k.row + 8 * half;
    const bf16* v = rows_of<bf16>(a.v, b, item.kvh) + (int64_t)kc * a.v.row + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      kf[ks] = *reinterpret_cast<const bf16x8*>(k + ks * 16);
      vf[ks] = *reinterpret_cast<const bf16x8*>(v + ks * 16);
    }
  }
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (item.it0 + s < item.nit) issue(item.it0 + s);
  wait_vm_lds<0>();
  const CapScale cs(a);
  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) { dk[dt][e] = 0.f; dv[dt][e] = 0.f; }
  for (int it = item.it0; it < item.nit; ++it) {
    ring_wait<NS, 2 * TT::PER + 1>(it + 1 < item.nit);
    block_barrier();
    if (it + NS - 1 < item.nit) issue(it + NS - 1);
    const bf16* Qs = ring + (it % NS) * Q::SZ;
    const bf16* Ds = Qs + Q::TSZ;
    const float* Ls = reinterpret_cast<const float*>(Qs + 2 * Q::TSZ);
    const int q0 = item.qlo + it % item.tiles * KB;
    float slope2 = 0.f;
    int64_t far0 = 0;
    if constexpr (BIAS) {
      slope2 = a.slopes[item.kvh * group + it / item.tiles] * LOG2E;
      far0 = position(a, b, q0) - mykey + 4 * half;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x16 s, dp;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<HD>(Qs, t * 32, ks * 16), kf[ks], ks ? s : f32x16{}, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_rows<HD>(Ds, t * 32, ks * 16), vf[ks], ks ? dp : f32x16{}, 0, 0, 0);
      }
      const float* stats = Ls + t * 32 + 4 * half;  // nlse, and KB behind it delta, of the lane's rows 8 e4 + j
      CapSlope slope;
      if constexpr (CAP) slope = tanh_ahead(s, dp, cs, stats + KB);
      const float base_far = (float)far0;
      mask_unseen<HD>(s, Qs, t * 32, mykey);
#pragma unroll
      for (int e4 = 0; e4 < 4; ++e4) {
        const f32x4 l4 = *reinterpret_cast<const f32x4*>(stats + 8 * e4), d4 = *reinterpret_cast<const f32x4*>(stats + KB + 8 * e4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int e = 4 * e4 + j;
          const float p = weight<CAP, BIAS>(s[e], l4[j], cs, slope2, base_far + (float)(t * 32 + 8 * e4 + j));
          dp[e] = p * (CAP ? slope.less(dp[e], d4[j]) * slope(s[e]) : dp[e] - d4[j]);
          s[e] = p;
        }
      }
#pragma unroll
      for (int g2 = 0; g2 < 2; ++g2) {
        const bf16x8 pb = g2 ? acc_rows_to_b<8>(s) : acc_rows_to_b<0>(s);
        const bf16x8 sb = g2 ? acc_rows_to_b<8>(dp) : acc_rows_to_b<0>(dp);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          dv[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<HD>(Ds, dt * 32, t * 32 + g2 * 16), pb, dv[dt], 0, 0, 0);
          dk[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<HD>(Qs, dt * 32, t * 32 + g2 * 16), sb, dk[dt], 0, 0, 0);
        }
      }
    }
  }
  block_barrier();
  dkv_store<HD>(a, item, dk, dv, reinterpret_cast<float*>(smem));
}

// dK and dV of head dimension 128, pipelined over 32-query tiles as flash_bwd_dkv128
template <bool CAP, bool BIAS>
__device__ __forceinline__ void range_dkv128_block(const RangeArgs& a, const KeyItem& item, unsigned char* __restrict__ smem) {
  constexpr int HD = 128, KS = 8, DT = 4, NS = 3;
  using TT = DmaRowTile<HD>;
  using Q = QueryStage<HD>;
  bf16* ring = reinterpret_cast<bf16*>(smem);
  const int group = a.Hq / a.Hkv, b = item.b;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, half = lane / 32, col = lane % 32;
  const int mykey = item.kb * QB + wave * 32 + col, kc = min(mykey, a.Sk - 1);
  const int wu = __builtin_amdgcn_readfirstlane(wave);
  // The tile being loaded (head h, queries q0 .. of 64), its stage slot, and the ranges of its rows.  Rows past
  // the last query that sees a key arrive as zeros, and see none.
  struct Fetch {
    int h, q0, slot;
    u32x4 q, d, r;
    uint32_t lds;
  } f;
  auto ranges = [&] {
    const bf16 *qh = rows_of<bf16>(a.q, b, f.h), *dh = rows_of<bf16>(a.dout, b, f.h);
    f.q = buffer_range(qh + (int64_t)f.q0 * a.q.row, qh + (int64_t)(item.qhi - 1) * a.q.row + HD);
    f.d = buffer_range(dh + (int64_t)f.q0 * a.dout.row, dh + (int64_t)(item.qhi - 1) * a.dout.row + HD);
    const int64_t rows = wu < 2 ? ((int64_t)b * a.Hq + f.h) * a.Sq : (int64_t)b * a.Sq;
    const float* v = (wu == 0 ? a.nlse : wu == 1 ? a.delta : wu == 2 ? (const float*)a.seen_lo : (const float*)a.seen_len) + rows;
    f.r = buffer_range(v + f.q0, v + item.qhi);
    f.lds = lds_addr(ring + f.slot * Q::SZ) + (uint32_t)wu * 1024u;
  };
  auto next_tile = [&] {  // past the item's last tile it wraps: loaded again, into a stage nobody reads
    f.q0 += KB;
    if (f.q0 >= item.qhi) {
      f.q0 = item.qlo;
      f.h = f.h + 1 < (item.kvh + 1) * group ? f.h + 1 : item.kvh * group;
    }
    f.slot = f.slot + 1 < NS ? f.slot + 1 : 0;
    ranges();
  };
  // load k of the 2 PER + 1 of a stage
  auto fetch = [&](auto K_) {
    constexpr int k = K_;
    if constexpr (k < TT::PER) TT::issue_range(f.q, k, a.q.row, f.lds);
    else if constexpr (k < 2 * TT::PER) TT::issue_range(f.d, k - TT::PER, a.dout.row, f.lds + Q::TSZ * 2);
    else dma4_range(f.r, 4u * (uint32_t)lane, lds_addr(ring + f.slot * Q::SZ + 2 * Q::TSZ) + (uint32_t)wu * KB * 4u);
  };
  static_assert(2 * TT::PER + 1 <= 2 * KS, "a load per group of the two steps");
  bf16x8 kf[KS], vf[KS];
  {
    const bf16* k = rows_of<bf16>(a.k, b, item.kvh) + (int64_t)kc * a.k.row + 8 * half;
    const bf16* v = rows_of<bf16>(a.v, b, item.kvh) + (int64_t)kc * a.v.row + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      kf[ks] = *reinterpret_cast<const bf16x8*>(k + ks * 16);
      vf[ks] = *reinterpret_cast<const bf16x8*>(v + ks * 16);
    }
  }
  if (item.it0 < item.nit) {
    f.h = item.kvh * group + item.it0 / item.tiles;
    f.q0 = item.qlo + item.it0 % item.tiles * KB;
    f.slot = 0;
    ranges();
    static_for<2 * TT::PER + 1>(fetch);
  }
  wait_vm_lds<0>();
  const CapScale cs(a);
  const int64_t first = BIAS ? position(a, b, 0) - mykey + 4 * half : 0;
  f32x16 dk[DT], dv[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) { dk[dt][e] = 0.f; dv[dt][e] = 0.f; }
  f32x16 s[2], dp[2];         // S and dP of the two tiles of a stage; after the softmax P and dS
  bf16x8 pb[2][2], sb[2][2];  // P and dS as operands, two 16-query halves each

  // One step, as there: the loads of a stage (FE), S and dP of tile T of the stage at `rows` (SC), the softmax of
  // the other tile, whose first query is sq0 and head's slope slope2, with the row vectors at `stats` (SM; with CAP behind
  // tanh_ahead, which gave `cap`), and dV and dK of tile T of the stage at `cols` (PV).
  auto step = [&](auto T_, auto SC_, auto SM_, auto PV_, auto FE_, const bf16* rows, const bf16* stats, int sq0,
                  float slope2, const bf16* cols, const CapSlope& cap) {
    constexpr int T = T_, U = T ^ 1;
    constexpr bool SC = SC_, SM = SM_, PV = PV_, FE = FE_;
    const bf16 *Qr = rows, *Dr = rows + Q::TSZ, *Qc = cols, *Dc = cols + Q::TSZ;
    const float* Ls = reinterpret_cast<const float*>(stats + 2 * Q::TSZ) + U * 32 + 4 * half;
    const float base_far = BIAS && SM ? (float)(first + sq0) : 0.f;
    auto cfrag = [&](auto QI) {
      constexpr int q = QI;
      return frag_cols<HD>(q % 2 ? Qc : Dc, ((q / 2) % DT) * 32, T * 32 + (q / 8) * 16);
    };
    bf16x8 fq[2], fd[2], fc[4];
    f32x4 l4[2], d4[2];
    auto stat = [&](auto I) {
      constexpr int n = I;
      l4[n % 2] = *reinterpret_cast<const f32x4*>(Ls + 8 * n);
      d4[n % 2] = *reinterpret_cast<const f32x4*>(Ls + KB + 8 * n);
    };
    if constexpr (SM) stat(std::integral_constant<int, 0>{});
    if constexpr (SC) {
      fq[0] = frag_rows<HD>(Qr, T * 32, 0);
      fd[0] = frag_rows<HD>(Dr, T * 32, 0);
    }
    if constexpr (PV) {
      fc[0] = cfrag(std::integral_constant<int, 0>{});
      fc[1] = cfrag(std::integral_constant<int, 1>{});
    }
    static_for<KS>([&](auto G) {
      constexpr int g = G, c = g & 1;
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (FE && T * KS + g < 2 * TT::PER + 1) fetch(std::integral_constant<int, T * KS + g>{});
      if constexpr (SC && g + 1 < KS) {
        fq[c ^ 1] = frag_rows<HD>(Qr, T * 32, (g + 1) * 16);
        fd[c ^ 1] = frag_rows<HD>(Dr, T * 32, (g + 1) * 16);
      }
      if constexpr (PV && g + 1 < KS) {
        fc[2 * (c ^ 1)] = cfrag(std::integral_constant<int, (2 * g + 2) % 16>{});
        fc[2 * (c ^ 1) + 1] = cfrag(std::integral_constant<int, (2 * g + 3) % 16>{});
      }
      if constexpr (SM && g % 2 == 1 && g + 1 < KS) stat(std::integral_constant<int, (g + 1) / 2>{});
      // four MFMAs, each followed by a quarter of the vector work
      constexpr int e0 = 2 * g, e1 = e0 + 1, lb = g / 2 % 2;
      float x0, x1, y0, y1;
      if constexpr (SC) s[T] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[c], kf[g], g ? s[T] : f32x16{}, 0, 0, 0);
      if constexpr (SM) {
        x0 = __builtin_fmaf(s[U][e0], CAP ? cs.out : cs.sl2, l4[lb][e0 % 4]);
        x1 = __builtin_fmaf(s[U][e1], CAP ? cs.out : cs.sl2, l4[lb][e1 % 4]);
        if constexpr (BIAS) {
          x0 = __builtin_fmaf(-slope2, fabsf(base_far + (float)(8 * (e0 / 4) + e0 % 4)), x0);
          x1 = __builtin_fmaf(-slope2, fabsf(base_far + (float)(8 * (e1 / 4) + e1 % 4)), x1);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (PV) mfma_acc<!SC>(dv[g % DT], fc[2 * c], pb[T][g / DT]);
      if constexpr (SM) {
        x0 = fast_exp2(x0);
        x1 = fast_exp2(x1);
        pin(x0, x1);
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (SC) dp[T] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fd[c], vf[g], g ? dp[T] : f32x16{}, 0, 0, 0);
      if constexpr (SM) {
        if constexpr (CAP) {
          y0 = cap.less(dp[U][e0], d4[lb][e0 % 4]) * cap(s[U][e0]);
          y1 = cap.less(dp[U][e1], d4[lb][e1 % 4]) * cap(s[U][e1]);
        } else {
          y0 = dp[U][e0] - d4[lb][e0 % 4];
          y1 = dp[U][e1] - d4[lb][e1 % 4];
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (PV) mfma_acc<!SC>(dk[g % DT], fc[2 * c + 1], sb[T][g / DT]);
      if constexpr (SM) {
        s[U][e0] = x0;
        s[U][e1] = x1;
        dp[U][e0] = x0 * y0;
        dp[U][e1] = x1 * y1;
        if constexpr (g == 3) { pb[U][0] = acc_rows_to_b<0>(s[U]); sb[U][0] = acc_rows_to_b<0>(dp[U]); }
        if constexpr (g == 7) { pb[U][1] = acc_rows_to_b<8>(s[U]); sb[U][1] = acc_rows_to_b<8>(dp[U]); }
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  constexpr std::integral_constant<int, 0> t0{};
  constexpr std::integral_constant<int, 1> t1{};
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  auto soft = [&](auto T_, auto SC_, auto PV_, auto FE_, const bf16* rows, const bf16* stats, int sq0, float slope2, const bf16* cols) {
    constexpr int U = T_ ^ 1;
    CapSlope cap;
    if constexpr (CAP) {
      cap = tanh_ahead(s[U], dp[U], cs, reinterpret_cast<const float*>(stats + 2 * Q::TSZ) + KB + U * 32 + 4 * half);
    }
    mask_unseen<HD>(s[U], stats, U * 32, mykey);
    step(T_, SC_, std::true_type{}, PV_, FE_, rows, stats, sq0, slope2, cols, cap);
  };
  auto arrive = [&] {
    wait_vm_lds<0>();
    block_barrier();  // every thread's loads of the stage are in; every wave is done with the last iteration
  };
  auto slope_of = [&](int h) { return BIAS ? a.slopes[h] * LOG2E : 0.f; };
  if (item.it0 < item.nit) {
    const bf16 *cur = ring, *prev;
    int qc = f.q0, qp;  // first queries of the stages cur and prev, and the slopes of their heads
    float mc = slope_of(f.h), mp;
    auto turn = [&] {   // the stage just loaded becomes cur
      prev = cur;
      qp = qc;
      mp = mc;
      cur = ring + f.slot * Q::SZ;
      qc = f.q0;
      mc = slope_of(f.h);
    };
    arrive();
    next_tile();
    step(t0, yes, no, no, yes, cur, cur, 0, 0.f, cur, CapSlope{});
    soft(t1, yes, no, yes, cur, cur, qc, mc, cur);
    for (int it = item.it0 + 1; it < item.nit; ++it) {
      turn();
      arrive();
      next_tile();  // into the stage before prev
      soft(t0, yes, yes, yes, cur, prev, qp + 32, mp, prev);
      soft(t1, yes, yes, yes, cur, cur, qc, mc, prev);
      acc_settled(dk, dv);  // register copies the compiler may place at the loop's end
    }
    acc_settled(dk, dv);
    soft(t0, no, yes, no, cur, cur, qc + 32, mc, cur);
    step(t1, no, no, yes, no, cur, cur, 0, 0.f, cur, CapSlope{});
    acc_settled(dk, dv);
    wait_vm_lds<0>();  // the last, unread loads: the ring becomes the output staging
  }
  block_barrier();
  dkv_store<HD>(a, item, dk, dv, reinterpret_cast<float*>(smem));
}

// The key block of sequence b whose queries are the r-th most (of up to NT blocks; beyond that block r itself: there are
// then enough items for their order not to matter).  Documents give the blocks of a launch very different lengths, and
// the longest, started last, would end it: 2 x 4096 tokens in 3 documents a row, 32 heads on 8, capped: 418 -> 371 us.
__device__ __forceinline__ int heavy_block(const RangeArgs& a, int b, int nkb, int r) {
  __shared__ int queries[NT], pick;
  if (nkb > NT) return r;
  const int t = threadIdx.x;
  if (t < nkb) {
    const int2 by = a.sees[(int64_t)b * nkb + t];
    queries[t] = by.y - by.x;
  }
  __syncthreads();
  if (t < nkb) {
    int rank = 0;
    for (int j = 0; j < nkb; ++j) rank += queries[j] > queries[t] || (queries[j] == queries[t] && j < t);
    if (rank == r) pick = t;
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(pick);
}

template <bool CAP, bool BIAS>
__global__ void __launch_bounds__(NT, 2) range_flash_dq128(RangeArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int nqb = (a.Sq + QB - 1) / QB;
  int unit, idx;  // unit: (sequence, query head)
  xcd_item(blockIdx.x, nqb * a.qsplit * a.Hq * a.B, nqb * a.qsplit, unit, idx);
  range_dq_block<128, CAP, BIAS>(a, nqb - 1 - idx / a.qsplit, idx % a.qsplit, unit % a.Hq, unit / a.Hq, smem);
}

template <bool CAP, bool BIAS>
__global__ void __launch_bounds__(NT) range_flash_dkv128(RangeArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int nkb = (a.Sk + QB - 1) / QB;
  int unit, idx;  // unit: (sequence, key/value head)
  xcd_item(blockIdx.x, nkb * a.nsplit * a.Hkv * a.B, nkb * a.nsplit, unit, idx);
  const int b = unit / a.Hkv;
  const KeyItem item(a, heavy_block(a, b, nkb, idx / a.nsplit), idx % a.nsplit, unit % a.Hkv, b);
  range_dkv128_block<CAP, BIAS>(a, item, smem);
}

// dQ and dK/dV items of head dimensions 32 and 64 in one launch: a unit is one (sequence, key/value head)
template <int HD, bool CAP, bool BIAS>
__global__ void __launch_bounds__(NT, 2) range_flash_bwd(RangeArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int nkb = (a.Sk + QB - 1) / QB, nqb = (a.Sq + QB - 1) / QB, group = a.Hq / a.Hkv;
  const int per_unit = nkb * a.nsplit + nqb * a.qsplit * group;
  int unit, idx;
  xcd_item(blockIdx.x, per_unit * a.Hkv * a.B, per_unit, unit, idx);
  const int kvh = unit % a.Hkv, b = unit / a.Hkv;
  if (idx < nkb * a.nsplit) {
    const KeyItem item(a, heavy_block(a, b, nkb, idx / a.nsplit), idx % a.nsplit, kvh, b);
    range_dkv_block<HD, CAP, BIAS>(a, item, smem);
  } else {
    idx -= nkb * a.nsplit;
    const int split = idx % a.qsplit;
    idx /= a.qsplit;
    range_dq_block<HD, CAP, BIAS>(a, nqb - 1 - idx / group, split, kvh * group + idx % group, b, smem);
  }
}

template <int HD>
constexpr size_t range_fwd_lds() {
  const size_t out = (size_t)QB * (HD + 4) * 4 + QB * 4;
  return std::max(Lds<HD>::NS * Lds<HD>::kv_stage, out);
}

// Allows kernel K its dynamic LDS, once per device
template <auto K>
void allow_lds(size_t bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  (void)hipGetDevice(&dev);
  const uint64_t bit = (uint64_t)1 << (dev % 64);
  if (done.load() & bit) return;
  (void)hipFuncSetAttribute((const void*)K, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  done |= bit;
}

template <int HD, bool EXACT, bool CAP, bool BIAS>
void fwd_launch(const RangeArgs& a, int pack, unsigned blocks, hipStream_t st) {
  allow_lds<range_flash_fwd<HD, EXACT, CAP, BIAS>>(range_fwd_lds<HD>());
  range_flash_fwd<HD, EXACT, CAP, BIAS><<<blocks, NT, range_fwd_lds<HD>(), st>>>(a, pack);
}

// f(std::bool_constant<x>, std::bool_constant<y>, std::bool_constant<z>)
template <typename F>
void with_flags(bool x, bool y, bool z, F&& f) {
  auto third = [&](auto X, auto Y) { if (z) f(X, Y, std::true_type{}); else f(X, Y, std::false_type{}); };
  auto second = [&](auto X) { if (y) third(X, std::true_type{}); else third(X, std::false_type{}); };
  if (x) second(std::true_type{}); else second(std::false_type{});
}

}  // namespace

// The query heads of a key/value head share a block's rows where that makes fewer blocks (few queries)
int range_mfma_pack(const RangeArgs& a) {
  const int group = a.Hq / a.Hkv;
  return cdiv((int64_t)a.Sq * group, QB) < group * cdiv(a.Sq, QB) ? group : 1;
}

int64_t range_mfma_items(const RangeArgs& a) {
  const int pack = range_mfma_pack(a);
  return cdiv((int64_t)a.Sq * pack, QB) * (a.Hq / pack) * a.B;
}

void range_mfma_fwd(const RangeArgs& a, hipStream_t st) {
  const unsigned blocks = (unsigned)(range_mfma_items(a) * a.nsplit);
  const int pack = range_mfma_pack(a);
  with_flags(a.o32 != nullptr, a.cap > 0.f, a.slopes != nullptr, [&](auto exact, auto cap, auto bias) {
    if (a.hd == 32) fwd_launch<32, exact.value, cap.value, bias.value>(a, pack, blocks, st);
    else if (a.hd == 64) fwd_launch<64, exact.value, cap.value, bias.value>(a, pack, blocks, st);
    else fwd_launch<128, exact.value, cap.value, bias.value>(a, pack, blocks, st);
  });
}

int range_mfma_keys() { return QB; }

// A share of at least so many tiles: with few items the chip is empty and a chain of tiles is all there is to wait for
// (one sequence of 300 tokens, 4 heads of 128 on 1: backward 50 us with 8, 40 with 3)
static int64_t tiles_per_share(int64_t items) { return items <= 64 ? 3 : 8; }

// As attention_dkv_splits: few key blocks are split over their queries' tiles, the longest by the causal count
int range_mfma_dkv_splits(const RangeArgs& a) {
  const int64_t items = cdiv(a.Sk, QB) * a.Hkv * a.B, tiles = (int64_t)(a.Hq / a.Hkv) * cdiv(a.Sq, KB);
  if (items == 0) return 1;
  const int64_t most = a.hd != 128 || tiles >= 140 || (tiles >= 48 && 256 % items == 0) ? 512 : 256;
  return (int)std::max<int64_t>(1, std::min<int64_t>({8, cdiv(most, items), tiles / tiles_per_share(items)}));
}

// Few query blocks share their keys' tiles, towards 512 items: a block of a long row alone is a chain of its tiles
// (captured: one sequence of 4096 tokens, one head of 64: backward 89 -> 46 us; 16 queries on 8192 keys, 8 heads of 128 on
// 1: 214 -> 59)
int range_mfma_dq_splits(const RangeArgs& a) {
  const int64_t items = cdiv(a.Sq, QB) * a.Hq * a.B;
  return items == 0 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({16, 512 / items, cdiv(a.Sk, KB) / tiles_per_share(items)}));
}

void range_mfma_bwd(const RangeArgs& a, hipStream_t st) {
  const int64_t nkb = cdiv(a.Sk, QB) * a.nsplit * a.Hkv * a.B, nqb = cdiv(a.Sq, QB) * a.qsplit * a.Hq * a.B;
  with_flags(a.cap > 0.f, a.slopes != nullptr, false, [&](auto cap, auto bias, auto) {
    constexpr bool CAP = decltype(cap)::value, BIAS = decltype(bias)::value;
    auto together = [&](auto hd) {
      constexpr int HD = decltype(hd)::value;
      constexpr size_t lds = std::max(Lds<HD>::dq_bytes(), QueryStage<HD>::bytes(ring_stages<HD>()));
      allow_lds<range_flash_bwd<HD, CAP, BIAS>>(lds);
      range_flash_bwd<HD, CAP, BIAS><<<(unsigned)(nkb + nqb), NT, lds, st>>>(a);
    };
    if (a.hd == 32) {
      together(std::integral_constant<int, 32>{});
    } else if (a.hd == 64) {
      together(std::integral_constant<int, 64>{});
    } else {
      constexpr size_t lds_kv = QueryStage<128>::bytes(3), lds_q = Lds<128>::dq_bytes();
      allow_lds<range_flash_dq128<CAP, BIAS>>(lds_q);
      allow_lds<range_flash_dkv128<CAP, BIAS>>(lds_kv);
      if (nqb) range_flash_dq128<CAP, BIAS><<<(unsigned)nqb, NT, lds_q, st>>>(a);
      if (nkb) range_flash_dkv128<CAP, BIAS><<<(unsigned)nkb, NT, lds_kv, st>>>(a);
    }
  });
}
