// Grouped-query attention over a range of keys per query, its scores capped by a tanh and lowered by the
// distance between query and key, forward and backward; and the key ranges of packed documents.
//
//   x_ij = scale q_i.k_j;  s_ij = cap tanh(x_ij / cap) - slope_h |pos_i - j|;  query i sees keys [lo_i, hi_i)
//   P_ij = exp(s_ij - lse_i), lse_i = log sum_j exp(s_ij) over the keys it sees;  o = P v
//   delta_i = dO_i.o_i;  dP = dO v^T;  dS = P (dP - delta) (1 - tanh^2);  dq = scale dS k
//   dk = scale dS^T q and dv = P^T dO, summed over the query heads of a key/value head
// A query that sees no key has o = 0, lse = -inf and no gradient.
//
// These kernels take fp32, on the fp32 matrix cores, tiled as in attention.hip (bf16: attention_ranges_mfma.hip):
// a block owns 32 rows of one side, its waves take every fourth tile of 32 rows of the other.  Tiles start at
// the first key (query) that a row of the block sees and end with the last; a tile that every row sees whole
// skips the mask.  What bounds them is the chain of one wave's tiles: loads, two products of 2 x 16 .. 64 MFMAs of 64 cycles
// and the softmax between them (3 x 777 tokens in 4 documents, 12 heads of 64 on 4: 36 us, of which the matrix cores
// need some 10), so few blocks are split into shares that a second kernel joins.
#include "attention_ranges.h"
#include "attention_rows.h"
#include <algorithm>

// attention_ranges_mfma.hip: bf16
int64_t range_mfma_items(const RangeArgs& a);
void range_mfma_fwd(const RangeArgs& a, hipStream_t st);
int range_mfma_keys();  // keys of a dK/dV block
int range_mfma_dkv_splits(const RangeArgs& a);
int range_mfma_dq_splits(const RangeArgs& a);
void range_mfma_bwd(const RangeArgs& a, hipStream_t st);

namespace {

constexpr int MAX_SPLITS = 256;  // shares of an item's keys

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// Score of x = scale q.k at distance `far` (x itself without cap and slopes)
struct Score {
  float cap, inv_cap, slope;
  bool has_cap, biased;
  __device__ Score(const RangeArgs& a, int h) {
    cap = a.cap;
    has_cap = a.cap > 0.f;
    inv_cap = has_cap ? 1.0f / a.cap : 0.f;
    biased = a.slopes != nullptr;
    slope = biased ? a.slopes[h] : 0.f;
  }
  __device__ float operator()(float x, float far, float& grad) const {
    grad = 1.f;
    if (has_cap) x = capped(x, cap, inv_cap, grad);
    if (biased) x = __builtin_fmaf(-slope, fabsf(far), x);
    return x;
  }
};

// rows_product as sums of 32 elements that are then added: 128 products in one chain leave a score twice as far off,
// and a weight is its exponential (84 tokens, 16 heads of 128, scores of 10: gradients 1.2e-6 off their norm against
// 9.4e-7).
template <int HD>
__device__ __forceinline__ f32x16 rows_product_parts(const RowFrag<HD>& a, const RowFrag<HD>& b) {
  f32x16 total;
#pragma unroll
  for (int n = 0; n < HD / 32; ++n) {
    f32x16 s;
    float zero = 0.f;
    if (n) asm volatile("" : "+v"(zero) : "v"(total[0]));  // one sum after the other: side by side they would spill
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = zero;
#pragma unroll
    for (int q = 4 * n; q < 4 * n + 4; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = mfma2(a.v[q][j], b.v[q][j], s);
    total = n ? total + s : s;
  }
  return total;
}

// The same for dP, of which nothing is an exponential: in parts at 128 only (their registers spill: 1425 tokens, 32
// heads of 128 on 8: backward 989 -> 1149 us captured, gradients 1.0e-6 off against 9.3e-7), one chain of 64 at most otherwise
template <int HD>
__device__ __forceinline__ f32x16 grad_product(const RowFrag<HD>& a, const RowFrag<HD>& b) {
  if constexpr (HD == 128) return rows_product_parts<HD>(a, b);
  else return rows_product<HD>(a, b);
}

__device__ __forceinline__ int acc_row(int e) { return 8 * (e / 4) + 4 * (threadIdx.x % 64 / 32) + e % 4; }

// One block per (32 queries, query head, sequence, share of their keys)
template <typename T, int HD>
__global__ void __launch_bounds__(NW * 64, HD == 128 ? 1 : HD == 64 ? 2 : 3) range_fwd(RangeArgs a) {
  __shared__ float red[NW * WAVE_LDS<HD>];
  const int nt = (a.Sq + TR - 1) / TR;
  int64_t id = blockIdx.x;
  const int split = id % a.nsplit;
  id /= a.nsplit;
  const int q0 = (nt - 1 - (int)(id % nt)) * TR;
  id /= nt;
  const int h = id % a.Hq, b = (int)(id / a.Hq), kvh = h / (a.Hq / a.Hkv);
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, q = q0 + lane % 32, qc = min(q, a.Sq - 1);
  float* mine = red + wave * WAVE_LDS<HD>;
  const T* kp = rows_of<T>(a.k, b, kvh);
  const T* vp = rows_of<T>(a.v, b, kvh);
  const int2 mask = seen_keys(a, b, qc);
  const WaveKeys wk(mask, q < a.Sq);
  const int64_t pos = position(a, b, qc);
  const Score score(a, h);
  // this share's keys: tiles of 32 from the first key seen on
  const int tiles = wk.hi > wk.lo ? (wk.hi - wk.lo + TR - 1) / TR : 0;
  const int t0 = (int)((int64_t)tiles * split / a.nsplit), t1 = (int)((int64_t)tiles * (split + 1) / a.nsplit);
  RowFrag<HD> qf;
  qf.load(rows_of<T>(a.q, b, h), qc, a.q.row);
#pragma unroll
  for (int i = 0; i < HD / 8; ++i) qf.v[i] *= a.scale;
  f32x16 o[HD / 32];
#pragma unroll
  for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
  float m = -INFINITY, l = 0.f;
  auto tile = [&](int k0, auto edge) {
    RowFrag<HD> kf;
    kf.load(kp, min(k0 + lane % 32, wk.hi - 1), a.k.row);
    ColFrag<HD> vf;  // on its way while the scores are formed
    vf.load(vp, k0, wk.hi - 1, a.v.row);
    f32x16 s = rows_product_parts<HD>(kf, qf);  // rows: keys; column: this lane's query
    const float base_far = (float)(pos - k0);
    float mt = -INFINITY, g;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = score(s[e], base_far - (float)acc_row(e), g);
      if (edge && !sees(mask, k0 + acc_row(e))) s[e] = -INFINITY;
      mt = fmaxf(mt, s[e]);
    }
    const float mn = fmaxf(m, pair_max(mt));
    const float base = weight_base(mn);
    const float corr = expf(m - base);
    float rs = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = expf(s[e] - base);
      rs += s[e];
    }
    l = l * corr + pair_sum(rs);
    m = mn;
#pragma unroll
    for (int dt = 0; dt < HD / 32; ++dt) o[dt] *= corr;
    if constexpr (edge) {
      kf.load(vp, min(k0 + lane % 32, wk.hi - 1), a.v.row);
      if (!kf.finite()) {  // 0 times what a query does not see could be a NaN
        cols_product_seen<HD>(o, vp, k0, a.v.row, s, mine, [&](int r) { return sees(mask, k0 + r); });
        return;
      }
    }
    vf.product(o, s);
  };
  for (int t = t0 + wave; t < t1; t += NW) {
    const int k0 = wk.lo + t * TR;
    if (wk.whole(k0, k0 + TR)) tile(k0, std::false_type{});
    else tile(k0, std::true_type{});
  }
  if (lane < TR) {
    mine[lane] = m;
    mine[TR + lane] = l;
  }
  __syncthreads();
  float M = -INFINITY, L = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) M = fmaxf(M, red[w * WAVE_LDS<HD> + lane % 32]);
  const float base = weight_base(M);
#pragma unroll
  for (int w = 0; w < NW; ++w)
    L += expf(red[w * WAVE_LDS<HD> + lane % 32] - base) * red[w * WAVE_LDS<HD> + TR + lane % 32];
  __syncthreads();
  const float wt = expf(m - base);
  put_partial<HD>(red, o, a.nsplit > 1 ? wt : L == 0.f ? 0.f : wt / L);
  __syncthreads();
  const int64_t row0 = ((int64_t)b * a.Sq * a.Hq + h);  // row of query i: row0 + i Hq
  if (a.nsplit > 1) {
    const int64_t n = (int64_t)a.B * a.Sq * a.Hq;
    store_rows<HD>(red, 1.0f, a.part + (n * split + row0) * HD, a.Hq * HD, q0, a.Sq, nullptr, nullptr);
    if (wave == 0 && lane < TR && q < a.Sq) a.part_ml[n * split + row0 + (int64_t)q * a.Hq] = make_float2(M, L);
    return;
  }
  store_rows<HD>(red, 1.0f, (T*)a.o + row0 * HD, a.Hq * HD, q0, a.Sq, nullptr, nullptr,
                 a.o32 ? a.o32 + row0 * HD : nullptr);
  if (wave == 0 && lane < TR && q < a.Sq) a.lse[((int64_t)b * a.Hq + h) * a.Sq + q] = base + logf(L);
}

// One row's sum of the shares s = s0, s0 + step, .. of the elements c .. c + 3, their weights given by weight(s)
template <int HD, typename F>
__device__ __forceinline__ f32x4 add_shares(const RangeArgs& a, int64_t r, int c, int s0, int step, F&& weight) {
  const int64_t n = (int64_t)a.B * a.Sq * a.Hq;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = s0; s < a.nsplit; s += step) o += weight(s) * ld4(a.part + (n * s + r) * HD + c);
  return o;
}
template <typename T, int HD>
__device__ __forceinline__ void store_joined(const RangeArgs& a, int64_t r, int c, f32x4 o, float base, float L) {
  o *= L == 0.f ? 0.f : 1.0f / L;
  st4((T*)a.o + r * HD + c, o);
  if (a.o32) st4(a.o32 + r * HD + c, o);
  if (c == 0) {
    const int64_t row = r / a.Hq, b = row / a.Sq;
    a.lse[(b * a.Hq + r % a.Hq) * a.Sq + row % a.Sq] = a.log2 ? (base + log2f(L)) * 0.6931471805599453f : base + logf(L);
  }
}
__device__ __forceinline__ float share_weight(const RangeArgs& a, float m, float base) {
  return a.log2 ? exp2f(m - base) : expf(m - base);
}

// The shares of a row (b, i, h) joined, a block per row: HD / 4 lanes per share, the shares spread over the block, so
// that a row of many shares takes a few round trips to memory and not one per share (16 rows of 16 shares: 5.6 ->
// 3.4 us).
template <typename T, int HD>
__global__ void __launch_bounds__(256) range_join(RangeArgs a) {
  constexpr int LR = HD / 4, NG = 256 / LR;  // lanes of a share, shares at a time
  __shared__ f32x4 sum[256];
  __shared__ float weight[MAX_SPLITS], top[4], tot[4];
  const int64_t n = (int64_t)a.B * a.Sq * a.Hq, r = blockIdx.x;
  const int t = threadIdx.x, c = (t % LR) * 4;
  float2 ml = make_float2(-INFINITY, 0.f);
  if (t < a.nsplit) ml = a.part_ml[n * t + r];
  const float m = wave_max(ml.x);
  if (t % 64 == 0) top[t / 64] = m;
  __syncthreads();
  const float base = weight_base(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
  const float w = share_weight(a, ml.x, base);
  weight[t] = w;
  const float l = wave_sum(w * ml.y);
  if (t % 64 == 0) tot[t / 64] = l;
  __syncthreads();
  f32x4 o = add_shares<HD>(a, r, c, t / LR, NG, [&](int s) { return weight[s]; });
  sum[t] = o;
  __syncthreads();
  if (t >= LR) return;
  const float L = (tot[0] + tot[1]) + (tot[2] + tot[3]);
#pragma unroll
  for (int g = 1; g < NG; ++g) o += sum[g * LR + t];
  store_joined<T, HD>(a, r, c, o, base, L);
}

// The same with a row's shares one after another, HD / 4 lanes per row, for many rows of few shares
constexpr int FEW_SPLITS = 8;
template <typename T, int HD>
__global__ void __launch_bounds__(256) range_join_few(RangeArgs a) {
  constexpr int LR = HD / 4;
  const int64_t n = (int64_t)a.B * a.Sq * a.Hq, r = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LR;
  const int c = (threadIdx.x % LR) * 4;
  if (r >= n) return;
  float2 ml[FEW_SPLITS];
  float M = -INFINITY, L = 0.f;
#pragma unroll
  for (int s = 0; s < FEW_SPLITS; ++s) {
    ml[s] = s < a.nsplit ? a.part_ml[n * s + r] : make_float2(-INFINITY, 0.f);
    M = fmaxf(M, ml[s].x);
  }
  const float base = weight_base(M);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < FEW_SPLITS; ++s) {
    if (s >= a.nsplit) break;
    const float w = share_weight(a, ml[s].x, base);
    L += w * ml[s].y;
    o += w * ld4(a.part + (n * s + r) * HD + c);
  }
  store_joined<T, HD>(a, r, c, o, base, L);
}

// [x, y): the first and last query that see a key of tile t of `width` keys
__device__ __forceinline__ void plan_tile(const RangeArgs& a, int width, int ntile, int t, int b) {
  __shared__ int first[4], last[4];
  const int k0 = t * width, k1 = min(k0 + width, a.Sk);
  int lo = INT32_MAX, hi = 0;
  for (int i = threadIdx.x; i < a.Sq; i += 256) {
    const int2 s = seen_keys(a, b, i);
    if (max(s.x, k0) < min(s.y, k1)) {
      lo = min(lo, i);
      hi = i + 1;
    }
  }
  lo = wave_min_i(lo);
  hi = wave_max_i(hi);
  if (threadIdx.x % 64 == 0) {
    first[threadIdx.x / 64] = lo;
    last[threadIdx.x / 64] = hi;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 4; ++w) {
      lo = min(lo, first[w]);
      hi = max(hi, last[w]);
    }
    a.sees[(int64_t)b * ntile + t] = lo < hi ? make_int2(lo, hi) : make_int2(0, 0);
  }
}

// What the backward needs first, in one launch: a block per (tile of `width` keys, sequence) for the queries that see
// it; then delta_i = dO_i.o_i and the other statistics per (sequence, head, query), HD / 4 lanes per row.
template <typename T, int HD>
__global__ void __launch_bounds__(256) range_prep(RangeArgs a, int width, int ntile) {
  constexpr int LR = HD / 4;
  const int nplan = ntile * a.B;
  if ((int)blockIdx.x < nplan) {
    plan_tile(a, width, ntile, blockIdx.x % ntile, blockIdx.x / ntile);
    return;
  }
  const int64_t r = ((int64_t)(blockIdx.x - nplan) * 256 + threadIdx.x) / LR;  // (b, i, h)
  const int c = (threadIdx.x % LR) * 4;
  const bool in = r < (int64_t)a.B * a.Sq * a.Hq;
  const int64_t row = r / a.Hq;
  const int h = (int)(r % a.Hq), b = (int)(row / a.Sq), i = (int)(row % a.Sq);
  float s = 0.f;
  if (in) {
    const f32x4 d = ld4(rows_of<T>(a.dout, b, h) + (int64_t)i * a.dout.row + c);
    const int64_t at = b * a.ob + i * a.orow + h * a.oh + c;
    const f32x4 o = a.o32 ? ld4(a.o32 + at) : ld4((const T*)a.o + at);
    s = (o[0] * d[0] + o[1] * d[1]) + (o[2] * d[2] + o[3] * d[3]);
  }
#pragma unroll
  for (int k = 1; k < LR; k <<= 1) s += __shfl_xor(s, k, WAVE);
  if (!in || c) return;
  a.delta[((int64_t)b * a.Hq + h) * a.Sq + i] = s;
  const float lse = weight_base(a.lse[((int64_t)b * a.Hq + h) * a.Sq + i]);
  a.nlse[((int64_t)b * a.Hq + h) * a.Sq + i] = a.log2 ? -1.4426950408889634f * lse : -lse;
  if (h == 0) {
    const int2 k = seen_keys(a, b, i);
    a.seen_lo[row] = k.x;
    a.seen_len[row] = k.y - k.x;
  }
}

// dq of 32 queries of head h: the share `split` of their keys' tiles
template <typename T, int HD>
__device__ __forceinline__ void range_dq(const RangeArgs& a, int qb, int split, int h, int b, float* red) {
  const int kvh = h / (a.Hq / a.Hkv), q0 = qb * TR;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, q = q0 + lane % 32, qc = min(q, a.Sq - 1);
  const T* kp = rows_of<T>(a.k, b, kvh);
  const T* vp = rows_of<T>(a.v, b, kvh);
  const int2 mask = seen_keys_kept(a, (int64_t)b * a.Sq + qc);
  const WaveKeys wk(mask, q < a.Sq);
  const int64_t pos = position(a, b, qc);
  const Score score(a, h);
  RowFrag<HD> qf, df;
  qf.load(rows_of<T>(a.q, b, h), qc, a.q.row);
  df.load(rows_of<T>(a.dout, b, h), qc, a.dout.row);
#pragma unroll
  for (int i = 0; i < HD / 8; ++i) qf.v[i] *= a.scale;
  const int64_t sidx = ((int64_t)b * a.Hq + h) * a.Sq + qc;
  const float nl = a.nlse[sidx], dl = a.delta[sidx];
  f32x16 dq[HD / 32];
#pragma unroll
  for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) dq[dt][e] = 0.f;
  auto tile = [&](int k0, auto edge) {
    const int kr = min(k0 + lane % 32, wk.hi - 1);
    RowFrag<HD> f;
    f.load(kp, kr, a.k.row);
    const bool plain = !edge || f.finite();
    f32x16 s = rows_product_parts<HD>(f, qf);
    f.load(vp, kr, a.v.row);
    const f32x16 dp = grad_product<HD>(f, df);
    const float base_far = (float)(pos - k0);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float g;
      const float x = score(s[e], base_far - (float)acc_row(e), g);
      s[e] = !edge || sees(mask, k0 + acc_row(e)) ? expf(x + nl) * (dp[e] - dl) * g : 0.f;
    }
    if (plain) cols_product<HD>(dq, kp, k0, wk.hi - 1, a.k.row, s);
    else cols_product_seen<HD>(dq, kp, k0, a.k.row, s, red + wave * WAVE_LDS<HD>, [&](int r) { return sees(mask, k0 + r); });
  };
  const int tiles = (wk.hi - wk.lo + TR - 1) / TR;
  const int t1 = (int)((int64_t)tiles * (split + 1) / a.qsplit);
  for (int t = (int)((int64_t)tiles * split / a.qsplit) + wave; t < t1; t += NW) {
    const int k0 = wk.lo + t * TR;
    if (wk.whole(k0, k0 + TR)) tile(k0, std::false_type{});
    else tile(k0, std::true_type{});
  }
  put_partial<HD>(red, dq, 1.0f);
  __syncthreads();
  if (a.qsplit > 1) store_rows<HD>(red, 1.0f, dq_part<HD>(a, split, b, h), a.Hq * HD, q0, a.Sq, nullptr, nullptr);
  else store_rows<HD>(red, a.scale, rows_out<T>(a.dq, b, h), a.dq.row, q0, a.Sq, a.rope_cos, a.rope_sin);
}

// dk and dv of 32 keys of key/value head kvh, summed over its query heads: the share `split` of the tiles of the
// queries that see one of them
template <typename T, int HD>
__device__ __forceinline__ void range_dkv(const RangeArgs& a, int kb, int split, int kvh, int b, float* red) {
  const int k0 = kb * TR, group = a.Hq / a.Hkv;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, half = lane / 32, key = k0 + lane % 32, kc = min(key, a.Sk - 1);
  RowFrag<HD> kf, vf;
  kf.load(rows_of<T>(a.k, b, kvh), kc, a.k.row);
  vf.load(rows_of<T>(a.v, b, kvh), kc, a.v.row);
#pragma unroll
  for (int i = 0; i < HD / 8; ++i) kf.v[i] *= a.scale;
  f32x16 dk[HD / 32], dv[HD / 32];
#pragma unroll
  for (int dt = 0; dt < HD / 32; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) { dk[dt][e] = 0.f; dv[dt][e] = 0.f; }
  const int2 by = a.sees[(int64_t)b * ((a.Sk + TR - 1) / TR) + kb];
  const int nt = (by.y - by.x + TR - 1) / TR;
  const int64_t row0 = (int64_t)b * a.Sq, all = (int64_t)group * nt;
  const int64_t it1 = all * (split + 1) / a.nsplit;
  for (int64_t it = all * split / a.nsplit + wave; it < it1; it += NW) {
    const int h = kvh * group + (int)(it / nt), q0 = by.x + (int)(it % nt) * TR, ql = by.y - 1;
    const T* qp = rows_of<T>(a.q, b, h);
    const T* dp_ = rows_of<T>(a.dout, b, h);
    const int64_t sb = ((int64_t)b * a.Hq + h) * a.Sq + q0;
    const int qr = min(q0 + lane % 32, ql);
    const Score score(a, h);
    RowFrag<HD> f;
    f.load(qp, qr, a.q.row);
    const int2 mine = seen_keys_kept(a, row0 + qr);
    // every key of the block is seen by every query of the tile
    const bool whole = q0 + TR <= by.y && __all(mine.x <= k0 && k0 + TR <= mine.y);
    const bool plain_q = whole || f.finite();
    f32x16 p = rows_product_parts<HD>(f, kf);  // rows: queries; column: this lane's key
    f.load(dp_, qr, a.dout.row);
    const bool plain_d = whole || f.finite();
    f32x16 ds = grad_product<HD>(f, vf);
    // the rows' statistics, four consecutive rows at a time (the arrays end with TR elements of room)
    f32x4 nl[4], dl[4];
    i32x4 lo[4], len[4];
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const int r = 8 * e4 + 4 * half;
      __builtin_memcpy(&nl[e4], a.nlse + sb + r, 16);
      __builtin_memcpy(&dl[e4], a.delta + sb + r, 16);
      __builtin_memcpy(&lo[e4], a.seen_lo + row0 + q0 + r, 16);
      __builtin_memcpy(&len[e4], a.seen_len + row0 + q0 + r, 16);
    }
    const float base_far = (float)(position(a, b, q0) - key);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const bool on = q0 + acc_row(e) <= ql && (uint32_t)(key - lo[e / 4][e % 4]) < (uint32_t)len[e / 4][e % 4];
      float g;
      const float x = score(p[e], base_far + (float)acc_row(e), g);
      p[e] = on ? expf(x + nl[e / 4][e % 4]) : 0.f;
      ds[e] = on ? p[e] * (ds[e] - dl[e / 4][e % 4]) * g : 0.f;
    }
    auto on = [&](int r) { return q0 + r <= ql && sees(seen_keys_kept(a, row0 + min(q0 + r, ql)), key); };
    float* tmp = red + wave * WAVE_LDS<HD>;
    if (plain_d) cols_product<HD>(dv, dp_, q0, ql, a.dout.row, p);
    else cols_product_seen<HD>(dv, dp_, q0, a.dout.row, p, tmp, on);
    if (plain_q) cols_product<HD>(dk, qp, q0, ql, a.q.row, ds);
    else cols_product_seen<HD>(dk, qp, q0, a.q.row, ds, tmp, on);
  }
  const bool parts = a.nsplit > 1;
  const int kvd = a.Hkv * HD;
  float* part = a.part + ((int64_t)split * 2 * a.B + b) * a.Sk * kvd + kvh * HD;
  put_partial<HD>(red, dk, 1.0f);
  __syncthreads();
  if (parts) store_rows<HD>(red, 1.0f, part, kvd, k0, a.Sk, nullptr, nullptr);
  else store_rows<HD>(red, a.scale, rows_out<T>(a.dk, b, kvh), a.dk.row, k0, a.Sk, a.rope_cos, a.rope_sin);
  __syncthreads();
  put_partial<HD>(red, dv, 1.0f);
  __syncthreads();
  if (parts) store_rows<HD>(red, 1.0f, part + (int64_t)a.B * a.Sk * kvd, kvd, k0, a.Sk, nullptr, nullptr);
  else store_rows<HD>(red, 1.0f, rows_out<T>(a.dv, b, kvh), a.dv.row, k0, a.Sk, nullptr, nullptr);
}

// dk/dv blocks and dq blocks in one launch
template <typename T, int HD>
__global__ void __launch_bounds__(NW * 64, bwd_waves(HD)) range_bwd(RangeArgs a) {
  __shared__ float red[NW * WAVE_LDS<HD>];
  const int nk = (a.Sk + TR - 1) / TR, nq = (a.Sq + TR - 1) / TR;
  const int64_t nkv = (int64_t)nk * a.nsplit * a.Hkv * a.B;
  int64_t id = blockIdx.x;
  if (id < nkv) {
    const int split = id % a.nsplit;
    id /= a.nsplit;
    const int kb = id % nk;
    id /= nk;
    range_dkv<T, HD>(a, kb, split, (int)(id % a.Hkv), (int)(id / a.Hkv), red);
  } else {
    id -= nkv;
    const int split = id % a.qsplit;
    id /= a.qsplit;
    const int qb = nq - 1 - (int)(id % nq);
    id /= nq;
    range_dq<T, HD>(a, qb, split, (int)(id % a.Hq), (int)(id / a.Hq), red);
  }
}

// Gradients of split items: the partial sums of rows [B, rows, heads, HD] added in order
struct JoinRows {
  const float* part;
  int64_t share, n;  // elements between shares, and of one
  int nsplit, rows, heads;
  HeadRows out;
  float scale;
  bool rope;
};
template <typename T, int HD>
__device__ __forceinline__ void join_rows(const RangeArgs& a, const JoinRows& j, int64_t e) {  // elements e .. e + 7
  constexpr int HH = HD / 2;
  const int64_t row = e / (j.heads * HD);
  const int h = (int)(e / HD % j.heads), d = (int)(e % HD), b = (int)(row / j.rows), i = (int)(row % j.rows);
  auto sum = [&](int64_t o, float* v) {
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = 0.f;
    for (int s = 0; s < j.nsplit; ++s) {
      const float* p = j.part + j.share * s + o;
      const f32x4 lo = ld4(p), hi = ld4(p + 4);
#pragma unroll
      for (int q = 0; q < 4; ++q) { v[q] += lo[q]; v[q + 4] += hi[q]; }
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] *= j.scale;
  };
  float v[8];
  sum(e, v);
  if (j.rope && a.rope_cos) {
    const bool first = d < HH;
    float p[8];
    sum(first ? e + HH : e - HH, p);
    const int64_t t = (int64_t)i * HH + d % HH;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float cs = a.rope_cos[t + q], sn = a.rope_sin[t + q];
      v[q] = first ? v[q] * cs + p[q] * sn : v[q] * cs - p[q] * sn;
    }
  }
  T* o = rows_out<T>(j.out, b, h) + (int64_t)i * j.out.row + d;
  st4(o, f32x4{v[0], v[1], v[2], v[3]});
  st4(o + 4, f32x4{v[4], v[5], v[6], v[7]});
}
template <typename T, int HD>
__global__ void __launch_bounds__(256) range_grad_join(RangeArgs a) {
  const int64_t nk = a.nsplit > 1 ? (int64_t)a.B * a.Sk * a.Hkv * HD : 0;
  const int64_t nq = a.qsplit > 1 ? (int64_t)a.B * a.Sq * a.Hq * HD : 0;
  const int64_t e = 8 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
  if (e < nk) join_rows<T, HD>(a, JoinRows{a.part, 2 * nk, nk, a.nsplit, a.Sk, a.Hkv, a.dk, a.scale, true}, e);
  else if (e < 2 * nk) join_rows<T, HD>(a, JoinRows{a.part + nk, 2 * nk, nk, a.nsplit, a.Sk, a.Hkv, a.dv, 1.0f, false}, e - nk);
  else if (e < 2 * nk + nq) join_rows<T, HD>(a, JoinRows{a.part_q, nq, nq, a.qsplit, a.Sq, a.Hq, a.dq, a.scale, true}, e - 2 * nk);
}

// ------------------------------------------------------------------------------------------ key ranges
// A block takes RT tokens of a row, PT consecutive ones per thread.  The last position at or before a token
// where a document starts, and where a token is no prefix token, are running maxima over the row; the next
// position where a prefix ends is a running minimum from its end.  What lies outside the block's tokens is
// searched for, outwards from them and no further than the document goes.  The block's tokens and the RT on either side
// are loaded together, since the time is that of the round trips to memory (4 rows of 131072 tokens, 200 documents each:
// 11.8 us of kernel time with one after the other, 7.2 so).  A document over many blocks is walked by each of them, RT tokens
// a round trip: the work grows with the square of its length (one document a row, 4 x 131072 tokens: 55 us, 84 with prefixes; one
// of 2^22: 2.7 ms).
constexpr int RT = 2048, RTH = 256, PT = RT / RTH;

// PT tokens of a row from i0 on (those below `end` exist) and the id before them
struct Tokens {
  int id[PT], before, i0, n;
  uint8_t flag[PT];
  __device__ __forceinline__ void load(const int32_t* ids, const uint8_t* flags, int i0_, int end) {
    i0 = i0_;
    n = max(0, min(PT, end - i0));
    before = n > 0 && i0 > 0 ? ids[i0 - 1] : 0;
#pragma unroll
    for (int j = 0; j < PT; ++j) {
      id[j] = 0;
      flag[j] = 0;
    }
    if (n == PT) {
      __builtin_memcpy(id, ids + i0, sizeof(id));
      if (flags) __builtin_memcpy(flag, flags + i0, sizeof(flag));
    } else {
#pragma unroll
      for (int j = 0; j < PT; ++j)
        if (j < n) {
          id[j] = ids[i0 + j];
          if (flags) flag[j] = flags[i0 + j];
        }
    }
  }
  __device__ __forceinline__ bool begins(int j) const { return j < n && (i0 + j == 0 || id[j] != (j ? id[j - 1] : before)); }
  __device__ __forceinline__ bool plain(int j) const { return j < n && !flag[j]; }
  __device__ __forceinline__ int last_begin() const {
    int r = -1;
#pragma unroll
    for (int j = 0; j < PT; ++j)
      if (begins(j)) r = i0 + j;
    return r;
  }
  __device__ __forceinline__ int last_plain() const {
    int r = -1;
#pragma unroll
    for (int j = 0; j < PT; ++j)
      if (plain(j)) r = i0 + j;
    return r;
  }
  __device__ __forceinline__ int first_stop() const {  // where a prefix from before them ends
    int r = INT32_MAX;
#pragma unroll
    for (int j = PT - 1; j >= 0; --j)
      if (begins(j) || plain(j)) r = i0 + j;
    return r;
  }
};

// the value of the threads before this one (maximum) or after it (minimum) combined: exclusive scans over the block
__device__ __forceinline__ int scan_before(int v, int none, int* lds) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o, WAVE);
    if (lane >= o) v = max(v, u);
  }
  if (lane == 63) lds[wave] = v;
  int r = __shfl_up(v, 1, WAVE);
  if (lane == 0) r = none;
  __syncthreads();
  for (int w = 0; w < wave; ++w) r = max(r, lds[w]);
  __syncthreads();
  return r;
}
__device__ __forceinline__ int scan_after(int v, int none, int* lds) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_down(v, o, WAVE);
    if (lane + o < 64) v = min(v, u);
  }
  if (lane == 0) lds[wave] = v;
  int r = __shfl_down(v, 1, WAVE);
  if (lane == 63) r = none;
  __syncthreads();
  for (int w = wave + 1; w < RTH / 64; ++w) r = min(r, lds[w]);
  __syncthreads();
  return r;
}
// the block's maxima of three values
__device__ __forceinline__ void block_max3(int (&v)[3], int (*lds)[3]) {
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    v[k] = wave_max_i(v[k]);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64][k] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int w = 0; w < RTH / 64; ++w) v[k] = max(v[k], lds[w][k]);
  __syncthreads();
}

__global__ void __launch_bounds__(RTH) key_ranges(int S, int nb, const int32_t* __restrict__ ids,
                                                  const uint8_t* __restrict__ flags, int32_t* __restrict__ start,
                                                  int32_t* __restrict__ end) {
  __shared__ int lds[RTH / 64], lds3[RTH / 64][3];
  const int64_t row = blockIdx.x / nb;
  const int c0 = (int)(blockIdx.x % nb) * RT, c1 = min(c0 + RT, S), at = (int)threadIdx.x * PT;
  ids += row * S;
  if (flags) flags += row * S;
  start += row * S;
  end += row * S;
  Tokens mine, prev, next;
  mine.load(ids, flags, c0 + at, c1);
  const bool continues = c0 > 0 && ids[c0] == ids[c0 - 1];  // the first token's document starts before it
  if (c0 > 0) prev.load(ids, flags, c0 - RT + at, c0);
  if (flags && c1 < S) next.load(ids, flags, c1 + at, min(c1 + RT, S));
  // the document of the first token: its start, and whether a token of it before c0 is no prefix token; and
  // where a prefix that runs over the block's end stops
  int doc = c0, plain = -1, stop = S;
  int found[3] = {-1, -1, -INT32_MAX};
  if (continues) {
    found[0] = prev.last_begin();
    if (flags) found[1] = prev.last_plain();
  }
  if (flags && c1 < S) found[2] = -next.first_stop();
  block_max3(found, lds3);
  bool back = continues && found[0] < 0, ahead = flags && c1 < S && found[2] == -INT32_MAX;
  if (continues) {
    doc = max(0, found[0]);
    plain = found[1];
  }
  if (flags && c1 < S && !ahead) stop = -found[2];
  for (int hi = c0 - RT, lo = c1 + RT; back || ahead; hi -= RT, lo += RT) {  // a document over several blocks
    found[0] = found[1] = -1;
    found[2] = -INT32_MAX;
    back = back && hi > 0;
    ahead = ahead && lo < S;
    if (back) {
      prev.load(ids, flags, hi - RT + at, hi);
      found[0] = prev.last_begin();
      if (flags) found[1] = prev.last_plain();
    }
    if (ahead) {
      next.load(ids, flags, lo + at, min(lo + RT, S));
      found[2] = -next.first_stop();
    }
    block_max3(found, lds3);
    if (back) {
      doc = max(0, found[0]);
      plain = max(plain, found[1]);
      back = found[0] < 0;
    }
    if (ahead && found[2] != -INT32_MAX) {
      stop = -found[2];
      ahead = false;
    }
  }
  int cur = max(doc, scan_before(mine.last_begin(), -1, lds)), lastp = -1;
  int stops[PT];
  if (flags) {
    lastp = max(plain, scan_before(mine.last_plain(), -1, lds));
    int nx = min(stop, scan_after(mine.first_stop(), INT32_MAX, lds));
#pragma unroll
    for (int j = PT - 1; j >= 0; --j) {
      stops[j] = nx;
      if (mine.begins(j) || mine.plain(j)) nx = mine.i0 + j;
    }
  }
  int first[PT], last[PT];
#pragma unroll
  for (int j = 0; j < PT; ++j) {
    const int i = mine.i0 + j;
    if (mine.begins(j)) cur = i;
    if (flags && mine.plain(j)) lastp = i;
    const bool live = mine.id[j] >= 0;
    first[j] = live ? cur : 0;
    last[j] = live ? (flags && lastp < cur ? stops[j] : i + 1) : 0;
  }
  if (mine.n == PT) {
    __builtin_memcpy(start + mine.i0, first, sizeof(first));
    __builtin_memcpy(end + mine.i0, last, sizeof(last));
  } else {
#pragma unroll
    for (int j = 0; j < PT; ++j)
      if (j < mine.n) {
        start[mine.i0 + j] = first[j];
        end[mine.i0 + j] = last[j];
      }
  }
}

template <typename T, typename F>
void dispatch_hd(int hd, F&& run) {
  if (hd == 32) run(T{}, std::integral_constant<int, 32>{});
  else if (hd == 64) run(T{}, std::integral_constant<int, 64>{});
  else run(T{}, std::integral_constant<int, 128>{});
}
template <typename F>
void dispatch(bool bf, int hd, F&& run) {
  if (bf) dispatch_hd<bf16>(hd, run);
  else dispatch_hd<float>(hd, run);
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Shares of a forward item's keys.  Few items: towards 512, two per compute unit, of at least 256 keys, or of one tile
// of 64 on the bf16 matrix cores where each sequence has a few queries, which then wait for little else.  A few
// queries of many long caches: towards 4096 shares of at least 1024 keys, since the caches' lengths differ and the longest
// share ends the launch (16 answers of up to 32768 keys, 128 items: 247 us towards 512, 233 towards 2048, 228 towards 4096);
// with more queries the partial sums would cost more than that.
int fwd_splits(bool bf, const RangeArgs& a) {
  const int64_t items = bf ? range_mfma_items(a) : cdiv(a.Sq, TR) * a.Hq * a.B;
  if (items == 0) return 1;
  const bool short_q = a.Sq <= TR;
  const int64_t few = std::min<int64_t>(512 / items, a.Sk / (bf && short_q ? 64 : 256));
  const int64_t many = short_q ? std::min<int64_t>(4096 / items, a.Sk / 1024) : 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>(MAX_SPLITS, std::max(few, many)));
}

}  // namespace

size_t range_fwd_ws_bytes(bool bf, const RangeArgs& a) {
  const int64_t ns = fwd_splits(bf, a), n = (int64_t)a.B * a.Sq * a.Hq;
  return ns > 1 ? up256(ns * n * a.hd * 4) + up256(ns * n * 8) : 0;
}

int64_t range_fwd_blocks(bool bf, const RangeArgs& a) {
  const int64_t ns = fwd_splits(bf, a), n = (int64_t)a.B * a.Sq * a.Hq;
  const int64_t items = bf ? range_mfma_items(a) : cdiv(a.Sq, TR) * a.Hq * a.B;
  return std::max(items * ns, ns > FEW_SPLITS ? n : ns > 1 ? cdiv(n * (a.hd / 4), 256) : 0);
}

void launch_range_fwd(bool bf, RangeArgs a, void* ws, hipStream_t st) {
  const int64_t n = (int64_t)a.B * a.Sq * a.Hq;
  a.nsplit = fwd_splits(bf, a);
  a.log2 = bf;
  if (a.nsplit > 1) {
    a.part = (float*)ws;
    a.part_ml = (float2*)((char*)ws + up256(a.nsplit * n * a.hd * 4));
  }
  dispatch(bf, a.hd, [&](auto t, auto hd) {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value;
    if constexpr (sizeof(T) == 2) range_mfma_fwd(a, st);
    else range_fwd<T, HD><<<(unsigned)(cdiv(a.Sq, TR) * a.Hq * a.B * a.nsplit), NW * 64, 0, st>>>(a);
    if (a.nsplit > FEW_SPLITS) range_join<T, HD><<<(unsigned)n, 256, 0, st>>>(a);
    else if (a.nsplit > 1) range_join_few<T, HD><<<(unsigned)cdiv(n * (HD / 4), 256), 256, 0, st>>>(a);
  });
}

namespace {

// Shares of a dk/dv block's query tiles: a block of few walks them one after another, a wave an iteration of some 8 us
// of latency.  Towards 512 blocks, keeping two iterations to a wave of the longest (2 x 333 tokens, 8 heads of 32 on 2: 52 ->
// 27 us, and 4.4 for the join).
int dkv_splits(const RangeArgs& a) {
  const int64_t items = cdiv(a.Sk, TR) * a.Hkv * a.B, tiles = (int64_t)(a.Hq / a.Hkv) * cdiv(a.Sq, TR);
  return items == 0 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({8, 512 / items, tiles / (2 * NW)}));
}

// and of a dq block's key tiles
int dq_splits(const RangeArgs& a) {
  const int64_t items = cdiv(a.Sq, TR) * a.Hq * a.B, tiles = cdiv(a.Sk, TR);
  return items == 0 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({16, 512 / items, tiles / (2 * NW)}));
}

// The backward's workspace at p (null: its size alone)
size_t bwd_layout(bool bf, RangeArgs& a, char* p) {
  size_t n = 0;
  auto take = [&](int64_t bytes) {
    char* r = p + n;
    n += up256(bytes);
    return r;
  };
  const int64_t rows = (int64_t)a.B * a.Sq;
  a.log2 = bf;
  a.delta = (float*)take((rows * a.Hq + TR) * 4);
  a.nlse = (float*)take((rows * a.Hq + TR) * 4);
  a.seen_lo = (int32_t*)take((rows + TR) * 4);
  a.seen_len = (int32_t*)take((rows + TR) * 4);
  a.sees = (int2*)take(a.B * cdiv(a.Sk, bf ? range_mfma_keys() : TR) * 8);
  a.nsplit = bf ? range_mfma_dkv_splits(a) : dkv_splits(a);
  a.part = a.nsplit > 1 ? (float*)take(2 * (int64_t)a.nsplit * a.B * a.Sk * a.Hkv * a.hd * 4) : nullptr;
  a.qsplit = bf ? range_mfma_dq_splits(a) : dq_splits(a);
  a.part_q = a.qsplit > 1 ? (float*)take(a.qsplit * rows * a.Hq * a.hd * 4) : nullptr;
  return n;
}

}  // namespace

size_t range_bwd_ws_bytes(bool bf, const RangeArgs& a) {
  RangeArgs t = a;
  return bwd_layout(bf, t, nullptr);
}

namespace {

// The blocks of a backward whose arguments bwd_layout has completed
struct BwdBlocks {
  int64_t prep, grads, join;
  explicit BwdBlocks(const RangeArgs& a) {
    const int rows = a.log2 ? range_mfma_keys() : TR;
    const int64_t q = (int64_t)a.B * a.Sq * a.Hq, k = (int64_t)a.B * a.Sk * a.Hkv;
    prep = cdiv(a.Sk, rows) * a.B + cdiv(q * (a.hd / 4), 256);
    grads = cdiv(a.Sk, rows) * a.nsplit * a.Hkv * a.B + cdiv(a.Sq, rows) * a.qsplit * a.Hq * a.B;
    join = cdiv(((a.nsplit > 1 ? 2 * k : 0) + (a.qsplit > 1 ? q : 0)) * a.hd / 8, 256);
  }
};

}  // namespace

int64_t range_bwd_blocks(bool bf, const RangeArgs& a) {
  RangeArgs t = a;
  bwd_layout(bf, t, nullptr);
  const BwdBlocks n(t);
  return std::max({n.prep, n.grads, n.join});
}

void launch_range_bwd(bool bf, RangeArgs a, void* ws, hipStream_t st) {
  bwd_layout(bf, a, (char*)ws);
  const int width = a.log2 ? range_mfma_keys() : TR, ntile = (int)cdiv(a.Sk, width);
  const BwdBlocks n(a);
  dispatch(bf, a.hd, [&](auto t, auto hd) {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value;
    range_prep<T, HD><<<(unsigned)n.prep, 256, 0, st>>>(a, width, ntile);
    if constexpr (sizeof(T) == 2) range_mfma_bwd(a, st);
    else range_bwd<T, HD><<<(unsigned)n.grads, NW * 64, 0, st>>>(a);
    if (n.join > 0) range_grad_join<T, HD><<<(unsigned)n.join, 256, 0, st>>>(a);
  });
}

void launch_key_ranges(int64_t B, int S, const int32_t* ids, const uint8_t* flags, int32_t* start, int32_t* end,
                       hipStream_t st) {
  const int nb = (int)cdiv(S, RT);
  const int64_t most = MAX_BLOCKS_256 / nb;  // rows of a launch
  for (int64_t b = 0; b < B; b += most) {
    const int64_t o = b * S;
    key_ranges<<<(unsigned)(std::min(most, B - b) * nb), RTH, 0, st>>>(S, nb, ids + o, flags ? flags + o : nullptr, start + o, end + o);
  }
}
