// Losses on the log-probabilities of answers, with their gradients: the clipped policy loss with a KL term
// and an entropy bonus, and the preference loss of paired log ratios.
//
// Arrays are [sequences, len] row-major; a token counts where its mask byte is not 0, and nothing is
// read of the others (their values may be anything).  Sums run in double in a fixed order.
#include "common.h"
#include "kernels.h"
#include <algorithm>

namespace {

// 4 consecutive tokens at any alignment
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint8_t u8x4u __attribute__((ext_vector_type(4), aligned(1)));

// e^x - 1 - x >= 0: its series up to x^9 where e^x - 1 and x cancel (next term below 3e-9 of the value)
__device__ __forceinline__ float kl_term(float x) {
  if (fabsf(x) >= 0.5f) return expm1f(x) - x;
  float p = 1.f / 362880.f;
  p = p * x + 1.f / 40320.f;
  p = p * x + 1.f / 5040.f;
  p = p * x + 1.f / 720.f;
  p = p * x + 1.f / 120.f;
  p = p * x + 1.f / 24.f;
  p = p * x + 1.f / 6.f;
  p = p * x + 0.5f;
  return p * x * x;
}

// Block-wide sums of N doubles, for blocks of whole waves; valid in thread 0.
template <int N>
__device__ __forceinline__ void block_sums(double (&v)[N], double* sm /* N x 16 */) {
  const int w = threadIdx.x / WAVE, l = threadIdx.x % WAVE, nw = blockDim.x / WAVE;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    v[k] = wave_sum(v[k]);
    if (l == 0) sm[k * 16 + w] = v[k];
  }
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      v[k] = 0.0;
      for (int i = 0; i < nw; ++i) v[k] += sm[k * 16 + i];
    }
  }
}
__device__ __forceinline__ int64_t wave_sum64(int64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor((long long)v, o, WAVE);
  return v;
}

// Tokens of mask[0, n) that count, summed over the lanes of a group of NT threads' own shares.
template <int NT>
__device__ __forceinline__ int count_share(const uint8_t* m, int64_t n, int tid) {
  typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(1)));
  int c = 0;
  const int64_t nv = n / 16;
  for (int64_t j = tid; j < nv; j += NT) {
    const u32x4u v = reinterpret_cast<const u32x4u*>(m)[j];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      // 1 in every byte that is not 0: its low 7 bits carry into bit 7, or bit 7 is set
      const uint32_t b = (((v[q] & 0x7f7f7f7fu) + 0x7f7f7f7fu) | v[q]) & 0x80808080u;
      c += __popc(b);
    }
  }
  if (tid < n - nv * 16) c += m[nv * 16 + tid] != 0;
  return c;
}

// ------------------------------------------------------------------ policy loss
constexpr int POL_SUMS = 6, POL_BLOCKS = 1024, POL_COUNT_BLOCKS = 256;
constexpr int POL_SMALL_TOKENS = 8192, POL_SMALL_SEQS = 1024;

// Weight of a token of a sequence with n tokens that count.
__device__ __forceinline__ double token_weight(const PolicyArgs& a, double tokens, double seqs, int n) {
  if (n == 0) return 0.0;
  if (a.seq_mean) return 1.0 / ((a.norm > 0 ? a.norm : seqs) * n);
  return 1.0 / (a.norm > 0 ? a.norm : tokens);
}

// Token i of sequence b at weight w: its terms into acc, its gradients returned.
// Which side of the clip a token is on is decided in the logarithm, on the exact difference of the two
// log-probabilities, so that the gradient's jump there does not hang on the rounding of e^x.
__device__ __forceinline__ void policy_token(const PolicyArgs& a, float lp, float old, float adv, float ref, float ent,
                                             double w, double (&acc)[POL_SUMS], float& g, float& ge) {
  const double x = (double)lp - (double)old;
  const float xf = (float)x, r = expf(xf);
  const bool rise = adv > 0.f && x > a.log_hi, fall = adv < 0.f && x < a.log_lo;
  const float held = rise ? 1.f + a.clip_high : fall ? 1.f - a.clip_low : r;
  float d = rise || fall ? 0.f : -r * adv;
  acc[0] += w * (double)(-held * adv);
  acc[3] += rise || fall ? w : 0.0;
  acc[4] += w * (double)kl_term(xf);
  acc[5] += w * (double)r;
  if (a.ref) {
    const float q = (float)((double)ref - (double)lp);
    acc[1] += w * (double)kl_term(q);
    if (a.kl_coef != 0.f) d -= a.kl_coef * expm1f(q);
  }
  if (a.ent) acc[2] += w * (double)ent;
  const float gw = (float)(w * a.grad_scale);
  g = gw * d;
  ge = -a.ent_coef * gw;
}

// Vectors j0, j0 + step, ... of 4 tokens
__device__ __forceinline__ void policy_walk(const PolicyArgs& a, int64_t j0, int64_t step, const int* nb, double tokens,
                                            double seqs, double (&acc)[POL_SUMS]) {
  const int64_t n = a.seqs * a.len;
  for (int64_t j = j0; 4 * j < n; j += step) {
    const int64_t i = 4 * j;
    int64_t b = (uint64_t)i >> 32 ? i / a.len : (int64_t)((uint32_t)i / (uint32_t)a.len);
    int64_t left = (b + 1) * a.len - i;  // tokens of sequence b from i on
    float g[4] = {0.f, 0.f, 0.f, 0.f}, ge[4] = {0.f, 0.f, 0.f, 0.f};
    const int m = (int)min((int64_t)4, n - i);
    uint8_t on[4] = {0, 0, 0, 0};
    if (m == 4) {
      const u8x4u v = *reinterpret_cast<const u8x4u*>(a.mask + i);
#pragma unroll
      for (int q = 0; q < 4; ++q) on[q] = v[q];
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < m) on[q] = a.mask[i + q];
    }
    if (on[0] | on[1] | on[2] | on[3]) {
      float lp[4] = {}, old[4] = {}, ref[4] = {}, ent[4] = {}, adv[4] = {};
      auto get = [&](const float* p, float (&v)[4]) {
        if (m == 4) {
          const f32x4u u = *reinterpret_cast<const f32x4u*>(p + i);
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = u[q];
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (q < m) v[q] = p[i + q];
        }
      };
      get(a.logp, lp);
      get(a.old, old);
      if (a.ref) get(a.ref, ref);
      if (a.ent) get(a.ent, ent);
      if (a.per_token) get(a.adv, adv);
      double w = token_weight(a, tokens, seqs, nb[b]);
      float ab = a.per_token ? 0.f : a.adv[b];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q < m) {
          if (left == 0) {
            ++b;
            left = a.len;
            w = token_weight(a, tokens, seqs, nb[b]);
            if (!a.per_token) ab = a.adv[b];
          }
          --left;
          if (on[q]) policy_token(a, lp[q], old[q], a.per_token ? adv[q] : ab, ref[q], ent[q], w, acc, g[q], ge[q]);
        }
      }
    }
    auto put = [&](float* p, const float (&v)[4]) {
      if (m == 4) {
        *reinterpret_cast<f32x4u*>(p + i) = f32x4u{v[0], v[1], v[2], v[3]};
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (q < m) p[i + q] = v[q];
      }
    };
    put(a.dlogp, g);
    if (a.dent) put(a.dent, ge);
  }
}

__device__ __forceinline__ void policy_out(const PolicyArgs& a, const double (&v)[POL_SUMS], int64_t tokens,
                                           int64_t seqs) {
  double l = v[0];  // an infinite KL or entropy counts only where it has a weight
  if (a.kl_coef != 0.f) l += (double)a.kl_coef * v[1];
  if (a.ent_coef != 0.f) l -= (double)a.ent_coef * v[2];
  a.loss[0] = (float)l;
#pragma unroll
  for (int k = 0; k < POL_SUMS; ++k) a.metrics[k] = (float)v[k];
  a.counts[0] = tokens;
  a.counts[1] = seqs;
}

// Counts of every sequence, and the block's totals: a wave per sequence, or the block where they are long.
__global__ void __launch_bounds__(1024) policy_count(PolicyArgs a, int* nb, int64_t* totals) {
  __shared__ int64_t sm[2][16];
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
  int64_t tokens = 0, seqs = 0;  // lane 0 of every wave
  if (a.len >= 16384) {
    __shared__ int part[16];
    for (int64_t b = blockIdx.x; b < a.seqs; b += gridDim.x) {
      const int c = (int)wave_sum64(count_share<1024>(a.mask + b * a.len, a.len, threadIdx.x));
      __syncthreads();
      if (lane == 0) part[wave] = c;
      __syncthreads();
      if (threadIdx.x == 0) {
        int n = 0;
        for (int w = 0; w < 16; ++w) n += part[w];
        nb[b] = n;
        tokens += n;
        seqs += n > 0;
      }
    }
  } else {
    for (int64_t b = (int64_t)blockIdx.x * 16 + wave; b < a.seqs; b += (int64_t)gridDim.x * 16) {
      const int n = (int)wave_sum64(count_share<WAVE>(a.mask + b * a.len, a.len, lane));
      if (lane == 0) {
        nb[b] = n;
        tokens += n;
        seqs += n > 0;
      }
    }
  }
  if (lane == 0) sm[0][wave] = tokens, sm[1][wave] = seqs;
  __syncthreads();
  if (threadIdx.x < 2) {
    int64_t v = 0;
    for (int w = 0; w < 16; ++w) v += sm[threadIdx.x][w];
    totals[2 * blockIdx.x + threadIdx.x] = v;
  }
}

// The sum of the count blocks' totals, in every thread (blockDim.x >= nblk).
__device__ __forceinline__ void policy_totals(const int64_t* totals, int nblk, int64_t& tokens, int64_t& seqs) {
  __shared__ int64_t sm[2][16];
  const bool in = (int)threadIdx.x < nblk;
  const int64_t t = wave_sum64(in ? totals[2 * threadIdx.x] : 0), s = wave_sum64(in ? totals[2 * threadIdx.x + 1] : 0);
  if (threadIdx.x % WAVE == 0) sm[0][threadIdx.x / WAVE] = t, sm[1][threadIdx.x / WAVE] = s;
  __syncthreads();
  tokens = seqs = 0;
  for (int w = 0; w < (int)blockDim.x / WAVE; ++w) tokens += sm[0][w], seqs += sm[1][w];
}

__global__ void __launch_bounds__(256) policy_tokens(PolicyArgs a, const int* nb, const int64_t* totals, int ncount,
                                                     double* sums) {
  __shared__ double sm[POL_SUMS * 16];
  int64_t tokens, seqs;
  policy_totals(totals, ncount, tokens, seqs);
  double acc[POL_SUMS] = {};
  policy_walk(a, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256, nb, (double)tokens, (double)seqs, acc);
  block_sums(acc, sm);
  if (threadIdx.x == 0) {
#pragma unroll
    for (int k = 0; k < POL_SUMS; ++k) sums[POL_SUMS * blockIdx.x + k] = acc[k];
  }
}

__global__ void __launch_bounds__(256) policy_finish(PolicyArgs a, const int64_t* totals, int ncount, const double* sums,
                                                     int nblk) {
  __shared__ double sm[POL_SUMS * 16];
  int64_t tokens, seqs;
  policy_totals(totals, ncount, tokens, seqs);
  double acc[POL_SUMS] = {};
  for (int i = threadIdx.x; i < nblk; i += 256)
#pragma unroll
    for (int k = 0; k < POL_SUMS; ++k) acc[k] += sums[POL_SUMS * i + k];
  block_sums(acc, sm);
  if (threadIdx.x == 0) policy_out(a, acc, tokens, seqs);
}

// Few tokens: one block does all of it.
__global__ void __launch_bounds__(1024) policy_small(PolicyArgs a) {
  __shared__ int nb[POL_SMALL_SEQS];
  __shared__ double sm[POL_SUMS * 16];
  __shared__ int64_t tot[2][16];
  const int n = (int)(a.seqs * a.len);
  for (int b = threadIdx.x; b < (int)a.seqs; b += 1024) nb[b] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 1024)
    if (a.mask[i]) atomicAdd(&nb[i / (int)a.len], 1);
  __syncthreads();
  int64_t tokens = 0, seqs = 0;
  for (int b = threadIdx.x; b < (int)a.seqs; b += 1024) tokens += nb[b], seqs += nb[b] > 0;
  tokens = wave_sum64(tokens);
  seqs = wave_sum64(seqs);
  if (threadIdx.x % WAVE == 0) tot[0][threadIdx.x / WAVE] = tokens, tot[1][threadIdx.x / WAVE] = seqs;
  __syncthreads();
  tokens = seqs = 0;
  for (int w = 0; w < 16; ++w) tokens += tot[0][w], seqs += tot[1][w];
  double acc[POL_SUMS] = {};
  policy_walk(a, threadIdx.x, 1024, nb, (double)tokens, (double)seqs, acc);
  block_sums(acc, sm);
  if (threadIdx.x == 0) policy_out(a, acc, tokens, seqs);
}

bool policy_is_small(int64_t seqs, int64_t len) { return seqs <= POL_SMALL_SEQS && seqs * len <= POL_SMALL_TOKENS; }

// ------------------------------------------------------------------ preference loss
constexpr int PREF_SUMS = 6, PREF_SMALL_ROWS = 512, PREF_SMALL_TOKENS = 8192;

// Sum of logp - ref over the tokens of [t0, t1) of a row that count, and their number: this thread's share.
template <int NT>
__device__ __forceinline__ void pref_share(const PreferenceArgs& a, int64_t row, int64_t t0, int64_t t1, int tid,
                                           double& s, int& n) {
  const int64_t o = row * a.len;
  for (int64_t t = t0 + 4 * tid; t < t1; t += 4 * NT) {
    if (t + 4 <= t1) {
      const u8x4u on = *reinterpret_cast<const u8x4u*>(a.mask + o + t);
      if (!(on[0] | on[1] | on[2] | on[3])) continue;
      const f32x4u l = *reinterpret_cast<const f32x4u*>(a.logp + o + t);
      f32x4u r = {0.f, 0.f, 0.f, 0.f};
      if (a.ref) r = *reinterpret_cast<const f32x4u*>(a.ref + o + t);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (on[q]) {
          s += (double)l[q] - (double)r[q];
          ++n;
        }
      }
    } else {
      for (int64_t u = t; u < t1; ++u) {
        if (a.mask[o + u]) {
          s += (double)a.logp[o + u] - (a.ref ? (double)a.ref[o + u] : 0.0);
          ++n;
        }
      }
    }
  }
}

// Pair p from its rows' sums and counts: its loss, rewards and terms; coef receives the rows' token gradients
// apart from the mean's 1 / pairs.
__device__ __forceinline__ void pref_pair(const PreferenceArgs& a, int64_t p, double sw, int nw, double sl, int nl,
                                          double (&acc)[PREF_SUMS], double& cw, double& cl) {
  cw = cl = 0.0;
  if (nw == 0 || nl == 0) {
    a.pair_loss[p] = 0.f;
    a.rewards[p] = a.rewards[p + a.pairs] = 0.f;
    return;
  }
  if (a.normalize) sw /= nw, sl /= nl;
  const double delta = sw - sl, h = a.beta * delta - a.margin, e = a.smoothing;
  double loss, dh;
  if (a.kind == 0) {
    const double soft = log1p(exp(-fabs(h)));  // log(1 + e^-|h|)
    loss = (1.0 - e) * (soft + fmax(-h, 0.0)) + (e > 0.0 ? e * (soft + fmax(h, 0.0)) : 0.0);
    if (h != h) loss = h;
    dh = e - 1.0 / (1.0 + exp(h));
  } else if (a.kind == 1) {
    loss = fmax(1.0 - h, 0.0);
    if (h != h) loss = h;
    dh = h < 1.0 ? -1.0 : h != h ? h : 0.0;
  } else {
    const double u = (h - 0.5) / a.beta;
    loss = u * u;
    dh = 2.0 * u / a.beta;
  }
  cw = a.beta * dh;
  cl = -cw;
  if (a.normalize) cw /= nw, cl /= nl;
  a.pair_loss[p] = (float)loss;
  a.rewards[p] = (float)(a.beta * sw);
  a.rewards[p + a.pairs] = (float)(a.beta * sl);
  acc[0] += loss;
  acc[1] += delta > 0.0 ? 1.0 : 0.0;
  acc[2] += a.beta * sw;
  acc[3] += a.beta * sl;
  acc[4] += h;
  acc[5] += 1.0;
}

// 1 / the number the mean divides by
__device__ __forceinline__ double pref_scale(const PreferenceArgs& a, double pairs) {
  return a.norm > 0 ? 1.0 / a.norm : pairs > 0 ? 1.0 / pairs : 0.0;
}
__device__ __forceinline__ void pref_out(const PreferenceArgs& a, const double (&v)[PREF_SUMS]) {
  const double s = pref_scale(a, v[5]);
  a.loss[0] = (float)(v[0] * s);
#pragma unroll
  for (int k = 0; k < 4; ++k) a.metrics[k] = (float)(v[k + 1] * s);
  a.counts[0] = (int64_t)v[5];
}

// dlogp of vectors j0, j0 + step, ... of 4 tokens; coef(row) is the gradient of a token that counts
template <typename F>
__device__ __forceinline__ void pref_walk(const PreferenceArgs& a, int64_t j0, int64_t step, const F& coef) {
  const int64_t n = 2 * a.pairs * a.len;
  for (int64_t j = j0; 4 * j < n; j += step) {
    const int64_t i = 4 * j;
    int64_t row = (uint64_t)i >> 32 ? i / a.len : (int64_t)((uint32_t)i / (uint32_t)a.len);
    int64_t left = (row + 1) * a.len - i;
    float c = coef(row);
    if (i + 4 <= n) {
      const u8x4u on = *reinterpret_cast<const u8x4u*>(a.mask + i);
      f32x4u g;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (left == 0) left = a.len, c = coef(++row);
        --left;
        g[q] = on[q] ? c : 0.f;
      }
      *reinterpret_cast<f32x4u*>(a.dlogp + i) = g;
    } else {
      for (int64_t u = i; u < n; ++u) {
        if (left == 0) left = a.len, c = coef(++row);
        --left;
        a.dlogp[u] = a.mask[u] ? c : 0.f;
      }
    }
  }
}

// Partial sums of chunk blockIdx.x mod cps of row blockIdx.x / cps
__global__ void __launch_bounds__(256) pref_sums(PreferenceArgs a, int cps, int64_t per, double* sums, int* ns) {
  __shared__ double sm[2 * 16];
  const int64_t items = 2 * a.pairs * cps;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t row = it / cps, t0 = (it % cps) * per;
    double v[2] = {0.0, 0.0};
    int n = 0;
    pref_share<256>(a, row, t0, min(a.len, t0 + per), threadIdx.x, v[0], n);
    v[1] = (double)n;
    block_sums(v, sm);
    if (threadIdx.x == 0) {
      sums[it] = v[0];
      ns[it] = (int)v[1];
    }
  }
}

// Every pair, one block: coef[row] = the gradient of the row's tokens
__global__ void __launch_bounds__(1024) pref_pairs(PreferenceArgs a, int cps, double* sums, int* ns, double* raw,
                                                   float* coef) {
  __shared__ double sm[PREF_SUMS * 16];
  __shared__ double scale;
  if (cps > 1) {  // a wave per row joins its chunks (into the first)
    for (int64_t row = threadIdx.x / WAVE; row < 2 * a.pairs; row += 16) {
      double s = 0.0;
      int64_t n = 0;
      for (int k = threadIdx.x % WAVE; k < cps; k += WAVE) s += sums[row * cps + k], n += ns[row * cps + k];
      s = wave_sum(s);
      n = wave_sum64(n);
      if (threadIdx.x % WAVE == 0) sums[row * cps] = s, ns[row * cps] = (int)n;
    }
    __threadfence_block();
    __syncthreads();
  }
  double acc[PREF_SUMS] = {};
  for (int64_t p = threadIdx.x; p < a.pairs; p += 1024) {
    const int64_t w = p * cps, l = (p + a.pairs) * cps;
    double cw, cl;
    pref_pair(a, p, sums[w], ns[w], sums[l], ns[l], acc, cw, cl);
    raw[p] = cw;
    raw[p + a.pairs] = cl;
  }
  block_sums(acc, sm);
  if (threadIdx.x == 0) {
    pref_out(a, acc);
    scale = pref_scale(a, acc[5]) * a.grad_scale;
  }
  __syncthreads();
  for (int64_t p = threadIdx.x; p < a.pairs; p += 1024) {
    coef[p] = (float)(raw[p] * scale);
    coef[p + a.pairs] = (float)(raw[p + a.pairs] * scale);
  }
}

__global__ void __launch_bounds__(256) pref_tokens(PreferenceArgs a, const float* coef) {
  pref_walk(a, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256, [&](int64_t r) { return coef[r]; });
}

// Few tokens: one block does all of it.
__global__ void __launch_bounds__(1024) pref_small(PreferenceArgs a) {
  __shared__ double sum[PREF_SMALL_ROWS], sm[PREF_SUMS * 16], scale;
  __shared__ int cnt[PREF_SMALL_ROWS];
  const int rows = (int)(2 * a.pairs);
  for (int row = threadIdx.x / WAVE; row < rows; row += 16) {
    double s = 0.0;
    int n = 0;
    pref_share<WAVE>(a, row, 0, a.len, threadIdx.x % WAVE, s, n);
    s = wave_sum(s);
    n = (int)wave_sum64(n);
    if (threadIdx.x % WAVE == 0) sum[row] = s, cnt[row] = n;
  }
  __syncthreads();
  double acc[PREF_SUMS] = {}, cw = 0.0, cl = 0.0;
  const int p = threadIdx.x;
  if (p < (int)a.pairs) pref_pair(a, p, sum[p], cnt[p], sum[p + a.pairs], cnt[p + a.pairs], acc, cw, cl);
  block_sums(acc, sm);
  if (threadIdx.x == 0) {
    pref_out(a, acc);
    scale = pref_scale(a, acc[5]) * a.grad_scale;
  }
  if (p < (int)a.pairs) sum[p] = cw, sum[p + a.pairs] = cl;
  __syncthreads();
  pref_walk(a, threadIdx.x, 1024, [&](int64_t r) { return (float)(sum[r] * scale); });
}

bool pref_is_small(int64_t pairs, int64_t len) {
  return 2 * pairs <= PREF_SMALL_ROWS && 2 * pairs * len <= PREF_SMALL_TOKENS;
}
// Chunks of a row: one where the rows alone make enough blocks
int pref_chunks(int64_t pairs, int64_t len) {
  if (2 * pairs >= 512) return 1;
  return (int)std::max<int64_t>(1, std::min(cdiv(len, 2048), cdiv(1024, 2 * pairs)));
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

size_t policy_ws_bytes(int64_t seqs, int64_t len) {
  if (policy_is_small(seqs, len)) return 0;
  return up256(POL_BLOCKS * POL_SUMS * sizeof(double)) + up256(POL_COUNT_BLOCKS * 2 * sizeof(int64_t)) +
         up256((size_t)seqs * sizeof(int));
}

void launch_policy_loss(const PolicyArgs& a, void* ws, hipStream_t st) {
  if (policy_is_small(a.seqs, a.len)) {
    policy_small<<<1, 1024, 0, st>>>(a);
    return;
  }
  double* sums = (double*)ws;
  int64_t* totals = (int64_t*)((char*)ws + up256(POL_BLOCKS * POL_SUMS * sizeof(double)));
  int* nb = (int*)((char*)totals + up256(POL_COUNT_BLOCKS * 2 * sizeof(int64_t)));
  const int64_t groups = a.len >= 16384 ? a.seqs : cdiv(a.seqs, 16);
  const int ncount = (int)std::min<int64_t>(POL_COUNT_BLOCKS, groups);
  const int nblk = (int)std::min<int64_t>(POL_BLOCKS, cdiv(a.seqs * a.len, 1024));
  policy_count<<<ncount, 1024, 0, st>>>(a, nb, totals);
  policy_tokens<<<nblk, 256, 0, st>>>(a, nb, totals, ncount, sums);
  policy_finish<<<1, 256, 0, st>>>(a, totals, ncount, sums, nblk);
}

size_t preference_ws_bytes(int64_t pairs, int64_t len) {
  if (pref_is_small(pairs, len)) return 0;
  const size_t n = 2 * (size_t)pairs, c = n * pref_chunks(pairs, len);
  return up256(c * sizeof(double)) + up256(c * sizeof(int)) + up256(n * sizeof(double)) + up256(n * sizeof(float));
}

void launch_preference_loss(const PreferenceArgs& a, void* ws, hipStream_t st) {
  if (pref_is_small(a.pairs, a.len)) {
    pref_small<<<1, 1024, 0, st>>>(a);
    return;
  }
  const int cps = pref_chunks(a.pairs, a.len);
  const size_t n = 2 * (size_t)a.pairs, c = n * cps;
  double* sums = (double*)ws;
  int* ns = (int*)((char*)sums + up256(c * sizeof(double)));
  double* raw = (double*)((char*)ns + up256(c * sizeof(int)));
  float* coef = (float*)((char*)raw + up256(n * sizeof(double)));
  const int64_t per = cdiv(cdiv(a.len, cps), 4) * 4;
  pref_sums<<<(unsigned)std::min<int64_t>(1 << 20, (int64_t)c), 256, 0, st>>>(a, cps, per, sums, ns);
  pref_pairs<<<1, 1024, 0, st>>>(a, cps, sums, ns, raw, coef);
  if (a.len > 0)
    pref_tokens<<<(unsigned)std::min<int64_t>(1 << 16, cdiv((int64_t)n * a.len, 1024)), 256, 0, st>>>(a, coef);
}
