// Losses on the log-probabilities of answers, with their gradients: the clipped policy loss with a KL term
// and an entropy bonus, and the preference loss of paired log ratios.
//
// Arrays are [sequences, len] row-major; a token counts where its mask byte is not 0, and what stands at the
// others, whatever it is, is selected away and reaches nothing.  Sums run in double in a fixed order.
//
// Both are bound by memory where they are large and by round trips to it where they are not.  Policy loss: the
// weights need the counts before the gradients can be written, so a first kernel counts (the mask alone), a
// second takes the tokens, 4 a thread with the next ones' mask on its way, and its last block or, above 2^17 tokens,
// a third kernel adds the blocks' sums; up to 8192 tokens one block does it all.  512 x 4096 tokens of which 0.4
// count, with reference, entropy and advantage per token: 3.5 + 13.7 + 3.9 us, 35 MB in the second, in which a copy
// of as many bytes takes 7.9 and the vector instructions, 360 per 4 tokens, 5.0; 37 x 1111: 2.8 + 7.5; 4 x 64: 3.6.
// Preference loss: the rows' sums, then the pairs and the gradients in one kernel whose blocks find their row's
// coefficient themselves (with the number of pairs that count).  256 pairs of 4096: 4.5 + 5.5 us, 17 MB at 1.7
// TB/s; 2 x 100: 4.1.
#include "common.h"
#include "kernels.h"
#include <algorithm>

namespace {

// 4 consecutive tokens at any alignment
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint8_t u8x4u __attribute__((ext_vector_type(4), aligned(1)));

// e^x - 1 - x >= 0, given ex = e^x: the series up to x^9 where the difference cancels (next term below 3e-9 of
// the value; from |x| = 1/2 on the difference keeps all but 2 bits).  With x added it is e^x - 1.  Infinite at x = +-inf:
// past 89 e^x is infinite and no less for an x of 128 taken away.
__device__ __forceinline__ float kl_term(float x, float ex) {
  float p = 1.f / 362880.f;
  p = p * x + 1.f / 40320.f;
  p = p * x + 1.f / 5040.f;
  p = p * x + 1.f / 720.f;
  p = p * x + 1.f / 120.f;
  p = p * x + 1.f / 24.f;
  p = p * x + 1.f / 6.f;
  p = p * x + 0.5f;
  const float near = p * x * x, far = (ex - 1.f) - fminf(x, 128.f);  // both, so that no branch holds up the next token
  return fabsf(x) >= 0.5f ? far : near;
}

// Sums over each 16 lanes, in all of them.
template <int CTRL>
__device__ __forceinline__ double row_add(double v) {
  uint32_t w[2];
  __builtin_memcpy(w, &v, 8);
  w[0] = (uint32_t)__builtin_amdgcn_mov_dpp((int)w[0], CTRL, 0xf, 0xf, true);
  w[1] = (uint32_t)__builtin_amdgcn_mov_dpp((int)w[1], CTRL, 0xf, 0xf, true);
  double o;
  __builtin_memcpy(&o, w, 8);
  return v + o;
}
__device__ __forceinline__ double row_total(double v) {
  return row_add<0x121>(row_add<0x122>(row_add<0x124>(row_add<0x128>(v))));  // row_ror 8, 4, 2, 1
}
__device__ __forceinline__ double read_lane(double v, int lane) {
  uint32_t w[2];
  __builtin_memcpy(w, &v, 8);
  w[0] = (uint32_t)__builtin_amdgcn_readlane((int)w[0], lane);
  w[1] = (uint32_t)__builtin_amdgcn_readlane((int)w[1], lane);
  __builtin_memcpy(&v, w, 8);
  return v;
}
// [a.low + a.high | b.low + b.high] of the wave's halves; with ROWS of its 16-lane rows 0 + 1 and 2 + 3,
// [a01 | b01 | a23 | b23]
template <bool ROWS>
__device__ __forceinline__ double swap_add(double a, double b) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  uint32_t x[2], y[2];
  __builtin_memcpy(x, &a, 8);
  __builtin_memcpy(y, &b, 8);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const u32x2 r = ROWS ? __builtin_amdgcn_permlane16_swap(x[k], y[k], false, false)
                         : __builtin_amdgcn_permlane32_swap(x[k], y[k], false, false);
    x[k] = r[0], y[k] = r[1];
  }
  __builtin_memcpy(&a, x, 8);
  __builtin_memcpy(&b, y, 8);
  return a + b;
}
// Sums of N doubles over the wave, in every lane: two exchanges leave a row of 16 lanes to each value, so that four of
// them take the last four steps at once (some 50 instructions for 6 values, one after the other 190: 37 x 1111 tokens of
// the policy loss 11.1 -> 9.9 us, 2 pairs of 100 5.3 -> 4.1).
template <int N>
__device__ __forceinline__ void wave_sums(double (&v)[N]) {
  constexpr int H = (N + 1) / 2, Q = (H + 1) / 2;
  double a[H], b[Q];
#pragma unroll
  for (int j = 0; j < H; ++j) a[j] = swap_add<false>(v[2 * j], v[2 * j + 1 < N ? 2 * j + 1 : N - 1]);
#pragma unroll
  for (int j = 0; j < Q; ++j) b[j] = row_total(swap_add<true>(a[2 * j], a[2 * j + 1 < H ? 2 * j + 1 : H - 1]));
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = read_lane(b[k / 4], (k % 2) * 32 + (k / 2 % 2) * 16);
}

// Block-wide sums of N doubles, for blocks of whole waves; valid in the first wave.
template <int N>
__device__ __forceinline__ void block_sums(double (&v)[N], double* sm /* N x 16 */) {
  const int w = threadIdx.x / WAVE, l = threadIdx.x % WAVE, nw = blockDim.x / WAVE;
  wave_sums(v);
  if (nw == 1) return;
  __syncthreads();
  if (l == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) sm[k * 16 + w] = v[k];
  }
  __syncthreads();
  if (w == 0) {
#pragma unroll
    for (int j = 0; j < N; j += 4) {  // a row of lanes per value
      const int k = j + l / 16;
      const double t = row_total(k < N && l % 16 < nw ? sm[k * 16 + l % 16] : 0.0);
#pragma unroll
      for (int q = 0; q < 4 && j + q < N; ++q) v[j + q] = read_lane(t, 16 * q);
    }
  }
}

// Tokens of mask[0, n) that count, summed over the lanes of a group of NT threads' own shares.
template <int NT>
__device__ __forceinline__ int count_share(const uint8_t* m, int64_t n, int tid) {
  typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(1)));
  int c = 0;
  auto add = [&](const u32x4u& v) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      // bit 7 of every byte that is not 0: its low 7 bits carry into it, or it is set
      const uint32_t b = (((v[q] & 0x7f7f7f7fu) + 0x7f7f7f7fu) | v[q]) & 0x80808080u;
      c += __popc(b);
    }
  };
  const u32x4u* p = reinterpret_cast<const u32x4u*>(m);
  const int64_t nv = n / 16;
  int64_t j = tid;
  for (; j + 3 * NT < nv; j += 4 * NT) {
    const u32x4u v0 = p[j], v1 = p[j + NT], v2 = p[j + 2 * NT], v3 = p[j + 3 * NT];
    add(v0), add(v1), add(v2), add(v3);
  }
  for (; j < nv; j += NT) add(p[j]);
  for (j = nv * 16 + tid; j < n; j += NT) c += m[j] != 0;
  return c;
}

// ------------------------------------------------------------------ policy loss
constexpr int POL_SUMS = 6, POL_BLOCKS = 1024, POL_COUNT_BLOCKS = WAVE, POL_LAST_BLOCKS = 128;
// policy_small: at most two vectors of 4 tokens and four of 16 mask bytes per thread of 64 to 1024.  One launch against
// two, us on the GPU: 4096 tokens 7.1 : 8.4, 8192 9.4 : 8.6, with sequence means 11.9 : 8.9; as issued, 8192 13.4 : 19.1
// and 13.1 : 18.8.
constexpr int POL_SMALL_TOKENS = 8192, POL_SMALL_SEQS = 1024;

// 1 / n for n > 0, to 2^-44: one step of Newton's method from the hardware's 2^-23
__device__ __forceinline__ double inverse(int n) {
  const double d = n, y = (double)__builtin_amdgcn_rcpf((float)n);
  return y * (2.0 - d * y);
}
// What a call has, known where its kernel is compiled: policy loss over 512 x 4096 tokens with all of it 22 us,
// with the same code asking for each 25.
enum { POL_REF = 1, POL_ENT = 2, POL_TOKEN_ADV = 4, POL_SEQ_MEAN = 8 };

// 1 / what the mean divides by, the number of tokens or of sequences that count or norm (0 where nothing
// counts): the weight of a token, or of a sequence with seq_mean
__device__ __forceinline__ double mean_scale(const PolicyArgs& a, int64_t tokens, int64_t seqs) {
  const double d = a.norm > 0 ? a.norm : (double)(a.seq_mean ? seqs : tokens);
  return d > 0 ? 1.0 / d : 0.0;
}

// A token's terms, times w, added to acc where it counts (whatever the others hold), and its gradient apart from
// the weight.  Which side of the clip a token is on is decided in the logarithm, on the exact difference of the two
// log-probabilities, so that the gradient's jump there does not hang on the rounding of e^x.
template <int F>
__device__ __forceinline__ float policy_token(const PolicyArgs& a, bool on, double w, float lp, float old, float adv,
                                              float ref, float ent, double (&acc)[POL_SUMS]) {
  auto add = [&](int k, float v) { acc[k] += w * (double)(on ? v : 0.f); };
  const double x = (double)lp - (double)old;
  const float xf = (float)x, r = expf(xf);
  const bool rise = adv > 0.f && x > a.log_hi, fall = adv < 0.f && x < a.log_lo, cut = rise || fall;
  const float kx = kl_term(xf, r);
  // The surrogate's terms have both signs, and where they cancel the rounding of e^x would be all that is left: near
  // 1 it is taken from its small part in double (the loss against 64 bits over 150 cases 2.7e-7 -> 2.5e-8).
  const double near1 = (1.0 + x) + (double)kx, e = fabsf(xf) >= 0.5f ? (double)r : near1, av = on ? adv : 0.f;
  const double held = rise ? 1.0 + (double)a.clip_high : fall ? 1.0 - (double)a.clip_low : e;
  const double ra = av == 0.0 ? 0.0 : held * av;  // no advantage: nothing, also where e^x is past the type
  float d = cut ? 0.f : -(float)ra;
  acc[0] -= w * ra;
  add(3, cut ? 1.f : 0.f);
  add(4, kx);
  add(5, r);
  if constexpr (F & POL_REF) {
    const float q = ref - lp, eq = expf(q), k = kl_term(q, eq);
    add(1, k);
    const float near = k + q, far = eq - 1.f;
    if (a.kl_coef != 0.f) d -= a.kl_coef * (fabsf(q) >= 0.5f ? far : near);
  }
  if constexpr (F & POL_ENT) add(2, ent);
  return on ? d : 0.f;
}

// sequence of token i
__device__ __forceinline__ int64_t seq_of(int64_t i, int64_t len) {
  return (uint64_t)i >> 32 ? i / len : (int64_t)((uint32_t)i / (uint32_t)len);
}

// 4 consecutive tokens i .. i + 3 of the flat arrays: the first in sequence b, those from token `turn` on in
// b + 1; the two sequences' counts and advantages.  vec: all four exist and sequences are at least that long (the
// others are taken one by one, from memory).
struct Tokens {
  uint32_t on;  // the mask's 4 bytes, taken apart where they are used (at once, they would be waited for)
  f32x4u lp, old, ref, ent, adv;
  int turn, nb0, nb1;
  float ab0, ab1;
  bool vec;
};
template <int F>
__device__ __forceinline__ void tokens_start(Tokens& v, const PolicyArgs& a, int64_t i, int64_t n, const int* nb) {
  v.vec = i + 4 <= n && a.len >= 4;
  if (!v.vec) return;
  const int64_t b = seq_of(i, a.len), left = (b + 1) * a.len - i;
  v.turn = left < 4 ? (int)left : 4;
  typedef uint32_t u32u __attribute__((aligned(1)));
  v.on = *reinterpret_cast<const u32u*>(a.mask + i);
  const int64_t b1 = v.turn < 4 ? b + 1 : b;
  if ((F & POL_SEQ_MEAN) && nb) v.nb0 = nb[b], v.nb1 = nb[b1];
  if (!(F & POL_TOKEN_ADV)) v.ab0 = a.adv[b], v.ab1 = a.adv[b1];
}
__device__ __forceinline__ bool tokens_any(const Tokens& v) {
  return v.vec && v.on;
}
template <int F>
__device__ __forceinline__ void tokens_load(Tokens& v, const PolicyArgs& a, int64_t i) {
  if (!v.vec) return;
  auto get = [&](const float* p) { return *reinterpret_cast<const f32x4u*>(p + i); };
  v.lp = get(a.logp);
  v.old = get(a.old);
  if (F & POL_REF) v.ref = get(a.ref);
  if (F & POL_ENT) v.ent = get(a.ent);
  if (F & POL_TOKEN_ADV) v.adv = get(a.adv);
}

// Their sums and gradients; nb: the sequences' counts.
template <int F>
__device__ __forceinline__ void tokens_run(const PolicyArgs& a, const Tokens& v, int64_t i, int64_t n, const int* nb,
                                           double scale, double (&acc)[POL_SUMS]) {
  if (v.vec) {
    f32x4u g = {0.f, 0.f, 0.f, 0.f}, ge = g;
    if (tokens_any(v)) {
      // a sequence whose count is 0 has no token here: its weight is not used
      const double w0 = (F & POL_SEQ_MEAN) ? scale * inverse(max(v.nb0, 1)) : scale;
      const double w1 = (F & POL_SEQ_MEAN) ? scale * inverse(max(v.nb1, 1)) : scale;
      const float g0 = (float)(w0 * a.grad_scale), g1 = (float)(w1 * a.grad_scale);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const bool first = q < v.turn;
        const bool on = (v.on >> 8 * q & 0xff) != 0;
        const float gw = first ? g0 : g1, ab = first ? v.ab0 : v.ab1;
        const float d = policy_token<F>(a, on, first ? w0 : w1, v.lp[q], v.old[q], (F & POL_TOKEN_ADV) ? v.adv[q] : ab,
                                        v.ref[q], v.ent[q], acc);
        g[q] = on ? gw * d : 0.f;
        ge[q] = on ? -a.ent_coef * gw : 0.f;
      }
    }
    *reinterpret_cast<f32x4u*>(a.dlogp + i) = g;
    if (F & POL_ENT) *reinterpret_cast<f32x4u*>(a.dent + i) = ge;
    return;
  }
#pragma unroll 1
  for (int64_t j = i; j < min(i + 4, n); ++j) {
    float g = 0.f, ge = 0.f;
    if (a.mask[j]) {
      const int64_t b = seq_of(j, a.len);
      const double w = (F & POL_SEQ_MEAN) ? scale * inverse(nb[b]) : scale;
      const float gw = (float)(w * a.grad_scale);
      g = gw * policy_token<F>(a, true, w, a.logp[j], a.old[j], a.adv[(F & POL_TOKEN_ADV) ? j : b],
                               (F & POL_REF) ? a.ref[j] : 0.f, (F & POL_ENT) ? a.ent[j] : 0.f, acc);
      ge = -a.ent_coef * gw;
    }
    a.dlogp[j] = g;
    if (F & POL_ENT) a.dent[j] = ge;
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
// It also clears the count of the token pass's blocks that are done.
__global__ void __launch_bounds__(1024) policy_count(PolicyArgs a, int* nb, int64_t* totals, int* done) {
  __shared__ int64_t sm[2][16];
  if (blockIdx.x == 0 && threadIdx.x == 0) *done = 0;
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
  int64_t tokens = 0, seqs = 0;  // lane 0 of every wave
  if (a.len >= 16384) {
    __shared__ int part[16];
    for (int64_t b = blockIdx.x; b < a.seqs; b += gridDim.x) {
      const int c = wave_total(count_share<1024>(a.mask + b * a.len, a.len, threadIdx.x));
      __syncthreads();
      if (lane == 0) part[wave] = c;
      __syncthreads();
      if (wave == 0) {
        const int n = wave_total(lane < 16 ? part[lane] : 0);
        if (lane == 0) nb[b] = n;
        tokens += n;
        seqs += n > 0;
      }
    }
  } else {
    for (int64_t b = (int64_t)blockIdx.x * 16 + wave; b < a.seqs; b += (int64_t)gridDim.x * 16) {
      const int n = wave_total(count_share<WAVE>(a.mask + b * a.len, a.len, lane));
      if (lane == 0) {
        nb[b] = n;
        tokens += n;
        seqs += n > 0;
      }
    }
  }
  if (lane == 0) sm[0][wave] = tokens, sm[1][wave] = seqs;
  __syncthreads();
  if (wave == 0) {
    tokens = wave_total(lane < 16 ? sm[0][lane] : (int64_t)0);
    seqs = wave_total(lane < 16 ? sm[1][lane] : (int64_t)0);
    if (lane == 0) totals[2 * blockIdx.x] = tokens, totals[2 * blockIdx.x + 1] = seqs;
  }
}

// Totals of the count's blocks (at most a wave's lanes of them), in every thread of full waves.
__device__ __forceinline__ void policy_totals(const int64_t* totals, int nblk, int64_t& tokens, int64_t& seqs) {
  const int l = threadIdx.x % WAVE;
  double t[2] = {l < nblk ? (double)totals[2 * l] : 0.0, l < nblk ? (double)totals[2 * l + 1] : 0.0};  // exact
  wave_sums(t);
  tokens = (int64_t)t[0];
  seqs = (int64_t)t[1];
}

// The tokens' pass.  A thread's tokens are requested once their mask says that one counts: asking for them with the
// mask, one round trip less, reads the others too and measured the same from 9600 tokens on, 11 % more for 512 x 2048.
// The blocks' sums are policy_finish's to add; or, with `done`, the last block's, in their order whichever it is: every
// block publishes its own (stores at device scope) before it counts itself (acquire and release), the last one reads
// them after.  That saves a launch, but the release writes the block's L2 back: 37 x 1111 tokens 18.5 -> 15.2 us as
// issued (10.7 -> 11.2 on the GPU), 128 x 1024 12.1 -> 12.0, 256 x 1024 11.2 -> 14.6, 512 x 4096 22 -> 48.
template <int F>
__global__ void __launch_bounds__(256) policy_tokens(PolicyArgs a, const int* nb, const int64_t* totals, int ncount,
                                                     double* sums, int* done) {
  __shared__ double sm[POL_SUMS * 16];
  __shared__ bool last;
  const int64_t n = a.seqs * a.len, step = 1024 * (int64_t)gridDim.x;
  int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
  Tokens v = {}, next = {};
  if (i < n) {
    tokens_start<F>(v, a, i, n, nb);
    if (tokens_any(v)) tokens_load<F>(v, a, i);
  }
  int64_t tokens, seqs;
  policy_totals(totals, ncount, tokens, seqs);
  const double scale = mean_scale(a, tokens, seqs);
  double acc[POL_SUMS] = {};
  while (i < n) {
    const int64_t in = i + step;
    if (in < n) tokens_start<F>(next, a, in, n, nb);  // the next mask is on its way while these are worked on
    tokens_run<F>(a, v, i, n, nb, scale, acc);
    v = next;
    i = in;
    if (i < n && tokens_any(v)) tokens_load<F>(v, a, i);
  }
  block_sums(acc, sm);
  if (!done) {
    if (threadIdx.x == 0) {
#pragma unroll
      for (int k = 0; k < POL_SUMS; ++k) sums[k * gridDim.x + blockIdx.x] = acc[k];
    }
    return;
  }
  if (threadIdx.x == 0) {
#pragma unroll
    for (int k = 0; k < POL_SUMS; ++k)
      __hip_atomic_store(&sums[k * gridDim.x + blockIdx.x], acc[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = __hip_atomic_fetch_add(done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
#pragma unroll
  for (int k = 0; k < POL_SUMS; ++k) acc[k] = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += 256)
#pragma unroll
    for (int k = 0; k < POL_SUMS; ++k)
      acc[k] += __hip_atomic_load(&sums[k * gridDim.x + i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  block_sums(acc, sm);
  if (threadIdx.x == 0) policy_out(a, acc, tokens, seqs);
}

__global__ void __launch_bounds__(256) policy_finish(PolicyArgs a, const int64_t* totals, int ncount, const double* sums,
                                                     int nblk) {
  __shared__ double sm[POL_SUMS * 16];
  double acc[POL_SUMS] = {};
  for (int i = threadIdx.x; i < nblk; i += 256)
#pragma unroll
    for (int k = 0; k < POL_SUMS; ++k) acc[k] += sums[k * nblk + i];
  int64_t tokens, seqs;
  policy_totals(totals, ncount, tokens, seqs);
  block_sums(acc, sm);
  if (threadIdx.x == 0) policy_out(a, acc, tokens, seqs);
}

// Sets nb[0, seqs) in LDS to the tokens that count of every sequence of a mask of n <= 64 blockDim.x bytes,
// and tot to the totals.  The counts are integers, whose atomic sums have no order.
__device__ __forceinline__ void count_block(const PolicyArgs& a, int n, int* nb, int* tot) {
  typedef uint8_t u8x16u __attribute__((ext_vector_type(16), aligned(1)));
  const int nt = blockDim.x, len = (int)a.len;
  u8x16u v[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {  // all requested at once
    const int i = 16 * (threadIdx.x + k * nt);
    if (i + 16 <= n) v[k] = *reinterpret_cast<const u8x16u*>(a.mask + i);
  }
  for (int b = threadIdx.x; b < (int)a.seqs; b += nt) nb[b] = 0;
  if (threadIdx.x < 2) tot[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int i = 16 * (threadIdx.x + k * nt);
    if (i < n) {
      int b = (uint32_t)i / (uint32_t)len, left = (b + 1) * len - i, c = 0;
      if (i + 16 <= n && left >= 16) {
#pragma unroll
        for (int q = 0; q < 16; ++q) c += v[k][q] != 0;
      } else {
#pragma unroll 1
        for (int j = i; j < min(i + 16, n); ++j) {
          if (left == 0) {
            if (c) atomicAdd(&nb[b], c);
            ++b, left = len, c = 0;
          }
          --left;
          c += a.mask[j] != 0;
        }
      }
      if (c) atomicAdd(&nb[b], c);
    }
  }
  __syncthreads();
  int tokens = 0, seqs = 0;
  for (int b = threadIdx.x; b < (int)a.seqs; b += nt) tokens += nb[b], seqs += nb[b] > 0;
  tokens = wave_total(tokens);
  seqs = wave_total(seqs);
  if (threadIdx.x % WAVE == 0 && tokens > 0) {
    atomicAdd(&tot[0], tokens);
    atomicAdd(&tot[1], seqs);
  }
  __syncthreads();
}

// Few tokens: one block does all of it.  A thread's tokens are requested before the counts are known, so that
// the block waits for memory once.
template <int F>
__global__ void __launch_bounds__(1024) policy_small(PolicyArgs a) {
  __shared__ int nb[POL_SMALL_SEQS], tot[2];
  __shared__ double sm[POL_SUMS * 16];
  constexpr int PER = POL_SMALL_TOKENS / 4096;
  const int n = (int)(a.seqs * a.len), nt = blockDim.x;
  Tokens v[PER] = {};
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = 4 * (threadIdx.x + k * nt);
    if (i < n) {
      tokens_start<F>(v[k], a, i, n, nullptr);
      tokens_load<F>(v[k], a, i);
    }
  }
  count_block(a, n, nb, tot);
  double acc[POL_SUMS] = {};
  const double scale = mean_scale(a, tot[0], tot[1]);
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = 4 * (threadIdx.x + k * nt);
    if (i < n) {
      if (v[k].vec) {
        const int b = (uint32_t)i / (uint32_t)a.len;
        v[k].nb0 = nb[b];
        v[k].nb1 = nb[v[k].turn < 4 ? b + 1 : b];
      }
      tokens_run<F>(a, v[k], i, n, nb, scale, acc);
    }
  }
  block_sums(acc, sm);
  if (threadIdx.x == 0) policy_out(a, acc, tot[0], tot[1]);
}

bool policy_is_small(int64_t seqs, int64_t len) { return seqs <= POL_SMALL_SEQS && seqs * len <= POL_SMALL_TOKENS; }

// ------------------------------------------------------------------ preference loss
constexpr int PREF_SUMS = 6, PREF_SMALL_ROWS = 512, PREF_SMALL_TOKENS = 8192, PREF_ROWS_PAIRS = 512;

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

// A pair from its rows' sums and counts: its loss and rewards; its terms go to acc, and cw and cl receive the rows'
// token gradients apart from the mean's 1 / pairs.
struct PairOut { float loss, rw, rl; };
__device__ __forceinline__ PairOut pref_pair(const PreferenceArgs& a, double sw, int nw, double sl, int nl,
                                             double (&acc)[PREF_SUMS], double& cw, double& cl) {
  cw = cl = 0.0;
  if (nw == 0 || nl == 0) return {0.f, 0.f, 0.f};
  if (a.normalize) sw /= nw, sl /= nl;
  const double delta = sw - sl, h = a.beta * delta - a.margin, e = a.smoothing;
  double loss, dh;
  if (a.kind == 0) {
    const double x = exp(-fabs(h)), soft = log1p(x);  // log(1 + e^-|h|)
    // a side without a weight adds nothing, also where it is infinite
    loss = (e < 1.0 ? (1.0 - e) * (soft + fmax(-h, 0.0)) : 0.0) + (e > 0.0 ? e * (soft + fmax(h, 0.0)) : 0.0);
    if (h != h) loss = h;
    // -(1 - e) sigmoid(-h) + e sigmoid(h), of which e - sigmoid(-h) would leave nothing at e = 1 and h far below 0
    const double near = 1.0 / (1.0 + x), far = x * near;  // sigmoid(|h|), sigmoid(-|h|)
    dh = h >= 0.0 ? e * near - (1.0 - e) * far : e * far - (1.0 - e) * near;
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
  acc[0] += loss;
  acc[1] += delta > 0.0 ? 1.0 : 0.0;
  acc[2] += a.beta * sw;
  acc[3] += a.beta * sl;
  acc[4] += h;
  acc[5] += 1.0;
  return {(float)loss, (float)(a.beta * sw), (float)(a.beta * sl)};
}
__device__ __forceinline__ void pair_out(const PreferenceArgs& a, int64_t p, const PairOut& o) {
  a.pair_loss[p] = o.loss;
  a.rewards[p] = o.rw;
  a.rewards[p + a.pairs] = o.rl;
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
    for (int64_t row = threadIdx.x / WAVE; row < 2 * a.pairs; row += blockDim.x / WAVE) {
      double s = 0.0;
      int64_t n = 0;
      for (int k = threadIdx.x % WAVE; k < cps; k += WAVE) s += sums[row * cps + k], n += ns[row * cps + k];
      s = wave_total(s);
      n = wave_total(n);
      if (threadIdx.x % WAVE == 0) sums[row * cps] = s, ns[row * cps] = (int)n;
    }
    __threadfence_block();
    __syncthreads();
  }
  double acc[PREF_SUMS] = {}, cw0 = 0.0, cl0 = 0.0;
  const int nt = blockDim.x;
  for (int64_t p = threadIdx.x; p < a.pairs; p += nt) {
    const int64_t w = p * cps, l = (p + a.pairs) * cps;
    double cw, cl;
    pair_out(a, p, pref_pair(a, sums[w], ns[w], sums[l], ns[l], acc, cw, cl));
    if (p < nt) {  // a thread's first pair stays in its registers
      cw0 = cw, cl0 = cl;
    } else {
      raw[p] = cw;
      raw[p + a.pairs] = cl;
    }
  }
  block_sums(acc, sm);
  if (threadIdx.x == 0) {
    pref_out(a, acc);
    scale = pref_scale(a, acc[5]) * a.grad_scale;
  }
  __syncthreads();
  for (int64_t p = threadIdx.x; p < a.pairs; p += nt) {
    coef[p] = (float)((p < nt ? cw0 : raw[p]) * scale);
    coef[p + a.pairs] = (float)((p < nt ? cl0 : raw[p + a.pairs]) * scale);
  }
}

__global__ void __launch_bounds__(256) pref_tokens(PreferenceArgs a, const float* coef) {
  pref_walk(a, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256, [&](int64_t r) { return coef[r]; });
}

// The same two steps in one launch, for few pairs of one chunk a row: block b < 2 pairs cpr takes a share of row
// b / cpr and finds the row's coefficient itself, the last block writes the pairs' outputs.  Against the two
// launches, us in all: 256 pairs of 4096 11.4 : 14.1, 1000 of 1000 17.2 : 15.1 (every block counts the pairs).
__global__ void __launch_bounds__(256) pref_rows(PreferenceArgs a, int cpr, int64_t per, const double* sums,
                                                 const int* ns) {
  __shared__ double sm[PREF_SUMS * 16];
  __shared__ int live[4];
  const int P = (int)a.pairs;
  if ((int64_t)blockIdx.x == 2 * a.pairs * cpr) {
    double acc[PREF_SUMS] = {}, cw, cl;
    for (int p = threadIdx.x; p < P; p += 256) {
      const PairOut o = pref_pair(a, sums[p], ns[p], sums[p + P], ns[p + P], acc, cw, cl);
      pair_out(a, p, o);
    }
    block_sums(acc, sm);
    if (threadIdx.x == 0) pref_out(a, acc);
    return;
  }
  const int64_t row = blockIdx.x / cpr, p = row < P ? row : row - P;
  const int64_t t0 = (blockIdx.x % cpr) * per, t1 = min(a.len, t0 + per), o = row * a.len;
  int n = 0;
  for (int q = threadIdx.x; q < P; q += 256) n += ns[q] > 0 && ns[q + P] > 0;
  double acc[PREF_SUMS] = {}, cw, cl;
  pref_pair(a, sums[p], ns[p], sums[p + P], ns[p + P], acc, cw, cl);
  n = wave_total(n);
  if (threadIdx.x % WAVE == 0) live[threadIdx.x / WAVE] = n;
  __syncthreads();
  n = live[0] + live[1] + live[2] + live[3];
  const float c = (float)((row < P ? cw : cl) * (pref_scale(a, n) * a.grad_scale));
  for (int64_t t = t0 + 4 * threadIdx.x; t < t1; t += 1024) {
    if (t + 4 <= t1) {
      const u8x4u on = *reinterpret_cast<const u8x4u*>(a.mask + o + t);
      *reinterpret_cast<f32x4u*>(a.dlogp + o + t) =
          f32x4u{on[0] ? c : 0.f, on[1] ? c : 0.f, on[2] ? c : 0.f, on[3] ? c : 0.f};
    } else {
      for (int64_t u = t; u < t1; ++u) a.dlogp[o + u] = a.mask[o + u] ? c : 0.f;
    }
  }
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
    s = wave_total(s);
    n = wave_total(n);
    if (threadIdx.x % WAVE == 0) sum[row] = s, cnt[row] = n;
  }
  __syncthreads();
  double acc[PREF_SUMS] = {}, cw = 0.0, cl = 0.0;
  const int p = threadIdx.x;
  if (p < (int)a.pairs) pair_out(a, p, pref_pair(a, sum[p], cnt[p], sum[p + a.pairs], cnt[p + a.pairs], acc, cw, cl));
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
         up256(sizeof(int)) + up256((size_t)seqs * sizeof(int));
}

namespace {
template <int F>
void policy_launch(const PolicyArgs& a, void* ws, hipStream_t st) {
  if (policy_is_small(a.seqs, a.len)) {
    const int n = (int)(a.seqs * a.len);
    policy_small<F><<<1, (int)std::min<int64_t>(1024, cdiv(std::max(n, 1), 256) * 64), 0, st>>>(a);
    return;
  }
  double* sums = (double*)ws;
  int64_t* totals = (int64_t*)((char*)ws + up256(POL_BLOCKS * POL_SUMS * sizeof(double)));
  int* done = (int*)((char*)totals + up256(POL_COUNT_BLOCKS * 2 * sizeof(int64_t)));
  int* nb = (int*)((char*)done + up256(sizeof(int)));
  const int nblk = (int)std::min<int64_t>(POL_BLOCKS, cdiv(a.seqs * a.len, 1024));
  const int64_t groups = a.len >= 16384 ? a.seqs : cdiv(a.seqs, 16);
  const int ncount = (int)std::min<int64_t>(POL_COUNT_BLOCKS, groups);
  policy_count<<<ncount, 1024, 0, st>>>(a, nb, totals, done);
  if (nblk <= POL_LAST_BLOCKS) {
    policy_tokens<F><<<nblk, 256, 0, st>>>(a, nb, totals, ncount, sums, done);
    return;
  }
  policy_tokens<F><<<nblk, 256, 0, st>>>(a, nb, totals, ncount, sums, nullptr);
  policy_finish<<<1, 256, 0, st>>>(a, totals, ncount, sums, nblk);
}
template <int... Fs>
void policy_dispatch(int f, const PolicyArgs& a, void* ws, hipStream_t st, std::integer_sequence<int, Fs...>) {
  (void)((f == Fs && (policy_launch<Fs>(a, ws, st), true)) || ...);
}
}  // namespace

void launch_policy_loss(const PolicyArgs& a, void* ws, hipStream_t st) {
  const int f = (a.ref ? POL_REF : 0) | (a.ent ? POL_ENT : 0) | (a.per_token ? POL_TOKEN_ADV : 0) |
                (a.seq_mean ? POL_SEQ_MEAN : 0);
  policy_dispatch(f, a, ws, st, std::make_integer_sequence<int, 16>{});
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
  const int64_t cpr = std::max<int64_t>(1, cdiv(a.len, 4096));
  if (cps == 1 && a.pairs <= PREF_ROWS_PAIRS && (int64_t)n * cpr < 1 << 20) {
    pref_rows<<<(unsigned)(n * cpr + 1), 256, 0, st>>>(a, (int)cpr, 4096, sums, ns);
    return;
  }
  // a thread per pair, or a wave per row where chunks are joined
  const int nt = (int)std::min<int64_t>(1024, cps > 1 ? 2 * a.pairs * 64 : cdiv(a.pairs, 64) * 64);
  pref_pairs<<<1, nt, 0, st>>>(a, cps, sums, ns, raw, coef);
  if (a.len > 0)
    pref_tokens<<<(unsigned)std::min<int64_t>(1 << 16, cdiv((int64_t)n * a.len, 1024)), 256, 0, st>>>(a, coef);
}
