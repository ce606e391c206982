// Log-probabilities of given tokens under rows of logits, and their gradient in the logits.
//
// For a row x of V logits, s = inv_temperature > 0, m = max x and S = sum exp(s (x_j - m)):
//   log p_j = s (x_j - m) - log S,   H = log S - sum p_j s (x_j - m)   (both terms >= 0: no cancellation)
// with S held as S - 1, the sum without the maximum's own term.
//   dx_j = s (g (1[j = t] - p_j) - h p_j (log p_j + H))   for upstream g = dlogp, h = dentropy.
// Everything is taken relative to m: x_j - m is exact where it matters, so logits of any magnitude
// lose nothing, and log p_t = s (x_t - m) - log S is small where p_t is near 1.  Exponentials are base 2
// with c = s log2(e); sums are fp32.
//
// What a row may hold: -inf adds nothing; the running maximum starts at the lowest finite value, so a row
// of only -inf ends with S = 0, S - 1 = -1 (told apart from one of lowest finite values, which is uniform); a NaN or
// +inf makes the row NaN through S.
#include "common.h"
#include "kernels.h"
#include <algorithm>
#include <cfloat>

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float TINY_T = -1e30f;  // a finite stand-in for -inf where it meets a zero factor

// 16 bytes of elements at any element alignment (8 bf16, 4 fp32); N of them, of either type
template <typename T> constexpr int VE = 16 / (int)sizeof(T);
template <typename T, int N>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[N]) {
  typedef T raw __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  const raw r = __builtin_nontemporal_load(reinterpret_cast<const raw*>(p));
#pragma unroll
  for (int q = 0; q < N; ++q) v[q] = to_f32(r[q]);
}
template <typename T, int N>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[N]) {
  typedef T raw __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  raw r;
#pragma unroll
  for (int q = 0; q < N; ++q) r[q] = from_f32<T>(v[q]);
  __builtin_nontemporal_store(r, reinterpret_cast<raw*>(p));
}

// Statistics of a part of a row: its maximum and the sums but for the maximum's own 1, so that they keep their bits
// where it is nearly all of the row (log p is then the logarithm of 1 plus them).  Of no logit, or only -inf: s = -1.
typedef RowPart Part;
__device__ __forceinline__ Part part_empty() { return {-FLT_MAX, -1.f, 0.f}; }

__device__ __forceinline__ void part_merge(Part& a, Part b, float c) {
  const bool up = b.m > a.m;
  const Part hi{up ? b.m : a.m, up ? b.s : a.s, up ? b.w : a.w}, lo{up ? a.m : b.m, up ? a.s : b.s, up ? a.w : b.w};
  // (an empty part's shift is -inf or NaN: it has nothing to move)
  const float d = fmaxf((lo.m - hi.m) * c, TINY_T), k = __builtin_amdgcn_exp2f(d), s = 1.f + lo.s;
  a = {hi.m, hi.s + k * s, hi.w + k * (lo.w + d * s)};
}
// The same while it runs: the logits at the maximum are counted apart.
struct Running { float m, s, w, n; };
__device__ __forceinline__ Part part_of(const Running& a) { return {a.m, a.s + (a.n - 1.f), a.w}; }
template <int N>
__device__ __forceinline__ void part_add(Running& a, const float (&v)[N], float c) {
  float mx = v[0];
#pragma unroll
  for (int q = 1; q < N; ++q) mx = fmaxf(mx, v[q]);
  if (mx > a.m) {
    const float d = fmaxf((a.m - mx) * c, TINY_T), k = __builtin_amdgcn_exp2f(d), s = a.s + a.n;
    a.w = k * (a.w + d * s);
    a.s = k * s;
    a.m = mx;
    a.n = 0.f;
  }
  a.n += (float)N;
#pragma unroll
  for (int q = 0; q < N; ++q) {
    const float t = (v[q] - a.m) * c, e = __builtin_amdgcn_exp2f(t);
    const float below = __builtin_amdgcn_fmed3f(t * -1e38f, 0.f, 1.f);  // 0 at the maximum, else 1
    a.n -= below;
    a.s += e * below;
    a.w += e * fmaxf(t, TINY_T);
  }
}
template <int LANES>
__device__ __forceinline__ void part_lanes(Part& a, float c) {  // the group's; lane 0's is the one to use
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    const Part b{__shfl_xor(a.m, o, WAVE), __shfl_xor(a.s, o, WAVE), __shfl_xor(a.w, o, WAVE)};
    part_merge(a, b, c);
  }
}

// What a row's statistics say about its target (x_t its logit).  s (x_t - m) by s itself: as a multiple of c it took
// three roundings for one, and a target at the lowest finite value overflowed.
__device__ __forceinline__ void row_finish(const Part& a, float xt, float inv_temp, int64_t row, float* logp, float* ent,
                                           float* stats) {
  // log(1 + s): of the rounded sum, and what its rounding left, which is exact
  const float u = 1.f + a.s, ls = logf(u) + (a.s - (u - 1.f)) * __builtin_amdgcn_rcpf(u);
  const bool none = a.s == -1.f;  // every logit -inf: no distribution
  logp[row] = none ? -INFINITY : (xt - a.m) * inv_temp - ls;
  if (ent) ent[row] = none ? 0.f : ls - a.w / u * LN2;
  if (stats) {
    stats[2 * row] = none ? -INFINITY : a.m;
    stats[2 * row + 1] = none ? 0.f : ls;
  }
}
__device__ __forceinline__ void row_ignored(int64_t row, float* logp, float* ent, float* stats) {
  logp[row] = 0.f;
  if (ent) ent[row] = 0.f;
  if (stats) stats[2 * row] = 0.f, stats[2 * row + 1] = 0.f;
}

// One row (or one of nsplit equal parts of it) per group of NT threads of a block; a block holds RPB groups.  One pass:
// the maximum and both sums as they run, rescaled where a 16-byte vector raises the maximum; what stands at the maximum
// is counted instead.
// Bound: memory, each logit read once, past the caches (8192 x 49152 fp32, a quarter of the rows ignored: 182 us,
// 6.6 TB/s, where a streaming copy reaches 6.3; with cached loads 212); 14 vector operations a logit are 0.45 of that.
// Two of them leave the maximum out of the sum: fp32 as fast without, bf16 51 : 55 us (4096 x 32000) and 512 logits
// a row 37 : 40 (60000 fp32), against a log p of 1e-4 to one part in 1000.
template <typename T, int NT, int RPB>
__global__ void __launch_bounds__(NT * RPB) logprob_rows(int64_t rows, int V, const T* __restrict__ x, int64_t ld,
                                                         const int32_t* __restrict__ tg, float inv_temp, int nsplit,
                                                         int per, Part* __restrict__ parts, float* __restrict__ logp,
                                                         float* __restrict__ ent, float* __restrict__ stats) {
  constexpr int NW = NT / WAVE, E = VE<T>, U = 32 / E;
  static_assert(NW == 1 || RPB == 1, "groups of one wave, or one group per block");
  __shared__ Part sm[NW];
  const float c = inv_temp * LOG2E;
  const int tid = threadIdx.x % NT;
  const int64_t items = rows * nsplit;
  for (int64_t it = (int64_t)blockIdx.x * RPB + threadIdx.x / NT; it < items; it += (int64_t)gridDim.x * RPB) {
    const int64_t row = it / nsplit;
    const int sp = (int)(it % nsplit), t = tg[row];
    if (t < 0 || t >= V) {
      if (nsplit == 1 && tid == 0) row_ignored(row, logp, ent, stats);
      continue;
    }
    const T* z = x + row * ld + (int64_t)sp * per;
    const int n = max(0, min(per, V - sp * per)), nv = n / E;
    Running run{-FLT_MAX, 0.f, 0.f, 0.f};
    int j = tid;
    for (; j + (U - 1) * NT < nv; j += U * NT) {
      float v[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u) load_vec(z + (int64_t)(j + u * NT) * E, v[u]);
#pragma unroll
      for (int u = 0; u < U; ++u) part_add(run, v[u], c);
    }
    for (; j < nv; j += NT) {
      float v[E];
      load_vec(z + (int64_t)j * E, v);
      part_add(run, v, c);
    }
    if (tid < n - nv * E) {
      const float v[1] = {to_f32(z[nv * E + tid])};
      part_add(run, v, c);
    }
    Part a = part_of(run);
    part_lanes<WAVE>(a, c);
    if constexpr (NW > 1) {
      __syncthreads();  // the row before has been read
      if (tid % WAVE == 0) sm[tid / WAVE] = a;
      __syncthreads();
      if (tid < WAVE) {
        a = sm[tid % NW];
        part_lanes<NW>(a, c);
      }
    }
    if (tid == 0) {
      if (nsplit > 1) parts[it] = a;
      else row_finish(a, to_f32(x[row * ld + t]), inv_temp, row, logp, ent, stats);
    }
  }
}

// Joins the nsplit <= 64 parts of every row, a wave per row (2.2 us for one).
template <typename T>
__global__ void __launch_bounds__(256) logprob_join(int64_t rows, int V, const T* __restrict__ x, int64_t ld,
                                                    const int32_t* __restrict__ tg, float inv_temp, int nsplit,
                                                    const Part* __restrict__ parts, float* __restrict__ logp,
                                                    float* __restrict__ ent, float* __restrict__ stats) {
  const float c = inv_temp * LOG2E;
  const int lane = threadIdx.x % WAVE;
  for (int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE; row < rows; row += (int64_t)gridDim.x * 4) {
    const int t = tg[row];
    if (t < 0 || t >= V) {
      if (lane == 0) row_ignored(row, logp, ent, stats);
      continue;
    }
    Part a = lane < nsplit ? parts[row * nsplit + lane] : part_empty();
    part_lanes<WAVE>(a, c);
    if (lane == 0) row_finish(a, to_f32(x[row * ld + t]), inv_temp, row, logp, ent, stats);
  }
}

// The gradient, element by element: a wave takes U x 64 x 16 bytes of consecutive logits of a row.  A row
// without a target, without a distribution or with zero upstream gradients gets zeros and is not read.
// zero_to > V: the columns [V, zero_to) get zeros.  dx may be x (same type and rows): a lane writes only
// what it has read.
// Bound: memory, one read and one write past the caches (4096 x 128256 bf16, a quarter of the rows without a gradient:
// 295 us, 6.2 TB/s; 999 x 32001 fp32 to bf16 with an entropy term 30 us, 6.0).  Two vectors a lane: 4096 x 128256 with
// 4 of them 319 us, with 1 294 but 39 for the other.
constexpr int BWD_U = 2;
template <typename T, typename OutT>
__global__ void __launch_bounds__(256) logprob_bwd(int64_t rows, int V, const T* x, int64_t ld,
                                                   const int32_t* __restrict__ tg, const float* __restrict__ stats,
                                                   const float* __restrict__ ent, const float* __restrict__ dlogp,
                                                   const float* __restrict__ dent, float s, OutT* dx, int64_t ldo,
                                                   int zero_to) {
  constexpr int U = BWD_U, E = VE<T>, CH = U * E * WAVE;
  const int lane = threadIdx.x % WAVE, W = max(V, zero_to);
  const int64_t per_row = (W + CH - 1) / CH, items = rows * per_row;
  const int64_t w0 = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  for (int64_t it = w0; it < items; it += (int64_t)gridDim.x * 4) {
    const int64_t row = it / per_row;
    const int j0 = (int)(it % per_row) * CH;
    const int t = tg[row];
    const float m = stats[2 * row], l2 = stats[2 * row + 1] * LOG2E, c = s * LOG2E;
    const bool on = t >= 0 && t < V && m != -INFINITY;
    const float g = on ? dlogp[row] * s : 0.f, h = on && dent ? dent[row] * s : 0.f, H = h != 0.f ? ent[row] : 0.f;
    const T* z = x + row * ld;
    OutT* o = dx + row * ldo;
    if (g == 0.f && h == 0.f) {
      const float zero[E] = {};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int j = j0 + (u * WAVE + lane) * E;
        if (j + E <= W) store_vec(o + j, zero);
        else
          for (int q = j; q < W; ++q) o[q] = from_f32<OutT>(0.f);
      }
      continue;
    }
    // without an entropy gradient an element is -g p; the target's is written apart, after its wave's stores
    // (1 - p_t is -(e^lp - 1), which keeps its bits where p_t is near 1); where p is 0, log p may be -inf or h log p past
    // the type
    auto grad = [&](float v) {
      const float q = (v - m) * c - l2, p = __builtin_amdgcn_exp2f(q);
      return h == 0.f ? -g * p : p == 0.f ? 0.f : -p * (g + h * (q * LN2 + H));
    };
    const bool mine = t >= j0 && t < j0 + CH;
    float dt = 0.f;
    if (mine) {
      const float q = (to_f32(z[t]) - m) * c - l2;
      dt = -g * expm1f(q * LN2);
      const float p = __builtin_amdgcn_exp2f(q);
      if (h != 0.f && p != 0.f) dt -= p * h * (q * LN2 + H);
    }
    if (j0 + CH <= V) {
      float v[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u) load_vec(z + j0 + (u * WAVE + lane) * E, v[u]);
      if (h == 0.f) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int q = 0; q < E; ++q) v[u][q] = -g * __builtin_amdgcn_exp2f((v[u][q] - m) * c - l2);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int q = 0; q < E; ++q) v[u][q] = grad(v[u][q]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) store_vec(o + j0 + (u * WAVE + lane) * E, v[u]);
    } else {
#pragma unroll 1
      for (int u = 0; u < U; ++u) {
        const int j = j0 + (u * WAVE + lane) * E;
        if (j + E <= V) {
          float v[E];
          load_vec(z + j, v);
#pragma unroll
          for (int q = 0; q < E; ++q) v[q] = grad(v[q]);
          store_vec(o + j, v);
        } else {
          for (int q = j; q < min(j + E, W); ++q) o[q] = from_f32<OutT>(q >= V ? 0.f : grad(to_f32(z[q])));
        }
      }
    }
    if (mine && lane == (t - j0) / E % WAVE) o[t] = from_f32<OutT>(dt);  // the lane that stored around it
  }
}

// Parts of a row, for the chip to have 512 blocks of at least 8192 logits.  Without : with parts, us: bf16 V 128256, 1 row
// 15.5 : 6.4, 8 rows 15.8 : 6.7; fp32 V 32000, 64 rows 11.4 : 8.9, V 128256 29 : 15.4; towards 1024 blocks instead, fp32
// V 49152, 500 rows 22.3 against 19.
int row_splits(int64_t rows, int64_t V) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({64, V / 8192, 512 / std::max<int64_t>(rows, 1)}));
}

constexpr int64_t GRID = 1 << 20;  // blocks of a launch at most; the kernels walk their rows

template <typename T>
void logprob_t(int64_t rows, int V, const void* x, int64_t ld, const int32_t* tg, float s, float* logp, float* ent,
               float* stats, void* ws, hipStream_t st) {
  const int ns = row_splits(rows, V);
  const int per = (int)(cdiv(cdiv(V, ns), 8) * 8);
  const T* z = (const T*)x;
  Part* parts = (Part*)ws;
  // A wave per row up to 24 KiB of logits where there are rows for the chip's waves, no exchange between
  // waves then (16384 rows, a wave : a block, us: bf16 V 4096 29 : 46, 8192 49 : 61, 16000 95 : 109; fp32 V 4096 45 : 56,
  // 6000 67 : 73, 8192 86 : 81; 2048 rows, bf16 V 6000 10.7 : 9.8)
  if (V <= 2048 || (rows >= 1024 && (int64_t)V * sizeof(T) <= 24576))
    logprob_rows<T, 64, 4><<<(unsigned)std::min(GRID, cdiv(rows * ns, 4)), 256, 0, st>>>(
        rows, V, z, ld, tg, s, ns, per, parts, logp, ent, stats);
  else
    logprob_rows<T, 256, 1><<<(unsigned)std::min(GRID, rows * ns), 256, 0, st>>>(rows, V, z, ld, tg, s, ns, per,
                                                                                  parts, logp, ent, stats);
  if (ns > 1)
    logprob_join<T><<<(unsigned)std::min(GRID, cdiv(rows, 4)), 256, 0, st>>>(rows, V, z, ld, tg, s, ns, parts, logp,
                                                                              ent, stats);
}

template <typename T, typename OutT>
void logprob_bwd_t(int64_t rows, int V, const void* x, int64_t ld, const int32_t* tg, const float* stats,
                   const float* ent, const float* dlogp, const float* dent, float s, void* dx, int64_t ldo,
                   int zero_to, hipStream_t st) {
  const int64_t waves = rows * cdiv(std::max(V, zero_to), BWD_U * VE<T> * WAVE);
  logprob_bwd<T, OutT><<<(unsigned)std::min(GRID, cdiv(waves, 4)), 256, 0, st>>>(
      rows, V, (const T*)x, ld, tg, stats, ent, dlogp, dent, s, (OutT*)dx, ldo, zero_to);
}

}  // namespace

size_t logprob_ws_bytes(int64_t rows, int64_t vocab) {
  const int ns = row_splits(rows, vocab);
  return ns > 1 ? (size_t)rows * ns * sizeof(Part) : 0;
}

void launch_logprob(bool bf, int64_t rows, int vocab, const void* logits, int64_t ld, const int32_t* targets,
                    float inv_temp, float* logp, float* ent, float* stats, void* ws, hipStream_t st) {
  if (rows <= 0) return;
  if (bf) logprob_t<bf16>(rows, vocab, logits, ld, targets, inv_temp, logp, ent, stats, ws, st);
  else logprob_t<float>(rows, vocab, logits, ld, targets, inv_temp, logp, ent, stats, ws, st);
}

void launch_logprob_bwd(bool bf, int64_t rows, int vocab, const void* logits, int64_t ld, const int32_t* targets,
                        const float* stats, const float* ent, const float* dlogp, const float* dent, float inv_temp,
                        bool out_bf, void* dlogits, int64_t ldo, int zero_to, hipStream_t st) {
  if (rows <= 0) return;
#define B_(T, O) \
  logprob_bwd_t<T, O>(rows, vocab, logits, ld, targets, stats, ent, dlogp, dent, inv_temp, dlogits, ldo, zero_to, st)
  if (bf && out_bf) B_(bf16, bf16);
  else if (bf) B_(bf16, float);
  else if (out_bf) B_(float, bf16);
  else B_(float, float);
#undef B_
}

// ------------------------------------------------------------------ from hidden states
namespace {

constexpr int64_t HEAD_ROWS = 16384;  // rows of one fused product: bounds its parts' memory

// Packing: the rows whose target is in the vocabulary, in order.  pos[r] is a row's place among them (-1: it has none),
// live[0] their number.  One block; a wave takes a run of rows, 64 at a time, as masks of the lanes that count.
__global__ void __launch_bounds__(1024) pack_rows(int rows, int V, const int32_t* __restrict__ tg, int32_t* __restrict__ pos,
                                                  int32_t* __restrict__ live) {
  __shared__ int total[16];
  constexpr int STEPS = HEAD_ROWS / 1024;
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, per = (rows + 1023) / 1024;
  const int r0 = wave * per * WAVE + lane;
  int32_t t[STEPS];
#pragma unroll
  for (int k = 0; k < STEPS; ++k) t[k] = k < per && r0 + k * WAVE < rows ? tg[r0 + k * WAVE] : -1;
  uint64_t m[STEPS];
  int n = 0;
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    m[k] = __ballot(t[k] >= 0 && t[k] < V);
    n += __popcll(m[k]);
  }
  if (lane == 0) total[wave] = n;
  __syncthreads();
  int at = 0, all = 0;
  for (int w = 0; w < 16; ++w) at += w < wave ? total[w] : 0, all += total[w];
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const bool on = m[k] >> lane & 1;
    if (k < per && r0 + k * WAVE < rows) pos[r0 + k * WAVE] = on ? at + __popcll(m[k] & ((1ull << lane) - 1)) : -1;
    at += __popcll(m[k]);
  }
  if (threadIdx.x == 0) live[0] = all;
}

// Copies the rows of x (16-byte chunks) that have a place there, with their targets, and clears the rows after them
// up to a multiple of 256; nothing to do where every row has one.
__global__ void __launch_bounds__(256) gather_rows(int rows, int chunks, const u32x4* __restrict__ x, int64_t ldx,
                                                   const int32_t* __restrict__ tg, const int32_t* __restrict__ pos,
                                                   const int32_t* __restrict__ live, u32x4* __restrict__ xp,
                                                   int32_t* __restrict__ tp) {
  const int n = live[0], r = blockIdx.x * 4 + threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
  if (n == rows) return;
  if (r < rows) {
    const int p = pos[r];
    if (p < 0) return;
    for (int k = lane; k < chunks; k += WAVE) xp[(int64_t)p * chunks + k] = x[r * ldx + k];
    if (lane == 0) tp[p] = tg[r];
  } else {
    const int p = n + r - rows;
    if (p >= (n + 255) / 256 * 256) return;
    for (int k = lane; k < chunks; k += WAVE) xp[(int64_t)p * chunks + k] = u32x4{0, 0, 0, 0};
    if (lane == 0) tp[p] = -1;
  }
}

// Joins the panels of every row (parts[p rows + row], or of its place where rows are packed): RJ rows per block of
// 256, 256 / RJ threads on each.  384 panels of 8192 rows: 10 us for 38 MB.
template <int RJ>
__global__ void __launch_bounds__(256) panel_join(int64_t rows, int V, int panels, const int32_t* __restrict__ tg,
                                                  float inv_temp, const Part* __restrict__ parts, const float* __restrict__ xt,
                                                  const int32_t* __restrict__ pos, const int32_t* __restrict__ live,
                                                  float* __restrict__ logp, float* __restrict__ ent,
                                                  float* __restrict__ stats) {
  constexpr int TR = 256 / RJ;  // threads per row
  __shared__ Part sm[4 * RJ];
  const float c = inv_temp * LOG2E;
  const int r = threadIdx.x % RJ, k = threadIdx.x / RJ;
  const int64_t row = (int64_t)blockIdx.x * RJ + r;
  const int t = row < rows ? tg[row] : -1;
  const bool on = t >= 0 && t < V;
  const int64_t at = !on ? 0 : pos && *live < rows ? pos[row] : row;
  Part a = part_empty();
  if (on) {
    int p = k;
    for (; p + 3 * TR < panels; p += 4 * TR) {
      Part b[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) b[u] = parts[(int64_t)(p + u * TR) * rows + at];
#pragma unroll
      for (int u = 0; u < 4; ++u) part_merge(a, b[u], c);
    }
    for (; p < panels; p += TR) part_merge(a, parts[(int64_t)p * rows + at], c);
  }
  // a wave holds 64 / RJ threads of each of the block's rows
  constexpr int LR = WAVE / RJ;
#pragma unroll
  for (int o = LR / 2 * RJ; o >= RJ; o >>= 1) {
    const Part b{__shfl_xor(a.m, o, WAVE), __shfl_xor(a.s, o, WAVE), __shfl_xor(a.w, o, WAVE)};
    part_merge(a, b, c);
  }
  if (threadIdx.x % WAVE < RJ) sm[threadIdx.x / WAVE * RJ + r] = a;
  __syncthreads();
  if (k == 0) {
    for (int w = 1; w < 4; ++w) part_merge(a, sm[w * RJ + r], c);
  }
  if (k == 0 && row < rows) {
    if (on) row_finish(a, xt[at], inv_temp, row, logp, ent, stats);
    else row_ignored(row, logp, ent, stats);
  }
}

size_t align256(size_t v) { return (v + 255) / 256 * 256; }

// Rows of fp32 logits held at once where they go through memory: within `bytes`, whole 128s if more than that; at most
// 2^20, since the product's row tiles of 64 are its grid's second dimension, which takes 65536
int64_t head_chunk(int64_t rows, int64_t vocab, int64_t bytes) {
  const int64_t r = std::min<int64_t>(bytes / (4 * vocab), 1 << 20);
  return std::max<int64_t>(1, std::min(rows, r > 128 ? r / 128 * 128 : r));
}
// Logits of heads of unaligned rows, a chunk at a time: the products' kernels for such rows, whose rate bounds it (1024 x
// 32000 x 769: fp32 617 us, 82 TFLOP/s; bf16 881 us on the vector units; 768 instead, 403 and 62)
constexpr int64_t HEAD_ODD_BYTES = 32 << 20;

// Whether a product is worth packing its rows for: 8 us of kernels against 250 us or more (at 1.2 PFLOP/s in bf16, a
// tenth of it in fp32), in which rows without a target would take their share.  With no such rows, a tenth, half of
// them, us: 8192 x 49152 x 2048 bf16 1405, 1299, 712 (without packing some 1395 each), 4096 x 32000 x 768 fp32 1558, 1411,
// 831; 333 x 32001 x 512 fp32, below this, 118 each.
bool head_packs(bool bf, int64_t n, int64_t vocab, int64_t d) {
  return n > 256 && (double)n * vocab * d >= (bf ? 1.5e11 : 1.5e10);
}
struct HeadLayout { size_t xt, parts, pos, tp, xp, total; };  // byte offsets in the workspace
HeadLayout head_layout(bool bf, int64_t n, int64_t vocab, int64_t d) {
  HeadLayout l{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += align256(bytes);
    return o;
  };
  l.xt = take((size_t)n * 4);
  l.parts = take((size_t)cdiv(vocab, gemm_rowstat_panel(bf, n, vocab, d)) * n * sizeof(Part));
  if (head_packs(bf, n, vocab, d)) {
    const int64_t np = cdiv(n, 256) * 256;
    l.pos = take((size_t)(n + 1) * 4);  // and the count
    l.tp = take((size_t)np * 4);
    l.xp = take((size_t)np * d * (bf ? 2 : 4));
  }
  l.total = at;
  return l;
}
// The logits of r rows, then the parts of the rows of the call's chunks: the last chunk has fewer rows, which are split
// further and can have more parts than the others (V 128256: 65 rows 455 parts, 64 rows 512).
size_t chunked_bytes(int64_t rows, int64_t r, int64_t vocab) {
  const int64_t last = (rows - 1) % r + 1;
  return align256((size_t)(r * vocab * 4)) + std::max(logprob_ws_bytes(r, vocab), logprob_ws_bytes(last, vocab));
}

}  // namespace

size_t head_logprob_ws_bytes(bool bf, int64_t rows, int64_t vocab, int64_t d) {
  const size_t chunked = chunked_bytes(rows, head_chunk(rows, vocab, HEAD_ODD_BYTES), vocab);
  const int64_t first = std::min(rows, HEAD_ROWS), last = (rows - 1) % HEAD_ROWS + 1;
  return std::max({head_layout(bf, first, vocab, d).total, head_layout(bf, last, vocab, d).total, chunked});
}

void launch_head_logprob(bool bf, int64_t rows, int vocab, int d, const void* x, int64_t ldx, const void* w,
                         int64_t ldw, const int32_t* targets, float inv_temp, float* logp, float* ent, float* stats,
                         void* ws, hipStream_t st) {
  if (rows <= 0) return;
  GemmArgs g{};
  g.N = vocab; g.K = d;
  g.lda = (int)ldx; g.a_kmajor = true;
  g.B = w; g.ldb = (int)ldw; g.b_kmajor = true;
  // the rows' statistics in the product's epilogue, a part per panel of columns
  bool fused = true;
  for (int64_t r0 = 0; fused && r0 < rows; r0 += HEAD_ROWS) {
    const int64_t n = std::min(HEAD_ROWS, rows - r0);
    g.M = (int)n;
    g.A = (const char*)x + r0 * ldx * (bf ? 2 : 4);
    g.stat_c = inv_temp * LOG2E;
    g.targets = targets + r0;
    const HeadLayout l = head_layout(bf, n, vocab, d);
    char* w0 = (char*)ws;
    g.stat_xt = (float*)(w0 + l.xt);
    g.stats = (Part*)(w0 + l.parts);
    g.stat_ld = n;
    int32_t* pos = nullptr;
    g.live = nullptr;
    if (!gemm_rowstat_takes(bf, g)) {  // all chunks or none: they differ in n alone
      fused = false;
      break;
    }
    if (head_packs(bf, n, vocab, d)) {
      pos = (int32_t*)(w0 + l.pos);
      int32_t* tp = (int32_t*)(w0 + l.tp);
      g.live = pos + n;
      g.A2 = w0 + l.xp; g.lda2 = d;
      g.targets2 = tp;
      const int per = bf ? 8 : 4;  // elements per 16 bytes
      pack_rows<<<1, 1024, 0, st>>>((int)n, vocab, g.targets, pos, pos + n);
      gather_rows<<<(unsigned)cdiv(n + 255, 4), 256, 0, st>>>((int)n, d / per, (const u32x4*)g.A, ldx / per, g.targets,
                                                              pos, pos + n, (u32x4*)(w0 + l.xp), tp);
    }
    gemm_rowstat(bf, g, st);
    const int panels = (int)cdiv(vocab, gemm_rowstat_panel(bf, n, vocab, d));
    float* e = ent ? ent + r0 : nullptr;
    float* q = stats ? stats + 2 * r0 : nullptr;
    if (n >= 256)
      panel_join<16><<<(unsigned)cdiv(n, 16), 256, 0, st>>>(n, vocab, panels, g.targets, inv_temp, g.stats, g.stat_xt, pos,
                                                            g.live, logp + r0, e, q);
    else
      panel_join<1><<<(unsigned)n, 256, 0, st>>>(n, vocab, panels, g.targets, inv_temp, g.stats, g.stat_xt, pos, g.live,
                                                 logp + r0, e, q);
  }
  if (fused) return;
  const int64_t r = head_chunk(rows, vocab, HEAD_ODD_BYTES);
  float* logits = (float*)ws;
  void* parts = (char*)ws + align256((size_t)(r * vocab * 4));
  g.C = logits; g.ldc = vocab; g.out_f32 = true; g.beta = 0.f;
  for (int64_t r0 = 0; r0 < rows; r0 += r) {
    const int64_t n = std::min(r, rows - r0);
    g.M = (int)n;
    g.A = (const char*)x + r0 * ldx * (bf ? 2 : 4);
    launch_gemm(bf, g, st);
    launch_logprob(false, n, vocab, logits, vocab, targets + r0, inv_temp, logp + r0, ent ? ent + r0 : nullptr,
                   stats ? stats + 2 * r0 : nullptr, parts, st);
  }
}
