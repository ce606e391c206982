// C entries of the stateless operators: argument checks, then the launchers of logprob.hip, losses.hip,
// attention_ranges.hip and dropout.hip.
#include <algorithm>
#include <cmath>

#include "../../include/asyncstage.h"
#include "common.h"
#include "kernels.h"

namespace {

int bad(const char* msg) { return set_error(STAGE_EINVAL, msg); }

int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? STAGE_OK : set_error(STAGE_EHIP, hipGetErrorString(e));
}

// nullptr, or what is wrong with a workspace of `need` bytes
const char* check_ws(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return nullptr;
  if (!ws || bytes < need) return "workspace smaller than the operator's workspace_bytes";
  if ((uintptr_t)ws % 256) return "workspace must be 256-byte aligned";
  return nullptr;
}

bool off(const void* p, size_t align) { return (uintptr_t)p % align != 0; }

// [a, a + na) and [b, b + nb) share a byte
bool meet(const void* a, size_t na, const void* b, size_t nb) {
  const char *x = (const char*)a, *y = (const char*)b;
  return a && b && na && nb && x < y + nb && y < x + na;
}

bool row_sizes(int64_t rows, int64_t vocab) {
  return rows >= 0 && rows < ((int64_t)1 << 31) && vocab >= 1 && vocab <= (1 << 24);
}
bool head_sizes(int64_t rows, int64_t vocab, int64_t d) {
  return row_sizes(rows, vocab) && d >= 1 && d <= (1 << 20);
}
bool grid_sizes(int64_t n, int64_t most, int64_t len) {  // n sequences of len
  return n >= 0 && n <= most && len >= 0 && len < ((int64_t)1 << 31) && (len == 0 || n < ((int64_t)1 << 40) / len);
}
bool policy_sizes(int64_t seqs, int64_t len) { return grid_sizes(seqs, ((int64_t)1 << 31) - 1, len); }
bool preference_sizes(int64_t pairs, int64_t len) {
  return pairs >= 0 && pairs <= (1 << 24) && grid_sizes(2 * pairs, 1 << 25, len);
}

const char* check_rows(int64_t rows, int64_t vocab, const int32_t* targets, float s, const float* logp,
                       const float* entropy, const float* stats) {
  if (!row_sizes(rows, vocab)) return "rows must be in [0, 2^31), vocab in [1, 2^24]";
  if (!(s > 0.f && s <= 0x1p60f)) return "inv_temperature must be in (0, 2^60]";
  if (rows > 0 && (!targets || !logp)) return "null targets or logp";
  if (off(targets, 4) || off(logp, 4) || off(entropy, 4) || off(stats, 4)) return "arrays must be 4-byte aligned";
  return nullptr;
}

// nullptr, or what is wrong with the sizes, ranges and numbers of an attention call
const char* check_attention(const attention_params_t* p, RangeArgs& a) {
  constexpr int64_t most = (int64_t)1 << 30;
  if (!p) return "null attention parameters";
  if (p->batch < 0 || p->batch > (1 << 24) || p->queries < 0 || p->queries > most || p->keys < 0 || p->keys > most)
    return "batch must be in [0, 2^24], queries and keys in [0, 2^30]";
  if (p->kv_heads < 1 || p->heads < p->kv_heads || p->heads > 4096 || p->heads % p->kv_heads)
    return "kv_heads must be at least 1 and divide heads (at most 4096)";
  if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128) return "head_dim must be 32, 64 or 128";
  if (!(p->scale >= 0x1p-60f && p->scale <= 0x1p60f)) return "scale must be in [2^-60, 2^60]";
  if (p->softcap != 0.f && !(p->softcap >= 0x1p-60f && p->softcap <= 0x1p100f && p->scale / p->softcap >= 0x1p-126f))
    return "softcap must be 0 (none) or in [2^-60, 2^100], scale / softcap at least 2^-126";
  if ((p->key_start != nullptr) != (p->key_end != nullptr)) return "key_start and key_end come together";
  if (off(p->key_start, 4) || off(p->key_end, 4) || off(p->q_start, 4) || off(p->slopes, 4))
    return "arrays must be 4-byte aligned";
  const int64_t blocks = ((p->queries + 31) / 32 + 1) * p->heads + ((p->keys + 31) / 32 + 1) * p->kv_heads;
  if (p->batch * blocks >= ((int64_t)1 << 25)) return "batch x (queries heads + keys kv_heads) is too large";
  a = RangeArgs{};
  a.B = (int)p->batch; a.Sq = (int)p->queries; a.Sk = (int)p->keys;
  a.Hq = p->heads; a.Hkv = p->kv_heads; a.hd = p->head_dim;
  a.key_start = p->key_start; a.key_end = p->key_end; a.q_start = p->q_start; a.slopes = p->slopes;
  a.scale = p->scale; a.cap = p->softcap;
  return nullptr;
}

// nullptr, or what is wrong with rows [batch, rows, heads, head_dim] at p with strides s (elements)
const char* check_rows_of(const void* p, const int64_t* s, int64_t rows, bool bf, HeadRows& out) {
  const int64_t per = bf ? 8 : 4, most = (int64_t)1 << 40;
  if (rows > 0 && !p) return "null rows";
  if (off(p, 16)) return "rows must be 16-byte aligned";
  for (int k = 0; k < 3; ++k)
    if (s[k] < 0 || s[k] > most || s[k] % per) return "strides must be whole 16 bytes, none negative, at most 2^40";
  if (s[1] > (1 << 24)) return "a row stride must be at most 2^24 elements";
  out = HeadRows{const_cast<void*>(p), s[0], s[2], (int)s[1]};
  return nullptr;
}
// what a kernel writes must not meet itself: sorted by stride, each dimension steps over the ones within it
bool apart(const int64_t* s, int64_t batch, int64_t rows, int64_t heads, int64_t hd) {
  int64_t st[3] = {s[0], s[1], s[2]}, n[3] = {batch, rows, heads};
  int64_t within = hd;
  bool used[3] = {};
  for (int k = 0; k < 3; ++k) {
    int best = -1;
    for (int j = 0; j < 3; ++j)
      if (!used[j] && n[j] > 1 && (best < 0 || st[j] < st[best])) best = j;
    if (best < 0) break;
    used[best] = true;
    if (st[best] < within) return false;
    within += st[best] * (n[best] - 1);
  }
  return true;
}
// Rows of n sequences, rows and heads (elements between them: s) of hd elements, and whether x and y, whose extents meet,
// share none: for some of the dimensions, of the same strides in both, what the other ones hold of x and of y lies side by
// side, and both together, as one, apart over them.  (Heads of one packed row, single tokens included; heads interleaved one
// by one; slices of a [B, heads, S, hd] tensor.)
struct Layout {
  const void* p;
  const int64_t* s;
  int64_t n[3], hd;
};
bool side_by_side(const Layout& x, const Layout& y, size_t esz) {
  if ((uintptr_t)y.p < (uintptr_t)x.p) return side_by_side(y, x, esz);
  const int64_t at = ((const char*)y.p - (const char*)x.p) / (int64_t)esz;  // both multiples of 16 bytes
  for (int outer = 0; outer < 8; ++outer) {
    int64_t wx = x.hd, wy = y.hd, st[3] = {}, n[3] = {1, 1, 1};
    bool same = true;
    for (int k = 0; k < 3; ++k) {
      if (outer >> k & 1) {
        same &= x.n[k] <= 1 || y.n[k] <= 1 || x.s[k] == y.s[k];
        n[k] = std::max(x.n[k], y.n[k]);
        st[k] = x.n[k] > 1 ? x.s[k] : y.s[k];  // the stride of a dimension of one is never used
      } else {
        wx += (x.n[k] - 1) * x.s[k];
        wy += (y.n[k] - 1) * y.s[k];
      }
    }
    if (same && wx <= at && apart(st, n[0], n[1], n[2], at + wy)) return true;
  }
  return false;
}
// bytes that rows span
size_t extent(const int64_t* s, int64_t batch, int64_t rows, int64_t heads, int64_t hd, size_t esz) {
  if (batch == 0 || rows == 0) return 0;
  return ((batch - 1) * s[0] + (rows - 1) * s[1] + (heads - 1) * s[2] + hd) * esz;
}

}  // namespace

extern "C" {

size_t token_logprob_workspace_bytes(int64_t rows, int64_t vocab) {
  return row_sizes(rows, vocab) ? logprob_ws_bytes(rows, vocab) : 0;
}

int token_logprob(int64_t rows, int64_t vocab, const void* logits, int64_t ld, int32_t logits_bf16,
                  const int32_t* targets, float inv_temperature, float* logp, float* entropy, float* stats,
                  void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (const char* m = check_rows(rows, vocab, targets, inv_temperature, logp, entropy, stats)) return bad(m);
  if (ld < vocab || ld > (1 << 28)) return bad("ld must be in [vocab, 2^28]");
  if (rows == 0) return STAGE_OK;
  if (!logits || off(logits, logits_bf16 ? 2 : 4)) return bad("logits null or not aligned to their type");
  if (const char* m = check_ws(workspace, workspace_bytes, logprob_ws_bytes(rows, vocab))) return bad(m);
  launch_logprob(logits_bf16 != 0, rows, (int)vocab, logits, ld, targets, inv_temperature, logp, entropy, stats,
                 workspace, (hipStream_t)hip_stream);
  return launched();
}

int token_logprob_backward(int64_t rows, int64_t vocab, const void* logits, int64_t ld, int32_t logits_bf16,
                           const int32_t* targets, const float* stats, const float* entropy, const float* dlogp,
                           const float* dentropy, float inv_temperature, void* dlogits, int64_t ld_out,
                           int32_t out_bf16, void* hip_stream) {
  if (const char* m = check_rows(rows, vocab, targets, inv_temperature, dlogp, entropy, stats)) return bad(m);
  if (ld < vocab || ld_out < vocab || ld > (1 << 28) || ld_out > (1 << 28))
    return bad("ld and ld_out must be in [vocab, 2^28]");
  if (dentropy && !entropy) return bad("dentropy needs the forward's entropy");
  if (rows == 0) return STAGE_OK;
  if (!logits || !dlogits || !stats) return bad("null logits, dlogits or stats");
  const size_t ei = logits_bf16 ? 2 : 4, eo = out_bf16 ? 2 : 4;
  if (off(logits, ei) || off(dlogits, eo) || off(dentropy, 4)) return bad("arrays must be aligned to their type");
  const bool same = logits == dlogits && ei == eo && ld == ld_out;
  if (!same && meet(logits, ((rows - 1) * ld + vocab) * ei, dlogits, ((rows - 1) * ld_out + vocab) * eo))
    return bad("dlogits may be logits itself (same type and ld) but not overlap it otherwise");
  launch_logprob_bwd(logits_bf16 != 0, rows, (int)vocab, logits, ld, targets, stats, entropy, dlogp, dentropy,
                     inv_temperature, out_bf16 != 0, dlogits, ld_out, 0, (hipStream_t)hip_stream);
  return launched();
}

size_t head_logprob_workspace_bytes(int64_t rows, int64_t vocab, int64_t d, int32_t is_bf16) {
  return rows > 0 && head_sizes(rows, vocab, d) ? head_logprob_ws_bytes(is_bf16 != 0, rows, vocab, d) : 0;
}

int head_logprob(int64_t rows, int64_t vocab, int64_t d, const void* x, int64_t ldx, const void* w, int64_t ldw,
                 int32_t is_bf16, const int32_t* targets, float inv_temperature, float* logp, float* entropy,
                 float* stats, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (const char* m = check_rows(rows, vocab, targets, inv_temperature, logp, entropy, stats)) return bad(m);
  if (!head_sizes(rows, vocab, d)) return bad("d must be in [1, 2^20]");
  if (ldx < d || ldw < d || ldx > (1 << 24) || ldw > (1 << 24)) return bad("ldx and ldw must be in [d, 2^24]");
  if (rows == 0) return STAGE_OK;
  const size_t e = is_bf16 ? 2 : 4;
  if (!x || !w || off(x, e) || off(w, e)) return bad("x or w null or not aligned to their type");
  if (const char* m = check_ws(workspace, workspace_bytes, head_logprob_ws_bytes(is_bf16 != 0, rows, vocab, d)))
    return bad(m);
  launch_head_logprob(is_bf16 != 0, rows, (int)vocab, (int)d, x, ldx, w, ldw, targets, inv_temperature, logp, entropy,
                      stats, workspace, (hipStream_t)hip_stream);
  return launched();
}

size_t policy_loss_workspace_bytes(int64_t seqs, int64_t len) {
  return policy_sizes(seqs, len) ? policy_ws_bytes(seqs, len) : 0;
}

int policy_loss(int64_t seqs, int64_t len, const float* logp, const float* old_logp, const float* ref_logp,
                const float* entropy, const float* advantages, const uint8_t* mask, const policy_hparams_t* hp,
                float* loss, float* dlogp, float* dentropy, float* metrics, int64_t* counts, void* workspace,
                size_t workspace_bytes, void* hip_stream) {
  if (!policy_sizes(seqs, len)) return bad("seqs and len must be in [0, 2^31), seqs len below 2^40");
  if (!hp) return bad("null hparams");
  if (!(hp->clip_low >= 0.f && hp->clip_low <= 1.f) || !(hp->clip_high >= 0.f) || !std::isfinite(hp->clip_high))
    return bad("clip_low must be in [0, 1], clip_high >= 0 and finite");
  if (!std::isfinite(hp->kl_coef) || !std::isfinite(hp->entropy_coef) || !std::isfinite(hp->grad_scale))
    return bad("kl_coef, entropy_coef and grad_scale must be finite");
  if (!(hp->norm >= 0.0) || !std::isfinite(hp->norm)) return bad("norm must be >= 0 and finite");
  if (hp->reduction != 0 && hp->reduction != 1) return bad("reduction must be 0 (tokens) or 1 (sequences)");
  const int64_t n = seqs * len;  // with no tokens, every array may be null
  if (n > 0 && hp->kl_coef != 0.f && !ref_logp) return bad("kl_coef needs ref_logp");
  if (n > 0 && hp->entropy_coef != 0.f && !entropy) return bad("entropy_coef needs entropy");
  if (n > 0 && (entropy != nullptr) != (dentropy != nullptr)) return bad("entropy and dentropy come together");
  if (!loss || !metrics || !counts) return bad("null loss, metrics or counts");
  if (n > 0 && (!logp || !old_logp || !advantages || !mask || !dlogp)) return bad("null array");
  if (off(logp, 4) || off(old_logp, 4) || off(ref_logp, 4) || off(entropy, 4) || off(advantages, 4) || off(loss, 4) ||
      off(dlogp, 4) || off(dentropy, 4) || off(metrics, 4) || off(counts, 8))
    return bad("arrays must be aligned to their type");
  for (const float* o : {dlogp, dentropy}) {
    for (const float* i : {logp, old_logp, ref_logp, entropy})
      if (meet(i, 4 * n, o, 4 * n)) return bad("a gradient may not overlap an input");
    if (meet(mask, n, o, 4 * n) || meet(advantages, 4 * (hp->advantage_per_token ? n : seqs), o, 4 * n))
      return bad("a gradient may not overlap an input");
  }
  if (meet(dlogp, 4 * n, dentropy, 4 * n)) return bad("dlogp and dentropy overlap");
  if (const char* m = check_ws(workspace, workspace_bytes, policy_ws_bytes(seqs, len))) return bad(m);
  PolicyArgs a{};
  a.seqs = n ? seqs : 0; a.len = n ? len : 0;
  a.logp = logp; a.old = old_logp; a.ref = ref_logp; a.ent = entropy; a.adv = advantages; a.mask = mask;
  a.per_token = hp->advantage_per_token != 0; a.seq_mean = hp->reduction;
  a.clip_low = hp->clip_low; a.clip_high = hp->clip_high; a.kl_coef = hp->kl_coef; a.ent_coef = hp->entropy_coef;
  a.log_lo = std::log1p(-(double)hp->clip_low); a.log_hi = std::log1p((double)hp->clip_high);
  a.norm = hp->norm; a.grad_scale = hp->grad_scale;
  a.loss = loss; a.dlogp = dlogp; a.dent = dentropy; a.metrics = metrics; a.counts = counts;
  launch_policy_loss(a, workspace, (hipStream_t)hip_stream);
  return launched();
}

size_t preference_loss_workspace_bytes(int64_t pairs, int64_t len) {
  return preference_sizes(pairs, len) ? preference_ws_bytes(pairs, len) : 0;
}

int preference_loss(int64_t pairs, int64_t len, const float* logp, const float* ref_logp, const uint8_t* mask,
                    const preference_hparams_t* hp, float* loss, float* dlogp, float* pair_loss, float* rewards,
                    float* metrics, int64_t* counts, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!preference_sizes(pairs, len)) return bad("pairs must be in [0, 2^24], len in [0, 2^31), 2 pairs len below 2^40");
  if (!hp) return bad("null hparams");
  if (hp->kind < 0 || hp->kind > 2) return bad("kind must be 0 (sigmoid), 1 (hinge) or 2 (square)");
  if (!(hp->beta > 0.f) || !std::isfinite(hp->beta)) return bad("beta must be positive and finite");
  if (!(hp->label_smoothing >= 0.f && hp->label_smoothing <= 1.f)) return bad("label_smoothing must be in [0, 1]");
  if (hp->label_smoothing != 0.f && hp->kind != 0) return bad("label_smoothing belongs to kind 0");
  if (!std::isfinite(hp->margin) || !std::isfinite(hp->grad_scale)) return bad("margin and grad_scale must be finite");
  if (!(hp->norm >= 0.0) || !std::isfinite(hp->norm)) return bad("norm must be >= 0 and finite");
  const int64_t n = 2 * pairs * len;
  if (!loss || !metrics || !counts) return bad("null loss, metrics or counts");
  if (pairs > 0 && (!pair_loss || !rewards)) return bad("null pair_loss or rewards");
  if (n > 0 && (!logp || !mask || !dlogp)) return bad("null array");
  if (off(logp, 4) || off(ref_logp, 4) || off(loss, 4) || off(dlogp, 4) || off(pair_loss, 4) || off(rewards, 4) ||
      off(metrics, 4) || off(counts, 8))
    return bad("arrays must be aligned to their type");
  if (meet(logp, 4 * n, dlogp, 4 * n) || meet(ref_logp, 4 * n, dlogp, 4 * n) || meet(mask, n, dlogp, 4 * n))
    return bad("dlogp may not overlap an input");
  if (const char* m = check_ws(workspace, workspace_bytes, preference_ws_bytes(pairs, len))) return bad(m);
  PreferenceArgs a{};
  a.pairs = pairs; a.len = len; a.logp = logp; a.ref = ref_logp; a.mask = mask;
  a.kind = hp->kind; a.normalize = hp->length_normalize != 0;
  a.beta = hp->beta; a.smoothing = hp->label_smoothing; a.margin = hp->margin;
  a.norm = hp->norm; a.grad_scale = hp->grad_scale;
  a.loss = loss; a.dlogp = dlogp; a.pair_loss = pair_loss; a.rewards = rewards; a.metrics = metrics; a.counts = counts;
  launch_preference_loss(a, workspace, (hipStream_t)hip_stream);
  return launched();
}

int attention_key_ranges(int64_t batch, int64_t length, const int32_t* documents, const uint8_t* prefix,
                         int32_t* key_start, int32_t* key_end, void* hip_stream) {
  if (batch < 0 || length < 0 || length > ((int64_t)1 << 30) || batch > ((int64_t)1 << 24) ||
      batch * ((length + 2047) / 2048) >= ((int64_t)1 << 31))
    return bad("batch must be in [0, 2^24], length in [0, 2^30], batch length / 2048 below 2^31");
  if (batch * length == 0) return STAGE_OK;
  if (!documents || !key_start || !key_end) return bad("null documents, key_start or key_end");
  if (off(documents, 4) || off(key_start, 4) || off(key_end, 4)) return bad("arrays must be 4-byte aligned");
  const size_t n = (size_t)(batch * length);
  for (const int32_t* o : {key_start, key_end})
    if (meet(documents, 4 * n, o, 4 * n) || meet(prefix, n, o, 4 * n)) return bad("the ranges may not overlap an input");
  if (meet(key_start, 4 * n, key_end, 4 * n)) return bad("key_start and key_end overlap");
  launch_key_ranges(batch, (int)length, documents, prefix, key_start, key_end, (hipStream_t)hip_stream);
  return launched();
}

size_t attention_workspace_bytes(const attention_params_t* p) {
  RangeArgs a;
  if (check_attention(p, a) || a.B == 0 || a.Sq == 0) return 0;
  return range_fwd_ws_bytes(p->is_bf16 != 0, a);
}

int attention_forward(const attention_params_t* p, const void* q, const void* k, const void* v, void* o, float* o_f32,
                      float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  RangeArgs a;
  if (const char* m = check_attention(p, a)) return bad(m);
  const bool bf = p->is_bf16 != 0;
  const size_t esz = bf ? 2 : 4;
  if (const char* m = check_rows_of(q, p->q_strides, a.B * p->queries, bf, a.q)) return bad(m);
  if (const char* m = check_rows_of(k, p->k_strides, a.B * p->keys, bf, a.k)) return bad(m);
  if (const char* m = check_rows_of(v, p->v_strides, a.B * p->keys, bf, a.v)) return bad(m);
  if (a.B == 0 || a.Sq == 0) return STAGE_OK;
  if (!o || !lse) return bad("null o or lse");
  if (off(o, 16) || off(o_f32, 16) || off(lse, 4)) return bad("o and o_f32 must be 16-byte aligned, lse to its type");
  if (o_f32 && !bf) return bad("o_f32 belongs to bf16: an fp32 o is the output itself");
  const size_t n = (size_t)(p->batch * p->queries * a.Hq), eq = extent(p->q_strides, a.B, a.Sq, a.Hq, a.hd, esz),
               ek = extent(p->k_strides, a.B, a.Sk, a.Hkv, a.hd, esz), ev = extent(p->v_strides, a.B, a.Sk, a.Hkv, a.hd, esz);
  struct { const void* p; size_t n; } outs[3] = {{o, n * a.hd * esz}, {o_f32, n * a.hd * 4}, {lse, n * 4}};
  for (int i = 0; i < 3; ++i) {
    if (meet(q, eq, outs[i].p, outs[i].n) || meet(k, ek, outs[i].p, outs[i].n) || meet(v, ev, outs[i].p, outs[i].n))
      return bad("an output may not overlap q, k or v");
    for (int j = 0; j < i; ++j)
      if (meet(outs[j].p, outs[j].n, outs[i].p, outs[i].n)) return bad("the outputs overlap");
  }
  if (range_fwd_blocks(bf, a) > MAX_BLOCKS_256) return bad("batch x queries x heads is too large for a launch");
  if (const char* m = check_ws(workspace, workspace_bytes, range_fwd_ws_bytes(bf, a))) return bad(m);
  a.o = o; a.o32 = o_f32; a.lse = lse;
  launch_range_fwd(bf, a, workspace, (hipStream_t)hip_stream);
  return launched();
}

size_t attention_backward_workspace_bytes(const attention_params_t* p) {
  RangeArgs a;
  if (check_attention(p, a) || a.B == 0) return 0;
  return range_bwd_ws_bytes(p->is_bf16 != 0, a);
}

int attention_backward(const attention_params_t* p, const void* q, const void* k, const void* v, const void* o,
                       const float* lse, const void* dout, const attention_grads_t* g, void* workspace,
                       size_t workspace_bytes, void* hip_stream) {
  RangeArgs a;
  if (const char* m = check_attention(p, a)) return bad(m);
  if (!g) return bad("null gradients");
  const bool bf = p->is_bf16 != 0;
  const size_t esz = bf ? 2 : 4;
  const int64_t nq = a.B * p->queries, nk = a.B * p->keys;
  if (const char* m = check_rows_of(q, p->q_strides, nq, bf, a.q)) return bad(m);
  if (const char* m = check_rows_of(k, p->k_strides, nk, bf, a.k)) return bad(m);
  if (const char* m = check_rows_of(v, p->v_strides, nk, bf, a.v)) return bad(m);
  if (const char* m = check_rows_of(dout, g->dout_strides, nq, bf, a.dout)) return bad(m);
  if (const char* m = check_rows_of(g->dq, g->dq_strides, nq, bf, a.dq)) return bad(m);
  if (const char* m = check_rows_of(g->dk, g->dk_strides, nk, bf, a.dk)) return bad(m);
  if (const char* m = check_rows_of(g->dv, g->dv_strides, nk, bf, a.dv)) return bad(m);
  if (nq + nk == 0) return STAGE_OK;
  HeadRows orows{};
  if (const char* m = check_rows_of(o, g->o_strides, nq, bf && !g->o_is_f32, orows)) return bad(m);
  if (nq > 0 && !lse) return bad("null lse");
  if (off(lse, 4)) return bad("lse must be aligned to its type");
  if (!apart(g->dq_strides, a.B, a.Sq, a.Hq, a.hd) || !apart(g->dk_strides, a.B, a.Sk, a.Hkv, a.hd) ||
      !apart(g->dv_strides, a.B, a.Sk, a.Hkv, a.hd))
    return bad("the rows of a gradient overlap");
  const size_t n = (size_t)nq * a.Hq;
  struct { const void* p; size_t n; } ins[6] = {{q, extent(p->q_strides, a.B, a.Sq, a.Hq, a.hd, esz)},
                                                {k, extent(p->k_strides, a.B, a.Sk, a.Hkv, a.hd, esz)},
                                                {v, extent(p->v_strides, a.B, a.Sk, a.Hkv, a.hd, esz)},
                                                {dout, extent(g->dout_strides, a.B, a.Sq, a.Hq, a.hd, esz)},
                                                {o, extent(g->o_strides, a.B, a.Sq, a.Hq, a.hd, g->o_is_f32 ? 4 : esz)}, {lse, n * 4}},
                                      outs[3] = {{g->dq, extent(g->dq_strides, a.B, a.Sq, a.Hq, a.hd, esz)},
                                                 {g->dk, extent(g->dk_strides, a.B, a.Sk, a.Hkv, a.hd, esz)},
                                                 {g->dv, extent(g->dv_strides, a.B, a.Sk, a.Hkv, a.hd, esz)}};
  for (auto& x : outs)
    for (auto& y : ins)
      if (meet(x.p, x.n, y.p, y.n)) return bad("a gradient may not overlap an input");
  // the three may be interleaved, as the heads of one packed row are
  const Layout lay[3] = {{g->dq, g->dq_strides, {a.B, a.Sq, a.Hq}, a.hd}, {g->dk, g->dk_strides, {a.B, a.Sk, a.Hkv}, a.hd},
                         {g->dv, g->dv_strides, {a.B, a.Sk, a.Hkv}, a.hd}};
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < i; ++j)
      if (meet(outs[j].p, outs[j].n, outs[i].p, outs[i].n) && !side_by_side(lay[j], lay[i], esz))
        return bad("the gradients overlap");
  if (range_bwd_blocks(bf, a) > MAX_BLOCKS_256)
    return bad("batch x (queries x heads x head_dim / 1024 + keys) is too large for a launch of the backward");
  if (const char* m = check_ws(workspace, workspace_bytes, range_bwd_ws_bytes(bf, a))) return bad(m);
  (g->o_is_f32 ? (void*&)a.o32 : a.o) = const_cast<void*>(o);
  a.ob = orows.batch; a.orow = orows.row; a.oh = orows.head;
  a.lse = const_cast<float*>(lse);
  launch_range_bwd(bf, a, workspace, (hipStream_t)hip_stream);
  return launched();
}

int dropout_add(int64_t rows, int64_t cols, const void* x, int64_t ldx, const void* residual, int64_t ldr, void* out,
                int64_t ldo, int32_t is_bf16, double p, uint64_t seed, uint64_t offset, void* hip_stream) {
  constexpr int64_t most = (int64_t)1 << 40;
  if (rows < 0 || cols < 0 || rows > most || cols > most || (cols > 0 && rows > most / cols))
    return bad("rows and cols must not be negative, rows cols at most 2^40");
  if (!(p >= 0.0 && p <= 65535.0 / 65536.0)) return bad("p must be in [0, 1 - 2^-16]");
  if (rows * cols == 0) return STAGE_OK;
  if (ldx < cols || ldo < cols || (residual && ldr < cols) || ldx > most || ldo > most || ldr > most)
    return bad("ldx, ldr and ldo must be in [cols, 2^40]");
  const size_t e = is_bf16 ? 2 : 4;
  if (!x || !out || off(x, e) || off(residual, e) || off(out, e)) return bad("x or out null or not aligned to their type");
  auto span = [&](int64_t ld) { return (size_t)((rows - 1) * ld + cols) * e; };
  if ((x != out || ldx != ldo) && meet(x, span(ldx), out, span(ldo))) return bad("out may be x itself but not overlap it otherwise");
  if ((residual != out || ldr != ldo) && meet(residual, span(ldr), out, span(ldo)))
    return bad("out may be the residual itself but not overlap it otherwise");
  launch_dropout(is_bf16 != 0, DropoutArgs{rows, cols, ldx, ldr, ldo, x, residual, out,
                                           (uint32_t)std::nearbyint(65536.0 * p), seed, offset}, (hipStream_t)hip_stream);
  return launched();
}

}  // extern "C"
