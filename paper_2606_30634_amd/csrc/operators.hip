// C entries of the stateless log-probability and loss operators: argument checks, then the launchers of
// logprob.hip and losses.hip.
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

}  // extern "C"
