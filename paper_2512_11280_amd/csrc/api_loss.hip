// C ABI of libadasd: log-probabilities and losses over vocabulary rows (argument validation, workspace carving, enqueue).
#include <cmath>

#include "internal.h"

namespace adasd {

namespace {
constexpr size_t kSliceBytes = (kXchgWords + kResultWords) * sizeof(uint64_t);
constexpr size_t kPerPosition = sizeof(LossCoef) + 2 * sizeof(double) + sizeof(float) + sizeof(uint64_t) + kSlicesPerPosition * kSliceBytes;
constexpr size_t kLossFixed = (size_t)kMaxLossSlices * kSliceBytes + (32 + kAddsUp) * sizeof(int32_t) +
                              kAddsUp * sizeof(double) + 8 * 256;
}  // namespace

// Room for the positions' arrays, and for the hand-off words of their slices at their longest (k_loss_join with a reference: 2048 vectors a
// slice; longer rows than 64 of them have none).
size_t loss_workspace_bytes_for(int64_t positions, int V, int dt) {
  const int epv = dt == ADASD_BF16 ? 8 : 4;
  const int64_t nv = ((int64_t)V + epv - 1) / epv, S = (nv + 8 * kBlock - 1) / (8 * kBlock);
  const int64_t slices = S > 1 && S <= kMaxSplit ? S * positions - kMaxLossSlices : 0, more = (slices + kSlicesPerPosition - 1) / kSlicesPerPosition;
  return kLossFixed + (size_t)((more > positions ? more : positions) + 1) * kPerPosition;
}

// (Offsets depend on the size of the workspace alone: a call of another shape finds words and counters where the one before left them, at
// zero.)
size_t loss_workspace_layout(size_t ws_bytes, LossWorkspace* ws, void* base) {
  if (ws_bytes <= kLossFixed) return 0;
  const size_t cap = (ws_bytes - kLossFixed) / kPerPosition;
  char* p = static_cast<char*>(base);
  auto take = [&](size_t bytes) {
    char* at = p;
    p += (bytes + 255) / 256 * 256;
    return at;
  };
  ws->slices = kMaxLossSlices + (int64_t)cap * kSlicesPerPosition;
  ws->sets = reinterpret_cast<uint64_t*>(take(cap * sizeof(uint64_t)));
  ws->done = reinterpret_cast<int32_t*>(take((32 + kAddsUp) * sizeof(int32_t)));
  ws->fresh = reinterpret_cast<double*>(take(kAddsUp * sizeof(double)));
  ws->xchg = reinterpret_cast<uint64_t*>(take((size_t)ws->slices * kSliceBytes));
  ws->coef = reinterpret_cast<LossCoef*>(take(cap * sizeof(LossCoef)));
  ws->term = reinterpret_cast<double*>(take(cap * sizeof(double)));
  ws->pair = reinterpret_cast<double*>(take(cap * sizeof(double)));
  ws->seq = reinterpret_cast<float*>(take(cap * sizeof(float)));
  return cap;
}

namespace {

bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_loss_shape(int B, int T, int V, int dt) {
  if (B < 0 || T < 0 || V < 1) return ADASD_ERR_INVALID_ARG;
  if (dt != ADASD_F32 && dt != ADASD_BF16) return ADASD_ERR_INVALID_ARG;
  if (V > ADASD_MAX_V || (int64_t)B * T > ADASD_MAX_ROWS) return ADASD_ERR_CAPACITY;
  return ADASD_OK;
}

// Whether the rows of a [B, T, V] array with these strides lie apart, in either order, and where the last one ends (elements).
bool rows_apart(int64_t B, int64_t T, int64_t V, int64_t& seq, int64_t& pos, int64_t* end) {
  if (B == 1) seq = T * V;                  // (strides that no address uses)
  if (T == 1) pos = V;
  constexpr int64_t kFar = (int64_t)1 << 40;   // (B * T is at most 2^20)
  if (seq < V || pos < V || seq > kFar || pos > kFar) return false;
  const int64_t last = (B - 1) * seq + (T - 1) * pos + V;
  *end = last;
  return B == 1 || T == 1 || seq >= (T - 1) * pos + V || pos >= (B - 1) * seq + V;
}
bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uintptr_t)b_bytes && y < x + (uintptr_t)a_bytes;
}

// Returns ADASD_OK with the rows and the workspace filled in (n == 0: nothing to read), or a negative error code.
int loss_setup(const adasd_rows* a, const void* ref, int64_t r_seq, int64_t r_pos, bool loss, LossRows* rows, LossWorkspace* ws) {
  if (!a) return ADASD_ERR_INVALID_ARG;
  int rc = check_loss_shape(a->B, a->T, a->V, (int)a->dt);
  if (rc) return rc;
  if (loss ? a->active != nullptr : a->weight != nullptr) return ADASD_ERR_INVALID_ARG;
  LossRows m{};
  m.T = a->T;
  m.V = a->V;
  m.n = a->B * a->T;
  if (m.n > 0) {
    if (!a->logits || !a->tokens) return ADASD_ERR_INVALID_ARG;
    int64_t z_seq = a->seq_stride, z_pos = a->pos_stride, z_end = 0, g_seq = a->d_seq_stride, g_pos = a->d_pos_stride, g_end = 0, r_end = 0;
    if (!rows_apart(a->B, a->T, a->V, z_seq, z_pos, &z_end)) return ADASD_ERR_INVALID_ARG;
    if (ref && !rows_apart(a->B, a->T, a->V, r_seq, r_pos, &r_end)) return ADASD_ERR_INVALID_ARG;
    const int64_t es = a->dt == ADASD_BF16 ? 2 : 4;
    if (a->dlogits) {
      if (!rows_apart(a->B, a->T, a->V, g_seq, g_pos, &g_end)) return ADASD_ERR_INVALID_ARG;
      const bool in_place = a->dlogits == a->logits && g_seq == z_seq && g_pos == z_pos;
      if (!in_place && overlap(a->dlogits, g_end * es, a->logits, z_end * es)) return ADASD_ERR_INVALID_ARG;
      if (ref && overlap(a->dlogits, g_end * es, ref, r_end * es)) return ADASD_ERR_INVALID_ARG;
    }
    if (!aligned_to(a->logits, es) || !aligned_to(ref, es) || !aligned_to(a->dlogits, es) || !aligned_to(a->tokens, 4) ||
        !aligned_to(a->weight, 4) || !aligned_to(a->logprob, 4) || !aligned_to(a->entropy, 4) || !aligned_to(a->status, 4))
      return ADASD_ERR_MISALIGNED;
    m.z = RowPlace{(char*)a->logits, z_seq, z_pos};
    m.ref = RowPlace{(char*)ref, r_seq, r_pos};
    m.g = RowPlace{(char*)a->dlogits, g_seq, g_pos};
    m.tokens = a->tokens;
    m.weight = a->weight;
    m.active = a->active;
    m.logprob = a->logprob;
    m.entropy = a->entropy;
    m.status = a->status;
    if (!a->workspace) return ADASD_ERR_WORKSPACE;
    if (!aligned_to(a->workspace, 256)) return ADASD_ERR_MISALIGNED;
    if (loss_workspace_layout(a->ws_bytes, ws, a->workspace) < (size_t)m.n) return ADASD_ERR_WORKSPACE;
  }
  *rows = m;
  return ADASD_OK;
}
int run(const LossRows& rows, int dt, const LossTerm& f, const LossWorkspace& ws, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  Scope sc(7, st);
  return launch_loss(rows, dt, f, ws, st) == hipSuccess ? ADASD_OK : ADASD_ERR_HIP;
}

}  // namespace

}  // namespace adasd

using namespace adasd;

extern "C" {

int adasd_loss_workspace_bytes(int B, int T, int V, adasd_dtype dt, size_t* bytes) {
  if (!bytes) return ADASD_ERR_INVALID_ARG;
  const int rc = check_loss_shape(B, T, V, (int)dt);
  if (rc) return rc;
  *bytes = loss_workspace_bytes_for((int64_t)B * T, V, (int)dt);
  return ADASD_OK;
}

static int token_logprob(const adasd_rows* a, void* stream, WordWait wait) {
  LossRows rows;
  LossWorkspace ws{};
  const int rc = loss_setup(a, nullptr, 0, 0, false, &rows, &ws);
  if (rc) return rc;
  if (rows.n == 0) return ADASD_OK;
  rows.g = RowPlace{};
  LossTerm f{};
  f.kind = kLogprob;
  f.wait = wait;
  return run(rows, (int)a->dt, f, ws, stream);
}

int adasd_token_logprob(const adasd_rows* a, void* stream) { return token_logprob(a, stream, kWaits); }

// For the tests, not part of the ABI: the same where records that are there count as not there, and where the last slice gives its
// rows up at once.
int adasd_test_logprob_unarrived(const adasd_rows* a, void* stream) { return token_logprob(a, stream, kNotThere); }
int adasd_test_logprob_given_up(const adasd_rows* a, void* stream) { return token_logprob(a, stream, kGivesUp); }

static int token_logprob_grad(const adasd_rows* a, const float* dlogprob, const float* dentropy, void* stream, WordWait wait) {
  LossRows rows;
  LossWorkspace ws{};
  const int rc = loss_setup(a, nullptr, 0, 0, false, &rows, &ws);
  if (rc) return rc;
  if (rows.n == 0) return ADASD_OK;
  if (!dlogprob || !a->dlogits) return ADASD_ERR_INVALID_ARG;
  if (!aligned_to(dlogprob, 4) || !aligned_to(dentropy, 4)) return ADASD_ERR_MISALIGNED;
  LossTerm f{};
  f.wait = wait;
  f.kind = kLogprob;
  f.dlogprob = dlogprob;
  f.dentropy = dentropy;
  return run(rows, (int)a->dt, f, ws, stream);
}

int adasd_token_logprob_grad(const adasd_rows* a, const float* dlogprob, const float* dentropy, void* stream) {
  return token_logprob_grad(a, dlogprob, dentropy, stream, kWaits);
}

// For the tests, as above: the slices form the others' sums from the logits whatever has been sent, or do not wait for them.
int adasd_test_logprob_grad_unarrived(const adasd_rows* a, const float* dlogprob, const float* dentropy, void* stream) {
  return token_logprob_grad(a, dlogprob, dentropy, stream, kNotThere);
}
int adasd_test_logprob_grad_given_up(const adasd_rows* a, const float* dlogprob, const float* dentropy, void* stream) {
  return token_logprob_grad(a, dlogprob, dentropy, stream, kGivesUp);
}

static int policy_loss(const adasd_rows* a, const adasd_policy_args* p, void* stream, WordWait wait) {
  if (!a || !p) return ADASD_ERR_INVALID_ARG;
  if (p->ref_logits && p->ref_logprob) return ADASD_ERR_INVALID_ARG;
  if (p->adv_per_seq != 0 && p->adv_per_seq != 1) return ADASD_ERR_INVALID_ARG;
  if (!(p->clip_low >= 0.f && p->clip_low <= 1.f) || !(p->clip_high >= 0.f)) return ADASD_ERR_INVALID_ARG;
  if (!std::isfinite(p->kl_coef) || !std::isfinite(p->entropy_coef)) return ADASD_ERR_INVALID_ARG;
  LossRows rows;
  LossWorkspace ws{};
  const int rc = loss_setup(a, p->ref_logits, p->r_seq_stride, p->r_pos_stride, true, &rows, &ws);
  if (rc) return rc;
  if (!p->loss || (rows.n > 0 && !p->advantage)) return ADASD_ERR_INVALID_ARG;
  if (!aligned_to(p->loss, 4) || !aligned_to(p->advantage, 4) || !aligned_to(p->old_logprob, 4) || !aligned_to(p->ref_logprob, 4) ||
      !aligned_to(p->grad_scale, 4) || !aligned_to(p->token_loss, 4) || !aligned_to(p->kl, 4))
    return ADASD_ERR_MISALIGNED;
  LossTerm f{};
  f.wait = wait;
  f.kind = kPolicy;
  f.advantage = p->advantage;
  f.adv_per_seq = p->adv_per_seq;
  f.old_logprob = p->old_logprob;
  f.ref_logprob = p->ref_logprob;
  f.grad_scale = p->grad_scale;
  f.clip_low = p->clip_low;
  f.clip_high = p->clip_high;
  f.kl_coef = p->ref_logprob || p->ref_logits ? p->kl_coef : 0.f;
  f.entropy_coef = p->entropy_coef;
  f.loss = p->loss;
  f.token_loss = p->token_loss;
  f.kl = p->kl;
  return run(rows, (int)a->dt, f, ws, stream);
}

int adasd_policy_loss(const adasd_rows* a, const adasd_policy_args* p, void* stream) { return policy_loss(a, p, stream, kWaits); }

// For the tests, as above.
int adasd_test_policy_loss_unarrived(const adasd_rows* a, const adasd_policy_args* p, void* stream) { return policy_loss(a, p, stream, kNotThere); }
int adasd_test_policy_loss_given_up(const adasd_rows* a, const adasd_policy_args* p, void* stream) { return policy_loss(a, p, stream, kGivesUp); }

int adasd_preference_loss(const adasd_rows* a, const adasd_preference_args* p, void* stream) {
  if (!a || !p) return ADASD_ERR_INVALID_ARG;
  if (p->kind < 0 || p->kind > 2 || (a->B & 1)) return ADASD_ERR_INVALID_ARG;
  if (!(p->beta > 0.f) || !std::isfinite(p->beta) || !std::isfinite(p->margin)) return ADASD_ERR_INVALID_ARG;
  if (!(p->label_smoothing >= 0.f && p->label_smoothing <= 1.f) || (p->kind != 0 && p->label_smoothing != 0.f)) return ADASD_ERR_INVALID_ARG;
  LossRows rows;
  LossWorkspace ws{};
  const int rc = loss_setup(a, nullptr, 0, 0, true, &rows, &ws);
  if (rc) return rc;
  if (!p->loss) return ADASD_ERR_INVALID_ARG;
  if (a->B > 0 && a->T == 0) return ADASD_ERR_INVALID_ARG;          // pairs without positions: nothing to prefer
  if (!aligned_to(p->loss, 4) || !aligned_to(p->ref_logprob, 4) || !aligned_to(p->pair_weight, 4) || !aligned_to(p->grad_scale, 4) ||
      !aligned_to(p->pair_loss, 4) || !aligned_to(p->pair_margin, 4) || !aligned_to(p->score, 4))
    return ADASD_ERR_MISALIGNED;
  LossTerm f{};
  f.wait = kWaits;
  f.kind = kPreference;
  f.pair_kind = p->kind;
  f.P = a->B / 2;
  f.beta = p->beta;
  f.margin = p->margin;
  f.smoothing = p->label_smoothing;
  f.ref_logprob = p->ref_logprob;
  f.pair_weight = p->pair_weight;
  f.grad_scale = p->grad_scale;
  f.loss = p->loss;
  f.pair_loss = p->pair_loss;
  f.pair_margin = p->pair_margin;
  f.score = p->score;
  return run(rows, (int)a->dt, f, ws, stream);
}

}  // extern "C"
