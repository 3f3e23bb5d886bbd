// Log-probabilities of tokens, the clipped policy loss and the preference loss over vocabulary rows, with their gradients.
//
// A gradient row needs the row's normaliser (and entropy, and KL) before its first element, and the preference loss those of whole
// sequences.
//   k_loss_sums  (slices of rows) the sums of each slice (loss_device.h).  One workgroup of a row folds them (hand_off), settles the
//                position: what is reported of it, and the five numbers of its gradient row.  The position that is done last adds up
//                the loss; of a pair's sequences, settles the pair.
//   k_loss_grad  (slices of rows) reads the logits again and forms the gradient.
//   k_loss_fused (a workgroup per row, which stays in registers) both in one, where the gradient needs nothing but its own row.
//   k_loss_pairs, k_loss_total: pairs and the sum of the loss where there are many positions.
// Sums over positions and sequences are in 64 bits and in a fixed order, whoever forms them.
#include "loss_device.h"
#include "sample_device.h"

namespace adasd {

namespace {

using namespace sampling;

// Vectors v0 .. v1 of a row that slice s of S works on.
__device__ __forceinline__ void slice_of(int nv, int s, int S, int& v0, int& v1) {
  const int chunk = slice_vectors(nv, S);
  v0 = min(s * chunk, nv);
  v1 = min(v0 + chunk, nv);
}
template <int DT> __device__ __forceinline__ uint4 load_vec_of(const char* row, int idx, int V) {
  return idx < V / Elem<DT>::per_vec ? load_vec_any(row, idx) : load_last_vec<DT>(row, V);
}
// The reference c of a row: what the logits of its token differ by, if that is a number (any value would do; near the typical
// difference the sums about it cancel least).
template <int DT> __device__ __forceinline__ float ref_shift(const char* row, const char* ref, int x, int V) {
  const int at = x >= 0 && x < V ? x : 0;
  const float d = (load_elem<DT>(row, at) - load_elem<DT>(ref, at)) * kLog2e;
  return fabsf(d) < INFINITY ? d : 0.f;
}

// What the numbers of a position are formed from, asked for ahead of the row.
struct PositionIn {
  float z, weight, a, h, old, ref;      // logit of the token; a: advantage or dlogprob; h: dentropy
  int x;
};
__device__ __forceinline__ PositionIn ask_position(const LossRows& rows, const LossTerm& f, int r, int b) {
  PositionIn in{};
  in.x = rows.tokens[r];
  in.weight = rows.weight ? rows.weight[r] : 1.f;
  if (f.kind == kLogprob) {
    if (f.dlogprob) in.a = f.dlogprob[r];
    if (f.dentropy) in.h = f.dentropy[r];
  } else {
    if (f.kind == kPolicy) in.a = f.advantage[f.adv_per_seq ? b : r];
    if (f.old_logprob) in.old = f.old_logprob[r];
    if (f.ref_logprob) in.ref = f.ref_logprob[r];
  }
  return in;
}
template <int DT> __device__ __forceinline__ void ask_logit(PositionIn& in, const char* row, int V) {
  in.z = load_elem<DT>(row, in.x >= 0 && in.x < V ? in.x : 0);
}

// What is reported of a position (lane 0 writes it), and the numbers of its gradient row, by one wavefront from the sums of the whole row.
template <bool REF>
__device__ __forceinline__ LossCoef settle_position(const LossRows& rows, const LossTerm& f, int r, const PositionIn& in, const LossSums& sums,
                                                    float c, double& term) {
  const int lane = threadIdx.x & 63;
  const bool known = in.x >= 0 && in.x < rows.V;
  const LossRow row = finish_loss_row<REF>(sums, c);
  const double lp = known ? (double)in.z - row.lse : (double)NAN;
  const double w = (double)in.weight;
  double a = 0.0, by_entropy = 0.0, by_kl = 0.0, loss = 0.0, kl = row.kl;
  term = 0.0;
  if (f.kind == kLogprob) {
    a = (double)in.a;
    by_entropy = (double)in.h;
  } else if (f.kind == kPolicy) {
    // one exponential for both ratios: the old policy's in the even lanes, the reference's in the odd ones
    const double grown = expm1_fine(lane & 1 ? (double)in.ref - lp : lp - (double)in.old);
    const double A = (double)in.a, ratio = f.old_logprob ? 1.0 + __shfl(grown, 0) : lp == lp ? 1.0 : lp, grown_ref = __shfl(grown, 1);
    if (A != 0.0) {
      const double free = ratio * A, held = fmin(fmax(ratio, 1.0 - (double)f.clip_low), 1.0 + (double)f.clip_high) * A;
      const bool clipped = held < free;
      loss = -(clipped ? held : free);
      a = clipped ? 0.0 : -free;
    }
    if (f.ref_logprob) {
      kl = grown_ref - ((double)in.ref - lp);
      if (f.kl_coef != 0.f) a -= (double)f.kl_coef * grown_ref;
    }
    if (f.kl_coef != 0.f) loss += (double)f.kl_coef * kl;
    if (f.entropy_coef != 0.f) loss -= (double)f.entropy_coef * row.H;
    term = w * loss;
    const double scale = w * (f.grad_scale ? (double)*f.grad_scale : 1.0);
    a *= scale;
    by_entropy = -scale * (double)f.entropy_coef;
    if (REF) by_kl = scale * (double)f.kl_coef;
  } else {
    term = w * (lp - (f.ref_logprob ? (double)in.ref : 0.0));
    a = w;
  }
  if (lane == 0) {
    if (rows.logprob) rows.logprob[r] = (float)lp;
    if (rows.entropy) rows.entropy[r] = (float)row.H;
    if (rows.status) rows.status[r] = (known ? 0u : (uint32_t)ADASD_ST_BAD_TOKEN) | (row.bad ? (uint32_t)ADASD_ST_NONFINITE : 0u);
    if (f.token_loss) f.token_loss[r] = (float)loss;
    if (f.kl) f.kl[r] = (float)kl;
  }
  // dz_j = a (1[j = x] - p_j) - by_entropy p_j (ln p_j + H) + by_kl p_j (ln p_j - ln q_j - KL)
  LossCoef k{};
  double k0 = -a;
  if (by_entropy != 0.0) {
    k0 -= by_entropy * (row.H - (row.lse - kNat * (double)sums.m));
    k.k1 = (float)(-by_entropy * kNat * row.inv_s);
  }
  if (REF && by_kl != 0.0) {
    k0 += by_kl * (kNat * (double)c - (row.lse - row.lse_ref) - row.kl);
    k.k2 = (float)(by_kl * kNat * row.inv_s);
  }
  k.m = sums.m;
  k.c = c;
  k.a = (float)a;
  k.k0 = k0 == 0.0 ? 0.f : (float)(k0 * row.inv_s);      // (nothing of the row enters a gradient of zeros)
  return k;
}

// The results of a position that does not count.
__device__ __forceinline__ void report_nothing(const LossRows& rows, const LossTerm& f, int r) {
  if (rows.logprob) rows.logprob[r] = 0.f;
  if (rows.entropy) rows.entropy[r] = 0.f;
  if (rows.status) rows.status[r] = 0u;
  if (f.token_loss) f.token_loss[r] = 0.f;
  if (f.kl) f.kl[r] = 0.f;
}

// ---- sums over positions.  One wavefront; the order of the additions is the same whether other workgroups' terms are read in the launch
// that forms them (FRESH) or in a later one.
template <bool FRESH> __device__ __forceinline__ double wave_total(const double* v, int n) {
  const int lane = threadIdx.x & 63;
  double t = 0.0;
  for (int base = 0; base < n; base += 8 * 64) {
    double x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = base + k * 64 + lane;
      x[k] = i < n ? (FRESH ? ld_agent(v + i) : v[i]) : 0.0;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) t += x[k];
  }
  return wave_sum(t);
}

__device__ __forceinline__ double softplus(double v) { return fmax(v, 0.0) + log1p(exp(-fabs(v))); }

// A pair's loss and slope from the terms of its positions, by one wavefront (lane 0 writes).
template <bool FRESH> __device__ __forceinline__ void settle_pair(const LossTerm& f, const LossWorkspace& ws, int i, int T) {
  const int P = f.P;
  const double chosen = wave_total<FRESH>(ws.term + (size_t)i * T, T), rejected = wave_total<FRESH>(ws.term + (size_t)(P + i) * T, T);
  const double beta = (double)f.beta, e = (double)f.smoothing, D = chosen - rejected;
  double m, loss, slope;
  if (f.pair_kind == 1) {
    m = D - (double)f.margin;
    const double d = m - 0.5 / beta;
    loss = d * d;
    slope = 2.0 * d;
  } else {
    m = beta * D - (double)f.margin;
    if (f.pair_kind == 2) {
      loss = fmax(1.0 - m, 0.0);
      slope = m < 1.0 ? -beta : 0.0;
    } else {
      // (a part with factor 0 is left out: its logarithm may be infinite)
      loss = (e < 1.0 ? (1.0 - e) * softplus(-m) : 0.0) + (e > 0.0 ? e * softplus(m) : 0.0);
      slope = beta * (e / (1.0 + exp(-m)) - (1.0 - e) / (1.0 + exp(m)));
    }
    if (m != m) loss = slope = m;
  }
  const double w = f.pair_weight ? (double)f.pair_weight[i] : 1.0 / (double)P;
  const double scale = w * (f.grad_scale ? (double)*f.grad_scale : 1.0);
  if ((threadIdx.x & 63) != 0) return;
  st_agent(ws.pair + i, w != 0.0 ? w * loss : 0.0);
  ws.seq[i] = w != 0.0 ? (float)(scale * slope) : 0.f;
  ws.seq[P + i] = w != 0.0 ? (float)(-scale * slope) : 0.f;
  if (f.pair_loss) f.pair_loss[i] = (float)loss;
  if (f.pair_margin) f.pair_margin[i] = (float)m;
  if (f.score) {
    f.score[i] = (float)chosen;
    f.score[P + i] = (float)rejected;
  }
}

// Whether this is the last of n to come to a counter, which is zero again then: all that the others stored before is to be read.
__device__ __forceinline__ bool last_of(int32_t* counter, int n) {
  stores_before_loads();
  if (!last_to_add(add_arrival(counter), n)) return false;
  set_arrival(counter, 0);
  return true;
}
// Position r is settled (one wavefront): the last of a pair settles the pair, the last of all adds up the loss.
__device__ __forceinline__ void position_done(const LossRows& rows, const LossTerm& f, const LossWorkspace& ws, int r, double term) {
  if (!f.loss) return;
  if ((threadIdx.x & 63) == 0) st_agent(ws.term + r, term);
  if (!f.adds_up) return;
  int n = rows.n;
  const double* v = ws.term;
  if (f.kind == kPreference) {
    const int b = r / rows.T, i = b < f.P ? b : b - f.P;
    if (!last_of(ws.done + 1 + i * ticket_stride(f.P, kAddsUp), 2 * rows.T)) return;
    settle_pair<true>(f, ws, i, rows.T);
    n = f.P;
    v = ws.pair;
  }
  if (!last_of(ws.done, n)) return;
  const double t = wave_total<true>(v, n);
  if ((threadIdx.x & 63) == 0) *f.loss = (float)t;
}

// Sums of a whole row by one wavefront (where the slices' records did not arrive, which never happens to calls that are ordered as they
// have to be).
template <int DT, bool REF> __device__ __noinline__ LossSums wave_row_sums(const char* row, const char* ref, int V, float c) {
  LossSums a = loss_empty();
#pragma unroll 1
  for (int idx = threadIdx.x & 63; idx < vectors_of<DT>(V); idx += 64) {
    const uint4 x = load_vec_of<DT>(row, idx, V);
    loss_push<DT, REF>(a, x, REF ? load_vec_of<DT>(ref, idx, V) : x, c);
  }
  return loss_fold_wave<REF>(a);
}

// A slice's vectors come in batches of four per thread, the next batch on its way.
constexpr int kSumsBatch = 4;
template <int DT, bool REF> __global__ void __launch_bounds__(kBlock) k_loss_sums(LossRows rows, LossTerm f, int S, int chunk, LossWorkspace ws) {
  __shared__ LossSums sh[kWaves];
  const int r = blockIdx.x / S, s = blockIdx.x - r * S, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = r / rows.T, t = r - b * rows.T, V = rows.V;
  if (!position_counts(rows, r)) {
    if (s != 0 || wave != 0) return;
    if (lane == 0) {
      report_nothing(rows, f, r);
      ws.coef[r] = LossCoef{};
    }
    position_done(rows, f, ws, r, 0.0);
    return;
  }
  PositionIn in = ask_position(rows, f, r, b);
  const char* row = row_at<DT>(rows.z, b, t);
  const char* ref = REF ? row_at<DT>(rows.ref, b, t) : nullptr;
  const int nv = vectors_of<DT>(V), v0 = min(s * chunk, nv), v1 = min(v0 + chunk, nv);
  auto load = [&](const char* from, int idx) { return idx < v1 ? load_vec_of<DT>(from, idx, V) : neutral_vec<DT>(); };
  uint4 next[kSumsBatch], nextr[kSumsBatch];
#pragma unroll
  for (int k = 0; k < kSumsBatch; ++k) next[k] = load(row, v0 + tid + k * kBlock);
  if (REF) {
#pragma unroll
    for (int k = 0; k < kSumsBatch; ++k) nextr[k] = load(ref, v0 + tid + k * kBlock);
  }
  ask_logit<DT>(in, row, V);
  const float c = REF ? ref_shift<DT>(row, ref, in.x, V) : 0.f;
  LossSums a = loss_empty();
  for (int base = v0; base < v1; base += kSumsBatch * kBlock) {
    uint4 x[kSumsBatch], xr[kSumsBatch];
#pragma unroll
    for (int k = 0; k < kSumsBatch; ++k) {
      x[k] = next[k];
      if (REF) xr[k] = nextr[k];
    }
    if (base + kSumsBatch * kBlock < v1) {
#pragma unroll
      for (int k = 0; k < kSumsBatch; ++k) {
        const int idx = base + tid + (k + kSumsBatch) * kBlock;
        next[k] = load(row, idx);
        if (REF) nextr[k] = load(ref, idx);
      }
    }
    loss_raise(a, vecs_max<DT, kSumsBatch>(x));
#pragma unroll
    for (int k = 0; k < kSumsBatch; ++k)
      if (base + k * kBlock < v1) loss_push_at<DT, REF>(a, x[k], REF ? xr[k] : x[k], c);
  }
  a = loss_fold_wave<REF>(a);
  if (lane == 0) sh[wave] = a;
  __syncthreads();
  if (wave != 0) return;
  a = loss_fold_wave<REF>(lane < kWaves ? sh[lane] : loss_empty());
  if (S > 1) {
    uint64_t w[kXchgWords];
    bool arrived = true;
    pack_pair(PairRecord{a.m, a.s, a.u, REF ? a.mr : a.m, REF ? a.sr : 0.f, REF ? a.w : 0.f}, w);
    if (!hand_off(PlainWords{ws.xchg + (size_t)r * S * kXchgWords}, s, S, Arrivals{ws.ticket, kTicketLossLen, r, rows.n}, f.wait, [] {}, w, arrived))
      return;
    a = loss_empty();
    if (lane < S) {
      const PairRecord p = unpack_pair(w);
      a = LossSums{p.mp, p.sp, p.up, p.uq, p.mq, p.sq};
    }
    a = loss_fold_wave<REF>(a);
    if (__builtin_expect(!arrived, 0)) a = wave_row_sums<DT, REF>(row, ref, V, c);
  }
  double term;
  const LossCoef k = settle_position<REF>(rows, f, r, in, a, c, term);
  if (lane == 0) ws.coef[r] = k;
  position_done(rows, f, ws, r, term);
}

__global__ void __launch_bounds__(64) k_loss_pairs(LossTerm f, int T, LossWorkspace ws) { settle_pair<false>(f, ws, blockIdx.x, T); }

__global__ void __launch_bounds__(64) k_loss_total(const double* v, int n, float* out) {
  const double t = wave_total<false>(v, n);
  if (threadIdx.x == 0) *out = (float)t;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {       // nearest, ties to even
  const bf16x2 v = __builtin_convertvector((floatx2{a, b}), bf16x2);
  uint32_t r;
  __builtin_memcpy(&r, &v, 4);
  return r;
}
// A whole vector of gradients, or the elements of the last one that the row has.
template <int DT> __device__ __forceinline__ void store_grad(char* row, int idx, int V, const float (&g)[Elem<DT>::per_vec]) {
  constexpr int EPV = Elem<DT>::per_vec;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DT == ADASD_BF16) w[i] = pack_bf16(g[2 * i % EPV], g[(2 * i + 1) % EPV]);
    else w[i] = __float_as_uint(g[i]);
  }
  if (idx < V / EPV) {
    vec16_any v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = w[i];
    *reinterpret_cast<vec16_any*>(row + (size_t)idx * 16) = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < EPV - 1; ++i) {
    const int j = idx * EPV + i;
    if (j >= V) break;
    if (DT == ADASD_BF16) reinterpret_cast<uint16_t*>(row)[j] = (uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2]);
    else reinterpret_cast<uint32_t*>(row)[j] = w[i];
  }
}

// The gradients of one vector: a 1[j = x] + e (k0 + k1 t + k2 dd).
template <int DT, bool ENT, bool REF>
__device__ __forceinline__ void grad_vec(const uint4& x, const uint4& xr, const LossCoef& k, float (&g)[Elem<DT>::per_vec]) {
  const float neg_m = -k.m;
#pragma unroll
  for (int h = 0; h < Elem<DT>::per_vec / 4; ++h) {
    float z[4], t[4], e[4], q[4];
    unpack4<DT>(x, h, z);
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = fma_log2e(z[i], neg_m);
    ex2_group(t, e);
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = ENT ? fmaf(k.k1, max_raw(t[i], -200.f), k.k0) : k.k0;
    if (REF) {
      float y[4];
      unpack4<DT>(xr, h, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float dd = fma_log2e(z[i] - y[i], -k.c);
        q[i] = fmaf(k.k2, e[i] > 0.f ? dd : 0.f, q[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) g[4 * h + i] = e[i] * q[i];
  }
}

template <int DT, bool ENT, bool REF>
__global__ void __launch_bounds__(kBlock) k_loss_grad(LossRows rows, int S, LossWorkspace ws, int by_sequence) {
  constexpr int EPV = Elem<DT>::per_vec;
  const int r = blockIdx.x, b = r / rows.T, t = r - b * rows.T, V = rows.V;
  LossCoef k = scalar_load(ws.coef + r);
  if (by_sequence) {
    const float d = scalar_load(ws.seq + b);
    k.a *= d;
    k.k0 = d == 0.f ? 0.f : k.k0 * d;
    if (d == 0.f) k.a = 0.f;
  }
  char* out = const_cast<char*>(row_at<DT>(rows.g, b, t));
  const char* row = row_at<DT>(rows.z, b, t);
  const char* ref = REF ? row_at<DT>(rows.ref, b, t) : nullptr;
  int v0, v1;
  slice_of(vectors_of<DT>(V), blockIdx.y, S, v0, v1);
  float g[EPV];
  if (k.a == 0.f && k.k0 == 0.f && k.k1 == 0.f && k.k2 == 0.f) {
#pragma unroll
    for (int i = 0; i < EPV; ++i) g[i] = 0.f;
    for (int idx = v0 + threadIdx.x; idx < v1; idx += kBlock) store_grad<DT>(out, idx, V, g);
    return;
  }
  const int x = rows.tokens[r];
  for (int idx = v0 + threadIdx.x; idx < v1; idx += kBlock) {
    const uint4 v = load_vec_of<DT>(row, idx, V);
    grad_vec<DT, ENT, REF>(v, REF ? load_vec_of<DT>(ref, idx, V) : v, k, g);
    if (idx == x / EPV) {
#pragma unroll
      for (int i = 0; i < EPV; ++i) g[i] += idx * EPV + i == x ? k.a : 0.f;
    }
    store_grad<DT>(out, idx, V, g);
  }
}

// ---- Many rows: one workgroup of T threads per row.  The row's first NB vectors per thread stay in registers (raw) from the load to
// the gradient, so that they are read once; what is longer, and the reference's row, is read again (from the cache behind the L2s,
// where the few hundred rows in work fit).
template <int W> struct FusedLoss {
  LossSums sums[W];
  LossCoef coef;
};
constexpr int kRefAhead = 4;      // vectors of the reference's row on their way
template <int DT, bool ENT, bool REF, int T, int NB>
__global__ void __launch_bounds__(T, 4) k_loss_fused(LossRows rows, LossTerm f, LossWorkspace ws) {
  constexpr int EPV = Elem<DT>::per_vec, W = T / 64;
  __shared__ FusedLoss<W> sh;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = rows.V, whole = V / EPV, nv = vectors_of<DT>(V);
  const int b = r / rows.T, t = r - b * rows.T;
  char* out = const_cast<char*>(row_at<DT>(rows.g, b, t));
  float g[EPV];
  auto zeros = [&] {
#pragma unroll
    for (int i = 0; i < EPV; ++i) g[i] = 0.f;
    for (int idx = tid; idx < nv; idx += T) store_grad<DT>(out, idx, V, g);
  };
  if (!position_counts(rows, r)) {
    if (tid == 0) report_nothing(rows, f, r);
    zeros();
    if (wave == 0) position_done(rows, f, ws, r, 0.0);
    return;
  }
  PositionIn in = ask_position(rows, f, r, b);
  const char* row = row_at<DT>(rows.z, b, t);
  const char* ref = REF ? row_at<DT>(rows.ref, b, t) : nullptr;
  auto load = [&](const char* from, int j) {
    const int idx = tid + j * T;
    if ((j + 1) * T <= whole) return load_vec_any(from, idx);
    return idx < nv ? load_vec_of<DT>(from, idx, V) : neutral_vec<DT>();
  };
  uint4 v[NB], q[kRefAhead];
#pragma unroll
  for (int j = 0; j < NB; ++j) v[j] = load(row, j);
  if (REF) {
#pragma unroll
    for (int j = 0; j < kRefAhead; ++j) q[j] = load(ref, j);
  }
  ask_logit<DT>(in, row, V);
  const float c = REF ? ref_shift<DT>(row, ref, in.x, V) : 0.f;
  LossSums a = loss_empty();
  a.m = vecs_max<DT, NB>(v);
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    if (j * T < nv) loss_push_at<DT, REF>(a, v[j], REF ? q[j % kRefAhead] : v[j], c);
    if (REF && j + kRefAhead < NB) q[j % kRefAhead] = load(ref, j + kRefAhead);
  }
  for (int idx = tid + NB * T; idx < nv; idx += T) {
    const uint4 x = load_vec_of<DT>(row, idx, V);
    loss_push<DT, REF>(a, x, REF ? load_vec_of<DT>(ref, idx, V) : x, c);
  }
  a = loss_fold_wave<REF>(a);
  if (lane == 0) sh.sums[wave] = a;
  __syncthreads();
  double term = 0.0;
  if (wave == 0) {
    a = loss_fold_wave<REF>(lane < W ? sh.sums[lane] : loss_empty());
    const LossCoef mine = settle_position<REF>(rows, f, r, in, a, c, term);
    if (lane == 0) sh.coef = mine;
  }
  if (REF) {
#pragma unroll
    for (int j = 0; j < kRefAhead; ++j) q[j] = load(ref, j);
  }
  __syncthreads();
  const LossCoef k = sh.coef;
  if (k.a == 0.f && k.k0 == 0.f && k.k1 == 0.f && k.k2 == 0.f) {
    zeros();
    if (wave == 0) position_done(rows, f, ws, r, term);
    return;
  }
  const int x = in.x;
  auto emit = [&](int idx, const uint4& z, const uint4& zr) {
    grad_vec<DT, ENT, REF>(z, zr, k, g);
    if (idx == x / EPV) {
#pragma unroll
      for (int i = 0; i < EPV; ++i) g[i] += idx * EPV + i == x ? k.a : 0.f;
    }
    store_grad<DT>(out, idx, V, g);
  };
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int idx = tid + j * T;
    if (idx < nv) emit(idx, v[j], REF ? q[j % kRefAhead] : v[j]);
    if (REF && j + kRefAhead < NB) q[j % kRefAhead] = load(ref, j + kRefAhead);
  }
  for (int idx = tid + NB * T; idx < nv; idx += T) {
    const uint4 z = load_vec_of<DT>(row, idx, V);
    emit(idx, z, REF ? load_vec_of<DT>(ref, idx, V) : z);
  }
  if (wave == 0) position_done(rows, f, ws, r, term);
}

}  // namespace

hipError_t launch_loss(const LossRows& rows, int dt, LossTerm f, const LossWorkspace& ws, hipStream_t st) {
  const int n = rows.n, epv = dt == ADASD_BF16 ? 8 : 4, nv = (rows.V + epv - 1) / epv;
  const bool ref = rows.ref.base != nullptr, ent = f.kind == kPolicy ? f.entropy_coef != 0.f : f.kind == kLogprob && f.dentropy;
  const bool by_ref = ref && f.kl_coef != 0.f;
  const bool fused = rows.g.base && f.kind != kPreference && ref == by_ref && n >= 256;
  const dim3 block(kBlock);
  f.adds_up = f.loss && n > 0 && n <= kAddsUp;
  if (fused) {
    const int T = nv <= 128 * 16 ? 128 : nv <= 256 * 16 ? 256 : nv <= 512 * 16 ? 512 : 1024;
#define ADASD_FUSED_CASE(DTV, ENTV, REFV, TV, NBV) \
    if (dt == DTV && ent == ENTV && ref == REFV && T == TV) \
      launch_kernel((k_loss_fused<DTV, ENTV, REFV, TV, NBV>), dim3(n), dim3(TV), st, rows, f, ws);
#define ADASD_FUSED_CASES(TV, NBV) \
    ADASD_FUSED_CASE(ADASD_BF16, false, false, TV, NBV) ADASD_FUSED_CASE(ADASD_BF16, true, false, TV, NBV) \
    ADASD_FUSED_CASE(ADASD_F32, false, false, TV, NBV) ADASD_FUSED_CASE(ADASD_F32, true, false, TV, NBV) \
    ADASD_FUSED_CASE(ADASD_BF16, false, true, TV, NBV) ADASD_FUSED_CASE(ADASD_BF16, true, true, TV, NBV) \
    ADASD_FUSED_CASE(ADASD_F32, false, true, TV, NBV) ADASD_FUSED_CASE(ADASD_F32, true, true, TV, NBV)
    ADASD_FUSED_CASES(128, 16) ADASD_FUSED_CASES(256, 16) ADASD_FUSED_CASES(512, 16) ADASD_FUSED_CASES(1024, 16)
#undef ADASD_FUSED_CASES
#undef ADASD_FUSED_CASE
  } else if (n > 0) {
    const int S = scan_split(n, rows.V, dt), chunk = slice_chunk(nv, S);
#define ADASD_LOSS_CASE(DTV, REFV) \
    if (dt == DTV && ref == REFV) launch_kernel((k_loss_sums<DTV, REFV>), dim3(n * S), block, st, rows, f, S, chunk, ws);
    ADASD_LOSS_CASE(ADASD_BF16, false) ADASD_LOSS_CASE(ADASD_BF16, true) ADASD_LOSS_CASE(ADASD_F32, false) ADASD_LOSS_CASE(ADASD_F32, true)
#undef ADASD_LOSS_CASE
    if (f.kind == kPreference && !f.adds_up) launch_kernel(k_loss_pairs, dim3(f.P), dim3(64), st, f, rows.T, ws);
    if (rows.g.base) {
      const int turns = 8, slices = (nv + turns * kBlock - 1) / (turns * kBlock);
      const dim3 pieces(n, slices);
#define ADASD_GRAD_CASE(DTV, ENTV, REFV) \
      if (dt == DTV && ent == ENTV && by_ref == REFV) \
        launch_kernel((k_loss_grad<DTV, ENTV, REFV>), pieces, block, st, rows, slices, ws, f.kind == kPreference ? 1 : 0);
      ADASD_GRAD_CASE(ADASD_BF16, false, false) ADASD_GRAD_CASE(ADASD_BF16, false, true) ADASD_GRAD_CASE(ADASD_BF16, true, false)
      ADASD_GRAD_CASE(ADASD_BF16, true, true) ADASD_GRAD_CASE(ADASD_F32, false, false) ADASD_GRAD_CASE(ADASD_F32, false, true)
      ADASD_GRAD_CASE(ADASD_F32, true, false) ADASD_GRAD_CASE(ADASD_F32, true, true)
#undef ADASD_GRAD_CASE
    }
  }
  if (f.loss && !f.adds_up) {
    const bool pairs = f.kind == kPreference;
    launch_kernel(k_loss_total, dim3(1), dim3(64), st, (const double*)(pairs ? ws.pair : ws.term), n == 0 ? 0 : pairs ? f.P : n, f.loss);
  }
  return hipGetLastError();
}

}  // namespace adasd
