// Log-probabilities of tokens, the clipped policy loss and the preference loss over vocabulary rows, with their gradients.
//
// A gradient row needs the row's normaliser (and entropy, and KL) before its first element, and the preference loss those of whole
// sequences: the rows are read, the few numbers of each position settled, and the rows read again for the gradient.
//   k_loss_sums  (slices of rows)  -> sums of each slice (loss_device.h)
//   k_loss_rows  (a wavefront per position) folds the slices, writes what is reported of the position, and the five numbers of its
//                gradient row
//   k_loss_pairs (a workgroup per pair; preference only) the scores of the two sequences, the pair's loss and slope
//   k_loss_grad  (slices of rows)  -> the gradient
//   k_loss_total (one workgroup)   adds up the loss
// Sums over positions and sequences are in 64 bits and in a fixed order.
#include "loss_device.h"

namespace adasd {

namespace {

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

template <int DT, bool REF> __global__ void __launch_bounds__(kBlock) k_loss_sums(LossRows rows, int S, float4* rec) {
  __shared__ LossSums sh[kWaves];
  const int r = blockIdx.x, s = blockIdx.y, tid = threadIdx.x;
  if (!position_counts(rows, r)) return;
  const int b = r / rows.T, t = r - b * rows.T, V = rows.V;
  const char* row = row_at<DT>(rows.z, b, t);
  const char* ref = REF ? row_at<DT>(rows.ref, b, t) : nullptr;
  const float c = REF ? ref_shift<DT>(row, ref, rows.tokens[r], V) : 0.f;
  int v0, v1;
  slice_of(vectors_of<DT>(V), s, S, v0, v1);
  LossSums a = loss_empty();
  for (int idx = v0 + tid; idx < v1; idx += kBlock) {
    const uint4 x = load_vec_of<DT>(row, idx, V);
    loss_push<DT, REF>(a, x, REF ? load_vec_of<DT>(ref, idx, V) : x, c);
  }
  a = loss_fold_wave<REF>(a);
  if ((tid & 63) == 0) sh[tid >> 6] = a;
  __syncthreads();
  if (tid < 64) {
    a = tid < kWaves ? sh[tid] : loss_empty();
    a = loss_fold_wave<REF>(a);
    if (tid == 0) {
      rec[2 * ((size_t)r * S + s)] = make_float4(a.m, a.s, a.u, a.w);
      rec[2 * ((size_t)r * S + s) + 1] = make_float4(a.mr, a.sr, c, 0.f);
    }
  }
}

// What is reported of a position, and the numbers of its gradient row (from the sums of the whole row).
template <int DT, bool REF>
__device__ __forceinline__ LossCoef settle_position(const LossRows& rows, const LossTerm& f, int r, const LossSums& sums, float c,
                                                    double& term) {
  const int b = r / rows.T, t = r - b * rows.T, x = rows.tokens[r];
  const bool known = x >= 0 && x < rows.V;
  const LossRow row = finish_loss_row<REF>(sums, c);
  const double lp = known ? (double)load_elem<DT>(row_at<DT>(rows.z, b, t), known ? x : 0) - row.lse : (double)NAN;
  const double w = rows.weight ? (double)rows.weight[r] : 1.0;
  double a = 0.0, by_entropy = 0.0, by_kl = 0.0;
  term = 0.0;
  if (f.kind == kLogprob) {
    if (f.dlogprob) a = (double)f.dlogprob[r];
    if (f.dentropy) by_entropy = (double)f.dentropy[r];
  } else if (f.kind == kPolicy) {
    const double A = (double)f.advantage[f.adv_per_seq ? b : r];
    const double ratio = f.old_logprob ? exp(lp - (double)f.old_logprob[r]) : lp == lp ? 1.0 : lp;
    double loss = 0.0, kl = row.kl;
    if (A != 0.0) {
      const double free = ratio * A, held = fmin(fmax(ratio, 1.0 - (double)f.clip_low), 1.0 + (double)f.clip_high) * A;
      const bool clipped = held < free;
      loss = -(clipped ? held : free);
      a = clipped ? 0.0 : -free;
    }
    if (f.ref_logprob) {
      const double d = (double)f.ref_logprob[r] - lp, grown = expm1(d);
      kl = grown - d;
      if (f.kl_coef != 0.f) a -= (double)f.kl_coef * grown;
    }
    if (f.kl_coef != 0.f) loss += (double)f.kl_coef * kl;
    if (f.entropy_coef != 0.f) loss -= (double)f.entropy_coef * row.H;
    term = w * loss;
    if (f.token_loss) f.token_loss[r] = (float)loss;
    if (f.kl) f.kl[r] = (float)kl;
    const double scale = w * (f.grad_scale ? (double)*f.grad_scale : 1.0);
    a *= scale;
    by_entropy = -scale * (double)f.entropy_coef;
    if (REF) by_kl = scale * (double)f.kl_coef;
  } else {
    term = w * (lp - (f.ref_logprob ? (double)f.ref_logprob[r] : 0.0));
    a = w;
  }
  if (rows.logprob) rows.logprob[r] = (float)lp;
  if (rows.entropy) rows.entropy[r] = (float)row.H;
  if (rows.status) rows.status[r] = (known ? 0u : (uint32_t)ADASD_ST_BAD_TOKEN) | (row.bad ? (uint32_t)ADASD_ST_NONFINITE : 0u);
  // dz_j = a (1[j = x] - p_j) - by_entropy p_j (ln p_j + H) + by_kl p_j (ln p_j - ln q_j - KL)
  LossCoef k{};
  const double inv_s = (double)row.inv_s;
  double k0 = -a;
  if (by_entropy != 0.0) {
    k0 -= by_entropy * (row.H - (row.lse - kNat * (double)sums.m));
    k.k1 = (float)(-by_entropy * kNat * inv_s);
  }
  if (REF && by_kl != 0.0) {
    k0 += by_kl * (kNat * (double)c - (row.lse - row.lse_ref) - row.kl);
    k.k2 = (float)(by_kl * kNat * inv_s);
  }
  k.m = sums.m;
  k.c = c;
  k.a = (float)a;
  k.k0 = k0 == 0.0 ? 0.f : (float)(k0 * inv_s);      // (nothing of the row enters a gradient of zeros)
  return k;
}

// The results of a position that does not count.
__device__ __forceinline__ void report_nothing(const LossRows& rows, const LossTerm& f, const LossWorkspace& ws, int r) {
  if (rows.logprob) rows.logprob[r] = 0.f;
  if (rows.entropy) rows.entropy[r] = 0.f;
  if (rows.status) rows.status[r] = 0u;
  if (f.token_loss) f.token_loss[r] = 0.f;
  if (f.kl) f.kl[r] = 0.f;
  ws.term[r] = 0.0;
}

template <int DT, bool REF> __global__ void __launch_bounds__(kBlock) k_loss_rows(LossRows rows, LossTerm f, int S, LossWorkspace ws) {
  const int r = blockIdx.x * kWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= rows.n) return;
  if (!position_counts(rows, r)) {
    if (lane == 0) {
      report_nothing(rows, f, ws, r);
      ws.coef[r] = LossCoef{};
    }
    return;
  }
  LossSums a = loss_empty();
  float c = 0.f;
  if (REF) c = ws.rec[2 * (size_t)r * S + 1].z;
  if (lane < S) {
    const float4 p = ws.rec[2 * ((size_t)r * S + lane)], q = ws.rec[2 * ((size_t)r * S + lane) + 1];
    a = LossSums{p.x, p.y, p.z, p.w, q.x, q.y};
  }
  a = loss_fold_wave<REF>(a);
  if (lane == 0) {
    double term;
    ws.coef[r] = settle_position<DT, REF>(rows, f, r, a, c, term);
    ws.term[r] = term;
  }
}

// Sum of v over the workgroup in 64 bits, in thread 0 (a fixed order).
__device__ __forceinline__ double block_sum(double v, double (&sh)[kWaves]) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) t += sh[w];
  return t;
}
__device__ __forceinline__ double strided_sum(const double* v, int n) {
  double t = 0.0;
  for (int i = threadIdx.x; i < n; i += kBlock) t += v[i];
  return t;
}

__device__ __forceinline__ double softplus(double v) { return fmax(v, 0.0) + log1p(exp(-fabs(v))); }

__global__ void __launch_bounds__(kBlock) k_loss_pairs(LossTerm f, int T, LossWorkspace ws) {
  __shared__ double sh[kWaves];
  const int i = blockIdx.x, P = f.P;
  const double chosen = block_sum(strided_sum(ws.term + (size_t)i * T, T), sh);
  const double rejected = block_sum(strided_sum(ws.term + (size_t)(P + i) * T, T), sh);
  if (threadIdx.x != 0) return;
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
      if (m != m) loss = slope = m;
    } else {
      // (a part with factor 0 is left out: its logarithm may be infinite)
      loss = (e < 1.0 ? (1.0 - e) * softplus(-m) : 0.0) + (e > 0.0 ? e * softplus(m) : 0.0);
      slope = beta * (e / (1.0 + exp(-m)) - (1.0 - e) / (1.0 + exp(m)));
      if (m != m) loss = slope = m;
    }
  }
  const double w = f.pair_weight ? (double)f.pair_weight[i] : 1.0 / (double)P;
  const double scale = w * (f.grad_scale ? (double)*f.grad_scale : 1.0);
  ws.pair[i] = w != 0.0 ? w * loss : 0.0;
  ws.seq[i] = w != 0.0 ? (float)(scale * slope) : 0.f;
  ws.seq[P + i] = w != 0.0 ? (float)(-scale * slope) : 0.f;
  if (f.pair_loss) f.pair_loss[i] = (float)loss;
  if (f.pair_margin) f.pair_margin[i] = (float)m;
  if (f.score) {
    f.score[i] = (float)chosen;
    f.score[P + i] = (float)rejected;
  }
}

__global__ void __launch_bounds__(kBlock) k_loss_total(const double* v, int n, float* out) {
  __shared__ double sh[kWaves];
  const double t = block_sum(strided_sum(v, n), sh);
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
__global__ void __launch_bounds__(kBlock) k_loss_grad(LossRows rows, int S, LossWorkspace ws, int by_sequence, const float* grad_scale) {
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

// ---- Many rows: one workgroup per row, which stays in its registers (T threads, up to NB vectors each, raw) from the load to the
// gradient: the logits are read once.
template <int W> struct FusedLoss {
  LossSums sums[W];
  LossCoef coef;
};
template <int DT, bool ENT, int T, int NB>
__global__ void __launch_bounds__(T) k_loss_fused(LossRows rows, LossTerm f, LossWorkspace ws) {
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
    if (tid == 0) report_nothing(rows, f, ws, r);
    zeros();
    return;
  }
  const char* row = row_at<DT>(rows.z, b, t);
  uint4 v[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int idx = tid + j * T;
    if ((j + 1) * T <= whole) v[j] = load_vec_any(row, idx);
    else if (idx < nv) v[j] = load_vec_of<DT>(row, idx, V);
    else v[j] = neutral_vec<DT>();
  }
  LossSums a = loss_empty();
  a.m = vecs_max<DT, NB>(v);
#pragma unroll
  for (int j = 0; j < NB; ++j)
    if (j * T < nv) loss_push_at<DT, false>(a, v[j], v[j], 0.f);
  a = loss_fold_wave<false>(a);
  if (lane == 0) sh.sums[wave] = a;
  __syncthreads();
  if (wave == 0) {
    a = loss_fold_wave<false>(lane < W ? sh.sums[lane] : loss_empty());
    if (lane == 0) {
      double term;
      sh.coef = settle_position<DT, false>(rows, f, r, a, 0.f, term);
      if (f.loss) ws.term[r] = term;
    }
  }
  __syncthreads();
  const LossCoef k = sh.coef;
  if (k.a == 0.f && k.k0 == 0.f && k.k1 == 0.f) {
    zeros();
    return;
  }
  const int x = rows.tokens[r];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int idx = tid + j * T;
    if (idx < nv) {
      grad_vec<DT, ENT, false>(v[j], v[j], k, g);
      if (idx == x / EPV) {
#pragma unroll
        for (int i = 0; i < EPV; ++i) g[i] += idx * EPV + i == x ? k.a : 0.f;
      }
      store_grad<DT>(out, idx, V, g);
    }
  }
}

}  // namespace

hipError_t launch_loss(const LossRows& rows, int dt, const LossTerm& f, const LossWorkspace& ws, hipStream_t st) {
  const int n = rows.n, epv = dt == ADASD_BF16 ? 8 : 4, nv = (rows.V + epv - 1) / epv;
  const bool ref = rows.ref.base != nullptr;
  const dim3 block(kBlock);
  const bool ent = f.kind == kPolicy ? f.entropy_coef != 0.f : f.kind == kLogprob && f.dentropy;
  const bool fused = rows.g.base && f.kind != kPreference && !ref && n >= 256 && nv <= 1024 * 20;
  if (fused) {
    const int NB = nv <= 1024 * 16 ? 16 : 20, T = NB == 20 ? 1024 : nv <= 128 * 16 ? 128 : nv <= 256 * 16 ? 256 : nv <= 512 * 16 ? 512 : 1024;
#define ADASD_FUSED_CASE(DTV, ENTV, TV, NBV) \
    if (dt == DTV && ent == ENTV && T == TV && NB == NBV) launch_kernel((k_loss_fused<DTV, ENTV, TV, NBV>), dim3(n), dim3(TV), st, rows, f, ws);
#define ADASD_FUSED_CASES(TV, NBV) ADASD_FUSED_CASE(ADASD_BF16, false, TV, NBV) ADASD_FUSED_CASE(ADASD_BF16, true, TV, NBV) \
    ADASD_FUSED_CASE(ADASD_F32, false, TV, NBV) ADASD_FUSED_CASE(ADASD_F32, true, TV, NBV)
    ADASD_FUSED_CASES(128, 16) ADASD_FUSED_CASES(256, 16) ADASD_FUSED_CASES(512, 16) ADASD_FUSED_CASES(1024, 16) ADASD_FUSED_CASES(1024, 20)
#undef ADASD_FUSED_CASES
#undef ADASD_FUSED_CASE
  } else if (n > 0) {
    const int S = scan_split(n, rows.V, dt);
    const dim3 grid(n, S), waves((n + kWaves - 1) / kWaves);
#define ADASD_LOSS_CASE(DTV, REFV) \
    if (dt == DTV && ref == REFV) { \
      launch_kernel((k_loss_sums<DTV, REFV>), grid, block, st, rows, S, ws.rec); \
      launch_kernel((k_loss_rows<DTV, REFV>), waves, block, st, rows, f, S, ws); \
    }
    ADASD_LOSS_CASE(ADASD_BF16, false) ADASD_LOSS_CASE(ADASD_BF16, true) ADASD_LOSS_CASE(ADASD_F32, false) ADASD_LOSS_CASE(ADASD_F32, true)
#undef ADASD_LOSS_CASE
    if (f.kind == kPreference) launch_kernel(k_loss_pairs, dim3(f.P), block, st, f, rows.T, ws);
    if (rows.g.base) {
      const int turns = 8, slices = (nv + turns * kBlock - 1) / (turns * kBlock);
      const dim3 pieces(n, slices);
      const bool by_ref = ref && f.kl_coef != 0.f;
#define ADASD_GRAD_CASE(DTV, ENTV, REFV) \
      if (dt == DTV && ent == ENTV && by_ref == REFV) \
        launch_kernel((k_loss_grad<DTV, ENTV, REFV>), pieces, block, st, rows, slices, ws, f.kind == kPreference ? 1 : 0, f.grad_scale);
      ADASD_GRAD_CASE(ADASD_BF16, false, false) ADASD_GRAD_CASE(ADASD_BF16, false, true) ADASD_GRAD_CASE(ADASD_BF16, true, false)
      ADASD_GRAD_CASE(ADASD_BF16, true, true) ADASD_GRAD_CASE(ADASD_F32, false, false) ADASD_GRAD_CASE(ADASD_F32, false, true)
      ADASD_GRAD_CASE(ADASD_F32, true, false) ADASD_GRAD_CASE(ADASD_F32, true, true)
#undef ADASD_GRAD_CASE
    }
  }
  if (f.loss) {
    const bool pairs = f.kind == kPreference;
    launch_kernel(k_loss_total, dim3(1), block, st, (const double*)(pairs ? ws.pair : ws.term), n == 0 ? 0 : pairs ? f.P : n, f.loss);
  }
  return hipGetLastError();
}

}  // namespace adasd
