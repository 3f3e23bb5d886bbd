// Log-probabilities of tokens, the clipped policy loss and the preference loss over vocabulary rows, with their gradients.
//
// A gradient row needs the row's normaliser (and entropy, and KL) before its first element, and the preference loss those of whole
// sequences.
//   k_loss_join  gradients that need nothing but their own row: the row stays in the registers of its workgroups between the sums and
//                the gradient, so that everything is read once and written once.  Rows of up to 2048 vectors: one to four wavefronts
//                each; longer ones: slices, whose workgroups exchange their sums.
//   k_loss_sums  (slices of rows) the sums alone: log-probabilities, the preference loss, rows too long for k_loss_join.  One workgroup of
//                a row folds its slices (hand_off).
//   k_loss_grad  (pieces of rows) reads the logits again and forms the gradient.
// Either way one wavefront settles the position: what is reported of it, and the six numbers of its gradient row.  Of few positions
// the one done last adds up the loss, or settles its pair; of many k_loss_pairs and k_loss_total do.
// Sums over positions and sequences are in 64 bits and in a fixed order, whoever forms them.
#include "loss_device.h"
#include "sample_device.h"

namespace adasd {

namespace {

using namespace sampling;

// A whole vector, `lane` vectors behind one at a uniform place (the address then is that place and one register); PAST: without a place in the
// caches.
template <bool PAST> __device__ __forceinline__ uint4 load_whole(const char* row, int at, int lane) {
  const vec16_any* from = reinterpret_cast<const vec16_any*>(row + (size_t)at * 16 + (uint32_t)lane * 16u);
  const vec16_any v = PAST ? __builtin_nontemporal_load(from) : *from;
  return make_uint4(v[0], v[1], v[2], v[3]);
}
template <int DT> __device__ __forceinline__ uint4 load_vec_of(const char* row, int idx, int V) {
  return idx < V / Elem<DT>::per_vec ? load_vec_any(row, idx) : load_last_vec<DT>(row, V);
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

// What is reported of a position, and the numbers of its gradient row, from the sums of the whole row.  Two neighbouring lanes (or more
// pairs of them) go through it together; the one that `writes` reports.  exps: see finish_loss_row.
template <bool REF>
__device__ __forceinline__ LossCoef settle_position(const LossRows& rows, const LossTerm& f, int r, const PositionIn& in, const LossSums& sums,
                                                    int exps, bool writes, double& term) {
  const bool odd = threadIdx.x & 1;
  const bool known = in.x >= 0 && in.x < rows.V;
  const LossRow row = finish_loss_row<REF>(sums, exps);
  const double above = known ? (double)in.z - row.lse : (double)NAN, lp = above > 0.0 ? 0.0 : above;      // (a token with all the mass, to rounding)
  const double w = (double)in.weight;
  double a = 0.0, by_entropy = 0.0, by_kl = 0.0, loss = 0.0, kl = row.kl;
  term = 0.0;
  if (f.kind == kLogprob) {
    a = known || in.a == 0.f ? (double)in.a : lp;           // (a gradient that hangs on a log-probability that is none)
    by_entropy = (double)in.h;
  } else if (f.kind == kPolicy) {
    // one exponential for both ratios: the old policy's in the even lanes, the reference's in the odd ones
    const double mine = expm1_fine(odd ? (double)in.ref - lp : lp - (double)in.old), other = __shfl_xor(mine, 1);
    const double grown_ref = odd ? mine : other, grown = odd ? other : mine;
    const double A = (double)in.a, ratio = f.old_logprob ? 1.0 + grown : lp == lp ? 1.0 : lp;
    if (A != 0.0) {
      const double free = ratio * A, held = fmin(fmax(ratio, 1.0 - (double)f.clip_low), 1.0 + (double)f.clip_high) * A;
      const bool clipped = held < free;
      loss = -(clipped ? held : free);
      a = clipped ? 0.0 : -free;
    }
    if (f.ref_logprob) {
      const double d = (double)in.ref - lp;
      kl = d < INFINITY ? grown_ref - d : d;
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
  if (writes) {
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
    k0 -= by_kl * (row.apart + row.kl);
    k.k2 = (float)(by_kl * kNat * row.inv_s);
  }
  k.mr = REF ? sums.mr : 0.f;
  k.a = (float)a;
  k.k0 = k0 == 0.0 ? 0.f : (float)(k0 * row.inv_s);      // (nothing of the row enters a gradient of zeros)
  k.m = fabsf(k.k0) < INFINITY ? sums.m : __uint_as_float(0x7fc00001u);      // (every element of a gradient that is no number is none)
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

// ---- sums over positions, of M arrays side by side.
constexpr int kTotalThreads = 1024;
template <int W, int M> struct TotalShared {
  double part[W][M];
};
// By a workgroup, in every thread.  (One wavefront took 0.7 us for each 512 terms: policy step of 200000 rows of 2000 443 -> 308 us.)
template <int M> __device__ __forceinline__ void block_totals(const double* const (&v)[M], int n, double (&t)[M]) {
  constexpr int U = 8 / M, W = kTotalThreads / 64;
  __shared__ TotalShared<W, M> sh;
  const int tid = threadIdx.x;
#pragma unroll
  for (int m = 0; m < M; ++m) t[m] = 0.0;
  for (int base = 0; base < n; base += U * kTotalThreads) {
    double x[M][U];
#pragma unroll
    for (int m = 0; m < M; ++m) {
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int i = base + k * kTotalThreads + tid;
        x[m][k] = i < n ? v[m][i] : 0.0;
      }
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
#pragma unroll
      for (int k = 0; k < U; ++k) t[m] += x[m][k];
    }
  }
#pragma unroll
  for (int m = 0; m < M; ++m) {
    t[m] = wave_sum(t[m]);
    if ((tid & 63) == 0) sh.part[tid >> 6][m] = t[m];
  }
  __syncthreads();
#pragma unroll
  for (int m = 0; m < M; ++m) {
    t[m] = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) t[m] += sh.part[w][m];
  }
}
// By a wavefront, of terms that come from other workgroups of the same launch: 64-bit words that say themselves that they are there (the
// lowest bit of the fraction is set; a cleared word is 0), cleared as they are read.  An infinity travels as the signalling NaN of the bits one
// above its own, which no term is (what arithmetic leaves is a quiet one).
__device__ __forceinline__ double flagged_term(double v) { return __longlong_as_double(__double_as_longlong(v) | 1ll); }
__device__ __forceinline__ double term_of(double flagged) {
  const long long w = __double_as_longlong(flagged);
  return (w & 0x7fffffffffffffffll) == 0x7ff0000000000001ll ? __longlong_as_double(w & ~1ll) : flagged;
}
template <int M> __device__ __forceinline__ void fresh_totals(double* const (&v)[M], int n, double (&t)[M]) {
  constexpr int U = 8 / M;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int m = 0; m < M; ++m) t[m] = 0.0;
  for (int base = 0; base < n; base += U * 64) {
    double x[M][U];
    auto look = [&] {
      bool there = true;
#pragma unroll
      for (int m = 0; m < M; ++m) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const int i = base + k * 64 + lane;
          x[m][k] = i < n ? ld_agent(v[m] + i) : 0.0;
        }
      }
#pragma unroll
      for (int m = 0; m < M; ++m) {
#pragma unroll
        for (int k = 0; k < U; ++k) there = there && (base + k * 64 + lane >= n || (__double_as_longlong(x[m][k]) & 1));
      }
      return __all(there) != 0;
    };
    bool there = look();
    // (all had been sent when the last one was counted: this ends at once, unless calls that share a workspace have not been ordered)
    for (int polls = kWaitPolls; !there && polls > 0; --polls) there = look();
#pragma unroll
    for (int m = 0; m < M; ++m) {
#pragma unroll
      for (int k = 0; k < U; ++k) {
        t[m] += there ? term_of(x[m][k]) : (double)NAN;
        if (base + k * 64 + lane < n) st_agent(v[m] + base + k * 64 + lane, 0.0);
      }
    }
  }
#pragma unroll
  for (int m = 0; m < M; ++m) t[m] = wave_sum(t[m]);
}

// A pair's loss and slope from its sequences' scores (thread 0 writes).
__device__ __forceinline__ void settle_pair(const LossTerm& f, const LossWorkspace& ws, int i, double chosen, double rejected) {
  const int P = f.P;
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
      // ln(1 + e^(-m)) = max(-m, 0) + ln(1 + e^-|m|), and the same of m
      const double E = exp_fine(-fabs(m)), tail = log1p_fine(E), small = E / (1.0 + E), large = 1.0 / (1.0 + E);
      // (a part with factor 0 is left out: it may be infinite)
      loss = tail + (e < 1.0 ? (1.0 - e) * fmax(-m, 0.0) : 0.0) + (e > 0.0 ? e * fmax(m, 0.0) : 0.0);
      slope = beta * (e * (m >= 0.0 ? large : small) - (1.0 - e) * (m >= 0.0 ? small : large));
    }
    if (m != m) loss = slope = m;
  }
  const double w = f.pair_weight ? (double)f.pair_weight[i] : 1.0 / (double)P;
  const double scale = w * (f.grad_scale ? (double)*f.grad_scale : 1.0);
  if (threadIdx.x != 0) return;
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

// Whether this is the last of n to come to a counter, which is zero again then.
__device__ __forceinline__ bool last_of(int32_t* counter, int n) {
  if (!last_to_add(add_arrival(counter), n)) return false;
  set_arrival(counter, 0);
  return true;
}
// Position r is settled (the workgroup's first wavefront): the last of a pair settles the pair; without pairs the last of all adds up the loss.
__device__ __forceinline__ void position_done(const LossRows& rows, const LossTerm& f, const LossWorkspace& ws, int r, double term) {
  if (!f.loss) return;
  const bool first = (threadIdx.x & 63) == 0;
  if (!f.adds_up) {
    if (first) ws.term[r] = term;
    return;
  }
  if (first) st_agent(ws.fresh + r, flagged_term(term));
  if (f.kind == kPreference) {
    const int b = r / rows.T, i = b < f.P ? b : b - f.P;
    if (!last_of(ws.done + 32 + i * ticket_stride(f.P, kAddsUp), 2 * rows.T)) return;
    double* const v[2] = {ws.fresh + i * rows.T, ws.fresh + (f.P + i) * rows.T};
    double score[2];
    fresh_totals<2>(v, rows.T, score);
    settle_pair(f, ws, i, score[0], score[1]);
    return;
  }
  if (!last_of(ws.done, rows.n)) return;
  double* const v[1] = {ws.fresh};
  double t[1];
  fresh_totals<1>(v, rows.n, t);
  if (first) *f.loss = (float)t[0];
}

// Sums of the vectors v0 .. v1 of a row by one wavefront (where the slices' records did not arrive, which never happens to calls that are
// ordered as they have to be).
template <int DT, bool REF> __device__ __noinline__ LossSums wave_sums(const char* row, const char* ref, int V, int v0, int v1) {
  LossSums a = loss_empty();
#pragma unroll 1
  for (int idx = v0 + (threadIdx.x & 63); idx < v1; idx += 64) {
    const uint4 x[1] = {load_vec_of<DT>(row, idx, V)}, xr[1] = {REF ? load_vec_of<DT>(ref, idx, V) : x[0]};
    loss_raise<DT, REF, 1>(a, x, xr);
    loss_push_at<DT, REF>(a, x[0], xr[0]);
  }
  return loss_fold_wave<REF>(a);
}

// The elements behind the last whole vector join the first lane's sums.
template <int DT, bool REF> __device__ __forceinline__ void push_tail(LossSums& a, const char* row, const char* ref, int V) {
  uint4 x[1] = {neutral_vec<DT>()}, xr[1] = {x[0]};
  if ((threadIdx.x & 63) == 0) {
    x[0] = load_last_vec<DT>(row, V);
    xr[0] = REF ? load_last_vec<DT>(ref, V) : x[0];
  }
  loss_raise<DT, REF, 1>(a, x, xr);
  loss_push_at<DT, REF>(a, x[0], xr[0]);
}

// The arrival words of the rows cut into slices: a set for each, however many there are (their last slices wait as those of few rows do: the
// launch has nothing else to do meanwhile.  Counts / sets: log-probabilities of 303 rows of 32003 float 11.4 / 10.9 us, of 256 of 128256 bf16
// of which 0.75 count 15.2 / 14.9, preference loss of 132 rows of 32003 bf16 15.9 / 15.1).
struct SetArrivals {
  uint64_t* base;
  int row;
  static constexpr int rows = 1;
  __device__ __forceinline__ uint64_t* set() const { return base + row; }
  __device__ __forceinline__ int32_t* count() const { return nullptr; }       // (of many rows)
};
// The kernel's arguments, read again where they are needed (they are in the scalar cache).  Held from the start they are more than the scalar
// registers, and each is put aside into a vector register and taken out again.
template <class T> __device__ __forceinline__ T arguments_again() {
  uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return scalar_load(reinterpret_cast<const T*>(at));
}
struct SumsArgs {
  LossRows rows;
  LossTerm f;
  LossWorkspace ws;
  int S, chunk, early;
};
// A slice's vectors come in batches of four per thread, the next batch on its way.
constexpr int kSumsBatch = 4;
template <int DT, bool REF, bool PAST>
__global__ void __launch_bounds__(kBlock) k_loss_sums(SumsArgs args) {
  maxima_without_nans();
  warm_kernargs<sizeof(SumsArgs)>();
  const LossRows& rows = args.rows;
  const int S = args.S, chunk = args.chunk, early = args.early;
  __shared__ LossSums sh[kWaves];
  const int r = blockIdx.x / S, s = blockIdx.x - r * S, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = r / rows.T, t = r - b * rows.T, V = rows.V;
  const PositionMark mark = ask_mark(rows, r);
  PositionIn in = ask_position(rows, args.f, r, b);
  const char* row = row_at<DT>(rows.z, b, t);
  const char* ref = REF ? row_at<DT>(rows.ref, b, t) : nullptr;
  // whole vectors; one that is not is the first thread's of the last slice
  const int whole = V / Elem<DT>::per_vec, v0 = min(s * chunk, whole), v1 = min(v0 + chunk, whole);
  const bool tail = V % Elem<DT>::per_vec != 0 && s == S - 1 && wave == 0;
  uint4 next[kSumsBatch], nextr[kSumsBatch];
  auto load_batch = [&](uint4 (&to)[kSumsBatch], const char* from, int base) {
    if (base + kSumsBatch * kBlock <= v1) {
#pragma unroll
      for (int k = 0; k < kSumsBatch; ++k) to[k] = load_whole<PAST>(from, base + k * kBlock, tid);
    } else {
#pragma unroll
      for (int k = 0; k < kSumsBatch; ++k)
        to[k] = base + k * kBlock + tid < v1 ? load_whole<PAST>(from, base + k * kBlock, tid) : neutral_vec<DT>();
    }
  };
  auto first_batch = [&] {
    load_batch(next, row, v0);
    if (REF) load_batch(nextr, ref, v0);
  };
  if (early) first_batch();
  if (!position_counts(mark)) {
    if (s != 0 || wave != 0) return;
    const SumsArgs late = arguments_again<SumsArgs>();
    if (lane == 0) {
      report_nothing(late.rows, late.f, r);
      late.ws.coef[r] = LossCoef{};
    }
    position_done(late.rows, late.f, late.ws, r, 0.0);
    return;
  }
  if (!early) first_batch();
  ask_logit<DT>(in, row, V);
  LossSums a = loss_empty();
  if (tail) push_tail<DT, REF>(a, row, ref, V);
  for (int base = v0; base < v1; base += kSumsBatch * kBlock) {
    uint4 x[kSumsBatch], xr[kSumsBatch];
#pragma unroll
    for (int k = 0; k < kSumsBatch; ++k) {
      x[k] = next[k];
      xr[k] = REF ? nextr[k] : next[k];
    }
    if (base + kSumsBatch * kBlock < v1) {
      load_batch(next, row, base + kSumsBatch * kBlock);
      if (REF) load_batch(nextr, ref, base + kSumsBatch * kBlock);
    }
    loss_raise<DT, REF, kSumsBatch>(a, x, xr);
#pragma unroll
    for (int k = 0; k < kSumsBatch; ++k)
      if (base + k * kBlock < v1) loss_push_at<DT, REF>(a, x[k], REF ? xr[k] : x[k]);
  }
  a = loss_fold_wave<REF>(a);
  if (lane == 0) sh[wave] = a;
  __syncthreads();
  if (wave != 0) return;
  const SumsArgs late = arguments_again<SumsArgs>();
  const LossTerm& f = late.f;
  const LossWorkspace& ws = late.ws;
  a = loss_fold_wave<REF>(lane < kWaves ? sh[lane] : loss_empty());
  if (S > 1) {
    uint64_t w[kXchgWords];
    bool arrived = true;
    pack_pair(PairRecord{a.m, a.s, a.u, REF ? a.mr : a.m, REF ? a.sr : 0.f, REF ? a.w : 0.f}, w);
    if (!hand_off(PlainWords{ws.xchg + (size_t)r * S * kXchgWords}, s, S, SetArrivals{ws.sets, r}, f.wait, [] {}, w, arrived))
      return;
    a = loss_empty();
    if (lane < S) {
      const PairRecord p = unpack_pair(w);
      a = LossSums{p.mp, p.sp, p.up, p.uq, p.mq, p.sq};
    }
    a = loss_fold_wave<REF>(a);
    if (__builtin_expect(!arrived, 0)) a = wave_sums<DT, REF>(row, ref, V, 0, vectors_of<DT>(V));
  }
  double term;
  const LossCoef k = settle_position<REF>(late.rows, f, r, in, a, S > 1 ? 4 : 3, lane == 0, term);
  if (lane == 0) ws.coef[r] = k;
  position_done(late.rows, f, ws, r, term);
}

__global__ void __launch_bounds__(kTotalThreads) k_loss_pairs(LossTerm f, int T, LossWorkspace ws) {
  const int i = blockIdx.x;
  const double* const v[2] = {ws.term + (size_t)i * T, ws.term + (size_t)(f.P + i) * T};
  double score[2];
  block_totals<2>(v, T, score);
  settle_pair(f, ws, i, score[0], score[1]);
}
__global__ void __launch_bounds__(kTotalThreads) k_loss_total(const double* terms, int n, float* out) {
  const double* const v[1] = {terms};
  double t[1];
  block_totals<1>(v, n, t);
  if (threadIdx.x == 0) *out = (float)t[0];
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {       // nearest, ties to even
  const bf16x2 v = __builtin_convertvector((floatx2{a, b}), bf16x2);
  uint32_t r;
  __builtin_memcpy(&r, &v, 4);
  return r;
}
// A whole vector of gradients, or the elements of the last one that the row has.  Stored past the caches: a gradient of more than a few
// hundred rows does not stay in them till it is read, and takes the place of logits that are still to be read (8192 rows of
// 128256 bf16 780 -> 738 us, preference loss of 512 rows of 128256 float 160 -> 129, KL over 1024 rows of 152064 229 -> 215).
template <int DT> __device__ __forceinline__ void grad_words(const float (&g)[Elem<DT>::per_vec], uint32_t (&w)[4]) {
  constexpr int EPV = Elem<DT>::per_vec;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DT == ADASD_BF16) w[i] = pack_bf16(g[2 * i % EPV], g[(2 * i + 1) % EPV]);
    else w[i] = __float_as_uint(g[i]);
  }
}
template <int DT> __device__ __forceinline__ void store_whole(char* row, int at, int lane, const float (&g)[Elem<DT>::per_vec]) {
  uint32_t w[4];
  grad_words<DT>(g, w);
  vec16_any v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = w[i];
  __builtin_nontemporal_store(v, reinterpret_cast<vec16_any*>(row + (size_t)at * 16 + (uint32_t)lane * 16u));
}
template <int DT> __device__ __forceinline__ void store_grad(char* row, int idx, int V, const float (&g)[Elem<DT>::per_vec]) {
  constexpr int EPV = Elem<DT>::per_vec;
  if (idx < V / EPV) return store_whole<DT>(row, idx, 0, g);
  uint32_t w[4];
  grad_words<DT>(g, w);
#pragma unroll
  for (int i = 0; i < EPV - 1; ++i) {
    const int j = idx * EPV + i;
    if (j >= V) break;
    if (DT == ADASD_BF16) reinterpret_cast<uint16_t*>(row)[j] = (uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2]);
    else reinterpret_cast<uint32_t*>(row)[j] = w[i];
  }
}

// The gradients of one vector, but for the token's a: e (k0 + k1 t + k2 dd).  (Where e is 0 they are 0; a row whose k0 is no number has no m either.)
template <int DT, bool ENT, bool REF>
__device__ __forceinline__ void grad_vec(const uint4& x, const uint4& xr, const LossCoef& k, float (&g)[Elem<DT>::per_vec]) {
  const float neg_m = -k.m, neg_mr = -k.mr;
#pragma unroll
  for (int h = 0; h < Elem<DT>::per_vec / 4; ++h) {
    float z[4], t[4], e[4], q[4];
    unpack4<DT>(x, h, z);
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = fma_log2e(z[i], neg_m);
    ex2_group(t, e);
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = ENT ? fmaf(k.k1, t[i], k.k0) : k.k0;
    if (REF) {
      float y[4];
      unpack4<DT>(xr, h, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = fmaf(k.k2, t[i] - fma_log2e(y[i], neg_mr), q[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) g[4 * h + i] = ENT || REF ? mass_times(e[i], q[i]) : e[i] * q[i];
  }
}

// Whether the gradient row is zeros, whatever the logits are.
__device__ __forceinline__ bool zero_row(const LossCoef& k) { return k.a == 0.f && k.k0 == 0.f && k.k1 == 0.f && k.k2 == 0.f; }
template <int DT> __device__ __forceinline__ void zero_vec(char* row, int idx, int V) {
  const float g[Elem<DT>::per_vec] = {};
  store_grad<DT>(row, idx, V, g);
}
template <int DT, bool REF>
__device__ __forceinline__ void form_grad(const uint4& z, const uint4& zr, const LossCoef& k, bool ent, float (&g)[Elem<DT>::per_vec]) {
  if (ent) grad_vec<DT, true, REF>(z, zr, k, g);
  else grad_vec<DT, false, REF>(z, zr, k, g);
}
template <int DT, bool REF>
__device__ __forceinline__ void emit_vec(char* out, int idx, int V, int x, const uint4& z, const uint4& zr, const LossCoef& k, bool ent) {
  constexpr int EPV = Elem<DT>::per_vec;
  float g[EPV];
  form_grad<DT, REF>(z, zr, k, ent, g);
  if (idx == x / EPV) {
#pragma unroll
    for (int i = 0; i < EPV; ++i) g[i] += idx * EPV + i == x ? k.a : 0.f;
  }
  store_grad<DT>(out, idx, V, g);
}

// Pieces of rows of `per` vectors, a wavefront each, from the last row to the first: the rows read last are still in the cache behind the L2s
// (preference loss of 2048 rows of 128256 bf16 of which 0.67 count: 210 -> 206 us).
constexpr int kPiece = 8 * 64, kMostPieces = 2048;      // (2^20 rows: no more than 2^31 pieces)
constexpr uint32_t kMostGroups = 1u << 22;
constexpr int kResidentWaves = 8 * 4 * 256;
constexpr int kGradAddsUp = 4096;     // pairs whose sum is formed beside the gradient, by one wavefront
template <int DT, bool REF, bool PAST>
__global__ void __launch_bounds__(kBlock) k_loss_grad(LossRows rows, int pieces, int per, LossWorkspace ws, int P, float* loss, int ent) {
  warm_kernargs<sizeof(LossRows) + 4 * sizeof(int) + sizeof(LossWorkspace) + sizeof(float*)>();
  const int lane = threadIdx.x & 63, V = rows.V, nv = vectors_of<DT>(V);
  const uint32_t step = (gridDim.x - (loss ? 1u : 0u)) * kWaves, units = (uint32_t)rows.n * (uint32_t)pieces;
  if (loss && blockIdx.x == gridDim.x - 1) {         // (the pairs' sum; its workgroup is one more than the rows take)
    if (threadIdx.x >= 64) return;
    double total = 0.0;
    for (int i = lane; i < P; i += 64) total += ws.pair[i];
    total = wave_sum(total);
    if (lane == 0) *loss = (float)total;
    return;
  }
  for (uint32_t unit = blockIdx.x * kWaves + uniform(threadIdx.x >> 6); unit < units; unit += step) {
    const uint32_t back = units - 1 - unit;
    const int r = (int)(back / (uint32_t)pieces), piece = (int)(back - (uint32_t)r * (uint32_t)pieces), b = r / rows.T, t = r - b * rows.T;
    LossCoef k = scalar_load(ws.coef + r);
    if (P > 0 && !zero_row(k)) {       // (a pair's slope, sequence by sequence; it may be no number, and this position one that does not count)
      const float d = scalar_load(ws.seq + b);
      k.a = d == 0.f ? 0.f : k.a * d;
      k.k0 = d == 0.f ? 0.f : k.k0 * d;
    }
    char* out = const_cast<char*>(row_at<DT>(rows.g, b, t));
    const char* row = row_at<DT>(rows.z, b, t);
    const char* ref = REF ? row_at<DT>(rows.ref, b, t) : nullptr;
    const int v0 = piece * per, v1 = min(v0 + per, nv);
    if (zero_row(k)) {
      for (int idx = v0 + lane; idx < v1; idx += 64) zero_vec<DT>(out, idx, V);
      continue;
    }
    const int x = rows.tokens[r];
    for (int idx = v0 + lane; idx < v1; idx += 64) {
      const uint4 z = idx < V / Elem<DT>::per_vec ? load_whole<PAST>(row, idx, 0) : load_last_vec<DT>(row, V);
      emit_vec<DT, REF>(out, idx, V, x, z, REF ? load_vec_of<DT>(ref, idx, V) : z, k, ent);
    }
  }
}

// ---- Everything in one launch, where a gradient row needs nothing but its own row.  A workgroup of four wavefronts has 4 / WPR rows, or
// (WPR = 4, S > 1) a slice of one.  The raw vectors, up to NB per thread and row, stay in its registers from the load to the gradient.
//
// The slices hand their sums to one workgroup (hand_off); it settles the position and sends the numbers of the gradient row to each of the
// others, into words that this slice alone reads and clears.  (All slices reading all records: 16 x 128256 in 63 slices waited 7.4 us for
// them; a count of those that have read one result, kept to clear it: 4.5 us more.)  Slices of a row are consecutive workgroups, and
// workgroups are started in order on each die, so who is waited for has mostly started; but other streams' work may hold the chip, and two calls
// that wait on two streams could hold each other's places.  So every wait is bounded: a slice that has waited in vain leaves a mark in
// the place of its result and ends, and who comes to send the result finds the mark and does the slice's part as well, from the logits
// (which are whole there: only the slice itself would have put its gradient in their place).
template <int W> struct JoinShared {
  LossSums sums[W];
  LossCoef coef[kWaves];
  int role;             // of a slice
  uint64_t left;        // slices whose part is to be done as well
};
enum { kWaitsFor = 0, kSettles = 1, kLeaves = 2 };
constexpr uint64_t kLeft = 2;        // in a result's first word: its slice has ended without it
// The slice's result, waited for and cleared (one wavefront).  False: the mark is left.
__device__ __forceinline__ bool await_result(uint64_t* at, WordWait wait, LossCoef& k) {
  const int lane = threadIdx.x & 63;
  uint64_t w = 1;
  auto look = [&](int polls) {
    for (;; --polls) {
      if (lane < kResultWords) w = __hip_atomic_load(at + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (__all((w & 1ull) != 0)) return true;
      if (polls <= 0) return false;
      __builtin_amdgcn_s_sleep(1);
    }
  };
  if (!look(wait == kWaits ? kWaitPolls : 0)) {
    uint64_t seen = 0;
    if (exchange_arrival(at, seen, kLeft)) return false;
    if (!look(kWaitPolls)) return false;          // (the result's other words have been sent with its first)
  }
  if (lane < kResultWords) __hip_atomic_store(at + lane, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  k.m = lane_value(word_lo(w), 0);
  k.a = lane_value(word_hi(w), 0);
  k.mr = lane_value(word_lo(w), 1);
  k.k0 = lane_value(word_hi(w), 1);
  k.k1 = lane_value(word_hi(w), 2);
  k.k2 = lane_value(word_hi(w), 3);
  return true;
}
// The result to all slices but `own`, lane by lane.  Returns what stood in the first word (kLeft: the slice has ended).
__device__ __forceinline__ uint64_t send_results(uint64_t* at, int S, int own, const LossCoef& k) {
  const int lane = threadIdx.x & 63;
  if (lane >= S || lane == own) return 0;
  at += lane * kResultWords;
  __hip_atomic_store(at + 1, record_word(bits_of(k.mr) | 1u, k.k0), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(at + 2, record_word(1u, k.k1), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(at + 3, record_word(1u, k.k2), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return __hip_atomic_exchange(at, record_word(bits_of(k.m), k.a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

struct JoinArgs {
  LossRows rows;
  LossTerm f;
  LossWorkspace ws;
  int S, chunk, ent, early;
};
// Wavefronts per SIMD that the registers are limited for (64 of data and about 50 more: four; 16: eight).
constexpr int join_waves(int nb, bool ref) { return !ref ? (nb <= 4 ? 8 : nb <= 8 ? 6 : 4) : (nb <= 2 ? 7 : nb <= 4 ? 5 : 4); }
template <int DT, bool REF, int NB, int WPR, bool PAST>
__global__ void __launch_bounds__(WPR > kWaves ? 64 * WPR : kBlock, join_waves(NB, REF))
k_loss_join(JoinArgs args) {
  maxima_without_nans();
  warm_kernargs<sizeof(JoinArgs)>();
  const LossRows& rows = args.rows;
  const int S = args.S, chunk = args.chunk, early = args.early;
  constexpr int RPB = WPR < kWaves ? kWaves / WPR : 1, TR = 64 * WPR;          // rows per workgroup, threads per row
  __shared__ JoinShared<WPR < kWaves ? kWaves : WPR> sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), V = rows.V;
  constexpr int EPV = Elem<DT>::per_vec;
  const int r0 = RPB > 1 ? blockIdx.x * RPB : blockIdx.x / S, s = RPB > 1 ? 0 : blockIdx.x - r0 * S;
  const int sub = wave / WPR, r = r0 + sub, me = tid & (TR - 1);
  const bool here = r < rows.n;
  const int b = here ? r / rows.T : 0, t = here ? r - b * rows.T : 0;
  const int r_here = here ? r : 0;
  const PositionMark mark = ask_mark(rows, r_here);
  int x = rows.tokens[r_here];
  const char* row = row_at<DT>(rows.z, b, t);
  const char* ref = REF ? row_at<DT>(rows.ref, b, t) : nullptr;
  // whole vectors; one that is not is the first thread's of the last slice
  const int whole = V / EPV, v0 = min(s * chunk, whole), v1 = min(v0 + chunk, whole);
  const bool tail = V % EPV != 0 && s == S - 1 && wave % WPR == 0;
  // what the positions are settled from, a pair of lanes for each row of the workgroup
  const int i = RPB > 1 ? min(lane >> 1, RPB - 1) : 0, ri = min(r0 + i, rows.n - 1), bi = ri / rows.T;
  PositionIn in{};
  PositionMark mark_i = mark;
  if (wave == 0 && s == S - 1) {
    in = ask_position(rows, args.f, ri, bi);
    if (RPB > 1) mark_i = ask_mark(rows, ri);
  }
  uint4 v[NB], q[NB];
  auto load_row = [&] {
    auto load = [&](const char* from, int j) {
      const int at = v0 + j * TR;
      if (at + TR <= v1) return load_whole<PAST>(from, at, me);
      return at + me < v1 ? load_whole<PAST>(from, at, me) : neutral_vec<DT>();
    };
#pragma unroll
    for (int j = 0; j < NB; ++j) v[j] = load(row, j);
    if (REF) {
#pragma unroll
      for (int j = 0; j < NB; ++j) q[j] = load(ref, j);
    }
  };
  if (early) load_row();
  const bool on = here && position_counts(mark), on_i = RPB > 1 ? r0 + i < rows.n && position_counts(mark_i) : on;
  if (on && !early) load_row();
  if (wave == 0 && on_i && s == S - 1) ask_logit<DT>(in, row_at<DT>(rows.z, bi, ri - bi * rows.T), V);
  if (on) {
    LossSums a = loss_empty();
    if (tail) push_tail<DT, REF>(a, row, ref, V);
    loss_raise<DT, REF, NB>(a, v, REF ? q : v);
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (v0 + j * TR < v1) loss_push_at<DT, REF>(a, v[j], REF ? q[j] : v[j]);
    a = loss_fold_wave<REF>(a);
    if (lane == 0) sh.sums[wave] = a;
  }
  __syncthreads();
  x = uniform(x);
  double term = 0.0;
  bool settles = S == 1;
  uint64_t found = 0;
  if (wave == 0) {
    const JoinArgs late = arguments_again<JoinArgs>();
    const LossRows& rows = late.rows;
    const LossTerm& f = late.f;
    const LossWorkspace& ws = late.ws;
    uint64_t* words = ws.xchg + (size_t)r * S * (kXchgWords + kResultWords);      // (S > 1: the records, then the results)
    uint64_t* results = words + S * kXchgWords;
    LossCoef k{};
    int role = kWaitsFor;
    if (RPB > 1 || on) {
      LossSums a;
      if (WPR > kWaves) {
        a = loss_fold_wave<REF>(lane < WPR ? sh.sums[lane] : loss_empty());
      } else {
        a = sh.sums[i * WPR];
#pragma unroll
        for (int n = 1; n < WPR; ++n) a = loss_merge<REF>(a, sh.sums[i * WPR + n]);
      }
      if (RPB == 1 && S > 1) {
        a.m = odd_bit(a.m);
        if (REF) a.mr = odd_bit(a.mr);
        bool arrived = true;
        uint64_t w[kXchgWords];
        pack_pair(PairRecord{a.m, a.s, a.u, REF ? a.mr : a.m, REF ? a.sr : 0.f, REF ? a.w : 0.f}, w);
        settles = hand_off(PlainWords{words}, s, S, SetArrivals{ws.sets, r}, f.wait,
                           [&] {
                             if (s == S - 1) return;
                             in = ask_position(rows, f, r, b);
                             ask_logit<DT>(in, row, V);
                           },
                           w, arrived);
        if (settles) {
          a = loss_empty();
          if (lane < S) {
            const PairRecord p = unpack_pair(w);
            a = LossSums{p.mp, p.sp, p.up, p.uq, p.mq, p.sq};
          }
          a = loss_fold_wave<REF>(a);
          if (__builtin_expect(!arrived, 0)) a = wave_sums<DT, REF>(row, ref, V, 0, vectors_of<DT>(V));
        } else if (!await_result(results + s * kResultWords, f.wait, k)) {
          role = kLeaves;
        }
      }
      if (settles) {
        role = kSettles;
        const bool writes = on_i && (RPB > 1 ? !(lane & 1) && lane < 2 * RPB : lane == 0);
        const LossCoef settled = settle_position<REF>(rows, f, ri, in, a, WPR > 1 ? (S > 1 ? 4 : 3) : 2, writes, term);
        if (on_i) k = settled;
        else term = 0.0;
        if (RPB == 1 && S > 1) found = send_results(results, S, s, k);
      }
    }
    if (RPB > 1 ? !(lane & 1) && lane < 2 * RPB && r0 + i < rows.n : lane == 0) {
      sh.coef[i] = k;
      sh.role = role;
      if (!on_i && s == 0) report_nothing(rows, f, ri);
      if (!rows.g.base) ws.coef[ri] = k;
      if (RPB > 1 && f.loss) ws.term[ri] = term;
    }
  }
  __syncthreads();
  if (!here || (RPB == 1 && sh.role == kLeaves)) return;
  const JoinArgs last = arguments_again<JoinArgs>();
  const int ent = last.ent;
  char* out = last.rows.g.base ? const_cast<char*>(row_at<DT>(last.rows.g, b, t)) : nullptr;
  const LossCoef k = sh.coef[sub];
  // (beside the other wavefronts' part of the gradient)
  if (RPB == 1 && wave == 0 && (sh.role == kSettles || (!on && s == 0))) position_done(last.rows, last.f, last.ws, r, term);
  int from = v0;
  asm("" : "+s"(from));          // (else the places of the loads are kept in scalar registers for the stores, more than there are)
  if (out) {
    const float none[EPV] = {};
    if (zero_row(k)) {
      for (int at = from; at + me < v1; at += TR) store_whole<DT>(out, at, me, none);
      if (tail && lane == 0) store_grad<DT>(out, whole, V, none);
    } else {
      const int x_at = x >= 0 ? x / EPV : -1, x_in = x & (EPV - 1);       // (uniform)
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int at = from + j * TR;
        if (at + me < v1) {
          float g[EPV];
          form_grad<DT, REF>(v[j], REF ? q[j] : v[j], k, ent, g);
          if (x_at >= at && x_at < at + TR) {
            const float a = x_at == at + me ? k.a : 0.f;
#pragma unroll
            for (int i = 0; i < EPV; ++i) g[i] += i == x_in ? a : 0.f;
          }
          store_whole<DT>(out, at, me, g);
        }
      }
      if (tail && lane == 0) {          // (its logits, from memory again: nobody has put a gradient there)
        const uint4 z = load_last_vec<DT>(row, V);
        emit_vec<DT, REF>(out, whole, V, x, z, REF ? load_last_vec<DT>(ref, V) : z, k, ent);
      }
    }
  }
  if (RPB > 1 || S == 1 || !on || sh.role != kSettles) return;
  // ---- the slices that have ended without their results
  uint64_t* results = last.ws.xchg + (size_t)r * S * (kXchgWords + kResultWords) + S * kXchgWords;
  if (wave == 0) {
    uint64_t left = __ballot(found == kLeft);
    if (lane == 0) sh.left = left;
    if (found == kLeft) {
#pragma unroll
      for (int n = 0; n < kResultWords; ++n)
        __hip_atomic_store(results + lane * kResultWords + n, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  __syncthreads();
  for (uint64_t left = sh.left; __builtin_expect(left != 0, 0); left &= left - 1) {
    const int other = __ffsll((long long)left) - 1, nv = vectors_of<DT>(V), u0 = min(other * chunk, nv), u1 = other == S - 1 ? nv : min(u0 + chunk, nv);
#pragma unroll 1
    for (int idx = u0 + tid; idx < u1; idx += TR) {
      if (zero_row(k)) {
        zero_vec<DT>(out, idx, V);
        continue;
      }
      const uint4 z = load_vec_of<DT>(row, idx, V);
      emit_vec<DT, REF>(out, idx, V, x, z, REF ? load_vec_of<DT>(ref, idx, V) : z, k, ent);
    }
  }
}

// How k_loss_join cuts rows of nv vectors: wavefronts per row, vectors in registers per thread, slices (0: too long) and vectors per slice.  (Each line's
// figures are of one build, the one it was decided in; later steps took 2 to 6 % off both sides.)
//  * Few rows: as many slices as are resident together, of eight wavefronts and up to 8 vectors per thread (with a reference's row four
//    wavefronts and up to 4 + 4); where those would not all be, and would be with twice the vectors, that.  (Us a call, eight wavefronts x 8 / four x
//    16: 64 rows of 32000 bf16 9.6 / 11.6, 512 19.7 / 21.2, 256 of 32003 float 18.8 / 21.0, 256 of 128256 bf16 30.6 / 28.4.  With a
//    reference, 4 + 4 / 8 + 8: 64 of 32000 11.8 / 14.7, 128 14.8 / 16.8, but 256 of 128256 64 / 59.)
//  * Many short rows: as few wavefronts per row as hold it, with as few registers as it takes (rows of 2000 bf16, four wavefronts
//    each / one / one of few registers: 200000 rows 752 / 432 / 304 us; of 8000, four / two / one: 50000 rows 428 / 303 / 282).
//  * Many long rows: eight wavefronts of 8 vectors per thread where those hold the row, else slices of four.  Bytes on their way are what the
//    chip's rate takes, and a workgroup asks for nothing while it exchanges sums and settles, so that several should take turns.
//    8192 rows of 128256 bf16, workgroups of 4 wavefronts x 16 vectors / 4 x 8 / 8 x 16 / 8 x 8 / 16 x 16 (no slices): 722 / 701 / 811 / 738 / 828 us;
//    2048 of which 0.7 count 169 / 159 / 176 / 166 / 192; 2624 rows of 152064 275 / 284 / 302 / 278 / 412.
//  * With a reference's row, twice the registers: four wavefronts of 8 + 8 vectors (1024 rows of 152064 bf16, 4 x (4 + 4) / 4 x (8 + 8) /
//    8 x (8 + 8): 299 / 222 / 234 us), eight where they hold the row (12480 rows of 32000 bf16 474 us, two slices 508).
struct JoinPlan {
  int wpr, nb, S, chunk;
};
JoinPlan join_plan(int n, int nv, bool ref) {
  const int most = ref ? 8 : 16, wpr_few = ref ? 4 : 8, nb_few = ref ? 4 : 8;
  const int64_t resident = ref ? 5 * 256 : 3 * 256;
  for (int turns = 1; turns <= nb_few; ++turns) {
    const int lanes = 64 * wpr_few * turns, S = (nv + lanes - 1) / lanes;
    if (S <= kMaxSplit && (int64_t)S * n <= resident) return {wpr_few, nb_few, S, slice_chunk(nv, S)};
  }
  for (int turns = nb_few + 1; turns <= most; ++turns) {
    const int S = (nv + turns * kBlock - 1) / (turns * kBlock);
    if (S <= kMaxSplit && (int64_t)S * n <= 4 * 256) return {4, most, S, slice_chunk(nv, S)};
  }
  for (int nb = most / 4; nb <= most; nb *= 2)
    if (nv <= 64 * nb) return {1, nb, 1, nv};
  if (nv <= 128 * most) return {2, most, 1, nv};
  if (ref && nv <= 256 * most) return {4, most, 1, nv};
  if (nv <= 512 * 8) return {8, 8, 1, nv};
  const int wpr = ref || nv <= kMaxSplit * 2048 ? 4 : 8, S = (nv + 512 * wpr - 1) / (512 * wpr);
  return {wpr, 8, S <= kMaxSplit ? S : 0, slice_chunk(nv, S)};
}

}  // namespace

// Logits of so many bytes are read past the caches.  Gradients of one launch read them once (1024 rows of 152064 bf16 and a reference's 223 -> 215
// us, 200000 rows of 2000 321 -> 306; 385 rows of 32003 float and a reference's, 50 MB each, which the cache behind the L2s can hold from
// the kernel that wrote them, took 35 us that way and 34 without).  Log-probabilities are often asked for ahead of a gradient, so only
// what that cache cannot hold (4096 rows of 128256 bf16 of which 0.64 count 123 -> 110); the second read of a preference loss likewise
// (200000 rows of 2000 bf16 480 -> 442 us; 256 of 128256, were it done there, 44 -> 45).
// Of so few bytes the logits are asked for before it is known whether their position counts: one latency less.
constexpr int64_t kEarly = (int64_t)16 << 20;
constexpr int64_t kJoinPast = (int64_t)64 << 20, kSumsPast = (int64_t)256 << 20;

hipError_t launch_loss(const LossRows& rows, int dt, LossTerm f, const LossWorkspace& ws, hipStream_t st) {
  const int n = rows.n, epv = dt == ADASD_BF16 ? 8 : 4, nv = (rows.V + epv - 1) / epv;
  const bool ref = rows.ref.base != nullptr, ent = f.kind == kPolicy ? f.entropy_coef != 0.f : f.kind == kLogprob && f.dentropy;
  const bool by_ref = ref && f.kl_coef != 0.f;
  const bool grad = rows.g.base != nullptr, own_row = grad && f.kind != kPreference && ref == by_ref;
  const dim3 block(kBlock);
  const JoinPlan plan = join_plan(n, nv, ref);
  const bool join = n > 0 && plan.S > 0 && (plan.S == 1 || (int64_t)plan.S * n <= ws.slices) && (own_row || plan.wpr < 4);
  const int64_t bytes = (int64_t)n * nv * 16;
  const bool early = bytes <= kEarly;
  const bool past = join ? own_row && bytes > kJoinPast : f.kind == kLogprob && bytes > kSumsPast;
  f.adds_up = f.loss && n > 0 && (join ? plan.wpr >= kWaves && n <= kJoinAddsUp : n <= kAddsUp);
  if (join) {
    LossRows some = rows;
    if (!own_row) some.g = RowPlace{};
    const unsigned groups = plan.wpr >= kWaves ? n * plan.S : (n + kWaves / plan.wpr - 1) / (kWaves / plan.wpr);
#define ADASD_JOIN_CASE(DTV, REFV, NBV, WPRV, PASTV) \
    if (dt == DTV && ref == REFV && plan.nb == NBV && plan.wpr == WPRV && past == PASTV) \
      launch_kernel((k_loss_join<DTV, REFV, NBV, WPRV, PASTV>), dim3(groups), dim3(WPRV > kWaves ? 64 * WPRV : kBlock), st, \
                    JoinArgs{some, f, ws, plan.S, plan.chunk, ent ? 1 : 0, early ? 1 : 0});
#define ADASD_JOIN_FEW(REFV, NBV, WPRV) \
    ADASD_JOIN_CASE(ADASD_BF16, REFV, NBV, WPRV, false) ADASD_JOIN_CASE(ADASD_F32, REFV, NBV, WPRV, false)
#define ADASD_JOIN_CASES(REFV, NBV, WPRV) \
    ADASD_JOIN_FEW(REFV, NBV, WPRV) ADASD_JOIN_CASE(ADASD_BF16, REFV, NBV, WPRV, true) ADASD_JOIN_CASE(ADASD_F32, REFV, NBV, WPRV, true)
    ADASD_JOIN_CASES(false, 4, 1) ADASD_JOIN_CASES(false, 8, 1) ADASD_JOIN_CASES(false, 16, 1) ADASD_JOIN_CASES(false, 16, 2)
    ADASD_JOIN_CASES(false, 8, 4) ADASD_JOIN_CASES(false, 8, 8)
    ADASD_JOIN_CASES(true, 2, 1) ADASD_JOIN_CASES(true, 4, 1) ADASD_JOIN_CASES(true, 8, 1) ADASD_JOIN_CASES(true, 8, 2)
    ADASD_JOIN_CASES(true, 8, 4) ADASD_JOIN_CASES(true, 8, 8)
    // (of few rows alone: 1024 slices of 4096 vectors, 64 MiB, at the most; 1280 of 1024)
    ADASD_JOIN_FEW(false, 16, 4) ADASD_JOIN_FEW(true, 4, 4)
#undef ADASD_JOIN_CASES
#undef ADASD_JOIN_FEW
#undef ADASD_JOIN_CASE
  } else if (n > 0) {
    const int S = scan_split(n, rows.V, dt), chunk = slice_chunk(nv, S);
#define ADASD_LOSS_CASE(DTV, REFV, PASTV) \
    if (dt == DTV && ref == REFV && past == PASTV) \
      launch_kernel((k_loss_sums<DTV, REFV, PASTV>), dim3(n * S), block, st, SumsArgs{rows, f, ws, S, chunk, early ? 1 : 0});
    ADASD_LOSS_CASE(ADASD_BF16, false, false) ADASD_LOSS_CASE(ADASD_BF16, true, false) ADASD_LOSS_CASE(ADASD_F32, false, false)
    ADASD_LOSS_CASE(ADASD_F32, true, false) ADASD_LOSS_CASE(ADASD_BF16, false, true) ADASD_LOSS_CASE(ADASD_F32, false, true)
#undef ADASD_LOSS_CASE
  }
  const bool pairs = f.kind == kPreference, grad_adds_up = pairs && grad && n > 0 && f.P <= kGradAddsUp;
  if (pairs && n > 0 && !f.adds_up) launch_kernel(k_loss_pairs, dim3(f.P), dim3(kTotalThreads), st, f, rows.T, ws);
  if (grad && n > 0 && !(join && own_row)) {
    // as many vectors per lane as leave each resident wavefront a piece, up to 8
    const int64_t lanes = ((int64_t)n * nv + kResidentWaves - 1) / kResidentWaves;
    const int fair = (int)min((int64_t)kPiece, (lanes + 63) / 64 * 64);
    const int per = max(fair, ((nv + kMostPieces - 1) / kMostPieces + 63) / 64 * 64), pieces = (nv + per - 1) / per;
    const uint32_t groups = ((uint32_t)n * (uint32_t)pieces + kWaves - 1) / kWaves;
    const bool last_past = bytes > kSumsPast;
    const dim3 grid((groups < kMostGroups ? groups : kMostGroups) + (grad_adds_up ? 1 : 0));
#define ADASD_GRAD_CASE(DTV, REFV, PASTV) \
    if (dt == DTV && by_ref == REFV && last_past == PASTV) \
      launch_kernel((k_loss_grad<DTV, REFV, PASTV>), grid, block, st, rows, pieces, per, ws, pairs ? f.P : 0, grad_adds_up ? f.loss : nullptr, \
                    ent ? 1 : 0);
    ADASD_GRAD_CASE(ADASD_BF16, false, false) ADASD_GRAD_CASE(ADASD_BF16, true, false) ADASD_GRAD_CASE(ADASD_F32, false, false)
    ADASD_GRAD_CASE(ADASD_F32, true, false) ADASD_GRAD_CASE(ADASD_BF16, false, true) ADASD_GRAD_CASE(ADASD_BF16, true, true)
    ADASD_GRAD_CASE(ADASD_F32, false, true) ADASD_GRAD_CASE(ADASD_F32, true, true)
#undef ADASD_GRAD_CASE
  }
  if (f.loss && (pairs ? !grad_adds_up : !f.adds_up))
    launch_kernel(k_loss_total, dim3(1), dim3(kTotalThreads), st, (const double*)(pairs ? ws.pair : ws.term), n == 0 ? 0 : pairs ? f.P : n, f.loss);
  return hipGetLastError();
}

}  // namespace adasd
