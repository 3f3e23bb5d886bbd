// Device helpers of the losses over vocabulary rows: partial sums of a slice of a row, their fold, and the gradient of a position.
//
// With x = z log2(e) (the float constant, see finish_loss_row) and m the largest x of the row, e_j = 2^(x_j - m):
//   s = sum e_j,   u = sum (x_j - m) e_j            log-normaliser and entropy,
//   w = sum e_j dd_j,  dd_j = (x_j - m) - (xr_j - mr)   (reference row zr, with its own mr) for the KL over the vocabulary.
// Each logit is taken about its own row's reference first: softmax does not see a row's offset, and the difference of two logits with different ones has
// lost what the KL is formed from (offsets of 300 and -300: 1e-3 of the KL, of 3e5 a tenth).
// The gradient of every loss here with respect to a row is
//   dz_j = a 1[j = x] + e_j (k0 + k1 (x_j - m) + k2 dd_j)
// with six numbers per position (m and mr among them): a is the derivative by the token's log-probability, k0 gathers -a and the constants of the
// entropy's and the KL's derivatives, k1 is the entropy's, k2 the KL's coefficient, all three over s.
#pragma once
#include "internal.h"
#include "stats_device.h"

namespace adasd {

struct LossSums {          // of a slice
  float m, s, u, w;        // of the row
  float mr, sr;            // of the reference's row
};
// Every reference has its lowest bit set (the flag of the hand-off words), from the first on: brought about afterwards it would cost each fold
// a factor next to 1 and two roundings.
__device__ __forceinline__ float odd_bit(float v) { return __uint_as_float(__float_as_uint(v) | 1u); }
// A row whose largest logit is beyond 2^26 in size is none of numbers here: a unit in the last place of m (8 at the border) is no small exponent.
constexpr float kLargestM = 67108864.f * kLog2e + 16.f;
// The lowest reference of any part of a row, below -kLargestM: a row that ends with it is none of numbers either.  Logits far below it (masks, of
// whatever finite value) have no mass about it, and a part of a row that holds nothing else stays at 0.  Were references to follow such
// logits, they would be off by up to a unit in their last place, which from 2^31 on is an exponent past the type's range; and the difference of two
// of them times a sum would pass it in the folds.  (-2^27: a unit is 16 there, e at most 2^24.)
constexpr float kLowestM = -134217728.f;
__device__ __forceinline__ LossSums loss_empty() { return LossSums{odd_bit(kLowestM), 0.f, 0.f, 0.f, odd_bit(kLowestM), 0.f}; }

// e v, and 0 where e is 0, whatever v is (a token, or a part of a row, without mass: v may be infinite, or no number).  One instruction; a comparison, a selection
// and the product were three.
__device__ __forceinline__ float mass_times(float e, float v) {
  float r;
  asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(r) : "v"(e), "v"(v));
  return r;
}

// One vector of the row (and of the reference's) joins a lane's sums, about the references that the sums have.  The vector's sums are
// formed on their own, so that a chain of additions is one per vector long.
template <int DT, bool REF>
__device__ __forceinline__ void loss_push_at(LossSums& a, const uint4& x, const uint4& xr) {
  constexpr int EPV = Elem<DT>::per_vec;
  const float neg_m = -a.m, neg_mr = -a.mr;
  float s[2], u[2], w[2], sr[2];
  auto join = [](float& sum, float v, bool first) { sum = first ? v : sum + v; };
#pragma unroll
  for (int g = 0; g < EPV / 4; ++g) {
    float z[4], t[4], e[4];
    unpack4<DT>(x, g, z);
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = fma_log2e(z[i], neg_m);
    ex2_group(t, e);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float held = max_raw(t[i], -200.f);                    // (masked logits: (-200) * 0 = 0; a NaN stays one through e)
      join(s[i & 1], e[i], g == 0 && i < 2);
      u[i & 1] = g == 0 && i < 2 ? held * e[i] : fmaf(held, e[i], u[i & 1]);
    }
    if (REF) {
      float y[4], tr[4], er[4];
      unpack4<DT>(xr, g, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) tr[i] = fma_log2e(y[i], neg_mr);
      ex2_group(tr, er);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        join(sr[i & 1], er[i], g == 0 && i < 2);
        join(w[i & 1], mass_times(e[i], t[i] - tr[i]), g == 0 && i < 2);
      }
    }
  }
  a.s += s[0] + s[1];
  a.u += u[0] + u[1];
  if (REF) {
    a.w += w[0] + w[1];
    a.sr += sr[0] + sr[1];
  }
}

// The sums about references that NV more vectors go by too: their largest logit, to a unit in its last place.
template <int DT, bool REF, int NV>
__device__ __forceinline__ void loss_raise(LossSums& a, const uint4 (&x)[NV], const uint4 (&xr)[NV]) {
  const float m = odd_bit(fmaxf(a.m, vecs_max<DT, NV>(x))), d = a.m - m, f = ex2(d);
  if (REF) {
    const float mr = odd_bit(fmaxf(a.mr, vecs_max<DT, NV>(xr))), dr = a.mr - mr;
    a.w = mass_times(f, fmaf(d - dr, a.s, a.w));
    a.sr *= ex2(dr);
    a.mr = mr;
  }
  a.u = (a.u + d * a.s) * f;
  a.s *= f;
  a.m = m;
}
// Sums of two parts of a row, about the larger references.
template <bool REF> __device__ __forceinline__ LossSums loss_merge(const LossSums& a, const LossSums& b) {
  LossSums r;
  r.m = fmaxf(a.m, b.m);
  const float da = a.m - r.m, db = b.m - r.m, fa = ex2(da), fb = ex2(db);
  r.s = a.s * fa + b.s * fb;
  r.u = (a.u + da * a.s) * fa + (b.u + db * b.s) * fb;
  r.w = 0.f;
  r.mr = kLowestM;
  r.sr = 0.f;
  if (REF) {
    r.mr = fmaxf(a.mr, b.mr);
    const float dra = a.mr - r.mr, drb = b.mr - r.mr;
    r.w = mass_times(fa, fmaf(da - dra, a.s, a.w)) + mass_times(fb, fmaf(db - drb, b.s, b.w));
    r.sr = a.sr * ex2(dra) + b.sr * ex2(drb);
  }
  return r;
}

// Over the lanes of a wavefront in 64 bits, uniform.
__device__ __forceinline__ double wave_sum_d(float v) {
  double t = (double)v;
  auto rotated = [&](auto rot) {
    const uint64_t w = (uint64_t)__double_as_longlong(t);
    const uint32_t lo = __float_as_uint(rot(__uint_as_float((uint32_t)w))), hi = __float_as_uint(rot(__uint_as_float((uint32_t)(w >> 32))));
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
  };
  t += rotated([](float x) { return dpp_rot<0x121>(x); });
  t += rotated([](float x) { return dpp_rot<0x122>(x); });
  t += rotated([](float x) { return dpp_rot<0x124>(x); });
  t += rotated([](float x) { return dpp_rot<0x128>(x); });
  auto of_row = [&](int lane) { return rotated([&](float x) { return lane_value(x, lane); }); };
  return (of_row(0) + of_row(16)) + (of_row(32) + of_row(48));
}
// One wavefront folds its lanes' sums; uniform results.  s (and sr and w, whose small difference the KL is) are folded in 64
// bits, six roundings fewer each: the absolute error of a log-probability before its rounding 5.0e-8 rms for 6.5e-8 in the build that this came with, for
// 0.3 us of 14 in a call of 193 rows; 3.4e-8 to 5.7e-8 now.
template <bool REF> __device__ __forceinline__ LossSums loss_fold_wave(const LossSums& a) {
  LossSums r = a;
  r.m = odd_bit(wave_max_f(a.m));                // (a NaN's lowest bit may be lost on the way)
  const float d = a.m - r.m, f = ex2(d);
  r.u = wave_sum_f((a.u + d * a.s) * f);
  r.s = (float)wave_sum_d(a.s * f);
  if (REF) {
    r.mr = odd_bit(wave_max_f(a.mr));
    const float dr = a.mr - r.mr;
    r.w = (float)wave_sum_d(mass_times(f, fmaf(d - dr, a.s, a.w)));
    r.sr = (float)wave_sum_d(a.sr * ex2(dr));
  }
  return r;
}

// What the whole row's sums say, in nats and 64 bits.  The sums hold 2^(z k), k the float nearest log2(e): the row at a temperature
// 1 / (1 + eps), eps = k ln 2 - 1 = -1.3e-8.  Dividing by k (and not by log2(e)) leaves an error of eps H in the
// log-normaliser, which is put right; in the entropy it is of the size of eps.
struct LossRow {
  double lse;              // log-normaliser
  double apart;            // ln s - ln sr
  double H, kl;
  double inv_s;            // 1 / s
  bool bad;
};
constexpr double kNat = 1.0 / (double)kLog2e;
constexpr double kTemperature = (double)kLog2e * kLn2 - 1.0;
// The chip's 2^x is short by 3.4e-9 of itself on average (v_exp_f32, 2^28 arguments in [-1, 0], [-2, -1], [-16, 0]; 2.6e-8 rms).  A sum has that once from
// its elements and once more from each fold that brought it here, `exps` times in all, but for the largest element, whose power is 1: added to the
// normaliser, or the log-probabilities of a long sequence add up 1.4e-8 each.
constexpr double kShort = 3.4e-9 / kLn2;
__device__ __forceinline__ double log2_sum(float s, int exps) { return log2_fine(s) + exps * kShort * fmax(1.0 - 1.0 / (double)s, 0.0); }
template <bool REF> __device__ __forceinline__ LossRow finish_loss_row(const LossSums& t, int exps) {
  LossRow r;
  const bool ok = t.s > 0.f && t.s < INFINITY && fabsf(t.u) < INFINITY && fabsf(t.m) <= kLargestM;
  const float s = ok ? t.s : NAN;
  const double l2 = log2_sum(s, exps), inv = 1.0 / (double)s;
  r.H = fmax(kNat * (l2 - (double)t.u * inv), 0.0);
  r.H = ok ? r.H : (double)NAN;
  r.lse = kNat * ((double)t.m + l2) + kTemperature * r.H;
  r.inv_s = inv;
  r.bad = !ok;
  r.apart = r.kl = 0.0;
  if (REF) {
    const bool okr = t.sr > 0.f && t.sr < INFINITY && fabsf(t.mr) <= kLargestM;
    const double l2r = log2_sum(okr ? t.sr : NAN, exps);
    r.apart = kNat * (l2 - l2r);
    r.kl = fmax(kNat * ((double)t.w * inv) - r.apart, 0.0);
    if (!ok || !okr || t.w != t.w) r.kl = (double)NAN;
    r.bad = r.bad || !okr;
  }
  return r;
}

// Whether a position counts, in two steps: what says so is asked for, and looked at where it is needed.
struct PositionMark {
  float weight;
  uint8_t active;
};
__device__ __forceinline__ PositionMark ask_mark(const LossRows& rows, int r) {
  return PositionMark{rows.weight ? rows.weight[r] : 1.f, rows.active ? rows.active[r] : (uint8_t)1};
}
__device__ __forceinline__ bool position_counts(const PositionMark& m) { return m.weight != 0.f && m.active != 0; }
template <int DT> __device__ __forceinline__ const char* row_at(const RowPlace& p, int b, int t) {
  return static_cast<const char*>(p.base) + ((int64_t)b * p.seq + (int64_t)t * p.pos) * Elem<DT>::bytes;
}

}  // namespace adasd
