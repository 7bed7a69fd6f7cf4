// The threshold of a row of scores: mass, root, and a bound of the root from group maxima.
#pragma once
#include "ekv_device.h"

namespace ekv {

// f += x^beta, d += x^(beta - 1) (0 for x = 0), x >= 0.  The products are spelled out, and what follows of the solve is
// compiled without contraction, so that every kernel that solves a row takes the same steps to the last bit.
template <int IB>
__device__ __forceinline__ void add_mass(float x, float beta, float& f, float& d) {
  if constexpr (IB == 0) {
    if (x > 0.f) { f += pow_beta(x, beta, 0); d += pow_beta_m1(x, beta, 0); }
  } else {
    const float y = IB == 1 ? (x > 0.f ? 1.f : 0.f) : pow_beta_m1(x, beta, IB);
    f = fmaf(x, y, f);
    d += y;
  }
}

// Root of sum (u - tau)_+^beta = 1 for u <= 0 with max u = 0: tau in [lo_init, 0), where lo_init >= -1
// is any point with mass >= 1.
// Safeguarded iteration inside a bracket [lo,hi], F(lo) >= 1 > F(hi).  From a left point the step is
// the exact root for the current support when beta is 1 or 2 (closed forms), Newton otherwise; from a
// right point a Newton step (F is convex, so it lands left of the root).  For beta in {1,2} the root is
// accepted as exact once a closed-form step leaves the support count unchanged.
// `eval(tau, F, D, cnt)` evaluates the mass, its negated derivative and the support count at tau.
// `seed`: where to take the first evaluation if it lies inside the bracket (NaN: none); `evals` counts
// the evaluations.
template <typename Eval>
__device__ __forceinline__ float solve_tau_core(Eval&& eval, float lo_init, float seed, int ibeta, int& supp,
                                                int& evals) {
#pragma clang fp contract(off)
  float lo = lo_init, hi = 0.f;
  float tau = (seed > lo && seed < hi) ? seed : lo;
  int pending_cnt = -1;
  int cnt = 0;
  bool last = false;                                         // tau is settled; evaluated once more for its support
  evals = 0;
  for (int it = 0;; ++it) {                                  // one call of `eval`: it is most of the code of every solve
    float F, D;
    eval(tau, F, D, cnt);
    ++evals;
    if (last) break;
    if (pending_cnt >= 0 && cnt == pending_cnt) break;       // exact step kept the support: done
    if (fabsf(F - 1.0f) <= 4e-7f) break;                     // float32 resolution of F: tau is the root
    pending_cnt = -1;
    float step;
    if (F >= 1.0f) {
      lo = tau;
      const float e = F - 1.0f;
      if (ibeta == 1) { step = e / (float)cnt; pending_cnt = cnt; }
      else if (ibeta == 2) {
        const float A = 0.5f * D;                            // sum (u - tau)
        const float disc = fmaf(A, A, -(float)cnt * e);
        if (disc > 0.f) { step = e / (A + sqrtf(disc)); pending_cnt = cnt; }
        else step = e / D;
      } else step = e / D;
    } else {
      hi = tau;
      step = D > 0.f ? (F - 1.0f) / D : -INFINITY;
    }
    float next = tau + step;
    if (next == tau) break;                                  // no representable progress
    if (!(next > lo && next < hi)) { next = 0.5f * (lo + hi); pending_cnt = -1; }
    last = hi - lo <= 1.2e-7f || (pending_cnt < 0 && fabsf(next - tau) <= 6e-8f);
    tau = next;
    if (it == 63 && !last) break;
  }
  supp = cnt;
  return tau;
}

// A certified lower bound of tau (relative to the row maximum) from group maxima relative to it: every group holds at
// least its maximum, so the mass of the maxima alone is a lower bound of the mass, and any point where it is >= 1 lies
// left of tau.  F^(1/beta) is a norm of (u - t)_+, hence convex in t: Newton's steps on it from a point where F >= 1
// stay left of the root.  They aim at a mass of 1.0001, which covers the rounding of the sums.  Below beta = 1 (alpha
// above 2) that fails, but sum x^beta >= (sum x)^beta there, so the point where the plain sum reaches 1 is a bound.
// `sums(f, d)` adds f and d up over all threads that hold maxima.
template <int R, typename Sums>
__device__ __forceinline__ float group_bound(const float (&u)[R], float t0, float beta, int ibeta, Sums&& sums) {
#pragma clang fp contract(off)
  if (beta < 1.f) { beta = 1.f; ibeta = 1; }
  return with_beta(ibeta, [&](auto ib) {
#pragma clang fp contract(off)
    constexpr int IB = decltype(ib)::value;
    const float target = 1.0f + 1e-4f / beta;
    float t = t0;
    for (int it = 0; it < 8; ++it) {
      float f = 0.f, d = 0.f;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        add_mass<IB>(fmaxf(u[k] - t, 0.f), beta, f, d);
      }
      sums(f, d);
      const float r = IB == 1 ? f : IB == 2 ? __builtin_amdgcn_sqrtf(f) : __builtin_exp2f(__builtin_log2f(f) / beta);
      if (!(r > target)) break;
      t += (r - target) * f * __builtin_amdgcn_rcpf(r * d);
      if (r < 1.02f) break;                                   // within two per cent of the norm: close enough
    }
    return t;
  });
}

}  // namespace ekv
