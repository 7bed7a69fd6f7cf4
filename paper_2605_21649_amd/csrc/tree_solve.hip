// Entmax attention of drafted rows, second launch: from a row's scores and group maxima to its threshold and output.
//
// One workgroup per row (drafted token, query head).  The mass of the group maxima bounds the threshold from below, so only the
// groups above that bound are read, and of them the candidates above it go to LDS, in the order of their wavefronts; one
// wavefront iterates to the exact root, then every wavefront adds up the value rows of its part of the support (V is read
// where a weight is not zero, nowhere else).  A row too flat for LDS is gone through in its scores instead, evaluation by evaluation.
// A chain of latencies (maxima, scores, root, lookups, values), several rows to a compute unit: 512 rows (tokens times query heads) of 21 000
// keys 11.4 us, 1472 of 131 000 24.6, 8032 of 512 19.3.  Rows with thousands of keys in their support are gone through in their scores: alpha 1.25,
// 131 000 keys, 256 rows 81 us by eight wavefronts each, 1024 rows 645 by four.
#include "ekv_solve.h"
#include "ekv_tree.h"

namespace ekv {

struct TreeSolveArgs {
  TreeArgs t;
  int32_t* supp;
  float beta; int ibeta;
  int rows;                                      // tokens * query heads
};

// Weighted sum of `n` value rows: weight and row of entry e are weight[e] and row[e] in LDS, rows `stride` elements apart; lane (r, c) adds
// channels 8c..8c+7 of entries r, r + 4, ...
template <typename T, typename W>
__device__ __forceinline__ void add_rows(const T* v, int64_t stride, const float* weight, const uint32_t* row, int n, float (&acc)[8], W&& scaled) {
  const int lane = threadIdx.x & 63, r = lane >> 4, c = lane & 15;
  for (int e0 = 0; e0 < n; e0 += 32) {
    Raw8<T> raw[8];
    float p[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int e = e0 + 4 * k + r, ec = min(e, n - 1);
      const uint32_t at = row[ec];
      p[k] = e < n ? scaled(weight[ec], at) : 0.f;
      load_raw8(v + (int64_t)at * stride + 8 * c, raw[k]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (e0 + 4 * k >= n) break;                // the same for the wavefront
      float x[8];
      widen8(raw[k], x);
      const bool in = e0 + 4 * k + r < n;
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = in ? fmaf(p[k], x[i], acc[i]) : acc[i];
    }
  }
}

template <typename TQ, typename TC, int NW>
__global__ __launch_bounds__(64 * NW) void tree_solve_kernel(const TreeSolveArgs S) {
#pragma clang fp contract(off)
  constexpr int NT = 64 * NW, SEG = 512, R = 8, kOneGroups = 64 * R, kRegs = 4;
  __shared__ float s_u[NW][SEG];
  __shared__ uint32_t s_at[NW][SEG];
  __shared__ float s_o[NW][kD];
  __shared__ float s_red[2][NW][3], s_one[NW < 2 ? 2 : NW];
  __shared__ int s_n[NW], s_supp;
  __shared__ float s_tau;
  __shared__ uint16_t s_list[kOneGroups];
  const TreeArgs& A = S.t;
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  const uint64_t lt = (1ull << lane) - 1;
  // consecutive rows, the heads of a token, on one XCD
  const int row = gridDim.x % kXcds == 0 ? (int)(blockIdx.x % kXcds * (gridDim.x / kXcds) + blockIdx.x / kXcds) : (int)blockIdx.x;
  const int n = row / A.Hq, hq = row - n * A.Hq;
  const int b = uniform(wave_last_at_most(A.start, A.B, n));   // sequence 0 for rows in front of its first: they are none's
  const int unit = b * A.L + hq / A.GL;
  const TreeList list = tree_list(A, unit);
  const TreeRows T = list.R;
  if (n < T.first || n >= T.first + T.count) return;         // of no sequence
  const int groups = (list.n_pos + kGroup - 1) / kGroup;     // of the cache; one more of drafted keys
  const TreeScores scores = tree_z(A, list, unit);
  const float* z = scores.z + ((n - T.first) * A.GL + hq - list.head) * kGroup;
  const float* zm = A.zmax + (size_t)row * A.n_groups;
  const float zd = lane < T.count ? z[groups * scores.group + lane] : -INFINITY;
  // Row maximum and bound: by one wavefront where its registers hold all maxima (rows of up to 32 704 cached tokens), which then lists the
  // groups above the bound for all; else by all, several groups to a register where there are more than registers (their
  // mass is still no more than the row's), and every wavefront looks up its own.
  const bool one = NW == 1 || groups < kOneGroups;           // (with NW 1 there are 128 groups at most)
  float m[R], zmax = 0.f, bound = 0.f;
  bool folded = false;
  auto relative = [&](auto&& sums) {
#pragma unroll
    for (int k = 0; k < R; ++k) m[k] -= zmax;
    const float eps = 4e-6f * fmaxf(1.f, fabsf(zmax)), t = group_bound(m, -1.0f - eps, S.beta, S.ibeta, sums);
    bound = fmaxf(t - eps, -1.0f - eps);
  };
  if (one) {
    if (w == 0) {
#pragma unroll
      for (int k = 0; k < R; ++k) m[k] = k * 64 + lane <= groups ? zm[k * 64 + lane] : -INFINITY;
      float mx = m[0];
#pragma unroll
      for (int k = 1; k < R; ++k) mx = fmaxf(mx, m[k]);
      zmax = wave_max(mx);
      int n_list = 0;
      if (zmax > -INFINITY) {
        relative([&](float& f, float& d) { f = wave_sum(f); d = wave_sum(d); });
#pragma unroll
        for (int k = 0; k < R; ++k) {
          const bool in = m[k] > bound && k * 64 + lane < groups;
          const uint64_t mk = __ballot(in);
          if (in) s_list[n_list + __popcll(mk & lt)] = (uint16_t)(k * 64 + lane);
          n_list += __popcll(mk);
        }
      }
      if constexpr (NW > 1) {
        if (lane == 0) { s_one[0] = zmax; s_one[1] = bound; s_supp = n_list; }
      } else {
        s_supp = n_list;
        wave_order();
      }
    }
    if constexpr (NW > 1) {
      __syncthreads();
      zmax = s_one[0]; bound = s_one[1];
    }
  } else {
    if constexpr (NW > 1) {
#pragma unroll
      for (int k = 0; k < R; ++k) m[k] = k * NT + tid <= groups ? zm[k * NT + tid] : -INFINITY;
      folded = groups >= R * NT;
      for (int g = R * NT + tid; g <= groups; g += R * NT) {
#pragma unroll
        for (int k = 0; k < R; ++k) {            // a maximum counts once: what lies behind the last is not it again
          const float x = zm[min(g + k * NT, groups)];
          m[k] = g + k * NT <= groups ? fmaxf(m[k], x) : m[k];
        }
      }
      float mx = m[0];
#pragma unroll
      for (int k = 1; k < R; ++k) mx = fmaxf(mx, m[k]);
      zmax = block_max(mx, s_one);
      if (zmax > -INFINITY) {
        int parity = 0;
        relative([&](float& f, float& d) {
          f = wave_sum(f); d = wave_sum(d);
          if (lane == 0) { s_red[parity][w][0] = f; s_red[parity][w][1] = d; }
          __syncthreads();
          f = 0.f; d = 0.f;
#pragma unroll
          for (int i = 0; i < NW; ++i) { f += s_red[parity][i][0]; d += s_red[parity][i][1]; }
          parity ^= 1;
        });
      }
    }
  }
  float* out = A.out + (size_t)row * kD;
  if (!(zmax > -INFINITY)) {                                 // no key at all
    if (tid < kD / 4) *reinterpret_cast<float4*>(out + 4 * tid) = make_float4(0.f, 0.f, 0.f, 0.f);
    if (tid == 0) { A.norm[row] = INFINITY; S.supp[row] = 0; }
    return;
  }
  const float lo_u = fminf(bound, -1e-7f), ud = zd - zmax;
  // each(u, position) for the keys of four groups at a time, 64 lanes
  auto each_four = [&](const int (&g)[4], auto&& each) {
    float zz[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) zz[k] = z[max(g[k], 0) * scores.group + lane];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (g[k] < 0) break;
      each(zz[k] - zmax, g[k] * kGroup + lane);
    }
  };
  auto each_group = [&](uint64_t mask, int base, auto&& each) {
    while (mask != 0) {
      int g[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        g[k] = mask != 0 ? base + __builtin_ctzll(mask) : -1;
        mask &= mask - 1;
      }
      each_four(g, each);
    }
  };
  // those of this wavefront's share of all groups that have a key above `above` (relative)
  auto each_candidate = [&](float above, auto&& each) {
    for (int base = 64 * w; base < groups; base += NT) {
      const float x = base + lane < groups ? zm[base + lane] : -INFINITY;
      each_group(__ballot(x - zmax > above), base, each);
    }
  };
  int count = 0;
  auto keep = [&](float u, int pos) {
    const bool in = u > bound;
    const uint64_t mk = __ballot(in);
    const int o = count + __popcll(mk & lt);
    if (in && o < SEG) { s_u[w][o] = u; s_at[w][o] = (uint32_t)pos; }
    count += __popcll(mk);
  };
  if (one) {
    const int n_list = uniform(s_supp);
    for (int i = 4 * w; i < n_list; i += 4 * NW) {
      int g[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) g[k] = i + k < n_list ? uniform(s_list[min(i + k, n_list - 1)]) : -1;
      each_four(g, keep);
    }
  } else if (folded) {
    each_candidate(bound, keep);
  } else {
#pragma unroll
    for (int k = 0; k < R; ++k) each_group(__ballot(m[k] > bound && k * NT + tid < groups), k * NT + 64 * w, keep);
  }
  if (lane == 0) s_n[w] = count;
  __syncthreads();
  bool fits = true;
#pragma unroll
  for (int i = 0; i < NW; ++i) fits &= s_n[i] <= SEG;
  int supp = 0, evals = 0;
  float tau;
  if (fits) {
    int total = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) total += s_n[i];
    if (w == 0 && total <= 64 * kRegs) {                     // the usual row: its candidates in one wavefront's registers
      float u[kRegs + 1];
#pragma unroll
      for (int k = 0; k < kRegs; ++k) {
        int e = lane + 64 * k, seg = 0;
#pragma unroll
        for (int i = 0; i < NW - 1; ++i) {
          const bool next = seg == i && e >= s_n[i];
          e -= next ? s_n[i] : 0;
          seg += next ? 1 : 0;
        }
        u[k] = lane + 64 * k < total ? s_u[seg][e] : -INFINITY;
      }
      u[kRegs] = ud;
      tau = with_beta(S.ibeta, [&](auto ib) {
        constexpr int IB = decltype(ib)::value;
        return solve_tau_core([&](float t, float& F, float& D, int& cnt) {
          float f = 0.f, d = 0.f;
          cnt = 0;
#pragma unroll
          for (int k = 0; k <= kRegs; ++k) {
            const float x = fmaxf(u[k] - t, 0.f);
            add_mass<IB>(x, S.beta, f, d);
            cnt += __popcll(__ballot(x > 0.f));
          }
          F = wave_sum(f); D = S.beta * wave_sum(d);
        }, lo_u, NAN, IB, supp, evals);
      });
      if (lane == 0) { s_tau = tau; s_supp = supp; }
    } else if (w == 0) {
      tau = with_beta(S.ibeta, [&](auto ib) {
        constexpr int IB = decltype(ib)::value;
        return solve_tau_core([&](float t, float& F, float& D, int& cnt) {
          float f = 0.f, d = 0.f;
          const float x0 = fmaxf(ud - t, 0.f);
          add_mass<IB>(x0, S.beta, f, d);
          cnt = __popcll(__ballot(x0 > 0.f));
#pragma unroll
          for (int i = 0; i < NW; ++i) {
            const int ni = s_n[i];
            for (int e = 0; e < ni; e += 64) {
              const float x = e + lane < ni ? fmaxf(s_u[i][e + lane] - t, 0.f) : 0.f;
              add_mass<IB>(x, S.beta, f, d);
              cnt += __popcll(__ballot(x > 0.f));
            }
          }
          F = wave_sum(f); D = S.beta * wave_sum(d);
        }, lo_u, NAN, IB, supp, evals);
      });
      if (lane == 0) { s_tau = tau; s_supp = supp; }
    }
    __syncthreads();
    tau = s_tau; supp = s_supp;
  } else {
    int parity = 0;
    tau = solve_tau_core([&](float t, float& F, float& D, int& cnt) {
      float f = 0.f, d = 0.f;
      int c = 0;
      auto mass = [&](float u, int) {
        const float x = u - t;
        if (x > 0.f) { f += pow_beta(x, S.beta, S.ibeta); d += pow_beta_m1(x, S.beta, S.ibeta); ++c; }
      };
      if (w == 0) mass(ud, 0);
      each_candidate(t, mass);
      f = wave_sum(f); d = wave_sum(d); c = wave_sum_i(c);
      if (lane == 0) { s_red[parity][w][0] = f; s_red[parity][w][1] = d; s_red[parity][w][2] = __int_as_float(c); }
      __syncthreads();
      F = 0.f; D = 0.f; cnt = 0;
#pragma unroll
      for (int i = 0; i < NW; ++i) { F += s_red[parity][i][0]; D += s_red[parity][i][1]; cnt += __float_as_int(s_red[parity][i][2]); }
      D *= S.beta;
      parity ^= 1;
    }, lo_u, NAN, S.ibeta, supp, evals);
    __syncthreads();
  }
  // weights and value rows of the support, in place
  const TreeLook<true> in_list(A, unit, list);
  const TreeLook<false> in_all(A, unit, list);
  auto value_row = [&](int pos) {
    return A.page_idx != nullptr ? in_list.row(pos, in_list.phys(in_list.page(pos))) : in_all.row(pos, in_all.phys(in_all.page(pos)));
  };
  auto scaled = [&](float p, uint32_t at) {
    if constexpr (sizeof(TC) == 1) return p * A.v_scale[page_div(at, A.page_div)];
    else return p;
  };
  float acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.f;
  int n_sup = 0;
  auto take = [&](float u, int pos, bool real) {             // a wavefront's next 64 entries, to its segment
    const float x = u - tau;
    const bool in = real && x > 0.f;
    const uint64_t mk = __ballot(in);
    const uint32_t at = value_row(in ? pos : 0);
    wave_order();
    if (in) {
      const int o = n_sup + __popcll(mk & lt);
      s_u[w][o] = pow_beta(x, S.beta, S.ibeta);
      s_at[w][o] = at;
    }
    n_sup += __popcll(mk);
    wave_order();
  };
  if (fits) {
    for (int e = 0; e < count; e += 64) {
      const int ec = min(e + lane, count - 1);
      take(s_u[w][ec], (int)s_at[w][ec], e + lane < count);
    }
    add_rows((const TC*)A.v_pool, kD, s_u[w], s_at[w], n_sup, acc, scaled);
  } else {
    each_candidate(tau, [&](float u, int pos) {
      take(u, pos, true);
      if (n_sup > SEG - 64) {
        add_rows((const TC*)A.v_pool, kD, s_u[w], s_at[w], n_sup, acc, scaled);
        n_sup = 0;
        wave_order();
      }
    });
    add_rows((const TC*)A.v_pool, kD, s_u[w], s_at[w], n_sup, acc, scaled);
  }
  if (w == NW - 1) {                                         // the drafted keys' share
    wave_order();
    const float x = ud - tau;
    const bool in = x > 0.f;
    const uint64_t mk = __ballot(in);
    if (in) {
      const int o = __popcll(mk & lt);
      s_u[w][o] = pow_beta(x, S.beta, S.ibeta);
      s_at[w][o] = (uint32_t)lane;
    }
    wave_order();
    add_rows((const TQ*)A.v_new + T.first * A.vs + list.hkv * kD, A.vs, s_u[w], s_at[w], __popcll(mk), acc, [](float p, uint32_t) { return p; });
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = column_sum(acc[i]);
  if constexpr (NW == 1) {
    if (lane < 16) store8(out + 8 * lane, acc);
  } else {
    if (lane < 16) store8(&s_o[w][8 * lane], acc);
    __syncthreads();
    if (tid < kD) {
      float o = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i) o += s_o[i][tid];
      out[tid] = o;
    }
  }
  if (tid == 0) { A.norm[row] = tau + zmax; S.supp[row] = supp; }
}

template <typename TQ, typename TC>
static void launch_solve_T(const TreeSolveArgs& s, hipStream_t st) {
  // Wavefronts to a row: one where short rows are many, four, or eight where rows are so few that a compute unit has two at most.  Calls, us, by the
  // launch's rows, tokens times query heads.  One / four / eight: 8032 rows of lists of 512 keys 38.9 / 62.6 / 101, of 1024 60.0 / 84.2 / 122, of 4096
  // 159 / 181 / 216, of 8000 273 / 292 / 329; 2144 of 4096 52.8 / 56.0 / 63.2; 1120 of 8000 54.7 / 50.1 / 55.8; 40 of 777 25.7 / 21.6 / 22.1.  Four /
  // eight: 512 of 20 972 61.7 / 61.1; of 131 072 keys 256 rows 97.7 / 95.4, 608 138 / 136, 1472 353 / 361, 2048 273 / 279 (one sequence).  The line at
  // two rows a compute unit is these rows'.  With large supports (alpha 1.25) eight win far beyond it: of 32 768 keys 64 rows 62.0 / 50.5, 608 162 /
  // 84.7, 2048 260 / 214, of 131 072 keys 256 rows 595 / 158, 608 667 / 214, 1024 802 / 353, 2048 1077 / 575, but 4160 of 4096 150 / 182; that such rows are
  // gone through in their scores at all is what costs them.
  if (s.rows > 8 * device_compute_units() && s.t.n_groups <= 128)
    hipLaunchKernelGGL((tree_solve_kernel<TQ, TC, 1>), dim3(s.rows), dim3(64), 0, st, s);
  else if (s.rows <= 2 * device_compute_units())
    hipLaunchKernelGGL((tree_solve_kernel<TQ, TC, 8>), dim3(s.rows), dim3(512), 0, st, s);
  else
    hipLaunchKernelGGL((tree_solve_kernel<TQ, TC, 4>), dim3(s.rows), dim3(256), 0, st, s);
}
void launch_tree_solve(const Dims& dm, const TreeArgs& a, bool codes, int32_t* supp, hipStream_t st) {
  const TreeSolveArgs s{a, supp, dm.beta, dm.ibeta, a.N * dm.Hq};
  if (dm.dtype == EKV_F32) {
    if (codes) launch_solve_T<float, e4m3_t>(s, st);
    else launch_solve_T<float, float>(s, st);
  } else {
    if (codes) launch_solve_T<bf16_t, e4m3_t>(s, st);
    else launch_solve_T<bf16_t, bf16_t>(s, st);
  }
}

}  // namespace ekv
