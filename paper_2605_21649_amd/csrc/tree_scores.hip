// Entmax attention of drafted rows, first launch: scores of every row with its list's keys and with the drafted keys that its mask
// names, and the maximum of every 64 of them (ekv_tree.h has the layout of the products).
//
// K is read once per block of rows; what bounds long lists is the scores' own bytes, 4 per row and key, beside K's.  So where rows are many
// a workgroup keeps a lower bound of every row's threshold, the root of the mass of the maxima that it has seen (32 a row, several
// groups folded into one), and a group none of whose keys is above it is not stored: its maximum is put down as -inf, nobody will read it.
// The drafted keys are a row's last group.  Hidden and missing keys score -inf.
// 64 rows a KV head, 4 x 128K tokens, 963 MB of K: 305 us, 232 (4.15 TB/s) with no score stored; 32 lists of 21 000 tokens, 16 rows, 172 MB of K:
// 51 us, 3.4 TB/s, seven tiles to a wavefront.
#include "ekv_solve.h"
#include "ekv_tree.h"

namespace ekv {

template <typename TQ, typename TC, int NQ, int WQ, bool LISTS>
__global__ __launch_bounds__(64 * (WQ == 1 ? 4 : WQ)) __attribute__((amdgpu_waves_per_eu(WQ == 1 ? 3 : WQ == 8 && NQ == 1 ? 4 : 2)))
void tree_scores_kernel(const TreeArgs A) {
  using S = TreeShape<TQ, TC, NQ, WQ, 1>;
  constexpr int kPer = kGroup / S::kKeys;        // tiles of a group
  extern __shared__ int pre_lds[];
  __shared__ __attribute__((aligned(16))) char s_tile[S::kLds];
  __shared__ int wsum[S::kWaves];
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6), c = lane & 15, j = lane >> 4;
  const int grp = WQ == 1 ? w : 0, tid = WQ == 1 ? lane : threadIdx.x;
  char* tile = s_tile + grp * S::kTileBytes;
  tree_work<S::kWork, S::kRows, kGroup>(A, pre_lds, wsum, [&](int, int unit, const TreeList& list, int blk, int st0, int st1, int steps, bool) {
    const TreeRows R = list.R;
    const int list_head = list.head, hkv = list.hkv;
    const int n_rows = R.count * A.GL;
    const int r0 = blk * S::kRows + (WQ > 1 ? w * 16 * NQ : 0);
    const TreeScores scores = tree_z(A, list, unit);
    TreeQuery<TQ, NQ> q;
    float* z[NQ]; float* zmax[NQ];
    bool there[NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      const int r = min(r0 + 16 * t + c, n_rows - 1), tok = r / A.GL;
      const size_t at = (size_t)(R.first + tok) * A.Hq + list_head + (r - tok * A.GL);
      there[t] = r0 + 16 * t + c < n_rows;
      z[t] = scores.z + min(r0 + 16 * t + c, n_rows - 1) * kGroup + 4 * j;
      zmax[t] = A.zmax + at * A.n_groups;
    }
    // a group's share of the steps, as tiles of the cache (the drafted keys are the last one's)
    const int n_g = st1 - st0, t0 = min(st0 + n_g * grp / S::kGroups, steps - 1) * kPer, t1 = min(st0 + n_g * (grp + 1) / S::kGroups, steps - 1) * kPer;
    const TreeLook<LISTS> look(A, unit, list);
    const int row = lane % S::kKeys;
    auto pos_of = [&](int t) { return min(t, t1 - 1) * S::kKeys + row; };
    TreeStage<TQ, TC, NQ, WQ, 1> stage;
    uint64_t valid_next = 0;
    auto fetch = [&](int t, int lp, int ph) {
      const int pos = pos_of(t);
      const uint32_t at_row = look.row(pos, ph);
      valid_next = __ballot(look.valid(pos, lp));
      stage.request(A, tid, [&](int i) { return (uint32_t)__shfl((int)at_row, i); });
    };
    q.load(A, R, list_head, r0);
    int lp1 = 0, ph1 = 0, lp2 = 0;
    if (t0 < t1) {
      const int lp0 = look.page(pos_of(t0));
      lp1 = look.page(pos_of(t0 + 1)); lp2 = look.page(pos_of(t0 + 2));
      const int ph0 = look.phys(lp0);
      ph1 = look.phys(lp1);
      fetch(t0, lp0, ph0);
    }
    float top[NQ];
    constexpr bool kHold = WQ > 1 && kPer == 1;
    constexpr int kSlots = 8;                              // maxima of a row: kSlots in each of its four lanes
    float held_top[kHold ? NQ : 1][4];                     // maxima of sixteen groups, lane (c, j) has those of 4j..4j+3
    float slot[kHold ? NQ : 1][kSlots], bound[kHold ? NQ : 1], most[kHold ? NQ : 1];
    if constexpr (kHold) {
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        bound[i] = most[i] = -INFINITY;
#pragma unroll
        for (int k = 0; k < kSlots; ++k) slot[i][k] = -INFINITY;
      }
    }
    // scores of the LDS tile to places from `to` on of the rows' scores, and into the maxima
    auto score = [&](const char* k, size_t to, auto drafted, uint64_t valid, const uint64_t (&seen)[NQ]) {
      constexpr bool kDrafted = decltype(drafted)::value != 0;
      constexpr uint64_t full = S::kKeys == 64 ? ~0ull : (1ull << (S::kKeys & 63)) - 1;
      f32x4_t d[S::kTiles][NQ];
      tree_scores_all<TQ, NQ, S::kTiles>(k, q, d);
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
#pragma unroll
        for (int m = 0; m < S::kTiles; ++m) {
          d[m][i] *= A.zscale;
          if (kDrafted || (valid & full) != full) {
            const uint32_t bits = (uint32_t)((kDrafted ? seen[i] : valid) >> (16 * m + 4 * j));
#pragma unroll
            for (int e = 0; e < 4; ++e) d[m][i][e] = bits >> e & 1 ? d[m][i][e] : -INFINITY;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) top[i] = fmaxf(top[i], d[m][i][e]);
        }
        bool store = there[i];
        if constexpr (kHold && !kDrafted) {
          top[i] = column_max(top[i]);
          if (top[i] <= bound[i]) { store = false; top[i] = -INFINITY; }
        }
        if (store) {
#pragma unroll
          for (int m = 0; m < S::kTiles; ++m) *reinterpret_cast<f32x4_t*>(z[i] + to + 16 * m) = d[m][i];
        }
      }
    };
    auto clear_top = [&]() {
#pragma unroll
      for (int i = 0; i < NQ; ++i) top[i] = -INFINITY;
    };
    auto store_top = [&](int group) {
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        const float x = column_max(top[i]);
        if (j == 0 && there[i]) zmax[i][group] = x;
      }
    };
    const uint64_t none[NQ] = {};
    auto ahead = [&](int t) {                              // tile t's data under way, the lookups of the two behind it
      const int ph2 = look.phys(lp2), lp3 = look.page(pos_of(t + 2));
      fetch(t, lp1, ph1);
      lp1 = lp2; ph1 = ph2; lp2 = lp3;
    };
    auto work = [&](const char* k, int t, uint64_t valid) {
      if (kPer == 1 || t % kPer == 0) clear_top();
      score(k, t / kPer * scores.group + t % kPer * S::kKeys, IntC<0>{}, valid, none);
      if constexpr (kHold) {
        const int seen_groups = t - t0, at = (seen_groups >> 2) & (kSlots - 1);
        const bool mine = j == (seen_groups & 3);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
#pragma unroll
          for (int k = 0; k < 4; ++k) held_top[i][k] = j == (t >> 2 & 3) && k == (t & 3) ? top[i] : held_top[i][k];
          most[i] = fmaxf(most[i], top[i]);
#pragma unroll
          for (int k = 0; k < kSlots; ++k) slot[i][k] = mine && k == at ? fmaxf(slot[i][k], top[i]) : slot[i][k];
        }
        if ((t & 15) == 15 || t == t1 - 1) {               // sixteen maxima of a row at a time, four in each of its lanes
          const int g0 = (t & ~15) + 4 * j;
#pragma unroll
          for (int i = 0; i < NQ; ++i) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (there[i] && g0 + k >= t0 && g0 + k <= t) zmax[i][g0 + k] = held_top[i][k];
          }
        }
        if ((seen_groups & 7) == 7) {                      // wave-uniform
#pragma unroll
          for (int i = 0; i < NQ; ++i) {
            float u[kSlots];
#pragma unroll
            for (int k = 0; k < kSlots; ++k) u[k] = slot[i][k] - most[i];
            const float eps = 4e-6f * fmaxf(1.f, fabsf(most[i]));
            // one key alone has mass 1 a step of 1 below it; the bound of fewer maxima is one of more
            const float from = fmaxf(bound[i] + eps - most[i], -1.0f - eps);
            const float b = group_bound(u, from, A.beta, A.ibeta, [&](float& f, float& d) {
              f = column_sum(f); d = column_sum(d);
            });
            if (most[i] > -INFINITY) bound[i] = fmaxf(bound[i], b + most[i] - eps);
          }
        }
      } else {
        if (kPer == 1 || t % kPer == kPer - 1) store_top(t / kPer);
      }
    };
    if constexpr (WQ == 1) {
      for (int t = t0; t < t1; ++t) {
        const uint64_t valid = valid_next;
        wave_order();                                      // the tile before is read
        stage.commit(tile, tid, valid);
        ahead(t + 1);
        wave_order();
        work(tile, t, valid);
      }
    } else if (t0 < t1) {
      // tile t + 1 goes to the half of LDS that nobody reads while tile t is worked on: one meeting a tile
      __syncthreads();                                     // the last list's tiles are read
      uint64_t valid = valid_next;
      stage.commit(tile, tid, valid);
      ahead(t0 + 1);
      for (int t = t0; t < t1; ++t) {
        __syncthreads();
        const uint64_t after = valid_next;
        if (t + 1 < t1) stage.commit(tile + ((t + 1 - t0) & 1) * S::kTileBytes, tid, after);
        ahead(t + 2);
        work(tile + ((t - t0) & 1) * S::kTileBytes, t, valid);
        valid = after;
      }
    }
    // the drafted keys, the list's last step; keys behind the last have no score, and nobody reads one
    if (st1 == steps && (WQ > 1 || w == S::kWaves - 1)) {
      clear_top();
#pragma unroll 1
      for (int d0 = 0; d0 < R.count; d0 += S::kKeys) {
        if constexpr (WQ > 1) __syncthreads(); else wave_order();
        stage_drafted<TQ, S, 1>(A, tile, tid, R, hkv, d0, [](int, uint4&) {});
        const int left = R.count - d0;
        const uint64_t there_keys = left >= 64 ? ~0ull : (1ull << left) - 1;
        uint64_t seen[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          const int r = min(r0 + 16 * i + c, n_rows - 1);
          seen[i] = (A.visible[R.first + r / A.GL] >> d0) & there_keys;
        }
        if constexpr (WQ > 1) __syncthreads(); else wave_order();
        score(tile, (steps - 1) * scores.group + d0, IntC<1>{}, 0, seen);
      }
      store_top(steps - 1);
    }
    if constexpr (WQ == 1) wave_order();
  });
}

// ------------------------------------------------------------------------------------------
static int score_rows(const Dims& dm, int list_rows) {
  if (list_rows <= 16) return 16;
  if (dm.dtype == EKV_F32) return 64;
  return list_rows <= 64 ? 64 : list_rows <= 128 ? 128 : 256;
}
static long long score_steps(const Dims& dm, bool dense, int lists, int list_rows) {
  const int rows = score_rows(dm, list_rows);
  const long long tokens = (long long)(dense ? dm.Mmax : dm.cap) * dm.P;
  return (long long)dm.B * lists * ((list_rows + rows - 1) / rows) * ((tokens + kGroup - 1) / kGroup + 1);
}
static int tree_groups(const Dims& dm, bool dense) {
  return (int)(((long long)(dense ? dm.Mmax : dm.cap) * dm.P + kGroup - 1) / kGroup) + 1;
}
bool tree_entmax_supported(const Dims& dm, bool dense, int lists, int most) {
  return score_steps(dm, dense, lists, most * (dm.Hq / lists)) <= 0x7fffffff;
}
size_t tree_entmax_ws_bytes(const Dims& dm, bool dense, int lists, int n_tokens) {
  const size_t rows = (size_t)n_tokens * dm.Hq, groups = (size_t)tree_groups(dm, dense);
  return tree_pre_bytes((size_t)dm.B * lists) + rows * groups * kGroup * sizeof(float) + ((rows * groups * sizeof(float) + 255) & ~(size_t)255);
}

template <typename TQ, typename TC, int NQ, int WQ>
static void launch_scores_shape(const TreeArgs& a, size_t lds, hipStream_t st) {
  if (a.page_idx != nullptr) hipLaunchKernelGGL((tree_scores_kernel<TQ, TC, NQ, WQ, true>), dim3(a.W), dim3(64 * (WQ == 1 ? 4 : WQ)), lds, st, a);
  else hipLaunchKernelGGL((tree_scores_kernel<TQ, TC, NQ, WQ, false>), dim3(a.W), dim3(64 * (WQ == 1 ? 4 : WQ)), lds, st, a);
}
template <typename TQ, typename TC>
static void launch_scores_T(const Dims& dm, TreeArgs& a, hipStream_t st) {
  const int list_rows = a.most * a.GL, rows = score_rows(dm, list_rows);
  a.blocks = (list_rows + rows - 1) / rows;
  const long long steps = score_steps(dm, a.page_idx == nullptr, a.L, list_rows);
  // Workgroups per compute unit.  A second and third one of four wavefronts share the waiting, but each goes through less of a row and bounds it
  // less closely.  us, two / three: lists of 512 8-bit keys, 64 sequences 40.2 / 39.3, 8 of 4096 tokens 49.3 / 48.1, 64 of 1024 61.7 / 62.7, 128K
  // 125 / 131, 4 of 128K 330 / 347; float32, which stores all, 4 of 64K 381 / 364.
  const bool third = rows == 16 || (rows == 64 && (dm.dtype == EKV_F32 || steps <= 8192));
  const int most = (rows == 256 ? 1 : third ? 3 : 2) * device_compute_units();
  a.W = (int)(steps < most ? steps : most);
  size_t lds = 0;
  if (a.U > kUnitsLdsMax) {
    launch_tree_prefix(a, kGroup, rows, st);
    a.pre_g = a.pre;
  } else {
    lds = (size_t)(a.U + 1) * sizeof(int);
  }
  if (rows == 16) launch_scores_shape<TQ, TC, 1, 1>(a, lds, st);
  else if (rows == 64) launch_scores_shape<TQ, TC, 1, 4>(a, lds, st);
  if constexpr (sizeof(TQ) == 2) {
    if (rows == 128) launch_scores_shape<TQ, TC, 1, 8>(a, lds, st);
    else if (rows == 256) launch_scores_shape<TQ, TC, 2, 8>(a, lds, st);
  }
}

void launch_tree_entmax(const Dims& dm, TreeArgs a, bool codes, int32_t* supp, void* ws, hipStream_t st) {
  const bool dense = a.page_idx == nullptr;
  a.n_groups = tree_groups(dm, dense);
  a.zstride = (size_t)a.n_groups * kGroup;
  a.pre = (int32_t*)ws;
  a.z = (float*)((char*)ws + tree_pre_bytes(a.U));
  a.zmax = a.z + (size_t)a.N * dm.Hq * a.zstride;
  a.zscale = dm.a * dm.scale;
  a.beta = dm.beta; a.ibeta = dm.ibeta;
  if (dm.dtype == EKV_F32) {
    if (codes) launch_scores_T<float, e4m3_t>(dm, a, st);
    else launch_scores_T<float, float>(dm, a, st);
  } else {
    if (codes) launch_scores_T<bf16_t, e4m3_t>(dm, a, st);
    else launch_scores_T<bf16_t, bf16_t>(dm, a, st);
  }
  launch_tree_solve(dm, a, codes, supp, st);
}

}  // namespace ekv
