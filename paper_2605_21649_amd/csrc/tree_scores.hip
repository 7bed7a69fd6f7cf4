// Entmax attention of drafted rows, first launch: scores of every row with its list's keys and with the drafted keys that its mask
// names, and the maximum of every 64 of them (ekv_tree.h has the layout of the products).
//
// K is read once per block of rows; what bounds long lists is the scores' own bytes, 4 per row and key, beside K's.
// The drafted keys are a row's last group.  Hidden and missing keys score -inf.
#include "ekv_tree.h"

namespace ekv {

constexpr int kGroup = 64;                       // keys per maximum

template <typename TQ, typename TC, int NQ, int WQ>
__global__ __launch_bounds__(kTreeThreads) __attribute__((amdgpu_waves_per_eu(2)))
void tree_scores_kernel(const TreeArgs A) {
  using S = TreeShape<TQ, TC, NQ, WQ, 1>;
  constexpr int kPer = kGroup / S::kKeys;        // tiles of a group
  extern __shared__ int pre_lds[];
  __shared__ __attribute__((aligned(16))) char s_tile[S::kLds];
  __shared__ int wsum[kTreeWaves];
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6), c = lane & 15, j = lane >> 4;
  const int grp = WQ == 1 ? w : 0, tid = WQ == 1 ? lane : threadIdx.x;
  char* tile = s_tile + grp * S::kSideBytes;
  tree_work<S::kRows, kGroup>(A, pre_lds, wsum, [&](int wg, int unit, const TreeRows& R, int blk, int st0, int st1, int steps, bool) {
    const int b = unit / A.L, list = unit - b * A.L, list_head = list * A.GL, hkv = list_head / (A.Hq / A.Hkv);
    const int g0 = min(st0, steps - 1), g1 = min(st1, steps - 1), n_rows = R.count * A.GL;
    const int r0 = blk * S::kRows + (WQ == 4 ? w * 16 * NQ : 0);
    TreeQuery<TQ, NQ> q;
    q.load(A, R, list_head, r0);
    float* z[NQ]; float* zmax[NQ];
    bool there[NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      const int r = min(r0 + 16 * t + c, n_rows - 1), tok = r / A.GL;
      const size_t at = (size_t)(R.first + tok) * A.Hq + list_head + (r - tok * A.GL);
      there[t] = r0 + 16 * t + c < n_rows;
      z[t] = A.z + at * A.zstride + 4 * j;
      zmax[t] = A.zmax + at * A.n_groups;
    }
    const int n_g = g1 - g0, t0 = (g0 + n_g * grp / S::kGroups) * kPer, t1 = (g0 + n_g * (grp + 1) / S::kGroups) * kPer;
    const TreeLook look(A, unit, hkv);
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
    int lp1 = 0, ph1 = 0, lp2 = 0;
    if (t0 < t1) {
      const int lp0 = look.page(pos_of(t0)), ph0 = look.phys(lp0);
      lp1 = look.page(pos_of(t0 + 1)); lp2 = look.page(pos_of(t0 + 2));
      ph1 = look.phys(lp1);
      fetch(t0, lp0, ph0);
    }
    const bool drafted = st1 == steps && (WQ == 4 || w == kTreeWaves - 1);
    const int t2 = drafted ? t1 + kPer : t1;
    float top[NQ];
    for (int t = t0; t < t2; ++t) {
      const bool cached = t < t1;
      uint64_t seen[NQ];
      bool all = false;
      if constexpr (WQ == 4) __syncthreads(); else wave_order();           // the tile before is read
      if (cached) {
        const uint64_t valid = valid_next;
        stage.commit(tile, tid, valid);
        const int ph2 = look.phys(lp2), lp3 = look.page(pos_of(t + 3));
        fetch(t + 1, lp1, ph1);
        lp1 = lp2; ph1 = ph2; lp2 = lp3;
#pragma unroll
        for (int i = 0; i < NQ; ++i) seen[i] = valid;
        constexpr uint64_t full = S::kKeys == 64 ? ~0ull : (1ull << (S::kKeys & 63)) - 1;
        all = (valid & full) == full;
      } else {
        constexpr int pieces = S::kRowBytes / 16;
        const int d0 = (t - t1) * S::kKeys;
#pragma unroll 1
        for (int i = tid; i < S::kKeys * pieces; i += S::kThreads) {
          const int key_row = i / pieces, piece = i % pieces, key = d0 + key_row;
          const int kc = R.first + min(key, R.count - 1);
          uint4 kv = load16((const char*)((const TQ*)A.k_new + kc * A.ks + hkv * kD) + 16 * piece);
          if (key >= R.count) kv = make_uint4(0u, 0u, 0u, 0u);
          *reinterpret_cast<uint4*>(tile + tree_piece<TQ>(key_row, piece)) = kv;
        }
        const int left = R.count - d0;
        const uint64_t there_keys = left >= 64 ? ~0ull : left > 0 ? (1ull << left) - 1 : 0;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          const int r = min(r0 + 16 * i + c, n_rows - 1);
          seen[i] = (A.visible[R.first + r / A.GL] >> d0) & there_keys;
        }
      }
      if constexpr (WQ == 4) __syncthreads(); else wave_order();
      if (kPer == 1 || t % kPer == 0) {
#pragma unroll
        for (int i = 0; i < NQ; ++i) top[i] = -INFINITY;
      }
      const int group = cached ? t / kPer : steps - 1, sub = kPer == 1 ? 0 : t % kPer * S::kKeys;
#pragma unroll
      for (int m = 0; m < S::kTiles; ++m) {
        f32x4_t d[NQ];
        tree_scores<TQ, NQ>(tile, m, q, d);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          d[i] *= A.zscale;
          if (!all) {
            const uint32_t bits = (uint32_t)(seen[i] >> (16 * m + 4 * j));
#pragma unroll
            for (int e = 0; e < 4; ++e) d[i][e] = bits >> e & 1 ? d[i][e] : -INFINITY;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) top[i] = fmaxf(top[i], d[i][e]);
          if (there[i]) *reinterpret_cast<f32x4_t*>(z[i] + (size_t)group * kGroup + sub + 16 * m) = d[i];
        }
      }
      if (kPer == 1 || t % kPer == kPer - 1) {
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          float x = fmaxf(top[i], __shfl_xor(top[i], 16));
          x = fmaxf(x, __shfl_xor(x, 32));
          if (j == 0 && there[i]) zmax[i][group] = x;
        }
      }
    }
    if constexpr (WQ == 1) wave_order();
  });
}

// ------------------------------------------------------------------------------------------
constexpr int kScoreWgs = 1024;

static int score_rows(const Dims& dm, int list_rows) {
  if (list_rows <= 16) return 16;
  if (dm.dtype == EKV_F32) return 64;
  return list_rows <= 32 ? 32 : list_rows <= 64 ? 64 : 128;
}
static long long score_steps(const Dims& dm, bool dense, int lists, int list_rows) {
  const int rows = score_rows(dm, list_rows);
  const long long tokens = (long long)(dense ? dm.Mmax : dm.cap) * dm.P;
  return (long long)dm.B * lists * ((list_rows + rows - 1) / rows) * ((tokens + kGroup - 1) / kGroup + 1);
}
static int tree_groups(const Dims& dm, bool dense) {
  return (int)(((long long)(dense ? dm.Mmax : dm.cap) * dm.P + kGroup - 1) / kGroup) + 1;
}
bool tree_entmax_supported(const Dims& dm, bool dense, int lists, int n_tokens, int most) {
  return score_steps(dm, dense, lists, most * (dm.Hq / lists)) <= 0x7fffffff && (long long)n_tokens * dm.Hq <= 0x7fffffff;
}
size_t tree_entmax_ws_bytes(const Dims& dm, bool dense, int lists, int n_tokens) {
  const size_t rows = (size_t)n_tokens * dm.Hq, groups = (size_t)tree_groups(dm, dense);
  return tree_pre_bytes((size_t)dm.B * lists) + rows * groups * kGroup * sizeof(float) + ((rows * groups * sizeof(float) + 255) & ~(size_t)255);
}

template <typename TQ, typename TC, int NQ, int WQ>
static void launch_scores_shape(const TreeArgs& a, size_t lds, hipStream_t st) {
  hipLaunchKernelGGL((tree_scores_kernel<TQ, TC, NQ, WQ>), dim3(a.W), dim3(kTreeThreads), lds, st, a);
}
template <typename TQ, typename TC>
static void launch_scores_T(const Dims& dm, TreeArgs& a, hipStream_t st) {
  const int list_rows = a.most * a.GL, rows = score_rows(dm, list_rows);
  a.blocks = (list_rows + rows - 1) / rows;
  const long long steps = score_steps(dm, a.page_idx == nullptr, a.L, list_rows);
  const int share = rows <= 32 ? kTreeWaves : 1, most = 2 * device_compute_units();
  const long long wgs = (steps + share - 1) / share;
  a.W = (int)(wgs < most ? wgs : most);
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
    if (rows == 32) launch_scores_shape<TQ, TC, 2, 1>(a, lds, st);
    else if (rows == 128) launch_scores_shape<TQ, TC, 2, 4>(a, lds, st);
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
