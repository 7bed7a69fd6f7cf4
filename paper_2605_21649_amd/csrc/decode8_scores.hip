// Scores of the entmax decode over the 8-bit cache; the solve that follows is that of decode.hip.
#include "ekv_attn8.h"

namespace ekv {

struct Score8Args {
  ScoreArgs s;                      // k_pool: the codes
  const float* k_scale;
};

// An item is one group of page slots (up to 64 tokens) of one unit, as in decode.hip, and a wavefront takes a contiguous range
// of them.  The page-list, block-table and scale entries of up to 64 page slots are fetched at once, one slot per lane.
// TILED: pages of 16, 32, 48 or 64 tokens, where a tile lies in one page and its place is wave-uniform.  Otherwise a tile may span
// pages and every lane looks up its own token's (the four tokens of a result lane are of one page).
// Columns of the MFMA beyond the G heads repeat them, so the lanes of copy t of the heads hold every tile's scores and store
// tile t's: 16 bytes a lane, 1 KB for four heads' 64 tokens with one instruction.
template <typename T, int G, int MODE, bool TILED, bool STREAM>
__global__ __launch_bounds__(kScoreThreads) void decode8_scores_kernel(const Score8Args A8) {
  const ScoreArgs& A = A8.s;
  constexpr bool DENSE = MODE == kAllPages, GROUPED = MODE != kPerHead;
  extern __shared__ int pre_lds[];
  __shared__ int wsum[kScoreWaves];
  const int P = A.P, gp = pmax_pages(P), GT = gp * P;
  const int batch_items = 64 / gp;
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const e4m3_t* k_pool = (const e4m3_t*)A.k_pool;
  const T* q = (const T*)A.q;
  const bool in_lds = A.pre_g == nullptr;
  if (in_lds) block_exclusive_prefix<kScoreThreads>(A.U, [&](int u) { return (unit_slots<MODE>(A, u) + gp - 1) / gp; }, pre_lds, wsum);
  const WaveItems wi = in_lds ? wave_item_range((const int*)pre_lds, A.U, w, Part{0, 1}) : wave_item_range(A.pre_g, A.U, w, Part{0, 1});
  const int last = (DENSE ? A.Mmax : A.cap) - 1;
  // the lane's token as a row of tile t and the first of its four tokens as results: page slot of the item and place in the page
  int k_slot[4], k_tok[4], z_slot[4], z_tok[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int pk = TILED ? 16 * t : min(16 * t + c, GT - 1), pz = TILED ? 16 * t : min(16 * t + 4 * g, GT - 4);
    k_slot[t] = pk / P; k_tok[t] = pk - k_slot[t] * P + (TILED ? c : 0);
    z_slot[t] = pz / P; z_tok[t] = pz - z_slot[t] * P + (TILED ? 4 * g : 0);
  }
  Query8<T, G> qb;
  int unit_now = -1, n = 0, n_slots = 0;
  size_t row0 = 0;
  int unit0 = wi.unit;
  for (int it0 = wi.begin; it0 < wi.end; it0 += batch_items) {
    const int it1 = min(it0 + batch_items, wi.end);
    // lane l: page slot l % gp of item it0 + l / gp (clamped to the last): unit, group, logical page, page of the pool, scale
    int l_unit, l_grp, l_lp, l_page;
    float l_scale;
    {
      const int my_it = min(it0 + lane / gp, it1 - 1);
      if (in_lds) {
        l_unit = lane_last_at_most((const int*)pre_lds, A.U, unit0, my_it, it1 - 1);
        l_grp = my_it - pre_lds[l_unit];
      } else {
        l_unit = lane_last_at_most(A.pre_g, A.U, unit0, my_it, it1 - 1);
        l_grp = my_it - A.pre_g[l_unit];
      }
      unit0 = __builtin_amdgcn_readlane(l_unit, 63);
      const int slot = min(l_grp * gp + lane % gp, last);
      const int b = GROUPED ? l_unit / A.Hkv : l_unit / A.Hq;
      const int hkv = GROUPED ? l_unit % A.Hkv : l_unit % A.Hq / (A.Hq / A.Hkv);
      l_lp = clampi(DENSE ? slot : A.page_idx[(size_t)l_unit * A.cap + slot], 0, A.Mmax - 1);
      const int phys = clampi(A.block_table[(size_t)b * A.Mmax + l_lp], 0, A.n_phys - 1);
      l_page = phys * A.HkvPool + hkv;
      l_scale = A8.k_scale[l_page];
    }
    auto of_slot = [&](int v, int in, int slot) {
      return TILED ? __builtin_amdgcn_readlane(v, in * gp + slot) : __shfl(v, in * gp + slot);
    };
    for (int it = it0; it < it1; ++it) {
      const int in = it - it0;
      const int unit = __builtin_amdgcn_readlane(l_unit, in * gp), grp = __builtin_amdgcn_readlane(l_grp, in * gp);
      KeyTile k[4];
      float scale[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int page = of_slot(l_page, in, k_slot[t]);
        scale[t] = __int_as_float(of_slot(__float_as_int(l_scale), in, k_slot[t]));
        load_keys<STREAM>(k_pool + ((size_t)page * P + k_tok[t]) * kD + 16 * g, k[t]);
      }
      if (unit != unit_now) {
        unit_now = unit;
        const int b = GROUPED ? unit / A.Hkv : unit / A.Hq;
        row0 = GROUPED ? (size_t)b * A.Hq + (unit % A.Hkv) * G : (size_t)unit;
        n = uniform_load(A.seq_lens + b);
        n_slots = DENSE ? clampi((n + P - 1) / P, 0, A.Mmax) : clampi(uniform_load(A.n_sel + unit), 0, A.cap);
        qb.load(q + row0 * kD);
      }
      f32x4_t z[4];
      float top = -INFINITY;
      const int stored = min(GT, (n_slots - grp * gp) * P);             // tokens of the group that the row has
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        z[t] = tile_scores<T, G>(k[t], scale[t], qb);
        const int left = 16 * t + 4 * g < stored ? n - (of_slot(l_lp, in, z_slot[t]) * P + z_tok[t]) : 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          z[t][r] = r < left ? A.zscale * z[t][r] : -INFINITY;
          top = fmaxf(top, z[t][r]);
        }
      }
      float* zrow = A.zbuf + (row0 + c % G) * A.zstride + (size_t)grp * GT + 4 * g;
      const int copy = c / G;
#pragma unroll
      for (int round = 0; round < (G == 8 ? 2 : 1); ++round) {
        const int t = G == 8 ? 2 * round + copy : copy;
        f32x4_t v;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float a = copy & 1 ? z[2 * round + 1][r] : z[2 * round][r], d = copy & 1 ? z[3][r] : z[2][r];
          v[r] = G != 8 && (copy & 2) ? d : a;
        }
        if (t < 4 && 16 * t + 4 * g < stored) *reinterpret_cast<f32x4_t*>(zrow + 16 * t) = v;
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (lane < G) A.pmax[(row0 + lane) * A.n_chunks_max + grp] = top;
    }
  }
}

template <typename T, int G, int MODE>
static void launch_G(const Dims& dm, const Score8Args& a, bool stream, dim3 grid, size_t lds, hipStream_t st) {
  const dim3 block(kScoreThreads);
  const bool tiled = dm.P % 16 == 0;
  if constexpr (MODE != kPerHead)
    if (stream) {
      if (tiled) hipLaunchKernelGGL((decode8_scores_kernel<T, G, MODE, true, true>), grid, block, lds, st, a);
      else hipLaunchKernelGGL((decode8_scores_kernel<T, G, MODE, false, true>), grid, block, lds, st, a);
      return;
    }
  if (tiled) hipLaunchKernelGGL((decode8_scores_kernel<T, G, MODE, true, false>), grid, block, lds, st, a);
  else hipLaunchKernelGGL((decode8_scores_kernel<T, G, MODE, false, false>), grid, block, lds, st, a);
}
template <typename T>
static void launch_T(const Dims& dm, int mode, const Score8Args& a, bool stream, dim3 grid, size_t lds, hipStream_t st) {
  const int G = mode == kPerHead ? 1 : dm.G;
  if (mode == kPerHead) { launch_G<T, 1, kPerHead>(dm, a, stream, grid, lds, st); return; }
  if (mode == kAllPages) {
    if (G == 1) launch_G<T, 1, kAllPages>(dm, a, stream, grid, lds, st);
    else if (G == 2) launch_G<T, 2, kAllPages>(dm, a, stream, grid, lds, st);
    else if (G == 4) launch_G<T, 4, kAllPages>(dm, a, stream, grid, lds, st);
    else launch_G<T, 8, kAllPages>(dm, a, stream, grid, lds, st);
    return;
  }
  if (G == 2) launch_G<T, 2, kGroupList>(dm, a, stream, grid, lds, st);
  else if (G == 4) launch_G<T, 4, kGroupList>(dm, a, stream, grid, lds, st);
  else launch_G<T, 8, kGroupList>(dm, a, stream, grid, lds, st);
}

void launch_scores8(const Dims& dm, int mode, ScoreArgs sa, const float* k_scale, int32_t* pre_ws, hipStream_t st) {
  const int gp = pmax_pages(dm.P);
  const long long items = (long long)sa.U * (((mode == kAllPages ? dm.Mmax : dm.cap) + gp - 1) / gp);
  long long wgs = (items + kScoreWaves - 1) / kScoreWaves;
  const long long most = (long long)device_compute_units() * 16;
  if (wgs > most) wgs = most;
  const bool pre_global = sa.U > kUnitsLdsMax;
  if (pre_global) {
    sa.pre_g = pre_ws;
    launch_unit_prefix(mode, sa, pre_ws, st);
  }
  const long long k_bytes = (long long)sa.U * (mode == kAllPages ? dm.Mmax : dm.cap) * dm.P * kD;
  const bool stream = mode != kPerHead && k_bytes >= kStreamKBytes;
  const Score8Args a{sa, k_scale};
  const size_t lds = pre_global ? 0 : (size_t)(sa.U + 1) * sizeof(int);
  const dim3 grid((unsigned)wgs);
  if (dm.dtype == EKV_F32) launch_T<float>(dm, mode, a, stream, grid, lds, st);
  else launch_T<bf16_t>(dm, mode, a, stream, grid, lds, st);
}

}  // namespace ekv
