// Scores of the entmax decode over the 8-bit cache; the solve that follows is that of decode.hip.
#include "ekv_attn8.h"

namespace ekv {

// An item is one group of page slots (up to 64 tokens) of one unit, as in decode.hip, and a wavefront takes a contiguous range
// of them.  The page-list, block-table and scale entries of up to 64 page slots are fetched at once, one slot per lane.
// OCTETS: pages of a multiple of 8 tokens, where eight tokens lie in one page and their place is wave-uniform.  Otherwise they may
// span pages and every lane looks up its own token's (the two tokens of a result lane are of one page).
template <typename T, int G, int MODE, bool OCTETS, bool STREAM>
__global__ __launch_bounds__(kScoreThreads) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 && OCTETS ? 4 : 3)))
void decode8_scores_kernel(const Score8Args A8) {
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
  const int ratio = A.Hq / A.Hkv;
  const Part part = MODE == kPerHead ? unit_part(A) : Part{0, 1};
  if (in_lds)
    block_exclusive_prefix<kScoreThreads>(A.U, [&](int u) {
      return part_length(part, u / ratio, (unit_slots<MODE>(A, u) + gp - 1) / gp); }, pre_lds, wsum);
  const WaveItems wi = in_lds ? wave_item_range((const int*)pre_lds, A.U, w, part) : wave_item_range(A.pre_g, A.U, w, part);
  const int last = (DENSE ? A.Mmax : A.cap) - 1;
  // Octet o of an item: page slot and token of its keys (of the lane's one, without OCTETS), and of the lane's first result
  int k_slot[8], k_tok[8], z_slot[8], z_tok[8];
  const int per_page = 65536 / P + 1;
#pragma unroll
  for (int o = 0; o < 8; ++o) {
    if constexpr (OCTETS) {
      const int p = min(8 * o, GT - 8);
      k_slot[o] = z_slot[o] = uniform(div64(p, per_page)); k_tok[o] = z_tok[o] = p - k_slot[o] * P;
    } else {
      const int pk = min(8 * o + key_token(c), GT - 1), pz = min(8 * o + 2 * g, GT - 2);
      k_slot[o] = div64(pk, per_page); k_tok[o] = pk - k_slot[o] * P;
      z_slot[o] = div64(pz, per_page); z_tok[o] = pz - z_slot[o] * P;
    }
  }
  const uint32_t lane_off = (OCTETS ? key_token(c) * kD : 0) + key_offset(c, g);
  const int head = column_head(c, G), copy = column_copy(c, G);
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
        if (MODE == kPerHead && part.count != 1) l_grp += part_first(part, l_unit / ratio, (unit_slots<MODE>(A, l_unit) + gp - 1) / gp);
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
      return OCTETS ? __builtin_amdgcn_readlane(v, in * gp + slot) : __shfl(v, in * gp + slot);
    };
    // chunk ck of the batch: octets 4 (ck % 2) .. 4 (ck % 2) + 3 of item ck / 2
    const int n_ck = (it1 - it0) * 2;
    auto request = [&](int ck, auto half, uint4 (&k)[4]) {
      constexpr int h = decltype(half)::value;
#pragma unroll
      for (int o = 0; o < 4; ++o) {
        const int page = of_slot(l_page, ck >> 1, k_slot[4 * h + o]);
        k[o] = load16<STREAM>(k_pool + ((size_t)page * P + k_tok[4 * h + o]) * kD + lane_off);
      }
    };
    int grp = 0, stored = 0;
    auto open_item = [&](int in) {
      const int unit = __builtin_amdgcn_readlane(l_unit, in * gp);
      grp = __builtin_amdgcn_readlane(l_grp, in * gp);
      if (unit != unit_now) {
        unit_now = unit;
        const int b = GROUPED ? unit / A.Hkv : unit / A.Hq;
        row0 = GROUPED ? (size_t)b * A.Hq + (unit % A.Hkv) * G : (size_t)unit;
        n = uniform_load(A.seq_lens + b);
        n_slots = DENSE ? clampi((n + P - 1) / P, 0, A.Mmax) : clampi(uniform_load(A.n_sel + unit), 0, A.cap);
        qb.load(q + row0 * kD);
      }
      stored = min(GT, (n_slots - grp * gp) * P);                       // tokens of the group that the row has
    };
    float top = -INFINITY;
    auto consume = [&](int ck, auto half, const uint4 (&k)[4]) {
      constexpr int h = decltype(half)::value;
      const int in = ck >> 1;
      float2 z[4];
#pragma unroll
      for (int o = 0; o < 4; ++o) {
        octet_scores<T, G>(k[o], __int_as_float(of_slot(__float_as_int(l_scale), in, k_slot[4 * h + o])), qb, z[o].x, z[o].y);
        const int p = 32 * h + 8 * o + 2 * g;
        const int lp = of_slot(l_lp, in, z_slot[4 * h + o]);  // by all lanes: behind the condition some sources would be idle
        const int left = p < stored ? n - (lp * P + z_tok[4 * h + o] + (OCTETS ? 2 * g : 0)) : 0;
        z[o].x = left > 0 ? A.zscale * z[o].x : -INFINITY;
        z[o].y = left > 1 ? A.zscale * z[o].y : -INFINITY;
        top = fmaxf(top, fmaxf(z[o].x, z[o].y));
      }
      // copy i of a head stores octet i: a whole line per head where there are four copies
      float* zrow = A.zbuf + (row0 + head) * A.zstride + (size_t)grp * GT + 32 * h + 2 * g;
#pragma unroll
      for (int o = 0; o < 4; o += G == 8 ? 2 : 4) {
        const float2 v = copy_pair<G>(z[o], z[o + 1], z[2], z[3], copy);
        if (copy < 4 && 32 * h + 8 * (o + copy) + 2 * g < stored) *reinterpret_cast<float2*>(zrow + 8 * (o + copy)) = v;
      }
      if (h == 1) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (g == 0 && copy == 0) A.pmax[(row0 + head) * A.n_chunks_max + grp] = top;
        top = -INFINITY;
      }
    };
    // two chunks (4 KB each) in flight, in alternating registers; every request of the loop is unconditional, so that no wait
    // at a join drains them, and the last pair is taken after it
    uint4 k0[4], k1[4];
    request(0, IntC<0>{}, k0);
    int ck = 0;
    for (; ck + 2 < n_ck; ck += 2) {
      open_item(ck >> 1);
      __builtin_amdgcn_sched_barrier(0);
      request(ck + 1, IntC<1>{}, k1);
      __builtin_amdgcn_sched_barrier(0);
      consume(ck, IntC<0>{}, k0);
      request(ck + 2, IntC<0>{}, k0);
      __builtin_amdgcn_sched_barrier(0);
      consume(ck + 1, IntC<1>{}, k1);
    }
    open_item(ck >> 1);
    request(ck + 1, IntC<1>{}, k1);
    __builtin_amdgcn_sched_barrier(0);
    consume(ck, IntC<0>{}, k0);
    consume(ck + 1, IntC<1>{}, k1);
  }
}

template <typename T, int G, int MODE>
static void launch_G(const Dims& dm, const Score8Args& a, bool stream, dim3 grid, size_t lds, hipStream_t st) {
  const dim3 block(kScoreThreads);
  const bool octets = dm.P % 8 == 0;
  if (stream && octets) hipLaunchKernelGGL((decode8_scores_kernel<T, G, MODE, true, true>), grid, block, lds, st, a);
  else if (stream) hipLaunchKernelGGL((decode8_scores_kernel<T, G, MODE, false, true>), grid, block, lds, st, a);
  else if (octets) hipLaunchKernelGGL((decode8_scores_kernel<T, G, MODE, true, false>), grid, block, lds, st, a);
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
  // Lists: the workgroups that a compute unit holds at a time (entmax over 2 % of a million tokens, a list per head: 18.2 us, with
  // four times as many 21.0).  All pages: four times as many (4 x 128K tokens 102.7 us, 108 without; 32 per compute unit 107).
  const long long most = (long long)device_compute_units() * (mode == kAllPages ? 16 : 4);
  if (wgs > most) wgs = most;
  const bool pre_global = sa.U > kUnitsLdsMax;
  // lists of the heads of a group are split over the XCDs as in decode.hip, by the same rule
  const bool split = mode == kPerHead && dm.G > 1 && !pre_global && 3 * wgs * kScoreWaves >= 2ll * kXcds * sa.U;
  sa.parts = split ? kXcds : 1;
  if (split) wgs = (wgs + kXcds - 1) / kXcds * kXcds;
  if (pre_global) {
    sa.pre_g = pre_ws;
    launch_unit_prefix(mode, sa, pre_ws, st);
  }
  const long long k_bytes = (long long)sa.U * (mode == kAllPages ? dm.Mmax : dm.cap) * dm.P * kD;
  // Loads through the caches or past them, by the capacity.  Whole calls, us, kept / past, K of every page: pages of 12 17 MB 19.1 / 18.5
  // (launched one by one 17.4 / 17.2), 34 MB 25.6 / 24.2 (23.1 / 23.7), 67 MB 38.9 / 36.8 (37.3 / 36.6), 134 MB 59.5 / 55.7, of 48 67 MB 37.9 /
  // 36.3, float32 268 MB 85.0 / 80.7; group lists 34 MB 21.8 / 21.6 (20.3 / 21.2), 67 MB 30.3 / 28.7 and 29.3 / 28.2, 134 MB 59.2 / 54.9, 268
  // MB 92.5 / 84.5; lists of heads without a group 34 MB 16.1 / 16.2, 67 MB 30.5 / 28.1 and 21.9 / 22.1, 134 MB 46.1 / 39.2, 268 MB
  // 74.7 / 66.1.  Lists per head of a group meet in the caches: 16 x 16K tokens, lists of 40 %, 78.4 / 91.6 (2 % of a million, which
  // hardly overlap, 35.4 / 31.7).
  const bool stream = (mode != kPerHead || dm.G == 1) && k_bytes >= kStream8Bytes;
  const Score8Args a{sa, k_scale};
  if (mode == kAllPages && launch_scores8_held(dm, a, items, k_bytes, st)) return;
  const size_t lds = pre_global ? 0 : (size_t)(sa.U + 1) * sizeof(int);
  const dim3 grid((unsigned)wgs);
  if (dm.dtype == EKV_F32) launch_T<float>(dm, mode, a, stream, grid, lds, st);
  else launch_T<bf16_t>(dm, mode, a, stream, grid, lds, st);
}

}  // namespace ekv
