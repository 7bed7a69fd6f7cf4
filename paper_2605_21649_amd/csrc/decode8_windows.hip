// Score pass over every page of a large 8-bit cache: the stores of the scores are put off and made by all of the GPU at once, as
// in decode_windows.hip (what mixed stores cost a stream of reads is told there).  Here they are twice as many beside the bytes read.
#include "ekv_attn8.h"

namespace ekv {

// PER workgroups of four wavefronts per compute unit, one or four, share its LDS for the scores held back, and have 128 KB of
// codes in flight: four items (8 KB) for each of four wavefronts or one for each of sixteen.
template <int PER> struct Windows8 {
  static constexpr int kHold = 8192 / PER;       // scores a wavefront holds back
  static constexpr int kFlight = 4 / PER;        // items it has in flight
  static constexpr int kUnitsMax = PER == 1 ? 4096 : 1024;    // the most units of such a launch
};

// Pages of 8, 16, 32 or 64 tokens: items of 64.
template <typename T, int G, int PT, int PER>
__global__ __launch_bounds__(kScoreThreads) __attribute__((amdgpu_waves_per_eu(PER)))
void decode8_windows_kernel(const Score8Args A8, uint32_t window) {
  const ScoreArgs& A = A8.s;
  constexpr int GP = 64 / PT, kBatchItems = 64 / GP;
  constexpr int kHold8 = Windows8<PER>::kHold, kFlight = Windows8<PER>::kFlight;
  constexpr int NB = kHold8 / (64 * G);            // items a wavefront holds
  static_assert(kBatchItems % kFlight == 0, "a batch begins with the first item of a turn");
  extern __shared__ int pre_lds[];
  __shared__ __attribute__((aligned(16))) float hold_z[kScoreWaves][kHold8];
  __shared__ float hold_max[kScoreWaves][NB * G];
  __shared__ int4 hold_at[kScoreWaves][NB];        // first row, group, scores stored per row
  __shared__ int wsum[kScoreWaves];
  static_assert(PER * (sizeof(hold_z) + sizeof(hold_max) + sizeof(hold_at) + sizeof(wsum) + (Windows8<PER>::kUnitsMax + 1) * sizeof(int)) <= 160 * 1024,
                "the LDS of a compute unit");
  const T* q = (const T*)A.q;
  const e4m3_t* k_pool = (const e4m3_t*)A.k_pool;
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const int head = column_head(c, G), copy = column_copy(c, G);
  const int lane_off = key_token(c) * kD + key_offset(c, g);
  block_exclusive_prefix<kScoreThreads>(A.U, [&](int u) { return (unit_slots<kAllPages>(A, u) + GP - 1) / GP; }, pre_lds, wsum);
  const WaveItems wi = wave_item_range((const int*)pre_lds, A.U, w, Part{0, 1});
  if (wi.begin >= wi.end) return;

  // lane l: page slot l % GP of item it0 + l / GP (clamped to the last item): unit, group, page of the pool, its scale
  struct Slots { int unit, grp, page; float scale; };
  int unit0 = wi.unit;                             // the batch's first unit, or one before
  auto look_up = [&](int it0) {
    const int my_it = min(it0 + lane / GP, wi.end - 1);
    const int lo = lane_last_at_most((const int*)pre_lds, A.U, unit0, my_it, min(it0 + kBatchItems, wi.end) - 1);
    unit0 = __builtin_amdgcn_readlane(lo, 63);
    Slots s{lo, my_it - pre_lds[lo], 0, 0.f};
    const int slot = min(s.grp * GP + lane % GP, A.Mmax - 1);
    s.page = clampi(A.block_table[(size_t)(lo / A.Hkv) * A.Mmax + slot], 0, A.n_phys - 1) * A.HkvPool + lo % A.Hkv;
    s.scale = A8.k_scale[s.page];
    return s;
  };
  int batch0 = wi.begin;
  Slots now = look_up(batch0), next = look_up(batch0 + kBatchItems);

  // octet o of an item; past the wavefront's range the buffer has no bytes and nothing is read
  auto request = [&](int it, int o, u32x4_t& a) {
    const int i = it - batch0, in = i < kBatchItems ? i : i - kBatchItems;
    const int here = __builtin_amdgcn_readlane(now.page, (in * GP + 8 * o / PT) & 63), behind = __builtin_amdgcn_readlane(next.page, (in * GP + 8 * o / PT) & 63);
    const int page = i < kBatchItems ? here : behind;
    const e4m3_t* kc = k_pool + ((size_t)page * PT + 8 * o % PT) * kD;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)kc, 0, it < wi.end ? 8 * kD : 0, kBufferFlags);
    a = __builtin_amdgcn_raw_buffer_load_b128(r, lane_off, 0, kBufferNt);
  };

  int held = 0;
  auto flush = [&]() __attribute__((always_inline)) {
    wave_order();
    for (int i0 = 0; i0 < held; i0 += 4) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = min(i0 + u, held - 1);
        const int4 at = hold_at[w][i];
        const int row0 = uniform(at.x), grp = uniform(at.y), lim = uniform(at.z);
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(A.zbuf + (size_t)row0 * A.zstride + (size_t)grp * 64, 0, -1, kBufferFlags);
#pragma unroll
        for (int s = 0; s < (G + 3) / 4; ++s) {
          const int h = 4 * s + g, tok = 4 * c;
          const u32x4_t v = *reinterpret_cast<const u32x4_t*>(&hold_z[w][i * 64 * G + min(h, G - 1) * 64 + ((tok + 16 * h) & 63)]);
          if (i0 + u < held && h < G && tok < lim)
            __builtin_amdgcn_raw_buffer_store_b128(v, r, (int)((h * A.zstride + tok) * 4), 0, kBufferThrough);
        }
      }
    }
    for (int i = lane; i < held; i += 64) {
      const int4 at = hold_at[w][i];
#pragma unroll
      for (int h = 0; h < G; ++h) A.pmax[(size_t)(at.x + h) * A.n_chunks_max + at.y] = hold_max[w][i * G + h];
    }
    held = 0;
    wave_order();
  };

  uint32_t due = (uint32_t)__builtin_amdgcn_s_memrealtime();
  due += window - due % window;
  int unit_now = -1, n = 0, n_slots = 0, row0 = 0;
  Query8<T, G> qb;
  auto process = [&](int it, u32x4_t (&a)[8]) __attribute__((always_inline)) {
    const int at = (it - batch0) * GP;
    const int unit = __builtin_amdgcn_readlane(now.unit, at), grp = __builtin_amdgcn_readlane(now.grp, at);
    if (unit != unit_now) {
      const int b = unit / A.Hkv;
      unit_now = unit;
      row0 = b * A.Hq + unit % A.Hkv * G;
      n = uniform_load(A.seq_lens + b);
      n_slots = clampi((n + PT - 1) / PT, 0, A.Mmax);
      qb.load(q + (size_t)row0 * kD);
      qb.wait();                                   // here: behind the branch the wait would drain the loads of K
    }
    float top = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float2 z[4];
#pragma unroll
      for (int o = 0; o < 4; ++o) {
        const float scale = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(now.scale), at + 8 * (4 * h + o) / PT));
        octet_scores<T, G>(__builtin_bit_cast(uint4, a[4 * h + o]), scale, qb, z[o].x, z[o].y);
        const int left = n - (grp * 64 + 32 * h + 8 * o + 2 * g);
        z[o].x = left > 0 ? A.zscale * z[o].x : -INFINITY;
        z[o].y = left > 1 ? A.zscale * z[o].y : -INFINITY;
        top = fmaxf(top, fmaxf(z[o].x, z[o].y));
        __builtin_amdgcn_sched_barrier(0);
        request(it + kFlight, 4 * h + o, a[4 * h + o]);
        __builtin_amdgcn_sched_barrier(0);
      }
      float* hz = &hold_z[w][held * 64 * G + head * 64];
#pragma unroll
      for (int o = 0; o < 4; o += G == 8 ? 2 : 4) {
        const float2 v = copy_pair<G>(z[o], z[o + 1], z[2], z[3], copy);
        if (copy < 4) *reinterpret_cast<float2*>(hz + ((32 * h + 8 * (o + copy) + 2 * g + 16 * head) & 63)) = v;
      }
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    if (g == 0 && copy == 0) hold_max[w][held * G + head] = top;
    if (lane == 0) hold_at[w][held] = make_int4(row0, grp, n_slots * PT - grp * 64, 0);
    if (it < wi.end) ++held;
    const uint32_t t = (uint32_t)__builtin_amdgcn_s_memrealtime();
    const bool tick = (int)(t - due) >= 0;
    if (held == NB || tick) flush();
    if (tick) due = t + window - t % window;
  };

  // the first requests in the order of their use
  u32x4_t a[kFlight][8];
#pragma unroll
  for (int i = 0; i < kFlight; ++i) {
#pragma unroll
    for (int o = 0; o < 8; ++o) {
      request(wi.begin + i, o, a[i][o]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  for (int it = wi.begin; it < wi.end; it += kFlight) {
    if (it == batch0 + kBatchItems) {
      batch0 = it;
      now = next;
      next = look_up(batch0 + kBatchItems);
    }
#pragma unroll
    for (int i = 0; i < kFlight; ++i) process(it + i, a[i]);
  }
  flush();
}

template <typename T, int G, int PER>
static void launch_windows_PT(const Dims& dm, const Score8Args& a, dim3 grid, size_t lds, uint32_t window, hipStream_t st) {
  const dim3 block(kScoreThreads);
  if (dm.P == 8) hipLaunchKernelGGL((decode8_windows_kernel<T, G, 8, PER>), grid, block, lds, st, a, window);
  else if (dm.P == 16) hipLaunchKernelGGL((decode8_windows_kernel<T, G, 16, PER>), grid, block, lds, st, a, window);
  else if (dm.P == 32) hipLaunchKernelGGL((decode8_windows_kernel<T, G, 32, PER>), grid, block, lds, st, a, window);
  else hipLaunchKernelGGL((decode8_windows_kernel<T, G, 64, PER>), grid, block, lds, st, a, window);
}
template <typename T, int PER>
static void launch_windows_T(const Dims& dm, const Score8Args& a, dim3 grid, size_t lds, uint32_t window, hipStream_t st) {
  if (dm.G == 1) launch_windows_PT<T, 1, PER>(dm, a, grid, lds, window, st);
  else if (dm.G == 2) launch_windows_PT<T, 2, PER>(dm, a, grid, lds, window, st);
  else if (dm.G == 4) launch_windows_PT<T, 4, PER>(dm, a, grid, lds, window, st);
  else launch_windows_PT<T, 8, PER>(dm, a, grid, lds, window, st);
}

// Whole calls, us, by chunks (decode8_scores.hip) / in windows by four workgroups per compute unit, heads four to a KV head: 1 x 65536
// tokens (67 MB of K) 30.4 / 28.8, 1 x 131072 51.0 / 44.6, 4 x 131072 uneven 123.9 / 119.3, 64 x 2048 59.6 / 51.6; eight heads,
// 1 x 32768 22.0 / 22.0, 1 x 65536 31.0 / 30.6, 1 x 524288 153 / 158; one head, 1 x 262144 69.1 / 65.5, 1 x 524288 123 / 113;
// float32 queries, 64 x 8192 134 / 125, pages of 8 tokens, 4 x 131072 134 / 128.  One workgroup per compute unit, whose lone
// wavefronts pay more for their start, needs a long call: 1 x 1048576 246 by chunks, 235 by four, 222 by one, 4 x 131072
// (466 MB) 113 / 112 / 119.  A window is what fills most of a wavefront's LDS at full rate, half of decode_windows.hip's.
bool launch_scores8_windows(const Dims& dm, const Score8Args& a, long long items, long long k_bytes, hipStream_t st) {
  const unsigned long long z_bytes = (unsigned long long)a.s.U * dm.G * a.s.zstride * 4;
  if ((dm.P != 8 && dm.P != 16 && dm.P != 32 && dm.P != 64) || a.s.U > Windows8<1>::kUnitsMax || k_bytes < (64ll << 20) ||
      z_bytes < (8u << 20) || (unsigned long long)a.s.zstride * dm.G * 4 > 0x7fffffffull) return false;
  const bool one = a.s.U > Windows8<4>::kUnitsMax || k_bytes >= (768ll << 20);
  const long long wgs = (items + kScoreWaves - 1) / kScoreWaves, most = (long long)device_compute_units() * (one ? 1 : 4);
  const dim3 grid((unsigned)(wgs < most ? wgs : most));
  const size_t lds = (size_t)(a.s.U + 1) * sizeof(int);
  const uint32_t window = 12800 / dm.G;
  if (dm.dtype == EKV_F32) {
    if (one) launch_windows_T<float, 1>(dm, a, grid, lds, window, st);
    else launch_windows_T<float, 4>(dm, a, grid, lds, window, st);
  } else {
    if (one) launch_windows_T<bf16_t, 1>(dm, a, grid, lds, window, st);
    else launch_windows_T<bf16_t, 4>(dm, a, grid, lds, window, st);
  }
  return true;
}

}  // namespace ekv
