// Score pass over every page of a large 8-bit cache: the stores of the scores are put off, as in decode_windows.hip (what mixed
// stores cost a stream of reads is told there; here they are twice as many beside the bytes read), until the LDS that holds them is
// full, which the wavefronts, as fast as one another, reach at about the same time.  A clock that makes them store together does
// not help here: 4 x 131072 tokens 115.5 us without, 115.8 with windows of 32 us, 117.9 with 16.
#include "ekv_attn8.h"

namespace ekv {

constexpr int kHold8 = 8192;            // scores a wavefront holds back
constexpr int kHold8UnitsMax = 4096;    // the most units of such a launch

// Pages of 8, 16, 32 or 64 tokens: items of 64 (with shorter ones a wavefront has less in flight: 4 x 65536 tokens in pages of 40 take
// 71 us by chunks and 84 like this).  One workgroup of four wavefronts per compute unit; a wavefront has one item (8 KB) in flight,
// each octet requested anew as it is consumed.  us, one item / two / four / eight, eight wavefronts with half the LDS each,
// sixteen with a quarter: 4 x 131072 tokens 112.9 / 112.9 / 115.2 / 124.4, 113.5, 116.2; 1 x 1048576 221 / 221 / 224 / 227, 234, 253;
// 64 x 8192 124 / 123 / 125 / 129, 126, 130.
template <typename T, int G, int PT>
__global__ __launch_bounds__(kScoreThreads) void decode8_held_kernel(const Score8Args A8) {
  const ScoreArgs& A = A8.s;
  constexpr int GP = 64 / PT, kBatchItems = 64 / GP;
  constexpr int NB = kHold8 / (64 * G);            // items a wavefront holds
  extern __shared__ int pre_lds[];
  __shared__ __attribute__((aligned(16))) float hold_z[kScoreWaves][kHold8];
  __shared__ float hold_max[kScoreWaves][NB * G];
  __shared__ int4 hold_at[kScoreWaves][NB];        // first row, group, scores stored per row
  __shared__ int wsum[kScoreWaves];
  static_assert(sizeof(hold_z) + sizeof(hold_max) + sizeof(hold_at) + sizeof(wsum) + (kHold8UnitsMax + 1) * sizeof(int) <= 160 * 1024,
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
  auto flush = [&]() {
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

  int unit_now = -1, n = 0, n_slots = 0, row0 = 0;
  Query8<T, G> qb;
  auto process = [&](int it, u32x4_t (&a)[8]) {
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
        request(it + 1, 4 * h + o, a[4 * h + o]);
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
    if (++held == NB) flush();
  };

  u32x4_t a[8];
#pragma unroll
  for (int o = 0; o < 8; ++o) {                    // in the order of their use
    request(wi.begin, o, a[o]);
    __builtin_amdgcn_sched_barrier(0);
  }
  for (int it = wi.begin; it < wi.end; ++it) {
    if (it == batch0 + kBatchItems) {
      batch0 = it;
      now = next;
      next = look_up(batch0 + kBatchItems);
    }
    process(it, a);
  }
  flush();
}

template <typename T, int G>
static void launch_held_PT(const Dims& dm, const Score8Args& a, dim3 grid, size_t lds, hipStream_t st) {
  const dim3 block(kScoreThreads);
  if (dm.P == 8) hipLaunchKernelGGL((decode8_held_kernel<T, G, 8>), grid, block, lds, st, a);
  else if (dm.P == 16) hipLaunchKernelGGL((decode8_held_kernel<T, G, 16>), grid, block, lds, st, a);
  else if (dm.P == 32) hipLaunchKernelGGL((decode8_held_kernel<T, G, 32>), grid, block, lds, st, a);
  else hipLaunchKernelGGL((decode8_held_kernel<T, G, 64>), grid, block, lds, st, a);
}
template <typename T>
static void launch_held_T(const Dims& dm, const Score8Args& a, dim3 grid, size_t lds, hipStream_t st) {
  if (dm.G == 1) launch_held_PT<T, 1>(dm, a, grid, lds, st);
  else if (dm.G == 2) launch_held_PT<T, 2>(dm, a, grid, lds, st);
  else if (dm.G == 4) launch_held_PT<T, 4>(dm, a, grid, lds, st);
  else launch_held_PT<T, 8>(dm, a, grid, lds, st);
}

// Whole calls, us, by chunks (decode8_scores.hip) / here, heads four to a KV head: 1 x 65536 tokens (67 MB of K) 30.4 / 27.1, 1 x
// 131072 51.0 / 42.7, 4 x 131072 uneven 123.9 / 112.9, 64 x 2048 59.6 / 51.6, 1 x 1048576 246 / 221; eight heads, 1 x 65536 31.0 /
// 30.6, 1 x 524288 153 / 145; one head, 1 x 262144 69.1 / 65.5, 1 x 524288 123 / 110.
bool launch_scores8_held(const Dims& dm, const Score8Args& a, long long items, long long k_bytes, hipStream_t st) {
  const unsigned long long z_bytes = (unsigned long long)a.s.U * dm.G * a.s.zstride * 4;
  if ((dm.P != 8 && dm.P != 16 && dm.P != 32 && dm.P != 64) || a.s.U > kHold8UnitsMax || k_bytes < (64ll << 20) ||
      z_bytes < (8u << 20) || (unsigned long long)a.s.zstride * dm.G * 4 > 0x7fffffffull) return false;
  const long long wgs = (items + kScoreWaves - 1) / kScoreWaves;
  const int cus = device_compute_units();
  const dim3 grid((unsigned)(wgs < cus ? wgs : cus));
  const size_t lds = (size_t)(a.s.U + 1) * sizeof(int);
  if (dm.dtype == EKV_F32) launch_held_T<float>(dm, a, grid, lds, st);
  else launch_held_T<bf16_t>(dm, a, grid, lds, st);
  return true;
}

}  // namespace ekv
