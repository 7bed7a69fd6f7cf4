// Append of several tokens per sequence to a cache in its own type (the 8-bit cache's is in cache8.hip), with the statistics of
// the pages that they reach (paper Sec. 4.2).
//
// One wavefront per run (rows with consecutive slots of one page), KV head and side (K or V).  Lane (r, c) has channels 8c..8c+7
// of the page's rows r, r + 4, ..: the rows' order of ekv_stats_build in the sums, whose result is that call's to the last bit.
// V and, without statistics, K are a copy; with statistics the run's page is gone through from its first token, the older ones
// from the cache and the new ones from their rows.  Bound by the bytes: rows read and written once, old keys of partly filled
// pages, records; 24000 tokens of prompts without statistics 196 MB in 49 us, 4.0 TB/s (a copy: 4.7).
#include "ekv_internal.h"
#include "ekv_stats.h"

namespace ekv {

constexpr int kAppendThreads = 256, kAppendWaves = kAppendThreads / 64;

struct AppendRowsArgs {
  const void* x[2]; int64_t stride[2];           // new rows: K, V
  void* pool[2];
  void* box; void* gauss; uint8_t* box8;         // null: no statistics
  const int64_t* slots; const int32_t* seq; const int32_t* pos;
  const int32_t* rows; int n_rows;               // row of x for each token; null: its own
  int T, block, B, Hkv, HkvPool, P, Mmax;        // T tokens, `block` of them per wavefront
  int64_t n_slots;                               // slots of the pool
};

// A page's statistics from the sums of a wavefront whose lane (r, c) went through rows r, r + 4, .. of channels 8c..8c+7: extremes, sums and
// squares relative to the first token k0, combined in the order of ekv_stats_build.  box_out, gauss_out, box8_out: the page's records.
template <typename T>
__device__ __forceinline__ void store_page_stats(const float (&mn)[8], const float (&mx)[8], const float (&s1)[8], const float (&s2)[8],
                                                 const float (&k0)[8], int cnt, T* box_out, T* gauss_out, uint8_t* box8_out) {
  const int lane = threadIdx.x & 63, r = lane >> 4, c = lane & 15;
  const float inv_n = 1.0f / (float)cnt;
  const float2 lo = rows_reduce(mn, [](float a, float b) { return fminf(a, b); }), hi = rows_reduce(mx, [](float a, float b) { return fmaxf(a, b); });
  const float2 d1 = rows_reduce(s1, [](float a, float b) { return a + b; }), d2 = rows_reduce(s2, [](float a, float b) { return a + b; });
  const bool up = r >> 1, far = r & 1;                     // channels 2 up + 4 far + 0, 1
  auto mine = [&](int i) { return far ? (up ? k0[i + 6] : k0[i + 4]) : (up ? k0[i + 2] : k0[i]); };
  auto variance = [&](float m1, float m2) { return fmaxf(fmaf(-m1, m1, m2 * inv_n), 0.f); };
  const float m1x = d1.x * inv_n, m1y = d1.y * inv_n;
  const int e = 2 * up + 4 * far;
  T* box = box_out + 8 * c + e; T* gauss = gauss_out + 8 * c + e;
  store2(box, lo);
  store2(box + kD, hi);
  store2(gauss, make_float2(mine(0) + m1x, mine(1) + m1y));
  store2(gauss + kD, make_float2(variance(m1x, d2.x), variance(m1y, d2.y)));
  if (box8_out != nullptr) {
    uint8_t* u = box8_out + 16 * c + e;
    *reinterpret_cast<uint16_t*>(u) = (uint16_t)(f32_to_e4m3_directed<false>(lo.x) | (f32_to_e4m3_directed<false>(lo.y) << 8));
    *reinterpret_cast<uint16_t*>(u + 8) = (uint16_t)(f32_to_e4m3_directed<true>(hi.x) | (f32_to_e4m3_directed<true>(hi.y) << 8));
  }
}

template <typename T>
__device__ __forceinline__ void append_rows_run(const AppendRowsArgs& A, int side, int h, int i0, int len, int64_t slot) {
  const int lane = threadIdx.x & 63, r = lane >> 4, c = lane & 15;
  const int P = A.P, t0 = (int)(slot % P), cnt = t0 + len;
  T* page = (T*)A.pool[side] + ((size_t)(slot / P) * A.HkvPool + h) * P * kD + 8 * c;
  const T* x = (const T*)A.x[side] + h * kD + 8 * c;
  const bool stats = side == 0 && A.box != nullptr;
  int b = -1, lp = -1;
  if (stats) { b = A.seq[i0]; lp = A.pos[i0]; }
  // where token t of the page is read
  auto source = [&](int t) -> const T* {
    if (t < t0) return page + (size_t)t * kD;
    const int i = i0 + t - t0;
    return x + (A.rows != nullptr ? min(max(A.rows[i], 0), A.n_rows - 1) : i) * A.stride[side];
  };
  float k0[8], mn[8], mx[8], s1[8], s2[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { mn[i] = INFINITY; mx[i] = -INFINITY; s1[i] = s2[i] = k0[i] = 0.f; }
  for (int base = stats ? 0 : t0 & ~3; base < cnt; base += 16) {        // sixteen rows of the page at a time
    Raw8<T> raw[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (base + 4 * q < cnt) load_raw8(source(min(max(base + 4 * q + r, stats ? 0 : t0), cnt - 1)), raw[q]);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int t = base + 4 * q + r;
      if (t >= t0 && t < cnt) {
        if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<uint4*>(page + (size_t)t * kD) = raw[q].a;
        } else {
          *reinterpret_cast<float4*>(page + (size_t)t * kD) = raw[q].a;
          *reinterpret_cast<float4*>(page + (size_t)t * kD + 4) = raw[q].b;
        }
      }
      if (stats && base + 4 * q < cnt) {
        const bool in = t < cnt;
        float y[8];
        widen8(raw[q], y);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (base == 0 && q == 0) k0[i] = __shfl(y[i], c);             // token 0
          mn[i] = fminf(mn[i], in ? y[i] : INFINITY);
          mx[i] = fmaxf(mx[i], in ? y[i] : -INFINITY);
          const float dx = in ? y[i] - k0[i] : 0.f;
          s1[i] += dx;
          s2[i] = fmaf(dx, dx, s2[i]);
        }
      }
    }
  }
  if (!stats || b < 0 || b >= A.B || lp < 0 || lp / P >= A.Mmax) return;
  const size_t rec = (((size_t)b * A.Hkv + h) * A.Mmax + lp / P) * 2 * kD;
  store_page_stats<T>(mn, mx, s1, s2, k0, cnt, (T*)A.box + rec, (T*)A.gauss + rec, A.box8 != nullptr ? A.box8 + rec : nullptr);
}

template <typename T>
__global__ __launch_bounds__(kAppendThreads) void append_rows_kernel(const AppendRowsArgs A) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // stretches of the rows per XCD, as in the 8-bit append: with fewer rows to a wavefront than to a page not every one begins a run
  const unsigned x = blockIdx.x % kXcds, each = gridDim.x / kXcds, rest = gridDim.x % kXcds;
  const long long wg = (long long)(x * each + min(x, rest) + blockIdx.x / kXcds);
  const long long id = wg * kAppendWaves + w, first = (id >> 1) / A.Hkv * A.block;
  const int side = (int)(id & 1), h = (int)((id >> 1) % A.Hkv);
  if (first >= A.T) return;
  const int i0 = (int)first;
  // lane l: tokens i0 + l and i0 + 64 + l; a token goes on the run of the one before it, or it does not
  auto slot_of = [&](int i) -> int64_t {
    const int64_t s = i >= 0 && i < A.T ? A.slots[i] : -1;
    return s >= 0 && s < A.n_slots ? s : -1;
  };
  const int64_t sa = slot_of(i0 + lane), sb = slot_of(i0 + 64 + lane);
  int64_t pa = __shfl_up((long long)sa, 1), pb = __shfl_up((long long)sb, 1);
  const int64_t before = slot_of(i0 - 1), sa63 = __shfl((long long)sa, 63);
  pa = lane == 0 ? before : pa;
  pb = lane == 0 ? sa63 : pb;
  const bool ga = sa > 0 && pa == sa - 1 && sa % A.P != 0, gb = sb > 0 && pb == sb - 1 && sb % A.P != 0;
  const uint64_t goes_on = __ballot(ga), goes_on2 = __ballot(gb);
  uint64_t begins = __ballot(sa >= 0 && !ga && lane < A.block);
  while (begins != 0) {
    const int l = __builtin_ctzll(begins);
    begins &= begins - 1;
    // tokens behind l that go on: ones from bit l + 1 of the two masks; a page has at most 64 tokens
    const uint64_t m = l == 63 ? goes_on2 : (goes_on >> (l + 1)) | (goes_on2 << (63 - l));
    const int len = 1 + (m == ~0ull ? 64 : __builtin_ctzll(~m));
    append_rows_run<T>(A, side, h, i0 + l, len, __shfl((long long)sa, l));
  }
}

void launch_cache_append(const Dims& dm, const ekv_cache_view& c, const ekv_stats_view* stats, const ekv_token_map& tok,
                         const int32_t* rows, int n_rows, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                         hipStream_t st) {
  AppendRowsArgs a{};
  a.x[0] = k_new; a.x[1] = v_new; a.stride[0] = k_stride; a.stride[1] = v_stride;
  a.pool[0] = c.k_pool; a.pool[1] = c.v_pool;
  if (stats != nullptr) { a.box = stats->box; a.gauss = stats->gauss; a.box8 = (uint8_t*)stats->box8; }
  a.slots = tok.slots; a.seq = tok.seq; a.pos = tok.pos;
  a.rows = rows; a.n_rows = n_rows;
  a.T = tok.max_tokens; a.B = dm.B; a.Hkv = dm.Hkv; a.HkvPool = dm.HkvPool; a.P = dm.P; a.Mmax = dm.Mmax;
  a.n_slots = (int64_t)c.n_phys_pages * dm.P;
  // Tokens per wavefront: one where there are few, so that a step's go on at once, up to 32 (64 with pages that long) where most
  // are prompts', of which one in P begins a run.  us, up to 4096 wavefronts / 16384 / 65536: 157 single tokens 8.4 / 8.5 / 8.5, 1000
  // 23.3 / 25.1 / 25.1, 2000 tokens of 20 chunks 11.8 / 14.4 / 18.5, 24000 of 6 prompts 64.1 / 64.3 / 70.6, 16411 float32 in pages of 12
  // 75.3 / 75.3 / 71.7, 16000 in pages of 64 48.9 / 45.0 / 62.1.
  a.block = 1;
  while (a.block < (dm.P < 64 ? 32 : 64) && (long long)a.T * dm.Hkv * 2 / a.block > 4096) a.block *= 2;
  const long long waves = (long long)((a.T + a.block - 1) / a.block) * dm.Hkv * 2;
  const dim3 grid((unsigned)((waves + kAppendWaves - 1) / kAppendWaves)), block(kAppendThreads);
  if (dm.dtype == EKV_F32) hipLaunchKernelGGL(append_rows_kernel<float>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(append_rows_kernel<bf16_t>, grid, block, 0, st, a);
}

}  // namespace ekv
