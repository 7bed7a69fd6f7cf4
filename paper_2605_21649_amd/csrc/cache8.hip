// Block tables and slots from request lengths, and the append that quantises into the 8-bit cache.
#include "ekv_cache8.h"
#include "ekv_internal.h"

namespace ekv {

// ------------------------------------------------------------------------------------------
// block tables and slots
// ------------------------------------------------------------------------------------------
// Where a row of a step goes depends on the lengths of all sequences before its own: two prefix sums over the batch (rows,
// new pages).  Every workgroup computes them for itself, in LDS, and then does its share of the rows: a few kilobytes read
// again by each from the caches cost less than a second launch (about 4 us) or a wait between workgroups.  Nothing is
// read that the launch writes (block-table entries of new pages are taken from the free list), so no order is needed.
// Bound by latency at the sizes of a decode step and by the writes of 16 bytes per row for prompts.
constexpr int kMapThreads = 256;
constexpr uint32_t kCountMost = 1u << 30;       // sums of rows stay here

struct MapArgs {
  const int32_t* seq_lens; const int32_t* n_new; int32_t* block_table; const int32_t* free_pages; const int32_t* n_free;
  ekv_token_map tok; int32_t* new_lens; int32_t* n_left;
  int B, P, Mmax, capacity, rows_per_block;
};

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, kCountMost); }    // a, b <= 2^30

// Exclusive prefix over the threads of a workgroup, saturating; total: the sum.  Starts and ends with a barrier.
__device__ __forceinline__ uint32_t block_exclusive_sat(uint32_t v, uint32_t* wsum, uint32_t& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t inc = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(inc, d);
    if (lane >= d) inc = sat_add(inc, o);
  }
  __syncthreads();
  if (lane == 63) wsum[w] = inc;
  __syncthreads();
  uint32_t base = __shfl_up(inc, 1);
  if (lane == 0) base = 0;
  uint32_t sum = 0;
#pragma unroll
  for (int i = 0; i < kMapThreads / 64; ++i) {
    if (i == w) base = sat_add(base, sum);
    sum = sat_add(sum, wsum[i]);
  }
  total = sum;
  return base;
}

__global__ __launch_bounds__(kMapThreads) void map_tokens_kernel(const MapArgs A) {
  extern __shared__ int32_t lds[];
  int32_t* start = lds;                          // [B + 1] first row of a sequence
  int32_t* have = lds + A.B + 1;                 // [B] its pages, with the pages taken in front of it: see below
  int32_t* len = have + A.B;                     // [B] its tokens, -1 if it is not served
  __shared__ uint32_t wsum[kMapThreads / 64];
  __shared__ int32_t taken_most[kMapThreads / 64];
  const int tid = threadIdx.x, B = A.B, P = A.P;
  const int room = A.Mmax * P;                   // at most 2^30
  const int n_free = min(max(A.n_free[0], 0), A.capacity);
  const int per = (B + kMapThreads - 1) / kMapThreads, b0 = min(tid * per, B), b1 = min(b0 + per, B);
  uint32_t rows = 0, total = 0;
  for (int b = b0; b < b1; ++b) rows = sat_add(rows, (uint32_t)min(max(A.n_new[b], 0), (int)kCountMost));
  uint32_t at = block_exclusive_sat(rows, wsum, total);
  uint32_t pages = 0;
  for (int b = b0; b < b1; ++b) {
    const int n = A.seq_lens[b], c = A.n_new[b];
    start[b] = (int)at;
    at = sat_add(at, (uint32_t)min(max(c, 0), (int)kCountMost));
    const bool fits = c > 0 && n >= 0 && n <= room && c <= room - n && at <= (uint32_t)A.tok.max_tokens;
    const int need = fits ? (n + c + P - 1) / P - (n + P - 1) / P : 0;
    pages += need;                               // of sequences whose rows lie below max_tokens: below 2^30 + B together
    len[b] = fits ? n : -1;
    have[b] = need;
  }
  if (tid == 0) start[B] = (int)total;
  uint32_t all_pages = 0;
  uint32_t before = block_exclusive_sat(pages, wsum, all_pages);
  int most = 0;
  for (int b = b0; b < b1; ++b) {
    const int need = have[b];
    const uint32_t end = before + need;
    const bool served = len[b] >= 0 && (need == 0 || end <= (uint32_t)n_free);
    if (served && need > 0) most = (int)end;
    // page p >= ceil(n / P) of the sequence is new page (p - ceil(n / P)) + before of the call: free_pages[have - p]
    const int n = len[b];
    have[b] = served ? n_free - 1 - (int)before + (n + P - 1) / P : 0;
    if (!served) len[b] = -1;
    before = end;
    if (blockIdx.x == 0) {
      const int c = A.n_new[b], was = A.seq_lens[b];
      A.tok.start[b] = start[b];
      A.tok.n_mapped[b] = served ? c : 0;
      A.new_lens[b] = served ? was + c : was;
    }
  }
  most = (int)wave_max_u((uint32_t)most);
  if ((tid & 63) == 0) taken_most[tid >> 6] = most;
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) {
    A.tok.start[B] = (int)total;
    for (int i = 0; i < kMapThreads / 64; ++i) most = max(most, taken_most[i]);
    A.n_left[0] = n_free - most;
  }
  const int r0 = blockIdx.x * A.rows_per_block, r1 = min(r0 + A.rows_per_block, A.tok.max_tokens);
  for (int i = r0 + tid; i < r1; i += kMapThreads) {
    int lo = 0, hi = B;                          // start[lo] <= i: the last such sequence has the row, if any has
    while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (start[mid] <= i) lo = mid; else hi = mid; }
    const int n = len[lo];
    int64_t slot = -1;
    int32_t pos = -1, seq = -1;
    if (n >= 0 && i < start[lo + 1]) {
      pos = n + (i - start[lo]);
      seq = lo;
      const int p = pos / P, t = pos - p * P;
      int32_t* entry = A.block_table + (size_t)lo * A.Mmax + p;
      int32_t phys;
      if (p < (n + P - 1) / P) phys = *entry;
      else {
        phys = A.free_pages[have[lo] - p];
        if (t == 0) *entry = phys;               // the page's first row writes its entry
      }
      slot = (int64_t)phys * P + t;
    }
    A.tok.slots[i] = slot;
    A.tok.seq[i] = seq;
    A.tok.pos[i] = pos;
  }
}

struct ReleaseArgs {
  const int32_t* release; const int32_t* seq_lens; const int32_t* block_table; int32_t* free_pages; const int32_t* n_free;
  int32_t* new_lens; int32_t* n_left;
  int B, P, Mmax, capacity;
};
// The pages of ended sequences, one after the other behind the free ones: one prefix sum, then every workgroup its share.
__global__ __launch_bounds__(kMapThreads) void release_pages_kernel(const ReleaseArgs A) {
  extern __shared__ int32_t pre[];               // [B + 1] pages returned before a sequence
  __shared__ uint32_t wsum[kMapThreads / 64];
  const int tid = threadIdx.x, B = A.B;
  const int n_free = min(max(A.n_free[0], 0), A.capacity);
  auto pages_of = [&](int b) { return A.release[b] != 0 ? (uint32_t)min((max(A.seq_lens[b], 0) + (int64_t)A.P - 1) / A.P, (int64_t)A.Mmax) : 0u; };
  const int per = (B + kMapThreads - 1) / kMapThreads, b0 = min(tid * per, B), b1 = min(b0 + per, B);
  uint32_t mine = 0, total = 0;
  for (int b = b0; b < b1; ++b) mine = sat_add(mine, pages_of(b));
  uint32_t at = block_exclusive_sat(mine, wsum, total);
  for (int b = b0; b < b1; ++b) {
    pre[b] = (int)at;
    at = sat_add(at, pages_of(b));
    if (blockIdx.x == 0) A.new_lens[b] = A.release[b] != 0 ? 0 : A.seq_lens[b];
  }
  if (tid == 0) pre[B] = (int)total;
  __syncthreads();
  const int give = (int)min(total, (uint32_t)(A.capacity - n_free));
  if (blockIdx.x == 0 && tid == 0) A.n_left[0] = n_free + give;
  for (int i = blockIdx.x * kMapThreads + tid; i < give; i += gridDim.x * kMapThreads) {
    int lo = 0, hi = B;
    while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (pre[mid] <= i) lo = mid; else hi = mid; }
    A.free_pages[n_free + i] = A.block_table[(size_t)lo * A.Mmax + (i - pre[lo])];
  }
}

// ------------------------------------------------------------------------------------------
// the quantising append
// ------------------------------------------------------------------------------------------
// One wavefront per run (rows with consecutive slots of one page), KV head and side (K or V): the scale needs the maximum
// of the whole run before the first code can be written.  Lane (r, c) has channels 8c..8c+7 of the page's rows r, r + 4, ..:
// whole lines with every load and store, and the rows' order of ekv_stats_build in the sums of the statistics, which are taken
// from the stored values and equal that call's to the last bit.  A lane reads and writes the same rows of the page, so older
// tokens that a grown scale rounds again need no exchange.  Rows of a chunk that the run does not have are read as one that
// it has, which no maximum or minimum minds.  The bytes are the new rows'; the conversions with a scale leave about ten
// instructions to an element of K with its statistics and three to one of V, without which the arithmetic was what bounded it.
constexpr int kAppendThreads = 256, kAppendWaves = kAppendThreads / 64;

struct AppendArgs {
  const void* x[2]; int64_t stride[2];           // new rows: K, V
  e4m3_t* pool[2]; float* scale[2];
  void* box; void* gauss; uint8_t* box8;         // null: no statistics
  const int64_t* slots; const int32_t* seq; const int32_t* pos;
  int T, block, B, Hkv, HkvPool, P, Mmax;        // T rows, `block` of them per wavefront
  int64_t n_slots;                               // slots of the pool
};

// Sum, minimum or maximum over the four rows of lanes of 8 values each: lane (r, c) gets entries e and e + 1, e = 2 (r / 2) + 4 (r % 2).
// The pairs are those of exchanges over 16 and then 32 lanes; each step passes on the half of the entries that the other needs.
template <typename F> __device__ __forceinline__ float2 rows_reduce(const float (&x)[8], F&& f) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[i]), __float_as_uint(x[i + 4]), false, false);
    y[i] = f(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  float z[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(y[i]), __float_as_uint(y[i + 2]), false, false);
    z[i] = f(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  return make_float2(z[0], z[1]);
}
__device__ __forceinline__ void store2(float* p, float2 v) { *reinterpret_cast<float2*>(p) = v; }
__device__ __forceinline__ void store2(bf16_t* p, float2 v) {
  *reinterpret_cast<uint32_t*>(p) = float_to_bf16_bits(v.x) | ((uint32_t)float_to_bf16_bits(v.y) << 16);
}

// ONE: pages of up to 16 tokens, one chunk (its registers let four wavefronts share a SIMD).
template <typename T, bool ONE>
__device__ __forceinline__ void append_run(const AppendArgs& A, int side, int h, int row0, int len, uint32_t slot) {
  const int lane = threadIdx.x & 63, r = lane >> 4, c = lane & 15;
  const int P = A.P, t0 = (int)(slot % (uint32_t)P), cnt = t0 + len;
  const size_t page = (size_t)(slot / (uint32_t)P) * A.HkvPool + h;
  e4m3_t* codes = A.pool[side] + page * P * kD + 8 * c;
  float* scale = A.scale[side] + page;
  const T* x = (const T*)A.x[side] + (int64_t)row0 * A.stride[side] + h * kD + 8 * c;
  const bool stats = side == 0 && A.box != nullptr;
  // sixteen rows of the page at a time
  Raw8<T> raw[4];
  Raw8<e4m3_t> old[4];
  // whether four rows of a chunk hold one of the run's, or one of the page's at all (wave-uniform: a step's single token has one
  // such four, and what the page does not hold yet costs nothing)
  auto any_new = [&](int chunk, int s) { return 16 * chunk + 4 * s + 3 >= t0 && 16 * chunk + 4 * s < cnt; };
  auto any_old = [&](int chunk, int s) { return 16 * chunk + 4 * s < t0; };
  auto request = [&](int chunk) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
      if (any_new(chunk, s)) load_raw8(x + (int64_t)min(max(16 * chunk + 4 * s + r - t0, 0), len - 1) * A.stride[side], raw[s]);
  };
  auto request_old = [&](int chunk) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
      if (any_old(chunk, s)) load_raw8(codes + (size_t)min(16 * chunk + 4 * s + r, t0 - 1) * kD, old[s]);
  };
  const int first = ONE ? 0 : t0 / 16, last = ONE ? 0 : (cnt - 1) / 16;
  const float s_was = t0 > 0 ? *scale : 0.f;
  int b = -1, lp = -1;
  if (stats) { b = A.seq[row0]; lp = A.pos[row0]; }
  uint32_t top = 0;
  for (int chunk = last; chunk >= first; --chunk) {        // downwards: the first chunk's rows stay in the registers
    request(chunk);
    if (chunk == first && stats && t0 > 0) request_old(0);
#pragma unroll
    for (int s = 0; s < 4; ++s)
      if (any_new(chunk, s)) top = max_bits(raw[s], top);
  }
  top = wave_max_u(max_as_float_bits<T>(top));
  if (top >= 0x7f800000u) {                                // infinities or NaN among them: once more without
    float m = 0.f;
    for (int chunk = last; chunk >= first; --chunk) {
      if constexpr (!ONE) request(chunk);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        if (!any_new(chunk, s)) continue;
        float v[8];
        widen8(raw[s], v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float f = __builtin_fabsf(v[i]);
          m = fmaxf(m, f < INFINITY ? f : 0.f);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    top = __float_as_uint(wave_max(m));
  }
  const float s_new = two_to(scale_exponent(__uint_as_float(top)));
  const bool grown = t0 > 0 && s_new > s_was;
  const float s = t0 == 0 || grown ? s_new : s_was;
  const bool beyond = !(__uint_as_float(top) <= kMaxCode * s);     // the largest scale is too small
  if (lane == 0 && (t0 == 0 || grown)) *scale = s;
  float k0[8], mn[8], mx[8], s1[8], s2[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { mn[i] = INFINITY; mx[i] = -INFINITY; s1[i] = s2[i] = k0[i] = 0.f; }
  for (int chunk = stats || grown ? 0 : first; chunk <= last; ++chunk) {
    const bool has_old = 16 * chunk < t0 && (stats || grown);      // the same for the whole wavefront, as all but `fresh`
    if (chunk > first) request(chunk);
    if (has_old && (chunk > 0 || !stats)) request_old(chunk);
    uint2 now[4];
    if (beyond) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (!any_new(chunk, q)) continue;
        float v[8];
        widen8(raw[q], v);
        now[q] = codes8_clamped(v, s);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (any_new(chunk, q)) now[q] = codes8(raw[q], s);
    }
    if (has_old) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (!any_old(chunk, q)) continue;
        if (grown) {
          float v[8];
          values8(old[q].a, s_was, v);
          old[q].a = make_uint2(codes4(v[0], v[1], v[2], v[3], s), codes4(v[4], v[5], v[6], v[7], s));
          __builtin_amdgcn_sched_barrier(0);
        }
        if (16 * chunk + 4 * q + r < t0) now[q] = old[q].a;
      }
    }
    const int from = grown ? 0 : t0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int t = 16 * chunk + 4 * q + r;
      if (t >= from && t < cnt) *reinterpret_cast<uint2*>(codes + (size_t)t * kD) = now[q];
    }
    if (stats) {
      auto add = [&](auto whole) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (!decltype(whole)::value && 16 * chunk + 4 * q >= cnt) break;
          float y[8];
          values8(now[q], s, y);
          const bool in = decltype(whole)::value || 16 * chunk + 4 * q + r < cnt;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (chunk == 0 && q == 0) k0[i] = __shfl(y[i], c);     // token 0
            mn[i] = fminf(mn[i], y[i]);
            mx[i] = fmaxf(mx[i], y[i]);
            const float dx = in ? y[i] - k0[i] : 0.f;
            s1[i] += dx;
            s2[i] = fmaf(dx, dx, s2[i]);
          }
          __builtin_amdgcn_sched_barrier(0);               // a row at a time: four at once cost registers and hide nothing more
        }
      };
      if (16 * chunk + 16 <= cnt) add(IntC<1>{}); else add(IntC<0>{});
    }
  }
  if (!stats || b < 0 || b >= A.B || lp < 0 || lp / P >= A.Mmax) return;
  const float inv_n = 1.0f / (float)cnt;
  const float2 lo = rows_reduce(mn, [](float a, float b) { return fminf(a, b); }), hi = rows_reduce(mx, [](float a, float b) { return fmaxf(a, b); });
  const float2 d1 = rows_reduce(s1, [](float a, float b) { return a + b; }), d2 = rows_reduce(s2, [](float a, float b) { return a + b; });
  const bool up = r >> 1, far = r & 1;                     // channels 2 up + 4 far + 0, 1
  auto mine = [&](int i) { return far ? (up ? k0[i + 6] : k0[i + 4]) : (up ? k0[i + 2] : k0[i]); };
  auto variance = [&](float m1, float m2) { return fmaxf(fmaf(-m1, m1, m2 * inv_n), 0.f); };
  const float m1x = d1.x * inv_n, m1y = d1.y * inv_n;
  const size_t rec = (((size_t)b * A.Hkv + h) * A.Mmax + lp / P) * 2 * kD;
  const int e = 2 * up + 4 * far;
  T* box = (T*)A.box + rec + 8 * c + e; T* gauss = (T*)A.gauss + rec + 8 * c + e;
  store2(box, lo);
  store2(box + kD, hi);
  store2(gauss, make_float2(mine(0) + m1x, mine(1) + m1y));
  store2(gauss + kD, make_float2(variance(m1x, d2.x), variance(m1y, d2.y)));
  if (A.box8 != nullptr) {
    uint8_t* u = A.box8 + rec + 16 * c + e;
    *reinterpret_cast<uint16_t*>(u) = (uint16_t)(f32_to_e4m3_directed<false>(lo.x) | (f32_to_e4m3_directed<false>(lo.y) << 8));
    *reinterpret_cast<uint16_t*>(u + 8) = (uint16_t)(f32_to_e4m3_directed<true>(hi.x) | (f32_to_e4m3_directed<true>(hi.y) << 8));
  }
}

template <typename T, bool ONE>
__global__ __launch_bounds__(kAppendThreads) __attribute__((amdgpu_waves_per_eu(ONE ? 4 : 3)))
void append8_kernel(const AppendArgs A) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Workgroups go to the XCDs in turn, and with fewer rows to a wavefront than to a page only every so many of them find the
  // beginning of a run: in stretches every XCD gets its share (16384 tokens, pages of 64: 44.7 -> 42.3 us with 64 rows to a
  // wavefront, 76 -> 48 with 16).
  const unsigned x = blockIdx.x % kXcds, each = gridDim.x / kXcds, rest = gridDim.x % kXcds;
  const int wg = (int)(x * each + min(x, rest) + blockIdx.x / kXcds);
  const int id = wg * kAppendWaves + w, side = id & 1, h = (id >> 1) % A.Hkv, i0 = (id >> 1) / A.Hkv * A.block;
  if (i0 >= A.T) return;
  // lane l: rows i0 + l and i0 + 64 + l; a row goes on the run of the one before it, or it does not
  auto slot_of = [&](int i) {
    const int64_t s = i >= 0 && i < A.T ? A.slots[i] : -1;
    return s >= 0 && s < A.n_slots ? (int)s : -1;          // n_slots < 2^30
  };
  const int sa = slot_of(i0 + lane), sb = slot_of(i0 + 64 + lane);
  int pa = __shfl_up(sa, 1), pb = __shfl_up(sb, 1);
  const int before = slot_of(i0 - 1);
  pa = lane == 0 ? before : pa;
  pb = lane == 0 ? __builtin_amdgcn_readlane(sa, 63) : pb;
  const bool ga = sa > 0 && pa == sa - 1 && sa % A.P != 0, gb = sb > 0 && pb == sb - 1 && sb % A.P != 0;
  const uint64_t goes_on = __ballot(ga), goes_on2 = __ballot(gb);
  uint64_t begins = __ballot(sa >= 0 && !ga && lane < A.block);
  while (begins != 0) {
    const int l = __builtin_ctzll(begins);
    begins &= begins - 1;
    // rows behind l that go on: ones from bit l + 1 of the two masks
    const uint64_t m = l == 63 ? goes_on2 : (goes_on >> (l + 1)) | (goes_on2 << (63 - l));
    const int len = 1 + (m == ~0ull ? 64 : __builtin_ctzll(~m));
    append_run<T, ONE>(A, side, h, i0 + l, len, (uint32_t)__builtin_amdgcn_readlane(sa, l));
  }
}

// ------------------------------------------------------------------------------------------
// launchers
// ------------------------------------------------------------------------------------------
void launch_map_tokens(const Dims& dm, const int32_t* seq_lens, const int32_t* n_new, int32_t* block_table,
                       const int32_t* free_pages, const int32_t* n_free, int capacity, const ekv_token_map& tok,
                       int32_t* new_lens, int32_t* n_left, hipStream_t st) {
  MapArgs a{seq_lens, n_new, block_table, free_pages, n_free, tok, new_lens, n_left, dm.B, dm.P, dm.Mmax, capacity, kMapThreads};
  const int blocks = (tok.max_tokens + a.rows_per_block - 1) / a.rows_per_block;
  const size_t lds = (size_t)(3 * dm.B + 1) * sizeof(int32_t);
  hipLaunchKernelGGL(map_tokens_kernel, dim3(blocks), dim3(kMapThreads), lds, st, a);
}

void launch_release_pages(const Dims& dm, const int32_t* release, const int32_t* seq_lens, const int32_t* block_table,
                          int32_t* free_pages, const int32_t* n_free, int capacity, int32_t* new_lens, int32_t* n_left,
                          hipStream_t st) {
  ReleaseArgs a{release, seq_lens, block_table, free_pages, n_free, new_lens, n_left, dm.B, dm.P, dm.Mmax, capacity};
  const long long pages = (long long)dm.B * dm.Mmax < capacity ? (long long)dm.B * dm.Mmax : capacity;
  const long long blocks = (pages + kMapThreads - 1) / kMapThreads;
  hipLaunchKernelGGL(release_pages_kernel, dim3((unsigned)(blocks < 256 ? blocks : 256)), dim3(kMapThreads),
                     (size_t)(dm.B + 1) * sizeof(int32_t), st, a);
}

void launch_cache8_append(const Dims& dm, const ekv_cache8_view& c, const ekv_stats_view* stats, const ekv_token_map& tok,
                          const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride, hipStream_t st) {
  AppendArgs a{};
  a.x[0] = k_new; a.x[1] = v_new; a.stride[0] = k_stride; a.stride[1] = v_stride;
  a.pool[0] = (e4m3_t*)c.k_pool; a.pool[1] = (e4m3_t*)c.v_pool; a.scale[0] = c.k_scale; a.scale[1] = c.v_scale;
  if (stats != nullptr) { a.box = stats->box; a.gauss = stats->gauss; a.box8 = (uint8_t*)stats->box8; }
  a.slots = tok.slots; a.seq = tok.seq; a.pos = tok.pos;
  a.T = tok.max_tokens; a.B = dm.B; a.Hkv = dm.Hkv; a.HkvPool = dm.HkvPool; a.P = dm.P; a.Mmax = dm.Mmax;
  a.n_slots = (int64_t)c.n_phys_pages * dm.P;
  // Rows per wavefront: one where there are few, so that a step's rows go on at once; up to 32 where most rows are prompts', of
  // which one in P begins a run and the others' wavefronts would only find that out, 64 with pages that long.  us, 4096
  // wavefronts / 16384 where there are rows enough: 4096 tokens of prompts 11.9 / 17.3, 1024 single tokens 19.4 / 22.5.  At most
  // 16 rows / 32 / 64, 16384 tokens of prompts: pages of 4 41 / 44 / 53 (10000 tokens), of 16 32.6 / 30.0 / 28.7 (32768: 56.0 /
  // 52.4 / 53.2), of 32 43.5 / 40.2 / 46.1, of 48 44.5 / 39.9 / 48.8, of 64 48.1 / 45.1 / 42.3.
  const bool one = dm.P <= 16;
  a.block = 1;
  while (a.block < (dm.P < 64 ? 32 : 64) && (long long)a.T * dm.Hkv * 2 / a.block > 4096) a.block *= 2;
  const long long waves = (long long)((a.T + a.block - 1) / a.block) * dm.Hkv * 2;
  const dim3 grid((unsigned)((waves + kAppendWaves - 1) / kAppendWaves)), block(kAppendThreads);
  if (dm.dtype == EKV_F32) {
    if (one) hipLaunchKernelGGL((append8_kernel<float, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((append8_kernel<float, false>), grid, block, 0, st, a);
  } else {
    if (one) hipLaunchKernelGGL((append8_kernel<bf16_t, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((append8_kernel<bf16_t, false>), grid, block, 0, st, a);
  }
}

}  // namespace ekv
