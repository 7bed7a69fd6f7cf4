// Softmax attention of one query token per sequence over the 8-bit cache: every page, or a page list per query head.
//
// One pass over K and V with the running maximum and sum; scores and weighted values both go through the matrix cores
// (ekv_attn8.h has the scores).  Steps of 32 tokens, four octets: lane (c, g) then holds the scores of its head for tokens 2g and
// 2g + 1 of each, and that is the layout in which the next product wants its rows (row c, eight tokens of group g), so the weights
// go from one product to the next without leaving the lane.  Float32 weights are three bf16 terms that sum to them exactly
// (8 + 8 + 8 bits); the columns that repeat the heads hold them: copy 0 of a head contributes the first term, copy 1 the
// second, copy 2 the third, as rows of one product (eight heads have two copies and take a second product).  Values are 8
// bytes of each token's row per lane, whole lines per load, transposed in pairs of tokens by byte permutes and widened with
// their page's scale (exact), so that sums are float32 sums of exact products.
// The maximum only has to keep exp in range: it is brought up to date, with the exchange and the rescaling that takes, when a
// score passes it by more than 2^kSlack, not at every step.
#include "ekv_attn8.h"

namespace ekv {

constexpr int kAttnWaves = 4;                    // wavefronts of a workgroup, or twice as many
constexpr int kStep = 32;                        // tokens per step of a wavefront
constexpr int kRec = kD + 2;                     // floats per head of a partial result: o[128], maximum, sum
constexpr float kSlack = 8.f;                    // weights stay below 2^8
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

struct Attn8Args {
  ScoreArgs s;                                   // q, lists, lengths, sizes; k_pool: codes; zscale: scale * log2(e)
  const float* k_scale; const float* v_scale; const e4m3_t* v_pool;
  float* out; float* lse;
  float* part;                                   // [grid + U][G][kRec]
  int32_t* pre;                                  // [U + 1] steps before a unit, for the join
  PageDiv page_div;
  int per_unit;                                  // 1: workgroup i has unit i, whole
};

template <bool DENSE>
__device__ __forceinline__ int unit_steps(const ScoreArgs& A, int u) {
  if (DENSE) return (int)(((int64_t)clampi(A.seq_lens[u / A.Hkv], 0, A.Mmax * A.P) + kStep - 1) / kStep);
  return (int)(((int64_t)clampi(A.n_sel[u], 0, A.cap) * A.P + kStep - 1) / kStep);
}

template <bool DENSE>
__global__ __launch_bounds__(1024) void attn8_prefix_kernel(const Attn8Args A) {
  __shared__ int wsum[16];
  block_exclusive_prefix<1024>(A.s.U, [&](int u) { return unit_steps<DENSE>(A.s, u); }, A.pre, wsum);
}

// A step's data as loaded.  K: the lane's codes of each octet; V: channels 8c..8c+7 of tokens 2g, 2g + 1 of each.
struct Step8 {
  uint4 k[4];
  uint2 v[8];
  float ks[4], vs[4];
  int left[4];                                   // valid tokens from the lane's first of an octet on (2 or more: both)
};
template <bool STREAM> __device__ __forceinline__ uint2 load8b(const e4m3_t* p) {
  typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
  if constexpr (STREAM) return __builtin_bit_cast(uint2, __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(p)));
  else return *reinterpret_cast<const uint2*>(p);
}

template <typename T, int G, bool DENSE, bool OCTETS, bool STREAM, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2)))
void attn8_kernel(const Attn8Args AA) {
  const ScoreArgs& A = AA.s;
  extern __shared__ int pre_lds[];
  __shared__ int wsum[NW];
  __shared__ float s_o[NW][G][kD];
  __shared__ float s_m[NW][G], s_l[NW][G];
  const int P = A.P, lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const e4m3_t* k_pool = (const e4m3_t*)A.k_pool;
  const uint32_t k_off = (OCTETS ? key_token(c) * kD : 0) + key_offset(c, g), v_off = (OCTETS ? 2 * g * kD : 0) + 8 * c;
  const int head = column_head(c, G), copy = column_copy(c, G);
  const bool in_lds = A.pre_g == nullptr;
  int first_unit = 0, begin = 0, end = 0;
  // Workgroups go to the XCDs in turn: each XCD gets a stretch of the steps, so that the lists of a group's heads, which name many
  // of the same pages, meet in one L2 (64 x 8192 tokens, lists of 32 pages, the same for a group: 51.1 -> 42.2 us a call).
  const int wg = !DENSE && gridDim.x % kXcds == 0 ? (int)(blockIdx.x % kXcds * (gridDim.x / kXcds) + blockIdx.x / kXcds) : (int)blockIdx.x;
  auto range = [&](auto pre) {                   // this workgroup's steps
    const int total = uniform(pre[A.U]), W = gridDim.x, i = wg, per = total / W, rem = total - per * W;
    begin = i * per + min(i, rem);
    end = begin + per + (i < rem ? 1 : 0);
    first_unit = wave_last_at_most(pre, A.U, begin);
  };
  if (AA.per_unit) {
    first_unit = wg;
    begin = 0;
    end = max(unit_steps<DENSE>(A, first_unit), 1);          // one step at least, if of nothing: it writes the row
  } else if (in_lds) {
    block_exclusive_prefix<(64 * NW)>(A.U, [&](int u) { return unit_steps<DENSE>(A, u); }, pre_lds, wsum);
    range((const int*)pre_lds);
    if (blockIdx.x == 0)
      for (int u = threadIdx.x; u <= A.U; u += (64 * NW)) AA.pre[u] = pre_lds[u];
  } else {
    range(A.pre_g);
  }
  const int last = (DENSE ? A.Mmax : A.cap) - 1;
  const uint32_t take1 = copy >= 1 ? 0xffff0000u : 0u, take2 = copy >= 2 ? 0xffff0000u : 0u;
  const uint32_t keep = copy < 3 ? ~0u : 0u, first = copy == 0 ? ~0u : 0u;

  int unit = first_unit;
  for (int at = begin; at < end;) {
    int u_begin = 0, u_end = 0;
    auto bounds = [&](auto pre) {
      while (at >= uniform(pre[unit + 1])) ++unit;
      u_begin = uniform(pre[unit]); u_end = uniform(pre[unit + 1]);
    };
    if (AA.per_unit) u_end = end;
    else if (in_lds) bounds((const int*)pre_lds);
    else bounds(A.pre_g);
    const int seg_end = min(end, u_end), n_steps = seg_end - at;
    const int b = DENSE ? unit / A.Hkv : unit / A.Hq, hkv = DENSE ? unit % A.Hkv : unit % A.Hq / (A.Hq / A.Hkv);
    const size_t row0 = DENSE ? (size_t)b * A.Hq + hkv * G : (size_t)unit;
    const int n = clampi(uniform_load(A.seq_lens + b), 0, A.Mmax * P);
    const int n_pos = DENSE ? n : clampi(uniform_load(A.n_sel + unit), 0, A.cap) * P;      // positions of the unit
    // a quarter of the segment for each wavefront
    const int st0 = at - u_begin + n_steps * w / NW, st1 = at - u_begin + n_steps * (w + 1) / NW;

    float m = -INFINITY, l = 0.f;
    f32x4_t acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (st0 < st1) {
      Query8<T, G> qb;
      qb.load((const T*)A.q + row0 * kD);
      // page slots [slot_base, slot_base + 64), one per lane
      int slot_base = -64, l_lp = 0, l_page = 0;
      float l_ks = 0.f, l_vs = 0.f;
      auto look_up = [&](int pos) {
        slot_base = uniform((int)page_div((uint32_t)pos, AA.page_div));
        const int slot = min(slot_base + lane, last);
        l_lp = clampi(DENSE ? slot : A.page_idx[(size_t)unit * A.cap + slot], 0, A.Mmax - 1);
        const int phys = clampi(A.block_table[(size_t)b * A.Mmax + l_lp], 0, A.n_phys - 1);
        l_page = phys * A.HkvPool + hkv;
        l_ks = AA.k_scale[l_page];
        l_vs = AA.v_scale[l_page];
      };
      auto request = [&](int st, Step8& x) {
        const int p0 = st * kStep;
        if ((int)page_div((uint32_t)(p0 + kStep - 1), AA.page_div) >= slot_base + 64) look_up(p0);
#pragma unroll
        for (int o = 0; o < 4; ++o) {
          if constexpr (OCTETS) {
            const int p = p0 + 8 * o, slot = uniform((int)page_div((uint32_t)p, AA.page_div)), tok = p - slot * P, sl = slot - slot_base;
            const int page = __builtin_amdgcn_readlane(l_page, sl);
            const size_t at = ((size_t)page * P + tok) * kD;
            x.k[o] = load16<STREAM>(k_pool + at + k_off);
#pragma unroll
            for (int e = 0; e < 2; ++e) x.v[2 * o + e] = load8b<STREAM>(AA.v_pool + at + v_off + e * kD);
            x.ks[o] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(l_ks), sl));
            x.vs[o] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(l_vs), sl));
            x.left[o] = p < n_pos ? n - (__builtin_amdgcn_readlane(l_lp, sl) * P + tok) - 2 * g : 0;
          } else {
            const int pk = p0 + 8 * o + key_token(c), pv = p0 + 8 * o + 2 * g;
            const int sk = (int)page_div((uint32_t)pk, AA.page_div), sv = (int)page_div((uint32_t)pv, AA.page_div);
            x.k[o] = load16<STREAM>(k_pool + ((size_t)__shfl(l_page, sk - slot_base) * P + (pk - sk * P)) * kD + k_off);
            const size_t at = ((size_t)__shfl(l_page, sv - slot_base) * P + (pv - sv * P)) * kD;
#pragma unroll
            for (int e = 0; e < 2; ++e) x.v[2 * o + e] = load8b<STREAM>(AA.v_pool + at + v_off + e * kD);
            x.ks[o] = __shfl(l_ks, sk - slot_base);
            x.vs[o] = __shfl(l_vs, sv - slot_base);
            const int lp = __shfl(l_lp, sv - slot_base);     // by all lanes: behind the condition some sources would be idle
            x.left[o] = pv < n_pos ? n - (lp * P + (pv - sv * P)) : 0;
          }
        }
      };
      auto consume = [&](Step8& x) {
        float2 z[4];
        float top = -INFINITY;
        bool some_out = false;
#pragma unroll
        for (int o = 0; o < 4; ++o) {
          octet_scores<T, G>(x.k[o], x.ks[o], qb, z[o].x, z[o].y);
          z[o].x = x.left[o] > 0 ? A.zscale * z[o].x : -INFINITY;
          z[o].y = x.left[o] > 1 ? A.zscale * z[o].y : -INFINITY;
          top = fmaxf(top, fmaxf(z[o].x, z[o].y));
          some_out |= x.left[o] < 2;
        }
        if (__any(some_out)) {                               // what a page holds behind the last token counts for nothing, NaN too,
#pragma unroll                                               // nor does the scale of a page that nobody has
          for (int o = 0; o < 4; ++o) {
            if (x.left[o] < 2) x.v[2 * o + 1] = make_uint2(0u, 0u);
            if (x.left[o] < 1) { x.v[2 * o] = make_uint2(0u, 0u); x.vs[o] = 1.f; }
          }
        }
        if (__any(top > m + kSlack)) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float m_new = fmaxf(m, top);
          const float f = m_new > -INFINITY ? __builtin_amdgcn_exp2f(m - m_new) : 1.f;
          m = m_new;
          l *= f;
          f32x4_t fr;                                        // the factors of result rows 4g..4g+3
#pragma unroll
          for (int r = 0; r < 4; ++r) fr[r] = __shfl(f, 4 * g + r);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][r] *= fr[r];
          }
        }
        const float m_use = m > -INFINITY ? m : 0.f;
        u32x4_t pa, pb;                                      // rows of the second product: this lane's term of its head's weights
#pragma unroll
        for (int o = 0; o < 4; ++o) {
          uint32_t bits[2], low[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float p = __builtin_amdgcn_exp2f((e ? z[o].y : z[o].x) - m_use);
            l += p;
            float y = p - __uint_as_float(__float_as_uint(p) & take1);
            if constexpr (G == 8) {
              const float rest = p - __uint_as_float(__float_as_uint(p) & 0xffff0000u);
              low[e] = __float_as_uint(rest - __uint_as_float(__float_as_uint(rest) & 0xffff0000u));
            } else {
              y -= __uint_as_float(__float_as_uint(y) & take2);
            }
            bits[e] = __float_as_uint(y) & keep;
          }
          pa[o] = __builtin_amdgcn_perm(bits[1], bits[0], 0x07060302u);
          if constexpr (G == 8) pb[o] = __builtin_amdgcn_perm(low[1], low[0], 0x07060302u) & first;
        }
        // channel 8c + i of tokens 0..7 of the lane, i = 0..7: pairs of tokens side by side, then widened
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t lo[4], hi[4];                             // (token 2j, 2j + 1) of channels 0, 1 and of channels 2, 3 of the half
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t a = half ? x.v[2 * j].y : x.v[2 * j].x, d = half ? x.v[2 * j + 1].y : x.v[2 * j + 1].x;
            lo[j] = __builtin_amdgcn_perm(d, a, 0x05010400u);
            hi[j] = __builtin_amdgcn_perm(d, a, 0x07030602u);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            u32x4_t vb;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t src = i < 2 ? lo[j] : hi[j];
              vb[j] = i & 1 ? widen2<true>(src, x.vs[j]) : widen2<false>(src, x.vs[j]);
            }
            const bf16x8_t vv = __builtin_bit_cast(bf16x8_t, vb);
            f32x4_t& d = acc[4 * half + i];
            if constexpr (G == 8) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, pb), vv, d, 0, 0, 0);
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, pa), vv, d, 0, 0, 0);
          }
        }
      };
      Step8 x0, x1;
      request(st0, x0);
      for (int st = st0; st < st1; st += 2) {
        request(min(st + 1, st1 - 1), x1);
        consume(x0);
        if (st + 1 >= st1) break;
        request(min(st + 2, st1 - 1), x0);
        consume(x1);
      }
    }
    // the wavefront's sums: row r of the second product is of head column_head(r), whose rows are pairs (the copies c % 2)
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    __syncthreads();                                         // the previous segment's partial results have been read
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float even = acc[i][0] + acc[i][1], odd = acc[i][2] + acc[i][3];
      if constexpr (G == 1) even += odd;
      if constexpr (G <= 2) { even += __shfl_xor(even, 16); odd += __shfl_xor(odd, 16); }
      if constexpr (G <= 4) { even += __shfl_xor(even, 32); odd += __shfl_xor(odd, 32); }
      constexpr int kGroups = G >= 2 ? G / 2 : 1;
      if (g < kGroups) {
        s_o[w][G >= 2 ? 2 * g : 0][8 * c + i] = even;
        if constexpr (G >= 2) s_o[w][2 * g + 1][8 * c + i] = odd;
      }
    }
    if (g == 0 && copy == 0) { s_m[w][head] = m; s_l[w][head] = l; }
    __syncthreads();
    const bool whole = at == u_begin && seg_end == u_end;    // the unit is this workgroup's alone: no record, no join
    float* rec = AA.part + (size_t)(wg + unit) * G * kRec;
    for (int e = threadIdx.x; e < G * kD; e += (64 * NW)) {
      const int h = e / kD, ch = e % kD;
      float M = s_m[0][h];
#pragma unroll
      for (int i = 1; i < NW; ++i) M = fmaxf(M, s_m[i][h]);
      float L = 0.f, o = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        const float f = s_m[i][h] > -INFINITY ? __builtin_amdgcn_exp2f(s_m[i][h] - M) : 0.f;
        L = fmaf(s_l[i][h], f, L);
        o = fmaf(s_o[i][h][ch], f, o);
      }
      if (whole) {
        AA.out[(row0 + h) * kD + ch] = L > 0.f ? o / L : (L == 0.f ? 0.f : o);
        if (ch == 0) AA.lse[row0 + h] = L == 0.f ? -INFINITY : M * kLn2 + __logf(L);
      } else {
        rec[h * kRec + ch] = o;
        if (ch == 0) { rec[h * kRec + kD] = M; rec[h * kRec + kD + 1] = L; }
      }
    }
    at = seg_end;
  }
}

// Joins the partial results of the units that several workgroups worked on, in their order, and writes those that have no token.
// One workgroup per unit and head; JG groups of 128 threads take the records in turn: eight, or two where the heads are many, which
// have few records each (8 x 128K tokens for 64 heads 7.5 -> 5.4 us).
template <int JG>
__global__ __launch_bounds__(JG * kD) void attn8_join_kernel(const Attn8Args A, int G, int W) {
  __shared__ float red[JG * kD / 64];
  __shared__ float g_o[JG][kD], g_l[JG];
  const int unit = blockIdx.x / G, h = blockIdx.x % G, tid = threadIdx.x, t = tid & (kD - 1), grp = tid >> 7;
  const size_t row = (size_t)unit * G + h;                   // [B][Hq]: units are (b, KV head) or (b, query head)
  const int begin = A.pre[unit], end = A.pre[unit + 1];
  if (begin == end) {
    if (tid < kD) A.out[row * kD + tid] = 0.f;
    if (tid == 0) A.lse[row] = -INFINITY;
    return;
  }
  const int total = A.pre[A.s.U], per = total / W, rem = total - per * W;
  auto wg_of = [&](int step) { return step < rem * (per + 1) ? step / (per + 1) : rem + (step - rem * (per + 1)) / per; };
  const int w0 = wg_of(begin), w1 = wg_of(end - 1);
  if (w0 == w1) return;                                      // written by that workgroup
  const float* rec0 = A.part + ((size_t)(w0 + unit) * G + h) * kRec;
  const int n = w1 - w0 + 1;
  // the first 4 JG records are fetched before the maximum is known, all there are as a rule
  float rm[4], rl[4], ro[4];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float* rec = rec0 + (size_t)min(i0 + u * JG, n - 1) * G * kRec;
      rm[u] = rec[kD]; rl[u] = rec[kD + 1]; ro[u] = rec[t];
    }
  };
  fetch(grp);
  float mx = fmaxf(fmaxf(rm[0], rm[1]), fmaxf(rm[2], rm[3]));
  for (int i = 4 * JG + tid; i < n; i += JG * kD) mx = fmaxf(mx, rec0[(size_t)i * G * kRec + kD]);
  const float M = block_max(mx, red);
  float L = 0.f, o = 0.f;
  for (int i0 = grp; i0 < n; i0 += 4 * JG) {
    if (i0 != grp) fetch(i0);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float f = i0 + u * JG < n && rm[u] > -INFINITY ? __builtin_amdgcn_exp2f(rm[u] - M) : 0.f;
      L = fmaf(rl[u], f, L);
      o = fmaf(ro[u], f, o);
    }
  }
  g_o[grp][t] = o;
  if (t == 0) g_l[grp] = L;
  __syncthreads();
  if (tid < kD) {
    float Ls = 0.f, os = 0.f;
    for (int i = 0; i < JG; ++i) { Ls += g_l[i]; os += g_o[i][tid]; }
    A.out[row * kD + tid] = Ls > 0.f ? os / Ls : (Ls == 0.f ? 0.f : os);
    if (tid == 0) A.lse[row] = Ls == 0.f ? -INFINITY : M * kLn2 + __logf(Ls);
  }
}

// Workgroups: the two that a compute unit holds, no more than there can be steps for their wavefronts.  With four a compute unit,
// half of which wait for the others to end, 8 x 128K tokens for 64 heads take 315 us for 299, lists of 4 x 128K 42.6 for 37.1;
// compiled for three or four wavefronts per SIMD (and as many workgroups) 306 / 39.9 and, with spills, 513 / 67.
// Workspaces are sized for kMostWgs.
constexpr int kMostWgs = 512;
static long long attn8_units(const Dims& dm, bool dense) { return (long long)dm.B * (dense ? dm.Hkv : dm.Hq); }
static int attn8_grid(const Dims& dm, bool dense, int most) {
  const long long steps = attn8_units(dm, dense) * (((long long)(dense ? dm.Mmax : dm.cap) * dm.P + kStep - 1) / kStep);
  const long long wgs = (steps + kAttnWaves - 1) / kAttnWaves;
  return (int)(wgs < most ? wgs : most);
}
static size_t attn8_pre_bytes(const Dims& dm, bool dense) { return (((size_t)attn8_units(dm, dense) + 1) * sizeof(int32_t) + 255) & ~(size_t)255; }

bool softmax8_supported(const Dims& dm, bool dense) {
  return attn8_units(dm, dense) * (((long long)(dense ? dm.Mmax : dm.cap) * dm.P + kStep - 1) / kStep) <= 0x7fffffff;
}

size_t softmax8_ws_bytes(const Dims& dm, bool dense) {
  const size_t recs = (size_t)attn8_units(dm, dense) + (size_t)attn8_grid(dm, dense, kMostWgs);
  return attn8_pre_bytes(dm, dense) + recs * (dense ? dm.G : 1) * kRec * sizeof(float);
}

// One workgroup per unit, without the prefix sums and the join, where no unit can be long and there are enough for the GPU, or
// they are so short that two launches take longer.  Calls, us, split / one workgroup per unit (of eight wavefronts where there are
// fewer than compute units): 512 units of 1024 tokens 37.4 / 28.6, of 2048 uneven ones 73 / 34.5, of 4096 110 / 76, of 8192 185 /
// 176, 256 of 1024 26.6 / 16.0, of 8192 103 / 91, 2048 lists of 512 tokens 70 / 59; 128 units of 2048 tokens 23.3 / 19.6, of 4096
// 35.1 / 38.8, 128 lists of 2622 28.2 / 25.2; 8 units of 256 tokens 11.0 / 8.7, of 1024 11.5 / 11.9, of 2048 11.6 / 17.8, 32 lists of
// 524 tokens 14.4 / 9.9, of 1049 15.9 / 13.2, of 2622 18.7 / 23.0.  The line is the capacity's: a long sequence among short ones
// is one workgroup's, at about 75 GB/s (8192 tokens: 28 us).
static bool attn8_per_unit(const Dims& dm, bool dense, int cus) {
  const long long tokens = (long long)(dense ? dm.Mmax : dm.cap) * dm.P, units = attn8_units(dm, dense);
  return tokens <= (units >= cus ? 8192 : units >= cus / 2 ? 2560 : 1024);
}

template <typename T, int G, bool DENSE, bool STREAM, int NW>
static void launch_attn8_NW(const Dims& dm, const Attn8Args& a, int W, size_t lds, hipStream_t st) {
  if (dm.P % 8 == 0) hipLaunchKernelGGL((attn8_kernel<T, G, DENSE, true, STREAM, NW>), dim3(W), dim3(64 * NW), lds, st, a);
  else hipLaunchKernelGGL((attn8_kernel<T, G, DENSE, false, STREAM, NW>), dim3(W), dim3(64 * NW), lds, st, a);
}
template <typename T, int G, bool DENSE>
static void launch_attn8(const Dims& dm, Attn8Args a, hipStream_t st) {
  const int cus = device_compute_units();
  // Loads through the caches or past them, by the capacity.  Whole calls, us, kept / past, K and V of every page: 34 MB 17.9 / 18.0, 67 MB 23.9 /
  // 23.8 (launched one by one 22.1 / 22.9), 134 MB 36.7 / 34.4, in pages of 12 37.4 / 35.0, 268 MB 59.9 / 55.3, 2 GB 335 / 298; lists of heads
  // without a group 43 MB 22.0 / 21.7 (19.9 / 20.9), 67 MB 18.8 / 18.6 (16.8 / 17.7), 134 MB 38.4 / 35.8, 268 MB 56.5 / 51.7 and 61.6 / 56.7.
  // Lists per head of a group meet in the caches: 16 x 16K tokens, lists of 40 %, 107 / 129 (4 x 128K, 4 %, which hardly overlap, 44.0 / 41.8).
  const bool stream = (DENSE || dm.G == 1) && (long long)a.s.U * (DENSE ? dm.Mmax : dm.cap) * dm.P * kD >= kStream8Bytes;
  if (attn8_per_unit(dm, DENSE, cus)) {
    a.per_unit = 1;
    if (a.s.U < cus) launch_attn8_NW<T, G, DENSE, false, 2 * kAttnWaves>(dm, a, a.s.U, 0, st);
    else if (stream) launch_attn8_NW<T, G, DENSE, true, kAttnWaves>(dm, a, a.s.U, 0, st);
    else launch_attn8_NW<T, G, DENSE, false, kAttnWaves>(dm, a, a.s.U, 0, st);
    return;
  }
  const int W = attn8_grid(dm, DENSE, 2 * cus < kMostWgs ? 2 * cus : kMostWgs);
  if (a.s.U > kUnitsLdsMax) {
    hipLaunchKernelGGL(attn8_prefix_kernel<DENSE>, dim3(1), dim3(1024), 0, st, a);
    a.s.pre_g = a.pre;
  }
  const size_t lds = a.s.pre_g != nullptr ? 0 : (size_t)(a.s.U + 1) * sizeof(int);
  if (stream) launch_attn8_NW<T, G, DENSE, true, kAttnWaves>(dm, a, W, lds, st);
  else launch_attn8_NW<T, G, DENSE, false, kAttnWaves>(dm, a, W, lds, st);
  if (a.s.U * G <= cus) hipLaunchKernelGGL(attn8_join_kernel<8>, dim3(a.s.U * G), dim3(8 * kD), 0, st, a, G, W);
  else hipLaunchKernelGGL(attn8_join_kernel<2>, dim3(a.s.U * G), dim3(2 * kD), 0, st, a, G, W);
}
template <typename T>
static void launch_attn8_T(const Dims& dm, bool dense, const Attn8Args& a, hipStream_t st) {
  if (!dense) launch_attn8<T, 1, false>(dm, a, st);
  else if (dm.G == 1) launch_attn8<T, 1, true>(dm, a, st);
  else if (dm.G == 2) launch_attn8<T, 2, true>(dm, a, st);
  else if (dm.G == 4) launch_attn8<T, 4, true>(dm, a, st);
  else launch_attn8<T, 8, true>(dm, a, st);
}

void launch_decode8_softmax(const Dims& dm, bool dense, const void* q, const ekv_cache8_view& c, const int32_t* page_idx,
                            const int32_t* n_sel, float* out, float* lse, void* ws, hipStream_t st) {
  Attn8Args a{};
  a.s = ScoreArgs{q, c.k_pool, c.block_table, c.seq_lens, page_idx, n_sel, nullptr, nullptr, dm.Hq, dm.Hkv, dm.P, dm.Mmax, dm.cap,
                  0, c.n_phys_pages, 0, dm.scale * kLog2e, dm.HkvPool, (int)attn8_units(dm, dense), nullptr, 1};
  a.k_scale = c.k_scale; a.v_scale = c.v_scale; a.v_pool = (const e4m3_t*)c.v_pool;
  a.out = out; a.lse = lse;
  a.pre = (int32_t*)ws;
  a.part = (float*)((char*)ws + attn8_pre_bytes(dm, dense));
  a.page_div = make_page_div(dm.P);
  if (dm.dtype == EKV_F32) launch_attn8_T<float>(dm, dense, a, st);
  else launch_attn8_T<bf16_t>(dm, dense, a, st);
}

}  // namespace ekv
