// Softmax attention of drafted rows over the cache and over the drafted keys that their masks name (ekv_tree.h has the layout).
//
// One pass over K and V with the running maximum and sum of every row.  The work of all lists is one sequence of steps (tiles of
// keys; the drafted keys are a list's last), of which every workgroup takes an even, contiguous share; a list that several
// workgroups share leaves partial results, two at most to a workgroup, which a second launch joins.
// bf16 products take float32 weights as three terms that sum to them exactly (8 + 8 + 8 bits), so sums are float32 sums of exact
// products, as in the single-token call.  The maximum only has to keep exp in range: it moves when a score passes it by 2^kSlack.
// What a mask hides counts for nothing, infinities and NaN in its value among them: such drafted values are taken out of the
// product (0 * NaN) and added by themselves to the rows that see them.
// An infinite value of the cache, which no mask hides, stays in the product: its channel is infinite, or NaN where one of the weight's terms is
// zero (looking for one in every tile would cost every call).
// Bound by the bytes with few rows (lists of 4 x 5243 tokens, 32 rows, 347 MB: 77 us, 4.5 TB/s) and by the products with many: 256 rows, 8 x
// 32K tokens, 0.37 TFLOP with the three terms in 395 us (the call's 412 without the join), 0.94 PFLOP/s, matrix units 53 % busy (a library product of 8192^2 bf16 matrices: 1.37).
#include "ekv_tree.h"

namespace ekv {

constexpr int kRec = kD + 2;
constexpr float kSlack = 8.f;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

// floats of a partial result: rows of outputs, then (maximum, sum) of every row
__host__ __device__ constexpr size_t tree_rec(int rows) { return (size_t)rows * kRec; }

__device__ __forceinline__ uint32_t top_halves(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
__device__ __forceinline__ float below(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

template <typename TQ, int NQ, int TILES> struct TreeSoftmax {
  f32x4_t o[NQ][8];                              // lane (c, j): channels 16 i + 4 j + 0..3 of row c
  float m[NQ], l[NQ];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      m[t] = -INFINITY; l[t] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[t][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
  }
  struct Weights { f32x4_t p[TILES][NQ]; };                // of a tile: lane (c, j) has keys 16 i + 4 j + 0..3 of row c
  // From an LDS tile of keys of the cache (bit i of valid: key i counts) or drafted ones (bit i of seen[t]: for the lane's row of tile t) to
  // weights; maxima and sums go on.  bad: drafted keys whose values are added here, by themselves, from v_bad.
  template <bool DRAFTED>
  __device__ __forceinline__ void weigh(const char* k, const TreeQuery<TQ, NQ>& q, float zscale, uint64_t valid, const uint64_t (&seen)[NQ],
                                        uint64_t bad, const TQ* v_bad, int64_t v_stride, Weights& out) {
    const int lane = threadIdx.x & 63, c = lane & 15, j = lane >> 4;
    constexpr uint64_t full = TILES == 4 ? ~0ull : (1ull << (16 * TILES & 63)) - 1;
    f32x4_t (&p)[TILES][NQ] = out.p;
    tree_scores_all<TQ, NQ, TILES>(k, q, p);
    if (DRAFTED || (valid & full) != full) {
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
          const uint32_t bits = (uint32_t)((DRAFTED ? seen[t] : valid) >> (16 * i + 4 * j));
#pragma unroll
          for (int e = 0; e < 4; ++e) p[i][t][e] = bits >> e & 1 ? p[i][t][e] : -INFINITY;
        }
      }
    }
    float top[NQ];
    bool higher = false;
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      top[t] = -INFINITY;
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) top[t] = fmaxf(top[t], p[i][t][e]);
      }
      top[t] *= zscale;
      higher |= top[t] > m[t] + kSlack;
    }
    if (__any(higher)) {
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        const float now = fmaxf(m[t], column_max(top[t])), f = now > -INFINITY ? __builtin_amdgcn_exp2f(m[t] - now) : 1.f;
        m[t] = now;
        l[t] *= f;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[t][i] *= f;
      }
    }
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      const float base = m[t] > -INFINITY ? -m[t] : 0.f;
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[i][t][e] = __builtin_amdgcn_exp2f(fmaf(p[i][t][e], zscale, base));
          l[t] += p[i][t][e];
        }
      }
    }
    if (DRAFTED && bad != 0) {
      for (uint64_t left = bad; left != 0; left &= left - 1) {
        const int key = __builtin_ctzll(left);
        const TQ* row = v_bad + (int64_t)key * v_stride + 4 * j;
        float w[NQ];
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
          w[t] = 0.f;
#pragma unroll
          for (int i = 0; i < TILES; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if ((key >> 4) == i && (key & 3) == e) {
                w[t] = __shfl(p[i][t][e], (((key >> 2) & 3) << 4) + c);
                p[i][t][e] = j == ((key >> 2) & 3) ? 0.f : p[i][t][e];
              }
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float x[4];
          if constexpr (sizeof(TQ) == 2) {
            const uint2 u = *reinterpret_cast<const uint2*>(row + 16 * i);
            x[0] = __uint_as_float(u.x << 16); x[1] = __uint_as_float(u.x & 0xffff0000u);
            x[2] = __uint_as_float(u.y << 16); x[3] = __uint_as_float(u.y & 0xffff0000u);
          } else {
            const float4 u = *reinterpret_cast<const float4*>(row + 16 * i);
            x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
          }
#pragma unroll
          for (int t = 0; t < NQ; ++t) {
            if (seen[t] >> key & 1) {
#pragma unroll
              for (int e = 0; e < 4; ++e) o[t][i][e] = fmaf(w[t], x[e], o[t][i][e]);
            }
          }
        }
      }
    }
  }
  // The weighted values of the tile.
  __device__ __forceinline__ void multiply(const char* v, const Weights& x) {
    const int lane = threadIdx.x & 63, c = lane & 15, j = lane >> 4;
    if constexpr (sizeof(TQ) == 2) {
#pragma unroll
      for (int i = 0; i < TILES; i += 2) {
        // 32 keys at a time, lane group j has keys 4j..4j+3 of either tile of sixteen: three terms of their weights
        bf16x8_t w[3][NQ];
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) { y[e] = x.p[i][t][e]; y[4 + e] = x.p[i + 1][t][e]; }
#pragma unroll
          for (int term = 0; term < 3; ++term) {
            u32x4_t r;
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = top_halves(y[2 * e], y[2 * e + 1]);
            w[term][t] = __builtin_bit_cast(bf16x8_t, r);
            if (term < 2) {
#pragma unroll
              for (int e = 0; e < 8; ++e) y[e] = below(y[e]);
            }
          }
        }
        // a sum's terms are apart from each other: 2 (4) channels' by the rows' tiles between them
        constexpr int CH = NQ == 1 ? 4 : 2;
#pragma unroll
        for (int ch = 0; ch < 8; ch += CH) {
          bf16x8_t a[CH];
#pragma unroll
          for (int h = 0; h < CH; ++h) {
            const int row = 16 * i + 4 * j + (c >> 2), piece = 2 * (ch + h) + ((c & 3) >> 1), half = (c & 1) * 8;
            const s16x4_t a0 = read_transposed(v + tree_piece<TQ>(row, piece) + half), a1 = read_transposed(v + tree_piece<TQ>(row + 16, piece) + half);
            a[h] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
          }
#pragma unroll
          for (int term = 2; term >= 0; --term) {                          // the smallest terms first
#pragma unroll
            for (int h = 0; h < CH; ++h) {
#pragma unroll
              for (int t = 0; t < NQ; ++t)
                o[t][ch + h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[h], w[term][t], o[t][ch + h], 0, 0, 0);
            }
          }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
#pragma unroll
        for (int ch = 0; ch < 8; ++ch) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float a = *reinterpret_cast<const float*>(v + tree_piece<TQ>(16 * i + 4 * j + e, 4 * ch + (c >> 2)) + 4 * (c & 3));
#pragma unroll
            for (int t = 0; t < NQ; ++t) o[t][ch] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, x.p[i][t][e], o[t][ch], 0, 0, 0);
          }
        }
      }
    }
  }
  __device__ __forceinline__ void add(const char* k, const char* v, const TreeQuery<TQ, NQ>& q, float zscale, uint64_t valid) {
    const uint64_t none[NQ] = {};
    Weights x;
    weigh<false>(k, q, zscale, valid, none, 0, nullptr, 0, x);
    multiply(v, x);
  }
};

template <typename TQ> __device__ __forceinline__ bool has_no_number(const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  bool no = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    no |= (w[i] & 0x7f800000u) == 0x7f800000u;
    if constexpr (sizeof(TQ) == 2) no |= (w[i] & 0x7f80u) == 0x7f80u;
  }
  return no;
}

template <typename TQ, typename TC, int NQ, int WQ, bool LISTS>
__global__ __launch_bounds__(64 * (WQ == 1 ? 4 : WQ)) __attribute__((amdgpu_waves_per_eu(2)))
void tree_softmax_kernel(const TreeArgs A) {
  using S = TreeShape<TQ, TC, NQ, WQ, 2>;
  extern __shared__ int pre_lds[];
  __shared__ __attribute__((aligned(16))) char s_tile[S::kLds];
  __shared__ uint32_t s_bad[S::kGroups][2];
  __shared__ int wsum[S::kWaves];
  constexpr int RS = kD + 4;                     // floats between rows of partial outputs in LDS
  static_assert(WQ > 1 || NQ * 16 * RS * 4 * 2 <= S::kLds, "two wavefronts' partial outputs take the tiles' place");
  __shared__ float s_m[S::kWaves][16 * NQ], s_l[S::kWaves][16 * NQ];
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6), c = lane & 15, j = lane >> 4;
  const int grp = WQ == 1 ? w : 0, tid = WQ == 1 ? lane : threadIdx.x;
  char* tile = s_tile + grp * S::kTileBytes;
  tree_work<S::kWork, S::kRows, S::kKeys>(A, pre_lds, wsum, [&](int wg, int unit, const TreeList& list, int blk, int st0, int st1, int steps, bool first) {
    const TreeRows R = list.R;
    const int list_head = list.head, hkv = list.hkv;
    const int tiles0 = min(st0, steps - 1), tiles1 = min(st1, steps - 1);          // the steps' tiles of the cache
    const bool drafted = st1 == steps;
    const int r0 = blk * S::kRows + (WQ > 1 ? w * 16 * NQ : 0);         // the wavefront's first row
    TreeQuery<TQ, NQ> q;
    TreeSoftmax<TQ, NQ, S::kTiles> acc;
    acc.clear();
    // a group's share of the tiles
    const int n_t = tiles1 - tiles0, t0 = tiles0 + n_t * grp / S::kGroups, t1 = tiles0 + n_t * (grp + 1) / S::kGroups;
    const TreeLook<LISTS> look(A, unit, list);
    const int row = lane % S::kKeys;
    auto pos_of = [&](int t) { return min(t, t1 - 1) * S::kKeys + row; };
    TreeStage<TQ, TC, NQ, WQ, 2> stage;
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
    auto ahead = [&](int t) {                              // tile t's data under way, the lookups of the two behind it
      const int ph2 = look.phys(lp2), lp3 = look.page(pos_of(t + 2));
      fetch(t, lp1, ph1);
      lp1 = lp2; ph1 = ph2; lp2 = lp3;
    };
    if constexpr (WQ == 1) {
      for (int t = t0; t < t1; ++t) {
        const uint64_t valid = valid_next;
        wave_order();                                      // the tile before is read
        stage.commit(tile, tid, valid);
        ahead(t + 1);
        wave_order();
        acc.add(tile, tile + S::kSideBytes, q, A.zscale, valid);
      }
    } else if (t0 < t1) {
      // tile t + 1 goes to the half of LDS that nobody reads while tile t is worked on: one meeting a tile
      __syncthreads();                                     // the last list's tiles are read
      uint64_t valid = valid_next;
      stage.commit(tile, tid, valid);
      ahead(t0 + 1);
      for (int t = t0; t < t1; ++t) {
        char* now = tile + ((t - t0) & 1) * S::kTileBytes;
        __syncthreads();
        const uint64_t after = valid_next;
        if (t + 1 < t1) stage.commit(tile + ((t + 1 - t0) & 1) * S::kTileBytes, tid, after);
        ahead(t + 2);
        acc.add(now, now + S::kSideBytes, q, A.zscale, valid);
        valid = after;
      }
    }
    // the drafted keys, whose tiles the groups take in turn
    if (drafted) {
#pragma unroll 1
      for (int d0 = WQ == 1 ? grp * S::kKeys : 0; d0 < R.count; d0 += S::kGroups * S::kKeys) {
        if constexpr (WQ > 1) __syncthreads(); else wave_order();
        if (tid < 2) s_bad[grp][tid] = 0;
        if constexpr (WQ > 1) __syncthreads(); else wave_order();
        stage_drafted<TQ, S, 2>(A, tile, tid, R, hkv, d0, [&](int key_row, uint4& v) {
          if (has_no_number<TQ>(v)) {
            atomicOr(&s_bad[grp][key_row >> 5], 1u << (key_row & 31));
            v = make_uint4(0u, 0u, 0u, 0u);
          }
        });
        const uint64_t there = R.count - d0 >= 64 ? ~0ull : (1ull << (R.count - d0)) - 1;
        uint64_t seen[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          const int r = min(r0 + 16 * i + c, R.count * A.GL - 1);
          seen[i] = (A.visible[R.first + r / A.GL] >> d0) & there;
        }
        if constexpr (WQ > 1) __syncthreads(); else wave_order();
        const uint64_t bad = (uint64_t)(uint32_t)uniform((int)s_bad[grp][0]) | (uint64_t)(uint32_t)uniform((int)s_bad[grp][1]) << 32;
        typename TreeSoftmax<TQ, NQ, S::kTiles>::Weights x;
        acc.template weigh<true>(tile, q, A.zscale, 0, seen, bad, (const TQ*)A.v_new + (int64_t)(R.first + d0) * A.vs + hkv * kD, A.vs, x);
        acc.multiply(tile + S::kSideBytes, x);
      }
    }
    // the rows' sums
#pragma unroll
    for (int t = 0; t < NQ; ++t) acc.l[t] = column_sum(acc.l[t]);
    const bool whole = st0 == 0 && st1 == steps;
    float* rec = A.part + tree_rec(S::kRows) * (2 * (size_t)wg + (first ? 0 : 1));
    auto put = [&](int r, int ch, float4 o, float m, float l) {            // four channels of row r of the block
      const int row = blk * S::kRows + r;
      if (row >= R.count * A.GL) return;
      if (whole) {
        const int tok = row / A.GL;
        const size_t to = (size_t)(R.first + tok) * A.Hq + list_head + (row - tok * A.GL);
        const float f = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);          // no key at all: a zero output; NaN stays
        *reinterpret_cast<float4*>(A.out + to * kD + ch) = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
        if (ch == 0) A.norm[to] = l == 0.f ? -INFINITY : m * kLn2 + __logf(l);
      } else {
        *reinterpret_cast<float4*>(rec + (size_t)r * kD + ch) = o;
        if (ch == 0) *reinterpret_cast<float2*>(rec + (size_t)S::kRows * kD + 2 * r) = make_float2(m, l);
      }
    };
    if constexpr (WQ > 1) {
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          put(w * 16 * NQ + 16 * t + c, 16 * i + 4 * j, make_float4(acc.o[t][i][0], acc.o[t][i][1], acc.o[t][i][2], acc.o[t][i][3]), acc.m[t], acc.l[t]);
      }
    } else {
      // two wavefronts hand theirs to the other two, and one of these to the first; then the first's go out
      float* so = reinterpret_cast<float*>(s_tile);
      if (j == 0) {
#pragma unroll
        for (int t = 0; t < NQ; ++t) { s_m[w][16 * t + c] = acc.m[t]; s_l[w][16 * t + c] = acc.l[t]; }
      }
      float f[NQ], M[NQ], Ls[NQ];
      __syncthreads();                                                     // the tiles are read
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        M[t] = fmaxf(fmaxf(s_m[0][16 * t + c], s_m[1][16 * t + c]), fmaxf(s_m[2][16 * t + c], s_m[3][16 * t + c]));
        f[t] = acc.m[t] > -INFINITY ? __builtin_amdgcn_exp2f(acc.m[t] - M[t]) : 0.f;
        Ls[t] = 0.f;
#pragma unroll
        for (int i = 0; i < S::kWaves; ++i) {
          const float mi = s_m[i][16 * t + c];
          Ls[t] = fmaf(s_l[i][16 * t + c], mi > -INFINITY ? __builtin_amdgcn_exp2f(mi - M[t]) : 0.f, Ls[t]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) acc.o[t][i] *= f[t];
      }
#pragma unroll
      for (int hand = 2; hand >= 1; hand >>= 1) {                          // wavefronts hand..2 hand-1 to 0..hand-1
        if (w >= hand && w < 2 * hand) {
#pragma unroll
          for (int t = 0; t < NQ; ++t) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              *reinterpret_cast<f32x4_t*>(so + ((size_t)(w - hand) * 16 * NQ + 16 * t + c) * RS + 16 * i + 4 * j) = acc.o[t][i];
          }
        }
        __syncthreads();
        if (w < hand) {
#pragma unroll
          for (int t = 0; t < NQ; ++t) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              acc.o[t][i] += *reinterpret_cast<const f32x4_t*>(so + ((size_t)w * 16 * NQ + 16 * t + c) * RS + 16 * i + 4 * j);
          }
        }
        __syncthreads();
      }
      if (w == 0) {
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            put(16 * t + c, 16 * i + 4 * j, make_float4(acc.o[t][i][0], acc.o[t][i][1], acc.o[t][i][2], acc.o[t][i][3]), M[t], Ls[t]);
        }
      }
    }
  });
}

// Joins the partial results of row blocks that several workgroups worked on, in their order: a wavefront per row, two channels a lane.
__global__ __launch_bounds__(256) void tree_join_kernel(const TreeArgs A, int rows, int keys) {
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
  const int most = A.most * A.GL, per = (most + 3) / 4;
  const int unit = (int)(blockIdx.x / (unsigned)per), r = (int)(blockIdx.x % (unsigned)per) * 4 + w;
  const TreeList l = tree_list(A, unit);
  const TreeRows R = l.R;
  if (r >= R.count * A.GL) return;
  const int blk = r / rows, steps = (l.n_pos + keys - 1) / keys + 1;
  const int total = A.pre[A.U], share = total / A.W, rem = total - share * A.W;
  const int begin = A.pre[unit] + blk * steps, end = begin + steps;
  auto wg_of = [&](int s) { return s < rem * (share + 1) ? s / (share + 1) : rem + (s - rem * (share + 1)) / share; };
  auto first_of = [&](int i) { return i * share + min(i, rem); };
  const int w0 = wg_of(begin), w1 = wg_of(end - 1);
  if (w0 == w1) return;                                                    // written by that workgroup
  const int in_blk = r - blk * rows;
  // the block is the second that workgroup w0 left if it began before the block did
  auto rec_of = [&](int i) { return A.part + tree_rec(rows) * (2 * (size_t)i + (i == w0 && first_of(i) < begin ? 1 : 0)); };
  float M = -INFINITY;
  for (int i = w0 + lane; i <= w1; i += 64) M = fmaxf(M, rec_of(i)[(size_t)rows * kD + 2 * in_blk]);
  M = wave_max(M);
  float L = 0.f;
  float2 o = make_float2(0.f, 0.f);
  for (int i0 = w0; i0 <= w1; i0 += 8) {                                   // eight records in flight
    float2 ml[8], x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float* rec = rec_of(min(i0 + k, w1));
      ml[k] = *reinterpret_cast<const float2*>(rec + (size_t)rows * kD + 2 * in_blk);
      x[k] = *reinterpret_cast<const float2*>(rec + (size_t)in_blk * kD + 2 * lane);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const bool in = i0 + k <= w1;                                        // else the last record over again, infinities and all
      const float f = in && ml[k].x > -INFINITY ? __builtin_amdgcn_exp2f(ml[k].x - M) : 0.f;
      x[k] = in ? x[k] : make_float2(0.f, 0.f);
      L = fmaf(in ? ml[k].y : 0.f, f, L);
      o.x = fmaf(x[k].x, f, o.x);
      o.y = fmaf(x[k].y, f, o.y);
    }
  }
  const int tok = r / A.GL;
  const size_t to = (size_t)(R.first + tok) * A.Hq + l.head + (r - tok * A.GL);
  const float f = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
  *reinterpret_cast<float2*>(A.out + to * kD + 2 * lane) = make_float2(o.x * f, o.y * f);
  if (lane == 0) A.norm[to] = L == 0.f ? -INFINITY : M * kLn2 + __logf(L);
}

__global__ __launch_bounds__(1024) void tree_prefix_kernel(const TreeArgs A, int keys, int rows) {
  __shared__ int wsum[16];
  block_exclusive_prefix<1024>(A.U, [&](int u) { return tree_unit_steps(A, u, keys, rows); }, A.pre, wsum);
}
void launch_tree_prefix(const TreeArgs& a, int keys, int rows, hipStream_t st) {
  hipLaunchKernelGGL(tree_prefix_kernel, dim3(1), dim3(1024), 0, st, a, keys, rows);
}

// ------------------------------------------------------------------------------------------
// workgroups of a launch at most; workspaces are sized for them
static int most_wgs(int rows) { return rows == 32 ? 1024 : 512; }

struct TreeDims { int rows, keys; };             // of a workgroup, of a tile
static long long list_tokens(const Dims& dm, bool dense) { return (long long)(dense ? dm.Mmax : dm.cap) * dm.P; }
// Blocks as large as the rows of a list, or of 64 rows where there is so little to go through that more workgroups count for more than reading
// keys once.  Calls, us, blocks of 64 / of 128 / of 256 rows: lists of 256 rows, 8 of 4000 tokens 27 / 38 / 34, 16 of 2049 8-bit 24 / 30 / 28, 64 of
// 1000 35 / 57 / 53, 32 of 4000 57 / 64 / 54, 16 of 32000 184 / 177 / 149, 64 of 16000 312 / 290 / 238; of 128 rows, 64 of 4096 57 / 71, 32 of 8000
// 65 / 73, 8 of 128000 205 / 184.  17 to 32 rows over every page: by two wavefronts, tiles of 32 keys, where there is enough.  Blocks of 64 / of 32:
// 16 caches of 2049 tokens 19.3 / 22.9, 8 of 4096 23.7 / 24.7, of 32 768 49.5 / 47.0, of 131 072 119 / 114, 32 of 8192 44.0 / 43.0, of 131 072 411 / 378,
// 64 of 4096 8-bit 36.8 / 31.6, 512 of 1024 56 / 55; page lists, 128 of 5243 84.5 / 85.5.
static TreeDims softmax_dims(const Dims& dm, bool dense, int lists, int list_rows) {
  if (dm.dtype == EKV_F32) return list_rows <= 16 ? TreeDims{16, 16} : TreeDims{64, 32};
  if (list_rows <= 16) return {16, 32};
  const long long all = list_tokens(dm, dense) * dm.B * lists;
  if (list_rows <= 32 && dense && all > 1ll << 17) return {32, 32};
  if (list_rows <= 64 || all <= (list_rows <= 128 ? 1ll << 19 : 3ll << 15)) return {64, 64};
  return {list_rows <= 128 ? 128 : 256, 64};
}
static long long softmax_steps(const Dims& dm, bool dense, int lists, int list_rows) {
  const TreeDims td = softmax_dims(dm, dense, lists, list_rows);
  return (long long)dm.B * lists * ((list_rows + td.rows - 1) / td.rows) * ((list_tokens(dm, dense) + td.keys - 1) / td.keys + 1);
}
bool tree_softmax_supported(const Dims& dm, bool dense, int lists, int most) {
  return softmax_steps(dm, dense, lists, most * (dm.Hq / lists)) <= 0x7fffffff;
}
size_t tree_softmax_ws_bytes(const Dims& dm, bool dense, int lists, int most) {
  const TreeDims td = softmax_dims(dm, dense, lists, most * (dm.Hq / lists));
  return tree_pre_bytes((size_t)dm.B * lists) + 2 * most_wgs(td.rows) * tree_rec(td.rows) * sizeof(float);
}

template <typename TQ, typename TC, int NQ, int WQ>
static void launch_softmax_shape(const TreeArgs& a, int grid, size_t lds, hipStream_t st) {
  if (a.page_idx != nullptr) hipLaunchKernelGGL((tree_softmax_kernel<TQ, TC, NQ, WQ, true>), dim3(grid), dim3(64 * (WQ == 1 ? 4 : WQ)), lds, st, a);
  else hipLaunchKernelGGL((tree_softmax_kernel<TQ, TC, NQ, WQ, false>), dim3(grid), dim3(64 * (WQ == 1 ? 4 : WQ)), lds, st, a);
}
template <typename TQ, typename TC>
static void launch_softmax_T(const Dims& dm, TreeArgs a, hipStream_t st) {
  const int list_rows = a.most * a.GL;
  const bool dense = a.page_idx == nullptr;
  const TreeDims td = softmax_dims(dm, dense, a.L, list_rows);
  const int cus = device_compute_units();
  a.blocks = (list_rows + td.rows - 1) / td.rows;
  const long long units = (long long)a.U * a.blocks, tokens = list_tokens(dm, dense);
  // A block of rows whole by one workgroup, without prefix sums, records and join, where blocks are many and no list can be long.  Calls, us,
  // split / whole, a sequence's KV heads one unit: of 16 rows, 8 units of 200 tokens 12.4 / 13.0, of 2000 14.9 / 29.4, 128 of 1000 26.4 / 20.9, of
  // 2000 36.3 / 34.9, 256 of 1000 38.4 / 28.9, of 2000 56.9 / 47.4, 512 of 4000 175 / 161, of 8000 328 / 309; of 64 rows, 32 of 1000 24.3 / 32.0, 128
  // of 2000 46.1 / 57.1, 256 of 1000 52.6 / 39.7, of 4000 108.9 / 113.5, 512 of 1000 85.9 / 60.7, of 4000 212 / 190; of 256 rows, 64 of 1000 55.3 /
  // 66.9, 128 of 3000 128 / 164, 512 of 1000 192 / 143.  The line is the capacity's: a long sequence among short ones is one workgroup's.
  const long long whole = units >= 2 * cus ? 8192 : units >= cus ? (td.rows == 16 ? 8192 : 2048) : units >= cus / 2 && td.rows == 16 ? 2048 : 0;
  a.per_unit = tokens <= whole;
  const long long steps = softmax_steps(dm, dense, a.L, list_rows);
  // 32 rows: four workgroups a compute unit where a block of rows is not in so many pieces that the join takes longer.  Calls, us, two / four, by
  // blocks of rows: 8 of 131 072 tokens 113 / 125, 16 of 32 768 66.6 / 73.7, 32 109 / 113, 48 132 / 136; 64 of 8192 60.0 / 61.4, of 32 768 177 / 181, of
  // 131 072 647 / 638, 128 of 8192 101 / 102, of 32 768 336 / 337, 256 of 4096 108 / 106, 512 of 16 384 660 / 653: from the line on within 3 % either way.
  const bool four = td.rows == 32 && units >= 64;
  const int per_cu = td.rows == 256 ? 1 : four ? 4 : 2, most = per_cu * cus < most_wgs(td.rows) ? per_cu * cus : most_wgs(td.rows), share = td.rows == 16 ? 4 : 1;
  const long long wgs = (steps + share - 1) / share;
  a.W = (int)(wgs < most ? wgs : most);
  size_t lds = 0;
  if (!a.per_unit) {
    if (a.U > kUnitsLdsMax) {
      launch_tree_prefix(a, td.keys, td.rows, st);
      a.pre_g = a.pre;
    } else {
      lds = (size_t)(a.U + 1) * sizeof(int);
    }
  }
  const int grid = a.per_unit ? (int)units : a.W;
  if (td.rows == 16) launch_softmax_shape<TQ, TC, 1, 1>(a, grid, lds, st);
  else if (td.rows == 64) launch_softmax_shape<TQ, TC, 1, 4>(a, grid, lds, st);
  if constexpr (sizeof(TQ) == 2) {
    if (td.rows == 32) launch_softmax_shape<TQ, TC, 1, 2>(a, grid, lds, st);
    if (td.rows == 128) launch_softmax_shape<TQ, TC, 1, 8>(a, grid, lds, st);
    else if (td.rows == 256) launch_softmax_shape<TQ, TC, 2, 8>(a, grid, lds, st);
  }
  if (!a.per_unit)
    hipLaunchKernelGGL(tree_join_kernel, dim3((unsigned)a.U * ((list_rows + 3) / 4)), dim3(256), 0, st, a, td.rows, td.keys);
}

void launch_tree_softmax(const Dims& dm, TreeArgs a, bool codes, void* ws, hipStream_t st) {
  a.pre = (int32_t*)ws;
  a.part = (float*)((char*)ws + tree_pre_bytes(a.U));
  a.zscale = dm.scale * kLog2e;
  if (dm.dtype == EKV_F32) {
    if (codes) launch_softmax_T<float, e4m3_t>(dm, a, st);
    else launch_softmax_T<float, float>(dm, a, st);
  } else {
    if (codes) launch_softmax_T<bf16_t, e4m3_t>(dm, a, st);
    else launch_softmax_T<bf16_t, bf16_t>(dm, a, st);
  }
}

}  // namespace ekv
