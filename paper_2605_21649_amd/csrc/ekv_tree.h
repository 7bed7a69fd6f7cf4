// Attention of drafted rows (a tree of up to 64 new tokens per sequence) over the cache: what its kernels share.
//
// A list's rows (the tree's tokens times the query heads that read the list) are columns of matrix products whose rows are the
// list's keys: S^T[key][row] = K Q^T.  A 16x16x32 bf16 product leaves rows 4j..4j+3 of column c in lane (c, j) = (lane % 16, lane / 16),
// and takes eight numbers of column c along the contraction from it: with the contraction's order chosen so that lane group j
// has keys 4j..4j+3 of two tiles of sixteen, weights go from one product to the next (O^T = V^T P^T) without leaving the lane.
// float32 caches and queries use the 16x16x4 float32 product in the same way, a key of the four after the other.
//
// Keys and values pass through LDS once for all rows of a workgroup: rows of a tile lie at their length, their 16-byte pieces in an
// order that their number turns (piece ^ row % 16), so that neither sixteen rows' same piece nor the transposing reads of V
// meet in a bank.  An 8-bit cache's codes become bf16 or float32 with their page's scale (exact) on the way into LDS.
// Two kinds of shape: up to 16 rows: every wavefront has all of them and keys of its own, nothing is waited for together; more: two, four
// or eight wavefronts share the keys, twice a tile's in LDS so that they meet once a tile, and have 16 or 32 rows each.  (17 to 32
// rows, two tiles of them in every wavefront with keys of its own: registers spill, and a spilled one read back waits for all loads
// under way; lists of 4 x 128K tokens, 32 rows, softmax 97 us, by four wavefronts that share, half of them idle, 83.)
#pragma once
#include "ekv_attn8.h"

namespace ekv {

constexpr int kTreeMost = 64;                    // drafted rows of a sequence: bits of a mask

struct TreeArgs {
  const void* q; const void* k_pool; const void* v_pool; const float* k_scale; const float* v_scale;
  const int32_t* block_table; const int32_t* seq_lens; const int32_t* page_idx; const int32_t* n_sel;      // every page: page_idx null, n_sel seq_lens
  const void* k_new; const void* v_new; int64_t ks, vs;
  const int32_t* start; const uint64_t* visible;
  int B, Hq, Hkv, HkvPool, P, Mmax, cap, n_phys, N, most;
  int L, GL;                                     // lists per sequence, query heads per list
  PageDiv page_div;
  float zscale;
  int U;                                         // B * L
  int W, per_unit;                               // workgroups; 1: workgroup i has block of rows i, whole
  int blocks;                                    // blocks of rows of the largest tree
  int32_t* pre; const int32_t* pre_g;            // steps before a list (all row blocks), [U + 1]; pre_g: where U is too large for LDS
  float* part;                                   // softmax: two partial results a workgroup
  float* out; float* norm;
  float* z; float* zmax; size_t zstride; int n_groups;      // entmax: scores and group maxima
  float beta; int ibeta;
};

// Drafted rows of a sequence: [first, first + count).
struct TreeRows { int first, count; };
__device__ __forceinline__ TreeRows tree_rows(const TreeArgs& A, int from, int to) {
  const int s0 = clampi(from, 0, A.N), s1 = clampi(to, s0, A.N);
  return {s0, min(s1 - s0, A.most)};
}
__device__ __forceinline__ TreeRows tree_rows(const TreeArgs& A, int b) { return tree_rows(A, uniform_load(A.start + b), uniform_load(A.start + b + 1)); }
// Positions of a list that may hold keys: all of the sequence's tokens, or the tokens of the selected pages.  n_sel[list_entry] says how many.
__device__ __forceinline__ int list_entry(const TreeArgs& A, int u) { return A.page_idx == nullptr ? u / A.L : u; }
__device__ __forceinline__ int list_positions(const TreeArgs& A, int entry) {
  if (A.page_idx == nullptr) return (int)min((int64_t)max(entry, 0), (int64_t)A.Mmax * A.P);
  return clampi(entry, 0, A.cap) * A.P;
}
// Steps of a list: tiles of `keys` positions and one for the drafted keys, for every block of `rows` rows; none without rows.
__device__ __forceinline__ int tree_blocks(const TreeArgs& A, int count, int rows) { return (count * A.GL + rows - 1) / rows; }
__device__ __forceinline__ int tree_unit_steps(const TreeArgs& A, int u, int keys, int rows) {
  const int b = u / A.L, s0 = A.start[b], s1 = A.start[b + 1], entry = A.n_sel[list_entry(A, u)];      // one wait for all
  const int count = tree_rows(A, s0, s1).count;
  return count > 0 ? tree_blocks(A, count, rows) * ((list_positions(A, entry) + keys - 1) / keys + 1) : 0;
}
// A list: its sequence, its first query head, its KV head, rows, the sequence's tokens and the list's positions.  Scalar loads, waited for once.
struct TreeList { int b, head, hkv, n, n_pos; TreeRows R; };
__device__ __forceinline__ TreeList tree_list(const TreeArgs& A, int u) {
  TreeList l;
  l.b = u / A.L;
  const int s0 = uniform_load(A.start + l.b), s1 = uniform_load(A.start + l.b + 1), n = uniform_load(A.seq_lens + l.b);
  const int entry = uniform_load(A.n_sel + list_entry(A, u));
  l.head = (u - l.b * A.L) * A.GL;
  l.hkv = l.head / (A.Hq / A.Hkv);
  l.R = tree_rows(A, s0, s1);
  l.n = (int)min((int64_t)max(n, 0), (int64_t)A.Mmax * A.P);
  l.n_pos = list_positions(A, entry);
  return l;
}

// Entmax scores of a list, [group of 64 keys][row][key]: what a workgroup stores of a group is in one piece.  (Rows one after the other, us
// before / now: 64 rows a KV head, 128K tokens 144 / 125, 2 of 128K 233 / 213, 8 of 32K 186 / 185, 4 of 128K 326 / 330; 256 rows, 128K
// 314 / 273.)  The lists of a sequence lie in the place of its rows.
constexpr int kGroup = 64;
struct TreeScores { float* z; size_t group; };           // floats from a group to the next
__device__ __forceinline__ TreeScores tree_z(const TreeArgs& A, const TreeList& l, int u) {
  const size_t rows = (size_t)l.R.count * A.GL;
  return {A.z + (l.R.first * (size_t)A.Hq + (u - l.b * A.L) * rows) * A.zstride, rows * kGroup};
}

// Largest value and sum of the four lanes (c, 0..3) of a column, in all four: two exchanges between registers, where __shfl_xor goes by LDS.
template <typename F> __device__ __forceinline__ float over_column(float x, F&& f) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float column_max(float x) { return over_column(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float column_sum(float x) { return over_column(x, [](float a, float b) { return a + b; }); }

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
__device__ __forceinline__ s16x4_t read_transposed(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4_t __attribute__((address_space(3)))*)(lds_char*)p);
}

// How a workgroup divides rows and keys.  TQ: type of queries and drafted rows, which the products have; TC: of the cache.  NQ: tiles of 16
// rows a wavefront, WQ: wavefronts that share the keys (1: none of four; 2, 4 or 8: all).  SIDES: K alone or K and V.
template <typename TQ, typename TC, int NQ, int WQ, int SIDES> struct TreeShape {
  static constexpr int kWaves = WQ == 1 ? 4 : WQ, kWork = 64 * kWaves;   // of the workgroup
  static constexpr int kGroups = kWaves / WQ;                            // groups of wavefronts with keys of their own
  static constexpr int kRows = 16 * NQ * WQ;                             // rows of a workgroup
  static constexpr int kKeys = (WQ == 1 || WQ == 2 && SIDES == 2 ? 32 : 64) * 2 / (int)sizeof(TQ);       // keys of a tile
  static constexpr int kTiles = kKeys / 16;
  static constexpr int kRowBytes = kD * (int)sizeof(TQ);
  static constexpr int kSideBytes = kKeys * kRowBytes;
  static constexpr int kThreads = 64 * WQ;                               // that stage a tile
  static constexpr int kTileBytes = SIDES * kSideBytes;
  static constexpr int kLds = WQ == 1 ? kGroups * kTileBytes : 2 * kTileBytes;
};
// where 16-byte piece `piece` of row `row` lies
template <typename TQ> __device__ __forceinline__ int tree_piece(int row, int piece) { return row * kD * (int)sizeof(TQ) + ((piece ^ (row & 15)) << 4); }

// A tile on its way from the cache to LDS: every thread has kLoads pieces of 16 bytes of each side.
template <typename TQ, typename TC, int NQ, int WQ, int SIDES> struct TreeStage {
  using S = TreeShape<TQ, TC, NQ, WQ, SIDES>;
  static constexpr int kPieces = kD * (int)sizeof(TC) / 16;              // of a row as stored
  static constexpr int kLoads = S::kKeys * kPieces / S::kThreads;
  static constexpr int kRowsApart = S::kThreads / kPieces;
  static constexpr bool kCodes = sizeof(TC) == 1;
  uint4 raw[SIDES][kLoads];
  float scale[SIDES][kCodes ? kLoads : 1];
  // tid: of the threads that stage; row_of(i): the cache row (page * P + token) of the tile's row i
  template <typename F> __device__ __forceinline__ void request(const TreeArgs& A, int tid, F&& row_of) {
    const int piece = tid % kPieces;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t row = row_of(tid / kPieces + i * kRowsApart);
      const size_t at = (size_t)row * (kD * sizeof(TC)) + 16 * piece;
      raw[0][i] = load16((const char*)A.k_pool + at);
      if constexpr (SIDES == 2) raw[1][i] = load16((const char*)A.v_pool + at);
      if constexpr (kCodes) {
        const uint32_t page = page_div(row, A.page_div);
        scale[0][i] = A.k_scale[page];
        if constexpr (SIDES == 2) scale[1][i] = A.v_scale[page];
      }
    }
  }
  // valid: bit i for the tile's row i; what is not valid becomes zero
  __device__ __forceinline__ void commit(char* lds, int tid, uint64_t valid) const {
    const int piece = tid % kPieces;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = tid / kPieces + i * kRowsApart;
      const bool in = (valid >> row) & 1;
#pragma unroll
      for (int s = 0; s < SIDES; ++s) {
        char* side = lds + s * S::kSideBytes;
        const uint32_t keep = in ? ~0u : 0u;
        const uint4 v = make_uint4(raw[s][i].x & keep, raw[s][i].y & keep, raw[s][i].z & keep, raw[s][i].w & keep);
        if constexpr (!kCodes) {
          *reinterpret_cast<uint4*>(side + tree_piece<TQ>(row, piece)) = v;
        } else if constexpr (sizeof(TQ) == 2) {
          const float f = in ? scale[s][i] : 1.f;
          *reinterpret_cast<bf16x8_t*>(side + tree_piece<TQ>(row, 2 * piece)) = widen_bf16(v.x, v.y, f);
          *reinterpret_cast<bf16x8_t*>(side + tree_piece<TQ>(row, 2 * piece + 1)) = widen_bf16(v.z, v.w, f);
        } else {
          const float f = in ? scale[s][i] : 1.f;
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
            *reinterpret_cast<float4*>(side + tree_piece<TQ>(row, 4 * piece + k)) = make_float4(a[0] * f, a[1] * f, b[0] * f, b[1] * f);
          }
        }
      }
    }
  }
};

// Lookups of a list's positions, a row of the tile per lane, in steps that are consumed a tile later each: page of the list, its
// physical page, and then the data.
template <bool LISTS> struct TreeLook {
  const TreeArgs* A; const int32_t* list; const int32_t* table;
  int P, n, n_pos, last, hkv;
  __device__ __forceinline__ TreeLook(const TreeArgs& a, int u, const TreeList& l) : A(&a), P(a.P), n(l.n), n_pos(l.n_pos), hkv(l.hkv) {
    table = a.block_table + (size_t)l.b * a.Mmax;
    list = LISTS ? a.page_idx + (size_t)u * a.cap : nullptr;
    last = (LISTS ? a.cap : a.Mmax) * P - 1;
  }
  __device__ __forceinline__ int slot(int pos) const { return (int)page_div((uint32_t)min(pos, last), A->page_div); }
  __device__ __forceinline__ int page(int pos) const {
    if constexpr (LISTS) return clampi(list[slot(pos)], 0, A->Mmax - 1);
    else return slot(pos);
  }
  __device__ __forceinline__ int phys(int lp) const { return clampi(table[lp], 0, A->n_phys - 1); }
  __device__ __forceinline__ uint32_t row(int pos, int ph) const {
    return ((uint32_t)ph * A->HkvPool + hkv) * P + (min(pos, last) - slot(pos) * P);
  }
  __device__ __forceinline__ bool valid(int pos, int lp) const { return pos < n_pos && (int64_t)lp * P + (pos - slot(pos) * P) < n; }
};

// A tile of drafted keys (and values): rows [d0, d0 + kKeys) of R, zeros behind the last.  The threads that stage a tile call it;
// found(row, v): a piece of the values, to be changed where it has to be.
template <typename TQ, typename S, int SIDES, typename F>
__device__ __forceinline__ void stage_drafted(const TreeArgs& A, char* lds, int tid, const TreeRows& R, int hkv, int d0, F&& found) {
  constexpr int kPieces = S::kRowBytes / 16, kTotal = S::kKeys * kPieces, kBatch = kTotal < 4 * S::kThreads ? kTotal / S::kThreads : 4;
  static_assert(kTotal % (kBatch * S::kThreads) == 0, "whole batches");
#pragma unroll 1
  for (int i0 = 0; i0 < kTotal; i0 += kBatch * S::kThreads) {
    uint4 k[kBatch], v[kBatch];
    const bool any = d0 + i0 / kPieces < R.count;                          // the same for the threads
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      k[q] = v[q] = make_uint4(0u, 0u, 0u, 0u);
      if (any) {
        const int i = i0 + q * S::kThreads + tid, row = R.first + min(d0 + i / kPieces, R.count - 1);
        k[q] = load16((const char*)((const TQ*)A.k_new + row * A.ks + hkv * kD) + 16 * (i % kPieces));
        if constexpr (SIDES == 2) v[q] = load16((const char*)((const TQ*)A.v_new + row * A.vs + hkv * kD) + 16 * (i % kPieces));
      }
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int i = i0 + q * S::kThreads + tid, row = i / kPieces, piece = i % kPieces;
      const uint32_t keep = d0 + row < R.count ? ~0u : 0u;
      k[q] = make_uint4(k[q].x & keep, k[q].y & keep, k[q].z & keep, k[q].w & keep);
      *reinterpret_cast<uint4*>(lds + tree_piece<TQ>(row, piece)) = k[q];
      if constexpr (SIDES == 2) {
        v[q] = make_uint4(v[q].x & keep, v[q].y & keep, v[q].z & keep, v[q].w & keep);
        found(row, v[q]);
        *reinterpret_cast<uint4*>(lds + S::kSideBytes + tree_piece<TQ>(row, piece)) = v[q];
      }
    }
  }
}

// Query operands of a wavefront's NQ tiles of rows: lane (c, j) has of row c of a tile channels 32 s + 8 j + 0..7 (bf16), 16 s + 4 j +
// 0..3 (float32).  Rows behind the last one repeat it.
template <typename TQ, int NQ> struct TreeQuery {
  static constexpr int kSteps = sizeof(TQ) == 2 ? 4 : 8;
  uint4 v[NQ][kSteps];
  __device__ __forceinline__ void load(const TreeArgs& A, const TreeRows& R, int list_head, int r0) {
    const int lane = threadIdx.x & 63, c = lane & 15, j = lane >> 4;
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      const int r = min(r0 + 16 * t + c, R.count * A.GL - 1), tok = r / A.GL;
      const TQ* row = (const TQ*)A.q + ((size_t)(R.first + tok) * A.Hq + list_head + (r - tok * A.GL)) * kD;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) v[t][s] = *reinterpret_cast<const uint4*>(row + (sizeof(TQ) == 2 ? 32 * s + 8 * j : 16 * s + 4 * j));
    }
  }
};

// S^T of M tiles of sixteen keys (from tile m0 of the LDS tile on) and a wavefront's rows: lane (c, j) gets keys 4j..4j+3 of row c.
template <typename TQ, int NQ, int M>
__device__ __forceinline__ void tree_scores(const char* k, int m0, const TreeQuery<TQ, NQ>& q, f32x4_t (&d)[M][NQ]) {
  const int lane = threadIdx.x & 63, c = lane & 15, j = lane >> 4;
  constexpr int kSums = sizeof(TQ) == 2 ? 1 : 4;       // float32: a product has 4 of the 128 channels, four sums of 8 each round less
  f32x4_t sum[kSums][M][NQ];
#pragma unroll
  for (int m = 0; m < M; ++m) {
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
#pragma unroll
      for (int e = 0; e < kSums; ++e) sum[e][m][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
  }
#pragma unroll
  for (int s = 0; s < TreeQuery<TQ, NQ>::kSteps; ++s) {
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const uint4 a = *reinterpret_cast<const uint4*>(k + tree_piece<TQ>(16 * (m0 + m) + c, 4 * s + j));
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        if constexpr (sizeof(TQ) == 2) {
          sum[0][m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, q.v[t][s]), sum[0][m][t], 0, 0, 0);
        } else {
          const f32x4_t x = __builtin_bit_cast(f32x4_t, a), y = __builtin_bit_cast(f32x4_t, q.v[t][s]);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[e][m][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], sum[e][m][t], 0, 0, 0);
        }
      }
    }
  }
#pragma unroll
  for (int m = 0; m < M; ++m) {
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      if constexpr (sizeof(TQ) == 2) d[m][t] = sum[0][m][t];
      else d[m][t] = (sum[0][m][t] + sum[1][m][t]) + (sum[2][m][t] + sum[3][m][t]);
    }
  }
}

// All tiles of the LDS tile: together, or in float32, whose sums take four registers for one, a tile after the other.
template <typename TQ, int NQ, int M>
__device__ __forceinline__ void tree_scores_all(const char* k, const TreeQuery<TQ, NQ>& q, f32x4_t (&d)[M][NQ]) {
  if constexpr (sizeof(TQ) == 2) {
    tree_scores<TQ, NQ, M>(k, 0, q, d);
  } else {
#pragma unroll
    for (int m = 0; m < M; ++m) {
      f32x4_t one[1][NQ];
      tree_scores<TQ, NQ, 1>(k, m, q, one);
#pragma unroll
      for (int t = 0; t < NQ; ++t) d[m][t] = one[0][t];
    }
  }
}

// Which workgroup this is among those that take the steps in order: stretches per XCD, so that row blocks of a list, and lists that
// name the same pages, meet in one L2.
__device__ __forceinline__ int tree_workgroup() {
  return gridDim.x % kXcds == 0 ? (int)(blockIdx.x % kXcds * (gridDim.x / kXcds) + blockIdx.x / kXcds) : (int)blockIdx.x;
}

// The work of a launch: the steps of all lists (for every block of `rows` rows its tiles of `keys` positions, and one step for the
// drafted keys), in order, of which every workgroup takes an even, contiguous share; or, per_unit, a block of rows whole.  seg(wg, unit, list,
// blk, st0, st1, steps, first) is called for every stretch [st0, st1) of a block's `steps`; first: the workgroup's first one.
// pre_lds: dynamic LDS for the steps before a list.
template <int THREADS, int ROWS, int KEYS, typename F>
__device__ __forceinline__ void tree_work(const TreeArgs& A, int* pre_lds, int* wsum, F&& seg) {
  const bool in_lds = A.pre_g == nullptr;
  const int wg = A.per_unit ? (int)blockIdx.x : tree_workgroup();
  int unit = 0, begin = 0, end = 0;
  auto range = [&](auto pre) {
    const int total = uniform(pre[A.U]), per = total / A.W, rem = total - per * A.W;
    begin = wg * per + min(wg, rem);
    end = begin + per + (wg < rem ? 1 : 0);
    unit = wave_last_at_most(pre, A.U, begin);
  };
  if (A.per_unit) {
    unit = wg / A.blocks;
    const TreeList l = tree_list(A, unit);
    const int steps = (l.n_pos + KEYS - 1) / KEYS + 1, blk = wg - unit * A.blocks;
    if (blk >= tree_blocks(A, l.R.count, ROWS)) return;
    begin = blk * steps;
    end = begin + steps;
  } else if (in_lds) {
    block_exclusive_prefix<THREADS>(A.U, [&](int u) { return tree_unit_steps(A, u, KEYS, ROWS); }, pre_lds, wsum);
    range((const int*)pre_lds);
    if (blockIdx.x == 0)
      for (int u = threadIdx.x; u <= A.U; u += THREADS) A.pre[u] = pre_lds[u];
  } else {
    range(A.pre_g);
  }
  for (int at = begin; at < end;) {
    int u_begin = 0, u_end = 0;
    auto bounds = [&](auto pre) {
      while (at >= uniform(pre[unit + 1])) ++unit;
      u_begin = uniform(pre[unit]); u_end = uniform(pre[unit + 1]);
    };
    if (A.per_unit) u_end = end;
    else if (in_lds) bounds((const int*)pre_lds);
    else bounds(A.pre_g);
    const TreeList l = tree_list(A, unit);
    const int steps = (l.n_pos + KEYS - 1) / KEYS + 1, blk = (at - u_begin) / steps, blk_begin = u_begin + blk * steps;
    const int seg_end = min(min(end, u_end), blk_begin + steps);
    seg(wg, unit, l, blk, at - blk_begin, seg_end - blk_begin, steps, at == begin);
    at = seg_end;
  }
}

// Workspace of the item prefix
static inline size_t tree_pre_bytes(size_t units) { return ((units + 1) * sizeof(int32_t) + 255) & ~(size_t)255; }
void launch_tree_prefix(const TreeArgs& a, int keys, int rows, hipStream_t st);
void launch_tree_solve(const Dims& dm, const TreeArgs& a, bool codes, int32_t* supp, hipStream_t st);
// api.hip fills in views, sizes and outputs; scratch is carved from ws.  codes: the cache is held in 8 bits.
void launch_tree_softmax(const Dims& dm, TreeArgs a, bool codes, void* ws, hipStream_t st);
void launch_tree_entmax(const Dims& dm, TreeArgs a, bool codes, int32_t* supp, void* ws, hipStream_t st);
// lists: page lists per sequence (query heads or KV heads), most: drafted rows of a sequence
// steps are counted in 31 bits, threads of a launch in 32
bool tree_softmax_supported(const Dims& dm, bool dense, int lists, int most);
bool tree_entmax_supported(const Dims& dm, bool dense, int lists, int most);
size_t tree_softmax_ws_bytes(const Dims& dm, bool dense, int lists, int most);
size_t tree_entmax_ws_bytes(const Dims& dm, bool dense, int lists, int n_tokens);

// cache type of an instantiation
template <typename TQ, bool CODES> struct TreeCache { using type = TQ; };
template <typename TQ> struct TreeCache<TQ, true> { using type = e4m3_t; };

}  // namespace ekv
