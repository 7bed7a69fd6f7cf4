// What the attention kernels over the 8-bit cache share: arguments, and tiles of 16 tokens on the matrix cores.
//
// Scores.  A 16x16x32 bf16 MFMA multiplies 16 rows (A) with 16 columns (B) over 32 channels; lane (c, g) = (lane % 16, lane / 16)
// holds eight channels of row c and of column c, and of the result rows 4g..4g+3 of column c.  Rows are tokens, columns the
// query heads of the group, repeated: column c is head c % G.  A lane's eight channels are the half of a 16-byte load of the
// page's codes, widened to bf16 with the page's scale (both exact), so nothing is exchanged between lanes; which channels
// meet in an instruction is the same for keys and queries and else of no account.  float32 queries are three bf16 terms
// whose sum is the query exactly, a product each.
#pragma once
#include "ekv_cache8.h"
#include "ekv_scores.h"

namespace ekv {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

struct Cache8Ptrs { const e4m3_t* pool; const float* scale; };

// e4m3 pairs -> bf16 times a power of two (exact); HI: the upper two codes
template <bool HI> __device__ __forceinline__ uint32_t widen2(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
}
__device__ __forceinline__ bf16x8_t widen_bf16(uint32_t lo, uint32_t hi, float scale) {
  const u32x4_t r = {widen2<false>(lo, scale), widen2<true>(lo, scale), widen2<false>(hi, scale), widen2<true>(hi, scale)};
  return __builtin_bit_cast(bf16x8_t, r);
}

// n / P for n < 2^30 and P a multiple of 4: n / 4 < 2^28 times ceil(2^32 / (P / 4)), whose error stays below one part
struct PageDiv { uint32_t magic; };
__host__ __device__ __forceinline__ uint32_t page_div(uint32_t n, PageDiv d) {
  const uint32_t n4 = n >> 2;
  return d.magic ? (uint32_t)(((uint64_t)n4 * d.magic) >> 32) : n4;
}
static inline PageDiv make_page_div(int P) {
  const uint32_t m = (uint32_t)P / 4;
  return {m == 1 ? 0u : (uint32_t)(((1ull << 32) + m - 1) / m)};
}

// The query operand of a group: column c is head c % G; word (u, half) holds channels 64 u + 16 g + 8 half + 0..7.
template <typename T, int G> struct Query8 {
  static constexpr int kTerms = sizeof(T) == 2 ? 1 : 3;
  bf16x8_t b[kTerms][2][2];
  __device__ __forceinline__ void load(const T* q /* the group's first head */) {
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const T* row = q + (c % G) * kD + 16 * g;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if constexpr (sizeof(T) == 2) {
          b[0][u][half] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(row + 64 * u + 8 * half));
        } else {
          float x[8];
          load8<float>((const float*)row + 64 * u + 8 * half, x);
#pragma unroll
          for (int t = 0; t < 3; ++t) {            // the upper 16 bits, then those of what is left: 24 bits in three steps
            u32x4_t w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t a = __float_as_uint(x[2 * i]) & 0xffff0000u, d = __float_as_uint(x[2 * i + 1]) & 0xffff0000u;
              w[i] = (a >> 16) | d;
              x[2 * i] -= __uint_as_float(a); x[2 * i + 1] -= __uint_as_float(d);
            }
            b[t][u][half] = __builtin_bit_cast(bf16x8_t, w);
          }
        }
      }
    }
  }
};

// A tile's keys as loaded: lane (c, g) has the codes of token c, channels 16 g + 0..15 and 64 + 16 g + 0..15.
struct KeyTile { uint4 a[2]; };
template <bool STREAM> __device__ __forceinline__ void load_keys(const e4m3_t* row /* of the lane's token, at channel 16 g */, KeyTile& k) {
  k.a[0] = load16<STREAM>(row);
  k.a[1] = load16<STREAM>(row + 64);
}
// q . k of the tile: lane (c, g), entry r: token 4 g + r, head c % G
template <typename T, int G>
__device__ __forceinline__ f32x4_t tile_scores(const KeyTile& k, float scale, const Query8<T, G>& q) {
  f32x4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int t = Query8<T, G>::kTerms - 1; t >= 0; --t) {        // the smallest terms first
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen_bf16(k.a[u].x, k.a[u].y, scale), q.b[t][u][0], d, 0, 0, 0);
      d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen_bf16(k.a[u].z, k.a[u].w, scale), q.b[t][u][1], d, 0, 0, 0);
    }
  }
  return d;
}

}  // namespace ekv
