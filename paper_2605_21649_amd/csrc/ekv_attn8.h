// What the attention kernels over the 8-bit cache share: arguments, and scores of eight tokens at a time on the matrix cores.
//
// A 16x16x32 bf16 MFMA multiplies 16 rows (A) with 16 columns (B) over 32 channels; lane (c, g) = (lane % 16, lane / 16)
// holds eight channels of row c and of column c, and the result's rows 4g..4g+3 of column c.  Eight tokens are 1 KB of codes, one
// 16-byte load a lane, and it has to be that whole kilobyte: loads that take half lines of sixteen tokens read K of 4 x
// 128K tokens in 111 us where these take 89.  So a row is half a token, (token c / 2, channels 64 (c % 2) + 16 g + 0..15 in
// lane (c, g)), and the columns are (head, half of the channels): a result counts where the halves are the same, and the
// two lanes of a head add theirs.  The 16 channels go through two instructions, widened to bf16 with the page's scale (both
// exact).  Columns beyond the heads repeat them: column c is head (c / 2) % G, half c % 2, copy (c / 2) / G.
// float32 queries are three bf16 terms whose sum is the query exactly, a product each.
#pragma once
#include "ekv_cache8.h"
#include "ekv_scores.h"

namespace ekv {

struct Score8Args {
  ScoreArgs s;                      // k_pool: the codes
  const float* k_scale;
};
// Score pass over every page with the stores put off (decode8_held.hip); false, with nothing launched, where it is not
// the faster one or the call has a form that it does not take.
bool launch_scores8_held(const Dims& dm, const Score8Args& a, long long items, long long k_bytes, hipStream_t st);

// Bytes of codes from which a call's pool passes the caches (non-temporal loads), where it is read once: every page, lists that the heads of
// a group share, lists of heads without a group.  Both sides are measured where the loads are chosen.
constexpr long long kStream8Bytes = 64ll << 20;

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

__device__ __forceinline__ int column_head(int c, int G) { return (c >> 1) & (G - 1); }
// which of the 16 / G lanes (c) of a head this is
__device__ __forceinline__ int column_copy(int c, int G) { return (c & 1) + 2 * ((c >> 1) / G); }

// The query operand of a group: word `half` has channels 64 (c % 2) + 16 g + 8 half + 0..7 of column c's head.
template <typename T, int G> struct Query8 {
  static constexpr int kTerms = sizeof(T) == 2 ? 1 : 3;
  bf16x8_t b[kTerms][2];
  __device__ __forceinline__ void load(const T* q /* the group's first head */) {
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const T* row = q + column_head(c, G) * kD + 64 * (c & 1) + 16 * g;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if constexpr (sizeof(T) == 2) {
        b[0][half] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(row + 8 * half));
      } else {
        float x[8];
        load8<float>((const float*)row + 8 * half, x);
#pragma unroll
        for (int t = 0; t < 3; ++t) {              // the upper 16 bits, then those of what is left: 24 bits in three steps
          u32x4_t w;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t a = __float_as_uint(x[2 * i]) & 0xffff0000u, d = __float_as_uint(x[2 * i + 1]) & 0xffff0000u;
            w[i] = (a >> 16) | d;
            x[2 * i] -= __uint_as_float(a); x[2 * i + 1] -= __uint_as_float(d);
          }
          b[t][half] = __builtin_bit_cast(bf16x8_t, w);
        }
      }
    }
  }
  // the loads are waited for here
  __device__ __forceinline__ void wait() {
#pragma unroll
    for (int t = 0; t < kTerms; ++t) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        u32x4_t w = __builtin_bit_cast(u32x4_t, b[t][half]);
        asm volatile("" : "+v"(w));
        b[t][half] = __builtin_bit_cast(bf16x8_t, w);
      }
    }
  }
};

// Of the pairs of scores of four octets (with eight heads, of the first two) the one that copy `copy` of the head puts away: octet
// `copy`'s, so that the copies' stores are whole lines; copies from 4 on have none.
template <int G> __device__ __forceinline__ float2 copy_pair(float2 z0, float2 z1, float2 z2, float2 z3, int copy) {
  const bool odd = copy & 1, upper = G != 8 && (copy & 2);
  const float ax = odd ? z1.x : z0.x, ay = odd ? z1.y : z0.y, bx = odd ? z3.x : z2.x, by = odd ? z3.y : z2.y;
  return make_float2(upper ? bx : ax, upper ? by : ay);
}

// n / P for 0 <= n < 64 and P <= 64, per_page = 65536 / P + 1: off by at most n / 65536 < 1 / P before the cut
__device__ __forceinline__ int div64(int n, int per_page) { return (n * per_page) >> 16; }

// Where in a page's eight tokens the lane's 16 codes are, and which token that is.
__device__ __forceinline__ int key_token(int c) { return c >> 1; }
__device__ __forceinline__ uint32_t key_offset(int c, int g) { return (c & 1) * 64 + g * 16; }
// q . k of eight tokens (k: the lane's codes): lane (c, g) gets tokens 2 g and 2 g + 1 for head column_head(c)
template <typename T, int G>
__device__ __forceinline__ void octet_scores(const uint4& k, float scale, const Query8<T, G>& q, float& z0, float& z1) {
  f32x4_t d = {0.f, 0.f, 0.f, 0.f};
  const bf16x8_t lo = widen_bf16(k.x, k.y, scale), hi = widen_bf16(k.z, k.w, scale);
#pragma unroll
  for (int t = Query8<T, G>::kTerms - 1; t >= 0; --t) {        // the smallest terms first
    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, q.b[t][0], d, 0, 0, 0);
    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, q.b[t][1], d, 0, 0, 0);
  }
  // the even lane's half of the channels and the odd neighbour's, in both
  z0 = dpp_move<0xA0>(d[0] + dpp_move<0xB1>(d[1]));
  z1 = dpp_move<0xA0>(d[2] + dpp_move<0xB1>(d[3]));
}

}  // namespace ekv
