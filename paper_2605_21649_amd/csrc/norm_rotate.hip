// Norm and rotation of a step's queries and keys, head by head: y = x / sqrt(mean x^2 + eps) * w, then channels (i, j) of each
// pair by the angle pos * freq[i]: (y_i cos - y_j sin, y_j cos + y_i sin).
//
// Sixteen lanes own one head of one token, lane c its channels 8c..8c+7: the mean is a DPP row sum, the partner of a channel is
// in the same lane (neighbours) or half the turned channels away (halves).  Angles are the same for all heads of a token: a
// workgroup computes them once, at most 64 a token, into LDS.  A position of a million times a frequency of one loses four digits in 32 bits, so
// the product is taken in 64, as turns, and only what is left of a whole turn goes to 32.  Sums and products are float32, rounded
// once.  Bound by the bytes: every head read and written once, 32768 tokens of 40 heads in bf16, 671 MB, in 163 us, 4.1 TB/s (a copy: 4.7).
#include "ekv_device.h"
#include "ekv_internal.h"

namespace ekv {

constexpr int kNormThreads = 256, kNormHeads = kNormThreads / 16;      // heads a workgroup has at hand at once
constexpr int kNormTokens = 2;                                         // tokens of a workgroup at most
constexpr int kBatch = 4;

struct NormRotateArgs {
  const void* x[2]; int64_t stride[2];           // queries, keys: rows of Hq and Hkv heads
  const void* w[2];                              // null: no norm
  void* y[2];
  const float* freq; const int32_t* pos;         // freq null: no rotation; pos null: every token is there
  float eps;
  int n, Hq, Hkv, half;                          // half: pairs that are turned
  int tokens, heads;                             // per workgroup
};

// eight channels in a row, or past the caches
template <bool STREAM> __device__ __forceinline__ void load_raw(const bf16_t* p, Raw8<bf16_t>& r) { r.a = load16<STREAM>(p); }
template <bool STREAM> __device__ __forceinline__ void load_raw(const float* p, Raw8<float>& r) {
  r.a = __builtin_bit_cast(float4, load16<STREAM>(p));
  r.b = __builtin_bit_cast(float4, load16<STREAM>(p + 4));
}
template <bool STREAM> __device__ __forceinline__ void store_row(bf16_t* p, const float (&x)[8]) { store16<STREAM>(p, pack8(x)); }
template <bool STREAM> __device__ __forceinline__ void store_row(float* p, const float (&x)[8]) {
  store16<STREAM>(p, __builtin_bit_cast(uint4, make_float4(x[0], x[1], x[2], x[3])));
  store16<STREAM>(p + 4, __builtin_bit_cast(uint4, make_float4(x[4], x[5], x[6], x[7])));
}

template <typename T, bool PAIRS, bool STREAM>
__global__ __launch_bounds__(kNormThreads) void norm_rotate_kernel(const NormRotateArgs A) {
  __shared__ float s_cos[kNormTokens][kD / 2], s_sin[kNormTokens][kD / 2];
  const int H = A.Hq + A.Hkv, blocks = (H + A.heads - 1) / A.heads;
  const int t0 = (int)(blockIdx.x / (unsigned)blocks) * A.tokens, h0 = (int)(blockIdx.x % (unsigned)blocks) * A.heads;
  const int nt = min(A.tokens, A.n - t0), nh = min(A.heads, H - h0);
  const int lane = threadIdx.x & 63, c = threadIdx.x & 15;
  const int total = nt * nh, mine = threadIdx.x >> 4;
  // Heads of a batch: sixteen at a time, kBatch of them under way, the next batch requested before this one is worked on, and the first
  // one before the angles.
  struct Batch { Raw8<T> raw[kBatch]; };
  auto place = [&](int base, int j, int& tok, int& side, int& h) {
    const int i = min(base + j * kNormHeads + mine, total - 1);
    tok = i / nh;
    h = h0 + (i - tok * nh);
    side = h < A.Hq ? 0 : 1;
    h -= side ? A.Hq : 0;
  };
  auto request = [&](int base, Batch& x) {
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (base + j * kNormHeads >= total) break;           // the same for the workgroup
      int tok, side, h;
      place(base, j, tok, side, h);
      load_raw<STREAM>((const T*)A.x[side] + (int64_t)(t0 + tok) * A.stride[side] + h * kD + 8 * c, x.raw[j]);
    }
  };
  Batch now, next;
  request(0, now);
  float w[2][8];
#pragma unroll
  for (int side = 0; side < 2; ++side)
    if (A.w[side] != nullptr) load8((const T*)A.w[side] + 8 * c, w[side]);
  if (A.half > 0) {
    for (int i = threadIdx.x; i < nt * A.half; i += kNormThreads) {
      const int t = i / A.half, k = i - t * A.half;
      double turns = (double)A.pos[t0 + t] * (double)A.freq[k] * 0.15915494309189533577;   // 1 / (2 pi)
      turns -= __builtin_rint(turns);
      sincospif(2.0f * (float)turns, &s_sin[t][k], &s_cos[t][k]);
    }
    __syncthreads();
  }
  // where the lane's channels are among the turned ones, and the lane that has their partners
  const bool turned = 8 * c < 2 * A.half, upper = !PAIRS && 8 * c >= A.half;
  const int angle = PAIRS ? 4 * c : 8 * c - (upper ? A.half : 0);
  const int partner = turned ? (lane & 48) | (c + (upper ? -1 : 1) * (A.half / 8)) : lane;
  for (int base = 0; base < total; base += kBatch * kNormHeads) {
    request(base + kBatch * kNormHeads, next);
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (base + j * kNormHeads >= total) break;
      int tok, side, h;
      place(base, j, tok, side, h);
      const int t = t0 + tok;
      float y[8];
      widen8(now.raw[j], y);
      float sq = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sq = fmaf(y[e], y[e], sq);
      sq = row16_sum(sq);
      if (A.w[side] != nullptr) {
        const float f = 1.0f / sqrtf(sq * (1.0f / kD) + A.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = y[e] * f * (side ? w[1][e] : w[0][e]);
      }
      if (A.half > 0) {
        if constexpr (PAIRS) {
          if (turned) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float cs = s_cos[tok][angle + e], sn = s_sin[tok][angle + e], a = y[2 * e], b = y[2 * e + 1];
              y[2 * e] = a * cs - b * sn;
              y[2 * e + 1] = b * cs + a * sn;
            }
          }
        } else {
          float other[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) other[e] = __shfl(y[e], partner);
          if (turned) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float cs = s_cos[tok][angle + e], sn = s_sin[tok][angle + e];
              y[e] = upper ? y[e] * cs + other[e] * sn : y[e] * cs - other[e] * sn;
            }
          }
        }
      }
      if (base + j * kNormHeads + mine < total && (A.pos == nullptr || A.pos[t] >= 0))
        store_row<STREAM>((T*)A.y[side] + ((size_t)t * (side ? A.Hkv : A.Hq) + h) * kD + 8 * c, y);
    }
    now = next;
  }
}

template <typename T, bool STREAM>
static void launch_norm_T(const NormRotateArgs& a, bool pairs, unsigned grid, hipStream_t st) {
  if (pairs) hipLaunchKernelGGL((norm_rotate_kernel<T, true, STREAM>), dim3(grid), dim3(kNormThreads), 0, st, a);
  else hipLaunchKernelGGL((norm_rotate_kernel<T, false, STREAM>), dim3(grid), dim3(kNormThreads), 0, st, a);
}

// A workgroup has sixteen heads of one token where heads are few, so that a step's are all under way at once; all heads of one token,
// or of two, where there are enough to fill the GPU and the angles want sharing.  us, 40 heads bf16, one token / two / three / four:
// 512 tokens 7.4 / 8.8 / 11.5, 1024 9.7 / 10.2 / 13.2, 2048 16.3 / 13.6 / 16.3 / 18.1, 8192 56 / 46 / 47, 32768 206 / 165 / 162 / 163.
// Heads and outputs past the caches from 32 MiB, kept / past: 1024 tokens (10 MB) 11.1 / 10.2, 4096 26.4 / 25.3, 8192 51.3 / 46.0, 32768
// 172 / 165; float32 1024 12.9 / 13.1, 4096 42.0 / 39.1, 16384 137 / 137; below the line the scoring and the attention that come next find them there.
constexpr long long kStreamHeadsBytes = 32ll << 20;

void launch_norm_rotate(const Dims& dm, const void* x_q, int64_t q_stride, const void* x_k, int64_t k_stride, const void* w_q,
                        const void* w_k, float eps, const float* freq, int n_freq, const int32_t* pos, int n, bool pairs, void* q_out,
                        void* k_out, hipStream_t st) {
  NormRotateArgs a{{x_q, x_k}, {q_stride, k_stride}, {w_q, w_k}, {q_out, k_out}, freq, pos, eps, n, dm.Hq, dm.Hkv, n_freq, 1, kNormHeads};
  const int H = dm.Hq + dm.Hkv;
  const long long heads = (long long)n * H;
  if (heads >= 16384) {
    a.heads = H;
    a.tokens = heads >= 65536 ? kNormTokens : 1;
  }
  const unsigned grid = (unsigned)((long long)((n + a.tokens - 1) / a.tokens) * ((H + a.heads - 1) / a.heads));
  const bool stream = heads * kD * (dm.dtype == EKV_F32 ? 4 : 2) >= kStreamHeadsBytes;
  if (dm.dtype == EKV_F32) {
    if (stream) launch_norm_T<float, true>(a, pairs, grid, st);
    else launch_norm_T<float, false>(a, pairs, grid, st);
  } else {
    if (stream) launch_norm_T<bf16_t, true>(a, pairs, grid, st);
    else launch_norm_T<bf16_t, false>(a, pairs, grid, st);
  }
}

}  // namespace ekv
