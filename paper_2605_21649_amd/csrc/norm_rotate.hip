// Norm and rotation of a step's queries and keys, head by head: y = x / sqrt(mean x^2 + eps) * w, then channels (i, j) of each
// pair by the angle pos * freq[i]: (y_i cos - y_j sin, y_j cos + y_i sin).
//
// Sixteen lanes own one head of one token, lane c its channels 8c..8c+7: the mean is a DPP row sum, the partner of a channel is
// in the same lane (neighbours) or half the turned channels away (halves).  Angles are the same for all heads of a token: a
// workgroup computes them once, at most 64 a token, into LDS.  A position of a million times a frequency of one loses four digits in 32 bits, so
// the product is taken in 64, as turns, and only what is left of a whole turn goes to 32.  Sums and products are float32, rounded
// once.  Bound by the bytes: every head read and written once.
#include "ekv_device.h"
#include "ekv_internal.h"

namespace ekv {

constexpr int kNormThreads = 256, kNormHeads = kNormThreads / 16;      // heads a workgroup has at hand at once
constexpr int kNormTokens = 4;                                         // tokens of a workgroup, where there are many

struct NormRotateArgs {
  const void* x[2]; int64_t stride[2];           // queries, keys: rows of Hq and Hkv heads
  const void* w[2];                              // null: no norm
  void* y[2];
  const float* freq; const int32_t* pos;         // freq null: no rotation; pos null: every token is there
  float eps;
  int n, Hq, Hkv, half;                          // half: pairs that are turned
  int tokens, heads;                             // per workgroup
};

template <typename T, bool PAIRS>
__global__ __launch_bounds__(kNormThreads) void norm_rotate_kernel(const NormRotateArgs A) {
  __shared__ float s_cos[kNormTokens][kD / 2], s_sin[kNormTokens][kD / 2];
  const int H = A.Hq + A.Hkv, blocks = (H + A.heads - 1) / A.heads;
  const int t0 = (int)(blockIdx.x / (unsigned)blocks) * A.tokens, h0 = (int)(blockIdx.x % (unsigned)blocks) * A.heads;
  const int nt = min(A.tokens, A.n - t0), nh = min(A.heads, H - h0);
  const int lane = threadIdx.x & 63, c = threadIdx.x & 15;
  if (A.half > 0) {
    for (int i = threadIdx.x; i < nt * A.half; i += kNormThreads) {
      const int t = i / A.half, k = i - t * A.half;
      double turns = (double)A.pos[t0 + t] * (double)A.freq[k] * 0.15915494309189533577;   // 1 / (2 pi)
      turns -= __builtin_rint(turns);
      sincospif(2.0f * (float)turns, &s_sin[t][k], &s_cos[t][k]);
    }
    __syncthreads();
  }
  float w[2][8];
#pragma unroll
  for (int side = 0; side < 2; ++side)
    if (A.w[side] != nullptr) load8((const T*)A.w[side] + 8 * c, w[side]);
  // where the lane's channels are among the turned ones, and the lane that has their partners
  const bool turned = 8 * c < 2 * A.half, upper = !PAIRS && 8 * c >= A.half;
  const int angle = PAIRS ? 4 * c : 8 * c - (upper ? A.half : 0);
  const int partner = turned ? (lane & 48) | (c + (upper ? -1 : 1) * (A.half / 8)) : lane;
  const int total = nt * nh;
  constexpr int kBatch = 4;
  for (int base = 0; base < total; base += kBatch * kNormHeads) {
    Raw8<T> raw[kBatch];
    int tok[kBatch], head[kBatch];
    const int i0 = base + (threadIdx.x >> 4);
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (base + j * kNormHeads >= total) break;           // the same for the workgroup
      const int i = min(i0 + j * kNormHeads, total - 1);
      tok[j] = i / nh; head[j] = h0 + (i - tok[j] * nh);
      const int side = head[j] < A.Hq ? 0 : 1, h = head[j] - (side ? A.Hq : 0);
      load_raw8((const T*)A.x[side] + (int64_t)(t0 + tok[j]) * A.stride[side] + h * kD + 8 * c, raw[j]);
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (base + j * kNormHeads >= total) break;
      const int side = head[j] < A.Hq ? 0 : 1, h = head[j] - (side ? A.Hq : 0), t = t0 + tok[j];
      float y[8];
      widen8(raw[j], y);
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
              const float cs = s_cos[tok[j]][angle + e], sn = s_sin[tok[j]][angle + e], a = y[2 * e], b = y[2 * e + 1];
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
              const float cs = s_cos[tok[j]][angle + e], sn = s_sin[tok[j]][angle + e];
              y[e] = upper ? y[e] * cs + other[e] * sn : y[e] * cs - other[e] * sn;
            }
          }
        }
      }
      if (i0 + j * kNormHeads < total && (A.pos == nullptr || A.pos[t] >= 0))
        store8((T*)A.y[side] + ((size_t)t * (side ? A.Hkv : A.Hq) + h) * kD + 8 * c, y);
    }
  }
}

void launch_norm_rotate(const Dims& dm, const void* x_q, int64_t q_stride, const void* x_k, int64_t k_stride, const void* w_q,
                        const void* w_k, float eps, const float* freq, int n_freq, const int32_t* pos, int n, bool pairs, void* q_out,
                        void* k_out, hipStream_t st) {
  NormRotateArgs a{{x_q, x_k}, {q_stride, k_stride}, {w_q, w_k}, {q_out, k_out}, freq, pos, eps, n, dm.Hq, dm.Hkv, n_freq, 1, kNormHeads};
  const int H = dm.Hq + dm.Hkv;
  if ((long long)n * H >= 16384) { a.tokens = kNormTokens; a.heads = H; }
  const long long grid = (long long)((n + a.tokens - 1) / a.tokens) * ((H + a.heads - 1) / a.heads);
  const dim3 g((unsigned)grid), block(kNormThreads);
  if (dm.dtype == EKV_F32) {
    if (pairs) hipLaunchKernelGGL((norm_rotate_kernel<float, true>), g, block, 0, st, a);
    else hipLaunchKernelGGL((norm_rotate_kernel<float, false>), g, block, 0, st, a);
  } else {
    if (pairs) hipLaunchKernelGGL((norm_rotate_kernel<bf16_t, true>), g, block, 0, st, a);
    else hipLaunchKernelGGL((norm_rotate_kernel<bf16_t, false>), g, block, 0, st, a);
  }
}

}  // namespace ekv
