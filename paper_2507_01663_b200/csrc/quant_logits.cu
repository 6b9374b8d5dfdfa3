// af_quant_logits: logits of a few tokens from a head in 4 bits.
#include "device_util.cuh"
#include "rollout.cuh"

namespace af {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 8;

__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// A warp per row of the head and eight tokens.
template <class Out>
__global__ void __launch_bounds__(kThreads) quant_logits_kernel(const uint4* __restrict__ hidden, const uint32_t* __restrict__ codes,
                                                                const __nv_bfloat16* __restrict__ scale, int T, int d, int V,
                                                                int group, int groups, Out* __restrict__ logits, int64_t pitch) {
  const int lane = threadIdx.x & 31;
  const int v = (int)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), t0 = (int)blockIdx.y * kTokens;
  if (v >= V) return;
  float acc[kTokens] = {};
  const int words = d / 8;
  for (int c = lane; c < words; c += 32) {
    const uint32_t w = __ldg(codes + (size_t)v * words + c);
    const float s = __bfloat162float(scale[(size_t)v * groups + c * 8 / group]);
    float q[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q[2 * i] = ((int)((w >> (4 * i)) & 15u) - 8) * s;
      q[2 * i + 1] = ((int)((w >> (4 * i + 16)) & 15u) - 8) * s;
    }
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
      if (t0 + t >= T) break;
      const uint4 x = __ldg(hidden + (size_t)(t0 + t) * words + c);
      const uint32_t h[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc[t] = fmaf(q[2 * i], __uint_as_float(h[i] << 16), acc[t]);
        acc[t] = fmaf(q[2 * i + 1], __uint_as_float(h[i] & 0xffff0000u), acc[t]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < kTokens; ++t) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc[t] += __shfl_xor_sync(0xffffffffu, acc[t], o);
    if (lane == 0 && t0 + t < T) put(logits + (int64_t)(t0 + t) * pitch + v, acc[t]);
  }
}

}  // namespace

af_status launch_quant_logits(af_ctx* ctx, const void* hidden, const QuantHead& h, int64_t T, void* logits, int32_t type,
                              int64_t pitch, cudaStream_t s) {
  const dim3 grid((h.V + kThreads / 32 - 1) / (kThreads / 32), (unsigned)((T + kTokens - 1) / kTokens));
  if (type == AF_F32)
    quant_logits_kernel<<<grid, kThreads, 0, s>>>(static_cast<const uint4*>(hidden), h.codes, h.scale, (int)T, h.d, h.V, h.group,
                                                  h.groups(), static_cast<float*>(logits), pitch);
  else
    quant_logits_kernel<<<grid, kThreads, 0, s>>>(static_cast<const uint4*>(hidden), h.codes, h.scale, (int)T, h.d, h.V, h.group,
                                                  h.groups(), static_cast<__nv_bfloat16*>(logits), pitch);
  return cudaGetLastError() == cudaSuccess ? AF_OK : AF_ERR_CUDA;
}

}  // namespace af
