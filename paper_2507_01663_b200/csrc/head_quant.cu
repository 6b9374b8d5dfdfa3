// af_quantize_head: an LM head in bf16 -> 4-bit codes with a scale per group, and the values they stand for.
//
// Per group of weights w:  s = max|w| / 7 rounded to five significant bits,  q = w / s rounded to the nearest whole
// number, halves away from zero,  value = s q.  |q| <= 7: s is at least 31/32 of max|w| / 7, so |w| / s is at most 7.23.
// Five bits times three are eight: every value is a bf16 exactly, and a head of these values scores like the codes do.
//
// The rounding needs no division per weight.  A quotient of an 8-bit by a 5-bit number is a half exactly, or off it
// by 1/255 of itself at least; w times 1/s (1 + 2^-20), exact within the fused multiply-add that also rounds it to a
// whole number, lies on the far side of every half and on the right side of everything else.
//
// A stream: 2 bytes read per weight, 1/2 (and 2 for the value) written.  152064 x 3584 in groups of 128 with the values: 371-408 us,
// 6.0-6.6 TB/s, about the rate of a copy; 4096 x 256: 2.6 us on the device.
#include "device_util.cuh"
#include "rollout.cuh"

namespace af {
namespace {

constexpr int kThreads = 128;
constexpr int kUnroll = 4;                         // loads of 16 bytes in flight per thread
constexpr float kWhole = 12582920.f;               // 1.5 * 2^23 + 8: adding it rounds to a whole number, digit in the low bits
constexpr uint32_t kLargest = 0x7b80, kSmallest = 0x0d80;   // 2^120 and 2^-100 as bf16

__device__ __forceinline__ uint32_t group_max(uint4 w, int lanes) {
  uint32_t m = __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
  for (int o = 1; o < lanes; o <<= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
  return max(m & 0xffffu, m >> 16);                // magnitudes order as their bits do, NaN and infinity on top
}

struct Scale { float s, inv; };
__device__ __forceinline__ Scale group_scale(uint32_t top) {
  if (top > kLargest) return {__uint_as_float(0x7fc00000u), 0.f};
  if (top < kSmallest) return {0.f, 0.f};
  uint32_t b = __float_as_uint(__fdiv_rn(__uint_as_float(top << 16), 7.f));
  b = (b + 0x3ffffu + ((b >> 19) & 1u)) & ~0x7ffffu;           // five significant bits, halves to the even neighbour
  const float s = __uint_as_float(b);
  return {s, __fmul_rn(__frcp_rn(s), 1.f + 0x1p-20f)};
}

// A warp takes 256 weights of a row at a time.  Where whole groups fill the head's rows, all of it is one row (kOneRow).
template <bool kOneRow, bool kValues>
__global__ void __launch_bounds__(kThreads) quantize_head_kernel(const uint4* __restrict__ W, int64_t steps, int64_t chunks,
                                                                 int32_t row_chunks, int lane_shift, int32_t groups,
                                                                 uint32_t* __restrict__ codes,
                                                                 __nv_bfloat16* __restrict__ scale, uint4* __restrict__ values) {
  const int lane = threadIdx.x & 31, lanes = 1 << lane_shift;      // a group's lanes: 8 weights each
  const int64_t first = ((int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * kUnroll;
  const int row_steps = (row_chunks + 31) / 32;
  if (first >= steps) return;
  uint4 w[kUnroll];
  int64_t at[kUnroll], group_at[kUnroll];
  bool in[kUnroll];
#pragma unroll
  for (int j = 0; j < kUnroll; ++j) {
    const int64_t step = first + j;
    if constexpr (kOneRow) {
      at[j] = step * 32 + lane;
      group_at[j] = at[j] >> lane_shift;
      in[j] = at[j] < chunks;
    } else {
      const int64_t row = step / row_steps;
      const int chunk = (int)(step - row * row_steps) * 32 + lane;
      at[j] = row * row_chunks + chunk;
      group_at[j] = row * groups + (chunk >> lane_shift);
      in[j] = step < steps && chunk < row_chunks;
    }
    w[j] = in[j] ? __ldcs(W + at[j]) : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int j = 0; j < kUnroll; ++j) {
    const Scale g = group_scale(group_max(w[j], lanes));
    const uint32_t half[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
    uint32_t word = 0, v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = fmaf(__uint_as_float(half[i] << 16), g.inv, kWhole), b = fmaf(__uint_as_float(half[i] & 0xffff0000u), g.inv, kWhole);
      word |= __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x5410) << (4 * i);
      if constexpr (kValues) v[i] = pack_bf16x2((a - kWhole) * g.s, (b - kWhole) * g.s);
    }
    if (g.s != g.s) word = 0x88888888u;
    if (in[j]) {
      codes[at[j]] = word;
      if ((lane & (lanes - 1)) == 0) scale[group_at[j]] = __float2bfloat16_rn(g.s);
      if constexpr (kValues) values[at[j]] = make_uint4(v[0], v[1], v[2], v[3]);
    }
  }
}

template <bool kOneRow, bool kValues>
cudaError_t quantize(const void* W, int32_t V, int32_t d, int32_t group, void* codes, void* scale, void* values, cudaStream_t s) {
  const int row_chunks = d / 8;
  const int64_t chunks = (int64_t)V * row_chunks;
  const int64_t steps = kOneRow ? (chunks + 31) / 32 : (int64_t)V * ((row_chunks + 31) / 32);
  // Every warp has one batch: CTAs that come and go overlap one's loads with another's stores better than those that stay and loop
  // (386 us against 459 for 152064 x 3584; with a loop that runs once 412, so with 256 threads 420, 8 loads at a time 452, 2 454).
  const int64_t per_block = kUnroll * (kThreads / 32), blocks = (steps + per_block - 1) / per_block;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;       // a head of more than 10^12 weights
  quantize_head_kernel<kOneRow, kValues><<<(unsigned)blocks, kThreads, 0, s>>>(
      static_cast<const uint4*>(W), steps, chunks, row_chunks, group == 32 ? 2 : group == 64 ? 3 : 4, (d + group - 1) / group,
      static_cast<uint32_t*>(codes), static_cast<__nv_bfloat16*>(scale), static_cast<uint4*>(values));
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_quantize_head(const void* W, int32_t V, int32_t d, int32_t group, void* codes, void* scale, void* values,
                                 cudaStream_t s) {
  if (d % group == 0)
    return values ? quantize<true, true>(W, V, d, group, codes, scale, values, s)
                  : quantize<true, false>(W, V, d, group, codes, scale, values, s);
  return values ? quantize<false, true>(W, V, d, group, codes, scale, values, s)
                : quantize<false, false>(W, V, d, group, codes, scale, values, s);
}

}  // namespace af
