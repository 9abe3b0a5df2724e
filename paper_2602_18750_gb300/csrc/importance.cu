// importance.cu -- the attention weights that a prompt's tokens receive, summed over its queries (Sec. 4.1 for
// prompt tokens): one warp per (sequence, KV head or all, key), a lane four channels.
#include "prompt_common.cuh"

namespace hill {
namespace {

constexpr int kWarps = 8;

template <int DT>
__device__ __forceinline__ float4 load4(const uint16_t* p) {
  const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
  const float2 x = unpack2<DT>(v.x), y = unpack2<DT>(v.y);
  return float4{x.x, x.y, y.x, y.y};
}

template <int DT>
__global__ void __launch_bounds__(kWarps * 32) hill_prompt_importance_kernel(const __grid_constant__ PromptArgs a) {
  const int lane = threadIdx.x & 31, b = blockIdx.z, row = blockIdx.y;
  pdl_wait();
  const Seq s = seq_at(a, b);
  const int j = blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (s.m > a.cap && j == 0 && lane == 0) raise_error(a.err, kErrDevArg);
  if (j >= min(s.m, a.cap)) return;
  float sum = 0.f;
  for (int g = a.kvh ? row : 0; g < (a.kvh ? row + 1 : a.Hkv); ++g) {
    const float4 k = load4<DT>(static_cast<const uint16_t*>(a.k) + (s.k0 + j) * a.k_st + g * a.k_sh + 4 * lane);
    for (int i = max(0, s.n - a.newest); i < s.n; ++i) {
      if (!sees(a, i + s.shift(), j)) continue;
      for (int h = g * a.G; h < (g + 1) * a.G; ++h) {
        const float4 q = load4<DT>(static_cast<const uint16_t*>(a.q) + (s.q0 + i) * a.q_st + h * a.q_sh + 4 * lane);
        const float z = warp_sum(q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w) * kLog2eInvSqrtD;
        sum += ex2(z - a.lse[(int64_t)(s.q0 + i) * a.H + h] * 1.4426950408889634f);
      }
    }
  }
  if (lane == 0) a.accum[((int64_t)b * (a.kvh ? a.Hkv : 1) + row) * a.cap + j] += sum;
}

}  // namespace

int importance_splits(int B, int Hkv, int64_t k_rows, int sms) { return 1; }

cudaError_t launch_prompt_importance(const PromptArgs& a, int dtype, int sms, cudaStream_t st, int* kernels) {
  *kernels = 1;
  const dim3 grid((a.cap + kWarps - 1) / kWarps, a.kvh ? a.Hkv : 1, a.B);
  return dtype ? launch_pdl(hill_prompt_importance_kernel<1>, grid, dim3(kWarps * 32), 0, st, 0, a)
               : launch_pdl(hill_prompt_importance_kernel<0>, grid, dim3(kWarps * 32), 0, st, 0, a);
}

}  // namespace hill
