// prompt.cu -- causal attention over packed prompts (Eq. 1 for every query of a prompt): one warp per
// (query row, query head), a lane four channels, the running maximum and sum of the softmax in one pass
// over the keys.
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
__global__ void __launch_bounds__(kWarps * 32) hill_prompt_attn_kernel(const __grid_constant__ PromptArgs a) {
  const int lane = threadIdx.x & 31, h = blockIdx.y, g = h / a.G;
  pdl_wait();
  if (blockIdx.x == 0 && h == 0)   // every sequence's offsets are looked at once
    for (int b = threadIdx.x; b < a.B; b += kWarps * 32) seq_at(a, b);
  const int t = blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (t >= a.q_rows) return;
  int b = 0;
  while (b < a.B && a.q_start[b + 1] <= t) ++b;
  if (b == a.B || t < a.q_start[b]) return;
  const Seq s = seq_at(a, b);
  const int pos = t - s.q0 + s.shift();
  const auto* K = static_cast<const uint16_t*>(a.k) + g * a.k_sh + 4 * lane;
  const auto* V = static_cast<const uint16_t*>(a.v) + g * a.v_sh + 4 * lane;
  const float4 q = load4<DT>(static_cast<const uint16_t*>(a.q) + t * a.q_st + h * a.q_sh + 4 * lane);
  float m = kNegHuge, l = 0.f;
  float4 o{0.f, 0.f, 0.f, 0.f};
  bool any = false;
  for (int j = 0; j <= min(pos, s.m - 1); ++j) {
    if (!sees(a, pos, j)) continue;
    any = true;
    const float4 k = load4<DT>(K + (s.k0 + j) * a.k_st), v = load4<DT>(V + (s.k0 + j) * a.v_st);
    const float z = warp_sum(q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w) * kLog2eInvSqrtD;
    const float mn = fmaxf(m, z), f = ex2(m - mn), p = ex2(z - mn);
    m = mn;
    l = l * f + p;
    o = float4{o.x * f + p * v.x, o.y * f + p * v.y, o.z * f + p * v.z, o.w * f + p * v.w};
  }
  const float inv = any ? 1.f / l : 0.f;
  const int64_t at = (int64_t)t * a.H + h;
  reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at * kHeadDim)[lane] =
      uint2{pack2<DT>(o.x * inv, o.y * inv), pack2<DT>(o.z * inv, o.w * inv)};
  if (a.lse && lane == 0) a.lse[at] = any ? m * 0.6931471805599453f + logf(l) : -INFINITY;
}

}  // namespace

cudaError_t launch_prompt_attn(const PromptArgs& a, int dtype, int sms, cudaStream_t st, int* kernels) {
  *kernels = 1;
  const dim3 grid((a.q_rows + kWarps - 1) / kWarps, a.H);
  return dtype ? launch_pdl(hill_prompt_attn_kernel<1>, grid, dim3(kWarps * 32), 0, st, 0, a)
               : launch_pdl(hill_prompt_attn_kernel<0>, grid, dim3(kWarps * 32), 0, st, 0, a);
}

}  // namespace hill
