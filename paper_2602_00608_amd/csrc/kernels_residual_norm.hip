// Gated residual with the norms on both of its sides: x' = x + s * g * P(h), y = N(x') * (1 + c) + b, rows of d channels.
#include "common.hpp"

namespace wmdec {
namespace {

constexpr int NT = 256;

__device__ __forceinline__ float block_sum(float v, float* s_red) {
  for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_red[threadIdx.x >> 6] = v;
  __syncthreads();
  return s_red[0] + s_red[1] + s_red[2] + s_red[3];
}

struct Params {
  ResidualNormArgs a;
};

// A workgroup takes a row, its values in LDS.
template <typename TX, typename TA>
__global__ __launch_bounds__(NT) void residual_norm_kernel(Params p) {
  __shared__ float s_v[kResidualNormMaxD];
  __shared__ float s_red[4];
  const ResidualNormArgs& a = p.a;
  const int d = a.d, n = blockIdx.x / a.t;
  const size_t row = (size_t)blockIdx.x * d, mod = (size_t)n * a.mod_stride;
  auto statistics = [&](const wmdec_norm& norm, float& mean, float& rstd) {
    mean = 0.f; rstd = 1.f;
    if (norm.kind == WMDEC_NORM_NONE) return;
    float sum = 0.f;
    if (norm.kind == WMDEC_NORM_LAYER) {
      for (int c = threadIdx.x; c < d; c += NT) sum += s_v[c];
      mean = block_sum(sum, s_red) / d;
    }
    sum = 0.f;
    for (int c = threadIdx.x; c < d; c += NT) sum += (s_v[c] - mean) * (s_v[c] - mean);
    rstd = 1.f / sqrtf(block_sum(sum, s_red) / d + norm.eps);
  };
  auto normalise = [&](const wmdec_norm& norm, float mean, float rstd, int c) {
    if (norm.kind == WMDEC_NORM_NONE) return s_v[c];
    return (s_v[c] - mean) * rstd * (norm.weight ? norm.weight[c] : 1.f) + (norm.bias ? norm.bias[c] : 0.f);
  };
  float mean, rstd;
  if (a.h) {
    for (int c = threadIdx.x; c < d; c += NT) s_v[c] = to_float(((const TA*)a.h)[row + c]);
    statistics(a.post, mean, rstd);
    for (int c = threadIdx.x; c < d; c += NT) {
      const float v = to_float(((const TX*)a.x)[row + c]) + a.res_scale * (a.gate ? a.gate[mod + c] : 1.f) * normalise(a.post, mean, rstd, c);
      const TX stored = from_float<TX>(v);
      ((TX*)a.x_out)[row + c] = stored;
      s_v[c] = to_float(stored);
    }
  } else {
    for (int c = threadIdx.x; c < d; c += NT) s_v[c] = to_float(((const TX*)a.x)[row + c]);
  }
  if (!a.y) return;
  statistics(a.pre, mean, rstd);
  for (int c = threadIdx.x; c < d; c += NT)
    ((TA*)a.y)[row + c] = from_float<TA>(normalise(a.pre, mean, rstd, c) * (1.f + (a.scale ? a.scale[mod + c] : 0.f)) + (a.shift ? a.shift[mod + c] : 0.f));
}

template <typename TX, typename TA>
int launch(const ResidualNormArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((residual_norm_kernel<TX, TA>), dim3((unsigned)(a.n * a.t)), dim3(NT), 0, s, Params{a});
  WMDEC_HIP(hipGetLastError());
  return WMDEC_OK;
}

}  // namespace

int launch_residual_norm(const ResidualNormArgs& a, int x_dtype, int act_dtype, hipStream_t s) {
  if (x_dtype == WMDEC_BF16) return launch<bf16_t, bf16_t>(a, s);
  if (x_dtype == WMDEC_F16) return launch<f16_t, f16_t>(a, s);
  if (act_dtype == WMDEC_BF16) return launch<float, bf16_t>(a, s);
  if (act_dtype == WMDEC_F16) return launch<float, f16_t>(a, s);
  return launch<float, float>(a, s);
}

}  // namespace wmdec
