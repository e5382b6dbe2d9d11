// Attention to states of another length: o = softmax(scale * q k^T over the valid keys) v.
#include "common.hpp"

namespace wmdec {
namespace {

// A wavefront takes one row (a token of one query head); a lane holds every 64th channel, scores are summed over the lanes key by
// key, with the running maximum and sum of the softmax.
template <typename T>
__global__ __launch_bounds__(64) void cross_attention_kernel(CrossArgs a) {
  const int lane = threadIdx.x, heads_q = a.heads * a.group;
  const long row = blockIdx.x;
  const int hq = (int)(row % heads_q), tok = (int)(row / heads_q % a.tq), n = (int)(row / ((long)heads_q * a.tq)), h = hq / a.group;
  const int len = a.lens ? min(max(a.lens[n], 0), a.tk) : a.tk;
  const T* q = (const T*)a.q + n * a.qs.sample + tok * a.qs.token + hq * a.qs.head;
  const T* k = (const T*)a.k + n * a.ks.sample + h * a.ks.head;
  const T* v = (const T*)a.v + n * a.vs.sample + h * a.vs.head;
  float qv[4], acc[4], m = -INFINITY, l = 0.f;
  for (int i = 0; i < 4; ++i) { qv[i] = lane + 64 * i < a.d ? to_float(q[lane + 64 * i]) : 0.f; acc[i] = 0.f; }
  const float c = a.scale * 1.4426950408889634f;
  for (int j = 0; j < len; ++j) {
    if (a.mask && !a.mask[(long)n * a.tk + j]) continue;
    float s = 0.f;
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < a.d) s = fmaf(qv[i], to_float(k[j * a.ks.token + lane + 64 * i]), s);
    for (int w = 32; w > 0; w >>= 1) s += __shfl_xor(s, w);
    s *= c;
    if (s == -INFINITY) continue;   // (weight zero, also where the maximum is -inf itself)
    const float top = fmaxf(m, s);
    const float keep = __builtin_amdgcn_exp2f(m - top), p = __builtin_amdgcn_exp2f(s - top);
    m = top;
    l = fmaf(l, keep, p);
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < a.d) acc[i] = fmaf(acc[i], keep, p * to_float(v[j * a.vs.token + lane + 64 * i]));
  }
  T* o = (T*)a.o + n * a.os.sample + tok * a.os.token + hq * a.os.head;
  for (int i = 0; i < 4; ++i)
    if (lane + 64 * i < a.d) o[lane + 64 * i] = from_float<T>(l == 0.f ? 0.f : acc[i] / l);
}

}  // namespace

size_t cross_attention_scratch_bytes(int, int, int, int, int, int, int) { return 0; }

int launch_cross_attention(const CrossArgs& a, int dtype, hipStream_t s) {
  const dim3 grid((unsigned)((long)a.n * a.tq * a.heads * a.group));
  if (dtype == WMDEC_F32) hipLaunchKernelGGL(cross_attention_kernel<float>, grid, dim3(64), 0, s, a);
  else if (dtype == WMDEC_BF16) hipLaunchKernelGGL(cross_attention_kernel<bf16_t>, grid, dim3(64), 0, s, a);
  else hipLaunchKernelGGL(cross_attention_kernel<f16_t>, grid, dim3(64), 0, s, a);
  WMDEC_HIP(hipGetLastError());
  return WMDEC_OK;
}

}  // namespace wmdec
