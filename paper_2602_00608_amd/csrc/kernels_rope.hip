// Rotary positions: pairs of channels of a head turn by position * frequency.
#include "common.hpp"

namespace wmdec {
namespace {

constexpr int NT = 256;
constexpr double kTwoPi = 6.283185307179586476925286766559;

struct FreqParams { double* freq; int axes; int dim[3]; wmdec_rope_scaling sc; };

__global__ void rope_frequencies_kernel(FreqParams p) {
  int j = blockIdx.x * blockDim.x + threadIdx.x, axis = 0;
  const int at = j;
  while (axis < p.axes && j >= p.dim[axis] / 2) j -= p.dim[axis++] / 2;
  if (axis == p.axes) return;
  const double d = p.dim[axis];
  const double base = p.sc.kind == WMDEC_ROPE_BASE ? p.sc.base * pow(p.sc.factor, d / (d - 2)) : p.sc.base;
  double f = pow(base, -2.0 * j / d);
  if (p.sc.kind == WMDEC_ROPE_LINEAR) f /= p.sc.factor;
  if (p.sc.kind == WMDEC_ROPE_RAMP) {
    const double w = fmin(fmax((p.sc.trained_length * f / kTwoPi - p.sc.low_turns) / (p.sc.high_turns - p.sc.low_turns), 0.0), 1.0);
    f *= w + (1.0 - w) / p.sc.factor;
  }
  p.freq[at] = f;
}

// One thread: one pair of one head of one token, or one channel that is copied.
template <typename T>
__global__ __launch_bounds__(NT) void rope_kernel(RopeArgs a) {
  const int pairs = a.rot / 2, units = pairs + (a.d - a.rot), heads = a.q.heads + a.k.heads;
  const long i = (long)blockIdx.x * NT + threadIdx.x, per_token = (long)units * heads;
  if (i >= per_token * a.n * a.t) return;
  const long token = i / per_token;
  const int n = (int)(token / a.t), t = (int)(token % a.t), u = (int)(i % units);
  int head = (int)(i % per_token / units);
  const bool second = head >= a.q.heads;
  const RopeTensor& x = second ? a.k : a.q;
  if (second) head -= a.q.heads;
  const T* in = (const T*)x.in + n * x.si.sample + t * x.si.token + head * x.si.head;
  T* out = (T*)x.out + n * x.so.sample + t * x.so.token + head * x.so.head;
  if (u >= pairs) {
    out[a.rot + u - pairs] = in[a.rot + u - pairs];
    return;
  }
  int axis = 0, j = u, first = 0;
  while (j >= a.layout.axis_dim[axis] / 2) { first += a.layout.axis_dim[axis]; j -= a.layout.axis_dim[axis++] / 2; }
  const int c0 = first + (a.layout.interleaved ? 2 * j : j), c1 = a.layout.interleaved ? c0 + 1 : c0 + a.layout.axis_dim[axis] / 2;
  double theta = (double)a.positions[n * a.positions_stride + (long)t * a.layout.axes + axis] * a.freq[u];
  if (a.layout.inverse) theta = -theta;
  double sn, cs;
  sincos(theta, &sn, &cs);
  const float c = (float)(cs * a.layout.magnitude), s = (float)(sn * a.layout.magnitude);
  const float v0 = to_float(in[c0]), v1 = to_float(in[c1]);
  out[c0] = from_float<T>(v0 * c - v1 * s);
  out[c1] = from_float<T>(v0 * s + v1 * c);
}

template <typename T>
int launch(const RopeArgs& a, hipStream_t s) {
  const long total = (long)(a.rot / 2 + a.d - a.rot) * (a.q.heads + a.k.heads) * a.n * a.t;
  WMDEC_REQUIRE((total + NT - 1) / NT < (1L << 31), WMDEC_ERR_UNSUPPORTED, "rope: too many elements");
  hipLaunchKernelGGL(rope_kernel<T>, dim3((unsigned)((total + NT - 1) / NT)), dim3(NT), 0, s, a);
  WMDEC_HIP(hipGetLastError());
  return WMDEC_OK;
}

}  // namespace

int launch_rope_frequencies(double* freq, int axes, const int* axis_dim, const wmdec_rope_scaling& sc, hipStream_t s) {
  FreqParams p{freq, axes, {0, 0, 0}, sc};
  int pairs = 0;
  for (int i = 0; i < axes; ++i) { p.dim[i] = axis_dim[i]; pairs += axis_dim[i] / 2; }
  hipLaunchKernelGGL(rope_frequencies_kernel, dim3((unsigned)((pairs + 63) / 64)), dim3(64), 0, s, p);
  WMDEC_HIP(hipGetLastError());
  return WMDEC_OK;
}

int launch_rope(const RopeArgs& a, int dtype, hipStream_t s) {
  switch (dtype) {
    case WMDEC_F32: return launch<float>(a, s);
    case WMDEC_BF16: return launch<bf16_t>(a, s);
    default: return launch<f16_t>(a, s);
  }
}

}  // namespace wmdec
