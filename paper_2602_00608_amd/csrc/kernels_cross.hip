// Attention to states of another length: o = softmax(scale * q k^T over the valid keys) v.  The kernels are in cross_device.hpp; here is what is decided on
// sizes alone, and the f16 kernels.
#include "cross_device.hpp"

namespace wmdec {

template int cross_launch<f16_t>(const CrossLaunch&, int, bool, hipStream_t);

namespace {

// channels of a head that the kernels are made for
int width_of(int d) { return d <= 128 ? (d + 31) / 32 * 32 : d <= 192 ? 192 : 256; }

// Ranges of keys of a row: workgroups for every compute unit twice, of 256 keys at least.  Independent of the batch, so that the bits of a sample are.
int splits_of(int tk, int heads, long rows) {
  const long units = heads * (rows <= 32 ? 1 : (rows + 127) / 128);
  const long want = (512 + units - 1) / units, most = tk / 256;
  return (int)max(1L, min(min(want, most), (long)kCrossMaxSplits));
}

}  // namespace

size_t cross_attention_scratch_bytes(int dtype, int tk, int n, int tq, int heads, int group, int d) {
  const long rows = (long)tq * group;
  const int splits = splits_of(tk, heads, rows);
  return splits == 1 ? 0 : (size_t)splits * n * heads * rows * (width_of(d) + 2) * sizeof(float);
}

int launch_cross_attention(const CrossArgs& a, int dtype, hipStream_t s) {
  CrossLaunch p;
  p.a = a;
  p.rows = a.tq * a.group;
  p.row_blocks = 0;
  p.splits = splits_of(a.tk, a.heads, p.rows);
  const int width = width_of(a.d);
  p.part = (float*)a.scratch;
  p.ml = (float2*)(p.part + (size_t)p.splits * a.n * a.heads * p.rows * width);
  const bool few = p.rows <= 32;
  if (dtype == WMDEC_F32) return cross_launch<float>(p, width, few, s);
  return dtype == WMDEC_BF16 ? cross_launch<bf16_t>(p, width, few, s) : cross_launch<f16_t>(p, width, few, s);
}

}  // namespace wmdec
