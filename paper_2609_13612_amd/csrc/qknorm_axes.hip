// Norm and rotation of query and key rows at positions of several axes
// (qknorm_kernel.hpp), and the table of their angles where every axis has its own
// ladder of frequencies.
#include "qknorm_kernel.hpp"

namespace af {

// T[n][i] = (cos, sin) of n theta^(-num[i] / den[i]), in 64 bits, rounded once.
__global__ __launch_bounds__(256) void axes_table_kernel(float2* __restrict__ T, int rows, AxesRungs r, double theta) {
  const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
  if (idx >= (long long)rows * r.half) return;
  const int n = (int)(idx / r.half), i = (int)(idx % r.half);
  double s, c;
  sincos((double)n * pow(theta, -(double)r.num[i] / (double)r.den[i]), &s, &c);
  T[idx] = make_float2((float)c, (float)s);
}

int launch_axes_table(float2* table, int rows, const AxesRungs& r, double theta, hipStream_t st) {
  const long long n = (long long)rows * r.half;
  hipLaunchKernelGGL(axes_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, table, rows, r, theta);
  return hipGetLastError() == hipSuccess ? 0 : -3;
}

template <bool FP32, int D>
static int dispatch_rope(int what, int rope, const QkNormParams& p, hipStream_t st) {
  switch (rope) {
    case ROPE_NEOX: return qknorm_launch_one<FP32, D, ROPE_NEOX, true>(what, p, st);
    case ROPE_INTERLEAVED: return qknorm_launch_one<FP32, D, ROPE_INTERLEAVED, true>(what, p, st);
  }
  return -2;
}

int launch_qknorm_axes(int what, bool fp32, int D, int rope, const QkNormParams& p, hipStream_t st) {
  if (D == 64) return fp32 ? dispatch_rope<true, 64>(what, rope, p, st) : dispatch_rope<false, 64>(what, rope, p, st);
  if (D == 128) return fp32 ? dispatch_rope<true, 128>(what, rope, p, st) : dispatch_rope<false, 128>(what, rope, p, st);
  return -2;
}

}  // namespace af
