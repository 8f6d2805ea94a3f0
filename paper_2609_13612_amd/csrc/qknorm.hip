// Norm and rotation of query and key rows at positions of one axis (qknorm_kernel.hpp).
#include "qknorm_kernel.hpp"

namespace af {

template <bool FP32, int D>
static int dispatch_rope(int what, int rope, const QkNormParams& p, hipStream_t st) {
  switch (rope) {
    case ROPE_NONE: return qknorm_launch_one<FP32, D, ROPE_NONE, false>(what, p, st);
    case ROPE_NEOX: return qknorm_launch_one<FP32, D, ROPE_NEOX, false>(what, p, st);
    case ROPE_INTERLEAVED: return qknorm_launch_one<FP32, D, ROPE_INTERLEAVED, false>(what, p, st);
  }
  return -2;
}

int launch_qknorm(int what, bool fp32, int D, int rope, const QkNormParams& p, hipStream_t st) {
  if (p.axes > 0) return launch_qknorm_axes(what, fp32, D, rope, p, st);
  if (D == 64) return fp32 ? dispatch_rope<true, 64>(what, rope, p, st) : dispatch_rope<false, 64>(what, rope, p, st);
  if (D == 128) return fp32 ? dispatch_rope<true, 128>(what, rope, p, st) : dispatch_rope<false, 128>(what, rope, p, st);
  return -2;
}

}  // namespace af
