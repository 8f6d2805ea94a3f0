// dK/dV pass under a window with sinks (dkdv_kernel.hpp): the window's pairs.  The key
// blocks that hold sinks start from what bwd_sinks.hip summed; with splits the
// reduction (bwd_dkdv_split.hip) adds it.
#include "dkdv_kernel.hpp"

namespace af {

template <int D, int ROPE>
static int launch_one(const BwdParams& p, hipStream_t st) {
  using QC = QTileCfg<D>;
  const long long blocks = (long long)((p.S + QC::KEYS - 1) / QC::KEYS) * p.B * p.Hkv * p.splits;
  if (p.splits > 1)
    hipLaunchKernelGGL((bwd_dkdv_kernel<D, ROPE, MASK_SINKS, false, false, EXT_NONE, true>), dim3((unsigned)blocks),
                       dim3(QC::THREADS), 0, st, p);
  else
    hipLaunchKernelGGL((bwd_dkdv_kernel<D, ROPE, MASK_SINKS, false, false, EXT_NONE, false>), dim3((unsigned)blocks),
                       dim3(QC::THREADS), 0, st, p);
  if (hipGetLastError() != hipSuccess) return -3;
  return p.splits > 1 ? launch_bwd_dkdv_reduce(D, ROPE, p, st) : 0;
}

template <int D>
static int dispatch_rope(int rope, const BwdParams& p, hipStream_t st) {
  switch (rope) {
    case ROPE_F16: return launch_one<D, ROPE_F16>(p, st);
    case ROPE_NEOX: return launch_one<D, ROPE_NEOX>(p, st);
    case ROPE_INTERLEAVED: return launch_one<D, ROPE_INTERLEAVED>(p, st);
  }
  return -2;
}

int launch_bwd_dkdv_sinks(int D, int rope, const BwdParams& p, hipStream_t st) {
  if (D == 64) return dispatch_rope<64>(rope, p, st);
  if (D == 128) return dispatch_rope<128>(rope, p, st);
  return -2;
}

}  // namespace af
