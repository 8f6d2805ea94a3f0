// Fused forward, bf16 (fwd_kernel.hpp), under a sliding window whose first keys
// stay visible: a workgroup visits the tiles that hold sinks, then those of its
// window, four waves to a workgroup as under a window alone.  With RoPE the keys
// are rotated once into the caller's workspace first: rotating them in the loop
// is the faster form only for calls of a few microseconds.
#include "fwd_kernel.hpp"

namespace af {

template <int D, int ROPE>
static int launch_one(const FwdParams& p0, hipStream_t st) {
  FwdParams p = p0;
  if constexpr (ROPE != ROPE_NONE) {
    RopeParams r{};
    r.x0 = p.k;
    r.y0 = p.k16;
    r.heads0 = p.Hkv;
    r.B = p.B;
    r.S = p.S;
    r.table = p.table;
    const int rc = launch_rope_f16(D, ROPE, r, st);
    if (rc != 0) return rc;
  }
  const int G = p.H / p.Hkv;
  p.heads_per_wg = heads_per_wg(G) < 4 ? heads_per_wg(G) : 4;
  const int P = 128 / p.heads_per_wg;
  const long long blocks = (long long)((p.S + P - 1) / P) * p.B * p.Hkv * (G / p.heads_per_wg);
  hipLaunchKernelGGL((fwd_bf16_kernel<D, ROPE, MASK_SINKS, false, false, EXT_NONE, ROPE != ROPE_NONE, 4>),
                     dim3((unsigned)blocks), dim3(256), 0, st, p);
  return hipGetLastError() == hipSuccess ? 0 : -3;
}

template <int D>
static int dispatch_rope(int rope, const FwdParams& p, hipStream_t st) {
  switch (rope) {
    case ROPE_NONE: return launch_one<D, ROPE_NONE>(p, st);
    case ROPE_NEOX: return launch_one<D, ROPE_NEOX>(p, st);
    case ROPE_INTERLEAVED: return launch_one<D, ROPE_INTERLEAVED>(p, st);
  }
  return -2;
}

int launch_fwd_sinks(int D, int rope, const FwdParams& p, hipStream_t st) {
  if (D == 64) return dispatch_rope<64>(rope, p, st);
  if (D == 128) return dispatch_rope<128>(rope, p, st);
  return -2;
}

}  // namespace af
