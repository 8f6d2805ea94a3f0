// Fused RoPE + masked attention backward, bf16 MFMA with fp32 accumulation,
// for gfx950.
//
// The passes of Section 4.4, no atomics: every output tile has exactly one
// writer.
//   1. bwd_pre:   partial maxima of |dO| per (batch, K/V head), and with RoPE
//                 K' = R K rotated once into the workspace (fp16): the later
//                 kernels read every K' tile many times.  Under a block mask
//                 Q' = R Q too.
//   2. bwd_dq:    one workgroup per 128 or 256 query rows (GQA heads packed, as
//                 in the forward); it loops over visible key tiles:
//                 dQ' += scale dS K',  dQ = R^T dQ'.  Before the loop it forms
//                 what else the passes need of its rows from the registers that
//                 hold them: sigma (the power of two that brings the group's
//                 largest |dO| into [1, 2)), delta_i = rowsum(dO_i * O_i), and
//                 for the dK/dV pass sigma dO and (without a block mask)
//                 Q' = R Q in fp16 in the workspace.  Since it forms P and dP for every visible key of
//                 its rows, it also sums the softmax backward's row term
//                 delta_i = sum_j P_ij dP_ij in fp32 (with P renormalised by
//                 its own row sum) and leaves it, and the renormalised LSE.
//   3. bwd_dkdv:  (bwd_dkdv.hip) one workgroup per 128 keys of one (batch,
//                 K/V head); it loops over the query heads of the GQA group
//                 and their visible query tiles, re-deriving P = exp(S - LSE)
//                 tile by tile:  dV += P^T dO,  dS = P o (dO V^T - delta),
//                 dK' += scale dS^T Q';  dK = R^T dK'.
// delta from rowsum(dO o O) equals sum_j P_ij dP_ij only for the exact O;
// the bf16 O a forward stores moves it by O's rounding, which reaches dK and
// dQ through P_ij (dP_ij - delta_i).  The dK/dV pass therefore runs last, on
// the dQ pass's sum; the dQ pass itself uses rowsum(dO o O).
//
// Scaling: the fp16 MFMA operands dO and dS carry the factor sigma, so their
// magnitudes sit near 1 whatever the gradient's scale (unscaled bf16
// gradients of 1e-6 would fall into fp16's subnormals, 6e-8 apart); the
// gradients leave multiplied by 1/sigma.  Multiplying by a power of two is
// exact, so results do not depend on the scale of dO.
// Register layouts follow the forward: the operand held in registers is the
// MFMA B operand (lane = its row), tiles staged in LDS are the A operand, and
// contractions over queries/keys read a transposed LDS copy stored with the
// perm16 row order that matches the score tile's register order.
//
// Precision: Q', K' and dS are fp16 MFMA operands.  With RoPE the rotated
// Q' and K' are the fp16 values the forward's scores came from, so P is
// re-derived from the same rounded operands that produced its LSE; without
// RoPE, Q and K are converted exactly from bf16 as they are staged.  dS in
// fp16 (2^-12 relative rounding instead of bf16's 2^-9) keeps the sums
// dK = dS^T Q and dQ = dS K accurate when attention concentrates on a few
// keys and their gradients grow.  dV = P^T dO sums P over many queries
// without normalisation, so it also runs on fp16 operands (P and sigma dO,
// the latter converted exactly from bf16).  Range: the rotated |Q'|, |K'|
// and |V| must stay below the fp16 maximum 65504, and |sigma dS| <= 4 D
// max|V| below it too, i.e. max|V| < 16376 / D (128 at D = 128).  In the dQ
// pass dP = dO V^T uses the bf16 inputs as they are.
#include "dq_kernel.hpp"

namespace af {

// ---------------------------------------------------------------- launch
namespace {
struct BwdPasses {
  template <int D, int ROPE, int MASK, bool ALIBI, int EXT>
  static int run(const BwdParams& p, hipStream_t st) {
    constexpr int RPB = 256 / (D / 16);
    const long long rows = (ROPE != ROPE_NONE) ? (long long)p.B * (p.Hkv + (p.bq_ptr ? p.H : 0)) * p.S : 0;
    const int k_blocks = (int)((rows + RPB - 1) / RPB);
    const int d_blocks = p.B * p.Hkv * p.dmax_chunks;
    hipLaunchKernelGGL((bwd_pre_kernel<D, ROPE>), dim3((unsigned)(d_blocks + k_blocks)), dim3(256), 0, st, p, d_blocks);
    const int nw = (EXT == EXT_NONE && p.bq_ptr) ? dq_waves(ROPE, true) : dq_waves(ROPE, false);
    BwdParams pq = p;
    pq.heads_per_wg = heads_per_wg(p.H / p.Hkv) < nw ? heads_per_wg(p.H / p.Hkv) : nw;
    const int P = 32 * nw / pq.heads_per_wg;
    const long long qblocks = (long long)((p.S + P - 1) / P) * p.B * p.Hkv * ((p.H / p.Hkv) / pq.heads_per_wg);
    if (EXT == EXT_NONE && p.bq_ptr)
      hipLaunchKernelGGL((bwd_dq_kernel<D, ROPE, MASK, ALIBI, true>), dim3((unsigned)qblocks), dim3(64 * nw), 0,
                         st, pq);
    else
      hipLaunchKernelGGL((bwd_dq_kernel<D, ROPE, MASK, ALIBI, false, EXT>), dim3((unsigned)qblocks),
                         dim3(64 * nw), 0, st, pq);
    if (hipGetLastError() != hipSuccess) return -3;
    // after the dQ pass, which replaced delta by sum_j P_ij dP_ij
    return launch_bwd_dkdv_bf16(D, ROPE, MASK, ALIBI, EXT, p, st);
  }
};
}  // namespace

int launch_bwd_bf16(int D, int rope, int mask, bool alibi, int ext, const BwdParams& p, hipStream_t st) {
  return bwd_dispatch<BwdPasses>(D, rope, mask, alibi, ext, p, st);
}

}  // namespace af
