// Backward under a sliding window whose first keys stay visible (sinks), bf16: the
// passes of bwd_bf16.hip, the dQ pass over the tiles with sinks and its window's,
// and between it and the dK/dV pass one more.
//
// A sink is seen by every later query, hundreds of times what another key is.  In the dK/dV pass,
// whose workgroups walk all queries of their keys, its block would run on alone
// long after the others; so that pass takes the pairs of the window only, for
// all keys alike, and this one the sinks' pairs past it,
//   (i, j) with j < sinks and i - j >= window:   dV_j += P_ij dO_i,  dK'_j += dS_ij Q'_i,
// split over the queries: the workgroups of 32 sinks share their (query head,
// query tile) steps and leave fp32 partial sums.  The dK/dV pass sums them in their
// order (no atomics) and starts from them, or, where it is split itself, its reduction
// adds them to its own; dK and dV are rotated and rounded once, after that.
//
// Without RoPE K and Q go through the workspace in fp16 too (ROPE_F16), so that the
// passes copy their tiles straight to LDS in workgroups of four waves: converted as
// they were staged, by eight, B4 H12 S2001 D64 window 256 took the dQ pass 61 us
// against 46.
#include "dq_kernel.hpp"

namespace af {

template <int D>
struct FarCfg {
  static constexpr int NW = 4;
  static constexpr int KS = D / 16, MT = D / 32;
  static constexpr int KP = D + 8;                       // pitch of the resident K' and V rows (16-byte reads)
  static constexpr int TILE = 32 * D;                    // a wave's own 32 query rows, swizzled
  static constexpr int IPT = 32 * (D / 8) / 64;          // 16-byte chunks of a tile per lane
  static constexpr int TILES = NW * 2 * TILE;            // Q' and dO of each wave
  static constexpr int SMEM = TILES + 2 * 32 * KP;
  static_assert(SMEM * 2 >= NW * MT * 16 * 64 * 4, "the waves' sums go through the same memory");
};

// Workgroup = 4 waves, one part of the steps of 32 sinks of one (batch, K/V
// head).  A wave takes every fourth 32-row query tile of its part, through its
// own LDS: no barriers; the next tile is on its way, in registers, while one is
// worked on.  K' and V rows (fp16) are shared.  Bound by reading Q' and dO, which the
// dQ pass has just written: B1 H32/8 S8192 D128 window 1024, 4 sinks 33 us, 117 MB at
// 3.6 TB/s; small calls by their chain, load -> products -> sums of the waves (B4 H12
// S2001 D64 window 256, 4 sinks 10.4 us, of 21 MB).
template <int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 2 : 1, D == 64 ? 2 : 1)))
void bwd_far_kernel(BwdParams p) {
  using C = FarCfg<D>;
  __shared__ __attribute__((aligned(16))) uint16_t smem[C::SMEM];
  __shared__ __attribute__((aligned(16))) float stat[C::NW][2][32];   // the tile's LSE (log2 units) and delta
  const int tid = threadIdx.x, lane = tid & 63, lq = lane & 31, lg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int S = p.S, W = p.window, G = p.H / p.Hkv;
  const int nfb = (p.sinks + 31) / 32;
  const int part = (int)(blockIdx.x % p.far_parts), rest = (int)(blockIdx.x / p.far_parts);
  const int fb = rest % nfb, bg = rest / nfb;
  const int b = bg / p.Hkv, g = bg % p.Hkv;
  const int nw = 32 * fb, n = nw + lq;       // the block's first key, this lane's key

  f32x16 dk[C::MT], dv[C::MT];
#pragma unroll
  for (int i = 0; i < C::MT; ++i) { dk[i] = f32x16{}; dv[i] = f32x16{}; }
  const float c2 = p.scale * kLog2e;
  const int tq = (nw + W) / 32, nq = (S + 31) / 32 - tq;   // query tiles from the first that sees key nw past its window
  const long long steps = (long long)G * nq;
  const int s_begin = (int)(steps * part / p.far_parts), s_end = (int)(steps * (part + 1) / p.far_parts);

  uint16_t* Qs = smem + wave * 2 * C::TILE;
  uint16_t* Os = Qs + C::TILE;
  float (*st)[32] = stat[wave];
  const SwzLane<D> z(lane);
  u32x4 qt[C::IPT], ot[C::IPT];   // the tile in flight
  float stat_t;
  auto load = [&](int s) {
    const size_t bh = (size_t)b * p.H + g * G + s / nq;
    const int mq = 32 * (tq + s % nq);
    const uint16_t* Q = static_cast<const uint16_t*>(p.qr16) + bh * S * D;
    const uint16_t* dO = static_cast<const uint16_t*>(p.do16) + bh * S * D;
#pragma unroll
    for (int i = 0; i < C::IPT; ++i) {
      const int it = lane + 64 * i;
      const size_t off = (size_t)min(mq + it / (D / 8), S - 1) * D + 8 * (it % (D / 8));
      qt[i] = ld16(Q + off);
      ot[i] = ld16(dO + off);
    }
    stat_t = (lg ? p.delta : p.lse2)[bh * S + min(mq + lq, S - 1)];
  };
  if (s_begin + wave < s_end) load(s_begin + wave);

  uint16_t* Ks = smem + C::TILES;
  uint16_t* Vs = Ks + 32 * C::KP;
  const uint16_t* Kg = static_cast<const uint16_t*>(p.kr16) + (size_t)bg * S * D;
  const uint16_t* Vg = static_cast<const uint16_t*>(p.v) + (size_t)bg * S * D;
  for (int it = tid; it < 32 * (D / 8); it += 256) {
    const int r = it / (D / 8), c = it % (D / 8);
    const size_t off = (size_t)min(nw + r, S - 1) * D + 8 * c;
    u32x4 v = ld16(Vg + off), k = ld16(Kg + off);
#pragma unroll
    for (int w = 0; w < 4; ++w) v[w] = pack_f16(bf_lo(v[w]), bf_hi(v[w]));
    *reinterpret_cast<u32x4*>(Vs + r * C::KP + 8 * c) = v;
    *reinterpret_cast<u32x4*>(Ks + r * C::KP + 8 * c) = k;
  }
  __syncthreads();

  for (int s = s_begin + wave; s < s_end; s += C::NW) {
    const int mq = 32 * (tq + s % nq);
#pragma unroll
    for (int i = 0; i < C::IPT; ++i) {   // (this wave's earlier reads are done: LDS is in order per wave)
      const int it = lane + 64 * i, at = swz_at<D>(it / (D / 8), 8 * (it % (D / 8)));
      *reinterpret_cast<u32x4*>(Qs + at) = qt[i];
      *reinterpret_cast<u32x4*>(Os + at) = ot[i];
    }
    st[lg][lq] = stat_t;
    if (s + C::NW < s_end) load(s + C::NW);
    f32x16 sc = f32x16{}, dp = f32x16{};
#pragma unroll
    for (int k = 0; k < C::KS; ++k) {
      const u32x4 bk = *reinterpret_cast<const u32x4*>(Ks + lq * C::KP + 16 * k + 8 * lg);
      const u32x4 bv = *reinterpret_cast<const u32x4*>(Vs + lq * C::KP + 16 * k + 8 * lg);
      sc = mfma32<true>(row_operand_swz<D>(Qs, z, 0, k), bk, sc);
      dp = mfma32<true>(row_operand_swz<D>(Os, z, 0, k), bv, dp);
    }
    // element r: query mq + 8 (r/4) + 4 lg + r%4, key n
    u32x4 pb[2], db[2];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const float4 l4 = *reinterpret_cast<const float4*>(&st[0][8 * a + 4 * lg]);
      const float4 d4 = *reinterpret_cast<const float4*>(&st[1][8 * a + 4 * lg]);
      const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
      float pr[4], ds[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = mq + 8 * a + 4 * lg + e;
        const bool ok = n < p.sinks && m - n >= W && m < S;
        pr[e] = ok ? fast_exp2(sc[4 * a + e] * c2 - lv[e]) : 0.f;
        ds[e] = ok ? (dp[4 * a + e] - dl[e]) * pr[e] : 0.f;
      }
      pb[a >> 1][2 * (a & 1)] = pack_f16(pr[0], pr[1]);
      pb[a >> 1][2 * (a & 1) + 1] = pack_f16(pr[2], pr[3]);
      db[a >> 1][2 * (a & 1)] = pack_f16(ds[0], ds[1]);
      db[a >> 1][2 * (a & 1) + 1] = pack_f16(ds[2], ds[3]);
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int mt = 0; mt < C::MT; ++mt) {
        dv[mt] = mfma32<true>(tr_operand_swz<D>(Os, z, 16 * hf, mt), pb[hf], dv[mt]);
        dk[mt] = mfma32<true>(tr_operand_swz<D>(Qs, z, 16 * hf, mt), db[hf], dk[mt]);
      }
  }

  // Sum the waves, 32 dims of dK' and dV each; [wave][tile][element][lane] in the tiles'
  // memory.  Rows past the sinks are neither written here nor read.
  float* xch = reinterpret_cast<float*>(smem) + lane;
  float* dst = p.far + (((size_t)bg * nfb + fb) * p.far_parts + part) * 2 * 32 * D + lq * D + 4 * lg;
#pragma unroll
  for (int what = 0; what < 2; ++what) {
    __syncthreads();   // every wave is past its tiles, or past the sums of dK'
    if (n < p.sinks) {
#pragma unroll
      for (int mt = 0; mt < C::MT; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r) xch[((wave * C::MT + mt) * 16 + r) * 64] = what ? dv[mt][r] : dk[mt][r];
    }
    __syncthreads();
    if (wave < C::MT && n < p.sinks) {
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        float4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < C::NW; ++w) {
          const float* y = xch + ((w * C::MT + wave) * 16 + 4 * a) * 64;
          x.x += y[0];
          x.y += y[64];
          x.z += y[128];
          x.w += y[192];
        }
        *reinterpret_cast<float4*>(dst + what * 32 * D + 32 * wave + 8 * a) = x;
      }
    }
  }
}

// ---------------------------------------------------------------- launch
template <int D, int ROPE>
static int launch_one(const BwdParams& p, hipStream_t st) {
  constexpr int RPB = 256 / (D / 16);
  const long long rows = (long long)p.B * p.Hkv * p.S;
  const int d_blocks = p.B * p.Hkv * p.dmax_chunks;
  hipLaunchKernelGGL((bwd_pre_kernel<D, ROPE>), dim3((unsigned)(d_blocks + (rows + RPB - 1) / RPB)), dim3(256), 0, st, p,
                     d_blocks);
  constexpr int NW = dq_waves(ROPE, false);
  const int G = p.H / p.Hkv;
  BwdParams pq = p;
  pq.heads_per_wg = heads_per_wg(G) < NW ? heads_per_wg(G) : NW;
  const int P = 32 * NW / pq.heads_per_wg;
  const long long qblocks = (long long)((p.S + P - 1) / P) * p.B * p.Hkv * (G / pq.heads_per_wg);
  hipLaunchKernelGGL((bwd_dq_kernel<D, ROPE, MASK_SINKS, false, false, EXT_NONE>), dim3((unsigned)qblocks), dim3(64 * NW),
                     0, st, pq);
  const long long far = (long long)p.B * p.Hkv * ((p.sinks + 31) / 32) * p.far_parts;
  hipLaunchKernelGGL((bwd_far_kernel<D>), dim3((unsigned)far), dim3(256), 0, st, p);
  if (hipGetLastError() != hipSuccess) return -3;
  return launch_bwd_dkdv_sinks(D, ROPE, p, st);
}

template <int D>
static int dispatch_rope(int rope, const BwdParams& p, hipStream_t st) {
  switch (rope) {
    case ROPE_NONE: return launch_one<D, ROPE_F16>(p, st);
    case ROPE_NEOX: return launch_one<D, ROPE_NEOX>(p, st);
    case ROPE_INTERLEAVED: return launch_one<D, ROPE_INTERLEAVED>(p, st);
  }
  return -2;
}

int launch_bwd_sinks(int D, int rope, const BwdParams& p, hipStream_t st) {
  if (D == 64) return dispatch_rope<64>(rope, p, st);
  if (D == 128) return dispatch_rope<128>(rope, p, st);
  return -2;
}

}  // namespace af
