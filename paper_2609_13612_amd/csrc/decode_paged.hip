// Decode attention over a paged key/value cache, or a contiguous one under a
// sliding window whose first tokens stay visible; bf16, fp32 accumulation.
//
// One query per sequence: with L cached keys it sits at position L - 1 and sees
// the keys n < L of its window, n >= L - window, and the sinks, n < sinks.  Each
// K and V element is used once per query head of its group, so the kernel is
// bound by reading the visible part of the cache once.
//
// The visible 32-key tiles of a sequence are numbered from 0: first the tiles
// that hold sinks, then those of the window.  Workgroup = 4 waves = one of nsplit
// shares of those tiles for one (sequence, K/V head, up to 32 query heads): wave w of
// share s takes tiles 4 s + w, 4 (s + nsplit) + w, ..., so shares are even whatever
// the length, the first tile's page is looked up before the length is known, and a
// sequence's result depends, at a given nsplit, on its own length alone.  (nsplit comes
// from the batch and the most keys a sequence may have.)  The four waves' (max, sum, O)
// are joined through LDS and leave as one partial per workgroup, or as the result
// where a sequence is one workgroup's; a second kernel joins the partials.
//
// A tile is two units of 16 keys.  Pages hold a multiple of 16, so a unit lies in
// one page and its address is wave-uniform: the page numbers are scalar loads,
// two a tile, one tile ahead of the keys.
//
// Products: S^T = K Q'^T (32 keys x 32 columns, the group's heads repeated), K
// straight from memory into registers as the A operand; O^T += V^T P^T, V
// through the wave's own LDS tile for the transposed read.  Without RoPE the
// bf16 query and keys meet exactly.  With it the query, rotated in fp32, is
// split into two bf16 values, q = hi + lo to 2^-16 of itself, and meets the
// cached keys in two products: the matrix units are idle nine tenths of the
// time, and neither range nor the LSE suffers from a 16-bit query.  P is rounded to
// bf16 (2^-8 of each weight at most, as the bf16 O is); sums, maxima and O stay
// fp32 to the end.
//
// Measured (K and V bytes of the visible keys over the whole time, D 128, H 32 of 8):
// 32 sequences of 8192 keys 187 us, 5.7 TB/s; the same with lengths from 2048 to 8192
// 131 us; one sequence of 4096 keys 8.7 us in a replayed graph and one of 16 keys 5.0,
// of which a launch is 1.7: there the chain length and page -> K and V -> products ->
// join -> second kernel is what lasts.
#include "common.hpp"
#include "launch.hpp"

namespace af {

template <int D>
struct PagedCfg {
  static constexpr int NW = 4;
  static constexpr int KS = D / 16;               // MFMA k-steps over the head dimension
  static constexpr int MT = D / 32;               // 32-row output tiles over the head dimension
  static constexpr int VP = D + 16;               // V tile pitch (transpose reads)
  static constexpr int QP = D + 8;                // pitch of the rotated heads' rows (16-byte reads)
  static constexpr int VT = 32 * VP;              // one wave's V tile (elements)
  static constexpr int VPL = 32 * (D / 8) / 64;   // 16-byte V chunks per lane per tile
  static_assert(VT * 2 >= MT * 4 * 32 * 16, "16 columns of a wave's O go through its V tile's memory");
};

// The bits below bit n.
__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }

// The visible tiles of a sequence with L keys: tiles [0, ns), then [t0, t0 + n - ns).
struct Visible {
  int L, lo, sinks, ns, t0, n;
  __device__ __forceinline__ Visible(const PagedParams& p, int len) {
    L = max(min(len, p.S), 0);
    lo = p.window > 0 ? max(0, L - p.window) : 0;
    sinks = min(p.sinks, lo);                     // (those still in the window are the window's)
    t0 = lo >> 5;
    ns = min((sinks + 31) >> 5, t0);
    n = ns + ((L + 31) >> 5) - t0;
  }
  __device__ __forceinline__ int tile(int i) const { return i < ns ? i : t0 + i - ns; }
};

// The sequence with the r-th most cached keys (the lower index first), of up to 64:
// where workgroups wait for others to end, the longest start first and the short ones
// fill the end.  One length a lane, ranked by counting the larger ones.
__device__ __forceinline__ int nth_longest(const PagedParams& p, int r, int lane) {
  const int key = lane < p.B ? max(min(p.lens[lane], p.S), 0) * 64 + (63 - lane) : -1;   // (S <= 2^20)
  int above = 0;
  for (int j = 0; j < p.B; ++j) above += __builtin_amdgcn_readlane(key, j) > key;
  return __ffsll((long long)__ballot(key >= 0 && above == r)) - 1;
}

// What a partial with maximum m counts in a sum of maximum M.  Scores that are all NaN
// leave m at -inf, as no visible key does, and NaN in the sums: those are added, times
// 0, and stay NaN.
__device__ __forceinline__ float part_weight(float m, float M) { return m == -INFINITY ? 0.f : fast_exp2(m - M); }

// Fold the (max, sum) pair (m2, l2) into (m, l).
__device__ __forceinline__ void merge_stats(float& m, float& l, float m2, float l2) {
  const float M = fmaxf(m, m2);
  l = l * part_weight(m, M) + l2 * part_weight(m2, M);
  m = M;
}

template <int D, int ROPE, bool ALIBI, bool PAGED>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void paged_split_kernel(PagedParams p) {
  using C = PagedCfg<D>;
  constexpr int NQ = ROPE == ROPE_NONE ? 1 : 2;   // bf16 parts of the query
  __shared__ __attribute__((aligned(16))) uint16_t smem[C::NW * C::VT];
  __shared__ float xml[2][C::NW][32];             // the waves' max and sum per column
  __shared__ __attribute__((aligned(16))) uint16_t qs[ROPE == ROPE_NONE ? 8 : NQ * 32 * C::QP];   // the rotated heads

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 31, lg = lane >> 5;
  const int split = blockIdx.x;
  const int b = p.by_length ? __builtin_amdgcn_readfirstlane(nth_longest(p, blockIdx.z, lane)) : (int)blockIdx.z;
  int g = blockIdx.y, hg = 0;
  if (p.hgroups > 1) {
    hg = g % p.hgroups;
    g /= p.hgroups;
  }
  const int G = p.G, h0 = hg * 32, nh = min(32, G - h0);   // this workgroup's heads of the group
  const int h = g * G + h0 + lq % nh;             // head of this lane's column
  const float c2 = p.scale * kLog2e;
  const float slope2 = ALIBI ? p.slopes[h] * kLog2e : 0.f;
  const uint16_t* __restrict__ K = static_cast<const uint16_t*>(p.k) + g * p.ks[1];
  const uint16_t* __restrict__ V = static_cast<const uint16_t*>(p.v) + g * p.vs[1];
  const int* __restrict__ table = PAGED ? p.table + (size_t)b * p.max_pages : nullptr;

  uint16_t* Vw = smem + wave * C::VT;
  const int tr_key = 4 * lg + ((lane & 15) >> 2);
  const int tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);

  f32x16 acc[C::MT];
#pragma unroll
  for (int i = 0; i < C::MT; ++i) acc[i] = f32x16{};
  float m_run = -INFINITY, l_run = 0.f;

  // The page of each unit of a tile (-1: none there, its keys are not visible).
  auto pages_of = [&](int n0, int (&pg)[2]) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (PAGED) {
        const int e = uniform_load(table + min((n0 + 16 * u) >> p.page_shift, p.max_pages - 1));
        pg[u] = (unsigned)e < (unsigned)p.num_pages ? e : -1;
      } else {
        pg[u] = b;
      }
    }
  };
  int pg[2] = {-1, -1}, pn[2] = {-1, -1};         // pages of the tile in flight, of the one after it
  int i = C::NW * split + wave;                   // this wave's tile
  const int step = C::NW * p.nsplit;
  const bool early = PAGED && p.window <= 0;      // its place does not depend on the length
  if (early) pages_of(32 * i, pg);
  // Query operand (B of S^T = K Q'^T): lane holds column lq's head, dims 16s + 8lg .. +7.
  // With RoPE the workgroup rotates its heads once, a thread two pairs of a head (words
  // qa and qb of the row), and hands them out through LDS.
  u32x4 qreg[NQ][C::KS];
  const uint32_t* qrows = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p.q) +
                                                            ((size_t)b * p.H + g * G + h0) * D);
  auto word_a = [&](int j) { return (j / (D / 4)) * (D / 2) + (ROPE == ROPE_NEOX ? j % (D / 4) : 2 * (j % (D / 4))); };
  auto word_b = [&](int j) { return word_a(j) + (ROPE == ROPE_NEOX ? D / 4 : 1); };
  const int items = nh * (D / 4);
  uint32_t qa = 0, qb = 0;
  if constexpr (ROPE == ROPE_NONE) {
    const uint16_t* Qh = reinterpret_cast<const uint16_t*>(qrows) + (lq % nh) * D;
#pragma unroll
    for (int s = 0; s < C::KS; ++s) qreg[0][s] = ld16(Qh + 16 * s + 8 * lg);
  } else {
    qa = qrows[word_a(min(tid, items - 1))];
    qb = qrows[word_b(min(tid, items - 1))];
  }
  const int len = p.lens ? uniform_load(p.lens + b) : p.S;
  const Visible vis(p, len);
  const int n_tiles = vis.n;
  if (C::NW * split >= n_tiles) {                 // (workgroup-uniform)
    if (p.nsplit == 1) {                          // an empty sequence: nothing else writes its rows
      for (int j = tid; j < nh * (D / 8); j += 256)
        st16(static_cast<uint16_t*>(p.o) + ((size_t)b * p.H + g * G + h0) * D + 8 * j, u32x4{0, 0, 0, 0});
      if (tid < nh) p.lse[(size_t)b * p.H + g * G + h0 + tid] = -INFINITY;
    }
    return;
  }
  const int L = vis.L, pos = L - 1;

  u32x4 kreg[C::KS], vreg[C::VPL];
  // Rows that are not there (no page; past a contiguous cache) read another
  // row's finite memory: page 0, or the last row.  Their keys are masked and
  // their V rows cleared before use.
  auto load_tile = [&](int n0, const int (&pg)[2]) {
    const uint16_t* kb[2];
    const uint16_t* vb[2];
    int last[2];                                  // last row of the unit that may be read
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int n = n0 + 16 * u;
      long long place;
      if constexpr (PAGED) {
        place = n & ((1 << p.page_shift) - 1);
        last[u] = 15;
      } else {
        place = min(n, p.S - 1);
        last[u] = max(0, min(15, p.S - 1 - n));
      }
      const long long page = max(pg[u], 0);
      kb[u] = K + page * p.ks[0] + place * p.ks[2];
      vb[u] = V + page * p.vs[0] + place * p.vs[2];
    }
    const int u = lq >> 4, r = min(lq & 15, u ? last[1] : last[0]);
    const uint16_t* krow = (u ? kb[1] : kb[0]) + (long long)r * p.ks[2] + 8 * lg;
#pragma unroll
    for (int s = 0; s < C::KS; ++s) kreg[s] = ld16(krow + 16 * s);
#pragma unroll
    for (int i = 0; i < C::VPL; ++i) {
      constexpr int RPI = 512 / D;                // rows an instruction reads
      const int vu = (i * RPI) >> 4;              // (an instruction stays inside a unit)
      const int vr = min((i * RPI & 15) + lane / (D / 8), last[vu]);
      vreg[i] = ld16(vb[vu] + (long long)vr * p.vs[2] + 8 * (lane % (D / 8)));
    }
  };

  [[maybe_unused]] float4 cs;                     // cos and sin of a thread's pairs, ahead of the tile's loads
  [[maybe_unused]] const float2* angles = p.rope + (size_t)pos * (D / 2);
  if constexpr (ROPE != ROPE_NONE) cs = *reinterpret_cast<const float4*>(angles + 2 * (tid % (D / 4)));
  if (i < n_tiles) {
    if (!early) pages_of(32 * vis.tile(i), pg);
    load_tile(32 * vis.tile(i), pg);
    if (i + step < n_tiles) pages_of(32 * vis.tile(i + step), pn);
  }

  if constexpr (ROPE != ROPE_NONE) {
    for (int j = tid; j < items; j += 256) {      // (256 is a multiple of D / 4: the same pairs of other heads)
      if (j != tid) {
        qa = qrows[word_a(j)];
        qb = qrows[word_b(j)];
      }
      float x[4] = {bf_lo(qa), bf_hi(qa), bf_lo(qb), bf_hi(qb)};
      if constexpr (ROPE == ROPE_NEOX) {
        rotate_pair<false>(x[0], x[2], cs.x, cs.y);
        rotate_pair<false>(x[1], x[3], cs.z, cs.w);
      } else {
        rotate_pair<false>(x[0], x[1], cs.x, cs.y);
        rotate_pair<false>(x[2], x[3], cs.z, cs.w);
      }
      const uint32_t ha = pack_bf16(x[0], x[1]), hb = pack_bf16(x[2], x[3]);
      const int head = j / (D / 4), a = word_a(j) - head * (D / 2), w = word_b(j) - head * (D / 2);
      uint32_t* row = reinterpret_cast<uint32_t*>(qs) + head * (C::QP / 2);
      row[a] = ha;
      row[w] = hb;
      row += 32 * C::QP / 2;
      row[a] = pack_bf16(x[0] - bf_lo(ha), x[1] - bf_hi(ha));
      row[w] = pack_bf16(x[2] - bf_lo(hb), x[3] - bf_hi(hb));
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int s = 0; s < C::KS; ++s)
        qreg[q][s] = *reinterpret_cast<const u32x4*>(qs + (32 * q + lq % nh) * C::QP + 16 * s + 8 * lg);
  }

  for (; i < n_tiles; i += step) {
    const int n0 = 32 * vis.tile(i);
    // some key of the tile is not visible: past the end, before the window, or without a page
    const bool edge = n0 + 32 > L || (n0 < vis.lo && n0 + 32 > vis.sinks) || pg[0] < 0 || pg[1] < 0;   // (wave-uniform)
    // Bit k: key n0 + k is visible.  (One wave-uniform mask for V's rows and for S; a test
    // of each key held registers that the loads in flight want: 8192 keys of 32 sequences,
    // H 32 of 8, D 128, all in 194 us against 187.)
    uint32_t seen = ~0u;
    if (edge) {
      seen = below(L - n0) & (~below(vis.lo - n0) | below(vis.sinks - n0));
      if (pg[0] < 0) seen &= 0xffff0000u;
      if (pg[1] < 0) seen &= 0x0000ffffu;
      // what lies in rows that are not visible may be anything: 0 x NaN is NaN
#pragma unroll
      for (int k = 0; k < C::VPL; ++k)
        if (!(seen >> (k * (512 / D) + lane / (D / 8)) & 1)) vreg[k] = u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int k = 0; k < C::VPL; ++k)   // (this wave's earlier transpose reads are done: LDS is in order per wave)
      *reinterpret_cast<u32x4*>(Vw + (k * (512 / D) + lane / (D / 8)) * C::VP + 8 * (lane % (D / 8))) = vreg[k];
    f32x16 st = f32x16{};
#pragma unroll
    for (int s = 0; s < C::KS; ++s)
#pragma unroll
      for (int q = 0; q < NQ; ++q) st = mfma32(kreg[s], qreg[q][s], st);
    if (i + step < n_tiles) {
      pg[0] = pn[0];
      pg[1] = pn[1];
      load_tile(32 * vis.tile(i + step), pg);
      if (i + 2 * step < n_tiles) pages_of(32 * vis.tile(i + 2 * step), pn);
    }

    // element r: key n0 + 8 (r/4) + 4 lg + r%4 of column lq
    if constexpr (ALIBI) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        st[r] = __builtin_fmaf(st[r], c2, slope2 * (float)(n0 + 8 * (r >> 2) + 4 * lg + (r & 3) - pos));
    }
    if (edge) {
#pragma unroll
      for (int r = 0; r < 16; ++r) st[r] = seen >> (4 * lg) >> (8 * (r >> 2) + (r & 3)) & 1 ? st[r] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[r]);
    mx = pair_max(mx);
    if constexpr (!ALIBI) mx *= c2;
    const float m_new = fmaxf(m_run, mx);
    if (__any(m_new > m_run + 8.f)) {   // raise the reference max (wave-uniform)
      const float alpha = (m_run == -INFINITY) ? 0.f : fast_exp2(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int k = 0; k < C::MT; ++k) acc[k] *= alpha;
      m_run = m_new;
    }
    const float m_use = (m_run == -INFINITY) ? 0.f : m_run;
    float pv[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      pv[r] = fast_exp2(ALIBI ? (st[r] - m_use) : __builtin_fmaf(st[r], c2, -m_use));
      l_run += pv[r];
    }
    u32x4 pop[2];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int w = 0; w < 4; ++w) pop[hf][w] = pack_bf16(pv[8 * hf + 2 * w], pv[8 * hf + 2 * w + 1]);
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int mt = 0; mt < C::MT; ++mt) {
        const uint16_t* base = Vw + (16 * hf + tr_key) * C::VP + 32 * mt + tr_col;
        const u32x2 lo2 = lds_read_tr16(base);
        const u32x2 hi2 = lds_read_tr16(base + 8 * C::VP);
        acc[mt] = mfma32(u32x4{lo2[0], lo2[1], hi2[0], hi2[1]}, pop[hf], acc[mt]);
      }
  }

  // Join the waves, 16 columns at a time: each leaves its O of those columns, as 16-byte
  // pieces [32-dim tile][piece][lane], in the memory of its own V tile, which no other
  // wave reads; then wave w sums dims 32 w .. of all four, each weighted by 2^(its max
  // - the common one).  (Sums of whole tiles over 48 KB of LDS, scaled before, took two
  // barriers: 16 keys of one sequence 5.8 us against 5.5.)
  const float l_tot = pair_sum(l_run);
  if (lg == 0) {
    xml[0][wave][lq] = m_run;
    xml[1][wave][lq] = l_tot;
  }
  const size_t bh = (size_t)b * p.H + h;
  for (int c0 = 0; c0 < nh; c0 += 16) {           // (one round for up to 16 heads of a group)
    const bool mine = lq >= c0 && lq < c0 + 16;
    const int at = 16 * lg + lq - c0;             // of 32 lanes
    if (c0 > 0) __syncthreads();                  // the round before has been read
    if (mine) {
      float4* own = reinterpret_cast<float4*>(Vw);
#pragma unroll
      for (int mt = 0; mt < C::MT; ++mt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          own[(4 * mt + q) * 32 + at] = float4{acc[mt][4 * q], acc[mt][4 * q + 1], acc[mt][4 * q + 2], acc[mt][4 * q + 3]};
    }
    __syncthreads();
    if (wave >= C::MT || !mine || lq >= nh) continue;
    float M = -INFINITY, l = 0.f;
    float4 o[4] = {};
#pragma unroll
    for (int w = 0; w < C::NW; ++w) M = fmaxf(M, xml[0][w][lq]);
#pragma unroll
    for (int w = 0; w < C::NW; ++w) {
      const float a = part_weight(xml[0][w][lq], M);
      l = __builtin_fmaf(xml[1][w][lq], a, l);
      const float4* from = reinterpret_cast<const float4*>(smem + w * C::VT);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float4 x = from[(4 * wave + q) * 32 + at];
        o[q].x = __builtin_fmaf(x.x, a, o[q].x);
        o[q].y = __builtin_fmaf(x.y, a, o[q].y);
        o[q].z = __builtin_fmaf(x.z, a, o[q].z);
        o[q].w = __builtin_fmaf(x.w, a, o[q].w);
      }
    }
    if (p.nsplit == 1) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      uint16_t* O = static_cast<uint16_t*>(p.o) + bh * D + 32 * wave + 4 * lg;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<u32x2*>(O + 8 * q) =
            u32x2{pack_bf16(o[q].x * inv, o[q].y * inv), pack_bf16(o[q].z * inv, o[q].w * inv)};
      if (wave == 0 && lg == 0) p.lse[bh] = l == 0.f ? -INFINITY : (M + __log2f(l)) * kLn2;
    } else {
      float* dst = p.part_acc + (bh * p.nsplit + split) * D + 32 * wave + 4 * lg;
#pragma unroll
      for (int q = 0; q < 4; ++q) *reinterpret_cast<float4*>(dst + 8 * q) = o[q];
      if (wave == 0 && lg == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * (bh * p.nsplit + split)) = float2{M, l};
    }
  }
}

// Join the partials of one (sequence, query head), none of an empty sequence: D /
// 4 lanes hold the dims, the groups of lanes take every NG-th partial.  The first
// PF of a group and the statistics are on their way before the length, which says
// how many there are, is known: one round trip to memory where they are all.
template <int D, int PF>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedParams p) {
  constexpr int LPR = D / 4, NG = 256 / LPR;
  __shared__ float4 red[NG][LPR];
  __shared__ float wml[2][4];
  const int t = threadIdx.x, c = t % LPR, grp = t / LPR;
  const int b = blockIdx.y;
  const size_t bh = (size_t)b * p.H + blockIdx.x;
  const float* ml = p.part_ml + 2 * bh * p.nsplit;
  const float* acc = p.part_acc + bh * p.nsplit * D + 4 * c;
  float4 x[PF];
  float mx[PF];
#pragma unroll
  for (int j = 0; j < PF; ++j) {
    const int i = min(grp + NG * j, p.nsplit - 1);
    x[j] = *reinterpret_cast<const float4*>(acc + (size_t)i * D);
    mx[j] = ml[2 * i];
  }
  float2 own = *reinterpret_cast<const float2*>(ml + 2 * min(t, p.nsplit - 1));
  const Visible vis(p, p.lens ? uniform_load(p.lens + b) : p.S);
  const int n = min(p.nsplit, (vis.n + 3) / 4);   // partials: the shares that have tiles
  float m = -INFINITY, l = 0.f;
  if (t < n) {
    m = own.x;
    l = own.y;
  }
  for (int i = t + 256; i < n; i += 256) {
    const float2 v = *reinterpret_cast<const float2*>(ml + 2 * i);
    merge_stats(m, l, v.x, v.y);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) merge_stats(m, l, __shfl_xor(m, o), __shfl_xor(l, o));
  if ((t & 63) == 0) {
    wml[0][t >> 6] = m;
    wml[1][t >> 6] = l;
  }
  __syncthreads();
  float M = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) M = fmaxf(M, wml[0][w]);
#pragma unroll
  for (int w = 0; w < 4; ++w) l = __builtin_fmaf(wml[1][w], part_weight(wml[0][w], M), l);
  float4 sum = {0.f, 0.f, 0.f, 0.f};
  auto fold = [&](float mi, const float4& y) {
    const float w = part_weight(mi, M);
    sum.x = __builtin_fmaf(w, y.x, sum.x);
    sum.y = __builtin_fmaf(w, y.y, sum.y);
    sum.z = __builtin_fmaf(w, y.z, sum.z);
    sum.w = __builtin_fmaf(w, y.w, sum.w);
  };
#pragma unroll
  for (int j = 0; j < PF; ++j)
    if (grp + NG * j < n) fold(mx[j], x[j]);
  for (int i = grp + NG * PF; i < n; i += NG) fold(ml[2 * i], *reinterpret_cast<const float4*>(acc + (size_t)i * D));
  red[grp][c] = sum;
  __syncthreads();
  if (grp == 0) {
#pragma unroll
    for (int i = 1; i < NG; ++i) {
      const float4 y = red[i][c];
      sum.x += y.x;
      sum.y += y.y;
      sum.z += y.z;
      sum.w += y.w;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.o) + bh * D + 4 * c) =
        u32x2{pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv)};
    if (t == 0) p.lse[bh] = l == 0.f ? -INFINITY : (M + __log2f(l)) * kLn2;
  }
}

// ---------------------------------------------------------------- launch
template <int D, int ROPE, bool ALIBI>
static int launch_one(const PagedParams& p, hipStream_t st) {
  const dim3 grid((unsigned)p.nsplit, (unsigned)(p.Hkv * p.hgroups), (unsigned)p.B);
  if (p.table) hipLaunchKernelGGL((paged_split_kernel<D, ROPE, ALIBI, true>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((paged_split_kernel<D, ROPE, ALIBI, false>), grid, dim3(256), 0, st, p);
  if (p.nsplit > 1) hipLaunchKernelGGL((paged_join_kernel<D, 4>), dim3((unsigned)p.H, (unsigned)p.B), dim3(256), 0, st, p);
  return hipGetLastError() == hipSuccess ? 0 : -3;
}

template <int D>
static int dispatch_rope(int rope, bool alibi, const PagedParams& p, hipStream_t st) {
  switch (rope) {
    case ROPE_NONE: return alibi ? launch_one<D, ROPE_NONE, true>(p, st) : launch_one<D, ROPE_NONE, false>(p, st);
    case ROPE_NEOX: return alibi ? launch_one<D, ROPE_NEOX, true>(p, st) : launch_one<D, ROPE_NEOX, false>(p, st);
    case ROPE_INTERLEAVED:
      return alibi ? launch_one<D, ROPE_INTERLEAVED, true>(p, st) : launch_one<D, ROPE_INTERLEAVED, false>(p, st);
  }
  return -2;
}

int launch_decode_paged(int D, int rope, bool alibi, const PagedParams& p, hipStream_t st) {
  if (D == 64) return dispatch_rope<64>(rope, alibi, p, st);
  if (D == 128) return dispatch_rope<128>(rope, alibi, p, st);
  return -2;
}

}  // namespace af
