// Attention of new tokens over paged keys and values, several tokens a sequence or
// one, behind a prefix that the whole batch shares; bf16, fp32 accumulation.
//
// Sequence b has n_b queries, the last n_b of its L_b own keys; query t of them sees
// the P keys of the prefix and its own keys 0 .. L_b - n_b + t:
//   s_j = scale q . k_j,  O = sum_j softmax(s)_j v_j,  LSE = log sum_j exp(s_j).
//
// A row is one (token, query head) of a K/V head's group of G: row r of a list of tokens
// is head r % G of token r / G.  Workgroup = NW waves = 32 NW rows against every ns-th
// 64-key tile of a list of key tiles.  What makes rows meet the prefix once:
//   * apart: the rows of all tokens of the batch are one list for the prefix's tiles, so
//     a workgroup's tile of K and V serves 32 NW rows of any sequences; the rows of a
//     sequence are a list for its own tiles.  Both kinds of workgroup run in one launch and leave
//     partials (max, sum, O), which a second kernel joins;
//   * joined: where sequences have tokens enough to fill tiles of rows by themselves, the
//     rows of a sequence walk the prefix's tiles and then their own: fewer partials, none
//     with one share.
// The tiles of a list are dealt out in turn to ns shares, so shares are even whatever the
// lengths, which are known on the device alone.  In calls of one token each, lists of up to
// 32 rows have a loop of their own (few_rows).
//
// Inside a workgroup the tiles go straight from the pages to LDS (attn_tiles.hpp), one
// 16-key unit of a page at a time, whose address is wave-uniform: lanes read the page numbers
// two tiles ahead, form an address each and hand them out as scalars.  The loop is the forward's: while the products S^T = K Q^T of the
// next tile run, this tile's scores become probabilities, and its P V runs while the next tile's
// scores are masked and reduced.  Q and K meet in bf16 exactly; P is rounded to bf16
// (2^-8 of each weight at most; the bf16 O is rounded as much), sums, maxima and O stay fp32.
//
// What lies in places that are no key of any row of the workgroup may be anything: scores
// are replaced and rows of V cleared in LDS after they landed.
//
// Bound by reading K and V where few rows meet them, from about 220 rows of a K/V head on by the
// products and the softmax between them.  Measured (D 128): 32 sequences' tokens behind 32768 shared
// keys, own keys to 1024, H 32 of 8, 57 to 58 us, of which the join 7: 224 MB, 4.5 TB/s in the
// first kernel.  3500 tokens of 6 sequences behind 32768: 1906 to 1999 us, 1.0 PFLOP/s, 81 to 85 % of a
// large library product's rate, matrix units busy 44 % of the cycles, 6.4 vector instructions to one of
// theirs, a third of the waves' time waiting; a
// tile of a workgroup of eight waves takes 1.75 us, of four waves, two of them on a CU, 1.9.
// Copies three tiles ahead instead of one (four stages, 32- or 64-key tiles) were nowhere
// faster: 1904 to 2120 us, and 60 to 140 for the first.
#include "attn_tiles.hpp"
#include "launch.hpp"

namespace af {

// The queries of a sequence: tokens [first, first + n), and its own keys.
struct Sequence {
  int b, first, n, keys;
};

__device__ __forceinline__ Sequence sequence_at(const TilesParams& p, int b) {
  Sequence s{b, b, 1, 0};
  if (p.starts) {
    s.first = min(max(uniform_load(p.starts + b), 0), p.T);
    s.n = min(max(uniform_load(p.starts + b + 1), s.first), p.T) - s.first;
  }
  s.keys = p.lens ? min(max(uniform_load(p.lens + b), 0), p.S) : p.S;
  return s;
}

// The sequence of a slot (a tile of rows) and the tile's first row.  Unless they are sorted
// by length, sequence b has the slots from first_b G / rows + b on, which leaves it room for a
// tile that is not full; its number is that of the sequences that start at or before the
// slot.  -1: no sequence's.
__device__ __forceinline__ int sequence_of(const TilesParams& p, int slot, int rows, int lane, int& r0) {
  if (p.by_length) {   // (up to 64 sequences with lengths) the longest one's slots first, so that short ones fill the end
    int count = 0, key = -1;
    if (lane < p.B) {
      int n = 1;
      if (p.starts) {
        const int first = min(max(p.starts[lane], 0), p.T);
        n = min(max(p.starts[lane + 1], first), p.T) - first;
      }
      count = (n * p.G + rows - 1) / rows;
      key = min(max(p.lens[lane], 0), p.S) * 64 + (63 - lane);   // (S <= 2^20)
    }
    int before = 0;
    for (int j = 0; j < p.B; ++j) before += __builtin_amdgcn_readlane(key, j) > key ? __builtin_amdgcn_readlane(count, j) : 0;
    const unsigned long long mine = __ballot(before <= slot && slot < before + count);
    if (!mine) return -1;
    const int b = __ffsll(mine) - 1;
    r0 = (slot - __builtin_amdgcn_readlane(before, b)) * rows;
    return b;
  }
  if (!p.starts) {
    const int per = (p.G + rows - 1) / rows;
    r0 = slot % per * rows;
    return slot / per;
  }
  int count = 0, mine = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    const int b = b0 + lane;
    const int at = b < p.B ? (int)((long long)min(max(p.starts[b], 0), p.T) * p.G / rows) + b : 0x7fffffff;
    const unsigned long long before = __ballot(at <= slot);
    if (before) mine = __builtin_amdgcn_readlane(at, 63 - __clzll(before));
    count += __popcll(before);
  }
  r0 = (slot - mine) * rows;
  return count - 1;
}

// All but the newest N copies of this wave have landed; this wave's LDS reads are done.
template <int N>
__device__ __forceinline__ void async_wait_but() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void lds_wait() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// What a partial with maximum m counts in a sum of maximum M.  Scores that are all NaN
// leave m at -inf, as no visible key does, and NaN in the sums: those are added, times
// 0, and stay NaN.
__device__ __forceinline__ float share_weight(float m, float M) { return m == -INFINITY ? 0.f : fast_exp2(m - M); }

// A row's sum of weights is that of a tile's, of SUM_TILES tiles' (l_run) and of those (l_old):
// in one sum the roundings of equal weights go the same way, and 2^20 keys in one share moved
// the LSE by 2.4e-4 (added a weight at a time by 1.9e-3).  Lists have up to 2^15 tiles: no sum
// is of more than 256 numbers.  (With the additions' errors kept in a register instead, 32
// sequences behind 32768 keys took 59.8 us against 58.2; one sum alone 57.7.)
constexpr int SUM_TILES = 128;

// A list of up to 32 rows (one token of a sequence and its heads; a prefix under a few
// sequences): the rows are one wave's, so the four waves take turns at its half tiles of 32
// keys, each with K and V of its own in LDS and no barrier before the end.  K of a wave's
// next half tile is on its way from this one's scores on, V from its products on.  Bound by
// the reads' latency.  Against the other loop: 8 sequences behind 4096 keys, H32/8 D128,
// 13.3 us to 15.5; 64 with 8128 own keys (H32/8 D128) 245 to 265; 189 sequences of up
// to 13 own keys behind 23, H16 D128, 34 to 44.
template <int D, class Place, class Entries>
__device__ __forceinline__ void few_rows(const TilesParams& p, uint16_t* smem, Place place_of, Entries entries16, int entries,
                                         int nt, int g, int nrows, int first, int shift_keys, int part, int lane, int wave) {
  using AT = AsyncTile<D, 1, 32>;
  constexpr int KS = D / 16, MT = D / 32, RPG = AT::RPG, CPR = D / 8, NI = AT::NI;
  const int lq = lane & 31, lg = lane >> 5;
  const AT at(lane, 0);
  uint16_t* kw = smem + wave * 2 * AT::ELEMS;
  uint16_t* vw = kw + AT::ELEMS;
  __shared__ float xml[2][4][32];                          // the waves' maximum and sum of every row

  const int row = min(lq, nrows - 1), token = row / p.G;
  const size_t at_row = (size_t)(first + token) * p.H + g * p.G + (row - token * p.G);
  const int lim = shift_keys + token;                      // the last own key that this lane's row sees; the least: shift_keys
  u32x4 qreg[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) qreg[s] = ld16(static_cast<const uint16_t*>(p.q) + at_row * D + 16 * s + 8 * lg);

  // Lanes 0, 1: K's units of a half tile, 2, 3: V's.
  const int lane_unit = lane & 1;
  const bool lane_v = lane & 2;
  const uint16_t* lane_base = static_cast<const uint16_t*>(lane_v ? p.v : p.k) + g * (lane_v ? p.vs[1] : p.ks[1]);
  const long long lane_page = lane_v ? p.vs[0] : p.ks[0];
  const uint32_t lane_place = (uint32_t)(lane_v ? p.vs[2] : p.ks[2]);
  const uint32_t voff_k = (uint32_t)(lane / CPR) * (uint32_t)(2 * p.ks[2]) + at.col;
  const uint32_t voff_v = (uint32_t)(lane / CPR) * (uint32_t)(2 * p.vs[2]) + at.col;
  struct Half {
    int n0, end;
    bool prefix;
    uint32_t valid;
    uint64_t base;
  };
  int batch = 0;
  auto half_at = [&](int h) {
    const int i = h >> 1;
    if (i >> 4 != batch) {
      batch = i >> 4;
      entries = entries16(16 * batch);
    }
    const int e = __shfl(entries, 4 * (i & 15) + 2 * (h & 1) + lane_unit);
    const auto t = place_of(i);
    Half x{t.n0 + 32 * (h & 1), t.end, t.prefix, 0, 0};
    const bool ok = (unsigned)e < (unsigned)p.num_pages;
    x.valid = (uint32_t)__ballot(ok) & 3u;
    const uint32_t place = (uint32_t)(x.n0 + 16 * lane_unit) & ((1u << p.page_shift) - 1);
    x.base = (uint64_t)(lane_base + (ok ? e : 0) * lane_page + (uint64_t)place * lane_place);
    return x;
  };
  auto load = [&](const Half& x, int lane0, long long place, uint32_t voff, uint16_t* dst) {
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)dst;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x.base, lane0 + j * RPG / 16);
      const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(x.base >> 32), lane0 + j * RPG / 16);
      const uint64_t base = ((uint64_t)hi << 32 | lo) + (uint64_t)(2 * (j * RPG % 16)) * (uint64_t)place;
      async_copy16((const void*)base, voff, __builtin_amdgcn_readfirstlane(lds + j * (AT::GROUP * 2)));
    }
  };
  auto load_k = [&](const Half& x) { load(x, 0, p.ks[2], voff_k, kw); };
  auto load_v = [&](const Half& x) { load(x, 2, p.vs[2], voff_v, vw); };

  f32x16 acc[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m] = f32x16{};
  float m_run = -INFINITY, l_run = 0.f, l_old = 0.f;       // log2 units
  const float c2 = p.scale * kLog2e;
  const int nh = 2 * nt;
  int h = wave;
  Half cur{};
  if (h < nh) {
    cur = half_at(h);
    load_k(cur);
    load_v(cur);
  }
  while (h < nh) {
    const bool more = h + 4 < nh;
    async_wait_but<NI>();                                  // K is there
    f32x16 sc = f32x16{};
#pragma unroll
    for (int s = 0; s < KS; ++s) sc = mfma32(at.row(kw, 0, s), qreg[s], sc);
    lds_wait();
    Half nxt = cur;
    if (more) {
      nxt = half_at(h + 4);
      load_k(nxt);
    }
    const bool whole = cur.n0 + 32 <= cur.end && cur.valid == 3u;
    if (!whole || (!cur.prefix && cur.n0 + 31 > shift_keys)) {
      const int seen = (cur.prefix ? cur.end - 1 : lim) - cur.n0 - 4 * lg;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int last = cur.valid >> (r >> 3) & 1 ? seen : -1;
        sc[r] = 8 * (r >> 2) + (r & 3) <= last ? sc[r] : -INFINITY;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[r]);
    const float m_new = fmaxf(m_run, pair_max(mx) * c2);
    if (__any(m_new > m_run + 8.f)) {
      const float alpha = (m_run == -INFINITY) ? 0.f : fast_exp2(m_run - m_new);
      l_run *= alpha;
      l_old *= alpha;
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[m] *= alpha;
      m_run = m_new;
    }
    const float m_use = (m_run == -INFINITY) ? 0.f : m_run;
    u32x4 pop[2];
    float w[16], rs = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      w[r] = fast_exp2(__builtin_fmaf(sc[r], c2, -m_use));
      rs += w[r];
    }
    l_run += rs;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int x = 0; x < 4; ++x) pop[hf][x] = pack_bf16(w[8 * hf + 2 * x], w[8 * hf + 2 * x + 1]);
    if (more) async_wait_but<NI>();                        // V is there
    else async_wait();
    if (!whole) {                                          // rows that are no key: 0 x NaN is NaN
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int n = cur.n0 + RPG * j + lane / CPR;
        if (n >= cur.end || !(cur.valid >> (j * RPG / 16) & 1))
          *reinterpret_cast<u32x4*>(vw + j * AT::GROUP + 8 * lane) = u32x4{0, 0, 0, 0};
      }
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) acc[mt] = mfma32(at.tr(vw, 16 * hf, mt), pop[hf], acc[mt]);
    lds_wait();
    if (more) load_v(nxt);
    cur = nxt;
    h += 4;
    if (h / 4 % SUM_TILES == 0) {
      l_old += l_run;
      l_run = 0.f;
    }
  }

  // Join the waves: each leaves its O in its own LDS, as 16-byte pieces [32-dim tile][piece]
  // [lane]; wave w sums dims 32 w .. of all four.
  const float l_tot = pair_sum(l_run + l_old);
  float4* mine = reinterpret_cast<float4*>(kw);
  static_assert(MT * 4 * 64 * 16 <= 2 * AT::ELEMS * 2, "a wave's O goes through its tiles' memory");
  static_assert(4 * 2 * AT::ELEMS <= 4 * AsyncTile<D, 4>::ELEMS, "the waves' tiles fit the workgroup's stages");
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int a = 0; a < 4; ++a)
      mine[(4 * mt + a) * 64 + lane] = float4{acc[mt][4 * a], acc[mt][4 * a + 1], acc[mt][4 * a + 2], acc[mt][4 * a + 3]};
  if (lg == 0) {
    xml[0][wave][lq] = m_run;
    xml[1][wave][lq] = l_tot;
  }
  __syncthreads();
  if (wave >= MT || lq >= nrows) return;
  float M = -INFINITY, l = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) M = fmaxf(M, xml[0][w][lq]);
  float4 o[4] = {};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float a = share_weight(xml[0][w][lq], M);
    l = __builtin_fmaf(xml[1][w][lq], a, l);
    const float4* from = reinterpret_cast<const float4*>(smem + w * 2 * AT::ELEMS);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 x = from[(4 * wave + q) * 64 + lane];
      o[q].x = __builtin_fmaf(x.x, a, o[q].x);
      o[q].y = __builtin_fmaf(x.y, a, o[q].y);
      o[q].z = __builtin_fmaf(x.z, a, o[q].z);
      o[q].w = __builtin_fmaf(x.w, a, o[q].w);
    }
  }
  if (p.parts > 1) {
    const size_t at_part = (size_t)part * p.T * p.H + at_row;
    float* dst = p.part_acc + at_part * D + 32 * wave + 4 * lg;
#pragma unroll
    for (int q = 0; q < 4; ++q) *reinterpret_cast<float4*>(dst + 8 * q) = o[q];
    if (wave == 0 && lg == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at_part) = float2{M, l};
  } else {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* dst = static_cast<uint16_t*>(p.o) + at_row * D + 32 * wave + 4 * lg;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<u32x2*>(dst + 8 * q) = u32x2{pack_bf16(o[q].x * inv, o[q].y * inv), pack_bf16(o[q].z * inv, o[q].w * inv)};
    if (wave == 0 && lg == 0) p.lse[at_row] = l == 0.f ? -INFINITY : (M + __log2f(l)) * kLn2;
  }
}

// Few: the call is of one token each with up to 32 heads to a K/V head, so that every
// sequence's list, and a prefix's under a few sequences, is few_rows'.  Other calls have a
// build without that loop: with it, and page numbers sixteen tiles at a time, prompts took
// up to 6 % longer (12 x 200 tokens behind 8192 keys, H12 D64: 71.5 us against 67.2).
template <int D, int NW, bool Few>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2)))
void paged_tiles_kernel(TilesParams p) {
  using AT = AsyncTile<D, NW>;
  constexpr int BN = 64, KS = D / 16, MT = D / 32, ROWS = 32 * NW, RPG = AT::RPG;
  __shared__ __attribute__((aligned(16))) uint16_t smem[4 * AT::ELEMS];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 31, lg = lane >> 5;

  // ---- what this workgroup does: rows [r0, r0 + ROWS) of a list of nrows, from token
  // `first` on; tiles share, share + ns, ... of the prefix's (np keys) and then the
  // sequence's; part: where its partial goes.
  const int g = blockIdx.x % p.Hkv;
  int i = blockIdx.x / p.Hkv, r0, nrows, first, np = 0, share, ns, part, shift_keys = 0;
  const int* table = p.table;
  const bool prefix_list = i < p.prefix_items;             // (apart: a list of all tokens' rows)
  int b = 0;
  if (prefix_list) {
    ns = p.nsp;
    share = i % ns;
    r0 = i / ns * ROWS;
    part = share;
  } else {
    i -= p.prefix_items;
    ns = p.nso;
    share = i % ns;
    b = __builtin_amdgcn_readfirstlane(sequence_of(p, i / ns, ROWS, lane, r0));
    r0 = __builtin_amdgcn_readfirstlane(r0);
    if (b < 0) return;
    table += (size_t)b * p.max_pages;
    part = p.nsp + share;
  }
  // Page numbers come by vector loads, lane l that of unit l % 4 (Few: the first 16 tiles'
  // at once, lane l that of tile l / 4).
  const int lane_unit = lane & 3;
  auto entry_of = [=](bool prefix, int n0) {
    const int* pages = prefix ? p.prefix_table : table;
    const int last = (prefix ? p.prefix_pages : p.max_pages) - 1;
    return pages[min((n0 + 16 * lane_unit) >> p.page_shift, last)];
  };
  int e[3], first16 = 0;
  if constexpr (Few) {        // (never joined: that takes 1024 rows a sequence)
    first16 = entry_of(prefix_list, BN * (share + (lane >> 2) * ns));
  } else if (!p.joined) {     // apart, the first tiles' places do not depend on any length: one trip to memory less
#pragma unroll
    for (int j = 0; j < 3; ++j) e[j] = entry_of(prefix_list, BN * (share + j * ns));
  }
  if (p.prefix_pages > 0 && (prefix_list || p.joined))
    np = p.prefix_len ? min(max(uniform_load(p.prefix_len), 0), p.P) : p.P;
  int own = 0;                                             // own keys that any row of the workgroup sees
  if (prefix_list) {
    nrows = p.T * p.G;
    first = 0;
  } else {
    const Sequence s = sequence_at(p, b);
    nrows = s.n * p.G;
    if (r0 >= nrows) return;
    first = s.first;
    shift_keys = s.keys - s.n;                             // token t sees its keys up to shift_keys + t
    own = max(0, shift_keys + (min(r0 + ROWS, nrows) - 1) / p.G + 1);
  }
  const int tp = (np + BN - 1) / BN, all = tp + (own + BN - 1) / BN;
  const int nt = all > share ? (all - share + ns - 1) / ns : 0;
  const bool direct = p.parts == 1;
  const int G = p.G;
  const int row = r0 + 32 * wave + lq, rowc = min(row, nrows - 1);
  const int token = rowc / G;                              // of the list
  const size_t at_row = (size_t)(first + token) * p.H + g * G + (rowc - token * G);   // of Q, O and LSE

  if (nt == 0) {                                           // no key: nothing to join, or an empty row
    for (int j = tid; j < ROWS && r0 + j < nrows; j += 64 * NW) {
      const int t = (r0 + j) / G;
      const size_t at = (size_t)(first + t) * p.H + g * G + (r0 + j - t * G);
      if (direct) {
        for (int d = 0; d < D; d += 8) st16(static_cast<uint16_t*>(p.o) + at * D + d, u32x4{0, 0, 0, 0});
        p.lse[at] = -INFINITY;
      } else {
        *reinterpret_cast<float2*>(p.part_ml + 2 * ((size_t)part * p.T * p.H + at)) = float2{-INFINITY, 0.f};
      }
    }
    return;
  }

  // ---- tiles
  // The units' addresses are formed in lanes (0 .. 3: K's of a tile, 4 .. 7: V's) and handed
  // out as scalars.
  struct Tile {
    int n0, end;          // its first key in the prefix or in the sequence, and where those end
    bool prefix;
    uint32_t valid;       // bit u: unit u has a page
    uint64_t base;        // lane u: K's unit u, lane 4 + u: V's
  };
  auto place_of = [=](int i) {   // of the workgroup's i-th tile
    Tile t{};
    const int idx = share + i * ns;
    t.prefix = prefix_list || idx < tp;                    // (apart, no length has to be known for it)
    t.n0 = BN * (t.prefix ? idx : idx - tp);
    t.end = t.prefix ? np : own;
    return t;
  };
  if constexpr (Few) {
    static_assert(NW == 4, "few_rows deals with four waves");
    auto entries16 = [=](int i) {                          // of the workgroup's tiles i .. i + 15
      const Tile t = place_of(i + (lane >> 2));
      return entry_of(t.prefix, t.n0);
    };
    if (nrows <= 32) {   // (not the last rows of a longer list: those walk the tiles beside the others and share their reads)
      few_rows<D>(p, smem, place_of, entries16, first16, nt, g, nrows, first, shift_keys, part, lane, wave);
      return;
    }
  }

  const bool live = r0 + 32 * wave < nrows;                // (a wave without rows only copies)
  const int lim = shift_keys + token;                      // the last own key that this lane's row sees
  const int lim_wave = shift_keys + min(r0 + 32 * wave, nrows - 1) / G;   // the least of the wave's

  const bool lane_v = lane & 4;
  const uint16_t* lane_base = static_cast<const uint16_t*>(lane_v ? p.v : p.k) + g * (lane_v ? p.vs[1] : p.ks[1]);
  const long long lane_page = lane_v ? p.vs[0] : p.ks[0];
  const uint32_t lane_place = (uint32_t)(lane_v ? p.vs[2] : p.ks[2]);
  auto settle = [&](Tile& t, int e) {
    const bool ok = (unsigned)e < (unsigned)p.num_pages;
    t.valid = (uint32_t)__ballot(ok) & 15u;
    const uint32_t place = (uint32_t)(t.n0 + 16 * lane_unit) & ((1u << p.page_shift) - 1);
    t.base = (uint64_t)(lane_base + (ok ? e : 0) * lane_page + (uint64_t)place * lane_place);
  };
  auto whole = [&](const Tile& t) { return t.n0 + BN <= t.end && t.valid == 15u; };

  const AT at(lane, wave);
  auto akst = [&](int par) { return smem + 2 * par * AT::ELEMS; };
  auto avst = [&](int par) { return smem + (2 * par + 1) * AT::ELEMS; };
  constexpr int CPR = D / 8;
  const int unit0 = wave * RPG / 16, row_in_unit = wave * RPG % 16 + lane / CPR;   // of the wave's first group
  auto unit_of = [&](int i) { return unit0 + NW * RPG / 16 * i; };
  const uint32_t voff_k = (uint32_t)row_in_unit * (uint32_t)(2 * p.ks[2]) + at.col;
  const uint32_t voff_v = (uint32_t)row_in_unit * (uint32_t)(2 * p.vs[2]) + at.col;
  auto load = [&](const Tile& t, int lane0, uint32_t voff, uint16_t* dst) {
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)dst;
#pragma unroll
    for (int i = 0; i < AT::NI; ++i) {
      const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)t.base, lane0 + unit_of(i));
      const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(t.base >> 32), lane0 + unit_of(i));
      async_copy16((const void*)((uint64_t)hi << 32 | lo), voff,
                   __builtin_amdgcn_readfirstlane(lds + (wave + NW * i) * (AT::GROUP * 2)));
    }
  };
  auto load_k = [&](const Tile& t, uint16_t* dst) { load(t, 0, voff_k, dst); };
  auto load_v = [&](const Tile& t, uint16_t* dst) { load(t, 4, voff_v, dst); };
  // Rows of V that are no key: 0 x NaN is NaN.  (Each lane clears what it copied.)
  auto clear = [&](const Tile& t, uint16_t* dst) {
    if (whole(t)) return;
#pragma unroll
    for (int i = 0; i < AT::NI; ++i) {
      const int n = t.n0 + 16 * unit_of(i) + row_in_unit;
      if (n >= t.end || !(t.valid >> unit_of(i) & 1))
        *reinterpret_cast<u32x4*>(dst + (wave + NW * i) * AT::GROUP + 8 * lane) = u32x4{0, 0, 0, 0};
    }
  };

  Tile cur_t = place_of(0), nxt_t = place_of(1), far_t = place_of(2);
  if constexpr (Few) {
#pragma unroll
    for (int j = 0; j < 3; ++j) e[j] = __shfl(first16, 4 * j + lane_unit);
  } else if (p.joined) {
    e[0] = entry_of(cur_t.prefix, cur_t.n0);
    e[1] = entry_of(nxt_t.prefix, nxt_t.n0);
    e[2] = entry_of(far_t.prefix, far_t.n0);
  }
  settle(cur_t, e[0]);
  settle(nxt_t, e[1]);
  settle(far_t, e[2]);
  load_k(cur_t, akst(0));
  load_v(cur_t, avst(0));
  if (nt > 1) load_k(nxt_t, akst(1));

  // Query operand (B of S^T = K Q^T): lane holds its row, dims 16 s + 8 lg .. +7.
  u32x4 qreg[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) qreg[s] = ld16(static_cast<const uint16_t*>(p.q) + at_row * D + 16 * s + 8 * lg);

  f32x16 acc[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m] = f32x16{};
  float m_run = -INFINITY, l_run = 0.f, l_old = 0.f, m_new = -INFINITY;   // log2 units
  const float c2 = p.scale * kLog2e;

  auto scores = [&](f32x16 (&sc)[2], const uint16_t* Ks) {
    sc[0] = f32x16{};
    sc[1] = f32x16{};
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) sc[kt] = mfma32(at.row(Ks, 32 * kt, s), qreg[s], sc[kt]);
  };
  auto pv = [&](const u32x4 (&pop)[2][2], const uint16_t* Vs) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[mt] = mfma32(at.tr(Vs, 32 * kt + 16 * hf, mt), pop[kt][hf], acc[mt]);
  };
  // Mask and maximum.  Element r of subtile kt is key n0 + 32 kt + 8 (r / 4) + r % 4 + 4 lg,
  // of unit 2 kt + r / 8.
  auto prepare = [&](f32x16 (&sc)[2], const Tile& t) {
    if (!whole(t) || (!t.prefix && t.n0 + BN - 1 > lim_wave)) {   // (wave-uniform)
      const int seen = (t.prefix ? t.end - 1 : lim) - t.n0 - 4 * lg;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int last = t.valid >> u & 1 ? seen : -1;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const float x = sc[u >> 1][8 * (u & 1) + r];
          sc[u >> 1][8 * (u & 1) + r] = 16 * u + 8 * (r >> 2) + (r & 3) <= last ? x : -INFINITY;
        }
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[kt][r]);
    m_new = fmaxf(m_run, pair_max(mx) * c2);
  };
  auto raise = [&]() {   // the reference maximum, where a row's grew by more than 2^8
    if (__any(m_new > m_run + 8.f)) {
      const float alpha = (m_run == -INFINITY) ? 0.f : fast_exp2(m_run - m_new);
      l_run *= alpha;
      l_old *= alpha;
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[m] *= alpha;
      m_run = m_new;
    }
  };
  auto probs = [&](const f32x16 (&sc)[2], u32x4 (&pop)[2][2]) {
    const float m_use = (m_run == -INFINITY) ? 0.f : m_run;
    float rs = 0.f;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      float e[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        e[r] = fast_exp2(__builtin_fmaf(sc[kt][r], c2, -m_use));
        rs += e[r];
      }
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int w = 0; w < 4; ++w) pop[kt][hf][w] = pack_bf16(e[8 * hf + 2 * w], e[8 * hf + 2 * w + 1]);
    }
    l_run += rs;
  };
  auto pin_values = [](u32x4 (&pp)[2][2], float& l) {   // (keeps the softmax work beside the next scores' products)
    asm volatile("" : "+v"(pp[0][0]), "+v"(pp[0][1]), "+v"(pp[1][0]), "+v"(pp[1][1]), "+v"(l));
  };

  f32x16 sa[2], sb[2];
  u32x4 pop[2][2];
  async_wait();
  clear(cur_t, avst(0));
  __syncthreads();
  if (live) {
    scores(sa, akst(0));
    prepare(sa, cur_t);
    raise();
  }
  __syncthreads();
  // Iteration t turns tile t's scores into its share of O while tile t + 1's scores are
  // formed; it copies K of tile t + 2 and V of tile t + 1 into the stage halves that the
  // last barrier freed.
  int t = 0;
  auto iteration = [&](f32x16 (&cur)[2], f32x16 (&nxt)[2], auto parity) {
    constexpr int PAR = decltype(parity)::value;   // t & 1
    if (t + 2 < nt) load_k(far_t, akst(PAR));
    load_v(nxt_t, avst(1 - PAR));
    Tile after = place_of(t + 3);
    int entry = entry_of(after.prefix, after.n0);
    if (live) {
      probs(cur, pop);
      scores(nxt, akst(1 - PAR));
      pin_values(pop, l_run);
      prepare(nxt, nxt_t);
      pv(pop, avst(PAR));
      raise();
    }
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(entry)::"memory");   // the copies, and the pages behind them
    clear(nxt_t, avst(1 - PAR));
    settle(after, entry);
    __syncthreads();
    nxt_t = far_t;
    far_t = after;
    ++t;
  };
  using P0 = std::integral_constant<int, 0>;
  using P1 = std::integral_constant<int, 1>;
  while (t + 2 < nt) {
    iteration(sa, sb, P0{});
    iteration(sb, sa, P1{});
    if (t % SUM_TILES == 0) {
      l_old += l_run;
      l_run = 0.f;
    }
  }
  if (t + 1 < nt) {
    iteration(sa, sb, P0{});
    if (live) {
      probs(sb, pop);
      pv(pop, avst(1));
    }
  } else if (live) {
    probs(sa, pop);
    pv(pop, avst(0));
  }

  // ---- the result, or this share's partial
  const float l_tot = pair_sum(l_run + l_old);
  if (!direct) {
    if (live && row < nrows) {
      const size_t at = (size_t)part * p.T * p.H + at_row;
      float* dst = p.part_acc + at * D + 4 * lg;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int a = 0; a < 4; ++a)
          *reinterpret_cast<float4*>(dst + 32 * mt + 8 * a) =
              float4{acc[mt][4 * a], acc[mt][4 * a + 1], acc[mt][4 * a + 2], acc[mt][4 * a + 3]};
      if (lg == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at) = float2{m_run, l_tot};
    }
    return;
  }
  const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
  if (live && row < nrows) {
    uint16_t* dst = static_cast<uint16_t*>(p.o) + at_row * D + 4 * lg;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int a = 0; a < 4; ++a)
        *reinterpret_cast<u32x2*>(dst + 32 * mt + 8 * a) =
            u32x2{pack_bf16(acc[mt][4 * a] * inv, acc[mt][4 * a + 1] * inv),
                  pack_bf16(acc[mt][4 * a + 2] * inv, acc[mt][4 * a + 3] * inv)};
    if (lg == 0) p.lse[at_row] = l_tot == 0.f ? -INFINITY : (m_run + __log2f(l_tot)) * kLn2;
  }
}

// Join the partials of rows (token, query head): D / 4 lanes hold a row's dims, GP groups
// of lanes take every GP-th partial, 256 / (D / 4) / GP rows to a workgroup.  A partial of
// a share without a visible key, (-inf, 0), has no O.
template <int D, int GP>
__global__ __launch_bounds__(256) void tiles_join_kernel(TilesParams p) {
  constexpr int LPR = D / 4, NG = 256 / LPR, NR = NG / GP;
  __shared__ float4 red[NG][LPR];
  __shared__ float2 stat[NG];
  const int c = threadIdx.x % LPR, grp = threadIdx.x / LPR, gp = grp % GP;
  const size_t rows = (size_t)p.T * p.H;
  const size_t r = (size_t)blockIdx.x * NR + grp / GP;
  bool live = r < rows;
  if (live && p.starts) {   // rows outside every sequence are left as they are
    const int token = (int)(r / p.H);
    live = token >= p.starts[0] && token < p.starts[p.B];
  }
  // What a partial (m2, l2, x) adds to (M, l, sum).
  float M = -INFINITY, l = 0.f;
  float4 sum = {0.f, 0.f, 0.f, 0.f};
  auto fold = [&](const float2& ml, const float4& x) {
    const float m = fmaxf(M, ml.x), a = share_weight(M, m), w = share_weight(ml.x, m);
    sum.x = __builtin_fmaf(sum.x, a, x.x * w);
    sum.y = __builtin_fmaf(sum.y, a, x.y * w);
    sum.z = __builtin_fmaf(sum.z, a, x.z * w);
    sum.w = __builtin_fmaf(sum.w, a, x.w * w);
    l = __builtin_fmaf(l, a, ml.y * w);
    M = m;
  };
  if (live) {
    // Four partials on their way at once; where there is no O, what is read in its place is not used.
    for (int i0 = gp; i0 < p.parts; i0 += 4 * GP) {
      float2 ml[4];
      float4 x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const size_t at = min(i0 + j * GP, p.parts - 1) * rows + r;
        ml[j] = *reinterpret_cast<const float2*>(p.part_ml + 2 * at);
        x[j] = *reinterpret_cast<const float4*>(p.part_acc + at * D + 4 * c);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i0 + j * GP < p.parts && !(ml[j].x == -INFINITY && ml[j].y == 0.f)) fold(ml[j], x[j]);
    }
  }
  if constexpr (GP > 1) {
    red[grp][c] = sum;
    if (c == 0) stat[grp] = float2{M, l};
    __syncthreads();
    if (gp != 0 || !live) return;
    for (int i = 1; i < GP; ++i) {
      const float2 ml = stat[grp + i];
      if (!(ml.x == -INFINITY && ml.y == 0.f)) fold(ml, red[grp + i][c]);
    }
  }
  if (!live) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.o) + r * D + 4 * c) =
      u32x2{pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv)};
  if (c == 0) p.lse[r] = l == 0.f ? -INFINITY : (M + __log2f(l)) * kLn2;
}

// ---------------------------------------------------------------- launch
template <int D>
static int launch_one(const TilesParams& p, int nw, hipStream_t st) {
  const dim3 grid((unsigned)((p.prefix_items + p.own_items) * p.Hkv));
  if (nw == 8) hipLaunchKernelGGL((paged_tiles_kernel<D, 8, false>), grid, dim3(512), 0, st, p);
  else if (!p.starts && p.G <= 32) hipLaunchKernelGGL((paged_tiles_kernel<D, 4, true>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((paged_tiles_kernel<D, 4, false>), grid, dim3(256), 0, st, p);
  if (hipGetLastError() != hipSuccess) return -3;   // (no join of what is not there)
  if (p.parts > 1) {
    const long long rows = (long long)p.T * p.H;
    constexpr int NG = 1024 / D;
    if (p.parts >= 8 && rows < (1 << 24)) hipLaunchKernelGGL((tiles_join_kernel<D, NG>), dim3((unsigned)rows), dim3(256), 0, st, p);
    else hipLaunchKernelGGL((tiles_join_kernel<D, 1>), dim3((unsigned)((rows + NG - 1) / NG)), dim3(256), 0, st, p);
  }
  return hipGetLastError() == hipSuccess ? 0 : -3;
}

int launch_paged_tiles(int D, const TilesParams& p, int nw, hipStream_t st) {
  if (D == 64) return launch_one<64>(p, nw, st);
  if (D == 128) return launch_one<128>(p, nw, st);
  return -2;
}

}  // namespace af
