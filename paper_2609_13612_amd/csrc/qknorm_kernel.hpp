// RMS norm of every head's query and key rows with learned weights, and their
// rotation, in one pass; its backward; and the same for new tokens whose keys
// and values go to a paged cache.
//
// A row x of D values at position p:
//   r = (mean(x^2) + eps)^-1/2,  y = w o (x r),  out = R_p y
// and with dy = R_p^T dout, g = w o dy, xh = x r:
//   dx = r (g - xh mean(g o xh)),   dw = sum over rows of dy o xh.
//
// D / 16 threads share a row; a thread holds dims 8c..8c+7 and D/2 + 8c.., so
// the pairs of both rotation kinds are its own and the row's sums are two or
// three DPP steps.  All arithmetic is fp32 on values read once; r is formed
// again in the backward, which reads x anyway, rather than stored.  A thread
// takes HPT heads of one position, whose cos/sin entries and weights it loads
// once, and has all their loads in flight before it uses any.
//
// Bound by HBM: B4 H64/8 S4096 D128 bf16 108 us forward, 5.6 TB/s, and 176 backward, 5.1;
// fp32 B1 H32/8 S8192 69 forward, 4.8, and 110 backward, 4.6.
//
// Rows may lie anywhere 16-byte aligned (strides per batch, head, position): a
// slice of a fused projection's output needs no copy first.
//
// AXES: positions of several axes (time, height, width of a patch of a video).  Pair
// i of a row turns by the position on its axis; what axis that is, two bits a pair,
// comes with the call.  Beside the rows a thread then reads up to four positions and
// gathers its 8 pairs' angles from as many rows of the table.  Such a call may leave
// the norm out (r = 1, no weights): its backward is the inverse rotation of dout alone.
// us of B1 H32/8 S8192 D128 bf16 in replayed graphs, three axes and one: forward 28.3 and
// 27.0, backward 52.4 and 48.5 (a thread gathers its angles for two heads there, for four in
// the forward; held to 128 registers for a fourth wave per SIMD, 53.5), without norm 27 each.
#pragma once
#include <type_traits>

#include "common.hpp"
#include "launch.hpp"

namespace af {

// ---------------------------------------------------------------- rows
// The thread's 16 values of a row: dims 8c.. in v[0..7], D/2 + 8c.. in v[8..15].
template <bool FP32>
struct RowChunk {
  u32x4 x[FP32 ? 4 : 2];
  __device__ __forceinline__ void load(const void* row, int d0, int d1) {
    if constexpr (FP32) {
      const float* p = static_cast<const float*>(row);
      x[0] = ld16(p + d0);
      x[1] = ld16(p + d0 + 4);
      x[2] = ld16(p + d1);
      x[3] = ld16(p + d1 + 4);
    } else {
      const uint16_t* p = static_cast<const uint16_t*>(row);
      x[0] = ld16(p + d0);
      x[1] = ld16(p + d1);
    }
  }
  __device__ __forceinline__ void store(void* row, int d0, int d1) const {
    if constexpr (FP32) {
      float* p = static_cast<float*>(row);
      st16(p + d0, x[0]);
      st16(p + d0 + 4, x[1]);
      st16(p + d1, x[2]);
      st16(p + d1 + 4, x[3]);
    } else {
      uint16_t* p = static_cast<uint16_t*>(row);
      st16(p + d0, x[0]);
      st16(p + d1, x[1]);
    }
  }
  __device__ __forceinline__ void get(float (&v)[16]) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (FP32) v[i] = __uint_as_float(x[i >> 2][i & 3]);
      else v[i] = (i & 1) ? bf_hi(x[i >> 3][(i & 7) >> 1]) : bf_lo(x[i >> 3][(i & 7) >> 1]);
    }
  }
  __device__ __forceinline__ void put(const float (&v)[16]) {
    if constexpr (FP32) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i >> 2][i & 3] = __float_as_uint(v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i >> 2][i & 3] = pack_bf16(v[2 * i], v[2 * i + 1]);
    }
  }
};

// The sum of x over the D / 16 (4 or 8) lanes of a row.
template <int D>
__device__ __forceinline__ float row_sum(float x) {
  auto dpp = [](float v, auto ctrl) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  x += dpp(x, std::integral_constant<int, 0xB1>{});    // quad_perm: lane ^ 1
  x += dpp(x, std::integral_constant<int, 0x4E>{});    // quad_perm: lane ^ 2
  if constexpr (D == 128) x += dpp(x, std::integral_constant<int, 0x141>{});   // row_half_mirror: the other four
  return x;
}

// What p.axis says of the thread's pairs (see Angles): two bits for each of its 8.
template <int D, int ROPE>
__device__ __forceinline__ uint32_t axes_of(const QkNormParams& p, int c) {
  // Values, not places, are chosen by lane here and below: a place that differs by lane
  // would go through memory (one token's append took 7.9 us instead of 3.9).
  // The words are values of their own before a lane chooses: the compiler makes one load of
  // arguments out of a choice between two, at the index of the wave's first lane (pairs 16 to
  // 31 of D 64 then took the axes of pairs 0 to 15).
  u32x4 axis;
#pragma unroll
  for (int w = 0; w < D / 32; ++w) {
    uint32_t x = p.axis[w];
    asm("" : "+s"(x));
    axis[w] = x;
  }
  auto word = [&](int w) {
    const uint32_t lo = w & 1 ? axis.y : axis.x;
    if constexpr (D == 64) return lo;
    const uint32_t hi = w & 1 ? axis.w : axis.z;
    return w & 2 ? hi : lo;
  };
  if constexpr (ROPE == ROPE_NEOX) return word(c >> 1) >> (16 * (c & 1)) & 0xffffu;
  const uint32_t lo = word(c >> 2) >> (8 * (c & 3)) & 0xffu, hi = word((D / 64) + (c >> 2)) >> (8 * (c & 3)) & 0xffu;
  return lo | hi << 8;
}

// The positions of a row of the call, of which there are n, on its axes.  Asked for before
// the row itself: the table's rows wait for them, and nothing else of the thread's does.
struct RowPositions {
  u32x4 at;   // (a vector, not an array: see axes_of)
  __device__ __forceinline__ void load(const QkNormParams& p, size_t row, size_t n) {
    const int* x = p.positions + row;
    const int last = p.axes - 1;
    at = u32x4{(uint32_t)x[0], (uint32_t)x[min(1, last) * n], (uint32_t)x[min(2, last) * n], (uint32_t)x[min(3, last) * n]};
  }
};

// cos and sin of the thread's 8 pairs at position pos: NeoX pair 8c + i is
// (v[i], v[8 + i]); interleaved pairs are (v[2i], v[2i + 1]), 4c + i and D/4 + 4c
// + i.  A position outside the table gives NaN, so its row comes out as NaN.
template <int D, int ROPE>
struct Angles {
  float c[8], s[8];
  __device__ __forceinline__ void load(const float2* __restrict__ table, int rows, int pos, int d0) {
    if constexpr (ROPE != ROPE_NONE) {
      const bool ok = (unsigned)pos < (unsigned)rows;
      const float2* t = table + (size_t)(ok ? pos : 0) * (D / 2);
      float4 e[4];
      const float4* lo = reinterpret_cast<const float4*>(t + (ROPE == ROPE_NEOX ? d0 : d0 / 2));
      const float4* hi = ROPE == ROPE_NEOX ? lo + 2 : reinterpret_cast<const float4*>(t + D / 4 + d0 / 2);
      e[0] = lo[0];
      e[1] = lo[1];
      e[2] = hi[0];
      e[3] = hi[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[2 * i] = ok ? e[i].x : NAN;
        s[2 * i] = ok ? e[i].y : NAN;
        c[2 * i + 1] = ok ? e[i].z : NAN;
        s[2 * i + 1] = ok ? e[i].w : NAN;
      }
    }
  }
  // The same, each pair at the position on its axis.  Two neighbours on one axis, in every
  // thread (p.by_two), share a load.
  __device__ __forceinline__ void load_axes(const QkNormParams& p, const RowPositions& pos, int ch) {
    const uint32_t rows = (uint32_t)p.rows;
    const bool ok = pos.at.x < rows && pos.at.y < rows && pos.at.z < rows && pos.at.w < rows;
    const u32x4 at = ok ? pos.at : u32x4{0, 0, 0, 0};
    uint32_t bits = axes_of<D, ROPE>(p, ch);
    asm volatile("" : "+v"(bits));   // (in the backward's loop the choices are formed anew, not kept in registers)
    auto entry = [&](int i) {
      const uint32_t a = bits >> (2 * i) & 3u;
      const uint32_t lo = a & 1u ? at.y : at.x, hi = a & 1u ? at.w : at.z, t = a & 2u ? hi : lo;
      const int pair = ROPE == ROPE_NEOX ? 8 * ch + i : (i < 4 ? 4 * ch + i : D / 4 + 4 * ch + i - 4);
      return p.table + (size_t)t * (D / 2) + pair;
    };
    if (p.by_two) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float4 e = *reinterpret_cast<const float4*>(entry(i));
        c[i] = e.x;
        s[i] = e.y;
        c[i + 1] = e.z;
        s[i + 1] = e.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 e = *entry(i);
        c[i] = e.x;
        s[i] = e.y;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      c[i] = ok ? c[i] : NAN;
      s[i] = ok ? s[i] : NAN;
    }
  }
  template <bool INVERSE>
  __device__ __forceinline__ void turn(float (&v)[16]) const {
    if constexpr (ROPE == ROPE_NEOX) {
#pragma unroll
      for (int i = 0; i < 8; ++i) rotate_pair<INVERSE>(v[i], v[8 + i], c[i], s[i]);
    } else if constexpr (ROPE == ROPE_INTERLEAVED) {
#pragma unroll
      for (int i = 0; i < 8; ++i) rotate_pair<INVERSE>(v[2 * i], v[2 * i + 1], c[i], s[i]);
    }
  }
};

// The thread's 16 weights (fp32 or bf16; 1 without any).
__device__ __forceinline__ void load_weights(float (&w)[16], const void* p, bool w32, int d0, int d1) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = 1.f;
  } else if (w32) {
    RowChunk<true> r;
    r.load(p, d0, d1);
    r.get(w);
  } else {
    RowChunk<false> r;
    r.load(p, d0, d1);
    r.get(w);
  }
}

template <int D>
__device__ __forceinline__ float inv_rms(const float (&v)[16], float eps) {
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) ss = __builtin_fmaf(v[i], v[i], ss);
  return 1.f / sqrtf(__builtin_fmaf(row_sum<D>(ss), 1.f / D, eps));
}

// Row i of a workgroup at position n of batch b, or, of short sequences, of p.per
// batches from p.per * b on: b and n of the row, and whether there is one.  (One batch
// a workgroup leaves most of its threads idle there: H32/8 S1 D128, B512 forward 10.0 us
// against 4.3 and backward 25.9 against 8.8, B4096 45.2 against 19.5 and 169 against 28.5.)
__device__ __forceinline__ bool place(const QkNormParams& p, int i, int& b, int& n) {
  if (p.per == 1) return n < p.S;
  b = b * p.per + i / p.S;
  n = i % p.S;
  return i < p.per * p.S && b < p.B;
}

// ---------------------------------------------------------------- forward
// Workgroup: 256 / (D / 16) positions of one batch (or of several short ones) and HPT
// heads of q or k.  blockIdx: x position block, y head group (q's, then k's), z batches.
// INVERSE: the backward of a rotation without norm.
template <bool FP32, int D, int ROPE, int HPT, bool AXES, bool INVERSE>
__global__ __launch_bounds__(256) void qknorm_rope_kernel(QkNormParams p) {
  constexpr int TPR = D / 16, EB = FP32 ? 4 : 2;
  const int groups0 = (p.heads[0] + HPT - 1) / HPT;
  const int t = (int)blockIdx.y >= groups0;              // q or k
  const int hg = (int)blockIdx.y - (t ? groups0 : 0);
  const int i = threadIdx.x / TPR;
  int b = blockIdx.z, n = (int)blockIdx.x * (256 / TPR) + i;
  if (!place(p, i, b, n)) return;                        // (rows' lanes leave together)
  const int c = threadIdx.x % TPR, d0 = 8 * c, d1 = D / 2 + 8 * c;
  const int nh = p.heads[t], h0 = hg * HPT;
  const char* x = static_cast<const char*>(p.x[t]) + (b * p.xs[t][0] + n * p.xs[t][2]) * EB;

  [[maybe_unused]] RowPositions pos;
  if constexpr (AXES) pos.load(p, (size_t)b * p.S + n, (size_t)p.B * p.S);
  RowChunk<FP32> r[HPT];
#pragma unroll
  for (int j = 0; j < HPT; ++j) r[j].load(x + min(h0 + j, nh - 1) * p.xs[t][1] * EB, d0, d1);
  Angles<D, ROPE> a;
  if constexpr (AXES) a.load_axes(p, pos, c);
  else a.load(p.table, p.rows, p.positions ? p.positions[(size_t)b * p.S + n] : n, d0);
  float w[16];
  load_weights(w, p.w[t], p.w32, d0, d1);
  char* y = static_cast<char*>(p.y[t]) +
            (INVERSE ? b * p.ys[t][0] + n * p.ys[t][2] : (long long)(((size_t)b * nh * p.S + n) * D)) * EB;
  const long long sh = INVERSE ? p.ys[t][1] : (long long)p.S * D;   // elements from head to head
#pragma unroll
  for (int j = 0; j < HPT; ++j) {
    float v[16];
    r[j].get(v);
    if (!AXES || p.norm) {
      const float inv = inv_rms<D>(v, p.eps);
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] *= inv * w[i];
    }
    a.template turn<INVERSE>(v);
    r[j].put(v);
    if (h0 + j < nh) r[j].store(y + (h0 + j) * sh * EB, d0, d1);
  }
}

// ---------------------------------------------------------------- new tokens
// Rows of token n: its H queries normed and rotated into y[0] [T, H, D], its
// keys likewise and its values as they are into the pages, at the token's slot
// (page * page_size + place in the page).  A slot outside the pages, -1 among
// them, is not written.
template <bool FP32, int D, int ROPE, int HPT, bool AXES>
__global__ __launch_bounds__(256) void qknorm_append_kernel(QkNormParams p) {
  constexpr int TPR = D / 16, EB = FP32 ? 4 : 2;
  const int gq = (p.heads[0] + HPT - 1) / HPT, gk = (p.heads[1] + HPT - 1) / HPT;
  const int t = ((int)blockIdx.y >= gq) + ((int)blockIdx.y >= gq + gk);   // q, k or v
  const int hg = (int)blockIdx.y - (t > 0 ? gq : 0) - (t > 1 ? gk : 0);
  const int n = (int)blockIdx.x * (256 / TPR) + (int)threadIdx.x / TPR;
  if (n >= p.S) return;
  const int c = threadIdx.x % TPR, d0 = 8 * c, d1 = D / 2 + 8 * c;
  const int nh = t ? p.heads[1] : p.heads[0], h0 = hg * HPT;
  const char* x = static_cast<const char*>(p.x[t]) + n * p.xs[t][2] * EB;

  [[maybe_unused]] RowPositions pos;
  if constexpr (AXES) {
    if (t < 2) pos.load(p, n, p.S);
  }
  RowChunk<FP32> r[HPT];
#pragma unroll
  for (int j = 0; j < HPT; ++j) r[j].load(x + min(h0 + j, nh - 1) * p.xs[t][1] * EB, d0, d1);
  char* y;
  long long sh;          // elements from head to head
  bool keep = true;
  if (t == 0) {
    y = static_cast<char*>(p.y[0]) + (size_t)n * nh * D * EB;
    sh = D;
  } else {
    const long long slot = p.slots[n];
    keep = slot >= 0 && slot < p.nslots;
    const long long s = keep ? slot : 0;
    y = static_cast<char*>(p.y[t]) +
        ((s >> p.page_shift) * p.ys[t][0] + (s & ((1 << p.page_shift) - 1)) * p.ys[t][2]) * EB;
    sh = p.ys[t][1];
  }
  if (t < 2) {
    Angles<D, ROPE> a;
    if constexpr (AXES) a.load_axes(p, pos, c);
    else a.load(p.table, p.rows, ROPE != ROPE_NONE ? p.positions[n] : 0, d0);
    float w[16];
    load_weights(w, p.w[t], p.w32, d0, d1);
#pragma unroll
    for (int j = 0; j < HPT; ++j) {
      float v[16];
      r[j].get(v);
      const float inv = p.norm ? inv_rms<D>(v, p.eps) : 1.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] *= inv * w[i];
      a.template turn<false>(v);
      r[j].put(v);
    }
  }
#pragma unroll
  for (int j = 0; j < HPT; ++j)
    if (keep && h0 + j < nh) r[j].store(y + (h0 + j) * sh * EB, d0, d1);
}

// ---------------------------------------------------------------- backward
// Workgroup w of the tensor's n takes every n-th unit (batch, head group,
// position block) and leaves the sum of its rows' dy o xh in part[w]; the
// second launch adds those up in the order of w, so the weights' gradients
// are the same in every call (no atomics).
template <bool FP32, int D, int ROPE, int HPT, bool AXES>
__global__ __launch_bounds__(256) void qknorm_rope_bwd_kernel(QkNormParams p) {
  constexpr int TPR = D / 16, R = 256 / TPR, EB = FP32 ? 4 : 2;
  __shared__ float red[16][256];
  const int t = (int)blockIdx.x >= p.wgs[0];
  const int wg = (int)blockIdx.x - (t ? p.wgs[0] : 0), nwg = p.wgs[t];
  const int c = threadIdx.x % TPR, d0 = 8 * c, d1 = D / 2 + 8 * c;
  const int nh = p.heads[t], groups = (nh + HPT - 1) / HPT, nblk = (p.S + R - 1) / R;
  float w[16], dw[16];
  load_weights(w, p.w[t], p.w32, d0, d1);
#pragma unroll
  for (int i = 0; i < 16; ++i) dw[i] = 0.f;
  const int units = (p.B + p.per - 1) / p.per * groups * nblk;
  for (int u = wg; u < units; u += nwg) {
    const int hb = u / nblk, h0 = (hb % groups) * HPT, i = threadIdx.x / TPR;
    int b = hb / groups, n = u % nblk * R + i;
    if (place(p, i, b, n)) {   // (rows' lanes together)
      [[maybe_unused]] RowPositions pos;
      if constexpr (AXES) pos.load(p, (size_t)b * p.S + n, (size_t)p.B * p.S);
      const char* x = static_cast<const char*>(p.x[t]) + (b * p.xs[t][0] + n * p.xs[t][2]) * EB;
      const char* dy = static_cast<const char*>(p.dy[t]) + ((size_t)b * nh * p.S + n) * D * EB;
      char* dx = static_cast<char*>(p.y[t]) + (b * p.ys[t][0] + n * p.ys[t][2]) * EB;
      RowChunk<FP32> rx[HPT], rd[HPT];
#pragma unroll
      for (int j = 0; j < HPT; ++j) {
        const int h = min(h0 + j, nh - 1);
        rx[j].load(x + h * p.xs[t][1] * EB, d0, d1);
        rd[j].load(dy + (size_t)h * p.S * D * EB, d0, d1);
      }
      Angles<D, ROPE> a;
      if constexpr (AXES) a.load_axes(p, pos, c);
      else a.load(p.table, p.rows, p.positions ? p.positions[(size_t)b * p.S + n] : n, d0);
#pragma unroll
      for (int j = 0; j < HPT; ++j) {
        if (h0 + j >= nh) break;
        float v[16], g[16];
        rx[j].get(v);
        rd[j].get(g);
        a.template turn<true>(g);
        const float inv = inv_rms<D>(v, p.eps);
        float gx = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          v[i] *= inv;                                   // xh
          dw[i] = __builtin_fmaf(g[i], v[i], dw[i]);
          g[i] *= w[i];
          gx = __builtin_fmaf(g[i], v[i], gx);
        }
        gx = row_sum<D>(gx) * (1.f / D);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = inv * __builtin_fmaf(-v[i], gx, g[i]);
        rx[j].put(v);
        rx[j].store(dx + (h0 + j) * p.ys[t][1] * EB, d0, d1);
      }
    }
  }
  if (!p.part) return;
#pragma unroll
  for (int i = 0; i < 16; ++i) red[i][threadIdx.x] = dw[i];
  __syncthreads();
  if ((int)threadIdx.x < D) {
    const int d = threadIdx.x, half = d / (D / 2), cc = (d % (D / 2)) / 8, e = 8 * half + d % 8;
    float sum = 0.f;
    for (int i = 0; i < R; ++i) sum += red[e][cc + TPR * i];
    p.part[((size_t)(t ? p.wgs[0] : 0) + wg) * D + d] = sum;
  }
}

// dw of q (blockIdx.y 0) or k: 32 dims a workgroup, 32 threads a dim.
template <int D>
__global__ __launch_bounds__(1024) void qknorm_dw_kernel(QkNormParams p) {
  __shared__ float red[32][33];
  const int t = blockIdx.y, lane = threadIdx.x & 31, row = threadIdx.x >> 5, d = 32 * blockIdx.x + lane;
  const float* part = p.part + (size_t)(t ? p.wgs[0] : 0) * D + d;
  float sum = 0.f;
  int i = row;
  for (; i + 7 * 32 < p.wgs[t]; i += 8 * 32) {   // eight loads in flight
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = part[(size_t)(i + 32 * j) * D];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += x[j];
  }
  for (; i < p.wgs[t]; i += 32) sum += part[(size_t)i * D];
  red[row][lane] = sum;
  __syncthreads();
  if (row == 0) {
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) sum += red[i][lane];
    if (p.w32) static_cast<float*>(p.dw[t])[d] = sum;
    else static_cast<uint16_t*>(p.dw[t])[d] = (uint16_t)(pack_bf16(sum, 0.f) & 0xffffu);
  }
}

// ---------------------------------------------------------------- launch
template <bool FP32, int D, int ROPE, bool AXES>
int qknorm_launch_one(int what, const QkNormParams& p0, hipStream_t st) {
  constexpr int R = 256 / (D / 16);
  QkNormParams p = p0;
  p.per = qknorm_per(p.S, D);
  const int nb = (p.B + p.per - 1) / p.per;
  // Heads a thread takes: more share its cos/sin and weights and keep more loads in
  // flight, one is done sooner.  us with 1 / 2 / 4 heads, bf16: append of 4500 tokens
  // H64/8 D128 46 / 43 / 40 (3384 workgroups with 4); backward B1 H32/8 S8192 D128 57.8 /
  // 54.8 / 55.9; captured in a graph, append H32/8 D128 with 1 / 4 heads of 1 token 2.5 /
  // 3.8, 128 2.9 / 4.0, 512 4.1 / 4.7, 1000 5.8 / 6.4 (384 workgroups with 4).
  constexpr int HPT = FP32 ? 2 : 4;
  const unsigned nblk = (unsigned)((p.S + R - 1) / R);
  if (what == QKNORM_BWD) {
    hipLaunchKernelGGL((qknorm_rope_bwd_kernel<FP32, D, ROPE, QKNORM_BWD_HPT, AXES>), dim3((unsigned)(p.wgs[0] + p.wgs[1])),
                       dim3(256), 0, st, p);
    if (p.part)
      hipLaunchKernelGGL((qknorm_dw_kernel<D>), dim3(D / 32, p.heads[1] ? 2 : 1), dim3(1024), 0, st, p);
    return hipGetLastError() == hipSuccess ? 0 : -3;
  }
  const int nk = what == QKNORM_APPEND ? 2 : 1;   // key tensors: the values go the keys' way
  auto groups = [&](int hpt) { return (unsigned)((p.heads[0] + hpt - 1) / hpt + nk * ((p.heads[1] + hpt - 1) / hpt)); };
  const bool one = (long long)nblk * groups(HPT) * nb < 512;
  const dim3 grid(nblk, groups(one ? 1 : HPT), (unsigned)nb);
  if (what == QKNORM_APPEND) {
    if (one) hipLaunchKernelGGL((qknorm_append_kernel<FP32, D, ROPE, 1, AXES>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((qknorm_append_kernel<FP32, D, ROPE, HPT, AXES>), grid, dim3(256), 0, st, p);
  } else if (what == QKNORM_FWD) {
    if (one) hipLaunchKernelGGL((qknorm_rope_kernel<FP32, D, ROPE, 1, AXES, false>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((qknorm_rope_kernel<FP32, D, ROPE, HPT, AXES, false>), grid, dim3(256), 0, st, p);
  } else if constexpr (AXES) {   // QKNORM_UNTURN
    if (one) hipLaunchKernelGGL((qknorm_rope_kernel<FP32, D, ROPE, 1, true, true>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((qknorm_rope_kernel<FP32, D, ROPE, HPT, true, true>), grid, dim3(256), 0, st, p);
  }
  return hipGetLastError() == hipSuccess ? 0 : -3;
}

}  // namespace af
