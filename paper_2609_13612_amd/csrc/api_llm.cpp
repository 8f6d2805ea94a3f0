// C-ABI entry points of include/attnfuse_llm.h: argument validation and dispatch
// to the kernel launchers.  Every argument is checked before the first HIP call;
// nothing here allocates, synchronises, throws or keeps state.
#include "attnfuse_llm.h"

#include <hip/hip_runtime.h>

#include <initializer_list>

#include "checks.hpp"
#include "launch.hpp"

using namespace af_api;

namespace {

constexpr int kMaxHeads = 1 << 14;

int element_bytes(int dtype) { return dtype == AF_DTYPE_FP32 ? 4 : 2; }

// Strides of an input (any >= 0) or an output (out: at least D apart in each
// dimension longer than 1), in whole 16-byte chunks.
struct Dim {
  long long n, stride;
};

bool strides_ok(std::initializer_list<Dim> dims, int D, int dtype, bool out) {
  for (const Dim& d : dims) {
    if (d.stride < 0 || d.stride * element_bytes(dtype) % 16 != 0) return false;
    if (d.stride > (1LL << 40)) return false;   // (offsets stay inside 64 bits)
    if (out && d.n > 1 && d.stride < D) return false;
  }
  return true;
}

bool any_alias(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins) {
  for (const void* o : outs)
    for (const void* i : ins)
      if (o && o == i) return true;
  return false;
}

bool outs_alias(std::initializer_list<const void*> outs) {
  for (auto a = outs.begin(); a != outs.end(); ++a)
    for (auto b = a + 1; b != outs.end(); ++b)
      if (*a && *a == *b) return true;
  return false;
}

int check_rope(int rope, float theta) {
  if (rope != AF_ROPE_NONE && rope != AF_ROPE_NEOX && rope != AF_ROPE_INTERLEAVED) return AF_ERR_INVALID_ARG;
  if (rope != AF_ROPE_NONE && !(std::isfinite(theta) && theta > 0.f)) return AF_ERR_INVALID_ARG;
  return AF_OK;
}

// Sizes of a norm call; H_kv 0: no keys.
bool qknorm_sizes(int B, int H, int H_kv, int S, int D, int dtype) {
  return B >= 1 && B <= kMaxHeads && H >= 1 && H <= kMaxHeads && H_kv >= 0 && H_kv <= kMaxHeads && S >= 1 && S <= kMaxS &&
         D >= 2 && D % 2 == 0 && (dtype == AF_DTYPE_BF16 || dtype == AF_DTYPE_FP32);
}

// Workgroups of the backward for q and k: one per unit (head group, position
// block), or about 1024 that share them, four for each CU (B1 H32/8 S8192 D128 with
// 768 / 1024 / 2048: 55.4 / 54.8 / 58.0 us; their sums are a second launch's work).
bool qknorm_wgs(int B, int H, int H_kv, int S, int D, int (&wgs)[2]) {
  const long long hpt = af::QKNORM_BWD_HPT, rows = 256 / (D / 16);
  const long long per = af::qknorm_per(S, D), blocks = (S + rows - 1) / rows * ((B + per - 1) / per);
  const long long uq = blocks * ((H + hpt - 1) / hpt), uk = blocks * ((H_kv + hpt - 1) / hpt), all = uq + uk, most = 1024;
  if (all >= (1LL << 31)) return false;
  const long long q = all <= most ? uq : uq * most / all, k = all <= most ? uk : most - q;
  wgs[0] = (int)(q < 1 ? 1 : q);
  wgs[1] = (int)(H_kv && k < 1 ? 1 : k);
  return true;
}

// ---------------------------------------------------------------- positions of several axes
// Which axis each of the D / 2 pairs turns by (n 0: positions of one axis for all).
struct Axes {
  int n = 0;
  uint8_t axis[64], rung[64], size[64];   // of a pair: its axis, how many pairs of that axis come before it, and the axis's pairs

  void fill(af::QkNormParams& p, int D) const {
    if (!n) return;
    p.axes = n;
    p.by_two = true;
    for (int i = 0; i < D / 2; ++i) {
      p.axis[i / 16] |= (uint32_t)axis[i] << (2 * (i % 16));
      p.by_two = p.by_two && axis[i] == axis[i & ~1];
    }
  }
};

int check_axes(int axes, const int* sections, int order, int D, Axes& out) {
  if (axes < 1 || axes > 4 || !sections || D < 2 || D % 2 != 0) return AF_ERR_INVALID_ARG;
  if (order != AF_SECTIONS_BLOCKS && order != AF_SECTIONS_TURNS) return AF_ERR_INVALID_ARG;
  long long sum = 0;
  for (int a = 0; a < axes; ++a) {
    if (sections[a] < 1 || sections[a] > D / 2) return AF_ERR_INVALID_ARG;
    sum += sections[a];
  }
  if (sum != D / 2) return AF_ERR_INVALID_ARG;
  if (!supported_d(D)) return AF_ERR_UNSUPPORTED;
  out.n = axes;
  int i = 0;
  auto give = [&](int a, int r) {
    out.axis[i] = (uint8_t)a;
    out.rung[i] = (uint8_t)r;
    out.size[i++] = (uint8_t)sections[a];
  };
  if (order == AF_SECTIONS_BLOCKS) {
    for (int a = 0; a < axes; ++a)
      for (int r = 0; r < sections[a]; ++r) give(a, r);
  } else {
    for (int r = 0; r < D / 2; ++r)
      for (int a = 0; a < axes; ++a)
        if (r < sections[a]) give(a, r);
  }
  return AF_OK;
}

// Page size -> shift, or -1 where the kernels have none.
int page_shift_of(int page_size) {
  for (int s = 4; s <= 20; ++s)
    if ((1 << s) == page_size) return s;
  return -1;
}

// ---------------------------------------------------------------- decode
struct PagedLayout {
  int hgroups, nsplit;
  bool by_length;
  size_t ml, acc, total;
};

// Workgroups that share a sequence's visible 32-key tiles for a head group: one for
// each CU over the whole batch, while every wave of theirs has a tile; then twice
// as many, while a share keeps 32 tiles (eight for each wave) and there are fewer
// than 1024, so that CUs with short sequences take more of the long ones.  A round of
// tiles takes a lone wave 1.4 us, 124 workgroups saturate the memory, and the
// second launch costs 4 us.  us with 1 / 2 / 4 / 8 / 16 / 32 shares, and those taken:
//   B1 H32/8 D128 4096 keys: 49 / 32 / 21 / 15.5 / 12.2 / 11.1, 32;  B8 H32/8 8192: 102 / 64 / 53 / 52 / 54 / 59, 8
//   B8 H64/8 lengths 8k to 32k: 356 / 198 / 137 / 129 / 123 / 129, 16;  B32 H32/8 window 1024: 26 / 29 / 32 / 42, 1
//   B48 H12 D64 3500 keys: 117 / 106 / 100 / 106, 2;  B70 H32/8 lengths to 1500: 60 / 68 / 73 / 88, 1
PagedLayout paged_layout(int B, int H, int H_kv, int S, int D, int window, int sinks) {
  PagedLayout L{};
  L.hgroups = (H / H_kv + 31) / 32;
  long long tiles = (S + 31) / 32;
  if (window > 0) {
    const long long most = (window + 30LL) / 32 + 1 + (sinks + 31LL) / 32;   // a window's edges cut two tiles
    tiles = tiles < most ? tiles : most;
  }
  const long long units = (long long)B * H_kv * L.hgroups;
  long long n = units < 256 ? (256 + units - 1) / units : 1;
  while (n > 1 && tiles < 4 * n) --n;
  while (units * n < 1024 && tiles >= 64 * n) n *= 2;
  L.nsplit = (int)n;
  // The longest sequences first, where more workgroups run than are resident (two to a
  // CU) and each is long enough to pay for the ranking (1 to 2 us of its start).  us
  // without / with, lengths from a quarter on: B32 H32/8 to 8192 139 / 130, B8 H64/8 to
  // 32768 133 / 122, B20 H16/16 to 3000 68 / 63, B64 H32/8 to 4000 134 / 125; not taken:
  // B48 H12 D64 to 1000 25.5 / 25.7 and to 3500 73.3 / 73.4.  Even lengths: B32 184.5 / 185.7.
  L.by_length = B > 1 && B <= 64 && units * n > 512 && tiles * D >= 4096 * n;
  const size_t parts = (size_t)B * H * L.nsplit;
  L.ml = 0;
  L.acc = align256(parts * 2 * sizeof(float));
  L.total = L.acc + align256(parts * D * sizeof(float));
  return L;
}

bool decode_sizes(int B, int H, int H_kv, int S, int D) {
  return B >= 1 && B < (1 << 16) && H >= 1 && H <= kMaxHeads && H_kv >= 1 && H % H_kv == 0 && S >= 1 && S <= kMaxS && D >= 2 && D % 2 == 0 &&
         (long long)B * H * ((S + 63) / 64) < (1LL << 31);
}

// The checks and the launch that both decode calls share; p holds the cache.
int decode_impl(af::PagedParams& p, const void* Q, const void* K, const void* V, const int* cache_lens, void* O, float* LSE,
                void* workspace, size_t workspace_bytes, int B, int H, int H_kv, int S, int D, int rope, float rope_theta,
                const float* rope_table, int rope_table_rows, int mask, int window, int sinks, const float* alibi_slopes,
                float softmax_scale, void* stream) {
  if (!Q || !K || !V || !O || !LSE || !workspace) return AF_ERR_INVALID_ARG;
  for (const void* x : {Q, K, V, (const void*)O, (const void*)workspace})
    if (!aligned16(x)) return AF_ERR_INVALID_ARG;
  if (!aligned4(LSE) || !aligned4(cache_lens) || !aligned4(p.table) || !aligned4(alibi_slopes)) return AF_ERR_INVALID_ARG;
  if (any_alias({O, LSE, workspace}, {Q, K, V, cache_lens, p.table, alibi_slopes}) || outs_alias({O, LSE, workspace}))
    return AF_ERR_INVALID_ARG;
  if (!decode_sizes(B, H, H_kv, S, D)) return AF_ERR_INVALID_ARG;
  int rc = check_rope(rope, rope_theta);
  if (rc != AF_OK || (rc = check_attn(mask, window, softmax_scale)) != AF_OK) return rc;
  if (sinks < 0 || (sinks > 0 && mask != AF_MASK_SLIDING_WINDOW)) return AF_ERR_INVALID_ARG;
  const void* outs[] = {O, LSE, workspace};
  if ((rc = check_table(rope, rope_table, rope_table_rows, S, outs, 3)) != AF_OK) return rc;
  if (mask != AF_MASK_SLIDING_WINDOW) window = 0;
  window = window < S ? window : S;
  sinks = sinks < S ? sinks : S;
  const PagedLayout L = paged_layout(B, H, H_kv, S, D, window, sinks);
  if (workspace_bytes < L.total) return AF_ERR_INVALID_ARG;
  if (!supported_d(D) || (sinks > 0 && alibi_slopes)) return AF_ERR_UNSUPPORTED;

  p.q = Q; p.k = K; p.v = V; p.lens = cache_lens;
  p.o = O; p.lse = LSE;
  p.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + L.ml);
  p.part_acc = reinterpret_cast<float*>(static_cast<char*>(workspace) + L.acc);
  p.B = B; p.H = H; p.Hkv = H_kv; p.S = S;
  p.window = window; p.sinks = sinks;
  p.by_length = cache_lens && L.by_length;
  p.nsplit = L.nsplit; p.G = H / H_kv; p.hgroups = L.hgroups;
  p.slopes = alibi_slopes;
  p.scale = softmax_scale;
  p.rope = reinterpret_cast<const float2*>(rope_table);
  return map_launch(af::launch_decode_paged(D, rope, alibi_slopes != nullptr, p, static_cast<hipStream_t>(stream)));
}

// attnfuse_qknorm_rope, or with axes.n > 0 attnfuse_qknorm_axes.
int qknorm_fwd(const void* Q, const void* K, void* Qr, void* Kr, const void* q_weight, const void* k_weight,
               int weight_dtype, int norm, float eps,
               long long q_stride_b, long long q_stride_h, long long q_stride_s,
               long long k_stride_b, long long k_stride_h, long long k_stride_s,
               int B, int H, int H_kv, int S, int D, int dtype,
               int rope, float rope_theta, const float* rope_table, int rope_table_rows,
               const int* positions, const Axes& axes, void* stream) {
  if (!Q || !Qr || !K != !Kr) return AF_ERR_INVALID_ARG;
  if (!K) H_kv = 0;
  else if (H_kv < 1) return AF_ERR_INVALID_ARG;
  for (const void* x : {Q, K, (const void*)Qr, (const void*)Kr, q_weight, k_weight})
    if (!aligned16(x)) return AF_ERR_INVALID_ARG;
  if (!qknorm_sizes(B, H, H_kv, S, D, dtype) || (norm && !(std::isfinite(eps) && eps >= 0.f))) return AF_ERR_INVALID_ARG;
  if (!norm && (q_weight || k_weight)) return AF_ERR_INVALID_ARG;
  if (weight_dtype != AF_DTYPE_BF16 && weight_dtype != AF_DTYPE_FP32) return AF_ERR_INVALID_ARG;
  if (!strides_ok({{B, q_stride_b}, {H, q_stride_h}, {S, q_stride_s}}, D, dtype, false)) return AF_ERR_INVALID_ARG;
  if (K && !strides_ok({{B, k_stride_b}, {H_kv, k_stride_h}, {S, k_stride_s}}, D, dtype, false)) return AF_ERR_INVALID_ARG;
  if (any_alias({Qr, Kr}, {q_weight, k_weight, positions}) || any_alias({Qr}, {K}) || any_alias({Kr}, {Q}) ||
      outs_alias({Qr, Kr}))
    return AF_ERR_INVALID_ARG;
  // in place: every row where it was
  const auto same = [&](int heads, long long sb, long long sh, long long ss) {
    return (S == 1 || ss == D) && (heads == 1 || sh == (long long)S * D) && (B == 1 || sb == (long long)heads * S * D);
  };
  if (Qr == Q && !same(H, q_stride_b, q_stride_h, q_stride_s)) return AF_ERR_INVALID_ARG;
  if (K && Kr == K && !same(H_kv, k_stride_b, k_stride_h, k_stride_s)) return AF_ERR_INVALID_ARG;
  int rc = check_rope(rope, rope_theta);
  if (rc != AF_OK) return rc;
  if (axes.n && (rope == AF_ROPE_NONE || !positions)) return AF_ERR_INVALID_ARG;
  const void* outs[] = {Qr, Kr};
  if ((rc = check_table(rope, rope_table, rope_table_rows, positions ? 1 : S, outs, 2)) != AF_OK) return rc;
  if (!aligned4(positions)) return AF_ERR_INVALID_ARG;
  if (!supported_d(D)) return AF_ERR_UNSUPPORTED;

  af::QkNormParams p{};
  p.x[0] = Q; p.x[1] = K;
  p.y[0] = Qr; p.y[1] = Kr;
  p.w[0] = q_weight; p.w[1] = k_weight;
  p.w32 = weight_dtype == AF_DTYPE_FP32;
  p.xs[0][0] = q_stride_b; p.xs[0][1] = q_stride_h; p.xs[0][2] = q_stride_s;
  p.xs[1][0] = k_stride_b; p.xs[1][1] = k_stride_h; p.xs[1][2] = k_stride_s;
  p.heads[0] = H; p.heads[1] = H_kv;
  p.B = B; p.S = S; p.eps = eps;
  p.norm = norm != 0;
  axes.fill(p, D);
  p.table = reinterpret_cast<const float2*>(rope_table);
  p.rows = rope_table_rows;
  p.positions = rope != AF_ROPE_NONE ? positions : nullptr;
  return map_launch(af::launch_qknorm(af::QKNORM_FWD, dtype == AF_DTYPE_FP32, D, rope, p, static_cast<hipStream_t>(stream)));
}

// attnfuse_qknorm_rope_bwd, or with axes.n > 0 attnfuse_qknorm_axes_bwd under a norm.
int qknorm_bwd(const void* Q, const void* K, const void* dQr, const void* dKr, void* dQ, void* dK,
               void* dq_weight, void* dk_weight, const void* q_weight, const void* k_weight,
               int weight_dtype, float eps,
               long long q_stride_b, long long q_stride_h, long long q_stride_s,
               long long k_stride_b, long long k_stride_h, long long k_stride_s,
               long long dq_stride_b, long long dq_stride_h, long long dq_stride_s,
               long long dk_stride_b, long long dk_stride_h, long long dk_stride_s,
               void* workspace, size_t workspace_bytes,
               int B, int H, int H_kv, int S, int D, int dtype,
               int rope, float rope_theta, const float* rope_table, int rope_table_rows,
               const int* positions, const Axes& axes, void* stream) {
  if (!Q || !dQr || !dQ || !K != !dKr || !K != !dK) return AF_ERR_INVALID_ARG;
  if (!K) { H_kv = 0; dk_weight = nullptr; }
  else if (H_kv < 1) return AF_ERR_INVALID_ARG;
  const bool weights = dq_weight != nullptr;
  if (K && !dk_weight != !dq_weight) return AF_ERR_INVALID_ARG;
  if (!weights) workspace = nullptr;
  else if (!workspace) return AF_ERR_INVALID_ARG;
  for (const void* x : {Q, K, dQr, dKr, (const void*)dQ, (const void*)dK, q_weight, k_weight, (const void*)workspace})
    if (!aligned16(x)) return AF_ERR_INVALID_ARG;
  if (!aligned4(dq_weight) || !aligned4(dk_weight) || !aligned4(positions)) return AF_ERR_INVALID_ARG;
  if (!qknorm_sizes(B, H, H_kv, S, D, dtype) || !(std::isfinite(eps) && eps >= 0.f)) return AF_ERR_INVALID_ARG;
  if (weight_dtype != AF_DTYPE_BF16 && weight_dtype != AF_DTYPE_FP32) return AF_ERR_INVALID_ARG;
  if (!strides_ok({{B, q_stride_b}, {H, q_stride_h}, {S, q_stride_s}}, D, dtype, false) ||
      !strides_ok({{B, dq_stride_b}, {H, dq_stride_h}, {S, dq_stride_s}}, D, dtype, true))
    return AF_ERR_INVALID_ARG;
  if (K && (!strides_ok({{B, k_stride_b}, {H_kv, k_stride_h}, {S, k_stride_s}}, D, dtype, false) ||
            !strides_ok({{B, dk_stride_b}, {H_kv, dk_stride_h}, {S, dk_stride_s}}, D, dtype, true)))
    return AF_ERR_INVALID_ARG;
  if (any_alias({dQ, dK, dq_weight, dk_weight, workspace}, {Q, K, dQr, dKr, q_weight, k_weight, positions, rope_table}) ||
      outs_alias({dQ, dK, dq_weight, dk_weight, workspace}))
    return AF_ERR_INVALID_ARG;
  int rc = check_rope(rope, rope_theta);
  if (rc != AF_OK) return rc;
  if (axes.n && (rope == AF_ROPE_NONE || !positions)) return AF_ERR_INVALID_ARG;
  if ((rc = check_table(rope, rope_table, rope_table_rows, positions ? 1 : S, nullptr, 0)) != AF_OK) return rc;
  if (!supported_d(D)) return AF_ERR_UNSUPPORTED;
  af::QkNormParams p{};
  if (!qknorm_wgs(B, H, H_kv, S, D, p.wgs)) return AF_ERR_INVALID_ARG;
  if (weights && workspace_bytes < (size_t)(p.wgs[0] + p.wgs[1]) * D * sizeof(float)) return AF_ERR_INVALID_ARG;

  p.x[0] = Q; p.x[1] = K;
  p.dy[0] = dQr; p.dy[1] = dKr;
  p.y[0] = dQ; p.y[1] = dK;
  p.w[0] = q_weight; p.w[1] = k_weight;
  p.dw[0] = dq_weight; p.dw[1] = dk_weight;
  p.w32 = weight_dtype == AF_DTYPE_FP32;
  p.xs[0][0] = q_stride_b; p.xs[0][1] = q_stride_h; p.xs[0][2] = q_stride_s;
  p.xs[1][0] = k_stride_b; p.xs[1][1] = k_stride_h; p.xs[1][2] = k_stride_s;
  p.ys[0][0] = dq_stride_b; p.ys[0][1] = dq_stride_h; p.ys[0][2] = dq_stride_s;
  p.ys[1][0] = dk_stride_b; p.ys[1][1] = dk_stride_h; p.ys[1][2] = dk_stride_s;
  p.heads[0] = H; p.heads[1] = H_kv;
  p.B = B; p.S = S; p.eps = eps;
  p.norm = true;
  axes.fill(p, D);
  p.table = reinterpret_cast<const float2*>(rope_table);
  p.rows = rope_table_rows;
  p.positions = rope != AF_ROPE_NONE ? positions : nullptr;
  p.part = static_cast<float*>(workspace);
  return map_launch(af::launch_qknorm(af::QKNORM_BWD, dtype == AF_DTYPE_FP32, D, rope, p, static_cast<hipStream_t>(stream)));
}

// The backward of attnfuse_qknorm_axes without norm: dx = R^T dout.
int qknorm_unturn(const void* dQr, const void* dKr, void* dQ, void* dK,
                  long long dq_stride_b, long long dq_stride_h, long long dq_stride_s,
                  long long dk_stride_b, long long dk_stride_h, long long dk_stride_s,
                  int B, int H, int H_kv, int S, int D, int dtype,
                  int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                  const int* positions, const Axes& axes, void* stream) {
  if (!dQr || !dQ || !dKr != !dK) return AF_ERR_INVALID_ARG;
  if (!dK) H_kv = 0;
  else if (H_kv < 1) return AF_ERR_INVALID_ARG;
  for (const void* x : {dQr, dKr, (const void*)dQ, (const void*)dK})
    if (!aligned16(x)) return AF_ERR_INVALID_ARG;
  if (!qknorm_sizes(B, H, H_kv, S, D, dtype)) return AF_ERR_INVALID_ARG;
  if (!strides_ok({{B, dq_stride_b}, {H, dq_stride_h}, {S, dq_stride_s}}, D, dtype, true)) return AF_ERR_INVALID_ARG;
  if (dK && !strides_ok({{B, dk_stride_b}, {H_kv, dk_stride_h}, {S, dk_stride_s}}, D, dtype, true)) return AF_ERR_INVALID_ARG;
  if (any_alias({dQ, dK}, {dQr, dKr, positions}) || outs_alias({dQ, dK})) return AF_ERR_INVALID_ARG;
  int rc = check_rope(rope, rope_theta);
  if (rc != AF_OK) return rc;
  if (rope == AF_ROPE_NONE || !positions || !aligned4(positions)) return AF_ERR_INVALID_ARG;
  const void* outs[] = {dQ, dK};
  if ((rc = check_table(rope, rope_table, rope_table_rows, 1, outs, 2)) != AF_OK) return rc;
  if (!supported_d(D)) return AF_ERR_UNSUPPORTED;

  af::QkNormParams p{};
  p.x[0] = dQr; p.x[1] = dKr;
  p.y[0] = dQ; p.y[1] = dK;
  const int heads[2] = {H, H_kv};
  for (int t = 0; t < 2; ++t) {
    p.xs[t][0] = (long long)heads[t] * S * D; p.xs[t][1] = (long long)S * D; p.xs[t][2] = D;
  }
  p.ys[0][0] = dq_stride_b; p.ys[0][1] = dq_stride_h; p.ys[0][2] = dq_stride_s;
  p.ys[1][0] = dk_stride_b; p.ys[1][1] = dk_stride_h; p.ys[1][2] = dk_stride_s;
  p.heads[0] = H; p.heads[1] = H_kv;
  p.B = B; p.S = S;
  axes.fill(p, D);
  p.table = reinterpret_cast<const float2*>(rope_table);
  p.rows = rope_table_rows;
  p.positions = positions;
  return map_launch(
      af::launch_qknorm(af::QKNORM_UNTURN, dtype == AF_DTYPE_FP32, D, rope, p, static_cast<hipStream_t>(stream)));
}

// attnfuse_qknorm_rope_append, or with axes.n > 0 attnfuse_qknorm_axes_append.
int qknorm_append(const void* Q, const void* K, const void* V, void* Qr, void* K_pages, void* V_pages,
                  const long long* slots, const void* q_weight, const void* k_weight, int weight_dtype,
                  int norm, float eps,
                  long long q_stride_t, long long q_stride_h, long long k_stride_t, long long k_stride_h,
                  long long v_stride_t, long long v_stride_h,
                  long long kp_stride_p, long long kp_stride_h, long long kp_stride_s,
                  long long vp_stride_p, long long vp_stride_h, long long vp_stride_s,
                  int T, int H, int H_kv, int D, int num_pages, int page_size, int dtype,
                  int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                  const int* positions, const Axes& axes, void* stream) {
  if (!Q || !K || !V || !Qr || !K_pages || !V_pages || !slots) return AF_ERR_INVALID_ARG;
  for (const void* x : {Q, K, V, (const void*)Qr, (const void*)K_pages, (const void*)V_pages, q_weight, k_weight})
    if (!aligned16(x)) return AF_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(slots) & 7u) != 0 || !aligned4(positions)) return AF_ERR_INVALID_ARG;
  if (!qknorm_sizes(1, H, H_kv, T, D, dtype) || H_kv < 1 || num_pages < 1 || page_size < 1) return AF_ERR_INVALID_ARG;
  if ((long long)num_pages * page_size >= (1LL << 31)) return AF_ERR_INVALID_ARG;
  if (norm ? !(std::isfinite(eps) && eps >= 0.f) : q_weight || k_weight) return AF_ERR_INVALID_ARG;
  if (weight_dtype != AF_DTYPE_BF16 && weight_dtype != AF_DTYPE_FP32) return AF_ERR_INVALID_ARG;
  if (!strides_ok({{T, q_stride_t}, {H, q_stride_h}}, D, dtype, false) ||
      !strides_ok({{T, k_stride_t}, {H_kv, k_stride_h}, {T, v_stride_t}, {H_kv, v_stride_h}}, D, dtype, false) ||
      !strides_ok({{num_pages, kp_stride_p}, {H_kv, kp_stride_h}, {page_size, kp_stride_s}}, D, dtype, true) ||
      !strides_ok({{num_pages, vp_stride_p}, {H_kv, vp_stride_h}, {page_size, vp_stride_s}}, D, dtype, true))
    return AF_ERR_INVALID_ARG;
  if (any_alias({Qr, K_pages, V_pages}, {Q, K, V, q_weight, k_weight, slots, positions}) ||
      outs_alias({Qr, K_pages, V_pages}))
    return AF_ERR_INVALID_ARG;
  int rc = check_rope(rope, rope_theta);
  if (rc != AF_OK) return rc;
  if (rope != AF_ROPE_NONE ? !positions : axes.n > 0) return AF_ERR_INVALID_ARG;
  const void* outs[] = {Qr, K_pages, V_pages};
  if ((rc = check_table(rope, rope_table, rope_table_rows, 1, outs, 3)) != AF_OK) return rc;
  const int shift = page_shift_of(page_size);
  if (!supported_d(D) || shift < 0) return AF_ERR_UNSUPPORTED;

  af::QkNormParams p{};
  p.x[0] = Q; p.x[1] = K; p.x[2] = V;
  p.y[0] = Qr; p.y[1] = K_pages; p.y[2] = V_pages;
  p.w[0] = q_weight; p.w[1] = k_weight;
  p.w32 = weight_dtype == AF_DTYPE_FP32;
  p.norm = norm != 0;
  p.eps = eps;
  p.xs[0][1] = q_stride_h; p.xs[0][2] = q_stride_t;
  p.xs[1][1] = k_stride_h; p.xs[1][2] = k_stride_t;
  p.xs[2][1] = v_stride_h; p.xs[2][2] = v_stride_t;
  p.ys[1][0] = kp_stride_p; p.ys[1][1] = kp_stride_h; p.ys[1][2] = kp_stride_s;
  p.ys[2][0] = vp_stride_p; p.ys[2][1] = vp_stride_h; p.ys[2][2] = vp_stride_s;
  p.heads[0] = H; p.heads[1] = H_kv;
  p.B = 1; p.S = T;
  axes.fill(p, D);
  p.table = reinterpret_cast<const float2*>(rope_table);
  p.rows = rope_table_rows;
  p.positions = rope != AF_ROPE_NONE ? positions : nullptr;
  p.slots = slots;
  p.nslots = (long long)num_pages * page_size;
  p.page_shift = shift;
  return map_launch(
      af::launch_qknorm(af::QKNORM_APPEND, dtype == AF_DTYPE_FP32, D, rope, p, static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------- new tokens over pages
struct TilesLayout {
  int nw, nsp, nso, prefix_items, own_items;
  bool joined, by_length;
  size_t acc, total;   // workspace: (max, sum) pairs, from acc on the accumulators
};

// How the work of T queries of B sequences (one_each: one of each) against up to S own
// keys and P of the prefix is cut (paged_tiles.hip says what is apart and joined): the
// waves to a workgroup and the numbers of shares with the least estimated time, from what a
// workgroup's tile takes, what starting and ending one takes, the rounds of workgroups that
// are resident together, the bytes of K and V at the rate they are read with, and the
// partials' bytes.  us with the prefix's tiles in n shares (own tiles in one), n taken first:
//   H32/8 D128: 4 sequences behind 500 keys 4 10.9, 2 10.9, 1 12.1;  32 behind 32768, own to 1024 32 58, 24 59, 16 67, 48 65;
//   64 behind 16384 16 49, 12 53, 20 53, 8 61;  256 behind 8192 of H64/8 2 130, 3 141, 4 156;
//   760 tokens of 4 behind 16384 in eight waves 5 221, 4 255, in four 4 227, 2 244;
//   881 tokens of 24 behind 16384 in eight waves 2 252, in four 264;  H12 D64, 24 behind 5001 8 14.7, 16 15.5, 24 17.6
// Joined where the rows of a sequence fill eight waves (3500 tokens of 6 sequences behind
// 32768: 1890, apart in four waves 2020); four waves at D 64 otherwise (1630 tokens of 12
// behind 8192: 69, in eight 76).
// (HIP: fewer than 2^32 threads in a dimension of a grid)
bool launches(long long workgroups, int threads) { return workgroups * threads < (1LL << 32); }
bool tiles_join_launches(long long rows, int D) { return launches((rows * D + 1023) / 1024, 256); }   // (paged_tiles.hip)

TilesLayout tiles_layout(int T, int B, bool one_each, int H, int H_kv, int S, int P, int D) {
  TilesLayout L{};
  const int G = H / H_kv;
  const long long rows = (long long)T * G;
  const bool many = rows >= 1024LL * B, apart = P > 0 && !many;
  L.joined = P > 0 && many;
  const int tiles_p = (P + 63) / 64, tiles_s = (S + 63) / 64, tiles_o = tiles_s + (L.joined ? tiles_p : 0);
  const bool sorted = B > 1 && B <= 64;
  const float partial = (float)T * H * D * 8.f / 5e6f;   // us
  const float read_o = (float)B * tiles_s * H_kv * D * 256.f / 5e6f, read = read_o + tiles_p * H_kv * D * 256.f / 5e6f;
  static const short kShares[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64};
  // Work and reading beside each other: the longer; with one token each, and a quarter of the
  // shorter, which does not overlap.
  const bool few = one_each && G <= 32;
  const auto both = [=](float a, float b) { return a > b ? a + (few ? 0.25f * b : 0.f) : b + (few ? 0.25f * a : 0.f); };
  float best = INFINITY;
  for (const int nw : {4, 8}) {
    if (nw == 4 ? many : !many && (D == 64 || rows <= 128)) continue;
    const long long R = 32 * nw;
    const long long lists = one_each ? B * ((G + R - 1) / R) : rows / R + B;   // tiles of rows of the sequences
    const long long flat = (rows + R - 1) / R;                                 // and of all tokens
    const bool few_o = nw == 4 && few, few_p = few_o && rows <= 32;           // lists of up to 32 rows
    const float slots = nw == 8 ? 256.f : 512.f, narrow = D == 64 ? 0.6f : 1.f, pair = (nw == 8 ? 1.75f : 2.f) * narrow;
    const float beside_p = few_o && !few_p ? 0.5f * read_o / flat : 0.f;   // what few rows' lists read before the prefix's go on
    const float units_o = (float)(lists * H_kv), units_p = (float)(flat * H_kv);
    if (!launches((lists + (apart ? flat : 0)) * H_kv, 64 * nw)) continue;    // (four waves, or many: tiles_sizes has seen to it)
    for (const int no : kShares) {
      if (no > 1 && (no > tiles_o || (apart && tiles_o / no < 4) || !tiles_join_launches((long long)T * H, D))) break;
      const float all_o = units_o * no;
      for (const int n : kShares) {
        if (n > 1 && (!apart || n > tiles_p)) break;
        if ((n > 1 || no > 1) && all_o + units_p * n > 1e6f) break;   // (nothing to gain, and few enough to launch)
        // (a workgroup of four waves alone on its CU, or beside short lists, is done with a tile sooner)
        const float alone = nw == 4 && (few ? 0.f : all_o) + (apart ? units_p * n : 0.f) <= 256.f ? 0.75f : 1.f, tile = alone * pair;
        const float one_o = (tiles_o + no - 1) / no * (few_o ? 0.55f * narrow : tile) + (few_o ? 6.5f : 5.f);
        float t;
        if (apart) {   // the prefix's workgroups start first; the others run in the slots they leave free, then alone
          const float one = (tiles_p + n - 1) / n * (few_p ? 0.55f * alone * narrow : tile) + (few_p ? 6.5f : 5.f) + beside_p;
          const float all = units_p * n, full = std::floor(all / slots);
          const float rest = all - full * slots;
          const float left = all_o - (rest > 0.f ? (slots - rest) * std::floor(one / one_o) : 0.f);
          t = (full + (rest > 0.f)) * one + (left > 0.f ? std::ceil(left / slots) * one_o : 0.f);
          t = both(t, read) + (n + no) * partial;
        } else {
          t = std::ceil(all_o / slots) * one_o;
          if (all_o > slots && sorted) {   // the longest first: as far as lengths differ, the end is filled (a quarter of
            const float fill = 0.75f * all_o / slots * one_o + 0.25f * one_o;          // the own keys is taken to be missing)
            t += ((fill > one_o ? fill : one_o) - t) * tiles_s / tiles_o;
          }
          t = both(t, read) + (no > 1 ? 2.f * no * partial + 3.f : 0.f);
        }
        if (t < best) {
          best = t;
          L.nw = nw;
          L.nsp = apart ? n : 0;
          L.nso = no;
          L.prefix_items = (int)(L.nsp * flat);
          L.own_items = (int)(no * lists);
        }
      }
    }
  }
  L.by_length = sorted && (long long)L.own_items * H_kv > (L.nw == 8 ? 256 : 512);
  const size_t parts = L.nsp + L.nso, all = parts > 1 ? parts * (size_t)T * H : 0;
  L.acc = align256(all * 2 * sizeof(float));
  L.total = L.acc + align256(all * D * sizeof(float));
  return L;
}

bool tiles_sizes(int T, int B, int H, int H_kv, long long S, long long P, int D) {
  if (!(T >= 1 && T <= kMaxS && B >= 1 && B < (1 << 16) && H >= 1 && H <= kMaxHeads && H_kv >= 1 && H % H_kv == 0 && S >= 1 &&
        S <= kMaxS && P >= 0 && P <= kMaxS && D >= 2 && D % 2 == 0 && (long long)T * H <= (1 << 30)))
    return false;
  // What one share of each list launches.  Many rows a sequence: at most 2^30 / 256 tiles of eight waves and 2^30 / 1024 sequences.
  const long long rows = (long long)T * (H / H_kv);
  return rows >= 1024LL * B ||
         (launches(2 * (rows / 128) * H_kv + (B + 1LL) * H_kv, 256) && (P == 0 || tiles_join_launches((long long)T * H, D)));
}

}  // namespace

extern "C" {

int attnfuse_qknorm_rope(const void* Q, const void* K, void* Qr, void* Kr, const void* q_weight, const void* k_weight,
                         int weight_dtype, float eps,
                         long long q_stride_b, long long q_stride_h, long long q_stride_s,
                         long long k_stride_b, long long k_stride_h, long long k_stride_s,
                         int B, int H, int H_kv, int S, int D, int dtype,
                         int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                         const int* positions, void* stream) {
  return qknorm_fwd(Q, K, Qr, Kr, q_weight, k_weight, weight_dtype, 1, eps, q_stride_b, q_stride_h, q_stride_s, k_stride_b,
                    k_stride_h, k_stride_s, B, H, H_kv, S, D, dtype, rope, rope_theta, rope_table, rope_table_rows, positions,
                    Axes{}, stream);
}

int attnfuse_qknorm_axes(const void* Q, const void* K, void* Qr, void* Kr, const void* q_weight, const void* k_weight,
                         int weight_dtype, int norm, float eps,
                         long long q_stride_b, long long q_stride_h, long long q_stride_s,
                         long long k_stride_b, long long k_stride_h, long long k_stride_s,
                         int B, int H, int H_kv, int S, int D, int dtype,
                         int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                         const int* positions, int axes, const int* sections, int section_order, void* stream) {
  Axes x;
  const int rc = check_axes(axes, sections, section_order, D, x);
  if (rc != AF_OK) return rc;
  return qknorm_fwd(Q, K, Qr, Kr, q_weight, k_weight, weight_dtype, norm, eps, q_stride_b, q_stride_h, q_stride_s, k_stride_b,
                    k_stride_h, k_stride_s, B, H, H_kv, S, D, dtype, rope, rope_theta, rope_table, rope_table_rows, positions,
                    x, stream);
}

int attnfuse_axes_table_fill(float* table, int rows, int D, float rope_theta, int axes, const int* sections,
                             int section_order, int frequencies, void* stream) {
  if (!table || !aligned16(table) || rows < 1 || rows > kMaxTableRows) return AF_ERR_INVALID_ARG;
  if (!(std::isfinite(rope_theta) && rope_theta > 0.f)) return AF_ERR_INVALID_ARG;
  if (frequencies != AF_FREQUENCIES_SHARED && frequencies != AF_FREQUENCIES_OWN) return AF_ERR_INVALID_ARG;
  Axes x;
  const int rc = check_axes(axes, sections, section_order, D, x);
  if (rc != AF_OK) return rc;
  af::AxesRungs r{};
  r.half = D / 2;
  for (int i = 0; i < D / 2; ++i) {
    r.num[i] = frequencies == AF_FREQUENCIES_OWN ? x.rung[i] : (uint8_t)i;
    r.den[i] = frequencies == AF_FREQUENCIES_OWN ? x.size[i] : (uint8_t)(D / 2);
  }
  return map_launch(af::launch_axes_table(reinterpret_cast<float2*>(table), rows, r, (double)rope_theta,
                                          static_cast<hipStream_t>(stream)));
}

size_t attnfuse_qknorm_rope_bwd_workspace_bytes(int B, int H, int H_kv, int S, int D, int dtype) {
  int wgs[2];
  if (!qknorm_sizes(B, H, H_kv, S, D, dtype) || !supported_d(D) || !qknorm_wgs(B, H, H_kv, S, D, wgs)) return 0;
  return (size_t)(wgs[0] + wgs[1]) * D * sizeof(float);
}

int attnfuse_qknorm_rope_bwd(const void* Q, const void* K, const void* dQr, const void* dKr, void* dQ, void* dK,
                             void* dq_weight, void* dk_weight, const void* q_weight, const void* k_weight,
                             int weight_dtype, float eps,
                             long long q_stride_b, long long q_stride_h, long long q_stride_s,
                             long long k_stride_b, long long k_stride_h, long long k_stride_s,
                             long long dq_stride_b, long long dq_stride_h, long long dq_stride_s,
                             long long dk_stride_b, long long dk_stride_h, long long dk_stride_s,
                             void* workspace, size_t workspace_bytes,
                             int B, int H, int H_kv, int S, int D, int dtype,
                             int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                             const int* positions, void* stream) {
  return qknorm_bwd(Q, K, dQr, dKr, dQ, dK, dq_weight, dk_weight, q_weight, k_weight, weight_dtype, eps, q_stride_b,
                    q_stride_h, q_stride_s, k_stride_b, k_stride_h, k_stride_s, dq_stride_b, dq_stride_h, dq_stride_s,
                    dk_stride_b, dk_stride_h, dk_stride_s, workspace, workspace_bytes, B, H, H_kv, S, D, dtype, rope,
                    rope_theta, rope_table, rope_table_rows, positions, Axes{}, stream);
}

int attnfuse_qknorm_axes_bwd(const void* Q, const void* K, const void* dQr, const void* dKr, void* dQ, void* dK,
                             void* dq_weight, void* dk_weight, const void* q_weight, const void* k_weight,
                             int weight_dtype, int norm, float eps,
                             long long q_stride_b, long long q_stride_h, long long q_stride_s,
                             long long k_stride_b, long long k_stride_h, long long k_stride_s,
                             long long dq_stride_b, long long dq_stride_h, long long dq_stride_s,
                             long long dk_stride_b, long long dk_stride_h, long long dk_stride_s,
                             void* workspace, size_t workspace_bytes,
                             int B, int H, int H_kv, int S, int D, int dtype,
                             int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                             const int* positions, int axes, const int* sections, int section_order, void* stream) {
  Axes x;
  const int rc = check_axes(axes, sections, section_order, D, x);
  if (rc != AF_OK) return rc;
  if (!norm) {
    if (q_weight || k_weight || dq_weight || dk_weight) return AF_ERR_INVALID_ARG;
    return qknorm_unturn(dQr, dKr, dQ, dK, dq_stride_b, dq_stride_h, dq_stride_s, dk_stride_b, dk_stride_h, dk_stride_s, B, H,
                         H_kv, S, D, dtype, rope, rope_theta, rope_table, rope_table_rows, positions, x, stream);
  }
  return qknorm_bwd(Q, K, dQr, dKr, dQ, dK, dq_weight, dk_weight, q_weight, k_weight, weight_dtype, eps, q_stride_b,
                    q_stride_h, q_stride_s, k_stride_b, k_stride_h, k_stride_s, dq_stride_b, dq_stride_h, dq_stride_s,
                    dk_stride_b, dk_stride_h, dk_stride_s, workspace, workspace_bytes, B, H, H_kv, S, D, dtype, rope,
                    rope_theta, rope_table, rope_table_rows, positions, x, stream);
}

int attnfuse_qknorm_rope_append(const void* Q, const void* K, const void* V, void* Qr, void* K_pages, void* V_pages,
                                const long long* slots, const void* q_weight, const void* k_weight, int weight_dtype,
                                int norm, float eps,
                                long long q_stride_t, long long q_stride_h, long long k_stride_t, long long k_stride_h,
                                long long v_stride_t, long long v_stride_h,
                                long long kp_stride_p, long long kp_stride_h, long long kp_stride_s,
                                long long vp_stride_p, long long vp_stride_h, long long vp_stride_s,
                                int T, int H, int H_kv, int D, int num_pages, int page_size, int dtype,
                                int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                                const int* positions, void* stream) {
  return qknorm_append(Q, K, V, Qr, K_pages, V_pages, slots, q_weight, k_weight, weight_dtype, norm, eps, q_stride_t,
                       q_stride_h, k_stride_t, k_stride_h, v_stride_t, v_stride_h, kp_stride_p, kp_stride_h, kp_stride_s,
                       vp_stride_p, vp_stride_h, vp_stride_s, T, H, H_kv, D, num_pages, page_size, dtype, rope,
                       rope_theta, rope_table, rope_table_rows, positions, Axes{}, stream);
}

int attnfuse_qknorm_axes_append(const void* Q, const void* K, const void* V, void* Qr, void* K_pages, void* V_pages,
                                const long long* slots, const void* q_weight, const void* k_weight, int weight_dtype,
                                int norm, float eps,
                                long long q_stride_t, long long q_stride_h, long long k_stride_t, long long k_stride_h,
                                long long v_stride_t, long long v_stride_h,
                                long long kp_stride_p, long long kp_stride_h, long long kp_stride_s,
                                long long vp_stride_p, long long vp_stride_h, long long vp_stride_s,
                                int T, int H, int H_kv, int D, int num_pages, int page_size, int dtype,
                                int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                                const int* positions, int axes, const int* sections, int section_order, void* stream) {
  Axes x;
  const int rc = check_axes(axes, sections, section_order, D, x);
  if (rc != AF_OK) return rc;
  return qknorm_append(Q, K, V, Qr, K_pages, V_pages, slots, q_weight, k_weight, weight_dtype, norm, eps, q_stride_t,
                       q_stride_h, k_stride_t, k_stride_h, v_stride_t, v_stride_h, kp_stride_p, kp_stride_h, kp_stride_s,
                       vp_stride_p, vp_stride_h, vp_stride_s, T, H, H_kv, D, num_pages, page_size, dtype, rope,
                       rope_theta, rope_table, rope_table_rows, positions, x, stream);
}

size_t attnfuse_decode_paged_workspace_bytes(int B, int H, int H_kv, int S_kv, int D, int window, int sinks) {
  if (!decode_sizes(B, H, H_kv, S_kv, D) || window < 0 || sinks < 0) return 0;
  return paged_layout(B, H, H_kv, S_kv, D, window < S_kv ? window : S_kv, sinks < S_kv ? sinks : S_kv).total;
}

int attnfuse_decode_paged(const void* Q, const void* K_pages, const void* V_pages, const int* block_table,
                          const int* cache_lens, void* O, float* LSE, void* workspace, size_t workspace_bytes,
                          long long kp_stride_p, long long kp_stride_h, long long kp_stride_s,
                          long long vp_stride_p, long long vp_stride_h, long long vp_stride_s,
                          int B, int H, int H_kv, int D, int num_pages, int page_size, int max_pages,
                          int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                          int mask, int window, int sinks,
                          const float* alibi_slopes, float softmax_scale, void* stream) {
  if (!block_table || num_pages < 1 || page_size < 1 || max_pages < 1) return AF_ERR_INVALID_ARG;
  if ((long long)max_pages * page_size > kMaxS) return AF_ERR_INVALID_ARG;
  if (!strides_ok({{num_pages, kp_stride_p}, {H_kv, kp_stride_h}, {page_size, kp_stride_s}}, 0, AF_DTYPE_BF16, false) ||
      !strides_ok({{num_pages, vp_stride_p}, {H_kv, vp_stride_h}, {page_size, vp_stride_s}}, 0, AF_DTYPE_BF16, false) ||
      kp_stride_s > (1 << 24) || vp_stride_s > (1 << 24))
    return AF_ERR_INVALID_ARG;
  const int shift = page_shift_of(page_size);
  if (shift < 0) return AF_ERR_UNSUPPORTED;
  af::PagedParams p{};
  p.table = block_table;
  p.max_pages = max_pages; p.num_pages = num_pages; p.page_shift = shift;
  p.ks[0] = kp_stride_p; p.ks[1] = kp_stride_h; p.ks[2] = kp_stride_s;
  p.vs[0] = vp_stride_p; p.vs[1] = vp_stride_h; p.vs[2] = vp_stride_s;
  return decode_impl(p, Q, K_pages, V_pages, cache_lens, O, LSE, workspace, workspace_bytes, B, H, H_kv,
                     max_pages * page_size, D, rope, rope_theta, rope_table, rope_table_rows, mask, window, sinks,
                     alibi_slopes, softmax_scale, stream);
}

size_t attnfuse_fwd_paged_workspace_bytes(int T, int B, int H, int H_kv, int D, int own_keys, int prefix_keys) {
  if (!tiles_sizes(T, B, H, H_kv, own_keys, prefix_keys, D)) return 0;
  const size_t one = T == B ? tiles_layout(T, B, true, H, H_kv, own_keys, prefix_keys, D).total : 0;
  const size_t any = tiles_layout(T, B, false, H, H_kv, own_keys, prefix_keys, D).total;
  return one > any ? one : any;
}

int attnfuse_fwd_paged(const void* Q, const void* K_pages, const void* V_pages, const int* block_table, const int* q_starts,
                       const int* cache_lens, const int* prefix_table, const int* prefix_len, void* O, float* LSE,
                       void* workspace, size_t workspace_bytes,
                       long long kp_stride_p, long long kp_stride_h, long long kp_stride_s,
                       long long vp_stride_p, long long vp_stride_h, long long vp_stride_s,
                       int T, int B, int H, int H_kv, int D, int num_pages, int page_size, int max_pages, int prefix_pages,
                       float softmax_scale, void* stream) {
  if (!Q || !K_pages || !V_pages || !block_table || !O || !LSE) return AF_ERR_INVALID_ARG;
  if (num_pages < 1 || page_size < 1 || max_pages < 1 || prefix_pages < 0) return AF_ERR_INVALID_ARG;
  if (prefix_pages > 0 ? !prefix_table : prefix_table || prefix_len) return AF_ERR_INVALID_ARG;
  if (!q_starts && T != B) return AF_ERR_INVALID_ARG;
  for (const void* x : {Q, K_pages, V_pages, (const void*)O, (const void*)workspace})
    if (!aligned16(x)) return AF_ERR_INVALID_ARG;
  for (const void* x : {(const void*)LSE, (const void*)block_table, (const void*)q_starts, (const void*)cache_lens,
                        (const void*)prefix_table, (const void*)prefix_len})
    if (!aligned4(x)) return AF_ERR_INVALID_ARG;
  if (any_alias({O, LSE, workspace}, {Q, K_pages, V_pages, block_table, q_starts, cache_lens, prefix_table, prefix_len}) ||
      outs_alias({O, LSE, workspace}))
    return AF_ERR_INVALID_ARG;
  const long long S = (long long)max_pages * page_size, P = (long long)prefix_pages * page_size;
  if (!tiles_sizes(T, B, H, H_kv, S, P, D)) return AF_ERR_INVALID_ARG;
  if (!strides_ok({{num_pages, kp_stride_p}, {H_kv, kp_stride_h}, {page_size, kp_stride_s}}, 0, AF_DTYPE_BF16, false) ||
      !strides_ok({{num_pages, vp_stride_p}, {H_kv, vp_stride_h}, {page_size, vp_stride_s}}, 0, AF_DTYPE_BF16, false) ||
      kp_stride_s > (1 << 24) || vp_stride_s > (1 << 24))
    return AF_ERR_INVALID_ARG;
  if (!(std::isfinite(softmax_scale) && softmax_scale > 0.f)) return AF_ERR_INVALID_ARG;
  const TilesLayout L = tiles_layout(T, B, !q_starts, H, H_kv, (int)S, (int)P, D);
  if (L.total > 0 && (!workspace || workspace_bytes < L.total)) return AF_ERR_INVALID_ARG;
  const int shift = page_shift_of(page_size);
  if (shift < 0 || !supported_d(D)) return AF_ERR_UNSUPPORTED;

  af::TilesParams p{};
  p.q = Q; p.k = K_pages; p.v = V_pages;
  p.ks[0] = kp_stride_p; p.ks[1] = kp_stride_h; p.ks[2] = kp_stride_s;
  p.vs[0] = vp_stride_p; p.vs[1] = vp_stride_h; p.vs[2] = vp_stride_s;
  p.table = block_table;
  p.max_pages = max_pages; p.num_pages = num_pages; p.page_shift = shift;
  p.lens = cache_lens; p.starts = q_starts;
  p.prefix_table = prefix_table; p.prefix_len = prefix_len; p.prefix_pages = prefix_pages;
  p.o = O; p.lse = LSE;
  p.part_ml = static_cast<float*>(workspace);
  p.part_acc = reinterpret_cast<float*>(static_cast<char*>(workspace) + L.acc);
  p.T = T; p.B = B; p.H = H; p.Hkv = H_kv; p.G = H / H_kv;
  p.S = (int)S; p.P = (int)P;
  p.joined = L.joined;
  p.nsp = L.nsp; p.nso = L.nso; p.parts = L.nsp + L.nso;
  p.prefix_items = L.prefix_items; p.own_items = L.own_items;
  p.by_length = cache_lens && L.by_length;
  p.scale = softmax_scale;
  return map_launch(af::launch_paged_tiles(D, p, L.nw, static_cast<hipStream_t>(stream)));
}

int attnfuse_decode_sinks(const void* Q, const void* K, const void* V, const int* cache_lens, void* O, float* LSE,
                          void* workspace, size_t workspace_bytes, int B, int H, int H_kv, int S_kv, int D,
                          int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                          int window, int sinks, float softmax_scale, void* stream) {
  if (sinks < 1) return AF_ERR_INVALID_ARG;
  af::PagedParams p{};
  p.ks[0] = p.vs[0] = (long long)H_kv * S_kv * D;
  p.ks[1] = p.vs[1] = (long long)S_kv * D;
  p.ks[2] = p.vs[2] = D;
  return decode_impl(p, Q, K, V, cache_lens, O, LSE, workspace, workspace_bytes, B, H, H_kv, S_kv, D, rope, rope_theta,
                     rope_table, rope_table_rows, AF_MASK_SLIDING_WINDOW, window, sinks, nullptr, softmax_scale, stream);
}

}  // extern "C"
