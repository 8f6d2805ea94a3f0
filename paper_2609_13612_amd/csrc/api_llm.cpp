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

}  // namespace

extern "C" {

int attnfuse_qknorm_rope(const void* Q, const void* K, void* Qr, void* Kr, const void* q_weight, const void* k_weight,
                         int weight_dtype, float eps,
                         long long q_stride_b, long long q_stride_h, long long q_stride_s,
                         long long k_stride_b, long long k_stride_h, long long k_stride_s,
                         int B, int H, int H_kv, int S, int D, int dtype,
                         int rope, float rope_theta, const float* rope_table, int rope_table_rows,
                         const int* positions, void* stream) {
  if (!Q || !Qr || !K != !Kr) return AF_ERR_INVALID_ARG;
  if (!K) H_kv = 0;
  else if (H_kv < 1) return AF_ERR_INVALID_ARG;
  for (const void* x : {Q, K, (const void*)Qr, (const void*)Kr, q_weight, k_weight})
    if (!aligned16(x)) return AF_ERR_INVALID_ARG;
  if (!qknorm_sizes(B, H, H_kv, S, D, dtype) || !(std::isfinite(eps) && eps >= 0.f)) return AF_ERR_INVALID_ARG;
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
  p.table = reinterpret_cast<const float2*>(rope_table);
  p.rows = rope_table_rows;
  p.positions = rope != AF_ROPE_NONE ? positions : nullptr;
  return map_launch(af::launch_qknorm(af::QKNORM_FWD, dtype == AF_DTYPE_FP32, D, rope, p, static_cast<hipStream_t>(stream)));
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
  p.table = reinterpret_cast<const float2*>(rope_table);
  p.rows = rope_table_rows;
  p.positions = rope != AF_ROPE_NONE ? positions : nullptr;
  p.part = static_cast<float*>(workspace);
  return map_launch(af::launch_qknorm(af::QKNORM_BWD, dtype == AF_DTYPE_FP32, D, rope, p, static_cast<hipStream_t>(stream)));
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
  if (rope != AF_ROPE_NONE && !positions) return AF_ERR_INVALID_ARG;
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
  p.table = reinterpret_cast<const float2*>(rope_table);
  p.rows = rope_table_rows;
  p.positions = rope != AF_ROPE_NONE ? positions : nullptr;
  p.slots = slots;
  p.nslots = (long long)num_pages * page_size;
  p.page_shift = shift;
  return map_launch(
      af::launch_qknorm(af::QKNORM_APPEND, dtype == AF_DTYPE_FP32, D, rope, p, static_cast<hipStream_t>(stream)));
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
