// Argument checks shared by the C-ABI entry points (api.cpp, api_llm.cpp).
#pragma once
#include <cmath>
#include <cstddef>
#include <cstdint>

#include "attnfuse.h"

namespace af_api {

constexpr int kMaxS = 1 << 20;
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

inline int map_launch(int rc) {
  if (rc == 0) return AF_OK;
  if (rc == -2) return AF_ERR_UNSUPPORTED;
  return AF_ERR_HIP;
}

// ---------------------------------------------------------------- caller-owned cos/sin table
// The table is [rows][D/2] (cos, sin) fp32 pairs; a RoPE call reads rows 0..S-1.
constexpr int kMaxTableRows = kMaxS;

inline size_t table_bytes(int rows, int D) { return (size_t)rows * (size_t)(D / 2) * 2 * sizeof(float); }

// Checks the table arguments of a call that rotates positions 0..S-1 (nothing
// without RoPE); a table given as an output would be a caller error too.
inline int check_table(int rope, const float* table, int rows, int S, const void* const* outs, int nouts) {
  if (rope == AF_ROPE_NONE) return AF_OK;
  if (!table || !aligned16(table) || rows < S || rows > kMaxTableRows) return AF_ERR_INVALID_ARG;
  for (int i = 0; i < nouts; ++i)
    if (outs[i] == static_cast<const void*>(table)) return AF_ERR_INVALID_ARG;
  return AF_OK;
}

// ---------------------------------------------------------------- validation
inline int check_common(int B, int H, int H_kv, int S, int D, int dtype, int rope, float rope_theta) {
  if (B < 1 || H < 1 || H_kv < 1 || S < 1 || S > kMaxS || D < 2 || (D & 1)) return AF_ERR_INVALID_ARG;
  if (H % H_kv != 0) return AF_ERR_INVALID_ARG;
  if (dtype != AF_DTYPE_BF16 && dtype != AF_DTYPE_FP32) return AF_ERR_INVALID_ARG;
  if (rope != AF_ROPE_NONE && rope != AF_ROPE_NEOX && rope != AF_ROPE_INTERLEAVED) return AF_ERR_INVALID_ARG;
  if (rope != AF_ROPE_NONE && !(std::isfinite(rope_theta) && rope_theta > 0.f)) return AF_ERR_INVALID_ARG;
  // grid sizes and element offsets must stay inside their integer types
  if ((long long)B * H * ((S + 63) / 64) >= (1LL << 31)) return AF_ERR_INVALID_ARG;
  return AF_OK;
}

inline int check_attn(int mask, int window, float scale) {
  if (mask != AF_MASK_NONE && mask != AF_MASK_CAUSAL && mask != AF_MASK_SLIDING_WINDOW) return AF_ERR_INVALID_ARG;
  if (mask == AF_MASK_SLIDING_WINDOW && window < 1) return AF_ERR_INVALID_ARG;
  if (!(std::isfinite(scale) && scale > 0.f)) return AF_ERR_INVALID_ARG;
  return AF_OK;
}

inline bool supported_d(int D) { return D == 64 || D == 128; }

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace af_api
