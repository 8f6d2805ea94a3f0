// Internal host-side interface between the C-ABI layer (api.cpp) and the
// kernel translation units.  Each launcher maps runtime enums onto one
// compile-time template instantiation and enqueues it on the given stream.
#pragma once
#include <hip/hip_runtime.h>

namespace af {

// Score-modification / normalisation variants beyond masks and ALiBi (the
// additive_bias and relu_attention combinators): a dense fp32 bias tensor
// added to the scaled scores, and P = max(s, 0) in place of the softmax.
enum { EXT_NONE = 0, EXT_BIAS = 1, EXT_RELU = 2, EXT_RELU_BIAS = 3 };

struct FwdParams {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  float* lse;
  int B, H, Hkv, S, window;
  const float* slopes;    // [H] or nullptr
  float scale;
  const float2* table;    // [rows >= S][D/2] (cos, sin); nullptr without RoPE
  int heads_per_wg;       // set by the bf16 launcher: query heads packed per workgroup
  void* k16;              // workspace [B, H_kv, S, D] fp16: K' = R K, or nullptr (keys rotated in the loop)
  const int* bq_ptr;      // block-sparse mask by 64-row query block (CSR row pointers), or nullptr
  const int* bk_idx;      // and the active 64-key blocks of each row
  const float* bias;      // dense bias: element (b, h, i, j) at bias[b*bias_sb + h*bias_sh + i*bias_sq + j]
  long long bias_sb, bias_sh, bias_sq;
  int sinks;              // > 0 under a sliding window: first keys that stay visible, window + sinks < S
};

constexpr int DMAX_PARTS = 256;   // a wave reads four per lane

struct BwdParams {
  const void* q;
  const void* k;
  const void* v;
  const void* o;
  const void* dout;
  const float* lse;
  void* dq;
  void* dk;
  void* dv;
  float* delta;           // workspace [B*H*S]: sigma * sum_j P_ij dP_ij (see dscale), from the dQ pass
  float* lse2;            // workspace [B*H*S]: LSE in log2 units (+inf for empty rows)
  void* do16;             // workspace [B,H,S,D] fp16: sigma * dO
  float* dscale;          // workspace [B*H_kv]: sigma, a power of two per (batch, K/V head)
  uint32_t* dmax;         // workspace [B*H_kv*dmax_chunks]: partial max |dO| (bf16 magnitude bits)
  int dmax_chunks;        // partial maxima per (batch, K/V head), at most DMAX_PARTS
  void* qr16;             // workspace [B,H,S,D] fp16: Q' = R Q (with RoPE, and Q itself with sinks; else nullptr)
  void* kr16;             // workspace [B,H_kv,S,D] fp16: K' = R K (as qr16)
  int B, H, Hkv, S, window;
  const float* slopes;
  float scale;
  const float2* table;
  int splits;             // dK/dV: workgroups that share a key block's query tiles (1: no partials)
  float* part;            // splits > 1: their partial dK' and dV, [splits][2][B*H_kv*S][D]
  int heads_per_wg;       // set by the launcher for the dQ kernel
  const int* bq_ptr;      // block-sparse mask by 64-row query block (CSR), or nullptr
  const int* bk_idx;
  const int* bk_ptr;      // the same mask by 64-key block (CSC), or nullptr
  const int* bq_idx;
  const float* bias;      // dense bias, as in FwdParams
  long long bias_sb, bias_sh, bias_sq;
  int sinks;              // as FwdParams
  float* far;             // sinks > 0: partial dK', dV of the sinks, [B*H_kv][32-key blocks of sinks][far_parts][2][32][D]
  int far_parts;
};

struct DecodeParams {
  const void* q;          // [B, H, D]
  const void* k;          // cache [B, H_kv, S, D], keys already rotated
  const void* v;          // cache [B, H_kv, S, D]
  const int* lens;        // device [B] cache lengths, or nullptr (all S)
  void* o;                // [B, H, D]
  float* lse;             // [B, H]
  float* part_ml;         // workspace [B, H, 4 nsplit, 2]: wave partial max and sum (log2 units)
  float* part_acc;        // workspace [B, H, 4 nsplit, D]: wave partial accumulator
  int B, H, Hkv, S;
  int window;             // > 0: sliding window of that many keys; 0: every cached key
  int chunk, nsplit;      // keys per phase-1 workgroup; chunks per sequence
  const float* slopes;
  float scale;
  const float2* table;
};

struct RopeParams {
  const void* x0;  void* y0;  int heads0;   // first tensor [B, heads0, S, D]
  const void* x1;  void* y1;  int heads1;   // optional second tensor (heads1 may be 0)
  int B, S;
  const float2* table;
};

// Norm and rotation of query and key rows (qknorm.hip).  Index 0 is q, 1 k, 2 v;
// strides in elements: batch (of a cache: page), head, position.
enum { QKNORM_FWD = 0, QKNORM_BWD = 1, QKNORM_APPEND = 2 };
constexpr int QKNORM_BWD_HPT = 2;   // heads a thread takes in the backward
// Batches whose rows share a workgroup of 256 / (D / 16) rows: several of them fit.
inline int qknorm_per(int S, int D) { return 2 * S <= 4096 / D ? 4096 / D / S : 1; }

struct QkNormParams {
  const void* x[3];       // inputs; rows at b xs[.][0] + h xs[.][1] + n xs[.][2]
  void* y[3];             // outputs: forward [B, heads, S, D]; append q' [T, H, D], the key and value pages; backward dx
  const void* dy[2];      // backward: the gradients of the outputs, [B, heads, S, D]
  const void* w[2];       // weights [D], nullptr: 1
  void* dw[2];            // backward: their gradients [D], of the weights' type
  long long xs[3][3], ys[3][3];
  int heads[2];           // H, H_kv (0: no k)
  int B, S;               // append: 1, the tokens
  int per;                // batches a workgroup takes the rows of (qknorm_per)
  bool w32, norm;         // weights are fp32; append: norm the rows
  float eps;
  const float2* table;    // [rows][D/2] (cos, sin)
  int rows;
  const int* positions;   // [B, S], nullptr: 0..S-1
  const long long* slots; // append: [T]
  long long nslots;       // append: pages * page size
  int page_shift;
  int wgs[2];             // backward: workgroups of q and of k
  float* part;            // backward: [wgs[0] + wgs[1]][D], their sums of the weights' gradients (nullptr: none wanted)
};

// Decode over a paged cache, or over a contiguous one with sinks (decode_paged.hip).
struct PagedParams {
  const void* q;          // [B, H, D]
  const void* k;          // pages, or the contiguous cache (a sequence is then a page of S keys)
  const void* v;
  long long ks[3], vs[3]; // their strides in elements: page, head, place
  const int* table;       // [B, max_pages] page numbers, or nullptr: contiguous
  int max_pages, num_pages, page_shift;
  const int* lens;        // device [B] cache lengths, or nullptr (all S)
  void* o;                // [B, H, D]
  float* lse;             // [B, H]
  float* part_ml;         // workspace [B, H, nsplit, 2]: partial max and sum (log2 units)
  float* part_acc;        // workspace [B, H, nsplit, D]
  int B, H, Hkv, S;       // S: the most keys a sequence may have
  int window, sinks;      // window 0: every cached key; sinks: first keys that stay visible
  int nsplit;             // workgroups that share a sequence's tiles for a head group
  bool by_length;         // the longest sequences' workgroups first (B <= 64, lens given)
  int G, hgroups;         // query heads of a K/V head, and their groups of up to 32
  const float* slopes;
  float scale;
  const float2* rope;     // [rows >= S][D/2] (cos, sin)
};

// Waves per workgroup, four or eight, of a dense bf16 forward that has both
// forms; rope: the rotation of its key tiles in the loop (ROPE_NONE where they
// are copied to LDS as they are); bias: 0 without one, 1 where one row serves
// every query, 2 a row per query.
int fwd_waves(int B, int H, int Hkv, int S, int D, int rope, int mask, int window, int bias);

// Return 0 on success, -2 when the variant is not compiled, -3 on a HIP error.
// ext: EXT_* (common.hpp); variants other than EXT_NONE run without ALiBi and block masks.
int launch_fwd_bf16(int D, int rope, int mask, bool alibi, int ext, const FwdParams& p, hipStream_t st);
// The same with p.k16 filled first (RoPE kinds only): two launches.
int launch_fwd_prerot(int D, int rope, int mask, bool alibi, int ext, const FwdParams& p, hipStream_t st);
int launch_fwd_fp32(int D, int rope, int mask, bool alibi, const FwdParams& p, hipStream_t st);
// A sliding window with p.sinks > 0 (forward with RoPE: p.k16 is filled first); the
// fp32 launchers go by p.sinks themselves.
int launch_fwd_sinks(int D, int rope, const FwdParams& p, hipStream_t st);
int launch_bwd_sinks(int D, int rope, const BwdParams& p, hipStream_t st);
int launch_bwd_dkdv_sinks(int D, int rope, const BwdParams& p, hipStream_t st);   // its last launch
int launch_bwd_dkdv_reduce(int D, int rope, const BwdParams& p, hipStream_t st);  // the reduction of a split pass
int launch_bwd_bf16(int D, int rope, int mask, bool alibi, int ext, const BwdParams& p, hipStream_t st);
// The dK/dV pass alone (the last launch of launch_bwd_bf16).
int launch_bwd_dkdv_bf16(int D, int rope, int mask, bool alibi, int ext, const BwdParams& p, hipStream_t st);
// The same with p.splits > 1 workgroups per key block, and the reduction of their partials.
int launch_bwd_dkdv_split(int D, int rope, int mask, bool alibi, int ext, const BwdParams& p, hipStream_t st);
int launch_bwd_fp32(int D, int rope, int mask, bool alibi, const BwdParams& p, hipStream_t st);
int launch_decode(int D, int rope, bool alibi, const DecodeParams& p, hipStream_t st);
int launch_rope(bool fp32, int D, int rope, bool inverse, const RopeParams& p, hipStream_t st);
// x0 (bf16) rotated into y0 (fp16); x1 unused.
int launch_rope_f16(int D, int rope, const RopeParams& p, hipStream_t st);
int launch_decode_paged(int D, int rope, bool alibi, const PagedParams& p, hipStream_t st);
int launch_qknorm(int what, bool fp32, int D, int rope, const QkNormParams& p, hipStream_t st);
int launch_rope_table(float2* table, int rows, int D, double theta, hipStream_t st);

// Static device scratch of the decode entry point that allocates nothing: its
// size, and its address on the current device (nullptr if it cannot be found).
constexpr size_t DECODE_SCRATCH_BYTES = (size_t)32 << 20;
void* decode_scratch_ptr();

}  // namespace af
