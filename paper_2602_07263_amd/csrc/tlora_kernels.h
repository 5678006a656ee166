// Launch wrappers of the gfx950 kernels.  Every pointer is a device pointer; every launch is
// asynchronous on the given stream.  The wrappers check nothing: the planner has already
// validated shapes and sized every table.
#pragma once
#include <hip/hip_runtime.h>

#include "tlora_internal.h"

namespace tlora {

// bf16 copies of the adapters in the layouts the MFMA kernels read (zero padded to rpad).
// atp: per job A_j^T [rpad, d_in], stacked in job order ([R + 32, d_in], trailing rows zero);  a_all: [d_in, R + 32] with job j in columns roff_j ..;  b_all: [R + 32, d_out]
// with job j in rows roff_j ..  (R = r_total; the 32 trailing columns / rows are zero).
// frags: laid out in the same launch.  host_tables (null: the job table is on the device already): HOST memory, table_bytes (a
// multiple of 4, at most kPackArgBytes) of tables that begin with the job table; the launch takes them by value and leaves them at
// `jobs`.  Not with max_rpad == 0, which packs nothing.
constexpr size_t kPackArgBytes = 3328;      // with the other arguments below the 4 KB of a launch's argument block
void launch_pack_adapters(JobDev* jobs, int num_jobs, int d_in, int d_out, int max_rpad, int r_total, uint16_t* atp, uint16_t* a_all,
                          uint16_t* b_all, const FragPack& frags, const void* host_tables, size_t table_bytes, hipStream_t st);
void launch_frag_pack(const FragPack& frags, hipStream_t st);

// out[c, r] = in[r, c]; bf16 [rows, cols] row-major, rows and cols multiples of 8, 16-byte aligned.
void launch_transpose_bf16(const uint16_t* in, uint16_t* out, int rows, int cols, hipStream_t st);

// Zero `bytes` (multiple of 16) of device memory with a plain store kernel.
void launch_zero_fill(void* ptr, size_t bytes, hipStream_t st);

// Copy `bytes` of HOST memory to device memory `dst` (4-byte aligned, room for bytes rounded up to 4) by value,
// through the arguments of small store kernels: no staging buffer, no copy node, nothing allocated.
void launch_table_write(const void* host_src, size_t bytes, void* dst, hipStream_t st);
// What a backward does about the transposed copy of W in its workspace.
enum WtAction {
  kWtKeep = 0,       // nothing: no dX product, or a copy that this very call has made before
  kWtMade = 1,       // notes that the call makes it
  kWtNone = 2,       // notes that the call does without, so that what lies there is not taken for a copy of its W
  kWtEnsure = 3,     // the caller promises that an earlier call made it: made now if that call did without
};
struct WtState {     // in the workspace, at a place that depends on d_in x d_out alone
  uint32_t made;
  uint32_t done;     // workgroups of a kWtEnsure launch that have finished
};
struct WtCall {
  int action = kWtKeep;
  WtState* state = nullptr;
  const uint16_t* W = nullptr;     // [rows, cols]
  uint16_t* Wt = nullptr;
  int rows = 0, cols = 0;
};
// Copy `bytes` (a multiple of 16) from pinned host memory, given by its device address, to device memory; and wt or frags.
void launch_table_copy(const void* src_device_view, void* dst, size_t bytes, const WtCall& wt, const FragPack& frags,
                       hipStream_t st);

// out_j[t, p] = sum_k act[t, k] * P_j[p, k]   (P_j = A_j^T packed, or B_j packed)
// row_index (null = identity): the row of `act` that holds token row t of the job-sorted order (token-indexed calls).
// writes the result as bf16 hi + lo planes (packed ragged layout, each job's rows zero padded to a multiple of
// 32) and bf16 `scale_j * S` into the per-tile K-extension matrices `Sx`.
// packed_is_atp: P_j = atp + atp_off_j (row stride K);  otherwise P_j = b_all + roff_j * K.
void launch_shrink(const JobDev* jobs, const TileDev* tiles, const ShrinkUnit* units, int num_units,
                   int shrink_rows, const uint16_t* act, int K, const uint16_t* packed, bool packed_is_atp,
                   uint16_t* S_hi, uint16_t* S_lo, uint16_t* Sx, const int32_t* row_index, hipStream_t st);
// Same result for K % 32 == 0 with streaming units (shrink_rows = 64 | 128 token rows x 128 rank columns).
void launch_shrink_stream(const JobDev* jobs, const TileDev* tiles, const ShrinkUnit* units, int num_units,
                          int shrink_rows, int stages, const uint16_t* act, int K, const uint16_t* packed,
                          bool packed_is_atp, uint16_t* S_hi, uint16_t* S_lo, uint16_t* Sx, const int32_t* row_index,
                          hipStream_t st);
// An activation [T, D] kept in 8 bits: codes [T, D] and scales, bf16 [T, groups], of 128 values each.
struct PackedX {
  const uint8_t* codes = nullptr;        // null: there is none
  const uint16_t* scales = nullptr;
  int groups = 0;
};
// Same result from codes (K % 64 == 0, units of 64 or 128 rows, at most kShrinkScales scales in a unit's rows).
constexpr int kShrinkScales = 20480;
void launch_shrink_codes(const JobDev* jobs, const TileDev* tiles, const ShrinkUnit* units, int num_units, int shrink_rows,
                         const PackedX& codes, int K, const uint16_t* packed, bool packed_is_atp, uint16_t* S_hi, uint16_t* S_lo,
                         uint16_t* Sx, hipStream_t st);
// Same result with the contraction cut into `splits` (K % 64 == 0, units of 32 rows; splits <= K / 64): `part` holds
// `splits` copies of part_stride floats (>= the packed S elements).  Writes all of Sx, zeros included: no fill needed.
void launch_shrink_split(const JobDev* jobs, const TileDev* tiles, const ShrinkUnit* units, int num_units, int splits, int T,
                         const uint16_t* act, int K, const uint16_t* packed, bool packed_is_atp, uint16_t* S_hi,
                         uint16_t* S_lo, uint16_t* Sx, const int32_t* row_index, float* part, int64_t part_stride,
                         hipStream_t st);

// out[t, n] = sum_k act[t, k] * Wop[k, n] + sum_p Sx_tile[t, p] * Eop[roff_first + p, n]
//   w_is_kn = true : W is [K, N] row-major (forward,  Eop = b_all [R + 32, N])
//   w_is_kn = false: W is [N, K] row-major (backward, Eop = a_all^T, stored [N, R + 32])
void launch_seg_gemm(bool w_is_kn, const TileDev* tiles, const uint16_t* act, const uint16_t* W,
                     const uint16_t* Sx, const uint16_t* packed, int r_total, uint16_t* out,
                     const int32_t* out_index /* null, or the output row of every row (scatter) */,
                     const int32_t* in_index /* null, or the row of `act` behind every row (gather; needs T * K * 2 < 4 GiB) */,
                     int T, int K, int N,
                     unsigned long long* clk /* null, or 2 zeroed words: every 64th workgroup adds the shader
                                                cycles and 100 MHz ticks of its K-loop */,
                     const GemmSplit& split /* taken when K % 32 == 0 */,
                     float* part /* splits x cut tiles x min(T, 256) x 256 floats */,
                     const GemmOperands& second /* another product of the same T, K, N and tiles in the same launch, if any
                                                   (K % 32 == 0, no indexes); `split` is then that of both */,
                     hipStream_t st);

// A direction of a small batch (T <= kSmallRows; K and N multiples of 64): S_j (dS_j) as hi / lo planes (null: not wanted) and,
// unless out is null, Y (dX).  act: as fragments if small_frags(small_blocks(T)).  rank_rows: A_j^T (B_j) packed, [R + 32, K];  expand_rows: B_j (A_j^T) packed, [R + 32, N].  part:
// splits x T x small_ld(N, R) floats.
void launch_small(bool w_is_kn, const JobDev* jobs, const TileDev* tiles, const uint16_t* act, const uint16_t* W,
                  const uint16_t* rank_rows, const uint16_t* expand_rows, int r_total, uint16_t* out, const int32_t* out_index,
                  const int32_t* in_index, int T, int K, int N, int splits, float* part, uint16_t* S_hi, uint16_t* S_lo,
                  hipStream_t st);

// partial[u] = sum_{t in unit u} U_j[t, p] * V[t, c], or G_j itself of a unit with all tokens of its job;  then G_j = scale_j * sum_u
// partial[u].  b: the units of dB_j (U = S_j, V = dY), a: of dA_j (U = dS_j, V = X); either may be empty.
struct GradSide {
  const GradUnit* units = nullptr;
  const uint16_t *Uhi = nullptr, *Ulo = nullptr, *V = nullptr;      // V: [T, D], rows through row_index if that is given
  int D = 0, count = 0;
  PackedX packed;                                                   // instead of V, of a without row_index; D a multiple of 16
};
void launch_rank_grad(const JobDev* jobs, const GradSide& b, const GradSide& a, float* partial, bool accumulate,
                      const int32_t* row_index, hipStream_t st);
// accumulate: G_j += ... instead of G_j = ...
void launch_grad_reduce(const JobDev* jobs, const GradGroup* groups, int num_groups, const float* partial, int D,
                        bool out_is_dA, bool accumulate, hipStream_t st);

// ---- cross entropy of the vocabulary projection (bf16) ----------------------------------------------------------------------
// The tokens that have a loss are listed first (`live`, in token order); everything after works on pieces of the list, `max_rows` rows
// from place `first` on, of which those before *live exist: the host does not know their number, so grids are sized for a full piece.
struct HeadStat {
  float ref, sum;                        // of a row's logits z in a tile of kGemmBN columns: sum of exp(z - ref)
};
struct HeadParams {
  const int32_t* live = nullptr;         // how many tokens the list has
  int first = 0, max_rows = 0;
  int vocab = 0, ld = 0, kext = 0;       // columns that count; elements per row of W and of E; K-steps behind the last whole one (0 | 32)
  int col_tiles = 0;                     // tiles of kGemmBN columns
  const int32_t* target = nullptr;       // [max_rows] of the piece
  float* target_logit = nullptr;         // [max_rows]
  HeadStat* stats = nullptr;             // [max_rows, col_tiles]
  const float* factor = nullptr;         // [max_rows] what a row of E W^T is multiplied by
};
constexpr int kHeadMaxSplits = 64;
constexpr int kHeadShare = 8;            // K-steps
// Bytes of the shares' sums of a product of at most max_rows rows, whatever their number turns out to be (head_shape): at most two
// rounds of tiles, and none of a contraction that is too short to be cut.
inline size_t head_part_bytes(int64_t max_rows, int tiles_n, int steps) {
  const int64_t most = steps / kHeadShare < kHeadMaxSplits ? steps / kHeadShare : kHeadMaxSplits;
  const int64_t tiles = (max_rows + kGemmBM - 1) / kGemmBM * tiles_n, rest = tiles < 255 ? tiles : 255;
  const int64_t shares = most < 2 ? 0 : rest * most < 512 ? rest * most : 512;
  return (size_t)shares * kGemmBM * kGemmBN * sizeof(float);
}
// Largest logit of a row in a tile up to which exp(z) needs no reference, and from which on sums of it hold their digits.
__host__ __device__ inline float head_reference(float m) {
  constexpr float kTop = 60.f, kBottom = -40.f;
  return m <= kTop && m >= kBottom ? 0.f : m == -__builtin_huge_valf() ? 0.f : m;
}
// E = exp(H.W - ref) as bf16 [max_rows, ld] (null: statistics alone), zero from vocab to the next multiple of 8; stats; target_logit.
// Tiles that are cut leave their shares in part (head_part_bytes), from which launch_head_logits_reduce makes the same.
void launch_head_logits(const HeadParams& head, const uint16_t* H, const uint16_t* W, uint16_t* E, int d, float* part, hipStream_t st);
void launch_head_logits_reduce(const HeadParams& head, uint16_t* E, int d, const float* part, hipStream_t st);
// dH[out_index[r]] = factor[r] * (E[r] . W^T).  The columns from vocab / 32 * 32 on come from E_tail [max_rows padded to 256, 32] and
// W_tail [d, 32] (null if there are none).  Cut tiles as above: launch_head_grad_reduce, which also makes the job losses (null: not
// wanted, or not with this piece).
void launch_head_grad(const HeadParams& head, const uint16_t* E, const uint16_t* E_tail, const uint16_t* W, const uint16_t* W_tail,
                      uint16_t* dH, const int32_t* out_index, int d, float* part, hipStream_t st);
struct CeTokens;
void launch_head_grad_reduce(const HeadParams& head, const CeTokens& c, uint16_t* dH, const int32_t* out_index, int d, const float* part,
                             int num_jobs, float* job_loss, hipStream_t st);

// The rest of the loss.
constexpr int kCeArgJobs = 256;          // segments of so many jobs travel as an argument of the launch
struct CeOffsets {
  int32_t at[kCeArgJobs + 1];
};
struct CeTokens {
  int32_t T = 0, vocab = 0, d = 0;
  const int32_t* offsets = nullptr;      // [J + 1] on the device
  const int32_t* targets = nullptr;      // [T]
  const float* weights = nullptr;        // [T] or null: ones
  int32_t *live = nullptr, *list = nullptr, *target = nullptr;    // the list of the tokens with a loss, and their targets
  float* share = nullptr;                // [T] what a token's loss counts for; null: no gradient
  float* token_loss = nullptr;           // [T]; written for the tokens with a loss
};
// Whatever the first launch of a call can do: the list, the shares (dloss instead of them if given), zeros in loss and lse (either
// may be null) and dH (null: no gradient) of the tokens without a loss, the last columns of W as W_tail (null: none), and with `rows`
// the rows H of a batch that is one piece.  host_offsets: [J + 1], left at c.offsets; of more than kCeArgJobs jobs by launches
// before.
struct CePrepare {
  const float* dloss = nullptr;
  float *loss = nullptr, *lse = nullptr;
  const uint16_t* H = nullptr;
  uint16_t *dH = nullptr, *rows = nullptr;
  const uint16_t* W = nullptr;
  int64_t ld = 0;
  uint16_t* W_tail = nullptr;
};
void launch_ce_prepare(const CeTokens& c, int num_jobs, const int64_t* host_offsets, const CePrepare& p, hipStream_t st);
void launch_ce_gather(const HeadParams& h, const CeTokens& c, const uint16_t* H, uint16_t* rows, int d, hipStream_t st);
// Statistics -> losses; E null: no gradient.
void launch_ce_finish(const HeadParams& h, const CeTokens& c, uint16_t* E, uint16_t* E_tail, float* factor, float* loss, float* lse,
                      hipStream_t st);
void launch_ce_jobs(const CeTokens& c, int num_jobs, float* job_loss, hipStream_t st);

// ---- residual stream and norms between two blocks -----------------------------------------------------------------------------
struct NormArgs {
  const void *X = nullptr, *Y = nullptr, *gamma_post = nullptr, *gamma_pre = nullptr;
  float eps = 0.f, res_scale = 1.f;
  int d = 0;
};
struct NormGrads {
  const void *dH = nullptr, *dXn = nullptr;
  void *dX = nullptr, *dY = nullptr;
  int sums = 0;                            // column sums that are wanted: 1 dgamma_post, 2 dgamma_pre, 4 dgates
};
struct NormJob {
  int32_t row0 = 0, row1 = 0;
  int32_t unit0 = 0, units = 0;          // of the launch
  const void* gate = nullptr;
  float* dgate = nullptr;
};
constexpr int kNormJobs = 96;            // jobs of a launch: they travel as its argument
struct NormJobs {
  int32_t n = 0;
  int32_t unit_base = 0;                 // units of the launches before this one
  NormJob job[kNormJobs];
};
void launch_norm_fwd(bool bf16, const NormArgs& a, const NormJobs& jobs, int rows, void* H, void* Xn, hipStream_t st);
bool norm_in_registers(bool bf16, int d);// the rows' width allows launch_norm_bwd_units, else the two launches behind it are taken
int norm_resident_units(bool bf16, int d);
// partial [units of all launches][3][d], or null: not wanted
void launch_norm_bwd_units(bool bf16, const NormArgs& a, const NormJobs& jobs, const NormGrads& g, int units, int unit_rows,
                           float* partial, hipStream_t st);
// row_stats: 4 floats per row, or null: not wanted
void launch_norm_bwd_rows(bool bf16, const NormArgs& a, const NormJobs& jobs, const NormGrads& g, int rows, float* row_stats,
                          hipStream_t st);
// partial [units of all launches][3][d]
void launch_norm_bwd_cols(bool bf16, const NormArgs& a, const NormJobs& jobs, const NormGrads& g, int units, int unit_rows,
                          const float* row_stats, float* partial, hipStream_t st);
void launch_norm_reduce(const float* partial, const NormJobs& jobs, int first_vector, int vectors, int d, float* gamma_post,
                        float* gamma_pre, int all_units, bool accumulate, hipStream_t st);

// ---- activations in 8 bits ------------------------------------------------------------------------------------------------------
void launch_ckpt_pack(bool bf16, const void* X, int64_t T, int d, uint8_t* codes, uint16_t* scales, hipStream_t st);
void launch_ckpt_unpack(bool bf16, const uint8_t* codes, const uint16_t* scales, int64_t T, int d, void* X, hipStream_t st);

// fp32 configuration: strided products on plain FMA units.
void launch_f32_units(const F32Unit* units, const F32Tile* tiles, int num_tiles, hipStream_t st);

// AdamW step over a device table of `count` tensors (max_n = the largest element count).
void launch_adamw(const AdamwDev* tensors, int count, int64_t max_n, hipStream_t st);

// Glue of the MLP block (bf16 = tensors are bf16, else fp32; d and n multiples of 8; rstd fp32 [T]).
void launch_rmsnorm_fwd(bool bf16, const void* X, const void* gamma, float eps, int T, int d, void* Xn, float* rstd,
                        hipStream_t st);
// dX = dOut + d/dX [RMSNorm(X) gamma] applied to (dXa + dXb [+ dXc]); dXc may be null
void launch_rmsnorm_bwd(bool bf16, const void* X, const void* gamma, const float* rstd, const void* dXa,
                        const void* dXb, const void* dXc, const void* dOut, int T, int d, void* dX, hipStream_t st);
void launch_swiglu_fwd(bool bf16, const void* G, const void* U, void* Z, int64_t n, hipStream_t st);
void launch_swiglu_bwd(bool bf16, const void* G, const void* U, const void* dZ, void* dG, void* dU, int64_t n,
                       hipStream_t st);
void launch_residual_add(bool bf16, const void* X, const void* D, void* Out, int64_t n, hipStream_t st);

// Row gather (dst[i] = src[index[i]]) / scatter (dst[index[i]] = src[i]); row_bytes a multiple of 16.
void launch_permute_rows(const void* src, void* dst, const int32_t* index, int64_t rows, int64_t row_bytes, bool scatter,
                         hipStream_t st);
// Copy of a row list with every entry forced into [0, rows)  (rows < 2^31).
void launch_clamp_index(const int32_t* src, int32_t* dst, int64_t rows, hipStream_t st);

// ---- attention half (bf16, head size 128) -----------------------------------------------------------------
constexpr int kAttnHeadDim = 128;
// 128 consecutive tokens [t0, t0 + 128) of the sequence that starts at token seq_start and has seq_len tokens
struct AttnTile {
  int32_t seq_start, seq_len, t0, pad;
};
// Causal grouped-query attention over [T, heads * 128] tensors (Q, O, dO, dQ: Hq heads; K, V, dK, dV: Hkv heads,
// Hq % Hkv == 0).  lse [T, Hq] fp32 = log2 of the softmax denominator (base-2 domain, including the maximum);
// D [T, Hq] fp32 is scratch of the backward.  The backward is deterministic (no atomics).
void launch_attn_fwd(const AttnTile* tiles, int n_tiles, const uint16_t* Q, const uint16_t* K, const uint16_t* V,
                     uint16_t* O, float* lse, int Hq, int Hkv, hipStream_t st);
void launch_attn_bwd(const AttnTile* tiles, int n_tiles, const uint16_t* Q, const uint16_t* K, const uint16_t* V,
                     const uint16_t* O, const uint16_t* dO, const float* lse, float* D, uint16_t* dQ, uint16_t* dK,
                     uint16_t* dV, int Hq, int Hkv, hipStream_t st);
// table [positions, 64, 2] fp32 = (cos, sin) of position * base^(-i / 64)
void launch_rope_table(float* table, int positions, float base, hipStream_t st);
// In-place rotary embedding of x [T, heads * 128] at positions pos [T] (all < the table's positions);
// inverse = the transposed rotation.
void launch_rope(uint16_t* x, const int32_t* pos, const float* table, int64_t T, int heads, bool inverse, hipStream_t st);

}  // namespace tlora
