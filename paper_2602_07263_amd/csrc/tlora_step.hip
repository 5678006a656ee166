// gfx950 kernels of a training step around the decoder layers: what the vocabulary projection's cross entropy does beside its two
// matrix products, the residual stream and norms between two blocks, and activations in 8 bits.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "tlora_device.h"
#include "tlora_kernels.h"

namespace tlora {
namespace {

__device__ __forceinline__ double wave_sum_double(double x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
  return x;
}
// sum over the 1024 threads of a workgroup, every thread gets it; the order is fixed
__device__ __forceinline__ double block_sum_1024(double x, double* red) {
  x = wave_sum_double(x);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < 16; ++w) t += red[w];
  __syncthreads();
  return t;
}

// ---------------------------------------------------------------------------------------------------
// Cross entropy.  Workgroup 0 lists the tokens that have a loss, in token order; workgroup 1 + j sums job j's weights and notes
// what each of its tokens' losses counts for (dloss, or weight / sum; nothing at weight 0).  Tokens without a loss get zeros.  Of the
// workgroups behind those, each of the first has 16 tokens, a wave per row: it clears the rows of dH without a loss, and where the
// batch is one piece moves the others' rows of H to their places, for which it counts the list up to its tokens itself (16 KB of
// targets at most, from the L2; a launch of its own that reads the list would cost more); the last copy the end of W.
// ---------------------------------------------------------------------------------------------------
__device__ __forceinline__ bool ce_live(int y, int vocab) { return (unsigned)y < (unsigned)vocab; }

__device__ __forceinline__ void copy_row(const uint16_t* src, uint16_t* dst, int d, int lane) {     // src null: zeros
  for (int i = lane * 8; i < d; i += 4096) {           // eight loads in flight: a row of 4096 takes one latency, not eight
    u32x4 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = src ? ldg16(src + min(i + k * 512, d - 8)) : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i + k * 512 < d) *reinterpret_cast<u32x4*>(dst + i + k * 512) = v[k];
  }
}

template <bool ARGS>
__global__ void __launch_bounds__(1024) ce_prepare_kernel(CeTokens c, int num_jobs, int32_t* __restrict__ table, const CeOffsets offsets,
                                                          CePrepare p, int row_groups) {
  __shared__ double red[16];
  __shared__ int counts[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (blockIdx.x == 0) {
    if (ARGS && tid <= num_jobs) table[tid] = offsets.at[tid];
    int base = 0;
    for (int t0 = 0; t0 < c.T; t0 += 8192) {          // eight neighbouring tokens per thread
      int y[8], n = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int t = t0 + tid * 8 + k;
        y[k] = t < c.T ? c.targets[t] : -1;
        n += ce_live(y[k], c.vocab) ? 1 : 0;
      }
      int before = n;                                  // tokens up to this thread's last, inside its wave
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(before, o, 64);
        if (lane >= o) before += v;
      }
      if (lane == 63) counts[wave] = before;
      __syncthreads();
      int at = base + before - n, all = 0;
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        if (w < wave) at += counts[w];
        all += counts[w];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (ce_live(y[k], c.vocab)) {
          c.list[at] = t0 + tid * 8 + k;
          c.target[at] = y[k];
          ++at;
        }
      base += all;
      __syncthreads();
    }
    if (tid == 0) *c.live = base;
    return;
  }
  if ((int)blockIdx.x <= num_jobs) {
    const int j = (int)blockIdx.x - 1;
    const int a = ARGS ? offsets.at[j] : table[j], b = ARGS ? offsets.at[j + 1] : table[j + 1];
    double w = 0.0;
    for (int t = a + tid; t < b; t += 1024) {
      const bool on = ce_live(c.targets[t], c.vocab);
      if (on) w += c.weights ? (double)c.weights[t] : 1.0;
      else {
        if (p.loss) p.loss[t] = 0.f;
        if (p.lse) p.lse[t] = 0.f;
      }
    }
    if (!c.share) return;
    const double total = block_sum_1024(w, red);
    for (int t = a + tid; t < b; t += 1024) {
      float g = 0.f;
      if (ce_live(c.targets[t], c.vocab)) {
        const double v = c.weights ? (double)c.weights[t] : 1.0;
        if (v == 0.0) g = 0.f;                         // (a token of weight 0 is left out, whatever the caller's gradient is)
        else if (p.dloss) g = p.dloss[t];
        else if (total != 0.0) g = (float)(v / total);
      }
      c.share[t] = g;
    }
    return;
  }
  const int group = (int)blockIdx.x - 1 - num_jobs;
  if (group < row_groups) {
    const int t0 = group * 16, t = t0 + wave;
    if (p.rows) {
      int n = 0;
      for (int i = tid; i < t0; i += 1024) n += ce_live(c.targets[i], c.vocab) ? 1 : 0;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
      if (lane == 0) counts[wave] = n;
      __syncthreads();
    }
    if (t >= c.T) return;
    if (!ce_live(c.targets[t], c.vocab)) {
      if (p.dH) copy_row(nullptr, p.dH + (int64_t)t * c.d, c.d, lane);
    } else if (p.rows) {
      int at = 0;
#pragma unroll
      for (int w = 0; w < 16; ++w) at += counts[w] + (w < wave && ce_live(c.targets[t0 + w], c.vocab) ? 1 : 0);
      copy_row(p.H + (int64_t)t * c.d, p.rows + (int64_t)at * c.d, c.d, lane);
    }
    return;
  }
  const int i = (group - row_groups) * 1024 + tid, n = i >> 5, v = c.vocab / 32 * 32 + (i & 31);
  if (n < c.d) p.W_tail[i] = v < c.vocab ? p.W[(int64_t)n * p.ld + v] : (uint16_t)0;
}

// job_loss_j = sum w loss / sum w, by the threads of a workgroup (sums: its block sum)
template <class Sum>
__device__ __forceinline__ void ce_job(const CeTokens& c, int j, int threads, float* job_loss, const Sum& sums) {
  const int a = c.offsets[j], b = c.offsets[j + 1];
  double w = 0.0, s = 0.0;
  for (int t = a + (int)threadIdx.x; t < b; t += threads)
    if (ce_live(c.targets[t], c.vocab)) {
      const double v = c.weights ? (double)c.weights[t] : 1.0;
      w += v;
      if (v != 0.0) s += v * (double)c.token_loss[t];   // (whatever the loss of a token without weight is)
    }
  w = sums(w);
  s = sums(s);
  if (threadIdx.x == 0) job_loss[j] = w != 0.0 ? (float)(s / w) : 0.f;
}
__global__ void __launch_bounds__(1024) ce_jobs_kernel(CeTokens c, float* __restrict__ job_loss) {
  __shared__ double red[16];
  ce_job(c, blockIdx.x, 1024, job_loss, [&](double x) { return block_sum_1024(x, red); });
}

// The rows of a piece's tokens side by side: a wave per row.
__global__ void __launch_bounds__(256) ce_gather_kernel(const int32_t* __restrict__ live, int first, int max_rows,
                                                        const int32_t* __restrict__ list, const uint16_t* __restrict__ src,
                                                        uint16_t* __restrict__ dst, int d) {
  const int r = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6);
  if (r >= min(*live - first, max_rows)) return;
  copy_row(src + (int64_t)list[first + r] * d, dst + (int64_t)r * d, d, threadIdx.x & 63);
}

// Cut tiles of logits: the shares added in order, then what head_softmax_tile makes of a whole tile.  A workgroup has 8 rows of a tile,
// 8 columns per thread.
__global__ void __launch_bounds__(256) head_logits_reduce_kernel(const float* __restrict__ part, HeadParams h, uint16_t* __restrict__ E,
                                                                 int steps) {
  const HeadShape shape = head_shape(h, h.col_tiles, steps);
  const int n_tail = shape.tiles_m * h.col_tiles - shape.split.n_direct;
  if ((int)blockIdx.x >= n_tail) return;
  int tm, tn;
  gemm_tile_of(shape.split.n_direct + (int)blockIdx.x, shape.tiles_m, h.col_tiles, tm, tn);
  const int R = (int)blockIdx.y * 8 + (int)(threadIdx.x >> 5), c = (int)(threadIdx.x & 31) * 8;
  const int t = tm * kGemmBM + R, col = tn * kGemmBN + c;
  if (t >= shape.rows) return;
  const int64_t stride = (int64_t)n_tail * kGemmBM * kGemmBN;
  const float* src = part + ((int64_t)blockIdx.x * kGemmBM + R) * kGemmBN + c;
  float z[8] = {};
#pragma unroll 4
  for (int k = 0; k < shape.split.splits; ++k, src += stride) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(src), b = *reinterpret_cast<const f32x4*>(src + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[e] += a[e];
      z[4 + e] += b[e];
    }
  }
  float m = -__builtin_huge_valf();
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (col + e < h.vocab) m = fmaxf(m, z[e]);
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  const float ref = head_reference(m);
  const int y = h.target[t] - col;
  if (y >= 0 && y < 8) {
    float zy = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) zy = y == e ? z[e] : zy;
    h.target_logit[t] = zy;
  }
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    z[e] = col + e < h.vocab ? __builtin_amdgcn_exp2f((z[e] - ref) * 1.44269504088896340736f) : 0.f;
    s += z[e];
  }
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) s += __shfl_xor(s, o, 64);
  if (c == 0) h.stats[(int64_t)t * h.col_tiles + tn] = HeadStat{ref, s};
  if (E && col < h.vocab) store8<true>(E, (int64_t)t * h.ld + col, z);
}

// dH rows of a piece whose tiles were cut: the shares in order, scaled, as gemm_reduce_kernel
// The workgroups behind `tiles` make the job losses: all tokens' are known by then.
__global__ void __launch_bounds__(256) head_grad_reduce_kernel(const float* __restrict__ part, HeadParams head, CeTokens c_tokens,
                                                               uint16_t* __restrict__ out, const int32_t* __restrict__ out_index, int N,
                                                               int tiles_n, int steps, int tiles, int num_jobs,
                                                               float* __restrict__ job_loss) {
  if ((int)blockIdx.x >= tiles) {
    __shared__ double jobs_red[4];
    const int j = ((int)blockIdx.x - tiles) * (int)gridDim.y + (int)blockIdx.y;
    if (j >= num_jobs) return;
    ce_job(c_tokens, j, 256, job_loss, [&](double x) {
      x = wave_sum_double(x);
      if ((threadIdx.x & 63) == 0) jobs_red[threadIdx.x >> 6] = x;
      __syncthreads();
      const double all = (jobs_red[0] + jobs_red[1]) + (jobs_red[2] + jobs_red[3]);
      __syncthreads();
      return all;
    });
    return;
  }
  const HeadShape h = head_shape(head, tiles_n, steps);
  const int n_tail = h.tiles_m * tiles_n - h.split.n_direct;
  if ((int)blockIdx.x >= n_tail) return;
  int tm, tn;
  gemm_tile_of(h.split.n_direct + (int)blockIdx.x, h.tiles_m, tiles_n, tm, tn);
  const int R = (int)blockIdx.y * 8 + (int)(threadIdx.x >> 5), c = (int)(threadIdx.x & 31) * 8;
  const int t = tm * kGemmBM + R, col = tn * kGemmBN + c;
  if (t >= h.rows || col >= N) return;
  const int64_t stride = (int64_t)n_tail * kGemmBM * kGemmBN;
  const float* src = part + ((int64_t)blockIdx.x * kGemmBM + R) * kGemmBN + c;
  f32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
#pragma unroll 8
  for (int k = 0; k < h.split.splits; ++k, src += stride) {
    a += *reinterpret_cast<const f32x4*>(src);
    b += *reinterpret_cast<const f32x4*>(src + 4);
  }
  const float f = head.factor[t];
  if (f == 0.f) a = b = f32x4{0, 0, 0, 0};
  a *= f;  b *= f;
  *reinterpret_cast<u32x4*>(out + (int64_t)out_index[t] * N + col) =
      u32x4{pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3])};
}

// A row's statistics become its logarithm of the sum and its loss; with GRAD its exponentials become those of the gradient: all
// relative to one reference rho, the target's less the sum itself, and factor = share * exp(rho - lse).  rho is 0 unless the sum
// itself is out of range for it or the factor would be (a gradient from above of 1e-20 beside lse 57 left a subnormal factor and a row
// wrong by a third), so that as a rule (logits within head_reference's bounds) one element of the row is touched; a tile that took a
// reference of its own is scaled.  A wave per row.
// The target's element is as large as all others together, and its rounding to bf16, of a relative delta, would be most of the row's
// error.  The factor, an fp32 number, takes a part a of it over: (1 - a) delta is left at the target, a delta comes to the others, and
// with T = (1 - p_y)^2 and N the others' sum of p^2 the squares, T (1 - a)^2 + N a^2 in directions that have nothing to do with each
// other, are smallest at a = T / (T + N).  N is taken from the tiles' sums, which is more than it is.  8192 logits of deviation 1 to 3:
// the error of dH before its own rounding 0.0012 of its norm without this, 0.0001 to 0.0004 with it.
template <bool GRAD>
__global__ void __launch_bounds__(256) ce_finish_kernel(HeadParams h, CeTokens c, uint16_t* __restrict__ E, uint16_t* __restrict__ E_tail,
                                                        float* __restrict__ factor, float* __restrict__ loss, float* __restrict__ lse) {
  const int r = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= min(*h.live - h.first, h.max_rows)) return;
  const int t = c.list[h.first + r];
  const HeadStat* const st = h.stats + (int64_t)r * h.col_tiles;
  float sum = 0.f;
  bool plain = true;
  for (int i = lane; i < h.col_tiles; i += 64) {
    const HeadStat s = st[i];
    plain = plain && s.ref == 0.f;
    sum += s.sum;
  }
  plain = __all(plain);
  float l;
  if (plain) {
    l = logf(wave_sum(sum));
  } else {
    float top = -__builtin_huge_valf();
    for (int i = lane; i < h.col_tiles; i += 64) top = fmaxf(top, st[i].ref + logf(st[i].sum));
    top = wave_max(top);
    if (!(fabsf(top) < __builtin_huge_valf())) top = 0.f;
    float s = 0.f;
    for (int i = lane; i < h.col_tiles; i += 64) s += st[i].sum * expf(st[i].ref - top);
    l = top + logf(wave_sum(s));
  }
  const float zy = h.target_logit[r];
  if (lane == 0) {
    const float v = l - zy;
    c.token_loss[t] = v;
    if (loss) loss[t] = v;
    if (lse) lse[t] = l;
  }
  if (!GRAD) return;
  // (one row has one share: all lanes agree.  With rho = l the factor is the share itself; 1 + absorb is 1 to within 2^-8)
  const float g = c.share[t], at_zero = fabsf(g) * expf(-l);
  const float rho = l >= -20.f && l <= 60.f && (g == 0.f || (at_zero >= 0x1p-125f && at_zero <= 0x1p127f)) ? 0.f : l;
  uint16_t* const row = E + (int64_t)r * h.ld;
  const int n8 = (h.vocab + 7) & ~7;
  if (!plain || rho != 0.f)
    for (int i = 0; i < h.col_tiles; ++i) {
      const float ref = st[i].ref;
      if (ref == rho) continue;
      const float f = expf(ref - rho);
      const int col = i * kGemmBN + lane * 4;
      if (col < n8) {
        u32x2* const p = reinterpret_cast<u32x2*>(row + col);
        const u32x2 v = *p;
        u32x2 o;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          o[e] = pack_bf16x2(__builtin_bit_cast(float, v[e] << 16) * f, __builtin_bit_cast(float, v[e] & 0xffff0000u) * f);
        *p = o;
      }
    }
  const int y = h.target[r];
  const float to_one = expm1f(zy - l), target = expf(l - rho) * to_one;
  const uint16_t at_y = (uint16_t)(pack_bf16x2(target, 0.f) & 0xffffu);
  float others = 0.f;
  for (int i = lane; i < h.col_tiles; i += 64) {
    const float p = st[i].sum * expf(st[i].ref - l) - (i == y / kGemmBN ? expf(zy - l) : 0.f);
    others += p > 0.f ? p * p : 0.f;
  }
  others = wave_sum(others);
  const float as_stored = bf16_float(at_y);
  const float absorb = as_stored != 0.f ? to_one * to_one / (to_one * to_one + others) * (target / as_stored - 1.f) : 0.f;
  __threadfence_block();                               // (the tail reads what other lanes may have scaled)
  const int k0 = h.vocab & ~31, rest = h.vocab - k0;
  if (rest && lane < 32) {
    uint16_t v = lane < rest ? row[k0 + lane] : (uint16_t)0;
    if (k0 + lane == y) v = at_y;
    E_tail[(int64_t)r * 32 + lane] = v;
  }
  if (lane == 0) {
    row[y] = at_y;
    factor[r] = g == 0.f ? 0.f : g * expf(rho - l) * (1.f + absorb);    // (0: a row of zeros, whatever the exponentials are)
  }
}

}  // namespace

void launch_ce_prepare(const CeTokens& c, int num_jobs, const int64_t* host_offsets, const CePrepare& p, hipStream_t st) {
  const int row_groups = p.dH || p.rows ? (c.T + 15) / 16 : 0;
  const dim3 grid(1 + num_jobs + row_groups + (p.W_tail ? (c.d + 31) / 32 : 0));
  int32_t* const table = const_cast<int32_t*>(c.offsets);
  CeOffsets args = {};
  if (num_jobs <= kCeArgJobs) {
    for (int j = 0; j <= num_jobs; ++j) args.at[j] = (int32_t)host_offsets[j];
    hipLaunchKernelGGL(ce_prepare_kernel<true>, grid, dim3(1024), 0, st, c, num_jobs, table, args, p, row_groups);
  } else {
    for (int j = 0, n; j <= num_jobs; j += n) {
      n = std::min(num_jobs + 1 - j, kCeArgJobs);
      for (int i = 0; i < n; ++i) args.at[i] = (int32_t)host_offsets[j + i];
      launch_table_write(args.at, sizeof(int32_t) * (size_t)n, table + j, st);
    }
    hipLaunchKernelGGL(ce_prepare_kernel<false>, grid, dim3(1024), 0, st, c, num_jobs, table, args, p, row_groups);
  }
}
void launch_ce_jobs(const CeTokens& c, int num_jobs, float* job_loss, hipStream_t st) {
  hipLaunchKernelGGL(ce_jobs_kernel, dim3(num_jobs), dim3(1024), 0, st, c, job_loss);
}
void launch_ce_gather(const HeadParams& h, const CeTokens& c, const uint16_t* H, uint16_t* rows, int d, hipStream_t st) {
  hipLaunchKernelGGL(ce_gather_kernel, dim3((h.max_rows + 3) / 4), dim3(256), 0, st, h.live, h.first, h.max_rows, c.list, H, rows, d);
}
// tiles that may be cut: less than a round
static int head_cut_tiles(const HeadParams& h, int tiles_n) { return std::min((h.max_rows + kGemmBM - 1) / kGemmBM * tiles_n, 255); }
void launch_head_logits_reduce(const HeadParams& h, uint16_t* E, int d, const float* part, hipStream_t st) {
  if (d % kGemmBK) return;                             // (none is)
  hipLaunchKernelGGL(head_logits_reduce_kernel, dim3(head_cut_tiles(h, h.col_tiles), std::min((h.max_rows + 7) / 8, kGemmBM / 8)), dim3(256), 0,
                     st, part, h, E, d / kGemmBK);
}
void launch_head_grad_reduce(const HeadParams& h, const CeTokens& c, uint16_t* dH, const int32_t* out_index, int d, const float* part,
                             int num_jobs, float* job_loss, hipStream_t st) {
  const int tiles_n = (d + kGemmBN - 1) / kGemmBN, tiles = head_cut_tiles(h, tiles_n), y = std::min((h.max_rows + 7) / 8, kGemmBM / 8);
  const int jobs = job_loss ? num_jobs : 0;
  HeadParams head = h;
  hipLaunchKernelGGL(head_grad_reduce_kernel, dim3(tiles + (jobs + y - 1) / y, y), dim3(256), 0, st, part, head, c, dH, out_index, d,
                     tiles_n, (h.vocab + kGemmBK - 1) / kGemmBK, tiles, jobs, job_loss);
}
void launch_ce_finish(const HeadParams& h, const CeTokens& c, uint16_t* E, uint16_t* E_tail, float* factor, float* loss, float* lse,
                      hipStream_t st) {
  const dim3 grid((h.max_rows + 3) / 4);
  if (E) hipLaunchKernelGGL(ce_finish_kernel<true>, grid, dim3(256), 0, st, h, c, E, E_tail, factor, loss, lse);
  else   hipLaunchKernelGGL(ce_finish_kernel<false>, grid, dim3(256), 0, st, h, c, E, E_tail, factor, loss, lse);
}

// ---------------------------------------------------------------------------------------------------
// Residual stream and norms between two blocks (see include/tlora.h).  fp32 arithmetic on the inputs as they are; every result is
// rounded once.  A launch has the jobs of one group as an argument, a workgroup finds its job by bisection.
// ---------------------------------------------------------------------------------------------------
namespace {

__device__ __forceinline__ int norm_job(const NormJobs& jobs, int unit) {
  int lo = 0, hi = jobs.n - 1;                          // the last job whose first unit is not beyond `unit`
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (jobs.job[mid].unit0 <= unit) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
template <bool BF>
__device__ __forceinline__ void load8_or(const void* p, int64_t i, float other, float (&v)[8]) {
  if (p) {
    load8<BF>(p, i, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = other;
  }
}

// units are rows
template <bool BF>
__global__ void __launch_bounds__(256) norm_fwd_kernel(NormArgs a, NormJobs jobs, void* __restrict__ H, void* __restrict__ Xn) {
  __shared__ float red[4];
  const NormJob jb = jobs.job[norm_job(jobs, blockIdx.x)];
  const int64_t row = (int64_t)(jb.row0 + (int)blockIdx.x - jb.unit0) * a.d;
  float ss = 0.f;
  if (a.gamma_post)
    for (int c = threadIdx.x * 8; c < a.d; c += 2048) {
      float y[8];
      load8<BF>(a.Y, row + c, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += y[e] * y[e];
    }
  const float r1 = a.gamma_post ? 1.0f / sqrtf(block_sum(ss, red) / (float)a.d + a.eps) : 1.0f;
  auto stream = [&](int c, float (&h)[8]) {
    float y[8], g[8], p[8];
    load8<BF>(a.Y, row + c, y);
    load8_or<BF>(a.gamma_post, c, 1.f, p);
    load8_or<BF>(jb.gate, c, 1.f, g);
    load8_or<BF>(a.X, row + c, 0.f, h);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] += a.res_scale * (g[e] * (y[e] * r1 * p[e]));
  };
  ss = 0.f;
  if (Xn)
    for (int c = threadIdx.x * 8; c < a.d; c += 2048) {
      float h[8];
      stream(c, h);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += h[e] * h[e];
    }
  const float r2 = Xn ? 1.0f / sqrtf(block_sum(ss, red) / (float)a.d + a.eps) : 0.f;
  for (int c = threadIdx.x * 8; c < a.d; c += 2048) {
    float h[8];
    stream(c, h);
    if (H) store8<BF>(H, row + c, h);
    if (Xn) {
      float g[8];
      load8<BF>(a.gamma_pre, c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = h[e] * r2 * g[e];
      store8<BF>(Xn, row + c, h);
    }
  }
}

// Rows of at most kNormRow features stay in registers: a thread has eight neighbouring features and the workgroup as many waves as
// the row needs.  A lane behind the row's end repeats its last features, which enter no sum.  Rows of up to twice that take two runs of
// eight per thread, where no column sums are kept beside them.
constexpr int kNormRow = 8192;
constexpr int norm_bwd_row(bool bf16) { return bf16 ? kNormRow : kNormRow / 2; }      // (fp32 operands take twice the registers)
static int norm_threads(int d) { return d <= kNormRow ? (d + 511) / 512 * 64 : (d + 1023) / 1024 * 64; }

// Sums over the workgroup; each use between two barriers has a slot of its own.
template <int N>
__device__ __forceinline__ void norm_sums(float (&x)[N], float (*slot)[16]) {
  const int waves = (int)blockDim.x >> 6, wave = (int)threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = wave_sum(x[i]);
  if (waves == 1) return;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if ((threadIdx.x & 63) == 0) slot[i][wave] = x[i];
  __syncthreads();
  const int w = (int)threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = row_sum(w < waves ? slot[i][w] : 0.f);
}
// Eight values as they lie in memory, fetched ahead of their use; p null: `other`.
template <bool BF>
struct Raw8 {
  u32x4 v[BF ? 1 : 2];
  __device__ __forceinline__ void fetch(const void* p, int64_t i) {
    const char* const at = static_cast<const char*>(p) + i * (BF ? 2 : 4);
#pragma unroll
    for (int k = 0; k < (BF ? 1 : 2); ++k) v[k] = ldg16(at + 16 * k);
  }
  __device__ __forceinline__ void get(float (&x)[8]) {
    // (kept as loaded until here: the compiler would convert right behind the load, and wait for it there)
#pragma unroll
    for (int k = 0; k < (BF ? 1 : 2); ++k) asm volatile("" : "+v"(v[k]));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (BF) {
        x[2 * e] = __builtin_bit_cast(float, v[0][e] << 16);
        x[2 * e + 1] = __builtin_bit_cast(float, v[0][e] & 0xffff0000u);
      } else {
        const uint32_t lo = v[0][e], hi = v[BF ? 0 : 1][e];     // (bit_cast of the element itself takes element 0)
        x[e] = __builtin_bit_cast(float, lo);
        x[4 + e] = __builtin_bit_cast(float, hi);
      }
    }
  }
};
__device__ __forceinline__ void fill8(float (&x)[8], float v) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = v;
}

// A row per workgroup, CH runs per thread: bound by HBM (31744 x 4096 bf16 193 us, 5.4 TB/s; read again for each sum, 256).
template <bool BF, int CH>
__global__ void __launch_bounds__(1024) norm_fwd_row_kernel(NormArgs a, NormJobs jobs, void* __restrict__ H, void* __restrict__ Xn) {
  __shared__ float red[2][1][16];
  const NormJob jb = jobs.job[norm_job(jobs, blockIdx.x)];
  const int64_t row = (int64_t)(jb.row0 + (int)blockIdx.x - jb.unit0) * a.d;
  const int c0 = (int)threadIdx.x * 8, step = (int)blockDim.x * 8;
  float y[CH][8], h[CH][8];
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    const int c = min(c0 + k * step, a.d - 8);
    load8<BF>(a.Y, row + c, y[k]);
    load8_or<BF>(a.X, row + c, 0.f, h[k]);
  }
  auto squares = [&](const float (&v)[CH][8]) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      float t = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) t += v[k][e] * v[k][e];
      s += c0 + k * step < a.d ? t : 0.f;
    }
    return s;
  };
  float r1 = 1.f;
  if (a.gamma_post) {
    float s[1] = {squares(y)};
    norm_sums(s, red[0]);
    r1 = 1.0f / sqrtf(s[0] / (float)a.d + a.eps);
  }
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    const int c = min(c0 + k * step, a.d - 8);
    float g[8], p[8];
    load8_or<BF>(jb.gate, c, 1.f, g);
    load8_or<BF>(a.gamma_post, c, 1.f, p);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[k][e] += a.res_scale * (g[e] * (y[k][e] * r1 * p[e]));
    if (H && c0 + k * step < a.d) store8<BF>(H, row + c, h[k]);
  }
  if (!Xn) return;
  float s[1] = {squares(h)};
  norm_sums(s, red[1]);
  const float r2 = 1.0f / sqrtf(s[0] / (float)a.d + a.eps);
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    const int c = c0 + k * step;
    if (c >= a.d) continue;
    float q[8];
    load8<BF>(a.gamma_pre, c, q);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[k][e] = h[k][e] * r2 * q[e];
    store8<BF>(Xn, row + c, h[k]);
  }
}

// 1 / sqrt(x): the instruction's estimate and one Newton step (which has no say about 0 and infinity)
__device__ __forceinline__ float rstd_of(float x) {
  const float r = __builtin_amdgcn_rsqf(x);
  const float better = r * fmaf(-0.5f * x * r, r, 1.5f);
  return x > 0.f && x < __builtin_huge_valf() ? better : r;
}

// D = dH + r2 (u - c2 hn) with u = dXn gamma_pre, hn = r2 H and c2 = mean(u hn); dY = r1 (v - c1 (r1 Y)) with v = res_scale gate
// gamma_post D and c1 = mean(v r1 Y).  Every reciprocal root stands beside the value that it is of: its square or cube would leave
// fp32 where the result does not.  Fused operations written out, so that every kernel rounds alike.
__device__ __forceinline__ float norm_D(float dH, float u, float hn, float r2, float c2) { return fmaf(r2, fmaf(-hn, c2, u), dH); }
__device__ __forceinline__ float norm_dY(float v, float y, float r1, float c1) { return r1 * fmaf(-(y * r1), c1, v); }
// sum D w, from the sums of dH w, u w and H w
__device__ __forceinline__ float norm_dot(float dHw, float uw, float hw, float r2, float c2) {
  return fmaf(r2, fmaf(-c2, r2 * hw, uw), dHw);
}

// Backward of a unit's rows, one after the other; with SUMS the unit's column sums stay in registers and leave as partial
// [unit][3][d] (dgamma_post, dgamma_pre, dgate; those that are wanted).  What holds a row up are the sums across the workgroup that follow one another: of Y^2
// for rstd_Y, with it of H^2 and dXn gamma_pre H for D, with that of D' = res_scale gate gamma_post D and Y for dY.  D is linear in
// what the second sums give (norm_D), so the last sum is put together from three that need rstd_Y alone (norm_dot); and
// Y^2 is summed for the row after, whose Y is loaded a row earlier than the rest.  So a row has one round of sums and one barrier.
// 31744 x 4096 bf16 with all sums 320 to 324 us (4.8 TB/s).
// BOTH: dX and dY are wanted.  Every lane then stores without a condition -- those behind the row's end its last features once more,
// the same values -- since behind a store that may not have been issued the compiler waits for all those that may.
template <bool BF, bool SUMS, bool BOTH>
__global__ void __launch_bounds__(norm_bwd_row(BF) / 8) norm_bwd_unit_kernel(NormArgs a, NormJobs jobs, NormGrads g, int unit_rows,
                                                             float* __restrict__ partial) {
  __shared__ float red[2][6][16];
  const NormJob jb = jobs.job[norm_job(jobs, blockIdx.x)];
  const int t0 = jb.row0 + ((int)blockIdx.x - jb.unit0) * unit_rows, t1 = min(t0 + unit_rows, jb.row1);
  const bool on = (int)threadIdx.x * 8 < a.d;
  const int c = on ? (int)threadIdx.x * 8 : a.d - 8;
  const float inv_d = 1.0f / (float)a.d;
  float agp[8], q[8];                        // res_scale * gate * gamma_post, and gamma_pre
  {
    float p[8];
    load8_or<BF>(jb.gate, c, 1.f, agp);
    load8_or<BF>(a.gamma_post, c, 1.f, p);
    load8_or<BF>(a.gamma_pre, c, 0.f, q);
#pragma unroll
    for (int e = 0; e < 8; ++e) agp[e] *= p[e] * a.res_scale;
  }
  // a job's gate and gamma_post are factors of whole columns: of D Y rstd_Y one sum serves both
  float sum_y[8] = {}, sum_h[8] = {};
  // (an operand that is not there is Y once more: around a branch in the loop the compiler would wait for all loads)
  Raw8<BF> ry, rx, rh, rn;
  const void *const X = a.X ? a.X : a.Y, *const dH = g.dH ? g.dH : a.Y, *const dXn = g.dXn ? g.dXn : a.Y;
  auto fetch = [&](int t) {
    const int64_t at = (int64_t)t * a.d + c;
    rx.fetch(X, at);
    rh.fetch(dH, at);
    rn.fetch(dXn, at);
  };
  auto squares = [&](const float (&v)[8]) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[e] * v[e];
    return on ? s : 0.f;
  };
  float y[8], r1 = 1.f;
  ry.fetch(a.Y, (int64_t)t0 * a.d + c);
  fetch(t0);
  ry.get(y);
  if (a.gamma_post) {
    float s[1] = {squares(y)};
    norm_sums(s, red[1]);
    r1 = rstd_of(s[0] * inv_d + a.eps);
  }
  ry.fetch(a.Y, (int64_t)min(t0 + 1, t1 - 1) * a.d + c);
  for (int t = t0; t < t1; ++t) {
    const int64_t at = (int64_t)t * a.d + c;
    float h[8], D[8], gq[8];
    rx.get(h);
    rh.get(D);
    rn.get(gq);
    fetch(min(t + 1, t1 - 1));
    if (!a.X) fill8(h, 0.f);
    if (!g.dH) fill8(D, 0.f);
    if (!g.dXn) fill8(gq, 0.f);
    float s[6] = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      h[e] += agp[e] * (y[e] * r1);
      const float w = agp[e] * y[e], u = gq[e] * q[e];
      s[0] += h[e] * h[e];
      s[1] += u * h[e];
      s[2] += D[e] * w;
      s[3] += u * w;
      s[4] += h[e] * w;
    }
    float next[8];
    ry.get(next);
    ry.fetch(a.Y, (int64_t)min(t + 2, t1 - 1) * a.d + c);
    s[5] = squares(next);
#pragma unroll
    for (int i = 0; i < 5; ++i) s[i] = on ? s[i] : 0.f;
    norm_sums(s, red[(t - t0) & 1]);
    float r2 = 0.f, c2 = 0.f;
    if (g.dXn) {
      r2 = rstd_of(s[0] * inv_d + a.eps);
      c2 = s[1] * r2 * inv_d;
    }
    const float c1 = a.gamma_post ? norm_dot(s[2], s[3], s[4], r2, c2) * r1 * inv_d : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float hn = h[e] * r2;
      D[e] = norm_D(D[e], gq[e] * q[e], hn, r2, c2);
      if (SUMS) {
        sum_y[e] += D[e] * (y[e] * r1);
        sum_h[e] += gq[e] * hn;
      }
    }
    if (BOTH || g.dX) store8<BF>(g.dX, at, D);
    if (BOTH || g.dY) {
#pragma unroll
      for (int e = 0; e < 8; ++e) D[e] = norm_dY(agp[e] * D[e], y[e], r1, c1);
      store8<BF>(g.dY, at, D);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = next[e];
    if (a.gamma_post) r1 = rstd_of(s[5] * inv_d + a.eps);
  }
  if (SUMS && on) {
    float* const o = partial + (int64_t)(jobs.unit_base + (int)blockIdx.x) * 3 * a.d + c;
    float p[8], gate[8], v[8];
    load8_or<BF>(jb.gate, c, 1.f, gate);
    load8_or<BF>(a.gamma_post, c, 1.f, p);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = gate[e] * a.res_scale * sum_y[e];
    if (g.sums & 1) store8<false>(o, 0, v);
    if (g.sums & 2) store8<false>(o, a.d, sum_h);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = p[e] * a.res_scale * sum_y[e];
    if (g.sums & 4) store8<false>(o, 2 * (int64_t)a.d, v);
  }
}

// rstd of Y and of H, and c2 of norm_D
struct NormRow {
  float r1, r2, c2, pad;
};

// Backward of one row per workgroup, two runs per thread; the column sums are left to norm_bwd_cols_kernel.
template <bool BF>
__global__ void __launch_bounds__(1024) norm_bwd_row_kernel(NormArgs a, NormJobs jobs, NormGrads g, NormRow* __restrict__ rows) {
  __shared__ float red[2][5][16];
  const NormJob jb = jobs.job[norm_job(jobs, blockIdx.x)];
  const int t = jb.row0 + (int)blockIdx.x - jb.unit0;
  const int64_t row = (int64_t)t * a.d;
  const int c0 = (int)threadIdx.x * 8, step = (int)blockDim.x * 8;
  const float inv_d = 1.0f / (float)a.d;
  float y[2][8], h[2][8], D[2][8], gq[2][8];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int c = min(c0 + k * step, a.d - 8);
    load8<BF>(a.Y, row + c, y[k]);
    load8_or<BF>(a.X, row + c, 0.f, h[k]);
    load8_or<BF>(g.dH, row + c, 0.f, D[k]);
    load8_or<BF>(g.dXn, row + c, 0.f, gq[k]);
  }
  float r1 = 1.f;
  if (a.gamma_post) {
    float s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += c0 + k * step < a.d ? y[k][e] * y[k][e] : 0.f;
    norm_sums(s, red[0]);
    r1 = rstd_of(s[0] * inv_d + a.eps);
  }
  float s[5] = {};                          // as norm_bwd_unit_kernel's
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int c = min(c0 + k * step, a.d - 8);
    float agp[8], p[8], q[8];
    load8_or<BF>(jb.gate, c, 1.f, agp);
    load8_or<BF>(a.gamma_post, c, 1.f, p);
    load8_or<BF>(g.dXn ? a.gamma_pre : nullptr, c, 0.f, q);
    const bool on = c0 + k * step < a.d;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      agp[e] *= p[e] * a.res_scale;
      const float w = agp[e] * y[k][e];
      h[k][e] += w * r1;
      gq[k][e] *= q[e];
      if (on) {
        s[0] += h[k][e] * h[k][e];
        s[1] += gq[k][e] * h[k][e];
        s[2] += D[k][e] * w;
        s[3] += gq[k][e] * w;
        s[4] += h[k][e] * w;
      }
    }
  }
  norm_sums(s, red[1]);
  float r2 = 0.f, c2 = 0.f;
  if (g.dXn) {
    r2 = rstd_of(s[0] * inv_d + a.eps);
    c2 = s[1] * r2 * inv_d;
  }
  const float c1 = a.gamma_post ? norm_dot(s[2], s[3], s[4], r2, c2) * r1 * inv_d : 0.f;
  if (rows && threadIdx.x == 0) rows[t] = NormRow{r1, r2, c2, 0.f};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int c = c0 + k * step;
    if (c >= a.d) continue;
#pragma unroll
    for (int e = 0; e < 8; ++e) D[k][e] = norm_D(D[k][e], gq[k][e], h[k][e] * r2, r2, c2);
    if (g.dX) store8<BF>(g.dX, row + c, D[k]);
    if (g.dY) {
      float agp[8], p[8];
      load8_or<BF>(jb.gate, c, 1.f, agp);
      load8_or<BF>(a.gamma_post, c, 1.f, p);
#pragma unroll
      for (int e = 0; e < 8; ++e) D[k][e] = norm_dY(agp[e] * (p[e] * a.res_scale) * D[k][e], y[k][e], r1, c1);
      store8<BF>(g.dY, row + c, D[k]);
    }
  }
}

// ---- wider rows: read again for every sum -----------------------------------------------------------------------------------
template <bool BF>
__device__ __forceinline__ void norm_elements(const NormArgs& a, const void* gate, const NormGrads& g, int64_t row, int c, float r1, float r2,
                                              float c2, float (&y)[8], float (&pn)[8], float (&h)[8], float (&gn)[8], float (&D)[8],
                                              float (&ag)[8]) {
  float p[8];
  load8<BF>(a.Y, row + c, y);
  load8_or<BF>(a.gamma_post, c, 1.f, p);
  load8_or<BF>(gate, c, 1.f, ag);
  load8_or<BF>(a.X, row + c, 0.f, h);
  load8_or<BF>(g.dH, row + c, 0.f, D);
  load8_or<BF>(g.dXn, row + c, 0.f, gn);
  float q[8];
  load8_or<BF>(a.gamma_pre, c, 0.f, q);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    pn[e] = p[e];
    ag[e] *= a.res_scale;
    h[e] += ag[e] * (y[e] * r1 * p[e]);
    D[e] = norm_D(D[e], gn[e] * q[e], h[e] * r2, r2, c2);
  }
}

// units are rows
template <bool BF>
__global__ void __launch_bounds__(256) norm_bwd_rows_kernel(NormArgs a, NormJobs jobs, NormGrads g, NormRow* __restrict__ rows) {
  __shared__ float red[4];
  const NormJob jb = jobs.job[norm_job(jobs, blockIdx.x)];
  const int t = jb.row0 + (int)blockIdx.x - jb.unit0;
  const int64_t row = (int64_t)t * a.d;
  const float inv_d = 1.0f / (float)a.d;
  float r1 = 1.f, r2 = 0.f, c2 = 0.f;
  if (a.gamma_post) {
    float ss = 0.f;
    for (int c = threadIdx.x * 8; c < a.d; c += 2048) {
      float y[8];
      load8<BF>(a.Y, row + c, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += y[e] * y[e];
    }
    r1 = 1.0f / sqrtf(block_sum(ss, red) * inv_d + a.eps);
  }
  float y[8], p[8], h[8], gn[8], D[8], ag[8];
  if (g.dXn) {
    float ss = 0.f, dot = 0.f;
    for (int c = threadIdx.x * 8; c < a.d; c += 2048) {
      norm_elements<BF>(a, jb.gate, g, row, c, r1, 0.f, 0.f, y, p, h, gn, D, ag);
      float q[8];
      load8<BF>(a.gamma_pre, c, q);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ss += h[e] * h[e];
        dot += gn[e] * q[e] * h[e];
      }
    }
    r2 = 1.0f / sqrtf(block_sum(ss, red) * inv_d + a.eps);
    c2 = block_sum(dot, red) * r2 * inv_d;
  }
  if (rows && threadIdx.x == 0) rows[t] = NormRow{r1, r2, c2, 0.f};
  float c1 = 0.f;
  if (a.gamma_post && g.dY) {
    float dot = 0.f;
    for (int c = threadIdx.x * 8; c < a.d; c += 2048) {
      norm_elements<BF>(a, jb.gate, g, row, c, r1, r2, c2, y, p, h, gn, D, ag);
#pragma unroll
      for (int e = 0; e < 8; ++e) dot += ag[e] * D[e] * p[e] * y[e];
    }
    c1 = block_sum(dot, red) * r1 * inv_d;
  }
  if (!g.dX && !g.dY) return;
  for (int c = threadIdx.x * 8; c < a.d; c += 2048) {
    norm_elements<BF>(a, jb.gate, g, row, c, r1, r2, c2, y, p, h, gn, D, ag);
    if (g.dX) store8<BF>(g.dX, row + c, D);
    if (g.dY) {
#pragma unroll
      for (int e = 0; e < 8; ++e) D[e] = norm_dY(ag[e] * D[e] * p[e], y[e], r1, c1);
      store8<BF>(g.dY, row + c, D);
    }
  }
}

// Column sums of a unit's rows: a workgroup has 512 columns, its four waves every fourth row.  partial [unit][3][d]: dgamma_post,
// dgamma_pre, dgate.
template <bool BF>
__global__ void __launch_bounds__(256) norm_bwd_cols_kernel(NormArgs a, NormJobs jobs, NormGrads g, const NormRow* __restrict__ rows,
                                                            int unit_rows, float* __restrict__ partial) {
  __shared__ float red[4][3][512];
  const NormJob jb = jobs.job[norm_job(jobs, blockIdx.x)];
  const int t0 = jb.row0 + ((int)blockIdx.x - jb.unit0) * unit_rows, t1 = min(t0 + unit_rows, jb.row1);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (int)blockIdx.y * 512 + lane * 8;
  float s[3][8] = {};
  if (c < a.d)
    for (int t = t0 + wave; t < t1; t += 4) {
      const NormRow r = rows[t];
      float y[8], p[8], h[8], gn[8], D[8], ag[8];
      norm_elements<BF>(a, jb.gate, g, (int64_t)t * a.d, c, r.r1, r.r2, r.c2, y, p, h, gn, D, ag);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float yn = y[e] * r.r1;
        s[0][e] += ag[e] * D[e] * yn;
        s[1][e] += gn[e] * (h[e] * r.r2);
        s[2][e] += a.res_scale * (D[e] * (yn * p[e]));
      }
    }
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) red[wave][k][lane * 8 + e] = s[k][e];
  __syncthreads();
  for (int i = threadIdx.x; i < 3 * 512; i += 256) {
    const int k = i >> 9, x = i & 511, col = (int)blockIdx.y * 512 + x;
    if (col < a.d && (g.sums >> k & 1))
      partial[((int64_t)(jobs.unit_base + (int)blockIdx.x) * 3 + k) * a.d + col] =
          (red[0][k][x] + red[1][k][x]) + (red[2][k][x] + red[3][k][x]);
  }
}

// Sums over units in a fixed order: 64 columns per workgroup, 16 slices of the units side by side.  Vectors 0 and 1 are the gammas', over all
// units; vector 2 + j the gate of the group's job j.
__global__ void __launch_bounds__(1024) norm_reduce_kernel(const float* __restrict__ partial, NormJobs jobs, int first_vector, int d,
                                                           float* gamma_post, float* gamma_pre, int all_units, int accumulate) {
  __shared__ float red[16][64];
  const int vec = (int)blockIdx.y + first_vector, x = threadIdx.x & 63, slice = threadIdx.x >> 6, c = (int)blockIdx.x * 64 + x;
  int u0 = 0, u1 = all_units, k = vec;
  float* out = vec == 0 ? gamma_post : gamma_pre;
  if (vec >= 2) {
    const NormJob& jb = jobs.job[vec - 2];
    out = jb.dgate;
    u0 = jobs.unit_base + jb.unit0;
    u1 = u0 + jb.units;
    k = 2;
  }
  if (!out) return;
  const int per = (u1 - u0 + 15) / 16, a = u0 + slice * per, b = min(a + per, u1);
  float s = 0.f;
  if (c < d) {
    const float* p = partial + ((int64_t)a * 3 + k) * d + c;
    int u = a;
    for (; u + 8 <= b; u += 8, p += 24 * (int64_t)d) {       // eight loads in flight
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = p[3 * (int64_t)d * i];
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
    for (; u < b; ++u, p += 3 * (int64_t)d) s += *p;
  }
  red[slice][x] = s;
  __syncthreads();
  if (slice == 0 && c < d) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += red[i][x];
    out[c] = accumulate ? out[c] + s : s;
  }
}

}  // namespace

void launch_norm_fwd(bool bf16, const NormArgs& a, const NormJobs& jobs, int rows, void* H, void* Xn, hipStream_t st) {
  if (rows == 0) return;
  if (a.d <= 2 * kNormRow) {
    const dim3 block(norm_threads(a.d));
#define TLORA_NORM_FWD(CH)                                                                                            \
  do {                                                                                                               \
    if (bf16) hipLaunchKernelGGL((norm_fwd_row_kernel<true, CH>), dim3(rows), block, 0, st, a, jobs, H, Xn);          \
    else      hipLaunchKernelGGL((norm_fwd_row_kernel<false, CH>), dim3(rows), block, 0, st, a, jobs, H, Xn);         \
  } while (0)
    if (a.d <= kNormRow) TLORA_NORM_FWD(1);
    else                 TLORA_NORM_FWD(2);
#undef TLORA_NORM_FWD
    return;
  }
  if (bf16) hipLaunchKernelGGL(norm_fwd_kernel<true>, dim3(rows), dim3(256), 0, st, a, jobs, H, Xn);
  else      hipLaunchKernelGGL(norm_fwd_kernel<false>, dim3(rows), dim3(256), 0, st, a, jobs, H, Xn);
}
bool norm_in_registers(bool bf16, int d) { return d <= norm_bwd_row(bf16); }
// Workgroups of the backward that the chip holds at a time: 16 waves to a CU, as its registers allow, or 8 for fp32.
int norm_resident_units(bool bf16, int d) {
  return norm_in_registers(bf16, d) ? 256 * (bf16 ? 16 : 8) / (norm_threads(d) / 64) : 512;
}
void launch_norm_bwd_units(bool bf16, const NormArgs& a, const NormJobs& jobs, const NormGrads& g, int units, int unit_rows,
                           float* partial, hipStream_t st) {
  if (units == 0) return;
  const dim3 block(norm_threads(a.d));
  const bool both = g.dX && g.dY;
#define TLORA_NORM_BWD(BF, SUMS)                                                                                              \
  do {                                                                                                                      \
    if (both) hipLaunchKernelGGL((norm_bwd_unit_kernel<BF, SUMS, true>), dim3(units), block, 0, st, a, jobs, g, unit_rows, partial);  \
    else      hipLaunchKernelGGL((norm_bwd_unit_kernel<BF, SUMS, false>), dim3(units), block, 0, st, a, jobs, g, unit_rows, partial); \
  } while (0)
  if (bf16) { if (partial) TLORA_NORM_BWD(true, true);  else TLORA_NORM_BWD(true, false); }
  else      { if (partial) TLORA_NORM_BWD(false, true); else TLORA_NORM_BWD(false, false); }
#undef TLORA_NORM_BWD
}
void launch_norm_bwd_rows(bool bf16, const NormArgs& a, const NormJobs& jobs, const NormGrads& g, int rows, float* row_stats,
                          hipStream_t st) {
  if (rows == 0) return;
  NormRow* const r = reinterpret_cast<NormRow*>(row_stats);
  if (a.d <= 2 * kNormRow) {
    const dim3 block((a.d + 1023) / 1024 * 64);      // (fp32 rows from kNormRow / 2 on too)
    if (bf16) hipLaunchKernelGGL(norm_bwd_row_kernel<true>, dim3(rows), block, 0, st, a, jobs, g, r);
    else      hipLaunchKernelGGL(norm_bwd_row_kernel<false>, dim3(rows), block, 0, st, a, jobs, g, r);
    return;
  }
  if (bf16) hipLaunchKernelGGL(norm_bwd_rows_kernel<true>, dim3(rows), dim3(256), 0, st, a, jobs, g, r);
  else      hipLaunchKernelGGL(norm_bwd_rows_kernel<false>, dim3(rows), dim3(256), 0, st, a, jobs, g, r);
}
void launch_norm_bwd_cols(bool bf16, const NormArgs& a, const NormJobs& jobs, const NormGrads& g, int units, int unit_rows,
                          const float* row_stats, float* partial, hipStream_t st) {
  if (units == 0) return;
  const dim3 grid(units, (a.d + 511) / 512);
  const NormRow* const r = reinterpret_cast<const NormRow*>(row_stats);
  if (bf16) hipLaunchKernelGGL(norm_bwd_cols_kernel<true>, grid, dim3(256), 0, st, a, jobs, g, r, unit_rows, partial);
  else      hipLaunchKernelGGL(norm_bwd_cols_kernel<false>, grid, dim3(256), 0, st, a, jobs, g, r, unit_rows, partial);
}
void launch_norm_reduce(const float* partial, const NormJobs& jobs, int first_vector, int vectors, int d, float* gamma_post,
                        float* gamma_pre, int all_units, bool accumulate, hipStream_t st) {
  if (vectors <= 0) return;
  hipLaunchKernelGGL(norm_reduce_kernel, dim3((d + 63) / 64, vectors), dim3(1024), 0, st, partial, jobs, first_vector, d, gamma_post,
                     gamma_pre, all_units, accumulate ? 1 : 0);
}

// ---------------------------------------------------------------------------------------------------
// Activations in 8 bits: 16 lanes of 8 values have a group of 128; a thread has four groups' values in flight.  Bound by memory (31744 x
// 12288 bf16: packing 219 to 245 us, 4.8 to 5.4 TB/s, unpacking 193 us, 6.1 TB/s; one group at a time and the maximum by exchanges through LDS, 259
// and 197).
// ---------------------------------------------------------------------------------------------------
namespace {

// Where a thread's values lie: row, group of the row, first column.  A workgroup has kCkptGroups consecutive groups, 16 at a time.
constexpr int kCkptSteps = 4, kCkptGroups = 16 * kCkptSteps;
struct CkptPlace {
  int64_t row, group;      // group: over all rows
  int col;
  bool on;
};
__device__ __forceinline__ CkptPlace ckpt_place(int64_t T, int d, int groups, int step) {
  const int64_t g0 = (int64_t)blockIdx.x * kCkptGroups;
  const int64_t r0 = g0 / groups;
  const int i = step * 16 + (int)(threadIdx.x >> 4), g = (int)(g0 - r0 * groups) + i, more = g / groups;
  CkptPlace p;
  p.row = r0 + more;
  p.group = g0 + i;
  p.col = (g - more * groups) * 128 + (int)(threadIdx.x & 15) * 8;
  p.on = p.row < T && p.col < d;
  return p;
}
// the largest of a lane's 16, in registers
template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true));
}

template <bool BF>
__global__ void __launch_bounds__(256) ckpt_pack_kernel(const void* __restrict__ X, int64_t T, int d, int groups,
                                                        uint8_t* __restrict__ codes, uint16_t* __restrict__ scales) {
  Raw8<BF> raw[kCkptSteps];
#pragma unroll
  for (int i = 0; i < kCkptSteps; ++i) {               // (what is not there repeats the last values)
    const CkptPlace p = ckpt_place(T, d, groups, i);
    raw[i].fetch(X, min(p.row, T - 1) * d + min(p.col, d - 8));
  }
#pragma unroll
  for (int i = 0; i < kCkptSteps; ++i) {
    const CkptPlace p = ckpt_place(T, d, groups, i);
    float v[8];
    raw[i].get(v);
    // the largest magnitude as an integer: infinities and NaN are the largest of all
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu);
    if (!p.on) top = 0;
    top = max_dpp<0xB1>(top);
    top = max_dpp<0x4E>(top);
    top = max_dpp<0x141>(top);
    top = max_dpp<0x140>(top);
    const float amax = __builtin_bit_cast(float, top);
    const bool finite = top < 0x7f000000u;             // below 2^127: 127 s, rounded, stays finite
    auto up = [](float x) { return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, x) + 0xffffu) & 0xffff0000u); };
    float s = up(amax / 127.0f);
    if (127.0f * s < amax) s = up(s * (1.0f + 0x1p-12f));  // (127 s is exact: the quotient had been rounded down onto the grid)
    s = fmaxf(s, 0x1p-100f);
    const float inv = 1.0f / s;
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // The fp32 quotient.  bf16: by the reciprocal and one correction, which is exact where the quotient has few bits, as at a tie;
      // any other quotient of two numbers of 8 bits is 2^-9 or more away from a tie.
      const float q = v[e] * inv;
      const float c = BF ? fmaf(fmaf(-q, s, v[e]), inv, q) : v[e] / s;
      const int code = finite ? (int)rintf(c) : 0;
      w[e >> 2] |= ((uint32_t)code & 0xffu) << (8 * (e & 3));
    }
    if (p.on) *reinterpret_cast<u32x2*>(codes + p.row * d + p.col) = u32x2{w[0], w[1]};
    if (p.row < T && (threadIdx.x & 15) == 0)
      scales[p.group] = finite ? (uint16_t)(__builtin_bit_cast(uint32_t, s) >> 16) : (uint16_t)0x7fc0;
  }
}

template <bool BF>
__global__ void __launch_bounds__(256) ckpt_unpack_kernel(const uint8_t* __restrict__ codes, const uint16_t* __restrict__ scales, int64_t T,
                                                          int d, int groups, void* __restrict__ X) {
  u32x2 w[kCkptSteps];
  uint16_t sc[kCkptSteps];
#pragma unroll
  for (int i = 0; i < kCkptSteps; ++i) {
    const CkptPlace p = ckpt_place(T, d, groups, i);
    w[i] = *reinterpret_cast<const u32x2*>(codes + min(p.row, T - 1) * d + min(p.col, d - 8));
    sc[i] = scales[min(p.group, T * groups - 1)];
  }
#pragma unroll
  for (int i = 0; i < kCkptSteps; ++i) {
    const CkptPlace p = ckpt_place(T, d, groups, i);
    const float s = bf16_float(sc[i]);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)(w[i][e >> 2] >> (8 * (e & 3))) * s;
    if (p.on) store8<BF>(X, p.row * d + p.col, v);
  }
}

}  // namespace

void launch_ckpt_pack(bool bf16, const void* X, int64_t T, int d, uint8_t* codes, uint16_t* scales, hipStream_t st) {
  const int groups = (d + 127) / 128;
  if (T == 0) return;
  const dim3 grid((unsigned)((T * groups + kCkptGroups - 1) / kCkptGroups));
  if (bf16) hipLaunchKernelGGL(ckpt_pack_kernel<true>, grid, dim3(256), 0, st, X, T, d, groups, codes, scales);
  else      hipLaunchKernelGGL(ckpt_pack_kernel<false>, grid, dim3(256), 0, st, X, T, d, groups, codes, scales);
}
void launch_ckpt_unpack(bool bf16, const uint8_t* codes, const uint16_t* scales, int64_t T, int d, void* X, hipStream_t st) {
  const int groups = (d + 127) / 128;
  if (T == 0) return;
  const dim3 grid((unsigned)((T * groups + kCkptGroups - 1) / kCkptGroups));
  if (bf16) hipLaunchKernelGGL(ckpt_unpack_kernel<true>, grid, dim3(256), 0, st, codes, scales, T, d, groups, X);
  else      hipLaunchKernelGGL(ckpt_unpack_kernel<false>, grid, dim3(256), 0, st, codes, scales, T, d, groups, X);
}

}  // namespace tlora
