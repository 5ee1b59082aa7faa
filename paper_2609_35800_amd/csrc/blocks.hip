// The blocks of an 8-bit cache that a new token's queries may score highest.
//
//   S_n = sum_g sum_d (q_gd > 0 ? q_gd hi_nd : q_gd lo_nd)
//       = sum_d (sum_g max(q_gd, 0)) hi_nd + (sum_g min(q_gd, 0)) lo_nd,
// so the queries of a KV head are summed first and a block costs one product of
// 2 D, whatever the group: 4 D bytes of bounds for block_size * 2 D of codes.  The
// sums are in 64 bits.  The products of two BF16 numbers have 16 bits, so the sums
// are exact unless the products lie more than 2^37 apart, and their order does not
// decide which block is chosen.
//
// One launch scores, one chooses: the k-th largest score of a (row, head) by a
// radix selection on order-preserving bit patterns, 11 bits a step from the top,
// ended as soon as a digit separates the k largest; then the chosen blocks' numbers
// are written in order.
#include "hg_attn.h"
#include "hg_device.h"

namespace hg {
namespace {

// Blocks of a row's attended tokens.
struct Blocks {
  int first, count;
};
__device__ __forceinline__ Blocks row_blocks(const SelectParams& p, int b) {
  const int len = clamp_to(p.lens[b], p.cache.max_tokens);
  const int start = p.starts ? min(clamp_to(p.starts[b], p.cache.max_tokens), len) : 0;
  if (start >= len) return Blocks{0, 0};
  const int n0 = start >> p.block_shift;
  return Blocks{n0, ((len - 1) >> p.block_shift) - n0 + 1};
}

constexpr int kScoreThreads = 256;
constexpr int kScoreBlocks = 64;  // blocks of a workgroup

template <int D>
__global__ __launch_bounds__(kScoreThreads) void scores_kernel(const SelectParams p, int groups) {
  constexpr int L = D / 8;  // lanes of a block, 8 channels each
  constexpr int kAtOnce = kScoreThreads / L;
  const PagedCache& c = p.cache;
  const int64_t item = blockIdx.x / groups;
  const int group = (int)(blockIdx.x - item * groups);
  const int b = (int)(item / c.H), h = (int)(item - (int64_t)b * c.H);
  const Blocks row = row_blocks(p, b);
  if (row.count <= p.budget || group * kScoreBlocks >= row.count) return;
  const int c8 = (threadIdx.x % L) * 8;

  double up[8], down[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) up[e] = down[e] = 0;
  for (int g = 0; g < p.R; ++g) {
    const u32x4 q = *(const u32x4*)(p.q.data + b * p.q.token_stride + (h * p.R + g) * p.q.head_stride + c8);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = e & 1 ? bf16_hi(q[e / 2]) : bf16_lo(q[e / 2]);
      // NaN goes into both
      up[e] += x < 0 ? 0.0f : x;
      down[e] += x > 0 ? 0.0f : x;
    }
  }
  for (int k = threadIdx.x / L; k < kScoreBlocks; k += kAtOnce) {
    const int i = group * kScoreBlocks + k;
    double s = -__builtin_inf();
    if (i < row.count) {
      const uint32_t t = (uint32_t)(row.first + i) << p.block_shift;
      const uint32_t pg = divide(t, c);
      const int page = c.table[(int64_t)b * c.max_pages + pg];
      if (page >= 0 && page < c.num_pages) {
        const uint32_t sub = (t - pg * (uint32_t)c.page_size) >> p.block_shift;
        const uint16_t* bounds = p.bounds + (((int64_t)page * c.H + h) * p.page_blocks + sub) * 2 * D + c8;
        const u32x4 lo = *(const u32x4*)bounds, hi = *(const u32x4*)(bounds + D);
        s = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float l = e & 1 ? bf16_hi(lo[e / 2]) : bf16_lo(lo[e / 2]), u = e & 1 ? bf16_hi(hi[e / 2]) : bf16_lo(hi[e / 2]);
          // a bound that no query has a factor for does not count, infinite ones too
          s = __builtin_fma(down[e], (double)(down[e] == 0 ? 0.0f : l), s);
          s = __builtin_fma(up[e], (double)(up[e] == 0 ? 0.0f : u), s);
        }
      }
    }
#pragma unroll
    for (int m = 1; m < L; m *= 2) s += __shfl_xor(s, m);
    if (i < row.count && threadIdx.x % L == 0) p.scores[item * p.row_blocks + i] = s;
  }
}

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kDigit = 11, kBins = 1 << kDigit;

// A score's bit pattern as an integer of the same order; NaN as -inf, -0 as 0.
__device__ __forceinline__ uint64_t order_of(double s) {
  s = s != s ? -__builtin_inf() : s + 0.0;
  const uint64_t u = (uint64_t)__double_as_longlong(s);
  return u >> 63 ? ~u : u | (1ull << 63);
}

__global__ __launch_bounds__(kSelectThreads) void select_kernel(const SelectParams p) {
  __shared__ int bins[kBins];
  __shared__ int sums[kSelectWaves], ties[kSelectWaves];
  __shared__ int found[3];
  const int64_t item = blockIdx.x;
  const int b = (int)(item / p.cache.H);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Blocks row = row_blocks(p, b);
  int32_t* out = p.blocks + item * p.budget;
  if (row.count <= p.budget) {
    for (int i = tid; i < p.budget; i += kSelectThreads) out[i] = i < row.count ? row.first + i : -1;
    return;
  }
  // blocks [lo, hi) of the row compete for `want` places
  const int lo = p.first, hi = row.count - p.last;
  int want = p.budget - p.first - p.last;
  const double* scores = p.scores + item * p.row_blocks;
  // chosen: keys >> shift above `least`, and the first `want` that equal it
  uint64_t least = 0;
  int shift = 64;
  bool all_equal = false;  // all that equal it
  while (want > 0 && shift > 0) {
    const int digit = min(kDigit, shift), size = 1 << digit;
    const int next = shift - digit;
    for (int i = tid; i < size; i += kSelectThreads) bins[i] = 0;
    __syncthreads();
    for (int i = lo + tid; i < hi; i += kSelectThreads) {
      const uint64_t key = order_of(scores[i]);
      if (shift == 64 || key >> shift == least) atomicAdd(&bins[(key >> next) & (size - 1)], 1);
    }
    __syncthreads();
    // sums from the highest bin down; a thread holds two neighbours
    const int top = size - 1 - 2 * tid;
    const int c0 = top >= 0 ? bins[top] : 0, c1 = top >= 1 ? bins[top - 1] : 0;
    const int s = lane_scan(c0 + c1);
    if (lane == 63) sums[wave] = s;
    __syncthreads();
    int past = s - c0 - c1;
    for (int w = 0; w < wave; ++w) past += sums[w];
    if (past < want && want <= past + c0) {
      found[0] = top;
      found[1] = past;
      found[2] = c0;
    } else if (past + c0 < want && want <= past + c0 + c1) {
      found[0] = top - 1;
      found[1] = past + c0;
      found[2] = c1;
    }
    __syncthreads();
    least = (least << digit) | (uint64_t)found[0];
    want -= found[1];
    shift = next;
    all_equal = found[2] == want;
    if (all_equal) break;
    __syncthreads();
  }
  // the chosen ones in order
  const bool any = p.budget > p.first + p.last;
  int at = 0, equal = 0;  // written, and equal ones passed
  for (int i0 = 0; i0 < row.count; i0 += kSelectThreads) {
    const int i = i0 + tid;
    bool take = i < row.count && (i < lo || i >= hi), tie = false;
    if (any && i >= lo && i < hi) {
      const uint64_t key = order_of(scores[i]) >> shift;
      take = key > least || (all_equal && key == least);
      tie = !all_equal && key == least;
    }
    const uint64_t tied = __ballot(tie);
    if (lane == 0) ties[wave] = __popcll(tied);
    __syncthreads();
    int rank = equal + __popcll(tied & ((1ull << lane) - 1)), tied_all = 0;
    for (int w = 0; w < kSelectWaves; ++w) {
      if (w < wave) rank += ties[w];
      tied_all += ties[w];
    }
    equal += tied_all;
    take = take || (tie && rank < want);
    const uint64_t taken = __ballot(take);
    if (lane == 0) sums[wave] = __popcll(taken);
    __syncthreads();
    int place = at + __popcll(taken & ((1ull << lane) - 1));
    for (int w = 0; w < kSelectWaves; ++w) {
      if (w < wave) place += sums[w];
      at += sums[w];
    }
    if (take) out[place] = row.first + i;
    __syncthreads();
  }
}

int64_t score_groups(const SelectParams& p) { return (p.row_blocks + kScoreBlocks - 1) / kScoreBlocks; }

}  // namespace

int64_t select_work_items(const SelectParams& p) {
  const int64_t items = (int64_t)p.cache.B * p.cache.H;
  const int64_t groups = score_groups(p);
  if (groups > kMaxWorkItems / kScoreThreads) return kMaxWorkItems + 1;
  const __int128 a = (__int128)items * groups * kScoreThreads, b = (__int128)items * kSelectThreads;
  const __int128 most = a > b ? a : b;
  return most > kMaxWorkItems ? kMaxWorkItems + 1 : (int64_t)most;
}

hipError_t launch_select_scores(const SelectParams& p, hipStream_t stream) {
  const int64_t groups = score_groups(p);
  const dim3 grid((uint32_t)((int64_t)p.cache.B * p.cache.H * groups)), threads(kScoreThreads);
  switch (p.D) {
    case 64: scores_kernel<64><<<grid, threads, 0, stream>>>(p, (int)groups); break;
    case 128: scores_kernel<128><<<grid, threads, 0, stream>>>(p, (int)groups); break;
    default: scores_kernel<256><<<grid, threads, 0, stream>>>(p, (int)groups); break;
  }
  return hipGetLastError();
}

hipError_t launch_select(const SelectParams& p, hipStream_t stream) {
  select_kernel<<<dim3((uint32_t)((int64_t)p.cache.B * p.cache.H)), dim3(kSelectThreads), 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace hg
