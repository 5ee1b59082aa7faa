// The blocks of an 8-bit cache that a new token's queries may score highest.
//
//   S_n = sum_g sum_d (q_gd > 0 ? q_gd hi_nd : q_gd lo_nd)
//       = sum_d (sum_g max(q_gd, 0)) hi_nd + (sum_g min(q_gd, 0)) lo_nd,
// so the queries of a KV head are summed first and a block costs one product of
// 2 D, whatever the group: 4 D bytes of bounds for block_size * 2 D of codes.  The
// sums are in 64 bits: exact as long as their terms, of 16 bits and a few for the
// sum over the queries, lie within 2^30 of one another, so that their order does not
// decide which block is chosen.
//
// Rows of up to kShort blocks (32768 tokens in blocks of 64) are scored and ranked
// by one workgroup for each head, which compares every score with every other. A
// longer row's scores are shared out to more workgroups; a second launch finds the
// k-th largest by a radix selection on order-preserving bit patterns, 11 bits a step
// from the first that differs, ended as soon as a digit separates the k largest.
// The trips to memory bound it: lengths, table, bounds.
// Measured: 64 rows of up to 104 blocks, 8 KV heads, 28 MB of bounds at most: 11.9 us
// (scores and a radix selection in two launches 22); one row of 2048 blocks, 4 KV
// heads: 6.3 to score, 8.4 to select.
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

// Comparing every score with every other costs the square of the blocks; the second
// launch, and shares that find nothing to do, cost every call whose table is wide
// enough for a longer row.  64 rows of up to 104 blocks, 8 KV heads, in a table of 300
// or 500: 11.9 us, with 256 in the place of 512 21.9.  Rows that are that long pay for
// it: 64 of 250 blocks take 25.5 us the one way, 27.1 the other, of 300 38.5 and 30.9,
// of 500 67.6 and 41.9; one row, 4 KV heads, 16.7 and 11.3, 28.4 and 11.6, 44.0 and 11.4.
constexpr int kShort = 512;
constexpr int kScoreThreads = 512, kScoreWaves = kScoreThreads / 64;

// A score's bit pattern as an integer of the same order; NaN as -inf, -0 as 0.
__device__ __forceinline__ uint64_t order_of(double s) {
  s = s != s ? -__builtin_inf() : s + 0.0;
  const uint64_t u = (uint64_t)__double_as_longlong(s);
  return u >> 63 ? ~u : u | (1ull << 63);
}

// Sum over L neighbouring lanes, in each of them.
template <int CTRL>
__device__ __forceinline__ double add_dpp(double s) {
  const uint64_t u = (uint64_t)__double_as_longlong(s);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)u, CTRL, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(u >> 32), CTRL, 0xF, 0xF, true);
  return s + __longlong_as_double((int64_t)(((uint64_t)hi << 32) | lo));
}
template <int L>
__device__ __forceinline__ double lanes_sum(double s) {
  s = add_dpp<0xB1>(s);   // quad_perm: lane ^ 1
  s = add_dpp<0x4E>(s);   // lane ^ 2
  s = add_dpp<0x141>(s);  // row_half_mirror: the other four of eight
  if constexpr (L >= 16) s = add_dpp<0x140>(s);  // row_mirror: the other eight
  if constexpr (L >= 32) s += __shfl_xor(s, 16);
  return s;
}

// Writes the numbers of the blocks that threads take, those of lower threads first,
// from out[at] on; returns how many.
template <int Waves>
__device__ __forceinline__ int put_taken(bool take, int block, int32_t* out, int at, int* sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t taken = __ballot(take);
  if (lane == 0) sums[wave] = __popcll(taken);
  __syncthreads();
  int place = at + __popcll(taken & ((1ull << lane) - 1)), all = 0;
#pragma unroll
  for (int w = 0; w < Waves; ++w) {
    if (w < wave) place += sums[w];
    all += sums[w];
  }
  if (take) out[place] = block;
  __syncthreads();
  return all;
}

// A workgroup: a (row, head), or one of `parts` shares of a long row's blocks.
template <int D>
__global__ __launch_bounds__(kScoreThreads) void score_kernel(const SelectParams p, int parts) {
  constexpr int L = D / 8;  // lanes of a block, 8 channels each
  constexpr int kAtOnce = kScoreThreads / L;
  constexpr int kShares = kScoreThreads / D < 4 ? kScoreThreads / D : 4;
  __shared__ double up_lds[kShares][D], down_lds[kShares][D];
  __shared__ uint64_t keys[kShort];
  __shared__ int sums[kScoreWaves];
  const PagedCache& c = p.cache;
  const int64_t item = blockIdx.x / parts;
  const int part = (int)(blockIdx.x - item * parts);
  const int b = (int)(item / c.H), h = (int)(item - (int64_t)b * c.H);
  const Blocks row = row_blocks(p, b);
  const bool all = row.count <= p.budget, brief = row.count <= kShort;
  if (part > 0 && (all || brief)) return;
  int32_t* out = p.blocks + item * p.budget;
  if (all) {
    for (int i = threadIdx.x; i < p.budget; i += kScoreThreads) out[i] = i < row.count ? row.first + i : -1;
    return;
  }
  const int c8 = (threadIdx.x % L) * 8;
  const int i0 = brief ? 0 : (int)((int64_t)row.count * part / parts), i1 = brief ? row.count : (int)((int64_t)row.count * (part + 1) / parts);
  if (i0 >= i1) return;  // more shares than blocks

  // Blocks are taken kAhead at a time and thread; the pages, then the bounds, of the
  // first are asked for before the queries are summed.
  constexpr int kAhead = 4;
  u32x4 lo[kAhead], hi[kAhead];
  bool in[kAhead];
  auto fetch = [&](int k0) __attribute__((always_inline)) {
    int page[kAhead];
    uint32_t sub[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = min(k0 + k * kAtOnce, i1 - 1);
      const uint32_t t = (uint32_t)(row.first + i) << p.block_shift;
      const uint32_t pg = divide(t, c);
      page[k] = c.table[(int64_t)b * c.max_pages + pg];
      sub[k] = (t - pg * (uint32_t)c.page_size) >> p.block_shift;
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      in[k] = page[k] >= 0 && page[k] < c.num_pages;
      const uint16_t* bounds = p.bounds + (((int64_t)(in[k] ? page[k] : 0) * c.H + h) * p.page_blocks + sub[k]) * 2 * D + c8;
      lo[k] = *(const u32x4*)bounds;
      hi[k] = *(const u32x4*)(bounds + D);
    }
  };
  // the sums over the queries: a thread has a channel and a share of the queries
  const int d = threadIdx.x % D, share = threadIdx.x / D;
  const uint16_t* q = p.q.data + b * p.q.token_stride + (int64_t)h * p.R * p.q.head_stride + d;
  const uint16_t q0 = share < p.R && share < kShares ? q[share * p.q.head_stride] : 0;
  int k0 = i0 + threadIdx.x / L;
  fetch(k0);
  if (share < kShares) {
    double u = 0, l = 0;
    for (int g = share; g < p.R; g += kShares) {
      const float x = bf16_as_float(g == share ? q0 : q[g * p.q.head_stride]);
      // NaN goes into both
      u += x < 0 ? 0.0f : x;
      l += x > 0 ? 0.0f : x;
    }
    up_lds[share][d] = u;
    down_lds[share][d] = l;
  }
  __syncthreads();
  double up[8], down[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    up[e] = up_lds[0][c8 + e];
    down[e] = down_lds[0][c8 + e];
#pragma unroll
    for (int s = 1; s < kShares; ++s) {
      up[e] += up_lds[s][c8 + e];
      down[e] += down_lds[s][c8 + e];
    }
  }
  while (k0 < i1) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (k0 + k * kAtOnce >= i1) break;
      double s = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float l = e & 1 ? bf16_hi(lo[k][e / 2]) : bf16_lo(lo[k][e / 2]), u = e & 1 ? bf16_hi(hi[k][e / 2]) : bf16_lo(hi[k][e / 2]);
        // a bound that no query has a factor for does not count, infinite ones too
        s = __builtin_fma(down[e], (double)(down[e] == 0 ? 0.0f : l), s);
        s = __builtin_fma(up[e], (double)(up[e] == 0 ? 0.0f : u), s);
      }
      s = lanes_sum<L>(s);
      const int i = k0 + k * kAtOnce;
      if (threadIdx.x % L == 0) {
        const uint64_t key = order_of(in[k] ? s : -__builtin_inf());
        if (brief) keys[i] = key;
        else p.keys[item * p.row_blocks + i] = key;
      }
    }
    k0 += kAtOnce * kAhead;
    if (k0 < i1) fetch(k0);
  }
  if (!brief) return;
  __syncthreads();
  // blocks [first, last) of the row compete for `want` places; 16 threads or fewer rank one
  const int first = p.first, last = row.count - p.last, want = p.budget - p.first - p.last;
  int sharers = 1;
  while (sharers < 16 && sharers * 2 * row.count <= kScoreThreads) sharers *= 2;
  const int i = threadIdx.x / sharers;
  bool take = i < row.count;
  if (i >= first && i < last) {
    const uint64_t key = keys[i];
    int before = 0;
#pragma unroll 4
    for (int k = first + (threadIdx.x & (sharers - 1)); k < last; k += sharers) before += keys[k] >= key + (k >= i);
    for (int m = 1; m < sharers; m *= 2) before += __shfl_xor(before, m);
    take = before < want;
  }
  put_taken<kScoreWaves>(take && threadIdx.x % sharers == 0, row.first + i, out, 0, sums);
}

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kDigit = 11, kBins = 1 << kDigit;
constexpr int kHeldKeys = 8192;  // of a row, in LDS; of longer rows they are read again for each digit

__global__ __launch_bounds__(kSelectThreads) void select_kernel(const SelectParams p) {
  extern __shared__ uint64_t held[];
  __shared__ int bins[kBins];
  __shared__ int sums[kSelectWaves], ties[kSelectWaves];
  __shared__ uint64_t differ[kSelectWaves];
  __shared__ int found[3];
  const int64_t item = blockIdx.x;
  const int b = (int)(item / p.cache.H);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Blocks row = row_blocks(p, b);
  if (row.count <= p.budget || row.count <= kShort) return;
  int32_t* out = p.blocks + item * p.budget;
  // blocks [lo, hi) of the row compete for `want` places
  const int lo = p.first, hi = row.count - p.last;
  int want = p.budget - p.first - p.last;
  const uint64_t* keys = p.keys + item * p.row_blocks;
  const bool in_lds = hi - lo <= kHeldKeys;
  auto key_of = [&](int i) __attribute__((always_inline)) { return in_lds ? held[i - lo] : keys[i]; };
  // the first bit in which the keys differ
  const uint64_t one = keys[lo];
  uint64_t bits = 0;
  for (int i = lo + tid; i < hi; i += kSelectThreads) {
    const uint64_t key = keys[i];
    if (in_lds) held[i - lo] = key;
    bits |= key ^ one;
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) bits |= __shfl_xor((unsigned long long)bits, m);
  if (lane == 0) differ[wave] = bits;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelectWaves; ++w) bits |= differ[w];
  // chosen: keys >> shift above `least`, and the first `want` that equal it
  int shift = bits ? 64 - __clzll(bits) : 0;
  uint64_t least = shift == 64 ? 0 : one >> shift;
  bool all_equal = false;  // all that equal it
  while (want > 0 && shift > 0) {
    const int digit = min(kDigit, shift), size = 1 << digit;
    const int next = shift - digit;
    for (int i = tid; i < size; i += kSelectThreads) bins[i] = 0;
    __syncthreads();
    for (int i = lo + tid; i < hi; i += kSelectThreads) {
      const uint64_t key = key_of(i);
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
      const uint64_t key = key_of(i), upper = shift == 64 ? 0 : key >> shift;
      take = upper > least || (all_equal && upper == least);
      tie = !all_equal && upper == least;
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
    at += put_taken<kSelectWaves>(take || (tie && rank < want), row.first + i, out, at, sums);
  }
}

// Workgroups that share a long row's blocks: about four a compute unit in all, each
// with a turn's blocks at least.
int score_parts(const SelectParams& p) {
  const int64_t items = (int64_t)p.cache.B * p.cache.H;
  const int64_t turn = kScoreThreads / (p.D / 8);
  const int64_t most = p.row_blocks <= kShort ? 1 : (p.row_blocks + turn - 1) / turn;
  const int64_t n = (1024 + items - 1) / items;
  return (int)(n < most ? n : most);
}

}  // namespace

int64_t select_work_items(const SelectParams& p) {
  const int64_t items = (int64_t)p.cache.B * p.cache.H;
  if (items > kMaxWorkItems / kSelectThreads) return kMaxWorkItems + 1;
  const int64_t a = items * score_parts(p) * kScoreThreads, b = items * kSelectThreads;
  return a > b ? a : b;
}

hipError_t launch_scores(const SelectParams& p, hipStream_t stream) {
  const int parts = score_parts(p);
  const dim3 grid((uint32_t)((int64_t)p.cache.B * p.cache.H * parts)), threads(kScoreThreads);
  switch (p.D) {
    case 64: score_kernel<64><<<grid, threads, 0, stream>>>(p, parts); break;
    case 128: score_kernel<128><<<grid, threads, 0, stream>>>(p, parts); break;
    default: score_kernel<256><<<grid, threads, 0, stream>>>(p, parts); break;
  }
  return hipGetLastError();
}

bool select_has_long_rows(const SelectParams& p) { return p.row_blocks > kShort && p.row_blocks > p.budget; }

hipError_t launch_select(const SelectParams& p, hipStream_t stream) {
  const int64_t n = p.row_blocks < kHeldKeys ? p.row_blocks : kHeldKeys;
  const size_t bytes = (size_t)n * sizeof(uint64_t);
  if (bytes > 32 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)select_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return e;
  }
  select_kernel<<<dim3((uint32_t)((int64_t)p.cache.B * p.cache.H)), dim3(kSelectThreads), bytes, stream>>>(p);
  return hipGetLastError();
}

}  // namespace hg
