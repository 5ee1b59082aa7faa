// Rows of a paged cache brought to new lengths: pages given up and taken, the
// block table, offsets, slots and positions of the new tokens.
//
//   have = ceil(len / size), want = ceil(target / size) pages of a row; entries
//   [want, have) of its table go on top of the free pages, then entries [have,
//   want) come off the top, both in the order of rows and entries.
// So the place of an entry on the stack is a sum over the rows before it: a scan
// over the rows, then each entry on its own.  All that bounds it is the chain of
// trips to memory: one workgroup does the rows, 1024 at a time; the tokens of a
// large call are mapped by a second launch over all compute units.
#include "hg_attn.h"
#include "hg_device.h"

namespace hg {
namespace {

constexpr int kResizeThreads = 1024, kResizeWaves = kResizeThreads / 64;
// Tokens up to which the one workgroup maps them itself, without a second launch.
constexpr int kFewTokens = 8192;

__device__ __forceinline__ int64_t lane_scan64(int64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const uint32_t lo = __shfl_up((int)(uint32_t)v, s), hi = __shfl_up((int)(v >> 32), s);
    if (lane >= s) v += (int64_t)(((uint64_t)hi << 32) | lo);
  }
  return v;
}

// Sum over the threads before this one, and over all.
struct Scan {
  int64_t before, all;
};
__device__ __forceinline__ Scan block_scan(int64_t v, int64_t* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t s = lane_scan64(v);
  if (lane == 63) lds[wave] = s;
  __syncthreads();
  Scan r = {s - v, 0};
#pragma unroll
  for (int w = 0; w < kResizeWaves; ++w) {
    const int64_t x = lds[w];
    if (w < wave) r.before += x;
    r.all += x;
  }
  __syncthreads();
  return r;
}

// A row: its pages, and the tokens it gains.  Lengths outside the table count as
// none (the call is refused then).
struct Row {
  int have, want, gain;
  bool good;
};
__device__ __forceinline__ Row read_row(const ResizeParams& p, int b) {
  Row r = {0, 0, 0, true};
  if (b >= p.B) return r;
  const int64_t most = (int64_t)p.max_pages * p.page_size;
  const int len = p.lens[b], target = p.targets[b];
  r.good = len >= 0 && len <= most && target >= 0 && target <= most;
  if (!r.good) return r;
  const uint32_t size = p.page_size;
  r.have = (int)(((uint32_t)len + size - 1) / size);
  r.want = (int)(((uint32_t)target + size - 1) / size);
  r.gain = max(target - len, 0);
  return r;
}

// Slot and position of token i, of the rows' lengths as they are after the call.
__device__ __forceinline__ void map_token(const ResizeParams& p, int i, int tokens) {
  int64_t slot = -1;
  int position = -1;
  if (i < tokens) {
    int lo = 0, hi = p.B;  // the last row that starts at or before i; rows without tokens end there too
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.cu[mid] <= i) lo = mid;
      else hi = mid;
    }
    position = p.lens[lo] - p.cu[lo + 1] + i;
    const uint32_t pg = (uint32_t)position / (uint32_t)p.page_size;
    slot = (int64_t)p.table[(int64_t)lo * p.max_pages + pg] * p.page_size + ((uint32_t)position - pg * (uint32_t)p.page_size);
  }
  if (p.slots) p.slots[i] = slot;
  if (p.positions) p.positions[i] = position;
}

__global__ __launch_bounds__(kResizeThreads) void resize_kernel(const ResizeParams p, int few) {
  __shared__ int64_t lds[kResizeWaves];
  __shared__ int64_t row_at[kResizeThreads];
  __shared__ int row_from[kResizeThreads], row_to[kResizeThreads];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n_free = *p.n_free;

  int64_t freed = 0, taken = 0, gained = 0, bad = 0;
  for (int b0 = 0; b0 < p.B; b0 += kResizeThreads) {
    const Row r = read_row(p, b0 + threadIdx.x);
    freed += max(r.have - r.want, 0);
    taken += max(r.want - r.have, 0);
    gained += r.gain;
    bad += !r.good;
  }
  freed = block_scan(freed, lds).all;
  taken = block_scan(taken, lds).all;
  gained = block_scan(gained, lds).all;
  bad = block_scan(bad, lds).all;
  const int64_t top = n_free + freed, left = top - taken;
  const int64_t room = p.slots || p.positions ? p.N : 0x7FFFFFFF;
  int flags = (left < 0 ? 1 : 0) | (bad ? 2 : 0) | (gained > room ? 4 : 0);
  if (n_free < 0 || n_free > p.num_pages || top > p.num_pages) flags |= 8;

  // pages given up, then pages taken; a wavefront takes a row
  for (int pass = 0; pass < 2 && !flags; ++pass) {
    int64_t before = 0;
    for (int b0 = 0; b0 < p.B; b0 += kResizeThreads) {
      const Row r = read_row(p, b0 + threadIdx.x);
      const int from = pass ? r.have : r.want, to = pass ? r.want : r.have;
      const Scan s = block_scan(max(to - from, 0), lds);
      row_at[threadIdx.x] = before + s.before;
      row_from[threadIdx.x] = from;
      row_to[threadIdx.x] = to;
      before += s.all;
      __syncthreads();
      for (int i = wave; i < min(kResizeThreads, p.B - b0); i += kResizeWaves) {
        int32_t* row = p.table + (int64_t)(b0 + i) * p.max_pages;
        const int f = row_from[i], n = row_to[i] - f;
        for (int k = lane; k < n; k += 64) {
          if (pass) {
            row[f + k] = p.free_pages[top - 1 - (row_at[i] + k)];
          } else {
            p.free_pages[n_free + row_at[i] + k] = row[f + k];
            row[f + k] = -1;
          }
        }
      }
      __syncthreads();
    }
  }
  // offsets of the new tokens, lengths
  int64_t before = 0;
  for (int b0 = 0; b0 < p.B; b0 += kResizeThreads) {
    const int b = b0 + threadIdx.x;
    const Row r = read_row(p, b);
    const Scan s = block_scan(r.gain, lds);
    if (b < p.B) {
      if (p.cu) p.cu[b] = flags ? 0 : (int)(before + s.before);
      if (!flags) p.lens[b] = p.targets[b];
    }
    before += s.all;
  }
  if (threadIdx.x == 0) {
    if (p.cu) p.cu[p.B] = flags ? 0 : (int)gained;
    if (!flags) *p.n_free = (int)left;
    p.result[0] = flags;
    p.result[1] = left < 0 ? (int)min(-left, (int64_t)0x7FFFFFFF) : 0;
    p.result[2] = (int)min(gained, (int64_t)0x7FFFFFFF);
    p.result[3] = flags ? (int)n_free : (int)left;
  }
  if (!few) return;
  __syncthreads();
  for (int i = threadIdx.x; i < p.N; i += kResizeThreads) map_token(p, i, flags ? 0 : (int)gained);
}

constexpr int kSlotThreads = 256, kSlotTokens = 4;

__global__ __launch_bounds__(kSlotThreads) void slots_kernel(const ResizeParams p) {
  const int tokens = p.cu[p.B];
  const int64_t i0 = (int64_t)blockIdx.x * (kSlotThreads * kSlotTokens) + threadIdx.x;
#pragma unroll
  for (int k = 0; k < kSlotTokens; ++k) {
    const int64_t i = i0 + k * kSlotThreads;
    if (i < p.N) map_token(p, (int)i, tokens);
  }
}

}  // namespace

bool resize_maps_slots(const ResizeParams& p) { return p.N <= kFewTokens || (!p.slots && !p.positions); }

hipError_t launch_resize(const ResizeParams& p, hipStream_t stream) {
  const bool few = (p.slots || p.positions) && resize_maps_slots(p);
  resize_kernel<<<dim3(1), dim3(kResizeThreads), 0, stream>>>(p, few ? 1 : 0);
  return hipGetLastError();
}

hipError_t launch_slots(const ResizeParams& p, hipStream_t stream) {
  constexpr int64_t tile = kSlotThreads * kSlotTokens;
  slots_kernel<<<dim3((uint32_t)((p.N + tile - 1) / tile)), dim3(kSlotThreads), 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace hg
