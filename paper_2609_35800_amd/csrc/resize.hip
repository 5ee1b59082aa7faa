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
// Measured: 4 rows that gain a token 6.2 us, 256 rows that gain five 7.4, 64 prompts of
// up to 6656 tokens (13000 pages of 16) 9.2 and 6.0 for the slots of 210000 tokens.
#include <type_traits>

#include "hg_attn.h"
#include "hg_device.h"

namespace hg {
namespace {

constexpr int kResizeThreads = 1024, kResizeWaves = kResizeThreads / 64;
// Tokens up to which the one workgroup maps them itself, without a second launch (four
// rows that gain 500, 1000, 2000 and 4000 each, and lose them: 14.4, 15.3, 17.4 and 21.6
// us in one launch, 17.1, 17.3, 17.5 and 17.9 in two).
constexpr int kFewTokens = 8192;
constexpr int kRowEntries = 4;  // entries of a row that one thread moves

// Sums over the lanes up to this one, of values below 2^32, in 64 bits.
__device__ __forceinline__ int64_t lane_scan64(uint32_t v) {
  return ((int64_t)lane_scan((int)(v >> 16)) << 16) + lane_scan((int)(v & 0xFFFF));
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

// What the rows before a row give up, need and gain, and all rows of a tile.
struct Sums {
  int64_t freed, taken, gained;
};

// Slot and position of token i, of the rows' lengths as they are after the call;
// cu: offsets of the rows' new tokens, in LDS if there are few.
__device__ __forceinline__ void map_token(const ResizeParams& p, const int32_t* cu, int i, int tokens) {
  int64_t slot = -1;
  int position = -1;
  if (i < tokens) {
    int lo = 0, hi = p.B;  // the last row that starts at or before i; rows without tokens end there too
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (cu[mid] <= i) lo = mid;
      else hi = mid;
    }
    position = p.lens[lo] - cu[lo + 1] + i;
    const uint32_t pg = (uint32_t)position / (uint32_t)p.page_size;
    slot = (int64_t)p.table[(int64_t)lo * p.max_pages + pg] * p.page_size + ((uint32_t)position - pg * (uint32_t)p.page_size);
  }
  if (p.slots) p.slots[i] = slot;
  if (p.positions) p.positions[i] = position;
}

__global__ __launch_bounds__(kResizeThreads) void resize_kernel(const ResizeParams p, int few) {
  __shared__ Sums wave_sums[2][kResizeWaves];
  __shared__ int64_t row_at[kResizeThreads];  // entries of the rows before it
  __shared__ int row_from[kResizeThreads], row_n[kResizeThreads];
  __shared__ int32_t cu_lds[kResizeThreads + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n_free = *p.n_free;

  // The row of this thread in a tile and the sums before it; `all` grows by the tile's.
  int turn = 0;
  auto scan = [&](const Row& r, Sums& all) __attribute__((always_inline)) {
    const uint32_t f = max(r.have - r.want, 0), t = max(r.want - r.have, 0), g = r.gain;
    Sums s = {lane_scan64(f), lane_scan64(t), lane_scan64(g)};
    Sums* sums = wave_sums[turn++ & 1];
    if (lane == 63) sums[wave] = s;
    s = Sums{s.freed - f, s.taken - t, s.gained - g};
    __syncthreads();
    Sums before = all;
    for (int w = 0; w < kResizeWaves; ++w) {
      if (w == wave) before = all;
      all.freed += sums[w].freed;
      all.taken += sums[w].taken;
      all.gained += sums[w].gained;
    }
    return Sums{s.freed + before.freed, s.taken + before.taken, s.gained + before.gained};
  };

  const bool single = p.B <= kResizeThreads;  // one tile: its rows stay in registers
  Sums all = {0, 0, 0}, before = {0, 0, 0};
  Row row = {0, 0, 0, true};
  bool good = true;
  for (int b0 = 0; b0 < p.B; b0 += kResizeThreads) {
    row = read_row(p, b0 + threadIdx.x);
    before = scan(row, all);
    good = good && row.good;
  }
  const bool bad = __syncthreads_or(!good);
  const int64_t top = n_free + all.freed, left = top - all.taken;
  const int64_t room = p.slots || p.positions ? p.N : 0x7FFFFFFF;
  int flags = (left < 0 ? 1 : 0) | (bad ? 2 : 0) | (all.gained > room ? 4 : 0);
  if (n_free < 0 || n_free > p.num_pages || top > p.num_pages) flags |= 8;

  // pages given up, then, once all are, pages taken
  for (int pass = 0; pass < 2 && !flags; ++pass) {
    if (pass ? all.taken == 0 : all.freed == 0) continue;
    Sums sum = {0, 0, 0};
    for (int b0 = 0; b0 < p.B; b0 += kResizeThreads) {
      if (!single) {
        row = read_row(p, b0 + threadIdx.x);
        before = scan(row, sum);
      }
      const int from = pass ? row.have : row.want, n = max((pass ? row.want : row.have) - from, 0);
      const int64_t at = pass ? before.taken : before.freed;
      auto move = [&](int b, int64_t at, int from, int k0, int n, auto step) __attribute__((always_inline)) {
        constexpr int kStep = decltype(step)::value, kAhead = kRowEntries;
        int32_t* entries = p.table + (int64_t)b * p.max_pages + from;
        for (; k0 < n; k0 += kStep * kAhead) {
          int32_t page[kAhead];
#pragma unroll
          for (int k = 0; k < kAhead; ++k) {
            const int e = k0 + k * kStep;
            page[k] = e >= n ? 0 : pass ? p.free_pages[top - 1 - (at + e)] : entries[e];
          }
#pragma unroll
          for (int k = 0; k < kAhead; ++k) {
            const int e = k0 + k * kStep;
            if (e >= n) break;
            entries[e] = pass ? page[k] : -1;
            if (!pass) p.free_pages[n_free + at + e] = page[k];
          }
        }
      };
      if (n > 0 && n <= kRowEntries) move(b0 + threadIdx.x, at, from, 0, n, std::integral_constant<int, 1>());
      // the rows of more: a wavefront each
      row_at[threadIdx.x] = at;
      row_from[threadIdx.x] = from;
      row_n[threadIdx.x] = n;
      __syncthreads();
      const int mine = wave + kResizeWaves * lane;  // row of the tile
      for (uint64_t many = __ballot(row_n[mine] > kRowEntries); many; many &= many - 1) {
        const int i = wave + kResizeWaves * (int)__builtin_ctzll(many);
        move(b0 + i, row_at[i], row_from[i], lane, row_n[i], std::integral_constant<int, 64>());
      }
      __syncthreads();
    }
  }
  // offsets of the new tokens, lengths
  Sums sum = {0, 0, 0};
  for (int b0 = 0; b0 < p.B; b0 += kResizeThreads) {
    const int b = b0 + threadIdx.x;
    if (!single) {
      row = read_row(p, b);
      before = scan(row, sum);
    }
    if (b < p.B) {
      const int at = flags ? 0 : (int)before.gained;
      if (p.cu) p.cu[b] = at;
      if (single) cu_lds[b] = at;
      if (!flags) p.lens[b] = p.targets[b];
    }
  }
  const int tokens = flags ? 0 : (int)all.gained;
  if (threadIdx.x == 0) {
    if (p.cu) p.cu[p.B] = tokens;
    if (single) cu_lds[p.B] = tokens;
    if (!flags) *p.n_free = (int)left;
    p.result[0] = flags;
    p.result[1] = left < 0 ? (int)min(-left, (int64_t)0x7FFFFFFF) : 0;
    p.result[2] = (int)min(all.gained, (int64_t)0x7FFFFFFF);
    p.result[3] = flags ? (int)n_free : (int)left;
  }
  if (!few) return;
  __syncthreads();
  if (single)
    for (int i = threadIdx.x; i < p.N; i += kResizeThreads) map_token(p, cu_lds, i, tokens);
  else
    for (int i = threadIdx.x; i < p.N; i += kResizeThreads) map_token(p, p.cu, i, tokens);
}

constexpr int kSlotThreads = 256, kSlotTokens = 4, kSlotRows = 2048;

__global__ __launch_bounds__(kSlotThreads) void slots_kernel(const ResizeParams p) {
  __shared__ int32_t cu_lds[kSlotRows + 1];
  const int tokens = p.cu[p.B];
  const bool held = p.B <= kSlotRows;
  if (held) {
    for (int b = threadIdx.x; b <= p.B; b += kSlotThreads) cu_lds[b] = p.cu[b];
    __syncthreads();
  }
  const int64_t i0 = (int64_t)blockIdx.x * (kSlotThreads * kSlotTokens) + threadIdx.x;
#pragma unroll
  for (int k = 0; k < kSlotTokens; ++k) {
    const int64_t i = i0 + k * kSlotThreads;
    if (i >= p.N) continue;
    if (held) map_token(p, cu_lds, (int)i, tokens);
    else map_token(p, p.cu, (int)i, tokens);
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
