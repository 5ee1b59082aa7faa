// What the decode kernels share: how the cached tokens of a call are cut into
// runs for the workgroups, and how the parts of a (row, head) are joined.  The
// kernels, decode.hip (BF16 cache) and decode8.hip (8-bit cache), say what a run's
// chunk is and attend over it; the reasons for the cut stand in decode.hip.
#pragma once

#include <type_traits>

#include "hg_attn.h"
#include "hg_device.h"

namespace hg {
namespace {

constexpr int kWaves = 4;
constexpr int kThreadsDecode = kWaves * 64;
constexpr int kJoin = 16;  // parts of an item joined in one step
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kNegInf = -__builtin_inff();

// exp2(a - m) with m = -inf (nothing seen) giving 0.
__device__ __forceinline__ float weight(float a, float m) {
  return __builtin_amdgcn_exp2f(a - (m == kNegInf ? 0.0f : m));
}

// Attended span of batch row b, and its chunks: at least one, so that an empty
// row is answered.  Lengths go up to 2^31 - 1, so what may lie a few chunks past
// one (a chunk's end, the tokens looked up ahead) is counted in uint32_t.
struct Span {
  int first, len;
};
__device__ __forceinline__ Span row_span(const DecodeParams& p, int b) {
  Span s;
  s.len = clamp_to(p.lens[b], p.cache.max_tokens);
  s.first = p.starts ? min(clamp_to(p.starts[b], p.cache.max_tokens), s.len) : 0;
  return s;
}
// Sum of values up to 2^27 in 64 bits, 16 bits at a time.
__device__ __forceinline__ int64_t lane_sum64(int v) {
  return ((int64_t)lane_sum(v >> 16) << 16) + lane_sum(v & 0xFFFF);
}

// 64-bit quotient, in 32 bits where both fit (almost always).
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
  return (((uint64_t)x | (uint64_t)y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

// An item, or a workgroup's part of it.
struct Segment {
  int b, pair;      // batch row; (head, row tile)
  Span span;
  int c0, c1;       // chunks
  int parts, part;  // of the item
  int slot0, step;  // slot of part k: slot0 + step k, of part 0 of several in a list share: one more
};
__device__ __forceinline__ int slot_of(const Segment& s, int k) { return s.slot0 + s.step * k + (s.step == 2 && k == 0 ? 1 : 0); }

// Rows that the lanes hold, lane's 64 j + lane: all of a call of kDecodeSlots / 2 items.
constexpr int kHeld = kDecodeSlots / 2 / 64;

// Maximum over the lanes, of values from 0 on.
template <int CTRL, int ROWS>
__device__ __forceinline__ int lane_max_step(int v) {
  return max(v, __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ int lane_max(int v) {
  v = lane_max_step<0x121, 0xF>(v);  // row_ror:1, 2, 4, 8
  v = lane_max_step<0x122, 0xF>(v);
  v = lane_max_step<0x124, 0xF>(v);
  v = lane_max_step<0x128, 0xF>(v);
  v = lane_max_step<0x142, 0xA>(v);  // row_bcast:15, 31
  return __builtin_amdgcn_readlane(lane_max_step<0x143, 0xC>(v), 63);
}

// Up to kDecodeSlots items: this workgroup's segment (false: none).  With Even, only
// if the longest segment is at most a quarter longer than the even share; `even`
// says whether.
template <bool Even, bool Few, class Count>
__device__ __forceinline__ bool equal_segment(const DecodeParams& p, int per_row, const Count& count, Segment& s, int64_t& total,
                                              bool& even) {
  even = true;
  const int lane = threadIdx.x & 63;
  Span span[kHeld];
  int n[kHeld];
  total = 0;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    n[j] = 0;
    span[j] = Span{0, 0};
    if (64 * j < p.cache.B && 64 * j + lane < p.cache.B) {
      span[j] = row_span(p, 64 * j + lane);
      n[j] = count(span[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (64 * j < p.cache.B) total += lane_sum64(n[j]);
  int per = max((int)((total * per_row + kDecodeSlots - 1) / kDecodeSlots), kWaves);
  int slots = kDecodeSlots, again = 0;
  if constexpr (Few) {
    // Half the slots, one workgroup a compute unit (one row of 131072 tokens, 4 KV
    // heads: 39.4 -> 35.2 us, 524288: 99.2 -> 91.5; 8 rows of 256 to 6656, 8 KV heads:
    // 19.7 -> 17.9; 30 such rows: 52.5, by half the slots 62.5), unless segments would
    // have to be more than half as long again as the even share (a quarter: 20 rows of
    // 1000 to 4000 take 28.0 us, not 27.2; as long again: the 30 rows 63.0, not 53.5).
    slots = kDecodeSlots / 2;
    again = per;
    per = max((int)((total * per_row + slots - 1) / slots), kWaves);
    // A join costs about six chunks' time: no item is cut for less (16 rows of 700
    // tokens, 8 KV heads, in one segment each 12.5 -> 11.3 us; one row of 1361 tokens,
    // 4 KV heads, and four of 2000 to 3008, 32, stay cut: 10.0 and 21.9, and 14.5 and
    // 27.0 where 24 chunks count as less).
    int longest = 0;
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (64 * j < p.cache.B) longest = max(longest, n[j]);
    longest = lane_max(longest);
    if (longest <= per + 6) per = longest;
  }
  const int most = per + (Few ? per / 2 : per / 4);
  while (true) {
    int segs = 0;
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (64 * j < p.cache.B) segs += lane_sum((n[j] + per - 1) / per);
    if (segs * per_row <= slots) break;
    per += max(per >> 3, 1);
    if (Few && slots < kDecodeSlots && per > most) {
      slots = kDecodeSlots;
      per = again;
    }
    if (Even && per > most) {
      even = false;
      return false;
    }
  }
  int before = 0;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    if (64 * j >= p.cache.B) return false;
    const int segs = (n[j] + per - 1) / per;
    const int sum = lane_scan(segs * per_row);
    const int past = __popcll(__ballot(before + sum <= (int)blockIdx.x));
    if (past < 64) {
      s.b = 64 * j + past;
      s.parts = __builtin_amdgcn_readlane(segs, past);
      s.span.first = __builtin_amdgcn_readlane(span[j].first, past);
      s.span.len = __builtin_amdgcn_readlane(span[j].len, past);
      const int rel = (int)blockIdx.x - before - __builtin_amdgcn_readlane(sum, past) + s.parts * per_row;
      s.pair = rel / s.parts;
      s.part = rel - s.pair * s.parts;
      const int chunks = count(s.span);
      s.c0 = (int)((int64_t)chunks * s.part / s.parts);
      s.c1 = (int)((int64_t)chunks * (s.part + 1) / s.parts);
      s.slot0 = (int)blockIdx.x - s.part;
      s.step = 1;
      return true;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  return false;
}

// The runs of a workgroup: one segment of an item, or a share of the list of all
// chunks.  count(span) is the number of chunks of a row, at least 1.  Mode says
// which: both, as the call has it, or one that the launch was chosen for.  In the
// list an item counts Extra chunks more than it has, the cost of turning to it.  With Few
// an item is cut into fewer segments, see equal_segment.
enum RunMode { kEither, kSegments, kShares };
__host__ __device__ __forceinline__ bool runs_are_shares(int64_t items) { return items > kDecodeSlots / 2; }

template <RunMode Mode, int Extra, bool Few>
struct Run {
  Segment sg;
  bool shares;
  int64_t u = 0, u1 = 1, per = 0, before = 0;  // before: place in the list of the row sg.b
  int64_t row_chunks = 0;                      // of all rows, for one head

  template <class Count>
  __device__ __forceinline__ bool begin(const DecodeParams& p, int per_row, const Count& count) {
    const int lane = threadIdx.x & 63;
    const int64_t items = (int64_t)p.cache.B * per_row;
    shares = Mode == kEither ? runs_are_shares(items) : Mode == kShares;
    bool even;
    if (!shares) return equal_segment<false, Few>(p, per_row, count, sg, row_chunks, even);
    // Items of about one length, a workgroup each, need no joins (64 rows of 3456 tokens,
    // 8 KV heads, over the 8-bit cache: 79.8 -> 73.8 us; 60 rows of 900 to 1100: 40.7 ->
    // 31.2; 60 of 700 to 1300 40.5 -> 32.5, and 38.9 if a segment may be an eighth longer).
    if (Extra > 0 && items <= kDecodeSlots && p.cache.B <= 64 * kHeld) {
      const bool some = equal_segment<true, false>(p, per_row, count, sg, row_chunks, even);
      if (even) {
        shares = false;
        return some;
      }
    }
    // this workgroup's share [u, u1) of the list
    row_chunks = 0;
    for (int b0 = 0; b0 < p.cache.B; b0 += 64)
      row_chunks += lane_sum64(b0 + lane < p.cache.B ? count(row_span(p, b0 + lane)) : 0);
    const int64_t total = (row_chunks + (int64_t)Extra * p.cache.B) * per_row;
    per = (total + kDecodeSlots - 1) / kDecodeSlots;
    u = blockIdx.x * per;
    u1 = u + per < total ? u + per : total;
    if (u >= u1) return false;
    // the row that holds u: rows are dropped 64 at a time, then one at a time
    sg.b = 0;
    for (int b0 = 0; b0 + 64 < p.cache.B; b0 += 64) {
      const int64_t n = (lane_sum64(count(row_span(p, b0 + lane))) + 64 * Extra) * per_row;
      if (before + n > u) break;
      before += n;
      sg.b = b0 + 64;
    }
    const int n = sg.b + lane < p.cache.B ? count(row_span(p, sg.b + lane)) : 0;
    for (int i = 0; i < 63; ++i) {
      const int64_t c = ((int64_t)__builtin_amdgcn_readlane(n, i) + Extra) * per_row;
      if (before + c > u) break;
      before += c;
      ++sg.b;
    }
    return true;
  }

  // The next item, or part of one; its values are wave-uniform.  False: none is left.
  template <class Count>
  __device__ __forceinline__ bool next(const DecodeParams& p, int per_row, const Count& count, Segment& s) {
    if (u >= u1) return false;
    if (shares) {
      sg.span = row_span(p, sg.b);
      const int64_t listed = (int64_t)count(sg.span) + Extra;
      sg.pair = (int)quotient(u - before, listed);
      const int64_t end = before + (sg.pair + 1) * listed, start = end - listed + Extra;  // of its chunks
      const int64_t stop = end < u1 ? end : u1;
      if (Extra > 0 && stop <= start) {  // the share ends before the item's first chunk
        u = u1;
        return false;
      }
      sg.c0 = (int)(u > start ? u - start : 0);
      sg.c1 = (int)(stop - start);
      const int w0 = (int)quotient(start, per), w1 = (int)quotient(end - 1, per);
      sg.parts = w1 - w0 + 1;
      sg.part = (int)blockIdx.x - w0;
      sg.slot0 = 2 * w0;
      sg.step = 2;
      u = stop;
      if (u == before + listed * per_row) before = u;
    } else {
      u = u1;
    }
    s = sg;
    s.b = __builtin_amdgcn_readfirstlane(sg.b);
    s.pair = __builtin_amdgcn_readfirstlane(sg.pair);
    s.span.first = __builtin_amdgcn_readfirstlane(sg.span.first);
    s.span.len = __builtin_amdgcn_readfirstlane(sg.span.len);
    s.c0 = __builtin_amdgcn_readfirstlane(sg.c0);
    s.c1 = __builtin_amdgcn_readfirstlane(sg.c1);
    s.parts = __builtin_amdgcn_readfirstlane(sg.parts);
    if (shares && before == u) ++sg.b;  // the row ends here
    return true;
  }
};

__device__ __forceinline__ int64_t shfl64(int64_t v, int src) {
  const uint32_t lo = __shfl((int)(uint32_t)v, src), hi = __shfl((int)(v >> 32), src);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// Results of segments pass between workgroups, on any die, in 8-byte accesses of
// agent scope: the stores go through the caches to memory and the loads past
// them.  A wavefront's stores are there once it has waited for them, so the
// arrival counter needs no write-back or invalidation of a whole L2 (with a
// release and acquire in their place a call of 512 segments took 81 us, not 58).
__device__ __forceinline__ void put_shared(float* p, float x, float y) {
  const uint64_t v = ((uint64_t)__float_as_uint(y) << 32) | __float_as_uint(x);
  __hip_atomic_store((uint64_t*)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 get_shared(const float* p) {
  const uint64_t v = __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return f32x2{__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}
__device__ __forceinline__ f32x4 get_shared4(const float* p) {
  const f32x2 a = get_shared(p), b = get_shared(p + 2);
  return f32x4{a[0], a[1], b[0], b[1]};
}

// Channels c4.. of query head hq from sum o of weight l (relative to m).
__device__ __forceinline__ void store_output(const DecodeParams& p, int b, int hq, int c4, f32x4 o, float m, float l) {
  const float inv = l > 0 ? 1.0f / l : (l == 0 ? 0.0f : l);
  *(q32x2*)(p.out.data + b * p.out.token_stride + hq * p.out.head_stride + c4) =
      q32x2{cvt_bf16x2(o[0] * inv, o[1] * inv), cvt_bf16x2(o[2] * inv, o[3] * inv)};
  if (p.lse && c4 == 0)
    p.lse[(int64_t)b * p.cache.H * p.R + hq] = l == 0 ? kNegInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int D>
__device__ __forceinline__ void put_part(float* part, int rows, int row, int c4, f32x4 o, float m, float l) {
  if (c4 == 0) put_shared(part + 2 * row, m, l);
  put_shared(part + 2 * rows + row * D + c4, o[0], o[1]);
  put_shared(part + 2 * rows + row * D + c4 + 2, o[2], o[3]);
}

// Counts this workgroup's arrival, its stores done; true for the last of `count`,
// which leaves the counter at zero.
__device__ __forceinline__ bool arrive(uint32_t* counter, int count, float* lds) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  uint32_t* last = (uint32_t*)lds;
  if (threadIdx.x == 0) {
    const uint32_t n = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *last = n == (uint32_t)(count - 1);
    if (*last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return *last != 0;
}

// Joins parts k0, k0 + every, .. (count of them) of an item and hands out the
// result, four channels a call.  A thread reads its channels and their row's
// statistics of up to 16 parts at a time (a part past the last is read as the
// last and left out), so up to 16 parts cost one trip to memory.  With few
// columns, several threads share one, each with a run of the parts.
template <int D, class Emit>
__device__ __forceinline__ void join_parts(const DecodeParams& p, const Segment& sg, int k0, int every, int count, int stride,
                                           int rows, float* lds, const Emit& emit) {
  const int columns = rows * (D / 4);
  const int share = max(kThreadsDecode / columns, 1);
  for (int i0 = 0; i0 < columns; i0 += kThreadsDecode) {
    const int s = share > 1 ? (int)threadIdx.x / columns : 0;
    const int i = share > 1 ? (int)threadIdx.x - s * columns : i0 + (int)threadIdx.x;
    const bool active = s < share && i < columns;
    const int row = active ? i / (D / 4) : 0, c4 = active ? (i % (D / 4)) * 4 : 0;
    const int w0 = share > 1 ? min(count * s / share, count) : 0, w1 = share > 1 ? min(count * (s + 1) / share, count) : count;
    f32x4 o = {0, 0, 0, 0};
    float m = kNegInf, l = 0;
    auto take = [&](auto size, int w) __attribute__((always_inline)) {
      constexpr int N = decltype(size)::value;
      f32x2 st[N];
      f32x4 x[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float* src = p.partial + (int64_t)slot_of(sg, k0 + every * min(w + k, w1 - 1)) * stride;
        st[k] = get_shared(src + 2 * row);
        x[k] = get_shared4(src + 2 * rows + row * D + c4);
      }
      float top = m;
#pragma unroll
      for (int k = 0; k < N; ++k) top = fmaxf(top, st[k][0]);
      const float down = weight(m, top);
      m = top;
      o *= down;
      l *= down;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float f = weight(st[k][0], m);
        const bool in = w + k < w1;
        l += in ? st[k][1] * f : 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += in ? x[k][e] * f : 0.0f;
      }
    };
    int w = w0;
    for (; w + 8 < w1; w += 16) take(std::integral_constant<int, 16>{}, w);
    for (; w + 3 < w1; w += 8) take(std::integral_constant<int, 8>{}, w);
    for (; w < w1; w += 3) take(std::integral_constant<int, 3>{}, w);
    if (share > 1) {  // the sharers' results in order
      float* sums = lds + 1;  // [kThreadsDecode][6], after the arrival word
      if (active) {
        float* t = sums + threadIdx.x * 6;
        t[0] = m;
        t[1] = l;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[2 + e] = o[e];
      }
      __syncthreads();
      if (active && s == 0) {
        float top = m;
        for (int k = 1; k < share; ++k) top = fmaxf(top, sums[(k * columns + i) * 6]);
        const float f0 = weight(m, top);
        o *= f0;
        l *= f0;
        m = top;
        for (int k = 1; k < share; ++k) {
          const float* t = sums + (k * columns + i) * 6;
          const float f = weight(t[0], m);
          l += t[1] * f;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] += t[2 + e] * f;
        }
      }
    }
    __syncthreads();  // every part is read before a result takes the place of one
    if (active && s == 0) emit(row, c4, o, m, l);
  }
}

// Joins the wavefronts of a workgroup, whose results are in LDS ([kWaves][rows]
// [D + 4] sums, then [kWaves][2][rows] maxima and weights), and the parts of an
// item in several.
template <int D>
__device__ __forceinline__ void finish_item(const DecodeParams& p, const Segment& sg, int h, int tile0, int rows, float* lds) {
  constexpr int pitch = D + 4;
  const float* part = lds;
  const float* stat = lds + kWaves * rows * pitch;
  const int b = sg.b, parts = sg.parts;
  __syncthreads();
  const int stride = decode_partial_floats(min(p.R, kDecodeRows), D);
  float* mine = p.partial + (int64_t)slot_of(sg, sg.part) * stride;
  for (int i = threadIdx.x; i < rows * (D / 4); i += kThreadsDecode) {
    const int row = i / (D / 4), c4 = (i % (D / 4)) * 4;
    f32x4 o = {0, 0, 0, 0};
    float m = kNegInf, l = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, stat[(w * 2) * rows + row]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = weight(stat[(w * 2) * rows + row], m);
      o += *(const f32x4*)(part + (w * rows + row) * pitch + c4) * f;
      l += stat[(w * 2 + 1) * rows + row] * f;
    }
    if (parts == 1)
      store_output(p, b, h * p.R + tile0 + row, c4, o, m, l);
    else
      put_part<D>(mine, rows, row, c4, o, m, l);
  }
  if (parts == 1) {
    __syncthreads();  // LDS is free for the next item
    return;
  }

  // The last workgroup to finish a part joins them.  Arrivals are counted at the
  // item's own slots: a group's at its first part's, the item's at part 1's,
  // with which no group starts (groups have five parts or more).
  const int group = parts <= kJoin ? 1 : (int)ceilf(sqrtf((float)parts));
  bool joins = true;
  if (group > 1) {
    const int k0 = sg.part - sg.part % group, count = min(group, parts - k0);
    float* first_part = p.partial + (int64_t)slot_of(sg, k0) * stride;
    joins = arrive(p.counters + slot_of(sg, k0), count, lds);
    if (joins)
      join_parts<D>(p, sg, k0, 1, count, stride, rows, lds, [&](int row, int c4, f32x4 o, float m, float l) {
        put_part<D>(first_part, rows, row, c4, o, m, l);
      });
  }
  if (joins && arrive(p.counters + slot_of(sg, 1), (parts + group - 1) / group, lds))
    join_parts<D>(p, sg, 0, group, (parts + group - 1) / group, stride, rows, lds,
                  [&](int row, int c4, f32x4 o, float m, float l) { store_output(p, b, h * p.R + tile0 + row, c4, o, m, l); });
  __syncthreads();
}

// LDS of a decode workgroup: the wavefronts' parts, or the results of threads
// that share a column.
inline size_t decode_lds_bytes(int R, int D) {
  const int rows = R < kDecodeRows ? R : kDecodeRows;
  const int parts = kWaves * rows * (D + 4 + 2), sums = 1 + 6 * kThreadsDecode;
  return sizeof(float) * (parts > sums ? parts : sums);
}

}  // namespace
}  // namespace hg
