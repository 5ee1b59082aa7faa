// Attention of one new token per batch row over the paged cache.
//
// For query head q of key/value head h, over the row's tokens t:
//   s_t = scale q.K_t,  m = max s_t,  p_t = exp(s_t - m),
//   out = sum p_t V_t / sum p_t,  lse = m + log sum p_t,
// in one pass with the running m and sum; parts (m, l, O) of a row join as
//   m = max m_i, l = sum l_i e^(m_i - m), O = sum O_i e^(m_i - m).
// Every K and V row is read once, 4 R operations an element for R query heads
// a KV head, so memory bounds it and the layout serves the loads:
//   * A wavefront takes 32 tokens at a time, K and V rows straight to
//     registers in 16-byte pieces; the products run on the matrix units as
//     S^T = K Q^T and O^T = V^T P^T (16x16x32 steps), the query heads of a KV head
//     as the (padded) 16 columns.  In both the query head of a lane is
//     lane % 16, so the softmax state and the rescaling of O stay in the lane.
//   * The result layout of S^T gives lane group g = lane / 16 the tokens
//     4g..4g+3 of each 16; the second product takes its 32 tokens in just that
//     order (tokens 4g + i and 16 + 4g + i for group g), so P goes from result
//     to operand without moving.  V rows arrive as 8 channels a lane, and the
//     lane's 8 tokens x 8 channels are transposed by byte permutes in place;
//     the channel order that this gives the product's rows is undone in the store.
//   * Keys of the next 32 tokens are loaded before the values are used, values
//     before the next softmax.
// Work is split by what the lengths on the GPU say, into at most kDecodeSlots
// runs, two workgroups a compute unit (how a call is cut does not change with
// the timing, so neither do results):
//   * up to kDecodeSlots / 2 (row, head)s, "items": each is cut into ceil(chunks /
//     per) equal segments, per stepping up from the even share until there is a
//     slot for every segment (twice the share is enough), and a workgroup takes
//     one;
//   * more items: a workgroup takes an even share of the list of all chunks, that
//     is whole items and at most one part of an item at either end.
// The wavefronts take the chunks of an item in turn and join through LDS.  An item
// in several parts is joined through the workspace by the last workgroup to
// finish one, in the order of the parts; past kJoin parts in two steps (groups of
// about the square root of the parts), since one compute unit reads a few tens of
// bytes a clock (64 rows x 128 parts joined in one step: 19 us, in two: 6).
//
// Measured: 64 rows of up to 6656 tokens, 64 query and 8 KV heads of 128 channels,
// 924 MB: 161 us, 5.7 TB/s; one row of 1361 tokens: 10.0 us.
#include <type_traits>

#include "hg_attn.h"
#include "hg_device.h"

namespace hg {
namespace {

constexpr int kWaves = 4;
constexpr int kThreadsDecode = kWaves * 64;
// Tokens of a wavefront's step: 8 KiB of keys and as much of values up to
// head_dim 128; 32 tokens at 256 would not fit the registers.
template <int D>
constexpr int kChunk = D == 256 ? 16 : 32;
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
template <int D>
__device__ __forceinline__ int span_chunks(const Span& s) {
  return max((int)(((uint32_t)(s.len - s.first) + kChunk<D> - 1) / kChunk<D>), 1);
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

// Rows of up to kDecodeSlots / 2 items: lane's rows 64 j + lane.
constexpr int kHeld = kDecodeSlots / 2 / 64;

// Up to kDecodeSlots / 2 items: this workgroup's segment (false: none).
template <int D>
__device__ __forceinline__ bool equal_segment(const DecodeParams& p, int per_row, Segment& s, int64_t& total) {
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
      n[j] = span_chunks<D>(span[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (64 * j < p.cache.B) total += lane_sum64(n[j]);
  int per = max((int)((total * per_row + kDecodeSlots - 1) / kDecodeSlots), kWaves);
  while (true) {
    int segs = 0;
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (64 * j < p.cache.B) segs += lane_sum((n[j] + per - 1) / per);
    if (segs * per_row <= kDecodeSlots) break;
    per += max(per >> 3, 1);
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
      const int chunks = span_chunks<D>(s.span);
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

// The state of one wavefront over its chunks of one (row, head, row tile).
template <int D>
struct Part {
  static constexpr int S = D / 32;   // 32-channel steps of the first product
  static constexpr int J = D / 16;   // 16-channel results of the second
  f32x4 acc[J];
  float m, l;
};

// Page of token t0 + lane % kChunk (-1: not before len), asked for one chunk ahead.
template <int D>
__device__ __forceinline__ int chunk_page(const DecodeParams& p, const int32_t* table, uint32_t t0, int len) {
  const uint32_t t = t0 + (threadIdx.x & (kChunk<D> - 1));
  return t < (uint32_t)len ? table[divide(t, p.cache)] : -1;
}
// Its row's offset, and which of the chunk's tokens are attended (row 0 of page
// 0 stands in for the others, so every load is inside the cache).
template <int D>
__device__ __forceinline__ int64_t chunk_rows(const DecodeParams& p, int page, uint32_t t0, uint32_t& seen) {
  const uint32_t t = t0 + (threadIdx.x & (kChunk<D> - 1));
  const bool in = page >= 0 && page < p.cache.num_pages;
  seen = (uint32_t)__ballot(in);
  const uint32_t at = t - divide(t, p.cache) * (uint32_t)p.cache.page_size;
  return in ? page * p.cache.page_stride + at * p.cache.token_stride : 0;
}

__device__ __forceinline__ int64_t shfl64(int64_t v, int src) {
  const uint32_t lo = __shfl((int)(uint32_t)v, src), hi = __shfl((int)(v >> 32), src);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

template <int D>
struct Loads {
  static constexpr int S = D / 32;
  static constexpr int VP = D >= 128 ? D / 128 : 1;  // pieces of a V row per lane
  static constexpr int VW = D >= 128 ? 4 : 2;        // dwords of a piece
  static constexpr int TT = kChunk<D> / 16;          // 16-token tiles
  q32x4 k[TT][S];
  uint32_t v[4 * TT][VP][VW];  // tokens 4g + i, then 16 + 4g + i
};

// Once: streaming (non-temporal) loads, see stream_chunks.
template <bool Once, class T>
__device__ __forceinline__ T load_row(const uint16_t* p) {
  if constexpr (Once) return __builtin_nontemporal_load((const T*)p);
  else return *(const T*)p;
}

template <int D, bool Once>
__device__ __forceinline__ void load_keys(Loads<D>& x, const uint16_t* K, int64_t off) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int tile = 0; tile < Loads<D>::TT; ++tile) {
    const uint16_t* row = K + shfl64(off, tile * 16 + (lane & 15)) + (lane >> 4) * 8;
#pragma unroll
    for (int s = 0; s < Loads<D>::S; ++s) x.k[tile][s] = load_row<Once, q32x4>(row + s * 32);
  }
}

template <int D, bool Once>
__device__ __forceinline__ void load_values(Loads<D>& x, const uint16_t* V, int64_t off) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
#pragma unroll
  for (int i = 0; i < 4 * Loads<D>::TT; ++i) {
    const uint16_t* row = V + shfl64(off, (i & 4) * 4 + g * 4 + (i & 3));
#pragma unroll
    for (int c = 0; c < Loads<D>::VP; ++c) {
      if constexpr (D >= 128) {
        const q32x4 y = load_row<Once, q32x4>(row + c * 128 + r * 8);
#pragma unroll
        for (int w = 0; w < 4; ++w) x.v[i][c][w] = y[w];
      } else {
        const q32x2 y = load_row<Once, q32x2>(row + r * 4);
        x.v[i][c][0] = y[0];
        x.v[i][c][1] = y[1];
      }
    }
  }
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

template <int D>
__global__ __launch_bounds__(kThreadsDecode, 2) void decode_kernel(const DecodeParams p) {
  constexpr int S = D / 32, J = D / 16;
  constexpr int VP = Loads<D>::VP, VW = Loads<D>::VW, TT = Loads<D>::TT;
  extern __shared__ float lds[];  // [kWaves][rows][D + 4] parts, then their m and l
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int per_row = p.cache.H * p.row_tiles;  // (head, row tile) pairs of a batch row

  // more items than slots: this workgroup's share [u, u1) of all chunks
  Segment sg;
  int64_t u = 0, u1 = 1, per = 0, before = 0;  // before: chunks of the rows before sg.b
  int64_t row_chunks = 0;                      // of all rows, for one head
  const bool shares = (int64_t)p.cache.B * per_row > kDecodeSlots / 2;
  if (shares) {
    for (int b0 = 0; b0 < p.cache.B; b0 += 64)
      row_chunks += lane_sum64(b0 + lane < p.cache.B ? span_chunks<D>(row_span(p, b0 + lane)) : 0);
    const int64_t total = row_chunks * per_row;
    per = (total + kDecodeSlots - 1) / kDecodeSlots;
    u = blockIdx.x * per;
    u1 = u + per < total ? u + per : total;
    if (u >= u1) return;
    // the row that holds u: rows are dropped 64 at a time, then one at a time
    sg.b = 0;
    for (int b0 = 0; b0 + 64 < p.cache.B; b0 += 64) {
      const int64_t n = lane_sum64(span_chunks<D>(row_span(p, b0 + lane))) * per_row;
      if (before + n > u) break;
      before += n;
      sg.b = b0 + 64;
    }
    const int n = sg.b + lane < p.cache.B ? span_chunks<D>(row_span(p, sg.b + lane)) : 0;
    for (int i = 0; i < 63; ++i) {
      const int64_t c = (int64_t)__builtin_amdgcn_readlane(n, i) * per_row;
      if (before + c > u) break;
      before += c;
      ++sg.b;
    }
  } else if (!equal_segment<D>(p, per_row, sg, row_chunks)) {
    return;
  }
  const bool streamed = row_chunks > p.stream_chunks;

  while (u < u1) {  // one item, or part of one, a turn
    if (shares) {
      sg.span = row_span(p, sg.b);
      const int64_t chunks = span_chunks<D>(sg.span);
      sg.pair = (int)quotient(u - before, chunks);
      const int64_t start = before + sg.pair * chunks, end = start + chunks;
      const int64_t stop = end < u1 ? end : u1;
      sg.c0 = (int)(u - start);
      sg.c1 = (int)(stop - start);
      const int w0 = (int)quotient(start, per), w1 = (int)quotient(end - 1, per);
      sg.parts = w1 - w0 + 1;
      sg.part = (int)blockIdx.x - w0;
      sg.slot0 = 2 * w0;
      sg.step = 2;
      u = stop;
      if (u == before + chunks * per_row) {
        before = u;
      }
    } else {
      u = u1;
    }
    const int b = __builtin_amdgcn_readfirstlane(sg.b), pair = __builtin_amdgcn_readfirstlane(sg.pair);
    const int first = __builtin_amdgcn_readfirstlane(sg.span.first), len = __builtin_amdgcn_readfirstlane(sg.span.len);
    const int c0 = __builtin_amdgcn_readfirstlane(sg.c0), c1 = __builtin_amdgcn_readfirstlane(sg.c1);
    const int parts = __builtin_amdgcn_readfirstlane(sg.parts);
    if (shares && before == u) ++sg.b;  // the row ends here
    const int h = pair / p.row_tiles, tile0 = (pair - h * p.row_tiles) * kDecodeRows;
    const int rows = min(p.R - tile0, kDecodeRows);

    // queries: lane's head is r, channels 32 s + 8 g ..
    q32x4 q[S];
    {
      const int hq = h * p.R + tile0 + min(r, rows - 1);
      const uint16_t* src = p.q.data + b * p.q.token_stride + hq * p.q.head_stride + g * 8;
#pragma unroll
      for (int s = 0; s < S; ++s) q[s] = *(const q32x4*)(src + s * 32);
    }
    const uint16_t* K = p.cache.K + h * p.cache.head_stride;
    const uint16_t* V = p.cache.V + h * p.cache.head_stride;

    Part<D> a;
#pragma unroll
    for (int j = 0; j < J; ++j) a.acc[j] = f32x4{0, 0, 0, 0};
    a.m = kNegInf;
    a.l = 0;

    // One chunk; the next one's keys are asked for once the scores are taken, its
    // values once these are used.
    Loads<D> x;
    auto step = [&](auto once, uint32_t seen, bool more, int64_t off_next) __attribute__((always_inline)) {
      constexpr bool Once = decltype(once)::value;
      f32x4 st[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        st[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < S; ++s)
          st[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x.k[t][s]),
                                                          __builtin_bit_cast(bf16x8, q[s]), st[t], 0, 0, 0);
      }
      if (more) load_keys<D, Once>(x, K, off_next);
      float sc[4 * TT];
      float top = kNegInf;
#pragma unroll
      for (int i = 0; i < 4 * TT; ++i) {
        const bool ok = (seen >> ((i & 4) * 4 + g * 4 + (i & 3))) & 1u;
        sc[i] = ok ? st[i >> 2][i & 3] * p.scale_log2 : kNegInf;
        top = fmaxf(top, sc[i]);
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m = fmaxf(a.m, top);
      const float down = weight(a.m, m);
      a.m = m;
      a.l *= down;
#pragma unroll
      for (int j = 0; j < J; ++j) a.acc[j] *= down;
      // The weights are rounded to BF16 for their product with the values, the type
      // that the matrix units take beside them; their sum is of the unrounded ones
      // (measured against 64 bits: 0.0017 to 0.0018, any BF16 output 0.0016 to 0.0017).
      uint32_t w[2 * TT];
#pragma unroll
      for (int i = 0; i < 4 * TT; i += 2) {
        const float p0 = weight(sc[i], m), p1 = weight(sc[i + 1], m);
        a.l += p0 + p1;
        w[i >> 1] = cvt_bf16x2(p0, p1);
      }
      // values that are not attended count as 0, whatever they hold
#pragma unroll
      for (int i = 0; i < 4 * TT; ++i) {
        const uint32_t keep = (uint32_t)((int32_t)(seen << (31 - ((i & 4) * 4 + g * 4 + (i & 3)))) >> 31);
#pragma unroll
        for (int cc = 0; cc < VP; ++cc)
#pragma unroll
          for (int e = 0; e < VW; ++e) x.v[i][cc][e] &= keep;
      }
#pragma unroll
      for (int cc = 0; cc < VP; ++cc)
#pragma unroll
        for (int e = 0; e < 2 * VW; ++e) {
          uint32_t y[2 * TT];  // channel e of the lane's piece, its tokens
#pragma unroll
          for (int i = 0; i < 2 * TT; ++i)
            y[i] = __builtin_amdgcn_perm(x.v[2 * i + 1][cc][e >> 1], x.v[2 * i][cc][e >> 1],
                                         (e & 1) ? 0x07060302u : 0x05040100u);
          const int j = cc * 2 * VW + e;
          if constexpr (TT == 2)
            a.acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, q32x4{y[0], y[1], y[2], y[3]}),
                __builtin_bit_cast(bf16x8, q32x4{w[0], w[1], w[2], w[3]}), a.acc[j], 0, 0, 0);
          else
            a.acc[j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, q32x2{y[0], y[1]}),
                                                                 __builtin_bit_cast(s16x4, q32x2{w[0], w[1]}), a.acc[j], 0, 0, 0);
        }
      if (more) load_values<D, Once>(x, V, off_next);
    };
    auto attend = [&](auto once) __attribute__((always_inline)) {
      constexpr bool Once = decltype(once)::value;
      int c = c0 + wave;
      const int32_t* table = p.cache.table + (int64_t)b * p.cache.max_pages;
      const uint32_t t0 = (uint32_t)first + (uint32_t)c * kChunk<D>;
      constexpr int kStep = kWaves * kChunk<D>;
      // pages are asked for two chunks ahead
      const int page = chunk_page<D>(p, table, t0, len);
      int page_next = chunk_page<D>(p, table, t0 + kStep, len);
      uint32_t seen;
      const int64_t off = chunk_rows<D>(p, page, t0, seen);
      load_keys<D, Once>(x, K, off);
      load_values<D, Once>(x, V, off);
      for (uint32_t t = t0 + kStep; c + kWaves < c1; c += kWaves, t += kStep) {
        uint32_t seen_next;
        const int64_t off_next = chunk_rows<D>(p, page_next, t, seen_next);
        page_next = chunk_page<D>(p, table, t + kStep, len);
        step(once, seen, true, off_next);
        seen = seen_next;
      }
      step(once, seen, false, 0);
    };
    if (c0 + wave < c1 && first < len) {
      if (streamed) attend(std::true_type());
      else attend(std::false_type());
    }
    a.l += __shfl_xor(a.l, 16);
    a.l += __shfl_xor(a.l, 32);

    // join the wavefronts
    constexpr int pitch = D + 4;
    float* part = lds;                          // [kWaves][rows][pitch]
    float* stat = lds + kWaves * rows * pitch;  // [kWaves][2][rows]
    if (g == 0 && r < rows) {
      stat[(wave * 2) * rows + r] = a.m;
      stat[(wave * 2 + 1) * rows + r] = a.l;
    }
    if (r < rows) {
      float* row = part + (wave * rows + r) * pitch;
#pragma unroll
      for (int cc = 0; cc < VP; ++cc)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 2 * VW; ++e) row[cc * 128 + (g * 4 + i) * 2 * VW + e] = a.acc[cc * 2 * VW + e][i];
    }
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
      continue;
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
}

template <int D>
hipError_t launch(const DecodeParams& p, hipStream_t stream) {
  const int rows = p.R < kDecodeRows ? p.R : kDecodeRows;
  // the wavefronts' parts, or the results of threads that share a column
  const int parts = kWaves * rows * (D + 4 + 2), sums = 1 + 6 * kThreadsDecode;
  const size_t bytes = sizeof(float) * (parts > sums ? parts : sums);
  if (bytes > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)decode_kernel<D>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)bytes);
    if (e != hipSuccess) return e;
  }
  decode_kernel<D><<<dim3(kDecodeSlots), dim3(kThreadsDecode), bytes, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

// Chunks of all rows past which a call's keys and values are streamed.  In a decode
// loop a layer's are read again once the other layers' have been: they are still in
// the 256 MiB last-level cache only if all layers' are.  A pool of pages within it
// is read through the caches (32 rows of up to 320 tokens, head_dim 256, 43 MB: 15.3
// us, streamed 16.5 with three such layers).  With a larger pool it depends on what
// the rows attend, which the kernel knows.  Measured with 28 layers in turn, read
// through the caches -> streamed (us): one row, 4 KV heads, 3 MiB 10.6 -> 11.0, 8 MiB
// 12.6 -> 13.1, 12 MiB 13.5 -> 13.3; four rows, 8 KV heads, 8 MiB 9.7 -> 10.1, 12 MiB
// 10.8 -> 10.6; with layers of 900 MiB together, 24 MiB 20.2 -> 20.0, 43 MiB at
// head_dim 256 17.1 -> 16.3, 128 MiB 38.3 -> 36.7, 256 MiB 61.2 -> 57.7.  (A layer of
// 128 MiB read again and again and nothing else: 33.0 -> 34.8.)  Row tiles of one head
// read the same rows, so with several the caches serve them.
int64_t decode_stream_chunks(const PagedCache& c, int D, int row_tiles) {
  const double pool = 4.0 * c.num_pages * c.page_size * c.H * D;
  if (pool <= (double)(256 << 20) || row_tiles > 1) return INT64_MAX;
  const int chunk = D == 64 ? kChunk<64> : D == 128 ? kChunk<128> : kChunk<256>;
  return ((int64_t)10 << 20) / ((int64_t)4 * c.H * D * chunk);
}

hipError_t launch_decode(const DecodeParams& p, int D, hipStream_t stream) {
  switch (D) {
    case 64: return launch<64>(p, stream);
    case 128: return launch<128>(p, stream);
    default: return launch<256>(p, stream);
  }
}

}  // namespace hg

extern "C" int64_t hg_test_decode_stream_chunks(int num_pages, int page_size, int H, int D, int row_tiles) {
  hg::PagedCache c = {};
  c.num_pages = num_pages;
  c.page_size = page_size;
  c.H = H;
  return hg::decode_stream_chunks(c, D, row_tiles);
}
