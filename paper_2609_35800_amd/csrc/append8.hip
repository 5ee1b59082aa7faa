// Appending new tokens to the 8-bit cache, keys and queries rotated.
//
// Per (row, head, block of tokens): k' = bf16(R(p) k); m = max |k'| over the new
// tokens; e the smallest with m <= 448 2^e, or the block's present one if larger;
// codes e4m3(k' / 2^e); lo, hi = min, max of k' per channel, joined with the
// block's present ones.  A power of two as scale makes k' / 2^e exact, so each key
// is rounded once, and what a block already holds changes only when the scale
// steps up, by an exact shift of the codes' exponents (codes that fall below the
// smallest normal one are rounded again).  e4m3 keeps its relative precision over
// 2^15 of range, so channels ten times the others cost the others nothing, and
// half an exponent step that a power of two wastes costs neither.
//
// The call moves N (Hq + 2H) D 2 bytes in, N (Hq 2 + 2H) D out: memory bounds it, a
// call of few tokens the chain row -> length -> page -> scale -> store.
//   * One token a row: a wavefront takes a head's key and value, or several queries.
//   * Several: a workgroup takes the tokens of a block for some of the heads.  A
//     thread keeps two units (16 channels of a token each) in registers between the
//     reduction and the store, so every input is read once, and keeps their angles
//     from head to head.  Maxima, and minima and maxima per channel, are taken on
//     BF16 bit patterns as 16-bit integers, two an instruction.
#include "hg_attn.h"
#include "hg_device.h"
#include "hg_e4m3.h"
#include "hg_rotate.h"

namespace hg {
namespace {

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t max_u16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
__device__ __forceinline__ uint32_t max_i16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2, a), __builtin_bit_cast(i16x2, b)));
}
__device__ __forceinline__ uint32_t min_i16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(i16x2, a), __builtin_bit_cast(i16x2, b)));
}
// BF16 bit patterns to integers of the same order, and back.
__device__ __forceinline__ uint32_t ordered(uint32_t x) {
  i16x2 v = __builtin_bit_cast(i16x2, x);
  v ^= (v >> 15) & (short)0x7FFF;
  return __builtin_bit_cast(uint32_t, v);
}
constexpr uint32_t kInf2 = 0x7F807F80u, kBelow2 = 0xFF80FF80u;  // infinities
constexpr uint32_t kMinusInf2 = 0x807F807Fu;                    // ordered(kBelow2); ordered(kInf2) is kInf2
// Each half of x that is NaN (or, with Finite, infinite) replaced by that of y.
template <bool Finite>
__device__ __forceinline__ uint32_t numbers(uint32_t x, uint32_t y) {
  const uint32_t top = Finite ? 0x7F80u : 0x7F81u;
  const uint32_t lo = (x & 0x7FFFu) >= top ? y & 0xFFFFu : x & 0xFFFFu;
  const uint32_t hi = ((x >> 16) & 0x7FFFu) >= top ? y & 0xFFFF0000u : x & 0xFFFF0000u;
  return lo | hi;
}

// Page of token `at` of row b, and its place there; false if it has none.
__device__ __forceinline__ bool find_page(const Append8Params& p, int b, int64_t at, int& page, uint32_t& place) {
  const PagedCache& c = p.a.cache;
  if (at < 0 || at >= c.max_tokens) return false;
  const uint32_t pg = divide((uint32_t)at, c);
  page = c.table[(int64_t)b * c.max_pages + pg];
  place = (uint32_t)at - pg * (uint32_t)c.page_size;
  return page >= 0 && page < c.num_pages;
}

// ------------------------------------------------------------ one token a row

constexpr int kTokenThreads = 256;

// Queries that a wavefront takes, and wavefronts of a token.
template <int D>
constexpr int kWaveQueries = 64 / (D / 16);
template <int D>
__host__ __device__ __forceinline__ int token_waves(const Append8Params& p) {
  return p.a.cache.H + (p.a.Hq + kWaveQueries<D> - 1) / kWaveQueries<D>;
}

template <int D>
__global__ __launch_bounds__(kTokenThreads) void append8_token_kernel(const Append8Params p) {
  constexpr int C = D / 16;  // units of a row
  const AppendParams& a = p.a;
  const int lane = threadIdx.x & 63;
  const int waves = token_waves<D>(p);
  const int64_t wave = (int64_t)blockIdx.x * (kTokenThreads / 64) + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int token = (int)(wave / waves), part = (int)(wave - (int64_t)token * waves);
  if (token >= a.N) return;
  const int64_t at = (int64_t)a.lens[token] - 1;

  if (part >= a.cache.H) {  // queries
    const int h = (part - a.cache.H) * kWaveQueries<D> + lane / C;
    const Unit un = unit_of(a, lane % C);
    Angles an;
    if (h >= a.Hq || !load_angles(a, un, token, at, an)) return;
    const uint16_t* src = a.q.data + token * a.q.token_stride + h * a.q.head_stride;
    u32x4 x = *(const u32x4*)(src + un.c0), y = *(const u32x4*)(src + un.c1);
    if (un.rotated) rotate(x, y, an, a.interleaved);
    uint16_t* o = a.q_out.data + token * a.q_out.token_stride + h * a.q_out.head_stride;
    *(u32x4*)(o + un.c0) = x;
    *(u32x4*)(o + un.c1) = y;
    return;
  }

  // lanes 0 .. C - 1 the key, 32 .. 32 + C - 1 the value
  const int h = part;
  const bool is_k = lane < 32, in = (lane & 31) < C;
  const Unit un = unit_of(a, in ? lane & 31 : 0);
  const hg_rows& rows = is_k ? a.k : a.v;
  const uint16_t* src = rows.data + token * rows.token_stride + h * rows.head_stride;
  u32x4 x = *(const u32x4*)(src + un.c0), y = *(const u32x4*)(src + un.c1);
  int page = 0;
  uint32_t place = 0;
  const bool stored = find_page(p, token, at, page, place);
  const int64_t block = ((int64_t)page * a.cache.H + h) * p.c.page_blocks + (place >> p.c.block_shift);
  const uint32_t held = place & ((1u << p.c.block_shift) - 1);
  float* scales = is_k ? p.c.k_scale : p.c.v_scale;
  const float present = stored && held ? scales[block] : 0.0f;
  uint16_t* bounds = p.c.bounds + block * 2 * D;
  const bool bounded = stored && p.c.bounds && is_k && in;
  u32x4 lo[2], hi[2];
  if (bounded && held) {
    lo[0] = *(const u32x4*)(bounds + un.c0);
    lo[1] = *(const u32x4*)(bounds + un.c1);
    hi[0] = *(const u32x4*)(bounds + D + un.c0);
    hi[1] = *(const u32x4*)(bounds + D + un.c1);
  }
  Angles an;
  if (!load_angles(a, un, token, at, an)) return;  // the wavefront's token
  if (is_k && un.rotated) rotate(x, y, an, a.interleaved);
  if (is_k && in && a.k_out.data) {
    uint16_t* o = a.k_out.data + token * a.k_out.token_stride + h * a.k_out.head_stride;
    *(u32x4*)(o + un.c0) = x;
    *(u32x4*)(o + un.c1) = y;
  }
  if (!stored) return;

  uint32_t most = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    most = max_u16(most, numbers<true>(x[w], 0) & 0x7FFF7FFFu);
    most = max_u16(most, numbers<true>(y[w], 0) & 0x7FFF7FFFu);
  }
  if (!in) most = 0;
  most = max(most & 0xFFFFu, most >> 16);
#pragma unroll
  for (int s = 1; s < C; s *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, s));
  const int needed = scale_exponent(most << 16);
  const int old = held ? stored_exponent(present, needed) : needed;
  const int e = max(old, needed);

  // what the block holds, on the new scale (the lanes that read the scale go first)
  uint8_t* codes = (is_k ? p.c.K : p.c.V) + page * a.cache.page_stride + h * a.cache.head_stride + place * a.cache.token_stride;
  const uint64_t grown = __ballot(in && e > old);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if (!(grown >> (32 * t) & 1)) continue;
    const float ratio = exponent_ratio(__builtin_amdgcn_readlane(old - e, 32 * t));
    uint8_t* first = (t ? p.c.V : p.c.K) + page * a.cache.page_stride + h * a.cache.head_stride + (place - held) * a.cache.token_stride;
    for (uint32_t i = lane; i < held * C; i += 64) {
      u32x4* piece = (u32x4*)(first + i / C * a.cache.token_stride + i % C * 16);
      u32x4 z = *piece;
#pragma unroll
      for (int w = 0; w < 4; ++w) z[w] = rescale_codes(z[w], ratio);
      *piece = z;
    }
  }
  if (!in) return;
  const float inv = exponent_inverse(e);
  *(u32x2*)(codes + un.c0) = to_codes8(x, inv);
  *(u32x2*)(codes + un.c1) = to_codes8(y, inv);
  if ((lane & 31) == 0) scales[block] = exponent_scale(e);
  if (bounded) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t z = i ? y[w] : x[w];
        const uint32_t low = ordered(numbers<false>(z, kInf2)), high = ordered(numbers<false>(z, kBelow2));
        lo[i][w] = ordered(held ? min_i16(low, ordered(numbers<false>(lo[i][w], kInf2))) : low);
        hi[i][w] = ordered(held ? max_i16(high, ordered(numbers<false>(hi[i][w], kBelow2))) : high);
      }
    *(u32x4*)(bounds + un.c0) = lo[0];
    *(u32x4*)(bounds + un.c1) = lo[1];
    *(u32x4*)(bounds + D + un.c0) = hi[0];
    *(u32x4*)(bounds + D + un.c1) = hi[1];
  }
}

// ------------------------------------------------------------ several tokens a row

// Threads for the units of a block, two each.
inline int block_threads(const Append8Params& p, int D) {
  const int n = (1 << p.c.block_shift) * (D / 16) / 2;
  return n < 64 ? 64 : n;
}

template <int D, bool Once>
__global__ __launch_bounds__(1024) void append8_block_kernel(const Append8Params p, int slice_rows) {
  constexpr int C = D / 16, kItems = 2;
  const AppendParams& a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = blockDim.x / 64;
  // the block: blocks of the rows' new tokens, counted 64 rows at a time
  __shared__ uint32_t most_lds[2][16];
  __shared__ uint32_t bound_lds[2][16][2][D / 2];
  int b = -1, rel = 0;
  int64_t before = 0;
  for (int b0 = 0; b0 < a.cache.B && b < 0; b0 += 64) {
    int n = 0;
    if (b0 + lane < a.cache.B) {
      const int lo = clamp_to(a.cu[b0 + lane], a.N), hi = clamp_to(a.cu[b0 + lane + 1], a.N);
      const int64_t len = a.lens[b0 + lane];
      if (hi > lo) n = (int)(((len - 1) >> p.c.block_shift) - ((len - (hi - lo)) >> p.c.block_shift)) + 1;
    }
    const int sum = lane_scan(n);
    const int past = __popcll(__ballot(before + sum <= (int64_t)blockIdx.x));
    if (past < 64) {
      b = b0 + past;
      rel = (int)(blockIdx.x - before) - __builtin_amdgcn_readlane(sum, past) + __builtin_amdgcn_readlane(n, past);
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  if (b < 0) return;
  b = __builtin_amdgcn_readfirstlane(b);
  const int lo_token = clamp_to(a.cu[b], a.N), n_new = clamp_to(a.cu[b + 1], a.N) - lo_token;
  const int64_t len = a.lens[b], start = len - n_new;  // the new tokens are [start, len) of the row
  const int64_t nb = (start >> p.c.block_shift) + rel, base = nb << p.c.block_shift;
  int page = 0;
  uint32_t place = 0;
  bool has_page = find_page(p, b, base, page, place);
  const uint32_t held = start > base ? (uint32_t)(start - base) : 0;

  // this thread's units and their angles
  const int unit = threadIdx.x % C;
  const Unit un = unit_of(a, unit);
  int token[kItems];
  uint32_t slot[kItems];
  bool active[kItems], stored[kItems];
  Angles an[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    slot[i] = threadIdx.x / C + i * (blockDim.x / C);
    const int64_t at = base + slot[i];
    active[i] = slot[i] < (1u << p.c.block_shift) && at >= start && at < len;
    token[i] = active[i] ? lo_token + (int)(at - start) : lo_token;
    if (active[i]) active[i] = load_angles(a, un, token[i], at, an[i]);
    stored[i] = active[i] && has_page && at < a.cache.max_tokens;
  }
  has_page = __syncthreads_or(stored[0] || stored[1]);  // a block without new tokens is left alone

  const int H = a.cache.H, rows = a.Hq + 2 * H;
  const int r0 = blockIdx.y * slice_rows, r1 = min(r0 + slice_rows, rows);
  auto load = [&](int r, u32x4 (&x)[kItems], u32x4 (&y)[kItems]) __attribute__((always_inline)) {
    const hg_rows& t = r < H ? a.k : r < 2 * H ? a.v : a.q;
    const int h = r < H ? r : r < 2 * H ? r - H : r - 2 * H;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      x[i] = y[i] = u32x4{0, 0, 0, 0};
      if (!active[i]) continue;
      const uint16_t* src = t.data + token[i] * t.token_stride + h * t.head_stride;
      x[i] = load_piece<Once>(src + un.c0);
      y[i] = load_piece<Once>(src + un.c1);
    }
  };
  u32x4 x[kItems], y[kItems], nx[kItems], ny[kItems];
  load(r0, nx, ny);
  int turn = 0;
  for (int r = r0; r < r1; ++r) {
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      x[i] = nx[i];
      y[i] = ny[i];
    }
    if (r + 1 < r1) load(r + 1, nx, ny);
    const bool is_k = r < H, is_q = r >= 2 * H;
    if ((is_k || is_q) && un.rotated)
#pragma unroll
      for (int i = 0; i < kItems; ++i)
        if (active[i]) rotate(x[i], y[i], an[i], a.interleaved);
    if (is_q || (is_k && a.k_out.data)) {
      const hg_rows& t = is_q ? a.q_out : a.k_out;
      const int h = is_q ? r - 2 * H : r;
#pragma unroll
      for (int i = 0; i < kItems; ++i)
        if (active[i]) {
          uint16_t* o = t.data + token[i] * t.token_stride + h * t.head_stride;
          store_piece<Once>(o + un.c0, x[i]);
          store_piece<Once>(o + un.c1, y[i]);
        }
    }
    if (is_q || !has_page) continue;

    // the largest magnitude of the block, and each channel's bounds; a second pass
    // leaves out what is not finite if there is any
    const int h = is_k ? r : r - H;
    const bool bounded = is_k && p.c.bounds;
    uint32_t most = 0;
    int buffer = 0;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
      buffer = turn++ & 1;
      most = 0;
      uint32_t lo[8], hi[8];
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        lo[w] = kInf2;
        hi[w] = kMinusInf2;
      }
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        if (!stored[i]) continue;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          const uint32_t z = w < 4 ? x[i][w & 3] : y[i][w & 3];
          if (pass == 0) {
            most = max_u16(most, z & 0x7FFF7FFFu);
            const uint32_t o = ordered(z);
            lo[w] = min_i16(lo[w], o);
            hi[w] = max_i16(hi[w], o);
          } else {
            most = max_u16(most, numbers<true>(z, 0) & 0x7FFF7FFFu);
            lo[w] = min_i16(lo[w], ordered(numbers<false>(z, kInf2)));
            hi[w] = max_i16(hi[w], ordered(numbers<false>(z, kBelow2)));
          }
        }
      }
      most = max(most & 0xFFFFu, most >> 16);
#pragma unroll
      for (int s = 1; s < 64; s *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, s));
      if (lane == 0) most_lds[buffer][wave] = most;
      if (bounded) {
#pragma unroll
        for (int s = C; s < 64; s *= 2)
#pragma unroll
          for (int w = 0; w < 8; ++w) {
            lo[w] = min_i16(lo[w], (uint32_t)__shfl_xor((int)lo[w], s));
            hi[w] = max_i16(hi[w], (uint32_t)__shfl_xor((int)hi[w], s));
          }
        if (lane < C) {
#pragma unroll
          for (int w = 0; w < 8; ++w) {
            const int c = ((w < 4 ? un.c0 : un.c1) + 2 * (w & 3)) / 2;
            bound_lds[buffer][wave][0][c] = lo[w];
            bound_lds[buffer][wave][1][c] = hi[w];
          }
        }
      }
      __syncthreads();
      most = 0;
      for (int w = 0; w < waves; ++w) most = max(most, most_lds[buffer][w]);
      if (most < 0x7F80u) break;
    }

    const int64_t block = ((int64_t)page * H + h) * p.c.page_blocks + (place >> p.c.block_shift);
    float* scale = (is_k ? p.c.k_scale : p.c.v_scale) + block;
    uint8_t* first = (is_k ? p.c.K : p.c.V) + page * a.cache.page_stride + h * a.cache.head_stride + place * a.cache.token_stride;
    const int needed = scale_exponent(most << 16);
    int e = needed;
    if (held) {
      const int old = stored_exponent(*scale, needed);
      e = max(old, needed);
      if (e > old) {
        const float ratio = exponent_ratio(old - e);
        for (uint32_t i = threadIdx.x; i < held * C; i += blockDim.x) {
          u32x4* piece = (u32x4*)(first + i / C * a.cache.token_stride + i % C * 16);
          u32x4 z = *piece;
#pragma unroll
          for (int w = 0; w < 4; ++w) z[w] = rescale_codes(z[w], ratio);
          *piece = z;
        }
      }
      __syncthreads();  // the old scale is read
    }
    if (threadIdx.x == 0) *scale = exponent_scale(e);
    const float inv = exponent_inverse(e);
#pragma unroll
    for (int i = 0; i < kItems; ++i)
      if (stored[i]) {
        uint8_t* o = first + slot[i] * a.cache.token_stride;
        *(u32x2*)(o + un.c0) = to_codes8(x[i], inv);
        *(u32x2*)(o + un.c1) = to_codes8(y[i], inv);
      }
    if (bounded) {
      uint16_t* bounds = p.c.bounds + block * 2 * D;
      for (int i = threadIdx.x; i < D; i += blockDim.x) {  // channel pairs of either bound
        const int which = i / (D / 2), c = i % (D / 2);
        uint32_t* o = (uint32_t*)(bounds + which * D) + c;
        uint32_t z = held ? ordered(numbers<false>(*o, which ? kBelow2 : kInf2)) : which ? kMinusInf2 : kInf2;
        for (int w = 0; w < waves; ++w) {
          const uint32_t v = bound_lds[buffer][w][which][c];
          z = which ? max_i16(z, v) : min_i16(z, v);
        }
        *o = ordered(z);
      }
    }
  }
}

// At most the blocks that the new tokens lie in: of a row's n >= 2 tokens the first
// and the last may lie alone in theirs.
int64_t most_blocks(const Append8Params& p) {
  const int64_t rows = p.a.cache.B < p.a.N ? p.a.cache.B : p.a.N;
  return (p.a.N >> p.c.block_shift) + 2 * rows;
}
// Heads (of keys, values and queries) of a workgroup: all, or fewer where that
// would leave the card idle.
int slice_rows_of(const Append8Params& p) {
  const int rows = p.a.Hq + 2 * p.a.cache.H;
  const int64_t slices = (2048 + most_blocks(p) - 1) / most_blocks(p);
  const int64_t n = (rows + slices - 1) / slices;
  return n < 1 ? 1 : (int)n;
}

template <int D>
hipError_t launch(const Append8Params& p, hipStream_t stream) {
  if (!p.a.cu) {
    const int64_t waves = (int64_t)p.a.N * token_waves<D>(p);
    append8_token_kernel<D><<<dim3((uint32_t)((waves + 3) / 4)), dim3(kTokenThreads), 0, stream>>>(p);
    return hipGetLastError();
  }
  const int slice = slice_rows_of(p), rows = p.a.Hq + 2 * p.a.cache.H;
  const dim3 grid((uint32_t)most_blocks(p), (uint32_t)((rows + slice - 1) / slice));
  const dim3 threads((uint32_t)block_threads(p, D));
  const double bytes = 1.0 * D * p.a.N * (4.0 * p.a.Hq + (p.a.k_out.data ? 8.0 : 6.0) * p.a.cache.H);
  if (bytes > (double)(256 << 20)) append8_block_kernel<D, true><<<grid, threads, 0, stream>>>(p, slice);
  else append8_block_kernel<D, false><<<grid, threads, 0, stream>>>(p, slice);
  return hipGetLastError();
}

}  // namespace

int64_t append8_work_items(const Append8Params& p, int D) {
  if (!p.a.cu) {
    const int64_t waves = (int64_t)p.a.N * (D == 64 ? token_waves<64>(p) : D == 128 ? token_waves<128>(p) : token_waves<256>(p));
    return (waves + 3) / 4 * kTokenThreads;
  }
  return most_blocks(p) * block_threads(p, D);
}

hipError_t launch_append8(const Append8Params& p, int D, hipStream_t stream) {
  return D == 64 ? launch<64>(p, stream) : D == 128 ? launch<128>(p, stream) : launch<256>(p, stream);
}

}  // namespace hg
