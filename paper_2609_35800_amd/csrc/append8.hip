// Appending new tokens to the 8-bit cache, keys and queries rotated.
//
// Per (row, head, block of tokens): k' = bf16(R(p) k); m = max |k'| over the new
// tokens; e the smallest with m <= 448 2^e, or the block's present one if larger;
// codes e4m3(k' / 2^e); lo, hi = min, max of k' per channel, joined with the
// block's present ones.  Present are those of the row's own tokens, from starts[b] on:
// what another row left in a page, its scale and bounds too, counts for nothing.
// A power of two as scale makes k' / 2^e exact, so each key
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
// Measured: four prompts of up to 3008 tokens, 32 heads, 255 MB, 56.4 us, 4.5 TB/s (a
// large copy 4.8); the kernel of one token a row 4.9 us for one row, 7.8 for 64 rows of
// 64 query and 8 KV heads.
#include <type_traits>

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

// First token of row b.
__device__ __forceinline__ int64_t row_start(const Append8Params& p, int b) { return p.starts ? p.starts[b] : 0; }

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
  const int64_t own = at - row_start(p, token);  // the row's tokens before this one
  const bool stored = find_page(p, token, at, page, place) && own >= 0;
  const int64_t block = ((int64_t)page * a.cache.H + h) * p.c.page_blocks + (place >> p.c.block_shift);
  // the row's tokens that the block holds, right before this one
  const uint32_t held = (uint32_t)min((int64_t)(place & ((1u << p.c.block_shift) - 1)), max(own, (int64_t)0));
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
  *(u32x2*)(codes + un.c0) = to_codes8<false>(x, inv);
  *(u32x2*)(codes + un.c1) = to_codes8<false>(y, inv);
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

// Maximum over the wavefront, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xF, 0xF, false));  // row_ror:1, 2, 4, 8
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false));
  auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(s[0], s[1]);
  s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(s[0], s[1]);
}

// Minima or maxima of words over the lanes with the same lane % C, in three steps:
// two words share a register after each of the first two, so that lanes 16 j .. of
// the result of words 0 .. 3 hold word 2 (j & 1) + (j >> 1).
template <class Op>
__device__ __forceinline__ uint32_t reduce_halves(uint32_t x, uint32_t y, const Op& op) {
  const auto s = __builtin_amdgcn_permlane32_swap(x, y, false, false);
  return op(s[0], s[1]);
}
template <int C, class Op>
__device__ __forceinline__ uint32_t reduce_rest(uint32_t x, uint32_t y, const Op& op) {
  const auto s = __builtin_amdgcn_permlane16_swap(x, y, false, false);
  uint32_t v = op(s[0], s[1]);
  if constexpr (C <= 8) v = op(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false));
  if constexpr (C <= 4) v = op(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, false));
  return v;
}

// The new tokens of one block, as a workgroup sees them.
struct Block {
  int page;
  uint32_t place;        // of the page
  uint32_t held;         // the row's tokens that it held before, 256 times the first one's place in it added
  int64_t index;         // of head 0's scale
  bool has_page;         // some token is stored
};

constexpr int kItems = 2;

// Heads [h0, h1) of the keys (Key), the values or (Query) the queries.
template <int D, bool Once, bool Key, bool Query>
__device__ __forceinline__ void append_heads(const Append8Params& p, const Block& blk, const Unit& un, const int (&token)[kItems],
                                             const uint32_t (&slot)[kItems], const bool (&active)[kItems],
                                             const bool (&stored)[kItems], const Angles (&an)[kItems], int h0, int h1,
                                             uint32_t (*most_lds)[16], uint32_t (*bound_lds)[16][2][D / 2]) {
  constexpr int C = D / 16;
  const AppendParams& a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = blockDim.x / 64;
  const hg_rows& in = Query ? a.q : Key ? a.k : a.v;
  const hg_rows& out = Query ? a.q_out : a.k_out;
  const bool copied = Query || (Key && a.k_out.data);
  const uint16_t* src[kItems];
  uint16_t* dst[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    src[i] = in.data + token[i] * in.token_stride + h0 * in.head_stride;
    if (copied) dst[i] = out.data + token[i] * out.token_stride + h0 * out.head_stride;
  }
  uint8_t* codes = (Key ? p.c.K : p.c.V) + blk.page * a.cache.page_stride + blk.place * a.cache.token_stride + h0 * a.cache.head_stride;
  float* scale = (Key ? p.c.k_scale : p.c.v_scale) + blk.index + (int64_t)h0 * p.c.page_blocks;
  uint32_t* bounds = (uint32_t*)p.c.bounds + (blk.index + (int64_t)h0 * p.c.page_blocks) * D;
  const bool bounded = Key && p.c.bounds;

  u32x4 nx[kItems], ny[kItems];
  auto load = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      nx[i] = ny[i] = u32x4{0, 0, 0, 0};
      if (active[i]) {
        nx[i] = load_piece<Once>(src[i] + un.c0);
        ny[i] = load_piece<Once>(src[i] + un.c1);
      }
      src[i] += in.head_stride;
    }
  };
  load();
  int turn = 0;
  for (int h = h0; h < h1; ++h) {
    u32x4 x[kItems], y[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      x[i] = nx[i];
      y[i] = ny[i];
    }
    if (h + 1 < h1) load();
    if ((Key || Query) && un.rotated)
#pragma unroll
      for (int i = 0; i < kItems; ++i) rotate(x[i], y[i], an[i], a.interleaved);
    if (copied) {
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        if (active[i]) {
          store_piece<Once>(dst[i] + un.c0, x[i]);
          store_piece<Once>(dst[i] + un.c1, y[i]);
        }
        dst[i] += out.head_stride;
      }
    }
    if constexpr (!Query) {
      if (!blk.has_page) continue;
      // the largest magnitude of the block, and each channel's bounds
      uint32_t most = 0;
      int buffer = 0;
      auto reduce = [&](auto only) __attribute__((always_inline)) {
        constexpr bool Numbers = decltype(only)::value;  // leave out what is not finite, or NaN
        const auto least = [](uint32_t a, uint32_t b) { return min_i16(a, b); };
        const auto largest = [](uint32_t a, uint32_t b) { return max_i16(a, b); };
        buffer = turn++ & 1;
        most = 0;
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int w2 = 0; w2 < 4; ++w2) {
          uint32_t l[2], u[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int w = 2 * w2 + k;
            l[k] = kInf2;
            u[k] = kMinusInf2;
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
              const uint32_t z = w < 4 ? x[i][w & 3] : y[i][w & 3];
              most = max_u16(most, stored[i] ? (Numbers ? numbers<true>(z, 0) : z) & 0x7FFF7FFFu : 0u);
              if constexpr (Key) {
                const uint32_t o = ordered(Numbers ? numbers<false>(z, kInf2) : z);
                l[k] = min_i16(l[k], stored[i] ? o : kInf2);
                u[k] = max_i16(u[k], stored[i] ? (Numbers ? ordered(numbers<false>(z, kBelow2)) : o) : kMinusInf2);
              }
            }
          }
          if constexpr (Key) {
            lo[w2] = reduce_halves(l[0], l[1], least);
            hi[w2] = reduce_halves(u[0], u[1], largest);
          }
        }
        most = wave_max(max(most & 0xFFFFu, most >> 16));
        if (lane == 0) most_lds[buffer][wave] = most;
        if (bounded) {
          const uint32_t l0 = reduce_rest<C>(lo[0], lo[1], least), l1 = reduce_rest<C>(lo[2], lo[3], least);
          const uint32_t u0 = reduce_rest<C>(hi[0], hi[1], largest), u1 = reduce_rest<C>(hi[2], hi[3], largest);
          if ((lane & 15) < C) {
            const int word = (lane >> 4 & 1) * 2 + (lane >> 5);  // of the pieces at c0 and c1
            bound_lds[buffer][wave][0][un.c0 / 2 + word] = l0;
            bound_lds[buffer][wave][0][un.c1 / 2 + word] = l1;
            bound_lds[buffer][wave][1][un.c0 / 2 + word] = u0;
            bound_lds[buffer][wave][1][un.c1 / 2 + word] = u1;
          }
        }
        __syncthreads();
        most = most_lds[buffer][0];
        for (int w = 1; w < waves; ++w) most = max(most, most_lds[buffer][w]);
      };
      reduce(std::false_type());
      const bool finite = most < 0x7F80u;
      if (!finite) reduce(std::true_type());

      const int needed = scale_exponent(most << 16);
      int e = needed;
      if (blk.held) {
        const int old = stored_exponent(*scale, needed);
        e = max(old, needed);
        if (e > old) {
          const float ratio = exponent_ratio(old - e);
          uint8_t* first = codes + (blk.held >> 8) * a.cache.token_stride;
          for (uint32_t i = threadIdx.x; i < (blk.held & 255) * C; i += blockDim.x) {
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
      auto store = [&](auto small) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kItems; ++i)
          if (stored[i]) {
            uint8_t* o = codes + slot[i] * a.cache.token_stride;
            *(u32x2*)(o + un.c0) = to_codes8<decltype(small)::value>(x[i], inv);
            *(u32x2*)(o + un.c1) = to_codes8<decltype(small)::value>(y[i], inv);
          }
      };
      if (finite && needed < 127 + 119) store(std::true_type());  // all within 448 2^e
      else store(std::false_type());
      if (bounded) {
        for (int i = threadIdx.x; i < D; i += blockDim.x) {  // channel pairs of either bound
          const int which = i / (D / 2), c = i % (D / 2);
          uint32_t* o = bounds + which * (D / 2) + c;
          uint32_t z = blk.held ? ordered(numbers<false>(*o, which ? kBelow2 : kInf2)) : which ? kMinusInf2 : kInf2;
          for (int w = 0; w < waves; ++w) {
            const uint32_t v = bound_lds[buffer][w][which][c];
            z = which ? max_i16(z, v) : min_i16(z, v);
          }
          *o = ordered(z);
        }
      }
      codes += a.cache.head_stride;
      scale += p.c.page_blocks;
      bounds += (int64_t)p.c.page_blocks * D;
    }
  }
}

// blockIdx.x: a block of a row's new tokens; blockIdx.y: some heads of the keys,
// then of the values, then of the queries.
template <int D, bool Once>
__global__ __launch_bounds__(1024) void append8_block_kernel(const Append8Params p, int kv_heads, int kv_slices, int q_heads) {
  constexpr int C = D / 16;
  const AppendParams& a = p.a;
  const int lane = threadIdx.x & 63;
  __shared__ uint32_t most_lds[2][16];
  __shared__ uint32_t bound_lds[2][16][2][D / 2];
  // the block: blocks of the rows' new tokens, counted 64 rows at a time
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
  // of the places before the first new token, those from the row's start on
  const uint32_t before_new = start > base ? (uint32_t)(start - base) : 0;
  const uint32_t own = (uint32_t)min(max(row_start(p, b) - base, (int64_t)0), (int64_t)1 << p.c.block_shift);
  const uint32_t from = min(own, before_new);
  Block blk = {0, 0, before_new > from ? from << 8 | (before_new - from) : 0, 0, false};
  const bool has_page = find_page(p, b, base, blk.page, blk.place);
  blk.index = (int64_t)blk.page * a.cache.H * p.c.page_blocks + (blk.place >> p.c.block_shift);

  // this thread's units and their angles
  const int slice = blockIdx.y;
  const bool is_k = slice < kv_slices, is_q = slice >= 2 * kv_slices;
  Unit un = unit_of(a, threadIdx.x % C);
  int token[kItems];
  uint32_t slot[kItems];
  bool active[kItems], stored[kItems];
  Angles an[kItems];
  Unit wanted = un;
  wanted.rotated = un.rotated && (is_k || is_q);
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    slot[i] = threadIdx.x / C + i * (blockDim.x / C);
    const int64_t at = base + slot[i];
    active[i] = slot[i] < (1u << p.c.block_shift) && at >= start && at < len;
    token[i] = active[i] ? lo_token + (int)(at - start) : lo_token;
    if (active[i]) active[i] = load_angles(a, wanted, token[i], at, an[i]);
    stored[i] = active[i] && has_page && at < a.cache.max_tokens && slot[i] >= own;
  }
  if (!is_q) blk.has_page = __syncthreads_or(stored[0] || stored[1]);  // a block without new tokens is left alone
  if (is_k)
    append_heads<D, Once, true, false>(p, blk, un, token, slot, active, stored, an, slice * kv_heads,
                                       min((slice + 1) * kv_heads, a.cache.H), most_lds, bound_lds);
  else if (!is_q)
    append_heads<D, Once, false, false>(p, blk, un, token, slot, active, stored, an, (slice - kv_slices) * kv_heads,
                                        min((slice - kv_slices + 1) * kv_heads, a.cache.H), most_lds, bound_lds);
  else
    append_heads<D, Once, false, true>(p, blk, un, token, slot, active, stored, an, (slice - 2 * kv_slices) * q_heads,
                                       min((slice - 2 * kv_slices + 1) * q_heads, a.Hq), most_lds, bound_lds);
}

// At most the blocks that the new tokens lie in: of a row's n >= 2 tokens the first
// and the last may lie alone in theirs.
int64_t most_blocks(const Append8Params& p) {
  const int64_t rows = p.a.cache.B < p.a.N ? p.a.cache.B : p.a.N;
  return (p.a.N >> p.c.block_shift) + 2 * rows;
}
// Heads of a workgroup: up to eight, which share their angles, fewer where that
// would leave the card idle (and more where a launch could not count the rest).
int heads_of(const Append8Params& p, int heads) {
  const int64_t all = most_blocks(p) * (p.a.Hq + 2 * (int64_t)p.a.cache.H);
  int64_t n = all / 2048;
  n = n < 1 ? 1 : n > 8 ? 8 : n;
  const int64_t least = (heads + 16383) / 16384;  // at most 3 * 16384 workgroups in y
  n = n < least ? least : n;
  return (int)(n < heads ? n : heads);
}
int slices_of(int heads, int each) { return heads ? (heads + each - 1) / each : 0; }

template <int D>
hipError_t launch(const Append8Params& p, hipStream_t stream) {
  if (!p.a.cu) {
    const int64_t waves = (int64_t)p.a.N * token_waves<D>(p);
    append8_token_kernel<D><<<dim3((uint32_t)((waves + 3) / 4)), dim3(kTokenThreads), 0, stream>>>(p);
    return hipGetLastError();
  }
  const int kv_heads = heads_of(p, p.a.cache.H), q_heads = p.a.Hq ? heads_of(p, p.a.Hq) : 1;
  const int kv_slices = slices_of(p.a.cache.H, kv_heads);
  const dim3 grid((uint32_t)most_blocks(p), (uint32_t)(2 * kv_slices + slices_of(p.a.Hq, q_heads)));
  const dim3 threads((uint32_t)block_threads(p, D));
  // Calls of more than half the 256 MiB last-level cache stream (255 MB: 64.6 -> 56.1
  // us, 128 MB: 37.4 -> 35.0, 98 MB: 28.2 both ways, 69 MB: 19.7 -> 21.7); with the
  // prompts' attention behind it both take the same (147 MB: 122.9 us together).
  const double bytes = 1.0 * D * p.a.N * (4.0 * p.a.Hq + (p.a.k_out.data ? 8.0 : 6.0) * p.a.cache.H);
  if (bytes > (double)(128 << 20)) append8_block_kernel<D, true><<<grid, threads, 0, stream>>>(p, kv_heads, kv_slices, q_heads);
  else append8_block_kernel<D, false><<<grid, threads, 0, stream>>>(p, kv_heads, kv_slices, q_heads);
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
