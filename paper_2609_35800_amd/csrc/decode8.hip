// Attention of one new token per batch row over the 8-bit cache, of all cached
// tokens or of those in the blocks listed.
//
// The mathematics, the cut into runs and the join of parts are decode.hip's, the
// keys and values code * scale.  Every code is read once: half the bytes of a BF16
// cache for the same products, so the vector work counts, and the layout keeps it
// small:
//   * A wavefront takes tiles of 16 tokens, each within one block and page, so a
//     tile has one address and one scale for keys and one for values, in scalar
//     registers; the lanes look up the tiles of the next 16 steps at once, 64 of them.
//   * Codes become BF16 by the conversion that takes a power-of-two scale along: two
//     an instruction, exact, and no scale is left for scores or weights.
//   * S^T = K Q^T and O^T = V^T P^T on the matrix units (16x16x32 steps), the query
//     heads of a KV head as the 16 columns, as in decode.hip.  A lane reads keys in
//     16-byte pieces, channels 64 p + 16 g .. of token r for lane = 16 g + r, and the
//     queries' channels are laid to match.  It reads the D/16 channels r D/16 .. of
//     the values of tokens 4 g .. 4 g + 3 of a tile: four words of four tokens are
//     transposed by eight byte permutes, then converted, and are an operand.
//   * Tokens outside the row are dealt with only in chunks that hold some.
// Measured: 64 rows of 256 to 6656 tokens, 64 query and 8 KV heads of 128 channels, 464
// MB: 89.4 us, 5.2 TB/s (the BF16 cache, 924 MB: 162), of 64 channels 59.3 us, 3.9 TB/s,
// of 256 166 us, 5.6 TB/s; one row of 131072 tokens, 4 KV heads, 134 MB: 35.0 us (57.5);
// one of 1361: 10.0.  1024 chosen tokens of each of the 64 rows, 112 MB of codes: the
// kernel 27.1 us.  A wavefront has a vector instruction running a fifth of its time, so
// with two on a SIMD its vector unit is busy about two fifths: memory bounds large
// calls, small ones the chain lengths -> (list ->) table -> codes -> parts -> their join.
#include "hg_attn.h"
#include "hg_decode.h"
#include "hg_device.h"
#include "hg_e4m3.h"

namespace hg {
namespace {

// 16-token tiles of a wavefront's step: 8 KiB of keys and as much of values.
template <int D>
constexpr int kTiles = D == 256 ? 2 : 4;

// Tiles of a row's span: those that hold its tokens, or those of the listed blocks.
__device__ __forceinline__ uint32_t span_tiles(const Decode8Params& p, const Span& s) {
  if (s.len <= s.first) return 0;
  if (!p.blocks) return ((uint32_t)(s.len - 1) >> 4) - ((uint32_t)s.first >> 4) + 1;
  const uint32_t n = ((uint32_t)(s.len - 1) >> p.c.block_shift) - ((uint32_t)s.first >> p.c.block_shift) + 1;
  return min(n, (uint32_t)p.budget) << (p.c.block_shift - 4);
}

// What turning to another item costs a workgroup with a share of the list, in
// chunks (64 rows of 256 to 6656 tokens, 8 KV heads: 98.7 us if it counts nothing, 90.3
// for 2, 89.4 for 4, 90.0 for 8; of 64 channels 70.5, 63.0, 59.3, 56.5, of 256 175, 168,
// 166, 167; 128 rows of 64 to 512 tokens 42.8, 34.4, 34.5, 33.1).
constexpr int kItemChunks = 4;

// What the lanes know of tiles: lane holds that of tile lane % kTiles of step lane / kTiles.
struct Tiles {
  int64_t off;       // of the first row
  uint32_t seen;     // which of the 16 tokens are attended
  float k_scale, v_scale;
};
__device__ __forceinline__ Tiles find_tile(const Decode8Params& p, int b, int h, const Span& s, uint32_t i, bool active) {
  const PagedCache& c = p.d.cache;
  Tiles x = {0, 0, 1.0f, 1.0f};  // row 0 of page 0 stands in, so every load is inside the cache
  if (!active) return x;
  uint32_t tile;
  if (p.blocks) {
    const int up = p.c.block_shift - 4;
    const uint32_t id = (uint32_t)p.blocks[((int64_t)b * c.H + h) * p.budget + (i >> up)];
    if (id > (uint32_t)(s.len - 1) >> p.c.block_shift) return x;  // -1 too
    tile = (id << up) + (i & ((1u << up) - 1));
  } else {
    tile = ((uint32_t)s.first >> 4) + i;
  }
  const int t = (int)(tile << 4);  // a tile of a block that starts before len: below 2^31
  const int lo = min(max(s.first - t, 0), 16), hi = min(max(s.len - t, 0), 16);
  if (hi <= lo) return x;
  const uint32_t pg = divide((uint32_t)t, c);
  const int page = c.table[(int64_t)b * c.max_pages + pg];
  if (page < 0 || page >= c.num_pages) return x;
  const uint32_t at = (uint32_t)t - pg * (uint32_t)c.page_size;
  const int64_t scale = ((int64_t)page * c.H + h) * p.c.page_blocks + (at >> p.c.block_shift);
  x.off = page * c.page_stride + at * c.token_stride;
  x.seen = ((1u << hi) - 1) & ~((1u << lo) - 1);
  x.k_scale = p.c.k_scale[scale];
  x.v_scale = p.c.v_scale[scale];
  return x;
}

// A step's tiles, wave-uniform: where they are, and what their tokens count for
// (taken later, so that the codes are asked for before the scales are there).
template <int D>
struct Place {
  int64_t off[kTiles<D>];
};
template <int D>
struct Step {
  uint64_t seen;
  float k_scale[kTiles<D>], v_scale[kTiles<D>];
};
template <int D>
__device__ __forceinline__ Place<D> take_place(const Tiles& x, int at) {
  Place<D> s;
#pragma unroll
  for (int j = 0; j < kTiles<D>; ++j) {
    const int lane = at * kTiles<D> + j;
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)x.off, lane), hi = __builtin_amdgcn_readlane((int)(x.off >> 32), lane);
    s.off[j] = (int64_t)(((uint64_t)hi << 32) | lo);
  }
  return s;
}
template <int D>
__device__ __forceinline__ Step<D> take_step(const Tiles& x, int at) {
  Step<D> s;
  s.seen = 0;
#pragma unroll
  for (int j = 0; j < kTiles<D>; ++j) {
    const int lane = at * kTiles<D> + j;
    s.seen |= (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)x.seen, lane) << (16 * j);
    s.k_scale[j] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x.k_scale), lane));
    s.v_scale[j] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x.v_scale), lane));
  }
  return s;
}

template <int D>
struct Loads8 {
  static constexpr int P = D / 64;   // 16-byte pieces of a key per lane
  static constexpr int W = D / 64;   // words of a value per lane
  static constexpr int TT = kTiles<D>;
  q32x4 k[TT][P];
  uint32_t v[TT][4][W];
};

// Once: streaming (non-temporal) loads, see decode8_stream_chunks.
template <bool Once, class T>
__device__ __forceinline__ T load_codes(const uint8_t* p) {
  if constexpr (Once) return __builtin_nontemporal_load((const T*)p);
  else return *(const T*)p;
}

// K: this lane's first piece of a tile.  From head_dim 128 on an access takes whole
// 128-byte lines, eight lanes a token: lane 16 g + r piece 4 (r / 8) + g of tokens
// r % 8 and 8 + r % 8 (half lines at a time, 16 tokens an access, the second half
// waits in the cache for the first: 64 rows 104 us).  swap_tokens then gives it
// pieces g and 4 + g of token r.
template <int D, bool Once>
__device__ __forceinline__ void load_keys(Loads8<D>& x, const uint8_t* K, int64_t token_stride, const Place<D>& s) {
#pragma unroll
  for (int j = 0; j < Loads8<D>::TT; ++j)
#pragma unroll
    for (int c = 0; c < Loads8<D>::P; ++c)
      x.k[j][c] = load_codes<Once, q32x4>(K + (s.off[j] + (c & 1) * 8 * token_stride) + (c >> 1) * 128);
}
__device__ __forceinline__ void swap_tokens(q32x4& a, q32x4& b) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {  // row_ror:8 into lanes 8 .. 15, or 0 .. 7, of each 16
    const int x = (int)a[w], y = (int)b[w];
    a[w] = (uint32_t)__builtin_amdgcn_update_dpp(x, y, 0x128, 0xF, 0xC, false);
    b[w] = (uint32_t)__builtin_amdgcn_update_dpp(y, x, 0x128, 0xF, 0x3, false);
  }
}
template <int D, bool Once>
__device__ __forceinline__ void load_values(Loads8<D>& x, const uint8_t* V, int64_t token_stride, const Place<D>& s) {
#pragma unroll
  for (int j = 0; j < Loads8<D>::TT; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint8_t* row = V + (s.off[j] + i * token_stride);
      if constexpr (D == 256) {
        const q32x4 y = load_codes<Once, q32x4>(row);
#pragma unroll
        for (int w = 0; w < 4; ++w) x.v[j][i][w] = y[w];
      } else if constexpr (D == 128) {
        const q32x2 y = load_codes<Once, q32x2>(row);
        x.v[j][i][0] = y[0];
        x.v[j][i][1] = y[1];
      } else {
        x.v[j][i][0] = load_codes<Once, uint32_t>(row);
      }
    }
}

// A segment as a wavefront sees it; wave-uniform.
struct Item {
  Segment sg;
  int h, tile0, rows;  // key/value head, query heads of the tile
  int steps;           // of this wavefront; 0 for a row without tokens
};
__device__ __forceinline__ Item item_of(const Segment& sg, const DecodeParams& d, int wave) {
  Item i;
  i.sg = sg;
  i.h = sg.pair / d.row_tiles;
  i.tile0 = (sg.pair - i.h * d.row_tiles) * kDecodeRows;
  i.rows = min(d.R - i.tile0, kDecodeRows);
  i.steps = sg.span.first < sg.span.len && sg.c0 + wave < sg.c1 ? (sg.c1 - sg.c0 - wave + kWaves - 1) / kWaves : 0;
  return i;
}

// Split: at most 8 query heads a KV head, which take the 16 columns twice, see below.
template <int D, RunMode Mode, bool Split>
__global__ __launch_bounds__(kThreadsDecode, 2) void decode8_kernel(const Decode8Params p) {
  constexpr int P = Loads8<D>::P, W = Loads8<D>::W, TT = kTiles<D>, J = D / 16;
  constexpr int kHeldSteps = 64 / TT;  // steps whose tiles the lanes hold
  extern __shared__ float lds[];  // [kWaves][rows][D + 4] parts, then their m and l
  const DecodeParams& d = p.d;
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int per_row = d.cache.H * d.row_tiles;  // (head, row tile) pairs of a batch row
  auto count = [&](const Span& s) __attribute__((always_inline)) { return (int)max((span_tiles(p, s) + TT - 1) / TT, 1u); };
  Run<Mode, Mode == kShares ? kItemChunks : 0, Mode == kSegments> run;
  Segment sg;
  if (!run.begin(d, per_row, count) || !run.next(d, per_row, count, sg)) return;
  const bool streamed = run.row_chunks > d.stream_chunks;

  const uint32_t rest_columns = r < 8 ? 0u : ~0u;  // Split: which columns take the weights' left-overs

  // One item, or part of one, a turn.  The first tiles of the next one are looked up
  // before this one's last step, which asks for their codes as for those of any other
  // step: they arrive while the workgroup joins its parts.
  const int64_t ts = d.cache.token_stride;
  Item it = item_of(sg, d, wave);
  Tiles held;
  Loads8<D> x;
  auto find = [&](const Item& i, int k0) __attribute__((always_inline)) {
    const int k = k0 + lane / TT;
    const uint32_t n = (uint32_t)(i.sg.c0 + wave + kWaves * k) * TT + lane % TT;
    return find_tile(p, i.sg.b, i.h, i.sg.span, n, k < i.steps && n < span_tiles(p, i.sg.span));
  };
  // this lane's first bytes of a head's keys and values
  auto keys_of = [&](int h) __attribute__((always_inline)) {
    return p.c.K + h * d.cache.head_stride + (P == 1 ? r * ts + g * 16 : (r & 7) * ts + ((r >> 3) * 4 + g) * 16);
  };
  auto values_of = [&](int h) __attribute__((always_inline)) {
    return p.c.V + h * d.cache.head_stride + 4 * g * ts + r * (D / 16);
  };
  auto begin = [&](auto once) __attribute__((always_inline)) {
    constexpr bool Once = decltype(once)::value;
    held = find(it, 0);
    if (it.steps > 0) {
      const Place<D> at = take_place<D>(held, 0);
      load_keys<D, Once>(x, keys_of(it.h), ts, at);
      load_values<D, Once>(x, values_of(it.h), ts, at);
    }
  };
  auto run_items = [&](auto once) __attribute__((always_inline)) {
    constexpr bool Once = decltype(once)::value;
    begin(once);
    while (true) {
      const Item now = it;
      const int b = now.sg.b, h = now.h, tile0 = now.tile0, rows = now.rows, steps = now.steps;

      // queries: lane's head is r (Split: r % 8), channels 64 c + 16 g + 8 i ..
      q32x4 q[P][2];
      {
        const int hq = h * d.R + tile0 + min(Split ? r & 7 : r, rows - 1);
        const uint16_t* src = d.q.data + b * d.q.token_stride + hq * d.q.head_stride + g * 16;
#pragma unroll
        for (int c = 0; c < P; ++c) {
          q[c][0] = *(const q32x4*)(src + c * 64);
          q[c][1] = *(const q32x4*)(src + c * 64 + 8);
        }
      }
      f32x4 acc[J];
#pragma unroll
      for (int j = 0; j < J; ++j) acc[j] = f32x4{0, 0, 0, 0};
      float m_run = kNegInf, l_run = 0;

      // One step; the next one's keys are asked for once the scores are taken, its
      // values once these are used.
      auto step = [&](const Step<D>& s, bool more, const uint8_t* K, const uint8_t* V, const Place<D>& next) __attribute__((always_inline)) {
        f32x4 st[TT];
#pragma unroll
        for (int j = 0; j < TT; ++j) {
          st[j] = f32x4{0, 0, 0, 0};
#pragma unroll
          for (int c = 0; c + 1 < P; c += 2) swap_tokens(x.k[j][c], x.k[j][c + 1]);
#pragma unroll
          for (int c = 0; c < P; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t lo = x.k[j][c][2 * i], hi = x.k[j][c][2 * i + 1];
              const q32x4 k = {codes_bf16<false>(lo, s.k_scale[j]), codes_bf16<true>(lo, s.k_scale[j]),
                               codes_bf16<false>(hi, s.k_scale[j]), codes_bf16<true>(hi, s.k_scale[j])};
              st[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[c][i]),
                                                              st[j], 0, 0, 0);
            }
        }
        if (more) load_keys<D, Once>(x, K, ts, next);
        const bool whole = s.seen == ~0ull >> (64 - 16 * TT);
        float sc[4 * TT];
#pragma unroll
        for (int i = 0; i < 4 * TT; ++i) sc[i] = st[i >> 2][i & 3] * d.scale_log2;
        const uint64_t mine = s.seen >> (4 * g);
        if (!whole) {
#pragma unroll
          for (int i = 0; i < 4 * TT; ++i) sc[i] = (mine >> (16 * (i >> 2) + (i & 3))) & 1 ? sc[i] : kNegInf;
        }
        float top = kNegInf;
#pragma unroll
        for (int i = 0; i < 4 * TT; ++i) top = fmaxf(top, sc[i]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m = fmaxf(m_run, top);
        const float down = weight(m_run, m);
        m_run = m;
        l_run *= down;
#pragma unroll
        for (int j = 0; j < J; ++j) acc[j] *= down;
        // The matrix units take the weights in the values' type, BF16: a weight goes in
        // as its nearest BF16 number and what that leaves, again rounded, 2^-16 of it
        // lost.  With up to 8 heads the left-overs are the weights of columns 8 .. 15,
        // which repeat the heads, and no product is added; with more they cost a
        // second one.  The weights' sum is of the unrounded ones.
        uint32_t w[2 * TT], w_rest[Split ? 1 : 2 * TT];
#pragma unroll
        for (int i = 0; i < 4 * TT; i += 2) {
          const float p0 = weight(sc[i], m), p1 = weight(sc[i + 1], m);
          l_run += p0 + p1;
          w[i >> 1] = cvt_bf16x2(p0, p1);
          const uint32_t taken = Split ? w[i >> 1] & rest_columns : w[i >> 1];
          const uint32_t rest = cvt_bf16x2(p0 - bf16_lo(taken), p1 - bf16_hi(taken));
          if constexpr (Split) w[i >> 1] = rest;
          else w_rest[i >> 1] = rest;
        }
        if (!whole) {  // values that are not attended count as 0, whatever they hold
#pragma unroll
          for (int i = 0; i < 4 * TT; ++i) {
            const uint32_t keep = (mine >> (16 * (i >> 2) + (i & 3))) & 1 ? ~0u : 0u;
#pragma unroll
            for (int c = 0; c < W; ++c) x.v[i >> 2][i & 3][c] &= keep;
          }
        }
#pragma unroll
        for (int u = 0; u < TT / 2; ++u)
#pragma unroll
          for (int c = 0; c < W; ++c) {
            uint32_t y[2][4];  // of a tile: the codes of channel 4 c + e of its four tokens
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const auto& v = x.v[2 * u + j];
              const uint32_t a0 = __builtin_amdgcn_perm(v[1][c], v[0][c], 0x05010400u), a1 = __builtin_amdgcn_perm(v[1][c], v[0][c], 0x07030602u);
              const uint32_t b0 = __builtin_amdgcn_perm(v[3][c], v[2][c], 0x05010400u), b1 = __builtin_amdgcn_perm(v[3][c], v[2][c], 0x07030602u);
              y[j][0] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
              y[j][1] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
              y[j][2] = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
              y[j][3] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
            }
            const float s0 = s.v_scale[2 * u], s1 = s.v_scale[2 * u + 1];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const q32x4 v = {codes_bf16<false>(y[0][e], s0), codes_bf16<true>(y[0][e], s0), codes_bf16<false>(y[1][e], s1),
                               codes_bf16<true>(y[1][e], s1)};
              acc[4 * c + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  __builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, q32x4{w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]}),
                  acc[4 * c + e], 0, 0, 0);
              if constexpr (!Split)
                acc[4 * c + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    __builtin_bit_cast(bf16x8, v),
                    __builtin_bit_cast(bf16x8, q32x4{w_rest[4 * u], w_rest[4 * u + 1], w_rest[4 * u + 2], w_rest[4 * u + 3]}),
                    acc[4 * c + e], 0, 0, 0);
            }
          }
        if (more) load_values<D, Once>(x, V, ts, next);
      };
      const uint8_t *K = keys_of(h), *V = values_of(h);
      for (int k = 1; k < steps; ++k) {
        const Step<D> s = take_step<D>(held, (k - 1) % kHeldSteps);
        if (k % kHeldSteps == 0) held = find(now, k);
        step(s, true, K, V, take_place<D>(held, k % kHeldSteps));
      }
      Step<D> s;
      if (steps > 0) s = take_step<D>(held, (steps - 1) % kHeldSteps);
      const bool more = Mode == kShares && run.next(d, per_row, count, sg);
      if (more) {
        it = item_of(sg, d, wave);
        held = find(it, 0);
      }
      if (steps > 0) {
        const bool ahead = more && it.steps > 0;
        Place<D> at = {};
        if (ahead) at = take_place<D>(held, 0);
        step(s, ahead, keys_of(it.h), values_of(it.h), at);
      } else if (more && it.steps > 0) {
        const Place<D> at = take_place<D>(held, 0);
        load_keys<D, Once>(x, keys_of(it.h), ts, at);
        load_values<D, Once>(x, values_of(it.h), ts, at);
      }
      l_run += __shfl_xor(l_run, 16);
      l_run += __shfl_xor(l_run, 32);
      if constexpr (Split) {  // the heads' two columns (row_ror:8)
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            acc[j][i] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(acc[j][i]), 0x128, 0xF, 0xF, false));
      }

      // the wavefront's result, for their join
      constexpr int pitch = D + 4;
      float* part = lds;                          // [kWaves][rows][pitch]
      float* stat = lds + kWaves * rows * pitch;  // [kWaves][2][rows]
      if (g == 0 && r < rows) {
        stat[(wave * 2) * rows + r] = m_run;
        stat[(wave * 2 + 1) * rows + r] = l_run;
      }
      if (r < rows) {
        float* row = part + (wave * rows + r) * pitch;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < J; ++e) row[(g * 4 + i) * J + e] = acc[e][i];
      }
      finish_item<D>(d, now.sg, h, tile0, rows, lds);
      if (!more) break;
    }
  };
  if (streamed) run_items(std::true_type());
  else run_items(std::false_type());
}

template <int D, RunMode Mode, bool Split>
hipError_t launch(const Decode8Params& p, hipStream_t stream) {
  const size_t bytes = decode_lds_bytes(p.d.R, D);
  if (bytes > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)decode8_kernel<D, Mode, Split>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)bytes);
    if (e != hipSuccess) return e;
  }
  decode8_kernel<D, Mode, Split><<<dim3(kDecodeSlots), dim3(kThreadsDecode), bytes, stream>>>(p);
  return hipGetLastError();
}
template <int D>
hipError_t launch(const Decode8Params& p, hipStream_t stream) {
  const bool shares = runs_are_shares((int64_t)p.d.cache.B * p.d.cache.H * p.d.row_tiles);
  if (p.d.R <= 8) return shares ? launch<D, kShares, true>(p, stream) : launch<D, kSegments, true>(p, stream);
  return shares ? launch<D, kShares, false>(p, stream) : launch<D, kSegments, false>(p, stream);
}

}  // namespace

// Chunks of all rows past which a call's codes are streamed: decode_stream_chunks'
// rule, in bytes.
int64_t decode8_stream_chunks(const PagedCache& c, int D, int row_tiles) {
  const double pool = 2.0 * c.num_pages * c.page_size * c.H * D;
  if (pool <= (double)(256 << 20) || row_tiles > 1) return INT64_MAX;
  const int chunk = 16 * (D == 256 ? kTiles<256> : kTiles<128>);
  return ((int64_t)10 << 20) / ((int64_t)2 * c.H * D * chunk);
}

hipError_t launch_decode8(const Decode8Params& p, int D, hipStream_t stream) {
  switch (D) {
    case 64: return launch<64>(p, stream);
    case 128: return launch<128>(p, stream);
    default: return launch<256>(p, stream);
  }
}

}  // namespace hg
