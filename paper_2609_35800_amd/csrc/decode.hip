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
// 924 MB: 162 us, 5.7 TB/s; one row of 1361 tokens: 10.0 us.
#include <type_traits>

#include "hg_attn.h"
#include "hg_decode.h"
#include "hg_device.h"

namespace hg {
namespace {

// Tokens of a wavefront's step: 8 KiB of keys and as much of values up to
// head_dim 128; 32 tokens at 256 would not fit the registers.
template <int D>
constexpr int kChunk = D == 256 ? 16 : 32;

template <int D>
__device__ __forceinline__ int span_chunks(const Span& s) {
  return max((int)(((uint32_t)(s.len - s.first) + kChunk<D> - 1) / kChunk<D>), 1);
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

template <int D>
__global__ __launch_bounds__(kThreadsDecode, 2) void decode_kernel(const DecodeParams p) {
  constexpr int S = D / 32, J = D / 16;
  constexpr int VP = Loads<D>::VP, VW = Loads<D>::VW, TT = Loads<D>::TT;
  extern __shared__ float lds[];  // [kWaves][rows][D + 4] parts, then their m and l
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int per_row = p.cache.H * p.row_tiles;  // (head, row tile) pairs of a batch row

  auto count = [](const Span& s) __attribute__((always_inline)) { return span_chunks<D>(s); };
  Run<kEither, 0, false> run;
  if (!run.begin(p, per_row, count)) return;
  const bool streamed = run.row_chunks > p.stream_chunks;

  Segment sg;
  while (run.next(p, per_row, count, sg)) {  // one item, or part of one, a turn
    const int b = sg.b, pair = sg.pair, first = sg.span.first, len = sg.span.len, c0 = sg.c0, c1 = sg.c1;
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
    finish_item<D>(p, sg, h, tile0, rows, lds);
  }
}

template <int D>
hipError_t launch(const DecodeParams& p, hipStream_t stream) {
  const size_t bytes = decode_lds_bytes(p.R, D);
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
