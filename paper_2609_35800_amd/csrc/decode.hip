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
//     S^T = K Q^T and O^T = V^T P^T (16x16x32), the query heads of a KV head
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
// The launch is kDecodeGroups workgroups, one per compute unit, each with an
// equal run of 32-token chunks of the list (batch row, KV head, chunk), so
// ragged rows and few long rows load the chip alike; the chunks of a run that
// belong to one (row, head) are dealt to the workgroup's wavefronts in turn,
// whose parts are joined through LDS.  A (row, head) that several workgroups
// share is joined through the workspace by the last one to arrive, in the order
// of the workgroups.
#include "hg_attn.h"
#include "hg_device.h"

namespace hg {
namespace {

constexpr int kWaves = 8;
constexpr int kThreadsDecode = kWaves * 64;
constexpr int kChunk = 32;                   // tokens of a wavefront's step
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kNegInf = -__builtin_inff();

// exp2(a - m) with m = -inf (nothing seen) giving 0.
__device__ __forceinline__ float weight(float a, float m) {
  return __builtin_amdgcn_exp2f(a - (m == kNegInf ? 0.0f : m));
}

// Chunks of batch row b, at least one so that an empty row is answered.
__device__ __forceinline__ void row_span(const DecodeParams& p, int b, int& first, int& len) {
  len = clamp_to(p.lens[b], p.cache.max_tokens);
  first = p.starts ? min(clamp_to(p.starts[b], p.cache.max_tokens), len) : 0;
}
__device__ __forceinline__ int64_t row_chunks(const DecodeParams& p, int b) {
  int first, len;
  row_span(p, b, first, len);
  return max((len - first + kChunk - 1) / kChunk, 1);
}

// The state of one wavefront over its chunks of one (row, head, row tile).
template <int D>
struct Part {
  static constexpr int S = D / 32;   // 32-channel steps of the first product
  static constexpr int J = D / 16;   // 16-channel results of the second
  f32x4 acc[J];
  float m, l;
};

// Row offsets of 32 tokens from t0 (lane i and i + 32: token t0 + i), and which are attended.
__device__ __forceinline__ int chunk_page(const DecodeParams& p, int b, int t0, int len, int64_t& off_in_page) {
  const int t = t0 + (threadIdx.x & 31);
  int page = -1;
  off_in_page = 0;
  if (t < len) {
    const uint32_t pg = divide((uint32_t)t, p.cache);
    page = p.cache.table[(int64_t)b * p.cache.max_pages + pg];
    off_in_page = ((uint32_t)t - pg * (uint32_t)p.cache.page_size) * p.cache.token_stride;
  }
  return page;
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
  q32x4 k[2][S];
  uint32_t v[8][VP][VW];
};

template <int D>
__device__ __forceinline__ void load_keys(Loads<D>& x, const uint16_t* K, int64_t off) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int tile = 0; tile < 2; ++tile) {
    const uint16_t* row = K + shfl64(off, tile * 16 + (lane & 15)) + (lane >> 4) * 8;
#pragma unroll
    for (int s = 0; s < Loads<D>::S; ++s) x.k[tile][s] = *(const q32x4*)(row + s * 32);
  }
}

template <int D>
__device__ __forceinline__ void load_values(Loads<D>& x, const uint16_t* V, int64_t off) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint16_t* row = V + shfl64(off, (i & 4) * 4 + g * 4 + (i & 3));
#pragma unroll
    for (int c = 0; c < Loads<D>::VP; ++c) {
      if constexpr (D >= 128) {
        const q32x4 y = *(const q32x4*)(row + c * 128 + r * 8);
#pragma unroll
        for (int w = 0; w < 4; ++w) x.v[i][c][w] = y[w];
      } else {
        const q32x2 y = *(const q32x2*)(row + r * 4);
        x.v[i][c][0] = y[0];
        x.v[i][c][1] = y[1];
      }
    }
  }
}

template <int D>
__global__ __launch_bounds__(kThreadsDecode) void decode_kernel(const DecodeParams p) {
  constexpr int S = D / 32, J = D / 16;
  constexpr int VP = Loads<D>::VP, VW = Loads<D>::VW;
  extern __shared__ float lds[];  // [kWaves][rows][D + 4] parts, then their m and l
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int per_row = p.cache.H * p.row_tiles;  // (head, row tile) pairs of a batch row

  // this workgroup's run [u0, u1) of the list of chunks
  int64_t total = 0;
  for (int b0 = 0; b0 < p.cache.B; b0 += 64) {
    int64_t n = b0 + lane < p.cache.B ? row_chunks(p, b0 + lane) : 0;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) n += shfl64(n, lane ^ o);
    total += n;
  }
  total *= per_row;
  int64_t per = (total + gridDim.x - 1) / gridDim.x;
  per = per < kWaves ? kWaves : per;  // one chunk per wavefront at least
  const int64_t u0 = blockIdx.x * per;
  const int64_t u1 = u0 + per < total ? u0 + per : total;
  if (u0 >= u1) return;

  // the batch row that holds u0, and the chunks before it
  int b = 0;
  int64_t before = 0;
  for (int b0 = 0; b0 < p.cache.B; b0 += 64) {
    const int64_t n = b0 + lane < p.cache.B ? row_chunks(p, b0 + lane) * per_row : 0;
    int64_t sum = n;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int64_t y = shfl64(sum, lane >= o ? lane - o : lane);
      sum += lane >= o ? y : 0;
    }
    const int past = __popcll(__ballot(b0 + lane < p.cache.B && before + sum <= u0));
    if (past < 64) {
      const int64_t add = shfl64(sum, past > 0 ? past - 1 : 0);
      b = b0 + past;
      before += past > 0 ? add : 0;
      break;
    }
    before += shfl64(sum, 63);
  }
  b = __builtin_amdgcn_readfirstlane(b);

  int64_t u = u0;
  while (u < u1) {  // one (row, head, row tile) a turn
    int first, len;
    row_span(p, b, first, len);
    first = __builtin_amdgcn_readfirstlane(first);
    len = __builtin_amdgcn_readfirstlane(len);
    const int64_t chunks = max((len - first + kChunk - 1) / kChunk, 1);
    const int pair = (int)((u - before) / chunks);
    const int64_t start = before + pair * chunks, end = start + chunks;
    const int h = pair / p.row_tiles, tile0 = (pair % p.row_tiles) * kDecodeRows;
    const int rows = min(p.R - tile0, kDecodeRows);
    const int64_t stop = end < u1 ? end : u1;
    const int c0 = (int)(u - start), c1 = (int)(stop - start);

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

    Loads<D> x;
    for (int c = c0 + wave; c < c1; c += kWaves) {
      int64_t off;
      const int page = chunk_page(p, b, first + c * kChunk, len, off);
      const bool in = page >= 0 && page < p.cache.num_pages;
      off = in ? off + page * p.cache.page_stride : 0;
      const uint32_t seen = (uint32_t)__ballot(in);
      if (seen == 0) continue;  // (row 0 of page 0 stands in for tokens not attended)
      load_keys<D>(x, K, off);
      load_values<D>(x, V, off);

      f32x4 st[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        st[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < S; ++s)
          st[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x.k[t][s]),
                                                          __builtin_bit_cast(bf16x8, q[s]), st[t], 0, 0, 0);
      }
      float sc[8];
      float top = kNegInf;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
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
      q32x4 w;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float p0 = weight(sc[i], m), p1 = weight(sc[i + 1], m);
        a.l += p0 + p1;
        w[i >> 1] = cvt_bf16x2(p0, p1);
      }
      if (seen != 0xFFFFFFFFu) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!((seen >> ((i & 4) * 4 + g * 4 + (i & 3))) & 1u))
#pragma unroll
            for (int cc = 0; cc < VP; ++cc)
#pragma unroll
              for (int e = 0; e < VW; ++e) x.v[i][cc][e] = 0;
      }
#pragma unroll
      for (int cc = 0; cc < VP; ++cc)
#pragma unroll
        for (int e = 0; e < 2 * VW; ++e) {
          q32x4 y;  // channel e of the lane's piece, its 8 tokens
#pragma unroll
          for (int i = 0; i < 4; ++i)
            y[i] = __builtin_amdgcn_perm(x.v[2 * i + 1][cc][e >> 1], x.v[2 * i][cc][e >> 1],
                                         (e & 1) ? 0x07060302u : 0x05040100u);
          const int j = cc * 2 * VW + e;
          a.acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, y),
                                                             __builtin_bit_cast(bf16x8, w), a.acc[j], 0, 0, 0);
        }
    }
    a.l += __shfl_xor(a.l, 16);
    a.l += __shfl_xor(a.l, 32);

    // join the wavefronts
    const int pitch = D + 4;
    float* part = lds;                                 // [kWaves][rows][pitch]
    float* stat = lds + (size_t)kWaves * rows * pitch;  // [kWaves][2][rows]
    if (g == 0 && r < rows) {
      stat[(wave * 2) * rows + r] = a.m;
      stat[(wave * 2 + 1) * rows + r] = a.l;
    }
    __syncthreads();
    if (r < rows) {
      float m = kNegInf;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, stat[(w * 2) * rows + r]);
      const float f = weight(a.m, m);
      float* row = part + ((size_t)wave * rows + r) * pitch;
#pragma unroll
      for (int cc = 0; cc < VP; ++cc)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 2 * VW; ++e)
            row[cc * 128 + (g * 4 + i) * 2 * VW + e] = a.acc[cc * 2 * VW + e][i] * f;
    }
    __syncthreads();
    const bool whole = u == start && stop == end;
    const int64_t w0 = start / per, w1 = (end - 1) / per;  // workgroups that share it
    // partial results: slot 0 for one begun by an earlier workgroup, 1 for one that goes on in the next
    const int stride = decode_partial_floats(min(p.R, kDecodeRows), D);
    float* mine = p.partial + (size_t)(blockIdx.x * 2 + (u == start ? 1 : 0)) * stride;
    for (int i = threadIdx.x; i < rows * (D / 4); i += kThreadsDecode) {
      const int row = i / (D / 4), c4 = (i % (D / 4)) * 4;
      f32x4 o = {0, 0, 0, 0};
      float m = kNegInf, l = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, stat[(w * 2) * rows + row]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        o += *(const f32x4*)(part + ((size_t)w * rows + row) * pitch + c4);
        l += stat[(w * 2 + 1) * rows + row] * weight(stat[(w * 2) * rows + row], m);
      }
      if (whole) {
        const int hq = h * p.R + tile0 + row;
        const float inv = l > 0 ? 1.0f / l : (l == 0 ? 0.0f : l);
        *(q32x2*)(p.out.data + b * p.out.token_stride + hq * p.out.head_stride + c4) =
            q32x2{cvt_bf16x2(o[0] * inv, o[1] * inv), cvt_bf16x2(o[2] * inv, o[3] * inv)};
        if (p.lse && c4 == 0)
          p.lse[(int64_t)b * p.cache.H * p.R + hq] = l == 0 ? kNegInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
      } else {
        if (c4 == 0) {
          mine[row] = m;
          mine[rows + row] = l;
        }
        *(f32x4*)(mine + 2 * rows + row * D + c4) = o;
      }
    }
    if (!whole) {
      __threadfence();
      __syncthreads();
      uint32_t* counter = p.counters + ((int64_t)b * per_row + pair);
      uint32_t* last = (uint32_t*)lds;
      if (threadIdx.x == 0) {
        const uint32_t n = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        *last = n == (uint32_t)(w1 - w0);
        if (*last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
      const bool join = *last != 0;
      __syncthreads();
      if (join) {
        __threadfence();
        for (int i = threadIdx.x; i < rows * (D / 4); i += kThreadsDecode) {
          const int row = i / (D / 4), c4 = (i % (D / 4)) * 4;
          float m = kNegInf;
          for (int64_t w = w0; w <= w1; ++w)
            m = fmaxf(m, p.partial[(size_t)(w * 2 + (w == w0 ? 1 : 0)) * stride + row]);
          f32x4 o = {0, 0, 0, 0};
          float l = 0;
          for (int64_t w = w0; w <= w1; ++w) {
            const float* q2 = p.partial + (size_t)(w * 2 + (w == w0 ? 1 : 0)) * stride;
            const float f = weight(q2[row], m);
            l += q2[rows + row] * f;
            o += *(const f32x4*)(q2 + 2 * rows + row * D + c4) * f;
          }
          const int hq = h * p.R + tile0 + row;
          const float inv = l > 0 ? 1.0f / l : (l == 0 ? 0.0f : l);
          *(q32x2*)(p.out.data + b * p.out.token_stride + hq * p.out.head_stride + c4) =
              q32x2{cvt_bf16x2(o[0] * inv, o[1] * inv), cvt_bf16x2(o[2] * inv, o[3] * inv)};
          if (p.lse && c4 == 0)
            p.lse[(int64_t)b * p.cache.H * p.R + hq] = l == 0 ? kNegInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
        }
      }
    }
    __syncthreads();  // the parts in LDS are free again
    u = stop;
    if (u == before + chunks * per_row) {
      before = u;
      ++b;
    }
  }
}

template <int D>
hipError_t launch(const DecodeParams& p, hipStream_t stream) {
  const int rows = p.R < kDecodeRows ? p.R : kDecodeRows;
  const size_t bytes = sizeof(float) * kWaves * rows * (D + 4 + 2);
  if (bytes > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)decode_kernel<D>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)bytes);
    if (e != hipSuccess) return e;
  }
  decode_kernel<D><<<dim3(kDecodeGroups), dim3(kThreadsDecode), bytes, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_decode(const DecodeParams& p, int D, hipStream_t stream) {
  return D == 64 ? launch<64>(p, stream) : D == 128 ? launch<128>(p, stream) : launch<256>(p, stream);
}

}  // namespace hg
