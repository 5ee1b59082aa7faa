// Appending new tokens to the paged cache, keys and queries rotated.
//
// Per token: q' = R(p) q, k' = R(p) k in fp32 with one rounding, k' and v to
// the token's place in its page.  The call moves N (Hq + 2H) D * 2 bytes in and
// out and computes 3 operations an element, so memory bounds it, and a call of
// few tokens the chain row -> length -> page -> store.  A unit is 16 channels
// of a row: two 16-byte pieces whose channels pair up (halves of the rotated
// channels, or 16 neighbours interleaved), so a pair never leaves its thread
// and in-place calls are safe.  A thread keeps its channels and walks over the
// rows (heads) of its token, so the table is read once per token and thread.
// Measured: one token 3.4 us and 64 tokens (64 and 8 heads) 4.1 us in a graph; a
// large call moves 5.3 TB/s, the rate of a large copy (5.0).
#include "hg_attn.h"
#include "hg_device.h"

namespace hg {
namespace {

constexpr int kAppendThreads = 256;

// Once: streaming (non-temporal) loads and stores, see launch.
template <bool Once>
__device__ __forceinline__ u32x4 load_piece(const uint16_t* p) {
  if constexpr (Once) return __builtin_nontemporal_load((const u32x4*)p);
  else return *(const u32x4*)p;
}
template <bool Once>
__device__ __forceinline__ void store_piece(uint16_t* p, u32x4 x) {
  if constexpr (Once) __builtin_nontemporal_store(x, (u32x4*)p);
  else *(u32x4*)p = x;
}

template <int D, bool Once>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(const AppendParams p, int row_slots) {
  constexpr int C = D / 16;              // units per row
  const int unit = threadIdx.x % C;
  const int slot = threadIdx.x / C;
  // row_slots is a power of two, at least 64 / C: a wavefront has one token
  const int tokens = kAppendThreads / C / row_slots;
  const int token = __builtin_amdgcn_readfirstlane((int)blockIdx.x * tokens + slot / row_slots);
  if (token >= p.N) return;

  // place in the cache
  int b = token, n = 1, j = 0;
  if (p.cu) {
    b = find_row(p.cu, p.cache.B, token);
    if (b >= p.cache.B) return;
    const int lo = p.cu[b];
    n = p.cu[b + 1] - lo;
    j = token - lo;
    if (j < 0) return;
  }
  const int64_t at = (int64_t)p.lens[b] - n + j;
  bool stored = at >= 0 && at < p.cache.max_tokens;
  int64_t place = 0;
  if (stored) {
    const uint32_t pg = divide((uint32_t)at, p.cache);
    const int page = p.cache.table[(int64_t)b * p.cache.max_pages + pg];
    stored = page >= 0 && page < p.cache.num_pages;
    place = page * p.cache.page_stride + ((uint32_t)at - pg * (uint32_t)p.cache.page_size) * p.cache.token_stride;
  }

  // the two pieces of this thread's units, and their pairs
  const bool rotated = unit * 16 < p.rot;
  int c0, c1, pair;
  if (rotated && !p.interleaved) {
    c0 = unit * 8;
    c1 = c0 + p.half;
    pair = unit * 8;
  } else {
    c0 = unit * 16;
    c1 = c0 + 8;
    pair = unit * 8;
  }
  float cs[8], sn[8];
  if (p.rot > 0) {
    int pos[3];
    bool inside = true;
    for (int a = 0; a < p.axes; ++a) {
      const int64_t v = p.positions ? (int64_t)p.positions[(int64_t)a * p.N + token] : at;
      inside = inside && v >= 0 && v < p.max_pos;
      pos[a] = (int)v;
    }
    if (!inside) return;
    if (p.axes == 1) pos[1] = pos[2] = pos[0];
    if (rotated) {
      const int a0 = pair < p.sec0 ? 0 : pair < p.sec1 ? 1 : 2;
      const int a7 = pair + 7 < p.sec0 ? 0 : pair + 7 < p.sec1 ? 1 : 2;
      if (a0 == a7) {
        const int64_t o = (int64_t)(a0 == 0 ? pos[0] : a0 == 1 ? pos[1] : pos[2]) * p.half + pair;
        const f32x4* c = (const f32x4*)(p.cos + o);
        const f32x4* s = (const f32x4*)(p.sin + o);
        const f32x4 ca = c[0], cb = c[1], sa = s[0], sb = s[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          cs[e] = ca[e];
          cs[e + 4] = cb[e];
          sn[e] = sa[e];
          sn[e + 4] = sb[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int i = pair + e;
          const int64_t o = (int64_t)(i < p.sec0 ? pos[0] : i < p.sec1 ? pos[1] : pos[2]) * p.half + i;
          cs[e] = p.cos[o];
          sn[e] = p.sin[o];
        }
      }
    }
  }

  const int rows = p.Hq + 2 * p.cache.H;
  for (int r = slot % row_slots; r < rows; r += row_slots) {
    const bool is_q = r < p.Hq;
    const bool is_k = !is_q && r < p.Hq + p.cache.H;
    const int h = is_q ? r : is_k ? r - p.Hq : r - p.Hq - p.cache.H;
    const uint16_t* base = is_q ? p.q.data : is_k ? p.k.data : p.v.data;
    const int64_t ts = is_q ? p.q.token_stride : is_k ? p.k.token_stride : p.v.token_stride;
    const int64_t hs = is_q ? p.q.head_stride : is_k ? p.k.head_stride : p.v.head_stride;
    const uint16_t* src = base + token * ts + h * hs;
    u32x4 x = load_piece<Once>(src + c0);
    u32x4 y = load_piece<Once>(src + c1);
    if (rotated && (is_q || is_k)) {
      if (!p.interleaved) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float a0 = bf16_lo(x[w]), a1 = bf16_hi(x[w]), b0 = bf16_lo(y[w]), b1 = bf16_hi(y[w]);
          const float c = cs[2 * w], s = sn[2 * w], d = cs[2 * w + 1], t = sn[2 * w + 1];
          x[w] = cvt_bf16x2(__builtin_fmaf(a0, c, -(b0 * s)), __builtin_fmaf(a1, d, -(b1 * t)));
          y[w] = cvt_bf16x2(__builtin_fmaf(b0, c, a0 * s), __builtin_fmaf(b1, d, a1 * t));
        }
      } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float a0 = bf16_lo(x[w]), b0 = bf16_hi(x[w]), a1 = bf16_lo(y[w]), b1 = bf16_hi(y[w]);
          const float c = cs[w], s = sn[w], d = cs[w + 4], t = sn[w + 4];
          x[w] = cvt_bf16x2(__builtin_fmaf(a0, c, -(b0 * s)), __builtin_fmaf(b0, c, a0 * s));
          y[w] = cvt_bf16x2(__builtin_fmaf(a1, d, -(b1 * t)), __builtin_fmaf(b1, d, a1 * t));
        }
      }
    }
    if (is_q) {
      uint16_t* o = p.q_out.data + token * p.q_out.token_stride + h * p.q_out.head_stride;
      store_piece<Once>(o + c0, x);
      store_piece<Once>(o + c1, y);
      continue;
    }
    if (is_k && p.k_out.data) {
      uint16_t* o = p.k_out.data + token * p.k_out.token_stride + h * p.k_out.head_stride;
      store_piece<Once>(o + c0, x);
      store_piece<Once>(o + c1, y);
    }
    if (stored) {
      uint16_t* o = (is_k ? p.cache.K : p.cache.V) + place + h * p.cache.head_stride;
      store_piece<Once>(o + c0, x);
      store_piece<Once>(o + c1, y);
    }
  }
}

// Rows that a workgroup's threads take of a token at once, and its tokens.
int row_slots_of(const AppendParams& p, int D) {
  const int C = D / 16, rows = p.Hq + 2 * p.cache.H;
  int row_slots = 64 / C;
  while (row_slots < rows && row_slots < kAppendThreads / C) row_slots *= 2;
  return row_slots;
}
int64_t workgroups(const AppendParams& p, int D) {
  const int tokens = kAppendThreads / (D / 16) / row_slots_of(p, D);
  return ((int64_t)p.N + tokens - 1) / tokens;
}

template <int D>
hipError_t launch(const AppendParams& p, hipStream_t stream) {
  const int row_slots = row_slots_of(p, D);
  // Calls that outgrow the 256 MiB last-level cache stream (four prompts of up to
  // 3008 tokens, 32 heads, 296 MB: 60.4 -> 55.5 us, 5.3 TB/s); what smaller ones
  // write is read from the caches by the attention that follows.
  const dim3 grid((uint32_t)workgroups(p, D));
  const double bytes = 4.0 * D * p.N * (p.Hq + (p.k_out.data ? 2.5 : 2.0) * p.cache.H);
  if (bytes > (double)(256 << 20)) append_kernel<D, true><<<grid, dim3(kAppendThreads), 0, stream>>>(p, row_slots);
  else append_kernel<D, false><<<grid, dim3(kAppendThreads), 0, stream>>>(p, row_slots);
  return hipGetLastError();
}

}  // namespace

int64_t append_work_items(const AppendParams& p, int D) { return workgroups(p, D) * kAppendThreads; }

hipError_t launch_append(const AppendParams& p, int D, hipStream_t stream) {
  return D == 64 ? launch<64>(p, stream) : D == 128 ? launch<128>(p, stream) : launch<256>(p, stream);
}

}  // namespace hg
