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
#include "hg_rotate.h"

namespace hg {
namespace {

constexpr int kAppendThreads = 256;

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

  const Unit un = unit_of(p, unit);
  const int c0 = un.c0, c1 = un.c1;
  Angles an;
  if (!load_angles(p, un, token, at, an)) return;

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
    if (un.rotated && (is_q || is_k)) rotate(x, y, an, p.interleaved);
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
