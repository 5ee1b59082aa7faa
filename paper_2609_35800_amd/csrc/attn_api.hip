// Host side of the attention calls: argument checks and launch.  The contract
// of every entry point is in include/headguard.h.

#include <math.h>
#include <string.h>

#include <algorithm>

#include "headguard.h"
#include "hg_attn.h"
#include "hg_host.h"

namespace {

using namespace hg;

constexpr double kLog2e = 1.4426950408889634;

// A strided BF16 operand: runs of `inner` elements at sums of index * stride.
struct View {
  const char* name;
  const uint16_t* data;
  int64_t inner;
  int64_t n[3], stride[3];
  int dims;
  bool empty() const {
    for (int i = 0; i < dims; ++i)
      if (n[i] <= 0) return true;
    return false;
  }
  // elements from the first to past the last
  __int128 extent() const {
    __int128 e = inner;
    for (int i = 0; i < dims; ++i) e += (__int128)(n[i] - 1) * stride[i];
    return e;
  }
  // dimensions by descending stride, those of one index left out
  View sorted() const {
    View v = *this;
    v.dims = 0;
    for (int i = 0; i < dims; ++i)
      if (n[i] != 1) {
        int k = v.dims++;
        for (; k > 0 && v.stride[k - 1] < stride[i]; --k) {
          v.n[k] = v.n[k - 1];
          v.stride[k] = v.stride[k - 1];
        }
        v.n[k] = n[i];
        v.stride[k] = stride[i];
      }
    return v;
  }
};

View rows_view(const char* name, const hg_rows& r, int64_t n, int64_t heads, int64_t D) {
  return View{name, r.data, D, {n, heads, 0}, {r.token_stride, r.head_stride, 0}, 2};
}
View pages_view(const char* name, const uint16_t* data, const hg_paged_cache& c) {
  return View{name, data, c.D, {c.num_pages, c.H, c.page_size}, {c.page_stride, c.head_stride, c.token_stride}, 3};
}

// Pointer, alignment and stride checks of one operand; a written one's rows
// must not overlap.
int check_view(const View& v, bool written) {
  if (v.empty()) return HG_OK;
  if (!v.data) return fail(HG_ERR_NULL, "%s is NULL", v.name);
  if (!aligned(v.data, 16)) return fail(HG_ERR_ALIGN, "%s is not 16-byte aligned", v.name);
  for (int i = 0; i < v.dims; ++i) {
    if (v.stride[i] < 0) return fail(HG_ERR_SHAPE, "%s has a negative stride", v.name);
    if (v.stride[i] % 8) return fail(HG_ERR_ALIGN, "%s has a stride of %lld, not a multiple of 8 elements", v.name,
                                     (long long)v.stride[i]);
  }
  if (v.extent() > ((__int128)1 << 60)) return fail(HG_ERR_SHAPE, "%s is too large", v.name);
  if (written) {
    const View s = v.sorted();
    int64_t inner = s.inner;
    for (int i = s.dims - 1; i >= 0; --i) {
      if (s.stride[i] < inner) return fail(HG_ERR_SHAPE, "rows of %s overlap one another", v.name);
      inner = (s.n[i] - 1) * s.stride[i] + inner;
    }
  }
  return HG_OK;
}

bool same_view(const View& a, const View& b) {
  const View x = a.sorted(), y = b.sorted();
  if (a.data != b.data || x.dims != y.dims) return false;
  for (int i = 0; i < x.dims; ++i)
    if (x.n[i] != y.n[i] || x.stride[i] != y.stride[i]) return false;
  return true;
}

// Whether elements i of a (at 0) and j of b (at delta) can be the same one,
// strides of dimensions d and up: delta = sum (i - j) stride + (less than a run).
bool meet(int64_t delta, const View& a, const View& b, int d) {
  if (d == a.dims) return delta < a.inner && -delta < b.inner;
  int64_t ea = a.inner, eb = b.inner;  // extents of the inner dimensions
  for (int i = d + 1; i < a.dims; ++i) {
    ea += (a.n[i] - 1) * a.stride[i];
    eb += (b.n[i] - 1) * b.stride[i];
  }
  // -eb < delta - x stride < ea
  const int64_t s = a.stride[d];
  if (s == 0) return true;
  auto floor_div = [](int64_t x, int64_t y) { return x / y - (x % y < 0); };
  const int64_t lo = std::max(floor_div(delta - ea, s), -(b.n[d] - 1));
  const int64_t hi = std::min(floor_div(delta + eb, s) + 1, a.n[d] - 1);
  if (hi - lo > 8) return true;  // not the strides of nested dimensions
  for (int64_t x = lo; x <= hi; ++x)
    if (meet(delta - x * s, a, b, d + 1)) return true;
  return false;
}

// Whether two operands may share an element: exact where their strides agree
// (views of one tensor), by their address ranges otherwise.
bool overlap(const View& a, const View& b) {
  if (a.empty() || b.empty()) return false;
  const int64_t delta = ((int64_t)(uintptr_t)b.data - (int64_t)(uintptr_t)a.data) / 2;
  if (delta >= (int64_t)a.extent() || -delta >= (int64_t)b.extent()) return false;
  if (a.dims != b.dims) return true;
  View x = a, y = b;  // by descending stride of either
  for (int i = 0; i < x.dims; ++i) {
    // a dimension of one index takes the other's stride
    if (x.n[i] == 1) x.stride[i] = y.stride[i];
    if (y.n[i] == 1) y.stride[i] = x.stride[i];
    if (x.stride[i] != y.stride[i]) return true;
  }
  for (int i = 0; i < x.dims; ++i)
    for (int k = i + 1; k < x.dims; ++k)
      if (x.stride[k] > x.stride[i]) {
        std::swap(x.stride[k], x.stride[i]);
        std::swap(x.n[k], x.n[i]);
        std::swap(y.stride[k], y.stride[i]);
        std::swap(y.n[k], y.n[i]);
      }
  return meet(delta, x, y, 0);
}

bool overlap(const View& a, const void* p, uint64_t bytes) {
  if (a.empty() || !p || bytes == 0) return false;
  const uintptr_t lo = (uintptr_t)a.data, hi = lo + (uintptr_t)a.extent() * 2;
  return (uintptr_t)p < hi && lo < (uintptr_t)p + bytes;
}

int check_head_dim(int D) {
  if (D != 64 && D != 128 && D != 256) return fail(HG_ERR_HEADDIM, "head_dim %d not in {64, 128, 256}", D);
  return HG_OK;
}

int check_scale(float scale) {
  if (!isfinite(scale) || !isfinite((float)(scale * kLog2e))) return fail(HG_ERR_VALUE, "scale is not finite");
  return HG_OK;
}

int check_array(const void* p, const char* name) {
  if (!p) return fail(HG_ERR_NULL, "%s is NULL", name);
  if (!aligned(p, 4)) return fail(HG_ERR_ALIGN, "%s is not 4-byte aligned", name);
  return HG_OK;
}

// Sizes of a paged cache (its pointers are checked with the operands).
int check_cache(const hg_paged_cache* c) {
  if (!c) return fail(HG_ERR_NULL, "cache is NULL");
  if (c->B < 0 || c->H <= 0 || c->page_size <= 0 || c->num_pages < 0 || c->max_pages < 0)
    return fail(HG_ERR_SHAPE, "cache sizes B, H, page_size, num_pages, max_pages = %d, %d, %d, %d, %d", c->B, c->H,
                c->page_size, c->num_pages, c->max_pages);
  int s = check_head_dim(c->D);
  if (s) return s;
  if (c->B > 0 && c->max_pages > 0) s = check_array(c->block_table, "block_table");
  return s;
}

PagedCache fill_cache(const hg_paged_cache* c) {
  PagedCache p;
  memset(&p, 0, sizeof p);
  p.K = c->K;
  p.V = c->V;
  p.table = c->block_table;
  p.page_stride = c->page_stride;
  p.head_stride = c->head_stride;
  p.token_stride = c->token_stride;
  p.B = c->B;
  p.H = c->H;
  p.page_size = c->page_size;
  p.num_pages = c->num_pages;
  p.max_pages = c->num_pages > 0 ? c->max_pages : 0;
  p.max_tokens = (int32_t)std::min<int64_t>((int64_t)p.max_pages * p.page_size, 0x7FFFFFFF);
  // t / d for t < 2^31: with k = floor(log2 d) and M = ceil(2^(32+k) / d), M d
  // exceeds 2^(32+k) by less than d < 2^(k+1), so t M / 2^(32+k) exceeds t / d by
  // less than 1 / d.
  const uint32_t d = (uint32_t)c->page_size;
  const int k = 31 - __builtin_clz(d);
  p.div_shift = (uint32_t)k;
  p.div_mul = (d & (d - 1)) == 0 ? 0u : (uint32_t)((((uint64_t)1 << (32 + k)) + d - 1) / d);
  return p;
}

// NULL, alignment and overlap of all operands, then the device and the
// pointers.  The `written` operands come first; operand i of them may be
// operand in_place[i] itself.
int check_operands(const View* views, int nv, int written, const Buf* arrays, int na, const int* in_place) {
  for (int i = 0; i < nv; ++i) {
    const int s = check_view(views[i], i < written);
    if (s) return s;
  }
  for (int i = 0; i < na; ++i) {
    if (arrays[i].bytes == 0) continue;
    if (!arrays[i].p) return fail(HG_ERR_NULL, "%s is NULL", arrays[i].name);
    if (!aligned(arrays[i].p, arrays[i].align))
      return fail(HG_ERR_ALIGN, "%s is not %u-byte aligned", arrays[i].name, (unsigned)arrays[i].align);
  }
  for (int i = 0; i < written; ++i) {
    for (int j = 0; j < nv; ++j) {
      if (j == i || (j < i && j < written)) continue;
      if (in_place && in_place[i] == j && same_view(views[i], views[j])) continue;
      if (overlap(views[i], views[j])) return fail(HG_ERR_POINTER, "%s overlaps %s", views[i].name, views[j].name);
    }
    for (int j = 0; j < na; ++j)
      if (overlap(views[i], arrays[j].p, arrays[j].bytes))
        return fail(HG_ERR_POINTER, "%s overlaps %s", views[i].name, arrays[j].name);
  }
  int s = check_device();
  if (s) return s;
  for (int i = 0; i < nv; ++i)
    if (!views[i].empty()) {
      s = check_device_ptr(views[i].data, views[i].name);
      if (s) return s;
    }
  return check_buffers(arrays, na);
}

// lse and workspace are written arrays: disjoint from every other operand.
int check_written_array(const Buf& w, const View* views, int nv, const Buf* arrays, int na) {
  if (!w.p || w.bytes == 0) return HG_OK;
  for (int i = 0; i < nv; ++i)
    if (overlap(views[i], w.p, w.bytes)) return fail(HG_ERR_POINTER, "%s overlaps %s", w.name, views[i].name);
  for (int i = 0; i < na; ++i) {
    if (arrays[i].p == w.p && arrays[i].name == w.name) continue;
    const uintptr_t a = (uintptr_t)w.p, b = (uintptr_t)arrays[i].p;
    if (arrays[i].bytes && b && a < b + arrays[i].bytes && b < a + w.bytes)
      return fail(HG_ERR_POINTER, "%s overlaps %s", w.name, arrays[i].name);
  }
  return HG_OK;
}

int row_tiles(int R) { return (R + kDecodeRows - 1) / kDecodeRows; }

// Bytes of the workspace that a decode call uses.
uint64_t decode_bytes(int R, int D) {
  return kDecodeCounterBytes + 2 * (uint64_t)kDecodeSlots * decode_partial_floats(std::min(R, kDecodeRows), D) * 4;
}

int check_groups(int Hq, int H) {
  if (Hq <= 0 || Hq % H) return fail(HG_ERR_SHAPE, "%d query heads are not a multiple of %d key/value heads", Hq, H);
  return HG_OK;
}

}  // namespace

extern "C" {

int hg_append_kv(const hg_paged_cache* cache, const hg_rotation* rot, const hg_append* a, hipStream_t stream) {
  int s = check_cache(cache);
  if (s) return s;
  if (!a) return fail(HG_ERR_NULL, "args is NULL");
  if (a->N < 0 || a->Hq < 0) return fail(HG_ERR_SHAPE, "N, Hq = %d, %d", a->N, a->Hq);
  if (!a->cu_new && a->N != cache->B)
    return fail(HG_ERR_SHAPE, "%d tokens for %d rows without cu_new", a->N, cache->B);
  AppendParams p;
  memset(&p, 0, sizeof p);
  if (rot && rot->rot_dim != 0) {
    if (rot->rot_dim < 0 || rot->rot_dim > cache->D || rot->rot_dim % 16)
      return fail(HG_ERR_SHAPE, "rot_dim %d is not a multiple of 16 within %d", rot->rot_dim, cache->D);
    if (rot->max_pos <= 0) return fail(HG_ERR_SHAPE, "max_pos %d", rot->max_pos);
    if (rot->interleaved != 0 && rot->interleaved != 1) return fail(HG_ERR_SHAPE, "interleaved must be 0 or 1");
    p.rot = rot->rot_dim;
    p.half = rot->rot_dim / 2;
    p.max_pos = rot->max_pos;
    p.interleaved = rot->interleaved;
    p.cos = rot->cos;
    p.sin = rot->sin;
    const int32_t* sec = rot->sections;
    p.axes = sec[0] || sec[1] || sec[2] ? 3 : 1;
    if (p.axes == 3) {
      if (sec[0] < 0 || sec[1] < 0 || sec[2] < 0 || (int64_t)sec[0] + sec[1] + sec[2] != p.half)
        return fail(HG_ERR_SHAPE, "sections %d, %d, %d do not add up to %d pairs", sec[0], sec[1], sec[2], p.half);
      if (!a->positions) return fail(HG_ERR_NULL, "sections need positions");
    }
    p.sec0 = p.axes == 3 ? sec[0] : p.half;
    p.sec1 = p.axes == 3 ? sec[0] + sec[1] : p.half;
    p.positions = a->positions;
  }
  if (a->N == 0 || cache->B == 0) return ok();
  if ((int64_t)a->Hq + 2 * (int64_t)cache->H > 0x7FFFFFFF - 1024)
    return fail(HG_ERR_SHAPE, "%d query and %d key/value heads", a->Hq, cache->H);
  p.cache = fill_cache(cache);
  p.N = a->N;
  p.Hq = a->Hq;
  if (append_work_items(p, cache->D) > kMaxWorkItems)
    return fail(HG_ERR_SHAPE, "grid too large for %d tokens of %d query and %d key/value heads", a->N, a->Hq, cache->H);
  const uint64_t table_bytes = (uint64_t)p.half * p.max_pos * 4;
  const int D = cache->D;
  const View views[] = {
      pages_view("K", cache->K, *cache),
      pages_view("V", cache->V, *cache),
      rows_view("q_out", a->q_out, a->N, a->Hq, D),
      rows_view("k_out", a->k_out, a->k_out.data ? a->N : 0, cache->H, D),
      rows_view("q", a->q, a->N, a->Hq, D),
      rows_view("k", a->k, a->N, cache->H, D),
      rows_view("v", a->v, a->N, cache->H, D),
  };
  const Buf arrays[] = {
      {a->lens, (uint64_t)cache->B * 4, 4, "lens"},
      {a->cu_new, a->cu_new ? ((uint64_t)cache->B + 1) * 4 : 0, 4, "cu_new"},
      {p.positions, p.positions ? (uint64_t)p.axes * a->N * 4 : 0, 4, "positions"},
      {p.cos, table_bytes, 16, "cos"},
      {p.sin, table_bytes, 16, "sin"},
      {cache->block_table, (uint64_t)cache->B * cache->max_pages * 4, 4, "block_table"},
  };
  const int in_place[] = {-1, -1, 4, 5};
  s = check_operands(views, 7, 4, arrays, 6, in_place);
  if (s) return s;
  p.q = a->q;
  p.k = a->k;
  p.v = a->v;
  p.q_out = a->q_out;
  p.k_out = a->k_out;
  p.lens = a->lens;
  p.cu = a->cu_new;
  LaunchSteps step;
  const hipError_t e = step([&] { return launch_append(p, D, stream); });
  if (e != hipSuccess) return fail(HG_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
  return ok();
}

int hg_decode_workspace(const hg_paged_cache* cache, int32_t Hq, uint64_t* bytes) {
  int s = check_cache(cache);
  if (!s) s = check_groups(Hq, cache->H);
  if (s) return s;
  if (!bytes) return fail(HG_ERR_NULL, "bytes is NULL");
  const int R = Hq / cache->H;
  // a word per (row, head, row tile) is spare: the size is part of the interface
  const uint64_t spare = ((uint64_t)cache->B * cache->H * row_tiles(R) * 4 + 255) & ~(uint64_t)255;
  *bytes = decode_bytes(R, cache->D) + spare;
  return ok();
}

int hg_decode_attention(const hg_paged_cache* cache, const hg_decode* a, hipStream_t stream) {
  int s = check_cache(cache);
  if (s) return s;
  if (!a) return fail(HG_ERR_NULL, "args is NULL");
  s = check_groups(a->Hq, cache->H);
  if (!s) s = check_scale(a->scale);
  if (s) return s;
  if (cache->B == 0) return ok();
  const int D = cache->D, R = a->Hq / cache->H;
  const uint64_t need = decode_bytes(R, D);
  if (!a->workspace)
    return fail(HG_ERR_NULL, "workspace is NULL but the call needs %llu bytes", (unsigned long long)need);
  if (a->workspace_bytes < need)
    return fail(HG_ERR_SHAPE, "the call needs a %llu-byte workspace (%llu bytes available)", (unsigned long long)need,
                (unsigned long long)a->workspace_bytes);
  const View views[] = {
      rows_view("out", a->out, cache->B, a->Hq, D),
      rows_view("q", a->q, cache->B, a->Hq, D),
      pages_view("K", cache->K, *cache),
      pages_view("V", cache->V, *cache),
  };
  const Buf arrays[] = {
      {a->lens, (uint64_t)cache->B * 4, 4, "lens"},
      {a->starts, a->starts ? (uint64_t)cache->B * 4 : 0, 4, "starts"},
      {cache->block_table, (uint64_t)cache->B * cache->max_pages * 4, 4, "block_table"},
      {a->lse, a->lse ? (uint64_t)cache->B * a->Hq * 4 : 0, 4, "lse"},
      {a->workspace, need, 256, "workspace"},
  };
  for (int i = 3; i < 5 && !s; ++i) s = check_written_array(arrays[i], views, 4, arrays, 5);
  if (!s) s = check_operands(views, 4, 1, arrays, 5, nullptr);
  if (s) return s;
  DecodeParams p;
  memset(&p, 0, sizeof p);
  p.cache = fill_cache(cache);
  p.q = a->q;
  p.out = a->out;
  p.lse = a->lse;
  p.lens = a->lens;
  p.starts = a->starts;
  p.scale_log2 = (float)(a->scale * kLog2e);
  p.R = R;
  p.row_tiles = row_tiles(R);
  p.stream_chunks = decode_stream_chunks(p.cache, D, p.row_tiles);
  p.counters = (uint32_t*)a->workspace;
  p.partial = (float*)((char*)a->workspace + kDecodeCounterBytes);
  LaunchSteps step;
  const hipError_t e = step([&] { return launch_decode(p, D, stream); });
  if (e != hipSuccess) return fail(HG_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
  return ok();
}

int hg_prefill_attention(const hg_prefill* a, hipStream_t stream) {
  if (!a) return fail(HG_ERR_NULL, "args is NULL");
  if (a->B < 0 || a->H <= 0 || a->Nq < 0 || a->Nk < 0 || (a->causal != 0 && a->causal != 1))
    return fail(HG_ERR_SHAPE, "B, H, Nq, Nk, causal = %d, %d, %d, %d, %d", a->B, a->H, a->Nq, a->Nk, a->causal);
  int s = check_head_dim(a->D);
  if (!s) s = check_groups(a->Hq, a->H);
  if (!s) s = check_scale(a->scale);
  if (s) return s;
  if (!a->cu_k && a->Nk != a->Nq)
    return fail(HG_ERR_SHAPE, "%d keys for %d queries without cu_k", a->Nk, a->Nq);
  if (a->Nk > kMaxKeys) return fail(HG_ERR_SHAPE, "%d keys exceed %d", a->Nk, kMaxKeys);
  if (a->B == 0 || a->Nq == 0) return ok();
  PrefillParams p;
  memset(&p, 0, sizeof p);
  p.B = a->B;
  p.Hq = a->Hq;
  p.H = a->H;
  p.Nq = a->Nq;
  p.Nk = a->Nk;
  if (prefill_work_items(p, a->D) > kMaxWorkItems)
    return fail(HG_ERR_SHAPE, "grid too large for %d queries of %d heads", a->Nq, a->Hq);
  const int D = a->D;
  const View views[] = {
      rows_view("out", a->out, a->Nq, a->Hq, D),
      rows_view("q", a->q, a->Nq, a->Hq, D),
      rows_view("k", a->k, a->Nk, a->H, D),
      rows_view("v", a->v, a->Nk, a->H, D),
  };
  // a stage of keys or values is addressed with 32-bit byte offsets
  if (a->k.token_stride > kMaxKeyStride || a->v.token_stride > kMaxKeyStride)
    return fail(HG_ERR_SHAPE, "token strides of k, v = %lld, %lld exceed %lld", (long long)a->k.token_stride,
                (long long)a->v.token_stride, (long long)kMaxKeyStride);
  const Buf arrays[] = {
      {a->cu_q, ((uint64_t)a->B + 1) * 4, 4, "cu_q"},
      {a->cu_k, a->cu_k ? ((uint64_t)a->B + 1) * 4 : 0, 4, "cu_k"},
      {a->lse, a->lse ? (uint64_t)a->Nq * a->Hq * 4 : 0, 4, "lse"},
  };
  s = check_written_array(arrays[2], views, 4, arrays, 3);
  if (!s) s = check_operands(views, 4, 1, arrays, 3, nullptr);
  if (s) return s;
  p.q = a->q;
  p.k = a->k;
  p.v = a->v;
  p.out = a->out;
  p.lse = a->lse;
  p.cu_q = a->cu_q;
  p.cu_k = a->cu_k ? a->cu_k : a->cu_q;
  p.causal = a->causal;
  p.scale_log2 = (float)(a->scale * kLog2e);
  LaunchSteps step;
  const hipError_t e = step([&] { return launch_prefill(p, D, stream); });
  if (e != hipSuccess) return fail(HG_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
  return ok();
}

}  // extern "C"
