// Argument checks that the attention calls share: strided operands, their
// overlaps, arrays, and the sizes of a paged cache.
#pragma once

#include <math.h>
#include <string.h>

#include <algorithm>

#include "headguard.h"
#include "hg_attn.h"
#include "hg_host.h"

namespace hg {

constexpr double kLog2e = 1.4426950408889634;

// A strided operand of BF16 values or 8-bit codes: runs of `inner` elements at
// sums of index * stride.
struct View {
  const char* name;
  const void* data;
  int64_t inner;
  int64_t n[3], stride[3];
  int dims;
  int size = 2;  // bytes of an element
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

inline View rows_view(const char* name, const hg_rows& r, int64_t n, int64_t heads, int64_t D) {
  return View{name, r.data, D, {n, heads, 0}, {r.token_stride, r.head_stride, 0}, 2};
}
inline View pages_view(const char* name, const uint16_t* data, const hg_paged_cache& c) {
  return View{name, data, c.D, {c.num_pages, c.H, c.page_size}, {c.page_stride, c.head_stride, c.token_stride}, 3};
}

// Pointer, alignment and stride checks of one operand; a written one's rows
// must not overlap.
inline int check_view(const View& v, bool written) {
  if (v.empty()) return HG_OK;
  if (!v.data) return fail(HG_ERR_NULL, "%s is NULL", v.name);
  if (!aligned(v.data, 16)) return fail(HG_ERR_ALIGN, "%s is not 16-byte aligned", v.name);
  for (int i = 0; i < v.dims; ++i) {
    if (v.stride[i] < 0) return fail(HG_ERR_SHAPE, "%s has a negative stride", v.name);
    if (v.stride[i] % (16 / v.size)) return fail(HG_ERR_ALIGN, "%s has a stride of %lld, not a multiple of %d elements", v.name,
                                                 (long long)v.stride[i], 16 / v.size);
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

inline bool same_view(const View& a, const View& b) {
  const View x = a.sorted(), y = b.sorted();
  if (a.data != b.data || x.dims != y.dims) return false;
  for (int i = 0; i < x.dims; ++i)
    if (x.n[i] != y.n[i] || x.stride[i] != y.stride[i]) return false;
  return true;
}

// Whether elements i of a (at 0) and j of b (at delta) can be the same one,
// strides of dimensions d and up: delta = sum (i - j) stride + (less than a run).
inline bool meet(int64_t delta, const View& a, const View& b, int d) {
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
inline bool overlap(const View& a, const View& b) {
  if (a.empty() || b.empty()) return false;
  if (a.size != b.size) {
    const __int128 x = (uintptr_t)a.data, y = (uintptr_t)b.data;
    return x < y + b.extent() * b.size && y < x + a.extent() * a.size;
  }
  const int64_t delta = ((int64_t)(uintptr_t)b.data - (int64_t)(uintptr_t)a.data) / a.size;
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

inline bool overlap(const View& a, const void* p, uint64_t bytes) {
  if (a.empty() || !p || bytes == 0) return false;
  const uintptr_t lo = (uintptr_t)a.data, hi = lo + (uintptr_t)a.extent() * a.size;
  return (uintptr_t)p < hi && lo < (uintptr_t)p + bytes;
}

inline int check_head_dim(int D) {
  if (D != 64 && D != 128 && D != 256) return fail(HG_ERR_HEADDIM, "head_dim %d not in {64, 128, 256}", D);
  return HG_OK;
}

inline int check_scale(float scale) {
  if (!isfinite(scale) || !isfinite((float)(scale * kLog2e))) return fail(HG_ERR_VALUE, "scale is not finite");
  return HG_OK;
}

inline int check_array(const void* p, const char* name) {
  if (!p) return fail(HG_ERR_NULL, "%s is NULL", name);
  if (!aligned(p, 4)) return fail(HG_ERR_ALIGN, "%s is not 4-byte aligned", name);
  return HG_OK;
}

// The rotation of an append call, into its parameters.
inline int check_rotation(const hg_rotation* rot, const hg_append* a, int D, AppendParams& p) {
  if (rot && rot->rot_dim != 0) {
    if (rot->rot_dim < 0 || rot->rot_dim > D || rot->rot_dim % 16)
      return fail(HG_ERR_SHAPE, "rot_dim %d is not a multiple of 16 within %d", rot->rot_dim, D);
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
  return HG_OK;
}

// Sizes of a paged cache (its pointers are checked with the operands).
inline int check_cache(const hg_paged_cache* c) {
  if (!c) return fail(HG_ERR_NULL, "cache is NULL");
  if (c->B < 0 || c->H <= 0 || c->page_size <= 0 || c->num_pages < 0 || c->max_pages < 0)
    return fail(HG_ERR_SHAPE, "cache sizes B, H, page_size, num_pages, max_pages = %d, %d, %d, %d, %d", c->B, c->H,
                c->page_size, c->num_pages, c->max_pages);
  int s = check_head_dim(c->D);
  if (s) return s;
  if (c->B > 0 && c->max_pages > 0) s = check_array(c->block_table, "block_table");
  return s;
}

inline PagedCache fill_cache(const hg_paged_cache* c) {
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
inline int check_operands(const View* views, int nv, int written, const Buf* arrays, int na, const int* in_place) {
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
inline int check_written_array(const Buf& w, const View* views, int nv, const Buf* arrays, int na) {
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

inline int row_tiles(int R) { return (R + kDecodeRows - 1) / kDecodeRows; }

// Bytes of the workspace that a decode call uses.
inline uint64_t decode_bytes(int R, int D) {
  return kDecodeCounterBytes + 2 * (uint64_t)kDecodeSlots * decode_partial_floats(std::min(R, kDecodeRows), D) * 4;
}

inline int check_groups(int Hq, int H) {
  if (Hq <= 0 || Hq % H) return fail(HG_ERR_SHAPE, "%d query heads are not a multiple of %d key/value heads", Hq, H);
  return HG_OK;
}

}  // namespace hg
