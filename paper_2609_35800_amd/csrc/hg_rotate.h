// Rotation of rows by their tokens' positions, as the append kernels do it: a
// unit is 16 channels of a row, two 16-byte pieces whose channels pair up (halves
// of the rotated channels, or 16 neighbours interleaved).
#pragma once

#include "hg_attn.h"
#include "hg_device.h"

namespace hg {
namespace {

// Once: streaming (non-temporal) loads and stores, for
// calls that outgrow the last-level cache.
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

// The pieces of unit `unit`, at channels c0 and c1, and its first pair.
struct Unit {
  int c0, c1, pair;
  bool rotated;
};
__device__ __forceinline__ Unit unit_of(const AppendParams& p, int unit) {
  Unit u;
  u.rotated = unit * 16 < p.rot;
  u.pair = unit * 8;
  if (u.rotated && !p.interleaved) {
    u.c0 = unit * 8;
    u.c1 = u.c0 + p.half;
  } else {
    u.c0 = unit * 16;
    u.c1 = u.c0 + 8;
  }
  return u;
}

// Cosines and sines of a unit's pairs for `token`, at index `at` of its row; false
// if a position is outside the table.
struct Angles {
  float cs[8], sn[8];
};
__device__ __forceinline__ bool load_angles(const AppendParams& p, const Unit& u, int token, int64_t at, Angles& an) {
  if (p.rot <= 0) return true;
  int pos[3];
  bool inside = true;
  for (int a = 0; a < p.axes; ++a) {
    const int64_t v = p.positions ? (int64_t)p.positions[(int64_t)a * p.N + token] : at;
    inside = inside && v >= 0 && v < p.max_pos;
    pos[a] = (int)v;
  }
  if (!inside) return false;
  if (p.axes == 1) pos[1] = pos[2] = pos[0];
  if (u.rotated) {
    const int pair = u.pair;
    const int a0 = pair < p.sec0 ? 0 : pair < p.sec1 ? 1 : 2;
    const int a7 = pair + 7 < p.sec0 ? 0 : pair + 7 < p.sec1 ? 1 : 2;
    if (a0 == a7) {
      const int64_t o = (int64_t)(a0 == 0 ? pos[0] : a0 == 1 ? pos[1] : pos[2]) * p.half + pair;
      const f32x4* c = (const f32x4*)(p.cos + o);
      const f32x4* s = (const f32x4*)(p.sin + o);
      const f32x4 ca = c[0], cb = c[1], sa = s[0], sb = s[1];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        an.cs[e] = ca[e];
        an.cs[e + 4] = cb[e];
        an.sn[e] = sa[e];
        an.sn[e + 4] = sb[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = pair + e;
        const int64_t o = (int64_t)(i < p.sec0 ? pos[0] : i < p.sec1 ? pos[1] : pos[2]) * p.half + i;
        an.cs[e] = p.cos[o];
        an.sn[e] = p.sin[o];
      }
    }
  }
  return true;
}

// A unit's pieces rotated in fp32, with one rounding.
__device__ __forceinline__ void rotate(u32x4& x, u32x4& y, const Angles& an, int interleaved) {
  if (!interleaved) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float a0 = bf16_lo(x[w]), a1 = bf16_hi(x[w]), b0 = bf16_lo(y[w]), b1 = bf16_hi(y[w]);
      const float c = an.cs[2 * w], s = an.sn[2 * w], d = an.cs[2 * w + 1], t = an.sn[2 * w + 1];
      x[w] = cvt_bf16x2(__builtin_fmaf(a0, c, -(b0 * s)), __builtin_fmaf(a1, d, -(b1 * t)));
      y[w] = cvt_bf16x2(__builtin_fmaf(b0, c, a0 * s), __builtin_fmaf(b1, d, a1 * t));
    }
  } else {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float a0 = bf16_lo(x[w]), b0 = bf16_hi(x[w]), a1 = bf16_lo(y[w]), b1 = bf16_hi(y[w]);
      const float c = an.cs[w], s = an.sn[w], d = an.cs[w + 4], t = an.sn[w + 4];
      x[w] = cvt_bf16x2(__builtin_fmaf(a0, c, -(b0 * s)), __builtin_fmaf(b0, c, a0 * s));
      y[w] = cvt_bf16x2(__builtin_fmaf(a1, d, -(b1 * t)), __builtin_fmaf(b1, d, a1 * t));
    }
  }
}

}  // namespace
}  // namespace hg
