// Attention over packed prompts, causal or full, grouped heads.
//
// For query i and key j of a row: s_ij = scale q_i.k_j, p_ij = exp(s_ij - m_i),
// out_i = sum_j p_ij v_j / sum_j p_ij, with the running maximum m_i and sum of
// a softmax over blocks of keys, so scores never leave the registers.  4 D
// operations per (query, key): the matrix units bound it.
//   * A wavefront holds 32 queries; a workgroup's wavefronts share stages of
//     keys and values in LDS (three and four buffers), which loads fill directly
//     while the stages before are used.
//   * S^T = K Q^T and O^T = V^T P^T on 32x32x16 matrix instructions: a lane's
//     query is lane % 32 in both results, so maximum, sum and rescaling stay in
//     the lane and its partner lane ^ 32.
//   * The result layout of S^T gives half h = lane / 32 the keys 8a + 4h + c
//     (c < 4) of each 32; the second product takes its 16 keys in that order
//     (16s + 4h + c, 16s + 8 + 4h + c), so P goes from result to operand in
//     place, and V is read from LDS transposed, 4 keys x 16 channels a read.
//   * Rows in LDS are swizzled in 16-byte pieces so that neither read meets
//     its own banks.
//   * The softmax of a stage costs the vector units about as long as its two
//     products the matrix units.  With eight wavefronts, those that share a SIMD
//     run half an iteration apart, so that one's softmax meets the other's
//     products (a wavefront's own did not overlap: with twice the queries a
//     wavefront and both kinds of work interleaved, 8.5 ms where this takes 5.5).
//   * The maximum a row is scaled by moves only when a block exceeds it by
//     2^8: weights up to 2^8 are as good in BF16 and fp32, and most blocks skip
//     the rescaling of O.
// A value that is not finite must not reach queries that do not see it (0 * NaN
// in the product): in blocks that some query sees in part, such values are
// staged as 0 and added afterwards to the queries that see them.
//
// Measured: 30001 tokens, 28 query and 4 KV heads of 128 channels, causal: 5.5 to 5.8
// ms on different cards, 1110 to 1180 TFLOP/s (a large matrix product: 1600).  By the
// counters the matrix units are busy 65 % of the cycles and no LDS read meets
// another's banks; the clock falls to 1.5 to 1.74 GHz, where calls of 40 and 80 us
// run at 2.4.
#include <type_traits>

#include "hg_attn.h"
#include "hg_device.h"

namespace hg {
namespace {

constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kNegInf = -__builtin_inff();
constexpr float kSlack = 8.0f;  // in powers of two
constexpr uint32_t kRawBufferWord3 = 0x00020000u;  // raw buffer, bounds checked in bytes

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void* lds_ptr;

template <int D>
__device__ __forceinline__ constexpr int key_swizzle(int row) {
  return D == 64 ? (row >> 1) & 7 : row & 15;
}
template <int D>
__device__ __forceinline__ constexpr int value_swizzle(int row) {
  return D == 64 ? ((row >> 1) & 1) << 2 : (row & 3) << 2;
}

// Both halves of x whose exponent is all ones (infinities, NaN) as a mask of their bits.
__device__ __forceinline__ uint32_t not_finite(uint32_t x) {
  const uint32_t lo = (x & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u;
  const uint32_t hi = (x & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u;
  return lo | hi;
}

// Maximum of a lane's value and its partner's in the other half of the wavefront.
__device__ __forceinline__ float other_half_max(float x) {
  const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

// Waits for this wavefront's LDS traffic, then for the workgroup; nothing moves across.
__device__ __forceinline__ void phase_end() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

template <int D, int W, int BN>
__global__ __launch_bounds__(W * 64, D == 256 ? 1 : 2) void prefill_kernel(const PrefillParams p) {
  constexpr int T = W * 64, BM = W * 32;
  constexpr bool kPairs = W == 8;     // two wavefronts a SIMD, half an iteration apart
  constexpr int S = D / 16;           // 16-channel steps of the first product
  constexpr int NB = D / 32;          // 32-channel blocks of the output
  constexpr int KB = BN / 32;         // 32-key blocks of a stage
  constexpr int C = D / 8;            // 16-byte pieces of a row
  constexpr int PIECES = BN * C / T;  // of each of K and V per thread and stage
  static_assert(PIECES * T == BN * C, "");
  __shared__ __attribute__((aligned(16))) uint16_t Ks[3][BN * D];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[4][BN * D];
  __shared__ int odd_stage[4];     // the stage in a buffer that holds values that are not finite

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int half = lane >> 5, col = lane & 31;

  // the row and tile of queries
  const int slot = blockIdx.x / p.Hq, hq = blockIdx.x % p.Hq;
  const int h = hq / (p.Hq / p.H);
  int b = -1, tile = 0, q_lo = 0, nq = 0, k_lo = 0, nk = 0;
  int before = 0;  // tiles of earlier rows
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    int q0 = 0, q1 = 0, k0 = 0, k1 = 0;
    if (b0 + lane < p.B) {
      q0 = p.cu_q[b0 + lane];
      q1 = p.cu_q[b0 + lane + 1];
      k0 = p.cu_k[b0 + lane];
      k1 = p.cu_k[b0 + lane + 1];
    }
    q0 = clamp_to(q0, p.Nq);
    k0 = clamp_to(k0, p.Nk);
    const int nq_row = max(clamp_to(q1, p.Nq) - q0, 0), nk_row = max(clamp_to(k1, p.Nk) - k0, 0);
    const int tiles = (nq_row + BM - 1) / BM;
    const int sum = lane_scan(tiles);
    const int row = __popcll(__ballot(before + sum <= slot));
    if (row < 64) {
      b = b0 + row;
      q_lo = __builtin_amdgcn_readlane(q0, row);
      nq = __builtin_amdgcn_readlane(nq_row, row);
      k_lo = __builtin_amdgcn_readlane(k0, row);
      nk = __builtin_amdgcn_readlane(nk_row, row);
      // a row's long tiles first
      tile = before + __builtin_amdgcn_readlane(sum, row) - 1 - slot;
      break;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  // (offsets that do not ascend can lead to a row without this tile)
  if (b < 0 || b >= p.B || tile < 0 || (int64_t)tile * BM >= nq) return;

  // queries, as the second operand of S^T: query col, channels 16 s + 8 half ..
  const int i0 = tile * BM + wave * 32;  // first query of the wavefront
  const int iq = i0 + col;
  const uint32_t flip = p.scale_log2 < 0 ? 0x80008000u : 0u;
  const float scale = fmaxf(fabsf(p.scale_log2), 1e-30f);  // (-inf) * 0 would be NaN
  q32x4 q[S];
  {
    const uint16_t* src = p.q.data + (int64_t)(q_lo + min(iq, nq - 1)) * p.q.token_stride + hq * p.q.head_stride + half * 8;
#pragma unroll
    for (int s = 0; s < S; ++s) q[s] = *(const q32x4*)(src + s * 16) ^ flip;
  }
  // last key of a query, of the wavefront's first, of the workgroup's first and last
  const int shift = nk - nq;
  const int last = p.causal ? min(iq + shift, nk - 1) : nk - 1;
  const int wave_first = p.causal ? min(i0 + shift, nk - 1) : nk - 1;
  const int group_first = p.causal ? min(tile * BM + shift, nk - 1) : nk - 1;
  const int group_last = p.causal ? min(min(tile * BM + BM, nq) - 1 + shift, nk - 1) : nk - 1;
  const int stages = group_last < 0 ? 0 : group_last / BN + 1;

  f32x16 acc[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[n][e] = 0;
  float m = kNegInf, l = 0;

  const uint16_t* K = p.k.data + (int64_t)k_lo * p.k.token_stride + h * p.k.head_stride;
  const uint16_t* V = p.v.data + (int64_t)k_lo * p.v.token_stride + h * p.v.head_stride;

  // Staging, one stage after the other: global memory -> LDS directly, 1 KiB a
  // wavefront and instruction, lane after lane, so a lane asks for the piece that
  // the swizzle puts in its place.  A stage's rows are read through a buffer
  // resource that ends with row nk - 1: rows past it are not read.  Values of
  // stages that some query sees in part go through registers (rows past the last
  // come back as 0), where those that are not finite are taken out.
  q32x4 vr[PIECES];
  const int stage_row = threadIdx.x / C, place = threadIdx.x % C;  // and every T / C rows
  struct Stream {
    const uint16_t* at;          // first row of the stage to be loaded
    int64_t left;                // bytes from there to the end of row nk - 1, or below 1
    int64_t stage;               // bytes of a stage
    uint32_t off[PIECES];        // this thread's pieces
  };
  auto open = [&](const uint16_t* base, int64_t stride, auto swizzle) __attribute__((always_inline)) {
    Stream x;
    x.at = base;
    x.left = nk > 0 ? (nk - 1) * stride * 2 + D * 2 : 0;
    x.stage = BN * stride * 2;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int row = stage_row + i * (T / C);
      x.off[i] = (uint32_t)(row * stride * 2 + (place ^ swizzle(row)) * 16);
    }
    return x;
  };
  auto resource = [&](const Stream& x) __attribute__((always_inline)) {
    const int32_t high = (int32_t)(x.left >> 32);
    const uint32_t bytes = high < 0 ? 0u : high > 0 ? 0xFFFFFFFFu : (uint32_t)x.left;
    const uint64_t at = (uint64_t)x.at;
    return q32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(at >> 32) & 0xFFFFu)),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), kRawBufferWord3};
  };
  auto advance = [&](Stream& x) __attribute__((always_inline)) {
    x.at += x.stage / 2;
    x.left -= x.stage;
  };
  Stream ks = open(K, p.k.token_stride, [](int row) { return key_swizzle<D>(row); });
  Stream vs = open(V, p.v.token_stride, [](int row) { return value_swizzle<D>(row); });
  // The instruction is written out: the compiler would have every later LDS read
  // wait for it.  phase_end and the counted waits order it, which count the
  // requests in the order written (it writes LDS, so no other access of memory
  // may move across it).  m0 holds the LDS address; the compiler warns of it because
  // it keeps nothing there itself.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  auto stage_direct = [&](Stream& x, uint16_t* buf) __attribute__((always_inline)) {
    const q32x4 r = resource(x);
    const uint32_t to = (uint32_t)(uintptr_t)(lds_ptr)buf + wave * 1024;
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(
                       __builtin_amdgcn_readfirstlane((int)(to + i * T * 16))),
                   "v"(x.off[i]), "s"(r)
                   : "m0", "memory");
    advance(x);
  };
#pragma clang diagnostic pop
  auto load_values = [&]() __attribute__((always_inline)) {
    const q32x4 words = resource(vs);
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)vs.at, 0, words[2], kRawBufferWord3);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) vr[i] = __builtin_amdgcn_raw_buffer_load_b128(r, vs.off[i], 0, 0);
    advance(vs);
  };
  auto store_values = [&](int stage, int buf) __attribute__((always_inline)) {
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t x = not_finite(vr[i][w]);
        odd |= x;
        vr[i][w] &= ~x;
      }
    if (odd) odd_stage[buf] = stage;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) *(q32x4*)&Vs[buf][(i * T + threadIdx.x) * 8] = vr[i];
  };

  f32x16 st[KB];
  q32x4 w[KB][2];
  // A matrix half: PV steps of O^T += V^T P^T (channel blocks of 32, 16 keys
  // each), then QK steps of S^T = K Q^T (key blocks of 32, 16 channels each), one
  // matrix instruction a step.  Its operand comes from LDS into a ring that is
  // refilled as soon as it is used, kRing steps ahead.
  constexpr int PV = NB * 2 * KB, QK = KB * S, kRing = 8;
  bf16x8 ring[kRing];
  const int k_base = col * D + (half ^ key_swizzle<D>(col)) * 8;
  auto read_key = [&](int t, int buf) __attribute__((always_inline)) {
    const int kb = t / S, s = t % S;
    return __builtin_bit_cast(bf16x8, *(const q32x4*)&Ks[buf][(k_base ^ (s * 16)) + kb * 32 * D]);
  };
  // V^T: a lane's 16 lanes read 4 keys x 16 channels, and take 4 keys of one channel
  const int v_key = 4 * half + ((lane & 15) >> 2);
  const int v_base = v_key * D + ((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ value_swizzle<D>(v_key)) * 8 + (lane & 1) * 4;
  auto read_value = [&](int t, int buf) __attribute__((always_inline)) {
    const int n = t / (2 * KB), x = t % (2 * KB);
    union {
      s16x4 part[2];
      bf16x8 all;
    } v;
#pragma unroll
    for (int y = 0; y < 2; ++y)
      v.part[y] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)&Vs[buf][(v_base ^ (n * 32)) + (x * 16 + y * 8) * D]);
    return v.all;
  };
  // Buffers: keys of stage i in i % 3, values in i % 4.
  auto next3 = [](int buf) __attribute__((always_inline)) { return buf == 2 ? 0 : buf + 1; };
  // Steps [from, to) of PV + QK, values of buffer vb, keys of kb; then the ring
  // holds the first PV steps of the values of buffer vb + 1.  Between them the
  // staging of stage i + 2 (with `edge` of values of stage i + 1, asked for before).
  auto matrix_half = [&](auto first, auto end, int i, int vb, int kbuf, bool stage, bool pending, bool edge) __attribute__((always_inline)) {
    constexpr int from = decltype(first)::value, to = decltype(end)::value;
    if constexpr (to > PV) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) st[kb][e] = 0;
    }
#pragma unroll
    for (int t = from; t < to; ++t) {
      bf16x8& f = ring[t % kRing];
      if (t < PV) {
        const int n = t / (2 * KB), x = t % (2 * KB);
        acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, __builtin_bit_cast(bf16x8, w[x >> 1][x & 1]), acc[n], 0, 0, 0);
      } else {
        const int kb = (t - PV) / S, s = (t - PV) % S;
        st[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, __builtin_bit_cast(bf16x8, q[s]), st[kb], 0, 0, 0);
      }
      const int r = t + kRing;
      if (r < to) f = r < PV ? read_value(r, vb) : read_key(r - PV, kbuf);
      else if (to == PV + QK) f = read_value(r - to, (vb + 1) & 3);
      if (stage) {
        if (t == from + 1 && pending) store_values(i + 1, (vb + 2) & 3);  // before newer requests: its wait is for all
        if (t == from + 3) stage_direct(ks, Ks[next3(next3(kbuf))]);
        if (t == from + 5) {
          if (edge) load_values();
          else stage_direct(vs, Vs[(vb + 3) & 3]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // values of a stage that are not finite, to the queries that see them
  auto add_odd = [&](int stage, int buf) __attribute__((always_inline)) {
    if (odd_stage[buf] != stage) return;
    for (int j = stage * BN; j < min(stage * BN + BN, nk); ++j)
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const uint32_t x = V[j * p.v.token_stride + n * 32 + 8 * (e >> 2) + 4 * half + (e & 3)];
          if ((x & 0x7F80u) == 0x7F80u && j <= last) acc[n][e] += bf16_as_float(x);
        }
  };
  // st -> w, the running maximum and sum; O is rescaled if the maximum moves.  The
  // weights are rounded to BF16 for their product with the values, the type that the
  // matrix units take beside them; their sum is of the unrounded ones.  Measured
  // against 64 bits the output is off by 0.0020 to 0.0022 (relative, rms), 0.0016 of
  // which any BF16 output has.
  auto softmax = [&](int j0, bool edge) __attribute__((always_inline)) {
    if (edge && j0 + BN - 1 > wave_first) {
      const int seen = last - j0 - 4 * half;  // keys of this lane's half up to here
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (kb * 32 + 8 * (e >> 2) + (e & 3) > seen) st[kb][e] = kNegInf;
    }
    float top = kNegInf;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, st[kb][e]);
    top = other_half_max(top) * scale;
    if (__any(top > m + kSlack)) {
      const float up = fmaxf(m, top);
      const float down = __builtin_amdgcn_exp2f(m - (up == kNegInf ? 0.0f : up));
      m = up;
      l *= down;
#pragma unroll
      for (int n = 0; n < NB; ++n) acc[n] *= down;
    }
    const float shift_m = m == kNegInf ? 0.0f : -m;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kb][e], scale, shift_m));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kb][e + 1], scale, shift_m));
        l += p0 + p1;
        w[kb][e >> 3][(e & 7) >> 1] = cvt_bf16x2(p0, p1);
      }
  };

  // Iteration i: the products of stage i - 1 with its values and of stage i with
  // its keys (matrix units), then the softmax of stage i (vector units).  Of the
  // two wavefronts of a SIMD one is half an iteration behind, so each kind of
  // work meets the other.  Stage i + 2 is asked for in iteration i's matrix half,
  // over stages that the later wavefronts last read in their iteration i - 1 (keys
  // of stage i - 1, values of i - 2), which has ended; the end of the matrix half
  // of iteration i + 1 waits for it, and its first reads come after that.  Every
  // matrix half asks for the same number of pieces, stages past the last too
  // (nothing is read for them), so the wait can count them.
  typedef std::integral_constant<int, 0> kStart;
  typedef std::integral_constant<int, PV> kProducts;
  typedef std::integral_constant<int, PV + QK> kEnd;
  int vb = 3, kbuf = 0;  // buffers of the values of stage i - 1, the keys of i
  // stages that every query of the workgroup sees whole (none if the first one
  // sees no key: with fewer keys than queries group_first can be far below 0)
  const int whole = max(group_first + 1, 0) / BN;
  auto iteration = [&](auto from, int i, bool edge) __attribute__((always_inline)) {
    __builtin_amdgcn_s_setprio(1);
    matrix_half(from, kEnd(), i, vb, kbuf, true, edge && i + 1 >= whole, edge);
    __builtin_amdgcn_s_setprio(0);
    if (edge && i > whole) add_odd(i - 1, vb);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * PIECES) : "memory");
    phase_end();
    softmax(i * BN, edge);
    if (kPairs) phase_end();
    vb = (vb + 1) & 3;
    kbuf = next3(kbuf);
  };
  if (stages > 0) {
    if (threadIdx.x < 4) odd_stage[threadIdx.x] = -1;
    stage_direct(ks, Ks[0]);
    if (whole < 1) load_values();
    else stage_direct(vs, Vs[0]);
    stage_direct(ks, Ks[1]);
    __syncthreads();
    if (whole < 1) store_values(0, 0);
    if (whole < 2) load_values();
    else stage_direct(vs, Vs[1]);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * PIECES) : "memory");
    __syncthreads();
    if (kPairs && wave >= W / 2) phase_end();
#pragma unroll
    for (int t = 0; t < kRing; ++t) ring[(PV + t) % kRing] = read_key(t, 0);
    if (whole > 2) iteration(kProducts(), 0, false);
    else iteration(kProducts(), 0, true);
    int i = 1;
    for (; i + 2 < whole; ++i) iteration(kStart(), i, false);
    for (; i < stages; ++i) iteration(kStart(), i, true);
    matrix_half(kStart(), kProducts(), i, vb, kbuf, false, false, false);
    add_odd(stages - 1, vb);
    if (kPairs && wave < W / 2) phase_end();
    // nothing may still be on its way to LDS when the workgroup leaves it
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }

  l += __shfl_xor(l, 32);
  const float inv = l > 0 ? 1.0f / l : (l == 0 ? 0.0f : l);
  uint16_t* o = p.out.data + (int64_t)(q_lo + iq) * p.out.token_stride + hq * p.out.head_stride + half * 8;
  // channels 8a + 4 half + c of both halves of the wavefront exchanged, so that a
  // lane stores 8 neighbours: 16 a .. of the first half's, 16 a + 8 .. of the second's
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      q32x4 y;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const int e = 8 * a + 2 * w;
        const auto both = __builtin_amdgcn_permlane32_swap(cvt_bf16x2(acc[n][e] * inv, acc[n][e + 1] * inv),
                                                           cvt_bf16x2(acc[n][e + 4] * inv, acc[n][e + 5] * inv), false, false);
        y[w] = both[0];
        y[w + 2] = both[1];
      }
      if (iq < nq) *(q32x4*)(o + n * 32 + a * 16) = y;
    }
  if (iq >= nq) return;
  if (p.lse && half == 0)
    p.lse[(int64_t)(q_lo + iq) * p.Hq + hq] = l == 0 ? kNegInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Tiles of all rows (at most one partly filled each) and heads, by the wavefronts
// of a workgroup.
int64_t workgroups(const PrefillParams& p, int waves) {
  return ((int64_t)p.Nq / (waves * 32) + (p.B < p.Nq ? p.B : p.Nq)) * p.Hq;
}

template <int D, int W, int BN>
hipError_t launch(const PrefillParams& p, hipStream_t stream) {
  prefill_kernel<D, W, BN><<<dim3((uint32_t)workgroups(p, W)), dim3(W * 64), 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

// At head_dim 128, rows of fewer than kShortRow keys on average take tiles of 128
// queries and stages of 32 keys, two workgroups a compute unit, which meet each
// other's work by chance; longer ones tiles of 256 queries, whose pairs do so by
// design and which read each stage half as often.  Measured, 128 -> 256 queries
// (us; query/KV heads): 30 tokens 32/32 5.2 -> 6.9, 16 x 60 32/8 11.6 -> 16.7, 8 x
// 170 28/4 16.2 -> 16.9, 4 x 600 28/4 30.4 -> 40.7, 1360 28/4 37.4 -> 38.1, 4 x 1400
// 28/4 87.6 -> 93.8, 8 x 1700 32/8 261 -> 260, 8 x 2200 32/8 395 -> 387, 5000 28/4 198
// -> 191.  At head_dim 64, 128 queries and 64 keys (8 x 2000 32/8 205, with 256
// queries 214; 1360 28/4 24.4 and 26.3).  At 256, O and Q leave registers for one
// wavefront a SIMD, and LDS for stages of 32 keys.
constexpr int kShortRow = 1700;

static bool long_rows(const PrefillParams& p, int D) { return D == 128 && (int64_t)p.Nk >= (int64_t)kShortRow * p.B; }

int64_t prefill_work_items(const PrefillParams& p, int D) {
  const int waves = long_rows(p, D) ? 8 : 4;
  return workgroups(p, waves) * waves * 64;
}

hipError_t launch_prefill(const PrefillParams& p, int D, hipStream_t stream) {
  if (D == 64) return launch<64, 4, 64>(p, stream);
  if (D == 256) return launch<256, 4, 32>(p, stream);
  return long_rows(p, D) ? launch<128, 8, 64>(p, stream) : launch<128, 4, 32>(p, stream);
}

}  // namespace hg
