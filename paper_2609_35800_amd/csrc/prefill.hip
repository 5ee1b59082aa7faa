// Attention over packed prompts, causal or full, grouped heads.
//
// For query i and key j of a row: s_ij = scale q_i.k_j, p_ij = exp(s_ij - m_i),
// out_i = sum_j p_ij v_j / sum_j p_ij, with the running maximum m_i and sum of
// a softmax over blocks of keys, so scores never leave the registers.  4 D
// operations per (query, key): the matrix units bound it.
//   * A wavefront holds 32 queries; a workgroup's wavefronts share blocks of
//     keys and values staged in LDS (two buffers, the next block loading while
//     this one is used).
//   * S^T = K Q^T and O^T = V^T P^T on 32x32x16 matrix instructions: a lane's
//     query is lane % 32 in both results, so maximum, sum and rescaling stay in
//     the lane and its partner lane ^ 32.
//   * The result layout of S^T gives half h = lane / 32 the keys 8a + 4h + c
//     (c < 4) of each 32; the second product takes its 16 keys in that order
//     (16s + 4h + c, 16s + 8 + 4h + c), so P goes from result to operand in
//     place, and V is read from LDS transposed, 4 keys x 16 channels a read.
//   * Rows in LDS are swizzled in 16-byte pieces so that neither read meets
//     its own banks.
//   * The maximum a row is scaled by moves only when a block exceeds it by
//     2^8: weights up to 2^8 are as good in BF16 and fp32, and most blocks skip
//     the rescaling of O.
// A value that is not finite must not reach queries that do not see it (0 * NaN
// in the product): in blocks that some query sees in part, such values are
// staged as 0 and added afterwards to the queries that see them.
#include "hg_attn.h"
#include "hg_device.h"

namespace hg {
namespace {

constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kNegInf = -__builtin_inff();
constexpr float kSlack = 8.0f;  // in powers of two

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

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

template <int D, int W, int BN>
__global__ __launch_bounds__(W * 64) void prefill_kernel(const PrefillParams p) {
  constexpr int T = W * 64, BM = W * 32;
  constexpr int S = D / 16;           // 16-channel steps of the first product
  constexpr int NB = D / 32;          // 32-channel blocks of the output
  constexpr int KB = BN / 32;         // 32-key blocks of a stage
  constexpr int C = D / 8;            // 16-byte pieces of a row
  constexpr int PIECES = BN * C / T;  // of each of K and V per thread and stage
  static_assert(PIECES * T == BN * C, "");
  __shared__ __attribute__((aligned(16))) uint16_t Ks[2][BN * D];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[2][BN * D];
  __shared__ int odd_stage[2];  // the stage in a buffer that holds values that are not finite

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int half = lane >> 5, col = lane & 31;

  // the row and tile of queries
  const int slot = blockIdx.x / p.Hq, hq = blockIdx.x % p.Hq;
  const int h = hq / (p.Hq / p.H);
  int b = -1, tile = 0, q_lo = 0, nq = 0;
  int before = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    int lo = 0, n = 0;
    if (b0 + lane < p.B) {
      lo = clamp_to(p.cu_q[b0 + lane], p.Nq);
      n = max(clamp_to(p.cu_q[b0 + lane + 1], p.Nq) - lo, 0);
    }
    const int tiles = (n + BM - 1) / BM;
    int sum = tiles;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int y = __shfl(sum, lane >= o ? lane - o : lane);
      sum += lane >= o ? y : 0;
    }
    const int past = __popcll(__ballot(before + sum <= slot));
    if (past < 64) {
      b = b0 + past;
      q_lo = __shfl(lo, past);
      nq = __shfl(n, past);
      const int t = __shfl(tiles, past);
      tile = t - 1 - (slot - before - (__shfl(sum, past) - t));  // long tiles of a row first
      break;
    }
    before += __shfl(sum, 63);
  }
  b = __builtin_amdgcn_readfirstlane(b);
  if (b < 0) return;
  q_lo = __builtin_amdgcn_readfirstlane(q_lo);
  nq = __builtin_amdgcn_readfirstlane(nq);
  tile = __builtin_amdgcn_readfirstlane(tile);
  const int k_lo = clamp_to(p.cu_k[b], p.Nk);
  const int nk = max(clamp_to(p.cu_k[b + 1], p.Nk) - k_lo, 0);

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
  // last key of a query, of the wavefront's queries and of the workgroup's
  const int shift = nk - nq;
  const int last = p.causal ? min(iq + shift, nk - 1) : nk - 1;
  const int wave_first = p.causal ? min(i0 + shift, nk - 1) : nk - 1;
  const int wave_last = p.causal ? min(i0 + 31 + shift, nk - 1) : nk - 1;
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
  q32x4 kr[PIECES], vr[PIECES];
  auto load_stage = [&](int stage) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int piece = threadIdx.x + i * T;
      const int64_t row = min(stage * BN + piece / C, nk - 1);
      kr[i] = *(const q32x4*)(K + row * p.k.token_stride + (piece % C) * 8);
      vr[i] = *(const q32x4*)(V + row * p.v.token_stride + (piece % C) * 8);
    }
  };
  auto store_stage = [&](int stage) {
    const int buf = stage & 1;
    if (stage * BN + BN - 1 > group_first) {
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
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int piece = threadIdx.x + i * T;
      const int row = piece / C, c = piece % C;
      *(q32x4*)&Ks[buf][row * D + ((c ^ key_swizzle<D>(row)) * 8)] = kr[i];
      *(q32x4*)&Vs[buf][row * D + ((c ^ value_swizzle<D>(row)) * 8)] = vr[i];
    }
  };

  if (threadIdx.x < 2) odd_stage[threadIdx.x] = -1;
  __syncthreads();
  if (stages > 0) {
    load_stage(0);
    store_stage(0);
  }
  __syncthreads();

  for (int stage = 0; stage < stages; ++stage) {
    const int buf = stage & 1;
    const bool more = stage + 1 < stages;
    if (more) load_stage(stage + 1);
    const int j0 = stage * BN;
    if (j0 <= wave_last) {
      f32x16 st[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) st[kb][e] = 0;
        const int row = kb * 32 + col;
#pragma unroll
        for (int s = 0; s < S; ++s) {
          const q32x4 k = *(const q32x4*)&Ks[buf][row * D + (((2 * s + half) ^ key_swizzle<D>(row)) * 8)];
          st[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[s]),
                                                           st[kb], 0, 0, 0);
        }
      }
      if (j0 + BN - 1 > wave_first) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (j0 + kb * 32 + 8 * (e >> 2) + 4 * half + (e & 3) > last) st[kb][e] = kNegInf;
      }
      float top = kNegInf;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, st[kb][e]);
      top = fmaxf(top, __shfl_xor(top, 32)) * scale;
      if (__any(top > m + kSlack)) {
        const float up = fmaxf(m, top);
        const float down = __builtin_amdgcn_exp2f(m - (up == kNegInf ? 0.0f : up));
        m = up;
        l *= down;
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[n] *= down;
      }
      const float shift_m = m == kNegInf ? 0.0f : -m;
      q32x4 w[KB][2];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kb][e], scale, shift_m));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kb][e + 1], scale, shift_m));
          l += p0 + p1;
          w[kb][e >> 3][(e & 7) >> 1] = cvt_bf16x2(p0, p1);
        }
      // V^T: lane's 16 lanes read 4 keys x 16 channels, and take 4 keys of one channel
      const int key = 4 * half + ((lane & 15) >> 2);
      const int piece = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), sub = (lane & 1) * 4;
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            union {
              s16x4 part[2];
              bf16x8 all;
            } v;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int row = kb * 32 + s * 16 + x * 8 + key;
              v.part[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (lds_s16x4*)&Vs[buf][row * D + (((n * 4 + piece) ^ value_swizzle<D>(row)) * 8) + sub]);
            }
            acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.all, __builtin_bit_cast(bf16x8, w[kb][s]), acc[n], 0, 0, 0);
          }
      if (j0 + BN - 1 > group_first && odd_stage[buf] == stage) {
        for (int j = j0; j < min(j0 + BN, nk); ++j)
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const uint32_t x = V[j * p.v.token_stride + n * 32 + 8 * (e >> 2) + 4 * half + (e & 3)];
              if ((x & 0x7F80u) == 0x7F80u && j <= last) acc[n][e] += bf16_as_float(x);
            }
      }
    }
    if (more) store_stage(stage + 1);
    __syncthreads();
  }

  l += __shfl_xor(l, 32);
  if (iq >= nq) return;
  const float inv = l > 0 ? 1.0f / l : (l == 0 ? 0.0f : l);
  uint16_t* o = p.out.data + (int64_t)(q_lo + iq) * p.out.token_stride + hq * p.out.head_stride;
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *(q32x2*)(o + n * 32 + 8 * (e >> 2) + 4 * half) =
          q32x2{cvt_bf16x2(acc[n][e] * inv, acc[n][e + 1] * inv), cvt_bf16x2(acc[n][e + 2] * inv, acc[n][e + 3] * inv)};
  if (p.lse && half == 0)
    p.lse[(int64_t)(q_lo + iq) * p.Hq + hq] = l == 0 ? kNegInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int D, int W, int BN>
hipError_t launch(const PrefillParams& p, hipStream_t stream) {
  // tiles of all rows: at most one partly filled each
  const int64_t slots = p.Nq / (W * 32) + (p.B < p.Nq ? p.B : p.Nq);
  prefill_kernel<D, W, BN><<<dim3((uint32_t)(slots * p.Hq)), dim3(W * 64), 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prefill(const PrefillParams& p, int D, hipStream_t stream) {
  return D == 64 ? launch<64, 4, 64>(p, stream) : D == 128 ? launch<128, 4, 64>(p, stream) : launch<256, 4, 64>(p, stream);
}

}  // namespace hg
