// Kernel parameters, launchers and device helpers of the attention calls
// (append, prefill, decode).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "headguard.h"

namespace hg {

// A batch row's pages; see hg_paged_cache.  num_pages = 0 comes with
// max_tokens = 0, so no token is looked up.
struct PagedCache {
  uint16_t *K, *V;
  const int32_t* table;
  int64_t page_stride, head_stride, token_stride;
  int32_t B, H, page_size, num_pages, max_pages;
  int32_t max_tokens;         // min(max_pages * page_size, 2^31 - 1)
  uint32_t div_mul, div_shift;  // t / page_size = mulhi(t, div_mul) >> div_shift (t < 2^31), or t >> div_shift
};

struct AppendParams {
  PagedCache cache;
  hg_rows q, k, v, q_out, k_out;
  const int32_t *lens, *cu, *positions;
  const float *cos, *sin;
  int32_t N, Hq;
  int32_t rot, half, max_pos, interleaved;  // rotated channels and pairs
  int32_t sec0, sec1;                       // first pair of axes 1 and 2 (half: one axis)
  int32_t axes;
};

struct DecodeParams {
  PagedCache cache;
  hg_rows q, out;
  float* lse;
  const int32_t *lens, *starts;
  float scale_log2;    // scale * log2(e)
  int32_t R;           // query heads per key/value head
  int32_t row_tiles;   // tiles of kDecodeRows query heads
  int64_t stream_chunks;  // see decode_stream_chunks
  uint32_t* counters;  // arrivals by slot; zero between calls
  float* partial;      // results of parts of items, by slot
};

struct PrefillParams {
  hg_rows q, k, v, out;
  float* lse;
  const int32_t *cu_q, *cu_k;
  int32_t B, Hq, H, Nq, Nk;
  int32_t causal;
  float scale_log2;
};

// The 8-bit cache: PagedCache's strides count codes, its K and V are not used.
struct Cache8 {
  uint8_t *K, *V;
  float *k_scale, *v_scale;
  uint16_t* bounds;
  int32_t block_shift;  // log2 of the tokens of a block
  int32_t page_blocks;  // blocks of a page
};

struct Append8Params {
  AppendParams a;
  Cache8 c;
  const int32_t* starts;  // the rows' first tokens, or NULL
};

struct Decode8Params {
  DecodeParams d;
  Cache8 c;
  const int32_t* blocks;
  int32_t budget;
};

struct SelectParams {
  PagedCache cache;
  hg_rows q;
  const int32_t *lens, *starts;
  const uint16_t* bounds;
  int32_t block_shift, page_blocks, D, R;
  int32_t budget, first, last;
  int32_t* blocks;
  uint64_t* keys;     // [B][H][row_blocks]: scores of long rows, as integers of their order
  int64_t row_blocks; // blocks of max_tokens
};

struct ResizeParams {
  int32_t B, page_size, num_pages, max_pages;
  int32_t *table, *lens, *free_pages, *n_free;
  int32_t N;
  const int32_t* targets;
  int32_t* cu;
  int64_t* slots;
  int32_t *positions, *result;
};

// Work-items of the call's launch (from the sizes in p alone).  The runtime takes
// at most kMaxWorkItems in a dimension: 2^32 are refused, and of more the bits
// above the 32nd are dropped without an error.
constexpr int64_t kMaxWorkItems = 0xFFFFFFFFll;
int64_t append_work_items(const AppendParams& p, int D);
int64_t prefill_work_items(const PrefillParams& p, int D);

int64_t append8_work_items(const Append8Params& p, int D);
int64_t select_work_items(const SelectParams& p);

int64_t decode_stream_chunks(const PagedCache& c, int D, int row_tiles);
int64_t decode8_stream_chunks(const PagedCache& c, int D, int row_tiles);

hipError_t launch_append(const AppendParams& p, int D, hipStream_t stream);
hipError_t launch_decode(const DecodeParams& p, int D, hipStream_t stream);
hipError_t launch_prefill(const PrefillParams& p, int D, hipStream_t stream);
hipError_t launch_append8(const Append8Params& p, int D, hipStream_t stream);
hipError_t launch_decode8(const Decode8Params& p, int D, hipStream_t stream);
hipError_t launch_scores(const SelectParams& p, hipStream_t stream);
bool select_has_long_rows(const SelectParams& p);  // whether launch_select has anything to do
hipError_t launch_select(const SelectParams& p, hipStream_t stream);
hipError_t launch_resize(const ResizeParams& p, hipStream_t stream);
hipError_t launch_slots(const ResizeParams& p, hipStream_t stream);
bool resize_maps_slots(const ResizeParams& p);  // whether launch_resize does launch_slots' work

// Decode: query heads of a row tile, workgroups of a launch, and floats of a
// part's result for a tile with `rows` query heads.  Every workgroup has two
// slots for such results, each with an arrival counter.  The counters come first
// in the workspace, at a place that no size of a call moves: a word that one call
// counts in must not be one that a call of another size writes results to.
constexpr int kDecodeRows = 16;
constexpr int kDecodeSlots = 512;
constexpr int kDecodeCounterBytes = 2 * kDecodeSlots * 4;
constexpr int64_t kMaxKeyStride = 1 << 24;  // between tokens of k, v
// Keys of a prefill call: tiles and stages that end past the last key are counted
// in int32_t, up to 256 queries and two stages of 64 keys further.
constexpr int32_t kMaxKeys = 0x7FFFFFFF - 512;
constexpr int decode_partial_floats(int rows, int D) { return 2 * rows + rows * D; }

typedef uint32_t q32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t q32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Two floats to BF16, nearest, ties to even (one conversion instruction).
__device__ __forceinline__ uint32_t cvt_bf16x2(float lo, float hi) {
  const f32x2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

__device__ __forceinline__ uint32_t divide(uint32_t t, const PagedCache& c) {
  return (c.div_mul ? __umulhi(t, c.div_mul) : t) >> c.div_shift;
}

__device__ __forceinline__ int32_t clamp_to(int32_t x, int32_t hi) { return min(max(x, 0), hi); }

// Inclusive sum over the lanes up to this one (DPP row shifts and broadcasts).
template <int CTRL, int ROWS>
__device__ __forceinline__ int lane_add(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int lane_scan(int v) {
  v = lane_add<0x111, 0xF>(v);  // row_shr:1, 2, 4, 8
  v = lane_add<0x112, 0xF>(v);
  v = lane_add<0x114, 0xF>(v);
  v = lane_add<0x118, 0xF>(v);
  v = lane_add<0x142, 0xA>(v);  // row_bcast:15, 31
  return lane_add<0x143, 0xC>(v);
}
__device__ __forceinline__ int lane_sum(int v) { return __builtin_amdgcn_readlane(lane_scan(v), 63); }

// Row of `cu` ([B+1] ascending) that holds token t: the number of rows that
// end at or before t, counted 64 rows at a time by the wavefront; t is uniform.
// B if t is past the last row.
__device__ __forceinline__ int find_row(const int32_t* cu, int B, int t) {
  const int lane = threadIdx.x & 63;
  int n = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const bool before = b0 + lane < B && cu[b0 + lane + 1] <= t;
    n += __popcll(__ballot(before));
  }
  return __builtin_amdgcn_readfirstlane(n);
}

}  // namespace hg
