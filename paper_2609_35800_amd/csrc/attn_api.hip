// Host side of the attention calls: argument checks and launch.  The contract
// of every entry point is in include/headguard.h.

#include <string.h>

#include "headguard.h"
#include "hg_attn.h"
#include "hg_checks.h"
#include "hg_host.h"

using namespace hg;

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
  s = check_rotation(rot, a, cache->D, p);
  if (s) return s;
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
