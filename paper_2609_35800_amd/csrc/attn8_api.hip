// Host side of the 8-bit cache's calls and of the page pool: argument checks and
// launch.  The contract of every entry point is in include/headguard.h.

#include <string.h>

#include "headguard.h"
#include "hg_attn.h"
#include "hg_checks.h"
#include "hg_host.h"

using namespace hg;

namespace {

// The paged cache that an 8-bit one is apart from its codes and scales.
hg_paged_cache as_paged(const hg_cache8& c) {
  hg_paged_cache p;
  memset(&p, 0, sizeof p);
  p.B = c.B;
  p.H = c.H;
  p.D = c.D;
  p.page_size = c.page_size;
  p.num_pages = c.num_pages;
  p.max_pages = c.max_pages;
  p.page_stride = c.page_stride;
  p.head_stride = c.head_stride;
  p.token_stride = c.token_stride;
  p.block_table = c.block_table;
  return p;
}

int check_cache8(const hg_cache8* c, hg_paged_cache& paged) {
  if (!c) return fail(HG_ERR_NULL, "cache is NULL");
  paged = as_paged(*c);
  const int s = check_cache(&paged);
  if (s) return s;
  if (c->block_size != 16 && c->block_size != 32 && c->block_size != 64 && c->block_size != 128)
    return fail(HG_ERR_SHAPE, "block_size %d not in {16, 32, 64, 128}", c->block_size);
  if (c->page_size % c->block_size)
    return fail(HG_ERR_SHAPE, "page_size %d is not a multiple of block_size %d", c->page_size, c->block_size);
  return HG_OK;
}

Cache8 fill_cache8(const hg_cache8* c) {
  Cache8 p;
  p.K = c->K;
  p.V = c->V;
  p.k_scale = c->k_scale;
  p.v_scale = c->v_scale;
  p.bounds = c->bounds;
  p.block_shift = __builtin_ctz(c->block_size);
  p.page_blocks = c->page_size / c->block_size;
  return p;
}

View codes_view(const char* name, const uint8_t* data, const hg_cache8& c) {
  return View{name, data, c.D, {c.num_pages, c.H, c.page_size}, {c.page_stride, c.head_stride, c.token_stride}, 3, 1};
}

// Blocks of all pages and heads, at most 2^50 (past every memory).
uint64_t cache_blocks(const hg_cache8& c) {
  const __int128 n = (__int128)c.num_pages * c.H * (c.page_size / c.block_size);
  return n > ((__int128)1 << 50) ? (uint64_t)1 << 50 : (uint64_t)n;
}

}  // namespace

extern "C" {

int hg_append_kv8(const hg_cache8* cache, const hg_rotation* rot, const hg_append* a, hipStream_t stream) {
  return hg_append_kv8_from(cache, rot, a, nullptr, stream);
}

int hg_append_kv8_from(const hg_cache8* cache, const hg_rotation* rot, const hg_append* a, const int32_t* starts,
                       hipStream_t stream) {
  hg_paged_cache paged;
  int s = check_cache8(cache, paged);
  if (s) return s;
  if (!a) return fail(HG_ERR_NULL, "args is NULL");
  if (a->N < 0 || a->Hq < 0) return fail(HG_ERR_SHAPE, "N, Hq = %d, %d", a->N, a->Hq);
  if (!a->cu_new && a->N != cache->B)
    return fail(HG_ERR_SHAPE, "%d tokens for %d rows without cu_new", a->N, cache->B);
  Append8Params p;
  memset(&p, 0, sizeof p);
  const int D = cache->D;
  s = check_rotation(rot, a, D, p.a);
  if (s) return s;
  if (a->N == 0 || cache->B == 0) return ok();
  if ((int64_t)a->Hq + 2 * (int64_t)cache->H > 0x7FFFFFFF - 1024)
    return fail(HG_ERR_SHAPE, "%d query and %d key/value heads", a->Hq, cache->H);
  p.a.cache = fill_cache(&paged);
  p.a.N = a->N;
  p.a.Hq = a->Hq;
  p.a.cu = a->cu_new;
  p.c = fill_cache8(cache);
  p.starts = starts;
  if (append8_work_items(p, D) > kMaxWorkItems)
    return fail(HG_ERR_SHAPE, "grid too large for %d tokens of %d query and %d key/value heads", a->N, a->Hq, cache->H);
  const uint64_t table_bytes = (uint64_t)p.a.half * p.a.max_pos * 4, blocks = cache_blocks(*cache);
  const View views[] = {
      codes_view("K", cache->K, *cache),
      codes_view("V", cache->V, *cache),
      rows_view("q_out", a->q_out, a->N, a->Hq, D),
      rows_view("k_out", a->k_out, a->k_out.data ? a->N : 0, cache->H, D),
      rows_view("q", a->q, a->N, a->Hq, D),
      rows_view("k", a->k, a->N, cache->H, D),
      rows_view("v", a->v, a->N, cache->H, D),
  };
  const Buf arrays[] = {
      {cache->k_scale, blocks * 4, 4, "k_scale"},
      {cache->v_scale, blocks * 4, 4, "v_scale"},
      {cache->bounds, cache->bounds ? blocks * 4 * D : 0, 16, "bounds"},
      {a->lens, (uint64_t)cache->B * 4, 4, "lens"},
      {starts, starts ? (uint64_t)cache->B * 4 : 0, 4, "starts"},
      {a->cu_new, a->cu_new ? ((uint64_t)cache->B + 1) * 4 : 0, 4, "cu_new"},
      {p.a.positions, p.a.positions ? (uint64_t)p.a.axes * a->N * 4 : 0, 4, "positions"},
      {p.a.cos, table_bytes, 16, "cos"},
      {p.a.sin, table_bytes, 16, "sin"},
      {cache->block_table, (uint64_t)cache->B * cache->max_pages * 4, 4, "block_table"},
  };
  const int in_place[] = {-1, -1, 4, 5};
  for (int i = 0; i < 3 && !s; ++i) s = check_written_array(arrays[i], views, 7, arrays, 10);
  if (!s) s = check_operands(views, 7, 4, arrays, 10, in_place);
  if (s) return s;
  p.a.q = a->q;
  p.a.k = a->k;
  p.a.v = a->v;
  p.a.q_out = a->q_out;
  p.a.k_out = a->k_out;
  p.a.lens = a->lens;
  LaunchSteps step;
  const hipError_t e = step([&] { return launch_append8(p, D, stream); });
  if (e != hipSuccess) return fail(HG_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
  return ok();
}

int hg_decode8_workspace(const hg_cache8* cache, int32_t Hq, uint64_t* bytes) {
  hg_paged_cache paged;
  const int s = check_cache8(cache, paged);
  return s ? s : hg_decode_workspace(&paged, Hq, bytes);
}

int hg_decode_attention8(const hg_cache8* cache, const hg_decode8* a, hipStream_t stream) {
  hg_paged_cache paged;
  int s = check_cache8(cache, paged);
  if (s) return s;
  if (!a) return fail(HG_ERR_NULL, "args is NULL");
  s = check_groups(a->Hq, cache->H);
  if (!s) s = check_scale(a->scale);
  if (s) return s;
  if (a->blocks ? a->budget <= 0 : a->budget != 0)
    return fail(HG_ERR_SHAPE, "budget %d %s blocks", a->budget, a->blocks ? "with" : "without");
  if (cache->B == 0) return ok();
  const int D = cache->D, R = a->Hq / cache->H;
  const uint64_t need = decode_bytes(R, D);
  if (!a->workspace)
    return fail(HG_ERR_NULL, "workspace is NULL but the call needs %llu bytes", (unsigned long long)need);
  if (a->workspace_bytes < need)
    return fail(HG_ERR_SHAPE, "the call needs a %llu-byte workspace (%llu bytes available)", (unsigned long long)need,
                (unsigned long long)a->workspace_bytes);
  const uint64_t blocks = cache_blocks(*cache);
  const View views[] = {
      rows_view("out", a->out, cache->B, a->Hq, D),
      rows_view("q", a->q, cache->B, a->Hq, D),
      codes_view("K", cache->K, *cache),
      codes_view("V", cache->V, *cache),
  };
  const Buf arrays[] = {
      {a->lens, (uint64_t)cache->B * 4, 4, "lens"},
      {a->starts, a->starts ? (uint64_t)cache->B * 4 : 0, 4, "starts"},
      {cache->block_table, (uint64_t)cache->B * cache->max_pages * 4, 4, "block_table"},
      {a->lse, a->lse ? (uint64_t)cache->B * a->Hq * 4 : 0, 4, "lse"},
      {a->workspace, need, 256, "workspace"},
      {cache->k_scale, blocks * 4, 4, "k_scale"},
      {cache->v_scale, blocks * 4, 4, "v_scale"},
      {a->blocks, a->blocks ? (uint64_t)cache->B * cache->H * a->budget * 4 : 0, 4, "blocks"},
  };
  for (int i = 3; i < 5 && !s; ++i) s = check_written_array(arrays[i], views, 4, arrays, 8);
  if (!s) s = check_operands(views, 4, 1, arrays, 8, nullptr);
  if (s) return s;
  Decode8Params p;
  memset(&p, 0, sizeof p);
  p.d.cache = fill_cache(&paged);
  p.d.q = a->q;
  p.d.out = a->out;
  p.d.lse = a->lse;
  p.d.lens = a->lens;
  p.d.starts = a->starts;
  p.d.scale_log2 = (float)(a->scale * kLog2e);
  p.d.R = R;
  p.d.row_tiles = row_tiles(R);
  p.d.stream_chunks = decode8_stream_chunks(p.d.cache, D, p.d.row_tiles);
  p.d.counters = (uint32_t*)a->workspace;
  p.d.partial = (float*)((char*)a->workspace + kDecodeCounterBytes);
  p.c = fill_cache8(cache);
  p.blocks = a->blocks;
  p.budget = a->budget;
  LaunchSteps step;
  const hipError_t e = step([&] { return launch_decode8(p, D, stream); });
  if (e != hipSuccess) return fail(HG_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
  return ok();
}

int hg_select_workspace(const hg_cache8* cache, uint64_t* bytes) {
  hg_paged_cache paged;
  const int s = check_cache8(cache, paged);
  if (s) return s;
  if (!bytes) return fail(HG_ERR_NULL, "bytes is NULL");
  const PagedCache c = fill_cache(&paged);
  const uint64_t row_blocks = ((uint64_t)c.max_tokens + cache->block_size - 1) / cache->block_size;
  const __int128 n = (__int128)cache->B * cache->H * row_blocks * 8;
  if (n > ((__int128)1 << 50)) return fail(HG_ERR_SHAPE, "scores of %d rows and %d heads are too large", cache->B, cache->H);
  *bytes = (uint64_t)n;
  return ok();
}

int hg_select_blocks(const hg_cache8* cache, const hg_select* a, hipStream_t stream) {
  uint64_t need = 0;
  int s = hg_select_workspace(cache, &need);
  if (s) return s;
  if (!a) return fail(HG_ERR_NULL, "args is NULL");
  s = check_groups(a->Hq, cache->H);
  if (s) return s;
  if (a->budget <= 0 || a->first < 0 || a->last < 0 || (int64_t)a->first + a->last > a->budget)
    return fail(HG_ERR_SHAPE, "budget, first, last = %d, %d, %d", a->budget, a->first, a->last);
  if (cache->B == 0) return ok();
  if (need && !a->workspace)
    return fail(HG_ERR_NULL, "workspace is NULL but the call needs %llu bytes", (unsigned long long)need);
  if (a->workspace_bytes < need)
    return fail(HG_ERR_SHAPE, "the call needs a %llu-byte workspace (%llu bytes available)", (unsigned long long)need,
                (unsigned long long)a->workspace_bytes);
  const int D = cache->D;
  const hg_paged_cache paged = as_paged(*cache);
  SelectParams p;
  memset(&p, 0, sizeof p);
  p.cache = fill_cache(&paged);
  const Cache8 c8 = fill_cache8(cache);
  p.block_shift = c8.block_shift;
  p.page_blocks = c8.page_blocks;
  p.row_blocks = ((int64_t)p.cache.max_tokens + cache->block_size - 1) / cache->block_size;
  p.D = cache->D;
  p.budget = a->budget;
  if (select_work_items(p) > kMaxWorkItems)
    return fail(HG_ERR_SHAPE, "grid too large for %d rows of %d heads and %lld blocks", cache->B, cache->H,
                (long long)p.row_blocks);
  const uint64_t blocks = cache_blocks(*cache);
  const View views[] = {rows_view("q", a->q, cache->B, a->Hq, D)};
  const Buf arrays[] = {
      {a->blocks, (uint64_t)cache->B * cache->H * a->budget * 4, 4, "blocks"},
      {a->workspace, need, 256, "workspace"},
      {cache->bounds, blocks * 4 * D, 16, "bounds"},
      {a->lens, (uint64_t)cache->B * 4, 4, "lens"},
      {a->starts, a->starts ? (uint64_t)cache->B * 4 : 0, 4, "starts"},
      {cache->block_table, (uint64_t)cache->B * cache->max_pages * 4, 4, "block_table"},
  };
  for (int i = 0; i < 2 && !s; ++i) s = check_written_array(arrays[i], views, 1, arrays, 6);
  if (!s) s = check_operands(views, 1, 0, arrays, 6, nullptr);
  if (s) return s;
  p.q = a->q;
  p.lens = a->lens;
  p.starts = a->starts;
  p.bounds = cache->bounds;
  p.R = a->Hq / cache->H;
  p.first = a->first;
  p.last = a->last;
  p.blocks = a->blocks;
  p.keys = (uint64_t*)a->workspace;
  LaunchSteps step;
  hipError_t e = step([&] { return launch_scores(p, stream); });
  if (e == hipSuccess && select_has_long_rows(p)) e = step([&] { return launch_select(p, stream); });
  if (e != hipSuccess) return fail(HG_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
  return ok();
}

int hg_resize_rows(const hg_page_pool* pool, const hg_resize* a, hipStream_t stream) {
  if (!pool) return fail(HG_ERR_NULL, "pool is NULL");
  if (!a) return fail(HG_ERR_NULL, "args is NULL");
  if (pool->B < 0 || pool->page_size <= 0 || pool->num_pages < 0 || pool->max_pages < 0 || a->N < 0 || pool->B == 0x7FFFFFFF)
    return fail(HG_ERR_SHAPE, "B, page_size, num_pages, max_pages, N = %d, %d, %d, %d, %d", pool->B, pool->page_size,
                pool->num_pages, pool->max_pages, a->N);
  const bool mapped = (a->slots || a->positions) && a->N > 0;
  if (mapped && !a->cu_new) return fail(HG_ERR_NULL, "slots and positions need cu_new");
  const Buf arrays[] = {
      {pool->block_table, (uint64_t)pool->B * pool->max_pages * 4, 4, "block_table"},
      {pool->lens, (uint64_t)pool->B * 4, 4, "lens"},
      {pool->free_pages, (uint64_t)pool->num_pages * 4, 4, "free_pages"},
      {pool->n_free, 4, 4, "n_free"},
      {a->cu_new, a->cu_new ? ((uint64_t)pool->B + 1) * 4 : 0, 4, "cu_new"},
      {a->slots, a->slots ? (uint64_t)a->N * 8 : 0, 8, "slots"},
      {a->positions, a->positions ? (uint64_t)a->N * 4 : 0, 4, "positions"},
      {a->result, 16, 4, "result"},
      {a->targets, (uint64_t)pool->B * 4, 4, "targets"},
  };
  int s = HG_OK;
  for (int i = 0; i < 8 && !s; ++i) s = check_written_array(arrays[i], nullptr, 0, arrays, 9);
  if (!s) s = check_operands(nullptr, 0, 0, arrays, 9, nullptr);
  if (s) return s;
  ResizeParams p;
  p.B = pool->B;
  p.page_size = pool->page_size;
  p.num_pages = pool->num_pages;
  p.max_pages = pool->max_pages;
  p.table = pool->block_table;
  p.lens = pool->lens;
  p.free_pages = pool->free_pages;
  p.n_free = pool->n_free;
  p.N = a->N;
  p.targets = a->targets;
  p.cu = a->cu_new;
  p.slots = a->slots;
  p.positions = a->positions;
  p.result = a->result;
  LaunchSteps step;
  hipError_t e = step([&] { return launch_resize(p, stream); });
  if (e == hipSuccess && mapped && !resize_maps_slots(p)) e = step([&] { return launch_slots(p, stream); });
  if (e != hipSuccess) return fail(HG_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
  return ok();
}

}  // extern "C"
