"""Host-side checks of the 8-bit cache's calls and the page pool, runnable without
a GPU: every refusal comes with its status before any device work."""
import ctypes as C
import math

import pytest
import torch

import cache8ref as ref
import paper_2609_35800_amd as hg
from test_attention_host import G, append, passed, rotation, rows

LIB = hg.library()


def cache8(**kw):
    f = dict(B=2, H=2, D=128, page_size=64, num_pages=8, max_pages=4, block_size=32, page_stride=2 * 64 * 128, head_stride=64 * 128,
             token_stride=128, K=1 * G, V=2 * G, k_scale=20 * G, v_scale=21 * G, bounds=22 * G, block_table=3 * G)
    f.update(kw)
    return hg.hg_cache8(**f)


def decode8(**kw):
    f = dict(Hq=4, scale=0.1, **rows("q", 4 * G, 4), **rows("out", 5 * G, 4), lse=None, lens=6 * G, starts=None,
             workspace=7 * G, workspace_bytes=1 << 30, blocks=None, budget=0)
    f.update(kw)
    return hg.hg_decode8(**f)


def select(**kw):
    f = dict(Hq=4, **rows("q", 4 * G, 4), lens=6 * G, starts=None, blocks=8 * G, budget=3, first=1, last=2, workspace=7 * G,
             workspace_bytes=1 << 30)
    f.update(kw)
    return hg.hg_select(**f)


def pool(**kw):
    f = dict(B=2, page_size=16, num_pages=8, max_pages=4, block_table=1 * G, lens=2 * G, free_pages=3 * G, n_free=4 * G)
    f.update(kw)
    return hg.hg_page_pool(**f)


def resize(**kw):
    f = dict(N=6, targets=5 * G, cu_new=6 * G, slots=7 * G, positions=8 * G, result=9 * G)
    f.update(kw)
    return hg.hg_resize(**f)


def test_sizes_of_the_structures():
    """As a C compiler lays them out: 4-byte fields, then 8-byte ones on 8-byte boundaries."""
    assert C.sizeof(hg.hg_cache8) == 7 * 4 + 4 + 3 * 8 + 6 * 8
    assert C.sizeof(hg.hg_decode8) == 8 + 2 * 24 + 4 * 8 + 8 + 8 + 8
    assert C.sizeof(hg.hg_select) == 8 + 24 + 3 * 8 + 16 + 16
    assert C.sizeof(hg.hg_page_pool) == 16 + 4 * 8
    assert C.sizeof(hg.hg_resize) == 8 + 5 * 8


def test_packed_arguments_match_the_structures():
    for packer, struct_type, n in ((hg._decode8_args, hg.hg_decode8, 15), (hg._select_args, hg.hg_select, 12),
                                   (hg._resize_args, hg.hg_resize, 6)):
        fields = struct_type._fields_
        assert len(fields) == n
        values = [0.5 if t is C.c_float else i + 1 for i, (_, t) in enumerate(fields)]
        raw = packer(*values)
        assert len(raw) == C.sizeof(struct_type)
        got = struct_type.from_buffer_copy(raw)
        assert [getattr(got, f) for f, _ in fields] == values


CACHE = [
    (dict(H=0), hg.HG_ERR_SHAPE), (dict(B=-1), hg.HG_ERR_SHAPE), (dict(D=96), hg.HG_ERR_HEADDIM), (dict(page_size=0), hg.HG_ERR_SHAPE),
    (dict(block_size=0), hg.HG_ERR_SHAPE), (dict(block_size=8), hg.HG_ERR_SHAPE), (dict(block_size=48), hg.HG_ERR_SHAPE),
    (dict(block_size=256), hg.HG_ERR_SHAPE), (dict(page_size=80), hg.HG_ERR_SHAPE), (dict(block_size=128), hg.HG_ERR_SHAPE),
    (dict(block_table=None), hg.HG_ERR_NULL), (dict(K=None), hg.HG_ERR_NULL), (dict(V=2 * G + 8), hg.HG_ERR_ALIGN),
    (dict(token_stride=136), hg.HG_ERR_ALIGN), (dict(head_stride=-128), hg.HG_ERR_SHAPE), (dict(k_scale=None), hg.HG_ERR_NULL),
    (dict(v_scale=21 * G + 2), hg.HG_ERR_ALIGN),
]


@pytest.mark.parametrize("kw,status", CACHE, ids=[str(c[0]) for c in CACHE])
def test_cache_refusals(kw, status):
    c = cache8(**kw)
    assert LIB.hg_append_kv8(c, None, append(), None) == status
    assert hg.hg_last_error()
    assert LIB.hg_decode_attention8(c, decode8(), None) == status


def test_null_arguments():
    n = C.c_uint64()
    assert LIB.hg_append_kv8(None, None, append(), None) == hg.HG_ERR_NULL
    assert LIB.hg_append_kv8(cache8(), None, None, None) == hg.HG_ERR_NULL
    assert LIB.hg_decode_attention8(None, decode8(), None) == hg.HG_ERR_NULL
    assert LIB.hg_decode_attention8(cache8(), None, None) == hg.HG_ERR_NULL
    assert LIB.hg_select_blocks(None, select(), None) == hg.HG_ERR_NULL
    assert LIB.hg_select_blocks(cache8(), None, None) == hg.HG_ERR_NULL
    assert LIB.hg_resize_rows(None, resize(), None) == hg.HG_ERR_NULL
    assert LIB.hg_resize_rows(pool(), None, None) == hg.HG_ERR_NULL
    assert LIB.hg_decode8_workspace(None, 4, C.byref(n)) == hg.HG_ERR_NULL
    assert LIB.hg_decode8_workspace(cache8(), 4, None) == hg.HG_ERR_NULL
    assert LIB.hg_select_workspace(cache8(), None) == hg.HG_ERR_NULL


APPEND = [
    (dict(N=-1), {}, {}, hg.HG_ERR_SHAPE), (dict(cu_new=None), {}, {}, hg.HG_ERR_SHAPE), (dict(v=None), {}, {}, hg.HG_ERR_NULL),
    (dict(lens=None), {}, {}, hg.HG_ERR_NULL), (dict(k=5 * G + 2), {}, {}, hg.HG_ERR_ALIGN),
    (dict(q_out_token_stride=384), {}, {}, hg.HG_ERR_SHAPE), (dict(q_out=4 * G + 256), {}, {}, hg.HG_ERR_POINTER),
    (dict(q_out=1 * G), {}, {}, hg.HG_ERR_POINTER), (dict(k_out=2 * G + 4096), {}, {}, hg.HG_ERR_POINTER),
    (dict(v=1 * G + 64), {}, {}, hg.HG_ERR_POINTER),  # BF16 values within the codes
    (dict(lens=20 * G + 4), {}, {}, hg.HG_ERR_POINTER), (dict(k=22 * G), {}, {}, hg.HG_ERR_POINTER),
    ({}, dict(rot_dim=24), {}, hg.HG_ERR_SHAPE), ({}, dict(section0=16, section1=24, section2=24), {}, hg.HG_ERR_NULL),
    ({}, {}, dict(V=1 * G + 2 * 64 * 128 - 128), hg.HG_ERR_POINTER), ({}, {}, dict(token_stride=112), hg.HG_ERR_SHAPE),
    ({}, {}, dict(v_scale=20 * G + 64), hg.HG_ERR_POINTER), ({}, {}, dict(bounds=2 * G), hg.HG_ERR_POINTER),
    ({}, {}, dict(bounds=22 * G + 8), hg.HG_ERR_ALIGN), ({}, {}, dict(k_scale=3 * G), hg.HG_ERR_POINTER),
]


@pytest.mark.parametrize("kw,rot,c,status", APPEND, ids=[str(c[:3]) for c in APPEND])
def test_append_refusals(kw, rot, c, status):
    assert LIB.hg_append_kv8(cache8(**c), rotation(**rot), append(**kw), None) == status
    assert hg.hg_last_error()


def test_append_calls_without_a_fault():
    assert passed(LIB.hg_append_kv8(cache8(), rotation(), append(), None))
    assert passed(LIB.hg_append_kv8(cache8(bounds=None), None, append(Hq=0, q=None, q_out=None, k_out=None), None))
    assert passed(LIB.hg_append_kv8(cache8(), rotation(), append(N=2, cu_new=None), None))
    # codes of K and V side by side: [pages][2][H][page_size][D]
    c = cache8(V=G + 2 * 64 * 128, page_stride=4 * 64 * 128)
    assert passed(LIB.hg_append_kv8(c, rotation(), append(), None))
    assert LIB.hg_append_kv8(cache8(), rotation(), append(N=0), None) == hg.HG_OK
    assert LIB.hg_append_kv8(cache8(B=0), rotation(), append(N=0, cu_new=None), None) == hg.HG_OK


def test_largest_append():
    a = dict(Hq=0, q=None, q_out=None, k_out=None, k_token_stride=0, v_token_stride=0)
    assert passed(LIB.hg_append_kv8(cache8(), None, append(N=2**29, **a), None))
    assert LIB.hg_append_kv8(cache8(), None, append(N=2**31 - 1, **a), None) == hg.HG_ERR_SHAPE
    c = cache8(B=2**28, block_table=None, max_pages=0, H=64, head_stride=0, page_stride=0, num_pages=0)
    assert LIB.hg_append_kv8(c, None, append(N=2**28, cu_new=None, **a), None) == hg.HG_ERR_SHAPE


def test_append_of_rows_that_begin_later():
    """The rows' first tokens are a read-only array beside the others; NULL is hg_append_kv8."""
    call = LIB.hg_append_kv8_from
    assert passed(call(cache8(), rotation(), append(), 30 * G, None)) and passed(call(cache8(), rotation(), append(), None, None))
    assert passed(call(cache8(), rotation(), append(N=2, cu_new=None), 30 * G, None))
    assert call(cache8(), rotation(), append(), 30 * G + 2, None) == hg.HG_ERR_ALIGN
    for written in (1 * G, 2 * G, 20 * G, 21 * G + 4, 22 * G):
        assert call(cache8(), rotation(), append(), written, None) == hg.HG_ERR_POINTER, written
    a = append()
    for written in (a.q_out, a.k_out):
        assert call(cache8(), rotation(), a, written, None) == hg.HG_ERR_POINTER
    assert passed(call(cache8(), rotation(), a, a.lens, None))  # read as well: rows without tokens
    assert call(None, None, a, 30 * G, None) == hg.HG_ERR_NULL and call(cache8(), None, None, 30 * G, None) == hg.HG_ERR_NULL
    t = torch.zeros(2, 2, dtype=torch.int32)
    c = hg.alloc_cache8(4, 2, 16, 64, t, 16, device="cpu")
    kv, lens = torch.zeros(2, 2, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    for bad in (lens.long(), lens[:1], torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises((TypeError, ValueError)):
            hg.hg_append_kv8(c, None, None, kv, kv, lens, starts=bad, stream=0)


DECODE = [
    (dict(Hq=3), hg.HG_ERR_SHAPE), (dict(Hq=0), hg.HG_ERR_SHAPE), (dict(scale=math.inf), hg.HG_ERR_VALUE), (dict(q=None), hg.HG_ERR_NULL),
    (dict(lens=None), hg.HG_ERR_NULL), (dict(workspace=None), hg.HG_ERR_NULL), (dict(workspace_bytes=1024), hg.HG_ERR_SHAPE),
    (dict(workspace=7 * G + 16), hg.HG_ERR_ALIGN), (dict(out=4 * G), hg.HG_ERR_POINTER), (dict(out=1 * G), hg.HG_ERR_POINTER),
    (dict(out=20 * G), hg.HG_ERR_POINTER), (dict(lse=5 * G), hg.HG_ERR_POINTER), (dict(lse=2 * G + 32), hg.HG_ERR_POINTER),
    (dict(workspace=2 * G), hg.HG_ERR_POINTER), (dict(workspace=21 * G), hg.HG_ERR_POINTER),
    (dict(blocks=8 * G), hg.HG_ERR_SHAPE), (dict(blocks=8 * G, budget=-1), hg.HG_ERR_SHAPE), (dict(budget=4), hg.HG_ERR_SHAPE),
    (dict(blocks=8 * G + 2, budget=4), hg.HG_ERR_ALIGN), (dict(blocks=5 * G, budget=4), hg.HG_ERR_POINTER),
    (dict(blocks=7 * G + 4096, budget=4), hg.HG_ERR_POINTER),
]


@pytest.mark.parametrize("kw,status", DECODE, ids=[str(c[0]) for c in DECODE])
def test_decode_refusals(kw, status):
    assert LIB.hg_decode_attention8(cache8(), decode8(**kw), None) == status
    assert hg.hg_last_error()


def test_decode_calls_without_a_fault():
    assert passed(LIB.hg_decode_attention8(cache8(), decode8(), None))
    assert passed(LIB.hg_decode_attention8(cache8(bounds=None), decode8(blocks=8 * G, budget=5), None))
    assert passed(LIB.hg_decode_attention8(cache8(num_pages=0, K=None, V=None, k_scale=None, v_scale=None), decode8(), None))
    assert LIB.hg_decode_attention8(cache8(B=0), decode8(), None) == hg.HG_OK
    # the BF16 call's workspace
    a, b = C.c_uint64(), C.c_uint64()
    assert LIB.hg_decode8_workspace(cache8(B=70), 40, C.byref(a)) == hg.HG_OK
    paged = hg.hg_paged_cache(B=70, H=2, D=128, page_size=64, num_pages=8, max_pages=4, block_table=3 * G)
    assert LIB.hg_decode_workspace(paged, 40, C.byref(b)) == hg.HG_OK and a.value == b.value


SELECT = [
    (dict(Hq=3), {}, hg.HG_ERR_SHAPE), (dict(budget=0), {}, hg.HG_ERR_SHAPE), (dict(first=-1), {}, hg.HG_ERR_SHAPE),
    (dict(first=2, last=2), {}, hg.HG_ERR_SHAPE), (dict(first=2**31 - 1, last=2**31 - 1), {}, hg.HG_ERR_SHAPE),
    (dict(q=None), {}, hg.HG_ERR_NULL), (dict(lens=None), {}, hg.HG_ERR_NULL), (dict(blocks=None), {}, hg.HG_ERR_NULL),
    (dict(workspace=None), {}, hg.HG_ERR_NULL), (dict(workspace_bytes=8), {}, hg.HG_ERR_SHAPE),
    (dict(workspace=7 * G + 128), {}, hg.HG_ERR_ALIGN), (dict(blocks=4 * G), {}, hg.HG_ERR_POINTER),
    (dict(blocks=22 * G), {}, hg.HG_ERR_POINTER), (dict(workspace=8 * G), {}, hg.HG_ERR_POINTER),
    (dict(blocks=6 * G), {}, hg.HG_ERR_POINTER), ({}, dict(bounds=None), hg.HG_ERR_NULL),
    ({}, dict(bounds=22 * G + 2), hg.HG_ERR_ALIGN), ({}, dict(block_size=24), hg.HG_ERR_SHAPE),
]


@pytest.mark.parametrize("kw,c,status", SELECT, ids=[str(c[:2]) for c in SELECT])
def test_select_refusals(kw, c, status):
    assert LIB.hg_select_blocks(cache8(**c), select(**kw), None) == status
    assert hg.hg_last_error()


def test_select_calls_without_a_fault():
    assert passed(LIB.hg_select_blocks(cache8(), select(), None))
    assert passed(LIB.hg_select_blocks(cache8(), select(budget=1, first=0, last=1), None))
    assert LIB.hg_select_blocks(cache8(B=0), select(), None) == hg.HG_OK
    n = C.c_uint64()
    # too many scores, and too many rows for a launch
    assert LIB.hg_select_workspace(cache8(B=2**30, H=2**10, max_pages=2**30), C.byref(n)) == hg.HG_ERR_SHAPE
    assert LIB.hg_select_blocks(cache8(B=2**22), select(workspace_bytes=2**60), None) == hg.HG_ERR_SHAPE


RESIZE = [
    ({}, dict(B=-1), hg.HG_ERR_SHAPE), ({}, dict(page_size=0), hg.HG_ERR_SHAPE), ({}, dict(num_pages=-1), hg.HG_ERR_SHAPE),
    ({}, dict(max_pages=-1), hg.HG_ERR_SHAPE), (dict(N=-1), {}, hg.HG_ERR_SHAPE), (dict(targets=None), {}, hg.HG_ERR_NULL),
    (dict(result=None), {}, hg.HG_ERR_NULL), (dict(cu_new=None), {}, hg.HG_ERR_NULL), ({}, dict(lens=None), hg.HG_ERR_NULL),
    ({}, dict(n_free=None), hg.HG_ERR_NULL), ({}, dict(free_pages=None), hg.HG_ERR_NULL), ({}, dict(block_table=None), hg.HG_ERR_NULL),
    (dict(slots=7 * G + 4), {}, hg.HG_ERR_ALIGN), (dict(positions=8 * G + 2), {}, hg.HG_ERR_ALIGN),
    (dict(targets=2 * G), {}, hg.HG_ERR_POINTER), (dict(slots=8 * G + 8), {}, hg.HG_ERR_POINTER),
    (dict(result=4 * G - 8), {}, hg.HG_ERR_POINTER), (dict(cu_new=1 * G + 16), {}, hg.HG_ERR_POINTER),
    ({}, dict(n_free=3 * G), hg.HG_ERR_POINTER),
]


@pytest.mark.parametrize("kw,p,status", RESIZE, ids=[str(c[:2]) for c in RESIZE])
def test_resize_refusals(kw, p, status):
    assert LIB.hg_resize_rows(pool(**p), resize(**kw), None) == status
    assert hg.hg_last_error()


def test_resize_calls_without_a_fault():
    assert passed(LIB.hg_resize_rows(pool(), resize(), None))
    assert passed(LIB.hg_resize_rows(pool(), resize(N=0, slots=None, positions=None, cu_new=None), None))
    assert passed(LIB.hg_resize_rows(pool(), resize(slots=None), None))
    assert passed(LIB.hg_resize_rows(pool(B=0, lens=None, block_table=None), resize(targets=None), None))


def test_binding_refuses_wrong_tensors():
    K = torch.zeros(4, 2, 64, 64, dtype=torch.uint8)
    s = torch.ones(4, 2, 2)
    bounds = torch.zeros(4, 2, 2, 2, 64, dtype=torch.bfloat16)
    t = torch.zeros(2, 2, dtype=torch.int32)
    c = hg.make_cache8(K, K.clone(), s, s.clone(), t, bounds)
    assert (c.block_size, c.page_size, c.token_stride) == (32, 64, 64)
    assert hg.make_cache8(K.view(torch.float8_e4m3fn), K.clone().view(torch.float8_e4m3fn), s, s, t).bounds is None
    for bad in (dict(K=K.float()), dict(V=K[:2]), dict(K=K.transpose(2, 3)), dict(k_scale=s.double()), dict(v_scale=s[:, :, :1]),
                dict(k_scale=torch.ones(4, 2, 3)), dict(k_scale=s[0]), dict(block_table=t.long()), dict(bounds=bounds.float()),
                dict(bounds=bounds[:, :, :1]), dict(V=K.view(torch.float8_e4m3fn)), dict(v_scale=s.transpose(0, 1).contiguous().transpose(0, 1))):
        kw = dict(K=K, V=K.clone(), k_scale=s, v_scale=s.clone(), block_table=t, bounds=bounds)
        kw.update(bad)
        with pytest.raises((TypeError, ValueError)):
            hg.make_cache8(**kw)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    kv = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    lens = torch.zeros(2, dtype=torch.int32)
    ws = torch.zeros(1, dtype=torch.uint8)
    blocks = torch.zeros(2, 2, 3, dtype=torch.int32)
    for bad in (dict(q=q.float()), dict(lens=lens.long()), dict(blocks=blocks[0]), dict(blocks=blocks.long()), dict(blocks=blocks[:, :1]),
                dict(workspace=None), dict(workspace=torch.zeros(8, dtype=torch.uint8)[::2]), dict(lse=torch.zeros(2, 3))):
        kw = dict(q=q, lens=lens, out=q.clone(), workspace=ws)
        kw.update(bad)
        with pytest.raises((TypeError, ValueError)):
            hg.hg_decode_attention8(c, **kw, stream=0)
    for bad in (dict(q=q[:1]), dict(blocks=blocks[0]), dict(blocks=None), dict(starts=lens.float()), dict(workspace=None)):
        kw = dict(q=q, lens=lens, blocks=blocks, workspace=ws)
        kw.update(bad)
        with pytest.raises((TypeError, ValueError, AttributeError)):
            hg.hg_select_blocks(c, **kw, stream=0)
    with pytest.raises(ValueError):
        hg.hg_append_kv8(c, None, q, kv, kv[:1], lens, q.clone(), stream=0)
    free = torch.zeros(9, dtype=torch.int32)
    n = torch.zeros(1, dtype=torch.int32)
    p = hg.make_page_pool(t, lens, free, n, 16)
    assert (p.B, p.num_pages, p.max_pages, p.page_size) == (2, 9, 2, 16)
    with pytest.raises((TypeError, ValueError)):
        hg.make_page_pool(t, lens.long(), free, n, 16)
    result = torch.zeros(4, dtype=torch.int32)
    for bad in (dict(targets=lens.long()), dict(result=result[:3]), dict(slots=torch.zeros(3, dtype=torch.int32)),
                dict(slots=torch.zeros(3, dtype=torch.int64), positions=torch.zeros(4, dtype=torch.int32)), dict(cu_new=lens)):
        kw = dict(targets=lens, result=result)
        kw.update(bad)
        with pytest.raises((TypeError, ValueError)):
            hg.hg_resize_rows(p, **kw, stream=0)
    for kw in (dict(targets=None, result=result), dict(targets=lens, result=None)):
        with pytest.raises(hg.HeadGuardError):
            hg.hg_resize_rows(p, **kw, stream=0)


def test_binding_tells_the_kinds_of_caches_apart():
    """A descriptor of one kind is not read as one of another."""
    K = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    t = torch.zeros(2, 2, dtype=torch.int32)
    paged = hg.make_paged_cache(K, K.clone(), t)
    eight = hg.alloc_cache8(4, 2, 16, 64, t, 16, device="cpu")
    assert (eight.block_size, eight.page_size, eight.num_pages) == (16, 16, 4) and len(eight.tensors) == 6
    q, kv = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    lens, ws, blocks = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.uint8), torch.zeros(2, 2, 3, dtype=torch.int32)
    pool = hg.alloc_page_pool(2, 2, 4, 16, device="cpu")
    for call in (lambda: hg.hg_append_kv(eight, None, q, kv, kv, lens, q.clone(), stream=0),
                 lambda: hg.hg_append_kv8(paged, None, q, kv, kv, lens, q.clone(), stream=0),
                 lambda: hg.hg_decode_attention(eight, q, lens, q.clone(), ws, stream=0),
                 lambda: hg.hg_decode_attention8(paged, q, lens, q.clone(), ws, stream=0),
                 lambda: hg.hg_select_blocks(paged, q, lens, blocks, ws, stream=0),
                 lambda: hg.hg_resize_rows(eight, lens, lens, stream=0),
                 lambda: hg.hg_append_kv8(pool, None, q, kv, kv, lens, q.clone(), stream=0)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        hg.alloc_cache8(4, 2, 80, 64, t, 64, device="cpu")
    with pytest.raises(hg.HeadGuardError):  # without bounds there is nothing to choose by
        hg.hg_select_blocks(hg.alloc_cache8(4, 2, 16, 64, t, 16, bounds=False, device="cpu"), q, lens, blocks,
                            torch.zeros(4096, dtype=torch.uint8), stream=0)


# ------------------------------------------------------------ the plain forms that the GPU's are compared with

def test_codes_of_the_plain_form():
    """Against the definition by hand, and torch's conversion in its range."""
    assert ref.VALUES[0x7E] == 448 and ref.VALUES[1] == 2.0 ** -9 and ref.VALUES[0x38] == 1 and math.isnan(ref.VALUES[0xFF])
    x = torch.tensor([0.0, 447.0, 432.0, 431.9, 1.0625, 1.1875, 2.0 ** -10, 1.5 * 2.0 ** -9, 1e9, -math.inf, math.nan], dtype=torch.float64)
    assert ref.VALUES[ref.to_codes(x)[:10].long()].tolist() == [0, 448, 448, 416, 1.0, 1.25, 0, 2.0 ** -8, 448, -448]
    assert int(ref.to_codes(x)[10]) & 0x7F == 0x7F
    y = torch.randn(100000, generator=torch.Generator().manual_seed(0), dtype=torch.float64) * 100
    y = y.clamp(-448, 448)
    assert torch.equal(ref.to_codes(y), y.float().to(torch.float8_e4m3fn).view(torch.uint8))


def test_scales_of_the_plain_form():
    assert ref.scale_of(448.0) == 1 and ref.scale_of(449.0) == 2 and ref.scale_of(224.0) == 0.5 and ref.scale_of(224.5) == 1
    assert ref.scale_of(0.0) == 2.0 ** -100 and ref.scale_of(3.3e38) == 2.0 ** 119


def test_pool_of_the_plain_form():
    p = ref.Pool([[-1, -1], [-1, -1]], [0, 0], [2, 1, 0], 3, 4)
    assert p.resize([5, 3], 10) == ([0, 0, 8, 0], [0, 5, 8], [0, 1, 2, 3, 4, 8, 9, 10, -1, -1], [0, 1, 2, 3, 4, 0, 1, 2, -1, -1])
    assert p.table == [[0, 1], [2, -1]]
    assert p.resize([9, 3], 10)[0] == [2, 0, 0, 0]
    assert p.resize([4, 5], None)[:2] == ([0, 0, 2, 0], [0, 0, 2]) and p.table == [[0, -1], [2, 1]]
