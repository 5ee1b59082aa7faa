"""Host-side checks of the attention calls, runnable without a GPU: every
refusal comes with its status before any device work, and the operands that
may share memory are told from those that may not."""
import ctypes as C
import math

import pytest
import torch

import paper_2609_35800_amd as hg

LIB = hg.library()
G = 1 << 32  # operands 4 GiB apart: never touched


def cache(**kw):
    f = dict(B=2, H=2, D=128, page_size=16, num_pages=8, max_pages=4, page_stride=2 * 16 * 128, head_stride=16 * 128,
             token_stride=128, K=1 * G, V=2 * G, block_table=3 * G)
    f.update(kw)
    return hg.hg_paged_cache(**f)


def rows(name, base, heads, D=128):
    return {name: base, name + "_token_stride": heads * D, name + "_head_stride": D}


def append(**kw):
    f = dict(N=6, Hq=4, **rows("q", 4 * G, 4), **rows("k", 5 * G, 2), **rows("v", 6 * G, 2), **rows("q_out", 7 * G, 4),
             **rows("k_out", 8 * G, 2), lens=9 * G, cu_new=10 * G, positions=None)
    f.update(kw)
    return hg.hg_append(**f)


def rotation(**kw):
    f = dict(cos=11 * G, sin=12 * G, max_pos=100, rot_dim=128, interleaved=0, section0=0, section1=0, section2=0)
    f.update(kw)
    return hg.hg_rotation(**f)


def decode(**kw):
    f = dict(Hq=4, scale=0.1, **rows("q", 4 * G, 4), **rows("out", 5 * G, 4), lse=None, lens=6 * G, starts=None,
             workspace=7 * G, workspace_bytes=1 << 30)
    f.update(kw)
    return hg.hg_decode(**f)


def prefill(**kw):
    f = dict(B=2, Hq=4, H=2, D=128, Nq=6, Nk=6, causal=1, scale=0.1, **rows("q", 4 * G, 4), **rows("k", 5 * G, 2),
             **rows("v", 6 * G, 2), **rows("out", 7 * G, 4), lse=None, cu_q=8 * G, cu_k=None)
    f.update(kw)
    return hg.hg_prefill(**f)


# What a call without a fault gives here: no device, or the made-up addresses refused.
PASSED = (hg.HG_ERR_NO_DEVICE, hg.HG_ERR_POINTER)


def passed(rc):
    return rc in PASSED and "overlap" not in hg.hg_last_error()


CACHE = [
    (dict(H=0), hg.HG_ERR_SHAPE), (dict(B=-1), hg.HG_ERR_SHAPE), (dict(page_size=0), hg.HG_ERR_SHAPE),
    (dict(num_pages=-1), hg.HG_ERR_SHAPE), (dict(max_pages=-1), hg.HG_ERR_SHAPE), (dict(D=96), hg.HG_ERR_HEADDIM),
    (dict(block_table=None), hg.HG_ERR_NULL), (dict(block_table=3 * G + 2), hg.HG_ERR_ALIGN),
    (dict(K=None), hg.HG_ERR_NULL), (dict(V=2 * G + 8), hg.HG_ERR_ALIGN), (dict(token_stride=132), hg.HG_ERR_ALIGN),
    (dict(head_stride=-128), hg.HG_ERR_SHAPE),
]


@pytest.mark.parametrize("kw,status", CACHE, ids=[str(c[0]) for c in CACHE])
def test_cache_refusals(kw, status):
    c = cache(**kw)
    assert LIB.hg_append_kv(c, None, append(), None) == status
    assert hg.hg_last_error()
    assert LIB.hg_decode_attention(c, decode(), None) == status


APPEND = [
    (dict(N=-1), {}, hg.HG_ERR_SHAPE), (dict(Hq=-1), {}, hg.HG_ERR_SHAPE), (dict(cu_new=None), {}, hg.HG_ERR_SHAPE),
    (dict(q=None), {}, hg.HG_ERR_NULL), (dict(v=None), {}, hg.HG_ERR_NULL), (dict(lens=None), {}, hg.HG_ERR_NULL),
    (dict(k=5 * G + 2), {}, hg.HG_ERR_ALIGN), (dict(q_token_stride=516), {}, hg.HG_ERR_ALIGN),
    (dict(q_token_stride=-512), {}, hg.HG_ERR_SHAPE),
    (dict(q_out_token_stride=384), {}, hg.HG_ERR_SHAPE),    # its rows overlap
    (dict(q_out=4 * G + 256), {}, hg.HG_ERR_POINTER),       # partly q
    (dict(k_out=4 * G), {}, hg.HG_ERR_POINTER), (dict(q_out=1 * G), {}, hg.HG_ERR_POINTER),
    (dict(lens=8 * G + 16), {}, hg.HG_ERR_POINTER),
    ({}, dict(rot_dim=24), hg.HG_ERR_SHAPE), ({}, dict(rot_dim=144), hg.HG_ERR_SHAPE),
    ({}, dict(rot_dim=-16), hg.HG_ERR_SHAPE), ({}, dict(max_pos=0), hg.HG_ERR_SHAPE),
    ({}, dict(interleaved=2), hg.HG_ERR_SHAPE), ({}, dict(cos=None), hg.HG_ERR_NULL),
    ({}, dict(sin=12 * G + 4), hg.HG_ERR_ALIGN), ({}, dict(section0=16, section1=24, section2=25), hg.HG_ERR_SHAPE),
    (dict(positions=13 * G), dict(section0=-16, section1=56, section2=24), hg.HG_ERR_SHAPE),
    ({}, dict(section0=16, section1=24, section2=24), hg.HG_ERR_NULL),  # no positions
]


@pytest.mark.parametrize("kw,rot,status", APPEND, ids=[str(c[:2]) for c in APPEND])
def test_append_refusals(kw, rot, status):
    assert LIB.hg_append_kv(cache(), rotation(**rot), append(**kw), None) == status
    assert hg.hg_last_error()


def test_append_nulls_and_empty_calls():
    assert LIB.hg_append_kv(None, None, append(), None) == hg.HG_ERR_NULL
    assert LIB.hg_append_kv(cache(), None, None, None) == hg.HG_ERR_NULL
    assert LIB.hg_append_kv(cache(), rotation(), append(N=0), None) == hg.HG_OK
    assert LIB.hg_append_kv(cache(B=0), rotation(), append(N=0, cu_new=None), None) == hg.HG_OK
    assert passed(LIB.hg_append_kv(cache(), rotation(), append(), None))
    # no queries, no packed keys, no rotation
    a = append(Hq=0, q=None, q_out=None, k_out=None)
    assert passed(LIB.hg_append_kv(cache(), None, a, None))


def test_views_of_one_tensor_are_told_apart():
    # q, k, v of one fused projection [N][4 + 2 + 2][128], rotated in place
    ts = 8 * 128
    base = 4 * G
    fused = dict(q=base, q_token_stride=ts, k=base + 4 * 256, k_token_stride=ts, v=base + 6 * 256, v_token_stride=ts,
                 q_out=base, q_out_token_stride=ts, k_out=base + 4 * 256, k_out_token_stride=ts)
    assert passed(LIB.hg_append_kv(cache(), rotation(), append(**fused), None))
    # keys before queries
    other = dict(fused, k=base, k_out=base, q=base + 2 * 256, q_out=base + 2 * 256)
    assert passed(LIB.hg_append_kv(cache(), rotation(), append(**other), None))
    # q_out on top of the keys, or one head further than q
    for bad in (dict(fused, q_out=base + 2 * 256), dict(fused, q_out=base + 256), dict(fused, k_out=base + 5 * 256)):
        assert LIB.hg_append_kv(cache(), rotation(), append(**bad), None) == hg.HG_ERR_POINTER
        assert "overlaps" in hg.hg_last_error()
    # K and V of one tensor: [pages][2][H][page_size][D], and [pages][H][page_size][2][D]
    c = cache(K=G, V=G + 2 * 16 * 128 * 2, page_stride=2 * 2 * 16 * 128)
    assert passed(LIB.hg_append_kv(c, rotation(), append(), None))
    c = cache(K=G, V=G + 256, page_stride=2 * 2 * 16 * 128, head_stride=2 * 16 * 128, token_stride=256)
    assert passed(LIB.hg_append_kv(c, rotation(), append(), None))
    for V in (G, G + 256, G + 2 * 16 * 128 * 2):
        assert LIB.hg_append_kv(cache(K=G, V=V), rotation(), append(), None) == hg.HG_ERR_POINTER
    # tokens of a page on top of one another
    assert LIB.hg_append_kv(cache(token_stride=64), rotation(), append(), None) == hg.HG_ERR_SHAPE


DECODE = [
    (dict(Hq=3), hg.HG_ERR_SHAPE), (dict(Hq=0), hg.HG_ERR_SHAPE), (dict(scale=math.inf), hg.HG_ERR_VALUE),
    (dict(scale=math.nan), hg.HG_ERR_VALUE), (dict(scale=3e38), hg.HG_ERR_VALUE), (dict(q=None), hg.HG_ERR_NULL),
    (dict(out=None), hg.HG_ERR_NULL), (dict(lens=None), hg.HG_ERR_NULL), (dict(workspace=None), hg.HG_ERR_NULL),
    (dict(workspace_bytes=1024), hg.HG_ERR_SHAPE), (dict(workspace=7 * G + 16), hg.HG_ERR_ALIGN),
    (dict(out=4 * G), hg.HG_ERR_POINTER), (dict(out=1 * G), hg.HG_ERR_POINTER), (dict(out=7 * G + 4096), hg.HG_ERR_POINTER),
    (dict(lse=5 * G), hg.HG_ERR_POINTER), (dict(lse=6 * G + 4), hg.HG_ERR_POINTER), (dict(lse=2), hg.HG_ERR_ALIGN),
    (dict(workspace=2 * G), hg.HG_ERR_POINTER), (dict(out_head_stride=64), hg.HG_ERR_SHAPE),
]


@pytest.mark.parametrize("kw,status", DECODE, ids=[str(c[0]) for c in DECODE])
def test_decode_refusals(kw, status):
    assert LIB.hg_decode_attention(cache(), decode(**kw), None) == status
    assert hg.hg_last_error()


def test_decode_workspace_and_empty_calls():
    n = C.c_uint64()
    # counters of the (row, head, tile of 16 query heads) and of 1024 slots, then the slots' results
    assert LIB.hg_decode_workspace(cache(B=70), 40, C.byref(n)) == hg.HG_OK
    assert n.value == -(-(70 * 2 * 2 + 1024) * 4 // 256) * 256 + 1024 * 16 * (128 + 2) * 4
    assert LIB.hg_decode_workspace(cache(), 4, None) == hg.HG_ERR_NULL
    assert LIB.hg_decode_workspace(cache(), 5, C.byref(n)) == hg.HG_ERR_SHAPE
    assert LIB.hg_decode_attention(None, decode(), None) == hg.HG_ERR_NULL
    assert LIB.hg_decode_attention(cache(), None, None) == hg.HG_ERR_NULL
    assert LIB.hg_decode_attention(cache(B=0), decode(), None) == hg.HG_OK
    assert passed(LIB.hg_decode_attention(cache(), decode(), None))
    assert passed(LIB.hg_decode_attention(cache(num_pages=0, K=None, V=None), decode(), None))


PREFILL = [
    (dict(B=-1), hg.HG_ERR_SHAPE), (dict(H=0), hg.HG_ERR_SHAPE), (dict(Nq=-1), hg.HG_ERR_SHAPE),
    (dict(causal=2), hg.HG_ERR_SHAPE), (dict(D=80), hg.HG_ERR_HEADDIM), (dict(Hq=5), hg.HG_ERR_SHAPE),
    (dict(scale=math.nan), hg.HG_ERR_VALUE), (dict(Nk=7), hg.HG_ERR_SHAPE), (dict(cu_q=None), hg.HG_ERR_NULL),
    (dict(k=None), hg.HG_ERR_NULL), (dict(v=6 * G + 4), hg.HG_ERR_ALIGN), (dict(v_head_stride=4), hg.HG_ERR_ALIGN),
    (dict(out=4 * G), hg.HG_ERR_POINTER), (dict(lse=7 * G), hg.HG_ERR_POINTER), (dict(lse=8 * G), hg.HG_ERR_POINTER),
    (dict(out_token_stride=0), hg.HG_ERR_SHAPE), (dict(Nq=1 << 30, Nk=1 << 30, Hq=256, H=256), hg.HG_ERR_SHAPE),
]


@pytest.mark.parametrize("kw,status", PREFILL, ids=[str(c[0]) for c in PREFILL])
def test_prefill_refusals(kw, status):
    assert LIB.hg_prefill_attention(prefill(**kw), None) == status
    assert hg.hg_last_error()


def test_prefill_empty_calls():
    assert LIB.hg_prefill_attention(None, None) == hg.HG_ERR_NULL
    assert LIB.hg_prefill_attention(prefill(B=0), None) == hg.HG_OK
    assert LIB.hg_prefill_attention(prefill(Nq=0, Nk=0), None) == hg.HG_OK
    assert passed(LIB.hg_prefill_attention(prefill(), None))
    assert passed(LIB.hg_prefill_attention(prefill(k_token_stride=0, k_head_stride=0), None))  # a broadcast key


def test_largest_launches():
    """A launch of 2^32 work-items is refused by the runtime, one of more cut short in silence."""
    # append, two 128-channel KV heads: four tokens a workgroup of 256
    a = dict(Hq=0, q=None, q_out=None, k_out=None, k_token_stride=0, v_token_stride=0)
    most = 4 * ((2**32 - 1) // 256)
    assert passed(LIB.hg_append_kv(cache(), None, append(N=most, **a), None))
    for n in (most + 1, 2**31 - 1):
        assert LIB.hg_append_kv(cache(), None, append(N=n, **a), None) == hg.HG_ERR_SHAPE
    # prefill of rows of one query: tiles of 128 queries and 256 work-items; of many keys: 256 and 512
    p = dict(H=1, out=16 * G, q_token_stride=0, k_token_stride=0, v_token_stride=0, cu_k=9 * G)
    for D, Hq, keys, tile in ((64, 64, 1, 128), (256, 16, 1, 128), (128, 64, 1, 128), (128, 64, 1700, 256)):
        slots = (2**32 - 1) // (2 * tile) // Hq
        most = next(n for n in range(slots, 0, -1) if n + n // tile <= slots)
        for n in (most, most + 1):
            rc = LIB.hg_prefill_attention(prefill(B=n, Nq=n, Nk=n * keys, Hq=Hq, D=D, **p, out_token_stride=Hq * D,
                                                  out_head_stride=D), None)
            assert passed(rc) if n == most else rc == hg.HG_ERR_SHAPE, (D, n)


def test_most_keys():
    """Keys so many that a tile or stage past the last one could not be counted in 32 bits."""
    for n, ok in ((2**31 - 513, True), (2**31 - 512, False), (2**31 - 1, False)):
        rc = LIB.hg_prefill_attention(prefill(Nk=n, k_token_stride=0, v_token_stride=0, cu_k=9 * G), None)
        assert passed(rc) if ok else rc == hg.HG_ERR_SHAPE, n


def test_binding_refuses_wrong_tensors():
    K = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    t = torch.zeros(2, 2, dtype=torch.int32)
    c = hg.make_paged_cache(K, K.clone(), t)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    ws = torch.zeros(1, dtype=torch.uint8)
    lens = torch.zeros(2, dtype=torch.int32)
    for bad in (dict(q=q.float()), dict(q=q[:1]), dict(q=q.transpose(1, 2)), dict(lens=lens.long()), dict(lens=lens[:1]),
                dict(out=q[:, :2]), dict(lse=torch.zeros(2, 3)), dict(lse=torch.zeros(2, 4, dtype=torch.float64))):
        kw = dict(q=q, lens=lens, out=q.clone(), workspace=ws)
        kw.update(bad)
        with pytest.raises((TypeError, ValueError)):
            hg.hg_decode_attention(c, **kw)
    with pytest.raises(ValueError):
        hg.make_paged_cache(K, K.transpose(1, 2).contiguous(), t)
    with pytest.raises(TypeError):
        hg.make_paged_cache(K.float(), K.float(), t)
    with pytest.raises(ValueError):
        hg.make_paged_cache(K, K.clone(), t.t())
    with pytest.raises(TypeError):
        hg.make_rotation(torch.zeros(4, 32, dtype=torch.float64), torch.zeros(4, 32))
    kv = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    for bad in (dict(v=kv[:1]), dict(q_out=None), dict(positions=torch.zeros(3, 2, dtype=torch.int32)),
                dict(cu_new=torch.zeros(2, dtype=torch.int32))):
        kw = dict(rotation=None, q=q, k=kv, v=kv, lens=lens, q_out=q.clone())
        kw.update(bad)
        with pytest.raises((TypeError, ValueError)):
            hg.hg_append_kv(c, **kw)


def test_binding_refuses_a_workspace_with_gaps():
    """The call writes workspace_bytes bytes from the workspace's address on."""
    K = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    c = hg.make_paged_cache(K, K.clone(), torch.zeros(2, 2, dtype=torch.int32))
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    lens = torch.zeros(2, dtype=torch.int32)
    whole = torch.zeros(2 * hg.hg_decode_workspace(c, 4), dtype=torch.uint8)
    for bad in (whole[::2], whole.view(2, -1).t(), whole[:1].expand(whole.numel())):
        with pytest.raises(ValueError):
            hg.hg_decode_attention(c, q, lens, q.clone(), bad, stream=0)
    with pytest.raises(ValueError):
        hg.hg_decode_attention(c, q, lens, q.clone(), None, stream=0)
    with pytest.raises(hg.HeadGuardError) as e:  # contiguous: only host memory is wrong with it
        hg.hg_decode_attention(c, q, lens, q.clone(), whole.view(2, -1)[1], stream=0)
    assert e.value.status in (hg.HG_ERR_NO_DEVICE, hg.HG_ERR_POINTER, hg.HG_ERR_ALIGN)


def test_descriptors_built_from_their_classes():
    """hg_paged_cache and hg_rotation are public structures: one filled by hand is as
    good as one of make_paged_cache or make_rotation, changed fields and copies too."""
    q, kv = torch.zeros(2, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 2, 128, dtype=torch.bfloat16)
    lens, pos3 = torch.zeros(2, dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32)
    out = torch.zeros_like(q)
    by_hand = hg.hg_paged_cache.from_buffer_copy(cache())
    for c in (cache(), by_hand):
        for r, positions in ((rotation(), None), (rotation(section0=16, section1=24, section2=24), pos3)):
            with pytest.raises(hg.HeadGuardError) as e:
                hg.hg_append_kv(c, r, q, kv, kv, lens, out, positions=positions, stream=0)
            assert passed(e.value.status)
        with pytest.raises(hg.HeadGuardError) as e:
            hg.hg_decode_attention(c, q, lens, out, torch.zeros(1, dtype=torch.uint8), stream=0)
        assert e.value.status == hg.HG_ERR_SHAPE  # the workspace
    with pytest.raises(ValueError):  # three axes
        hg.hg_append_kv(cache(), rotation(section0=16, section1=24, section2=24), q, kv, kv, lens, out,
                        positions=pos3[0].contiguous(), stream=0)
    K = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    made = hg.make_paged_cache(K, K.clone(), torch.zeros(2, 2, dtype=torch.int32))
    made.D = 96
    with pytest.raises(hg.HeadGuardError) as e:
        hg.hg_decode_attention(made, q[..., :96], lens, out[..., :96], torch.zeros(1, dtype=torch.uint8), stream=0)
    assert e.value.status == hg.HG_ERR_HEADDIM


def test_pages_of_one_head_page_or_token():
    """Strides of a dimension of one index do not matter, those of K and V may differ there."""
    table = torch.zeros(2, 2, dtype=torch.int32)
    tokens_first = torch.zeros(4, 16, 1, 64, dtype=torch.bfloat16).transpose(1, 2)
    heads_first = torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16)
    assert tokens_first.shape == heads_first.shape and tokens_first.stride() != heads_first.stride()
    c = hg.make_paged_cache(tokens_first, heads_first, table)
    assert (c.page_stride, c.token_stride) == (16 * 64, 64)
    wide = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    c = hg.make_paged_cache(wide[::2][:1], wide[2:], table)  # one page
    assert (c.head_stride, c.token_stride) == (16 * 64, 64)
    one = torch.zeros(3, 2, 1, 64, dtype=torch.bfloat16)  # pages of one token
    c = hg.make_paged_cache(one, one.clone().as_strided(one.shape, (128, 64, 8, 1)), table)
    assert (c.page_stride, c.head_stride) == (128, 64)
    with pytest.raises(ValueError):
        hg.make_paged_cache(wide, wide.transpose(0, 1).contiguous().transpose(0, 1), table)


def test_packed_arguments_match_the_structures():
    """The binding packs the argument structures into bytes: same size, same fields."""
    for packer, struct_type, n in ((hg._append_args, hg.hg_append, 20), (hg._prefill_args, hg.hg_prefill, 23),
                                   (hg._decode_args, hg.hg_decode, 13)):
        fields = struct_type._fields_
        assert len(fields) == n
        values = [0.5 if t is C.c_float else i + 1 for i, (_, t) in enumerate(fields)]
        raw = packer(*values)
        assert len(raw) == C.sizeof(struct_type)
        got = struct_type.from_buffer_copy(raw)
        assert [getattr(got, f) for f, _ in fields] == values
