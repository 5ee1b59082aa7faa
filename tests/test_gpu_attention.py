"""The attention calls (append, prefill, decode) on the GPU against plain
64-bit forms on the CPU, at the sizes, layouts and masks where they can go
wrong; bounds derived in attnref."""
import math
import random

import pytest
import torch

import attnref
from attnref import assert_close

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def randn(g, *shape):
    return torch.randn(*shape, generator=g).to(BF)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def bits(t):
    return t.contiguous().view(torch.int16)


def make_pages(lens, H, D, page_size, seed, token_major=False, interleaved_kv=False, spare=3, fill=float("nan")):
    """Pages filled with `fill`, a shuffled block table for rows of `lens` tokens.
    Returns K, V [pages, H, page_size, D] (views on the GPU), the table (host)."""
    need = [-(-n // page_size) for n in lens]
    total = sum(need) + spare
    order = list(range(total))
    random.Random(seed).shuffle(order)
    cols = max(max(need), 1) + 1
    rows, at = [], 0
    for n in need:
        rows.append(order[at:at + n] + [-7] * (cols - n))  # entries past a row's pages are not read
        at += n
    shape = (total, page_size, H, D) if token_major else (total, H, page_size, D)
    if interleaved_kv:
        kv = torch.full((shape[0], 2) + shape[1:], fill, dtype=BF, device="cuda")
        K, V = kv[:, 0], kv[:, 1]
    else:
        K = torch.full(shape, fill, dtype=BF, device="cuda")
        V = torch.full(shape, fill, dtype=BF, device="cuda")
    if token_major:
        K, V = K.transpose(1, 2), V.transpose(1, 2)
    return K, V, rows


def put(K, rows, b, t0, x):
    """Write x [n, H, D] to tokens t0.. of row b."""
    ps = K.shape[2]
    t = torch.arange(t0, t0 + x.shape[0])
    page = torch.tensor(rows[b])[t // ps]
    K[page.cuda(), :, (t % ps).cuda()] = x.cuda()


# ------------------------------------------------------------ append

APPEND = [  # D, Hq, H, rot, interleaved, sections, page_size, token_major, new lengths (None: one token a row)
    (128, 28, 4, 128, 0, (16, 24, 24), 16, False, None),
    (128, 8, 8, 128, 1, None, 16, True, [5, 0, 1, 40]),
    (64, 6, 2, 32, 0, None, 7, False, [33, 2]),
    (64, 3, 3, 48, 1, (8, 12, 4), 1, False, [3, 9, 1]),
    (256, 16, 8, 256, 0, None, 64, False, [65]),
    (256, 1, 1, 64, 0, (9, 13, 10), 100, True, [101, 1]),
    (128, 64, 1, 0, 0, None, 32, False, [2, 31]),
    (64, 130, 70, 64, 0, None, 16, False, [4]),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", APPEND, ids=str)
def test_append(case, in_place):
    import paper_2609_35800_amd as hg
    D, Hq, H, rot, inter, sections, ps, token_major, new = case
    g = gen(D + Hq)
    B = 3 if new is None else len(new)
    n_new = [1] * B if new is None else new
    before = [random.Random(b).choice([0, 1, ps - 1, ps, 37]) for b in range(B)]
    lens = [a + n for a, n in zip(before, n_new)]
    K, V, rows = make_pages(lens, H, D, ps, 5, token_major, interleaved_kv=not token_major)
    k0, v0 = bits(K).clone(), bits(V).clone()
    N = sum(n_new)
    qkv = randn(g, N, Hq + 2 * H, D)
    dev = qkv.cuda()
    q, k, v = dev[:, :Hq], dev[:, Hq:Hq + H], dev[:, Hq + H:]
    q_out = q if in_place else torch.zeros(N, Hq, D, dtype=BF, device="cuda")
    k_out = k if in_place else None
    max_pos = 400
    cos, sin = attnref.table(max_pos, max(rot // 2, 1))
    rotation = hg.make_rotation(cos.cuda(), sin.cuda(), inter, sections) if rot else None
    positions = torch.randint(0, max_pos, (3, N) if sections else (N,), generator=g, dtype=torch.int32)
    use_positions = sections is not None or inter == 1
    cu = [0]
    for n in n_new:
        cu.append(cu[-1] + n)
    cache = hg.make_paged_cache(K, V, i32(rows))
    hg.hg_append_kv(cache, rotation, q, k, v, i32(lens), q_out, cu_new=None if new is None else i32(cu),
                    positions=positions.cuda() if use_positions else None, k_out=k_out)
    torch.cuda.synchronize()
    Kh, Vh, qh = K.cpu(), V.cpu(), q_out.cpu()
    written = torch.zeros(K.shape[0], ps, dtype=torch.bool)
    for b in range(B):
        for j in range(n_new[b]):
            t, idx = cu[b] + j, before[b] + j
            page, off = rows[b][idx // ps], idx % ps
            written[page, off] = True
            if rot:
                i = torch.arange(rot // 2)
                if sections:
                    axis = (i >= sections[0]).long() + (i >= sections[0] + sections[1]).long()
                    pos = positions[axis, t].long()
                else:
                    pos = torch.full((rot // 2,), int(positions[t]) if use_positions else idx)
                c, s = cos[pos, i], sin[pos, i]
            else:
                c = s = torch.zeros(0)
            wq, tq = attnref.rotate(qkv[t, :Hq], c, s, inter)
            wk, tk = attnref.rotate(qkv[t, Hq:Hq + H], c, s, inter)
            assert_close(qh[t], wq, tq, f"q of token {t}")
            assert_close(Kh[page, :, off], wk, tk, f"key of token {t}")
            assert torch.equal(bits(Vh[page, :, off]), bits(qkv[t, Hq + H:])), f"value of token {t}"
            if in_place:
                assert torch.equal(bits(k[t].cpu()), bits(Kh[page, :, off]))
    keep = ~written.view(-1, 1, ps, 1).expand(K.shape).cuda()
    assert bool((bits(K) == k0)[keep].all()) and bool((bits(V) == v0)[keep].all()), "other tokens were written"
    if not in_place:
        assert torch.equal(bits(dev), bits(qkv.cuda()))


@pytest.mark.parametrize("D,inter", [(64, 0), (128, 1), (256, 0)])
def test_append_large_calls(D, inter):
    """Calls past 256 MiB stream; every element against the bound, in 64 bits."""
    import paper_2609_35800_amd as hg
    Hq, H, ps = 3, 2, 100
    lens = [(300 << 20) // (4 * D * (Hq + 2 * H)) - 77, 77]
    K, V, rows = make_pages(lens, H, D, ps, 1, fill=0.0)
    N = sum(lens)
    gpu = torch.Generator(device="cuda").manual_seed(D)
    qkv = torch.randn((N, Hq + 2 * H, D), generator=gpu, device="cuda").to(BF)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    cos, sin = (t.cuda() for t in attnref.table(max(lens), D // 2))
    q_out = torch.zeros((N, Hq, D), dtype=BF, device="cuda")
    cu = [0, lens[0], N]
    hg.hg_append_kv(hg.make_paged_cache(K, V, i32(rows)), hg.make_rotation(cos, sin, inter), q, k, v, i32(lens), q_out,
                    cu_new=i32(cu))
    torch.cuda.synchronize()
    pos = torch.cat([torch.arange(n, device="cuda") for n in lens])
    c, s = cos[pos].double().unsqueeze(1), sin[pos].double().unsqueeze(1)
    a, b = (slice(0, None, 2), slice(1, None, 2)) if inter else (slice(0, D // 2), slice(D // 2, D))
    where = torch.cat([torch.tensor(rows[i], device="cuda")[torch.arange(n, device="cuda") // ps] for i, n in enumerate(lens)])
    off = torch.cat([torch.arange(n, device="cuda") % ps for n in lens])
    for got, x in ((q_out, q), (K[where, :, off], k)):
        xa, xb = x[..., a].double(), x[..., b].double()
        for part, one, two, sign in ((a, xa, xb, -1), (b, xb, xa, 1)):
            want = one * c + sign * two * s
            tol = want.abs() * 2.0 ** -8 * (1 + 2.0 ** -6) + 2.0 ** -21 * ((one * c).abs() + (two * s).abs())
            assert bool(((got[..., part].double() - want).abs() <= tol).all())
    assert torch.equal(bits(V[where, :, off]), bits(v))


def test_append_skips_what_has_no_place():
    """Padding tokens, pages outside the cache, indexes past the table and
    positions outside the rotation's: no other byte changes."""
    import paper_2609_35800_amd as hg
    D, Hq, H, ps = 64, 2, 2, 4
    g = gen(3)
    K = torch.full((4, H, ps, D), float("nan"), dtype=BF, device="cuda")
    V = K.clone()
    table = i32([[0, 9], [1, -1], [2, 3]])  # 9 and -1: no such pages
    cu = i32([0, 3, 4, 6])                  # tokens 6 and 7 belong to no row
    N = 8
    q, k, v = (randn(g, N, Hq, D).cuda() for _ in range(3))
    q_out = torch.full_like(q, float("nan"))
    cos, sin = attnref.table(10, D // 2)
    lens = i32([5, 5, 10])      # row 0: tokens 2, 3, 4 (4: page 9); row 1: token 4 (page -1); row 2: tokens 8, 9 (past the table)
    positions = i32([0, 1, 2, 3, 10, -1, 0, 0])  # tokens 4 and 5: outside
    cache = hg.make_paged_cache(K, V, table)
    hg.hg_append_kv(cache, hg.make_rotation(cos.cuda(), sin.cuda()), q, k, v, lens, q_out, cu_new=cu, positions=positions)
    torch.cuda.synchronize()
    got = torch.isfinite(K.float()).all(-1).all(1).cpu()
    want = torch.zeros(4, ps, dtype=torch.bool)
    want[0, 2] = want[0, 3] = True
    assert torch.equal(got, want) and torch.equal(torch.isfinite(V.float()).all(-1).all(1).cpu(), want)
    assert torch.isfinite(q_out.float()).all(-1).all(1).cpu().tolist() == [True] * 4 + [False] * 4


# ------------------------------------------------------------ decode

def check_decode(lens, Hq, H, D, ps, seed=0, starts=None, token_major=False, interleaved_kv=False, scale=None,
                 peak=1.0, calls=1, q_pad=0, stream=None):
    import paper_2609_35800_amd as hg
    g = gen(seed)
    B = len(lens)
    K, V, rows = make_pages(lens, H, D, ps, seed, token_major, interleaved_kv)
    first = starts or [0] * B
    host = []
    for b in range(B):
        lo = min(first[b], lens[b])
        k, v = randn(g, lens[b] - lo, H, D) * peak, randn(g, lens[b] - lo, H, D)
        host.append((k, v))
        if lens[b] > lo:  # tokens outside [first, len) stay NaN
            put(K, rows, b, lo, k)
            put(V, rows, b, lo, v)
    q = randn(g, B, Hq, D)
    wide = torch.zeros(B, Hq + q_pad, D, dtype=BF, device="cuda")
    wide[:, :Hq] = q.cuda()
    out = torch.full((B, Hq, D), float("nan"), dtype=BF, device="cuda")
    lse = torch.full((B, Hq), float("nan"), dtype=torch.float32, device="cuda")
    cache = hg.make_paged_cache(K, V, i32(rows))
    ws = hg.alloc_decode_workspace(cache, Hq)
    s = D ** -0.5 if scale is None else scale
    args = (cache, wide[:, :Hq], i32(lens), out, ws)
    kw = dict(starts=None if starts is None else i32(starts), lse=lse, scale=scale, stream=stream)
    torch.cuda.synchronize()
    hg.hg_decode_attention(*args, **kw)
    torch.cuda.synchronize()
    o1, l1 = out.clone(), lse.clone()
    for _ in range(calls - 1):  # the workspace is ready again, the result the same
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        torch.cuda.synchronize()
        hg.hg_decode_attention(*args, **kw)
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(o1)) and torch.equal(lse, l1)
    G = Hq // H
    for b in range(B):
        for h in range(H):
            k, v = host[b]
            o, l, to, tl = attnref.attend(q[b, h * G:(h + 1) * G], k[:, h], v[:, h], s)
            assert_close(out[b, h * G:(h + 1) * G], o, to, f"row {b} head {h} of {lens[b]} tokens")
            assert_close(lse[b, h * G:(h + 1) * G], l, tl, f"lse of row {b} head {h}")


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,H", [(4, 4), (14, 2), (8, 1), (17, 1), (40, 1)])
def test_decode_lengths(D, Hq, H):
    check_decode([0, 1, 2, 31, 32, 33, 64, 255, 256, 257, 600], Hq, H, D, 16, seed=D + Hq, calls=2)


@pytest.mark.parametrize("ps", [1, 3, 7, 32, 100, 700])
def test_decode_page_sizes(ps):
    check_decode([ps, 3 * ps - 1 if ps < 300 else 699, 500, 1], 6, 2, 128, ps, seed=ps, token_major=ps % 2 == 0,
                 interleaved_kv=ps % 2 == 1, q_pad=3)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_decode_starts(D):
    """Left-padded rows and windows; rows that the start leaves empty."""
    check_decode([300, 300, 300, 300, 300, 5], 4, 2, D, 16, seed=D, starts=[0, 1, 33, 299, 300, 9])


@pytest.mark.parametrize("B", [63, 64, 65, 200])
def test_decode_many_rows(B):
    lens = [random.Random(b).choice([0, 1, 5, 40, 90]) for b in range(B)]
    check_decode(lens, 4, 2, 64, 16, seed=B, calls=3)


def test_decode_one_long_row():
    """One row over every workgroup, and beside short ones."""
    check_decode([40001], 4, 1, 128, 64, seed=1, calls=3)
    check_decode([3, 30000, 0, 17], 2, 1, 64, 16, seed=2, calls=3)


# rows of tokens, Hq, H, D: calls one after the other, cut into segments (up to 256
# (row, head, tile)s) and into even shares (more), joined in one step and in two.
_RAGGED = [700, 40, 1, 2000, 333, 0, 64, 1500]
CHANGING = [
    [([50] * 40 + [700] * 24, 32, 32, 128), (_RAGGED * 2, 32, 32, 128), ([50] * 40 + [700] * 24, 32, 32, 128)],
    [([900, 20, 3000] * 30, 8, 4, 128), ([9000], 8, 4, 128), ([900, 20, 3000] * 30, 8, 4, 128), ([9000, 5], 8, 4, 128)],
    [(_RAGGED, 40, 1, 64), ([5000, 77], 4, 2, 256), (_RAGGED * 20, 7, 7, 128), ([20001], 16, 1, 256), (_RAGGED, 40, 1, 64)],
]


@pytest.mark.parametrize("calls", CHANGING, ids=["rows", "joins", "heads"])
def test_one_decode_workspace_for_calls_of_changing_size(calls):
    """Every call gives what it gives with a workspace of its own, bit for bit, and leaves no arrival behind."""
    import paper_2609_35800_amd as hg
    made = []
    for i, (lens, Hq, H, D) in enumerate(calls):
        K, V, rows = make_pages(lens, H, D, 16, i, spare=0, fill=0.0)
        g = torch.Generator(device="cuda").manual_seed(i)
        K.normal_(generator=g)
        V.normal_(generator=g)
        q = torch.randn((len(lens), Hq, D), generator=g, device="cuda").to(BF)
        made.append((hg.make_paged_cache(K, V, i32(rows)), q, i32(lens)))
    size = max(hg.hg_decode_workspace(cache, q.shape[1]) for cache, q, _ in made)
    shared = torch.zeros(size, dtype=torch.uint8, device="cuda")
    for turn in range(2):
        for i, (cache, q, lens) in enumerate(made):
            got = []
            for ws in (shared, hg.alloc_decode_workspace(cache, q.shape[1])):
                out = torch.full_like(q, float("nan"))
                lse = torch.full(q.shape[:2], float("nan"), dtype=torch.float32, device="cuda")
                hg.hg_decode_attention(cache, q, lens, out, ws, lse=lse)
                got.append((out, lse))
            torch.cuda.synchronize()
            (o, l), (o1, l1) = got
            assert not bool(torch.isnan(o1).any()) and not bool(torch.isnan(l1).any())
            assert torch.equal(bits(o), bits(o1)) and torch.equal(l, l1), f"turn {turn}, call {i}"


def test_decode_peaked_and_scaled():
    check_decode([700, 33], 8, 2, 128, 16, seed=4, peak=20.0)
    check_decode([700, 33], 8, 2, 128, 16, seed=5, scale=-0.5)
    check_decode([700, 33], 8, 2, 128, 16, seed=6, scale=0.0)


def test_decode_pages_outside_the_cache_are_not_attended():
    import paper_2609_35800_amd as hg
    g = gen(8)
    D, H, ps = 128, 2, 16
    K, V = randn(g, 4, H, ps, D).cuda(), randn(g, 4, H, ps, D).cuda()
    table = i32([[0, 4, 2], [-1, -5, 1 << 30]])
    q = randn(g, 2, H, D)
    out = torch.full((2, H, D), float("nan"), dtype=BF, device="cuda")
    lse = torch.zeros(2, H, device="cuda")
    cache = hg.make_paged_cache(K, V, table)
    hg.hg_decode_attention(cache, q.cuda(), i32([40, 48]), out, hg.alloc_decode_workspace(cache, H), lse=lse)
    torch.cuda.synchronize()
    for h in range(H):
        k = torch.cat([K[0, h].cpu(), K[2, h, :8].cpu()])
        v = torch.cat([V[0, h].cpu(), V[2, h, :8].cpu()])
        o, l, to, tl = attnref.attend(q[0, h:h + 1], k, v, D ** -0.5)
        assert_close(out[0, h:h + 1], o, to, "row 0")
        assert_close(lse[0, h:h + 1], l, tl, "lse of row 0")
    assert bool((out[1] == 0).all()) and bool((lse[1] == -math.inf).all())
    # lengths outside the table are clamped to it
    hg.hg_decode_attention(cache, q.cuda(), i32([1 << 30, -3]), out, hg.alloc_decode_workspace(cache, H), lse=lse)
    torch.cuda.synchronize()
    k, v = torch.cat([K[0, 0].cpu(), K[2, 0].cpu()]), torch.cat([V[0, 0].cpu(), V[2, 0].cpu()])
    o, l, to, tl = attnref.attend(q[0, :1], k, v, D ** -0.5)
    assert_close(out[0, :1], o, to, "clamped row")
    assert bool((out[1] == 0).all())


def test_offsets_past_32_bits():
    """Pages past 2^31 elements (4 GiB per tensor): append there, then decode."""
    import paper_2609_35800_amd as hg
    g = gen(9)
    D, H, ps, pages = 128, 8, 64, 35000  # 2.3e9 elements
    K = torch.empty(pages, H, ps, D, dtype=BF, device="cuda")
    V = torch.empty_like(K)
    last = pages - 1
    rows = [[last, 0, pages // 2]]
    n = 150
    k, v, q = randn(g, n, H, D), randn(g, n, H, D), randn(g, 1, H, D)
    cache = hg.make_paged_cache(K, V, i32(rows))
    hg.hg_append_kv(cache, None, None, k.cuda(), v.cuda(), i32([n]), cu_new=i32([0, n]))
    out = torch.zeros(1, H, D, dtype=BF, device="cuda")
    hg.hg_decode_attention(cache, q.cuda(), i32([n]), out, hg.alloc_decode_workspace(cache, H))
    torch.cuda.synchronize()
    assert torch.equal(bits(K[last].cpu()), bits(k[:64].transpose(0, 1)))
    assert torch.equal(bits(V[pages // 2, :, :22].cpu()), bits(v[128:].transpose(0, 1)))
    for h in range(H):
        o, _, to, _ = attnref.attend(q[0, h:h + 1], k[:, h], v[:, h], D ** -0.5)
        assert_close(out[0, h:h + 1], o, to, f"head {h}")


@pytest.mark.parametrize("D", [64, 128, 256])
def test_decode_longest_rows(D):
    """Rows that end at token 2^31 - 1, over pages of 2^30 tokens that are one
    broadcast row: equal scores, so out is the value and lse the score and the
    logarithm of the tokens.  Weights are 1 and the values small whole numbers, so
    a lane's sums are exact; the join of up to 512 parts adds 2^-15 at most."""
    import paper_2609_35800_amd as hg
    g = gen(D)
    ps, top = 1 << 30, (1 << 31) - 1
    k, q = randn(g, D), randn(g, 5, 1, D)
    v = torch.randint(-2, 3, (D,), generator=g).to(BF)
    K, V = (x.cuda().view(1, 1, 1, D).expand(1, 1, ps, D) for x in (k, v))
    table = [[0, 0], [0, 0], [-1, 0], [0, -1], [0, 0]]
    starts = [0, top - 5, top - 300, ps - 40, top]
    tokens = [top, 5, 300, 40, 0]
    cache = hg.make_paged_cache(K, V, i32(table))
    out = torch.full((5, 1, D), float("nan"), dtype=BF, device="cuda")
    lse = torch.full((5, 1), float("nan"), dtype=torch.float32, device="cuda")
    hg.hg_decode_attention(cache, q.cuda(), i32([top] * 5), out, hg.alloc_decode_workspace(cache, 1), starts=i32(starts), lse=lse)
    torch.cuda.synchronize()
    for b, n in enumerate(tokens):
        x = q[b, 0].double() * k.double()
        s = float(x.sum()) * D ** -0.5
        want = s + math.log(n) if n else -math.inf
        tol = 2 * D * 2.0 ** -23 * D ** -0.5 * float(x.abs().sum()) + 2.0 ** -20 * (1 + abs(want)) + 2.0 ** -15 if n else 0.0
        assert_close(lse[b], torch.tensor([want], dtype=torch.float64), torch.tensor([tol], dtype=torch.float64), f"row {b}")
        assert torch.equal(out[b, 0].cpu(), v if n else torch.zeros_like(v)), f"row {b}"


@pytest.mark.parametrize("D", [64, 128, 256])
def test_decode_large_caches(D):
    """Pages past 256 MiB are read by streaming loads."""
    import paper_2609_35800_amd as hg
    g = gen(D)
    H, ps = 2, 64
    pages = (300 << 20) // (4 * H * ps * D)
    K = torch.full((pages, H, ps, D), float("nan"), dtype=BF, device="cuda")
    V = torch.full((pages, H, ps, D), float("nan"), dtype=BF, device="cuda")
    lens = [500, 0, 1, 77]
    free = iter(random.Random(D).sample(range(pages), 40))
    rows = [[next(free) for _ in range(8)] for _ in lens]
    host = [(randn(g, n, H, D), randn(g, n, H, D)) for n in lens]
    for b, (k, v) in enumerate(host):
        if lens[b]:
            put(K, rows, b, 0, k)
            put(V, rows, b, 0, v)
    q = randn(g, 4, 3 * H, D)
    out = torch.full((4, 3 * H, D), float("nan"), dtype=BF, device="cuda")
    cache = hg.make_paged_cache(K, V, i32(rows))
    hg.hg_decode_attention(cache, q.cuda(), i32(lens), out, hg.alloc_decode_workspace(cache, 3 * H))
    torch.cuda.synchronize()
    for b, (k, v) in enumerate(host):
        for h in range(H):
            o, _, to, _ = attnref.attend(q[b, 3 * h:3 * h + 3], k[:, h], v[:, h], D ** -0.5)
            assert_close(out[b, 3 * h:3 * h + 3], o, to, f"row {b} head {h}")


@pytest.mark.parametrize("D", [64, 128, 256])
def test_decode_streamed(D):
    """Pages and attended tokens past 256 MiB, read by streaming loads: long rows among short ones."""
    import paper_2609_35800_amd as hg
    H, Hq, ps = 8, 24, 64
    longest = (300 << 20) // (4 * H * D) // 4
    lens = [longest, 3, 3 * longest, 0, 65]
    K, V, rows = make_pages(lens, H, D, ps, D, spare=0, fill=0.0)
    g = torch.Generator(device="cuda").manual_seed(D)
    K.normal_(generator=g)
    V.normal_(generator=g)
    q = torch.randn((5, Hq, D), generator=g, device="cuda").to(BF)
    out = torch.full_like(q, float("nan"))
    lse = torch.full((5, Hq), float("nan"), dtype=torch.float32, device="cuda")
    cache = hg.make_paged_cache(K, V, i32(rows))
    hg.hg_decode_attention(cache, q, i32(lens), out, hg.alloc_decode_workspace(cache, Hq), lse=lse)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        at = torch.arange(n)
        page, off = torch.tensor(rows[b])[at // ps].cuda(), (at % ps).cuda()
        for h in (0, 5, 7):
            k, v = K[page, h, off].cpu(), V[page, h, off].cpu()
            heads = slice(3 * h, 3 * h + 3)
            o, l, to, tl = attnref.attend(q[b, heads].cpu(), k, v, D ** -0.5)
            assert_close(out[b, heads], o, to, f"row {b} head {h}")
            assert_close(lse[b, heads], l, tl, f"lse of row {b} head {h}")


def test_decode_many_rows_and_one_long():
    """Even shares of all chunks, with a row that a hundred workgroups share."""
    lens = [random.Random(b).choice([0, 1, 33, 40]) for b in range(150)]
    lens[70] = 60000
    check_decode(lens, 4, 2, 64, 64, seed=7, calls=2)
    lens[70], lens[149] = 20, 9000
    check_decode(lens, 18, 2, 128, 16, seed=8, calls=2)


# ------------------------------------------------------------ prefill

def check_prefill(nq, nk, Hq, H, D, causal, seed=0, scale=None, peak=1.0, fused=False, poison=False):
    """Rows of nq[b] queries and nk[b] keys.  poison: keys and values that some
    query does not see are NaN or infinite; those queries must not notice."""
    import paper_2609_35800_amd as hg
    g = gen(seed)
    B = len(nq)
    cq, ck = [0], [0]
    for a, b in zip(nq, nk):
        cq.append(cq[-1] + a)
        ck.append(ck[-1] + b)
    q, k, v = randn(g, cq[-1], Hq, D), randn(g, ck[-1], H, D) * peak, randn(g, ck[-1], H, D)
    if poison:
        for b in range(B):
            if nk[b] > 2:
                v[ck[b + 1] - 1, :, ::3] = float("inf")
                v[ck[b + 1] - 2, :, 1::5] = float("nan")
                k[ck[b + 1] - 1, :, 5] = float("nan")
    if fused:
        assert cq == ck
        dev = torch.cat([q, k, v], 1).cuda()
        qd, kd, vd = dev[:, :Hq], dev[:, Hq:Hq + H], dev[:, Hq + H:]
    else:  # heads before tokens in memory
        qd, kd, vd = (x.transpose(0, 1).contiguous().cuda().transpose(0, 1) for x in (q, k, v))
    out = torch.full((cq[-1], Hq, D), float("nan"), dtype=BF, device="cuda")
    lse = torch.full((cq[-1], Hq), float("nan"), dtype=torch.float32, device="cuda")
    hg.hg_prefill_attention(qd, kd, vd, i32(cq), out, cu_k=None if cq == ck else i32(ck), causal=causal, scale=scale, lse=lse)
    torch.cuda.synchronize()
    s = D ** -0.5 if scale is None else scale
    for b in range(B):
        rows = list(range(nq[b]))
        if len(rows) > 24:  # the ends, tile borders and a sample
            rows = sorted(set([0, 1, 31, 32, 63, 64, 127, 128, nq[b] - 2, nq[b] - 1] +
                              random.Random(seed).sample(rows, 10)) & set(rows))
        last = [i + nk[b] - nq[b] if causal else nk[b] - 1 for i in rows]
        if poison:  # queries that see none of the poisoned keys
            keep = [x for x in range(len(rows)) if last[x] < nk[b] - 2 or nk[b] <= 2]
            rows, last = [rows[x] for x in keep], [last[x] for x in keep]
        if not rows:
            continue
        at = torch.tensor(rows) + cq[b]
        for h in range(H):
            G = Hq // H
            kk, vv = k[ck[b]:ck[b + 1], h], v[ck[b]:ck[b + 1], h]
            for hq in sorted({h * G, h * G + G - 1}):
                o, l, to, tl = attnref.attend(q[at, hq], kk, vv, s, last=last)
                assert_close(out[at.cuda(), hq], o, to, f"row {b} of {nq[b]} x {nk[b]}, head {hq}")
                assert_close(lse[at.cuda(), hq], l, tl, f"lse of row {b}, head {hq}")


LENGTHS = [1, 0, 31, 32, 33, 64, 65, 130, 0, 300]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,H", [(2, 2), (7, 1), (6, 3)])
def test_prefill_packed(D, Hq, H, causal):
    check_prefill(LENGTHS, LENGTHS, Hq, H, D, causal, seed=D + Hq, fused=Hq == 6)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_prefill_more_and_fewer_keys(D, causal):
    """Keys of an earlier turn before the queries'; queries without keys (fewer
    keys than queries: the first see none; no keys at all)."""
    check_prefill([5, 130, 40, 200, 7, 1], [300, 131, 3, 70, 0, 257], 4, 2, D, causal, seed=D)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_prefill_longer(D):
    check_prefill([1361, 514], [1361, 514], 4, 2, D, True, seed=D, peak=4.0)


@pytest.mark.parametrize("causal", [True, False])
def test_prefill_long_rows(causal):
    """Tiles of 256 queries (long rows on average), beside short and empty rows."""
    check_prefill([3301, 3, 0, 290, 257, 6400], [3301, 3, 0, 290, 257, 6400], 4, 2, 128, causal, seed=11, fused=True)
    check_prefill([130, 700, 1, 0], [9001, 2000, 64, 77], 2, 1, 128, causal, seed=12)
    check_prefill([2000, 300], [1900, 1700], 2, 2, 128, causal, seed=13, peak=4.0)


def test_prefill_long_rows_masked_places():
    check_prefill([3500, 200, 1801], [3500, 200, 1801], 2, 1, 128, True, seed=14, poison=True)


@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.0])
def test_prefill_scales(scale):
    check_prefill([200, 3], [200, 3], 2, 1, 128, True, seed=3, scale=scale)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_prefill_what_masked_places_hold_does_not_matter(D):
    check_prefill([70, 200, 33, 3], [70, 200, 33, 3], 4, 2, D, True, seed=D, poison=True)


@pytest.mark.parametrize("D,nq,nk", [(64, 300, 200), (64, 200, 110), (128, 200, 130), (128, 40, 3), (256, 300, 250),
                                     (256, 200, 130), (128, 2000, 1900)])
def test_prefill_first_queries_far_before_the_keys(D, nq, nk):
    """Fewer keys than queries by a stage or more: the first queries see none, and
    nothing of the row before, whose last values are not finite, reaches any."""
    import paper_2609_35800_amd as hg
    g = gen(D + nq)
    Hq, H, n0 = 4, 2, max(nk, 128)
    q, k, v = randn(g, n0 + nq, Hq, D), randn(g, n0 + nk, H, D), randn(g, n0 + nk, H, D)
    v[n0 - 128:n0, :, ::2] = float("inf")
    v[n0 - 128:n0, :, 1::4] = float("nan")
    out = torch.full((n0 + nq, Hq, D), float("nan"), dtype=BF, device="cuda")
    lse = torch.full((n0 + nq, Hq), float("nan"), dtype=torch.float32, device="cuda")
    hg.hg_prefill_attention(q.cuda(), k.cuda(), v.cuda(), i32([0, n0, n0 + nq]), out, cu_k=i32([0, n0, n0 + nk]), lse=lse)
    torch.cuda.synchronize()
    empty = nq - nk
    assert bool((out[n0:n0 + empty] == 0).all()) and bool((lse[n0:n0 + empty] == -math.inf).all())
    rows = sorted({empty, empty + 1, empty + 31, nq // 2, nq - 1} & set(range(empty, nq)))
    at = torch.tensor(rows) + n0
    for hq in range(Hq):
        o, l, to, tl = attnref.attend(q[at, hq], k[n0:, hq // 2], v[n0:, hq // 2], D ** -0.5, last=[i - empty for i in rows])
        assert_close(out[at.cuda(), hq], o, to, f"head {hq}")
        assert_close(lse[at.cuda(), hq], l, tl, f"lse of head {hq}")


def test_prefill_values_not_finite_reach_the_queries_that_see_them():
    _values_not_finite(150)
    _values_not_finite(2000)  # tiles of 256 queries


def _values_not_finite(n):
    import paper_2609_35800_amd as hg
    g = gen(2)
    D = 128
    q, k, v = (randn(g, n, 1, D).cuda() for _ in range(3))
    v[100, 0, 3] = float("inf")
    v[140, 0, 5] = float("nan")
    v[10, 0, 7] = float("-inf")
    out = torch.zeros_like(q)
    hg.hg_prefill_attention(q, k, v, i32([0, n]), out)
    torch.cuda.synchronize()
    o = out[:, 0].float().cpu()
    i = torch.arange(n)
    assert bool((o[i >= 100, 3] == math.inf).all()) and bool(torch.isfinite(o[i < 100, 3]).all())
    assert bool(torch.isnan(o[i >= 140, 5]).all()) and bool(torch.isfinite(o[i < 140, 5]).all())
    assert bool((o[i >= 10, 7] == -math.inf).all()) and bool(torch.isfinite(o[i < 10, 7]).all())
    others = [c for c in range(D) if c not in (3, 5, 7)]
    assert bool(torch.isfinite(o[:, others]).all())


@pytest.mark.parametrize("D,n", [(64, 150), (128, 150), (256, 150), (128, 2000)])
def test_prefill_values_not_finite_stay_with_their_head(D, n):
    """Such values at a tile's border, within its diagonal and in a later row reach
    the queries of their own key/value head from their key on, and no others."""
    import paper_2609_35800_amd as hg
    g = gen(D + n)
    Hq, H, first = 6, 2, 37
    N = first + n
    q, k, v = randn(g, N, Hq, D).cuda(), randn(g, N, H, D).cuda(), randn(g, N, H, D).cuda()
    odd = [(0, 128, 3, math.inf), (0, 64, D - 1, -math.inf), (1, 129, 7, math.nan), (1, 31, 0, math.inf), (1, n - 1, 9, math.inf)]
    for h, j, c, x in odd:
        v[first + j, h, c] = x
    out = torch.zeros_like(q)
    hg.hg_prefill_attention(q, k, v, i32([0, first, N]), out)
    torch.cuda.synchronize()
    want = torch.zeros(N, Hq, D)
    for h, j, c, x in odd:
        want[first + j:, 3 * h:3 * h + 3, c] = x
    o = out.float().cpu()
    finite = torch.isfinite(want)
    assert bool(torch.isfinite(o[finite]).all())
    assert bool(((o == want) | (torch.isnan(o) & torch.isnan(want)))[~finite].all())


@pytest.mark.parametrize("D,nq,nk,stride", [(64, 150, 150, 1 << 24), (128, 40, 140, 1 << 24), (256, 140, 140, 1 << 24),
                                            (128, 300, 3500, 1 << 20)])
@pytest.mark.parametrize("causal", [True, False])
def test_prefill_rows_past_4_gib(D, nq, nk, stride, causal):
    """More than 4 GiB between a row's first key and its last, up to 32 MiB from one to the next."""
    import paper_2609_35800_amd as hg
    g = gen(D + nk)
    Hq, H = 4, 2
    base = torch.empty(nk + 2, stride, dtype=BF, device="cuda")
    kd, vd = base[:, :H * D].view(nk + 2, H, D), base[:, 4096:4096 + H * D].view(nk + 2, H, D)
    q, k, v = randn(g, 3 + nq, Hq, D), randn(g, nk + 2, H, D), randn(g, nk + 2, H, D)
    kd.copy_(k)
    vd.copy_(v)
    assert nk * stride * 2 > 1 << 32 and kd.stride(0) == stride
    out = torch.full((3 + nq, Hq, D), float("nan"), dtype=BF, device="cuda")
    hg.hg_prefill_attention(q.cuda(), kd, vd, i32([0, 3, 3 + nq]), out, cu_k=i32([0, 2, 2 + nk]), causal=causal)
    torch.cuda.synchronize()
    rows = sorted({0, 31, 32, nq // 2, nq - 2, nq - 1})
    last = [i + nk - nq if causal else nk - 1 for i in rows]
    at = torch.tensor(rows) + 3
    for hq in range(Hq):
        o, _, to, _ = attnref.attend(q[at, hq], k[2:, hq // 2], v[2:, hq // 2], D ** -0.5, last=last)
        assert_close(out[at.cuda(), hq], o, to, f"head {hq}")


def test_prefill_rows_outside_the_offsets_are_not_written():
    import paper_2609_35800_amd as hg
    g = gen(2)
    q, k, v = (randn(g, 20, 2, 64).cuda() for _ in range(3))
    out = torch.full_like(q, float("nan"))
    hg.hg_prefill_attention(q, k, v, i32([3, 8, 8, 15]), out)
    torch.cuda.synchronize()
    assert torch.isfinite(out.float()).all(-1).all(-1).cpu().tolist() == [False] * 3 + [True] * 12 + [False] * 5


def test_prefill_of_the_largest_launch():
    """Rows of one query up to the launch limit: every one is answered."""
    import paper_2609_35800_amd as hg
    Hq, D = 4096, 64
    slots = (2**32 - 1) // 256 // Hq
    n = next(n for n in range(slots, 0, -1) if n + n // 128 <= slots)
    g = gen(1)
    q, k = randn(g, 1, Hq, D).cuda().expand(n, Hq, D), randn(g, 1, 1, D).cuda().expand(n, 1, D)
    v = torch.arange(n, device="cuda").remainder(251).to(BF).view(n, 1, 1).expand(n, 1, D).contiguous()
    out = torch.full((n, Hq, D), float("nan"), dtype=BF, device="cuda")
    hg.hg_prefill_attention(q, k, v, torch.arange(n + 1, dtype=torch.int32, device="cuda"), out)
    torch.cuda.synchronize()
    assert bool((out == v).all())  # a softmax over one key is 1
    with pytest.raises(hg.HeadGuardError) as e:
        hg.hg_prefill_attention(q[:1].expand(n + 1, Hq, D), k[:1].expand(n + 1, 1, D), k[:1].expand(n + 1, 1, D),
                                torch.zeros(n + 2, dtype=torch.int32, device="cuda"), torch.empty(n + 1, Hq, D, dtype=BF, device="cuda"))
    assert e.value.status == hg.HG_ERR_SHAPE


def test_prefill_offsets_are_clamped():
    """Offsets outside the operands, or not ascending: nothing outside is read or written, rows that
    make sense are answered."""
    import paper_2609_35800_amd as hg
    g = gen(4)
    n, D = 200, 64
    qd = torch.full((n + 40, 2, D), float("nan"), dtype=BF, device="cuda")
    q, k, v = (randn(g, n, 2, D) for _ in range(3))
    qd[20:20 + n] = q.cuda()
    out = torch.full((n + 40, 2, D), 3.0, dtype=BF, device="cuda")
    cu = [0, 50, 150, -7, 120, 1 << 30]  # rows: 50, 100, none, [0, 120) again, [120, n)
    hg.hg_prefill_attention(qd[20:20 + n], k.cuda(), v.cuda(), i32(cu), out[20:20 + n])
    torch.cuda.synchronize()
    assert bool((out[:20] == 3).all()) and bool((out[20 + n:] == 3).all())
    for h in range(2):  # the fourth row starts with the first one's tokens: the same values, causal
        o, _, to, _ = attnref.attend(q[:50, h], k[:50, h], v[:50, h], D ** -0.5, last=list(range(50)))
        assert_close(out[20:70, h], o, to, f"head {h}")


# ------------------------------------------------------------ streams, graphs, errors

def _layer(hg, seed=0):
    """A small layer: prompts appended and attended, then one token a row."""
    g = gen(seed)
    B, Hq, H, D, ps = 3, 4, 2, 128, 16
    n = [20, 1, 40]
    cu = [0, 20, 21, 61]
    K, V, rows = make_pages([m + 1 for m in n], H, D, ps, seed, fill=0.0)
    cos, sin = attnref.table(64, D // 2)
    s = dict(cache=hg.make_paged_cache(K, V, i32(rows)), rot=hg.make_rotation(cos.cuda(), sin.cuda()),
             qkv=randn(g, 61, Hq + 2 * H, D).cuda(), one=randn(g, B, Hq + 2 * H, D).cuda(), cu=i32(cu), lens=i32(n),
             lens1=i32([m + 1 for m in n]), q=torch.zeros(61, Hq, D, dtype=BF, device="cuda"),
             k=torch.zeros(61, H, D, dtype=BF, device="cuda"), o=torch.zeros(61, Hq, D, dtype=BF, device="cuda"),
             q1=torch.zeros(B, Hq, D, dtype=BF, device="cuda"), o1=torch.zeros(B, Hq, D, dtype=BF, device="cuda"), K=K, V=V)
    s["ws"] = hg.alloc_decode_workspace(s["cache"], Hq)
    return s


def _run_layer(hg, s, stream=None):
    x, y = s["qkv"], s["one"]
    hg.hg_append_kv(s["cache"], s["rot"], x[:, :4], x[:, 4:6], x[:, 6:], s["lens"], s["q"], cu_new=s["cu"], k_out=s["k"],
                    stream=stream)
    hg.hg_prefill_attention(s["q"], s["k"], x[:, 6:], s["cu"], s["o"], stream=stream)
    hg.hg_append_kv(s["cache"], s["rot"], y[:, :4], y[:, 4:6], y[:, 6:], s["lens1"], s["q1"], stream=stream)
    hg.hg_decode_attention(s["cache"], s["q1"], s["lens1"], s["o1"], s["ws"], stream=stream)


def _results(s):
    return {n: s[n].clone() for n in ("q", "k", "o", "q1", "o1", "K", "V")}


def _reset(s):
    for n in ("q", "k", "o", "q1", "o1", "K", "V"):
        s[n].zero_()


def test_another_stream_and_graph_replays():
    import paper_2609_35800_amd as hg
    s = _layer(hg)
    _run_layer(hg, s)
    torch.cuda.synchronize()
    want = _results(s)
    assert all(bool((t != 0).any()) for t in want.values())
    _reset(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _run_layer(hg, s, stream=side)
    side.synchronize()
    got = _results(s)
    assert all(torch.equal(bits(got[n]), bits(want[n])) for n in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _run_layer(hg, s)
    for _ in range(3):
        _reset(s)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = _results(s)
        assert all(torch.equal(bits(got[n]), bits(want[n])) for n in want)
    del graph


def test_launch_failures_touch_nothing(monkeypatch):
    import paper_2609_35800_amd as hg
    s = _layer(hg)
    monkeypatch.setenv("HG_FAIL_LAUNCH", "0")
    x = s["qkv"]
    for call in (lambda: hg.hg_append_kv(s["cache"], s["rot"], x[:, :4], x[:, 4:6], x[:, 6:], s["lens"], s["q"],
                                         cu_new=s["cu"], k_out=s["k"]),
                 lambda: hg.hg_prefill_attention(s["q"], s["k"], x[:, 6:], s["cu"], s["o"]),
                 lambda: hg.hg_decode_attention(s["cache"], s["q1"], s["lens1"], s["o1"], s["ws"])):
        with pytest.raises(hg.HeadGuardError) as e:
            call()
        assert e.value.status == hg.HG_ERR_HIP
    torch.cuda.synchronize()
    assert all(bool((t == 0).all()) for t in _results(s).values())


def test_host_memory_is_refused():
    import paper_2609_35800_amd as hg
    s = _layer(hg)
    with pytest.raises(hg.HeadGuardError) as e:
        hg.hg_decode_attention(s["cache"], s["q1"].cpu(), s["lens1"], s["o1"], s["ws"])
    assert e.value.status == hg.HG_ERR_POINTER
    with pytest.raises(hg.HeadGuardError) as e:
        hg.hg_prefill_attention(s["q"], s["k"], s["k"], s["cu"].cpu(), s["o"])
    assert e.value.status == hg.HG_ERR_POINTER
