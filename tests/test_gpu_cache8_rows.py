"""Rows of the 8-bit cache over their lives: rows that begin inside a block, on
pages that other rows filled before, tokens taken back; every value through both
forms of the append; the weights of attention; the ways of ranking blocks; calls on a
stream of their own."""
import math

import pytest
import torch

import attnref
import cache8ref as ref
from attnref import assert_close
from test_gpu_cache8 import BF, Cache, check_select, gen, i32, offsets, randn, raw

pytestmark = pytest.mark.gpu


def append_from(codes, scales, bounds, row, page_size, block, start, x, first):
    """ref.append of a row whose tokens begin at `first`: what its first block held
    before, and its scale and bounds, are no tokens of the row."""
    n = x.shape[0]
    skip = min(max(first - start, 0), n)
    x, start = x[skip:], start + skip
    if not len(x):
        return
    base = start // block * block
    page, off, sub = row[base // page_size], base % page_size, base % page_size // block
    place = slice(off, off + min(max(first - base, 0), start - base))  # before the row's first token
    before = codes[page, :, place].clone()
    if first >= start:
        scales[page, :, sub] = math.nan
        if bounds is not None:
            bounds[page, :, sub] = math.nan
    ref.append(codes, scales, bounds, row, page_size, block, start, x)
    codes[page, :, place] = before


def recycle(c, seed):
    """Pages as another row with keys and values up to 1e6 left them."""
    g = gen(seed)
    for t in (c.K, c.V):
        t.copy_(torch.randint(0, 0x7F, t.shape, generator=g, dtype=torch.uint8))
    c.ks.fill_(2.0 ** 14)
    c.vs.fill_(2.0 ** 13)
    if c.bounds is not None:
        c.bounds[..., 0, :] = -4e6
        c.bounds[..., 1, :] = 4e6


ROWS = [  # D, H, block, pages of blocks, token_major, starts, tokens of each call (None: one of every row)
    (128, 4, 16, 1, False, [5, 0, 31, 16], [[3, 40, 1, 16], None, None]),
    (64, 2, 32, 3, True, [31, 33, 90], [None, None, [2, 70, 40], None]),
    (256, 2, 64, 1, False, [1, 63], [[70, 1], None, [5, 0], None]),
    (128, 8, 128, 1, True, [100, 127, 5], [None, [29, 1, 200], None]),
]


@pytest.mark.parametrize("case", ROWS, ids=str)
def test_rows_that_begin_inside_a_block(case):
    """Left-padded rows on recycled pages: codes, scales and bounds of the row's tokens alone, the
    same on pages of any past, every other byte as it was."""
    import paper_2609_35800_amd as hg
    D, H, block, pages, token_major, starts, calls = case
    B, ps = len(starts), block * pages
    total = [s + sum(1 if n is None else n[b] for n in calls) for b, s in enumerate(starts)]
    fresh, used = (Cache(total, H, D, ps, block, 3, token_major) for _ in range(2))
    recycle(used, D)
    g = gen(D + block)
    at = list(starts)
    for i, n in enumerate(calls):
        counts = [1] * B if n is None else n
        x = randn(g, sum(counts), 2 * H, D) * 2.0 ** (2 * i - 3)  # scales grow from call to call
        ends, cu = [a + n for a, n in zip(at, counts)], offsets(counts)
        for c in (fresh, used):
            state = c.host()
            hg.hg_append_kv8(c.descriptor(), None, None, x[:, :H].cuda(), x[:, H:].cuda(), i32(ends), cu_new=None if n is None else i32(cu),
                             starts=i32(starts))
            torch.cuda.synchronize()
            for b in range(B):
                for k, part in ((0, x[cu[b]:cu[b + 1], :H]), (1, x[cu[b]:cu[b + 1], H:])):
                    append_from(state[k], state[k + 2], state[4] if k == 0 else None, c.rows[b], ps, block, at[b], part, starts[b])
            for name, got, want in zip(("K", "V", "k_scale", "v_scale", "bounds"), c.host(), state):
                same = (got == want) | (raw(got) == raw(want))
                assert bool(same.all()), f"call {i}: {name}: {int((~same).sum())} differ"
        at = ends
        for b in range(B):
            for t in range(starts[b], at[b]):
                page, off = used.rows[b][t // ps], t % ps
                for p, q in ((fresh.K, used.K), (fresh.V, used.V)):
                    assert torch.equal(p[page, :, off], q[page, :, off])
                for p, q in ((fresh.ks, used.ks), (fresh.vs, used.vs), (fresh.bounds, used.bounds)):
                    assert torch.equal(raw(p[page, :, off // block]), raw(q[page, :, off // block]))


@pytest.mark.parametrize("single", [True, False])
def test_new_tokens_before_the_rows_first(single):
    """Padding that comes with the call is rotated, not stored, and counts for nothing, huge or NaN;
    starts past the row, and before the cache."""
    import paper_2609_35800_amd as hg
    D, H, block = 64, 2, 16
    starts = [9, 40, -5, 3, 2 ** 31 - 1]
    counts = [1] * 5 if single else [12, 6, 3, 40, 2]
    lens = [10, 20, 4, 41, 2] if not single else [9, 40, 4, 4, 2]
    B, N = len(starts), sum(counts)
    cu = offsets(counts)
    g = gen(2)
    c = Cache([48] * B, H, D, 2 * block, block)
    recycle(c, 1)
    k, v = randn(g, N, H, D), randn(g, N, H, D)
    at = [n - m for n, m in zip(lens, counts)]
    for b in range(B):
        for j in range(counts[b]):
            if at[b] + j < starts[b]:
                k[cu[b] + j], v[cu[b] + j] = (1e30, math.nan) if j % 2 else (math.nan, -1e30)
    k_out = torch.zeros(N, H, D, dtype=BF, device="cuda")
    cos, sin = attnref.table(64, D // 2)
    state = c.host()
    hg.hg_append_kv8(c.descriptor(), hg.make_rotation(cos.cuda(), sin.cuda()), None, k.cuda(), v.cuda(), i32(lens),
                     cu_new=None if single else i32(cu), k_out=k_out, starts=i32(starts))
    torch.cuda.synchronize()
    kh = k_out.cpu()
    assert bool((raw(kh) != 0).any(-1).any(-1)[[cu[b] + j for b in range(B) for j in range(counts[b]) if at[b] + j >= 0]].all())
    for b in range(B):
        lo, hi, first = cu[b], cu[b + 1], max(starts[b], 0)
        append_from(state[0], state[2], state[4], c.rows[b], c.ps, block, at[b], kh[lo:hi], first)
        append_from(state[1], state[3], None, c.rows[b], c.ps, block, at[b], v[lo:hi], first)
    for got, want in zip(c.host(), state):
        assert bool(((got == want) | (raw(got) == raw(want))).all())


@pytest.mark.parametrize("single", [True, False])
def test_rows_whose_first_tokens_were_skipped(single):
    """A call skipped a block's first tokens (positions outside the rotation's); the next one says
    where the row begins."""
    import paper_2609_35800_amd as hg
    D, H, block = 128, 2, 32
    g = gen(4)
    c = Cache([40], H, D, block, block)
    recycle(c, 7)
    cos, sin = attnref.table(64, D // 2)
    rotation = hg.make_rotation(cos.cuda(), sin.cuda())
    x = randn(g, 10, 2 * H, D)
    state = c.host()
    hg.hg_append_kv8(c.descriptor(), rotation, None, x[:5, :H].cuda(), x[:5, H:].cuda(), i32([5]), cu_new=i32([0, 5]),
                     positions=i32([-1] * 5))
    torch.cuda.synchronize()
    assert all(torch.equal(raw(a), raw(b)) for a, b in zip(c.host(), state))
    n = 1 if single else 5
    k_out = torch.empty(n, H, D, dtype=BF, device="cuda")
    hg.hg_append_kv8(c.descriptor(), rotation, None, x[5:5 + n, :H].cuda(), x[5:5 + n, H:].cuda(), i32([5 + n]),
                     cu_new=None if single else i32([0, n]), k_out=k_out, starts=i32([5]))
    torch.cuda.synchronize()
    append_from(state[0], state[2], state[4], c.rows[0], block, block, 5, k_out.cpu(), 5)
    append_from(state[1], state[3], None, c.rows[0], block, block, 5, x[5:5 + n, H:], 5)
    for got, want in zip(c.host(), state):
        assert bool(((got == want) | (raw(got) == raw(want))).all())
    assert float(c.ks[c.rows[0][0], 0, 0]) < 1


def test_rows_from_token_0_by_either_entry():
    """hg_append_kv8 is hg_append_kv8_from without starts, and with starts of 0."""
    import paper_2609_35800_amd as hg
    D, H, block, B = 64, 2, 16, 3
    lib = hg.library()
    got = []
    for entry in range(3):
        g = gen(1)
        c = Cache([40] * B, H, D, block, block)
        d = c.descriptor()
        lens, starts = i32([0] * B), i32([0] * B)
        for n in (17, 1, 5):
            x = randn(g, B * n, 2 * H, D).cuda()
            lens += n
            cu = i32(offsets([n] * B)) if n > 1 else None
            k, v = x[:, :H], x[:, H:]
            if entry:
                hg.hg_append_kv8(d, None, None, k, v, lens, cu_new=cu, starts=starts if entry == 2 else None)
            else:
                a = hg.hg_append(N=B * n, k=k.data_ptr(), k_token_stride=2 * H * D, k_head_stride=D, v=v.data_ptr(),
                                 v_token_stride=2 * H * D, v_head_stride=D, lens=lens.data_ptr(),
                                 cu_new=None if cu is None else cu.data_ptr())
                assert lib.hg_append_kv8(d, None, a, torch.cuda.current_stream().cuda_stream) == hg.HG_OK
            torch.cuda.synchronize()
        got.append(c.host())
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(raw(a), raw(b))
    assert bool(torch.isfinite(got[0][2]).any())


def test_left_padded_rows_served_from_recycled_pages():
    """Append, choose and attend with one array of starts, captured: replays with other starts and
    lengths give the eager run's results, the choice goes by the rows' own keys, and pages of any
    past the same answers."""
    import paper_2609_35800_amd as hg
    D, Hq, H, block, B, T, budget = 128, 8, 2, 16, 3, 160, 4
    cos, sin = attnref.table(T, D // 2)

    def setup(past):
        c = Cache([T] * B, H, D, 2 * block, block, 9)
        if past:
            recycle(c, past)
        s = dict(c=c, d=c.descriptor(), starts=i32([0] * B), lens=i32([0] * B), rotation=hg.make_rotation(cos.cuda(), sin.cuda()))
        s["x"] = torch.zeros(B, Hq + 2 * H, D, dtype=BF, device="cuda")
        s["q"], s["out"] = (torch.zeros(B, Hq, D, dtype=BF, device="cuda") for _ in range(2))
        s["k"] = torch.zeros(B, H, D, dtype=BF, device="cuda")
        s["blocks"] = torch.zeros(B, H, budget, dtype=torch.int32, device="cuda")
        s["ws"], s["sws"] = hg.alloc_decode8_workspace(s["d"], Hq), hg.alloc_select_workspace(s["d"])
        return s

    def step(s):
        x, k = s["x"], s["starts"]
        hg.hg_append_kv8(s["d"], s["rotation"], x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:], s["lens"], s["q"], k_out=s["k"], starts=k)
        hg.hg_select_blocks(s["d"], s["q"], s["lens"], s["blocks"], s["sws"], starts=k)
        hg.hg_decode_attention8(s["d"], s["q"], s["lens"], s["out"], s["ws"], starts=k, blocks=s["blocks"])

    eager, other, graphed = setup(0), setup(3), setup(5)
    step(graphed)  # rows without tokens
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    g = gen(1)
    for starts in ([7, 32, 45], [20, 3, 31]):
        keys = [[] for _ in range(B)]
        for n in range(46, 46 + 100):
            lens = [min(max(n - 46 + s + 1, 0), T) for s in starts]
            x = randn(g, B, Hq + 2 * H, D).cuda()
            for s in (eager, other, graphed):
                s["lens"].copy_(i32(lens))
                s["starts"].copy_(i32(starts))
                s["x"].copy_(x)
            step(eager)
            step(other)
            graph.replay()
            torch.cuda.synchronize()
            for name in ("q", "k", "blocks", "out"):
                assert torch.equal(raw(eager[name]), raw(graphed[name])) and torch.equal(raw(eager[name]), raw(other[name])), (n, name)
            for b in range(B):
                keys[b].append(eager["k"][b].double().cpu())
        # the last step against the formulas, bounds of the keys that the row has had
        K, V, ks, vs, _ = eager["c"].host()
        R = Hq // H
        for b in range(B):
            all_keys = torch.stack(keys[b])  # [n, H, D], of tokens starts[b] ..
            n0 = starts[b] // block
            for h in range(H):
                limits = []
                for i in range(n0, (lens[b] - 1) // block + 1):
                    own = all_keys[max(i * block - starts[b], 0):(i + 1) * block - starts[b], h]
                    limits.append(torch.stack((own.amin(0), own.amax(0))))
                q = eager["q"][b, h * R:(h + 1) * R].cpu()
                want = ref.select(q, limits, n0, budget, 1, 2)
                assert eager["blocks"][b, h].tolist() == want
                t = [t for i in want if i >= 0 for t in range(max(i * block, starts[b]), min((i + 1) * block, lens[b]))]
                c = eager["c"]
                o, _, to, _ = attnref.attend(q, c.gather(K, ks, b, h, t), c.gather(V, vs, b, h, t), D ** -0.5)
                assert_close(eager["out"][b, h * R:(h + 1) * R], o, to, f"row {b} head {h}")


@pytest.mark.parametrize("single", [True, False])
def test_tokens_taken_back_stay_counted(single):
    """Drafts far out, taken back by the pool: the block keeps their scale and bounds under the tokens
    that take their places, the bounds stay limits of the row's keys, and a row that shrinks to the
    block's first token begins it anew."""
    import paper_2609_35800_amd as hg
    D, H, block = 64, 2, 16
    g = gen(12)
    pool = hg.alloc_page_pool(1, 4, 4, block)
    table, lens, _, _ = pool.tensors
    c = hg.alloc_cache8(4, H, block, D, table, block)
    K, V, ks, vs, bounds, _ = c.tensors
    result = i32([0] * 4)
    state = [K.cpu(), V.cpu(), ks.cpu(), vs.cpu(), bounds.cpu()]

    def resize(n):
        hg.hg_resize_rows(pool, i32([n]), result)
        torch.cuda.synchronize()
        assert int(result[0]) == 0

    def append(n, size):
        x = randn(g, n, 2 * H, D) * size
        start = int(lens[0])
        resize(start + n)
        for t in range(1 if not single else n):
            a, z = (0, n) if not single else (t, t + 1)
            hg.hg_append_kv8(c, None, None, x[a:z, :H].cuda(), x[a:z, H:].cuda(), i32([start + z]),
                             cu_new=None if single else i32([0, n]))
            ref.append(state[0], state[2], state[4], table[0].tolist(), block, block, start + a, x[a:z, :H])
            ref.append(state[1], state[3], None, table[0].tolist(), block, block, start + a, x[a:z, H:])
        torch.cuda.synchronize()
        for got, want in zip((K, V, ks, vs, bounds), state):
            assert bool((got.cpu() == want).all())
        return x

    append(block, 1.0)  # a block of its own before
    kept = append(4, 1.0)
    page = int(table[0, 1])
    fine = ks[page].clone()
    drafts = append(5, 100.0)
    coarse = ks[page].clone()
    assert bool((coarse > 16 * fine).all())
    resize(block + 4)
    new = append(3, 1.0)
    assert torch.equal(ks[page], coarse)
    keys = torch.cat((kept, new))[:, :H]
    lo, hi = bounds[page, :, 0, 0].cpu(), bounds[page, :, 0, 1].cpu()
    assert bool((keys >= lo).all()) and bool((keys <= hi).all())
    counted = torch.cat((keys, drafts[:, :H]))
    assert torch.equal(lo, counted.amin(0)) and torch.equal(hi, counted.amax(0))
    # what the codes stand for is off by half a step of the coarse scale at most
    got = ref.values(K[page, :, :7].cpu(), ks[page, :, :1].expand(H, 7).cpu()).transpose(0, 1)
    x = keys.double()
    assert bool(((got - x).abs() <= torch.maximum(x.abs() * 2.0 ** -4, coarse.cpu().double().view(1, H, 1) * 2.0 ** -10) * 3).all())
    # to the block's first token, and back
    resize(block)
    again = append(2, 1.0)
    page = int(table[0, 1])
    assert bool((ks[page] < coarse / 16).all())
    assert torch.equal(bounds[page, :, 0, 1].cpu(), again[:, :H].amax(0))


@pytest.mark.parametrize("single", [True, False])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_every_value_becomes_its_nearest_code_in_every_row(single, D):
    """All BF16 numbers up to 448, infinities and NaN beside one 448 (scale 1): every row is compared,
    of one token each or as a single row."""
    import paper_2609_35800_amd as hg
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF)
    x = every[~(every.float().abs() > 448) | torch.isinf(every.float())]
    block = 16
    x = torch.cat((x, torch.zeros(-len(x) % (D - 1), dtype=BF))).view(-1, 1, D - 1)
    v = torch.cat((torch.full((len(x), 1, 1), 448.0, dtype=BF), x), 2)
    n = len(v)
    lens = [1] * n if single else [n]
    c = Cache(lens, 1, D, block, block)
    hg.hg_append_kv8(c.descriptor(), None, None, v.cuda(), v.cuda(), i32(lens), cu_new=None if single else i32([0, n]))
    torch.cuda.synchronize()
    want = ref.to_codes(v.double())[:, 0]
    assert int((want & 0x7F).unique().numel()) == 128  # every code of either sign, NaN among them
    t = torch.zeros(n, dtype=torch.long) if single else torch.arange(n)
    rows = torch.tensor(c.rows)
    page = (rows[:, 0] if single else rows[0][t // block]).cuda()
    for codes, scales in ((c.K, c.ks), (c.V, c.vs)):
        got = codes[page, 0, (t % block).cuda()].cpu()
        assert bool(ref.same_codes(got, want).all()) and bool((scales[page] == 1).all())


WEIGHTS = [(1, 64), (7, 128), (8, 64), (8, 256), (9, 128), (16, 64), (20, 128), (24, 256), (33, 64)]  # query heads a KV head, D


@pytest.mark.parametrize("R,D", WEIGHTS, ids=str)
@pytest.mark.parametrize("n", [2, 3, 17, 64, 1500])
def test_weights_keep_more_than_bf16(R, D, n):
    """Values of 1 and -1 that all but cancel, so that the weights' own errors show.

    Queries are 1 in one channel and 0 elsewhere, so a score s is one product, exact, times the scale
    and log2 e: with |s| <= 2, |s| 2^-22 bounds these roundings, and with the exponential's few units
    2^-20 is a weight's error and as much its sum's, relative.  A sum of n terms in fp32 adds n 2^-24 of
    A = sum p |v| / sum p = 1, for weights and products each.  The two roundings of a weight lose 2^-16
    of it.  The output's own is 2^-8 of it.  Rounded to BF16 once, a weight would lose 2^-8."""
    import paper_2609_35800_amd as hg
    H, block = 2, 16
    Hq, g = H * R, gen(100 * R + n)
    c = Cache([n, n], H, D, block, block)
    K, V, ks, vs, _ = c.host()
    for b in range(2):
        for h in range(H):
            for t in range(n):
                page, off = c.rows[b][t // block], t % block
                K[page, h, off] = ref.to_codes(-2.0 * torch.rand(D, generator=g, dtype=torch.float64) * 64)
                V[page, h, off] = ref.to_codes(torch.where(torch.rand(D, generator=g) < 0.5, 1.0, -1.0).double() * 256)
    ks.fill_(2.0 ** -6)
    vs.fill_(2.0 ** -8)
    for dst, src in ((c.K, K), (c.V, V), (c.ks, ks), (c.vs, vs)):
        dst.copy_(src)
    q = torch.zeros(2, Hq, D, dtype=BF)
    for i in range(Hq):
        q[:, i, i % D] = 1.0
    out = torch.full((2, Hq, D), math.nan, dtype=BF, device="cuda")
    d = c.descriptor()
    ws = hg.alloc_decode8_workspace(d, Hq)
    hg.hg_decode_attention8(d, q.cuda(), i32([n, n]), out, ws, scale=1.0)
    torch.cuda.synchronize()
    for b in range(2):
        for h in range(H):
            k, v = c.gather(K, ks, b, h, range(n)), c.gather(V, vs, b, h, range(n))
            assert bool((v.abs() == 1).all())
            exact = torch.softmax(q[b, h * R:(h + 1) * R].double() @ k.T, -1) @ v
            tol = 2.0 ** -8 * exact.abs() * (1 + 2.0 ** -6) + 2.0 ** -16 + 2 * 2.0 ** -20 + 2 * n * 2.0 ** -24
            assert_close(out[b, h * R:(h + 1) * R], exact, tol, f"row {b} head {h}")


def test_weights_keep_more_than_bf16_in_shares_of_the_list():
    """The same where workgroups take shares of the list of chunks, with blocks chosen too."""
    import paper_2609_35800_amd as hg
    D, H, block, B = 64, 4, 16, 200
    for R in (4, 12):
        g = gen(R)
        lens = [int(x) for x in torch.randint(1, 90, (B,), generator=g)]
        c = Cache(lens, H, D, block, block)
        K = ref.to_codes(-2.0 * torch.rand(c.K.shape, generator=g, dtype=torch.float64) * 64)
        V = ref.to_codes(torch.where(torch.rand(c.V.shape, generator=g) < 0.5, 256.0, -256.0).double())
        c.K.copy_(K)
        c.V.copy_(V)
        c.ks.fill_(2.0 ** -6)
        c.vs.fill_(2.0 ** -8)
        ks, vs = c.ks.cpu(), c.vs.cpu()
        q = torch.zeros(B, H * R, D, dtype=BF)
        for i in range(H * R):
            q[:, i, i % D] = 1.0
        d = c.descriptor()
        out = torch.full((B, H * R, D), math.nan, dtype=BF, device="cuda")
        for listed in (False, True):
            blocks = i32([[[0, 2, 3]] * H] * B) if listed else None
            hg.hg_decode_attention8(d, q.cuda(), i32(lens), out, hg.alloc_decode8_workspace(d, H * R), scale=1.0, blocks=blocks)
            torch.cuda.synchronize()
            for b in range(0, B, 7):
                n = lens[b]
                t = [i for i in range(n) if not listed or i // block in [0, 2, 3][:-(-n // block)]]
                for h in range(H):
                    k, v = c.gather(K, ks, b, h, t), c.gather(V, vs, b, h, t)
                    exact = torch.softmax(q[b, h * R:(h + 1) * R].double() @ k.T, -1) @ v
                    tol = 2.0 ** -8 * exact.abs() * (1 + 2.0 ** -6) + 2.0 ** -16 + 2 * 2.0 ** -20 + 2 * len(t) * 2.0 ** -24
                    assert_close(out[b, h * R:(h + 1) * R], exact, tol, f"row {b} head {h}")


@pytest.mark.parametrize("D,H,B", [(64, 1, 3), (128, 2, 20), (256, 1, 1)])
def test_selection_where_the_way_of_ranking_changes(D, H, B):
    """Rows of about 256 and 512 blocks, ranked by one workgroup or by two launches, in one call, with
    starts, ties and without."""
    block = 16
    lens = [block * n - 3 for n in (128, 129, 255, 256, 257, 258, 511, 512, 513, 600)]
    lens = (lens * 2)[:B] if B > 1 else [block * 257]
    starts = [(i * 37) % 70 for i in range(len(lens))]
    for budget, first, last in ((40, 1, 2), (1, 0, 0), (255, 0, 3), (256, 1, 1)):
        check_select(lens, 4 * H, H, D, block, budget, first, last, 2, starts, seed=budget)

    def few(c, x):
        x.copy_(torch.randint(-1, 2, x.shape[:3], generator=gen(5)).float()[..., None, None].expand(x.shape))

    check_select(lens[:4], 2, 1, D, block, 33, 0, 1, edit=few, q=torch.ones(len(lens[:4]), 2, D, dtype=BF))


def test_calls_take_their_place_on_their_stream():
    """Inputs made by work that is still running on a stream: calls on that stream, as the current one
    or named, wait for it, and work behind them for their results; nothing else is waited for."""
    import paper_2609_35800_amd as hg
    D, Hq, H, block, n = 128, 4, 2, 16, 100
    c = Cache([n + 1], H, D, block, block)
    K, V, ks, vs = c.fill([n], gen(1))
    c.bounds.copy_(torch.tensor([-3.0, 3.0]).view(1, 1, 1, 2, 1).expand(c.bounds.shape))
    d = c.descriptor()
    ws, sws = hg.alloc_decode8_workspace(d, Hq), hg.alloc_select_workspace(d)
    x = randn(gen(2), 1, Hq + 2 * H, D).cuda()
    state = [t.clone() for t in (c.K, c.V, c.ks, c.vs, c.bounds)]
    late, done = torch.empty_like(x), torch.empty(1, Hq, D, dtype=BF, device="cuda")
    blocks, out, q = i32([[[0] * 4] * H]), torch.empty_like(done), torch.empty_like(done)
    pool = hg.make_page_pool(i32([[3, -1]]), i32([7]), i32([0, 1, 2, 3, 4]), i32([3]), 16)
    targets, length, result = i32([0]), i32([0]), i32([0] * 4)
    weight = torch.randn(4096, 4096, device="cuda") / 64
    big = weight.clone()

    def calls(stream):
        hg.hg_resize_rows(pool, targets, result, stream=stream)
        hg.hg_append_kv8(d, None, late[:, :Hq], late[:, Hq:Hq + H], late[:, Hq + H:], length, q, stream=stream)
        hg.hg_select_blocks(d, q, length, blocks, sws, stream=stream)
        hg.hg_decode_attention8(d, q, length, out, ws, blocks=blocks, stream=stream)

    def run(side, named):
        for t, s in zip((c.K, c.V, c.ks, c.vs, c.bounds), state):
            t.copy_(s)
        for t in (late, done, out, q, targets, length, blocks, result):
            t.zero_()
        pool.tensors[1].fill_(7)
        pool.tensors[0].copy_(i32([[3, -1]]))
        pool.tensors[3].fill_(3)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            y = big
            for _ in range(20):  # some milliseconds
                y = y @ weight
            z = y.sum() * 0
            late.copy_(x + z.to(BF))
            targets.copy_(20 + z)
            length.copy_(n + 1 + z)
            if not named:
                calls(None)
        if named:
            calls(side)
        with torch.cuda.stream(side):
            done.copy_(out)
            result.add_(0)
        side.synchronize()
        return [t.clone() for t in (done, q, blocks, result, pool.tensors[1], c.K, c.V, c.ks, c.vs, c.bounds)]

    want = run(torch.cuda.current_stream(), False)
    torch.cuda.synchronize()
    assert want[3].tolist() == [0, 0, 13, 2] and int(want[4]) == 20
    assert bool((want[0] != 0).any()) and torch.equal(raw(want[1]), raw(x[:, :Hq]))
    side = torch.cuda.Stream()
    for named in (False, True):
        for a, b in zip(run(side, named), want):
            assert torch.equal(raw(a), raw(b))
