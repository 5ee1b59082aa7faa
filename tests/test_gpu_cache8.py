"""The 8-bit cache's calls on the GPU (append, decode, blocks chosen by a score)
against plain forms on the CPU: codes, scales, bounds and chosen blocks bit for
bit, attention within attnref's bounds; and the pages of rows."""
import math
import random

import pytest
import torch

import attnref
import cache8ref as ref
from attnref import assert_close

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
F8 = torch.float8_e4m3fn


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g).to(BF)


def raw(t):
    """The bytes of a tensor, for comparison."""
    t = t.contiguous()
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32, 8: torch.int64}[t.element_size()])


def offsets(n):
    cu = [0]
    for x in n:
        cu.append(cu[-1] + x)
    return cu


class Cache:
    """An 8-bit cache of junk (NaN codes and scales) with shuffled pages for rows of `lens` tokens."""

    def __init__(self, lens, H, D, page_size, block, seed=0, token_major=False, spare=2, junk=0x7F, bounds=True, device="cuda"):
        need = [-(-n // page_size) for n in lens]
        self.pages = sum(need) + spare
        order = list(range(self.pages))
        random.Random(seed).shuffle(order)
        cols = max(max(need, default=0), 1) + 1
        self.rows, at = [], 0
        for n in need:
            self.rows.append(order[at:at + n] + [-7] * (cols - n))  # entries past a row's pages are not read
            at += n
        self.H, self.D, self.ps, self.block = H, D, page_size, block
        shape = (self.pages, page_size, H, D) if token_major else (self.pages, H, page_size, D)
        self.K, self.V = (torch.full(shape, junk, dtype=torch.uint8, device=device) for _ in range(2))
        if token_major:
            self.K, self.V = self.K.transpose(1, 2), self.V.transpose(1, 2)
        n = page_size // block
        self.ks, self.vs = (torch.full((self.pages, H, n), math.nan, device=device) for _ in range(2))
        self.bounds = torch.full((self.pages, H, n, 2, D), math.nan, dtype=BF, device=device) if bounds else None
        self.table = torch.tensor(self.rows, dtype=torch.int32, device=device).view(len(lens), cols)

    def descriptor(self):
        import paper_2609_35800_amd as hg
        return hg.make_cache8(self.K, self.V, self.ks, self.vs, self.table, self.bounds)

    def host(self):
        return [t.cpu().clone() if t is not None else None for t in (self.K, self.V, self.ks, self.vs, self.bounds)]

    def fill(self, lens, g, starts=None, peak=1.0):
        """Random codes and scales for the rows' tokens; returned on the CPU too."""
        K, V, ks, vs, _ = self.host()
        for b, n in enumerate(lens):
            lo = 0 if starts is None else min(starts[b], n)
            for t in range(lo // self.block * self.block, n, self.block):
                page, off = self.rows[b][t // self.ps], t % self.ps
                for scales in (ks, vs):
                    scales[page, :, off // self.block] = torch.randint(-3, 2, (self.H,), generator=g).float().exp2() * peak / 64
                a, z = max(t, lo), min(t + self.block, n)
                for codes in (K, V):
                    x = torch.randn((self.H, z - a, self.D), generator=g, dtype=torch.float64) * 40
                    codes[page, :, a % self.ps:a % self.ps + z - a] = ref.to_codes(x.clamp(-448, 448))
        for dst, src in ((self.K, K), (self.V, V), (self.ks, ks), (self.vs, vs)):
            dst.copy_(src)
        return K, V, ks, vs

    def gather(self, codes, scales, b, h, tokens):
        """Values [n, D] of a row's tokens (those in no page left out)."""
        t = torch.as_tensor(tokens, dtype=torch.long)
        page = torch.tensor(self.rows[b])[t // self.ps]
        good = (page >= 0) & (page < self.pages)
        page, off = page[good], t[good] % self.ps
        return ref.values(codes[page, h, off], scales[page, h, off // self.block])


# ------------------------------------------------------------ codes

def test_every_value_becomes_its_nearest_code():
    """All BF16 numbers up to 448, infinities and NaN as values beside one 448 (scale 1),
    one token a row and several tokens a row."""
    import paper_2609_35800_amd as hg
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(BF)
    x = every.float()
    x = every[~(x.abs() > 448) | torch.isinf(x)]
    D, block = 64, 16
    x = torch.cat((x, torch.zeros(-len(x) % (D - 1), dtype=BF))).view(-1, 1, D - 1)
    v = torch.cat((torch.full((len(x), 1, 1), 448.0, dtype=BF), x), 2)
    n = len(v)
    for new in ([1] * n, [n]):
        c = Cache(new, 1, D, block, block)
        hg.hg_append_kv8(c.descriptor(), None, None, v.cuda(), v.cuda(), i32(new),
                         cu_new=None if len(new) > 1 else i32([0, n]))
        torch.cuda.synchronize()
        want = ref.to_codes(v.double())[:, 0]
        for codes, scales in ((c.K, c.ks), (c.V, c.vs)):
            for b in range(len(new)):
                t = torch.arange(new[b])
                page = torch.tensor(c.rows[b])[t // block].cuda()
                got = codes[page, 0, (t % block).cuda()].cpu()
                w = want[b:b + 1] if len(new) > 1 else want
                assert bool(ref.same_codes(got, w).all())
                assert bool((scales[page] == 1).all())
                if len(new) > 1 and b > 70:
                    break


def test_every_code_at_every_scale_is_read_exactly():
    """Rows of one token: the output is the value itself, for all codes and scales."""
    import paper_2609_35800_amd as hg
    B, D = 220, 256
    c = Cache([1] * B, 1, D, 16, 16)
    codes = torch.arange(256, dtype=torch.uint8)
    codes = torch.where((codes & 0x7F) == 0x7F, 0, codes)
    scale = torch.tensor([2.0 ** (e - 100) for e in range(B)])
    page = torch.tensor([r[0] for r in c.rows])
    c.V[page.cuda(), 0, 0] = codes.cuda()
    c.K[page.cuda(), 0, 0] = 0
    c.ks[page.cuda(), 0, 0] = c.vs[page.cuda(), 0, 0] = scale.cuda()
    q = torch.ones((B, 1, D), dtype=BF, device="cuda")
    out = torch.empty_like(q)
    d = c.descriptor()
    hg.hg_decode_attention8(d, q, i32([1] * B), out, hg.alloc_decode8_workspace(d, 1))
    torch.cuda.synchronize()
    want = ref.VALUES[codes.long()].view(1, D) * scale.double().view(B, 1)
    assert torch.equal(out[:, 0].double().cpu(), want)


# ------------------------------------------------------------ append

APPEND = [  # D, Hq, H, rot, interleaved, sections, block, pages of blocks, token_major, tokens before, new (None: one a row)
    (128, 28, 4, 128, 0, (16, 24, 24), 16, 1, False, [0, 1, 15, 16, 37], None),
    (64, 6, 2, 32, 0, None, 32, 3, True, [31, 32, 95, 96], None),
    (256, 16, 8, 256, 1, None, 128, 1, False, [0, 127, 200], None),
    (128, 8, 8, 128, 1, None, 64, 1, True, [0, 3, 63, 64, 130], [5, 0, 1, 70, 200]),
    (64, 6, 2, 32, 0, None, 16, 5, False, [9, 0, 80], [33, 2, 17]),
    (64, 3, 3, 48, 1, (8, 12, 4), 16, 1, False, [0, 5, 100], [3, 9, 1]),
    (256, 16, 8, 256, 0, None, 128, 2, False, [100], [300]),
    (256, 1, 1, 64, 0, (9, 13, 10), 32, 1, True, [1, 0], [101, 1]),
    (128, 64, 1, 0, 0, None, 128, 1, False, [0, 7], [2, 131]),
    (64, 130, 70, 64, 0, None, 64, 1, False, [70], [4]),
    (128, 0, 2, 128, 0, None, 16, 2, False, [3], [40]),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", APPEND, ids=str)
def test_append(case, in_place):
    """Two calls, the second with keys and values up to eight times the first's, so that
    scales grow under tokens that are there."""
    import paper_2609_35800_amd as hg
    D, Hq, H, rot, inter, sections, block, blocks, token_major, before, new = case
    g = gen(D + Hq + block)
    B, ps = len(before), block * blocks
    calls = [(before, offsets(before)), (None if new is None else new, None)]
    n_new = [1] * B if new is None else new
    lens = [a + n for a, n in zip(before, n_new)]
    c = Cache(lens, H, D, ps, block, 5, token_major)
    max_pos = 500
    cos, sin = attnref.table(max_pos, max(rot // 2, 1))
    rotation = hg.make_rotation(cos.cuda(), sin.cuda(), inter, sections) if rot else None
    use_positions = sections is not None or inter == 1
    d = c.descriptor()
    start = [0] * B
    for call in range(2):
        counts = before if call == 0 else n_new
        N = sum(counts)
        if N == 0:
            continue
        cu = offsets(counts)
        ends = [a + n for a, n in zip(start, counts)]
        qkv = randn(g, N, Hq + 2 * H, D) * torch.randint(0, 4, (N, Hq + 2 * H, 1), generator=g).float().exp2().to(BF) ** call
        dev = qkv.cuda()
        q, k, v = dev[:, :Hq], dev[:, Hq:Hq + H], dev[:, Hq + H:]
        q_out = (q if in_place else torch.zeros(N, Hq, D, dtype=BF, device="cuda")) if Hq else None
        k_out = k if in_place else torch.zeros(N, H, D, dtype=BF, device="cuda")
        positions = torch.randint(0, max_pos, (3, N) if sections else (N,), generator=g, dtype=torch.int32)
        state = c.host()
        hg.hg_append_kv8(d, rotation, q if Hq else None, k, v, i32(ends), q_out,
                         cu_new=None if call == 1 and new is None else i32(cu),
                         positions=positions.cuda() if use_positions else None, k_out=k_out)
        torch.cuda.synchronize()
        kh = k_out.cpu()
        for b in range(B):
            for j in range(counts[b]):
                t, idx = cu[b] + j, start[b] + j
                i = torch.arange(rot // 2)
                if rot and sections:
                    axis = (i >= sections[0]).long() + (i >= sections[0] + sections[1]).long()
                    pos = positions[axis, t].long()
                else:
                    pos = torch.full((rot // 2,), int(positions[t]) if use_positions else idx)
                cs, sn = (cos[pos, i], sin[pos, i]) if rot else (torch.zeros(0), torch.zeros(0))
                if Hq:
                    assert_close(q_out[t].cpu(), *attnref.rotate(qkv[t, :Hq], cs, sn, inter), f"q of token {t}")
                assert_close(kh[t], *attnref.rotate(qkv[t, Hq:Hq + H], cs, sn, inter), f"key of token {t}")
            lo, hi = cu[b], cu[b + 1]
            ref.append(state[0], state[2], state[4], c.rows[b], ps, block, start[b], kh[lo:hi])
            ref.append(state[1], state[3], None, c.rows[b], ps, block, start[b], qkv[lo:hi, Hq + H:])
        # everything else as it was, junk among it
        for name, got, want in zip(("K", "V", "k_scale", "v_scale", "bounds"), c.host(), state):
            if name == "bounds":
                same = (got == want) | (raw(got) == raw(want))
            else:
                same = raw(got) == raw(want)
            assert bool(same.all()), f"call {call}: {name}: {int((~same).sum())} differ"
        start = ends
    if not in_place:
        assert torch.equal(raw(dev), raw(qkv.cuda()))


@pytest.mark.parametrize("single", [True, False])
def test_append_of_numbers_that_are_not(single):
    """Infinities become the largest code, NaN stays; neither counts for the scale; zeros
    get the smallest scale; a block of NaN alone has the bounds inf, -inf."""
    import paper_2609_35800_amd as hg
    D, H, block = 128, 4, 16
    g = gen(1)
    before, n = 3, 1 if single else 18
    c = Cache([before + n], H, D, block, block)
    x = randn(g, before, H, D).cuda()
    d = c.descriptor()
    hg.hg_append_kv8(d, None, None, x, x, i32([before]), cu_new=i32([0, before]))
    y = randn(g, n, H, D)
    y[0, 0, 3], y[0, 0, 5], y[-1, 0, 7] = math.inf, -math.inf, math.nan
    y[:, 1] = math.nan
    y[:, 2] = 0.0
    y[0, 3], y[0, 3, 0] = 3.0e38, -math.inf
    state = c.host()
    hg.hg_append_kv8(d, None, None, y.cuda(), y.cuda(), i32([before + n]), cu_new=None if single else i32([0, n]))
    torch.cuda.synchronize()
    ref.append(state[0], state[2], state[4], c.rows[0], block, block, before, y)
    ref.append(state[1], state[3], None, c.rows[0], block, block, before, y)
    got = c.host()
    for i in range(2):
        assert bool(ref.same_codes(got[i], state[i]).all())
        assert torch.equal(raw(got[i + 2]), raw(state[i + 2]))
    assert bool(((got[4] == state[4]) | (torch.isnan(got[4]) & torch.isnan(state[4]))).all())
    if not single:
        page = c.rows[0][1]
        assert float(got[2][page, 2, 0]) == 2.0 ** -100
        assert bool((got[4][page, 1, 0, 0] == math.inf).all()) and bool((got[4][page, 1, 0, 1] == -math.inf).all())


def test_append_of_the_smallest_and_largest():
    """Scales at both ends of their range, and steps from one end to the other."""
    import paper_2609_35800_amd as hg
    D, H, block = 64, 1, 16
    c = Cache([40], H, D, block, block)
    d = c.descriptor()
    state = c.host()
    g = gen(2)
    at = 0
    for n, size in ((2, 2.0 ** -120), (1, 2.0 ** -90), (3, 1.0), (2, 2.0 ** 120), (16, 2.0 ** -126), (1, 3.0e38), (4, 1.75 * 2.0 ** 8), (2, 1.7578125 * 2.0 ** 8)):
        x = (randn(g, n, H, D).clamp(-1, 1).float() * size).to(BF)
        x[-1, 0, 0] = size
        hg.hg_append_kv8(d, None, None, x.cuda(), x.cuda(), i32([at + n]), cu_new=i32([0, n]) if n > 1 else None)
        torch.cuda.synchronize()
        ref.append(state[0], state[2], state[4], c.rows[0], block, block, at, x)
        ref.append(state[1], state[3], None, c.rows[0], block, block, at, x)
        at += n
        got = c.host()
        for i in range(2):
            # a rounding to 0 keeps its sign
            assert bool(ref.same_codes(got[i], state[i]).all()) and torch.equal(raw(got[i + 2]), raw(state[i + 2])), (at, size)
        assert bool(((got[4] == state[4]) | (torch.isnan(got[4]) & torch.isnan(state[4]))).all())


def test_append_skips_what_has_no_place():
    """Padding tokens, pages outside the cache, indexes past the table, positions outside
    the rotation's: no other byte changes, and blocks without new tokens keep their scales."""
    import paper_2609_35800_amd as hg
    D, Hq, H, block = 64, 2, 2, 16
    g = gen(3)
    c = Cache([64], H, D, block, block, spare=0)
    c.table = i32([[0, 9], [1, -1], [2, 3]])
    c.rows = [[0, 9], [1, -1], [2, 3]]
    cu = [0, 20, 24, 30]  # tokens 30 and 31 belong to no row
    N = 32
    q, k, v = (randn(g, N, H, D) for _ in range(3))
    q_out = torch.full((N, Hq, D), math.nan, dtype=BF, device="cuda")
    k_out = torch.full((N, H, D), math.nan, dtype=BF, device="cuda")
    cos, sin = attnref.table(40, D // 2)
    lens = [20, 18, 34]  # row 0: 16 .. in page 9; row 1: 16, 17 in page -1; row 2: 28 .., 32 and 33 past the table
    positions = torch.arange(N, dtype=torch.int32) % 40
    positions[3], positions[21], positions[24:28] = -1, 40, 1000  # row 2: nothing of block 1 but 28 .. 31 remain
    state = c.host()
    hg.hg_append_kv8(c.descriptor(), hg.make_rotation(cos.cuda(), sin.cuda()), q.cuda(), k.cuda(), v.cuda(), i32(lens), q_out,
                     cu_new=i32(cu), positions=positions.cuda(), k_out=k_out)
    torch.cuda.synchronize()
    ok = (positions >= 0) & (positions < 40)
    kh = k_out.cpu()
    for b in range(3):
        lo, hi = cu[b], cu[b + 1]
        start = lens[b] - (hi - lo)
        n = min(hi - lo, 32 - start)
        ref.append(state[0], state[2], state[4], c.rows[b], block, block, start, kh[lo:lo + n].nan_to_num(), ok[lo:lo + n])
        ref.append(state[1], state[3], None, c.rows[b], block, block, start, v[lo:lo + n], ok[lo:lo + n])
    for got, want in zip(c.host(), state):
        assert bool(((got == want) | (raw(got) == raw(want))).all())
    done = torch.isfinite(q_out.float()).all(-1).all(1).cpu()
    ok[30:] = False
    assert torch.equal(done, ok) and torch.equal(torch.isfinite(kh.float()).all(-1).all(1), ok)
    # one token a row: skipped tokens leave everything alone
    before = c.host()
    hg.hg_append_kv8(c.descriptor(), hg.make_rotation(cos.cuda(), sin.cuda()), None, k[:3].cuda(), v[:3].cuda(), i32([17, 18, 33]),
                     positions=i32([0, 1, 2]))
    hg.hg_append_kv8(c.descriptor(), hg.make_rotation(cos.cuda(), sin.cuda()), None, k[:3].cuda(), v[:3].cuda(), i32([0, 5, 6]),
                     positions=i32([0, -1, 40]))
    torch.cuda.synchronize()
    assert all(torch.equal(raw(a), raw(b)) for a, b in zip(before, c.host()))


def test_append_without_bounds_and_large():
    """A call past 256 MiB streams; every element against the definition, on the GPU in 64 bits."""
    import paper_2609_35800_amd as hg
    D, Hq, H, block = 128, 1, 4, 64
    lens = [(300 << 20) // (D * (4 * Hq + 6 * H)) - 77, 77]
    N = sum(lens)
    c = Cache(lens, H, D, 128, block, junk=0, bounds=False)
    gpu = torch.Generator(device="cuda").manual_seed(D)
    qkv = torch.randn((N, Hq + 2 * H, D), generator=gpu, device="cuda").to(BF)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    q_out = torch.empty((N, Hq, D), dtype=BF, device="cuda")
    hg.hg_append_kv8(c.descriptor(), None, q, k, v, i32(lens), q_out, cu_new=i32([0, lens[0], N]))
    torch.cuda.synchronize()
    assert torch.equal(raw(q_out), raw(q))
    index = torch.cat([torch.arange(n) for n in lens])
    page = torch.cat([torch.tensor(c.rows[b])[torch.arange(n) // 128] for b, n in enumerate(lens)]).cuda()
    off = (index % 128).cuda()
    local = torch.cat((index[:lens[0]] // block, lens[0] // block + 1 + index[lens[0]:] // block)).cuda()
    for codes, scales, x in ((c.K, c.ks, k), (c.V, c.vs, v)):
        most = torch.zeros((int(local.max()) + 1, H), device="cuda").scatter_reduce(
            0, local.view(-1, 1).expand(N, H), x.abs().amax(-1).float(), "amax")
        want = torch.exp2(torch.ceil(torch.log2(most.double() / 448)))[local]
        assert torch.equal(scales[page, :, off // block].double(), want)
        exact = x.double() / want.unsqueeze(-1)
        assert torch.equal(codes[page, :, off], exact.float().to(F8).view(torch.uint8))


# ------------------------------------------------------------ decode

def check_decode(lens, Hq, H, D, block, pages=1, seed=0, starts=None, token_major=False, scale=None, peak=1.0, calls=1,
                 blocks=None, workspace=None, c=None):
    """blocks [B][H][budget] (host) or None."""
    import paper_2609_35800_amd as hg
    g = gen(seed)
    B = len(lens)
    c = c or Cache(lens, H, D, block * pages, block, seed, token_major)
    K, V, ks, vs = c.fill(lens, g, starts, peak)
    q = randn(g, B, Hq, D)
    scale = D ** -0.5 if scale is None else scale
    out = torch.full((B, Hq, D), math.nan, dtype=BF, device="cuda")
    lse = torch.full((B, Hq), math.nan, device="cuda")
    d = c.descriptor()
    ws = hg.alloc_decode8_workspace(d, Hq) if workspace is None else workspace
    listed = None if blocks is None else i32(blocks)
    first = None
    for _ in range(calls):
        out.fill_(math.nan)
        hg.hg_decode_attention8(d, q.cuda(), i32(lens), out, ws, starts=None if starts is None else i32(starts), lse=lse,
                                scale=scale, blocks=listed)
        torch.cuda.synchronize()
        if first is None:
            first = out.clone(), lse.clone()
        assert torch.equal(raw(out), raw(first[0])) and torch.equal(raw(lse), raw(first[1]))
    assert int(ws[:4096].sum()) == 0  # 1024 counters, ready for the next call
    R = Hq // H
    for b in range(B):
        lo, hi = (0 if starts is None else min(starts[b], lens[b])), lens[b]
        n = (hi - 1) // block - lo // block + 1 if hi > lo else 0
        for h in range(H):
            tokens = list(range(lo, hi))
            if blocks is not None:
                tokens = [t for i in blocks[b][h][:n] if i >= 0 for t in range(i * block, i * block + block) if lo <= t < hi]
            k, v = c.gather(K, ks, b, h, tokens), c.gather(V, vs, b, h, tokens)
            o, l, to, tl = attnref.attend(q[b, h * R:(h + 1) * R], k, v, scale)
            assert_close(out[b, h * R:(h + 1) * R], o, to, f"row {b} head {h}")
            assert_close(lse[b, h * R:(h + 1) * R], l, tl, f"log-sum of row {b} head {h}")


DECODE = [  # Hq, H, D, block, pages of blocks
    (28, 4, 128, 16, 1), (8, 8, 64, 32, 3), (16, 8, 256, 64, 1), (5, 1, 128, 128, 2), (24, 1, 128, 16, 4), (35, 1, 256, 32, 1),
    (40, 2, 64, 128, 1), (8, 4, 128, 64, 5),
]
EDGES = [0, 1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 257, 513]


@pytest.mark.parametrize("case", DECODE, ids=str)
@pytest.mark.parametrize("starts", [False, True])
def test_decode_lengths(case, starts):
    Hq, H, D, block, pages = case
    r = random.Random(Hq + D)
    check_decode(EDGES, Hq, H, D, block, pages, starts=[r.randint(0, n + 1) for n in EDGES] if starts else None, calls=2,
                 token_major=starts)


@pytest.mark.parametrize("D,H,R", [(64, 1, 1), (128, 2, 7), (256, 1, 16), (128, 1, 20)])
def test_decode_one_long_row(D, H, R):
    """Rows split over many workgroups, and joined in two steps."""
    check_decode([9001], H * R, H, D, 64, calls=2)
    check_decode([9001, 3], H * R, H, D, 16, starts=[4321, 1])


@pytest.mark.parametrize("D", [64, 128, 256])
def test_decode_many_rows(D):
    """More (row, head)s than slots: workgroups take shares of the list of chunks."""
    r = random.Random(D)
    check_decode([r.choice([0, 1, 70, 200, 333]) for _ in range(90)], 8, 4, D, 16, 2, calls=2)


@pytest.mark.parametrize("B,T", [(1, 2300007), (520, 4490)])
def test_decode_long_segments(B, T):
    """Wavefronts of more steps than their lanes hold tiles of (16), in segments and in shares
    of the list; the reference in 64 bits on the GPU, attnref's bounds."""
    import paper_2609_35800_amd as hg
    D, block = 64, 32
    n = -(-T // block)
    gpu = torch.Generator(device="cuda").manual_seed(B)
    K, V = (torch.randn((B * n, 1, block, D), generator=gpu, device="cuda").mul_(30).clamp_(-448, 448).to(F8).view(torch.uint8)
            for _ in range(2))
    ks, vs = (torch.randint(-7, -3, (B * n, 1, 1), generator=gpu, device="cuda").float().exp2() for _ in range(2))
    table = torch.randperm(B * n, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(B, n).cuda()
    d = hg.make_cache8(K, V, ks, vs, table)
    q = torch.randn((B, 1, D), generator=gpu, device="cuda").to(BF)
    lens = torch.full((B,), T, dtype=torch.int32, device="cuda")
    lens[B // 2] -= 1 if B > 1 else 0
    out, lse = torch.empty_like(q), torch.empty((B, 1), device="cuda")
    hg.hg_decode_attention8(d, q, lens, out, hg.alloc_decode8_workspace(d, 1), lse=lse)
    torch.cuda.synchronize()
    for b in range(0, B, 40):
        page = table[b].long()
        k = (K[page].view(F8).double() * ks[page].double().unsqueeze(-1)).view(-1, D)[:int(lens[b])]
        v = (V[page].view(F8).double() * vs[page].double().unsqueeze(-1)).view(-1, D)[:int(lens[b])]
        s = (k @ q[b, 0].double()) * D ** -0.5
        p = torch.softmax(s, 0)
        E = D * 2.0 ** -23 * D ** -0.5 * float((k.abs() @ q[b, 0].double().abs()).max())
        tol = (2.0 ** -7 * (1 + 2.0 ** -6) + 4 * E) * (p @ v.abs())
        assert bool(((out[b, 0].double() - p @ v).abs() <= tol).all()), b
        exact = float(torch.logsumexp(s, 0))
        assert abs(float(lse[b, 0]) - exact) <= 2 * E + 2.0 ** -20 * (1 + abs(exact)), b


def test_calls_past_4_gib():
    """A pool of 5 GiB of codes, whose last pages the rows use: append, choose, attend."""
    import paper_2609_35800_amd as hg
    D, H, ps, block = 128, 8, 64, 32
    pages = (5 << 30) // (H * ps * D)
    K, V = (torch.zeros((pages, H, ps, D), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.ones((pages, H, ps // block), device="cuda") for _ in range(2))
    bounds = torch.zeros((pages, H, ps // block, 2, D), dtype=BF, device="cuda")
    small = Cache([300, 700], H, D, ps, block)
    table = torch.where(small.table >= 0, pages - small.pages + small.table, small.table)
    far = hg.make_cache8(K, V, ks, vs, table, bounds)
    near = small.descriptor()
    g = gen(8)
    x = randn(g, 1000, 2 * H, D).cuda()
    q = randn(g, 2, 16, D).cuda()
    lens = i32([300, 700])
    got = []
    for d in (near, far):
        hg.hg_append_kv8(d, None, None, x[:, :H], x[:, H:], lens, cu_new=i32([0, 300, 1000]))
        y = randn(gen(9), 2, 2 * H, D).cuda() * 3
        hg.hg_append_kv8(d, None, None, y[:, :H], y[:, H:], lens + 1)
        blocks = torch.empty((2, H, 6), dtype=torch.int32, device="cuda")
        out = torch.empty_like(q)
        hg.hg_select_blocks(d, q, lens + 1, blocks, hg.alloc_select_workspace(d))
        hg.hg_decode_attention8(d, q, lens + 1, out, hg.alloc_decode8_workspace(d, 16), blocks=blocks)
        torch.cuda.synchronize()
        got.append((blocks, out))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(raw(got[0][1]), raw(got[1][1]))
    used = sorted(p for r, n in zip(small.rows, (301, 701)) for p in r[:-(-n // ps)])
    for a, b in ((small.ks, ks), (small.vs, vs), (small.bounds, bounds)):
        for p in used[:3]:
            n = a[p]
            m = b[pages - small.pages + p]
            keep = torch.isfinite(n)
            assert torch.equal(n[keep], m[keep])
    del K, V, far
    torch.cuda.empty_cache()


def test_decode_peaked_and_scaled():
    check_decode([100, 700], 4, 2, 128, 16, peak=64.0)
    check_decode([100, 700], 4, 2, 128, 16, scale=-0.3)
    check_decode([100, 700], 4, 2, 64, 32, scale=0.0)


def test_decode_tokens_without_a_page():
    import paper_2609_35800_amd as hg
    c = Cache([200, 64], 2, 128, 32, 16)
    for b, i, page in ((0, 1, -1), (0, 3, c.pages), (1, 0, 2 ** 31 - 1), (1, 1, -2 ** 31)):
        c.rows[b][i] = page
    c.table.copy_(torch.tensor(c.rows, dtype=torch.int32))
    g = gen(1)
    lens = [200, 64]
    good = Cache([200, 64], 2, 128, 32, 16)
    K, V, ks, vs = good.fill(lens, g)
    for dst, src in ((c.K, K), (c.V, V), (c.ks, ks), (c.vs, vs)):
        dst.copy_(src)
    q = randn(g, 2, 4, 128)
    out = torch.full((2, 4, 128), math.nan, dtype=BF, device="cuda")
    lse = torch.full((2, 4), math.nan, device="cuda")
    d = c.descriptor()
    ws = hg.alloc_decode8_workspace(d, 4)
    # lengths past the table are clamped to it
    hg.hg_decode_attention8(d, q.cuda(), i32(lens), out, ws, lse=lse)
    torch.cuda.synchronize()
    for h in range(2):
        t = [i for i in range(200) if i // 32 not in (1, 3)]
        o, l, to, tl = attnref.attend(q[0, 2 * h:2 * h + 2], c.gather(K, ks, 0, h, t), c.gather(V, vs, 0, h, t), 128 ** -0.5)
        assert_close(out[0, 2 * h:2 * h + 2], o, to, "row 0")
        assert_close(lse[0, 2 * h:2 * h + 2], l, tl, "log-sum of row 0")
    assert bool((out[1] == 0).all()) and bool((lse[1] == -math.inf).all())
    # no tokens at all: negative lengths, an empty table
    hg.hg_decode_attention8(d, q.cuda(), i32([-5, 0]), out.fill_(math.nan), ws, lse=lse)
    torch.cuda.synchronize()
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_decode_lists_of_blocks():
    """Lists in any order, with places left empty, blocks twice and blocks that are not the row's."""
    block, lens, starts = 32, [0, 5, 100, 700, 1000], [0, 2, 40, 0, 333]
    H, budget = 3, 24
    r = random.Random(4)
    lists = []
    for n in lens:
        have = -(-n // block)
        lists.append([[r.choice([-1, -9, have, have + 5, 2 ** 31 - 1] + 9 * [r.randrange(max(have, 1))]) for _ in range(budget)]
                      for _ in range(H)])
    check_decode(lens, 6, H, 128, block, 2, starts=starts, blocks=lists, calls=2)
    check_decode(lens, 6, H, 64, block, 1, blocks=lists)
    check_decode(lens, 60, H, 256, block, 1, blocks=[[x[:1] for x in y] for y in lists])
    check_decode([40 * 128], 1, 1, 128, 128, blocks=[[list(range(39, -1, -1))]])  # all of them, backwards


def test_decode_one_workspace_for_every_call():
    import paper_2609_35800_amd as hg
    K = torch.zeros((4, 2, 16, 256), dtype=BF, device="cuda")
    big = hg.alloc_decode_workspace(hg.make_paged_cache(K, K.clone(), i32([[0]] * 90)), 32)
    check_decode([600, 20], 8, 2, 128, 16, workspace=big)
    # a call of the BF16 cache between
    cache = hg.make_paged_cache(K, K.clone(), i32([[0, 1, 2, 3]]))
    out = torch.empty((1, 32, 256), dtype=BF, device="cuda")
    hg.hg_decode_attention(cache, torch.zeros_like(out), i32([64]), out, big)
    check_decode([3, 4, 500] * 30, 4, 4, 256, 32, workspace=big)
    check_decode([2000], 16, 1, 64, 64, workspace=big)


def test_decode_junk_values_do_not_leak():
    """Infinite and NaN values in one attended token reach only their own channels and heads."""
    import paper_2609_35800_amd as hg
    c = Cache([70], 2, 128, 16, 16)
    g = gen(6)
    K, V, ks, vs = c.fill([70], g)
    page = c.rows[0][2]
    c.V[page, 0, 5, 9] = 0x7F  # token 37
    q = randn(g, 1, 4, 128).cuda()
    out, clean = torch.empty_like(q), torch.empty_like(q)
    d = c.descriptor()
    ws = hg.alloc_decode8_workspace(d, 4)
    hg.hg_decode_attention8(d, q, i32([70]), out, ws)
    hg.hg_decode_attention8(d, q, i32([37]), clean, ws)
    torch.cuda.synchronize()
    assert torch.isnan(out[0, :2, 9]).all()
    out[0, :2, 9] = 0
    assert torch.isfinite(out).all() and torch.isfinite(clean).all()
    hg.hg_decode_attention8(d, q, i32([70]), out, ws, starts=i32([38]))
    assert torch.isfinite(out).all()


# ------------------------------------------------------------ blocks chosen by their bounds

def check_select(lens, Hq, H, D, block, budget, first, last, pages=1, starts=None, seed=0, q=None, edit=None):
    import paper_2609_35800_amd as hg
    g = gen(seed)
    B = len(lens)
    c = Cache(lens, H, D, block * pages, block, seed)
    x = torch.randn(c.bounds.shape, generator=g)
    x = torch.stack((x.amin(3), x.amax(3)), 3).to(BF)
    if edit:
        edit(c, x)
    c.bounds.copy_(x)
    c.table.copy_(torch.tensor(c.rows, dtype=torch.int32))
    q = randn(g, B, Hq, D) if q is None else q
    blocks = torch.full((B, H, budget), -99, dtype=torch.int32, device="cuda")
    d = c.descriptor()
    ws = hg.alloc_select_workspace(d)
    for _ in range(2):
        ws.fill_(255)
        hg.hg_select_blocks(d, q.cuda(), i32(lens), blocks, ws, starts=None if starts is None else i32(starts), first=first, last=last)
        torch.cuda.synchronize()
        got = blocks.cpu().tolist()
        for b in range(B):
            lo, hi = (0 if starts is None else min(starts[b], lens[b])), lens[b]
            ids = range(lo // block, (hi - 1) // block + 1) if hi > lo else []
            for h in range(H):
                limits = []
                for i in ids:
                    page = c.rows[b][i * block // c.ps]
                    limits.append(x[page, h, i * block % c.ps // block] if 0 <= page < c.pages else None)
                want = ref.select(q[b, h * (Hq // H):(h + 1) * (Hq // H)], limits, lo // block, budget, first, last)
                assert got[b][h] == want, f"row {b} head {h}"
    return c


SELECT = [  # Hq, H, D, block, pages, budget, first, last
    (28, 4, 128, 16, 1, 8, 1, 2), (8, 8, 64, 32, 3, 3, 0, 0), (2, 1, 256, 64, 1, 1, 0, 1), (6, 2, 128, 128, 2, 2, 1, 1),
    (16, 1, 64, 16, 2, 40, 0, 3), (3, 3, 256, 16, 1, 12, 5, 7),
]


@pytest.mark.parametrize("case", SELECT, ids=str)
@pytest.mark.parametrize("starts", [False, True])
def test_select_lengths(case, starts):
    Hq, H, D, block, pages, budget, first, last = case
    r = random.Random(D + budget)
    lens = [0, 1, block, block + 1, budget * block, budget * block + 1, (budget + 1) * block, 1500, 2001]
    check_select(lens, Hq, H, D, block, budget, first, last, pages, [r.randint(0, n + 1) for n in lens] if starts else None)


@pytest.mark.parametrize("budget", [1, 64, 1000])
def test_select_of_a_long_row(budget):
    check_select([16 * 2500 + 3], 2, 1, 64, 16, budget, 0, 0 if budget == 1 else 1)


def test_select_in_a_wide_table():
    """A row of 513 blocks, the shortest that several workgroups score, in a table for
    200000: more workgroups than blocks."""
    import paper_2609_35800_amd as hg
    g = gen(3)
    c = Cache([16 * 513], 1, 64, 16, 16)
    c.table = torch.full((1, 200000), -1, dtype=torch.int32, device="cuda")
    c.table[0, :513] = i32(c.rows[0][:513])
    x = torch.randn(c.bounds.shape, generator=g)
    x = torch.stack((x.amin(3), x.amax(3)), 3).to(BF)
    c.bounds.copy_(x)
    d = c.descriptor()
    q = randn(g, 1, 2, 64)
    ws = hg.alloc_select_workspace(d)
    for n in (513, 512, 40):
        blocks = torch.full((1, 1, 30), -99, dtype=torch.int32, device="cuda")
        hg.hg_select_blocks(d, q.cuda(), i32([16 * n]), blocks, ws)
        torch.cuda.synchronize()
        assert blocks[0, 0].tolist() == ref.select(q[0], [x[c.rows[0][i], 0, 0] for i in range(n)], 0, 30, 1, 2)


def test_select_ties_go_to_the_lower_block():
    """Few different scores, the same everywhere, and infinities of either sign."""
    def few(c, x):
        x.copy_(torch.randint(-1, 2, x.shape[:3], generator=gen(5)).float()[..., None, None].expand(x.shape))

    def same(c, x):
        x.fill_(1.0)

    def wild(c, x):
        x[::3, :, :, 1] = math.inf
        x[1::3, :, :, 0] = -math.inf
        x[2::3, :, :, 1, 0] = math.nan

    q = torch.ones(1, 2, 64, dtype=BF)
    for edit in (few, same):
        for budget in (1, 7, 130):
            check_select([16 * 1200], 2, 1, 64, 16, budget, 0, 1, edit=edit, q=q)
    check_select([16 * 300], 2, 1, 64, 16, 60, 0, 0, edit=wild)
    check_select([16 * 300], 2, 1, 64, 16, 60, 0, 0, edit=wild, q=torch.zeros(1, 2, 64, dtype=BF))
    check_select([16 * 300], 2, 1, 64, 16, 250, 1, 1, edit=wild, q=torch.full((1, 2, 64), math.nan).to(BF))


def test_select_near_scores_and_missing_pages():
    """Scores that fp32 could not tell apart; blocks without a page come last, lower ones first."""
    def near(c, x):
        x[..., 0, :] = 1024.0
        x[..., 1, :] = 1024.0
        x[..., 1, 0] = 0.0
        x[..., 0, 0] = -(2.0 ** -20) * torch.randint(1, 200, x.shape[:3], generator=gen(9))

    q = torch.ones(1, 1, 128, dtype=BF)
    q[0, 0, 0] = -2.0 ** -10
    check_select([16 * 700], 1, 1, 128, 16, 50, 0, 0, edit=near, q=q)

    def lost(c, x):
        for i in range(0, 100, 3):
            c.rows[0][i] = [-1, c.pages, -2 ** 31][i % 3]

    check_select([16 * 100], 2, 2, 128, 16, 80, 1, 2, edit=lost)


def test_sparse_attention_is_the_attention_of_the_chosen_blocks():
    """Append, choose, attend, as a decode step does; all blocks chosen give the dense result bit for bit."""
    import paper_2609_35800_amd as hg
    D, Hq, H, block, ps = 128, 8, 2, 16, 32
    lens = [5, 300, 777]
    g = gen(11)
    c = Cache([n + 1 for n in lens], H, D, ps, block)
    d = c.descriptor()
    N = sum(lens)
    x = randn(g, N, 2 * H, D).cuda()
    hg.hg_append_kv8(d, None, None, x[:, :H], x[:, H:], i32(lens), cu_new=i32(offsets(lens)))
    y = randn(g, 3, Hq + 2 * H, D).cuda()
    q, k, v = y[:, :Hq], y[:, Hq:Hq + H], y[:, Hq + H:]
    cos, sin = attnref.table(800, D // 2)
    q_rot = torch.empty((3, Hq, D), dtype=BF, device="cuda")
    ends = i32([n + 1 for n in lens])
    hg.hg_append_kv8(d, hg.make_rotation(cos.cuda(), sin.cuda()), q, k, v, ends, q_rot)
    ws, sws = hg.alloc_decode8_workspace(d, Hq), hg.alloc_select_workspace(d)
    out, dense = torch.empty_like(q_rot), torch.empty_like(q_rot)
    K, V, ks, vs, bounds = c.host()
    for budget in (5, 49):
        blocks = torch.empty((3, H, budget), dtype=torch.int32, device="cuda")
        hg.hg_select_blocks(d, q_rot, ends, blocks, sws)
        hg.hg_decode_attention8(d, q_rot, ends, out, ws, blocks=blocks)
        hg.hg_decode_attention8(d, q_rot, ends, dense, ws)
        torch.cuda.synchronize()
        if budget == 49:
            assert torch.equal(raw(out), raw(dense))
            continue
        R = Hq // H
        for b, n in enumerate(lens):
            for h in range(H):
                qh = q_rot[b, h * R:(h + 1) * R].cpu()
                ids = range(n // block + 1)
                limits = [bounds[c.rows[b][i * block // ps], h, i * block % ps // block] for i in ids]
                want = ref.select(qh, limits, 0, budget, 1, 2)
                assert blocks[b, h].tolist() == want
                t = [t for i in want if i >= 0 for t in range(i * block, min(i * block + block, n + 1))]
                o, _, to, _ = attnref.attend(qh, c.gather(K, ks, b, h, t), c.gather(V, vs, b, h, t), D ** -0.5)
                assert_close(out[b, h * R:(h + 1) * R], o, to, f"row {b} head {h}")


# ------------------------------------------------------------ pages of rows

def check_resize(hg, pool, sim, targets, room, slots=True, positions=True):
    """One call against the plain form, pool and outputs."""
    table, lens, free, n_free = pool.tensors
    B = table.shape[0]
    cu = torch.full((B + 1,), -5, dtype=torch.int32, device="cuda")
    s = torch.full((room,), -5, dtype=torch.int64, device="cuda") if slots else None
    p = torch.full((room,), -5, dtype=torch.int32, device="cuda") if positions else None
    result = torch.full((4,), -5, dtype=torch.int32, device="cuda")
    hg.hg_resize_rows(pool, i32(targets), result, cu_new=cu, slots=s, positions=p)
    torch.cuda.synchronize()
    want = sim.resize(targets, room if slots or positions else None)
    assert result.tolist() == want[0]
    assert cu.tolist() == want[1]
    if slots:
        assert s.tolist() == want[2]
    if positions:
        assert p.tolist() == want[3]
    assert table.cpu().tolist() == sim.table and lens.tolist() == sim.lens
    assert int(n_free) == sim.n and free[:sim.n].tolist() == sim.free[:sim.n]
    return want[0][0]


def new_pool(hg, B, max_pages, num_pages, ps):
    pool = hg.alloc_page_pool(B, max_pages, num_pages, ps)
    table, lens, free, n_free = (t.cpu().tolist() for t in pool.tensors)
    return pool, ref.Pool(table, lens, free, n_free[0], ps)


@pytest.mark.parametrize("B,max_pages,num_pages,ps,room", [(1, 4, 4, 16, 64), (5, 7, 30, 16, 200), (33, 9, 200, 1, 300),
                                                           (70, 50, 1500, 7, 9000), (1100, 3, 2500, 16, 20000)])
def test_resize_random_calls(B, max_pages, num_pages, ps, room):
    import paper_2609_35800_amd as hg
    pool, sim = new_pool(hg, B, max_pages, num_pages, ps)
    r = random.Random(B)
    seen = set()
    for i in range(24):
        most = max_pages * ps
        kind = i % 6
        if kind == 0:
            targets = [r.randint(0, most) if r.random() < 0.7 else 0 for _ in range(B)]
        elif kind in (1, 2, 3):
            targets = [min(most, n + r.choice([0, 1, 1, 1, 3])) for n in sim.lens]
        elif kind == 4:
            targets = [max(0, n - r.randint(0, ps)) for n in sim.lens]
        else:
            targets = [r.randint(0, n) if r.random() < 0.5 else n for n in sim.lens]
            if i > 12 and B > 1:
                targets[r.randrange(B)] = r.choice([-1, most + 1, 2 ** 31 - 1, -2 ** 31])
        seen.add(check_resize(hg, pool, sim, targets, room, slots=i % 4 != 3, positions=i % 5 != 4))
    assert 0 in seen
    held = sorted(p for b, row in enumerate(sim.table) for p in row[:sim.pages(sim.lens[b])])
    assert sorted(held + sim.free[:sim.n]) == list(range(num_pages))  # no page is lost or had twice


def test_resize_refusals_on_the_gpu():
    """Each reason alone, several at once; nothing of the pool changes."""
    import paper_2609_35800_amd as hg
    pool, sim = new_pool(hg, 3, 4, 6, 16)
    assert check_resize(hg, pool, sim, [16, 17, 0], 64) == 0
    assert check_resize(hg, pool, sim, [64, 17, 40], 200) == 1
    assert check_resize(hg, pool, sim, [65, 17, 0], 200) == 2
    assert check_resize(hg, pool, sim, [16, 17, 5], 4) == 4
    assert check_resize(hg, pool, sim, [64, 64, -3], 50) == 7
    assert check_resize(hg, pool, sim, [16, 17, 5], 5) == 0
    pool.tensors[3].fill_(7)
    sim.n = 7
    assert check_resize(hg, pool, sim, [16, 17, 6], 5) & 8
    pool.tensors[3].fill_(-1)
    sim.n = -1
    assert check_resize(hg, pool, sim, [16, 17, 6], 5) & 8
    # a length that is not the table's
    pool.tensors[3].fill_(2)
    sim.n = 2
    pool.tensors[1][1] = 1000
    sim.lens[1] = 1000
    assert check_resize(hg, pool, sim, [16, 17, 6], 5) == 2


def test_resize_large_and_empty():
    import paper_2609_35800_amd as hg
    pool, sim = new_pool(hg, 3, 40000, 90000, 16)
    assert check_resize(hg, pool, sim, [500000, 1, 640000], 1200000) == 0
    assert check_resize(hg, pool, sim, [0, 640000, 17], 700000) == 0
    assert check_resize(hg, pool, sim, [0, 0, 0], 5, slots=False, positions=False) == 0
    pool, sim = new_pool(hg, 0, 4, 6, 16)
    check_resize(hg, pool, sim, [], 3)
    pool, sim = new_pool(hg, 2, 0, 6, 16)
    assert check_resize(hg, pool, sim, [0, 0], 3) == 0
    assert check_resize(hg, pool, sim, [0, 1], 3) & 2
    pool, sim = new_pool(hg, 2, 3, 0, 16)
    assert check_resize(hg, pool, sim, [0, 1], 3) == 1


# ------------------------------------------------------------ together, captured

def test_a_captured_step_of_all_calls():
    """Rows grow, keys and values are appended, blocks chosen and attended, in one graph;
    every replay gives the eager run's pool, cache, choice and output."""
    import paper_2609_35800_amd as hg
    D, Hq, H, block, ps, B, budget = 128, 8, 2, 16, 32, 3, 4

    def setup():
        pool = hg.alloc_page_pool(B, 12, 30, ps)
        c = hg.alloc_cache8(30, H, ps, D, pool.tensors[0], block)
        s = dict(pool=pool, cache=c, targets=i32([0] * B), result=i32([0] * 4), cu=i32([0] * (B + 1)),
                 positions=torch.zeros(3 * B, dtype=torch.int32, device="cuda"),
                 slots=torch.zeros(3 * B, dtype=torch.int64, device="cuda"))
        s["x"] = torch.zeros((3 * B, Hq + 2 * H, D), dtype=BF, device="cuda")
        s["q"] = torch.zeros((3 * B, Hq, D), dtype=BF, device="cuda")
        s["last"] = torch.zeros((B, Hq, D), dtype=BF, device="cuda")
        s["blocks"] = torch.zeros((B, H, budget), dtype=torch.int32, device="cuda")
        s["out"] = torch.zeros((B, Hq, D), dtype=BF, device="cuda")
        s["ws"], s["sws"] = hg.alloc_decode8_workspace(c, Hq), hg.alloc_select_workspace(c)
        cos, sin = attnref.table(400, D // 2)
        s["rotation"] = hg.make_rotation(cos.cuda(), sin.cuda())
        return s

    def step(s):
        lens = s["pool"].tensors[1]
        hg.hg_resize_rows(s["pool"], s["targets"], s["result"], cu_new=s["cu"], slots=s["slots"], positions=s["positions"])
        x = s["x"]
        hg.hg_append_kv8(s["cache"], s["rotation"], x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:], lens, s["q"], cu_new=s["cu"],
                         positions=s["positions"])
        torch.index_select(s["q"], 0, (s["cu"][1:] - 1).clamp_min(0).long(), out=s["last"])
        hg.hg_select_blocks(s["cache"], s["last"], lens, s["blocks"], s["sws"])
        hg.hg_decode_attention8(s["cache"], s["last"], lens, s["out"], s["ws"], blocks=s["blocks"])

    eager, graphed = setup(), setup()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(graphed)  # nothing grows: targets are 0
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    r = random.Random(1)
    g = gen(0)
    lens = [0] * B
    for i in range(60):
        if i % 20 == 19:
            lens = [0 if b == i % B else n - 2 for b, n in enumerate(lens)]
        else:
            lens = [n + r.randint(1, 3) for n in lens]
        x = randn(g, 3 * B, Hq + 2 * H, D).cuda()
        for s in (eager, graphed):
            s["targets"].copy_(torch.tensor(lens, dtype=torch.int32))
            s["x"].copy_(x)
        step(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert int(eager["result"][0]) == 0
        for n in ("result", "cu", "slots", "positions", "q", "blocks", "out"):
            assert torch.equal(raw(eager[n]), raw(graphed[n])), (i, n)
        for a, b in zip(eager["cache"].tensors + eager["pool"].tensors, graphed["cache"].tensors + graphed["pool"].tensors):
            assert torch.equal(raw(a), raw(b)), i
    # the last step's output is the formula's over the cache as it stands
    K, V, ks, vs, bounds, table = (t.cpu() for t in eager["cache"].tensors)
    R = Hq // H
    for b, n in enumerate(lens):
        rows = table[b].tolist()
        for h in range(H):
            limits = [bounds[rows[i * block // ps], h, i * block % ps // block] for i in range((n - 1) // block + 1)]
            want = ref.select(eager["last"][b, h * R:(h + 1) * R].cpu(), limits, 0, budget, 1, 2)
            assert eager["blocks"][b, h].tolist() == want
            t = torch.tensor([t for i in want if i >= 0 for t in range(i * block, min(i * block + block, n))], dtype=torch.long)
            page, off = torch.tensor(rows)[t // ps], t % ps
            o, _, to, _ = attnref.attend(eager["last"][b, h * R:(h + 1) * R].cpu(),
                                         ref.values(K[page, h, off], ks[page, h, off // block]),
                                         ref.values(V[page, h, off], vs[page, h, off // block]), D ** -0.5)
            assert_close(eager["out"][b, h * R:(h + 1) * R], o, to, f"row {b} head {h}")


def test_on_a_stream_of_its_own():
    """Work behind a busy default stream is not waited for by another stream's calls, and ordered on its own."""
    import paper_2609_35800_amd as hg
    c = Cache([100], 2, 128, 16, 16)
    g = gen(1)
    K, V, ks, vs = c.fill([100], g)
    d = c.descriptor()
    q = randn(g, 1, 4, 128).cuda()
    want, out = torch.empty_like(q), torch.empty_like(q)
    ws = hg.alloc_decode8_workspace(d, 4)
    hg.hg_decode_attention8(d, q, i32([100]), want, ws)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    lens = i32([100])
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        hg.hg_decode_attention8(d, q, lens, out, ws)
    s.synchronize()
    assert torch.equal(raw(out), raw(want))
    out.zero_()
    torch.cuda.synchronize()
    hg.hg_decode_attention8(d, q, lens, out, ws, stream=s)
    s.synchronize()
    assert torch.equal(raw(out), raw(want))
