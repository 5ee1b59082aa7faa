"""Performance cases of the operators around a KV cache in 8 bits: rows that
grow and shrink in paged memory, appending to the 8-bit cache, attention of one
new token over it, and the same over blocks that a score selects.

A case names one operator (`op`) and its sizes:
  resize   hg_resize_rows: rows grow to their target lengths (pages taken from the
           free ones, block table, offsets, slots and positions of the new tokens)
           and shrink back, as drafted tokens that are taken back, or prompts that
           come and go;
  append   hg_append_kv8: keys of new tokens rotated, keys and values put into the
           cache's pages as e4m3 codes with one power-of-two scale for each block of
           tokens and head, bounds of each block's keys kept for the selection;
  decode   hg_decode_attention8: one new token per row over its cached tokens;
  sparse   hg_select_blocks and hg_decode_attention8: one new token per row over the
           `budget` blocks that its queries may score highest.
Hq query heads share H key/value heads.  Rows have min_len to max_len tokens,
drawn from `ragged`; page_size 0 is one page of max_len tokens (rounded up to
whole blocks) per row.  The shapes are those of the package's workloads (caches
of 7B to 72B vision-language models), one layer a call.
"""
from __future__ import annotations

import math
import random

import torch

own = False

OPS = ("resize", "append", "decode", "sparse")
F8 = torch.float8_e4m3fn


def _case(name, op, B, Hq, H, D, min_len, max_len, ragged=1, page_size=16, block=16, new="one", sections=False,
          interleaved=False, left_pad=False, lse=False, token_major=False, budget=16, first=1, last=2):
    return dict(name=name, op=op, B=B, Hq=Hq, H=H, D=D, min_len=min_len, max_len=max_len, ragged=ragged, page_size=page_size,
                block=block, new=new, sections=sections, interleaved=interleaved, left_pad=left_pad, lse=lse,
                token_major=token_major, budget=budget, first=first, last=last)


def listed():
    return [
        # one token for each of four rows, taken back: the shortest step of a serving loop
        _case("resize token", "resize", 4, 1, 1, 64, 1361, 1361),
        # five drafted tokens for each of 256 rows, taken back
        _case("resize drafts", "resize", 256, 1, 1, 64, 256, 6656, new="5"),
        # 64 prompts with tiled images admitted, and released
        _case("resize prompts", "resize", 64, 1, 1, 64, 256, 6656, new="all"),
        # the next token of one prompt with one image, 7B model with four KV
        # heads, rotation by three position axes (time, height, width)
        _case("append token", "append", 1, 28, 4, 128, 1361, 1361, sections=True),
        # the next tokens of 64 rows of a 72B model
        _case("append tokens batch", "append", 64, 64, 8, 128, 256, 6656, page_size=64, block=64),
        # four prompts with tiled images just projected, one page a row, 32 KV heads
        _case("append prompts", "append", 4, 32, 32, 128, 700, 3008, page_size=0, block=64, new="all"),
        # one prompt, one new token: the shortest call of a decode loop
        _case("decode token", "decode", 1, 28, 4, 128, 1361, 1361),
        # 64 rows of a 72B model, lengths from a text prompt's to a long one's
        _case("decode batch", "decode", 64, 64, 8, 128, 256, 6656, page_size=64, block=64),
        # a long video: one row of 128K tokens
        _case("decode 128k", "decode", 1, 28, 4, 128, 131072, 131072, lse=True),
        # four left-padded prompts of one page each, no grouping, a quarter of the cache read
        _case("sparse layer cache", "sparse", 4, 32, 32, 128, 700, 3008, page_size=0, block=32, left_pad=True, budget=24),
        # 64 rows of a 72B model, at most 1024 tokens of each attended
        _case("sparse batch", "sparse", 64, 64, 8, 128, 256, 6656, page_size=64, block=64, budget=16),
        # a long video, 4096 of 128K tokens attended
        _case("sparse 128k", "sparse", 1, 28, 4, 128, 131072, 131072, page_size=64, block=64, budget=64, lse=True),
    ]


def draw(rng):
    """A case of the same ranges: one row to large batches, lengths of one
    token to long ones, every head layout, page and block size and option."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(OPS)
    block = rng.choice([16, 16, 32, 64, 64, 128])
    page_size = rng.choice([0, 1, 1, 2, 3, 4]) * block
    H, G = rng.choice([(4, 7), (32, 1), (8, 4), (8, 8), (8, 2), (1, 8), (5, 3), (2, 16), (1, 24)])
    longest = log(1, 131072 if op in ("decode", "sparse") else 30000)
    new = {"resize": ["one", "5", "all", "some"], "append": ["one", "one", "all", "some"]}.get(op, ["one"])
    budget = log(1, 128)
    first = rng.randint(0, min(2, budget))
    c = dict(op=op, B=log(1, 256 if op == "resize" else 64), Hq=H * G, H=H, D=rng.choice([64, 128, 128, 128, 256]),
             min_len=max(1, longest // rng.choice([1, 2, 4, 20])), max_len=longest, ragged=rng.randrange(1 << 20),
             page_size=page_size, block=block, new=rng.choice(new), sections=rng.random() < 0.3,
             interleaved=rng.random() < 0.3, left_pad=rng.random() < 0.3, lse=rng.random() < 0.5,
             token_major=rng.random() < 0.3, budget=budget, first=first, last=rng.randint(0, min(3, budget - first)))
    if op == "resize":
        c.update(Hq=1, H=1, D=64, page_size=rng.choice([1, 16, 16, 64, 100, 256]), block=1)
    # at most the largest listed case of the operator, in operations, bytes and cache
    limits = [(work(x), _cache_elements(x)) for x in listed() if x["op"] == op]
    while (work(c)["flops"] > max(w["flops"] for w, _ in limits) or work(c)["bytes"] > max(w["bytes"] for w, _ in limits)
           or _cache_elements(c) > max(n for _, n in limits)):
        if c["B"] > 1:
            c["B"] //= 2
        else:
            c["max_len"] = max(1, c["max_len"] // 2)
            c["min_len"] = max(1, c["min_len"] // 2)
    # a budget past the blocks of every row makes no other work
    c["budget"] = min(c["budget"], 2 * -(-c["max_len"] // c["block"]))
    c["first"] = min(c["first"], c["budget"])
    c["last"] = min(c["last"], c["budget"] - c["first"])
    return c


def _cache_elements(c):
    return c["B"] * c["H"] * c["max_len"] * c["D"]


def _lens(c):
    r = random.Random(c["ragged"])
    return [r.randint(c["min_len"], c["max_len"]) for _ in range(c["B"])]


def _new(c, lens):
    """New tokens of each row, counted in its length."""
    r = random.Random(c["ragged"] + 1)
    if c["new"] == "all":
        return list(lens)
    if c["new"] == "some":
        return [r.randint(0, n) for n in lens]
    return [min(n, 1 if c["new"] == "one" else int(c["new"])) for n in lens]


def _starts(c, lens):
    """Left-padded rows end together at max_len: row b's tokens are [max_len - len, max_len)."""
    return [c["max_len"] - n for n in lens] if c["left_pad"] else [0] * len(lens)


def _ends(c, lens):
    return [c["max_len"]] * len(lens) if c["left_pad"] else lens


def _page_size(c):
    return c["page_size"] or -(-c["max_len"] // c["block"]) * c["block"]


def _sections(D):
    """Frequencies per position axis: a quarter, three eighths, three eighths."""
    return (D // 8, 3 * D // 16, 3 * D // 16)


def _table(c, ends, spare):
    """Block table (host) of rows of `ends` tokens, and the pages left over."""
    ps = _page_size(c)
    need = [-(-n // ps) for n in ends]
    total = sum(need) + spare
    order = torch.randperm(total, generator=torch.Generator().manual_seed(c["ragged"])).to(torch.int32)
    if c["page_size"] == 0:
        order = order.sort().values
    table = torch.full((len(ends), max(max(need), 1)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, order[at:], total


def _scale_of(amax):
    """The smallest power of two 2^e, e in [-100, 119], with amax <= 448 2^e."""
    m, x = torch.frexp(amax.clamp_min(2.0 ** -99))
    e = x - 9 + (m > 0.875).to(x.dtype)
    return torch.ldexp(torch.ones_like(amax), e.clamp(-100, 119))


def _pages8(c, total, g):
    """Pages of an earlier use: codes, scales and key bounds."""
    H, D, block, ps = c["H"], c["D"], c["block"], _page_size(c)
    n = ps // block
    s = {}
    for name in ("K", "V"):
        x = torch.empty((total, H, n, block, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        if name == "K":
            # keys near one another are alike, and four channels a head are ten times the others
            x += torch.empty((total, H, n, 1, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
            x *= _outliers(H, D, g).view(1, H, 1, 1, D)
            s["bounds"] = torch.stack((x.amin(3), x.amax(3)), 3)
        scale = _scale_of(x.abs().amax((-1, -2)).float())
        s[name.lower() + "_scale"] = scale
        codes = (x / scale.to(torch.bfloat16)[..., None, None]).to(F8).view(torch.uint8).view(total, H, ps, D)
        if c["token_major"]:
            codes = codes.transpose(1, 2).contiguous().transpose(1, 2)
        s[name] = codes
    return s


def _outliers(H, D, g):
    """Scale of the key channels: four per head ten times the others."""
    scale = torch.ones((H, D), device="cuda")
    scale.scatter_(-1, torch.rand((H, D), generator=g, device="cuda").topk(4, dim=-1).indices, 10.0)
    return scale.to(torch.bfloat16)


def _offsets(n):
    cu = [0]
    for x in n:
        cu.append(cu[-1] + x)
    return cu


def _inputs(case, seed):
    """The tensors of a case; `lens` and the like also as host lists."""
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 31)
    B, Hq, H, D = c["B"], c["Hq"], c["H"], c["D"]
    lens = _lens(c)
    s = dict(case=c, lens_h=lens)

    def i32(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    if c["op"] == "resize":
        # which rows and pages are in use differs with the seed
        c = dict(c, ragged=c["ragged"] + 7919 * seed)
        lens = _lens(c)
        new = _new(c, lens)
        now = [a - b for a, b in zip(lens, new)]
        ps = _page_size(c)
        columns = -(-c["max_len"] // ps)
        # pages for rows of the greatest length
        table, free, total = _table(c, now, B * columns - sum(-(-n // ps) for n in now))
        wide = torch.full((B, columns), -1, dtype=torch.int32)
        wide[:, :table.shape[1]] = table[:, :wide.shape[1]]
        s.update(table=wide.cuda(), lens=i32(now), targets=i32(lens), back=i32(now), num_pages=total, n_free=i32([len(free)]))
        s["free"] = torch.full((total,), -1, dtype=torch.int32, device="cuda")
        s["free"][:len(free)] = free.cuda()
        # room for the tokens of a call, as a captured step has it
        room = max(sum(_new(c, [c["max_len"]] * B)), sum(new)) if c["new"] in ("one", "5") else c["max_len"] * B
        s.update(cu=torch.empty(B + 1, dtype=torch.int32, device="cuda"), slots=torch.empty(room, dtype=torch.int64, device="cuda"),
                 positions=torch.empty(room, dtype=torch.int32, device="cuda"), grown=i32([0] * 4), shrunk=i32([0] * 4))
        return s
    if c["op"] == "append":
        new = _new(c, lens)
        cu = _offsets(new)
        N = cu[-1]
        table, _, total = _table(c, lens, 1 if c["page_size"] else 0)
        s.update(_pages8(c, total, g), table=table.cuda(), lens=i32(lens), new_h=new, cu_h=cu,
                 cu_new=None if c["new"] == "one" else i32(cu))
        # the fused projection's output: queries, keys, values of a token side by side
        qkv = torch.empty((N, Hq + 2 * H, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        qkv[:, Hq:Hq + H] *= _outliers(H, D, g)
        s.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + H], v=qkv[:, Hq + H:])
        T = c["max_len"] + 1
        freq = 1e6 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
        angle = torch.arange(T, device="cuda", dtype=torch.float64).view(T, 1) * freq
        s.update(cos=angle.cos().float(), sin=angle.sin().float())
        # image tokens: the axes' positions differ
        s["positions"] = torch.randint(0, T, (3, N), generator=g, device="cuda", dtype=torch.int32) if c["sections"] else None
        s["q_out"] = torch.empty((N, Hq, D), dtype=torch.bfloat16, device="cuda")
        # prompts' attention reads the rotated keys packed
        s["k_out"] = torch.empty((N, H, D), dtype=torch.bfloat16, device="cuda") if c["new"] == "all" else None
        # the blocks that the rows' new tokens lie in
        blocks = [-(-n // c["block"]) - (n - m) // c["block"] if m else 0 for n, m in zip(lens, new)]
        s.update(block_rows=torch.repeat_interleave(torch.arange(B), torch.tensor(blocks)).cuda(),
                 block_cu=torch.tensor(_offsets(blocks), device="cuda"))
        return s
    ends = _ends(c, lens)
    table, _, total = _table(c, ends, 1 if c["page_size"] else 0)
    s.update(_pages8(c, total, g), table=table.cuda(), lens=i32(ends), ends_h=ends, starts_h=_starts(c, lens))
    s["starts"] = i32(s["starts_h"]) if c["left_pad"] else None
    s["q"] = torch.empty((B, Hq, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((B, Hq), dtype=torch.float32, device="cuda") if c["lse"] else None
    if c["op"] == "sparse":
        s["blocks"] = torch.empty((B, H, c["budget"]), dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2609_35800_amd as hg
        s["hg"] = hg
        if case["op"] == "resize":
            s["pool"] = hg.make_page_pool(s["table"], s["lens"], s["free"], s["n_free"], _page_size(case))
        else:
            s["cache"] = hg.make_cache8(s["K"], s["V"], s["k_scale"], s["v_scale"], s["table"], s["bounds"])
        if case["op"] == "append":
            s["rotation"] = hg.make_rotation(s["cos"], s["sin"], interleaved=case["interleaved"],
                                             sections=_sections(case["D"]) if case["sections"] else None)
        if case["op"] in ("decode", "sparse"):
            s["workspace"] = hg.alloc_decode8_workspace(s["cache"], case["Hq"])
        if case["op"] == "sparse":
            s["select_workspace"] = hg.alloc_select_workspace(s["cache"])
    return s


def run(state):
    return _own(state) if own else _plain(state)


def _appended(s):
    out = {"q": s["q_out"], "K": s["K"].view(F8), "V": s["V"].view(F8), "k_scale": s["k_scale"], "v_scale": s["v_scale"],
           "bounds": s["bounds"]}
    return dict(out, k=s["k_out"]) if s["k_out"] is not None else out


def _attended(s):
    return {n: s[n] for n in ("out", "lse", "blocks") if s.get(n) is not None}


def _resized(s):
    return {n: s[n] for n in ("table", "lens", "free", "n_free", "cu", "slots", "positions", "grown", "shrunk")}


def _own(s):
    hg, c = s["hg"], s["case"]
    if c["op"] == "resize":
        hg.hg_resize_rows(s["pool"], s["targets"], s["grown"], cu_new=s["cu"], slots=s["slots"], positions=s["positions"])
        hg.hg_resize_rows(s["pool"], s["back"], s["shrunk"])
        return _resized(s)
    if c["op"] == "append":
        hg.hg_append_kv8(s["cache"], s["rotation"], s["q"], s["k"], s["v"], s["lens"], s["q_out"], cu_new=s["cu_new"],
                         positions=s["positions"], k_out=s["k_out"])
        return _appended(s)
    if c["op"] == "sparse":
        hg.hg_select_blocks(s["cache"], s["q"], s["lens"], s["blocks"], s["select_workspace"], starts=s["starts"],
                            first=c["first"], last=c["last"])
        hg.hg_decode_attention8(s["cache"], s["q"], s["lens"], s["out"], s["workspace"], starts=s["starts"], lse=s["lse"],
                                blocks=s["blocks"])
    else:
        hg.hg_decode_attention8(s["cache"], s["q"], s["lens"], s["out"], s["workspace"], starts=s["starts"], lse=s["lse"])
    return _attended(s)


# ------------------------------------------------------------ the plain form, in 32 bits

def _plain(s):
    op = s["case"]["op"]
    if op == "resize":
        _resize(s, s["targets"], s["grown"], True)
        _resize(s, s["back"], s["shrunk"], False)
        return _resized(s)
    return {"append": _append, "decode": _decode, "sparse": _sparse}[op](s)


def _resize(s, targets, result, mapped):
    """Pages of the rows that shrink go on the free ones, pages of those that
    grow come off them, both by row and column; nothing changes if they do not do."""
    ps, table, free = _page_size(s["case"]), s["table"], s["free"]
    B, columns = table.shape
    total = s["num_pages"]
    lens, want = s["lens"].long(), targets.long()
    have_pages, want_pages = (lens + ps - 1) // ps, (want + ps - 1) // ps
    at = torch.arange(columns, device=table.device)
    freed = (at >= want_pages.view(B, 1)) & (at < have_pages.view(B, 1))
    taken = (at >= have_pages.view(B, 1)) & (at < want_pages.view(B, 1))
    n = s["n_free"].long()
    pushed = n + freed.sum()
    left = pushed - taken.sum()
    new = (want - lens).clamp_min(0)
    count = new.sum()
    outside = ((want < 0) | (want > columns * ps)).any()
    room = s["slots"].numel() if mapped else 1 << 40
    flags = (left < 0).long() + 2 * outside.long() + 4 * (count > room).long() + 8 * (pushed > total).long()
    ok = flags == 0
    # one place past the end takes what is not pushed
    stack = torch.cat((free, free.new_zeros(1)))
    place = torch.where(freed, n + freed.flatten().cumsum(0).view(B, columns) - 1, total)
    stack = stack.scatter(0, place.clamp(0, total).flatten(), table.flatten())[:total]
    source = pushed - taken.flatten().cumsum(0).view(B, columns)
    grown = torch.where(taken, stack[source.clamp(0, max(total - 1, 0))], torch.where(freed, -1, table))
    result.copy_(torch.stack((flags.view(()), (-left).clamp_min(0).view(()), count, torch.where(ok, left, n).view(()))))
    if mapped:
        cu = torch.nn.functional.pad(new.cumsum(0), (1, 0)) * ok
        s["cu"].copy_(cu)
        token = torch.arange(room, device=table.device)
        row = (torch.searchsorted(cu, token, right=True) - 1).clamp_max(B - 1)
        index = lens[row] + token - cu[row]
        inside = token < cu[-1]
        page = grown[row, (index // ps).clamp(0, columns - 1)]
        s["slots"].copy_(torch.where(inside, page * ps + index % ps, -1))
        s["positions"].copy_(torch.where(inside, index, -1))
    table.copy_(torch.where(ok, grown, table))
    free.copy_(torch.where(ok, stack, free))
    s["lens"].copy_(torch.where(ok, want, lens))
    s["n_free"].copy_(torch.where(ok, left, n))


def _angles(s, index):
    """cos, sin [N, 1, D/2] of every token's frequencies."""
    c = s["case"]
    if s["positions"] is None:
        return s["cos"][index].unsqueeze(1), s["sin"][index].unsqueeze(1)
    axis = torch.repeat_interleave(torch.arange(3, device=index.device), torch.tensor(_sections(c["D"]), device=index.device))
    p = s["positions"].long()[axis].t()  # [N, D/2]
    i = torch.arange(c["D"] // 2, device=index.device)
    return s["cos"][p, i].unsqueeze(1), s["sin"][p, i].unsqueeze(1)


def _rotate(x, cos, sin, interleaved):
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _append(s):
    c = s["case"]
    H, D, block, ps = c["H"], c["D"], c["block"], _page_size(c)
    dev = s["lens"].device
    N = s["q"].shape[0]
    token = torch.arange(N, device=dev)
    if s["cu_new"] is None:
        row, first = token, s["lens"].long() - 1
        index = first
    else:
        cu = s["cu_new"].long()
        row = torch.searchsorted(cu, token, right=True) - 1
        first = s["lens"].long() - (cu[1:] - cu[:-1])
        index = first[row] + token - cu[row]
    # keys in 64 bits: a scale steps where a block's largest one passes a border
    cos, sin = _angles(s, index)
    s["q_out"].copy_(_rotate(s["q"].float(), cos, sin, c["interleaved"]))
    k = _rotate(s["k"].double(), cos.double(), sin.double(), c["interleaved"]).to(torch.bfloat16)
    if s["k_out"] is not None:
        s["k_out"].copy_(k)
    # the blocks of the new tokens: row, page and place in it; tokens that they held before
    rows = s["block_rows"]
    nb = rows.shape[0]
    base = first // block
    b_index = base[rows] + torch.arange(nb, device=dev) - s["block_cu"][rows]
    b_page = s["table"][rows, b_index * block // ps].long()
    b_sub = b_index * block % ps // block
    held = (first[rows] - b_index * block).clamp_min(0)
    local = s["block_cu"][row] + index // block - base[row]
    page, off = b_page[local], index % ps
    for_d = local.view(N, 1, 1).expand(N, H, D)
    for x, codes, name in ((k, s["K"], "k_scale"), (s["v"], s["V"], "v_scale")):
        most = torch.zeros((nb, H), device=dev).scatter_reduce(0, local.view(N, 1).expand(N, H), x.abs().amax(-1).float(), "amax")
        old = s[name][b_page, :, b_sub]
        scale = torch.where(held.view(nb, 1) > 0, torch.maximum(old, _scale_of(most)), _scale_of(most))
        # what the rows' first blocks held, on the new scale
        t = torch.arange(block, device=dev)
        place = (b_page.view(nb, 1), slice(None), b_sub.view(nb, 1) * block + t)
        was = codes[place]  # [nb, block, H, D]
        again = (was.view(F8).float() * (old / scale).view(nb, 1, H, 1)).to(F8).view(torch.uint8)
        codes[place] = torch.where((t < held.view(nb, 1)).view(nb, block, 1, 1), again, was)
        codes[page, :, off] = (x.float() / scale[local].unsqueeze(-1)).to(F8).view(torch.uint8)
        s[name][b_page, :, b_sub] = scale
    for i, how in ((0, "amin"), (1, "amax")):
        old = torch.where(held.view(nb, 1, 1) > 0, s["bounds"][b_page, :, b_sub, i], math.inf if i == 0 else -math.inf)
        s["bounds"][b_page, :, b_sub, i] = old.float().scatter_reduce(0, for_d, k.float(), how).to(torch.bfloat16)
    return _appended(s)


def _values(s, name, page, sub_off, head=None):
    """Cached keys or values in fp32: of all heads of the pages, or of tokens (page, place) of a head."""
    codes, scale, block = s[name], s[name.lower() + "_scale"], s["case"]["block"]
    if head is None:
        x = codes[page].view(F8).float()                                    # [B, P, H, ps, D]
        x = x * scale[page].repeat_interleave(block, -1).unsqueeze(-1)
        return x.transpose(1, 2).flatten(2, 3)                              # [B, H, T, D]
    return codes[page, head, sub_off].view(F8).float() * scale[page, head, sub_off // block].unsqueeze(-1)


def _attend(s, K, V, seen):
    """q [B, Hq, D] over K, V [B, H, T, D], tokens `seen` [B, 1 or H, T]."""
    c = s["case"]
    B, Hq, H, D = c["B"], c["Hq"], c["H"], c["D"]
    x = torch.matmul(s["q"].float().view(B, H, Hq // H, D), K.transpose(2, 3)) * D ** -0.5
    x = torch.where(seen.unsqueeze(2), x, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = (x - m).exp()
    t = p.sum(-1, keepdim=True)
    s["out"].copy_((torch.matmul(p, V) / t).view(B, Hq, D))
    if s["lse"] is not None:
        s["lse"].copy_((m + t.log()).view(B, Hq))
    return _attended(s)


def _decode(s):
    page = s["table"].long().clamp_min(0)
    K, V = _values(s, "K", page, None), _values(s, "V", page, None)
    t = torch.arange(K.shape[2], device=K.device)
    seen = t < s["lens"].view(-1, 1)
    if s["starts"] is not None:
        seen &= t >= s["starts"].view(-1, 1)
    return _attend(s, K, V, seen.unsqueeze(1))


def _sparse(s):
    c = s["case"]
    B, Hq, H, D, block, budget, ps = c["B"], c["Hq"], c["H"], c["D"], c["block"], c["budget"], _page_size(c)
    dev = s["q"].device
    lens = s["lens"].long().view(B, 1, 1)
    starts = torch.zeros_like(lens) if s["starts"] is None else s["starts"].long().view(B, 1, 1)
    # what a block's keys can score at most, summed over the group, in 64 bits: the order of the scores decides
    page = s["table"].long().clamp_min(0)
    bounds = s["bounds"][page].permute(0, 2, 1, 3, 4, 5).flatten(2, 3)  # [B, H, NB, 2, D]
    NB = bounds.shape[2]
    q = s["q"].double().view(B, H, Hq // H, D)
    up, down = q.clamp_min(0).sum(2), q.clamp_max(0).sum(2)
    score = (torch.matmul(bounds[..., 0, :].double(), down.unsqueeze(-1)) +
             torch.matmul(bounds[..., 1, :].double(), up.unsqueeze(-1))).squeeze(-1)
    n = torch.arange(NB, device=dev).view(1, 1, NB)
    n0, n1 = starts // block, (lens - 1) // block
    inside = (n >= n0) & (n <= n1)
    score = torch.where((n < n0 + c["first"]) | (n > n1 - c["last"]), math.inf, score)
    score = torch.where(inside, score, -math.inf)
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :budget]
    best = torch.where((best >= n0) & (best <= n1), best, NB)
    best = best.sort(-1).values
    s["blocks"].fill_(-1)
    s["blocks"][..., :best.shape[-1]] = torch.where(best < NB, best, -1)
    # tokens of the chosen blocks
    chosen = s["blocks"].long()
    t = (chosen.unsqueeze(-1) * block + torch.arange(block, device=dev)).flatten(2)  # [B, H, budget * block]
    seen = (t >= starts) & (t < lens) & (chosen >= 0).repeat_interleave(block, -1)
    t = torch.where(seen, t, 0)
    at = page.gather(1, (t // ps).flatten(1)).view_as(t)
    h = torch.arange(H, device=dev).view(1, H, 1)
    return _attend(s, _values(s, "K", at, t % ps, h), _values(s, "V", at, t % ps, h), seen)


# ------------------------------------------------------------ work

def work(case):
    """Bytes: inputs read once, outputs written once.  Operations: the
    rotation's six per pair, two for a code; two products of 2 D per query head
    and key attended, 4 D per block scored."""
    c = case
    lens = _lens(c)
    B, Hq, H, D, block = c["B"], c["Hq"], c["H"], c["D"], c["block"]
    if c["op"] == "resize":
        ps = _page_size(c)
        new = _new(c, lens)
        pages = sum(-(-n // ps) - -(-(n - m) // ps) for n, m in zip(lens, new))
        # lengths and targets twice, lengths back, offsets; pages moved from and to the free ones; slots and positions
        return {"bytes": 28 * B + 20 * pages + 12 * sum(new) + 44, "flops": 0}
    if c["op"] == "append":
        new = _new(c, lens)
        N = sum(new)
        blocks = sum(-(-n // block) - (n - m) // block for n, m in zip(lens, new) if m)
        nbytes = N * D * (4 * Hq + 4 * H + 2 * H + (2 * H if c["new"] == "all" else 0)) + blocks * H * (8 + 4 * D) \
            + 4 * D * min(N, c["max_len"] + 1) + (12 * N if c["sections"] else 0) + 4 * B
        return {"bytes": nbytes, "flops": N * D * (3 * Hq + 7 * H)}
    ends, starts = _ends(c, lens), _starts(c, lens)
    attended, scored = sum(lens), 0
    if c["op"] == "sparse":
        rows = [(-(-e // block) - a // block, n) for a, e, n in zip(starts, ends, lens)]
        attended = sum(min(n, c["budget"] * block) for _, n in rows)
        scored = sum(n for n, _ in rows if n > c["budget"])
    io = B * Hq * (4 * D + (4 if c["lse"] else 0))
    scales = 8 * H * (attended // block)
    nbytes = attended * H * D * 2 + scales + io + (4 * B * H * c["budget"] + 4 * D * H * scored if c["op"] == "sparse" else 0)
    return {"bytes": nbytes, "flops": 4 * attended * Hq * D + 4 * scored * H * D}


# ------------------------------------------------------------ in 64 bits

def exact(case, seed):
    """From the definitions, row by row, in 64 bits; what is stored in 8 bits
    is not rounded to them here."""
    s = _inputs(case, seed)
    return {"resize": _resize_exact, "append": _append_exact, "decode": _attend_exact, "sparse": _attend_exact}[case["op"]](s)


def _resize_exact(s):
    """Page by page on the host."""
    ps = _page_size(s["case"])
    table, free = s["table"].cpu().tolist(), s["free"].cpu().tolist()
    n = int(s["n_free"])
    lens = s["lens"].cpu().tolist()
    out = {}
    for key, targets in (("grown", s["targets"].cpu().tolist()), ("shrunk", s["back"].cpu().tolist())):
        for b, t in enumerate(targets):
            for p in range(-(-t // ps), -(-lens[b] // ps)):
                free[n] = table[b][p]
                table[b][p] = -1
                n += 1
        for b, t in enumerate(targets):
            for p in range(-(-lens[b] // ps), -(-t // ps)):
                n -= 1
                table[b][p] = free[n]
        if key == "grown":
            cu, slots, positions = [0], [], []
            for b, t in enumerate(targets):
                for i in range(lens[b], t):
                    slots.append(table[b][i // ps] * ps + i % ps)
                    positions.append(i)
                cu.append(len(slots))
            fill = [-1] * (s["slots"].numel() - len(slots))
            out.update(cu=cu, slots=slots + fill, positions=positions + fill)
        out[key] = [0, 0, sum(max(0, t - m) for t, m in zip(targets, lens)), n]
        lens = targets
    out.update(table=table, lens=lens, free=free, n_free=[n])
    return {k: torch.tensor(v) for k, v in out.items()}


def _append_exact(s):
    c = s["case"]
    D, H, block, ps = c["D"], c["H"], c["block"], _page_size(c)
    N = s["q"].shape[0]
    index = torch.tensor([t for n, m in zip(s["lens_h"], s["new_h"]) for t in range(n - m, n)], device="cuda").long()
    q, k = s["q"].double().clone(), s["k"].double().clone()
    edges = _sections(D)
    for i in range(D // 2):
        p = index if s["positions"] is None else s["positions"][0 if i < edges[0] else 1 if i < edges[0] + edges[1] else 2].long()
        co, si = s["cos"][p, i].double().view(N, 1), s["sin"][p, i].double().view(N, 1)
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + D // 2)
        for x, src in ((q, s["q"]), (k, s["k"])):
            xa, xb = src[..., a].double(), src[..., b].double()
            x[..., a], x[..., b] = xa * co - xb * si, xb * co + xa * si
    res = {"q": q, "K": s["K"].view(F8).double(), "V": s["V"].view(F8).double(), "k_scale": s["k_scale"].double(),
           "v_scale": s["v_scale"].double(), "bounds": s["bounds"].double()}
    if s["k_out"] is not None:
        res["k"] = k
    table = s["table"].cpu().tolist()
    stored = {"K": k.to(torch.bfloat16).double(), "V": s["v"].double()}
    for b, (lo, n, m) in enumerate(zip(s["cu_h"], s["lens_h"], s["new_h"])):
        at = n - m
        while at < n:  # a block of the row: tokens at .. to
            to = min(n, at // block * block + block)
            page, off = table[b][at // ps], at % ps
            begin, sub = off // block * block, off // block
            for name in ("K", "V"):
                x = stored[name][lo + at - n + m:lo + to - n + m].transpose(0, 1)  # [H, tokens, D]
                most = x.abs().amax((1, 2))
                # log2 of most / 448 is whole only at a border, where it is exact
                scale = 2.0 ** torch.log2(most.clamp_min(2.0 ** -90) / 448).ceil()
                scales = res[name.lower() + "_scale"]
                if off > begin:
                    old = scales[page, :, sub].clone()
                    scale = torch.maximum(scale, old)
                    res[name][page, :, begin:off] *= (old / scale).view(H, 1, 1)
                scales[page, :, sub] = scale
                fine = (k if name == "K" else stored["V"])[lo + at - n + m:lo + to - n + m].transpose(0, 1)
                res[name][page, :, off:off + to - at] = fine / scale.view(H, 1, 1)
                if name == "K":
                    lower, upper = fine.amin(1), fine.amax(1)
                    if off > begin:
                        lower = torch.minimum(lower, res["bounds"][page, :, sub, 0])
                        upper = torch.maximum(upper, res["bounds"][page, :, sub, 1])
                    res["bounds"][page, :, sub, 0], res["bounds"][page, :, sub, 1] = lower, upper
            at = to
    return res


def _attend_exact(s):
    c = s["case"]
    G, D, block, ps = c["Hq"] // c["H"], c["D"], c["block"], _page_size(c)
    outs, lses, lists = [], [], []
    for b in range(c["B"]):
        lo, hi = s["starts_h"][b], s["ends_h"][b]
        table = s["table"][b].long()
        for h in range(c["H"]):
            q = s["q"][b, h * G:(h + 1) * G].double()
            t = torch.arange(lo, hi, device="cuda")
            if c["op"] == "sparse":
                ids = list(range(lo // block, (hi - 1) // block + 1))
                if len(ids) > c["budget"]:
                    n = torch.tensor(ids, device="cuda")
                    limits = s["bounds"][table[n * block // ps], h, n * block % ps // block].double()  # [n, 2, D]
                    score = torch.maximum(q.unsqueeze(1) * limits[:, 0], q.unsqueeze(1) * limits[:, 1]).sum((0, 2))
                    score[:c["first"]] = math.inf
                    score[len(ids) - c["last"]:] = math.inf
                    rank = score.sort(descending=True, stable=True).indices[:c["budget"]]
                    n = n[rank].sort().values
                    ids = n.tolist()
                    t = (n.view(-1, 1) * block + torch.arange(block, device="cuda")).flatten()
                    t = t[(t >= lo) & (t < hi)]
                lists.append(ids + [-1] * (c["budget"] - len(ids)))
            page, off = table[t // ps], t % ps
            K, V = (s[n][page, h, off].view(F8).double() * s[n.lower() + "_scale"][page, h, off // block].double().unsqueeze(-1)
                    for n in ("K", "V"))
            x = q @ K.t() / math.sqrt(D)
            outs.append(torch.softmax(x, -1) @ V)
            lses.append(torch.logsumexp(x, -1))
    res = {"out": torch.stack(outs).view(c["B"], c["Hq"], D)}
    if c["lse"]:
        res["lse"] = torch.stack(lses).view(c["B"], c["Hq"])
    if c["op"] == "sparse":
        res["blocks"] = torch.tensor(lists, dtype=torch.int32).view(c["B"], c["H"], c["budget"])
    return res
