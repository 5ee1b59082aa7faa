"""Performance cases of the attention operators that fill and read the KV
cache: appending rotated keys and values to a paged cache, attention over
packed prompts, and attention of one new token over the paged cache.

A case names one operator (`op`) and its sizes:
  append   hg_append_kv: keys and values of new tokens rotated and put into the
           cache's pages, the queries of the same tokens rotated beside them;
  prefill  hg_prefill_attention: whole prompts of different lengths, packed;
  decode   hg_decode_attention: one new token per row over its cached tokens.
Hq query heads share H key/value heads.  Rows have min_len to max_len tokens,
drawn from `ragged`; page_size 0 is the quantizer's own layer cache, one page
of T = max_len tokens per row.  The shapes are those of the package's workloads
(caches of 7B to 72B vision-language models), one layer a call.
"""
from __future__ import annotations

import math
import random

import torch

own = False

OPS = ("append", "decode", "prefill")


def _case(name, op, B, Hq, H, D, min_len, max_len, ragged=1, page_size=16, new="one", sections=False,
          interleaved=False, left_pad=False, causal=True, lse=False, token_major=False):
    return dict(name=name, op=op, B=B, Hq=Hq, H=H, D=D, min_len=min_len, max_len=max_len, ragged=ragged,
                page_size=page_size, new=new, sections=sections, interleaved=interleaved, left_pad=left_pad,
                causal=causal, lse=lse, token_major=token_major)


def listed():
    return [
        # the next token of one prompt with one image, 7B model with four KV
        # heads, rotation by three position axes (time, height, width)
        _case("append token", "append", 1, 28, 4, 128, 1361, 1361, sections=True),
        # the next tokens of 64 rows of a 72B model
        _case("append tokens batch", "append", 64, 64, 8, 128, 256, 6656),
        # four prompts with tiled images just projected, into the layer cache
        # that the quantizer takes, 32 KV heads
        _case("append prompts", "append", 4, 32, 32, 128, 700, 3008, page_size=0, new="all"),
        # one prompt, one new token: the shortest call of a decode loop
        _case("decode token", "decode", 1, 28, 4, 128, 1361, 1361),
        # four prompts in the quantizer's layer cache, left-padded to one length, no grouping
        _case("decode layer cache", "decode", 4, 32, 32, 128, 700, 3008, page_size=0, left_pad=True),
        # short prompts at head_dim 256, two query heads a KV head
        _case("decode short 256", "decode", 32, 16, 8, 256, 32, 320, page_size=64, token_major=True),
        # 64 rows of a 72B model, lengths from a text prompt's to a long one's
        _case("decode batch", "decode", 64, 64, 8, 128, 256, 6656),
        # a long video: one row of 128K tokens
        _case("decode 128k", "decode", 1, 28, 4, 128, 131072, 131072),
        # one prompt with one image
        _case("prefill prompt", "prefill", 1, 28, 4, 128, 1360, 1360),
        # 32 short prompts at head_dim 256
        _case("prefill short 256", "prefill", 32, 16, 8, 256, 32, 320),
        # eight prompts with tiled images
        _case("prefill packed", "prefill", 8, 32, 8, 128, 900, 3456, lse=True),
        # one long prompt: a video of about 30000 tokens
        _case("prefill long", "prefill", 1, 28, 4, 128, 30001, 30001),
    ]


def draw(rng):
    """A case of the same ranges: one row to large batches, lengths of one
    token to long ones, every head layout, page size and option."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(OPS)
    D = rng.choice([64, 128, 128, 128, 256])
    H, G = rng.choice([(4, 7), (32, 1), (8, 4), (8, 8), (8, 2), (1, 8), (5, 3), (2, 16), (1, 24)])
    B = log(1, 64)
    longest = log(1, 131072 if op == "decode" else 30000)
    new = rng.choice(["one", "all"]) if op == "append" else "one"
    c = dict(op=op, B=B, Hq=H * G, H=H, D=D, min_len=max(1, longest // rng.choice([1, 2, 4, 20])), max_len=longest,
             ragged=rng.randrange(1 << 20), page_size=rng.choice([0, 16, 16, 64, 1, 100, 256]), new=new,
             sections=rng.random() < 0.3, interleaved=rng.random() < 0.3, left_pad=rng.random() < 0.3,
             causal=rng.random() < 0.8, lse=rng.random() < 0.5, token_major=rng.random() < 0.3)
    # at most the largest listed case of the operator, in operations, bytes and cache
    limits = [(work(x), _cache_elements(x)) for x in listed() if x["op"] == op]
    while (work(c)["flops"] > max(w["flops"] for w, _ in limits) or work(c)["bytes"] > max(w["bytes"] for w, _ in limits)
           or (op != "prefill" and _cache_elements(c) > max(n for _, n in limits))):
        if c["B"] > 1:
            c["B"] //= 2
        else:
            c["max_len"] = max(1, c["max_len"] // 2)
            c["min_len"] = max(1, c["min_len"] // 2)
    return c


def _cache_elements(c):
    return c["B"] * c["H"] * c["max_len"] * c["D"]


def _lens(c):
    r = random.Random(c["ragged"])
    return [r.randint(c["min_len"], c["max_len"]) for _ in range(c["B"])]


def _sections(D):
    """Frequencies per position axis: a quarter, three eighths, three eighths."""
    return (D // 8, 3 * D // 16, 3 * D // 16)


def _starts(c, lens):
    """Left-padded rows end together at T: row b's tokens are [T - len, T)."""
    return [c["max_len"] - n for n in lens] if c["left_pad"] else [0] * len(lens)


def _ends(c, lens):
    return [c["max_len"]] * len(lens) if c["left_pad"] else lens


def _pages(c, ends, g):
    """K, V pages [pages, H, page_size, D] of an earlier use, and the table of the rows' pages."""
    B, H, D = c["B"], c["H"], c["D"]
    ps = c["page_size"] or c["max_len"]
    need = [-(-n // ps) for n in ends]
    total = sum(need) if c["page_size"] == 0 else sum(need) + sum(need) // 16 + 1
    order = torch.arange(total) if c["page_size"] == 0 else torch.randperm(total, generator=torch.Generator().manual_seed(c["ragged"]))
    table = torch.full((B, max(need)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n].to(torch.int32)
        at += n
    shape = (total, ps, H, D) if c["token_major"] else (total, H, ps, D)
    K = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    V = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    if c["token_major"]:
        K, V = K.transpose(1, 2), V.transpose(1, 2)
    K.mul_(_outliers(H, D, g).view(1, H, 1, D))
    return K, V, table.cuda()


def _outliers(H, D, g):
    """Scale of the key channels: four per head ten times the others."""
    scale = torch.ones((H, D), device="cuda")
    scale.scatter_(-1, torch.rand((H, D), generator=g, device="cuda").topk(4, dim=-1).indices, 10.0)
    return scale.to(torch.bfloat16)


def _inputs(case, seed):
    """The tensors of a case; `lens` and the like also as host lists."""
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 29)
    B, Hq, H, D = c["B"], c["Hq"], c["H"], c["D"]
    lens = _lens(c)
    s = dict(case=c, lens_h=lens)

    def i32(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    if c["op"] == "append":
        s["lens"] = i32(lens)
        new = lens if c["new"] == "all" else [1] * B
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        N = cu[-1]
        s.update(cu_h=cu, cu_new=i32(cu) if c["new"] == "all" else None)
        s["K"], s["V"], s["table"] = _pages(c, lens, g)
        # the fused projection's output: queries, keys, values of a token side by side
        qkv = torch.empty((N, Hq + 2 * H, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        qkv[:, Hq:Hq + H] *= _outliers(H, D, g)
        s.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + H], v=qkv[:, Hq + H:])
        T = c["max_len"] + 1
        freq = 1e6 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
        angle = torch.arange(T, device="cuda", dtype=torch.float64).view(T, 1) * freq
        s.update(cos=angle.cos().float(), sin=angle.sin().float())
        if c["sections"]:  # image tokens: the axes' positions differ
            s["positions"] = torch.randint(0, T, (3, N), generator=g, device="cuda", dtype=torch.int32)
        else:
            s["positions"] = None
        s["q_out"] = torch.empty((N, Hq, D), dtype=torch.bfloat16, device="cuda")
        # prompts' attention reads the rotated keys packed
        s["k_out"] = torch.empty((N, H, D), dtype=torch.bfloat16, device="cuda") if c["new"] == "all" else None
    elif c["op"] == "decode":
        ends = _ends(c, lens)
        s.update(ends_h=ends, starts_h=_starts(c, lens), lens=i32(ends))
        s["starts"] = i32(s["starts_h"]) if c["left_pad"] else None
        s["K"], s["V"], s["table"] = _pages(c, ends, g)
        s["q"] = torch.empty((B, Hq, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((B, Hq), dtype=torch.float32, device="cuda") if c["lse"] else None
    else:
        cu = [0]
        for n in lens:
            cu.append(cu[-1] + n)
        N = cu[-1]
        s.update(cu_h=cu, cu=i32(cu))
        s["q"] = torch.empty((N, Hq, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        s["k"] = torch.empty((N, H, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        s["k"].mul_(_outliers(H, D, g))
        # values as the fused projection left them
        s["v"] = torch.empty((N, Hq + 2 * H, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)[:, Hq + H:]
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((N, Hq), dtype=torch.float32, device="cuda") if c["lse"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2609_35800_amd as hg
        s["hg"] = hg
        if case["op"] != "prefill":
            s["cache"] = hg.make_paged_cache(s["K"], s["V"], s["table"])
        if case["op"] == "append":
            s["rotation"] = hg.make_rotation(s["cos"], s["sin"], interleaved=case["interleaved"],
                                             sections=_sections(case["D"]) if case["sections"] else None)
        if case["op"] == "decode":
            s["workspace"] = hg.alloc_decode_workspace(s["cache"], case["Hq"])
    return s


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    hg, c = s["hg"], s["case"]
    if c["op"] == "append":
        hg.hg_append_kv(s["cache"], s["rotation"], s["q"], s["k"], s["v"], s["lens"], s["q_out"], cu_new=s["cu_new"],
                        positions=s["positions"], k_out=s["k_out"])
        return {"q": s["q_out"], "K": s["K"], "V": s["V"], "k": s["k_out"]} if s["k_out"] is not None else {
            "q": s["q_out"], "K": s["K"], "V": s["V"]}
    if c["op"] == "decode":
        hg.hg_decode_attention(s["cache"], s["q"], s["lens"], s["out"], s["workspace"], starts=s["starts"], lse=s["lse"])
    else:
        hg.hg_prefill_attention(s["q"], s["k"], s["v"], s["cu"], s["out"], causal=c["causal"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]} if c["lse"] else {"out": s["out"]}


# ------------------------------------------------------------ the plain form, in 32 bits

def _token_index(s):
    """Cache row and index of every new token."""
    c = s["case"]
    dev = s["lens"].device
    if s["cu_new"] is None:
        row = torch.arange(c["B"], device=dev)
        return row, s["lens"].long() - 1
    cu = s["cu_new"].long()
    token = torch.arange(s["q"].shape[0], device=dev)
    row = torch.searchsorted(cu, token, right=True) - 1
    return row, s["lens"].long()[row] - (cu[row + 1] - token)


def _angles(s, index):
    """cos, sin [N, 1, D/2] of every token's frequencies."""
    c = s["case"]
    half = c["D"] // 2
    if s["positions"] is None:
        return s["cos"][index].unsqueeze(1), s["sin"][index].unsqueeze(1)
    axis = torch.repeat_interleave(torch.arange(3, device=index.device), torch.tensor(_sections(c["D"]), device=index.device))
    p = s["positions"].long()[axis].t()  # [N, D/2]
    i = torch.arange(half, device=index.device)
    return s["cos"][p, i].unsqueeze(1), s["sin"][p, i].unsqueeze(1)


def _rotate(x, cos, sin, interleaved):
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _plain(s):
    c = s["case"]
    if c["op"] == "append":
        row, index = _token_index(s)
        cos, sin = _angles(s, index)
        ps = s["K"].shape[2]
        page = s["table"].long()[row, index // ps]
        q = _rotate(s["q"].float(), cos, sin, c["interleaved"]).to(torch.bfloat16)
        k = _rotate(s["k"].float(), cos, sin, c["interleaved"]).to(torch.bfloat16)
        s["K"][page, :, index % ps] = k
        s["V"][page, :, index % ps] = s["v"]
        return {"q": q, "K": s["K"], "V": s["V"], "k": k} if s["k_out"] is not None else {"q": q, "K": s["K"], "V": s["V"]}
    if c["op"] == "decode":
        return _decode(s, torch.float32)
    return _prefill(s, torch.float32)


def _finish(s, out, lse, dtype):
    if dtype == torch.float32:
        out = out.to(torch.bfloat16)
    return {"out": out, "lse": lse} if s["case"]["lse"] else {"out": out}


def _decode(s, dtype):
    c = s["case"]
    B, Hq, H, D = c["B"], c["Hq"], c["H"], c["D"]
    out = torch.empty((B, Hq, D), dtype=dtype, device="cuda")
    lse = torch.empty((B, Hq), dtype=dtype, device="cuda")
    ps = s["K"].shape[2]
    for b in range(B):
        lo, hi = s["starts_h"][b], s["ends_h"][b]
        pages = s["table"][b, :-(-hi // ps)].long()
        K = s["K"][pages].transpose(0, 1).reshape(H, -1, D)[:, lo:hi].to(dtype)
        V = s["V"][pages].transpose(0, 1).reshape(H, -1, D)[:, lo:hi].to(dtype)
        q = s["q"][b].to(dtype).view(H, Hq // H, D)
        x = torch.matmul(q, K.transpose(1, 2)) * D ** -0.5
        m = x.amax(-1, keepdim=True)
        p = (x - m).exp()
        t = p.sum(-1, keepdim=True)
        out[b] = (torch.matmul(p, V) / t).view(Hq, D)
        lse[b] = (m + t.log()).view(Hq)
    return _finish(s, out, lse, dtype)


def _prefill(s, dtype, scores=1 << 29):
    c = s["case"]
    Hq, H, D = c["Hq"], c["H"], c["D"]
    G = Hq // H
    N = s["q"].shape[0]
    out = torch.empty((N, Hq, D), dtype=dtype, device="cuda")
    lse = torch.empty((N, Hq), dtype=dtype, device="cuda")
    for lo, hi in zip(s["cu_h"], s["cu_h"][1:]):
        n = hi - lo
        K = s["k"][lo:hi].to(dtype).permute(1, 2, 0).contiguous()  # [H, D, n]
        V = s["v"][lo:hi].to(dtype).transpose(0, 1).contiguous()
        step = max(1, min(n, scores // (Hq * n)))  # queries at a time
        for i in range(0, n, step):
            j = min(n, i + step)
            q = s["q"][lo + i:lo + j].to(dtype).view(j - i, H, G, D).permute(1, 2, 0, 3).reshape(H, G * (j - i), D)
            x = torch.matmul(q, K).view(H, G, j - i, n) * D ** -0.5
            if c["causal"]:
                t = torch.arange(n, device="cuda")
                x.masked_fill_(t.view(1, n) > t[i:j].view(j - i, 1), -math.inf)
            m = x.amax(-1, keepdim=True)
            p = x.sub_(m).exp_()
            t = p.sum(-1, keepdim=True)
            o = torch.matmul(p.view(H, G * (j - i), n), V).view(H, G, j - i, D) / t
            out[lo + i:lo + j] = o.permute(2, 0, 1, 3).reshape(j - i, Hq, D)
            lse[lo + i:lo + j] = (m + t.log()).view(Hq, j - i).t()
    return _finish(s, out, lse, dtype)


# ------------------------------------------------------------ work

def work(case):
    """Bytes: inputs read once, outputs written once.  Operations: the
    rotation's six per pair; two products of 2 D per query head and key seen."""
    c = case
    lens = _lens(c)
    Hq, H, D = c["Hq"], c["H"], c["D"]
    if c["op"] == "append":
        N = sum(lens) if c["new"] == "all" else c["B"]
        rows = Hq + 2 * H
        nbytes = N * D * 2 * (2 * rows + (H if c["new"] == "all" else 0)) + 4 * D * min(N, c["max_len"] + 1) \
            + (12 * N if c["sections"] else 0) + 4 * c["B"]
        return {"bytes": nbytes, "flops": N * (Hq + H) * D * 3}
    if c["op"] == "decode":
        nbytes = sum(lens) * H * D * 4 + c["B"] * Hq * (4 * D + (4 if c["lse"] else 0))
        return {"bytes": nbytes, "flops": 4 * sum(lens) * Hq * D}
    N = sum(lens)
    nbytes = N * D * 4 * (Hq + H) + (4 * N * Hq if c["lse"] else 0)
    seen = sum(n * (n + 1) // 2 if c["causal"] else n * n for n in lens)
    return {"bytes": nbytes, "flops": 4 * seen * Hq * D}


# ------------------------------------------------------------ in 64 bits

def exact(case, seed):
    """From the definitions, token by token, pair by pair (append) and row by
    row (attention), in 64 bits."""
    c = case
    s = _inputs(case, seed)
    if c["op"] == "append":
        return _append_exact(s)
    G, D = c["Hq"] // c["H"], c["D"]
    outs, lses = [], []
    if c["op"] == "decode":
        ps = s["K"].shape[2]
        for b in range(c["B"]):
            at = torch.arange(s["starts_h"][b], s["ends_h"][b], device="cuda")
            page, off = s["table"][b].long()[at // ps], at % ps
            o, l = [], []
            for h in range(c["H"]):
                K, V = s["K"][page, h, off].double(), s["V"][page, h, off].double()
                x = s["q"][b, h * G:(h + 1) * G].double() @ K.t() / math.sqrt(D)
                o.append(torch.softmax(x, -1) @ V)
                l.append(torch.logsumexp(x, -1))
            outs.append(torch.cat(o).unsqueeze(0))
            lses.append(torch.cat(l).unsqueeze(0))
    else:
        for lo, hi in zip(s["cu_h"], s["cu_h"][1:]):
            n = hi - lo
            o = torch.empty((n, c["Hq"], D), dtype=torch.float64, device="cuda")
            l = torch.empty((n, c["Hq"]), dtype=torch.float64, device="cuda")
            step = max(1, (1 << 28) // n)
            for hq in range(c["Hq"]):
                K, V = s["k"][lo:hi, hq // G].double(), s["v"][lo:hi, hq // G].double()
                for i in range(0, n, step):
                    j = min(n, i + step)
                    seen = j if c["causal"] else n
                    x = s["q"][lo + i:lo + j, hq].double() @ K[:seen].t() / math.sqrt(D)
                    if c["causal"]:
                        x += torch.full((j - i, seen), -math.inf, dtype=torch.float64, device="cuda").triu_(i + 1)
                    o[i:j, hq] = torch.softmax(x, -1) @ V[:seen]
                    l[i:j, hq] = torch.logsumexp(x, -1)
            outs.append(o)
            lses.append(l)
    res = {"out": torch.cat(outs)}
    if c["lse"]:
        res["lse"] = torch.cat(lses)
    return res


def _append_exact(s):
    c = s["case"]
    D, ps = c["D"], s["K"].shape[2]
    N = s["q"].shape[0]
    K, V = s["K"].double(), s["V"].double()
    # cache place of every token, from the host's lists
    place = []
    table = s["table"].cpu().tolist()
    for b, (lo, hi) in enumerate(zip(s["cu_h"], s["cu_h"][1:])):
        for t in range(s["lens_h"][b] - (hi - lo), s["lens_h"][b]):
            place.append((table[b][t // ps], t % ps, t))
    page, off, index = torch.tensor(place, device="cuda").t()
    q, k = s["q"].double().clone(), s["k"].double().clone()
    edges = _sections(D)
    for i in range(D // 2):
        if s["positions"] is None:
            p = index
        else:
            axis = 0 if i < edges[0] else 1 if i < edges[0] + edges[1] else 2
            p = s["positions"][axis].long()
        co, si = s["cos"][p, i].double().view(N, 1), s["sin"][p, i].double().view(N, 1)
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + D // 2)
        for x, src in ((q, s["q"]), (k, s["k"])):
            xa, xb = src[..., a].double(), src[..., b].double()
            x[..., a], x[..., b] = xa * co - xb * si, xb * co + xa * si
    K[page, :, off] = k
    V[page, :, off] = s["v"].double()
    res = {"q": q, "K": K, "V": V}
    if s["k_out"] is not None:
        res["k"] = k
    return res
