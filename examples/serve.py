"""A small decoder with random weights, served through the package: prompts
with an image each are prefilled, their image KV quantized in place, and tokens
decoded from the cache.

    python examples/serve.py [--layers 4] [--rows 4] [--new-tokens 16] [--base kivi] [--bits 2]
    python examples/serve.py --cache8 [--budget 8]

What runs where:
  * prefill, per layer: the fused projection of all prompts' tokens, packed;
    hg_append_kv rotates queries and keys and stores keys and values in the
    layer's cache; hg_prefill_attention attends within each prompt;
  * hg_fake_quantize takes the image span of the whole cache to low-bit levels
    in place (protected heads and text stay), as the method does after prefill;
  * decode, per layer: hg_append_kv adds the new token of every row,
    hg_decode_attention reads the row's cache.  A step is captured once as a HIP
    graph and replayed.
The cache is the quantizer's, [L][B][H][T][D]; a layer of it is the paged cache
of one page of T tokens per row.

With --cache8 the cache is paged and in 8 bits (Decoder8): hg_resize_rows takes the
pages of the prompts and of every new token on the GPU, hg_append_kv8 fills them,
hg_decode_attention8 reads them, with --budget only the blocks of 16 tokens that
hg_select_blocks picks for each row and KV head.  A step is captured here too: the
lengths, tables and free pages that it changes are all GPU memory.  A step that the
pool has no pages for changes nothing: its append takes the new tokens' offsets from
hg_resize_rows, and there are none then; check() raises after the steps.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_35800_amd as hg  # noqa: E402

BF = torch.bfloat16


class Decoder:
    """Embedding, L layers of attention and residual, output projection; BF16."""

    def __init__(self, layers, rows, prompt_lens, img_start, img_len, new_tokens, Hq=8, H=2, D=128, vocab=512, base="kivi",
                 bits=2, seed=0):
        self._model(layers, rows, max(prompt_lens) + new_tokens, Hq, H, D, vocab, seed)
        self.K = torch.zeros((layers, rows, H, self.T, D), dtype=BF, device="cuda")
        self.V = torch.zeros_like(self.K)
        table = torch.arange(rows, dtype=torch.int32, device="cuda").view(rows, 1)
        self.caches = [hg.make_paged_cache(self.K[l], self.V[l], table) for l in range(layers)]
        self.workspace = hg.alloc_decode_workspace(self.caches[0], Hq)
        # the quantizer's side: a span shared by the rows, one head in eight protected
        self.cfg = hg.make_config(L=layers, B=rows, H=H, T=self.T, D=D, img_start=img_start, img_len=img_len, bits=bits,
                                  base=base, keys_only=0)
        self.mask = torch.zeros(layers * H, dtype=torch.uint8).numpy()
        self.mask[::8] = 1
        self.quantize_workspace = hg.alloc_fake_workspace(self.cfg, self.mask)
        # decode state
        self.lens = torch.tensor(prompt_lens, dtype=torch.int32, device="cuda")

    def _model(self, layers, rows, T, Hq, H, D, vocab, seed):
        """Weights, the rotation of up to T positions, a step's tokens and queries."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.L, self.B, self.Hq, self.H, self.D, self.T = layers, rows, Hq, H, D, T
        width = Hq * D

        def weight(*shape):
            return (torch.randn(shape, generator=g, device="cuda") * shape[0] ** -0.5).to(BF)

        self.embedding = (torch.randn((vocab, width), generator=g, device="cuda")).to(BF)
        self.qkv = [weight(width, (Hq + 2 * H) * D) for _ in range(layers)]
        self.out = [weight(width, width) for _ in range(layers)]
        self.head = weight(width, vocab)
        angle = torch.arange(T, device="cuda", dtype=torch.float64).view(-1, 1) * 1e4 ** (
            -torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
        self.rotation = hg.make_rotation(angle.cos().float(), angle.sin().float())
        self.token = torch.zeros(rows, dtype=torch.int64, device="cuda")
        self.q = torch.empty((rows, Hq, D), dtype=BF, device="cuda")
        self.o = torch.empty_like(self.q)

    def _split(self, x):
        n = x.shape[0]
        x = x.view(n, self.Hq + 2 * self.H, self.D)
        return x[:, :self.Hq], x[:, self.Hq:self.Hq + self.H], x[:, self.Hq + self.H:]

    def _logits(self, h):
        return torch.nn.functional.rms_norm(h, h.shape[-1:]) @ self.head

    def prefill(self, tokens, cu):
        """Packed prompt tokens and their offsets; returns the last tokens' logits."""
        h = self.embedding[tokens]
        n = h.shape[0]
        q_rot = torch.empty((n, self.Hq, self.D), dtype=BF, device="cuda")
        k_rot = torch.empty((n, self.H, self.D), dtype=BF, device="cuda")
        o = torch.empty_like(q_rot)
        for l in range(self.L):
            q, k, v = self._split(torch.nn.functional.rms_norm(h, h.shape[-1:]) @ self.qkv[l])
            self._append(l, q, k, v, q_rot, cu_new=cu, k_out=k_rot)
            hg.hg_prefill_attention(q_rot, k_rot, v, cu, o)
            h = h + o.view(n, -1) @ self.out[l]
        logits = self._logits(h[cu[1:].long() - 1])
        self.token.copy_(logits.argmax(-1))
        return logits

    def _grow(self):
        self.lens += 1

    def _append(self, l, q, k, v, q_out, **kw):
        hg.hg_append_kv(self.caches[l], self.rotation, q, k, v, self.lens, q_out, **kw)

    def _attend(self, l):
        hg.hg_decode_attention(self.caches[l], self.q, self.lens, self.o, self.workspace)

    def quantize_images(self):
        hg.hg_fake_quantize(self.cfg, self.K, self.V, self.mask, self.K, self.V, self.quantize_workspace)

    def step(self):
        """One new token per row; returns the logits."""
        self._grow()
        h = self.embedding[self.token]
        for l in range(self.L):
            q, k, v = self._split(torch.nn.functional.rms_norm(h, h.shape[-1:]) @ self.qkv[l])
            self._append(l, q, k, v, self.q)
            self._attend(l)
            h = h + self.o.view(self.B, -1) @ self.out[l]
        logits = self._logits(h)
        self.token.copy_(logits.argmax(-1))
        return logits


class Decoder8(Decoder):
    """The same over a paged cache in 8 bits, whose rows take their pages from one
    pool for all layers; budget: blocks that a row and KV head attend (None: all)."""

    def __init__(self, layers, rows, prompt_lens, new_tokens, Hq=8, H=2, D=128, vocab=512, seed=0, page_size=32, block_size=16,
                 budget=None):
        self._model(layers, rows, max(prompt_lens) + new_tokens, Hq, H, D, vocab, seed)
        most = -(-self.T // page_size)
        pages = sum(-(-(n + new_tokens) // page_size) for n in prompt_lens)
        self.pool = hg.alloc_page_pool(rows, most, pages, page_size)
        self.table, self.lens, self.free_pages, self.n_free = self.pool.tensors
        self.caches = [hg.alloc_cache8(pages, H, page_size, D, self.table, block_size) for _ in range(layers)]
        self.workspace = hg.alloc_decode8_workspace(self.caches[0], Hq)
        self.budget = budget
        if budget is not None:
            self.blocks = torch.empty((rows, H, budget), dtype=torch.int32, device="cuda")
            self.select_workspace = hg.alloc_select_workspace(self.caches[0])
        self.targets = torch.tensor(prompt_lens, dtype=torch.int32, device="cuda")
        self.result = torch.zeros(4, dtype=torch.int32, device="cuda")
        self.refused = torch.zeros(1, dtype=torch.int32, device="cuda")  # reasons of all calls so far
        self.cu_new = torch.zeros(rows + 1, dtype=torch.int32, device="cuda")

    def _resize(self):
        hg.hg_resize_rows(self.pool, self.targets, self.result, cu_new=self.cu_new)
        self.refused |= self.result[:1]

    def check(self):
        """Raises if the pool refused a call (waits for the GPU)."""
        reasons = int(self.refused)
        if reasons:
            raise RuntimeError(f"rows were not resized: reasons {reasons}, {int(self.result[1])} pages missing in the last call")

    def prefill(self, tokens, cu):
        self._resize()
        self.check()
        return super().prefill(tokens, cu)

    def _grow(self):
        self.targets += 1
        self._resize()

    def _append(self, l, q, k, v, q_out, cu_new=None, **kw):
        # the offsets of a refused resize are all 0: no token is new, and the cache stays as it is
        hg.hg_append_kv8(self.caches[l], self.rotation, q, k, v, self.lens, q_out, cu_new=self.cu_new, **kw)

    def _attend(self, l):
        blocks = None
        if self.budget is not None:
            blocks = self.blocks
            hg.hg_select_blocks(self.caches[l], self.q, self.lens, blocks, self.select_workspace)
        hg.hg_decode_attention8(self.caches[l], self.q, self.lens, self.o, self.workspace, blocks=blocks)

    def release(self):
        """Gives all rows' pages back."""
        self.targets.zero_()
        self._resize()

    def quantize_images(self):
        pass  # the cache is in 8 bits as it is


def prompts(rows, img_start, img_len, seed=0, vocab=512):
    """Row lengths (text, image, text of its own length), packed tokens, offsets."""
    g = torch.Generator().manual_seed(seed + 1)
    lens = [img_start + img_len + int(torch.randint(1, 40, (1,), generator=g)) for _ in range(rows)]
    tokens = torch.randint(0, vocab, (sum(lens),), generator=g).cuda()
    cu = torch.tensor([sum(lens[:i]) for i in range(rows + 1)], dtype=torch.int32, device="cuda")
    return lens, tokens, cu


def serve(layers=4, rows=4, new_tokens=16, img_start=16, img_len=256, base="kivi", bits=2, graph=True, seed=0,
          cache8=False, budget=None):
    """Serves random prompts; returns the decoder and the new tokens [rows, new_tokens]."""
    lens, tokens, cu = prompts(rows, img_start, img_len, seed)
    if cache8:
        model = Decoder8(layers, rows, lens, new_tokens, seed=seed, budget=budget)
    else:
        model = Decoder(layers, rows, lens, img_start, img_len, new_tokens, base=base, bits=bits, seed=seed)
    model.prefill(tokens, cu)
    model.quantize_images()
    new = [model.token.clone()]
    run = model.step
    if graph and new_tokens > 2:
        model.step()  # warms the libraries up outside the capture; it is also the first step
        new.append(model.token.clone())
        torch.cuda.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            model.step()
        run = captured.replay
    while len(new) < new_tokens:
        run()
        new.append(model.token.clone())
    torch.cuda.synchronize()
    if cache8:
        model.check()
    return model, torch.stack(new, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--rows", type=int, default=4)
    ap.add_argument("--new-tokens", type=int, default=16)
    ap.add_argument("--base", choices=sorted(hg.BASES), default="kivi")
    ap.add_argument("--bits", type=int, choices=[2, 3, 4], default=2)
    ap.add_argument("--cache8", action="store_true", help="a paged cache in 8 bits")
    ap.add_argument("--budget", type=int, help="with --cache8: blocks of 16 tokens attended by a row and KV head")
    a = ap.parse_args()
    _, new = serve(a.layers, a.rows, a.new_tokens, base=a.base, bits=a.bits, cache8=a.cache8, budget=a.budget)
    for row, tokens in enumerate(new.tolist()):
        print(f"row {row}: {tokens}")


if __name__ == "__main__":
    main()
