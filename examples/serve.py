"""A small decoder with random weights, served through the package: prompts
with an image each are prefilled, their image KV quantized in place, and tokens
decoded from the cache.

    python examples/serve.py [--layers 4] [--rows 4] [--new-tokens 16] [--base kivi] [--bits 2]

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
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.L, self.B, self.Hq, self.H, self.D = layers, rows, Hq, H, D
        width = Hq * D

        def weight(*shape):
            return (torch.randn(shape, generator=g, device="cuda") * shape[0] ** -0.5).to(BF)

        self.embedding = (torch.randn((vocab, width), generator=g, device="cuda")).to(BF)
        self.qkv = [weight(width, (Hq + 2 * H) * D) for _ in range(layers)]
        self.out = [weight(width, width) for _ in range(layers)]
        self.head = weight(width, vocab)
        self.T = max(prompt_lens) + new_tokens
        self.K = torch.zeros((layers, rows, H, self.T, D), dtype=BF, device="cuda")
        self.V = torch.zeros_like(self.K)
        table = torch.arange(rows, dtype=torch.int32, device="cuda").view(rows, 1)
        self.caches = [hg.make_paged_cache(self.K[l], self.V[l], table) for l in range(layers)]
        angle = torch.arange(self.T, device="cuda", dtype=torch.float64).view(-1, 1) * 1e4 ** (
            -torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
        self.rotation = hg.make_rotation(angle.cos().float(), angle.sin().float())
        self.workspace = hg.alloc_decode_workspace(self.caches[0], Hq)
        # the quantizer's side: a span shared by the rows, one head in eight protected
        self.cfg = hg.make_config(L=layers, B=rows, H=H, T=self.T, D=D, img_start=img_start, img_len=img_len, bits=bits,
                                  base=base, keys_only=0)
        self.mask = torch.zeros(layers * H, dtype=torch.uint8).numpy()
        self.mask[::8] = 1
        self.quantize_workspace = hg.alloc_fake_workspace(self.cfg, self.mask)
        # decode state
        self.lens = torch.tensor(prompt_lens, dtype=torch.int32, device="cuda")
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
            hg.hg_append_kv(self.caches[l], self.rotation, q, k, v, self.lens, q_rot, cu_new=cu, k_out=k_rot)
            hg.hg_prefill_attention(q_rot, k_rot, v, cu, o)
            h = h + o.view(n, -1) @ self.out[l]
        logits = self._logits(h[cu[1:].long() - 1])
        self.token.copy_(logits.argmax(-1))
        return logits

    def quantize_images(self):
        hg.hg_fake_quantize(self.cfg, self.K, self.V, self.mask, self.K, self.V, self.quantize_workspace)

    def step(self):
        """One new token per row; returns the logits."""
        self.lens += 1
        h = self.embedding[self.token]
        for l in range(self.L):
            q, k, v = self._split(torch.nn.functional.rms_norm(h, h.shape[-1:]) @ self.qkv[l])
            hg.hg_append_kv(self.caches[l], self.rotation, q, k, v, self.lens, self.q)
            hg.hg_decode_attention(self.caches[l], self.q, self.lens, self.o, self.workspace)
            h = h + self.o.view(self.B, -1) @ self.out[l]
        logits = self._logits(h)
        self.token.copy_(logits.argmax(-1))
        return logits


def prompts(rows, img_start, img_len, seed=0, vocab=512):
    """Row lengths (text, image, text of its own length), packed tokens, offsets."""
    g = torch.Generator().manual_seed(seed + 1)
    lens = [img_start + img_len + int(torch.randint(1, 40, (1,), generator=g)) for _ in range(rows)]
    tokens = torch.randint(0, vocab, (sum(lens),), generator=g).cuda()
    cu = torch.tensor([sum(lens[:i]) for i in range(rows + 1)], dtype=torch.int32, device="cuda")
    return lens, tokens, cu


def serve(layers=4, rows=4, new_tokens=16, img_start=16, img_len=256, base="kivi", bits=2, graph=True, seed=0):
    """Serves random prompts; returns the decoder and the new tokens [rows, new_tokens]."""
    lens, tokens, cu = prompts(rows, img_start, img_len, seed)
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
    return model, torch.stack(new, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--rows", type=int, default=4)
    ap.add_argument("--new-tokens", type=int, default=16)
    ap.add_argument("--base", choices=sorted(hg.BASES), default="kivi")
    ap.add_argument("--bits", type=int, choices=[2, 3, 4], default=2)
    a = ap.parse_args()
    _, new = serve(a.layers, a.rows, a.new_tokens, base=a.base, bits=a.bits)
    for row, tokens in enumerate(new.tolist()):
        print(f"row {row}: {tokens}")


if __name__ == "__main__":
    main()
