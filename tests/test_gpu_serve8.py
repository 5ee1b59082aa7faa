"""The serving example over the paged cache in 8 bits: rows take their pages on the
GPU, steps are captured, and each step's attention is the formula's over the cache
as it stands, of all blocks or of the chosen ones."""
import pytest
import torch

import attnref
import cache8ref as ref
from attnref import assert_close
from examples import serve

pytestmark = pytest.mark.gpu


def raw(t):
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


@pytest.mark.parametrize("budget", [None, 6])
def test_graph_and_eager_serve_the_same(budget):
    a, ta = serve.serve(layers=2, rows=3, new_tokens=40, img_len=100, cache8=True, budget=budget, graph=True)
    b, tb = serve.serve(layers=2, rows=3, new_tokens=40, img_len=100, cache8=True, budget=budget, graph=False)
    assert torch.equal(ta, tb) and ta.shape == (3, 40)
    for x, y in zip([a.pool] + a.caches, [b.pool] + b.caches):
        for s, t in zip(x.tensors, y.tensors):
            assert torch.equal(raw(s), raw(t))
    assert a.result.tolist()[0] == 0
    held = [p for row, n in zip(a.table.tolist(), a.lens.tolist()) for p in row[:-(-n // 32)]]
    assert sorted(held + a.free_pages[:int(a.n_free)].tolist()) == list(range(len(a.free_pages)))
    a.release()
    torch.cuda.synchronize()
    assert int(a.n_free) == len(a.free_pages) and a.lens.tolist() == [0, 0, 0] and bool((a.table == -1).all())


@pytest.mark.parametrize("budget", [None, 5])
def test_each_step_attends_over_the_cache(budget):
    lens, tokens, cu = serve.prompts(3, 16, 100)
    m = serve.Decoder8(1, 3, lens, 4, budget=budget)
    m.prefill(tokens, cu)
    G, ps, block = m.Hq // m.H, 32, 16
    for _ in range(3):
        m.step()
        torch.cuda.synchronize()
        K, V, ks, vs, bounds, table = (t.cpu() for t in m.caches[0].tensors)
        for b, n in enumerate(m.lens.tolist()):
            row = table[b].long()
            for h in range(m.H):
                q = m.q[b, h * G:(h + 1) * G].cpu()
                t = torch.arange(n)
                if budget is not None:
                    limits = [bounds[row[i * block // ps], h, i * block % ps // block] for i in range((n - 1) // block + 1)]
                    want = ref.select(q, limits, 0, budget, 1, 2)
                    assert m.blocks[b, h].tolist() == want
                    t = torch.tensor([x for i in want for x in range(i * block, min(i * block + block, n))])
                page, off = row[t // ps], t % ps
                o, _, to, _ = attnref.attend(q, ref.values(K[page, h, off], ks[page, h, off // block]),
                                             ref.values(V[page, h, off], vs[page, h, off // block]), m.D ** -0.5)
                assert_close(m.o[b, h * G:(h + 1) * G], o, to, f"row {b} head {h}")
    assert m.lens.tolist() == [n + 3 for n in lens]


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("budget", [None, 5])
def test_steps_past_the_pool_change_nothing(graph, budget):
    """Rows outgrow their pages: the steps that the pool refuses leave lengths, table and every byte of
    the cache alone, and the model says so; prompts without pages are refused before they are stored."""
    lens, tokens, cu = serve.prompts(2, 16, 40)
    m = serve.Decoder8(2, 2, lens, 2, budget=budget)
    m.prefill(tokens, cu)
    m.step()
    run = m.step
    if graph:
        torch.cuda.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            m.step()
        run = captured.replay
    state, refused = None, 0
    for _ in range(70):
        run()
        torch.cuda.synchronize()
        now = [raw(t).clone() for x in [m.pool] + m.caches for t in x.tensors]
        if int(m.result[0]):
            assert all(torch.equal(a, b) for a, b in zip(state, now))
            refused += 1
        else:
            assert refused == 0
            m.check()
        state = now
    assert 0 < refused < 70
    with pytest.raises(RuntimeError):
        m.check()
    small = serve.Decoder8(1, 2, [8, 8], 1)
    small.targets.copy_(torch.tensor(lens, dtype=torch.int32))
    with pytest.raises(RuntimeError):
        small.prefill(tokens, cu)
    assert not bool(small.caches[0].tensors[0].any()) and small.lens.tolist() == [0, 0]
