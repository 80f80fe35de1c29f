"""Chunks in buffers that are much longer than their tokens (a padded batch, a captured graph's static
buffers): the unused rows change nothing, neither the outputs nor how the attention is cut into pieces."""
import pytest

from tests.gpu_helpers import log
from tests.test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,lens,most,total", [
    # one narrow tile per unit, cut into pieces for a long cache; the buffer alone holds eight tiles per compute unit
    (64, 8, [4, 3], 4, 1024), (8, 8, [8, 1], 8, 8192), (2, 2, [30, 0], 32, 32768),
    # planned pieces: more columns than a narrow tile
    (8, 8, [40, 3], 40, 16384), (16, 4, [100], 100, 8192),
])
def test_long_buffers(torch_cuda, dtype, hq, hkv, lens, most, total):
    log(f"{dtype} heads {hq}/{hkv} lens {lens} in {total} rows")
    slots = [[2000] + [600] * (hkv - 1), [30] * hkv][:len(lens)]
    c = Case(hq, hkv, 64, dtype, slots, max_tokens=total, max_chunk=most)
    x = c.tokens(lens, 2.0, tail=total - sum(lens))
    log(f"worst {c.attend(*x, lens):.3f} of the bound")
    c.cache.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_replays_with_other_lengths(torch_cuda, dtype):
    """A graph captured once over buffers of 4096 rows: every replay takes the lengths, tokens and cache of
    its time, as eager calls on another cache do, bit for bit."""
    import torch

    from tests.packed_reference import cu_of
    hq, hkv, total = 8, 2, 4096
    cases = [Case(hq, hkv, 64, dtype, [[2000, 40], [3, 3], [0, 700]], max_tokens=total, max_chunk=8) for _ in range(2)]
    q, k, v = cases[0].tokens([total], 2.0)
    cu = cu_of([8, 0, 3]).cuda()
    outs = [torch.zeros_like(q) for _ in cases]

    def step(c, out):
        c.chunk.attend(0, q, k, v, cu, out=out)
        c.chunk.append(0, k, v, q, cu)
    for c, out in zip(cases, outs):
        step(c, out)
    assert torch.equal(*outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cases[0], outs[0])
    for i, lens in enumerate(([1, 1, 1], [0, 0, 0], [8, 8, 8], [0, 5, 0])):
        for a, b in zip((q, k, v), cases[0].tokens([total], 2.0)):
            a.copy_(b)
        cu.copy_(cu_of(lens))
        outs[0].fill_(i)
        outs[1].fill_(i)
        graph.replay()
        step(cases[1], outs[1])
        torch.cuda.synchronize()
        assert torch.equal(*outs) and (outs[0][sum(lens):] == i).all(), lens
        for a, b in zip(cases[0].cache.export(0, 2100), cases[1].cache.export(0, 2100)):
            assert torch.equal(a, b)
    cases[0].cache.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tail", [0, 3000])
def test_many_rows(torch_cuda, dtype, tail):
    """More rows than a wave has lanes and more units than the planning workgroup has threads; sampled rows."""
    import numpy as np

    from tests.gpu_helpers import f64
    from tests.packed_reference import cu_of
    rng = np.random.default_rng(7)
    B, hkv = 100, 8
    slots = rng.integers(0, 70, (B, hkv))
    slots[41, 3] = 1500
    lens = [int(x) for x in rng.integers(0, 4, B)]
    lens[0], lens[41], lens[99] = 5, 90, 66
    c = Case(8, hkv, 64, dtype, slots, max_tokens=sum(lens) + tail, max_chunk=90, extra=100)
    q, k, v = c.tokens(lens, 2.0, tail=tail)
    out = f64(c.chunk.attend(0, q, k, v, cu_of(lens).cuda(), out=torch_cuda.zeros_like(q)))
    c.chunk.append(0, k, v, q, cu_of(lens).cuda())
    L = c.cache.lengths(0).cpu().numpy()
    sample = (0, 41, 63, 64, 65, 99)
    c.ref.units = [c.ref.units[b] for b in sample]
    lo = np.concatenate([[0], np.cumsum(lens)])
    rows = np.concatenate([np.arange(lo[b], lo[b + 1]) for b in sample])
    mine = [lens[b] for b in sample]
    want, bound, _ = c.ref.chunk(*(f64(t)[rows] for t in (q, k, v)), mine, commit=mine)
    assert (np.abs(out[rows] - want) <= bound).all()
    assert (L[list(sample)] == c.ref.lengths()).all()
    c.cache.check()


@pytest.mark.parametrize("dtype,page", [("bf16", 4096), ("fp32", 1024)])
def test_one_page_a_unit(torch_cuda, dtype, page):
    """Pages as large as a unit, and rows of many 64-token blocks that never open a slot."""
    lens = [700, 3]
    c = Case(4, 2, 64, dtype, [[100, 0], [900, 33]], page=page, extra=100, max_tokens=800, max_chunk=700)
    x = c.tokens(lens, [1000.0, 50.0])
    x[1][:, 0, 0] = 2.0   # the first head merges everything
    log(f"worst {c.attend(*x, lens):.3f} of the bound")
    c.append(*x, lens)
    c.cache.check()
