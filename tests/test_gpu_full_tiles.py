"""Attention over full caches by the tiles that a call takes: narrow ones keep two terms of every probability, also where a
row has many columns; a row's results in batches of several kinds; infinities that queries see in chunks."""
import math

import pytest
import torch

from tests import full_reference as R
from tests.test_gpu_full import ROOM, Case

pytestmark = pytest.mark.gpu


def takes_wide_tiles(case):
    """Whether the call rounds its probabilities to one bf16 term: 128 columns, bf16, groups of up to 128 heads, unless the
    cache's capacity bounds the work to be small."""
    cfg, T = case.full.cfg, case.q.shape[0]
    G = case.hq // case.hkv
    if case.q.dtype != torch.bfloat16 or case.max_chunk * G <= 32 or G > 128:
        return False
    tiles = T * G // 32 + cfg.batch
    return tiles * case.hkv * cfg.max_pages * cfg.page_size > 1 << 18


@pytest.fixture(params=[0, 1 << 19], ids=["small", "roomy"])
def room(request):
    ROOM[0] = request.param
    yield
    ROOM[0] = 0


@pytest.mark.parametrize("held,lens,hq,hkv,d,narrow", [
    ([0, 0, 0, 5], [1, 7, 33, 4], 8, 1, 64, True), ([100, 31, 32, 33, 0, 500], [2, 1, 0, 40, 3, 5], 8, 2, 128, True),
    ([1000, -1, 64], [16, 9, 15], 15, 3, 64, True), ([300], [40], 4, 2, 128, True),
    ([200, 900], [2, 3], 131, 1, 64, True),                                   # groups past 128 heads
    ([0, 700, 77, 3000, 20], [300, 129, 0, 257, 1], 8, 8, 128, False)])
def test_tiles_by_their_own_bound(torch_cuda, room, held, lens, hq, hkv, d, narrow):
    """Each call within the bound of the tiles that it takes: 2^-16 of the probabilities in narrow ones."""
    import paper_2403_09636_amd as P
    c = Case(P, held, lens, hq=hq, hkv=hkv, d=d, page=32, tail=1)
    c.wide = takes_wide_tiles(c)
    assert c.wide == (not narrow or ROOM[0] > 0 and hq // hkv <= 128)
    c.run()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [1, 3, 40])
def test_a_row_alone_and_among_others(torch_cuda, dtype, m):
    """One row's tokens in calls of one row, of a few and of 80 (other cuts of its keys, other tiles): each result within
    the bound of the tiles that the call takes."""
    import paper_2403_09636_amd as P
    n, hq, hkv, d, page = 1500, 8, 2, 64, 32
    first = None
    for rows, width in ((1, None), (1, 4096), (4, None), (4, 4096), (80, None)):
        lens = [m] + [1 + (b * 5) % m for b in range(1, rows)]
        held = [n] + [(b * 37) % 600 for b in range(1, rows)]
        c = Case(P, held, lens, hq=hq, hkv=hkv, d=d, dtype=dtype, page=page, seed=rows, width=width)
        if first is None:
            first = [x.clone() for x in (c.q[:m], *c.row(0))]
        c.q[:m] = first[0]
        for pool, rows_ in ((c.K, first[1]), (c.V, first[2])):
            for p in range(n + m):
                pool[int(c.table[0, p // page]), :, p % page] = rows_[:, p]
        c.put()
        c.wide = takes_wide_tiles(c)
        c.run(rows={0, rows - 1})


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m", [3, 40, 150])
def test_infinite_values_that_some_queries_see(torch_cuda, room, dtype, m):
    """Values of infinity and NaN among the cached tokens and among the new ones: they reach exactly the tokens that see
    them, as themselves; infinities of both signs make NaN; all other elements are as without them."""
    import paper_2403_09636_amd as P
    n, hq, hkv, d, page = 90, 8, 2, 64, 32
    c = Case(P, [20, n, 5], [2, m, 1], hq=hq, hkv=hkv, d=d, dtype=dtype, page=page, scale=0.5)
    spoiled = {10: (math.inf, 7), 11: (-math.inf, 64), 12: (math.nan, 89), 13: (math.inf, n), 14: (-math.inf, n + m // 2),
               15: (math.nan, n + m - 1), 63: (math.inf, n + m - 1)}   # element: value, position

    def spoil(e, x, p):
        c.V[int(c.table[1, p // page]), :, p % page, e] = x
    for e, (x, p) in spoiled.items():
        spoil(e, x, p)
    spoil(16, math.inf, 3)            # both signs: seen one after the other
    spoil(16, -math.inf, n + 1)
    c.put()
    out, lse = (x.cpu() for x in c.attend())
    s = slice(c.cu[1], c.cu[2])
    pos = n + torch.arange(m)
    for e, (x, p) in spoiled.items():
        got, seen = out[s, :, e].float(), pos >= p
        assert (got[seen].isnan() if math.isnan(x) else got[seen] == x).all(), (e, x, p)
        assert got[~seen].isfinite().all(), (e, x, p)
    both = out[s, :, 16].float()
    assert (both[pos < n + 1] == math.inf).all() and both[pos >= n + 1].isnan().all()
    # the elements that nothing spoils, and the spoiled ones where they are not seen
    K, V = c.row(1)
    V = V.clone()
    V[~V.isfinite()] = 0
    o, z, eo, ez = R.attend(c.q[s], K, V, n, takes_wide_tiles(c))
    rest = [e for e in range(d) if e not in spoiled and e != 16]
    R.close(out[s][..., rest], o[..., rest], eo[..., rest], "other elements")
    for e, (x, p) in spoiled.items():
        unseen = pos < p
        R.close(out[s][unseen][..., e], o[unseen][..., e], eo[unseen][..., e], f"element {e} before it is seen")
    R.close(lse[s], z, ez, "lse")
    c.check(out, lse, rows=[0, 2])
