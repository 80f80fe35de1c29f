"""Appends near the end of the page pool: a unit whose pages are not there takes none, so that others
get theirs and the pool is used to its last page."""
import pytest
import torch

from tests.gpu_helpers import log
from tests.packed_reference import cu_of
from tests.test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


def opening(c, lens):
    """Tokens that each open a slot."""
    q, k, v = c.tokens(lens, 1.0)
    k[..., 0] = -1
    return q, k, v


def append(c, x, lens):
    q, k, v = x
    slot = torch.full((sum(lens), c.hkv), -9, dtype=torch.int32, device="cuda")
    c.chunk.append(0, k, v, q, cu_of(lens).cuda(), slot_index=slot)
    return slot.tolist()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("page,many", [(8, 48), (32, 192)])   # one launch; several
def test_a_refused_unit_takes_no_pages(torch_cuda, dtype, page, many):
    slots = [[page], [page], [2 * page], [0]]            # full pages: any new slot needs one
    c = Case(1, 1, 64, dtype, slots, page=page, num_pages=4 + 5, max_chunk=many)
    before = c.cache.export(0, 2 * page)
    lens = [many, 3, 1, page]                            # 6 pages of the 5 left; 1 each
    slot = append(c, opening(c, lens), lens)
    assert c.cache.lengths(0).flatten().tolist() == [page, page + 3, 2 * page + 1, page]
    assert slot[:many] == [[-1]] * many
    assert slot[many:] == [[page], [page + 1], [page + 2], [2 * page]] + [[i] for i in range(page)]
    for a, b in zip(before[:2], c.cache.export(0, 2 * page)):
        assert torch.equal(a[0], b[0])
    assert c.cache.pages_used() == 7 and c.cache.status() == 3
    lens = [page + 1, 0, 0, 0]                           # the two pages that are left
    slot = append(c, opening(c, lens), lens)
    assert slot == [[page + i] for i in range(page + 1)]
    assert c.cache.lengths(0).flatten().tolist() == [2 * page + 1, page + 3, 2 * page + 1, page]
    assert c.cache.pages_used() == 9


@pytest.mark.parametrize("n", [40, 100])
def test_the_last_page(torch_cuda, n):
    """Many units at once take exactly the pages that there are; the next slot of each is refused."""
    rows, hkv = 24, 16
    need = rows * hkv * -(-n // 8)
    c = Case(16, hkv, 64, "bf16", [[0] * hkv] * rows, page=8, num_pages=need, max_tokens=rows * n, max_chunk=n)
    x = opening(c, [n] * rows)
    log(f"{need} pages")
    append(c, x, [n] * rows)
    c.cache.check()
    assert c.cache.pages_used() == need and (c.cache.lengths(0) == n).all()
    K, V, _ = c.cache.export(0, n)
    want = x[1].view(rows, n, hkv, 64).transpose(1, 2).clone()
    want[..., 0] = 0
    assert torch.equal(K, want) and torch.equal(V, x[2].view(rows, n, hkv, 64).transpose(1, 2))
    more = 8 - n % 8 + 1 if n % 8 else 1
    append(c, opening(c, [more] * rows), [more] * rows)
    assert (c.cache.lengths(0) == n).all() and c.cache.status() == 3
    for a, b in zip((K, V), c.cache.export(0, n)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_appends_after_decode_steps_used_up_the_pool(torch_cuda, dtype):
    """Refused decode steps and refused chunks in turns; units with room in their last page take theirs."""
    for hq in (1, 8):
        c = Case(hq, 1, 64, dtype, [[32], [32], [30]], num_pages=4, max_chunk=2)
        for i in range(3):
            q, k, v = opening(c, [1, 1, 0 if i else 1])
            q, k, v = (torch.cat([t, t[:1]])[:3] for t in (q, k, v))
            if i:
                k[2, :, 0] = 1   # merges
            c.cache.decode_step(0, q, k, v)
            L = c.cache.lengths(0).flatten().tolist()
            assert sorted(L[:2]) == [32, 33 + i] and L[2] == 31 + (i > 0) and c.cache.pages_used() == 4
            assert c.cache.status() == 3
            lens = [0, 0, 2 if i else 1]   # the third unit's page holds 32
            append(c, opening(c, lens), lens)
            assert c.cache.lengths(0).flatten().tolist() == L[:2] + [32]
            lens = [L[0] == 32, L[1] == 32, 0]   # the unit without a page
            append(c, opening(c, [int(x) for x in lens]), [int(x) for x in lens])
            assert c.cache.lengths(0).flatten().tolist() == L[:2] + [32] and c.cache.pages_used() == 4
