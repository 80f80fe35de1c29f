"""Tokens of full caches that are dropped (rows not in use, or full): each of their rows in the outputs is written, by the whole
chip."""
import math
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [2, 70])
def test_dropped_tokens_are_written_by_the_whole_chip(torch_cuda, rows):
    """A row that is not in use, with 8192 tokens: 134 MB of zeros and their lse take about as long as a fill of them, within
    a factor of ten (one workgroup alone would take a hundred times as long).  Every one of them is written."""
    import paper_2403_09636_amd as P
    T, hq, d = 8192, 64, 128
    cfg = P.make_full_config(rows, hq, 8, d, page_size=32, max_pages=4, num_pages=4)
    full = P.DMCFull(cfg, max_tokens=T + 1, max_chunk=T)
    full.page_table.zero_()
    for b, held in ((rows - 1, -1), (rows - 1, 128)):   # not in use; full
        lengths = torch.zeros(rows, dtype=torch.int32)
        lengths[b] = held
        full.lengths.copy_(lengths)
        cu = torch.zeros(rows + 1, dtype=torch.int32)
        cu[1:] = 1   # row 0 has one token
        cu[b + 1:] += T
        cu = cu.cuda()
        q = torch.randn(T + 1, hq, d, device="cuda").bfloat16()
        full.k_pages.zero_()
        full.v_pages.fill_(2.0)
        out, lse = torch.full_like(q, 7.0), torch.full((T + 1, hq), 7.0, device="cuda")

        def best(fn):
            took = []
            for _ in range(5):
                torch.cuda.synchronize()
                t0 = time.perf_counter()
                fn()
                torch.cuda.synchronize()
                took.append(time.perf_counter() - t0)
            return min(took)

        call = best(lambda: full.attend(0, q, cu_seqlens=cu, out=out, lse=lse))
        assert (out[1:] == 0).all() and (lse[1:] == -math.inf).all() and (out[0] == 2.0).all()
        assert int(full.flags) == (0 if held < 0 else 2)
        full.flags.zero_()
        fill = best(lambda: out.zero_())
        assert call <= 10 * max(fill, 20e-6), f"{call * 1e6:.0f} us, a fill {fill * 1e6:.0f} us"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [5, 64, 65, 700])
def test_every_dropped_token_of_many_rows(torch_cuda, dtype, rows):
    """Unused and full rows of 0 to 300 tokens among others (17 heads: items that end inside a wave); rows behind the last
    one and rows of other tokens stay as they were or get their own results."""
    import paper_2403_09636_amd as P
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    g = torch.Generator().manual_seed(rows)
    hq, d, page, width, tail = 17, 64, 8, 2, 5
    lens = torch.randint(0, 4, (rows,), generator=g)
    held = torch.randint(-2, 20, (rows,), generator=g)   # (capacity 16: full rows among them)
    held.clamp_(max=16)
    for b, n, m in ((1, -1, 300), (rows - 1, 16, 111), (rows // 2, 14, 37)):
        held[b], lens[b] = n, m
    cfg = P.make_full_config(rows, hq, 1, d, dtype, page_size=page, max_pages=width, num_pages=2)
    T = int(lens.sum()) + tail
    full = P.DMCFull(cfg, max_tokens=T, max_chunk=300)
    full.page_table.copy_(torch.tensor([0, 1], dtype=torch.int32).expand(rows, 2))
    full.lengths.copy_(held.int())
    full.k_pages.zero_()
    full.v_pages.fill_(3.0)
    cu = torch.cat([torch.zeros(1, dtype=torch.long), lens.cumsum(0)])
    q = torch.randn(T, hq, d, generator=g).to(dt).cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((T, hq), 7.0, device="cuda")
    full.attend(0, q, cu_seqlens=cu.int().cuda(), out=out, lse=lse)
    want, z = torch.full((T,), 7.0), torch.full((T,), 7.0)
    for b in range(rows):
        n = int(held[b])
        for i in range(int(lens[b])):
            t = int(cu[b]) + i
            room = n >= 0 and n + i < page * width
            want[t], z[t] = (3.0, math.log(n + i + 1)) if room else (0.0, -math.inf)
    # (equal scores of 0 and equal values: the weighted mean of 3 rounds by a few 2^-24; bf16 then holds 3 itself)
    off = 0.0 if dtype == "bf16" else 3.0 * 20 * 2.0 ** -24
    assert ((out.cpu().float() - want[:, None, None]).abs() <= off * (want == 3.0)[:, None, None]).all()
    got = lse.cpu()
    live = z.isfinite()
    assert torch.equal(got[~live], z[~live, None].expand(-1, hq))
    assert ((got[live] - z[live, None]).abs() <= 2.0 ** -20 * (1 + z[live, None].abs())).all()
