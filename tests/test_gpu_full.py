"""Attention over full caches on the GPU: against softmax attention in 64 bits, over rows of any length, pages,
chunks, masked places with anything in them, streams and graphs."""
import math

import pytest
import torch

from tests import full_reference as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


ROOM = [0]


@pytest.fixture(params=[0, 1 << 19], ids=["small", "roomy"])
def room(request):
    """Caches as large as their rows, and such that could hold half a million tokens a row: joined in one launch
    from narrow tiles or in two, from wide ones where a row has many columns."""
    ROOM[0] = request.param
    yield
    ROOM[0] = 0


class Case:
    """Rows of held[b] cached tokens and lens[b] new ones (in the pages already); every other place of the pools
    holds NaN."""

    def __init__(self, P, held, lens, hq=4, hkv=2, d=64, dtype="bf16", page=32, seed=1, tail=0, packed=True, width=None,
                 max_chunk=None, scale=2.0, num_layers=1, layer=0):
        g = torch.Generator().manual_seed(seed)
        self.wide = (max(max(lens), 1) if max_chunk is None else max_chunk) * (hq // hkv) > 32   # columns of a row
        self.held, self.lens, self.page, self.layer, self.hq, self.hkv, self.d = held, lens, page, layer, hq, hkv, d
        need = [-(-(n + m) // page) if n >= 0 else 0 for n, m in zip(held, lens)]
        width = max(max(need), 1, ROOM[0] // page) if width is None else width
        cfg = P.make_full_config(len(lens), hq, hkv, d, dtype, page_size=page, max_pages=width, num_pages=sum(need) + 2)
        T = sum(lens) + tail
        self.max_chunk = max(max(lens), 1) if max_chunk is None else max_chunk
        self.full = P.DMCFull(cfg, max_tokens=T, max_chunk=self.max_chunk, num_layers=num_layers)
        self.table = R.fill_tables(self.full, need, g, spare=2)
        self.full.lengths.copy_(torch.tensor(held, dtype=torch.int32))
        dt = DT[dtype]
        self.K, self.V = (torch.full((cfg.num_pages, hkv, page, d), math.nan, dtype=dt) for _ in range(2))
        for b, (n, m) in enumerate(zip(held, lens)):
            for p0 in range(0, max(n + m, 0) if n >= 0 else 0, page):
                c = min(page, n + m - p0)
                at = int(self.table[b, p0 // page])
                self.K[at, :, :c] = torch.randn(hkv, c, d, generator=g).to(dt)
                self.V[at, :, :c] = torch.randn(hkv, c, d, generator=g).to(dt)
        self.q = (torch.randn(T, hq, d, generator=g) * scale).to(dt)
        self.cu = [0]
        for m in lens:
            self.cu.append(self.cu[-1] + m)
        self.cu_dev = torch.tensor(self.cu, dtype=torch.int32, device="cuda") if packed else None
        self.put()

    def put(self):
        self.full.k_pages.fill_(math.nan)
        self.full.v_pages.fill_(math.nan)
        self.full.k_pages[self.layer] = self.K.cuda()
        self.full.v_pages[self.layer] = self.V.cuda()

    def attend(self, **kw):
        out = torch.full(self.q.shape, 7.0, dtype=self.q.dtype, device="cuda")
        lse = torch.full(self.q.shape[:2], 7.0, device="cuda")
        return self.full.attend(self.layer, self.q.cuda(), cu_seqlens=self.cu_dev, out=out, lse=lse, **kw)

    def row(self, b):
        n, m = self.held[b], self.lens[b]
        return (R.rows_of(x, self.table, b, n + m, self.page) for x in (self.K, self.V))

    def check(self, out, lse, rows=None):
        for b, (n, m) in enumerate(zip(self.held, self.lens)):
            s = slice(self.cu[b], self.cu[b + 1])
            if m == 0 or (rows is not None and b not in rows):
                continue
            if n < 0:
                assert (out[s] == 0).all() and (lse[s] == -math.inf).all(), f"row {b} is not in use"
                continue
            o, z, eo, ez = R.attend(self.q[s], *self.row(b), n, self.wide)
            R.close(out[s], o, eo, f"out of row {b}")
            R.close(lse[s], z, ez, f"lse of row {b}")
        end = self.cu[-1]
        assert (out[end:] == 7).all() and (lse[end:] == 7).all(), "tokens behind the last row"

    def run(self, rows=None, **kw):
        out, lse = self.attend(**kw)
        self.check(out.cpu(), lse.cpu(), rows)
        self.full.check()
        return out, lse


STEP = [0, 1, 30, 31, 32, 63, 64, -1, 127, 255, 256, 300, 511, 700]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 1), (6, 2), (34, 2)])
@pytest.mark.parametrize("page", [8, 32])
def test_step(torch_cuda, room, dtype, d, hq, hkv, page):
    if (dtype, d, hq, page) == ("fp32", 128, 34, 8):
        pytest.skip("an earlier kernel for it (32 columns, registers spilled) faulted once, cause not found; that kernel is gone")
    import paper_2403_09636_amd as P
    Case(P, STEP, [1] * len(STEP), hq=hq, hkv=hkv, d=d, dtype=dtype, page=page, packed=False).run()


@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_step_of_other_pages(torch_cuda, room, page, dtype):
    import paper_2403_09636_amd as P
    Case(P, [0, 15, 16, 1023, 1024, 1500], [1] * 6, hq=8, hkv=2, d=128, dtype=dtype, page=page, packed=False).run()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 1, 128, "bf16"), (1, 1, 64, "bf16"), (2, 1, 64, "fp32"), (3, 1, 128, "fp32")])
def test_step_of_one_long_row(torch_cuda, hq, hkv, d, dtype):
    """One row over all workgroups: hundreds of records to join."""
    import paper_2403_09636_amd as P
    Case(P, [140001], [1], hq=hq, hkv=hkv, d=d, dtype=dtype, page=64, packed=False).run()


CHUNKS = [([0, 0, 0, 5], [1, 7, 33, 4]), ([100, 31, 32, 33, 0, 500], [2, 1, 0, 40, 3, 5]), ([1000, -1, 64], [16, 9, 15])]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (4, 1), (8, 1), (15, 3)])
@pytest.mark.parametrize("i", range(len(CHUNKS)))
def test_chunks(torch_cuda, room, dtype, d, hq, hkv, i):
    import paper_2403_09636_amd as P
    held, lens = CHUNKS[i]
    Case(P, held, lens, hq=hq, hkv=hkv, d=d, dtype=dtype, page=(32, 8, 64)[i], tail=3).run()


@pytest.mark.parametrize("hq,hkv,d,dtype,page", [(8, 8, 128, "bf16", 32), (16, 2, 64, "bf16", 16), (71, 1, 64, "bf16", 32),
                                                (6, 2, 128, "bf16", 128), (4, 2, 64, "fp32", 32), (2, 1, 128, "fp32", 8)])
def test_pieces(torch_cuda, room, hq, hkv, d, dtype, page):
    """Long chunks: whole prompts in an empty cache, pieces behind a context, few tokens among them."""
    import paper_2403_09636_amd as P
    Case(P, [0, 700, 77, 3000, 20], [300, 129, 0, 257, 1], hq=hq, hkv=hkv, d=d, dtype=dtype, page=page, tail=1).run()


def test_two_tokens_of_one_row_over_everything(torch_cuda, room):
    import paper_2403_09636_amd as P
    Case(P, [0, 40000, 0], [0, 200, 0], hq=8, hkv=1, d=128, page=32).run()


@pytest.mark.parametrize("cols", [1, 2, 3, 4, 5, 8, 9, 16, 17, 32, 33, 64, 65, 128, 129])
def test_column_counts(torch_cuda, room, cols):
    """Every kind of column tile, full and not."""
    import paper_2403_09636_amd as P
    Case(P, [333, 64], [cols, min(cols, 2)], hq=1, hkv=1, d=64).run()
    if cols < 65:
        Case(P, [333, 64], [1, 1], hq=cols, hkv=1, d=128, packed=False).run()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens", [[1, 1, 1], [6, 3, 1], [150, 40, 1]])
def test_what_a_query_does_not_see_never_reaches_it(torch_cuda, room, dtype, lens):
    """Infinities and NaN in later tokens of the same chunk (and behind every row, as everywhere here): each token's
    outputs are those of a row that ends with it, bit for bit."""
    import paper_2403_09636_amd as P
    held = [90, 20, 64]
    c = Case(P, held, lens, hq=8, hkv=2, d=64, dtype=dtype, page=32)
    clean = c.attend()
    c.check(*(x.cpu() for x in clean))
    for bad in (math.inf, -math.inf, math.nan):
        for pool in (c.K, c.V):
            keep = pool.clone()
            first = {}   # the first spoiled token of every row
            for b, (n, m) in enumerate(zip(held, lens)):
                first[b] = max(m - max(m // 3, 1), 1)
                for i in range(first[b], m):
                    p = n + i
                    pool[int(c.table[b, p // c.page]), :, p % c.page, (i * 7) % 64] = bad
            c.put()
            out, lse = c.attend()
            for b, m in enumerate(lens):
                s = slice(c.cu[b], c.cu[b] + min(first[b], m))
                assert torch.equal(out[s], clean[0][s]) and torch.equal(lse[s], clean[1][s]), (bad, b)
            pool.copy_(keep)
    c.put()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_infinite_values_that_are_seen(torch_cuda, room, dtype):
    import paper_2403_09636_amd as P
    c = Case(P, [100, 3], [1, 1], hq=2, hkv=1, d=64, dtype=dtype, packed=False, scale=0.5)
    c.V[int(c.table[0, 1]), 0, 5, 10] = math.inf
    c.V[int(c.table[0, 2]), 0, 1, 11] = -math.inf
    c.V[int(c.table[0, 0]), 0, 7, 12] = math.nan
    c.put()
    out, _ = c.attend()
    out = out.cpu()
    assert (out[0, :, 10] == math.inf).all() and (out[0, :, 11] == -math.inf).all() and out[0, :, 12].isnan().all()
    rest = [i for i in range(64) if i not in (10, 11, 12)]
    K, V = c.row(0)
    V = V.clone()
    V[0, :, 10:13] = 0
    o, _, eo, _ = R.attend(c.q[:1], K, V, 100)
    R.close(out[:1, :, rest], o[..., rest], eo[..., rest], "other elements")
    assert out[1].isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_scores_of_any_size(torch_cuda, room, dtype):
    """One key far above the others, all far below zero, and all equal."""
    import paper_2403_09636_amd as P
    c = Case(P, [200, 200, 200], [1, 1, 1], hq=1, hkv=1, d=64, dtype=dtype, packed=False, scale=1.0)
    c.q[:] = 1.0
    for b, val in enumerate((0.0, -60.0, 3.0)):
        for p in range(201):
            c.K[int(c.table[b, p // 32]), :, p % 32] = val
    c.K[int(c.table[0, 3]), :, 9] = 100.0
    c.put()
    out, lse = c.attend()
    c.check(out.cpu(), lse.cpu())


def test_rows_that_are_full_and_pages_that_do_not_exist(torch_cuda):
    import paper_2403_09636_amd as P
    c = Case(P, [60, 10], [4, 4], hq=4, hkv=2, d=64, page=32)
    c.full.lengths.copy_(torch.tensor([62, 10], dtype=torch.int32))   # room for two of row 0's tokens
    out, lse = c.attend()
    out, lse = out.cpu(), lse.cpu()
    assert (out[2:4] == 0).all() and (lse[2:4] == -math.inf).all()
    K, V = (R.rows_of(x, c.table, 0, 64, 32) for x in (c.K, c.V))
    o, z, eo, ez = R.attend(c.q[:2], K, V, 62, c.wide)
    R.close(out[:2], o, eo, "tokens that have room")
    R.close(lse[:2], z, ez, "their lse")
    c.check(out, lse, rows=[1])
    assert int(c.full.flags) == 2
    for page in (32, 8):
        d = Case(P, [60, 10], [4, 4], hq=4, hkv=2, d=64, page=page)
        table = d.table.clone()
        table[0, 1] = d.full.cfg.num_pages
        table[0, 0] = -7
        d.full.page_table.copy_(table)
        out, lse = d.attend()
        d.check(out.cpu(), lse.cpu(), rows=[1])
        assert int(d.full.flags) == 8


def test_bad_boundaries_raise_the_flag(torch_cuda):
    import paper_2403_09636_amd as P
    for cu, held in (([0, 5, 2, 9], None), ([-3, 3, 6, 9], None), ([0, 3, 6, 99], None), ([0, 9, 9, 9], None), (None, [2 ** 31 - 1, 1, 1])):
        c = Case(P, [40, 50, 60], [3, 3, 3], hq=2, hkv=1)
        if cu:
            c.cu_dev.copy_(torch.tensor(cu, dtype=torch.int32))
        if held:
            c.full.lengths.copy_(torch.tensor(held, dtype=torch.int32))
        c.attend(max_chunk=3)
        assert int(c.full.flags) & 4, cu


def test_same_bits_every_time_and_in_any_batch(torch_cuda, room):
    import paper_2403_09636_amd as P
    c = Case(P, [3000, 10, 700, 64], [3, 1, 2, 5], hq=8, hkv=2, d=128)
    first = c.attend()
    for _ in range(3):
        again = c.attend()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_strided_tensors_and_layers(torch_cuda, room):
    import paper_2403_09636_amd as P
    c = Case(P, [100, 33, 0], [2, 1, 3], hq=4, hkv=2, d=64, num_layers=3, layer=2)
    plain = c.attend()
    x = torch.zeros(6, 9, 80, dtype=torch.bfloat16, device="cuda")
    x[:, 2:6, :64] = c.q.cuda()
    y = torch.full((6, 4, 3, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    c.full.attend(2, x[:, 2:6, :64], cu_seqlens=c.cu_dev, out=y[:, :, 1])
    assert torch.equal(y[:, :, 1], plain[0]) and (y[:, :, 0] == 5).all() and (y[:, :, 2] == 5).all()
    one = c.q[:1, :1].cuda().expand(6, 4, 64)
    got, _ = c.full.attend(2, one, cu_seqlens=c.cu_dev)
    want, _ = c.full.attend(2, one.contiguous(), cu_seqlens=c.cu_dev)
    assert torch.equal(got, want)


def test_two_objects_on_two_streams(torch_cuda):
    import paper_2403_09636_amd as P
    cases = [Case(P, [2000, 900, 31], [1, 1, 1], hq=8, hkv=1, d=128, packed=False, seed=s) for s in (1, 2)]
    want = [c.attend() for c in cases]
    q = [c.q.cuda() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(5):
        for i, (c, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                got[i].append(c.full.attend(0, q[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for o, z in got[i]:
            assert torch.equal(o, want[i][0]) and torch.equal(z, want[i][1])


def test_a_captured_step_serves_later_ones(torch_cuda):
    """Append and attend of two layers and the new lengths, captured once and replayed, against the same steps made
    eagerly on a second cache, with other work between; two graphs share the workspace."""
    import paper_2403_09636_amd as P
    B, hq, hkv, d, page, steps = 5, 8, 2, 64, 16, 40
    f = R.inv_freqs(d).cuda()
    cfg = P.make_full_config(B, hq, hkv, d, page_size=page, max_pages=6, rotary_dim=d)
    caches = [P.DMCFull(cfg, inv_freq=f, num_layers=2) for _ in range(2)]
    g = torch.Generator().manual_seed(4)
    table = torch.randperm(B * 6, generator=g).int().view(B, 6)
    start = torch.tensor([0, 13, 40, -1000, 20], dtype=torch.int32)
    pools = [torch.randn(caches[0].k_pages.shape, generator=g).bfloat16() for _ in range(2)]   # what the rows hold already
    for c in caches:
        c.page_table.copy_(table)
        c.lengths.copy_(start)
        c.k_pages.copy_(pools[0])
        c.v_pages.copy_(pools[1])
    data = [[torch.randn(B, h, d, generator=g).bfloat16().cuda() for h in (hq, hkv, hkv)] for _ in range(steps)]
    live = [torch.empty_like(x) for x in data[0]]
    outs = [torch.empty_like(live[0]) for _ in range(2)]
    lses = [torch.empty(B, hq, device="cuda") for _ in range(2)]
    turned = torch.empty_like(live[0])

    def step(c, q, k, v):
        res = []
        for layer in range(2):
            c.append(layer, k, v, q=q, q_out=turned)
            res.append(c.attend(layer, turned, out=outs[layer], lse=lses[layer]))
        c.lengths.add_(1)
        return res

    # warm up on a third cache, so that the two under test only see their steps
    step(P.DMCFull(cfg, inv_freq=f, num_layers=2), *live)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], *live)
    for i in range(steps):
        for x, y in zip(live, data[i]):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (*outs, *lses)]
        step(caches[1], *data[i])
        for x, y in zip(got, (*outs, *lses)):
            assert torch.equal(x, y), f"step {i}"
    assert torch.equal(caches[0].lengths, caches[1].lengths)
    caches[0].check()


def test_prompts_then_pieces_then_steps(torch_cuda):
    """A layer as it is served: packed prompts rotated and attended without a cache (DMCRotation, DMCCausal) and
    appended, then a piece, a draft and single tokens over the cache: every token's output is the one that causal
    attention of the whole rotated sequence gives."""
    import paper_2403_09636_amd as P
    hq, hkv, d, page = 8, 2, 128, 32
    prompts, piece, steps = [70, 1, 33], [5, 64, 40], 3
    f = R.inv_freqs(d)
    g = torch.Generator().manual_seed(9)
    total = [p + c + steps for p, c in zip(prompts, piece)]
    seqs = [[torch.randn(n, h, d, generator=g).bfloat16() for h in (hq, hkv, hkv)] for n in total]

    def packed(lo, hi):
        return [torch.cat([s[i][a:b] for s, a, b in zip(seqs, lo, hi)]).cuda() for i in range(3)]

    def bounds(lens):
        return torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()], dtype=torch.int32, device="cuda")

    cfg = P.make_full_config(3, hq, hkv, d, page_size=page, max_pages=6, rotary_dim=d)
    full = P.DMCFull(cfg, max_tokens=200, max_chunk=128, inv_freq=f.cuda())
    full.page_table.copy_(torch.randperm(18, generator=g).int().view(3, 6))
    got = [[] for _ in range(3)]

    def collect(out, lens):
        for b, x in enumerate(out.cpu().split(lens)):
            got[b].append(x)

    # the prompts, by causal attention and then into the cache
    q, k, v = packed([0] * 3, prompts)
    rot = P.DMCRotation(P.make_rotary_config(hq, hkv, d), f.cuda())
    pos = torch.cat([torch.arange(n) for n in prompts]).int().cuda()
    cu = bounds(prompts)
    qr, kr = rot.forward(q, k, pos)
    causal = P.DMCCausal(P.make_causal_config(hq, hkv, d), 200)
    collect(causal.forward(qr, kr, v, cu)[0], prompts)
    turned = full.append(0, k, v, q=q, cu_seqlens=cu)
    assert torch.equal(turned, qr), "append and rotation turn alike"
    over, _ = full.attend(0, turned, cu_seqlens=cu)
    direct = torch.cat([x[0] for x in got])
    full.lengths.add_(torch.tensor(prompts, dtype=torch.int32, device="cuda"))
    at = list(prompts)
    for lens in (piece, [1] * 3, [1] * 3, [1] * 3):
        q, k, v = packed(at, [a + n for a, n in zip(at, lens)])
        cu = None if lens == [1] * 3 else bounds(lens)
        qr = full.append(0, k, v, q=q, cu_seqlens=cu)
        collect(full.attend(0, qr, cu_seqlens=cu)[0], lens)
        full.lengths.add_(torch.tensor(lens, dtype=torch.int32, device="cuda"))
        at = [a + n for a, n in zip(at, lens)]
    full.check()
    for b, n in enumerate(total):
        qs, ks, vs = seqs[b]
        pos = torch.arange(n)
        qt, kt = (R.turn(x, pos, f, d, "halves")[0].bfloat16() for x in (qs, ks))
        # rotated queries and keys may have been rounded to the other side of a step: 2^-7 of an element, at
        # random, which moves a score by no more than 2^-7 (|q| . |k|) / sqrt(d)
        o, _, eo, _ = R.attend(qt, kt.transpose(0, 1), vs.transpose(0, 1), 0)
        size = vs.double().abs().amax(0).repeat_interleave(hq // hkv, 0)
        R.close(torch.cat(got[b]), o, eo + 2.0 ** -6 * size, f"row {b}")
    # the prompts' attention over the cache they have just entered (P of DMCCausal is rounded to bf16: 2^-8)
    size = torch.cat([s[2][:p].double().abs().amax(0, keepdim=True).expand(p, -1, -1) for s, p in zip(seqs, prompts)])
    assert ((over.cpu().double() - direct.double()).abs() <= 2.0 ** -6 * size.repeat_interleave(hq // hkv, 1)).all()


def test_pools_past_four_gigabytes(torch_cuda):
    """A row's pages spread over 6 GB pools: appended and attended by addresses past 32 bits, bit for bit as in a
    small pool."""
    import paper_2403_09636_amd as P
    hq, hkv, d, page = 8, 2, 128, 64
    pages = (6 << 30) // (hkv * page * d * 2)
    res = []
    for n in (pages, 40):
        cfg = P.make_full_config(2, hq, hkv, d, page_size=page, max_pages=20, num_pages=n, rotary_dim=d)
        full = P.DMCFull(cfg, max_tokens=800, max_chunk=400, inv_freq=R.inv_freqs(d).cuda())
        ids = torch.arange(40, dtype=torch.int32) * (n // 40) + (n // 40 - 1)
        full.page_table.copy_(ids.view(2, 20).flip(1))
        g = torch.Generator().manual_seed(2)
        q, k, v = (torch.randn(800, h, d, generator=g).bfloat16().cuda() for h in (hq, hkv, hkv))
        cu = torch.tensor([0, 400, 800], dtype=torch.int32, device="cuda")
        for _ in range(3):
            qr = full.append(0, k, v, q=q, cu_seqlens=cu)
            out = full.attend(0, qr, cu_seqlens=cu)
            full.lengths.add_(400)
        full.lengths.sub_(1)
        res.append((*out, *full.attend(0, qr[:2].contiguous())))
        full.check()
        del full
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_many_rows(torch_cuda):
    """The largest batch (the rows' table takes 32 KB of LDS), most rows empty or short."""
    import paper_2403_09636_amd as P
    g = torch.Generator().manual_seed(6)
    held = torch.randint(-3, 12, (4096,), generator=g).tolist()
    held[77], held[4000], held[4095] = 900, 500, 130
    c = Case(P, held, [1] * 4096, hq=2, hkv=1, d=64, page=16, packed=False)
    out, lse = c.attend()
    c.check(out.cpu(), lse.cpu(), rows=set(range(0, 4096, 37)) | {76, 77, 78, 4000, 4095})
    lens = torch.randint(0, 4, (3000,), generator=g).tolist()
    c = Case(P, held[:3000], lens, hq=2, hkv=1, d=64, page=16)
    out, lse = c.attend()
    c.check(out.cpu(), lse.cpu(), rows=set(range(0, 3000, 37)) | {76, 77, 78, 2999})


def test_many_rows_of_wide_chunks(torch_cuda, room):
    """More than 64 rows (their sums in LDS beside the wide tiles' ring; fp32 tiles of 64 columns), long chunks among
    short and empty ones."""
    import paper_2403_09636_amd as P
    g = torch.Generator().manual_seed(16)
    for dtype in ("bf16", "fp32"):
        held = torch.randint(-2, 90, (300,), generator=g).tolist()
        lens = torch.randint(0, 9, (300,), generator=g).tolist()
        held[11], lens[11], held[298], lens[298], held[150], lens[150] = 700, 150, 0, 90, 60, 40
        c = Case(P, held, lens, hq=4, hkv=1, d=64, page=16, dtype=dtype, tail=1)
        out, lse = c.attend()
        c.check(out.cpu(), lse.cpu(), rows=set(range(0, 300, 13)) | {10, 11, 12, 150, 298, 299})
        c.full.check()


def test_counters_are_left_at_zero(torch_cuda, room):
    import paper_2403_09636_amd as P
    for held, lens, hq, hkv in (([900], [1], 16, 4), ([140001], [1], 8, 1), ([3000, 5, 700], [2, 1, 3], 8, 2)):
        c = Case(P, held, lens, hq=hq, hkv=hkv, d=64, packed=len(held) > 1)
        for _ in range(3):
            c.attend()
        at = -c.full.workspace.data_ptr() % 256
        assert not c.full.workspace[at:at + P.binding.DMC_FULL_COUNTER_BYTES].any()


def test_calls_without_lse_and_flags(torch_cuda):
    import ctypes
    import paper_2403_09636_amd as P
    lib = P.binding.lib
    c = Case(P, [100, -1, 33, 2000], [1, 1, 1, 1], hq=8, hkv=2, d=128, packed=False)
    want, _ = c.attend()
    q, out, f = c.q.cuda(), torch.zeros_like(want), c.full
    st = (ctypes.c_int64 * 2)(8 * 128, 128)
    ptr = [ctypes.c_void_p(t.data_ptr()) for t in (q, f.lengths, f.page_table, f.k_pages, f.v_pages, out)]
    assert lib.dmc_full_attend(ctypes.byref(f.cfg), ptr[0], st, None, 4, 1, *ptr[1:], st, None, None, f._ws, f._ws_bytes,
                               torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(out, want)
    kv = torch.randn(4, 2, 128, device="cuda").bfloat16()
    st = (ctypes.c_int64 * 2)(2 * 128, 128)
    p = ctypes.c_void_p(kv.data_ptr())
    assert lib.dmc_full_append(ctypes.byref(f.cfg), p, st, p, st, None, None, None, None, 4, *ptr[1:3], *ptr[3:5], None, None,
                               None, torch.cuda.current_stream().cuda_stream) == 0
    for b, n in ((0, 100), (2, 33), (3, 2000)):
        at = int(c.table[b, n // 32])
        assert torch.equal(f.k_pages[0, at, :, n % 32], kv[b]) and torch.equal(f.v_pages[0, at, :, n % 32], kv[b])


@pytest.mark.parametrize("chunk,hq", [(5, 8), (40, 8)])
def test_captured_chunks_at_other_lengths(torch_cuda, chunk, hq):
    """Drafts (two launches) and pieces (wide tiles), captured once; replayed over caches of other lengths, pages and
    boundaries, and compared with eager calls."""
    import paper_2403_09636_amd as P
    B, hkv, d, page, width = 6, 2, 64, 32, 400
    g = torch.Generator().manual_seed(chunk)
    cfg = P.make_full_config(B, hq, hkv, d, page_size=page, max_pages=width, num_pages=600)
    a, b = (P.DMCFull(cfg, max_tokens=B * chunk, max_chunk=chunk) for _ in range(2))
    for x in (a, b):
        for pool, s in ((x.k_pages, 1), (x.v_pages, 2)):
            pool.copy_(torch.randn(pool.shape, generator=torch.Generator().manual_seed(s)).bfloat16())
    q, out, cu = torch.empty(B * chunk, hq, d, device="cuda").bfloat16(), torch.zeros(B * chunk, hq, d, device="cuda").bfloat16(), \
        torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    lse = torch.zeros(B * chunk, hq, device="cuda")
    a.attend(0, q, cu_seqlens=cu, out=out, lse=lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.attend(0, q, cu_seqlens=cu, out=out, lse=lse)
    for i in range(6):
        lens = torch.randint(0, chunk + 1, (B,), generator=g)
        held = torch.randint(-1, (60, 500, 12000)[i % 3], (B,), generator=g)
        table = torch.randint(0, 600, (B, width), generator=g)   # (shared pages are only read here)
        cu.copy_(torch.cat([torch.zeros(1, dtype=torch.long), lens.cumsum(0)]).int())
        q.copy_(torch.randn(q.shape, generator=g).bfloat16())
        for x in (a, b):
            x.lengths.copy_(held.int())
            x.page_table.copy_(table.int())
        out.fill_(3)
        lse.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        o, z = torch.full_like(out, 3), torch.full_like(lse, 3)
        b.attend(0, q, cu_seqlens=cu, out=o, lse=z)
        assert torch.equal(out, o) and torch.equal(lse, z), f"replay {i}"
    a.check()


def test_the_largest_batch_with_wide_chunks(torch_cuda):
    """4096 rows: their sums (32 KB) beside the ring of the wide tiles (64 KB) and the workgroup's places."""
    import paper_2403_09636_amd as P
    held, lens = [-1] * 4096, [0] * 4096
    for b, n, m in ((0, 40, 70), (1, 0, 0), (2000, 300, 33), (4094, 7, 1), (4095, 600, 140)):
        held[b], lens[b] = n, m
    c = Case(P, held, lens, hq=4, hkv=1, d=128, page=32, tail=1)
    out, lse = c.attend()
    c.check(out.cpu(), lse.cpu(), rows={0, 1, 2000, 4094, 4095})
    c.full.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [32, 33, 48, 63, 64, 65])
def test_about_as_many_units_as_workgroups(torch_cuda, room, dtype, rows):
    """256 to 520 units of 8 kv heads and up to 500 keys: cut equally, left whole, or in ranges."""
    import paper_2403_09636_amd as P
    g = torch.Generator().manual_seed(rows)
    held = torch.randint(-40, 500, (rows,), generator=g).tolist()
    held[0], held[-1] = 499, 320
    c = Case(P, held, [1] * rows, hq=16, hkv=8, d=64, dtype=dtype, packed=False)
    out, lse = c.attend()
    c.check(out.cpu(), lse.cpu(), rows=set(range(0, rows, 7)) | {rows - 1})
    c.full.check()


@pytest.mark.parametrize("tokens", [255, 256, 257, 400, 512, 520])
def test_prompts_of_about_as_many_units_as_workgroups(torch_cuda, room, tokens):
    import paper_2403_09636_amd as P
    Case(P, [0], [tokens], hq=32, hkv=8, d=64).run()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_calls_of_either_kind_on_one_workspace(torch_cuda, dtype):
    """Small calls (joined within their launch) and large ones (joined by a second) in turn on one object; every one gives
    the same bits as on an object of its own."""
    import paper_2403_09636_amd as P
    B, hq, hkv, d, page, width = 4, 16, 8, 64, 32, 64
    g = torch.Generator().manual_seed(3)
    cfg = P.make_full_config(B, hq, hkv, d, dtype, page_size=page, max_pages=width)
    make = lambda: P.DMCFull(cfg, max_tokens=1200, max_chunk=300)
    a, pools = make(), [torch.randn(make().k_pages.shape, generator=g).to(DT[dtype]) for _ in range(2)]
    table = torch.randperm(B * width, generator=g).view(B, width).int()
    held = torch.tensor([1500, 40, 0, 700], dtype=torch.int32)

    def fill(x):
        x.k_pages.copy_(pools[0])
        x.v_pages.copy_(pools[1])
        x.page_table.copy_(table)
        x.lengths.copy_(held)
        return x
    fill(a)
    calls = []
    for lens in ([1, 1, 1, 1], [300, 300, 300, 300], [2, 0, 7, 1], [300, 5, 280, 300], [60, 1, 0, 2]):
        cu = torch.tensor([0] + lens).cumsum(0).int().cuda()
        q = torch.randn(sum(lens), hq, d, generator=g).to(DT[dtype]).cuda()
        calls.append((q, cu, fill(make()).attend(0, q, cu_seqlens=cu)))
    for _ in range(3):
        for q, cu, want in calls:
            got = a.attend(0, q, cu_seqlens=cu)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), cu.tolist()
    a.check()
