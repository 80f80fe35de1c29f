"""The position rotation and the append to a full cache on the GPU, against the formulas in 64 bits."""
import pytest
import torch

from tests import full_reference as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _rotation(P, hq, hkv, d, dtype, r, pairs):
    f = R.inv_freqs(r) if r else None
    rot = P.DMCRotation(P.make_rotary_config(hq, hkv, d, dtype, rotary_dim=r, pairs=pairs), None if f is None else f.cuda())
    return rot, f


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,r", [(64, 64), (64, 16), (128, 128), (128, 48), (128, 0)])
@pytest.mark.parametrize("pairs", ["halves", "adjacent"])
@pytest.mark.parametrize("tokens,hq,hkv", [(1, 4, 2), (3, 5, 5), (70, 6, 1)])
def test_rotation_and_gradients(torch_cuda, dtype, d, r, pairs, tokens, hq, hkv):
    import paper_2403_09636_amd as P
    g = torch.Generator().manual_seed(tokens * 131 + d + r)
    rot, f = _rotation(P, hq, hkv, d, dtype, r, pairs)
    q, k, dq, dk = (torch.randn(tokens, h, d, generator=g).to(DT[dtype]) for h in (hq, hkv, hq, hkv))
    pos = torch.randint(-50, 9000, (tokens,), generator=g).int()
    pos[-1] = 2 ** 31 - 1
    got = rot.forward(q.cuda(), k.cuda(), pos.cuda())
    back = rot.backward(dq.cuda(), dk.cuda(), pos.cuda())
    for name, x, y, inverse in (("q", q, got[0], False), ("k", k, got[1], False), ("dq", dq, back[0], True), ("dk", dk, back[1], True)):
        R.close(y, *R.turn(x, pos, f, r, pairs, inverse), name)


@pytest.mark.parametrize("pairs", ["halves", "adjacent"])
def test_gradient_against_differences(torch_cuda, pairs):
    """The rotation is linear: the change of sum(out * g) along any direction e is sum(e * gradient), without
    any error of its own; sums of 2 d products of fp32 results, each within 2^-20 of their size."""
    import paper_2403_09636_amd as P
    rot, _ = _rotation(P, 2, 1, 64, "fp32", 64, pairs)
    g = torch.Generator().manual_seed(5)
    q, k, gq, gk, eq, ek = (torch.randn(33, h, 64, generator=g) for h in (2, 1, 2, 1, 2, 1))
    pos = torch.arange(33, dtype=torch.int32) * 1001
    dq, dk = (x.cpu().double() for x in rot.backward(gq.cuda(), gk.cuda(), pos.cuda()))
    step = [rot.forward(a.cuda(), b.cuda(), pos.cuda()) for a, b in ((q + eq, k + ek), (q, k))]
    for i, (e, gr, grad) in enumerate(((((q + eq) - q).double(), gq, dq), (((k + ek) - k).double(), gk, dk))):
        change = ((step[0][i].cpu().double() - step[1][i].cpu().double()) * gr.double()).sum((1, 2))
        size = ((step[0][i].abs() + step[1][i].abs()).cpu().double() * gr.abs()).sum((1, 2)) + (e.abs() * grad.abs()).sum((1, 2))
        # (a pair's error is of its larger element's size: at most both sizes, 2 more)
        assert ((change - (e * grad).sum((1, 2))).abs() <= 4 * 2.0 ** -20 * size).all()


def test_strides_broadcast_and_in_place(torch_cuda):
    import paper_2403_09636_amd as P
    hq, hkv, d, T = 4, 2, 128, 37
    rot, f = _rotation(P, hq, hkv, d, "bf16", 128, "halves")
    g = torch.Generator().manual_seed(8)
    x = torch.randn(T, hq + 2 * hkv, d + 8, generator=g).bfloat16()
    pos = torch.randint(0, 500, (T,), generator=g).int()
    X = x.cuda()
    view = [X[:, :hq, :d], X[:, hq:hq + hkv, :d]]
    want = [R.turn(v.cpu(), pos, f, 128, "halves") for v in view]
    for out, w in zip(rot.forward(*view, pos.cuda()), want):
        R.close(out, *w, "views")
    rot.forward(*view, pos.cuda(), q_out=view[0], k_out=view[1])   # in place
    for v, w in zip(view, want):
        R.close(v, *w, "in place")
    assert torch.equal(X[:, hq + hkv:].cpu(), x[:, hq + hkv:]) and torch.equal(X[..., d:].cpu(), x[..., d:])
    one = torch.randn(1, 1, d, generator=g).bfloat16()
    qo, ko = rot.forward(one.cuda().expand(T, hq, d), one.cuda().expand(T, hkv, d), pos.cuda())
    R.close(qo, *R.turn(one.expand(T, hq, d), pos, f, 128, "halves"), "broadcast")
    R.close(ko, *R.turn(one.expand(T, hkv, d), pos, f, 128, "halves"), "broadcast")


def test_many_tokens_in_groups(torch_cuda):
    """Enough tokens that a workgroup takes four, the last group not full."""
    import paper_2403_09636_amd as P
    rot, f = _rotation(P, 32, 32, 128, "bf16", 128, "adjacent")
    T = 4099
    q, k = (torch.randn(T, 32, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 7
    qo, ko = rot.forward(q, k, pos)
    for t in (0, 1, 2, 3, 4, 2047, 4095, 4096, 4097, 4098):
        s = slice(t, t + 1)
        R.close(qo[s], *R.turn(q[s].cpu(), pos[s].cpu(), f, 128, "adjacent"), f"q of token {t}")
        R.close(ko[s], *R.turn(k[s].cpu(), pos[s].cpu(), f, 128, "adjacent"), f"k of token {t}")
    back = rot.backward(qo, ko, pos)   # there and back: two roundings of at most 2^-8 of the pair's size
    for x, y in ((q, back[0]), (k, back[1])):
        pair = x.float().unflatten(-1, (64, 2)).norm(dim=-1, keepdim=True).expand(-1, -1, -1, 2).flatten(-2)
        assert ((x.float() - y.float()).abs() <= 3.0 * 2.0 ** -8 * pair).all()


class Case:
    """A full cache of 64-bit and GPU sides for appends."""

    def __init__(self, P, lens, held, hq=4, hkv=2, d=64, dtype="bf16", page=16, r=64, pairs="halves", width=None, seed=1,
                 tail=0, packed=True):
        self.g = torch.Generator().manual_seed(seed)
        self.lens, self.held, self.page, self.r, self.pairs = lens, held, page, r, pairs
        need = [-(-(max(n, 0) + m) // page) for n, m in zip(held, lens)]
        width = max(max(need), 1) if width is None else width
        self.f = R.inv_freqs(r) if r else None
        cfg = P.make_full_config(len(lens), hq, hkv, d, dtype, page_size=page, max_pages=width, num_pages=sum(need) + 3,
                                 rotary_dim=r, pairs=pairs)
        T = sum(lens) + tail
        self.full = P.DMCFull(cfg, max_tokens=T, max_chunk=max(max(lens), 1), inv_freq=None if not r else self.f.cuda(), num_layers=2)
        self.table = R.fill_tables(self.full, [min(n, width) for n in need], self.g, spare=1)
        self.full.lengths.copy_(torch.tensor(held, dtype=torch.int32))
        dt = DT[dtype]
        self.pools = [torch.randn(2, cfg.num_pages, hkv, page, d, generator=self.g).to(dt) for _ in range(2)]
        self.full.k_pages.copy_(self.pools[0])
        self.full.v_pages.copy_(self.pools[1])
        self.q, self.k, self.v = (torch.randn(T, h, d, generator=self.g).to(dt) for h in (hq, hkv, hkv))
        cu = [0]
        for m in lens:
            cu.append(cu[-1] + m)
        self.cu = cu
        self.cu_dev = torch.tensor(cu, dtype=torch.int32, device="cuda") if packed else None

    def run(self, queries=True, layer=1):
        q_out = torch.full(self.q.shape, 7.0, dtype=self.q.dtype, device="cuda")
        kw = dict(q=self.q.cuda(), q_out=q_out) if queries else {}
        self.full.append(layer, self.k.cuda(), self.v.cuda(), cu_seqlens=self.cu_dev, **kw)
        self.compare(q_out if queries else None, layer)

    def compare(self, q_out, layer, bad_pages=()):
        K, V = self.pools[0].double(), self.pools[1].double()
        off = torch.zeros_like(K)
        q_want, q_off = torch.full(self.q.shape, 7.0, dtype=torch.float64), torch.zeros(self.q.shape, dtype=torch.float64)
        capacity = self.full.cfg.max_pages * self.page
        for b, (n, m) in enumerate(zip(self.held, self.lens)):
            s = slice(self.cu[b], self.cu[b] + m)
            pos = n + torch.arange(m)
            kt, ko = R.turn(self.k[s], pos, self.f, self.r, self.pairs)
            qt, qo = R.turn(self.q[s], pos, self.f, self.r, self.pairs)
            for i in range(m):
                p = n + i
                if n < 0 or p >= capacity:
                    q_want[s.start + i] = 0
                    continue
                q_want[s.start + i], q_off[s.start + i] = qt[i], qo[i]
                at = int(self.table[b, p // self.page])
                if not 0 <= at < self.full.cfg.num_pages:
                    continue
                K[layer, at, :, p % self.page], off[layer, at, :, p % self.page] = kt[i], ko[i]
                V[layer, at, :, p % self.page] = self.v[s.start + i].double()
        R.close(self.full.k_pages, K, off, "keys")
        R.close(self.full.v_pages, V, torch.zeros_like(V), "values")
        if q_out is not None:
            R.close(q_out, q_want, q_off, "queries")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,r,pairs", [(64, 64, "halves"), (128, 64, "adjacent"), (128, 128, "halves"), (64, 0, "halves")])
@pytest.mark.parametrize("page", [8, 32, 128])
def test_append_packed_rows(torch_cuda, dtype, d, r, pairs, page):
    import paper_2403_09636_amd as P
    c = Case(P, [3, 0, 1, 40, 0, 17], [0, 5, 31, 7, 0, 100], d=d, r=r, pairs=pairs, dtype=dtype, page=page, tail=2)
    c.run()
    c.full.check()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 1), (9, 3), (64, 8)])
@pytest.mark.parametrize("queries", [True, False])
def test_append_one_token_per_row(torch_cuda, hq, hkv, queries):
    import paper_2403_09636_amd as P
    held = [0, 1, 31, 32, 33, -1, 200, 7]
    c = Case(P, [1] * len(held), held, hq=hq, hkv=hkv, d=128, r=128, page=32, packed=False)
    c.run(queries)
    c.full.check()


def test_append_many_rows_and_tokens(torch_cuda):
    """More rows than lanes (two steps of the row search), rows without tokens among them, and enough tokens for
    groups of four."""
    import paper_2403_09636_amd as P
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 60, (150,), generator=g).tolist()
    held = torch.randint(-1, 40, (150,), generator=g).tolist()
    c = Case(P, lens, held, hq=2, hkv=1, d=64, r=32, page=16, tail=3, seed=4)
    c.run()
    big = Case(P, [1500, 0, 2700], [3, 0, 1], hq=28, hkv=2, d=128, r=128, page=64, seed=5)
    big.run()


def test_append_where_there_is_no_room(torch_cuda):
    import paper_2403_09636_amd as P
    c = Case(P, [4, 6, 2, 3], [30, 10, 32, 0], width=2, page=16)   # row 0 has room for 2, row 2 for none
    c.run()
    assert int(c.full.flags) == 2
    with pytest.raises(P.DMCError, match="row is full"):
        c.full.check()


def test_append_to_pages_that_do_not_exist(torch_cuda):
    import paper_2403_09636_amd as P
    c = Case(P, [20, 20, 20], [0, 0, 0], page=16, r=0)
    c.table[0, 1], c.table[1, 0], c.table[2, 1] = -5, c.full.cfg.num_pages, 2 ** 31 - 1
    c.full.page_table.copy_(c.table)
    c.run()
    assert int(c.full.flags) == 8
    with pytest.raises(P.DMCError, match="outside the pool"):
        c.full.check()


def test_bad_boundaries_and_lengths_raise_the_flag(torch_cuda):
    import paper_2403_09636_amd as P
    for cu, held in (([0, 3, 2, 6], [0, 0, 0]), ([0, 3, 5, 900], [0, 0, 0]), ([-4, 3, 5, 6], [0, 0, 0]), ([0, 2, 4, 6], [0, 2 ** 31 - 1, 0])):
        c = Case(P, [2, 2, 2], [0, 0, 0], page=16, r=64)
        c.cu_dev.copy_(torch.tensor(cu, dtype=torch.int32))
        c.full.lengths.copy_(torch.tensor(held, dtype=torch.int32))
        c.full.append(0, c.k.cuda(), c.v.cuda(), q=c.q.cuda(), cu_seqlens=c.cu_dev)
        assert int(c.full.flags) & 4, (cu, held)
        assert torch.equal(c.full.k_pages[1].cpu(), c.pools[0][1])   # nothing outside the layer


def test_append_in_place_queries_and_views(torch_cuda):
    import paper_2403_09636_amd as P
    c = Case(P, [5, 9], [2, 0], hq=4, hkv=2, d=128, r=128, page=8)
    x = torch.cat([c.q, c.k, c.v], 1).cuda()   # views of one projection
    q = x[:, :4]
    got = c.full.append(1, x[:, 4:6], x[:, 6:], q=q, q_out=q, cu_seqlens=c.cu_dev)
    assert got is q
    c.compare(q, 1)
