"""Chunks of new tokens on a paged cache (dmc_chunk_attend, dmc_chunk_append) against a float64
token-by-token reference: outputs and slots within bounds derived from the arithmetic
(chunk_reference), slot indexes and lengths exact; and together with prompts and decode steps."""
import math

import numpy as np
import pytest
import torch

from tests.chunk_reference import Reference
from tests.gpu_helpers import f64, log
from tests.packed_reference import cu_of, dtype_of
from workloads import decision_logits

pytestmark = pytest.mark.gpu


class Case:
    """A cache with given slots per unit and the reference on the same stored values."""

    def __init__(self, hq, hkv, d, dtype, slots, page=32, extra=256, num_pages=None, bias=0.0, omega="lead",
                 shared=False, max_tokens=700, max_chunk=None, seed=0, layers=1, layer=0):
        import paper_2403_09636_amd as P
        self.P, self.rng = P, np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.dtype, self.bias = hq, hkv, d, dtype, bias
        self.layer = layer
        slots = np.array(slots)
        B, most = slots.shape[0], max(1, int(slots.max()))
        cfg = P.make_config(layers, B, hq, hkv, d, dtype, page, most + extra, num_pages, bias, omega,
                            max_prompt_len=min(512, most + extra),
                            decision_src="shared_layer" if shared else "per_head")
        self.cache = P.DMCCache(cfg)
        # whatever the pages hold where nothing was written: NaN
        pool = cfg.num_pages * 2 * page * d * (4 if dtype == "fp32" else 2)
        at = self.cache._ws_ptr - self.cache.workspace.data_ptr()
        self.cache.workspace[at:at + pool].fill_(0xFF)
        K, V = (torch.from_numpy(self.rng.standard_normal((B, hkv, most, d), dtype=np.float32)).to(dtype_of(dtype))
                for _ in range(2))
        K[..., 0] = 0
        z = torch.from_numpy(self.rng.uniform(0.2, 3.0, (B, hkv)).astype(np.float32)) * torch.from_numpy(slots > 0)
        if most:
            self.cache.import_(layer, K.cuda(), V.cuda(), torch.from_numpy(slots).int().cuda(), z.cuda())
        self.ref = Reference(f64(K), f64(V), slots, f64(z), hq, bias, omega, shared, dtype)
        self.chunk = P.DMCChunk(self.cache, max_tokens, max_chunk)

    def tokens(self, lens, cr=2.0, tail=0, fused=False):
        T = sum(lens) + tail
        cr = np.broadcast_to(np.asarray(cr, float), (self.hkv,))
        x = self.rng.standard_normal((T, self.hq + 2 * self.hkv, self.d), dtype=np.float32)
        x[:, self.hq:self.hq + self.hkv, 0] = decision_logits(self.rng.uniform(size=(T, self.hkv)), cr[None], self.bias)
        x = torch.from_numpy(x).to(dtype_of(self.dtype)).cuda()
        q, k, v = x[:, :self.hq], x[:, self.hq:self.hq + self.hkv], x[:, self.hq + self.hkv:]
        return (q, k, v) if fused else (q.contiguous(), k.contiguous(), v.contiguous())

    def attend(self, q, k, v, lens, rows=None):
        """The chunk's attention on both sides; the cache must stay as it is."""
        L = self.cache.lengths(self.layer).clone()
        out = torch.full((q.shape[0], self.hq, self.d), 5.0, dtype=q.dtype, device="cuda")
        self.chunk.attend(self.layer, q, k, v, cu_of(lens).cuda(), out=out)
        want, bound, _ = self.ref.chunk(f64(q), f64(k), f64(v), lens)
        n = sum(lens)
        assert (out[n:] == 5.0).all(), "rows behind the last chunk were written"
        err = np.abs(f64(out[:n]) - want[:n])
        bad = ~(err <= bound[:n])
        assert not bad.any(), f"{bad.sum()} of {bad.size} outside; worst {np.nanmax(err / bound[:n]):.2f} of its bound"
        assert torch.equal(self.cache.lengths(self.layer), L)
        return float((err / bound[:n]).max()) if n else 0.0

    def append(self, q, k, v, lens, accepted=None, check=True):
        slot = torch.full((q.shape[0], self.hkv), -9, dtype=torch.int32, device="cuda")
        acc = None if accepted is None else torch.tensor(accepted, dtype=torch.int32, device="cuda")
        self.chunk.append(self.layer, k, v, q, cu_of(lens).cuda(), accepted=acc, slot_index=slot)
        _, _, want = self.ref.chunk(f64(q), f64(k), f64(v), lens, commit=lens if accepted is None else accepted,
                                    attend=False)
        n = sum(lens)
        got = slot.cpu().numpy()
        assert (got[:n] == want[:n]).all(), "slot indexes"
        assert (got[n:] == -9).all()
        if check:
            self.ref.check_cache(self.cache, self.layer)


SHAPES = [
    # hq, hkv, d, slots per unit [B][hkv], chunk lengths, compression of the chunk
    (1, 1, 64, [[0]], [1], 2.0),
    (2, 1, 64, [[1]], [1], 8.0),
    (4, 4, 64, [[5, 33, 0, 64], [0, 0, 0, 0], [31, 32, 1, 100]], [3, 0, 7], [1, 2, 4, 8]),
    (8, 2, 128, [[40, 77], [200, 3]], [5, 8], 2.0),
    (8, 1, 128, [[300]], [4], 2.0),
    (4, 2, 64, [[17, 90]], [64], 4.0),
    (4, 2, 128, [[17, 90], [0, 250], [64, 1]], [65, 128, 33], [1, 30]),
    (8, 2, 64, [[130, 12]], [150], 1.0),
    (8, 1, 64, [[0], [95]], [200, 20], 1000.0),
    (2, 2, 128, [[700, 10]], [40], [3, 3]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("page", [8, 32, 64])
@pytest.mark.parametrize("hq,hkv,d,slots,lens,cr", SHAPES)
def test_attend_and_append(torch_cuda, dtype, page, hq, hkv, d, slots, lens, cr):
    log(f"{dtype} page {page} heads {hq}/{hkv} d {d} lens {lens}")
    c = Case(hq, hkv, d, dtype, slots, page, max_chunk=max(lens))
    x = c.tokens(lens, cr, tail=len(lens) - 1, fused=page == 32)
    worst = c.attend(*x, lens)
    c.append(*x, lens)
    c.ref.restart(c.cache, c.layer)
    y = c.tokens(lens, cr)
    log(f"worst {worst:.3f}, after the append {c.attend(*y, lens):.3f} of the bound")
    c.cache.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("omega,shared,bias", [("lead", True, 0.0), ("group_mean", False, 1.5), ("uniform", False, -0.5),
                                               ("group_mean", True, 0.0)])
@pytest.mark.parametrize("lens", [[6, 3], [70, 90]])
def test_variants(torch_cuda, dtype, omega, shared, bias, lens):
    c = Case(8, 2, 64, dtype, [[40, 40], [9, 9]], bias=bias, omega=omega, shared=shared)
    x = c.tokens(lens, 3.0)
    c.attend(*x, lens)
    c.append(*x, lens)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,chunk", [(1, 1, 2), (8, 1, 3), (8, 2, 40), (4, 1, 90)])
def test_long_caches_in_pieces(torch_cuda, dtype, hq, hkv, chunk):
    """Few units of long caches: a tile's blocks go to many workgroups that meet in the combine pass."""
    c = Case(hq, hkv, 64, dtype, [[5000] + [700] * (hkv - 1)])
    c.attend(*c.tokens([chunk], 2.0), [chunk])


@pytest.mark.parametrize("hq,hkv,chunk", [(8, 2, 12), (8, 2, 9), (8, 1, 16), (2, 2, 33)])
def test_few_columns_on_large_caches(torch_cuda, hq, hkv, chunk):
    """Room for 64K slots or more in the layer: more than 32 columns are one wide tile."""
    lens = [chunk, 0, chunk - 1]
    c = Case(hq, hkv, 64, "bf16", [[700] * hkv, [0] * hkv, [31] * hkv], extra=24000, max_chunk=chunk)
    x = c.tokens(lens, 2.0)
    c.attend(*x, lens)
    c.append(*x, lens)
    c.ref.restart(c.cache, c.layer)
    c.attend(*c.tokens(lens, 2.0), lens)
    c.cache.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_accepted_tokens(torch_cuda, dtype):
    """Drafts of which a part is accepted, then decode steps and further chunks: one conversation."""
    c = Case(8, 2, 128, dtype, [[60, 31], [0, 0], [100, 7], [32, 64]], max_chunk=8)
    for accepted in ([3, 1, 0, 5], [0, 8, 8, 1]):
        lens = [5, 8, 8, 5]
        x = c.tokens(lens, [1.5, 6])
        c.attend(*x, lens)
        c.append(*x, lens, accepted=accepted)
        c.ref.restart(c.cache, c.layer)
        q, k, v = c.tokens([1] * 4, [1.5, 6])
        out = c.cache.decode_step(c.layer, q, k, v)
        want, bound, _ = c.ref.chunk(f64(q), f64(k), f64(v), [1] * 4, commit=[1] * 4)
        # (the decode kernels' probabilities and scores: the bound of the same arithmetic, and their
        # product of two bf16 terms is finer)
        assert (np.abs(f64(out) - want) <= bound).all()
        c.ref.check_cache(c.cache, c.layer)
        c.ref.restart(c.cache, c.layer)
    c.cache.check()


def test_long_draft_accepted_in_part(torch_cuda):
    """Accepted counts on both sides of 64-token blocks."""
    c = Case(4, 2, 64, "bf16", [[20, 3], [0, 0], [50, 50]], max_chunk=200)
    lens = [200, 130, 129]
    x = c.tokens(lens, [2, 40])
    c.append(*x, lens, accepted=[64, 65, 128])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_packed_prompts_against_padded_ones(torch_cuda, dtype):
    """Whole prompts packed onto an empty cache: dmc_prefill_attend's outputs, slots and cache."""
    import paper_2403_09636_amd as P
    hq, hkv, d, lens = 8, 2, 64, [150, 0, 64, 301]
    c = Case(hq, hkv, d, dtype, [[0, 0]] * 4, extra=400)
    q, k, v = c.tokens(lens, [2, 5])
    out = c.chunk.attend(0, q, k, v, cu_of(lens).cuda())
    c.append(q, k, v, lens)
    other = P.DMCCache(c.cache.cfg)
    pad = [torch.zeros(4, 301, t.shape[1], d, dtype=t.dtype, device="cuda") for t in (q, k, v)]
    for x, t in zip(pad, (q, k, v)):
        for b, (lo, n) in enumerate(zip(cu_of(lens), lens)):
            x[b, :n] = t[lo:lo + n]
    ref = other.prefill_attend(0, pad[1], pad[2], pad[0], prompt_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    want = torch.cat([ref[b, :n] for b, n in enumerate(lens)])
    _, bound, _ = Reference(*(np.zeros((4, hkv, 0, d)),) * 2, np.zeros((4, hkv), int), np.zeros((4, hkv)), hq,
                            dtype=dtype).chunk(f64(q), f64(k), f64(v), lens)
    assert (np.abs(f64(out) - f64(want)) <= 2 * bound).all()
    assert torch.equal(c.cache.lengths(0), other.lengths(0))
    c.cache.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("at", [0, 11, 39])
def test_non_finite_tokens(torch_cuda, dtype, bad, at):
    """A token of NaN or infinity (k past element 0, v, q) reaches the outputs from its own on that see its
    slot, and no output before it, no other row; a value alone reaches its element only."""
    for hq, hkv in ((4, 4), (8, 2)):
        lens = [40, 10]
        c = Case(hq, hkv, 64, dtype, [[50] * hkv, [3] * hkv])
        q, k, v = c.tokens(lens, 2.0)
        clean = [t.clone() for t in (q, k, v)]
        k[at, :, 1:], v[at], q[at, :, 1:] = bad, bad, bad
        out = c.chunk.attend(0, q, k, v, cu_of(lens).cuda())
        want, bound, _ = c.ref.chunk(*(f64(t) for t in clean), lens)
        ok = np.ones(50, bool)
        ok[at:40] = False
        assert (np.abs(f64(out) - want)[ok] <= bound[ok]).all()
        assert not out[at].isfinite().any()
        # a value element alone
        v2 = clean[2].clone()
        v2[at, :, 5] = math.inf
        out = f64(c.chunk.attend(0, *clean[:2], v2, cu_of(lens).cuda()))
        rest = [e for e in range(64) if e != 5]
        assert (np.abs(out - want)[..., rest] <= bound[..., rest]).all()
        assert (np.abs(out - want)[ok] <= bound[ok]).all()
        assert (out[at:40, :, 5] == math.inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("slots", [0, 50])
@pytest.mark.parametrize("lens,most", [([6], 6), ([6], 40), ([40], 40), ([1], 40)])
def test_a_token_whose_own_score_is_not_finite(torch_cuda, dtype, bad, slots, lens, most):
    """A score of NaN or +infinity on the token's own state makes its whole row NaN, as a softmax does, also
    where nothing else is visible; k and v are finite, so no other row changes."""
    c = Case(8, 2, 64, dtype, [[slots] * 2], max_chunk=most)
    q, k, v = c.tokens(lens, 2.0)
    k[0, :, 1] = 1.0
    want, bound, _ = c.ref.chunk(f64(q), f64(k), f64(v), lens)
    # an empty cache: the first token's state is its own k, so that the score has the infinity's sign
    q[0, :, 1] = bad
    out = f64(c.chunk.attend(0, q, k, v, cu_of(lens).cuda()))
    assert np.isnan(out[0]).all()
    assert (np.abs(out - want)[1:] <= bound[1:]).all()


def test_no_room(torch_cuda):
    """A unit without slots or pages for its chunk keeps its cache; others take theirs."""
    P = torch_cuda and __import__("paper_2403_09636_amd")
    for lens in ([10, 10], [70, 10]):
        # unit (0, 0) at capacity
        c = Case(2, 2, 64, "bf16", [[20, 4], [3, 3]], extra=max(lens) - 2)
        q, k, v = c.tokens(lens, 1.0)
        k[..., 0] = -1   # every token opens a slot
        slot = torch.zeros(sum(lens), 2, dtype=torch.int32, device="cuda")
        before = c.cache.export(0)
        c.chunk.append(0, k, v, q, cu_of(lens).cuda(), slot_index=slot)
        n = lens[0]
        assert c.cache.lengths(0).tolist() == [[20, 4 + n], [13, 13]]
        assert (slot[:n, 0] == -1).all() and slot[:n, 1].tolist() == list(range(4, 4 + n))
        after = c.cache.export(0)
        for a, b in zip(before[:2], after[:2]):
            assert torch.equal(a[0, 0], b[0, 0]) and torch.equal(a[1, 0, :3], b[1, 0, :3])
        with pytest.raises(P.DMCError) as e:
            c.cache.check()
        assert e.value.status == 3
    # the pool: 4 pages for the four units, one to spare; two need one each
    c = Case(2, 2, 64, "bf16", [[30, 30], [3, 3]], num_pages=5)
    lens = [4, 4]
    q, k, v = c.tokens(lens)
    k[..., 0] = -1
    c.chunk.append(0, k, v, q, cu_of(lens).cuda())
    L = c.cache.lengths(0).tolist()
    assert sorted(L[0]) == [30, 34] and L[1] == [7, 7]
    assert c.cache.status() == 3


@pytest.mark.parametrize("what", ["longer", "range", "decreasing", "accepted"])
def test_bad_lengths_raise_the_flag(torch_cuda, what):
    """Lengths that the host cannot see: clamped, flagged, nothing out of range."""
    c = Case(4, 2, 64, "bf16", [[20, 20], [9, 9]], max_chunk=16)
    T = 40
    q, k, v = c.tokens([T])
    cu = dict(longer=[0, 30, 40], range=[-3, 12, 99], decreasing=[0, 12, 5], accepted=[0, 10, 20])[what]
    cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
    acc = torch.tensor([11, -1], dtype=torch.int32, device="cuda") if what == "accepted" else None
    out = torch.full((T, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    if what != "accepted":
        c.chunk.attend(0, q, k, v, cu, out=out)
        assert c.cache.status() == 1
        if what == "longer":   # the first 16 tokens of the row as if it ended there
            want, bound, _ = c.ref.chunk(f64(q[:16]), f64(k[:16]), f64(v[:16]), [16, 0])
            assert (np.abs(f64(out[:16]) - want) <= bound).all() and (out[16:30] == 5.0).all()
    c.chunk.append(0, k, v, q, cu, accepted=acc)
    assert c.cache.status() == 1
    if what == "accepted":
        want = c.ref.chunk(f64(q), f64(k), f64(v), [10, 10], commit=[10, 0], attend=False)
        c.ref.check_cache(c.cache)


def test_layers_strides_and_views(torch_cuda):
    """A later layer, head-major and broadcast inputs, outputs in a larger buffer; importance from q[..., 0]."""
    c = Case(4, 2, 64, "bf16", [[70, 5], [12, 40]], layers=3, layer=2)
    lens = [9, 80]
    q, k, v = c.tokens(lens, 2.0)
    k, v = k[:, :1].contiguous().expand(-1, 2, -1), v[:, :1].contiguous().expand(-1, 2, -1)
    q = q.transpose(0, 1).contiguous().transpose(0, 1)
    buf = torch.full((89, 7, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    c.chunk.attend(2, q, k, v, cu_of(lens).cuda(), out=buf[:, 1:5])
    want, bound, _ = c.ref.chunk(f64(q), f64(k), f64(v), lens)
    assert (np.abs(f64(buf[:, 1:5]) - want) <= bound).all()
    assert (buf[:, 0] == 3.0).all() and (buf[:, 5:] == 3.0).all()
    slot = torch.empty(89, 2, dtype=torch.int32, device="cuda")
    c.chunk.append(2, k, v, q[..., 0], cu_of(lens).cuda(), slot_index=slot)
    _, _, s = c.ref.chunk(f64(q), f64(k), f64(v), lens, commit=lens, attend=False)
    assert (slot.cpu().numpy() == s).all()
    c.ref.check_cache(c.cache, 2)
    assert c.cache.lengths(0).sum() == 0 and c.cache.lengths(1).sum() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_streams_and_graphs(torch_cuda, dtype):
    """Attend and append captured once and replayed: every replay continues the cache as eager calls do on
    another one, bit for bit, with eager work between; and the same from another stream."""
    lens = [5, 0, 9]
    cases = [Case(8, 2, 64, dtype, [[2000, 40], [3, 3], [0, 7]], max_chunk=9) for _ in range(2)]
    cu = cu_of(lens).cuda()
    xs = [cases[0].tokens(lens, 2.0) for _ in range(4)]
    q, k, v = (t.clone() for t in xs[0])
    outs = [torch.zeros(14, 8, 64, dtype=q.dtype, device="cuda") for _ in range(2)]

    def step(c, out, q, k, v):
        c.chunk.attend(0, q, k, v, cu, out=out)
        c.chunk.append(0, k, v, q, cu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cases[0], outs[0], q, k, v)
    torch.cuda.current_stream().wait_stream(side)
    step(cases[1], outs[1], *xs[0])
    assert torch.equal(*outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cases[0], outs[0], q, k, v)
    for x in xs[1:]:
        for a, b in zip((q, k, v), x):
            a.copy_(b)
        graph.replay()
        step(cases[1], outs[1], *x)
        torch.cuda.synchronize()
        assert torch.equal(*outs)
        for a, b in zip(cases[0].cache.export(0, 2100), cases[1].cache.export(0, 2100)):
            assert torch.equal(a, b)
    cases[0].cache.check()


def test_nothing_to_do(torch_cuda):
    c = Case(4, 2, 64, "bf16", [[5, 6]])
    for T, lens in ((0, [0]), (6, [0])):
        q, k, v = c.tokens([T])
        out = torch.ones_like(q)
        c.chunk.attend(0, q, k, v, cu_of(lens).cuda(), out=out)
        c.chunk.append(0, k, v, q, cu_of(lens).cuda())
        assert (out == 1).all() and c.cache.lengths(0).tolist() == [[5, 6]]
    c.cache.check()


def test_refusals(torch_cuda):
    """What the host can see is refused before anything is enqueued."""
    import ctypes

    import paper_2403_09636_amd as P
    from paper_2403_09636_amd import binding as Bd
    c = Case(4, 2, 64, "bf16", [[5, 6], [7, 0]], max_tokens=16)
    cfg = P.make_config(1, 2, 4, 2, 64, window=4, max_slots_per_seq=64)
    with pytest.raises(P.DMCError, match="window"):
        P.DMCChunk(P.DMCCache(cfg), 16)
    for total, chunk, msg in ((-1, 8, "total_tokens"), (8, 0, "max_chunk"), (1 << 25, 8, "tokens in a call")):
        assert Bd.lib.dmc_chunk_workspace_bytes(c.cache.handle, total, chunk) == 0 and msg in Bd.last_error()
    q, k, v = c.tokens([8, 9])
    with pytest.raises(P.DMCError, match="17 tokens"):
        c.chunk.attend(0, q, k, v, cu_of([8, 9]).cuda())
    with pytest.raises(P.DMCError, match="17 tokens"):
        c.chunk.append(0, k, v, q, cu_of([8, 9]).cuda())
    with pytest.raises(P.DMCError, match="layer"):
        c.chunk.append(1, k[:16], v[:16], q[:16], cu_of([8, 8]).cuda())

    ok = dict(layer=0, ptr=q.data_ptr(), cu=q.data_ptr(), total=8, chunk=8, ws=c.chunk._ws, nbytes=c.chunk._ws_bytes,
              qs=(256, 64), ks=(128, 64), os=(256, 64), out=q.data_ptr())

    def call(append, **kw):
        a = dict(ok, **kw)
        qs, ks, os_ = ((ctypes.c_int64 * 2)(*a[x]) for x in ("qs", "ks", "os"))
        if append:
            return Bd.lib.dmc_chunk_append(c.cache.handle, a["layer"], a["ptr"], ks, a["ptr"], ks, a["ptr"], qs, a["cu"],
                                           None, a["total"], a["chunk"], None, a["ws"], a["nbytes"], None)
        return Bd.lib.dmc_chunk_attend(c.cache.handle, a["layer"], a["ptr"], qs, a["ptr"], ks, a["ptr"], ks, a["cu"],
                                       a["total"], a["chunk"], a["out"], os_, a["ws"], a["nbytes"], None)
    for append in (False, True):
        for kw, status, msg in ((dict(layer=-1), 1, "layer"), (dict(ptr=None), 1, "non-NULL"), (dict(ptr=8), 1, "aligned"),
                                (dict(cu=None), 1, "cu_seqlens"), (dict(ks=(-8, 64)), 1, "non-negative"),
                                (dict(ks=(132, 64)), 1, "multiples"), (dict(ks=(1 << 24, 64)), 2, "32 MiB"),
                                (dict(qs=(1 << 24, 64)), 2, "32 MiB"), (dict(qs=(-8, 64)), 1, "non-negative"),
                                (dict(ws=None), 1, "workspace"), (dict(ws=16), 1, "256-byte"),
                                (dict(nbytes=256), 1, "workspace has"), (dict(chunk=0), 1, "max_chunk"),
                                (dict(total=-2), 1, "total_tokens")):
            assert call(append, **kw) == status, (append, kw, Bd.last_error())
            assert msg in Bd.last_error(), (kw, Bd.last_error())
    for kw, msg in ((dict(out=None), "out"), (dict(out=8), "aligned"), (dict(os=(256, 0)), "overlap"),
                    (dict(os=(192, 64)), "overlap")):
        assert call(False, **kw) == 1 and msg in Bd.last_error()
    torch.cuda.synchronize()
    assert c.cache.lengths(0).tolist() == [[5, 6], [7, 0]]


def test_append_alone_flags_boundaries(torch_cuda):
    for cu in ([0, 12, 5], [-1, 4, 9], [0, 4, 99]):
        c = Case(4, 2, 64, "bf16", [[20, 20], [9, 9]], max_chunk=16)
        q, k, v = c.tokens([20])
        c.chunk.append(0, k, v, q, torch.tensor(cu, dtype=torch.int32, device="cuda"))
        assert c.cache.status() == 1


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("chunk", [3, 30])
def test_many_units_are_planned(torch_cuda, dtype, chunk):
    """More than 64 units (pieces planned by their lengths), ragged, some empty, some far longer; sampled rows."""
    rng = np.random.default_rng(1)
    B, hkv = 40, 2
    slots = rng.integers(0, 60, (B, hkv))
    slots[3] = (1500, 4)
    slots[17] = 0
    lens = [int(x) for x in rng.integers(0, chunk + 1, B)]
    lens[3], lens[17] = chunk, chunk
    c = Case(4, hkv, 64, dtype, slots, max_tokens=sum(lens), max_chunk=chunk, extra=64)
    q, k, v = c.tokens(lens, 2.0)
    out = f64(c.chunk.attend(0, q, k, v, cu_of(lens).cuda()))
    c.ref.units = [c.ref.units[b] for b in (3, 17, 30)]
    lo = np.concatenate([[0], np.cumsum(lens)])
    rows = np.concatenate([np.arange(lo[b], lo[b + 1]) for b in (3, 17, 30)])
    want, bound, _ = c.ref.chunk(*(f64(t)[rows] for t in (q, k, v)), [lens[b] for b in (3, 17, 30)])
    assert (np.abs(out[rows] - want) <= bound).all()
    c.cache.check()


@pytest.mark.parametrize("dtype,hq,page", [("bf16", 4, 32), ("bf16", 16, 32), ("bf16", 8, 16), ("fp32", 8, 32)])
def test_pages_beyond_4_gb(torch_cuda, dtype, hq, page):
    """Another layer holds the pool's first 4 GB, so that this layer's pages lie past 32-bit offsets."""
    d, units = 128, 8
    slots = -(-2 ** 32 // (2 * d * (4 if dtype == "fp32" else 2)) // units) + page
    pages = units * -(-slots // page) + 64
    c = Case(hq, 4, d, dtype, [[0] * 4] * 2, page=page, extra=slots, num_pages=pages, layers=2, layer=1, max_tokens=64,
             max_chunk=4)
    full = torch.zeros((2, 4, slots, d), dtype=dtype_of(dtype), device="cuda")
    c.cache.import_(0, full, full, torch.full((2, 4), slots, dtype=torch.int32, device="cuda"),
                    torch.ones((2, 4), device="cuda"))
    del full
    assert c.cache.pages_used() * page * 2 * d * (4 if dtype == "fp32" else 2) > 2 ** 32
    narrow, wide = c.chunk, c.P.DMCChunk(c.cache, 64, 40)
    for chunk, lens in ((narrow, [4, 3]), (wide, [40, 17]), (wide, [1, 33]), (narrow, [2, 4])):
        c.chunk = chunk
        x = c.tokens(lens, 1.5)
        c.attend(*x, lens)
        c.append(*x, lens)
        c.ref.restart(c.cache, c.layer)
    c.cache.check()


def test_two_handles_at_once(torch_cuda):
    """Attention from two handles on two streams over one cache, and a handle whose bound on a row's
    tokens is far above the call's."""
    c = Case(8, 2, 64, "bf16", [[2000, 40], [300, 3], [0, 7]], max_tokens=64, max_chunk=8)
    other = c.P.DMCChunk(c.cache, 64, 2 ** 31 - 1)
    lens = [5, 8, 2]
    x, cu = c.tokens(lens, 2.0), cu_of(lens).cuda()
    want, bound, _ = c.ref.chunk(*(f64(t) for t in x), lens)
    sides = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.zeros_like(x[0]) for _ in range(4)] for _ in sides]
    torch.cuda.synchronize()
    for i in range(4):
        for side, chunk, out in zip(sides, (c.chunk, other), outs):
            chunk.attend(0, *x, cu, out=out[i], stream=side)
    torch.cuda.synchronize()
    for out in outs:
        assert (np.abs(f64(out[0]) - want) <= bound).all()
        assert all(torch.equal(o, out[0]) for o in out)


def test_closed_cache(torch_cuda):
    c = Case(4, 2, 64, "bf16", [[5, 6]], max_tokens=16)
    x = c.tokens([4])
    c.cache.close()
    for call in (lambda: c.chunk.attend(0, *x, cu_of([4]).cuda()), lambda: c.P.DMCChunk(c.cache, 16),
                 lambda: c.chunk.append(0, x[1], x[2], x[0], cu_of([4]).cuda())):
        with pytest.raises(c.P.DMCError, match="NULL"):
            call()
