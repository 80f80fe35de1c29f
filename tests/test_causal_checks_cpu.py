"""Refusals of the causal attention calls, without a GPU: the binding's tensor checks (shapes, types,
layouts, overlap, device) and the C ABI's own (configuration, counts, pointers, strides, workspace),
all before any HIP call."""
import ctypes

import pytest
import torch

import paper_2403_09636_amd as P
from paper_2403_09636_amd import binding as Bd

DEV = torch.device("cuda", 0)
T, HQ, HKV, D = 6, 4, 2, 64
BF = torch.bfloat16


def _args(backward=True):
    a = dict(q=torch.zeros(T, HQ, D, dtype=BF), k=torch.zeros(T, HKV, D, dtype=BF),
             v=torch.zeros(T, HKV, D, dtype=BF), cu_seqlens=torch.zeros(3, dtype=torch.int32),
             out=torch.zeros(T, HQ, D, dtype=BF), lse=torch.zeros(T, HQ))
    if backward:
        a.update(dout=torch.zeros(T, HQ, D, dtype=BF), dq=torch.zeros(T, HQ, D, dtype=BF),
                 dk=torch.zeros(T, HKV, D, dtype=BF), dv=torch.zeros(T, HKV, D, dtype=BF))
    return a


def _raises(fn, msg):
    with pytest.raises(P.DMCError) as e:
        fn()
    assert msg in str(e.value), str(e.value)


def _check(a):
    Bd.check_causal_args(P.make_causal_config(HQ, HKV, D), DEV, **a)


def test_valid_arguments_fail_on_the_device_only():
    _raises(lambda: _check(_args()), "is on cpu")
    _raises(lambda: _check(_args(False)), "is on cpu")


@pytest.mark.parametrize("name,bad,msg", [
    ("q", torch.zeros(T, HQ, D), "dtype"), ("k", torch.zeros(T + 1, HKV, D, dtype=BF), "shape"),
    ("v", torch.zeros(T, HQ, D, dtype=BF), "shape"), ("dout", torch.zeros(T, HQ, D // 2, dtype=BF), "shape"),
    ("out", torch.zeros(T, D, HQ, dtype=BF).transpose(1, 2), "contiguous last dimension"),
    ("q", torch.zeros(T, HQ, D + 4, dtype=BF)[..., :D], "multiples of 8"),
    ("k", torch.zeros(T * HKV * D + 8, dtype=BF)[1:1 + T * HKV * D].view(T, HKV, D), "aligned"),
    ("cu_seqlens", torch.zeros(3, dtype=torch.int64), "dtype"), ("cu_seqlens", torch.zeros(2, 3, dtype=torch.int32), "shape"),
    ("cu_seqlens", torch.zeros(0, dtype=torch.int32), "empty"),
    ("cu_seqlens", torch.zeros(6, dtype=torch.int32)[::2], "contiguous"),
    ("lse", torch.zeros(T, HQ, dtype=BF), "dtype"), ("lse", torch.zeros(HQ, T), "shape"),
    ("dk", torch.zeros(T, HQ, D, dtype=BF), "shape"),
])
def test_tensor_rejections(name, bad, msg):
    a = _args()
    a[name] = bad
    _raises(lambda: _check(a), msg)


@pytest.mark.parametrize("first,second", [("dq", "q"), ("dk", "v"), ("dv", "dk"), ("dq", "out"), ("dq", "dout")])
def test_outputs_that_share_memory(first, second):
    a = _args()
    a[second] = a[second][:, :HKV] if first in ("dk", "dv") else a[second]
    a[first] = a[second]
    _raises(lambda: _check(a), "overlaps")


def test_interleaved_views_of_one_buffer_are_apart():
    a = _args()
    buf = torch.zeros(T, HQ + 2 * HKV, D, dtype=BF)
    a["dq"], a["dk"], a["dv"] = buf[:, :HQ], buf[:, HQ:HQ + HKV], buf[:, HQ + HKV:]
    _raises(lambda: _check(a), "is on cpu")
    a["dk"] = buf[:, HQ - 1:HQ - 1 + HKV]
    _raises(lambda: _check(a), "dk overlaps dq")
    x = torch.zeros(2 * T, HQ, D, dtype=BF)
    a["dq"], a["q"] = x[:T], x[T - 1:2 * T - 1]
    _raises(lambda: _check(a), "dq overlaps q")


def _call(backward, cfg=None, ptr=4096, ws=1 << 14, ws_bytes=1 << 30, total=T, seqs=2, cu=4096, lse=4096, **strides):
    """The C entry with made-up addresses, refused before anything is read."""
    cfg = cfg or P.make_causal_config(HQ, HKV, D)
    names = ["q", "k", "v", "out"] + (["dout", "dq", "dk", "dv"] if backward else [])
    heads = dict(q=HQ, out=HQ, dout=HQ, dq=HQ)
    st = {n: (ctypes.c_int64 * 2)(*strides.get(n, (heads.get(n, HKV) * D, D))) for n in names}
    p = {n: ctypes.c_void_p(ptr) for n in names}
    head = [ctypes.byref(cfg), *(x for n in ("q", "k", "v") for x in (p[n], st[n])), cu, seqs, total,
            p["out"], st["out"], lse]
    if not backward:
        return Bd.lib.dmc_causal_forward(*head, ws, ws_bytes, None)
    return Bd.lib.dmc_causal_backward(*head, *(x for n in ("dout", "dq", "dk", "dv") for x in (p[n], st[n])),
                                      ws, ws_bytes, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw,status,msg", [
    (dict(cfg=P.make_causal_config(3, 2, 64)), 1, "multiple"), (dict(cfg=P.make_causal_config(0, 1, 64)), 1, "head counts"),
    (dict(cfg=P.make_causal_config(4, 2, 96)), 2, "head_dim"), (dict(cfg=P.CausalConfig(4, 2, 64, 7)), 1, "dtype"),
    (dict(cfg=P.make_causal_config(8192, 2, 64)), 2, "4096"),
    (dict(total=-1), 1, "counts"), (dict(seqs=-1), 1, "counts"), (dict(total=1 << 29), 2, "tokens"),
    (dict(ptr=None), 1, "non-NULL"), (dict(ptr=4104), 1, "aligned"), (dict(q=(-8, 64)), 1, "non-negative"),
    (dict(k=(HKV * D + 4, D)), 1, "multiples of 8"), (dict(v=(1 << 24, D)), 2, "32 MiB"),
    (dict(k=(HKV * D, 1 << 60)), 1, "address space"), (dict(cu=None), 1, "cu_seqlens"), (dict(lse=None), 1, "lse"),
    (dict(seqs=1 << 28, total=1 << 28, cfg=P.make_causal_config(64, 1, 64), q=(4096, 64), out=(4096, 64), dout=(4096, 64),
          dq=(4096, 64), k=(64, 64), v=(64, 64), dk=(64, 64), dv=(64, 64), ws_bytes=1 << 60), 2, "one launch"),
])
def test_c_refusals(backward, kw, status, msg):
    assert _call(backward, **kw) == status
    assert msg in Bd.last_error()


@pytest.mark.parametrize("strides", [(HQ * D, 0), (0, D), (HQ * D - 8, D), (D, T * D - 8), (64, 64)])
def test_output_rows_that_overlap(strides):
    assert _call(False, out=strides) == 1 and "overlap" in Bd.last_error()
    assert _call(True, dq=strides) == 1 and "overlap" in Bd.last_error()


def test_workspace_refusals():
    n = Bd.lib.dmc_causal_workspace_bytes(ctypes.byref(P.make_causal_config(HQ, HKV, D)), T)
    assert n >= HQ * T * 8
    for backward in (False, True):
        assert _call(backward, ws=None) == 1 and "workspace" in Bd.last_error()
        assert _call(backward, ws=4096 + 16) == 1 and "256-byte" in Bd.last_error()
        assert _call(backward, ws_bytes=n - 1) == 1 and "workspace has" in Bd.last_error()
    assert Bd.lib.dmc_causal_workspace_bytes(ctypes.byref(P.make_causal_config(3, 2, 64)), T) == 0
    assert Bd.lib.dmc_causal_workspace_bytes(ctypes.byref(P.make_causal_config(4, 2, 64)), -1) == 0


@pytest.mark.parametrize("backward", [False, True])
def test_nothing_to_do_reads_nothing(backward):
    assert _call(backward, total=0, ptr=None, cu=None, lse=None) == 0
    assert _call(backward, seqs=0, ptr=None, cu=None, lse=None) == 0


def test_config_struct_matches_header():
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "dmc.h")).read()
    body = re.search(r"typedef struct dmc_causal_config \{(.*?)\} dmc_causal_config;", text, re.S)
    names = re.findall(r"^\s*int32_t\s+([a-z_]+);", body.group(1), re.M)
    assert names == [f[0] for f in P.CausalConfig._fields_]


def test_one_pass_checks_agree_with_the_full_ones():
    """_PackedCall accepts what check_causal_args accepts (on its device) and returns its addresses;
    whatever it declines goes to the full check."""
    call = Bd._PackedCall(BF, torch.device("cpu"), D, 2)

    def quick(a):
        ins = [(a["q"], HQ), (a["k"], HKV), (a["v"], HKV), (a["out"], HQ), (a["dout"], HQ)]
        return call.tensors(T, ins, [(a["dq"], HQ), (a["dk"], HKV), (a["dv"], HKV)])
    a = _args()
    ptrs, st = quick(a)
    assert ptrs[0] == a["q"].data_ptr() and ptrs[-1] == a["dv"].data_ptr()
    assert list(st) == [HQ * D, D, HKV * D, D, HKV * D, D] + [HQ * D, D] * 3 + [HKV * D, D] * 2
    x = torch.zeros(T, HQ + 2 * HKV, D, dtype=BF)
    a["q"], a["k"], a["v"] = x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]
    assert quick(a) is not None
    for name, bad in (("q", torch.zeros(T, HQ, D)), ("k", torch.zeros(T, HQ, D, dtype=BF)),
                      ("v", torch.zeros(T, HKV, D + 4, dtype=BF)[..., :D]), ("dq", a["q"]), ("dk", a["v"]),
                      ("dout", torch.zeros(T, D, HQ, dtype=BF).transpose(1, 2)), ("dv", a["dk"]), ("out", None),
                      ("k", torch.zeros(T * HKV * D + 8, dtype=BF)[1:1 + T * HKV * D].view(T, HKV, D))):
        assert quick(dict(a, **{name: bad})) is None, name
    assert call.array(a["lse"], call.f32, (T, HQ)) == a["lse"].data_ptr()
    assert call.array(a["lse"], call.f32, (HQ, T)) is None and call.array(a["lse"], call.i32, (T, HQ)) is None
    assert call.array(a["lse"].t(), call.f32, (HQ, T)) is None and call.array(3, call.f32, ()) is None
    assert call.array(a["cu_seqlens"], call.i32) and call.array(a["lse"], call.f32) is None
    assert call.array(a["cu_seqlens"][:0], call.i32) is None and call.rows([1, 2]) == 0
