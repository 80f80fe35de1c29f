"""Refusals of the rotation and full-cache calls, without a GPU: the binding's tensor checks and the C ABI's own,
all before any HIP call."""
import ctypes
import os
import re

import pytest
import torch

import paper_2403_09636_amd as P
from paper_2403_09636_amd import binding as Bd

DEV = torch.device("cuda", 0)
CPU = torch.device("cpu")
T, B, HQ, HKV, D, R = 6, 3, 4, 2, 64, 32
BF, I32 = torch.bfloat16, torch.int32


def _raises(fn, msg):
    with pytest.raises(P.DMCError) as e:
        fn()
    assert msg in str(e.value), str(e.value)


def _rotary():
    return dict(q=torch.zeros(T, HQ, D, dtype=BF), k=torch.zeros(T, HKV, D, dtype=BF), positions=torch.zeros(T, dtype=I32),
                inv_freq=torch.zeros(R // 2), q_out=torch.zeros(T, HQ, D, dtype=BF), k_out=torch.zeros(T, HKV, D, dtype=BF))


def _check_rotary(a):
    Bd.check_rotary_args(P.make_rotary_config(HQ, HKV, D, rotary_dim=R), DEV, **a)


CFG = P.make_full_config(B, HQ, HKV, D, page_size=8, max_pages=4, num_pages=12, rotary_dim=R)


def _storage():
    return dict(k_pages=torch.zeros(1, 12, HKV, 8, D, dtype=BF), v_pages=torch.zeros(1, 12, HKV, 8, D, dtype=BF),
                page_table=torch.zeros(B, 4, dtype=I32), lengths=torch.zeros(B, dtype=I32), flags=torch.zeros(1, dtype=I32),
                inv_freq=torch.zeros(R // 2))


def _append():
    return dict(storage=_storage(), k=torch.zeros(T, HKV, D, dtype=BF), v=torch.zeros(T, HKV, D, dtype=BF),
                q=torch.zeros(T, HQ, D, dtype=BF), q_out=torch.zeros(T, HQ, D, dtype=BF), cu_seqlens=torch.zeros(B + 1, dtype=I32))


def _attend():
    return dict(storage=_storage(), q=torch.zeros(T, HQ, D, dtype=BF), out=torch.zeros(T, HQ, D, dtype=BF),
                lse=torch.zeros(T, HQ), cu_seqlens=torch.zeros(B + 1, dtype=I32))


def _check_append(a):
    Bd.check_full_append_args(CFG, DEV, **a)


def _check_attend(a):
    Bd.check_full_attend_args(CFG, DEV, **a)


def test_valid_arguments_fail_on_the_device_only():
    for args, check in ((_rotary, _check_rotary), (_append, _check_append), (_attend, _check_attend)):
        _raises(lambda: check(args()), "is on cpu")
    a = _rotary()
    a["q_out"], a["k_out"] = a["q"], a["k"]   # in place
    _raises(lambda: _check_rotary(a), "is on cpu")
    a = _append()
    a["q_out"] = a["q"]
    _raises(lambda: _check_append(a), "is on cpu")
    a.update(q=None, q_out=None)
    _raises(lambda: _check_append(a), "is on cpu")
    a = _append()
    a.update(k=a["k"][:B], v=a["v"][:B], q=None, q_out=None, cu_seqlens=None)
    _raises(lambda: _check_append(a), "is on cpu")


@pytest.mark.parametrize("name,bad,msg", [
    ("q", torch.zeros(T, HQ, D), "dtype"), ("k", torch.zeros(T + 1, HKV, D, dtype=BF), "shape"),
    ("q_out", torch.zeros(T, HKV, D, dtype=BF), "shape"), ("k_out", torch.zeros(T, D, HKV, dtype=BF).transpose(1, 2), "contiguous last"),
    ("q", torch.zeros(T, HQ, D + 4, dtype=BF)[..., :D], "multiples of 8"), ("positions", torch.zeros(T, dtype=torch.int64), "dtype"),
    ("positions", torch.zeros(T - 1, dtype=I32), "shape"), ("positions", torch.zeros(2 * T, dtype=I32)[::2], "contiguous"),
    ("inv_freq", torch.zeros(R), "shape"), ("inv_freq", torch.zeros(R // 2, dtype=torch.float64), "dtype"), ("inv_freq", None, "Tensor"),
])
def test_rotation_rejections(name, bad, msg):
    a = _rotary()
    a[name] = bad
    _raises(lambda: _check_rotary(a), msg)


def test_rotation_outputs_that_share_memory():
    x = torch.zeros(T + 1, HQ, D, dtype=BF)
    for name, kw in (("q_out overlaps q", dict(q=x[:T], q_out=x[1:])), ("k_out overlaps q", dict(q=x[:T], k_out=x[:T, :HKV])),
                     ("q_out overlaps k", dict(q_out=x[:T], k=x[:T, :HKV])), ("k_out overlaps q_out", dict(q_out=x[:T], k_out=x[:T, 1:1 + HKV])),
                     ("k_out overlaps k", dict(k=x[:T, :HKV], k_out=x[:T, 1:1 + HKV]))):
        _raises(lambda: _check_rotary({**_rotary(), **kw}), name)
    a = _rotary()
    a["positions"] = a["q_out"].view(I32).view(-1)[:T]
    _raises(lambda: _check_rotary(a), "q_out overlaps positions")


@pytest.mark.parametrize("name,bad,msg", [
    ("k", torch.zeros(T, HKV, D), "dtype"), ("v", torch.zeros(T + 1, HKV, D, dtype=BF), "shape"), ("q", torch.zeros(T, HKV, D, dtype=BF), "shape"),
    ("q_out", None, "go together"), ("q", None, "go together"), ("cu_seqlens", torch.zeros(B, dtype=I32), "shape"),
    ("cu_seqlens", torch.zeros(B + 1, dtype=torch.int64), "dtype"), ("cu_seqlens", None, "one for each"),
    ("v", torch.zeros(T * HKV * D + 8, dtype=BF)[1:1 + T * HKV * D].view(T, HKV, D), "aligned"),
])
def test_append_rejections(name, bad, msg):
    a = _append()
    a[name] = bad
    _raises(lambda: _check_append(a), msg)


@pytest.mark.parametrize("name,bad,msg", [
    ("q", torch.zeros(T, HQ, D), "dtype"), ("out", torch.zeros(T, HQ, 2 * D, dtype=BF), "shape"), ("lse", torch.zeros(T, HQ, dtype=BF), "dtype"),
    ("lse", torch.zeros(HQ, T).t(), "contiguous"), ("cu_seqlens", None, "one for each"), ("cu_seqlens", torch.zeros(2 * B + 2, dtype=I32)[::2], "contiguous"),
])
def test_attend_rejections(name, bad, msg):
    a = _attend()
    a[name] = bad
    _raises(lambda: _check_attend(a), msg)


def test_outputs_that_share_memory_with_the_cache():
    a = _append()
    a["k"] = a["storage"]["k_pages"].view(-1, HKV, D)[:T]
    _raises(lambda: _check_append(a), "k_pages overlaps k")
    a = _append()
    a["q_out"] = a["storage"]["v_pages"].view(-1, HQ, D)[:T]
    _raises(lambda: _check_append(a), "q_out overlaps v_pages")
    a = _append()
    a["q_out"] = a["k"].expand(T, HKV, D).repeat(1, 2, 1)
    a["k"] = a["q_out"][:, :HKV]
    _raises(lambda: _check_append(a), "q_out overlaps k")
    a = _attend()
    a["out"] = a["q"]
    _raises(lambda: _check_attend(a), "out overlaps q")
    a = _attend()
    a["out"] = a["storage"]["k_pages"].view(-1, HQ, D)[:T]
    _raises(lambda: _check_attend(a), "out overlaps k_pages")
    a = _attend()
    a["lse"] = a["out"].view(torch.float32).view(-1)[:T * HQ].view(T, HQ)
    _raises(lambda: _check_attend(a), "lse overlaps out")


def test_objects_refuse():
    f = torch.zeros(R // 2)
    _raises(lambda: P.DMCRotation(P.make_rotary_config(HQ, HKV, D, rotary_dim=R), None, device="cpu"), "inv_freq")
    _raises(lambda: P.DMCRotation(P.make_rotary_config(HQ, HKV, D, rotary_dim=R), f, device=DEV), "is on cpu")
    _raises(lambda: P.DMCFull(CFG, inv_freq=None, device="cpu"), "inv_freq")
    _raises(lambda: P.DMCFull(CFG, max_chunk=0, inv_freq=f, device="cpu"), "max_chunk")
    _raises(lambda: P.DMCFull(CFG, num_layers=0, inv_freq=f, device="cpu"), "num_layers")
    full = P.DMCFull(CFG, max_tokens=4, max_chunk=2, inv_freq=f, num_layers=2, device="cpu")
    for name in ("k_pages", "v_pages", "page_table", "lengths", "flags"):
        with pytest.raises(AttributeError):
            setattr(full, name, None)
    q = torch.zeros(5, HQ, D, dtype=BF)
    _raises(lambda: full.attend(0, q, cu_seqlens=torch.zeros(B + 1, dtype=I32)), "the workspace holds 4")
    _raises(lambda: full.attend(0, q[:3], cu_seqlens=torch.zeros(B + 1, dtype=I32), max_chunk=3), "the workspace holds 2")
    _raises(lambda: full.attend(2, q[:3]), "layer 2")
    _raises(lambda: full.append(-1, q[:3, :HKV], q[:3, :HKV]), "layer -1")
    full.flags.fill_(4)
    _raises(full.check, "out of range")
    full.flags.fill_(6)
    _raises(full.check, "full")


def _st(h):
    return (ctypes.c_int64 * 2)(h * D, D)


def _c_rotate(cfg=None, ptr=4096, total=T, positions=4096, freq=4096, q=None, q_out=None):
    cfg = cfg or P.make_rotary_config(HQ, HKV, D, rotary_dim=R)
    p = ctypes.c_void_p(ptr)
    return Bd.lib.dmc_rotate(ctypes.byref(cfg), p, q or _st(HQ), p, _st(HKV), positions, freq, total, 0, p, q_out or _st(HQ), p,
                             _st(HKV), None)


def _c_append(cfg=CFG, ptr=4096, q=4096, total=T, cu=4096, lens=4096, table=4096, kp=4096, freq=4096, q_out=4096):
    p = ctypes.c_void_p(ptr)
    return Bd.lib.dmc_full_append(ctypes.byref(cfg), p, _st(HKV), p, _st(HKV), q, _st(HQ), freq, cu, total, lens, table, kp, kp,
                                  q_out, _st(HQ), None, None)


def _c_attend(cfg=CFG, ptr=4096, total=T, chunk=2, cu=4096, lens=4096, table=4096, kp=4096, ws=1 << 14, ws_bytes=1 << 40, out=None):
    p = ctypes.c_void_p(ptr)
    return Bd.lib.dmc_full_attend(ctypes.byref(cfg), p, _st(HQ), cu, total, chunk, lens, table, kp, kp, p, out or _st(HQ), None,
                                  None, ws, ws_bytes, None)


def _full(**kw):
    c = P.FullConfig(*(getattr(CFG, n) for n, _ in P.FullConfig._fields_))
    for n, x in kw.items():
        setattr(c, n, x)
    return c


@pytest.mark.parametrize("call", [_c_append, _c_attend])
@pytest.mark.parametrize("kw,status,msg", [
    (dict(num_q_heads=3), 1, "multiple"), (dict(num_kv_heads=0), 1, "head counts"), (dict(num_q_heads=8192), 2, "4096"),
    (dict(head_dim=96), 2, "head_dim"), (dict(dtype=5), 1, "dtype"), (dict(rotary_dim=24), 1, "rotary_dim"),
    (dict(rotary_dim=80), 1, "rotary_dim"), (dict(rotary_dim=-16), 1, "rotary_dim"), (dict(rotary_pairs=2), 1, "rotary_pairs"),
    (dict(batch=0), 1, "batch"), (dict(batch=4097), 2, "4096 rows"), (dict(max_pages=0), 1, "max_pages"), (dict(num_pages=0), 1, "num_pages"),
    (dict(page_size=12), 1, "page_size"), (dict(page_size=4), 1, "page_size"), (dict(page_size=1 << 17), 1, "page_size"),
    (dict(max_pages=1 << 28), 2, "2^30"),
])
def test_c_config_refusals(call, kw, status, msg):
    assert call(cfg=_full(**kw)) == status
    assert msg in Bd.last_error()


@pytest.mark.parametrize("call", [_c_append, _c_attend])
@pytest.mark.parametrize("kw,status,msg", [
    (dict(total=-1), 1, "total_tokens"), (dict(total=1 << 27), 2, "too many tokens"), (dict(cu=None), 1, "one for each"),
    (dict(lens=None), 1, "non-NULL"), (dict(table=None), 1, "non-NULL"), (dict(kp=None), 1, "non-NULL"), (dict(kp=4104), 1, "aligned"),
    (dict(ptr=None), 1, "non-NULL"), (dict(ptr=4104), 1, "aligned"),
])
def test_c_refusals(call, kw, status, msg):
    assert call(**kw) == status
    assert msg in Bd.last_error()


def test_c_refusals_of_one_call():
    assert _c_append(freq=None) == 1 and "inv_freq" in Bd.last_error()
    assert _c_append(q_out=None) == 1 and "q_out" in Bd.last_error()
    assert _c_attend(chunk=0) == 1 and "max_chunk" in Bd.last_error()
    assert _c_attend(chunk=1 << 25) == 2 and "too many" in Bd.last_error()
    n = Bd.lib.dmc_full_workspace_bytes(ctypes.byref(CFG), T, 2)
    assert n > 0
    assert _c_attend(ws=None) == 1 and "workspace" in Bd.last_error()
    assert _c_attend(ws=4096 + 16) == 1 and "256-byte" in Bd.last_error()
    assert _c_attend(ws_bytes=n - 1) == 1 and "workspace has" in Bd.last_error()
    assert _c_attend(out=(ctypes.c_int64 * 2)(0, D)) == 1 and "overlap" in Bd.last_error()
    assert Bd.lib.dmc_full_workspace_bytes(ctypes.byref(_full(batch=0)), T, 2) == 0
    assert Bd.lib.dmc_full_workspace_bytes(ctypes.byref(CFG), -1, 2) == 0
    assert Bd.lib.dmc_full_workspace_bytes(ctypes.byref(CFG), T, 0) == 0
    # a larger chunk never takes less
    sizes = [Bd.lib.dmc_full_workspace_bytes(ctypes.byref(CFG), 4096, c) for c in (1, 4, 8, 9, 16, 17, 32, 33, 64, 65, 1000)]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("kw,status,msg", [
    (dict(total=-1), 1, "counts"), (dict(total=1 << 29), 2, "tokens"), (dict(ptr=None), 1, "non-NULL"), (dict(ptr=4104), 1, "aligned"),
    (dict(positions=None), 1, "positions"), (dict(freq=None), 1, "inv_freq"), (dict(cfg=P.make_rotary_config(0, 1, 64)), 1, "head counts"),
    (dict(cfg=P.make_rotary_config(HQ, HKV, 96, rotary_dim=32)), 2, "head_dim"), (dict(cfg=P.RotaryConfig(HQ, HKV, D, 9, R, 0)), 1, "dtype"),
    (dict(cfg=P.make_rotary_config(HQ, HKV, D, rotary_dim=40)), 1, "rotary_dim"), (dict(cfg=P.RotaryConfig(HQ, HKV, D, 0, R, 3)), 1, "pairs"),
    (dict(q=(ctypes.c_int64 * 2)(-8, 64)), 1, "non-negative"), (dict(q_out=(ctypes.c_int64 * 2)(D, D)), 1, "overlap"),
])
def test_c_rotation_refusals(kw, status, msg):
    assert _c_rotate(**kw) == status
    assert msg in Bd.last_error()


def test_nothing_to_do_reads_nothing():
    assert _c_rotate(total=0, ptr=None, positions=None, freq=None) == 0
    assert _c_append(total=0, ptr=None, q=None, cu=None, lens=None, table=None, kp=None, freq=None) == 0
    assert _c_attend(total=0, ptr=None, cu=None, lens=None, table=None, kp=None, ws=None, ws_bytes=0) == 0


@pytest.mark.parametrize("name,struct", [("dmc_rotary_config", P.RotaryConfig), ("dmc_full_config", P.FullConfig)])
def test_config_structs_match_the_header(name, struct):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "dmc.h")).read()
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, re.S)
    assert re.findall(r"^\s*int32_t\s+([a-z_]+);", body.group(1), re.M) == [f[0] for f in struct._fields_]


def test_one_pass_checks_agree_with_the_full_ones():
    """What the one-pass checks accept on their device has the full check's approval; whatever they decline goes to
    it."""
    full = P.DMCFull(CFG, max_tokens=T, max_chunk=2, inv_freq=torch.zeros(R // 2), device="cpu")
    rot = P.DMCRotation(P.make_rotary_config(HQ, HKV, D, rotary_dim=R), full._storage["inv_freq"], device="cpu")
    pool_k, pool_q = full.k_pages.view(-1, HKV, D)[:T], full.v_pages.view(-1, HQ, D)[:T]
    x = torch.zeros(T + 1, HQ + HKV, D, dtype=BF)

    def agree(quick, check, a, good):
        if good:
            assert quick(**a) is not None
            check(a)   # does not raise
        else:
            assert quick(**a) is None

    def append(a):
        Bd.check_full_append_args(CFG, CPU, full._storage, **a)

    def attend(a):
        Bd.check_full_attend_args(CFG, CPU, full._storage, **a)

    def rotate(a):
        Bd.check_rotary_args(rot.cfg, CPU, inv_freq=rot.inv_freq, **a)

    ok = {n: t for n, t in _append().items() if n != "storage"}
    agree(full._quick_append, append, ok, True)
    assert full._quick_append(**ok)[2:6] == tuple(ok[n].data_ptr() for n in ("k", "v", "q", "q_out"))
    agree(full._quick_append, append, dict(ok, q=None, q_out=None), True)
    agree(full._quick_append, append, dict(ok, q=x[:T, :HQ], k=x[:T, HQ:]), True)
    for bad in (dict(k=pool_k), dict(v=pool_k), dict(q=pool_q), dict(q_out=pool_q), dict(q_out=x[1:, :HQ], k=x[:T, HQ:]),
                dict(k=ok["k"].float()), dict(v=ok["v"][:3]), dict(q_out=ok["q"]), dict(cu_seqlens=None), dict(q=None),
                dict(cu_seqlens=full.page_table.view(-1)[:B + 1]), dict(q_out=ok["q_out"].transpose(0, 1)), dict(k="k"), dict(q_out=None)):
        agree(full._quick_append, append, dict(ok, **bad), False)
    ok = {n: t for n, t in _attend().items() if n != "storage"}
    agree(full._quick_attend, attend, ok, True)
    assert full._quick_attend(**ok)[2:5] == tuple(ok[n].data_ptr() for n in ("q", "out", "lse"))
    for bad in (dict(out=pool_q), dict(out=ok["q"]), dict(lse=ok["lse"].t()), dict(lse=torch.zeros(T, HQ, dtype=BF)),
                dict(lse=full.k_pages.view(torch.float32).view(-1)[:T * HQ].view(T, HQ)), dict(q=ok["q"].float()),
                dict(out=ok["out"][..., :32]), dict(cu_seqlens=ok["cu_seqlens"].long()), dict(q=None)):
        agree(full._quick_attend, attend, dict(ok, **bad), False)
    ok = {n: t for n, t in _rotary().items() if n != "inv_freq"}
    agree(rot._quick, rotate, ok, True)
    for bad in (dict(q_out=ok["q"]), dict(k_out=x[:T, :HKV], q_out=x[:T, :HQ]), dict(positions=ok["q_out"].view(I32).view(-1)[:T]),
                dict(positions=ok["positions"].long()), dict(q=ok["q"][:0]), dict(k=ok["k"][1:]), dict(k_out=None)):
        agree(rot._quick, rotate, dict(ok, **bad), False)


def test_strides_are_those_of_the_call():
    full = P.DMCFull(CFG, max_tokens=T, max_chunk=2, inv_freq=torch.zeros(R // 2), device="cpu")
    a = {n: t for n, t in _attend().items() if n != "storage"}
    wide = torch.zeros(T, HQ, 2 * D, dtype=BF)
    first = full._quick_attend(**a)[-1]
    assert list(first) == [HQ * D, D, HQ * D, D] and full._quick_attend(**a)[-1] is first
    assert list(full._quick_attend(**dict(a, q=wide[..., :D]))[-1]) == [2 * HQ * D, 2 * D, HQ * D, D]
    assert list(first) == [HQ * D, D, HQ * D, D]   # (the earlier call's array stays as it was)


def test_strides_of_two_threads_do_not_mix():
    """One object used from two threads with tensors of other strides: each call gets its own, also if the other
    thread's call comes between the comparison with the kept strides and the use of their array."""
    call = Bd._RowsCall(BF, DEV, D, 2)

    class Between(int):
        def __eq__(self, other):
            call.strides(72, 128)
            return int(self) == int(other)
        __hash__ = int.__hash__
    assert tuple(call.strides(64, 128)) == (64, 128)
    assert tuple(call.strides(Between(64), 128)) == (64, 128)
    assert tuple(call.strides(64, 128)) == (64, 128)


def test_more_tokens_than_a_launch_takes():
    """2^24 tokens, 256 threads each, would be 2^32 threads."""
    for total in ((1 << 23) + 1, 1 << 24):
        assert _c_rotate(total=total) == 2 and "8388608" in Bd.last_error()
        assert _c_append(total=total) == 2 and "too many tokens" in Bd.last_error()
