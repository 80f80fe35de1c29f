"""Refusals of the chunk calls without a GPU: the binding's tensor checks, and a NULL cache."""
import pytest
import torch

import paper_2403_09636_amd as P
from paper_2403_09636_amd import binding as Bd

DEV = torch.device("cuda", 0)
T, B, HQ, HKV, D = 6, 2, 4, 2, 64
BF = torch.bfloat16


def _args(out=True):
    a = dict(q=torch.zeros(T, HQ, D, dtype=BF), k=torch.zeros(T, HKV, D, dtype=BF),
             v=torch.zeros(T, HKV, D, dtype=BF), cu_seqlens=torch.zeros(B + 1, dtype=torch.int32))
    if out:
        a["out"] = torch.zeros(T, HQ, D, dtype=BF)
    else:
        a.update(accepted=torch.zeros(B, dtype=torch.int32), slot_index=torch.zeros(T, HKV, dtype=torch.int32))
    return a


def _raises(a, msg):
    cfg = P.make_config(1, B, HQ, HKV, D, "bf16", max_slots_per_seq=64)
    with pytest.raises(P.DMCError) as e:
        Bd.check_chunk_args(cfg, DEV, **a)
    assert msg in str(e.value), str(e.value)


def test_valid_arguments_fail_on_the_device_only():
    _raises(_args(), "is on cpu")
    _raises(_args(False), "is on cpu")
    a = _args(False)
    a["q"] = torch.zeros(T, HQ, dtype=BF)   # q[..., 0] alone
    _raises(a, "is on cpu")
    for out in (True, False):
        a = {n: t[:0] if n not in ("cu_seqlens", "accepted") else t for n, t in _args(out).items()}
        _raises(a, "is on cpu")


@pytest.mark.parametrize("out,name,bad,msg", [
    (True, "q", torch.zeros(T, HQ, dtype=BF), "shape"), (True, "q", torch.zeros(T, HQ, D), "dtype"),
    (True, "k", torch.zeros(T + 1, HKV, D, dtype=BF), "shape"), (True, "v", torch.zeros(T, HQ, D, dtype=BF), "shape"),
    (True, "k", torch.zeros(T, D, HKV, dtype=BF).transpose(1, 2), "contiguous last dimension"),
    (True, "v", torch.zeros(T, HKV, D + 4, dtype=BF)[..., :D], "multiples of 8"),
    (True, "out", torch.zeros(T * HQ * D + 8, dtype=BF)[1:1 + T * HQ * D].view(T, HQ, D), "aligned"),
    (True, "cu_seqlens", torch.zeros(B, dtype=torch.int32), "shape"),
    (True, "cu_seqlens", torch.zeros(B + 1, dtype=torch.int64), "dtype"),
    (False, "q", torch.zeros(T, HKV, dtype=BF), "shape"), (False, "q", torch.zeros(T, HQ), "dtype"),
    (False, "accepted", torch.zeros(B + 1, dtype=torch.int32), "shape"),
    (False, "accepted", torch.zeros(B), "dtype"), (False, "slot_index", torch.zeros(HKV, T, dtype=torch.int32), "shape"),
    (False, "slot_index", torch.zeros(T, HKV, dtype=torch.int64), "dtype"),
])
def test_tensor_rejections(out, name, bad, msg):
    a = _args(out)
    a[name] = bad
    _raises(a, msg)


@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_out_that_shares_memory(name):
    a = _args()
    x = torch.zeros(T, HQ + 1, D, dtype=BF)
    a["out"], a[name] = x[:, :HQ], x[:, :a[name].shape[1]]
    _raises(a, f"out overlaps {name}")


def test_null_cache():
    lib = Bd.lib
    assert lib.dmc_chunk_workspace_bytes(None, 8, 8) == 0 and "NULL" in Bd.last_error()
    st = (Bd.c_int64 * 2)(64, 64)
    assert lib.dmc_chunk_attend(None, 0, 16, st, 16, st, 16, st, 16, 8, 8, 16, st, 256, 1 << 30, None) == 1
    assert lib.dmc_chunk_append(None, 0, 16, st, 16, st, 16, st, 16, None, 8, 8, None, 256, 1 << 30, None) == 1
    assert "NULL" in Bd.last_error()
