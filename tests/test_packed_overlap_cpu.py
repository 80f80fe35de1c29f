"""The arrays of the packed calls (lse, cu_seqlens, slot_index, accepted) that share memory with what a
call writes are refused, by the full checks and by the one-pass ones; arrays between a tensor's rows are
not."""
import pytest
import torch

import paper_2403_09636_amd as P
from paper_2403_09636_amd import binding as Bd

DEV = torch.device("cuda", 0)
T, B, HQ, HKV, D = 6, 2, 4, 2, 64
F32, I32 = torch.float32, torch.int32
CAUSAL = P.make_causal_config(HQ, HKV, D, "fp32")
CACHE = P.make_config(1, B, HQ, HKV, D, "fp32", max_slots_per_seq=64)
CALL = Bd._PackedCall(F32, torch.device("cpu"), D, 4)


def packed(heads, n=T):
    return torch.zeros(n, heads, D)


def causal_args(backward):
    a = dict(q=packed(HQ), k=packed(HKV), v=packed(HKV), cu_seqlens=torch.zeros(B + 1, dtype=I32), out=packed(HQ),
             lse=torch.zeros(T, HQ))
    if backward:
        a.update(dout=packed(HQ), dq=packed(HQ), dk=packed(HKV), dv=packed(HKV))
    return a


def chunk_args(append):
    a = dict(q=packed(HQ), k=packed(HKV), v=packed(HKV), cu_seqlens=torch.zeros(B + 1, dtype=I32))
    if append:
        a.update(accepted=torch.zeros(B, dtype=I32), slot_index=torch.zeros(T, HKV, dtype=I32))
    else:
        a["out"] = packed(HQ)
    return a


def span(t):
    return t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()


def quick_causal(a):
    ins, outs = [(a["q"], HQ), (a["k"], HKV), (a["v"], HKV)], [(a["out"], HQ)]
    if "dout" not in a:
        return CALL.tensors(T, ins, outs, (span(a["cu_seqlens"]),), (span(a["lse"]),))
    return CALL.tensors(T, [*ins, *outs, (a["dout"], HQ)], [(a["dq"], HQ), (a["dk"], HKV), (a["dv"], HKV)],
                        (span(a["cu_seqlens"]), span(a["lse"])))


def quick_chunk(a):
    ins = [(a["q"], HQ), (a["k"], HKV), (a["v"], HKV)]
    if "out" in a:
        return CALL.tensors(T, ins, [(a["out"], HQ)], (span(a["cu_seqlens"]),))
    return CALL.tensors(T, ins, (), (span(a["cu_seqlens"]), span(a["accepted"])), (span(a["slot_index"]),))


def refusal(fn):
    with pytest.raises(P.DMCError) as e:
        fn()
    return str(e.value)


def part(t, dtype, shape, at=8):
    """An array inside the memory of t."""
    n = torch.Size(shape).numel()
    return t.flatten()[at:at + n].view(dtype).view(shape)


@pytest.mark.parametrize("backward,array,tensors", [
    (False, "lse", ("q", "k", "v", "out")), (True, "lse", ("dq", "dk", "dv")), (False, "cu_seqlens", ("out",)),
    (True, "cu_seqlens", ("dq", "dk", "dv"))])
def test_causal_arrays(backward, array, tensors):
    ok = causal_args(backward)
    assert quick_causal(ok) is not None
    assert "is on cpu" in refusal(lambda: Bd.check_causal_args(CAUSAL, DEV, **ok))
    for name in tensors:
        a = dict(ok)
        a[array] = part(a[name], a[array].dtype, a[array].shape)
        assert quick_causal(a) is None, name
        msg = refusal(lambda: Bd.check_causal_args(CAUSAL, DEV, **a))
        assert "overlaps" in msg and array in msg and name in msg


def test_lse_that_holds_the_boundaries():
    a = causal_args(False)
    a["cu_seqlens"] = part(a["lse"], I32, (B + 1,))
    assert quick_causal(a) is None
    assert "lse overlaps cu_seqlens" in refusal(lambda: Bd.check_causal_args(CAUSAL, DEV, **a))


def test_lse_of_a_backward_may_lie_in_an_input():
    a = causal_args(True)
    a["lse"] = part(a["q"], F32, (T, HQ))
    assert quick_causal(a) is not None
    assert "is on cpu" in refusal(lambda: Bd.check_causal_args(CAUSAL, DEV, **a))


@pytest.mark.parametrize("append,array,tensors", [(True, "slot_index", ("k", "v", "q", "cu_seqlens", "accepted")),
                                                  (False, "cu_seqlens", ("out",))])
def test_chunk_arrays(append, array, tensors):
    ok = chunk_args(append)
    assert quick_chunk(ok) is not None
    assert "is on cpu" in refusal(lambda: Bd.check_chunk_args(CACHE, DEV, **ok))
    for name in tensors:
        a = dict(ok)
        if a[name].dim() == 3:
            a[array] = part(a[name], a[array].dtype, a[array].shape, 0)
        else:
            a[name] = part(a[array], I32, a[name].shape, 1)
        assert quick_chunk(a) is None, name
        msg = refusal(lambda: Bd.check_chunk_args(CACHE, DEV, **a))
        assert "overlaps" in msg and array in msg and name in msg


def test_slot_index_beside_what_is_read_of_q():
    """Only element 0 of each query row is read: slots in the rest of the rows are apart."""
    a = chunk_args(True)
    buf = torch.zeros(T * HQ * D)
    a["q"] = buf.view(T, HQ, D)
    a["slot_index"] = buf[1:1 + T * HKV].view(I32).view(T, HKV)
    assert quick_chunk(a) is None   # (left to the full check)
    assert "is on cpu" in refusal(lambda: Bd.check_chunk_args(CACHE, DEV, **a))
    a["q"] = a["q"][..., 0]
    assert "is on cpu" in refusal(lambda: Bd.check_chunk_args(CACHE, DEV, **a))
    a["slot_index"] = buf[D - 4:D - 4 + T * HKV].view(I32).view(T, HKV)
    assert "slot_index overlaps q" in refusal(lambda: Bd.check_chunk_args(CACHE, DEV, **a))


def test_arrays_between_rows():
    a = causal_args(False)
    buf = torch.zeros(T, HQ * D + 64)
    a["out"] = buf[:, :HQ * D].view(T, HQ, D)
    a["lse"] = buf[2, HQ * D:HQ * D + T * HQ].view(T, HQ)
    assert "is on cpu" in refusal(lambda: Bd.check_causal_args(CAUSAL, DEV, **a))
    a["lse"] = buf.flatten()[2 * (HQ * D + 64) + HQ * D - 1:][:T * HQ].view(T, HQ)
    assert "lse overlaps out" in refusal(lambda: Bd.check_causal_args(CAUSAL, DEV, **a))
    a["lse"] = buf.flatten()[3 * (HQ * D + 64) - T * HQ + 1:][:T * HQ].view(T, HQ)
    assert "lse overlaps out" in refusal(lambda: Bd.check_causal_args(CAUSAL, DEV, **a))


def test_touches_is_exact():
    """Against the elements themselves, for strided tensors and every place of a short array."""
    gen = torch.Generator().manual_seed(0)
    for _ in range(60):
        t, h, d = (int(torch.randint(1, n, (), generator=gen)) for n in (5, 4, 4))
        st = (int(torch.randint(0, 12, (), generator=gen)), int(torch.randint(0, 12, (), generator=gen)), 1)
        buf = torch.zeros(80, dtype=torch.int16)
        x = buf.as_strided((t, h, d), st, 20)
        mine = {20 + i * st[0] + j * st[1] + e for i in range(t) for j in range(h) for e in range(d)}
        for lo in range(80):
            for n in (1, 3):
                want = not mine.isdisjoint(range(lo, lo + n))
                assert Bd._touches(x, buf.data_ptr() + 2 * lo, buf.data_ptr() + 2 * (lo + n)) == want, (x.shape, st, lo, n)
