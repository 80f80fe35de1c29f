"""DMCFull and DMCRotation objects without a GPU: what a new one holds, which calls it takes, what missing tensors are told."""
import pytest
import torch

import paper_2403_09636_amd as P

B, HQ, HKV, D = 3, 4, 2, 64
BF, I32 = torch.bfloat16, torch.int32
CFG = P.make_full_config(B, HQ, HKV, D, page_size=8, max_pages=4, num_pages=12)


def test_a_new_page_table_names_no_page():
    """Before the program has written a row's pages, a call that would use them finds page ids outside the pool (and says
    so by the flag) instead of page 0 for every row."""
    full = P.DMCFull(CFG, device="cpu")
    assert (full.page_table == -1).all()
    assert not full.lengths.any() and not full.flags.any()


def _step(tokens, heads):
    return torch.zeros(tokens, heads, D, dtype=BF)


def test_append_takes_more_tokens_than_the_workspace_is_for():
    """max_tokens is the attention's: append needs no workspace, so that the default object (one token per row) takes a
    prompt too."""
    full = P.DMCFull(CFG, device="cpu")
    cu = torch.tensor([0, 9, 9, 20], dtype=I32)
    k, v, q = _step(20, HKV), _step(20, HKV), _step(20, HQ)
    assert full._quick_append(k, v, q, torch.empty_like(q), cu)[0] == 20
    assert full._quick_append(k, v, None, None, cu)[0] == 20
    with pytest.raises(P.DMCError, match="the workspace holds 3"):
        full.attend(0, q, cu_seqlens=cu)


def _told(fn, name):
    with pytest.raises(P.DMCError) as e:
        fn()
    assert f"{name} must be a torch.Tensor" in str(e.value), str(e.value)


@pytest.mark.parametrize("bad", [None, "q", 3.0, [1.0]])
def test_what_is_no_tensor_is_named(bad):
    """The checks' message, whether or not the outputs are the caller's."""
    full = P.DMCFull(CFG, device="cpu")
    rot = P.DMCRotation(P.make_rotary_config(HQ, HKV, D, rotary_dim=0), device="cpu")
    q, k, lse, pos = _step(B, HQ), _step(B, HKV), torch.zeros(B, HQ), torch.zeros(B, dtype=I32)
    _told(lambda: full.attend(0, bad), "q")
    _told(lambda: full.attend(0, bad, out=q), "q")
    _told(lambda: full.attend(0, bad, lse=lse), "q")
    _told(lambda: full.attend(0, bad, out=q, lse=lse), "q")
    _told(lambda: full.append(0, bad, k), "k")
    _told(lambda: full.append(0, k, bad), "v")
    if bad is not None:   # (None: no queries)
        _told(lambda: full.append(0, k, k.clone(), q=bad), "q")
        _told(lambda: full.append(0, k, k.clone(), q=bad, q_out=q), "q")
    for fn in (rot.forward, rot.backward):
        _told(lambda: fn(bad, k, pos), "q")
        _told(lambda: fn(q, bad, pos), "k")
        _told(lambda: fn(bad, k, pos, q.clone(), k.clone()), "q")
        _told(lambda: fn(q, k, bad), "positions")
