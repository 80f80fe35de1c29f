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
