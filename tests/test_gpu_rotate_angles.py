"""Cosines and sines of the rotation where they are small: there a rounding of the angle itself would show."""
import math

import pytest
import torch

from tests import full_reference as R

pytestmark = pytest.mark.gpu

# Pairs (1, 0) of fp32 come out as (cos a, sin a).  Their errors: the library's sine and cosine of pi x, at most 4 steps
# (2^-23) of the value; what the angle's fraction has below 32 bits enters by a product and a sum, rounded once each (2^-24 of
# the value, and of a term no larger than 2^-23 of 1: 2^-47); the turns themselves, three roundings of 2^-53 of at most
# 2^18 turns, 2 pi times that: 2^-30.
LOOSE = 4 * 2.0 ** -23 + 2 * 2.0 ** -24
LEAST = 2.0 ** -30 + 2.0 ** -47


def _angles():
    g = torch.Generator().manual_seed(11)
    f = (0.2 + 0.8 * torch.rand(32, generator=g)).float()
    pos = torch.randint(0, 1 << 20, (4096,), generator=g).int()
    return f, pos, pos.double()[:, None] * f.double()


def _close(c, s, a, inverse):
    seen = 0
    for got, want in ((c, a.cos()), (s, -a.sin() if inverse else a.sin())):
        small = want.abs() <= 0.05
        seen += int(small.sum())
        off = (got.double() - want).abs()
        bad = small & (off > LOOSE * want.abs() + LEAST)
        assert not bad.any(), f"{int(bad.sum())} of {int(small.sum())} too far off, by up to {off[small].max().item():.2e}"
    assert seen > 5000


@pytest.mark.parametrize("inverse", [False, True])
def test_small_cosines_and_sines(torch_cuda, inverse):
    import paper_2403_09636_amd as P
    f, pos, a = _angles()
    rot = P.DMCRotation(P.make_rotary_config(1, 1, 64, "fp32", rotary_dim=64), f.cuda())
    x = torch.zeros(len(pos), 1, 64, device="cuda")
    x[..., :32] = 1.0
    turn = rot.backward if inverse else rot.forward
    for y in turn(x, x.clone(), pos.cuda()):
        y = y[:, 0].cpu()
        _close(y[:, :32], y[:, 32:], a, inverse)


def test_small_cosines_and_sines_of_appended_keys(torch_cuda):
    import paper_2403_09636_amd as P
    f, _, _ = _angles()
    cfg = P.make_full_config(1, 1, 1, 64, "fp32", page_size=256, max_pages=16, rotary_dim=64, pairs="adjacent")
    full = P.DMCFull(cfg, max_tokens=4096, inv_freq=f.cuda())
    full.page_table.copy_(torch.arange(16, dtype=torch.int32).view(1, 16))
    x = torch.zeros(4096, 1, 64, device="cuda")
    x[..., 0::2] = 1.0
    cu = torch.tensor([0, 4096], dtype=torch.int32, device="cuda")
    q = full.append(0, x, x.clone(), q=x.clone(), cu_seqlens=cu)
    full.check()
    a = torch.arange(4096).double()[:, None] * f.double()
    for y in (q[:, 0].cpu(), full.k_pages[0, :, 0].reshape(4096, 64).cpu()):
        _close(y[:, 0::2], y[:, 1::2], a, False)
