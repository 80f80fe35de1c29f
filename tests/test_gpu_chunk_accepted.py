"""Accepted counts outside a row's tokens raise the invalid-argument flag and are clamped, also in rows
without tokens and beside rows that are right."""
import pytest
import torch

from tests.gpu_helpers import f64
from tests.packed_reference import cu_of
from tests.test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("most", [16, 200])   # one launch; several
@pytest.mark.parametrize("lens,accepted,bad", [
    ([0, 6], [0, 6], False), ([0, 6], [1, 6], True), ([0, 6], [-1, 6], True), ([6, 0], [3, 5], True),
    ([0, 0], [0, 2], True), ([0, 0], [0, 0], False), ([6, 4], [6, 5], True), ([6, 4], [6, -7], True)])
def test_accepted_out_of_range(torch_cuda, most, lens, accepted, bad):
    c = Case(4, 2, 64, "bf16", [[20, 3], [9, 31]], max_chunk=most)
    q, k, v = c.tokens(lens, 2.0, tail=3)
    acc = torch.tensor(accepted, dtype=torch.int32, device="cuda")
    c.chunk.append(0, k, v, q, cu_of(lens).cuda(), accepted=acc)
    assert c.cache.status() == (1 if bad else 0)
    held = [min(max(a, 0), n) for a, n in zip(accepted, lens)]
    c.ref.chunk(f64(q), f64(k), f64(v), lens, commit=held, attend=False)
    c.ref.check_cache(c.cache)
