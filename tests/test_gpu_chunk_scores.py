"""A score of -infinity has weight 0: a token whose own score it is comes out as the rest of what it sees,
and as NaN where that is nothing, as a softmax gives it."""
import math

import numpy as np
import pytest

from tests.gpu_helpers import f64
from tests.packed_reference import cu_of
from tests.test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("slots", [0, 50, 3000])   # nothing, a few blocks, blocks in several pieces
@pytest.mark.parametrize("lens,most", [([6], 6), ([6], 40), ([40], 40), ([1], 1)])
def test_own_score_of_minus_infinity(torch_cuda, dtype, slots, lens, most):
    c = Case(8, 2, 64, dtype, [[slots] * 2], max_chunk=most)
    q, k, v = c.tokens(lens, 1.0)
    k[..., 0] = -1.0       # every token opens a slot
    q[:, :, 1] = 1.0
    k[0, :, 1] = -1e30     # (for the reference: a weight that vanishes)
    want, bound, _ = c.ref.chunk(f64(q), f64(k), f64(v), lens)
    k[0, :, 1] = -math.inf
    out = f64(c.chunk.attend(0, q, k, v, cu_of(lens).cuda()))
    rows = slice(0 if slots else 1, None)
    assert (np.abs(out - want)[rows] <= bound[rows]).all()
    if slots == 0:
        assert np.isnan(out[0]).all()
