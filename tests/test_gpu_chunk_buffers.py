"""Chunks in buffers that are much longer than their tokens (a padded batch, a captured graph's static
buffers): the unused rows change nothing, neither the outputs nor how the attention is cut into pieces."""
import pytest

from tests.gpu_helpers import log
from tests.test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,lens,most,total", [
    # one narrow tile per unit, cut into pieces for a long cache; the buffer alone holds eight tiles per compute unit
    (64, 8, [4, 3], 4, 1024), (8, 8, [8, 1], 8, 8192), (2, 2, [30, 0], 32, 32768),
    # planned pieces: more columns than a narrow tile
    (8, 8, [40, 3], 40, 16384), (16, 4, [100], 100, 8192),
])
def test_long_buffers(torch_cuda, dtype, hq, hkv, lens, most, total):
    log(f"{dtype} heads {hq}/{hkv} lens {lens} in {total} rows")
    slots = [[2000] + [600] * (hkv - 1), [30] * hkv][:len(lens)]
    c = Case(hq, hkv, 64, dtype, slots, max_tokens=total, max_chunk=most)
    x = c.tokens(lens, 2.0, tail=total - sum(lens))
    log(f"worst {c.attend(*x, lens):.3f} of the bound")
    c.cache.check()
