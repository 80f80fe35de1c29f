"""Appends of short rows, which take one launch, against the same appends by the launches of longer
rows: the same arithmetic, so lengths, slot indexes, slots and z are equal bit for bit."""
import numpy as np
import pytest
import torch

from tests.gpu_helpers import log
from tests.packed_reference import cu_of, dtype_of
from workloads import decision_logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hq,hkv,d,page", [("bf16", 32, 32, 128, 32), ("bf16", 32, 8, 64, 32), ("bf16", 16, 8, 64, 8),
                                                 ("fp32", 8, 8, 64, 16), ("fp32", 4, 2, 128, 64)])
@pytest.mark.parametrize("partly", [False, True])
def test_one_launch_and_several(torch_cuda, dtype, hq, hkv, d, page, partly):
    import paper_2403_09636_amd as P
    B, most = 40, 64
    rng = np.random.default_rng(hkv * d + page)
    cfg = P.make_config(1, B, hq, hkv, d, dtype, page_size=page, max_slots_per_seq=700, max_prompt_len=1)
    caches = [P.DMCCache(cfg) for _ in range(2)]
    chunks = [P.DMCChunk(caches[0], B * most, most), P.DMCChunk(caches[1], B * most, 10 * most)]
    crs = np.array([(1.0, 2.0, 4.0, 16.0)[g % 4] for g in range(hkv)])
    for step in range(10):
        log(f"step {step}")
        lens = [int(x) for x in rng.integers(0, (5, 9, most + 1)[step % 3], B)]
        T = sum(lens)
        x = rng.standard_normal((T, hq + 2 * hkv, d), dtype=np.float32)
        x[:, hq:hq + hkv, 0] = decision_logits(rng.uniform(size=(T, hkv)), crs[None])
        x = torch.from_numpy(x).to(dtype_of(dtype)).cuda()
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        accepted = torch.tensor([int(rng.integers(0, n + 1)) for n in lens], dtype=torch.int32).cuda() if partly else None
        slots = [torch.full((T, hkv), -7, dtype=torch.int32, device="cuda") for _ in chunks]
        for chunk, slot in zip(chunks, slots):
            chunk.append(0, k, v, q, cu_of(lens).cuda(), accepted=accepted, slot_index=slot)
        assert torch.equal(*slots)
        L = [c.lengths(0) for c in caches]
        assert torch.equal(*L)
        dense = max(1, int(L[0].max()))
        for a, b in zip(*(c.export(0, dense) for c in caches)):
            assert torch.equal(a, b)
        assert caches[0].pages_used() == caches[1].pages_used()
    for c in caches:
        c.check()
