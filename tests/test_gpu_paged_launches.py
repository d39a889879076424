"""Sizes of launches and workspaces of the paged cache and of rotary positions."""
import numpy as np
import pytest
import torch

from tests.paged_util import Serving
from tests.test_gpu_paged import check, queries

pytestmark = pytest.mark.gpu
F16 = torch.float16


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


def test_a_workspace_serves_whatever_the_cap_on_workgroups_is_by_then(B):
    s = Serving(B, 128, 32, 4, 16, 2, n=3, max_length=900, seed=8)
    s.append([800, 300, 33])
    new = [1, 90, 2]
    s.append(new)
    seqs, q = s.seqs(new), queries(s, sum(new), 4, F16)
    sizes = []
    for cap in (1, 0, 7, 1 << 20):
        for p in s.plans:
            B.srft_plan_set_max_workgroups(p.handle, cap)
        sizes.append((B.srft_pool_attention_workspace_bytes(s.pool, seqs, sum(new), 8), B.srft_pool_append_workspace_bytes(s.pool, seqs, sum(new))))
    assert len(set(sizes)) == 1
    whole = torch.full((sizes[0][0] + (1 << 16),), 0xA5, dtype=torch.uint8, device="cuda")
    space, outs = whole[: sizes[0][0]], []
    for cap in (1, 1 << 20, 0):
        for p in s.plans:
            B.srft_plan_set_max_workgroups(p.handle, cap)
        out = torch.full_like(q, float("nan"))
        B.srft_pool_attention(s.pool, seqs, q, 0.1, out, space)
        torch.cuda.synchronize()
        assert bool((whole[sizes[0][0]:] == 0xA5).all())
        check(s, q, new, 0.1, out, 4)
        outs.append(out)
    assert torch.equal(outs[1], outs[2])                     # (a cap above the launch's own size is none)
    s.close()
