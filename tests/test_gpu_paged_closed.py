"""Pools that are closed under a table of them."""
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
def test_a_table_knows_which_of_its_pools_are_closed(monkeypatch, native):
    from paper_2605_05699_amd import binding as B
    B.lib()
    if not native:
        monkeypatch.setattr(B, "_fast_pool_copy", B._not_made)
    plan = B.Plan(64, 32, 3)
    pools = [B.PagePool.empty(plan, plan, 2, 16, 4, 2) for _ in range(3)]
    table, rest, gone = B.PoolTable(pools), B.PoolTable(pools[:1] + pools[2:]), B.PoolTable(pools[1:])
    del gone
    gc.collect()
    pairs = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    B.srft_pool_copy(table, pairs, pairs[:0])
    pools[1].close()
    with pytest.raises(B.SrftError) as e:
        B.srft_pool_copy(table, pairs, pairs[:0])
    assert e.value.status == -1
    pools[0].k[1].copy_(torch.rand_like(pools[0].k[1]))
    B.srft_pool_copy(rest, pairs, pairs[:0])
    torch.cuda.synchronize()
    assert torch.equal(pools[0].k[1][0], pools[0].k[1][1])
    seqs = B.PagedSeqs(*(torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((1, 1), (1, 2), (1,), (2,))), max_new=1, max_length=16)
    x, space = torch.zeros(1, 2, 64, dtype=torch.float16, device="cuda"), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    for call in (lambda: B.srft_pool_append(pools[1], seqs, x, x, space), lambda: B.srft_pool_attention(pools[1], seqs, x, 0.1, x, space)):
        with pytest.raises(B.SrftError) as e:
            call()
        assert e.value.status == -1
    for p in pools:
        p.close()
