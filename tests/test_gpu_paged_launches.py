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


# ---- launches of more workgroups than 2^32 threads in one dimension
def test_rotary_of_more_tokens_than_one_dimension_of_a_launch_holds(B):
    from tests.test_gpu_rotary import check as turned_right
    n = (1 << 26) + 5                                        # (of 64 threads each)
    x = torch.randn(n, 1, 2, device="cuda").half()
    y = torch.full_like(x, float("nan"))
    positions = torch.arange(n, device="cuda", dtype=torch.int32) % 100_003
    freq = torch.tensor([0.3], device="cuda", dtype=torch.float64)
    B.srft_rotary([(x, y)], positions, freq)
    torch.cuda.synchronize()
    assert not bool(torch.isnan(y).any())
    for at in (0, 1 << 20, (1 << 25) - 500, (1 << 26) - 995):
        turned_right(y[at: at + 1000], x[at: at + 1000], positions[at: at + 1000], freq, "half", 1.0, False)


def test_attention_of_a_prompt_among_many_sequences(B):
    """A prompt of 2048 tokens among 4095 sequences of one: 2^24 workgroups of 256 threads, were every sequence as long."""
    d, R, n, long_, group = 64, 32, 4096, 2048, 64
    plans = [B.Plan(d, 32, 5 + i, None, 8) for i in range(2)]
    pool = B.PagePool.empty(*plans, 1, R, long_ // R, 2 * n)
    t = lambda a: torch.tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")      # noqa: E731
    at = 1000                                                # the prompt's place among the sequences
    new = np.ones(n, np.int64)
    new[at] = long_
    table = np.full((n, long_ // R), -1)
    table[at] = np.arange(long_ // R)[::-1]
    windows = np.stack([np.arange(n) * 2] * 2, 1)
    windows[at, 1] += 1
    starts = np.concatenate([[0], np.cumsum(new)])
    seqs = B.PagedSeqs(t(table), t(windows), t(new), t(starts), max_new=long_, max_length=long_)
    total = int(new.sum())
    k, v = (torch.randn(total, 1, d, device="cuda").half() for _ in "kv")
    q = torch.randn(total, group, d, device="cuda").half()
    out = torch.full_like(q, float("nan"))
    space = torch.empty(max(B.srft_pool_append_workspace_bytes(pool, seqs, total), B.srft_pool_attention_workspace_bytes(pool, seqs, total, group)),
                        dtype=torch.uint8, device="cuda")
    B.srft_pool_append(pool, seqs, k, v, space)
    B.srft_pool_attention(pool, seqs, q, 0.125, out, space)
    alone = B.PagedSeqs(t(table[at: at + 1]), t(windows[at: at + 1]), t(new[at: at + 1]), t([0, long_]), max_new=long_, max_length=long_)
    rows = slice(int(starts[at]), int(starts[at]) + long_)
    want = torch.full_like(q[rows], float("nan"))
    B.srft_pool_attention(pool, alone, q[rows], 0.125, want, space)
    torch.cuda.synchronize()
    # two calls that cut the keys elsewhere: each is off by some roundings of 2^-11 of a value's size
    assert float((out[rows].float() - want.float()).abs().max()) <= 8 * 2.0 ** -11 * float(v.abs().max())
    # a sequence of one token answers its value: the transform there and back, with the window's rows rounded to fp16 in between
    others = torch.ones(total, dtype=torch.bool, device="cuda")
    others[rows] = False
    error = (out[others].float() - v[others].float()).norm(dim=-1) / v[others].float().norm(dim=-1)
    assert float(error.max()) <= 3 * 2.0 ** -11
    pool.close()


def test_copies_of_more_pairs_than_one_dimension_of_a_launch_holds(B):
    plan = B.Plan(64, 32, 3)
    pool = B.PagePool.empty(plan, plan, 2, 16, 8, 4)
    for x in (*pool.k, *pool.v):
        x.copy_(torch.randint(0, 100, x.shape, device="cuda").to(x.dtype))
    before = [x.clone() for x in (*pool.k, *pool.v)]
    n = (1 << 24) + 3                                        # (of 256 threads each); pairs of -1 are skipped
    pages, windows = (torch.full((m, 2), -1, dtype=torch.int32, device="cuda") for m in (n, 5))
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")      # noqa: E731
    pages[0], pages[1 << 22], pages[-1] = ints(0, 1), ints(2, 3), ints(4, 5)
    windows[-1] = ints(0, 3)
    B.srft_pool_copy(B.PoolTable([pool]), pages, windows)
    torch.cuda.synchronize()
    for i, (x, old) in enumerate(zip((*pool.k, *pool.v), before)):
        for a, b in ([(0, 1), (2, 3), (4, 5)] if i % 3 < 2 else [(0, 3)]):
            old[b] = old[a]
        assert torch.equal(x, old)
    pool.close()


def test_rotary_in_place_where_a_stride_does_not_count(B):
    """One token, one head: what their strides are is nothing that in and out can differ in."""
    from tests.test_gpu_rotary import check as turned_right
    positions, freq = torch.tensor([70], dtype=torch.int32, device="cuda"), torch.rand(32, device="cuda", dtype=torch.float64)
    for shape, a, b in (((1, 5, 64), (320, 64, 1), (8, 64, 1)), ((1, 1, 64), (64, 64, 1), (8, 128, 1))):
        x = torch.randn(shape, device="cuda").half()
        first = x.clone()
        B.srft_rotary([(x.as_strided(shape, a), x.as_strided(shape, b))], positions, freq)
        torch.cuda.synchronize()
        turned_right(x, first, positions, freq, "half", 1.0, False)
    with pytest.raises(B.SrftError) as e:
        B.srft_rotary([(x, x.view(torch.bfloat16))], positions, freq)
    assert e.value.status == -7


def test_the_merge_has_workgroups_for_rows_that_there_are(B):
    """A prompt of 32,768 tokens among 4095 sequences of one, 512 query heads on 8: were every sequence as long, the merge's workgroups
    would be more than 32 bits count, and the call refused."""
    plan = B.Plan(64, 32, 3)
    pool = B.PagePool.empty(plan, plan, 8, 16, 1, 1)
    n, long_ = 4096, 32768
    t = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")      # noqa: E731
    seqs = B.PagedSeqs(t(n, long_ // 16), t(n, 2), t(n), t(n + 1), max_new=long_, max_length=long_)
    assert B.srft_pool_attention_workspace_bytes(pool, seqs, long_ + n - 1, 512) > 0
    pool.close()


@pytest.mark.parametrize("new", [[300, 1, 0, 17, 16, 257, 2, 256, 0, 1], [0, 0, 600, 0, 1, 5, 40, 8, 9, 0], [1] * 9 + [513]])
@pytest.mark.parametrize("cap", [0, 2, 11])
def test_rows_of_chunks_among_rows_of_few(B, new, cap):
    """Blocks of rows that several workgroups share, of sequences between others that have none."""
    s = Serving(B, 64, 32, 8, 32, 2, n=len(new), max_length=1200, seed=sum(new))
    s.append([200, 0, 31, 500, 7, 0, 64, 33, 1, 450])
    s.append(new)
    q = queries(s, sum(new), 2, F16)
    for p in s.plans:
        B.srft_plan_set_max_workgroups(p.handle, cap)
    out = s.run(q, new, 0.125)
    torch.cuda.synchronize()
    check(s, q, new, 0.125, out, 2)
    s.close()
