"""Attention of sequences with pages in common, in numbers: more sequences and groups than a wavefront or two have lanes, and than LDS has bounds for."""
import numpy as np
import pytest
import torch

from tests.paged_util import Serving
from tests.test_gpu_paged_shared import check, fork, prefixes_of, queries, share

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


# 63, 64, 127 and 128 items, 63 to 65 groups, 128 and more items, and 255, 256 and 300 groups
COUNTS = [(42, 21), (43, 21), (85, 42), (86, 42), (100, 50), (126, 63), (128, 64), (131, 65), (200, 100), (510, 255), (512, 256), (600, 300)]


@pytest.mark.parametrize("n,n_groups", COUNTS)
@pytest.mark.parametrize("chunks", [False, True])
def test_groups_of_two(B, n, n_groups, chunks):
    groups = [2 * g for g in range(n_groups)] + [2 * n_groups if n_groups * 2 <= n else n]
    R, pages = 16, [1 + g % 3 for g in range(n_groups)]
    s = fork(Serving(B, 64, 32, 4, R, 2, n=n, max_length=112, seed=n), groups, pages)
    new = [1] * n
    if chunks:
        for b in (0, 3, n // 2, n - 1):
            new[b] = 20
    s.append([a + int(x) for a, x in zip(new, s.rng.integers(0, 30, n))])
    q = queries(s, new, 4, torch.float16)
    out = share(s, q, new, 0.125, prefixes_of(B, groups, [R * p for p in pages]))
    check(s, out, q, new, 0.125, 4)
    s.close()


@pytest.mark.parametrize("n,n_groups", [(100, 50), (200, 100), (600, 300)])
def test_bounds_that_do_not_ascend(B, n, n_groups):
    """All sequences begin with the same pages, so that any groups are groups; bounds below and far above those around them, on both sides of 64 and 256."""
    R = 16
    s = fork(Serving(B, 64, 32, 4, R, 2, n=n, max_length=112, seed=n + 1), [0, n], [3])
    new = [1] * n
    s.append([a + int(x) for a, x in zip(new, s.rng.integers(0, 30, n))])
    q = queries(s, new, 4, torch.float16)
    for lost in ((5, 63), (64, 65), (n_groups // 2, n_groups - 1), (0, n_groups)):
        groups = [min(2 * g, n) for g in range(n_groups + 1)]
        for i, g in enumerate(lost):
            if g <= n_groups:
                groups[g] = (-3, 0, 2 ** 31 - 1)[(i + g) % 3]
        out = share(s, q, new, 0.125, prefixes_of(B, groups, [R * (1 + g % 3) for g in range(n_groups)]))
        check(s, out, q, new, 0.125, 4)
    s.close()


@pytest.mark.parametrize("workgroups", [1, 7, 0])
@pytest.mark.parametrize("heads,group", [(2, 1), (4, 8)])
def test_any_number_of_workgroups(B, workgroups, heads, group):
    """150 sequences in groups of one to five, some of them without new tokens, some in no group."""
    n, R = 150, 16
    rng = np.random.default_rng(workgroups + group)
    groups = [2]
    while groups[-1] + 5 < n - 3:
        groups.append(groups[-1] + int(rng.integers(1, 6)))
    pages = [int(x) for x in rng.integers(0, 4, len(groups) - 1)]
    s = fork(Serving(B, 128, 32, 8, R, heads, n=n, max_length=160, seed=group), groups, pages)
    new = [int(x) for x in rng.choice([0, 1, 1, 1, 2, 5], n)]
    s.append([a + int(x) for a, x in zip(new, rng.integers(1, 30, n))])
    q = queries(s, new, group, torch.bfloat16)
    B.srft_plan_set_max_workgroups(s.plans[0].handle, workgroups)
    out = share(s, q, new, 0.1, prefixes_of(B, groups, [R * p for p in pages]))
    B.srft_plan_set_max_workgroups(s.plans[0].handle, 0)
    check(s, out, q, new, 0.1, group)
    s.close()
