"""Pools of windows alone: sequences shorter than a page, and page tables whose numbers name nothing."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests.paged_util import Serving
from tests.test_gpu_paged import check, queries

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


def windows_only(B, d, g, bits, R, heads, n, max_length, seed):
    s = Serving(B, d, g, bits, R, heads, n=n, max_length=max_length, seed=seed)
    s.pool.close()
    s.pool = B.PagePool.empty(*s.plans, heads, R, 0, 2 * n + 1)
    for _, _, w in (s.pool.k, s.pool.v):
        w.fill_(float("nan"))
    assert s.pool.n_pages == 0 and s.pool.k[0].numel() == 0
    return s


@pytest.mark.parametrize("d,g,bits,R,heads", [(128, 32, 4, 64, 2), (256, 32, 8, 128, 1), (64, 16, 4, 32, 3), (96, 32, 4, 256, 1)])
@pytest.mark.parametrize("group,dtype", [(1, F16), (6, BF16)])
@pytest.mark.parametrize("chunk", [False, True])
def test_sequences_shorter_than_a_page(B, d, g, bits, R, heads, group, dtype, chunk):
    s = windows_only(B, d, g, bits, R, heads, 5, R - 1, seed=d + R + group)
    s.append([0, 1, R - 4, R // 2, 0])
    for new in ([R - 2, 3, 0, R // 2 - 1, 20] if chunk else [1, 1, 1, 0, 1],):
        s.append(new)
        q = queries(s, sum(new), group, dtype)
        out = s.run(q, new, d ** -0.5)
        torch.cuda.synchronize()
        check(s, q, new, d ** -0.5, out, group)
        for which in (0, 1):                                 # the windows are what was appended
            for b in range(s.n):
                assert np.array_equal(s.window(which, b)[: int(s.length[b])].view(np.uint16), s.tokens[which][b].view(np.uint16))
    s.close()


@pytest.mark.parametrize("new", [[1, 1, 1], [40, 3, 20]])
def test_tokens_in_pages_that_cannot_be_there_count_for_nothing(B, new):
    d, R, heads, group = 128, 16, 2, 4
    s = windows_only(B, d, 32, 4, R, heads, 3, 100, seed=3)
    s.free = [0, 5, -1, 1 << 30] * 10                        # page numbers: none of them exists
    s.append([33, 0, 16])
    s.append(new)
    torch.cuda.synchronize()
    there = [np.arange(100) >= n // R * R for n in s.length]
    tails = {(w, b): s.window(w, b)[: int(s.length[b]) % R].astype(np.float64) @ s.matrix(w).T for w in (0, 1) for b in range(3)}
    s.values = lambda w, b: np.concatenate([np.zeros((int(s.length[b]) // R * R, heads, d)), tails[w, b]])
    q = queries(s, sum(new), group, F16)
    out = s.run(q, new, 0.09)
    torch.cuda.synchronize()
    check(s, q, new, 0.09, out, group, there)
    pairs = torch.tensor([[0, 1], [5, 0], [-1, 2]], dtype=torch.int32, device="cuda")        # copies skip them too
    before = s.pool.k[2].clone()
    B.srft_pool_copy(B.PoolTable([s.pool]), pairs, pairs[:0])
    torch.cuda.synchronize()
    assert torch.equal(before.view(torch.int16), s.pool.k[2].view(torch.int16))
    s.close()


def test_buffers_of_no_page(B):
    plan, h = B.Plan(128, 32, 1), C.c_void_p()
    window = torch.zeros(2, 2, 16, 128, dtype=F16, device="cuda")
    codes = torch.zeros(1, 2, 16, 64, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(1, 2, 16, 4, device="cuda")

    def create(codes_at, scales_at, window_at, pages=0):
        buf = B._PoolBuffers(codes_at, scales_at, window_at)
        return B.lib().srft_pool_create(C.byref(h), plan.handle, plan.handle, 2, 16, pages, 2, C.byref(buf), C.byref(buf))
    w, c, s = window.data_ptr(), codes.data_ptr(), scales.data_ptr()
    assert create(c, s, w) == create(c, None, w) == create(None, s, w) == -7                  # (buffers of pages, and no page)
    assert create(None, None, None) == create(None, None, w, 1) == create(None, s, w, 1) == create(c, None, w, 1) == -1
    assert create(None, None, w, -1) == -7
    assert create(None, None, w) == 0 and B.lib().srft_pool_destroy(h) == 0
    kv = (codes[:0], scales[:0], window)
    B.PagePool(plan, plan, kv, kv).close()
