"""Strides that lead nowhere: of one token, of one head, of no token.  Tensors keep odd ones there, and no call may look at them."""
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


@pytest.fixture(params=["native", "ctypes"])
def way(request, B, monkeypatch):
    if request.param == "ctypes":
        for name in ("rotary", "pool_append", "pool_attention"):
            monkeypatch.setattr(B, "_fast_" + name, B._not_made)
    return request.param


def odd(t, dims):
    return t.as_strided(t.shape, [s + 3 if i in dims else s for i, s in enumerate(t.stride())])


def test_one_token_and_one_head(B, way):
    s = Serving(B, 64, 32, 4, 32, 1, n=1, max_length=96, seed=5)
    s.append([40])
    x = [torch.from_numpy(s.draw(1)).cuda() for _ in "kv"]
    s.grow([1])
    for i in range(2):
        s.tokens[i][0] = np.concatenate([s.tokens[i][0], x[i].cpu().numpy()])
    seqs = s.seqs([1])
    space = torch.empty(B.srft_pool_append_workspace_bytes(s.pool, seqs, 1), dtype=torch.uint8, device="cuda")
    B.srft_pool_append(s.pool, seqs, odd(x[0], (0, 1)), odd(x[1], (1,)), space)
    assert np.array_equal(s.window(0, 0)[:9], s.tokens[0][0][32:]) and np.array_equal(s.window(1, 0)[:9], s.tokens[1][0][32:])
    q = queries(s, 1, 4, F16)
    out = torch.full_like(q, float("nan"))
    s.run(odd(q, (0,)), [1], 0.125, out=odd(out, (0,)))
    torch.cuda.synchronize()
    check(s, q, [1], 0.125, out, 4)
    positions, freq = torch.tensor([5], dtype=torch.int32, device="cuda"), torch.rand(32, dtype=torch.float64, device="cuda")
    a, b = torch.empty_like(q), torch.empty_like(q)
    B.srft_rotary([(q, a)], positions, freq)
    B.srft_rotary([(odd(q, (0,)), odd(b, (0,)))], positions, freq)
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    s.close()


def test_no_token(B, way):
    s = Serving(B, 64, 32, 4, 32, 1, n=1, max_length=96, seed=6)
    s.append([40])
    nothing = torch.empty(0, dtype=F16, device="cuda").as_strided((0, 1, 64), (3, 5, 7))
    seqs, space = s.seqs([0]), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    B.srft_pool_append(s.pool, seqs, nothing, nothing, space)
    B.srft_pool_attention(s.pool, seqs, nothing, 0.1, nothing, space)
    B.srft_rotary([(nothing, nothing)], torch.empty(0, dtype=torch.int32, device="cuda"), torch.rand(32, dtype=torch.float64, device="cuda"))
    torch.cuda.synchronize()
    s.close()
