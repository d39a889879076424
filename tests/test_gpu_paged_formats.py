"""The paged cache in every format: head dimension, group size, code width; decode steps, two blocks of rows, chunks, and the records themselves."""
import pytest
import torch

from tests.paged_util import Serving
from tests.test_gpu_paged import check, queries
from tests.test_gpu_paged_batches import batch, stored_as_quantized

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
EVERY = [(d, g, bits) for d in range(32, 257, 32) for g in sorted({16, *(g for g in range(32, d + 1, 32) if d % g == 0)}) for bits in (4, 8)]


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("d,g,bits", EVERY)
@pytest.mark.parametrize("group,new,dtype", [(2, [1, 1, 0, 1], F16), (8, [3, 4, 1, 2], BF16), (2, [70, 1, 33, 140], F16)])
def test_every_format(B, d, g, bits, group, new, dtype):
    R, heads = {0: (16, 2), 1: (32, 3), 2: (64, 1), 3: (128, 1)}[(d // 32 + g // 16 + bits) % 4]
    s = Serving(B, d, g, bits, R, heads, n=4, max_length=6 * R + 150, seed=d + g + bits + group)
    new = batch(s, [R - 1, 6 * R + 3, 0, 2 * R], new)
    torch.cuda.synchronize()
    stored_as_quantized(s)
    q = queries(s, sum(new), group, dtype)
    out = s.run(q, new, d ** -0.5)
    torch.cuda.synchronize()
    check(s, q, new, d ** -0.5, out, group)
    s.close()
