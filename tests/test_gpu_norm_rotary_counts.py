"""Gradients of norms with rotary positions where a workgroup comes to its tokens several times, and weights' gradients whose every addition shows."""
import pytest
import torch

from tests.test_gpu_norm_rotary import BF16, F16, F32, backward, check_gradients, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


# n, d, rot, heads, types of x and dy.  At most 512 workgroups have a tensor, with as many tokens at a time as their lanes and angles allow: (4099, 128) with 32
# heads three times four tokens, the last time three of one workgroup, with 8 once; in fp32 two tokens five times, and eight twice; and so on.
CASES = [(4099, 128, 128, (32, 8), BF16, BF16), (4099, 128, 128, (32, 8), F32, F32), (1100, 1024, 1024, (24, 1), F16, F16), (2081, 96, 64, (10, 5, 70), F32, BF16),
         (700003, 2, 2, (1, 2), F32, F32), (3001, 34, 34, (7, 64), F16, F32), (5001, 64, 0, (64, 3), BF16, F32), (1025, 256, 256, (16, 16, 2, 40), F16, F16),
         (513, 512, 64, (130,), BF16, BF16)]


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("n,d,rot,heads,x_type,dy_type", CASES)
def test_tokens_that_a_workgroup_comes_to_later(B, layout, n, d, rot, heads, x_type, dy_type):
    gen, x, w, positions, freq = inputs(n, d, rot, heads, (x_type, x_type), n + d, (F32, BF16, None, F16)[: len(heads)])
    dy = [torch.randn(t.shape, device="cuda", generator=gen).to(dy_type) for t in x]
    dx, dw = backward(B, dy, x, w, positions, freq, layout, 1.25)
    for a in zip(dx, dw, dy, x, w):
        check_gradients(*a, positions, freq, layout, 1.25)


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("n,d,rot,heads,x_type,dy_type", [*CASES, (2051, 64, 64, (40, 7), BF16, BF16), (4099, 64, 64, (3, 1), BF16, BF16), (1, 128, 128, (1,), F16, F16)])
def test_every_row_counts_once(B, layout, n, d, rot, heads, x_type, dy_type):
    """Rows of 1 and -1 at position 0, gradients of 1, 2 and 3: r is 1, and all sums of weights' gradients are whole numbers below 2^24, so that fp32 holds every
    one of them.  A row that is left out or added twice changes every channel."""
    gen = torch.Generator("cuda")
    gen.manual_seed(n + d)
    x = [(2 * torch.randint(0, 2, (n, h, d), device="cuda", generator=gen) - 1).to(x_type) for h in heads]
    dy = [(torch.randint(1, 4, t.shape, device="cuda", generator=gen) * (2 * torch.randint(0, 2, t.shape, device="cuda", generator=gen) - 1)).to(dy_type) for t in x]
    dx, dw = [torch.full_like(t, float("nan")) for t in x], [torch.full((d,), float("nan"), device="cuda") for _ in x]
    positions, freq = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.rand(rot // 2, dtype=torch.float64, device="cuda")
    space = torch.full((B.srft_norm_rotary_backward_workspace_bytes(len(x), d),), 0xFF, dtype=torch.uint8, device="cuda")
    B.srft_norm_rotary_backward([(a, b, None, c, e) for a, b, c, e in zip(dy, x, dx, dw)], positions, freq, 2.0 ** -100, space, layout=layout)
    torch.cuda.synchronize()
    for a, b, c, e in zip(dy, x, dx, dw):
        a, b = a.long(), b.long()
        assert torch.equal(e.long(), (a * b).sum((0, 1))) and torch.equal(e, e.round())
        if d & (d - 1) == 0:                                 # (the mean is whole too, in steps of 1 / d)
            want = a.double() - b.double() * (a * b).sum(-1, keepdim=True).double() / d
            assert torch.equal(c, want.to(x_type))
