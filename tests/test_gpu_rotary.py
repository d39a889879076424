"""Rotary positions on the GPU against the definition in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
STEP = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


def turned(x, positions, freq, layout, factor, inverse):
    y, rot = x.clone(), 2 * len(freq)
    t = positions.double()[:, None] * freq * (-1.0 if inverse else 1.0)
    c, s = (torch.cos(t) * factor)[:, None], (torch.sin(t) * factor)[:, None]
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def check(got, x, positions, freq, layout, factor, inverse):
    want = turned(x.double(), positions, freq, layout, factor, inverse)
    rot, step = 2 * len(freq), STEP[got.dtype]
    # sine and cosine within two units in the last place of fp32 and three roundings on them, of magnitudes |a| + |b|; then the result's own
    size = x.double().abs()
    if rot:
        half = (size[..., :rot // 2], size[..., rot // 2:rot]) if layout == "half" else (size[..., 0:rot:2], size[..., 1:rot:2])
        pair = abs(factor) * (half[0] + half[1])
        size = size.clone()
        size[..., :rot] = torch.cat([pair, pair], -1) if layout == "half" else torch.stack([pair, pair], -1).flatten(-2)
    bound = size * (7 * 2.0 ** -24) + want.abs() * step * 1.001 + (2.0 ** -25 if got.dtype == F16 else 0.0)
    bound[..., rot:] = want[..., rot:].abs() * (step if got.dtype != x.dtype else 0.0) + (2.0 ** -25 if got.dtype == F16 and x.dtype != F16 else 0.0)
    worst = ((got.double() - want).abs() - bound).max()
    assert float(worst) <= 0.0, float(worst)


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("d,rot", [(128, 128), (96, 64), (64, 32), (256, 256), (80, 20), (6, 2), (128, 0), (2, 2), (34, 34), (1024, 1024)])
@pytest.mark.parametrize("types", [(F16, F16), (BF16, F16), (F32, F32), (F32, BF16), (F16, F32)])
def test_against_the_definition(B, layout, d, rot, types):
    gen = torch.Generator("cuda")
    gen.manual_seed(d + rot)
    n = 37
    x = [torch.randn(n, h, d, device="cuda", generator=gen).to(types[0]) for h in (5, 1, 2)]
    y = [torch.full(t.shape, float("nan"), device="cuda", dtype=types[1]) for t in x]
    positions = torch.randint(0, 1 << 20, (n,), device="cuda", generator=gen, dtype=torch.int32)
    positions[:3] = torch.tensor([0, 1, 2 ** 31 - 1], dtype=torch.int32)
    freq = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / max(rot, 1))
    for inverse in (False, True):
        B.srft_rotary(zip(x, y), positions, freq, layout=layout, factor=1.25, inverse=inverse)
        torch.cuda.synchronize()
        for a, b in zip(x, y):
            check(b, a, positions, freq, layout, 1.25, inverse)


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (0, 3), (8, 8), (4, 4)])
def test_strides_and_offsets_mixed_types_and_in_place(B, layout, offset, pad):
    gen = torch.Generator("cuda")
    gen.manual_seed(3)
    n, d, rot = 19, 64, 48
    positions = torch.randint(0, 5000, (n,), device="cuda", generator=gen, dtype=torch.int32)
    freq = torch.rand(rot // 2, device="cuda", generator=gen, dtype=torch.float64)

    def view(heads, dtype):
        wide = torch.randn(n * heads * (d + pad) + offset, device="cuda", generator=gen).to(dtype)
        return wide, wide[offset:].view(n, heads, d + pad)[..., :d]
    (w1, x1), (w2, x2), (w3, y1), (w4, y2) = view(3, F16), view(2, F32), view(3, F16), view(2, BF16)
    outside = [w.clone() for w in (w3, w4)]
    x3 = x1.transpose(0, 0)[::1]
    first = x1.clone()
    B.srft_rotary([(x1, y1), (x2, y2)], positions, freq, layout=layout)
    torch.cuda.synchronize()
    check(y1, x1, positions, freq, layout, 1.0, False)
    check(y2, x2, positions, freq, layout, 1.0, False)
    for w, old, heads in ((w3, outside[0], 3), (w4, outside[1], 2)):        # nothing between the rows is touched
        assert torch.equal(w[:offset], old[:offset])
        assert torch.equal(w[offset:].view(n, heads, d + pad)[..., d:], old[offset:].view(n, heads, d + pad)[..., d:])
    B.srft_rotary([(x3, x3)], positions, freq, layout=layout)               # in place
    torch.cuda.synchronize()
    assert torch.equal(x1.contiguous().view(torch.int16), y1.contiguous().view(torch.int16))
    check(x1, first, positions, freq, layout, 1.0, False)


def test_the_inverse_is_the_gradient(B):
    """<g, J dx> of the call equals <inverse call of g, dx>, and differences of the call agree with it."""
    gen = torch.Generator("cuda")
    gen.manual_seed(5)
    n, h, d, rot = 11, 3, 40, 24
    positions = torch.randint(0, 100000, (n,), device="cuda", generator=gen, dtype=torch.int32)
    freq = torch.rand(rot // 2, device="cuda", generator=gen, dtype=torch.float64)
    x, dx, g = (torch.randn(n, h, d, device="cuda", generator=gen) for _ in range(3))
    for layout in ("half", "pairs"):
        def call(t, inverse=False):
            out = torch.empty_like(t)
            B.srft_rotary([(t, out)], positions, freq, layout=layout, factor=0.7, inverse=inverse)
            return out
        formula = turned(g.double(), positions, freq, layout, 0.7, True)
        got = call(g, True)
        # (7 roundings of 2^-24 on |a| + |b|, which is at most 2 max |g|)
        assert float((got.double() - formula).abs().max()) <= 16 * 2.0 ** -24 * float(g.abs().max())
        # the map is linear: a difference over a step as large as x itself is exact up to the two calls' roundings
        left = float((g.double() * (call(x + dx).double() - call(x).double())).sum())
        right = float((got.double() * ((x + dx).double() - x.double())).sum())
        assert abs(left - right) <= 24 * 2.0 ** -24 * float((g.abs().double().sum()) * (x.abs().max() + dx.abs().max()).double())


def test_refusals_and_nothing_to_do(B):
    x = torch.randn(4, 2, 64, device="cuda")
    y, pos, freq = torch.empty_like(x), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(16, dtype=torch.float64, device="cuda")
    for bad in (([(x, y[:3])], pos, freq), ([(x, y)], pos[:3], freq), ([(x, y)], pos.long(), freq), ([(x, y)], pos, freq.float()), ([(x.cpu(), y)], pos, freq),
                ([(x.transpose(1, 2), y.transpose(1, 2))], pos, freq), ([(x.double(), y)], pos, freq), ([(x, y)], pos, freq[:, None])):
        with pytest.raises(ValueError):
            B.srft_rotary(*bad)
    with pytest.raises(B.SrftError) as e:
        B.srft_rotary([(x, y)], pos, torch.ones(33, dtype=torch.float64, device="cuda"))
    assert e.value.status == -7
    with pytest.raises(B.SrftError) as e:
        B.srft_rotary([(x, y)] * 5, pos, freq)
    assert e.value.status == -7
    with pytest.raises(KeyError):
        B.srft_rotary([(x, y)], pos, freq, layout="other")
    B.srft_rotary([], pos, freq)
    B.srft_rotary([(x[:0], y[:0])], pos[:0], freq)
    torch.cuda.synchronize()
