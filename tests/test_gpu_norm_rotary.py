"""RMS norms with rotary positions on the GPU, and their gradients, against the definition in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
STEP = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
TINY = {F32: 2.0 ** -126, F16: 2.0 ** -25, BF16: 2.0 ** -126}             # half a step of the smallest numbers (fp32 and bf16: where they end for sure)
U = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


def parts(rot, layout):
    return (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))


def turned(x, positions, freq, layout, factor, sign=1.0):
    y, rot = x.clone(), 2 * len(freq)
    t = sign * positions.double()[:, None] * freq
    c, s = (torch.cos(t) * factor)[:, None], (torch.sin(t) * factor)[:, None]
    a, b = parts(rot, layout)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def sizes(x, rot, layout, factor):
    """|a| + |b| of every channel's pair, times the factor: what the roundings of a turn are relative to."""
    y = x.abs()
    if rot:
        a, b = parts(rot, layout)
        pair = abs(factor) * (y[..., a] + y[..., b])
        y = y.clone()
        y[..., a], y[..., b] = pair, pair
    return y


def norm_error(d):
    """Relative error of r in fp32: a mean of d squares added up by up to 64 lanes (16 in a lane, six steps between them; every square and
    sum half a step, all of one sign, halved by the root), the division, the sum with eps, the root and its inverse."""
    return (0.5 * (24 + d / 64) + 3.5) * U


def check(got, x, weight, positions, freq, layout, factor):
    d, rot = x.shape[-1], 2 * len(freq)
    x, w = x.double(), torch.ones(d, device="cuda", dtype=torch.float64) if weight is None else weight.double()
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    want = turned(n, positions, freq, layout, factor)
    # r, two products, then as a turn: sine and cosine within two units in the last place and three roundings on them, of |a| + |b|
    bound = sizes(n, rot, layout, factor) * (norm_error(d) + 2 * U + 7 * U) * 1.01 + want.abs() * STEP[got.dtype] * 1.001 + TINY[got.dtype]
    worst = ((got.double() - want).abs() - bound).max() if got.numel() else torch.zeros(())
    assert float(worst) <= 0.0, float(worst)


SHAPES = [(258, 130), (128, 128), (96, 64), (64, 32), (256, 256), (80, 20), (6, 2), (128, 0), (2, 2), (34, 34), (1024, 1024), (512, 64), (192, 96)]


def inputs(n, d, rot, heads, types, seed, weights=(F32, F16, None)):
    gen = torch.Generator("cuda")
    gen.manual_seed(seed)
    x = [(torch.randn(n, h, d, device="cuda", generator=gen) * 10.0 ** (torch.randint(-3, 4, (n, h, 1), device="cuda", generator=gen) / 2)).to(types[0]) for h in heads]
    w = [None if t is None else (1 + 0.5 * torch.randn(d, device="cuda", generator=gen)).to(t) for t in weights]
    positions = torch.randint(0, 1 << 20, (n,), device="cuda", generator=gen, dtype=torch.int32)
    positions[: min(3, n)] = torch.tensor([0, 1, 2 ** 31 - 1], dtype=torch.int32)[: min(3, n)]
    freq = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / max(rot, 1))
    return gen, x, w, positions, freq


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("d,rot", SHAPES)
@pytest.mark.parametrize("types", [(F16, F16), (BF16, F16), (F32, F32), (F32, BF16), (F16, F32), (BF16, BF16)])
def test_against_the_definition(B, layout, d, rot, types):
    _, x, w, positions, freq = inputs(37, d, rot, (5, 1, 2), types, d + rot)
    y = [torch.full(t.shape, float("nan"), device="cuda", dtype=types[1]) for t in x]
    B.srft_norm_rotary(zip(x, w, y), positions, freq, EPS, layout=layout, factor=1.25)
    torch.cuda.synchronize()
    for a, b, c in zip(x, w, y):
        check(c, a, b, positions, freq, layout, 1.25)


@pytest.mark.parametrize("n,heads", [(1, (1,)), (1, (14, 2)), (3, (64, 8)), (1000, (1, 1)), (4099, (3, 1)), (2051, (40, 7))])
def test_counts_of_tokens_and_heads(B, n, heads):
    _, x, w, positions, freq = inputs(n, 64, 64, heads, (F16, F16), n, (BF16, F32))
    y = [torch.full_like(t, float("nan")) for t in x]
    B.srft_norm_rotary(zip(x, w, y), positions, freq, EPS)
    torch.cuda.synchronize()
    for a, b, c in zip(x, w, y):
        check(c, a, b, positions, freq, "half", 1.0)


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (0, 3), (8, 8), (4, 4)])
def test_strides_and_offsets_mixed_types_and_in_place(B, layout, offset, pad):
    gen, _, w, positions, freq = inputs(19, 64, 48, (), (F16,), 3, (BF16, F32))
    n, d = 19, 64

    def view(heads, dtype):
        wide = torch.randn(n * heads * (d + pad) + offset, device="cuda", generator=gen).to(dtype)
        return wide, wide[offset:].view(n, heads, d + pad)[..., :d]
    (_, x1), (_, x2), (w3, y1), (w4, y2) = view(3, F16), view(2, F32), view(3, F16), view(2, BF16)
    outside = [t.clone() for t in (w3, w4)]
    wide_weight = torch.cat([w[0][:1], w[0]])[1:]                         # (an address that is aligned to nothing but its element)
    first = x1.clone()
    B.srft_norm_rotary([(x1, wide_weight, y1), (x2, w[1], y2)], positions, freq, EPS, layout=layout)
    torch.cuda.synchronize()
    check(y1, x1, wide_weight, positions, freq, layout, 1.0)
    check(y2, x2, w[1], positions, freq, layout, 1.0)
    for t, old, heads in ((w3, outside[0], 3), (w4, outside[1], 2)):      # nothing between the rows is touched
        assert torch.equal(t[:offset], old[:offset])
        assert torch.equal(t[offset:].view(n, heads, d + pad)[..., d:], old[offset:].view(n, heads, d + pad)[..., d:])
    B.srft_norm_rotary([(x1, wide_weight, x1)], positions, freq, EPS, layout=layout)           # in place
    torch.cuda.synchronize()
    assert torch.equal(x1.contiguous().view(torch.int16), y1.contiguous().view(torch.int16))
    check(x1, first, wide_weight, positions, freq, layout, 1.0)


def test_rows_of_zeros_and_rows_that_are_not_numbers(B):
    x = torch.randn(4, 3, 96, device="cuda").half()
    x[1, 1] = 0.0
    x[2, 0, 17], x[2, 2, 3], x[3, 1, 90] = float("inf"), float("nan"), 65504.0
    y, w = torch.empty_like(x), torch.ones(96, device="cuda")
    pos, freq = torch.arange(4, dtype=torch.int32, device="cuda"), torch.rand(24, dtype=torch.float64, device="cuda")
    B.srft_norm_rotary([(x, w, y)], pos, freq, EPS)
    torch.cuda.synchronize()
    assert not y[1, 1].any()
    bad = torch.zeros(4, 3, dtype=torch.bool, device="cuda")
    bad[2, 0] = bad[2, 2] = True
    assert bool(torch.isnan(y[bad]).any(-1).all()) and bool(torch.isfinite(y[~bad]).all())     # (a row, and no other)
    good = x.clone()
    good[2] = 1.0
    ones = torch.empty_like(good)
    B.srft_norm_rotary([(good, w, ones)], pos, freq, EPS)
    torch.cuda.synchronize()
    check(ones, good, w, pos, freq, "half", 1.0)
    assert torch.equal(ones[:2], y[:2])


# ------------------------------------------------------------------------------------------------------------- gradients
def gradients(dy, x, weight, positions, freq, layout, factor):
    """(dx, dweight, and what the roundings of each are relative to): the formula in 64 bits."""
    d, rot = x.shape[-1], 2 * len(freq)
    x, w = x.double(), torch.ones(d, device="cuda", dtype=torch.float64) if weight is None else weight.double()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    g, size = turned(dy.double(), positions, freq, layout, factor, -1.0), sizes(dy.double(), rot, layout, factor)
    dn, h = g * w, x * r
    dx = r * (dn - h * (dn * h).mean(-1, keepdim=True))
    of = r * (size * w.abs() + h.abs() * (size * w.abs() * h.abs()).mean(-1, keepdim=True))
    return dx, (g * h).flatten(0, 1).sum(0), of, (size * h.abs()).flatten(0, 1).sum(0)


def check_gradients(dx, dweight, dy, x, weight, positions, freq, layout, factor):
    d, rows = x.shape[-1], x.shape[0] * x.shape[1]
    want, sums, of, of_sums = gradients(dy, x, weight, positions, freq, layout, factor)
    # the turn (7), its product with the weight, r three times and in the mean the sum of products as that of the squares, and six more products,
    # quotients and differences
    bound = of * (7 * U + 4 * norm_error(d) + (24 + d / 64) * U + 8 * U) * 1.01 + want.abs() * STEP[dx.dtype] * 1.001 + TINY[dx.dtype]
    worst = ((dx.double() - want).abs() - bound).max()
    assert float(worst) <= 0.0, float(worst)
    if dweight is not None:
        # a term: the turn, r and two products; and the additions that a term goes through: at most all rows one after the other
        bound = of_sums * (7 * U + norm_error(d) + 3 * U + min(rows, 4096) * U) * 1.01 + TINY[F32]
        worst = ((dweight.double() - sums).abs() - bound).max()
        assert float(worst) <= 0.0, float(worst)


def backward(B, dy, x, w, positions, freq, layout, factor, want_weights=True):
    dx = [torch.full_like(t, float("nan")) for t in x]
    dw = [torch.full((t.shape[-1],), float("nan"), device="cuda") if want_weights else None for t in x]
    space = torch.full((B.srft_norm_rotary_backward_workspace_bytes(len(x), x[0].shape[-1]),), 0xFF, dtype=torch.uint8, device="cuda")
    B.srft_norm_rotary_backward(zip(dy, x, w, dx, dw), positions, freq, EPS, space if want_weights else None, layout=layout, factor=factor)
    torch.cuda.synchronize()
    return dx, dw


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("d,rot", SHAPES)
@pytest.mark.parametrize("types", [(F16, F16), (BF16, BF16), (F32, F32), (F32, BF16), (F16, F32)])
def test_gradients_against_the_formula(B, layout, d, rot, types):
    gen, x, w, positions, freq = inputs(37, d, rot, (5, 1, 2), types, 7 * d + rot)
    dy = [torch.randn(t.shape, device="cuda", generator=gen).to(types[1]) for t in x]
    dx, dw = backward(B, dy, x, w, positions, freq, layout, 1.25)
    for a in zip(dx, dw, dy, x, w):
        check_gradients(*a, positions, freq, layout, 1.25)


@pytest.mark.parametrize("n,heads", [(1, (1,)), (1, (14, 2)), (3, (64, 8)), (1000, (1, 1)), (4099, (3, 1)), (2051, (40, 7))])
def test_gradients_of_counts_of_tokens_and_heads(B, n, heads):
    gen, x, w, positions, freq = inputs(n, 64, 64, heads, (BF16, BF16), n, (BF16, F32))
    dy = [torch.randn(t.shape, device="cuda", generator=gen).to(BF16) for t in x]
    dx, dw = backward(B, dy, x, w, positions, freq, "half", 1.0)
    again, sums = backward(B, dy, x, w, positions, freq, "half", 1.0)
    for a in zip(dx, dw, dy, x, w):
        check_gradients(*a, positions, freq, "half", 1.0)
    assert all(torch.equal(a, b) for a, b in zip(dx + dw, again + sums))  # (one order of additions)


@pytest.mark.parametrize("offset,pad", [(1, 0), (0, 3), (8, 8), (4, 4)])
def test_gradients_of_strides_in_place_and_without_weights(B, offset, pad):
    n, d = 21, 64
    gen, _, w, positions, freq = inputs(n, d, 48, (), (F16,), 9, (BF16, None))

    def view(heads, dtype):
        wide = torch.randn(n * heads * (d + pad) + offset, device="cuda", generator=gen).to(dtype)
        return wide[offset:].view(n, heads, d + pad)[..., :d]
    x, dy = [view(3, F16), view(2, F32)], [view(3, F16), view(2, F32)]
    dx, dw = backward(B, dy, x, w, positions, freq, "half", 0.7)
    for a in zip(dx, dw, dy, x, w):
        check_gradients(*a, positions, freq, "half", 0.7)
    alone, _ = backward(B, dy, x, w, positions, freq, "half", 0.7, want_weights=False)
    assert all(torch.equal(a, b) for a, b in zip(dx, alone))
    over_x, over_dy = [t.clone() for t in x], [t.clone() for t in dy]     # (contiguous, and in place of either)
    B.srft_norm_rotary_backward([(dy[0], over_x[0], w[0], over_x[0], None), (over_dy[1], x[1], w[1], over_dy[1], None)], positions, freq, EPS, None, factor=0.7)
    torch.cuda.synchronize()
    for got, (i, t) in ((over_x[0], (0, dy[0])), (over_dy[1], (1, dy[1]))):
        check_gradients(got, None, t, x[i], w[i], positions, freq, "half", 0.7)


def test_gradients_against_differences(B):
    """A central difference of <dy, call(x + h v)> along a direction v, and along one of the weights, in fp32."""
    gen, (x,), _, positions, freq = inputs(5, 32, 24, (3,), (F32,), 11, (F32,))
    x, w = torch.randn(x.shape, device="cuda", generator=gen), 1 + 0.3 * torch.randn(32, device="cuda", generator=gen)
    dy, v, u = torch.randn(x.shape, device="cuda", generator=gen), torch.randn(x.shape, device="cuda", generator=gen), torch.randn(32, device="cuda", generator=gen)
    for layout in ("half", "pairs"):
        def call(x, w):
            y = torch.empty_like(x)
            B.srft_norm_rotary([(x, w, y)], positions, freq, EPS, layout=layout, factor=1.5)
            return y.double()
        (dx,), (dw,) = backward(B, [dy], [x], [w], positions, freq, layout, 1.5)
        h, g = 2.0 ** -8, dy.double()
        # the call's roundings, 20 of 2^-24 of at most 1.5 sqrt(2) |n| |w|, over 2 h; the third derivative along v times h^2 / 6, which for rows of
        # 32 channels near 1 is below 30 |v|^3 / |x|^3 of an output's size
        for left, right in (((g * (call(x + h * v, w) - call(x - h * v, w))).sum() / (2 * h), (dx.double() * ((x + h * v).double() - (x - h * v).double())).sum() / (2 * h)),
                            ((g * (call(x, w + h * u) - call(x, w - h * u))).sum() / (2 * h), (dw.double() * ((w + h * u).double() - (w - h * u).double())).sum() / (2 * h))):
            size = float((g.abs() * sizes(call(x, w), 24, layout, 1.0)).sum())
            assert abs(float(left - right)) <= size * (20 * U / h + 30 * h * h), (float(left), float(right))


def test_no_tokens_and_refusals(B):
    x = torch.randn(4, 2, 64, device="cuda")
    y, pos, freq, w = torch.empty_like(x), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(16, dtype=torch.float64, device="cuda"), torch.ones(64, device="cuda")
    space, dw = torch.empty(B.srft_norm_rotary_backward_workspace_bytes(2, 64), dtype=torch.uint8, device="cuda"), torch.full((64,), 3.0, device="cuda")
    B.srft_norm_rotary([], pos, freq, EPS)
    B.srft_norm_rotary([(x[:0], w, y[:0])], pos[:0], freq, EPS)
    B.srft_norm_rotary_backward([(x[:0], x[:0], w, y[:0], dw)], pos[:0], freq, EPS, space)
    torch.cuda.synchronize()
    assert not dw.any()
    for bad in (([(x, w, y[:3])], pos, freq), ([(x, w[:63], y)], pos, freq), ([(x, w.double(), y)], pos, freq), ([(x, w.cpu(), y)], pos, freq), ([(x, w, y)], pos[:3], freq),
                ([(x, w, y)], pos.long(), freq), ([(x, w, y)], pos, freq.float()), ([(x.cpu(), w, y)], pos, freq), ([(x.double(), w, y)], pos, freq)):
        with pytest.raises(ValueError):
            B.srft_norm_rotary(*bad, EPS)
    for bad in ([(x, x, w, y.half(), dw)], [(x, x, w, y, dw[:63])], [(x, x, w, y, dw.half())], [(x[:3], x, w, y, dw)]):
        with pytest.raises(ValueError):
            B.srft_norm_rotary_backward(bad, pos, freq, EPS, space)
    with pytest.raises(ValueError):
        B.srft_norm_rotary_backward([(x, x, w, y, dw)] * 2, pos, freq, EPS, space[:-1])
    wide = torch.empty(4, 2, 128, device="cuda")
    for call, status in ((lambda: B.srft_norm_rotary([(x, w, y)], pos, freq, 0.0), -7), (lambda: B.srft_norm_rotary([(x, w, y)], pos, freq, float("nan")), -7),
                         (lambda: B.srft_norm_rotary([(x, w, y)] * 5, pos, freq, EPS), -7),
                         (lambda: B.srft_norm_rotary([(wide[..., :64], w, wide.flatten()[: x.numel()].view(x.shape))], pos, freq, EPS), -7),     # in place with other strides
                         (lambda: B.srft_norm_rotary_backward([(x, x, w, y, dw), (x, x, w, y.clone(), dw)], pos, freq, EPS, space), -7),         # one dweight for two
                         (lambda: B.srft_norm_rotary_backward([(x, x, w, y, dw)], pos, freq, EPS, None), -1)):
        with pytest.raises(B.SrftError) as e:
            call()
        assert e.value.status == status


def test_native_marshalling_and_ctypes_make_the_same_calls(B):
    """With a stream named the binding goes through ctypes."""
    gen, x, w, positions, freq = inputs(33, 96, 64, (4, 2), (BF16, BF16), 21, (F32, None))
    dy, stream = [torch.randn(t.shape, device="cuda", generator=gen).to(F16) for t in x], torch.cuda.current_stream()
    space = torch.empty(B.srft_norm_rotary_backward_workspace_bytes(2, 96), dtype=torch.uint8, device="cuda")
    results = []
    for s in (None, stream):
        y, dx, dw = [torch.full_like(t, float("nan")) for t in x], [torch.full_like(t, float("nan")) for t in x], [torch.full((96,), float("nan"), device="cuda") for _ in x]
        B.srft_norm_rotary(list(zip(x, w, y)), positions, freq, EPS, layout="pairs", factor=1.5, stream=s)
        B.srft_norm_rotary_backward(list(zip(dy, x, w, dx, [dw[0], None])), positions, freq, EPS, space, layout="pairs", factor=1.5, stream=s)
        torch.cuda.synchronize()
        results.append([*y, *dx, dw[0]])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    for a, b, c in zip(x, w, results[0][:2]):
        check(c, a, b, positions, freq, "pairs", 1.5)


def test_captured_gradients_of_a_step_after_another(B):
    """Forward and backward in one graph, replayed with other rows and positions, an eager backward with a workspace of its own between the replays."""
    n, d, heads = 300, 128, (6, 2)
    gen, x, w, positions, freq = inputs(n, d, 128, heads, (BF16, F32), 21, (F32, F32))
    dy = [torch.randn(t.shape, device="cuda", generator=gen) for t in x]
    y, dx, dw = [torch.empty_like(t) for t in dy], [torch.empty_like(t) for t in x], [torch.empty(d, device="cuda") for _ in x]
    space = torch.empty(B.srft_norm_rotary_backward_workspace_bytes(2, d), dtype=torch.uint8, device="cuda")

    def calls():
        B.srft_norm_rotary(zip(x, w, y), positions, freq, EPS, layout="pairs")
        B.srft_norm_rotary_backward(zip(dy, x, w, dx, dw), positions, freq, EPS, space, layout="pairs")
    calls()                                                  # (first launches load the kernels)
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        calls()
    for step in range(5):
        for t in (*x, *dy):
            t.copy_(torch.randn(t.shape, device="cuda", generator=gen))
        positions.add_(1000 * step + 1)
        for t in (*y, *dx, *dw):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        eager = backward(B, dy, x, w, positions, freq, "pairs", 1.0)
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(dx[i], eager[0][i]) and torch.equal(dw[i], eager[1][i]), (step, i)
            check(y[i], x[i], w[i], positions, freq, "pairs", 1.0)
            check_gradients(dx[i], dw[i], dy[i], x[i], w[i], positions, freq, "pairs", 1.0)
