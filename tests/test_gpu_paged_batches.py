"""The paged cache over batches as they are served: 63 and more sequences, 17 to 32 rows a key head in every format, tens of thousands of tokens."""
import numpy as np
import pytest
import torch

from tests.paged_util import HALF_STEP, Serving
from tests.test_gpu_paged import FORMATS, check, queries

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


def batch(s, prompts, new):
    s.append([int(x) for x in prompts])
    s.append([int(x) for x in new])
    return [int(x) for x in new]


def stored_as_quantized(s):
    """Every sequence's pages and windows, of K and V, against the quantizer over all of them at once."""
    R, d = s.R, s.d
    for which in (0, 1):
        full = [int(n) // R * R for n in s.length]
        rows = np.concatenate([t[:f] for t, f in zip(s.tokens[which], full)]).reshape(-1, d)
        want_codes, want_scales = (t.cpu().numpy() for t in s.plans[which].quantize(torch.from_numpy(rows).cuda()))
        codes, scales, window = (t.cpu().numpy() for t in (s.pool.k if which == 0 else s.pool.v))
        pages = np.concatenate([s.table[b, : f // R] for b, f in enumerate(full)])
        assert np.array_equal(codes[pages].swapaxes(1, 2).reshape(want_codes.shape), want_codes)
        assert np.array_equal(scales[pages].swapaxes(1, 2).reshape(want_scales.shape).view(np.uint32), want_scales.view(np.uint32))
        for b, f in enumerate(full):
            tail = window[s.windows[b, 1]].swapaxes(0, 1)[: int(s.length[b]) - f]
            assert np.array_equal(tail.view(np.uint16), s.tokens[which][b][f:].view(np.uint16)), b


@pytest.mark.parametrize("n", [62, 63, 64, 65, 257, 1000])
@pytest.mark.parametrize("caps", [0, 5])
@pytest.mark.parametrize("kind", ["decode", "mixed"])
def test_many_short_sequences(B, n, caps, kind):
    """Sequences without tokens lie at the first, the last and the 64th places, and at random ones."""
    rng = np.random.default_rng(n + caps)
    s = Serving(B, 64, 32, 4, 16, 2, n=n, max_length=112, seed=n)
    prompts = rng.integers(0, 60, n)
    new = rng.integers(0, 2, n) if kind == "decode" else np.where(rng.random(n) < 0.1, rng.integers(20, 50, n), rng.integers(0, 3, n))
    for b in (0, 62, 63, 64, n - 1):
        if b < n:
            prompts[b] = new[b] = 0
    new = batch(s, prompts, new)
    torch.cuda.synchronize()
    stored_as_quantized(s)
    q = queries(s, sum(new), 2, F16)
    for p in s.plans:
        B.srft_plan_set_max_workgroups(p.handle, caps)
    out = s.run(q, new, 0.125)
    torch.cuda.synchronize()
    check(s, q, new, 0.125, out, 2)
    s.close()


@pytest.mark.parametrize("d,g,bits,R,heads,transform", FORMATS)
@pytest.mark.parametrize("group,new,dtype", [(8, [3, 4, 1, 0], F16), (32, [1, 1, 0, 1], BF16), (5, [6, 1, 4, 2], F16)])
def test_two_blocks_of_rows_a_key_head(B, d, g, bits, R, heads, transform, group, new, dtype):
    s = Serving(B, d, g, bits, R, heads, n=4, max_length=6 * R + 8, seed=3 * d + g + group, transform=transform)
    new = batch(s, [R - 2, 6 * R, 0, 3 * R + 5], new)
    q = queries(s, sum(new), group, dtype)
    out = s.run(q, new, d ** -0.5)
    torch.cuda.synchronize()
    check(s, q, new, d ** -0.5, out, group)
    s.close()


@pytest.mark.parametrize("new,group", [([1, 1], 8), ([4, 3], 8), ([40, 1], 2)])
@pytest.mark.parametrize("d,bits,R", [(128, 4, 32), (256, 8, 64)])
def test_long_sequences(B, new, group, d, bits, R):
    s = Serving(B, d, 32, bits, R, 1, n=2, max_length=40_100, seed=d + group)
    new = batch(s, [40_000, 17_003], new)
    q = queries(s, sum(new), group, F16)
    out = s.run(q, new, 2.0 * d ** -0.5)
    torch.cuda.synchronize()
    check(s, q, new, 2.0 * d ** -0.5, out, group)
    s.close()


@pytest.mark.parametrize("d,g,bits,group", [(128, 32, 4, 8), (128, 32, 8, 16), (64, 16, 4, 8), (256, 32, 8, 4), (128, 32, 4, 24)])
def test_scores_of_a_decode_step_are_exact_but_for_32_bits(B, d, g, bits, group):
    """Scores of four natural units' spread over 4000 tokens in pages.  What the scan rounds to fp16 is a weight times a scale, and the
    output: 2^-11 of each at most, 2.0e-4 of the size in the root mean square (a uniform error over one binade's mantissas), together 2.9e-4.  32-bit
    sums of scores add less than 1e-4 at that spread, together 3.1e-4.  Queries rounded to fp16,
    without what that leaves, would make it 6e-4, which the definition with that mistake shows."""
    tolerance = 4.5e-4
    s = Serving(B, d, g, bits, 16, 2, n=2, max_length=4000, seed=d + bits, lam_spread=0.2)
    new = batch(s, [3999, 3983], [1, 1])                     # (no token is in a window then)
    q = queries(s, 2, group, F16)
    scores = np.einsum("hgd,nhd->hgn", q[0].double().cpu().numpy().reshape(2, group, d) @ s.inverse(0), s.values(0, 0))
    scale = float(np.float32(4.0 / scores.std()))
    out = s.run(q, new, scale).double().cpu().numpy()
    want, _ = s.attention(q.double().cpu().numpy(), new, scale, group, HALF_STEP[F16])

    def error(x):
        return float(np.sqrt(np.mean((np.linalg.norm(x - want, axis=-1) / np.linalg.norm(want, axis=-1)) ** 2)))
    rotated = (q.double().cpu().numpy() @ s.inverse(0))
    up = 2.0 ** (14 - np.floor(np.log2(np.abs(rotated).max(-1, keepdims=True))))
    planted = ((rotated * up).astype(np.float16) / up) @ np.linalg.inv(s.inverse(0))
    wrong, _ = s.attention(planted, new, scale, group, HALF_STEP[F16])
    assert error(out) <= tolerance, error(out)
    assert np.hypot(error(wrong), 2.9e-4) > tolerance, error(wrong)
    s.close()
