"""Sliding attention over pages on the GPU: the last tokens and the first ones, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from tests.paged_util import HALF_STEP, Serving

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


def hidden_of(recent, sinks):
    return lambda row, token: (token <= row - recent) & (token >= sinks)


def slide(s, q, new, scale, recent, sinks, seqs=None, stream=None, fill=0xFF):
    B, seqs, out = s.B, seqs or s.seqs(new), torch.full_like(q, float("nan"))
    space = torch.full((B.srft_pool_attention_sliding_workspace_bytes(s.pool, seqs, q.shape[0], q.shape[1]),), fill, dtype=torch.uint8, device="cuda")
    B.srft_pool_attention_sliding(s.pool, seqs, q, scale, recent, sinks, out, space, stream)
    torch.cuda.synchronize()
    return out


def queries(s, new, group, dtype):
    return torch.from_numpy(s.rng.standard_normal((int(sum(new)), s.heads * group, s.d))).to(dtype).cuda()


def check(s, out, q, new, scale, group, recent, sinks, there=None):
    want, err = s.attention(q.double().cpu().numpy(), new, scale, group, HALF_STEP[q.dtype], there, hidden_of(recent, sinks))
    off = np.abs(out.double().cpu().numpy() - want) - err
    assert np.isfinite(off).all() and off.max() <= 0.0, (float(off.max()), recent, sinks)


FORMATS = [(128, 32, 4, 16, 2, "dft", torch.float16), (64, 32, 4, 32, 1, "dft", torch.bfloat16), (96, 16, 4, 16, 4, "dft", torch.float16),
           (256, 32, 8, 64, 2, "dft", torch.bfloat16), (256, 16, 4, 32, 1, "dft", torch.float16), (128, 128, 8, 128, 1, "dft", torch.float16),
           (192, 64, 4, 16, 2, "dft", torch.float16), (32, 32, 8, 32, 2, "dft", torch.float16), (128, 32, 4, 16, 2, "hadamard", torch.float16),
           (160, 32, 8, 256, 1, "dft", torch.bfloat16), (224, 16, 4, 16, 2, "dft", torch.float16)]
REACHES = [(1, 0), (1, 3), (2, 0), (17, 16), (64, 1), (100, 0), (130, 70), (333, 200)]


@pytest.mark.parametrize("d,g,bits,R,heads,transform,dtype", FORMATS)
@pytest.mark.parametrize("new,group", [((1, 1, 1, 1, 1), 4), ((3, 1, 2, 0, 5), 6), ((40, 1, 97, 300, 2), 3)])
def test_against_the_definition(B, d, g, bits, R, heads, transform, dtype, new, group):
    s = Serving(B, d, g, bits, R, heads, n=5, max_length=700, seed=d + g + sum(new), transform=transform)
    s.append([a + b for a, b in zip(new, (3, 690 - new[1], 200, 123, 390))])
    q = queries(s, new, group, dtype)
    for recent, sinks in REACHES:
        out = slide(s, q, new, d ** -0.5, recent, sinks)
        check(s, out, q, new, d ** -0.5, group, recent, sinks)
    s.close()


@pytest.mark.parametrize("recent,sinks", [(700, 0), (1, 699), (350, 350), (1 << 40, 0), (1, 1 << 40), (1 << 62, 1 << 62)])
def test_what_sees_everything_is_causal_attention(B, recent, sinks):
    s = Serving(B, 128, 32, 4, 16, 2, n=3, max_length=700, seed=1)
    new = [1, 70, 4]
    s.append([700, 200, 40])
    q = queries(s, new, 4, torch.float16)
    assert torch.equal(slide(s, q, new, 0.1, recent, sinks), s.run(q, new, 0.1))
    s.close()


@pytest.mark.parametrize("new", [[1, 1, 1], [150, 1, 60]])
def test_pages_that_nobody_sees_are_not_read(B, new):
    """Their entries in the table name nothing, or a page whose scales are not numbers."""
    s = Serving(B, 128, 32, 4, 16, 2, n=3, max_length=1500, seed=2)
    s.append([1500, 900, 333])
    recent, sinks, group = 200, 20, 4
    q = queries(s, new, group, torch.float16)
    whole = slide(s, q, new, 0.09, recent, sinks)
    check(s, whole, q, new, 0.09, group, recent, sinks)
    table, spare = s.table.copy(), s.free[0]                 # (a page that nobody has written: its scales are not numbers)
    for b, n in enumerate(s.length):
        lowest = max(int(n) - new[b] - recent + 1, 0)
        for j in range(-(-sinks // 16), lowest // 16):
            table[b, j] = (-1, 10 ** 9, spare)[j % 3]
    seqs = s.seqs(new)
    seqs.page_table.copy_(torch.tensor(table))
    assert torch.equal(slide(s, q, new, 0.09, recent, sinks, seqs), whole)
    s.close()


@pytest.mark.parametrize("new", [[1, 1, 1], [150, 1, 60]])
def test_pages_that_do_not_exist_are_not_seen(B, new):
    s = Serving(B, 96, 32, 4, 16, 2, n=3, max_length=600, seed=3)
    s.append([600, 500, 333])
    there = []
    for b, n in enumerate(s.length):
        mask = np.ones(int(n), bool)
        for j in s.rng.choice(int(n) // 16, 9, replace=False):
            s.table[b, j] = -5
            mask[16 * j: 16 * j + 16] = False
        there.append(mask)
    group = 4
    q = queries(s, new, group, torch.float16)
    held = s.table.copy()
    seqs = s.seqs(new)
    s.table[s.table < 0] = 0                                 # (what the definition reads there is not seen)
    for recent, sinks in ((5, 0), (40, 17), (250, 1)):
        out = slide(s, q, new, 0.1, recent, sinks, seqs)
        check(s, out, q, new, 0.1, group, recent, sinks, there)
    assert (held < 0).any()
    s.close()


def test_rows_that_see_nothing_are_zero(B):
    s = Serving(B, 64, 32, 4, 16, 2, n=2, max_length=64, seed=4)
    s.append([32, 48])
    s.table[:] = -1                                          # no page exists and no token is behind the pages
    for new in ([1, 1], [30, 40]):
        q = queries(s, new, 2, torch.float16)
        assert not slide(s, q, new, 0.1, 7, 3).any()
    # more new tokens than tokens: those in front of the first one see nothing
    seqs = s.seqs([4, 4])
    seqs.lengths.fill_(2)
    seqs.windows.copy_(torch.tensor(s.slots))
    s.pool.k[2].fill_(1.0)
    s.pool.v[2].fill_(1.0)
    out = slide(s, queries(s, [4, 4], 2, torch.float16), [4, 4], 0.1, 1, 0, seqs)
    assert not out[[0, 1, 4, 5]].any() and bool((out[[2, 3, 6, 7]].float() - 1.0).abs().max() < 2e-3)
    s.close()


@pytest.mark.parametrize("workgroups", [1, 2, 3, 17, 0])
def test_any_number_of_workgroups(B, workgroups):
    s = Serving(B, 128, 32, 4, 16, 2, n=70, max_length=400, seed=5)
    length = s.rng.integers(1, 400, 70)
    s.append(list(length))
    for new in (np.ones(70, int), np.where(np.arange(70) % 9 == 0, np.minimum(length, 30), 1)):
        q = queries(s, new, 4, torch.float16)
        B.srft_plan_set_max_workgroups(s.plans[0].handle, workgroups)
        out = slide(s, q, list(new), 0.1, 90, 6)
        check(s, out, q, list(new), 0.1, 4, 90, 6)
    B.srft_plan_set_max_workgroups(s.plans[0].handle, 0)
    s.close()


@pytest.mark.parametrize("workgroups", [1, 3, 40, 0])
@pytest.mark.parametrize("recent", [33, 1000])
def test_more_blocks_of_rows_than_lanes(B, workgroups, recent):
    """75 blocks of 256 rows to a key head of the second sequence, behind and in front of others; with 1000 seen, everything."""
    s = Serving(B, 64, 32, 4, 16, 2, n=5, max_length=400, seed=19)
    new, group = [17, 300, 0, 1, 40], 64
    s.append([a + b for a, b in zip(new, (20, 70, 30, 100, 0))])
    q = queries(s, new, group, torch.float16)
    B.srft_plan_set_max_workgroups(s.plans[0].handle, workgroups)
    out = slide(s, q, new, 0.1, recent, 5)
    check(s, out, q, new, 0.1, group, recent, 5)
    B.srft_plan_set_max_workgroups(s.plans[0].handle, 0)
    s.close()


@pytest.mark.parametrize("workgroups", [1, 7, 0])
@pytest.mark.parametrize("recent", [20, 1000])
def test_blocks_of_rows_that_see_nothing(B, workgroups, recent):
    """More new tokens than tokens, in chunks of several key heads and sequences: the rows in front of the first token are zero, the others as ever."""
    s = Serving(B, 64, 32, 4, 16, 2, n=3, max_length=400, seed=20)
    s.append([60, 70, 33])
    new, group = [150, 300, 33], 16
    seqs, q = s.seqs(new), queries(s, new, group, torch.float16)
    B.srft_plan_set_max_workgroups(s.plans[0].handle, workgroups)
    out = slide(s, q, new, 0.1, recent, 3, seqs)
    B.srft_plan_set_max_workgroups(s.plans[0].handle, 0)
    seeing = torch.cat([torch.arange(a + n - m, a + n) for a, n, m in zip((0, 150, 450), new, (60, 70, 33))]).cuda()
    nothing = torch.ones(sum(new), dtype=torch.bool, device="cuda")
    nothing[seeing] = False
    assert not out[nothing].any()
    check(s, out[seeing], q[seeing], [60, 70, 33], 0.1, group, recent, 3)
    s.close()


def test_captured_steps_over_growing_sequences(B):
    """One graph, replayed with the next step's table, windows and lengths, beside eager calls on another stream and workspace."""
    s = Serving(B, 128, 32, 4, 16, 2, n=4, max_length=300, seed=6)
    s.append([30, 100, 1, 250])
    new, group, recent, sinks = [1] * 4, 4, 37, 5
    seqs, q = s.seqs(new), queries(s, new, group, torch.float16)
    out = torch.empty_like(q)
    space = torch.empty(B.srft_pool_attention_sliding_workspace_bytes(s.pool, seqs, 4, q.shape[1]), dtype=torch.uint8, device="cuda")
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        B.srft_pool_attention_sliding(s.pool, seqs, q, 0.1, recent, sinks, out, space)       # (first launches load the kernels)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        B.srft_pool_attention_sliding(s.pool, seqs, q, 0.1, recent, sinks, out, space)
    for step in range(20):
        s.append(new)
        now = s.seqs(new)
        for name in ("page_table", "windows", "lengths", "starts"):
            getattr(seqs, name).copy_(getattr(now, name))
        q.copy_(queries(s, new, group, torch.float16))
        torch.cuda.synchronize()
        out.fill_(float("nan"))
        graph.replay()
        eager = slide(s, q, new, 0.1, recent, sinks, now)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), step
        check(s, out, q, new, 0.1, group, recent, sinks)
    s.close()


def test_strides_streams_and_repeats(B):
    s = Serving(B, 64, 32, 8, 32, 2, n=3, max_length=500, seed=7)
    s.append([500, 77, 222])
    new, group = [20, 1, 3], 4
    wide = torch.full((24, 8, 80), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[..., :64] = queries(s, new, group, torch.bfloat16)
    q, seqs = wide[..., :64], s.seqs(new)
    out = torch.full((24, 9, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    space = torch.empty(B.srft_pool_attention_sliding_workspace_bytes(s.pool, seqs, 24, 8), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    B.srft_pool_attention_sliding(s.pool, seqs, q, -0.13, 45, 9, out[:, :8, :64], space, stream)
    torch.cuda.synchronize()
    check(s, out[:, :8, :64], q, new, -0.13, group, 45, 9)
    assert bool((out[:, 8] == 7.0).all()) and bool((out[..., 64:] == 7.0).all())
    again = slide(s, q, new, -0.13, 45, 9, fill=0)
    assert torch.equal(again, out[:, :8, :64])
    s.close()


@pytest.mark.parametrize("gains", [(1000.0, 1e-3, 1.0), (1e-3, 300.0, 0.1), (1e-4, 1e-4, 1e-4)])
@pytest.mark.parametrize("q_gain,dtype", [(1.0, torch.float16), (1e5, torch.bfloat16), (1e-8, torch.bfloat16)])
@pytest.mark.parametrize("new", [[1, 3], [1, 70]])
def test_magnitudes_of_first_and_last_tokens(B, gains, q_gain, dtype, new):
    """What lies between them is of another size, and seen by no row."""
    s = Serving(B, 128, 32, 4, 16, 2, n=2, max_length=500, seed=17, lam_spread=1.5)
    for gain, tokens in zip(gains, ([16, 16], [160, 240], [80, 150])):
        s.append(tokens, gain)
    s.append(new, gains[2])
    q = (q_gain * queries(s, new, 4, torch.float32)).to(dtype)
    scale = 0.09 / (max(gains[0], gains[2]) * q_gain)
    out = slide(s, q, new, scale, 70, 16)
    check(s, out, q, new, scale, 4, 70, 16)
    s.close()


@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0, 1e-30])
def test_softmax_scales(B, scale):
    s = Serving(B, 64, 32, 8, 16, 2, n=2, max_length=300, seed=18)
    s.append([100, 200])
    new = [1, 60]
    s.append(new)
    q = queries(s, new, 2, torch.float16)
    check(s, slide(s, q, new, scale, 33, 20), q, new, scale, 2, 33, 20)
    s.close()


def test_refusals(B):
    s = Serving(B, 64, 32, 4, 16, 2, n=2, max_length=64, seed=8)
    s.append([20, 30])
    seqs, q = s.seqs([1, 1]), torch.zeros(2, 4, 64, dtype=torch.float16, device="cuda")
    space = torch.empty(B.srft_pool_attention_sliding_workspace_bytes(s.pool, seqs, 2, 4), dtype=torch.uint8, device="cuda")
    for bad, kind in (((q, 0.1, 0, 0, q), -7), ((q, 0.1, -1, 0, q), -7), ((q, 0.1, 1, -1, q), -7), ((q, float("inf"), 1, 1, q), -7)):
        with pytest.raises(B.SrftError) as e:
            B.srft_pool_attention_sliding(s.pool, seqs, *bad, space)
        assert e.value.status == kind
    for bad in ((q.float(), 0.1, 1, 0, q), (q, 0.1, 1, 0, q[:1]), (q, 0.1, 1, 0, q.bfloat16()), (q, 0.1, 1 << 63, 0, q), (q, 0.1, 1, 1 << 64, q)):
        with pytest.raises(ValueError):
            B.srft_pool_attention_sliding(s.pool, seqs, *bad, space)
    with pytest.raises(ValueError):
        B.srft_pool_attention_sliding(s.pool, seqs, q, 0.1, 1, 0, q, space[:-1])
    s.close()
