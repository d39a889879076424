"""Attention of sequences that have their first pages in common, on the GPU, against the definition in 64 bits."""
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


def fork(s, groups, pages, gain=1.0):
    """The first pages[g] pages of the sequences groups[g] .. groups[g + 1] are those of the first of them."""
    first = np.zeros(s.n, int)
    for g, p in enumerate(pages):
        if groups[g] < groups[g + 1]:
            first[groups[g]] = p * s.R
    s.append(list(first), gain)
    for g, p in enumerate(pages):
        for b in range(groups[g] + 1, groups[g + 1]):
            s.table[b, :p] = s.table[groups[g], :p]
            s.length[b] = p * s.R
            for i in range(2):
                s.tokens[i][b] = s.tokens[i][groups[g]].copy()
    return s


def prefixes_of(B, groups, tokens):
    to = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")      # noqa: E731
    return B.SharedPrefixes(to(groups), to(tokens))


def share(s, q, new, scale, prefixes, seqs=None, stream=None, fill=0xFF):
    B, seqs, out = s.B, seqs or s.seqs(new), torch.full_like(q, float("nan"))
    space = torch.full((B.srft_pool_attention_shared_workspace_bytes(s.pool, seqs, prefixes, q.shape[0], q.shape[1]),), fill, dtype=torch.uint8, device="cuda")
    B.srft_pool_attention_shared(s.pool, seqs, prefixes, q, scale, out, space, stream)
    torch.cuda.synchronize()
    return out


def queries(s, new, group, dtype):
    return torch.from_numpy(s.rng.standard_normal((int(sum(new)), s.heads * group, s.d))).to(dtype).cuda()


def check(s, out, q, new, scale, group, there=None):
    want, err = s.attention(q.double().cpu().numpy(), new, scale, group, HALF_STEP[q.dtype], there)
    off = np.abs(out.double().cpu().numpy() - want) - err
    assert np.isfinite(off).all() and off.max() <= 0.0, float(off.max())


FORMATS = [(128, 32, 4, 16, 2, "dft", torch.float16), (64, 32, 4, 32, 1, "dft", torch.bfloat16), (96, 16, 4, 16, 4, "dft", torch.float16),
           (256, 32, 8, 64, 2, "dft", torch.bfloat16), (256, 16, 4, 32, 1, "dft", torch.float16), (128, 128, 8, 128, 1, "dft", torch.float16),
           (192, 64, 4, 16, 2, "dft", torch.float16), (32, 32, 8, 32, 2, "dft", torch.float16), (128, 32, 4, 16, 2, "hadamard", torch.float16),
           (160, 32, 8, 256, 1, "dft", torch.bfloat16), (224, 16, 4, 16, 2, "dft", torch.float16)]
#: new tokens of nine sequences in the groups 0 .. 2, 2 .. 3, 3 .. 3, 3 .. 8 (the last one in none): decode steps, steps of a few tokens, one of whose
#: sequences has none, chunks and both; rows of a chunk in a group that has few of them; groups of many rows in calls of few
STEPS = [((5, 1, 3, 60, 1, 0, 1, 1, 2), 4), ((1,) * 9, 4), ((1,) * 9, 1), ((2, 1, 4, 0, 3, 1, 5, 1, 1), 3), ((3,) * 9, 8), ((40, 1, 2, 70, 1, 0, 150, 1, 20), 3), ((1,) * 9, 24),
         ((1,) * 9, 14), ((1, 1, 1, 1, 1, 0, 1, 0, 1), 18)]
GROUPS = [0, 2, 3, 3, 8]


@pytest.mark.parametrize("d,g,bits,R,heads,transform,dtype", FORMATS)
@pytest.mark.parametrize("new,group", STEPS)
def test_against_the_definition(B, d, g, bits, R, heads, transform, dtype, new, group):
    pages = [1 + 200 // R, 2, 1, 1 + 300 // R]
    s = fork(Serving(B, d, g, bits, R, heads, n=9, max_length=1200, seed=d + g + sum(new) + group, transform=transform), GROUPS, pages)
    own = [3, 17, 1, 2 * R + 5, 1, R, 30, 0, 70]
    s.append([a + b for a, b in zip(new, own)])
    q = queries(s, new, group, dtype)
    out = share(s, q, new, d ** -0.5, prefixes_of(B, GROUPS, [R * p + (R // 2 if p == pages[0] else 0) for p in pages]))
    check(s, out, q, new, d ** -0.5, group)
    s.close()


@pytest.mark.parametrize("workgroups", [1, 2, 3, 5, 40, 0])
@pytest.mark.parametrize("group", [1, 4])
def test_any_number_of_workgroups(B, workgroups, group):
    """From one workgroup for everything (all rows' keys whole) to shares that split every prefix."""
    n, R = 70, 16
    groups = [0, 1, 30, 33, 66]
    s = fork(Serving(B, 128, 32, 4, R, 2, n=n, max_length=700, seed=5), groups, [3, 20, 37, 8])
    own = s.rng.integers(0, 60, n)
    for new in (np.ones(n, int), np.where(np.arange(n) % 11 == 0, 30, 1)):
        s.append(list(new + own * (s.length < 600)))
        B.srft_plan_set_max_workgroups(s.plans[0].handle, workgroups)
        q = queries(s, new, group, torch.float16)
        out = share(s, q, list(new), 0.1, prefixes_of(B, groups, [48, 320, 592, 128]))
        check(s, out, q, list(new), 0.1, group)
    B.srft_plan_set_max_workgroups(s.plans[0].handle, 0)
    s.close()


@pytest.mark.parametrize("workgroups", [1, 3, 40, 0])
def test_more_blocks_of_rows_than_lanes(B, workgroups):
    """75 blocks of 256 rows to a key head of one sequence's own tokens, and 80 of what its group has in common."""
    s = fork(Serving(B, 64, 32, 4, 16, 2, n=5, max_length=400, seed=19), [0, 3, 5], [4, 3])
    new, group = [17, 300, 3, 1, 40], 64
    s.append([a + b for a, b in zip(new, (0, 7, 30, 20, 0))])
    q = queries(s, new, group, torch.float16)
    B.srft_plan_set_max_workgroups(s.plans[0].handle, workgroups)
    out = share(s, q, new, 0.1, prefixes_of(B, [0, 3, 5], [64, 48]))
    check(s, out, q, new, 0.1, group)
    B.srft_plan_set_max_workgroups(s.plans[0].handle, 0)
    s.close()


def test_only_the_first_sequence_of_a_group_has_its_table_read_for_the_pages_in_common(B):
    s = fork(Serving(B, 128, 32, 4, 16, 2, n=6, max_length=700, seed=9), [0, 3, 6], [20, 30])
    s.append([1, 40, 20, 7, 16, 5])
    for new in ([1] * 6, [0, 2, 1, 5, 1, 0], [1, 35, 18, 2, 1, 3]):
        q = queries(s, new, 4, torch.float16)
        whole = share(s, q, new, 0.1, prefixes_of(B, [0, 3, 6], [320, 480]))
        check(s, whole, q, new, 0.1, 4)
        table = s.table.copy()
        for b0, b1, p in ((0, 3, 20), (3, 6, 30)):
            with_new = [b for b in range(b0, b1) if new[b] > 0]
            common = min(p, *((int(s.length[b]) - new[b]) // 16 for b in with_new))
            for b in range(b0, b1):
                if b != with_new[0]:
                    table[b, :common] = [-1, 10 ** 9][b % 2]
        seqs = s.seqs(new)
        seqs.page_table.copy_(torch.tensor(table))
        assert torch.equal(share(s, q, new, 0.1, prefixes_of(B, [0, 3, 6], [320, 480]), seqs), whole)
    s.close()


def test_a_prefix_counts_as_far_as_all_hold_it_without_their_new_tokens(B):
    """The sequences' new tokens reach into the pages that they have in common: as much as is in front of them is shared."""
    R = 16
    s = fork(Serving(B, 64, 32, 4, R, 2, n=4, max_length=300, seed=10), [0, 4], [10])
    new = [1, 30, 47, 3]                                     # (of the pages in common: queries of tokens that the cache holds already)
    q = queries(s, new, 4, torch.float16)
    for tokens in (0, 5, 16, 113, 160, 161, 10 ** 6, 2 ** 31 - 1, -7):
        out = share(s, q, new, 0.1, prefixes_of(B, [0, 4], [tokens]))
        check(s, out, q, new, 0.1, 4)
    s.close()


def test_pages_in_common_that_do_not_exist_are_not_seen(B):
    R = 16
    s = fork(Serving(B, 96, 32, 4, R, 2, n=5, max_length=600, seed=11), [0, 5], [30])
    s.append([1, 30, 17, 60, 5])
    lost = [2, 3, 17, 29]
    s.table[:, lost] = 10 ** 6
    there = []
    for b in range(5):
        mask = np.ones(int(s.length[b]), bool)
        for j in lost:
            mask[R * j: R * j + R] = False
        there.append(mask)
    for new in ([1] * 5, [1, 28, 10, 50, 2]):
        q, seqs = queries(s, new, 4, torch.float16), s.seqs(new)
        out = share(s, q, new, 0.1, prefixes_of(B, [0, 5], [480]), seqs)
        held, s.table = s.table, np.where(s.table == 10 ** 6, 0, s.table)
        check(s, out, q, new, 0.1, 4, there)
        s.table = held
    # no page in common exists
    s.table[:, :30] = -1
    new = [1] * 5
    q, seqs = queries(s, new, 4, torch.float16), s.seqs(new)
    out = share(s, q, new, 0.1, prefixes_of(B, [0, 5], [480]), seqs)
    s.table[:, :30] = 0
    check(s, out, q, new, 0.1, 4, [np.arange(int(n)) >= 480 for n in s.length])
    s.close()


def test_groups_out_of_order_stay_within_the_sequences(B):
    """A bound below the one in front of it, or past the last sequence, is taken as that; tables that are the same give the same answers."""
    s = fork(Serving(B, 64, 32, 4, 16, 2, n=6, max_length=300, seed=12), [0, 6], [8])
    s.append([1, 2, 3, 20, 5, 6])
    new = [1] * 6
    q = queries(s, new, 4, torch.float16)
    for groups in ([0, 4, 2, 6], [-5, 3, 3, 100], [5, 0, 0, 6], [2 ** 31 - 1] * 4, [-2 ** 31, 2, 2 ** 31 - 1, 3]):
        out = share(s, q, new, 0.1, prefixes_of(B, groups, [128, 128, 128]))
        check(s, out, q, new, 0.1, 4)
    s.close()


def test_no_groups_are_causal_attention(B):
    s = fork(Serving(B, 128, 32, 4, 16, 2, n=3, max_length=300, seed=13), [0, 3], [8])
    s.append([1, 50, 3])
    new = [1, 40, 2]
    q = queries(s, new, 4, torch.float16)
    whole = s.run(q, new, 0.1)
    assert torch.equal(share(s, q, new, 0.1, prefixes_of(B, [0], [])), whole)
    check(s, whole, q, new, 0.1, 4)
    for groups in ([0, 1, 2, 3], [1, 1], [3, 3]):            # (one sequence, or none: nothing is shared; the keys may be shared out in other parts)
        check(s, share(s, q, new, 0.1, prefixes_of(B, groups, [128] * (len(groups) - 1))), q, new, 0.1, 4)
    s.close()


def test_captured_steps_over_growing_sequences(B):
    """One graph of a decode step, replayed while the sequences grow and the groups change, beside eager calls with a workspace of their own."""
    s = fork(Serving(B, 128, 32, 4, 16, 2, n=5, max_length=300, seed=14), [0, 5], [9])
    s.append([1, 20, 3, 15, 40])
    new, group = [1] * 5, 4
    seqs, q, prefixes = s.seqs(new), queries(s, new, group, torch.float16), prefixes_of(B, [0, 3, 5], [144, 144])
    out = torch.empty_like(q)
    space = torch.empty(B.srft_pool_attention_shared_workspace_bytes(s.pool, seqs, prefixes, 5, q.shape[1]), dtype=torch.uint8, device="cuda")
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        B.srft_pool_attention_shared(s.pool, seqs, prefixes, q, 0.1, out, space)             # (first launches load the kernels)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        B.srft_pool_attention_shared(s.pool, seqs, prefixes, q, 0.1, out, space)
    for step in range(20):
        s.append(new)
        now = s.seqs(new)
        for name in ("page_table", "windows", "lengths", "starts"):
            getattr(seqs, name).copy_(getattr(now, name))
        prefixes.groups.copy_(torch.tensor([[0, 3, 5], [0, 5, 5], [1, 2, 4], [0, 2, 5]][step % 4]))
        prefixes.tokens.copy_(torch.tensor([[144, 100], [144, 0], [144, 144], [32, 144]][step % 4]))
        q.copy_(queries(s, new, group, torch.float16))
        torch.cuda.synchronize()
        out.fill_(float("nan"))
        graph.replay()
        eager = share(s, q, new, 0.1, prefixes, now)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), step
        check(s, out, q, new, 0.1, group)
    s.close()


def test_strides_streams_and_repeats(B):
    s = fork(Serving(B, 64, 32, 8, 32, 2, n=3, max_length=500, seed=15), [0, 3], [7])
    s.append([100, 77, 222])
    new, group = [20, 1, 3], 4
    wide = torch.full((24, 8, 80), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[..., :64] = queries(s, new, group, torch.bfloat16)
    q, seqs, prefixes = wide[..., :64], s.seqs(new), prefixes_of(B, [0, 3], [224])
    out = torch.full((24, 9, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    space = torch.empty(B.srft_pool_attention_shared_workspace_bytes(s.pool, seqs, prefixes, 24, 8), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    B.srft_pool_attention_shared(s.pool, seqs, prefixes, q, -0.13, out[:, :8, :64], space, stream)
    torch.cuda.synchronize()
    check(s, out[:, :8, :64], q, new, -0.13, group)
    assert bool((out[:, 8] == 7.0).all()) and bool((out[..., 64:] == 7.0).all())
    assert torch.equal(share(s, q, new, -0.13, prefixes, fill=0), out[:, :8, :64])
    s.close()


@pytest.mark.parametrize("gains", [(1000.0, 1e-3), (1e-3, 300.0), (1e-4, 1e-4)])
@pytest.mark.parametrize("q_gain,dtype", [(1.0, torch.float16), (1e5, torch.bfloat16), (1e-8, torch.bfloat16)])
@pytest.mark.parametrize("new", [[1, 1, 3], [1, 70, 20]])
def test_magnitudes_of_what_is_common_and_of_what_is_not(B, gains, q_gain, dtype, new):
    s = fork(Serving(B, 128, 32, 4, 16, 2, n=3, max_length=500, seed=17, lam_spread=1.5), [0, 3], [12], gains[0])
    s.append([a + b for a, b in zip(new, (7, 100, 44))], gains[1])
    q = q_gain * queries(s, new, 4, torch.float32)
    q = q.to(dtype)
    scale = 0.09 / (max(gains) * q_gain)
    out = share(s, q, new, scale, prefixes_of(B, [0, 3], [192]))
    check(s, out, q, new, scale, 4)
    s.close()


@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0, 1e-30])
def test_softmax_scales(B, scale):
    s = fork(Serving(B, 64, 32, 8, 16, 2, n=4, max_length=500, seed=18), [0, 2, 4], [12, 9])
    new = [1, 60, 2, 1]
    s.append([a + b for a, b in zip(new, (7, 100, 44, 1))])
    q = queries(s, new, 2, torch.float16)
    out = share(s, q, new, scale, prefixes_of(B, [0, 2, 4], [192, 144]))
    check(s, out, q, new, scale, 2)
    s.close()


def test_refusals(B):
    s = fork(Serving(B, 64, 32, 4, 16, 2, n=2, max_length=64, seed=16), [0, 2], [1])
    s.append([4, 5])
    seqs, q, prefixes = s.seqs([1, 1]), torch.zeros(2, 4, 64, dtype=torch.float16, device="cuda"), prefixes_of(B, [0, 2], [16])
    space = torch.empty(B.srft_pool_attention_shared_workspace_bytes(s.pool, seqs, prefixes, 2, 4), dtype=torch.uint8, device="cuda")
    with pytest.raises(B.SrftError) as e:
        B.srft_pool_attention_shared_workspace_bytes(s.pool, seqs, prefixes_of(B, [0, 1, 2, 2], [16] * 3), 2, 4)         # more groups than sequences
    assert e.value.status == -7
    with pytest.raises(B.SrftError) as e:
        B.srft_pool_attention_shared(s.pool, seqs, prefixes, q, float("nan"), q, space)
    assert e.value.status == -7
    for bad in ((q.float(), 0.1, q), (q, 0.1, q[:1]), (q, 0.1, q.bfloat16())):
        with pytest.raises(ValueError):
            B.srft_pool_attention_shared(s.pool, seqs, prefixes, *bad, space)
    with pytest.raises(ValueError):
        B.srft_pool_attention_shared(s.pool, seqs, prefixes, q, 0.1, q, space[:-1])
    for bad in ((prefixes.groups[:2], prefixes.groups), (prefixes.groups.long(), prefixes.tokens), (prefixes.groups.cpu(), prefixes.tokens), (prefixes.groups, prefixes.tokens[None])):
        with pytest.raises(ValueError):
            B.SharedPrefixes(*bad)
    s.close()
