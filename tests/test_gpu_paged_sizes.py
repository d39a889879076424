"""Sizes at which attention over pages is refused: the workspace's call, the call and the header's bounds agree."""
import pytest
import torch

from tests.paged_util import Serving

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


UNITS = 0x7FFFFF00                                           # what units of work stay below


def fits(n_seq, heads, max_length, n_new, group, start=0, n_groups=0):
    """The header's bounds on units of work (start: what a block counts for besides its tiles)."""
    tiles, items = max_length // 32 + 2 + start, n_seq + n_groups
    of_items = 3 * items + 8 if n_groups else 2 * items
    return of_items * heads * tiles < UNITS and ((2 if n_groups else 1) * n_new * group // 256 + items) * heads * max(tiles, 8) < UNITS


@pytest.fixture(scope="module")
def pool(B):
    s = Serving(B, 64, 32, 4, 256, 1, n=32, max_length=512, seed=1)
    s.append([300] * 32)
    yield s
    s.close()


def sequences(s, n_seq, max_length, table=None):
    """The first n_seq of them, with a bound that their lengths do not come near (no call here reads a table of that size but `table`)."""
    to = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")      # noqa: E731
    small = s.B.PagedSeqs(to(s.table[:n_seq]), to(s.windows[:n_seq]), to(s.length[:n_seq]), to(list(range(n_seq + 1))), 1, max_length)
    if table is None:
        small.struct.max_pages = max(1, max_length // s.R)   # (sizes are looked at, nothing else)
    else:
        small = s.B.PagedSeqs(table, small.windows, small.lengths, small.starts, 1, max_length)
    return small


def status(B, call):
    try:
        call()
        return 0
    except B.SrftError as e:
        return e.status


def bound(fit):
    """The largest max_length below 2^30 that fits."""
    low, high = 0, (1 << 30) - 1
    while low < high:
        middle = (low + high + 1) // 2
        low, high = (middle, high) if fit(middle) else (low, middle - 1)
    return low


@pytest.mark.parametrize("n_seq", [1, 31, 32])
def test_sliding(B, pool, n_seq):
    for start, name in ((0, "srft_pool_attention_workspace_bytes"), (6, "srft_pool_attention_sliding_workspace_bytes")):
        last = bound(lambda m: fits(n_seq, 1, m, n_seq, 2, start))
        for max_length in {last, last + 1, last - 192, last + 192, (1 << 30) - 1, 1 << 29, 512}:
            seqs, want = sequences(pool, n_seq, max_length), 0 if max_length <= last and max_length < 1 << 30 else -7
            assert status(B, lambda: getattr(B, name)(pool.pool, seqs, n_seq, 2)) == want, (name, max_length, last)


@pytest.mark.parametrize("n_groups", [0, 1, 16])
def test_shared(B, pool, n_groups):
    to = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")      # noqa: E731
    prefixes = B.SharedPrefixes(to(list(range(n_groups + 1))), to([16] * n_groups))
    last = bound(lambda m: fits(32, 1, m, 32, 2, 6 if n_groups else 0, n_groups))
    assert n_groups == 0 or last < (1 << 30) - 200
    for max_length in {last, last + 1, last - 192, last + 192, (1 << 30) - 1, 512}:
        seqs, want = sequences(pool, 32, max_length), 0 if max_length <= last and max_length < 1 << 30 else -7
        assert status(B, lambda: B.srft_pool_attention_shared_workspace_bytes(pool.pool, seqs, prefixes, 32, 2)) == want, (max_length, last)


def test_between_the_bounds(B, pool):
    """A length that the causal form answers and the sliding form does not: with a reach that covers every length the call is the causal one in this, too."""
    s, max_length = pool, (1 << 30) - 200
    assert fits(32, 1, max_length, 32, 2) and not fits(32, 1, max_length, 32, 2, start=6)
    table = torch.full((32, max_length // s.R), -1, dtype=torch.int32, device="cuda")
    table[:, : s.max_pages] = torch.tensor(s.table)
    seqs = sequences(s, 32, max_length, table)
    q = torch.randn(32, 2, 64, device="cuda").half()
    want, out, none = torch.empty_like(q), torch.full_like(q, float("nan")), torch.full_like(q, 7.0)
    space = torch.empty(B.srft_pool_attention_workspace_bytes(s.pool, seqs, 32, 2), dtype=torch.uint8, device="cuda")
    B.srft_pool_attention(s.pool, seqs, q, 0.1, want, space)
    for stream in (None, torch.cuda.current_stream()):
        out.fill_(float("nan"))
        B.srft_pool_attention_sliding(s.pool, seqs, q, 0.1, max_length, 0, out, space, stream)
        assert torch.equal(out, want)
        with pytest.raises(B.SrftError) as e:
            B.srft_pool_attention_sliding(s.pool, seqs, q, 0.1, max_length - 1, 0, none, space, stream)
        assert e.value.status == -7
    call = B.lib().srft_pool_attention_sliding               # (the call itself, with a workspace that is large enough)
    args = (s.pool.handle, seqs.address, q.data_ptr(), 1, 32, 2, 128, 64, 0.1)
    assert call(*args, 5, 3, none.data_ptr(), 128, 64, space.data_ptr(), None) == -7
    empty = torch.zeros(1, dtype=torch.int32, device="cuda")
    out.fill_(float("nan"))
    B.srft_pool_attention_shared(s.pool, seqs, B.SharedPrefixes(empty, empty[:0]), q, 0.1, out, space)
    assert torch.equal(out, want)
    torch.cuda.synchronize()
    assert bool((none == 7.0).all())


def test_a_refused_reach_is_refused_at_any_size(B, pool):
    s, q = pool, torch.zeros(32, 2, 64, device="cuda").half()
    space = torch.empty(B.srft_pool_attention_sliding_workspace_bytes(s.pool, sequences(s, 32, 512), 32, 2), dtype=torch.uint8, device="cuda")
    for max_length in (0, 1, 512):
        seqs = sequences(s, 32, max_length)
        for recent, sinks in ((0, 0), (0, 1 << 40), (-1, 5), (1, -1), (1 << 40, -1)):
            with pytest.raises(B.SrftError) as e:
                B.srft_pool_attention_sliding(s.pool, seqs, q, 0.1, recent, sinks, q, space)
            assert e.value.status == -7
