"""Starts that give the same new tokens to several sequences: calls keep to their buffers."""
import numpy as np
import pytest
import torch

from tests.paged_util import Serving

pytestmark = pytest.mark.gpu
F16 = torch.float16
GUARD = 1 << 16


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


def ints(a):
    return torch.tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")


def guarded(need):
    whole = torch.full((need + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
    return whole, whole[GUARD: GUARD + need]


def untouched(whole):
    return bool((whole[:GUARD] == 0xA5).all()) and bool((whole[-GUARD:] == 0xA5).all())


@pytest.mark.parametrize("R,starts,lengths", [(16, [0, 1600, 0, 1600], [1600, 0, 1600]), (16, [0, 1024] * 32 + [0], [1024, 5] * 32), (32, [1000, 0, 1000, 0, 1000], [999] * 4),
                                              (16, [0, 700] * 200 + [0], [1 << 30] * 400), (64, [-7, 1 << 30, 3, -2, 640, 0, 640], [640] * 6)])
def test_append_keeps_to_its_workspace(B, R, starts, lengths):
    n_new, n = max(min(x, 1600) for x in starts), len(lengths)
    heads, d, max_length = 2, 64, 2048
    plans = [B.Plan(d, 32, 5 + i) for i in range(2)]
    used = n * (max_length // R)
    pool = B.PagePool.empty(*plans, heads, R, used + 4, 2 * n)
    for _, s, _ in (pool.k, pool.v):
        s.fill_(float("nan"))
    table = np.arange(used).reshape(n, -1)                   # (the last four pages are nobody's)
    seqs = B.PagedSeqs(ints(table), ints(np.arange(2 * n).reshape(n, 2)), ints(lengths), ints(starts), max_new=n_new, max_length=max_length)
    x = torch.randn(n_new, heads, d, device="cuda").half()
    whole, space = guarded(B.srft_pool_append_workspace_bytes(pool, seqs, n_new))
    B.srft_pool_append(pool, seqs, x, x, space)
    torch.cuda.synchronize()
    assert untouched(whole)
    listed, room = int(space[:4].view(torch.int32)), (space.numel() - 16) // 16
    assert 0 <= listed <= room
    for _, s, _ in (pool.k, pool.v):
        filled = ~torch.isnan(s).flatten(1).any(1)
        assert int(filled.sum()) == listed and not bool(filled[-4:].any())
    pool.close()


def test_zeros_behind_the_last_sequence_are_no_overlap(B):
    """A step of two sequences in arrays for four whose rest is zeros."""
    s = Serving(B, 64, 32, 4, 16, 2, n=4, max_length=64, seed=3)
    s.append([20, 40, 0, 0])
    kv = [s.draw(30) for _ in range(2)]
    s.grow([13, 17, 0, 0])
    for i in range(2):
        for b, rows in enumerate((slice(0, 13), slice(13, 30))):
            s.tokens[i][b] = np.concatenate([s.tokens[i][b], kv[i][rows]])
    seqs = s.seqs([13, 17, 0, 0])
    seqs.starts.copy_(ints([0, 13, 30, 0, 0]))
    whole, space = guarded(B.srft_pool_append_workspace_bytes(s.pool, seqs, 30))
    B.srft_pool_append(s.pool, seqs, *[torch.from_numpy(x).cuda() for x in kv], space)
    torch.cuda.synchronize()
    assert untouched(whole)
    for which in (0, 1):
        for b in (0, 1):
            n = int(s.length[b])
            full = n // 16 * 16
            want, scales = s.plans[which].quantize(torch.from_numpy(np.ascontiguousarray(s.tokens[which][b][:full].reshape(-1, 64))).cuda())
            got = s.stored(which, b)
            assert np.array_equal(got[0].reshape(want.shape), want.cpu().numpy()) and np.array_equal(got[1].reshape(scales.shape), scales.cpu().numpy())
            assert np.array_equal(s.window(which, b)[: n - full], s.tokens[which][b][full:])
    s.close()


@pytest.mark.parametrize("n,new,length", [(65, 40, 300), (66, 700, 900), (4096, 32768, 1 << 20)])
def test_attention_keeps_to_its_workspace(B, n, new, length):
    """Every second sequence brings all rows.  The last case comes to more pairs of tiles of keys and blocks of rows than 32 bits count."""
    d, R, heads = 64, 256, 1
    plans = [B.Plan(d, 32, 5 + i) for i in range(2)]
    pool = B.PagePool.empty(*plans, heads, R, 1, 1)
    table = torch.full((n, length // R), -1, dtype=torch.int32, device="cuda")               # (no page is there: a tile costs little)
    windows = torch.full((n, 2), -1, dtype=torch.int32, device="cuda")
    starts = ints([new * (i % 2) for i in range(n + 1)])
    seqs = B.PagedSeqs(table, windows, ints([length] * n), starts, max_new=new, max_length=length)
    if n == 4096:
        tiles = sum((length - new + (r + 1) * 256) // 64 for r in range(new // 256))
        assert tiles * (n // 2) > 1 << 31
    q = torch.randn(new, heads, d, device="cuda").half()
    rows = q.numel() * 2
    out_whole, out = guarded(rows)
    whole, space = guarded(B.srft_pool_attention_workspace_bytes(pool, seqs, new, heads))
    assert space.data_ptr() % 256 == 0
    B.srft_pool_attention(pool, seqs, q, 0.1, out.view(F16).view(new, heads, d), space)
    torch.cuda.synchronize()
    assert untouched(whole) and untouched(out_whole)
    pool.close()
