"""Sliding attention where no row sees the last full page any more: what lies in pages that nobody sees takes no part."""
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


def slide(s, q, scale, recent, sinks, seqs):
    B, out = s.B, torch.full_like(q, float("nan"))
    space = torch.full((B.srft_pool_attention_sliding_workspace_bytes(s.pool, seqs, q.shape[0], q.shape[1]),), 0xFF, dtype=torch.uint8, device="cuda")
    B.srft_pool_attention_sliding(s.pool, seqs, q, scale, recent, sinks, out, space)
    torch.cuda.synchronize()
    return out


def lost_pages(s, new, recent, sinks, pages):
    """The page tables with `pages` in turn in the place of those that no row sees."""
    table = s.table.copy()
    for b, n in enumerate(s.length):
        lowest = max(int(n) - new[b] - recent + 1, 0)
        for j in range(-(-sinks // s.R), min(lowest, int(n) // s.R * s.R) // s.R):
            table[b, j] = pages[(b + j) % len(pages)]
    return table


# (pages of 16 tokens end inside a tile of 64 keys, or of 32 at d > 128; lengths a token or more behind a page's end)
@pytest.mark.parametrize("d,g,bits,R,heads", [(128, 32, 4, 16, 2), (64, 16, 4, 32, 1), (128, 128, 8, 16, 2), (256, 32, 8, 16, 2), (192, 64, 4, 16, 2), (96, 32, 8, 64, 1)])
@pytest.mark.parametrize("new,group", [(1, 4), (2, 12), (9, 6)])        # steps of one block of rows, of two, and chunks
def test_the_last_full_page_is_seen_by_nobody(B, d, g, bits, R, heads, new, group):
    n = 40
    s = Serving(B, d, g, bits, R, heads, n=n, max_length=256, seed=d + R + new, spare=4)
    s.append([R + new + i * 3 % 150 for i in range(n)])
    new = [new] * n
    spare = s.free[:2]                                       # (pages that nobody has written: their scales are not numbers; those of the second are large ones)
    for _, scales, _ in (s.pool.k, s.pool.v):
        scales[int(spare[1])] = 1e30
    q = torch.from_numpy(s.rng.standard_normal((sum(new), heads * group, d))).half().cuda()
    reached = 0
    for recent, sinks in ((1, 1), (2, 4), (1, 17), (7, 33), (1, 0), (3, 50)):
        seqs = s.seqs(new)
        whole = slide(s, q, d ** -0.5, recent, sinks, seqs)
        want, err = s.attention(q.double().cpu().numpy(), new, d ** -0.5, group, HALF_STEP[q.dtype], None,
                                lambda row, token: (token <= row - recent) & (token >= sinks))
        off = np.abs(whole.double().cpu().numpy() - want) - err
        assert np.isfinite(off).all() and off.max() <= 0.0, (float(off.max()), recent, sinks)
        for pages in ((spare[0],), (spare[1],), (-1,), (10 ** 9,), (spare[0], -1, spare[1])):
            table = lost_pages(s, new, recent, sinks, pages)
            reached += int(sum(table[b, int(m) // R - 1] != s.table[b, int(m) // R - 1] for b, m in enumerate(s.length)))
            seqs.page_table.copy_(torch.tensor(table))
            assert torch.equal(slide(s, q, d ** -0.5, recent, sinks, seqs), whole), (recent, sinks, pages)
    assert reached > 0                                       # (sequences whose last full page was one of them)
    s.close()
