"""The steps of attention layers as a program makes them: norms and positions of a step's queries and keys, the append of its keys and values, and
attention of a layer that sees everything, of one with a sliding reach and of one whose sequences share their prompt's pages."""
import numpy as np
import pytest
import torch

from tests.paged_util import HALF_STEP, Serving
from tests.test_gpu_norm_rotary import EPS, check as check_norm
from tests.test_gpu_paged_sliding import hidden_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


class Steps:
    """Buffers of steps of n tokens over one pool, and the calls of a step: norm_rotary, append, three kinds of attention."""

    def __init__(self, B, s, new, group, recent, sinks, groups, tokens):
        gen = torch.Generator("cuda")
        gen.manual_seed(7)
        n, d, heads = int(sum(new)), s.d, s.heads
        self.B, self.s, self.new, self.group, self.recent, self.sinks = B, s, list(new), group, recent, sinks
        self.packed = torch.zeros(n, heads * (group + 2), d, dtype=torch.bfloat16, device="cuda")        # q, k and v of a projection, next to each other
        self.q_in, self.k_in = self.packed[:, : heads * group], self.packed[:, heads * group: heads * (group + 1)]
        self.q, self.k, self.v = (torch.empty(n, h, d, dtype=torch.float16, device="cuda") for h in (heads * group, heads, heads))
        self.weights = [(1 + 0.3 * torch.randn(d, device="cuda", generator=gen)).to(torch.bfloat16) for _ in range(2)]
        self.freq = 10000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
        self.positions = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.seqs = s.seqs(self.new)
        to = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")      # noqa: E731
        self.prefixes = B.SharedPrefixes(to(groups), to(tokens))
        self.out = [torch.empty_like(self.q) for _ in range(3)]
        sizes = (B.srft_pool_append_workspace_bytes(s.pool, self.seqs, n), B.srft_pool_attention_workspace_bytes(s.pool, self.seqs, n, heads * group),
                 B.srft_pool_attention_sliding_workspace_bytes(s.pool, self.seqs, n, heads * group),
                 B.srft_pool_attention_shared_workspace_bytes(s.pool, self.seqs, self.prefixes, n, heads * group))
        self.space = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")       # one for all: the calls follow one another on a stream
        self.scale = d ** -0.5

    def calls(self):
        B, s = self.B, self.s
        B.srft_norm_rotary([(self.q_in, self.weights[0], self.q), (self.k_in, self.weights[1], self.k)], self.positions, self.freq, EPS)
        self.v.copy_(self.packed[:, s.heads * (self.group + 1):])
        B.srft_pool_append(s.pool, self.seqs, self.k, self.v, self.space)
        B.srft_pool_attention(s.pool, self.seqs, self.q, self.scale, self.out[0], self.space)
        B.srft_pool_attention_sliding(s.pool, self.seqs, self.q, self.scale, self.recent, self.sinks, self.out[1], self.space)
        B.srft_pool_attention_shared(s.pool, self.seqs, self.prefixes, self.q, self.scale, self.out[2], self.space)

    def inputs(self):
        """The next tokens, where they go, and the sequences with them."""
        s = self.s
        before = s.length.copy()
        s.grow(self.new)
        now = s.seqs(self.new)
        for name in ("page_table", "windows", "lengths", "starts"):
            getattr(self.seqs, name).copy_(getattr(now, name))
        self.positions.copy_(torch.tensor(np.concatenate([np.arange(a, a + t) for a, t in zip(before, self.new)]), dtype=torch.int32))
        self.packed.copy_(torch.from_numpy(s.rng.standard_normal(self.packed.shape)))
        for t in (self.q, self.k, self.v, *self.out):
            t.fill_(float("nan"))
        torch.cuda.synchronize()

    def check(self):
        torch.cuda.synchronize()
        s = self.s
        check_norm(self.q, self.q_in, self.weights[0], self.positions, self.freq, "half", 1.0)
        check_norm(self.k, self.k_in, self.weights[1], self.positions, self.freq, "half", 1.0)
        at = 0
        for b, t in enumerate(self.new):
            for i, x in enumerate((self.k, self.v)):
                s.tokens[i][b] = np.concatenate([s.tokens[i][b], x[at: at + t].cpu().numpy()])
                tail = int(s.length[b]) % s.R
                assert np.array_equal(s.window(i, b)[:tail].view(np.uint16), s.tokens[i][b][int(s.length[b]) - tail:].view(np.uint16)), (b, i)
            at += t
        q = self.q.double().cpu().numpy()
        for out, hidden in zip(self.out, (None, hidden_of(self.recent, self.sinks), None)):
            want, err = s.attention(q, self.new, self.scale, self.group, HALF_STEP[torch.float16], hidden=hidden)
            off = np.abs(out.double().cpu().numpy() - want) - err
            assert np.isfinite(off).all() and off.max() <= 0.0, float(off.max())


def conversations(B, d, g, bits, R, heads, n, prompt, seed):
    """n sequences that go on from one prompt: its pages are in all their tables, its last tokens copied into a window of each."""
    s = Serving(B, d, g, bits, R, heads, n=n, max_length=prompt + 200, seed=seed)
    s.append([prompt] + [0] * (n - 1))
    for b in range(1, n):
        s.table[b, : prompt // R] = s.table[0, : prompt // R]
        s.length[b] = prompt
        for i in range(2):
            s.tokens[i][b] = s.tokens[i][0].copy()
    pairs = torch.tensor([[s.windows[0, 1], s.windows[b, 1]] for b in range(1, n)], dtype=torch.int32, device="cuda")
    B.srft_pool_copy(B.PoolTable([s.pool]), torch.zeros(0, 2, dtype=torch.int32, device="cuda"), pairs)
    return s


@pytest.mark.parametrize("d,g,bits,R,heads,n,prompt,group", [(128, 32, 4, 16, 2, 5, 100, 4), (64, 32, 8, 32, 2, 3, 333, 1), (256, 256, 4, 64, 1, 12, 130, 8)])
def test_a_captured_decode_step(B, d, g, bits, R, heads, n, prompt, group):
    s = conversations(B, d, g, bits, R, heads, n, prompt, seed=d + n)
    steps = Steps(B, s, [1] * n, group, 50, 3, [0, n], [prompt])
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    steps.inputs()
    with torch.cuda.stream(stream):
        steps.calls()                                        # (an ordinary step; first launches load the kernels)
    steps.check()
    with torch.cuda.graph(graph, stream=stream):
        steps.calls()
    for _ in range(R + 5):                                   # past a page of every sequence
        steps.inputs()
        graph.replay()
        steps.check()
    s.close()


def test_chunks_and_decode_steps_in_turn(B):
    s = conversations(B, 128, 32, 4, 16, 2, 4, 200, seed=3)
    for new in ([30, 1, 0, 17], [1, 1, 1, 1], [0, 40, 2, 1], [1, 1, 1, 1]):
        steps = Steps(B, s, new, 4, 64, 10, [0, 4], [200])
        steps.inputs()
        steps.calls()
        steps.check()
    s.close()


def test_calls_on_two_streams_at_once(B):
    """Sliding and shared attention of decode steps and chunks over one pool, a workspace to each stream."""
    s = conversations(B, 128, 32, 4, 16, 2, 6, 1000, seed=3)
    new = [1, 90, 1, 40, 2, 1]
    s.append(new)
    gen = torch.Generator("cuda")
    gen.manual_seed(9)
    q = torch.randn(sum(new), 8, 128, device="cuda", generator=gen).half()
    seqs, to = s.seqs(new), lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")      # noqa: E731
    prefixes = B.SharedPrefixes(to([0, 6]), to([992]))
    streams = [torch.cuda.Stream() for _ in range(2)]
    sizes = [B.srft_pool_attention_sliding_workspace_bytes(s.pool, seqs, *q.shape[:2]), B.srft_pool_attention_shared_workspace_bytes(s.pool, seqs, prefixes, *q.shape[:2])]
    space = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    out = [[torch.full_like(q, float("nan")) for _ in range(8)] for _ in streams]
    torch.cuda.synchronize()
    for i in range(8):
        B.srft_pool_attention_sliding(s.pool, seqs, q, 0.1, 300, 4, out[0][i], space[0], streams[0])
        B.srft_pool_attention_shared(s.pool, seqs, prefixes, q, 0.1, out[1][i], space[1], streams[1])
    torch.cuda.synchronize()
    for got, hidden in zip(out, (hidden_of(300, 4), None)):
        assert all(torch.equal(t, got[0]) for t in got)
        want, err = s.attention(q.double().cpu().numpy(), new, 0.1, 4, HALF_STEP[torch.float16], hidden=hidden)
        off = np.abs(got[0].double().cpu().numpy() - want) - err
        assert np.isfinite(off).all() and off.max() <= 0.0, float(off.max())
    s.close()


@pytest.mark.parametrize("new,group", [([1, 1, 1], 4), ([70, 1, 100], 4)])
def test_pages_past_four_gibibytes(B, new, group):
    """Page numbers whose records begin past 2^32 bytes of codes (8 KB a page), the two kinds of pages in turn."""
    pages = 530_000
    s = Serving(B, 128, 32, 4, 16, 8, n=3, max_length=600, seed=4, spare=pages)
    high = sorted(p for p in s.free if p * 8192 >= 1 << 32)
    assert len(high) > 120
    s.free = [p for pair in zip(range(120), high) for p in pair]
    s.append([400, 0, 0])
    for b in (1, 2):
        s.table[b, :25] = s.table[0, :25]
        s.length[b] = 400
        for i in range(2):
            s.tokens[i][b] = s.tokens[i][0].copy()
    s.append([a + 20 for a in new])
    assert int(s.table[0, :25].max()) * 8192 >= 1 << 32
    q = torch.from_numpy(s.rng.standard_normal((sum(new), 8 * group, 128))).half().cuda()
    seqs, to = s.seqs(new), lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")      # noqa: E731
    prefixes = B.SharedPrefixes(to([0, 3]), to([400]))
    space = torch.empty(max(B.srft_pool_attention_sliding_workspace_bytes(s.pool, seqs, *q.shape[:2]),
                            B.srft_pool_attention_shared_workspace_bytes(s.pool, seqs, prefixes, *q.shape[:2])), dtype=torch.uint8, device="cuda")
    sliding, shared = torch.full_like(q, float("nan")), torch.full_like(q, float("nan"))
    B.srft_pool_attention_sliding(s.pool, seqs, q, 0.1, 150, 20, sliding, space)
    B.srft_pool_attention_shared(s.pool, seqs, prefixes, q, 0.1, shared, space)
    torch.cuda.synchronize()
    for out, hidden in ((sliding, hidden_of(150, 20)), (shared, None)):
        want, err = s.attention(q.double().cpu().numpy(), new, 0.1, group, HALF_STEP[torch.float16], hidden=hidden)
        off = np.abs(out.double().cpu().numpy() - want) - err
        assert np.isfinite(off).all() and off.max() <= 0.0, float(off.max())
    s.close()
