"""The native marshalling of rotary positions and of the paged cache against the same calls through ctypes: equal to the bit, and the
same refusals."""
import pytest
import torch

from tests.paged_util import Serving

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
NAMES = ("rotary", "pool_append", "pool_attention", "pool_copy")


@pytest.fixture(scope="module")
def B():
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


def through(B, monkeypatch, native):
    """The same calls, natively or not: (results, what was raised); native calls are counted."""
    made = dict.fromkeys(NAMES, 0)
    for name in NAMES:
        f = getattr(B._marshal, name)

        def call(*a, f=f, name=name):
            status = f(*a) if native else None
            made[name] += status is not None
            return status
        monkeypatch.setattr(B, "_fast_" + name, call)
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(7, 6, 64, generator=gen, device="cuda")
    pos, freq = torch.arange(7, dtype=torch.int32, device="cuda") * 1000, 10000.0 ** -torch.linspace(0, 1, 16, dtype=torch.float64, device="cuda")
    out = [torch.empty(7, 6, 64, dtype=t, device="cuda") for t in (torch.float32, F16, BF16)]
    B.srft_rotary([(x, out[0]), (x.half(), out[1]), (x[:, :4].bfloat16(), out[2][:, 2:])], pos, freq, layout="pairs", factor=0.5)
    B.srft_rotary(((x, out[0]) for _ in range(1)), pos, freq, inverse=True)
    got = [out[0], out[1], out[2][:, 2:]]
    s = Serving(B, 64, 16, 8, 16, 2, n=2, max_length=96, seed=3)
    s.append([40, 9])
    s.append([1, 12])
    q = torch.randn(13, 8, 64, generator=gen, device="cuda")
    for t in (F16, BF16):
        got.append(s.run(q.to(t)[:, 1:5], [1, 12], 0.3))
    pairs = torch.tensor([[0, s.pool.n_pages - 1]], dtype=torch.int32, device="cuda")
    B.srft_pool_copy(B.PoolTable([s.pool]), pairs, pairs[:0])
    got += [*s.pool.k, *s.pool.v]
    raised, space = [], torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    seqs, k = s.seqs([1, 12]), torch.zeros(13, 2, 64, dtype=F16, device="cuda")
    for call in (lambda: B.srft_rotary([(x, out[1].double())], pos, freq), lambda: B.srft_rotary([(x, out[0])] * 5, pos, freq),
                 lambda: B.srft_rotary([(x, out[0])], pos.long(), freq), lambda: B.srft_rotary([(x[..., :30], out[0][..., :30])], pos, freq),
                 lambda: B.srft_pool_append(s.pool, seqs, k, k[:, :1], space), lambda: B.srft_pool_append(s.pool, seqs, k, k, space[:16]),
                 lambda: B.srft_pool_append(s.pool, seqs, k, k, space[8:]), lambda: B.srft_pool_attention(s.pool, seqs, q, 1.0, q, space),
                 lambda: B.srft_pool_attention(s.pool, seqs, q.half(), float("nan"), q.half(), space), lambda: B.srft_pool_copy(B.PoolTable([s.pool]), pairs[0], pairs),
                 lambda: B.srft_pool_copy(B.PoolTable([s.pool]), pairs.long(), pairs)):
        with pytest.raises((ValueError, B.SrftError)) as e:
            call()
        raised.append((type(e.value), str(e.value)))
    torch.cuda.synchronize()
    s.close()
    return [g.clone() for g in got], raised, made


@pytest.mark.parametrize("side", [False, True])
def test_native_calls_are_the_same(B, monkeypatch, side):
    def both():
        return [through(B, monkeypatch, native) for native in (True, False)]
    if side:
        with torch.cuda.stream(torch.cuda.Stream()):
            (got, raised, made), (want, also, none) = both()
    else:
        (got, raised, made), (want, also, none) = both()
    assert all(made.values()) and not any(none.values())
    assert raised == also
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.uint8) if a.is_contiguous() else a, b.view(torch.uint8) if b.is_contiguous() else b)
