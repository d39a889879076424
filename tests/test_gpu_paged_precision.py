"""What attention over pages must not lose: many small weights behind a dominant one, long sequences, and the exact scores of decode steps."""
import numpy as np
import pytest
import torch

from tests.paged_util import HALF_STEP, Serving

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2605_05699_amd import binding
    binding.lib()
    return binding


def give(s, new, kv):
    """Append kv = [k, v], fp16 [tokens, heads, d] each."""
    s.grow(new)
    at = 0
    for b, t in enumerate(new):
        for i in range(2):
            s.tokens[i][b] = np.concatenate([s.tokens[i][b], kv[i][at: at + t]])
        at += t
    seqs = s.seqs(new)
    space = torch.empty(s.B.srft_pool_append_workspace_bytes(s.pool, seqs, int(sum(new))), dtype=torch.uint8, device="cuda")
    s.B.srft_pool_append(s.pool, seqs, *[torch.from_numpy(x).cuda() for x in kv], space)


@pytest.mark.parametrize("d,bits,behind", [(64, 8, 24.5), (64, 8, 26.0), (128, 4, 28.0), (256, 8, 26.0)])
@pytest.mark.parametrize("rows", [40, 1])
def test_many_small_weights_behind_a_dominant_one(B, d, bits, behind, rows):
    """The first key's weight is 2^behind times every other's, and its value is zero: the others' sum is all there is.  One workgroup has all
    of the keys, so that no other maximum helps.

    A weight of 2^-behind is rounded to fp16 under 2^7 of a row's largest, where the step is 2^-24: off by up to 2^(behind - 32) of it, all
    of them alike.  The exponent, some 18 natural units, comes from fp16 roundings of q' and of the keys: 3 of 2^-11 each.  The record's
    error is no part of it (the definition takes the record), the output's rounding is 2^-11."""
    n, R = 32768 + 77, 256
    s = Serving(B, d, 32, bits, R, 1, n=1, max_length=n + rows, seed=d, lam_spread=0.0)
    rng = np.random.default_rng(1)
    k, v = np.zeros((n + rows, 1, d), np.float16), np.empty((n + rows, 1, d), np.float16)
    k[0, 0] = rng.choice([-4.0, 4.0], d)
    v[:] = rng.choice([-1.0, 1.0], d)
    v[0] = 0.0
    give(s, [n], [k[:n], v[:n]])
    give(s, [rows], [k[n:], v[n:]])
    q = torch.from_numpy(np.repeat(k[:1], rows, 0)).cuda()
    first = (s.values(0, 0)[0, 0] @ s.inverse(0).T) @ k[0, 0].astype(np.float64)               # <q, k> of the record's first key
    scale = behind * np.log(2.0) / first
    for p in s.plans:
        B.srft_plan_set_max_workgroups(p.handle, 1)
    out = s.run(q, [rows], float(scale))
    torch.cuda.synchronize()
    want, _ = s.attention(q.double().cpu().numpy(), [rows], float(np.float32(scale)), 1, HALF_STEP[F16])
    got = out.double().cpu().numpy()
    tolerance = 2.0 ** (behind - 32) + 3 * 2.0 ** -11 * behind * np.log(2.0) * 1.1 + 4 * 2.0 ** -11
    error = np.linalg.norm(got - want, axis=-1) / np.linalg.norm(want, axis=-1)
    assert error.max() <= tolerance, (float(error.max()), tolerance)
    s.close()


@pytest.mark.parametrize("d,g,bits", [(128, 32, 4), (128, 32, 8), (64, 16, 4), (64, 32, 8), (32, 32, 4), (96, 96, 4), (256, 32, 4)])
@pytest.mark.parametrize("new,group", [([1, 1], 8), ([3, 4], 8), ([60, 1], 2)])
def test_channels_whose_codes_are_small_beside_large_queries(B, d, g, bits, new, group):
    """Half of each group's channels have a lambda 2^12 times the others': these have small codes, mostly 0, and a transformed query 2^12 times as large.
    What they add to a score is small, and what their sizes cost has to be too.  Some keys are a hundred times the others, so that an error that all
    of a row's products share is none that cancels.  (As everywhere: three roundings of 2^-11 of each product, 32-bit sums.)"""
    from tests.test_gpu_paged import check, queries
    s = Serving(B, d, g, bits, 32, 2, n=2, max_length=400, seed=d + g, lam_spread=0.3)
    s.pool.close()
    for lam in s.lam:
        lam[1::2] *= np.float32(2.0 ** -12)
    s.plans = [B.Plan(d, g, d + g + i, s.lam[i], bits) for i in range(2)]
    s.pool = B.PagePool(*s.plans, s.pool.k, s.pool.v)
    for more, gain in (([200, 37], 0.01), ([20, 19], 1.0), ([60, 40], 0.01)):
        s.append(more, gain)
    s.append(new, 0.01)
    q = queries(s, sum(new), group, F16)
    scores = [np.abs(q[0, :group].double().cpu().numpy() @ s.inverse(0) @ s.values(0, 0)[:, 0].T).max(), 1e-30]
    scale = float(np.float32(3.0 / max(scores)))
    out = s.run(q, new, scale)
    torch.cuda.synchronize()
    check(s, q, new, scale, out, group)
    s.close()
