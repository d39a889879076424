"""The paged cache on the GPU: append, attention and copies, against the definitions in 64 bits (tests/paged_util.py)."""
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


FORMATS = [(128, 32, 4, 16, 2, "dft"), (64, 32, 4, 32, 1, "dft"), (96, 16, 4, 16, 4, "dft"), (256, 32, 8, 64, 2, "dft"), (256, 16, 4, 32, 1, "dft"),
           (128, 128, 8, 128, 3, "dft"), (192, 64, 4, 16, 2, "dft"), (32, 32, 8, 32, 2, "dft"), (128, 32, 4, 16, 2, "hadamard"), (256, 256, 4, 16, 2, "dft"),
           (160, 32, 8, 256, 1, "dft"), (224, 16, 4, 16, 2, "dft"), (256, 64, 4, 16, 2, "dft")]


# ---------------------------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("d,g,bits,R,heads,transform", FORMATS)
def test_append_is_the_quantizer_bit_for_bit_and_the_window_is_exact(B, d, g, bits, R, heads, transform):
    s = Serving(B, d, g, bits, R, heads, n=5, max_length=5 * R + 20, seed=11 * d + g, transform=transform)
    schedule = [[1, 0, R, 2 * R + 3, R - 1], [R, 1, 1, 1, 1], [0, 0, 0, 1, 0], [1, 3 * R, R // 2, R - 4, 2], [R - 1, 1, 5, 0, R + 1]]
    for new in schedule:
        s.append(new)
        torch.cuda.synchronize()
    for which in (0, 1):
        used = set()
        for b in range(s.n):
            n = int(s.length[b])
            full = n // R * R
            assert s.tokens[which][b].shape[0] == n
            codes, scales = s.stored(which, b)
            x = torch.from_numpy(np.ascontiguousarray(s.tokens[which][b][:full].reshape(-1, d))).cuda()
            if full:
                want_codes, want_scales = (t.cpu().numpy() for t in s.plans[which].quantize(x))
                assert np.array_equal(codes.reshape(want_codes.shape), want_codes), (which, b)
                assert np.array_equal(scales.reshape(want_scales.shape).view(np.uint32), want_scales.view(np.uint32)), (which, b)
            assert np.array_equal(s.window(which, b)[: n - full].view(np.uint16), s.tokens[which][b][full:].view(np.uint16)), (which, b)
            used |= set(s.table[b, : n // R].tolist())
        # pages and windows of nobody are as they were
        codes, scales, window = s.pool.k if which == 0 else s.pool.v
        for p in set(range(s.pool.n_pages)) - used:
            assert not codes[p].any() and bool(torch.isnan(scales[p]).all()), p
        for w in set(range(s.pool.n_windows)) - set(s.slots.ravel().tolist()):
            assert bool(torch.isnan(window[w]).all()), w
    s.close()


def test_append_does_not_depend_on_the_split_into_calls(B):
    results = []
    for parts in ([[70, 33]], [[1, 0], [30, 33], [39, 0]], [[16, 17], [54, 16]]):
        s = Serving(B, 128, 32, 4, 16, 2, n=2, max_length=80, seed=5)
        whole = [s.draw(103) for _ in range(2)]
        at = np.array([0, 70])
        for new in parts:
            rows = np.concatenate([np.arange(at[b], at[b] + t) for b, t in enumerate(new)])
            at += new
            s.grow(new)
            seqs = s.seqs(new)
            space = torch.empty(B.srft_pool_append_workspace_bytes(s.pool, seqs, len(rows)), dtype=torch.uint8, device="cuda")
            B.srft_pool_append(s.pool, seqs, *[torch.from_numpy(np.ascontiguousarray(x[rows])).cuda() for x in whole], space)
        torch.cuda.synchronize()
        results.append([x for which in (0, 1) for b in (0, 1) for x in (*s.stored(which, b), s.window(which, b)[: int(s.length[b]) % 16])])
        s.close()
    for other in results[1:]:
        for x, y in zip(results[0], other):
            assert np.array_equal(x.view(np.uint8), y.view(np.uint8))


def test_append_takes_strided_tokens_and_skips_pages_and_windows_that_do_not_exist(B):
    d, R, heads = 128, 16, 2
    s = Serving(B, d, 32, 4, R, heads, n=3, max_length=64, seed=9)
    new = [33, 20, 5]
    packed = torch.from_numpy(np.random.default_rng(1).standard_normal((58, 3, heads, d)).astype(np.float16)).cuda()
    k, v = packed[:, 0].transpose(1, 2).contiguous().transpose(1, 2), packed[:, 2]
    k = torch.empty(58, heads, d + 8, dtype=torch.float16, device="cuda")[:, :, :d].copy_(packed[:, 0])
    s.grow(new)
    s.table[0, 1] = s.pool.n_pages                           # out of range, both ways; a window likewise
    s.table[1, 0] = -7
    bad_window = s.windows[2].copy()
    s.windows[2] = [1 << 30, -1]
    seqs = s.seqs(new)
    space = torch.empty(B.srft_pool_append_workspace_bytes(s.pool, seqs, 58), dtype=torch.uint8, device="cuda")
    B.srft_pool_append(s.pool, seqs, k, v, space)
    torch.cuda.synchronize()
    for which, x in ((0, packed[:, 0]), (1, packed[:, 2])):
        codes, scales, window = s.pool.k if which == 0 else s.pool.v
        want_codes, want_scales = s.plans[which].quantize(x[:16].transpose(0, 1).reshape(-1, d).contiguous())
        page = int(s.table[0, 0])
        assert torch.equal(codes[page].reshape(want_codes.shape), want_codes) and torch.equal(scales[page].reshape(want_scales.shape), want_scales)
        written = [p for p in range(s.pool.n_pages) if not bool(torch.isnan(scales[p]).any())]
        assert written == [page]
        assert torch.equal(window[int(s.windows[0, 1]), :, :1].transpose(0, 1), x[32:33])
        assert torch.equal(window[int(s.windows[1, 1]), :, :4].transpose(0, 1), x[49:53])
        assert bool(torch.isnan(window[bad_window]).all())
    s.close()


# ------------------------------------------------------------------------------------------------------------- attention
def check(s, q, new, scale, out, group, there=None):
    want, bound = s.attention(q.double().cpu().numpy(), new, scale, group, HALF_STEP[q.dtype], there)
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    worst = np.abs(got - want) / bound
    assert worst.max() <= 1.0, (float(worst.max()), np.unravel_index(worst.argmax(), worst.shape))


def queries(s, n, group, dtype, gain=1.0, seed=3):
    x = np.random.default_rng(seed).standard_normal((n, s.heads * group, s.d)) * gain
    return torch.from_numpy(x).cuda().to(dtype)


F16, BF16 = torch.float16, torch.bfloat16


# (prompts, then the new tokens of the step that is tested)
@pytest.mark.parametrize("d,g,bits,R,heads,transform", FORMATS)
@pytest.mark.parametrize("group,dtype", [(1, F16), (6, BF16)])
def test_a_decode_step(B, d, g, bits, R, heads, transform, group, dtype):
    s = Serving(B, d, g, bits, R, heads, n=7, max_length=6 * R + 8, seed=7 * d + g + group, transform=transform)
    s.append([0, 1, R - 1, R, 3 * R + 5, 6 * R, 2 * R])
    new = [1, 1, 1, 1, 1, 0, 1]
    s.append(new)
    q = queries(s, sum(new), group, dtype)
    out = s.run(q, new, d ** -0.5)
    torch.cuda.synchronize()
    check(s, q, new, d ** -0.5, out, group)
    s.close()


@pytest.mark.parametrize("d,g,bits,R,heads,transform", FORMATS)
@pytest.mark.parametrize("group,dtype", [(4, BF16), (3, F16)])
def test_chunks_behind_prefixes(B, d, g, bits, R, heads, transform, group, dtype):
    s = Serving(B, d, g, bits, R, heads, n=4, max_length=4 * R + 310, seed=5 * d + g + group, transform=transform)
    s.append([R + 3, 0, 2 * R, 0])
    new = [130, 300, 1, 40]
    s.append(new)
    q = queries(s, sum(new), group, dtype)
    out = s.run(q, new, d ** -0.5)
    torch.cuda.synchronize()
    check(s, q, new, d ** -0.5, out, group)
    s.close()


@pytest.mark.parametrize("group,new", [(8, [4, 3, 4]), (8, [4, 5, 4]), (32, [1, 2, 9]), (33, [1, 1, 1]), (64, [1, 4, 5]), (1, [32, 33, 31]), (1, [256, 257, 255]),
                                       (5, [51, 52, 103]), (1, [1, 513, 2])])
def test_numbers_of_rows_around_those_where_the_kernels_change(B, group, new):
    s = Serving(B, 64, 32, 4, 16, 2, n=3, max_length=1100, seed=group)
    s.append([100, 77, 500])
    s.append(new)
    q = queries(s, sum(new), group, F16)
    out = s.run(q, new, 0.125)
    torch.cuda.synchronize()
    check(s, q, new, 0.125, out, group)
    s.close()


@pytest.mark.parametrize("caps", [1, 3, 7])
def test_the_same_rows_whatever_the_number_of_workgroups(B, caps):
    """Shares that end inside a sequence, several sequences to a workgroup, whole ones between two parts."""
    s = Serving(B, 128, 32, 4, 16, 2, n=6, max_length=900, seed=21)
    s.append([800, 0, 33, 400, 16, 90])
    new = [1, 70, 1, 20, 2, 64]
    s.append(new)
    q = queries(s, sum(new), 4, F16)
    for p in s.plans:
        B.srft_plan_set_max_workgroups(p.handle, caps)
    out = s.run(q, new, 0.09)
    torch.cuda.synchronize()
    check(s, q, new, 0.09, out, 4)
    s.close()


@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0, 1e-30])
def test_softmax_scales(B, scale):
    s = Serving(B, 128, 32, 4, 16, 2, n=2, max_length=300, seed=33)
    s.append([100, 200])
    new = [1, 60]
    s.append(new)
    q = queries(s, 61, 2, F16)
    out = s.run(q, new, scale)
    torch.cuda.synchronize()
    check(s, q, new, scale, out, 2)
    s.close()


@pytest.mark.parametrize("gain,q_gain,dtype", [(1000.0, 1e-4, F16), (1e-4, 3000.0, F16), (1.0, 1e6, BF16), (1000.0, 1e-9, BF16)])
@pytest.mark.parametrize("new", [[1, 3], [1, 70]])
def test_magnitudes_far_from_one(B, gain, q_gain, dtype, new):
    s = Serving(B, 128, 32, 4, 16, 2, n=2, max_length=300, seed=34, lam_spread=1.5)
    s.append([100, 200], gain)
    s.append(new, gain)
    q = queries(s, sum(new), 2, dtype, q_gain)
    scale = 0.09 / (gain * q_gain)
    out = s.run(q, new, scale)
    torch.cuda.synchronize()
    check(s, q, new, scale, out, 2)
    s.close()


def test_magnitudes_that_grow_and_fall_along_a_sequence(B):
    s = Serving(B, 128, 32, 4, 32, 1, n=2, max_length=900, seed=35)
    for gain in (1e-3, 1.0, 300.0, 0.1, 1e-3, 30.0):
        s.append([64, 100], gain)
    new = [1, 40]
    s.append(new)
    for rows in (new,):
        q = queries(s, sum(rows), 4, F16, 0.05)
        out = s.run(q, rows, 0.02)
        torch.cuda.synchronize()
        check(s, q, rows, 0.02, out, 4)
    s.close()


@pytest.mark.parametrize("new", [[1, 1, 1, 1], [50, 20, 33, 8]])
def test_pages_and_windows_that_do_not_exist_count_for_nothing_and_rows_that_see_nothing_are_zero(B, new):
    s = Serving(B, 128, 32, 4, 16, 2, n=4, max_length=300, seed=41)
    s.append([160, 35, 0, 64])
    s.append(new)
    there = [np.ones(300, bool) for _ in range(4)]
    keep = s.table.copy(), s.windows.copy()
    values = {(w, b): s.values(w, b) for w in (0, 1) for b in range(4)}
    s.table[0, 2], s.table[0, 5], s.table[1, 0] = -1, s.pool.n_pages, 1 << 30
    there[0][32:48] = there[0][80:96] = there[1][0:16] = False
    s.windows[2, 1] = s.pool.n_windows
    there[2][int(s.length[2]) // 16 * 16:] = False
    s.table[3] = -5
    there[3][: int(s.length[3]) // 16 * 16] = False
    seqs = s.seqs(new)
    s.table, s.windows = keep
    s.values = lambda w, b: values[w, b]
    q = queries(s, sum(new), 4, F16)
    out = s.run(q, new, 0.09, seqs=seqs)
    torch.cuda.synchronize()
    check(s, q, new, 0.09, out, 4, there)
    if new[2] == 1:                                          # its only token is in the window
        assert not out[2].any()
    s.close()


@pytest.mark.parametrize("n", [1, 2])
@pytest.mark.parametrize("group,bound", [(4, 40), (4, 8), (1, 300)])
def test_fewer_new_tokens_than_the_bound(B, n, group, bound):
    """What a replayed graph does: launches for `bound` new tokens, and one of them (or none) in the device arrays."""
    s = Serving(B, 128, 32, 4, 16, 2, n=n, max_length=400, seed=60 + n)
    s.append([70] * n)
    new = [1] + [0] * (n - 1)
    q = queries(s, bound, group, F16)
    out = s.run(q, new, 0.1, seqs=s.seqs(new, max_new=bound))
    check(s, q[:1], new, 0.1, out[:1], group)
    assert out[1:].isnan().all()
    none = s.run(q, new, 0.1, seqs=s.seqs([0] * n, max_new=bound))
    assert none.isnan().all()
    s.close()


def test_sequences_without_tokens_and_bounds_that_cut(B):
    s = Serving(B, 64, 32, 4, 16, 2, n=4, max_length=100, seed=43)
    s.append([40, 0, 17, 3])
    # nothing new in 1; more new rows than tokens in 3 (the first two are in no place: they see nothing)
    new = [2, 0, 1, 5]
    q = queries(s, 8, 2, F16)
    out = s.run(q, new, 0.1)
    torch.cuda.synchronize()
    got = out.clone()
    assert not got[3:5].any() and bool(torch.isfinite(got).all())
    want, bound = s.attention(q.double().cpu().numpy(), new, 0.1, 2, HALF_STEP[F16])
    rows = [0, 1, 2, 5, 6, 7]
    assert (np.abs(got.double().cpu().numpy() - want)[rows] <= bound[rows]).all()
    # no sequence, no row, no length
    B.srft_pool_attention(s.pool, s.seqs(new, max_new=0), q, 0.1, out, torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))
    s.length[:] = 0
    out = s.run(q, new, 0.1)
    torch.cuda.synchronize()
    assert not out.any()
    # starts out of order and out of range: no access outside (what the rows hold is not said)
    seqs = s.seqs(new)
    seqs.starts.copy_(torch.tensor([-4, 1 << 30, 3, -2, 100], dtype=torch.int32))
    seqs.lengths.copy_(torch.tensor([1 << 30, -3, 60, 7], dtype=torch.int32))
    s.run(q, new, 0.1, seqs=seqs)
    torch.cuda.synchronize()
    s.close()


def test_strides_and_another_stream(B):
    s = Serving(B, 96, 32, 4, 32, 2, n=2, max_length=300, seed=44)
    side = torch.cuda.Stream()
    s.append([100, 5])
    new = [3, 60]
    s.append(new)
    torch.cuda.synchronize()
    packed = queries(s, 63, 8, F16)                          # [tokens, 16 heads]: q is every other token row of a wider tensor
    q = packed[:, 4:12]
    wide = torch.full((63, 20, 104), float("nan"), dtype=F16, device="cuda")
    out = wide[:, 2:10, :96]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s.run(q, new, 0.1, out=out, stream=side)
    side.synchronize()
    check(s, q, new, 0.1, out, 4)
    assert bool(torch.isnan(wide[:, :2]).all()) and bool(torch.isnan(wide[:, 10:]).all()) and bool(torch.isnan(wide[..., 96:]).all())
    s.close()


def test_a_step_in_a_graph_follows_what_the_device_arrays_hold(B):
    s = Serving(B, 128, 32, 4, 16, 2, n=3, max_length=200, seed=45)
    s.append([30, 0, 100])
    new = [1, 1, 1]
    q = queries(s, 3, 4, F16)
    dev = [torch.zeros(3, 2, 128, dtype=F16, device="cuda") for _ in range(2)]
    s.grow(new)
    seqs = s.seqs(new)
    out = torch.empty_like(q)
    space = torch.empty(max(B.srft_pool_append_workspace_bytes(s.pool, seqs, 3), B.srft_pool_attention_workspace_bytes(s.pool, seqs, 3, 8)),
                        dtype=torch.uint8, device="cuda")

    def step():
        B.srft_pool_append(s.pool, seqs, *dev, space)
        B.srft_pool_attention(s.pool, seqs, q, 0.1, out, space)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(20):
        if i:
            s.grow(new)
        fresh = [s.draw(3) for _ in range(2)]
        for which in (0, 1):
            for b in range(3):
                s.tokens[which][b] = np.concatenate([s.tokens[which][b], fresh[which][b: b + 1]])
            dev[which].copy_(torch.from_numpy(fresh[which]))
        now = s.seqs(new)
        for name in ("page_table", "windows", "lengths"):
            getattr(seqs, name).copy_(getattr(now, name))
        graph.replay()
        torch.cuda.synchronize()
        if i % 5 == 0 or i == 19:
            check(s, q, new, 0.1, out, 4)
        again = s.run(q, new, 0.1, seqs=seqs)
        torch.cuda.synchronize()
        assert torch.equal(again, out)
    s.close()


def test_a_pool_beyond_four_gigabytes(B):
    """Page numbers whose byte offsets pass 32 bits."""
    d, R, heads = 128, 16, 8
    plans = [B.Plan(d, 32, 70 + i) for i in range(2)]
    pages = 600_000                                          # 4.9 GB of codes each
    pool = B.PagePool.empty(*plans, heads, R, pages, 2)
    x = [torch.randn(33, heads, d, device="cuda").half() for _ in range(2)]
    t = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")      # noqa: E731
    outs = []
    for table in ([[pages - 1, 599_000]], [[0, 1]]):
        seqs = B.PagedSeqs(t(table), t([[0, 1]]), t([33]), t([0, 33]), max_new=33, max_length=33)
        space = torch.empty(max(B.srft_pool_append_workspace_bytes(pool, seqs, 33), B.srft_pool_attention_workspace_bytes(pool, seqs, 33, 8)),
                            dtype=torch.uint8, device="cuda")
        B.srft_pool_append(pool, seqs, *x, space)
        for rows in (33, 1):
            step = B.PagedSeqs(t(table), t([[0, 1]]), t([33]), t([0, rows]), max_new=rows, max_length=33)
            out = torch.empty(rows, heads, d, dtype=F16, device="cuda")
            B.srft_pool_attention(pool, step, x[0][:rows], 0.1, out, space)
            outs.append(out)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3]) and bool(outs[0].any())
    pool.close()


# ------------------------------------------------------------------------------------------------------------------ copy
@pytest.mark.parametrize("layers,d,g,bits,R,heads", [(1, 128, 32, 4, 16, 2), (3, 96, 16, 8, 32, 1), (70, 64, 64, 4, 16, 2)])
def test_copies_in_every_layer_and_nowhere_else(B, layers, d, g, bits, R, heads):
    gen = torch.Generator("cuda")
    gen.manual_seed(layers)
    plan = B.Plan(d, g, 3, None, bits)

    def buffers():
        return (torch.randint(0, 256, (9, heads, R, plan.code_bytes), device="cuda", generator=gen, dtype=torch.uint8),
                torch.rand(9, heads, R, plan.groups, device="cuda", generator=gen), torch.randn(5, heads, R, d, device="cuda", generator=gen).half())
    pools = [B.PagePool(plan, plan, buffers(), buffers()) for _ in range(layers)]
    before = [[t.clone() for t in (*p.k, *p.v)] for p in pools]
    pages = [[0, 4], [8, 5], [0, 7], [9, 1], [2, -1], [3, 3], [1 << 30, 2]]
    windows = [[1, 0], [5, 2], [1, 4]]
    t = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")      # noqa: E731
    table = B.PoolTable(pools)
    B.srft_pool_copy(table, t(pages), t(windows))
    B.srft_pool_copy(table, torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for p, old in zip(pools, before):
        for i, x in enumerate(old):
            want = x.clone()
            for a, b in ([[0, 4], [8, 5], [0, 7]] if i % 3 < 2 else [[1, 0], [1, 4]]):
                want[b] = x[a]
            assert torch.equal((*p.k, *p.v)[i], want)
    for p in pools:
        p.close()


# -------------------------------------------------------------------------------------------------------------- refusals
def test_refusals(B):
    L = B.lib()
    plan, other, wide = B.Plan(128, 32, 1), B.Plan(64, 32, 1), B.Plan(128, 32, 1, None, 8)
    s = Serving(B, 128, 32, 4, 16, 2, n=2, max_length=64, seed=50)
    k, v = s.pool.k, s.pool.v
    for args, status in (((plan, wide, k, v), None), ((plan, plan, (k[0][:, :1], k[1][:, :1], k[2][:, :1]), (v[0][:, :1], v[1][:, :1], v[2][:, :1])), None)):
        with pytest.raises((B.SrftError, ValueError)):
            B.PagePool(*args)
    buf = B._PoolBuffers(k[0].data_ptr(), k[1].data_ptr(), k[2].data_ptr())
    import ctypes as C
    h = C.c_void_p()

    def create(pk=plan.handle, pv=plan.handle, heads=2, R=16, pages=1, windows=1, kb=C.byref(buf), vb=C.byref(buf)):
        rc = L.srft_pool_create(C.byref(h), pk, pv, heads, R, pages, windows, kb, vb)
        assert h.value is None
        return rc
    assert create(pk=None) == create(pv=None) == create(kb=None) == create(vb=None) == -1
    assert create(heads=0) == create(heads=1) == create(heads=-2) == create(R=0) == create(R=8) == create(R=48) == create(R=512) == -7
    assert create(pages=0) == create(windows=0) == create(pages=1 << 31) == -7
    assert create(pv=other.handle) == create(pv=wide.handle) == -8
    assert create(kb=C.byref(B._PoolBuffers(None, buf.scales_dev, buf.window_f16_dev))) == -1
    assert create(kb=C.byref(B._PoolBuffers(buf.codes_dev, buf.scales_dev + 4, buf.window_f16_dev))) == -5
    s.append([20, 3])
    new = [2, 2]
    seqs, q = s.seqs(new), queries(s, 4, 3, F16)
    out = torch.empty_like(q)
    space = torch.empty(B.srft_pool_attention_workspace_bytes(s.pool, seqs, 4, 6), dtype=torch.uint8, device="cuda")

    def attend(q=q, out=out, scale=0.1, space=space, seqs=seqs):
        B.srft_pool_attention(s.pool, seqs, q, scale, out, space)
    for bad in (dict(q=q.float()), dict(out=out.bfloat16()), dict(out=out[:3]), dict(q=q.cpu()), dict(space=space[:-1]), dict(space=space.cpu()),
                dict(q=q[..., :64]), dict(q=q.transpose(0, 2))):
        with pytest.raises(ValueError):
            attend(**bad)
    for bad, status in ((dict(scale=float("nan")), -7), (dict(scale=float("inf")), -7), (dict(q=q[:, :5], out=out[:, :5]), -7)):
        with pytest.raises(B.SrftError) as e:
            attend(**bad)
        assert e.value.status == status
    odd = torch.empty(4, 6, 132, dtype=F16, device="cuda")[..., :128]
    with pytest.raises(B.SrftError) as e:
        attend(q=odd)
    assert e.value.status == -5

    def raw(**over):
        a = dict(pool=s.pool.handle, seqs=seqs.address, q=q.data_ptr(), type=1, n=4, heads=6, qt=768, qh=128, scale=0.1, out=out.data_ptr(), ot=768, oh=128,
                 space=space.data_ptr())
        a.update(over)
        return L.srft_pool_attention(*a.values(), None)
    assert raw(pool=None) == raw(seqs=None) == raw(q=None) == raw(out=None) == raw(space=None) == -1
    assert raw(type=0) == raw(type=7) == raw(n=-1) == raw(heads=0) == raw(heads=130) == raw(n=1 << 31) == -7
    assert raw(space=space.data_ptr() + 128) == raw(q=q.data_ptr() + 8) == raw(qt=772) == -5
    for field, value, status in (("n_seq", -1, -7), ("n_seq", 4097, -7), ("max_new", -1, -7), ("max_length", 1 << 30, -7), ("max_length", 97, -7),
                                 ("max_pages", -1, -7), ("page_table_dev", None, -1), ("lengths_dev", None, -1), ("starts_dev", 4 * 77 + 2, -5)):
        bad = B._PagedSeqs.from_buffer_copy(seqs.struct)
        setattr(bad, field, value)
        assert raw(seqs=C.addressof(bad)) == status, field
        assert L.srft_pool_append(s.pool.handle, C.addressof(bad), q.data_ptr(), q.data_ptr(), 4, 256, 128, 256, 128, space.data_ptr(), None) == status, field
    assert L.srft_pool_append(s.pool.handle, seqs.address, q.data_ptr(), q.data_ptr() + 2, 4, 256, 128, 256, 128, space.data_ptr(), None) == -5
    assert L.srft_pool_append(s.pool.handle, seqs.address, q.data_ptr(), q.data_ptr(), 4, 256, 124, 256, 128, space.data_ptr(), None) == -5
    assert L.srft_pool_append(s.pool.handle, seqs.address, None, q.data_ptr(), 4, 256, 128, 256, 128, space.data_ptr(), None) == -1
    one = (C.c_void_p * 2)(s.pool.handle, None)
    assert L.srft_pool_copy(one, 2, None, 0, None, 0, None) == -1 and L.srft_pool_copy(one, 1, None, 1, None, 0, None) == -1
    assert L.srft_pool_copy(one, -1, None, 0, None, 0, None) == L.srft_pool_copy(one, 1, None, -1, None, 0, None) == -7
    torch.cuda.synchronize()
    s.close()
