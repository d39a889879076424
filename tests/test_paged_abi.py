"""Rotary positions and the paged cache at the C boundary, without a GPU: what is refused before any HIP call, and the layouts of the
structures that Python fills."""
import ctypes as C
import subprocess
from pathlib import Path

import pytest
import torch

from paper_2605_05699_amd import binding as B

HEADER = Path(__file__).resolve().parent.parent / "include"


@pytest.fixture(scope="module")
def L():
    return B.lib()


def test_structures_are_the_headers(tmp_path):
    """Compiled as C, by the host compiler."""
    of = {"srft_rotary_rows": B._RotaryRows, "srft_pool_buffers": B._PoolBuffers, "srft_paged_seqs": B._PagedSeqs}
    lines = [f'printf("{n} %zu\\n", sizeof({n}));' for n in of]
    lines += [f'printf("{n}.{f[0]} %zu\\n", offsetof({n}, {f[0]}));' for n, s in of.items() for f in s._fields_]
    (tmp_path / "a.c").write_text("#include <stddef.h>\n#include <stdint.h>\n#include <stdio.h>\n#include \"srft_kv.h\"\nint main(void) {" + "\n".join(lines) + "return 0; }")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", str(HEADER), str(tmp_path / "a.c"), "-o", str(tmp_path / "a")], check=True)
    got = dict(x.split() for x in subprocess.run([str(tmp_path / "a")], check=True, capture_output=True, text=True).stdout.splitlines())
    for n, s in of.items():
        assert int(got[n]) == C.sizeof(s)
        for f in s._fields_:
            assert int(got[f"{n}.{f[0]}"]) == getattr(s, f[0]).offset, (n, f[0])


def rotary(L, rows=None, count=1, tokens=4, d=64, rot=64, layout=0, positions=4096, freq=4096, factor=1.0, **over):
    """Addresses that nothing may read: every call here is refused, or has nothing to do."""
    if rows is None:
        rows = (B._RotaryRows * max(count, 1))()
        for r in rows:
            for k, v in dict(dict(in_dev=1 << 20, out_dev=2 << 20, in_token=128, in_head=64, out_token=128, out_head=64, n_heads=2, in_type=1, out_type=1), **over).items():
                setattr(r, k, v)
    return L.srft_rotary(rows, count, tokens, d, rot, layout, positions, freq, factor, 0, None)


def test_rotary_refusals(L):
    assert L.srft_rotary(None, 1, 4, 64, 64, 0, 4096, 4096, 1.0, 0, None) == -1
    assert rotary(L, positions=None) == rotary(L, freq=None) == rotary(L, in_dev=None) == rotary(L, out_dev=None) == -1
    for bad in (dict(count=5), dict(count=-1), dict(tokens=-1), dict(d=0), dict(d=63), dict(d=1026), dict(rot=-2), dict(rot=3), dict(rot=66),
                dict(layout=2), dict(layout=-1), dict(n_heads=0), dict(n_heads=-1), dict(in_type=3), dict(out_type=-1), dict(n_heads=1 << 30)):
        assert rotary(L, **bad) == -7, bad
    assert rotary(L, in_dev=(1 << 20) + 1) == rotary(L, out_dev=(1 << 20) + 1) == rotary(L, positions=4098) == rotary(L, freq=4100) == -5
    assert rotary(L, in_type=0, in_dev=(1 << 20) + 2) == -5                   # (aligned to its element)
    assert rotary(L, tokens=0) == rotary(L, count=0) == 0
    assert rotary(L, tokens=0, layout=2) == -7                                # (a no-op is checked all the same)


def test_pools_without_a_plan(L):
    h, buf = C.c_void_p(77), B._PoolBuffers(1 << 20, 1 << 20, 1 << 20)
    assert L.srft_pool_create(None, None, None, 2, 16, 1, 1, C.byref(buf), C.byref(buf)) == -1
    assert L.srft_pool_create(C.byref(h), None, None, 2, 16, 1, 1, C.byref(buf), C.byref(buf)) == -1
    assert h.value is None
    assert L.srft_pool_destroy(None) == 0
    seqs = B._PagedSeqs(1, 1, 16, 1, 4096, 4096, 4096, 4096)
    at = C.addressof(seqs)
    assert L.srft_pool_append_workspace_bytes(None, at, 1) == L.srft_pool_attention_workspace_bytes(None, at, 1, 2) == -1
    assert L.srft_pool_append(None, at, 4096, 4096, 1, 1, 1, 1, 1, 4096, None) == -1
    assert L.srft_pool_attention(None, at, 4096, 1, 1, 2, 1, 1, 0.1, 4096, 1, 1, 4096, None) == -1


def test_copies_without_a_pool(L):
    none = (C.c_void_p * 1)(None)
    assert L.srft_pool_copy(None, 0, None, 0, None, 0, None) == 0
    assert L.srft_pool_copy(None, 1, None, 0, None, 0, None) == -1
    assert L.srft_pool_copy(none, 1, None, 0, None, 0, None) == -1
    for n in ((-1, 0, 0), (1, -1, 0), (1, 0, -1), (1, 1 << 31, 0), (1, 0, 1 << 31), (1, 1 << 30, 1 << 30)):
        assert L.srft_pool_copy(none, n[0], 4096, n[1], 4096, n[2], None) == -7, n


def test_binding_refuses_what_is_not_on_the_device():
    x, pos, freq = torch.zeros(4, 2, 64), torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    for items in ([(x, x)], [(x, x[:3])], [(x.double(), x.double())], [(x.transpose(0, 2), x.transpose(0, 2))]):
        with pytest.raises(ValueError):
            B.srft_rotary(items, pos, freq)
    with pytest.raises(ValueError):
        B.srft_rotary([(x, x)], pos[:3], freq)
    with pytest.raises(KeyError):
        B.srft_rotary([(x, x)], pos, freq, layout="other")
    B.srft_rotary([], pos, freq)
    table, windows, lengths, starts = (torch.zeros(s, dtype=torch.int32) for s in ((2, 3), (2, 2), (2,), (3,)))
    for bad in ((table[0], windows, lengths, starts), (table, windows[:, :1], lengths, starts), (table, windows, lengths, lengths), (table, windows, lengths, starts)):
        with pytest.raises(ValueError):
            B.PagedSeqs(*bad, 1, 16)
    with pytest.raises(ValueError):
        B.srft_pool_copy(B.PoolTable([]), lengths, windows)


@pytest.mark.parametrize("name, n", [("rotary", 6), ("pool_append", 7), ("pool_attention", 7), ("pool_copy", 4)])
def test_native_calls_leave_what_is_not_on_the_device_to_the_binding(L, name, n):
    f, x = getattr(B._marshal, name), torch.zeros(4, 2, 64, dtype=torch.float16)
    for a in (x, None, 0, "x", 1.0, True, [(x, x)], [x], torch.nn.Parameter(x), 1 << 70):
        assert f(*([a] * n)) is None
    assert f() is None and f(*[x] * (n + 1)) is None
    pos, freq = torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    assert B._marshal.rotary([(x, x)], pos, freq, 0, 1.0, False) is None
    assert B._marshal.pool_append(64, 64, 2, 64, x, x, x) is None and B._marshal.pool_attention(64, 64, 64, x, 0.1, x, x) is None
    assert B._marshal.pool_copy(64, 1, pos.view(2, 2), pos.view(2, 2)) is None
