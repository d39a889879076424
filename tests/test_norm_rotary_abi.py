"""Norms with rotary positions at the C boundary, without a GPU: what is refused before any HIP call, and the structures that Python fills."""
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
    of = {"srft_norm_rows": B._NormRows, "srft_norm_grad_rows": B._NormGradRows}
    lines = [f'printf("{n} %zu\\n", sizeof({n}));' for n in of]
    lines += [f'printf("{n}.{f[0]} %zu\\n", offsetof({n}, {f[0]}));' for n, s in of.items() for f in s._fields_]
    (tmp_path / "a.c").write_text("#include <stddef.h>\n#include <stdint.h>\n#include <stdio.h>\n#include \"srft_kv.h\"\nint main(void) {" + "\n".join(lines) + "return 0; }")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", str(HEADER), str(tmp_path / "a.c"), "-o", str(tmp_path / "a")], check=True)
    got = dict(x.split() for x in subprocess.run([str(tmp_path / "a")], check=True, capture_output=True, text=True).stdout.splitlines())
    for n, s in of.items():
        assert int(got[n]) == C.sizeof(s)
        for f in s._fields_:
            assert int(got[f"{n}.{f[0]}"]) == getattr(s, f[0]).offset, (n, f[0])


def forward(L, rows=None, count=1, tokens=4, d=64, rot=64, layout=0, positions=4096, freq=4096, eps=1e-6, weight_dev=4 << 20, weight_type=0, reserved=0, **over):
    """Addresses that nothing may read: every call here is refused, or has nothing to do."""
    if rows is None:
        rows = (B._NormRows * max(count, 1))()
        for r in rows:
            for k, v in dict(dict(in_dev=1 << 20, out_dev=2 << 20, in_token=128, in_head=64, out_token=128, out_head=64, n_heads=2, in_type=1, out_type=1), **over).items():
                setattr(r.x, k, v)
            r.weight_dev, r.weight_type, r.reserved = weight_dev, weight_type, reserved
    return L.srft_norm_rotary(rows, count, tokens, d, rot, layout, positions, freq, 1.0, eps, None)


def backward(L, count=1, tokens=4, d=64, rot=64, layout=0, positions=4096, freq=4096, eps=1e-6, workspace=64 << 20, apart=True, **over):
    rows = (B._NormGradRows * max(count, 1))()
    for i, r in enumerate(rows):
        for k, v in dict(dict(dy_dev=1 << 20, x_dev=2 << 20, dx_dev=3 << 20, weight_dev=4 << 20, dweight_dev=(5 + (i if apart else 0)) << 20, dy_token=128, dy_head=64,
                              x_token=128, x_head=64, dx_token=128, dx_head=64, n_heads=2, dy_type=1, x_type=1, weight_type=0), **over).items():
            setattr(r, k, v)
    return L.srft_norm_rotary_backward(rows, count, tokens, d, rot, layout, positions, freq, 1.0, eps, workspace, None)


BAD = (dict(count=5), dict(count=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(d=0), dict(d=63), dict(d=1026), dict(rot=-2), dict(rot=3), dict(rot=66), dict(layout=2),
       dict(layout=-1), dict(n_heads=0), dict(n_heads=-1), dict(n_heads=1 << 30), dict(eps=0.0), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")),
       dict(eps=1e-39), dict(eps=1e39), dict(weight_type=3))


def test_refusals(L):
    assert L.srft_norm_rotary(None, 1, 4, 64, 64, 0, 4096, 4096, 1.0, 1e-6, None) == -1
    assert forward(L, positions=None) == forward(L, freq=None) == forward(L, in_dev=None) == forward(L, out_dev=None) == -1
    for bad in (*BAD, dict(in_type=3), dict(out_type=-1), dict(reserved=1)):
        assert forward(L, **bad) == -7, bad
    assert forward(L, in_dev=(1 << 20) + 1) == forward(L, out_dev=(1 << 20) + 1) == forward(L, positions=4098) == forward(L, freq=4100) == forward(L, weight_dev=4098) == -5
    assert forward(L, out_dev=1 << 20, out_type=2) == forward(L, out_dev=1 << 20, out_token=256) == forward(L, out_dev=1 << 20, out_head=128) == -7
    assert forward(L, tokens=0) == forward(L, count=0) == forward(L, tokens=0, weight_dev=None) == 0
    assert forward(L, tokens=0, layout=2) == -7                              # (a no-op is checked all the same)


def test_refusals_of_gradients(L):
    assert L.srft_norm_rotary_backward(None, 1, 4, 64, 64, 0, 4096, 4096, 1.0, 1e-6, 4096, None) == -1
    for name in ("positions", "freq", "dy_dev", "x_dev", "dx_dev", "workspace"):
        assert backward(L, **{name: None}) == -1, name
    for bad in (*BAD, dict(x_type=3), dict(dy_type=-1), dict(count=2, apart=False)):
        assert backward(L, **bad) == -7, bad
    for bad in (dict(dy_dev=(1 << 20) + 1), dict(x_dev=(1 << 20) + 1), dict(dx_dev=(1 << 20) + 1), dict(positions=4098), dict(freq=4100), dict(weight_dev=4098), dict(dweight_dev=4098),
                dict(workspace=4096 + 8)):
        assert backward(L, **bad) == -5, bad
    for bad in (dict(dx_dev=1 << 20, dy_type=2), dict(dx_dev=1 << 20, dx_token=256), dict(dx_dev=2 << 20, dx_head=128)):
        assert backward(L, **bad) == -7, bad
    assert backward(L, count=0) == backward(L, tokens=0, dweight_dev=None) == 0
    size = L.srft_norm_rotary_backward_workspace_bytes
    assert size(0, 64) == 0 and size(2, 64) == 2 * size(1, 64) > 0
    assert size(5, 64) == size(-1, 64) == size(1, 63) == size(1, 1026) == size(1, 0) == -7


def test_binding_refuses_what_is_not_on_the_device():
    x, pos, freq, w = torch.zeros(4, 2, 64), torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64), torch.ones(64)
    for items in ([(x, w, x)], [(x, None, x)], [(x, w, x[:3])], [(x.double(), w, x.double())], [(x.transpose(0, 2), w, x.transpose(0, 2))]):
        with pytest.raises(ValueError):
            B.srft_norm_rotary(items, pos, freq, 1e-6)
    with pytest.raises(ValueError):
        B.srft_norm_rotary([(x, w, x)], pos[:3], freq, 1e-6)
    for items in ([(x, x, w, x, w)], [(x, x, None, x, None)], [(x, x, w, x.half(), w)], [(x, x, w, x, w[:3])]):
        with pytest.raises(ValueError):
            B.srft_norm_rotary_backward(items, pos, freq, 1e-6, None)
    B.srft_norm_rotary([], pos, freq, 1e-6)
    B.srft_norm_rotary_backward([], pos, freq, 1e-6, None)
