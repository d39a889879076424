"""Sliding and shared attention at the C boundary, without a GPU: what is refused before any HIP call, and the structure that Python fills."""
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
    s = B._SharedPrefixes
    lines = ['printf("size %zu\\n", sizeof(srft_shared_prefixes));'] + [f'printf("{f[0]} %zu\\n", offsetof(srft_shared_prefixes, {f[0]}));' for f in s._fields_]
    (tmp_path / "a.c").write_text("#include <stddef.h>\n#include <stdint.h>\n#include <stdio.h>\n#include \"srft_kv.h\"\nint main(void) {" + "\n".join(lines) + "return 0; }")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", str(HEADER), str(tmp_path / "a.c"), "-o", str(tmp_path / "a")], check=True)
    got = dict(x.split() for x in subprocess.run([str(tmp_path / "a")], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(got["size"]) == C.sizeof(s)
    for f in s._fields_:
        assert int(got[f[0]]) == getattr(s, f[0]).offset, f[0]


def test_without_a_pool(L):
    seqs, shared = B._PagedSeqs(1, 1, 16, 1, 4096, 4096, 4096, 4096), B._SharedPrefixes(1, 0, 4096, 4096)
    at, of = C.addressof(seqs), C.addressof(shared)
    assert L.srft_pool_attention_sliding_workspace_bytes(None, at, 1, 2) == -1
    assert L.srft_pool_attention_sliding(None, at, 4096, 1, 1, 2, 1, 1, 0.1, 1, 0, 4096, 1, 1, 4096, None) == -1
    assert L.srft_pool_attention_shared_workspace_bytes(None, at, of, 1, 2) == L.srft_pool_attention_shared_workspace_bytes(None, at, None, 1, 2) == -1
    assert L.srft_pool_attention_shared(None, at, of, 4096, 1, 1, 2, 1, 1, 0.1, 4096, 1, 1, 4096, None) == -1
    assert L.srft_pool_attention_shared(None, at, None, 4096, 1, 1, 2, 1, 1, 0.1, 4096, 1, 1, 4096, None) == -1


def test_binding_refuses_prefixes_that_are_not_on_the_device():
    groups, tokens = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for bad in ((groups, tokens), (groups, tokens[:1]), (groups[None], tokens), (groups, tokens.long())):
        with pytest.raises(ValueError):
            B.SharedPrefixes(*bad)


@pytest.mark.parametrize("name, n", [("norm_rotary", 6), ("norm_backward", 7), ("pool_sliding", 9), ("pool_shared", 8)])
def test_native_calls_leave_what_is_not_on_the_device_to_the_binding(L, name, n):
    f, x = getattr(B._marshal, name), torch.zeros(4, 2, 64, dtype=torch.float16)
    for a in (x, None, 0, "x", 1.0, True, [(x, x)], [x], [(x, None, x)], [(x, x, None, x, None)], torch.nn.Parameter(x), 1 << 70):
        assert f(*([a] * n)) is None
    assert f() is None and f(*[x] * (n + 1)) is None
    pos, freq = torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    assert B._marshal.norm_rotary([(x, None, x)], pos, freq, 0, 1.0, 1e-6) is None
    assert B._marshal.norm_backward([(x, x, None, x, None)], pos, freq, 0, 1.0, 1e-6, None) is None
    assert B._marshal.pool_sliding(64, 64, 64, x, 0.1, 1, 1, x, x) is None and B._marshal.pool_shared(64, 64, 64, 64, x, 0.1, x, x) is None
