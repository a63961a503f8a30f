"""A workspace of the largest batch serves every smaller one: sizes do not shrink
where a call grows (host code only)."""
import ctypes

import pytest

from paper_2608_19659_amd import fleetsieve as fs


def size(fn, *args):
    out = ctypes.c_size_t()
    assert fn(*args, ctypes.byref(out)) == fs.FS_OK, args
    return out.value


def grows(sizes, what):
    for (a, m), (b, n) in zip(sizes, sizes[1:]):
        assert m <= n, (what, a, m, b, n)


ROWS = [*range(0, 200), *range(200, 8200, 13), *range(8200, 70000, 997), 1 << 17, 1 << 20, (1 << 31) - 1]


@pytest.mark.parametrize("name", ["fs_linear_workspace_size", "fs_project_workspace_size", "fs_gated_project_workspace_size"])
@pytest.mark.parametrize("N,K", [(5120, 5120), (20480, 5120), (5120, 20480), (1001, 1999), (777, 2049), (64, 131071), (1, 4096)])
def test_projections_by_rows(name, N, K):
    fn = getattr(fs.load_library(), name)
    grows([(M, size(fn, M, N, K)) for M in ROWS], (name, N, K))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [1, 3, 8, 12, 40, 200, 300, 1000])
def test_states(heads, D):
    fn = fs.load_library().fs_state_attention_workspace_size
    pool = ctypes.byref(fs._StatePool(None, 4, heads, D))
    tokens = [*range(0, 8200, 11), *range(8200, 200000, 997), 1 << 20, (1 << 31) // heads - 1]
    for S in (1, 2, 64, 4096):
        grows([(T, size(fn, pool, heads, T, S)) for T in tokens], (heads, D, S))
    for T in (64, 65, 389, 8192, 179966):
        grows([(S, size(fn, pool, heads, T, S)) for S in range(0, 4097, 7)], (heads, D, T))
