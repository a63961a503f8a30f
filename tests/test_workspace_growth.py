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
