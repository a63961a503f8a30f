"""Workspace sizes of the projections and of state attention, and what they refuse:
host code only (no GPU needed)."""
import ctypes

import pytest

from paper_2608_19659_amd import fleetsieve as fs


@pytest.fixture(scope="module")
def lib():
    return fs.load_library()


def size(fn, *args):
    out = ctypes.c_size_t()
    status = fn(*args, ctypes.byref(out))
    return status, out.value


def pool(n_states=4, n_heads=2, head_dim=64):
    return fs._StatePool(None, n_states, n_heads, head_dim)


@pytest.mark.parametrize("M,N,K", [(0, 5, 5), (1, 1, 1), (1, 5120, 5120), (64, 5120, 20480), (8192, 5120, 20480), (333, 1001, 1999), (5, 7, 0)])
def test_projections_hold_codes_scales_and_parts(lib, M, N, K):
    _, plain = size(lib.fs_linear_workspace_size, M, N, K)
    status, got = size(lib.fs_project_workspace_size, M, N, K)
    # a block for each CU at most has a part, of 256 x 256 sums at most
    assert status == fs.FS_OK and plain <= got <= plain + 256 * 256 * 256 * 4 + (1 << 12)
    status, gated = size(lib.fs_gated_project_workspace_size, M, N, K)
    assert status == fs.FS_OK and gated >= size(lib.fs_linear_workspace_size, M, 2 * N, K)[1]


@pytest.mark.parametrize("args,status", [((-1, 1, 1), fs.FS_ERR_INVALID_ARGUMENT), ((1, -1, 1), fs.FS_ERR_INVALID_ARGUMENT),
                                         ((1, 1, -1), fs.FS_ERR_INVALID_ARGUMENT), ((1 << 31, 1, 1), fs.FS_ERR_INVALID_ARGUMENT),
                                         ((1, 1 << 31, 1), fs.FS_ERR_INVALID_ARGUMENT), ((1, 1, fs.MAX_INNER + 1), fs.FS_ERR_UNSUPPORTED)])
def test_projections_refused(lib, args, status):
    for fn in (lib.fs_project_workspace_size, lib.fs_gated_project_workspace_size):
        assert size(fn, *args)[0] == status
    assert lib.fs_project_workspace_size(1, 1, 1, None) == fs.FS_ERR_INVALID_ARGUMENT


def test_a_gated_product_has_two_rows_a_channel(lib):
    assert size(lib.fs_gated_project_workspace_size, 1, (1 << 30) - 1, 1)[0] == fs.FS_OK
    assert size(lib.fs_gated_project_workspace_size, 1, 1 << 30, 1)[0] == fs.FS_ERR_INVALID_ARGUMENT
    assert size(lib.fs_gated_project_workspace_size, 1, 1 << 62, 1)[0] == fs.FS_ERR_INVALID_ARGUMENT
    assert size(lib.fs_project_workspace_size, (1 << 31) - 1, (1 << 31) - 1, 64)[0] == fs.FS_OK  # too many tiles: the call's refusal


def test_states_of_segments(lib):
    fn = lib.fs_state_attention_workspace_size
    assert size(fn, ctypes.byref(pool()), 4, 64, 64) == (fs.FS_OK, 0)  # no sequence has two segments
    status, got = size(fn, ctypes.byref(pool(n_heads=8, head_dim=128)), 40, 8192, 4)
    assert status == fs.FS_OK and 0 < got <= 2 * 256 * 128 * 128 * 4 + 256
    status, got = size(fn, ctypes.byref(pool(n_heads=1)), 1, (1 << 31) - 1, 1)
    assert status == fs.FS_OK and got <= 2 * 257 * 64 * 64 * 4


@pytest.mark.parametrize("D,at_once", [(128, 256), (64, 512)])
@pytest.mark.parametrize("heads,T,S", [(1, 65, 1), (1, 129, 2), (2, 32768, 1), (8, 8192, 4), (8, 8192, 300), (12, 389, 23), (3, 179966, 27)])
def test_states_of_the_most_segments(lib, D, at_once, heads, T, S):
    """As many sequences of a token more than whole segments as there may be: places for
    all of their segments, and not for one more a sequence."""
    L = max(64, -(-(T * heads // at_once) // 64) * 64)
    long = min(S, T // (L + 1))
    lengths = [L + 1] * long
    if long:
        lengths[0] += (T - sum(lengths)) // L * L
    places = sum(-(-n // L) for n in lengths)
    status, got = size(lib.fs_state_attention_workspace_size, ctypes.byref(pool(n_heads=heads, head_dim=D)), heads, T, S)
    assert status == fs.FS_OK
    assert places * heads * D * D * 4 <= got <= (places + min(S, T // L)) * heads * D * D * 4


@pytest.mark.parametrize("change,args,status", [
    (dict(head_dim=80), (2, 5, 1), fs.FS_ERR_UNSUPPORTED), (dict(head_dim=256), (2, 5, 1), fs.FS_ERR_UNSUPPORTED),
    (dict(n_heads=0), (2, 5, 1), fs.FS_ERR_INVALID_ARGUMENT), (dict(n_states=-1), (2, 5, 1), fs.FS_ERR_INVALID_ARGUMENT),
    (dict(n_heads=4097), (4097, 5, 1), fs.FS_ERR_UNSUPPORTED), ({}, (3, 5, 1), fs.FS_ERR_INVALID_ARGUMENT),
    ({}, (0, 5, 1), fs.FS_ERR_INVALID_ARGUMENT), ({}, (65536, 5, 1), fs.FS_ERR_UNSUPPORTED),
    ({}, (2, -1, 1), fs.FS_ERR_INVALID_ARGUMENT), ({}, (2, 1 << 31, 1), fs.FS_ERR_INVALID_ARGUMENT),
    ({}, (32, 1 << 27, 1), fs.FS_ERR_INVALID_ARGUMENT), ({}, (2, 5, -1), fs.FS_ERR_INVALID_ARGUMENT),
    ({}, (2, 5, fs.MAX_SEQUENCES + 1), fs.FS_ERR_UNSUPPORTED)], ids=str)
def test_states_refused(lib, change, args, status):
    assert size(lib.fs_state_attention_workspace_size, ctypes.byref(pool(**change)), *args)[0] == status


def test_calls_without_a_context_or_a_pool(lib):
    assert size(lib.fs_state_attention_workspace_size, None, 2, 5, 1)[0] == fs.FS_ERR_INVALID_ARGUMENT
    n = None
    assert lib.fs_project(n, n, 0, 1, n, n, 1, n, n, 0, n, 0, 1, 1, 1, n, 0, 1, n, 0, n) == fs.FS_ERR_INVALID_ARGUMENT
    assert lib.fs_gated_project(n, n, 0, 1, n, n, 1, n, n, 0, 1, 1, 1, n, 0, 1, n, 0, n) == fs.FS_ERR_INVALID_ARGUMENT
    assert lib.fs_state_attention(n, n, n, 0, n, 0, n, 0, 1, 1, 1, 1, n, n, n, 1, n, 1.0, n, n, 0, n) == fs.FS_ERR_INVALID_ARGUMENT


def test_names_that_are_none():
    with pytest.raises(fs.FleetSieveError) as e:
        fs._activation("tanh")
    assert e.value.status == fs.FS_ERR_INVALID_ARGUMENT
    assert set(fs.ACTIVATIONS) == {"none", "relu", "gelu", "gelu_tanh", "silu"}
