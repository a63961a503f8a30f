"""Projections whose tiles are cut along the inner dimension, and those that are not,
for every tile that there is and both finishes: against the products of fs_linear,
whose tiles are never cut.  What a cut call did is read from its workspace: a count
for each cut tile, of the parts that arrived."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_serving import bits, env, note  # noqa: E402, F401

# (rows, channels, inner elements, tile, parts of a cut tile, cut tiles of an XCD): tiles
# of 16 x 16, 16 x 32, 32 x 32, 64 x 32, 64 x 64, 128 x 64, 128 x 128, 256 x 128 and 256 x
# 256 weight rows; all tiles cut and some, inner elements that are a multiple of 16 and odd
CUT = [
    (5, 16, 7568, 0, 7, 1), (5, 16, 7541, 0, 7, 1), (5, 4110, 8304, 0, 8, 1), (9, 4101, 8289, 0, 8, 1),
    (10, 1285, 12688, 1, 5, 6), (12, 1282, 12701, 1, 5, 6), (10, 9106, 8832, 1, 8, 4), (12, 9129, 8841, 1, 8, 4),
    (81, 161, 10336, 2, 10, 3), (84, 161, 10265, 2, 10, 3), (20, 8202, 6192, 2, 6, 1), (32, 8203, 6187, 2, 6, 1),
    (289, 209, 5120, 3, 5, 5), (273, 226, 5159, 3, 5, 5), (47, 8225, 11280, 3, 11, 1), (42, 8235, 11321, 3, 11, 1),
    (326, 325, 6752, 4, 6, 5), (324, 332, 6803, 4, 6, 5), (34, 16537, 2864, 4, 2, 1), (36, 16518, 2865, 4, 2, 1),
    (534, 513, 6112, 5, 5, 6), (518, 514, 6169, 5, 5, 6), (1623, 1223, 3232, 5, 3, 1), (1638, 1219, 3233, 5, 3, 1),
    (1035, 963, 9776, 6, 3, 9), (775, 1217, 9861, 6, 3, 9), (2321, 3410, 2160, 6, 2, 1), (2338, 3397, 2113, 6, 2, 1),
    (2191, 3684, 2144, 7, 2, 1), (2982, 2725, 2147, 7, 2, 1), (2471, 1941, 17200, 8, 3, 10),
    (1946, 2461, 17005, 8, 3, 10), (4416, 3753, 4112, 8, 4, 2), (4369, 3719, 4131, 8, 4, 2),
]
GATED_CUT = [
    (5, 8, 7536, 0, 7, 1), (5, 8, 7533, 0, 7, 1), (13, 2051, 8336, 0, 8, 1), (6, 2049, 8323, 0, 8, 1),
    (5, 642, 12704, 1, 5, 6), (9, 645, 12697, 1, 5, 6), (10, 4550, 8832, 1, 8, 4), (12, 4546, 8835, 1, 8, 4),
    (130, 57, 10256, 2, 10, 3), (162, 41, 10301, 2, 10, 3), (28, 4114, 6144, 2, 6, 1), (19, 4122, 6171, 2, 6, 1),
    (294, 105, 5120, 3, 5, 5), (313, 97, 5131, 3, 5, 5), (53, 4113, 11280, 3, 11, 1), (46, 4118, 11251, 3, 10, 1),
    (324, 161, 6784, 4, 6, 5), (261, 198, 6781, 4, 6, 5), (33, 8193, 2864, 4, 2, 1), (39, 8208, 2861, 4, 2, 1),
    (523, 257, 6192, 5, 5, 6), (586, 228, 6123, 5, 5, 5), (1348, 737, 3264, 5, 3, 1), (1219, 820, 3233, 5, 3, 1),
    (1046, 481, 9776, 6, 3, 9), (774, 612, 9789, 6, 3, 9), (2434, 1659, 2112, 6, 2, 1), (2311, 1724, 2131, 6, 2, 1),
    (2692, 1475, 2128, 7, 2, 1), (2180, 1820, 2123, 7, 2, 1), (1932, 1219, 17344, 8, 3, 10),
    (2441, 961, 17025, 8, 3, 10), (3753, 2284, 4112, 8, 4, 2), (4471, 1873, 4117, 8, 4, 2),
]
WHOLE = [
    (5, 16, 112, 0, 1, 0), (5, 16, 101, 0, 1, 0), (306, 193, 112, 1, 1, 0), (193, 306, 101, 1, 1, 0),
    (402, 289, 112, 2, 1, 0), (310, 389, 101, 2, 1, 0), (612, 386, 112, 3, 1, 0), (617, 385, 101, 3, 1, 0),
    (389, 1154, 112, 4, 1, 0), (386, 1165, 101, 4, 1, 0), (771, 1218, 112, 5, 1, 0), (772, 1229, 101, 5, 1, 0),
    (5, 16439, 112, 6, 1, 0), (5, 16612, 101, 6, 1, 0), (130, 16479, 112, 7, 1, 0), (129, 16469, 101, 7, 1, 0),
    (257, 16441, 112, 8, 1, 0), (258, 16510, 101, 8, 1, 0),
]
GATED_WHOLE = [
    (5, 8, 112, 0, 1, 0), (5, 8, 101, 0, 1, 0), (305, 97, 112, 1, 1, 0), (209, 146, 101, 1, 1, 0),
    (403, 145, 112, 2, 1, 0), (402, 145, 101, 2, 1, 0), (612, 194, 112, 3, 1, 0), (390, 309, 101, 3, 1, 0),
    (578, 402, 112, 4, 1, 0), (578, 401, 111, 4, 1, 0), (706, 673, 112, 5, 1, 0), (583, 803, 101, 5, 1, 0),
    (5, 8197, 112, 6, 1, 0), (5, 8199, 101, 6, 1, 0), (130, 8363, 112, 7, 1, 0), (131, 8281, 103, 7, 1, 0),
    (258, 8332, 112, 8, 1, 0), (258, 8195, 103, 8, 1, 0),
]


def inputs(M, rows, N, K):
    g = torch.Generator(device="cuda:0").manual_seed(M + rows)
    x = torch.randn(M, K, device="cuda:0", generator=g).to(torch.bfloat16)
    w = torch.randint(-127, 128, (rows, K), device="cuda:0", generator=g, dtype=torch.int8)
    sw = torch.rand(rows, device="cuda:0", generator=g) / (100.0 * math.sqrt(K))
    return x, w, sw, torch.randn(M, N, device="cuda:0", generator=g).to(torch.bfloat16)


def run(env, gated, M, N, K, tile, parts, rest):
    fs, ctx = env
    note(f"{'gated ' if gated else ''}project {M}x{N}x{K}, tile {tile} in {parts} parts")
    rows = 2 * N if gated else N
    x, w, sw, res = inputs(M, rows, N, K)
    lib = fs.load_library()
    before = fs._size(lib.fs_linear_workspace_size, M, rows, K)
    need = fs._size(lib.fs_gated_project_workspace_size if gated else lib.fs_project_workspace_size, M, N, K)
    value = fs.linear(ctx, x, w[rows - N:], sw[rows - N:], out_dtype=torch.float32)
    room = torch.empty(need + 4096, dtype=torch.uint8, device="cuda:0")
    for fill in (255, 1):
        room.fill_(fill)
        if gated:
            got = fs.gated_project(ctx, x, w, sw, activation="none", workspace=room[:need])
            want = (fs.linear(ctx, x, w[:N], sw[:N], out_dtype=torch.float32) * value).to(torch.bfloat16)
        else:
            got = fs.project(ctx, x, w, sw, residual=res, workspace=room[:need])
            want = (value + res.float()).to(torch.bfloat16)
        assert torch.equal(bits(got), bits(want))
        assert (room[need:] == fill).all()
        if need > before:
            counts = room[before:before + 1024].view(torch.int32).tolist()
            used = [c for c in counts if c != int.from_bytes([fill] * 4, "little", signed=True)]
            assert len(used) == 8 * rest and set(used) <= {0, parts} and (not rest or parts in used), counts
        else:
            assert rest == 0


@pytest.mark.parametrize("case", CUT + WHOLE, ids=str)
def test_project(env, case):
    run(env, False, *case)


@pytest.mark.parametrize("case", GATED_CUT + GATED_WHOLE, ids=str)
def test_gated(env, case):
    run(env, True, *case)


@pytest.mark.parametrize("M,N,K", [(34, 333, 2900), (129, 5120, 20480), (8192, 5120, 5120)])
def test_a_workspace_of_the_most_rows_serves_fewer(env, M, N, K):
    fs, ctx = env
    note(f"a workspace of {M} rows for fewer, {N}x{K}")
    ws = torch.empty(fs._size(fs.load_library().fs_project_workspace_size, M, N, K), dtype=torch.uint8, device="cuda:0")
    x, w, sw, res = inputs(M, N, N, K)
    for m in (1, 5, 16, 17, 33, 100, 128, 129, 3000, 7168, 8192):
        if m <= M:
            want = (fs.linear(ctx, x[:m], w, sw, out_dtype=torch.float32) + res[:m].float()).to(torch.bfloat16)
            assert torch.equal(bits(fs.project(ctx, x[:m], w, sw, residual=res[:m], workspace=ws)), bits(want)), m
