"""Projections with norm, activation and residual, and gated projections, on the
GPU against plain 64-bit statements of them; without a norm and an activation bit
for bit against the projection."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import layer_reference as ref  # noqa: E402
from test_gpu_serving import TYPES, bits, env, gen, note  # noqa: E402, F401

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
EPS = 1e-5


def inputs(M, N, K, dtype="bf16", seed=0, rows=None):
    g = gen(M * 31 + N * 7 + K + seed)
    rows = N if rows is None else rows
    x = (torch.randn(M, K, generator=g) * torch.exp(torch.randn(M, 1, generator=g))).to(TYPES[dtype])
    w = torch.randint(-127, 128, (rows, K), generator=g, dtype=torch.int8)
    w_scale = (torch.rand(rows, generator=g) + 0.2) / (73.0 * math.sqrt(max(K, 1)))
    return x, w, w_scale, torch.randn(rows, generator=g), torch.rand(K, generator=g) + 0.3


def d(t):
    return None if t is None else t.to("cuda:0")


def close(got, want, room, what=""):
    got = got.double().cpu()
    off = (got - want).abs()
    assert torch.isfinite(got).all(), what
    worst = (off - room).argmax()
    assert (off <= room).all(), (what, float(off.flatten()[worst]), float(room.flatten()[worst]))


# rows and channels that fill no tile, odd inner sizes (each tile, by the rule that these calls choose by, cut and
# whole: test_gpu_cut_products.py)
SIZES = [(1, 1, 1), (1, 64, 64), (1, 2500, 512), (2, 33, 100), (3, 4100, 528), (4, 9000, 64), (4, 131, 2048), (7, 130, 257),
         (16, 256, 1024), (17, 100, 4097), (33, 512, 384), (64, 320, 5120), (65, 65, 65), (100, 2048, 640), (127, 129, 1040),
         (255, 257, 128), (300, 700, 272), (513, 511, 1024), (777, 1100, 333), (2048, 768, 512), (2500, 3001, 129),
         (4096, 2600, 256)]
FEATURES = [dict(norm=True, act="silu", bias=False, residual=False), dict(norm=False, act="gelu", bias=True, residual=True),
            dict(norm=True, act="none", bias=True, residual=True)]


@pytest.mark.parametrize("features", FEATURES, ids=lambda f: "-".join(k if v is True else v for k, v in f.items() if v))
@pytest.mark.parametrize("M,N,K", SIZES)
def test_project(env, M, N, K, features):
    fs, ctx = env
    dtype, out = ["bf16", "f16", "f32"][(M + N) % 3], ["f32", "bf16", "f16"][(N + K) % 3]
    note(f"project {M}x{N}x{K} {dtype}->{out} {features}")
    x, w, sw, bias, gain = inputs(M, N, K, dtype)
    bias = bias if features["bias"] else None
    res = (torch.randn(M, N, generator=gen(5)) * 3).to(TYPES[out]) if features["residual"] else None
    norm = fs.Norm(d(gain), EPS) if features["norm"] else None
    got = fs.project(ctx, d(x), d(w), d(sw), norm=norm, bias=d(bias), activation=features["act"], residual=d(res),
                     out_dtype=TYPES[out])
    want, room = ref.project(x, w, sw, (gain, EPS) if norm else None, bias, features["act"], res, TYPES[out])
    assert got.dtype == TYPES[out]
    close(got, want, room)


@pytest.mark.parametrize("features", [dict(norm=True, act="silu", bias=False), dict(norm=False, act="gelu_tanh", bias=True)],
                         ids=lambda f: f["act"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gated(env, M, N, K, features):
    fs, ctx = env
    dtype, out = ["bf16", "f16", "f32"][(M + N) % 3], ["f32", "bf16", "f16"][(N + K) % 3]
    note(f"gated {M}x{N}x{K} {dtype}->{out} {features}")
    x, w, sw, bias, gain = inputs(M, N, K, dtype, rows=2 * N)
    bias = bias if features["bias"] else None
    norm = fs.Norm(d(gain), EPS) if features["norm"] else None
    got = fs.gated_project(ctx, d(x), d(w), d(sw), norm=norm, bias=d(bias), activation=features["act"], out_dtype=TYPES[out])
    want, room = ref.gated(x, w, sw, (gain, EPS) if norm else None, bias, features["act"], TYPES[out])
    assert got.shape == (M, N) and got.dtype == TYPES[out]
    close(got, want, room)


@pytest.mark.parametrize("act", ACTS)
def test_activations_over_their_range(env, act):
    """One inner element and weights of one: y is x, from nearly nothing to far
    beyond where a sigmoid is 0 or 1."""
    fs, ctx = env
    y = torch.cat([torch.linspace(-30, 30, 4001), 10.0 ** torch.linspace(-25, 3, 400), -(10.0 ** torch.linspace(-25, 3, 400))])
    x, w, sw = y[:, None].contiguous(), torch.full((3, 1), 127, dtype=torch.int8), torch.full((3,), 1 / 127.0)
    got = fs.project(ctx, d(x), d(w), d(sw), activation=act, out_dtype=torch.float32)
    want, room = ref.project(x, w, sw, act=act)
    close(got, want, room, act)
    both = fs.gated_project(ctx, d(x), d(w[:2]), d(sw[:2]), activation=act)
    want, room = ref.gated(x, w[:2], sw[:2], act=act)
    close(both, want, room, act)


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,N,K", [(1, 100, 64), (3, 5000, 528), (20, 333, 700), (300, 1001, 256), (2048, 768, 512)])
def test_without_extras_it_is_the_projection(env, M, N, K, out):
    """Bit for bit, and with a residual that plus the residual in one more step."""
    fs, ctx = env
    note(f"plain project {M}x{N}x{K} {out}")
    x, w, sw, bias, _ = inputs(M, N, K, "bf16")
    a = (ctx, d(x), d(w), d(sw))
    assert torch.equal(bits(fs.project(*a, bias=d(bias), out_dtype=TYPES[out])), bits(fs.linear(*a, d(bias), TYPES[out])))
    res = torch.randn(M, N, generator=gen(1)).to(TYPES[out])
    want = (fs.linear(*a, None, torch.float32).cpu() + res.float()).to(TYPES[out])
    assert torch.equal(bits(fs.project(*a, residual=d(res), out_dtype=TYPES[out])), bits(want))
    # the stream's own memory takes the result
    place = d(res).clone()
    assert fs.project(*a, residual=place, out=place).data_ptr() == place.data_ptr()
    assert torch.equal(bits(place), bits(want))
    # a gate of all ones and no activation: the values' projection
    ones = torch.cat([torch.zeros(N), torch.zeros(N)])
    ones[:N] = 1.0
    sw2 = torch.cat([torch.zeros(N), sw])
    got = fs.gated_project(ctx, d(x), d(torch.cat([w, w])), d(sw2), bias=d(ones), activation="none", out_dtype=TYPES[out])
    assert torch.equal(bits(got), bits(fs.linear(*a, torch.zeros(N, device="cuda:0"), TYPES[out])))


@pytest.mark.parametrize("offset,x_pad,w_pad,out_pad,gain_at", [(0, 16, 48, 8, 4), (1, 3, 5, 1, 1), (4, 4, 12, 2, 3), (16, 0, 0, 3, 0)])
@pytest.mark.parametrize("M,N,K", [(1, 70, 208), (4, 41, 96), (5, 70, 200), (40, 600, 1030), (130, 260, 520), (300, 300, 256)])
def test_strides_and_what_lies_between_rows(env, M, N, K, offset, x_pad, w_pad, out_pad, gain_at):
    fs, ctx = env
    note(f"project strided {M}x{N}x{K} +{offset} {x_pad} {w_pad} {out_pad} {gain_at}")
    x, w, sw, bias, gain = inputs(M, N, K, "bf16", rows=2 * N)

    def strided(t, pad, fill, at=0):
        flat = torch.full((at + t.shape[0] * (t.shape[1] + pad),), fill, dtype=t.dtype, device="cuda:0")
        view = flat[at:].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
        view.copy_(t)
        return flat, view
    _, dx = strided(x, x_pad, math.nan, offset)
    _, dw = strided(w, w_pad, -99, offset)
    dg = torch.full((gain_at + K + 1,), math.nan, device="cuda:0")
    dg[gain_at:gain_at + K] = d(gain)
    norm = fs.Norm(dg[gain_at:gain_at + K], EPS)
    res = torch.randn(M, N, generator=gen(9)).to(torch.float16)
    for gate in (False, True):
        flat, out = strided(res, out_pad, 5.0)
        if gate:
            fs.gated_project(ctx, dx, dw, d(sw), norm=norm, bias=d(bias), out=out)
            want, room = ref.gated(x, w, sw, (gain, EPS), bias, "silu", torch.float16)
        else:
            fs.project(ctx, dx, dw[:N], d(sw[:N]), norm=norm, bias=d(bias[:N]), activation="gelu", residual=out, out=out)
            want, room = ref.project(x, w[:N], sw[:N], (gain, EPS), bias[:N], "gelu", res, torch.float16)
        close(out, want, room)
        if out_pad:
            assert (flat.view(M, N + out_pad)[:, N:] == 5.0).all()


@pytest.mark.parametrize("M,K", [(1, 64), (3, 2048), (6, 333), (9, 9000), (2, 41000)])
def test_rows_at_the_ends_of_their_type(env, M, K):
    """Rows whose squares pass binary32 or vanish in it, of zeros, of no numbers."""
    fs, ctx = env
    for dtype in (torch.float32, torch.bfloat16):
        x, w, sw, _, gain = inputs(M, 40, K, "f32", rows=80)
        for scale in (1e36, 1e18, 1e-18, 1e-28, 0.0):
            y = (x / x.abs().max() * scale).to(dtype)
            got = fs.project(ctx, d(y), d(w[:40]), d(sw[:40]), norm=fs.Norm(d(gain), EPS), out_dtype=torch.float32)
            want, room = ref.project(y, w[:40], sw[:40], (gain, EPS))
            close(got, want, room * (1 if K < 20481 else 2), scale)  # a thread of a longer row adds 40 elements in 8 parts more
        for bad in (math.nan, math.inf, -math.inf):
            y = x.to(dtype).clone()
            y[M - 1, K // 2] = bad
            for got in (fs.project(ctx, d(y), d(w), d(sw), norm=fs.Norm(d(gain), EPS)),
                        fs.gated_project(ctx, d(y), d(w), d(sw), norm=fs.Norm(None, EPS)),
                        fs.project(ctx, d(y), d(w), d(sw), activation="relu")):
                assert torch.isnan(got[M - 1]).all() and torch.isfinite(got[:M - 1]).all()
    y = x.clone()
    y[0], gain[:] = 1e30, 1e20
    got = fs.project(ctx, d(y), d(w), d(sw), norm=fs.Norm(d(gain), EPS))
    assert torch.isnan(got[0]).all()


def test_norm_without_gains_and_large_eps(env):
    fs, ctx = env
    for M, K in ((1, 512), (3, 100), (40, 600)):
        x, w, sw, _, _ = inputs(M, 70, K, "f16")
        for eps in (2.0 ** -80, 0.5, 2.0 ** 80):
            got = fs.project(ctx, d(x), d(w), d(sw), norm=fs.Norm(None, eps), out_dtype=torch.float32)
            want, room = ref.project(x, w, sw, (torch.ones(K), eps))
            close(got, want, room, (M, K, eps))


@pytest.mark.parametrize("N", [255, 300])
@pytest.mark.parametrize("M", [2, 9])
def test_weight_rows_far_apart(env, N, M):
    """A gate's and its value's row more than 2^31 bytes apart."""
    fs, ctx = env
    note(f"weight rows far apart, {N} channels, {M} rows")
    K, stride = 64, 1 << 23
    x, w, sw, bias, gain = inputs(M, N, K, "bf16", rows=2 * N)
    far = torch.empty(2 * N * stride, dtype=torch.int8, device="cuda:0").view(2 * N, stride)[:, :K]
    far.copy_(w)
    got = fs.gated_project(ctx, d(x), far, d(sw), bias=d(bias))
    want, room = ref.gated(x, w, sw, None, bias, "silu", torch.bfloat16)
    close(got, want, room)


def test_no_inner_elements_and_nothing_to_do(env):
    fs, ctx = env
    e = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda:0")  # noqa: E731
    w = lambda *s: torch.zeros(*s, dtype=torch.int8, device="cuda:0")  # noqa: E731
    one = torch.ones(6, device="cuda:0")
    res = e(3, 6) + 2
    got = fs.project(ctx, e(3, 0), w(6, 0), one, norm=fs.Norm(None), bias=one, activation="relu", residual=res)
    assert (got == 3.0).all()
    assert (fs.gated_project(ctx, e(3, 0), w(6, 0), one, bias=2 * one, activation="none") == 4.0).all()
    assert fs.project(ctx, e(0, 8), w(6, 8), one).shape == (0, 6)
    assert fs.gated_project(ctx, e(0, 8), w(6, 8), one).shape == (0, 3)
    assert fs.gated_project(ctx, e(2, 8), w(0, 8), one[:0]).shape == (2, 0)


def test_arguments_that_are_refused(env):
    fs, ctx = env
    dev = "cuda:0"
    h = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=dev)  # noqa: E731
    i8 = lambda *s: torch.zeros(*s, dtype=torch.int8, device=dev)  # noqa: E731
    f = lambda *s: torch.zeros(*s, device=dev)  # noqa: E731
    square = h(8, 8)
    cases = [
        lambda: fs.project(ctx, h(2, 8), i8(3, 9), f(3)),
        lambda: fs.project(ctx, h(2, 8), i8(3, 8), f(2)),
        lambda: fs.project(ctx, h(2, 8), i8(3, 8), f(3), bias=f(4)),
        lambda: fs.project(ctx, h(2, 8), i8(3, 8), f(3), activation="tanh"),
        lambda: fs.project(ctx, h(2, 8), i8(3, 8), f(3), residual=f(2, 3)),
        lambda: fs.project(ctx, h(2, 8), i8(3, 8), f(3), residual=h(2, 4)),
        lambda: fs.project(ctx, h(2, 8), i8(3, 8), f(3), norm=fs.Norm(f(7))),
        lambda: fs.project(ctx, h(2, 8), i8(3, 8), f(3), norm=fs.Norm(h(8))),
        lambda: fs.project(ctx, h(2, 8), i8(3, 8), f(3), norm=fs.Norm(None, 0.0)),
        lambda: fs.project(ctx, h(2, 8), i8(3, 8), f(3), norm=fs.Norm(None, math.nan)),
        lambda: fs.project(ctx, h(2, 8), i8(3, 8), f(3), norm=fs.Norm(None, math.inf)),
        lambda: fs.project(ctx, h(2, 8), i8(3, 8), f(3), workspace=torch.empty(4096, dtype=torch.uint8)),
        lambda: fs.project(ctx, square, i8(8, 8), f(8), out=square),
        lambda: fs.project(ctx, h(2, 8), i8(3, 8), f(3), out=h(4, 3)[::2], residual=f(2, 3)),
        lambda: fs.gated_project(ctx, h(2, 8), i8(3, 8), f(3)),
        lambda: fs.gated_project(ctx, h(2, 8), i8(6, 8), f(3)),
        lambda: fs.gated_project(ctx, h(2, 8), i8(6, 8), f(6), out=h(2, 6)),
        lambda: fs.gated_project(ctx, h(2, 8).cpu(), i8(6, 8), f(6)),
    ]
    for i, call in enumerate(cases):
        with pytest.raises(fs.FleetSieveError) as e:
            call()
        assert e.value.status == fs.FS_ERR_INVALID_ARGUMENT, (i, str(e.value))
    for call in (lambda ws: fs.project(ctx, h(2, 64), i8(3, 64), f(3), workspace=ws),
                 lambda ws: fs.gated_project(ctx, h(2, 64), i8(6, 64), f(6), workspace=ws)):
        with pytest.raises(fs.FleetSieveError) as e:
            call(i8(8).view(torch.uint8))
        assert e.value.status == fs.FS_ERR_WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("M", [1, 4, 70])
def test_streams_graphs_and_plans(env, M):
    """A run as a layer has it: into the gated block and out of it, added to the
    stream; eager on two streams, and captured and replayed with other inputs
    between."""
    fs, ctx = env
    note(f"feed-forward block in a graph, {M} rows")
    K, F = 512, 1040
    x, w, sw, _, gain = inputs(M, F, K, "bf16", rows=2 * F)
    _, w2, sw2, _, _ = inputs(M, K, F, "bf16")
    h = d(x)
    side = torch.cuda.Stream()
    spaces = [torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0") for _ in range(2)]
    a = (d(w), d(sw), fs.Norm(d(gain), EPS), d(w2), d(sw2))

    def block(h, stream=None, ws=None):
        gated = fs.gated_project(ctx, h, a[0], a[1], norm=a[2], stream=stream, workspace=ws)
        return fs.project(ctx, gated, a[3], a[4], residual=h, stream=stream, workspace=ws)
    want = block(h)
    side.wait_stream(torch.cuda.current_stream())
    got = block(h, side, spaces[0])
    side.synchronize()
    assert torch.equal(bits(got), bits(want))
    mid, room = ref.gated(x, w, sw, (gain, EPS), None, "silu", torch.bfloat16)
    end, _ = ref.project(mid.to(torch.bfloat16), w2, sw2, residual=x)
    # the block's inner rounding and codes move it by a step of 8 bits of each row at most
    assert ((want.double().cpu() - end).norm() / end.norm()) < 0.02
    graph = torch.cuda.CUDAGraph()
    fixed = h.clone()
    with torch.cuda.graph(graph, stream=side):
        out = block(fixed, side, spaces[1])
    for i in range(4):
        fixed.copy_(torch.randn(M, K, generator=gen(i)))
        want = block(fixed)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(want)), i
    # plans hold the memory that they run on
    plan = fs.GatedProjectPlan(ctx, h.clone(), a[0].clone(), a[1].clone(), norm=fs.Norm(d(gain).clone(), EPS))
    filler = [torch.full((1 << 20,), 77, dtype=torch.int8, device="cuda:0") for _ in range(4)]
    assert torch.equal(bits(plan.run()), bits(fs.gated_project(ctx, h, a[0], a[1], norm=a[2])))
    del filler


def test_results_are_the_same_on_every_run(env):
    fs, ctx = env
    for M, N, K in ((1, 2560, 5120), (3, 1000, 2048), (60, 777, 1333), (700, 1100, 640)):
        x, w, sw, bias, gain = inputs(M, N, K, "bf16", rows=2 * N)
        plan = fs.GatedProjectPlan(ctx, d(x), d(w), d(sw), norm=fs.Norm(d(gain), EPS), bias=d(bias))
        first = bits(plan.run().clone())
        assert all(torch.equal(bits(plan.run()), first) for _ in range(3))


# long inner dimensions, along which the tiles of some of these are cut (that they are is
# seen to in test_gpu_cut_products.py)
CUT = [(5, 40, 2048), (16, 200, 8192), (9, 515, 5000), (20, 1000, 20480), (33, 2000, 3001), (64, 640, 4096), (64, 5120, 20480),
       (64, 20480, 2560), (100, 2000, 9999), (130, 1300, 4096), (300, 4000, 4096), (700, 2560, 6144), (1500, 5120, 4096),
       (2500, 5121, 3333), (5000, 5120, 4096)]


@pytest.mark.parametrize("M,N,K", CUT)
def test_products_cut_along_the_inner_dimension(env, M, N, K):
    """The same whole numbers, so the bits of the projection that is not cut; twice on
    a workspace of any contents."""
    fs, ctx = env
    note(f"cut {M}x{N}x{K}")
    g = torch.Generator(device="cuda:0").manual_seed(M + N)
    x = torch.randn(M, K, device="cuda:0", generator=g).to(torch.bfloat16)
    w = torch.randint(-127, 128, (2 * N, K), device="cuda:0", generator=g, dtype=torch.int8)
    sw = torch.rand(2 * N, device="cuda:0", generator=g) / (100.0 * math.sqrt(K))
    res = torch.randn(M, N, device="cuda:0", generator=g).to(torch.bfloat16)
    gate, value = (fs.linear(ctx, x, w[r], sw[r], out_dtype=torch.float32) for r in (slice(0, N), slice(N, 2 * N)))
    ws = torch.empty(1 << 28, dtype=torch.uint8, device="cuda:0")
    for fill in (255, 1):
        ws.fill_(fill)
        got = fs.project(ctx, x, w[:N], sw[:N], residual=res, workspace=ws)
        assert torch.equal(bits(got), bits((gate + res.float()).to(torch.bfloat16)))
        for _ in range(2):
            got = fs.gated_project(ctx, x, w, sw, activation="none", workspace=ws)
            assert torch.equal(bits(got), bits((gate * value).to(torch.bfloat16)))


def test_cut_products_in_a_graph(env):
    fs, ctx = env
    M, N, K = 64, 640, 8192
    x, w, sw, _, gain = inputs(M, N, K, "bf16", rows=2 * N)
    a = (ctx, d(x), d(w), d(sw))
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda:0")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = fs.gated_project(*a, norm=fs.Norm(a[3][:0].new_ones(K), EPS), stream=side, workspace=ws)
    for i in range(4):
        a[1].copy_(torch.randn(M, K, generator=gen(i)))
        want = fs.gated_project(*a, norm=fs.Norm(None, EPS))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(want)), i
