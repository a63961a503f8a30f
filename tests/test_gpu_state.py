"""State attention on the GPU, token by token and in chunks, against its
recurrence in 64 bits."""
import ctypes
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import layer_reference as ref  # noqa: E402
from test_gpu_serving import STEP, TYPES, bits, env, gen, note  # noqa: E402, F401


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


class Batch:
    """Sequences with new tokens, the tokens that their states hold, and whether
    these are kept: rows as parts of wider ones, states in a pool of another order
    with places that hold no numbers between."""

    def __init__(self, news, held, keep, heads, group, D, dtype, seed=0, extra=0, pad=0, decay=None):
        g = gen(sum(news) + 7 * D + heads + seed)
        self.news, self.held, self.keep, self.heads, self.group, self.D, self.dtype = news, held, keep, heads, group, D, dtype
        T = sum(news) + extra
        wide = torch.randn(T, (heads * (group + 2)) * D + pad, generator=g).to(TYPES[dtype])
        cut = lambda a, n: wide[:, a * D:(a + n) * D].unflatten(1, (n, D))  # noqa: E731
        self.wide, self.q, self.k, self.v = wide, cut(0, heads * group), cut(heads * group, heads), cut(heads * (group + 1), heads)
        S = len(news)
        order = torch.randperm(S + 2, generator=g).tolist()
        self.index = [order[s] if keep[s] else -1 - s for s in range(S)]
        self.pool = torch.randn(S + 2, heads, D, D, generator=g) * 4
        for p in order[S:]:
            self.pool[p] = math.nan
        for s in range(S):
            if keep[s] and not held[s] and news[s]:
                self.pool[order[s]] = math.nan  # a new sequence's place may hold anything
        self.decay = -(2.0 ** -torch.linspace(0, 8, heads)) if decay is None else torch.tensor(decay)
        self.cu = [0]
        for n in news:
            self.cu.append(self.cu[-1] + n)
        self.scale = D ** -0.5

    def device(self):
        wide, H, G, D = self.wide.to("cuda:0"), self.heads, self.group, self.D
        cut = lambda a, n: wide[:, a * D:(a + n) * D].unflatten(1, (n, D))  # noqa: E731
        ctx_lens = [n + h for n, h in zip(self.news, self.held)]
        return dict(states=self.pool.to("cuda:0"), q=cut(0, H * G), k=cut(H * G, H), v=cut(H * (G + 1), H),
                    state_index=i32(self.index), ctx_lens=i32(ctx_lens), cu_q=i32(self.cu), max_q=max(self.news + [0]),
                    log_decay=self.decay.to("cuda:0"), scale=self.scale)

    def check(self, out, states):
        out, states = out.cpu(), states.cpu()
        pool = self.pool.clone()
        for s, n in enumerate(self.news):
            if n == 0:
                continue
            rows = slice(self.cu[s], self.cu[s] + n)
            start = self.pool[self.index[s]] if self.keep[s] and self.held[s] else torch.zeros_like(self.pool[0])
            want, state, room, state_room = ref.state_attend(self.q[rows], self.k[rows], self.v[rows], start, self.decay, self.scale)
            got = out[rows].double()
            off = (got - want).abs()
            room = room + (want.abs() + room) * STEP[self.dtype] + (2.0 ** -25 if self.dtype == "f16" else 0.0)
            assert torch.isfinite(got).all(), s
            assert (off <= room).all(), (s, n, float(off.max()), float((off / room.clamp(min=1e-300)).max()))
            if self.keep[s]:
                mine = states[self.index[s]].double()
                off = (mine - state).abs()
                assert (off <= state_room + 2.0 ** -149).all(), (s, n, float((off / state_room.clamp(min=1e-300)).max()))
                pool[self.index[s]] = states[self.index[s]]
        assert torch.equal(bits(states), bits(pool))  # every other place as it was


def run(env, batch, **kw):
    fs, ctx = env
    note(f"state {batch.news[:6]} held {batch.held[:6]} heads {batch.heads}x{batch.group} D{batch.D} {batch.dtype}")
    a = batch.device()
    out = fs.state_attention(ctx, **a, **kw)
    batch.check(out, a["states"])
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,heads,group", [(128, 1, 5), (64, 3, 1), (128, 2, 1), (64, 2, 17), (128, 40, 2)])
@pytest.mark.parametrize("news", [[1], [1] * 5, [2, 1, 8, 3]], ids=str)
def test_token_by_token(env, news, D, heads, group, dtype):
    n = len(news)
    run(env, Batch(news, [9, 0, 3, 100, 1][:n], [True, True, False, True, True][:n], heads, group, D, dtype))


@pytest.mark.parametrize("S,heads", [(30, 4), (130, 1), (140, 4), (600, 1)])
def test_many_sequences_token_by_token(env, S, heads):
    """Each width of a block's columns."""
    run(env, Batch([1] * S, [s % 3 for s in range(S)], [s % 7 != 6 for s in range(S)], heads, 2, 64, "bf16"))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,heads,group", [(128, 2, 3), (64, 3, 1), (64, 1, 9), (128, 1, 1)])
@pytest.mark.parametrize("n", [9, 16, 17, 63, 64, 65, 100, 128, 200, 256])
def test_chunks(env, n, D, heads, group, dtype):
    run(env, Batch([n], [0 if n % 2 else 30], [True], heads, group, D, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,heads,group", [(128, 1, 2), (64, 4, 1)])
@pytest.mark.parametrize("news", [[257], [512, 100], [700, 1, 300, 0, 8, 9, 1000], [1, 1, 1500, 256, 255]], ids=str)
def test_segments(env, news, D, heads, group, dtype):
    n = len(news)
    run(env, Batch(news, [0, 4, 50, 0, 0, 7, 9][:n], [True, True, False, True, True, True, True][:n], heads, group, D, dtype))


def test_more_sequences_than_a_wavefront_and_segments_among_them(env):
    news = [(37 * s) % 11 for s in range(150)]
    news[70], news[3], news[149] = 900, 260, 400
    run(env, Batch(news, [s % 4 for s in range(150)], [s % 5 != 4 for s in range(150)], 2, 1, 64, "bf16"))


def test_long_segments(env):
    """So many heads and tokens that a segment has more than four chunks."""
    run(env, Batch([2500, 300], [3, 0], [True, True], 64, 1, 64, "bf16", decay=[-(2.0 ** -(s % 9)) for s in range(64)]))


# (heads, sequences and tokens enough that a block has several chunks, one or two of a
# segment's own sum among them)
MANY = [(128, 64, 3, [330, 300], 0), (128, 96, 5, [257, 64, 400], 0), (64, 200, 4, [449, 130], 0), (128, 128, 1, [200, 450], 0),
        (64, 128, 2, [700, 9], 0), (128, 64, 3, [330, 300], 3), (64, 128, 3, [250, 251], 1), (128, 20, 3, [3000], 0),
        (64, 40, 3, [5000, 1000], 0), (128, 20, 4, [2000, 1999], 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,heads,group,news,pad", MANY, ids=str)
def test_blocks_of_many_chunks(env, D, heads, group, news, pad, dtype):
    fs, ctx = env
    note(f"many chunks D{D} {heads}x{group} {news} pad{pad} {dtype}")
    g = torch.Generator(device="cuda:0").manual_seed(sum(news) + heads)
    T, S = sum(news), len(news)
    wide = torch.randn(T, heads * (group + 2) * D + pad, device="cuda:0", generator=g).to(TYPES[dtype])
    cut = lambda a, n: wide[:, a * D:(a + n) * D].unflatten(1, (n, D))  # noqa: E731
    q, k, v = cut(0, heads * group), cut(heads * group, heads), cut(heads * (group + 1), heads)
    pool = torch.randn(S, heads, D, D, device="cuda:0", generator=g) * 3
    start = pool.clone()
    decay = -torch.exp2(-torch.linspace(0, 9, heads, device="cuda:0"))
    cu = [0]
    for n in news:
        cu.append(cu[-1] + n)
    held = [0] + [7] * (S - 1)
    out = fs.state_attention(ctx, pool, q, k, v, i32(list(range(S))), i32([n + h for n, h in zip(news, held)]), i32(cu), max(news), decay)
    for s, n in enumerate(news):
        rows = slice(cu[s], cu[s] + n)
        for h in range(0, heads, 16):  # so many heads at a time
            of = slice(h, min(h + 16, heads))
            qs = slice(of.start * group, of.stop * group)
            first = start[s, of] if held[s] else torch.zeros_like(start[s, of])
            want, state, room, state_room = ref.state_attend_at_once(q[rows, qs], k[rows, of], v[rows, of], first, decay[of], D ** -0.5)
            got = out[rows, qs].double()
            room = room + (want.abs() + room) * STEP[dtype] + (2.0 ** -25 if dtype == "f16" else 0.0)
            assert ((got - want).abs() <= room).all(), (s, h)
            assert ((pool[s, of].double() - state).abs() <= state_room + 2.0 ** -149).all(), (s, h)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("at", [0, 63, 64, 130, 199])
def test_no_numbers_in_blocks_of_many_chunks(env, at, dtype):
    fs, ctx = env
    heads, group, D, n = 200, 3, 64, 200
    g = torch.Generator(device="cuda:0").manual_seed(at)
    make = lambda h: torch.randn(2 * n, h, D, device="cuda:0", generator=g).to(TYPES[dtype])  # noqa: E731
    q, k, v = make(heads * group), make(heads), make(heads)
    decay = -torch.full((heads,), 0.02, device="cuda:0")
    where = (i32([0, 1]), i32([n, n]), i32([0, n, 2 * n]), n, decay)
    pools = [torch.zeros(2, heads, D, D, device="cuda:0") for _ in range(2)]
    want = fs.state_attention(ctx, pools[0], q, k, v, *where)
    v[n + at, 7, 9] = math.nan
    got = fs.state_attention(ctx, pools[1], q, k, v, *where)
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[n + at:, 7 * group:8 * group, 9] = True
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit])
    hit = torch.zeros_like(pools[0], dtype=torch.bool)
    hit[1, 7, :, 9] = True
    assert torch.isnan(pools[1][hit]).all() and torch.equal(pools[1][~hit], pools[0][~hit])


@pytest.mark.parametrize("n", [1, 8, 100, 600])
@pytest.mark.parametrize("decay", [0.0, -1e-7, -30.0, -1e30, -math.inf])
def test_decays_from_all_to_nothing(env, n, decay):
    run(env, Batch([n, n], [5, 0], [True, True], 1, 2, 64, "bf16", decay=[decay]))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [3, 70, 300])
@pytest.mark.parametrize("pad", [1, 3, 8])
def test_rows_at_any_alignment(env, n, pad, dtype):
    fs, ctx = env
    b = Batch([n, 2], [4, 0], [True, True], 2, 2, 64, dtype, pad=pad)
    a = b.device()
    T, heads, D = a["q"].shape
    flat = torch.full((T * heads * D + 9,), 7.0, dtype=a["q"].dtype, device="cuda:0")
    out = flat[pad:pad + T * heads * D].view(T, heads, D)
    fs.state_attention(ctx, **a, out=out)
    b.check(out, a["states"])
    assert (flat[:pad] == 7.0).all() and (flat[pad + T * heads * D:] == 7.0).all()


@pytest.mark.parametrize("scale", [0.0, -2.0, 100.0])
def test_scales_and_values_of_any_size(env, scale):
    for size in (1e-4, 1.0, 300.0):
        for n in (2, 90):
            b = Batch([n], [2], [True], 1, 1, 64, "f16" if size < 100 else "bf16")
            b.wide *= size
            b.scale = scale
            run(env, b)


@pytest.mark.parametrize("news", [[1, 1], [5, 2], [200, 1], [600, 70]], ids=str)
def test_rows_behind_the_last_sequence_are_left(env, news):
    fs, ctx = env
    b = Batch(news, [1, 0], [True, True], 2, 1, 64, "bf16", extra=5)
    a = b.device()
    out = torch.full(a["q"].shape, 9.0, dtype=torch.bfloat16, device="cuda:0")
    fs.state_attention(ctx, **a, out=out)
    b.check(out, a["states"])
    assert (out[-5:] == 9.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("n,at", [(5, 2), (64, 0), (64, 40), (150, 70), (700, 300)])
def test_what_is_no_number_reaches_what_it_should(env, n, at, bad, dtype):
    """A value, a key, a query of one token: outputs before it, other columns and
    heads stay as they were."""
    fs, ctx = env
    clean = Batch([n], [3], [True], 2, 1, 64, dtype)
    a = clean.device()
    want, pool = fs.state_attention(ctx, **a).cpu(), a["states"].cpu()
    for what in ("q", "k", "v"):
        a = clean.device()
        a[what][at, 1, 5] = bad
        got, states = fs.state_attention(ctx, **a).cpu(), a["states"].cpu()[clean.index[0]]
        assert torch.equal(bits(got[:, 0]), bits(want[:, 0])), what
        assert torch.equal(bits(got[:at, 1]), bits(want[:at, 1])), what
        assert torch.equal(bits(states[0]), bits(pool[clean.index[0], 0])), what
        if what == "q":
            assert not torch.isfinite(got[at, 1]).any()
            assert torch.equal(bits(got[at + 1:]), bits(want[at + 1:])) and torch.isfinite(states).all()
        elif what == "k":
            assert not torch.isfinite(got[at:, 1]).any()
            assert not torch.isfinite(states[1, 5]).any() and torch.isfinite(states[1, :5]).all()
        else:
            assert not torch.isfinite(got[at:, 1, 5]).any() and torch.isfinite(got[at:, 1, :5]).all()
            assert not torch.isfinite(states[1, :, 5]).any() and torch.isfinite(states[1, :, 6:]).all()


def test_a_prompt_in_parts_is_the_prompt(env):
    """The state carries over, whichever form each part takes."""
    fs, ctx = env
    whole = Batch([400], [0], [True], 2, 2, 128, "bf16")
    a = whole.device()
    fs.state_attention(ctx, **a)
    want = a["states"].cpu()[whole.index[0]].double()
    b = whole.device()
    out = torch.empty(400, 4, 128, dtype=torch.bfloat16, device="cuda:0")
    at = 0
    for n in (300, 1, 8, 64, 27):
        part = {x: b[x][at:at + n] for x in "qkv"}
        fs.state_attention(ctx, b["states"], **part, state_index=b["state_index"], ctx_lens=i32([at + n]), cu_q=i32([0, n]),
                           max_q=n, log_decay=b["log_decay"], out=out[at:at + n])
        at += n
    whole.check(out, b["states"])
    assert (b["states"].cpu()[whole.index[0]].double() - want).norm() < 1e-4 * want.norm()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [7, 64, 1000])
def test_states_are_binary32(env, n, dtype):
    """Every term of a state may lose 2^-23 of itself (22 bits) and is added with some
    70 others and partial sums, each rounded by 2^-24 of what is there: if these fall
    either way sqrt(70) of them, together less than 2^-20 of the terms' sizes in the
    root mean square."""
    fs, ctx = env
    b = Batch([n], [5], [True], 3, 1, 64, dtype)
    a = b.device()
    fs.state_attention(ctx, **a)
    got = a["states"].cpu()[b.index[0]].double()
    _, want, _, room = ref.state_attend(b.q, b.k, b.v, b.pool[b.index[0]], b.decay, b.scale)
    lam = torch.exp(b.decay.double())[:, None, None]
    size = b.pool[b.index[0]].double().abs()
    for t in range(n):
        size = lam * size + (b.k[t].double()[:, :, None] * b.v[t].double()[:, None, :]).abs()
    assert (got - want).norm() < 2.0 ** -20 * size.norm()


def test_results_are_the_same_on_every_run(env):
    fs, ctx = env
    for news in ([1] * 9, [300, 1, 70], [1200]):
        b = Batch(news, [1] * len(news), [True] * len(news), 2, 3, 128, "bf16")
        first = None
        for _ in range(4):
            a = b.device()
            got = bits(fs.state_attention(ctx, **a)), bits(a["states"])
            first = first or got
            assert torch.equal(got[0], first[0]) and torch.equal(got[1], first[1])


@pytest.mark.parametrize("news", [[1, 1, 1], [300, 1, 9], [40, 600]], ids=str)
def test_streams_graphs_workspaces(env, news):
    fs, ctx = env
    b = Batch(news, [2] * len(news), [True] * len(news), 2, 2, 64, "bf16")
    side = torch.cuda.Stream()
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda:0")
    a = b.device()
    side.wait_stream(torch.cuda.current_stream())
    ws.fill_(255)
    torch.cuda.synchronize()
    out = fs.state_attention(ctx, **a, stream=side, workspace=ws)
    side.synchronize()
    b.check(out, a["states"])
    # captured, and replayed over other rows: each replay goes on from the states before it
    a, twin = b.device(), b.device()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = fs.state_attention(ctx, **a, stream=side, workspace=ws)
    for i in range(4):
        for x in "qkv":
            new = torch.randn(a[x].shape, generator=gen(i)).to(a[x].dtype)
            a[x].copy_(new)
            twin[x].copy_(new)
        graph.replay()
        want = fs.state_attention(ctx, **twin)
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(want)) and torch.equal(bits(a["states"]), bits(twin["states"])), i


def test_a_layer_of_state_attention(env):
    """The operators together, as a layer calls them: normed projection, attention,
    projection onto the stream, gated block, projection onto the stream."""
    fs, ctx = env
    H, G, D, hidden, F = 2, 2, 64, 256, 320
    news = [70, 1, 5]
    b = Batch(news, [3, 8, 0], [True] * 3, H, G, D, "bf16")
    a, g = b.device(), gen(4)

    def weight(n, k):
        return torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8), torch.full((n,), 1 / (73 * math.sqrt(k)))
    shapes = ((H * (G + 2) * D, hidden), (hidden, H * G * D), (2 * F, hidden), (hidden, F))
    (qkv, so, up, down) = [weight(*s) for s in shapes]
    dev = lambda p: tuple(t.to("cuda:0") for t in p)  # noqa: E731
    x = torch.randn(sum(news), hidden, generator=g).to(torch.bfloat16)
    h = x.to("cuda:0").clone()
    norm = fs.Norm(None, 1e-6)
    rows = fs.project(ctx, h, *dev(qkv), norm=norm).unflatten(1, (-1, D))
    a.update(q=rows[:, :H * G], k=rows[:, H * G:H * (G + 1)], v=rows[:, H * (G + 1):])
    seen = fs.state_attention(ctx, **a)
    fs.project(ctx, seen.flatten(1), *dev(so), residual=h, out=h)
    fs.project(ctx, fs.gated_project(ctx, h, *dev(up), norm=norm), *dev(down), residual=h, out=h)

    real = [w.double() * s.double()[:, None] for w, s in (qkv, so, up, down)]
    want = x.double()
    unit = lambda t: t / (t.pow(2).mean(1, keepdim=True) + 1e-6).sqrt()  # noqa: E731
    r = (unit(want) @ real[0].t()).unflatten(1, (-1, D))
    parts = []
    for s, n in enumerate(news):
        at = slice(b.cu[s], b.cu[s] + n)
        start = b.pool[b.index[s]] if b.held[s] else torch.zeros(H, D, D)
        parts.append(ref.state_attend(r[at, :H * G], r[at, H * G:H * (G + 1)], r[at, H * (G + 1):], start, b.decay, b.scale)[0])
    want = want + torch.cat(parts).flatten(1) @ real[1].t()
    wide = unit(want) @ real[2].t()
    want = want + (torch.nn.functional.silu(wide[:, :F]) * wide[:, F:]) @ real[3].t()
    # eight bits leave a row off by about 0.7% at each of the four products
    change = want - x.double()
    assert (h.double().cpu() - want).norm() < 0.1 * change.norm()


def test_nothing_to_do_and_no_pool(env):
    fs, ctx = env
    e = lambda *s: torch.zeros(*s, dtype=torch.float16, device="cuda:0")  # noqa: E731
    decay = torch.zeros(1, device="cuda:0")
    none = i32([])
    pool = torch.ones(1, 1, 64, 64, device="cuda:0")
    assert fs.state_attention(ctx, pool, e(0, 1, 64), e(0, 1, 64), e(0, 1, 64), none, none, i32([0]), 0, decay).shape == (0, 1, 64)
    assert fs.state_attention(ctx, pool, e(0, 1, 64), e(0, 1, 64), e(0, 1, 64), i32([0]), i32([5]), i32([0, 0]), 0, decay).shape == (0, 1, 64)
    assert (pool == 1).all()
    b = Batch([3, 80], [0, 0], [False, False], 1, 1, 64, "bf16")
    a = b.device()
    a["states"] = torch.empty(0, 1, 64, 64, device="cuda:0")
    want = b.device()
    assert torch.equal(bits(fs.state_attention(ctx, **a)), bits(fs.state_attention(ctx, **want)))


def test_lengths_and_states_out_of_range(env, monkeypatch):
    fs, ctx = env
    b = Batch([2, 70], [3, 1], [True, True], 1, 1, 64, "bf16")
    wrong = [dict(state_index=i32([0, 4])), dict(state_index=i32([1, 1])), dict(cu_q=i32([0, 2, 73])), dict(cu_q=i32([1, 2, 72])),
             dict(cu_q=i32([0, 5, 2])), dict(max_q=69), dict(ctx_lens=i32([-1, 80])), dict(log_decay=torch.tensor([0.1], device="cuda:0")),
             dict(log_decay=torch.tensor([math.nan], device="cuda:0"))]
    monkeypatch.setenv("FS_VALIDATE", "1")
    run(env, b)
    for i, change in enumerate(wrong):
        a = b.device()
        a.update(change)
        with pytest.raises(fs.FleetSieveError) as e:
            fs.state_attention(ctx, **a)
        assert e.value.status == fs.FS_ERR_INVALID_ARGUMENT, i
        assert torch.equal(bits(a["states"]), bits(b.pool))
    a = b.device()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(fs.FleetSieveError) as e:
            fs.state_attention(ctx, **a, stream=side, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0"))
    assert e.value.status == fs.FS_ERR_DEVICE
    monkeypatch.delenv("FS_VALIDATE")
    # an index beyond the pool is none, a positive decay 0, tokens beyond the batch are none
    a = b.device()
    a.update(state_index=i32([7, b.index[1]]), log_decay=torch.tensor([0.5], device="cuda:0"), cu_q=i32([0, 2, 5000]))
    got = fs.state_attention(ctx, **a)
    twin = Batch([2, 70], [3, 1], [False, True], 1, 1, 64, "bf16", decay=[0.0])
    twin.wide, twin.q, twin.k, twin.v, twin.pool, twin.index = b.wide, b.q, b.k, b.v, b.pool, [-1, b.index[1]]
    twin.check(got, a["states"])


def test_arguments_that_are_refused(env):
    fs, ctx = env
    b = Batch([2], [3], [True], 2, 2, 64, "bf16")
    f = lambda *s: torch.zeros(*s, device="cuda:0")  # noqa: E731
    bad, few = fs.FS_ERR_INVALID_ARGUMENT, fs.FS_ERR_UNSUPPORTED
    a = b.device()
    cases = [(bad, dict(states=a["states"][..., :32])), (bad, dict(states=a["states"].half())), (bad, dict(states=a["states"][0])),
             (bad, dict(q=a["q"][:, :3])), (bad, dict(k=a["k"][:1])), (bad, dict(v=a["v"].float())), (bad, dict(q=a["q"].cpu())),
             (few, dict(q=f(2, 4, 64), k=f(2, 2, 64), v=f(2, 2, 64))), (bad, dict(cu_q=i32([0]))), (bad, dict(ctx_lens=i32([1, 2]))),
             (bad, dict(state_index=i32([1]).long())), (bad, dict(log_decay=f(1))), (bad, dict(scale=math.inf)), (bad, dict(max_q=-1)),
             (few, dict(states=f(1, 2, 80, 80), q=f(2, 4, 80).half(), k=f(2, 2, 80).half(), v=f(2, 2, 80).half())),
             (bad, dict(out=f(2, 4, 64))), (few, dict(state_index=i32([0] * 4097), ctx_lens=i32([0] * 4097), cu_q=i32([0] * 4098)))]
    for i, (status, change) in enumerate(cases):
        with pytest.raises(fs.FleetSieveError) as e:
            fs.state_attention(ctx, **{**a, **change})
        assert e.value.status == status, (i, str(e.value))
    long = Batch([600], [3], [True], 2, 2, 64, "bf16").device()
    with pytest.raises(fs.FleetSieveError) as e:
        fs.state_attention(ctx, **long, workspace=torch.empty(1024, dtype=torch.uint8, device="cuda:0"))
    assert e.value.status == fs.FS_ERR_WORKSPACE_TOO_SMALL
    assert torch.equal(bits(a["states"]), bits(b.pool))


@pytest.mark.parametrize("T,S", [(16384, 64), (16384, 4096), (70, 4096), (3, 4096)])
def test_sequences_that_overlap_end_without_harm(env, T, S):
    """All rows given to every other sequence: more segments than the workspace, which
    ends with its last byte, has places for."""
    fs, ctx = env
    note(f"state of overlapping sequences, {T} rows, {S} sequences")
    heads, group, D = 8, 2, 64
    q = torch.zeros(T, heads * group, D, dtype=torch.bfloat16, device="cuda:0")
    k = torch.zeros(T, heads, D, dtype=torch.bfloat16, device="cuda:0")
    pool = torch.ones(2, heads, D, D, device="cuda:0")
    decay = torch.full((heads,), -0.5, device="cuda:0")
    index, lens, cu = i32([-1] * S), i32([T] * S), i32([0, T] * (S // 2) + [0])
    like = fs._StatePool(None, 2, heads, D)
    need = fs._size(fs.load_library().fs_state_attention_workspace_size, ctypes.byref(like), heads * group, T, S)
    room = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda:0")
    out = fs.state_attention(ctx, pool, q, k, k, index, lens, cu, T, decay, workspace=room[:need])
    torch.cuda.synchronize()
    assert (room[need:] == 77).all() and (pool == 1).all() and out.shape == q.shape
    run(env, Batch([70, 300], [3, 1], [True, True], 1, 2, 64, "bf16"))


def test_keys_values_and_queries_of_one_tensor_and_steps_in_a_row(env):
    """One tensor for all three, and 40 calls of a token each against one of 40."""
    fs, ctx = env
    note("40 steps and a prompt of 40")
    H, D = 3, 128
    x = torch.randn(40, H, D, generator=gen(5)).bfloat16()
    decay = torch.tensor([0.0, -0.1, -math.inf])
    want, state, room, state_room = ref.state_attend(x, x, x, torch.zeros(H, D, D), decay, D ** -0.5)
    pools = [torch.full((1, H, D, D), math.nan, device="cuda:0") for _ in range(2)]
    dx, dd = x.to("cuda:0"), decay.to("cuda:0")
    whole = fs.state_attention(ctx, pools[0], dx, dx, dx, i32([0]), i32([40]), i32([0, 40]), 40, dd)
    steps = [fs.state_attention(ctx, pools[1], dx[t:t + 1], dx[t:t + 1], dx[t:t + 1], i32([0]), i32([t + 1]), i32([0, 1]), 1, dd)
             for t in range(40)]
    for out, pool in ((whole, pools[0]), (torch.cat(steps), pools[1])):
        off = (out.cpu().double() - want).abs()
        assert (off <= room + (want.abs() + room) * STEP["bf16"]).all()
        assert ((pool[0].cpu().double() - state).abs() <= state_room + 2.0 ** -149).all()
