"""The serving operators on the GPU at the edges of what they accept: values
that are no numbers or nearly none, sizes near 2^31, buffers longer than what
is in them, windows on every kernel, workspaces of any contents."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import serving_reference as ref  # noqa: E402
from test_gpu_serving import STEP, TYPES, attention_case, bits, env, gen, note, wide  # noqa: E402, F401


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("value", [math.inf, -math.inf])
@pytest.mark.parametrize("D,page,length", [(64, 64, 1), (128, 16, 150), (64, 32, 1200)])
def test_an_infinite_query_gives_no_numbers(env, D, page, length, value, dtype):
    """Keys of one sign at the infinity's element, so that all its logits have one too."""
    fs, ctx = env
    note(f"infinite query D{D} page{page} {length} {value} {dtype}")
    c = ref.Paged([length], 1, D, page, seed=3)
    c.k[..., 5] = c.k[..., 5].abs().clamp(min=1)
    q = torch.randn(1, 3, D, generator=gen(length)).to(TYPES[dtype])
    q[0, 1, 5] = value
    got = fs.cache_attention(ctx, c.device(fs), q.to("cuda:0"), c.table.to("cuda:0"), i32([length]), i32([0, 1]), 1).cpu()
    assert torch.isnan(got[0, 1]).all() and torch.isfinite(got[0, ::2]).all()


@pytest.mark.parametrize("new", [3, 200])
def test_a_scale_that_is_not_finite_reaches_rows_that_see_it(env, new):
    """A code of zero under an infinite scale is no number, whatever the sign
    of the sum that the others make."""
    fs, ctx = env
    note(f"scales that are not finite, {new} tokens")
    for of, scale in (("k_scale", math.inf), ("k_scale", math.nan), ("v_scale", math.inf), ("v_scale", math.nan)):
        c = wide([300], 1, 64, 16, seed=5) if new > 100 else ref.Paged([300], 1, 64, 16, seed=5)
        page = int(c.table[0, 299 // 16])  # tokens 288 .. 299
        c.k[page] = -50
        c.k[page, ..., 7] = 0
        getattr(c, of)[page] = scale
        q = torch.rand(new, 1, 64, generator=gen(2)).to(torch.bfloat16) + 0.5
        got = fs.cache_attention(ctx, c.device(fs), q.to("cuda:0"), c.table.to("cuda:0"), i32([300]), i32([0, new]), new).cpu()
        sees = torch.arange(300 - new, 300) >= 288
        assert torch.isnan(got[sees]).all() and torch.isfinite(got[~sees]).all()


def test_an_appended_infinity_makes_its_page_no_numbers(env):
    fs, ctx = env
    for value in (math.inf, -math.inf):
        kv = fs.KVCache.empty(4, 2, 64, 16, "cuda:0")
        k, v = torch.ones(20, 2, 64, device="cuda:0"), torch.ones(20, 2, 64, device="cuda:0")
        k[18, 1, 3], v[2, 0, 9] = value, value
        slots = torch.arange(20, dtype=torch.int32, device="cuda:0")
        fs.cache_append(ctx, kv, k, v, slots)
        rk, rv = (t.cpu() for t in fs.cache_read(ctx, kv, slots))
        assert torch.isnan(rk[16:, 1]).all() and torch.isnan(rv[:16, 0]).all()
        assert torch.isfinite(rk[:, 0]).all() and torch.isfinite(rk[:16]).all()
        assert torch.isfinite(rv[:, 1]).all() and torch.isfinite(rv[16:]).all()
        q = torch.ones(1, 2, 64, dtype=torch.float16, device="cuda:0")
        got = fs.cache_attention(ctx, kv, q, i32([[0, 1]]), i32([20]), i32([0, 1]), 1).cpu()
        assert torch.isnan(got).all()  # head 0 by a value, head 1 by a key


@pytest.mark.parametrize("new,length", [(1, 1), (1, 150), (3, 4000), (200, 300)])
def test_logits_far_below_zero(env, new, length):
    """Logits of about -1.6e34, the same for all tokens: the mean of the values that a row sees."""
    fs, ctx = env
    note(f"logits far below zero, {new} of {length}")
    c = wide([length], 1, 64, 64, seed=9) if new > 100 else ref.Paged([length], 1, 64, 64, seed=9)
    c.k[:] = 100
    c.k_scale[:] = 0.02
    q = torch.full((new, 2, 64), -1e33, dtype=torch.bfloat16)
    got = fs.cache_attention(ctx, c.device(fs), q.to("cuda:0"), c.table.to("cuda:0"), i32([length]), i32([0, new]), new).cpu()
    _, v = c.values(0)
    for j in range(new):
        seen = v[:length - new + 1 + j, 0]
        assert ((got[j].double() - seen.mean(dim=0)).abs() <= 2.0 ** -8 * seen.mean(dim=0).abs() + 2.0 ** -10 * seen.abs().amax()).all()


@pytest.mark.parametrize("group,news,length,room", [(5, [300, 10], 4000, 600), (5, [300, 1, 0], 4000, 900), (2, [9, 3], 100, 40)])
def test_a_buffer_of_more_rows_than_the_sequences_have(env, group, news, length, room, monkeypatch):
    """All rows of the sequences are computed, and the rows behind them are left as they are."""
    fs, ctx = env
    note(f"padded rows {news} in {room}")
    heads, D, S = 8, 64, len(news)
    c = ref.Paged([length - 7 * s for s in range(S)], heads, D, 64, seed=room)
    starts = [sum(news[:s]) for s in range(S + 1)]
    q = torch.randn(room, heads * group, D, generator=gen(room)).to(torch.bfloat16)
    out = torch.full((room, heads * group, D), 7.0, dtype=torch.bfloat16, device="cuda:0")
    fs.cache_attention(ctx, c.device(fs), q.to("cuda:0"), c.table.to("cuda:0"), i32(c.lengths), i32(starts), max(news), out=out)
    got = out.cpu()
    monkeypatch.setenv("FS_VALIDATE", "1")  # such a buffer is no error
    fs.cache_attention(ctx, c.device(fs), q.to("cuda:0"), c.table.to("cuda:0"), i32(c.lengths), i32(starts), max(news), out=out)
    assert torch.equal(bits(out), bits(got))
    for s, n in enumerate(news):
        if n == 0:
            continue
        k, v = c.values(s)
        # of a long prompt the first and last tokens
        for rows in ([range(n)] if n < 20 else [range(4), range(n - 4, n)]):
            part = q[starts[s] + rows[0]:starts[s] + rows[-1] + 1]
            first = c.lengths[s] - n + rows[0]
            want = ref.attend(part, k, v, first, D ** -0.5)
            bound = ref.attention_bound(part, k, v, first, D ** -0.5, 0, want, STEP["bf16"])
            assert ((got[starts[s] + rows[0]:starts[s] + rows[-1] + 1].double() - want).abs() <= bound).all()
    assert (got[starts[-1]:] == 7.0).all()


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 3, 2 ** 30])
def test_windows_near_the_largest_number(env, window):
    """Also where the cache has fewer tokens than are new, so that positions are negative."""
    attention_case(env, [5, 40, 0], [10, 3, 4], 1, 2, 64, 16, window, "bf16")
    attention_case(env, [60], [200], 1, 2, 64, 64, window, "f16", cache=wide([60], 1, 64, 64, seed=3))


def test_tokens_of_a_page_that_do_not_follow_one_another_are_refused(env, monkeypatch):
    fs, ctx = env
    note("tokens that do not follow")
    monkeypatch.setenv("FS_VALIDATE", "1")
    kv = fs.KVCache.empty(4, 1, 64, 64, "cuda:0")
    x = torch.ones(6, 1, 64, device="cuda:0")
    for slots in ([3, 70, 4], [3, -1, 4], [5, 5], [5, 4], [64, 65, 3, 130, 66], [0, 1, 64, 0], [-1, 9, 10, 12]):
        with pytest.raises(fs.FleetSieveError) as e:
            fs.cache_append(ctx, kv, x[:len(slots)], x[:len(slots)], i32(slots))
        assert e.value.status == fs.FS_ERR_INVALID_ARGUMENT and "do not follow" in str(e.value), slots
    assert not kv.k.any() and not kv.k_scale.any()
    for slots in ([3, 4, 70], [3, -1, 70, 71], [62, 63, 64, 65], [127, 128, 5, 6, -1, 200], [-1, -1]):
        fs.cache_append(ctx, kv, x[:len(slots)], x[:len(slots)], i32(slots))
        k, _ = fs.cache_read(ctx, kv, i32([s for s in slots if s >= 0]))
        assert ((k - 1).abs() < 1e-6).all()


def test_checks_that_wait_are_refused_under_capture(env, monkeypatch):
    """The capture goes on, and what it recorded before and after replays."""
    fs, ctx = env
    note("checks under capture")
    kv = fs.KVCache.empty(2, 1, 64, 16, "cuda:0")
    x, slots = torch.ones(3, 1, 64, device="cuda:0"), i32([1, 2, 3])
    q, table, lens, cu = torch.ones(1, 1, 64, device="cuda:0").half(), i32([[0]]), i32([4]), i32([0, 1])
    side = torch.cuda.Stream()
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda:0")
    plans = [fs.AppendPlan(ctx, kv, x, x, slots, stream=side), fs.ReadPlan(ctx, kv, slots, stream=side),
             fs.AttentionPlan(ctx, kv, q, table, lens, cu, 1, stream=side, workspace=ws)]
    y = torch.zeros(4, device="cuda:0")
    torch.cuda.synchronize()
    monkeypatch.setenv("FS_VALIDATE", "1")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y.add_(1.0)
        for plan in plans:
            with pytest.raises(fs.FleetSieveError) as e:
                plan.run()
            assert e.value.status == fs.FS_ERR_DEVICE and "captured" in str(e.value)
        y.add_(1.0)
    for i in range(1, 4):
        graph.replay()
        torch.cuda.synchronize()
        assert (y == 2.0 * i).all()


@pytest.mark.parametrize("T,max_q,width", [(16384, 16384, 2048), (25, 25, 16384)])
def test_sequences_that_overlap_end_without_harm(env, T, max_q, width):
    """Rows 0 .. T - 1 given to 2048 sequences: more units of work than 32 bits count."""
    fs, ctx = env
    note(f"overlapping sequences, {T} rows")
    S, heads, group, D = 4096, 8, 5, 64
    c = ref.Paged([70], heads, D, 64, seed=1)
    kv = c.device(fs)
    q = torch.zeros(T, heads * group, D, dtype=torch.bfloat16, device="cuda:0")
    table = torch.zeros(S, width, dtype=torch.int32, device="cuda:0")
    lens = torch.full((S,), width * 64, dtype=torch.int32, device="cuda:0")
    cu = i32([0, T] * (S // 2) + [0])
    fs.cache_attention(ctx, kv, q, table, lens, cu, max_q)
    torch.cuda.synchronize()
    attention_case(env, [70, 300], [3, 1], 1, 2, 64, 16, 0, "bf16")


def test_a_row_of_nearly_two_to_the_31_elements(env):
    """Its last eight pass 2^31 - 1; nothing behind the row is read or written."""
    fs, ctx = env
    cols = 2 ** 31 - 1
    note(f"quantize 1x{cols}")
    x = torch.zeros(cols + 65, dtype=torch.float16, device="cuda:0")
    for at in range(0, cols, 1 << 28):
        n = min(1 << 28, cols - at)
        x[at:at + n] = (torch.arange(at, at + n, dtype=torch.int64, device="cuda:0") % 201 - 100).half()
    x[cols:] = 5000.0
    codes = torch.full((cols + 65,), 77, dtype=torch.int8, device="cuda:0")
    scale = torch.empty(1, device="cuda:0")
    fs._check(fs.load_library().fs_quantize_rows(ctx.handle, x.data_ptr(), fs.F16, 1, cols, cols + 65, codes.data_ptr(), cols + 65,
                                                 scale.data_ptr(), fs._stream(x.device, None)))
    assert scale.item() == float(torch.tensor(100.0) / 127.0)
    inverse = torch.tensor(127.0, device="cuda:0") / torch.tensor(100.0, device="cuda:0")
    for at in (0, 1 << 30, cols - (1 << 20)):
        want = torch.round(x[at:min(at + (1 << 20), cols)].float() * inverse).to(torch.int8)
        assert torch.equal(codes[at:at + want.numel()], want)
    assert (codes[cols:] == 77).all()


def test_more_rows_than_a_launch_has_blocks(env):
    fs, ctx = env
    rows, cols = 2 ** 24 + 5, 4
    note(f"quantize {rows}x{cols}")
    x = torch.randn(rows, cols, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(3)).half()
    codes, scale = fs.quantize_rows(ctx, x)
    a = x.float().abs().amax(dim=1, keepdim=True)
    assert torch.equal(scale, a[:, 0] / torch.full_like(a[:, 0], 127.0))
    assert torch.equal(codes, torch.round(x.float() * (torch.full_like(a, 127.0) / a)).to(torch.int8))


def test_more_channels_than_a_launch_of_one_row_has_tiles(env):
    fs, ctx = env
    N, K = 2 ** 28 + 5, 16
    note(f"linear 1x{N}x{K}")
    g = torch.Generator("cuda:0").manual_seed(4)
    w = torch.randint(-127, 128, (N, K), generator=g, dtype=torch.int8, device="cuda:0")
    sw = torch.full((N,), 0.01, device="cuda:0")
    x = torch.randn(1, K, generator=g, device="cuda:0").bfloat16()
    y = fs.linear(ctx, x, w, sw)
    codes, scale = fs.quantize_rows(ctx, x)
    for at in (0, N // 2, N - 4096):
        total = (w[at:at + 4096].double() * codes.double()).sum(dim=1)  # exact: below 2^53
        assert torch.equal(y[0, at:at + 4096], (total.float() * scale * sw[:4096]).bfloat16())


def test_products_of_nearly_two_to_the_31_channels(env):
    fs, ctx = env
    g = torch.Generator("cuda:0").manual_seed(5)
    most = 2 ** 31 - 1
    w = torch.empty(most, 1, dtype=torch.int8, device="cuda:0")
    w.view(torch.uint8).random_(0, 256, generator=g)
    sw = torch.full((most,), 0.5, device="cuda:0")
    a, sa = torch.full((1, 1), 3, dtype=torch.int8, device="cuda:0"), torch.ones(1, device="cuda:0")
    N = (2 ** 23 - 8) * 256
    note(f"matmul 1x{N}x1")
    y = fs.scaled_matmul(ctx, a, sa, w[:N], sw[:N], out_dtype=torch.float16)
    for at in (0, N // 2 - 300, N - 5000):
        assert torch.equal(y[0, at:at + 5000], (w[at:at + 5000, 0].float() * 1.5).half()[:min(5000, N - at)])
    del y
    with pytest.raises(fs.FleetSieveError) as e:
        fs.scaled_matmul(ctx, a, sa, w, sw, out_dtype=torch.float16)
    assert e.value.status == fs.FS_ERR_UNSUPPORTED


def test_more_tokens_than_a_launch_reads(env):
    fs, ctx = env
    T = 2 ** 28 + 20
    note(f"read of {T} tokens")
    c = ref.Paged([640], 1, 64, 16, seed=2)
    kv = c.device(fs)
    kv.k_scale.fill_(0.01)
    slots = torch.arange(T, dtype=torch.int32, device="cuda:0") % 637
    out = torch.empty(T, 1, 64, dtype=torch.float16, device="cuda:0")
    cache = kv._struct()
    import ctypes
    fs._check(fs.load_library().fs_cache_read(ctx.handle, ctypes.byref(cache), T, slots.data_ptr(), out.data_ptr(), None, fs.F16,
                                              fs._stream(out.device, None)))
    for at in (0, 2 ** 27 - 100, T - 4000):
        s = slots[at:at + 4000].long()
        assert torch.equal(out[at:at + 4000], (kv.k[s // 16, :, s % 16].float() * kv.k_scale[s // 16][:, :, None]).half())


# ------------------------------------------------ each attention kernel by itself --
@pytest.fixture(params=[1, 2], ids=["16rows", "256rows"])
def one_kernel(env, request):
    """Every sequence by the kernel of 16 rows, or by that of 256, whatever the sizes."""
    fs, ctx = env
    ctx.set_option(fs.OPT_ATTENTION_KERNEL, request.param)
    yield request.param
    ctx.set_option(fs.OPT_ATTENTION_KERNEL, 0)


def test_kernels_that_are_none(env):
    fs, ctx = env
    for value in (-1, 3):
        with pytest.raises(fs.FleetSieveError) as e:
            ctx.set_option(fs.OPT_ATTENTION_KERNEL, value)
        assert e.value.status == fs.FS_ERR_INVALID_ARGUMENT


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("window", [0, 1, 40, 300])
@pytest.mark.parametrize("D,page,heads,group", [(128, 64, 2, 5), (128, 32, 1, 3), (128, 16, 1, 8), (64, 64, 2, 2), (64, 32, 3, 4),
                                                (64, 16, 1, 1)])
def test_windows(env, one_kernel, D, page, heads, group, window, dtype):
    lengths, news = [200, 33, 530, 1, 130, 0, 90, 64, 65], [200, 1, 137, 1, 16, 2, 90, 64, 63]
    attention_case(env, lengths, news, heads, group, D, page, window, dtype, seed=window)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lengths,news,heads,group,window", [([3000, 2900], [150, 700], 1, 2, 1000), ([2600], [300], 2, 1, 0),
                                                             ([4100], [1537], 1, 1, 700), ([260] * 12, [256] * 12, 2, 1, 100),
                                                             ([100, 300], [250, 200], 1, 2, 70)])
def test_windows_over_cut_contexts(env, one_kernel, D, lengths, news, heads, group, window):
    attention_case(env, lengths, news, heads, group, D, 64 if D == 128 else 32, window, "bf16" if D == 128 else "f16")


@pytest.mark.parametrize("D,page", [(128, 64), (128, 16), (64, 32), (64, 64)])
def test_pages_below_the_window_may_be_anything(env, one_kernel, D, page):
    """Entries that are no pages, and pages whose scales are no numbers."""
    lengths, new, window = [900], 290, 100
    c = ref.Paged(lengths, 1, D, page, seed=6)
    good = ref.Paged(lengths, 1, D, page, seed=6)
    first = 900 - new - window + 1  # of the tokens that are seen
    for i in range(first // page):
        if i % 3 == 0:
            c.k_scale[int(c.table[0, i])] = math.nan
            c.v_scale[int(c.table[0, i])] = math.inf
        else:
            c.table[0, i] = -1 if i % 3 == 1 else 1 << 30
    with pytest.MonkeyPatch.context() as m:
        m.setattr(c, "values", good.values)
        attention_case(env, lengths, [new], 1, 2, D, page, window, "f16", cache=c)


def counted_plans(fs, ctx, kernel, make_workspace):
    """Plans whose blocks count the parts of the items that they cut: items of 24
    and 15 tiles in runs of 4 (the kernel of 16 rows) or 8, fewer than twelve
    parts each."""
    c = ref.Paged([1500, 900], 1, 128, 64, seed=1)
    kv, table, lens = c.device(fs), c.table.to("cuda:0"), i32([1500, 900])
    for n, group in ((1, 5), (3, 4)) if kernel == 1 else ((1, 5), (300, 2)):
        q = torch.randn(2 * n, group, 128, generator=gen(n)).to(torch.bfloat16).to("cuda:0")
        yield c, q, fs.AttentionPlan(ctx, kv, q, table, lens, i32([0, n, 2 * n]), n, workspace=make_workspace())


def test_counts_of_parts_in_workspaces_of_any_contents(env, one_kernel):
    """Words that look like counts, with any number of arrivals in their low 12
    bits: results are the same, and what was counted is left at zero."""
    fs, ctx = env
    note(f"counts of parts, kernel {one_kernel}")
    g = torch.Generator().manual_seed(7)
    any_word = torch.randint(-2 ** 62, 2 ** 62, (512,), generator=g)
    contents = [torch.full((512,), 1), torch.full((512,), -1), (torch.arange(512) << 12) + torch.arange(512) % 13 + 1,
                (any_word & ~0xfff) + torch.arange(512) % 13 + 1]
    results = {}
    for words in contents:
        assert (words != 0).all()

        def workspace():
            ws = torch.full((80 << 20,), 255, dtype=torch.uint8, device="cuda:0")
            ws[:4096] = words.contiguous().view(torch.uint8).to("cuda:0")
            return ws
        for c, q, plan in counted_plans(fs, ctx, one_kernel, workspace):
            n = q.shape[0] // 2
            ws = plan._keep[-1]
            for _ in range(3):
                got = plan.run().clone()
                assert torch.equal(bits(got), bits(results.setdefault(n, got)))
                # parts were counted: a counter that came back at zero, and none left in between
                counters = ws[:4096].view(torch.int64).cpu()
                assert (counters == 0).any() and ((counters == 0) | (counters == words)).all()
    for n, got in results.items():
        k, v = c.values(0)
        q = next(q for _, q, _ in counted_plans(fs, ctx, one_kernel, workspace) if q.shape[0] == 2 * n).cpu()
        want = ref.attend(q[:n], k, v, 1500 - n, 128 ** -0.5)
        bound = ref.attention_bound(q[:n], k, v, 1500 - n, 128 ** -0.5, 0, want, STEP["bf16"])
        assert ((got.cpu()[:n].double() - want).abs() <= bound).all()


def test_cut_items_are_the_same_on_every_run(env, one_kernel):
    """Whichever block arrives last adds the parts in their order."""
    fs, ctx = env
    note(f"every run, kernel {one_kernel}")
    ws = torch.zeros(80 << 20, dtype=torch.uint8, device="cuda:0")
    for _, _, plan in counted_plans(fs, ctx, one_kernel, lambda: ws):
        first = plan.run().clone()
        for _ in range(40):
            assert torch.equal(bits(plan.run()), bits(first))


# ------------------------------------------------------ tensors and streams --
def every_plan(fs, ctx, stream=None, workspace=None):
    """(call, the tensors that it is given) for every serving call."""
    dev = "cuda:0"
    i8 = lambda *s: torch.ones(*s, dtype=torch.int8, device=dev)  # noqa: E731
    f = lambda *s: torch.ones(*s, device=dev)  # noqa: E731
    h = lambda *s: torch.ones(*s, device=dev, dtype=torch.float16)  # noqa: E731
    kv = fs.KVCache.empty(4, 2, 64, 16, dev)
    cache = [kv.k, kv.v, kv.k_scale, kv.v_scale]
    t = dict(a=i8(2, 64), a_scale=f(2), w=i8(3, 64), w_scale=f(3), bias=f(3), out=h(2, 3))
    yield lambda: fs.scaled_matmul(ctx, **t, stream=stream, workspace=workspace), list(t.values())
    u = dict(x=h(2, 64), w=i8(3, 64), w_scale=f(3), bias=f(3), out=h(2, 3))
    yield lambda: fs.linear(ctx, **u, stream=stream, workspace=workspace), list(u.values())
    n = dict(k=h(2, 2, 64), v=h(2, 2, 64), slots=i32([0, 1]), q=h(2, 4, 64), positions=i32([0, 1]), cos=f(3, 32), sin=f(3, 32),
             q_out=h(2, 4, 64))
    yield lambda: fs.cache_append(ctx, kv, **n, stream=stream), list(n.values()) + cache
    slots, outs = i32([0, 1]), (h(2, 2, 64), h(2, 2, 64))
    yield lambda: fs.cache_read(ctx, kv, slots, torch.float16, outs, stream=stream), [slots, *outs] + cache
    s = dict(q=h(2, 4, 64), block_table=i32([[0]]), ctx_lens=i32([2]), cu_q=i32([0, 2]), max_q=2, out=h(2, 4, 64))
    yield (lambda: fs.cache_attention(ctx, kv, **s, stream=stream, workspace=workspace),
           [x for x in s.values() if isinstance(x, torch.Tensor)] + cache)
    x = h(2, 64)
    yield lambda: fs.quantize_rows(ctx, x, stream=stream), [x]


def test_every_tensor_is_held_against_the_context_device(env, monkeypatch):
    fs, ctx = env
    seen, check = [], fs._same_device

    def record(ctx, **tensors):
        seen.extend(t for t in tensors.values() if t is not None)
        check(ctx, **tensors)
    monkeypatch.setattr(fs, "_same_device", record)
    for call, tensors in every_plan(fs, ctx, workspace=torch.empty(80 << 20, dtype=torch.uint8, device="cuda:0")):
        seen.clear()
        call()
        assert {t.data_ptr() for t in tensors} <= {t.data_ptr() for t in seen}


def test_workspaces_that_are_refused(env):
    fs, ctx = env
    size = 80 << 20
    for ws in (torch.empty(size, dtype=torch.uint8), torch.empty(size // 4, dtype=torch.float32, device="cuda:0"),
               torch.empty(2 * size, dtype=torch.uint8, device="cuda:0")[::2]):
        for i, (call, _) in enumerate(every_plan(fs, ctx, workspace=ws)):
            if i not in (0, 1, 4):  # calls without a workspace
                continue
            with pytest.raises(fs.FleetSieveError) as e:
                call()
            assert e.value.status == fs.FS_ERR_INVALID_ARGUMENT and "workspace" in str(e.value)


def later(stream):
    """Work of some tens of milliseconds ahead of what `stream` is given next."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(50_000_000)


def test_outputs_for_another_stream_are_not_memory_that_the_current_one_still_reads(env):
    fs, ctx = env
    note("outputs for another stream")
    n = 1 << 11
    w, sw = torch.ones(n, 64, dtype=torch.int8, device="cuda:0"), torch.ones(n, device="cuda:0")
    x = torch.ones(n, 64, dtype=torch.bfloat16, device="cuda:0")
    side, current = torch.cuda.Stream(), torch.cuda.current_stream()
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda:0")
    for _ in range(2):  # the second time both pools hold memory
        read = torch.full((n, n), 7.0, dtype=torch.bfloat16, device="cuda:0")
        torch.cuda.synchronize()
        later(current)
        copy = torch.empty_like(read)
        copy.copy_(read)
        del read  # its memory is the current stream's again, which has yet to copy it
        out = fs.linear(ctx, x, w, sw, stream=side, workspace=ws)
        torch.cuda.synchronize()
        assert (copy == 7.0).all() and torch.isfinite(out).all() and not (out == 7.0).any()
        del out, copy


def test_inputs_and_workspaces_given_back_while_another_stream_works_on_them(env):
    fs, ctx = env
    note("inputs for another stream")
    n, K = 1 << 10, 1 << 11
    w, sw = torch.ones(64, K, dtype=torch.int8, device="cuda:0"), torch.ones(64, device="cuda:0")
    side = torch.cuda.Stream()
    own = fs.Context(0)
    x = torch.ones(n, K, dtype=torch.bfloat16, device="cuda:0")
    want = fs.linear(ctx, x, w, sw)
    torch.cuda.synchronize()
    later(side)
    got = fs.linear(own, x, w, sw, stream=side)
    old = own.workspace(0).numel()
    del x
    own.workspace(4 * old)  # another workspace: the one in use is given back
    filler = [torch.full((n, K), 3.0, dtype=torch.bfloat16, device="cuda:0"), torch.full((old,), 255, dtype=torch.uint8, device="cuda:0")]
    torch.cuda.synchronize()
    assert torch.equal(bits(got), bits(want))
    del filler
    own.close()


def test_the_most_sequences_of_a_call(env, one_kernel):
    lengths = [(13 * s) % 90 for s in range(4096)]
    attention_case(env, lengths, [1 + s % 2 if s % 500 == 0 else 1 for s in range(4096)], 1, 1, 128, 64, 0, "bf16")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("offset", [1, 3, 4])
def test_outputs_that_start_anywhere(env, dtype, offset):
    """Outputs from any element of their memory on: the same bits, and nothing beside them."""
    fs, ctx = env
    note(f"outputs at +{offset} {dtype}")
    ty = TYPES[dtype]

    def place(*shape, of=ty):
        flat = torch.full((offset + math.prod(shape) + 9,), 5, dtype=of, device="cuda:0")
        return flat, flat[offset:offset + math.prod(shape)].view(shape)

    def untouched(flat, view):
        return (flat[:offset] == 5).all() and (flat[offset + view.numel():] == 5).all()
    T, heads, group, D = 37, 2, 3, 64
    c = ref.Paged([60], heads, D, 16, seed=4)
    x = torch.randn(T, heads * (group + 2), D, generator=gen(3)).to(ty).to("cuda:0")
    q, k, v = x[:, :heads * group], x[:, heads * group:heads * (group + 1)], x[:, heads * (group + 1):]
    angle = torch.rand(60, 16, generator=gen(5)).to("cuda:0")
    slots = i32(c.slots(0, 60 - T, 60))
    turn = dict(positions=i32(list(range(60 - T, 60))), cos=angle.cos(), sin=angle.sin())
    flat, out = place(T, heads * group, D)
    got = fs.cache_append(ctx, c.device(fs), k, v, slots, q=q, q_out=out, **turn)
    assert torch.equal(bits(got), bits(fs.cache_append(ctx, c.device(fs), k, v, slots, q=q, **turn))) and untouched(flat, out)
    kv = c.device(fs)
    both = [place(T, heads, D) for _ in range(2)]
    fs.cache_read(ctx, kv, slots, ty, tuple(view for _, view in both))
    for (flat, view), want in zip(both, fs.cache_read(ctx, kv, slots, ty)):
        assert torch.equal(bits(view), bits(want)) and untouched(flat, view)
    if dtype != "f32":
        flat, out = place(T, heads * group, D)
        call = lambda **kw: fs.cache_attention(ctx, kv, q, c.table.to("cuda:0"), i32([60]), i32([0, T]), T, **kw)  # noqa: E731
        assert torch.equal(bits(call(out=out)), bits(call())) and untouched(flat, out)


def test_plans_hold_the_memory_that_they_run_on(env):
    """Also where a cache's tensors are exchanged for others."""
    import gc
    import weakref
    fs, ctx = env
    for make in (lambda kv, x, i: fs.AppendPlan(ctx, kv, x, x, i), lambda kv, x, i: fs.ReadPlan(ctx, kv, i),
                 lambda kv, x, i: fs.AttentionPlan(ctx, kv, x, i[None], i + 1, i32([0, 1]), 1)):
        kv = fs.KVCache.empty(2, 1, 64, 16, "cuda:0")
        x, i = torch.ones(1, 1, 64, dtype=torch.float16, device="cuda:0"), i32([0])
        plan = make(kv, x, i)
        held = [weakref.ref(t) for t in (kv.k, kv.v, kv.k_scale, kv.v_scale)]
        for name in ("k", "v", "k_scale", "v_scale"):
            setattr(kv, name, getattr(kv, name).clone())
        gc.collect()
        assert all(r() is not None for r in held)
        plan.run()
    torch.cuda.synchronize()
