"""The serving operators on the GPU against plain 64-bit statements of them:
row quantisation, the product of codes, the paged cache's append and read,
attention over it.  Integers and what is defined in binary32 steps are
compared bit for bit, the rest within bounds derived from the formats."""
import math
import random
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import serving_reference as ref  # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def note(msg):
    print(f"[gpu] {msg}", file=sys.stderr, flush=True)


@pytest.fixture(scope="module")
def env():
    from paper_2608_19659_amd import fleetsieve as fs
    if not torch.cuda.is_available():
        pytest.skip("no ROCm device")
    return fs, fs.Context(0)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def bits(t):
    t = t.cpu().contiguous()
    return t.view({1: torch.int8, 2: torch.int16, 4: torch.int32}[t.element_size()])


# ------------------------------------------------------------ quantisation --
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,stride", [(1, 1, 1), (3, 17, 40), (5, 64, 64), (2, 5120, 5120), (7, 1999, 2001),
                                              (4, 20480, 20480), (2, 40001, 40008)])
def test_quantize_rows(env, dtype, rows, cols, stride):
    fs, ctx = env
    note(f"quantize {dtype} {rows}x{cols}/{stride}")
    x = (torch.randn(rows, stride, generator=gen(cols)) * 3).to(TYPES[dtype])
    x[0, :cols] = 0.0
    view = x.to("cuda:0")[:, :cols]
    codes, scale = (t.cpu() for t in fs.quantize_rows(ctx, view))
    want, want_scale = ref.quantize(x[:, :cols])
    # the binary32 quotient and product are each off by 2^-24 of at most 127
    assert ((codes.double() - want).abs() <= 0.5 + 127 * 2.0 ** -22).all()
    assert ((scale.double() - want_scale).abs() <= 2.0 ** -24 * want_scale).all()
    assert (codes[0] == 0).all() and scale[0] == 0
    # the definition in binary32 steps, bit for bit
    f = x[:, :cols].float()
    a = f.abs().amax(dim=1, keepdim=True)
    again = torch.where(a < ref.TINY, torch.zeros_like(f), torch.round(f * (torch.full_like(a, 127.0) / a)))
    assert torch.equal(codes, again.to(torch.int8))


def test_quantize_rows_that_are_no_numbers(env):
    fs, ctx = env
    x = torch.randn(4, 300, generator=gen(1))
    x[0, 7], x[1, 299], x[2, 0] = math.nan, math.inf, 1e-31
    x[2, 1:] = 0.0
    x[3] *= 1e37
    codes, scale = (t.cpu() for t in fs.quantize_rows(ctx, x.to("cuda:0")))
    assert math.isnan(scale[0]) and math.isinf(scale[1])
    assert scale[2] == 0 and (codes[2] == 0).all()
    assert math.isfinite(scale[3]) and codes[3].abs().max() == 127


# ----------------------------------------------------------------- product --
def products(M, N, K, seed, lo=-127, hi=127):
    g = gen(seed)
    a = torch.randint(lo, hi + 1, (M, K), generator=g, dtype=torch.int8)
    w = torch.randint(lo, hi + 1, (N, K), generator=g, dtype=torch.int8)
    return a, torch.rand(M, generator=g) + 0.01, w, torch.rand(N, generator=g) * 1e-3, torch.randn(N, generator=g)


def in_steps(a, sa, w, sw, bias):
    """The product's definition: an exact sum, then binary32 steps."""
    total = (a.double() @ w.double().t())  # exact: below 2^53
    y = total.float() * sa[:, None] * sw[None]
    return y if bias is None else y + bias


SIZES = [(1, 1, 1), (1, 64, 64), (1, 7168, 512), (2, 33, 100), (7, 130, 257), (16, 256, 1024), (17, 100, 4097),
         (31, 1001, 1999), (33, 512, 384), (64, 320, 5120), (65, 65, 65), (100, 2048, 640), (127, 129, 1040),
         (128, 896, 256), (255, 257, 128), (256, 256, 2048), (300, 700, 272), (513, 511, 1024), (1024, 1024, 130),
         (777, 1100, 1333), (2048, 768, 512)]


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_scaled_matmul(env, M, N, K, out):
    fs, ctx = env
    note(f"matmul {M}x{N}x{K} {out}")
    a, sa, w, sw, bias = products(M, N, K, M + N + K)
    if M % 2:
        bias = None
    t = lambda x: None if x is None else x.to("cuda:0")  # noqa: E731
    got = fs.scaled_matmul(ctx, t(a), t(sa), t(w), t(sw), t(bias), out_dtype=TYPES[out]).cpu()
    want = in_steps(a, sa, w, sw, bias).to(TYPES[out])
    assert torch.equal(bits(got), bits(want))
    exact = ref.product(a, sa, w, sw, bias)
    room = exact.abs() + (bias.abs()[None] if bias is not None else 0)
    assert ((got.double() - exact).abs() <= (STEP[out] + 2.0 ** -22) * room + 2.0 ** -24).all()


@pytest.mark.parametrize("offset,a_pad,w_pad,out_pad", [(0, 16, 48, 8), (1, 3, 5, 1), (4, 4, 12, 2), (16, 0, 0, 3)])
@pytest.mark.parametrize("M,N,K", [(5, 70, 200), (40, 600, 1030), (130, 260, 520), (300, 300, 256)])
def test_scaled_matmul_strides(env, M, N, K, offset, a_pad, w_pad, out_pad):
    fs, ctx = env
    note(f"matmul strided {M}x{N}x{K} +{offset} {a_pad} {w_pad} {out_pad}")
    a, sa, w, sw, bias = products(M, N, K, M + offset)

    def strided(x, pad, fill, at=0):
        flat = torch.full((at + x.shape[0] * (x.shape[1] + pad),), fill, dtype=x.dtype, device="cuda:0")
        view = flat[at:].view(x.shape[0], x.shape[1] + pad)[:, :x.shape[1]]
        view.copy_(x)
        return flat, view
    _, da = strided(a, a_pad, 99, offset)
    _, dw = strided(w, w_pad, -99, offset)
    flat, out = strided(torch.zeros(M, N, dtype=torch.bfloat16), out_pad, 5.0)
    fs.scaled_matmul(ctx, da, sa.to("cuda:0"), dw, sw.to("cuda:0"), bias.to("cuda:0"), out=out)
    want = in_steps(a, sa, w, sw, bias).to(torch.bfloat16)
    assert torch.equal(bits(out.cpu()), bits(want))
    assert (flat.view(M, N + out_pad)[:, N:] == 5.0).all()  # nothing beyond the rows


@pytest.mark.parametrize("M", [1, 20, 70, 300])
def test_scaled_matmul_of_the_largest_codes(env, M):
    fs, ctx = env
    K = 131071
    a, w = torch.full((M, K), -128, dtype=torch.int8), torch.full((48, K), -128, dtype=torch.int8)
    one = lambda n: torch.ones(n, device="cuda:0")  # noqa: E731
    got = fs.scaled_matmul(ctx, a.to("cuda:0"), one(M), w.to("cuda:0"), one(48), out_dtype=torch.float32)
    assert (got.cpu().double() == float(torch.tensor(K * 16384.0))).all()


def test_scaled_matmul_without_inner_elements(env):
    fs, ctx = env
    e = lambda *s: torch.zeros(*s, dtype=torch.int8, device="cuda:0")  # noqa: E731
    f = lambda n: torch.ones(n, device="cuda:0")  # noqa: E731
    got = fs.scaled_matmul(ctx, e(3, 0), f(3), e(5, 0), f(5), bias=f(5) * 2, out_dtype=torch.float32)
    assert (got == 2).all()
    assert fs.scaled_matmul(ctx, e(0, 8), f(0), e(5, 8), f(5)).shape == (0, 5)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 96, 64), (1, 200, 5120), (2, 31, 999), (4, 100, 1024), (9, 65, 333),
                                   (64, 128, 1000), (200, 300, 640), (3, 40, 30011)])
def test_linear_is_the_two_calls(env, M, N, K, dtype):
    fs, ctx = env
    note(f"linear {M}x{N}x{K} {dtype}")
    x = (torch.randn(M, K + 3, generator=gen(K)) * 2).to(TYPES[dtype]).to("cuda:0")[:, :K]
    _, _, w, sw, bias = products(1, N, K, 5)
    w, sw, bias = (t.to("cuda:0") for t in (w, sw, bias))
    codes, scale = fs.quantize_rows(ctx, x)
    two = fs.scaled_matmul(ctx, codes, scale, w, sw, bias, out_dtype=TYPES[dtype])
    one = fs.linear(ctx, x, w, sw, bias)
    assert torch.equal(bits(one), bits(two))


def test_linear_with_rows_that_are_no_numbers(env):
    fs, ctx = env
    for M in (3, 70, 300):
        x = torch.randn(M, 200, generator=gen(M))
        x[1, 5], x[2, 199] = math.nan, math.inf
        x[0] = 0.0
        _, _, w, sw, _ = products(1, 50, 200, 5)
        y = fs.linear(ctx, x.to("cuda:0"), w.to("cuda:0"), sw.to("cuda:0")).cpu()
        assert (y[0] == 0).all() and not torch.isfinite(y[1:3]).any() and torch.isfinite(y[3:]).all()


# ------------------------------------------------------------------- cache --
def enter_in_steps(codes, scales, x, slots, page):
    """The append's definition in binary32 steps: codes [pages, H, page, D]."""
    done = 0
    T = len(slots)
    while done < T:
        if slots[done] < 0:
            done += 1
            continue
        at, first, n = slots[done] // page, slots[done] % page, 1
        while done + n < T and slots[done + n] == slots[done] + n and slots[done + n] // page == at:
            n += 1
        new = x[done:done + n]  # [n, H, D]
        a = new.abs().amax(dim=(0, 2))
        made = torch.where(a < ref.TINY, torch.zeros_like(a), a / torch.full_like(a, 127.0))
        old = scales[at] if first else torch.zeros_like(made)
        now = torch.maximum(old, made)
        inverse = torch.where(now > 0, torch.ones_like(now) / now, torch.zeros_like(now))
        ratio = torch.where(now > 0, old / now, torch.zeros_like(now))
        grew = now != old
        for h in range(codes.shape[1]):
            if first and grew[h]:
                codes[at, h, :first] = torch.round(codes[at, h, :first].float() * ratio[h]).to(torch.int8)
            codes[at, h, first:first + n] = torch.round(new[:, h] * inverse[h]).clamp(-127, 127).to(torch.int8)
        scales[at] = now
        done += n


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("D,page,R,heads,group", [(128, 64, 128, 2, 5), (64, 16, 32, 3, 1), (128, 16, 128, 1, 8),
                                                  (64, 64, 0, 5, 3), (128, 32, 6, 2, 2), (64, 32, 64, 1, 1)])
@pytest.mark.parametrize("steps", [[(1, 1, 1)], [(70, 1, 0), (3, 16, 65)], [(5, 200, 31), (1, 1, 1), (1, 64, 1)]])
def test_append(env, dtype, D, page, R, heads, group, steps):
    """Several steps into one cache: the codes held are those of the
    definition bit for bit, and their values near the 64-bit ones."""
    fs, ctx = env
    note(f"append {dtype} D{D} page{page} R{R} {heads}x{group} {steps}")
    S = 3
    totals = [sum(st[s] for st in steps) for s in range(S)]
    c = ref.Paged(totals, heads, D, page, seed=page + D, spare=2)
    kv = c.device(fs)
    k, ks, v, vs = c.k.clone(), c.k_scale.clone(), c.v.transpose(2, 3).contiguous(), c.v_scale.clone()
    g = gen(D + page)
    reach = max(totals) + 3
    angle = torch.rand(reach, max(1, R // 2), generator=g) * 6
    cos, sin = (angle.cos(), angle.sin()) if R else (None, None)
    held = [0] * S
    true = [([], []) for _ in range(S)]
    left_out = set()
    for number, st in enumerate(steps):
        T = sum(st)
        rows = torch.randn(T, heads * (group + 2), D, generator=g) * (1.0 + number)
        rows = rows.to(TYPES[dtype])
        q, kn, vn = rows[:, :heads * group], rows[:, heads * group:heads * (group + 1)], rows[:, heads * (group + 1):]
        slots, positions = [], []
        for s in range(S):
            slots += c.slots(s, held[s], held[s] + st[s])
            positions += range(held[s], held[s] + st[s])
            held[s] += st[s]
        if T > 4:
            slots[T - 1] = -1  # the last token is left out
            left_out.add((max(s for s in range(S) if st[s]), positions[T - 1]))
        pos = torch.tensor(positions, dtype=torch.int32)
        dev = rows.to("cuda:0")
        dq, dk, dv = dev[:, :heads * group], dev[:, heads * group:heads * (group + 1)], dev[:, heads * (group + 1):]
        on = lambda t: None if t is None else t.to("cuda:0")  # noqa: E731
        out = fs.cache_append(ctx, kv, dk, dv, torch.tensor(slots, dtype=torch.int32, device="cuda:0"), q=dq,
                              positions=on(pos), cos=on(cos), sin=on(sin))
        h = R // 2

        def turned(x):
            x = x.float().clone()
            if R:
                co, si = cos[pos.long()][:, None], sin[pos.long()][:, None]
                a, b = x[..., :h].clone(), x[..., h:R].clone()
                x[..., :h], x[..., h:R] = a * co - b * si, b * co + a * si
            return x
        assert torch.equal(bits(out), bits(turned(q).to(TYPES[dtype])))
        exact = ref.rotate(q, cos, sin, pos)
        # two products and a sum in binary32, each within 2^-24 of at most |a| + |b|
        assert ((out.cpu().double() - exact).abs() <= STEP[dtype] * exact.abs() + 2.0 ** -21 * q.double().abs().amax()).all()
        enter_in_steps(k, ks, turned(kn), slots, page)
        enter_in_steps(v, vs, vn.float(), slots, page)
        at = 0
        for s in range(S):
            true[s][0].append(ref.rotate(kn, cos, sin, pos)[at:at + st[s]])
            true[s][1].append(vn[at:at + st[s]].double())
            at += st[s]
    torch.cuda.synchronize()
    for s in range(S):
        n = totals[s]
        if n == 0:
            continue
        sl = torch.tensor(c.slots(s, 0, n), dtype=torch.int32, device="cuda:0")
        kk, vv = (t.cpu() for t in fs.cache_read(ctx, kv, sl))
        at, place = sl.cpu().long() // page, sl.cpu().long() % page
        assert torch.equal(kk, k[at, :, place].float() * ks[at][:, :, None])
        assert torch.equal(vv, v[at, :, place].float() * vs[at][:, :, None])
        for got, want, scale in ((kk, true[s][0], ks), (vv, true[s][1], vs)):
            want = torch.cat(want)
            # half a step at the append and at each growth of the page's scale
            room = 0.5 * (1 + 2 * len(steps)) * scale[at].double()[:, :, None] * 1.001
            there = torch.tensor([(s, p) not in left_out for p in range(n)])
            assert ((got.double() - want).abs() <= room)[there].all()
    used = torch.isfinite(c.k_scale).all(dim=1)
    assert torch.equal(kv.k_scale.cpu()[used], ks[used]) and torch.equal(kv.v_scale.cpu()[used], vs[used])
    assert torch.equal(kv.k.cpu(), k)
    got_v = kv.v.cpu().transpose(2, 3)
    assert torch.equal(got_v, v)


def test_append_of_a_long_batch(env):
    """More tokens than blocks take one by one, in pages of several lengths."""
    fs, ctx = env
    note("append long")
    heads, D, page = 2, 64, 32
    lengths = [1500, 33, 1001, 64, 7]
    c = ref.Paged(lengths, heads, D, page, seed=8)
    kv = c.device(fs)
    T = sum(lengths)
    g = gen(4)
    kn, vn = torch.randn(T, heads, D, generator=g), torch.randn(T, heads, D, generator=g)
    slots = [x for s, n in enumerate(lengths) for x in c.slots(s, 0, n)]
    fs.cache_append(ctx, kv, kn.to("cuda:0"), vn.to("cuda:0"), torch.tensor(slots, dtype=torch.int32, device="cuda:0"))
    k, ks, v, vs = c.k.clone(), c.k_scale.clone(), c.v.transpose(2, 3).contiguous(), c.v_scale.clone()
    enter_in_steps(k, ks, kn, slots, page)
    enter_in_steps(v, vs, vn, slots, page)
    assert torch.equal(kv.k.cpu(), k) and torch.equal(kv.v.cpu().transpose(2, 3), v)


def test_append_of_values_that_are_no_numbers(env):
    """A NaN makes its page and head's scale NaN, and no other's; a fresh use of the page clears it."""
    fs, ctx = env
    kv = fs.KVCache.empty(4, 2, 64, 16, "cuda:0")
    x = torch.ones(20, 2, 64, device="cuda:0")
    x[18, 1, 3] = math.nan
    slots = torch.arange(20, dtype=torch.int32, device="cuda:0")
    fs.cache_append(ctx, kv, x, torch.ones_like(x), slots)
    nan = torch.isnan(kv.k_scale).cpu()
    assert nan.sum() == 1 and nan[1, 1] and not torch.isnan(kv.v_scale).any()
    fs.cache_append(ctx, kv, torch.ones_like(x), torch.zeros_like(x), slots)
    assert not torch.isnan(kv.k_scale).any() and (kv.v_scale[:2] == 0).all()
    k, v = fs.cache_read(ctx, kv, slots, dtype=torch.float16)
    assert ((k - 1).abs() < 1e-3).all() and (v == 0).all()


def test_slots_out_of_range_are_left_out_or_refused(env, monkeypatch):
    fs, ctx = env
    kv = fs.KVCache.empty(2, 1, 64, 16, "cuda:0")
    x = torch.ones(3, 1, 64, device="cuda:0")
    bad = torch.tensor([5, 32, 1 << 30], dtype=torch.int32, device="cuda:0")
    fs.cache_append(ctx, kv, x, x, bad)
    k, _ = fs.cache_read(ctx, kv, bad)
    assert (k[0] == 1).all() and (k[1:] == 0).all()
    monkeypatch.setenv("FS_VALIDATE", "1")
    for call in (lambda: fs.cache_append(ctx, kv, x, x, bad), lambda: fs.cache_read(ctx, kv, bad)):
        with pytest.raises(fs.FleetSieveError) as e:
            call()
        assert e.value.status == fs.FS_ERR_INVALID_ARGUMENT
    order = torch.tensor([3, 5, 6], dtype=torch.int32, device="cuda:0")
    with pytest.raises(fs.FleetSieveError):
        fs.cache_append(ctx, kv, x, x, order)
    far = torch.tensor([0, 1, 9], dtype=torch.int32, device="cuda:0")
    table = torch.ones(9, 32, device="cuda:0")
    with pytest.raises(fs.FleetSieveError):
        fs.cache_append(ctx, kv, x, x, far.clone().fill_(0) + torch.arange(3, device="cuda:0", dtype=torch.int32),
                        positions=far, cos=table, sin=table)


# --------------------------------------------------------------- attention --
def attention_case(env, lengths, news, heads, group, D, page, window, dtype, seed=0, spread=1.0, q_std=1.2, scale=None,
                   cache=None):
    fs, ctx = env
    note(f"attention {lengths} {news} {heads}x{group} D{D} page{page} window{window} {dtype}")
    c = cache or ref.Paged(lengths, heads, D, page, seed=seed + D + page, spread=spread)
    T = sum(news)
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    wide = (torch.randn(T, heads * (group + 1), D, generator=gen(seed + T)) * q_std).to(TYPES[dtype])
    q = wide[:, :heads * group]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    scale = scale if scale is not None else D ** -0.5
    got = fs.cache_attention(ctx, c.device(fs), wide.to("cuda:0")[:, :heads * group], c.table.to("cuda:0"),
                             i32(lengths), i32(starts), max(news), scale=scale, window=window).cpu()
    for s, n in enumerate(news):
        k, v = c.values(s)
        part = q[starts[s]:starts[s] + n]
        first = lengths[s] - n
        want = ref.attend(part, k, v, first, scale, window)
        bound = ref.attention_bound(part, k, v, first, scale, window, want, STEP[dtype])
        off = (got[starts[s]:starts[s] + n].double() - want).abs()
        assert (off <= bound).all(), (s, float((off / bound).max()))
    return c, got


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,page,heads,group", [(128, 64, 2, 5), (128, 16, 1, 1), (64, 32, 3, 4), (64, 64, 1, 16),
                                                (128, 32, 2, 17), (64, 16, 2, 8)])
def test_decode_attention(env, dtype, D, page, heads, group):
    lengths = [1, 2, 15, 16, 17, 63, 64, 65, 128, 129, 300, 0, 257]
    attention_case(env, lengths, [1] * len(lengths), heads, group, D, page, 0, dtype)


@pytest.mark.parametrize("window", [0, 1, 5, 64, 100])
@pytest.mark.parametrize("D,page,heads,group,dtype", [(128, 64, 2, 5, "bf16"), (64, 16, 1, 1, "f16"), (64, 32, 2, 3, "bf16"),
                                                      (128, 16, 1, 2, "f16")])
def test_chunk_attention(env, window, D, page, heads, group, dtype):
    lengths, news = [70, 33, 200, 1, 130, 0, 90], [70, 1, 37, 1, 16, 2, 90]
    attention_case(env, lengths, news, heads, group, D, page, window, dtype)


@pytest.mark.parametrize("window", [0, 300])
def test_attention_over_a_split_context(env, window):
    attention_case(env, [5000, 1, 3000], [1, 1, 3], 1, 5, 128, 64, window, "bf16")
    attention_case(env, [9000], [1], 2, 1, 64, 16, window, "f16")


def test_long_chunk_attention(env):
    attention_case(env, [700, 513], [600, 257], 1, 2, 64, 64, 0, "bf16")
    attention_case(env, [390], [300], 1, 1, 128, 32, 0, "f16")
    attention_case(env, [2200, 40], [130, 1], 1, 4, 64, 32, 700, "f16")


def test_attention_of_one_large_logit(env):
    """One token far above many: the rest keep their weight."""
    lengths = [4000]
    c = ref.Paged(lengths, 1, 64, 64, seed=3, spread=0.0)
    c.k[:] = 0
    first = int(c.table[0, 0])
    c.k[first, 0, 0, 0] = 127
    q = torch.zeros(1, 1, 64, dtype=torch.bfloat16)
    q[0, 0, 0] = 26.5
    fs, ctx = env
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    got = fs.cache_attention(ctx, c.device(fs), q.to("cuda:0"), c.table.to("cuda:0"), i32(lengths), i32([0, 1]), 1).cpu()
    k, v = c.values(0)
    want = ref.attend(q, k, v, 3999, 0.125)
    bound = ref.attention_bound(q, k, v, 3999, 0.125, 0, want, STEP["bf16"])
    assert ((got.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("new", [1, 150])
def test_attention_over_pages_of_zeros_and_of_very_different_scales(env, new):
    for scales in ([0.0, 1.0], [1e-3, 1e3], [1e-30, 1.0], [0.0, 0.0]):
        c = ref.Paged([200], 1, 64, 16, seed=2)
        for i in range(13):
            c.v_scale[int(c.table[0, i])] = scales[i % 2]
        attention_case(env, [200], [new], 1, 2, 64, 16, 0, "bf16", cache=c)


@pytest.mark.parametrize("new", [1, 40, 200])
def test_attention_with_queries_that_are_no_numbers_or_zero(env, new):
    fs, ctx = env
    lengths = [300]
    c = ref.Paged(lengths, 1, 64, 64, seed=3)
    q = torch.randn(new, 2, 64, generator=gen(new)).to(torch.bfloat16)
    q[0, 0, 5] = math.nan
    q[0, 1] = 0.0
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    got = fs.cache_attention(ctx, c.device(fs), q.to("cuda:0"), c.table.to("cuda:0"), i32(lengths), i32([0, new]),
                             new).cpu()
    assert torch.isnan(got[0, 0]).all() and torch.isfinite(got[0, 1]).all() and torch.isfinite(got[1:]).all()
    k, v = c.values(0)
    mean = v[:300 - new + 1, 0].mean(dim=0)
    assert ((got[0, 1].double() - mean).abs() <= 2.0 ** -8 * mean.abs() + 2.0 ** -10 * v.abs().amax()).all()


@pytest.mark.parametrize("new", [1, 100])
def test_attention_reads_no_page_outside_the_window(env, new):
    """Table entries that no query sees may be anything, and what lies in
    their pages too."""
    c = ref.Paged([400], 1, 64, 16, seed=6)
    want_c, _ = attention_case(env, [400], [new], 1, 2, 64, 16, 60, "f16", cache=c)
    for i in range((400 - new - 59) // 16):
        c.table[0, i] = -1 if i % 2 else 1 << 30
    with pytest.MonkeyPatch.context() as m:
        m.setattr(c, "values", ref.Paged([400], 1, 64, 16, seed=6).values)
        attention_case(env, [400], [new], 1, 2, 64, 16, 60, "f16", cache=c)


def test_attention_of_many_sequences(env):
    r = random.Random(3)
    lengths = [r.choice([0, 1, 5, 40, 70]) for _ in range(700)]
    attention_case(env, lengths, [1] * 700, 1, 1, 64, 16, 0, "f16")


def test_attention_with_places_of_no_tokens(env):
    attention_case(env, [100, 50, 0, 30], [0, 3, 0, 0], 2, 2, 64, 16, 0, "bf16")


def test_attention_far_into_a_large_cache(env):
    """Offsets beyond 2^31 bytes: pages at the end of a cache of 2.6 GB."""
    fs, ctx = env
    note("attention far")
    n_pages, heads, D, page = 160_000, 1, 128, 128 // 2
    kv = fs.KVCache.empty(n_pages * 2, heads, D, page, "cuda:0")
    last = n_pages * 2 - 2
    x = torch.randn(70, heads, D, generator=gen(9))
    y = torch.randn(70, heads, D, generator=gen(10))
    slots = torch.arange(last * page, last * page + 70, dtype=torch.int32, device="cuda:0")
    fs.cache_append(ctx, kv, x.to("cuda:0"), y.to("cuda:0"), slots)
    k, v = (t.cpu() for t in fs.cache_read(ctx, kv, slots))
    q = torch.randn(70, 2, D, generator=gen(11)).to(torch.bfloat16)
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda:0")  # noqa: E731
    for n in (1, 70):
        got = fs.cache_attention(ctx, kv, q[:n].to("cuda:0"), i32([[last, last + 1]]), i32([70]), i32([0, n]), n).cpu()
        want = ref.attend(q[:n], k, v, 70 - n, D ** -0.5)
        bound = ref.attention_bound(q[:n], k, v, 70 - n, D ** -0.5, 0, want, STEP["bf16"])
        assert ((got.double() - want).abs() <= bound).all()


def test_attention_is_the_same_on_every_run(env):
    fs, ctx = env
    c = ref.Paged([3000, 900], 2, 128, 64, seed=1)
    kv = c.device(fs)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    for n in (1, 300):
        q = torch.randn(2 * n, 10, 128, generator=gen(n)).to(torch.bfloat16).to("cuda:0")
        plan = fs.AttentionPlan(ctx, kv, q, c.table.to("cuda:0"), i32([3000, 900]), i32([0, n, 2 * n]), n)
        one = plan.run().clone()
        for _ in range(5):
            assert torch.equal(bits(plan.run()), bits(one))


def test_calls_on_another_stream_and_in_a_graph(env):
    """The operators enqueue on the stream they are given, and a graph that
    records them replays with new contents."""
    fs, ctx = env
    note("graph")
    c = ref.Paged([700], 1, 64, 64, seed=1)
    kv = c.device(fs)
    x = torch.randn(5, 256, device="cuda:0").to(torch.bfloat16)
    w = torch.randint(-127, 128, (96, 256), dtype=torch.int8, device="cuda:0")
    sw = torch.rand(96, device="cuda:0")
    q = torch.randn(1, 4, 64, device="cuda:0").to(torch.bfloat16)
    kn = torch.randn(1, 1, 64, device="cuda:0").to(torch.bfloat16)
    slot = torch.tensor(c.slots(0, 699, 700), dtype=torch.int32, device="cuda:0")
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda:0")  # noqa: E731
    table, lens, cu = c.table.to("cuda:0"), i32([700]), i32([0, 1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = lambda: torch.empty(64 << 20, dtype=torch.uint8, device="cuda:0")  # noqa: E731
    plans = [fs.LinearPlan(ctx, x, w, sw, stream=side, workspace=ws()), fs.AppendPlan(ctx, kv, kn, kn, slot, stream=side),
             fs.AttentionPlan(ctx, kv, q, table, lens, cu, 1, stream=side, workspace=ws())]
    for p in plans:
        p.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for p in plans:
            p.run()
    for i in range(4):
        x.copy_(torch.randn(5, 256, generator=gen(i)).to(torch.bfloat16))
        q.copy_(torch.randn(1, 4, 64, generator=gen(i)).to(torch.bfloat16))
        kn.copy_(torch.randn(1, 1, 64, generator=gen(i + 50)).to(torch.bfloat16))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [plans[0].out.clone(), plans[2].out.clone()]
        assert torch.equal(bits(fs.linear(ctx, x, w, sw)), bits(got[0]))
        assert torch.equal(bits(fs.cache_attention(ctx, kv, q, table, lens, cu, 1)), bits(got[1]))


def test_lengths_and_pages_out_of_range_are_refused(env, monkeypatch):
    fs, ctx = env
    c = ref.Paged([70, 20], 1, 64, 16, seed=1)
    kv = c.device(fs)
    q = torch.randn(2, 1, 64, device="cuda:0").to(torch.float16)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    good = (c.table.to("cuda:0"), i32([70, 20]), i32([0, 1, 2]))
    holes = c.table.clone()
    holes[1, 0] = c.n_pages
    monkeypatch.setenv("FS_VALIDATE", "1")
    fs.cache_attention(ctx, kv, q, *good, 1)
    for bad in ((good[0], i32([7000, 20]), good[2]), (good[0], i32([-1, 20]), good[2]), (good[0], good[1], i32([0, 2, 1])),
                (holes.to("cuda:0"), good[1], good[2]), (good[0], good[1], i32([0, 0, 2]))):
        with pytest.raises(fs.FleetSieveError) as e:
            fs.cache_attention(ctx, kv, q, *bad, 1)
        assert e.value.status == fs.FS_ERR_INVALID_ARGUMENT


# ---------------------------------------------------------------- refusals --
def test_arguments_that_are_refused(env):
    fs, ctx = env
    dev = "cuda:0"
    i8 = lambda *s: torch.zeros(*s, dtype=torch.int8, device=dev)  # noqa: E731
    f = lambda *s: torch.zeros(*s, device=dev)  # noqa: E731
    h = lambda *s: torch.zeros(*s, device=dev, dtype=torch.float16)  # noqa: E731
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    kv = fs.KVCache.empty(4, 2, 64, 16, dev)
    cases = [
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.quantize_rows(ctx, torch.zeros(2, 3))),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.quantize_rows(ctx, f(2, 3).double())),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.quantize_rows(ctx, f(3, 2).t())),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.scaled_matmul(ctx, i8(2, 8), f(2), i8(3, 9), f(3))),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.scaled_matmul(ctx, i8(2, 8), f(3), i8(3, 8), f(3))),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.scaled_matmul(ctx, i8(2, 8), f(2), i8(3, 8), f(3), bias=f(2))),
        (fs.FS_ERR_UNSUPPORTED, lambda: fs.scaled_matmul(ctx, i8(1, 131072), f(1), i8(1, 131072), f(1))),
        (fs.FS_ERR_WORKSPACE_TOO_SMALL, lambda: fs.linear(ctx, h(2, 64), i8(3, 64), f(3), workspace=i8(8).view(torch.uint8))),
        (fs.FS_ERR_UNSUPPORTED, lambda: fs.cache_read(ctx, fs.KVCache.empty(4, 2, 80, 16, dev), i32([0]))),
        (fs.FS_ERR_UNSUPPORTED, lambda: fs.cache_read(ctx, fs.KVCache.empty(4, 2, 64, 8, dev), i32([0]))),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.cache_read(ctx, kv, i32([0]).long())),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.cache_append(ctx, kv, h(1, 2, 64), f(1, 2, 64), i32([0]))),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.cache_append(ctx, kv, h(1, 2, 64), h(1, 2, 64), i32([0]), cos=f(1, 32))),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.cache_append(ctx, kv, h(1, 2, 64), h(1, 2, 64), i32([0]), positions=i32([0]),
                                                             cos=f(1, 33), sin=f(1, 33))),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.cache_append(ctx, kv, h(1, 1, 64), h(1, 1, 64), i32([0]))),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.cache_attention(ctx, kv, h(1, 3, 64), i32([[0]]), i32([1]), i32([0, 1]), 1)),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.cache_attention(ctx, kv, h(1, 2, 64), i32([[0]]), i32([1]), i32([0]), 1)),
        (fs.FS_ERR_UNSUPPORTED, lambda: fs.cache_attention(ctx, kv, f(1, 2, 64), i32([[0]]), i32([1]), i32([0, 1]), 1)),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.cache_attention(ctx, kv, h(1, 2, 64), i32([[0]]), i32([1]), i32([0, 1]), 1,
                                                                window=-1)),
        (fs.FS_ERR_INVALID_ARGUMENT, lambda: fs.cache_attention(ctx, kv, h(1, 2, 64), i32([[0]]), i32([1]), i32([0, 1]), 1,
                                                                scale=math.inf)),
        (fs.FS_ERR_UNSUPPORTED, lambda: fs.cache_attention(ctx, kv, h(1, 2, 64), i32([[0]] * 4097), i32([1] * 4097),
                                                           i32([0] * 4097 + [1]), 1)),
    ]
    for i, (status, call) in enumerate(cases):
        with pytest.raises(fs.FleetSieveError) as e:
            call()
        assert e.value.status == status, (i, str(e.value))


def test_nothing_to_do_is_no_error(env):
    fs, ctx = env
    kv = fs.KVCache.empty(2, 1, 64, 16, "cuda:0")
    e = lambda *s: torch.zeros(*s, device="cuda:0", dtype=torch.float16)  # noqa: E731
    none = torch.zeros(0, dtype=torch.int32, device="cuda:0")
    fs.cache_append(ctx, kv, e(0, 1, 64), e(0, 1, 64), none)
    fs.cache_read(ctx, kv, none)
    cu = torch.zeros(2, dtype=torch.int32, device="cuda:0")
    fs.cache_attention(ctx, kv, e(0, 1, 64), cu[None], cu[:1], cu, 0)
    codes, scale = fs.quantize_rows(ctx, e(0, 5))
    assert codes.shape == (0, 5) and scale.shape == (0,)


# ------------------------------------- attention of many rows over long tables --
def wide(lengths, heads, D, page, seed, spread=1.0):
    """A cache whose block table has room for far longer contexts: the host
    then expects work enough for the kernel of many rows."""
    c = ref.Paged(lengths, heads, D, page, seed=seed, spread=spread)
    table = torch.full((len(lengths), 16384), -7, dtype=torch.int32)
    table[:, :c.table.shape[1]] = c.table
    c.table = table
    return c


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("window", [0, 1, 40, 300])
@pytest.mark.parametrize("D,page,heads,group", [(128, 64, 2, 5), (64, 16, 1, 1), (64, 32, 3, 4), (128, 16, 1, 8),
                                                (128, 32, 1, 17), (64, 64, 2, 2)])
def test_many_rows(env, D, page, heads, group, window, dtype):
    lengths, news = [200, 33, 530, 1, 130, 0, 90, 64, 65], [200, 1, 137, 1, 16, 2, 90, 64, 63]
    attention_case(env, lengths, news, heads, group, D, page, window, dtype,
                   cache=wide(lengths, heads, D, page, seed=window + D + page))


@pytest.mark.parametrize("lengths,news,heads,group", [([1500], [1100], 1, 1), ([3000, 2900], [150, 700], 1, 2),
                                                      ([4000], [130], 2, 1), ([260] * 12, [256] * 12, 2, 1),
                                                      ([600, 100, 90], [500, 1, 90], 1, 3)])
def test_many_rows_cut_over_blocks(env, lengths, news, heads, group):
    attention_case(env, lengths, news, heads, group, 64, 64, 0, "bf16", cache=wide(lengths, heads, 64, 64, seed=7))
    attention_case(env, lengths, news, heads, group, 128, 16, 0, "f16", cache=wide(lengths, heads, 128, 16, seed=8))


def test_many_rows_of_a_sequence_with_more_tokens_than_its_cache(env):
    lengths, news = [100, 300], [250, 200]
    attention_case(env, lengths, news, 1, 2, 64, 32, 0, "f16", cache=wide(lengths, 1, 64, 32, seed=4))


def test_many_rows_with_one_large_logit(env):
    fs, ctx = env
    lengths, new = [4000], 160
    c = wide(lengths, 1, 64, 64, seed=3, spread=0.0)
    c.k[:] = 0
    c.k[int(c.table[0, 0]), 0, 0, 0] = 127
    q = torch.zeros(new, 1, 64, dtype=torch.bfloat16)
    q[:, 0, 0] = torch.linspace(-20.0, 26.5, new)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    got = fs.cache_attention(ctx, c.device(fs), q.to("cuda:0"), c.table.to("cuda:0"), i32(lengths), i32([0, new]), new).cpu()
    k, v = c.values(0)
    want = ref.attend(q, k, v, 4000 - new, 0.125)
    bound = ref.attention_bound(q, k, v, 4000 - new, 0.125, 0, want, STEP["bf16"])
    assert ((got.double() - want).abs() <= bound).all()


def test_many_rows_over_pages_of_zeros_and_of_very_different_scales(env):
    for scales in ([0.0, 1.0], [1e-3, 1e3], [1e-30, 1.0], [0.0, 0.0]):
        c = wide([200], 1, 64, 16, seed=2)
        for i in range(13):
            c.v_scale[int(c.table[0, i])] = scales[i % 2]
        attention_case(env, [200], [150], 1, 2, 64, 16, 0, "bf16", cache=c)


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_attention_scales(env, scale):
    c = wide([300, 200], 1, 64, 64, seed=12)
    attention_case(env, [300, 200], [150, 1], 1, 2, 64, 64, 0, "bf16", scale=scale, q_std=0.3, cache=c)


def test_many_rows_with_queries_that_are_no_numbers_or_zero(env):
    fs, ctx = env
    new = 200
    c = wide([300], 1, 64, 64, seed=3)
    q = torch.randn(new, 2, 64, generator=gen(new)).to(torch.bfloat16)
    q[0, 0, 5], q[7, 1, 0] = math.nan, math.inf
    q[0, 1] = 0.0
    q[9] *= 1e30
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    got = fs.cache_attention(ctx, c.device(fs), q.to("cuda:0"), c.table.to("cuda:0"), i32([300]), i32([0, new]), new,
                             ).cpu()
    none = torch.zeros(new, 2, dtype=torch.bool)
    none[0, 0] = none[7, 1] = True
    assert torch.isnan(got[none]).all() and torch.isfinite(got[~none]).all()
    k, v = c.values(0)
    mean = v[:101, 0].mean(dim=0)
    assert ((got[0, 1].double() - mean).abs() <= 2.0 ** -8 * mean.abs() + 2.0 ** -10 * v.abs().amax()).all()


def test_a_page_that_is_no_number_reaches_only_rows_that_see_it(env):
    """A NaN scale: later rows are NaN, rows before the page are not."""
    fs, ctx = env
    for c, new in ((wide([300], 1, 64, 16, seed=5), 200), (ref.Paged([300], 1, 64, 16, seed=5), 40)):
        at = 280  # a page of tokens 272 .. 287
        c.v_scale[int(c.table[0, at // 16])] = math.nan
        q = torch.randn(new, 1, 64, generator=gen(2)).to(torch.bfloat16)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
        got = fs.cache_attention(ctx, c.device(fs), q.to("cuda:0"), c.table.to("cuda:0"), i32([300]), i32([0, new]),
                                 new).cpu()
        sees = torch.arange(300 - new, 300) >= 272
        assert torch.isnan(got[sees]).all() and torch.isfinite(got[~sees]).all()


def test_workspaces_of_any_contents(env):
    """The counters of arrived parts take no contents of the workspace for a count."""
    fs, ctx = env
    c = ref.Paged([3000, 900], 1, 128, 64, seed=1)
    kv = c.device(fs)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    q = torch.randn(2, 5, 128, generator=gen(1)).to(torch.bfloat16).to("cuda:0")
    results = []
    for fill in (0, 255, 1):
        ws = torch.full((256 << 20,), fill, dtype=torch.uint8, device="cuda:0")
        plan = fs.AttentionPlan(ctx, kv, q, c.table.to("cuda:0"), i32([3000, 900]), i32([0, 1, 2]), 1, workspace=ws)
        results += [plan.run().clone(), plan.run().clone()]
    assert all(torch.equal(bits(r), bits(results[0])) for r in results)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("N,K", [(100, 16), (16, 512), (33, 528), (4096, 64), (4097, 1040), (5120, 640), (8193, 1536),
                                 (8200, 48), (30, 5120), (4200, 6160), (6, 20480)])
def test_linear_of_few_rows(env, M, N, K, dtype):
    """Rows that start on multiples of 16 bytes, whose codes may be made where
    they are used: the bits are those of the two calls."""
    fs, ctx = env
    note(f"few {M}x{N}x{K} {dtype}")
    x = (torch.randn(M, K + 16, generator=gen(K)) * 2).to(TYPES[dtype])[:, :K]
    if M > 2:
        x[1] = 0.0
        x[2, K - 1], x[2, 0] = 1e4, -1e-3
    x = x.to("cuda:0")
    _, _, w, sw, bias = products(1, N, K, 5)
    wide = torch.full((N, K + 32), 77, dtype=torch.int8)
    wide[:, :K] = w
    w, sw, bias = wide.to("cuda:0")[:, :K], sw.to("cuda:0"), bias.to("cuda:0")
    codes, scale = fs.quantize_rows(ctx, x)
    for b in (bias, None):
        two = fs.scaled_matmul(ctx, codes, scale, w, sw, b, out_dtype=TYPES[dtype])
        out = torch.full((M, N + 5), 9.0, dtype=TYPES[dtype], device="cuda:0")
        one = fs.linear(ctx, x, w, sw, b, out=out[:, :N])
        assert torch.equal(bits(one.contiguous()), bits(two))
        assert (out[:, N:] == 9.0).all()


def test_linear_of_few_rows_that_are_no_numbers(env):
    fs, ctx = env
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn(4, 256, generator=gen(4)).to(dtype)
        x[1, 5], x[2, 199] = math.nan, -math.inf
        x[0] = 0.0
        _, _, w, sw, _ = products(1, 50, 256, 5)
        y = fs.linear(ctx, x.to("cuda:0"), w.to("cuda:0"), sw.to("cuda:0")).cpu()
        assert (y[0] == 0).all() and not torch.isfinite(y[1:3]).any() and torch.isfinite(y[3:]).all()


@pytest.mark.parametrize("K", [1, 15, 16, 17, 129, 511, 513, 1030, 1999])
@pytest.mark.parametrize("M,N", [(5, 41), (20, 1001), (40, 3001), (70, 2003), (130, 1999), (300, 2500), (1000, 1001), (2500, 3001)])
def test_linear_with_weights_at_any_alignment(env, M, N, K):
    fs, ctx = env
    note(f"linear, weights at any alignment, {M}x{N}x{K}")
    x = (torch.randn(M, K, generator=gen(M + K)) * 2).bfloat16().to("cuda:0")
    g = torch.Generator(device="cuda:0").manual_seed(N)
    # a part of wider rows, from an odd place on
    w = torch.randint(-127, 128, (N, K + 2), generator=g, dtype=torch.int8, device="cuda:0")[:, 1:K + 1]
    sw, bias = torch.rand(N, generator=g, device="cuda:0") * 1e-3, torch.randn(N, generator=g, device="cuda:0")
    # codes beside the rows' own must not count
    ws = torch.randint(-128, 128, (1 << 23,), generator=g, dtype=torch.int8, device="cuda:0").view(torch.uint8)
    codes, scale = fs.quantize_rows(ctx, x)
    one = fs.linear(ctx, x, w, sw, bias, out_dtype=torch.float32, workspace=ws)
    total = torch.round(codes.double() @ w.double().t().contiguous())  # exact: below 2^53
    want = total.float() * scale[:, None] * sw[None] + bias
    assert torch.equal(one, want)


@pytest.mark.parametrize("heads,group", [(1, 5), (3, 1), (8, 4), (1, 17)])
@pytest.mark.parametrize("lengths", [[1000], [4000, 1, 700, 64], [2100, 0, 65, 2049, 1024, 3],
                                     [300 + 211 * (i % 7) for i in range(24)], [(37 * i) % 1400 for i in range(60)]])
def test_decode_attention_cut_between_items(env, lengths, heads, group):
    attention_case(env, lengths, [1] * len(lengths), heads, group, 128 if heads < 8 else 64, 64 if group > 1 else 16, 0, "bf16")


@pytest.mark.parametrize("lengths,news,heads,group", [([3900] + [40 + 61 * i for i in range(40)], [79] + [1] * 40, 8, 3),
                                                      ([2300, 70, 0, 900], [300, 1, 1, 1], 4, 2)])
def test_one_prompt_beside_users(env, lengths, news, heads, group):
    attention_case(env, lengths, news, heads, group, 64, 32, 0, "f16")


@pytest.mark.parametrize("new,length", [(1100, 9000), (1537, 4100)])
def test_many_rows_in_many_parts(env, new, length):
    attention_case(env, [length], [new], 1, 5, 64, 64, 0, "bf16")


@pytest.mark.parametrize("lengths,news,heads,group,window", [([300, 290, 280], [300, 290, 280], 8, 4, 0),
                                                             ([700, 650], [600, 580], 8, 3, 100),
                                                             ([816, 900, 1, 0], [700, 690, 1, 1], 4, 4, 60),
                                                             ([1200, 1100], [500, 31], 4, 8, 0)])
def test_many_rows_over_short_contexts(env, lengths, news, heads, group, window):
    attention_case(env, lengths, news, heads, group, 64, 64, window, "bf16")
