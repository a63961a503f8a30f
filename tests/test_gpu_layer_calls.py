"""Projections and state attention as calls: every tensor is checked, memory that
another stream works on is left alone, contexts and plans side by side."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_serving import bits, env, gen, note  # noqa: E402, F401


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


def plans(fs, ctx, **kw):
    """Each call as a plan, with the tensors that it is given."""
    h = lambda *s: torch.randn(*s, device="cuda:0").to(torch.bfloat16)  # noqa: E731
    x, w, sw = h(9, 64), torch.ones(6, 64, dtype=torch.int8, device="cuda:0"), torch.ones(6, device="cuda:0")
    bias, gain, res, out = torch.ones(6, device="cuda:0"), torch.ones(64, device="cuda:0"), h(9, 6), h(9, 6)
    a = dict(states=torch.zeros(3, 1, 64, 64, device="cuda:0"), q=h(30, 2, 64), k=h(30, 1, 64), v=h(30, 1, 64),
             state_index=i32([2, 0]), ctx_lens=i32([9, 22]), cu_q=i32([0, 9, 30]))
    decay, seen = torch.zeros(1, device="cuda:0"), h(30, 2, 64)
    gated = h(9, 3)
    return [(lambda: fs.ProjectPlan(ctx, x, w, sw, fs.Norm(gain), bias, "silu", res, out=out, **kw), [x, w, sw, bias, gain, res, out]),
            (lambda: fs.GatedProjectPlan(ctx, x, w, sw, fs.Norm(gain), bias, out=gated, **kw), [x, w, sw, bias, gain, gated]),
            (lambda: fs.StateAttentionPlan(ctx, **a, max_q=21, log_decay=decay, out=seen, **kw), [*a.values(), decay, seen])]


def test_every_tensor_is_held_against_the_context_device(env, monkeypatch):
    fs, ctx = env
    seen, check = [], fs._same_device

    def record(ctx, **tensors):
        seen.extend(t for t in tensors.values() if t is not None)
        check(ctx, **tensors)
    monkeypatch.setattr(fs, "_same_device", record)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda:0")
    for call, tensors in plans(fs, ctx, workspace=ws):
        seen.clear()
        plan = call()
        assert {t.data_ptr() for t in (*tensors, ws)} <= {t.data_ptr() for t in seen}
        assert {t.data_ptr() for t in tensors if t is not plan.out} <= {t.data_ptr() for t in plan._keep if t is not None}


def test_workspaces_that_are_refused(env):
    fs, ctx = env
    size = 1 << 22
    for ws in (torch.empty(size, dtype=torch.uint8), torch.empty(size // 4, dtype=torch.float32, device="cuda:0"),
               torch.empty(2 * size, dtype=torch.uint8, device="cuda:0")[::2]):
        for call, _ in plans(fs, ctx, workspace=ws):
            with pytest.raises(fs.FleetSieveError) as e:
                call()
            assert e.value.status == fs.FS_ERR_INVALID_ARGUMENT and "workspace" in str(e.value)
    off = torch.empty(size + 1, dtype=torch.uint8, device="cuda:0")[1:]
    for call, _ in plans(fs, ctx, workspace=off):
        with pytest.raises(fs.FleetSieveError) as e:
            call().run()
        assert e.value.status == fs.FS_ERR_INVALID_ARGUMENT


def test_memory_given_back_while_another_stream_works_on_it(env):
    fs, ctx = env
    note("inputs for another stream")
    T, H, D = 2000, 2, 64
    g = torch.Generator(device="cuda:0").manual_seed(1)
    make = lambda *s: torch.randn(*s, device="cuda:0", generator=g).to(torch.bfloat16)  # noqa: E731
    q, k, v = make(T, H, D), make(T, H, D), make(T, H, D)
    states, decay = torch.zeros(1, H, D, D, device="cuda:0"), -torch.ones(H, device="cuda:0") / 50
    where = dict(state_index=i32([0]), ctx_lens=i32([T]), cu_q=i32([0, T]), max_q=T, log_decay=decay)
    want = fs.state_attention(ctx, states.clone(), q, k, v, **where)
    side, own = torch.cuda.Stream(), fs.Context(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    got = fs.state_attention(own, states, q, k, v, **where, stream=side)
    old = own.workspace(0).numel()
    del q, k, v
    own.workspace(4 * old)  # another one: the one in use is given back
    filler = [torch.full((T, H, D), 3.0, dtype=torch.bfloat16, device="cuda:0") for _ in range(3)]
    filler.append(torch.full((old,), 255, dtype=torch.uint8, device="cuda:0"))
    torch.cuda.synchronize()
    assert torch.equal(bits(got), bits(want))
    del filler
    own.close()


def test_two_calls_at_once(env):
    """On two streams, with workspaces of their own, of products that are cut and
    prompts in segments."""
    fs, ctx = env
    g = torch.Generator(device="cuda:0").manual_seed(2)
    make = lambda *s: torch.randn(*s, device="cuda:0", generator=g).to(torch.bfloat16)  # noqa: E731
    streams = [torch.cuda.Stream() for _ in range(2)]
    jobs = []
    for n in range(2):
        x, w = make(64, 8192), torch.randint(-127, 128, (1280, 8192), device="cuda:0", generator=g, dtype=torch.int8)
        sw = torch.full((1280,), 1e-4, device="cuda:0")
        q, k, v = make(1500, 4, 64), make(1500, 2, 64), make(1500, 2, 64)
        a = dict(state_index=i32([0, 1]), ctx_lens=i32([700, 800]), cu_q=i32([0, 700, 1500]), max_q=800,
                 log_decay=torch.tensor([-0.01, -0.1], device="cuda:0"))
        pool = torch.zeros(2, 2, 64, 64, device="cuda:0")
        ws = [torch.empty(1 << 25, dtype=torch.uint8, device="cuda:0") for _ in range(2)]
        jobs.append((x, w, sw, pool, q, k, v, a, ws))

    def run(job, stream):
        x, w, sw, pool, q, k, v, a, ws = job
        on = [dict(stream=stream, workspace=s) for s in ws]
        return (fs.gated_project(ctx, x, w, sw, norm=fs.Norm(None), **on[0]),
                fs.state_attention(ctx, pool.clone(), q, k, v, **a, **on[1]))
    want = [run(job, None) for job in jobs]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for job, stream in zip(jobs, streams):
            with torch.cuda.stream(stream):
                got.append([run(job, stream) for _ in range(4)])
        torch.cuda.synchronize()
        for mine, right in zip(got, want):
            for pair in mine:
                assert all(torch.equal(bits(a), bits(b)) for a, b in zip(pair, right))


def test_far_rows_and_many_states(env):
    """Offsets past 2^31 elements: a pool of more than 2^31 floats, rows that lie far apart."""
    fs, ctx = env
    note("a large pool")
    P, H, D = 70000, 2, 128  # 2.3 * 10^9 floats
    pool = torch.empty(P, H, D, D, device="cuda:0")
    first, last = 1, P - 1
    start = torch.randn(2, H, D, D, generator=gen(1))
    pool[first], pool[last] = start[0].to("cuda:0"), start[1].to("cuda:0")
    for n in (1, 70):
        wide = 1 << 25  # elements from token to token
        flat = torch.empty(2 * n * wide, dtype=torch.bfloat16, device="cuda:0").view(2 * n, wide)
        rows = torch.randn(2 * n, 4 * H * D, generator=gen(n)).to(torch.bfloat16)
        flat[:, :4 * H * D] = rows.to("cuda:0")
        cut = lambda t, a, b: t[:, a * D:b * D].unflatten(1, (b - a, D))  # noqa: E731
        small = torch.stack([pool[first], pool[last]])
        a = dict(ctx_lens=i32([n + 5, n + 5]), cu_q=i32([0, n, 2 * n]), max_q=n, log_decay=torch.tensor([-0.1, -0.01], device="cuda:0"))
        near = rows.to("cuda:0")
        want = fs.state_attention(ctx, small, cut(near, 0, 4), cut(near, 4, 6), cut(near, 6, 8), i32([0, 1]), **a)
        got = fs.state_attention(ctx, pool, cut(flat, 0, 4), cut(flat, 4, 6), cut(flat, 6, 8), i32([first, last]), **a)
        assert torch.equal(bits(got), bits(want))
        assert torch.equal(pool[first], small[0]) and torch.equal(pool[last], small[1])
        del flat
    assert math.isfinite(float(pool[last].sum()))
