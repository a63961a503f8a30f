"""State attention in chunks where the terms of a state, of an output or of a decay
lie many powers of two apart: each is held to its own size, not to the largest's."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import layer_reference as ref  # noqa: E402
from test_gpu_serving import STEP, TYPES, bits, env, gen, note  # noqa: E402, F401

LEAST = 2.0 ** -120  # what is below binary32's normal numbers, times keys and queries of a few units


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


def attend(env, q, k, v, state, decay, scale, held=5):
    """Outputs and state of one sequence whose state is `state`, as 64-bit numbers."""
    fs, ctx = env
    n = q.shape[0]
    pool = state[None].to("cuda:0").contiguous()
    out = fs.state_attention(ctx, pool, q.to("cuda:0"), k.to("cuda:0"), v.to("cuda:0"), i32([0]), i32([n + held]),
                             i32([0, n]), n, decay.to("cuda:0"), scale=scale)
    return out.double().cpu(), pool[0].double().cpu()


def spread(shape, g, least, most):
    """Numbers of either sign between 10^least and 10^most, even over the logarithm."""
    size = 10.0 ** (torch.rand(shape, generator=g) * (most - least) + least)
    return size * (torch.randint(0, 2, shape, generator=g) * 2 - 1)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,group", [(64, 2), (128, 3), (128, 1)])
@pytest.mark.parametrize("n", [9, 64, 200, 700])
def test_keys_that_meet_one_row_each(env, n, D, group, dtype):
    """A token's key has one element, so a row of the state has the terms of few tokens
    and nothing hides a decayed one.  Each term: its decay 2 steps of binary32 and
    the product of two powers one, the value times it one, the value as parts 4 (2^-22);
    up to 12 chunks later a decay's rounding and a product's each, and as many sums of
    two steps: 56 steps of 2^-24 at most, below 2^-18."""
    heads = 5
    g = gen(n + D)
    decay = torch.tensor([-0.05, -0.25, -0.7, -1.3, -1.9])
    k = torch.zeros(n, heads, D)
    at = (torch.arange(n)[:, None] * torch.tensor([1, 3, 5, 7, 9])) % D
    k.scatter_(2, at[..., None], torch.randn(n, heads, 1, generator=g) + 2.0)
    k, v = k.to(TYPES[dtype]), torch.randn(n, heads, D, generator=g).to(TYPES[dtype])
    # a query sees some of the rows
    q = (torch.randn(n, heads * group, D, generator=g) * (torch.rand(n, heads * group, D, generator=g) < 0.1)).to(TYPES[dtype])
    state = torch.randn(heads, D, D, generator=g)
    note(f"keys of one element, {n} tokens, D{D}x{group} {dtype}")
    got, mine = attend(env, q, k, v, state, decay, 1.0)
    want, end, room, _ = ref.state_attend(q, k, v, state, decay, 1.0)
    size = ref.state_attend(k, k.abs(), v.abs(), state.abs(), decay, 1.0)[1]  # the state's terms without their signs
    off = (mine - end).abs()
    assert (off <= size * 2.0 ** -18 + LEAST).all(), float((off / (size + LEAST)).max())
    room = room + (want.abs() + room) * STEP[dtype] + (2.0 ** -25 if dtype == "f16" else 0.0)
    assert ((got - want).abs() <= room + LEAST).all(), float(((got - want).abs() - room).max())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,group", [(64, 1), (128, 2)])
@pytest.mark.parametrize("least,most", [(-3, 7), (-3, 12), (-20, 20)])
@pytest.mark.parametrize("n", [9, 64, 150])
def test_states_of_many_sizes(env, n, least, most, D, group, dtype):
    """Elements of a column of the state from 10^least to 10^most, and queries that see
    only rows whose elements are small: an output is off by its own terms' share."""
    heads = 2
    g = gen(n + most)
    state = spread((heads, D, D), g, least, most)
    rows = torch.arange(D) % 2 == 0
    state[:, rows] = spread((heads, D, D), g, least, least + 1)[:, rows]
    make = lambda h: torch.randn(n, h, D, generator=g)  # noqa: E731
    q = (make(heads * group) * rows).to(TYPES[dtype])
    k, v = (make(heads) * 10.0 ** min(0, least)).to(TYPES[dtype]), make(heads).to(TYPES[dtype])
    decay, scale = torch.tensor([-1e-3, -0.1]), 1.0
    note(f"states of 1e{least} to 1e{most}, {n} tokens, D{D}x{group} {dtype}")
    got, mine = attend(env, q, k, v, state, decay, scale)
    want, end, room, state_room = ref.state_attend(q, k, v, state, decay, scale)
    room = room + (want.abs() + room) * STEP[dtype] + (2.0 ** -25 if dtype == "f16" else 0.0)
    seen = (want.abs() < 6e4) if dtype == "f16" else torch.ones_like(want, dtype=torch.bool)
    off = (got - want).abs()[seen]
    assert (off <= room[seen]).all(), float((off / room[seen].clamp(min=1e-300)).max())
    assert ((mine - end).abs() <= state_room).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [9, 64, 130])
def test_values_that_only_one_token_has(env, n, dtype):
    """Value columns in which the tokens' values lie far apart, and tokens whose own
    value is zero there: an output is the decayed products of earlier tokens."""
    heads, group, D = 3, 2, 64
    g = gen(n)
    v = spread((n, heads, D), g, -4, 3) * (torch.rand(n, heads, D, generator=g) < 0.05)
    q, k = torch.randn(n, heads * group, D, generator=g), torch.randn(n, heads, D, generator=g)
    q, k, v = (x.to(TYPES[dtype]) for x in (q, k, v))
    decay = torch.tensor([-0.5, -1.0, -2.0])
    state = torch.zeros(heads, D, D)
    note(f"values far apart, {n} tokens {dtype}")
    got, mine = attend(env, q, k, v, state, decay, 0.25)
    want, end, room, state_room = ref.state_attend(q, k, v, state, decay, 0.25)
    room = room + (want.abs() + room) * STEP[dtype] + (2.0 ** -25 if dtype == "f16" else 0.0)
    off = (got - want).abs()
    # of a decayed product what is below 2^-126 may be lost, in either of its parts, times
    # values of up to 1e3 of some seven tokens: 2 * 2^-126 * 7 * 1e3 < 2^-112
    assert (off <= room + 2.0 ** -112).all(), float((off - room).max())
    assert ((mine - end).abs() <= state_room + 2.0 ** -112).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("what", ["state", "value", "key"])
def test_no_numbers_beside_elements_far_apart(env, what, bad, dtype):
    """A column, a row or a token that is no number, among states of many sizes: other
    columns and earlier tokens stay as they were."""
    heads, D, n, at = 2, 64, 100, 70
    g = gen(3)
    state = spread((heads, D, D), g, -6, 6)
    make = lambda h: torch.randn(n, h, D, generator=g).to(TYPES[dtype])  # noqa: E731
    q, k, v, decay = make(heads), make(heads), make(heads), torch.tensor([-0.5, -1.0])
    note(f"no numbers among many sizes: {what} {bad} {dtype}")
    want, end, room, state_room = ref.state_attend(q, k, v, state, decay, 1e-4)
    room = room + (want.abs() + room) * STEP[dtype] + (2.0 ** -25 if dtype == "f16" else 0.0)
    hit, lost = torch.zeros(n, heads, D, dtype=torch.bool), torch.zeros(heads, D, D, dtype=torch.bool)
    if what == "state":
        state[1, 3, 9] = bad
        hit[:, 1, 9], lost[1, 3, 9] = True, True
    elif what == "value":
        v[at, 1, 9] = bad
        hit[at:, 1, 9], lost[1, :, 9] = True, True
    else:
        k[at, 1, 9] = bad
        hit[at:, 1], lost[1, 9] = True, True
    got, mine = attend(env, q, k, v, state, decay, 1e-4)
    assert not torch.isfinite(got[hit]).any() and ((got - want).abs() <= room + LEAST)[~hit].all()
    assert not torch.isfinite(mine[lost]).any() and ((mine - end).abs() <= state_room + LEAST)[~lost].all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [65, 200, 1000])
def test_dense_states_to_their_own_norm(env, n, dtype):
    """Of random keys and values a state's terms add up as their squares do, and so do
    their errors: ref.state_norm says what is left beside the state's own norm
    (a part of the values less is beyond it)."""
    g = gen(n)
    heads, D = 3, 64
    q, k, v = (torch.randn(n, heads, D, generator=g).to(TYPES[dtype]) for _ in range(3))
    state, decay = torch.randn(heads, D, D, generator=g) * 4, torch.tensor([-1.0, -2.0 ** -4, -2.0 ** -8])
    note(f"dense states, {n} tokens {dtype}")
    _, mine = attend(env, q, k, v, state, decay, 0.125)
    end = ref.state_attend(q, k, v, state, decay, 0.125)[1]
    for h in range(heads):
        off = float((mine[h] - end[h]).norm() / end[h].norm())
        assert off < ref.state_norm(n, float(decay[h])), (h, off)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("news", [[100], [70, 1, 300], [900]], ids=str)
def test_replays_are_the_eager_calls(env, news, dtype):
    """States of many sizes and fast decays, captured and replayed, each replay from the
    states of the one before."""
    fs, ctx = env
    heads, group, D, S = 2, 2, 64, len(news)
    note(f"replays of states of many sizes, {news} {dtype}")
    g = gen(sum(news))
    cu = [0]
    for n in news:
        cu.append(cu[-1] + n)
    make = lambda h: torch.randn(cu[-1], h, D, generator=g).to(TYPES[dtype]).to("cuda:0")  # noqa: E731
    q, k, v = make(heads * group), make(heads), make(heads)
    pools = [spread((S, heads, D, D), gen(1), -6, 3).to("cuda:0") for _ in range(2)]
    where = (i32(list(range(S))), i32([n + 5 for n in news]), i32(cu), max(news), torch.tensor([-0.7, -0.01], device="cuda:0"))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    ws = torch.empty(16 << 20, dtype=torch.uint8, device="cuda:0")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = fs.state_attention(ctx, pools[0], q, k, v, *where, stream=side, workspace=ws)
    for i in range(4):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gen(i)))
        graph.replay()
        want = fs.state_attention(ctx, pools[1], q, k, v, *where)
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(want)) and torch.equal(bits(pools[0]), bits(pools[1])), i
