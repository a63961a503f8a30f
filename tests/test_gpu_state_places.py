"""State attention in the workspace that it asks for: no segment is left out, whatever
the lengths are, and a workspace of the most tokens serves fewer."""
import ctypes

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_serving import bits, env, gen, note  # noqa: E402, F401


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


def size(fs, heads, D, T, S):
    like = fs._StatePool(None, S, heads, D)
    return fs._size(fs.load_library().fs_state_attention_workspace_size, ctypes.byref(like), heads, T, S)


def attend(fs, ctx, x, news, D, workspace):
    heads, S = x.shape[1], len(news)
    cu = [0]
    for n in news:
        cu.append(cu[-1] + n)
    pool = torch.zeros(S, heads, D, D, device="cuda:0")
    out = torch.full_like(x, float("nan"))
    fs.state_attention(ctx, pool, x, x, x, i32(list(range(S))), i32(news), i32(cu), max(news),
                       torch.full((heads,), -0.5, device="cuda:0"), out=out, workspace=workspace)
    return out, pool


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [1, 3, 5])
def test_every_segment_has_a_place(env, heads, D):
    """Tokens a little above and below where the least length of a segment goes up."""
    fs, ctx = env
    step = 64 * (256 if D == 128 else 512) // heads
    note(f"places, {heads} heads of {D}")
    for T in (step - 1, step, step + 1, step + 40, step + 64, step + step // 64, step + step // 64 + 1, 2 * step + 1, 2 * step + 70):
        x = torch.randn(T, heads, D, generator=gen(T)).to(torch.bfloat16).to("cuda:0")
        most = T // 65
        for news in ([T], [T - 130, 65, 65], [65] * min(most, 300), [T - 65 * min(most - 2, 200)] + [65] * min(most - 2, 200)):
            total = sum(news)
            need = size(fs, heads, D, total, len(news))
            room = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda:0")
            out, pool = attend(fs, ctx, x[:total], news, D, room[:need])
            assert torch.isfinite(out.float()).all() and torch.isfinite(pool).all() and (room[need:] == 77).all(), (T, news[:3])


def test_a_workspace_of_the_most_tokens_serves_fewer(env):
    fs, ctx = env
    heads, D, T = 8, 128, 2112
    note("a workspace of the most tokens")
    ws = torch.empty(size(fs, heads, D, T, 64), dtype=torch.uint8, device="cuda:0")
    x = torch.randn(T, heads, D, generator=gen(1)).to(torch.bfloat16).to("cuda:0")
    for news in ([2112], [2048], [1000, 1048], [33] * 62, [32] * 64, [300, 1, 70], [1] * 64):
        total = sum(news)
        want = attend(fs, ctx, x[:total], news, D, None)
        got = attend(fs, ctx, x[:total], news, D, ws)
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(got, want)), news[:3]
