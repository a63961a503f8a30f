"""State attention in chunks: the decay of tokens far back in a chunk."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import layer_reference as ref  # noqa: E402
from test_gpu_serving import TYPES, env, gen, note  # noqa: E402, F401


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [40, 64])
def test_far_tokens_decay_like_near_ones(env, n, D):
    """Each token's key has an element of its own, so a row of the state is one token's
    decayed value.  Steps of 2^-24: the power 3 (its two factors and their product), the
    value times it 1, three parts of 8 bits 1, the products and sums with nothing
    6: less than 2^-20 of the term, however far back the token is."""
    fs, ctx = env
    note(f"decays of {n} tokens, D{D}")
    decay = torch.tensor([-0.03, -0.11, -0.37, -0.77, -1.1, -1.23])
    heads, g = len(decay), gen(n + D)
    k = torch.zeros(n, heads, D)
    k[torch.arange(n), :, torch.arange(n)] = 1.0
    q, v = torch.randn(n, heads, D, generator=g).bfloat16(), torch.randn(n, heads, D, generator=g).bfloat16()
    pool = torch.zeros(1, heads, D, D, device="cuda:0")
    fs.state_attention(ctx, pool, q.to("cuda:0"), k.bfloat16().to("cuda:0"), v.to("cuda:0"), i32([0]), i32([n]), i32([0, n]), n,
                       decay.to("cuda:0"))
    want = ref.state_attend(q, k, v, torch.zeros(heads, D, D), decay, 1.0)[1]
    off = (pool[0].double().cpu() - want).abs()
    # a part below 2^-126 may be lost
    assert (off <= want.abs() * 2.0 ** -20 + 2.0 ** -125).all(), float((off / want.abs().clamp(min=2.0 ** -100)).max())
