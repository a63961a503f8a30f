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
