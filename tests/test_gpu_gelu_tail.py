"""gelu of negative arguments, whose value is small beside them."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_serving import env, note  # noqa: E402, F401


@pytest.mark.parametrize("gated", [False, True])
def test_gelu_to_its_own_size(env, gated):
    """Rows of one element 127 m / 2^14, whose scale m / 2^14 and projection are exact: what
    is off is the activation, by less than 2^-20 (1 + |y|) of itself and a rounding."""
    fs, ctx = env
    note("gelu of negative arguments")
    y = -127.0 * torch.arange(1, 1651, dtype=torch.float32) / 2.0 ** 14
    x, one = y[:, None].to("cuda:0"), torch.ones(1, device="cuda:0")
    w = torch.ones(1, 1, dtype=torch.int8, device="cuda:0")
    if gated:  # the value is 1
        zero = torch.zeros(1, 1, dtype=torch.int8, device="cuda:0")
        got = fs.gated_project(ctx, x, torch.cat([w, zero]), torch.cat([one, one]), bias=torch.cat([0 * one, one]), activation="gelu")
    else:
        got = fs.project(ctx, x, w, one, activation="gelu")
    y = y.double()
    want = 0.5 * y * torch.special.erfc(-y * math.sqrt(0.5))
    off = (got[:, 0].double().cpu() - want).abs() / want.abs()
    assert (off <= 2.0 ** -20 * (1 + y.abs()) + 2.0 ** -24).all(), float(off.max())
