"""The norm of long rows whose values are as large as their type's largest."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import layer_reference as ref  # noqa: E402
from test_gpu_serving import TYPES, env, gen, note  # noqa: E402, F401


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [64, 65536, 65537, 131071])
@pytest.mark.parametrize("M", [1, 3])
def test_rows_of_the_largest_values(env, M, K, dtype):
    """Sums of squares beyond binary32.  A thread adds up to 128 elements of a row, all
    of one sign, wavefronts and blocks two dozen sums more; the factor is its root, and as
    a number below the normal ones has 2^-22 more: within twice what the shorter
    rows' bound has."""
    fs, ctx = env
    note(f"rows of the largest values, {M}x{K} {dtype}")
    g = gen(K)
    most = torch.finfo(TYPES[dtype]).max
    x = torch.full((M, K), most, dtype=TYPES[dtype]) * (torch.randint(0, 2, (M, K), generator=g) * 2 - 1).to(TYPES[dtype])
    w = torch.randint(-127, 128, (80, K), generator=g, dtype=torch.int8)
    sw, gain = torch.rand(80, generator=g) / 1000.0, torch.rand(K, generator=g) * 0.5 + 0.3
    d = lambda t: t.to("cuda:0")  # noqa: E731
    got = fs.project(ctx, d(x), d(w[:40]), d(sw[:40]), norm=fs.Norm(d(gain), 1e-5), out_dtype=torch.float32)
    want, room = ref.project(x, w[:40], sw[:40], (gain, 1e-5))
    assert ((got.double().cpu() - want).abs() <= 2 * room).all()
    got = fs.gated_project(ctx, d(x), d(w), d(sw), norm=fs.Norm(d(gain), 1e-5), out_dtype=torch.float32)
    want, room = ref.gated(x, w, sw, (gain, 1e-5))
    assert ((got.double().cpu() - want).abs() <= 2 * room).all()
