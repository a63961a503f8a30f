"""What the parts of decayed values make of a state, on the CPU: the bound that the
states are held to tells as many parts as there are from one fewer."""
import pytest
import torch

import layer_reference as ref


def state_of_parts(k, v, decay, dtype, count):
    """The state after k and v [n, D] in chunks of 64 tokens, decayed values in parts;
    sums in 64 bits."""
    state = torch.zeros(k.shape[1], v.shape[1], dtype=torch.float64)
    for at in range(0, k.shape[0], 64):
        kc, vc = k[at:at + 64], v[at:at + 64].float()
        n = kc.shape[0]
        fade = torch.exp(decay * torch.arange(n - 1, -1, -1, dtype=torch.float64))
        x = (vc.double() * fade[:, None]).float()
        state = torch.exp(decay * n) * state + kc.double().t() @ ref.in_parts(x, dtype, count).double()
    return state


@pytest.mark.parametrize("dtype,parts", [(torch.bfloat16, 3), (torch.float16, 2)], ids=["bf16", "f16"])
@pytest.mark.parametrize("n", [65, 200, 1000])
def test_a_part_fewer_is_beyond_the_bound(n, dtype, parts):
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn(n, 64, generator=g).to(dtype) for _ in range(2))
    for rate in (-1.0, -2.0 ** -4, -2.0 ** -8):
        decay = torch.tensor(rate, dtype=torch.float64)
        _, want, _, _ = ref.state_attend(k[:, None], k[:, None], v[:, None], torch.zeros(1, 64, 64), decay[None], 1.0)

        def off(count):
            return float((state_of_parts(k, v, decay, dtype, count) - want[0]).norm() / want[0].norm())
        most = ref.state_norm(n, rate)
        assert off(parts) < most / 2 and off(parts - 1) > most, (rate, off(parts), off(parts - 1), most)
