"""The probe's layers with a state a head: all of the operators between a residual
stream and itself, against the same layers in plain arithmetic."""
import pytest
import torch

import layer_reference as ref
from paper_2608_19659_amd import fleetsieve as fs
from paper_2608_19659_amd import probe

pytestmark = pytest.mark.gpu
SMALL = probe.Decoder(hidden=256, q_heads=8, kv_heads=4, head_dim=64, ffn=512, layers=4, attention="state")


@pytest.fixture(scope="module")
def ctx():
    torch.cuda.init()
    return fs.Context(0)


def plain(shard, new, held, states):
    """The layers in binary64, activations not quantised."""
    D, hq, hkv, ffn = shard.decoder.head_dim, shard.hq, shard.hkv, shard.ffn
    h, decay = shard.x.double().cpu(), shard.log_decay.cpu()
    norm = lambda x: x / (x.pow(2).mean(1, keepdim=True) + probe.EPS).sqrt()  # noqa: E731
    for i, layer in enumerate(shard.weights):
        qkv, out, up, down = [c.double().cpu() * s.double().cpu()[:, None] for c, s in layer]
        rows = (norm(h) @ qkv.t()).view(-1, hq + 2 * hkv, D)
        seen, row = [], 0
        for s, (n, m) in enumerate(zip(new, held)):
            at = rows[row:row + n]
            start = states[i][s] if m > n else torch.zeros(hkv, D, D)
            seen.append(ref.state_attend(at[:, :hq], at[:, hq:hq + hkv], at[:, hq + hkv:], start, decay, D ** -0.5)[0])
            row += n
        h = h + torch.cat(seen).flatten(1) @ out.t()
        wide = norm(h) @ up.t()
        h = h + (torch.nn.functional.silu(wide[:, :ffn]) * wide[:, ffn:]) @ down.t()
    return h


@pytest.mark.parametrize("tp", [1, 4])
@pytest.mark.parametrize("new,held", [([1], [200]), ([1, 1, 1], [70, 1, 333]), ([150], [150]), ([1, 40, 3], [128, 100, 3])],
                         ids=str)
def test_layers(ctx, tp, new, held):
    """As of the layers over a cache: four projections of two layers in eight bits
    leave about 2%, and a tenth would be a wrong path."""
    shard = probe.Shard(ctx, SMALL, tp, new, held, layers=2, seed=tp)
    states = [s.cpu().clone() for s in shard.states]
    got = shard.forward()
    shard.stream.synchronize()
    want = plain(shard, new, held, states)
    change = want - shard.x.double().cpu()
    off = (got.double().cpu() - want).norm() / change.norm()
    assert off < 0.1, float(off)


def test_the_captured_layers_are_the_eager_ones(ctx):
    new, held = [1, 1, 5, 90], [70, 1, 333, 90]
    shard = probe.Shard(ctx, SMALL, 2, new, held, layers=2)
    graph, out = shard.capture()
    for i in range(4):
        with torch.cuda.stream(shard.stream):
            shard.x.normal_()
            before = [s.clone() for s in shard.states]
            want = shard.forward()
            after = [s.clone() for s in shard.states]
            for s, b in zip(shard.states, before):
                s.copy_(b)
            graph.replay()
        shard.stream.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
        assert all(torch.equal(s, a) for s, a in zip(shard.states, after))


def test_its_times(ctx):
    classes = (probe.Class("chat", 96, 16, 40.0, 1.0),)
    times = probe.measure(ctx, SMALL, [1, 2], [1, 4], classes, layers=2)
    assert all(0.0 < fast <= slow for fast, slow in times.prefill.values())
    assert all(0.0 < fast <= slow for steps in times.step.values() for fast, slow in steps.values())
