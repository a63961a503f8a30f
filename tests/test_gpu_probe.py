"""The probe's layers: the serving operators together, against the same
layers in plain arithmetic, and the planner's calls on what it measured."""
import pytest
import torch

import serving_reference as ref
from paper_2608_19659_amd import fleetsieve as fs
from paper_2608_19659_amd import probe
from paper_2608_19659_amd.synth import Problem

pytestmark = pytest.mark.gpu
SMALL = probe.Decoder(hidden=256, q_heads=8, kv_heads=4, head_dim=64, ffn=512, layers=4)


@pytest.fixture(scope="module")
def ctx():
    torch.cuda.init()
    return fs.Context(0)


def plain(shard, new, held):
    """The layers in binary64, activations not quantised, new keys and
    values not either."""
    w = [[(c.double().cpu() * s.double().cpu()[:, None]) for c, s in layer] for layer in shard.weights]
    h = shard.x.double().cpu()
    D, hq, hkv = shard.decoder.head_dim, shard.hq, shard.hkv
    norm = lambda x: x / (x.pow(2).mean(1, keepdim=True) + torch.finfo(torch.bfloat16).eps).sqrt()  # noqa: E731
    cos, sin, at = shard.cos.cpu(), shard.sin.cpu(), shard.positions.cpu()
    for i, (qkv, out, up, down) in enumerate(w):
        rows = (norm(h) @ qkv.t()).view(-1, hq + 2 * hkv, D)
        q, k = ref.rotate(rows[:, :hq], cos, sin, at), ref.rotate(rows[:, hq:hq + hkv], cos, sin, at)
        v, seen, row = rows[:, hq + hkv:], [], 0
        cache = shard.before[i]
        for s, (n, m) in enumerate(zip(new, held)):
            pages = shard.table[s].cpu()[torch.arange(m) // probe.PAGE].long()
            place = torch.arange(m) % probe.PAGE
            ks = cache[0][pages, :, place].double() * cache[2][pages].double()[:, :, None]
            vs = cache[1][pages, :, :, place].double() * cache[3][pages].double()[:, :, None]
            ks[m - n:], vs[m - n:] = k[row:row + n], v[row:row + n]
            seen.append(ref.attend(q[row:row + n], ks, vs, m - n, D ** -0.5))
            row += n
        h = h + torch.cat(seen).view(-1, hq * D) @ out.t()
        wide = norm(h) @ up.t()
        h = h + (torch.nn.functional.silu(wide[:, :shard.ffn]) * wide[:, shard.ffn:]) @ down.t()
    return h


@pytest.mark.parametrize("tp", [1, 4])
@pytest.mark.parametrize("new,held", [([1], [200]), ([1, 1, 1], [70, 1, 333]), ([150], [150]), ([1, 40, 3], [128, 100, 3])],
                         ids=str)
def test_layers(ctx, tp, new, held):
    """Eight bits leave an activation off by up to 1/254 of its row's largest,
    about 0.7% of the row in the root mean square, and a new key or value likewise; four
    projections of two layers add up to about 2%, and what is stored in bfloat16
    adds less.  A tenth would be a wrong path, which is off by the whole."""
    shard = probe.Shard(ctx, SMALL, tp, new, held, layers=2, seed=tp)
    shard.before = [[t.cpu().clone() for t in (c.k, c.v, c.k_scale, c.v_scale)] for c in shard.caches]
    got = shard.forward()
    shard.stream.synchronize()
    want = plain(shard, new, held)
    change = want - shard.x.double().cpu()
    off = (got.double().cpu() - want).norm() / change.norm()
    assert off < 0.1, float(off)


def test_the_captured_layers_are_the_eager_ones(ctx):
    new, held = [1, 1, 5], [70, 1, 333]
    shard = probe.Shard(ctx, SMALL, 2, new, held, layers=2)
    graph, out = shard.capture()
    # the new tokens' codes are entered anew on every run; the scales of their pages
    # only grow to what the same tokens need, so a run after the first changes nothing
    for i in range(4):
        with torch.cuda.stream(shard.stream):
            shard.x.normal_()
        want = [shard.forward() for _ in range(2)][-1]
        with torch.cuda.stream(shard.stream):
            graph.replay()
        shard.stream.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))


def test_probe_to_plan(ctx):
    classes = (probe.Class("chat", 96, 16, 40.0, 1.0), probe.Class("code", 160, 4, 60.0, 1.0))
    times = probe.measure(ctx, SMALL, [1, 2, 4], [1, 4], classes, layers=2)
    assert all(0.0 < fast <= slow for fast, slow in times.prefill.values())
    problem = Problem(tp=[1, 2, 4], levels=probe.LEVELS, demand=[c.demand for c in classes], slo=[c.slo for c in classes],
                      budget=16)
    iv = probe.intervals(problem, classes, times)
    says = probe.plan(ctx, problem, iv, samples=64)
    # no cell is measured, so no fleet is certified; the fast side is no worse
    assert says["state"] == "undecided"
    assert says["slow"]["fulfilment"] <= says["fast"]["fulfilment"]
    assert says["gap"] == pytest.approx(says["fast"]["fulfilment"] - says["slow"]["fulfilment"])
    assert says["measure_next"] is not None
