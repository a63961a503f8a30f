"""Probes a fleet's cells on this GPU, for a planner that has no measurements yet.

A cell is (class, TP degree, load): what one tensor-parallel replica of a
served model does at that load.  The command runs, on one GPU, the work of one
rank of such a replica: decoder layers whose projections are 8-bit products, with
the norm before them and the activation or the residual stream behind
(fs_project, fs_gated_project), whose keys and values go rotated into a paged 8-bit
cache (fs_cache_append) and whose attention reads it (fs_cache_attention), or which
keep a decaying state a head instead (fs_state_attention, --attention state), once
as decode steps of several batch sizes and once as the prefill of a prompt.  From
the times come an interval for every cell's capacity and tail; the planner's own calls
(fs_certify, fs_score_candidates) then say what the fleet would be and which
cell is worth a real measurement first.

    python -m paper_2608_19659_amd.probe
    python -m paper_2608_19659_amd.probe --tp 2 4 8 --batch 1 8 64 --budget 32
    python -m paper_2608_19659_amd.probe --attention state

What a rank's time leaves out is the sum over the replica's ranks after the
output and the down projection.  The fast side of an interval has it hidden
behind other work, the slow side has it exposed, at the rate and latency given
(--link-gbs, --hop-us).  The vocabulary's projection, sampling and scheduling
are in neither.  Weights and inputs are random; nothing here depends on
their values.  torch supplies memory, streams and graphs.
"""
from __future__ import annotations

import argparse
import json
import math
from dataclasses import dataclass, field

import numpy as np

from . import fleetsieve as fs
from .synth import Intervals, Problem

QUANTUM = 1.0 / 64.0  # capacity grid, req/s
UNSERVED = 1.0e6      # tail of a cell whose load no batch sustains: seconds past every SLO, yet a number
PAGE = 64
ATTENTIONS = ("cache", "state")
EPS = 2.0 ** -7  # of the norms: bfloat16's step


@dataclass(frozen=True)
class Decoder:
    """A decoder's sizes.  The defaults have 31 billion weights.  attention:
    "cache" of every token's keys and values, or "state", one matrix a head."""
    hidden: int = 5120
    q_heads: int = 40
    kv_heads: int = 8
    head_dim: int = 128
    ffn: int = 20480
    layers: int = 80
    attention: str = "cache"

    def check(self, tp: int):
        if self.attention not in ATTENTIONS:
            raise ValueError(f"attention must be one of {', '.join(ATTENTIONS)}, got {self.attention!r}")
        if tp < 1 or self.q_heads % tp or self.kv_heads % tp or self.ffn % tp:
            raise ValueError(f"{self.q_heads} and {self.kv_heads} heads and {self.ffn} columns do not divide over TP {tp}")


@dataclass(frozen=True)
class Class:
    """A workload class: tokens of a prompt and of an answer, requests per
    second, seconds a request may take."""
    name: str
    prompt: int
    answer: int
    demand: float
    slo: float


CLASSES = (Class("chat", 1024, 256, 16.0, 3.0), Class("code", 2048, 32, 12.0, 0.6))
LEVELS = (1.0, 2.0, 4.0, 8.0, 16.0, 32.0)


# ---------------------------------------------------------------- the work --
class Shard:
    """One rank's layers for a batch: sequence s has new[s] new tokens and
    held[s] tokens in its cache after them.  `layers` of the decoder's layers
    exist, each with weights and a cache of its own, so that one layer's do not wait in a
    cache of the GPU for their next use; the others' time is theirs."""

    def __init__(self, ctx, decoder: Decoder, tp: int, new, held, layers: int = 8, stream=None, seed: int = 0):
        import torch
        decoder.check(tp)
        if len(new) != len(held) or any(n < 1 or h < n for n, h in zip(new, held)):
            raise ValueError("every sequence needs a new token and holds its new tokens")
        self.ctx, self.decoder, self.layers = ctx, decoder, min(layers, decoder.layers)
        self.hq, self.hkv, D = decoder.q_heads // tp, decoder.kv_heads // tp, decoder.head_dim
        self.ffn = decoder.ffn // tp
        dev = torch.device("cuda", ctx.device)
        self.stream = stream if stream is not None else torch.cuda.Stream(dev)
        g = torch.Generator(device=dev).manual_seed(seed)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731

        def weight(n, k):
            w = torch.randint(-127, 128, (n, k), dtype=torch.int8, device=dev, generator=g)
            return w, torch.full((n,), 1.0 / (73.0 * math.sqrt(k)), device=dev)  # 73: deviation of the codes

        self.cu, self.held, self.max_new = i32(np.concatenate([[0], np.cumsum(new)])), i32(held), max(new)
        self.norm = fs.Norm(None, EPS)
        self.x = torch.randn((sum(new), decoder.hidden), device=dev, generator=g).to(torch.bfloat16)
        self.weights = []
        for _ in range(self.layers):
            self.weights.append((weight((self.hq + 2 * self.hkv) * D, decoder.hidden), weight(decoder.hidden, self.hq * D),
                                 weight(2 * self.ffn, decoder.hidden), weight(decoder.hidden, self.ffn)))
        if decoder.attention == "state":
            # a head keeps half of what it holds for 0.7 to 177 tokens
            self.log_decay = -torch.exp2(torch.linspace(0.0, -8.0, self.hkv, device=dev))
            self.index = torch.arange(len(held), dtype=torch.int32, device=dev)
            self.states = [torch.randn((len(held), self.hkv, D, D), device=dev, generator=g) for _ in range(self.layers)]
            torch.cuda.current_stream(dev).synchronize()
            return
        # each sequence's pages lie side by side in the pool
        pages = [-(-h // PAGE) for h in held]
        first = np.concatenate([[0], np.cumsum(pages)])
        table = np.zeros((len(held), max(pages)), np.int32)
        for s, n in enumerate(pages):
            table[s, :n] = np.arange(first[s], first[s] + n)
        at = np.concatenate([np.arange(h - n, h) for n, h in zip(new, held)])
        self.slots = i32(np.concatenate([first[s] * PAGE + np.arange(h - n, h)
                                         for s, (n, h) in enumerate(zip(new, held))]))
        self.positions, self.table = i32(at), i32(table)
        angle = torch.outer(torch.arange(max(held), device=dev, dtype=torch.float32),
                            10000.0 ** (-torch.arange(0, D, 2, device=dev, dtype=torch.float32) / D))
        self.cos, self.sin = angle.cos().contiguous(), angle.sin().contiguous()
        self.caches = []
        for _ in range(self.layers):
            cache = fs.KVCache.empty(int(first[-1]), self.hkv, D, PAGE, dev)
            for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
                codes.random_(-127, 128, generator=g)
                scale.fill_(1.0 / 73.0)
            self.caches.append(cache)
        torch.cuda.current_stream(dev).synchronize()

    def layer(self, i: int, h, workspace=None):
        """A layer's share of the residual stream h, added to it in place."""
        (qkv, qkv_s), (out, out_s), (up, up_s), (down, down_s) = self.weights[i]
        n, D, hq, hkv = h.shape[0], self.decoder.head_dim, self.hq, self.hkv
        on = dict(stream=self.stream, workspace=workspace)
        rows = fs.project(self.ctx, h, qkv, qkv_s, norm=self.norm, **on).view(n, hq + 2 * hkv, D)
        q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
        if self.decoder.attention == "state":
            seen = fs.state_attention(self.ctx, self.states[i], q, k, v, self.index, self.held, self.cu, self.max_new,
                                      self.log_decay, **on)
        else:
            q = fs.cache_append(self.ctx, self.caches[i], k, v, self.slots, q, self.positions, self.cos, self.sin,
                                stream=self.stream)
            seen = fs.cache_attention(self.ctx, self.caches[i], q, self.table, self.held, self.cu, self.max_new, **on)
        fs.project(self.ctx, seen.view(n, hq * D), out, out_s, residual=h, out=h, **on)
        gated = fs.gated_project(self.ctx, h, up, up_s, norm=self.norm, **on)
        return fs.project(self.ctx, gated, down, down_s, residual=h, out=h, **on)

    def forward(self, workspace=None):
        import torch
        with torch.cuda.stream(self.stream):
            h = self.x.clone()
            for i in range(self.layers):
                self.layer(i, h, workspace)
        return h

    def capture(self):
        """(graph, its output): the layers as one launch."""
        import torch
        self.forward()  # the context's workspace has its size after this
        self.stream.synchronize()
        workspace = self.ctx.workspace(0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=self.stream):
            out = self.forward(workspace)
        self._keep = workspace
        return graph, out

    def seconds(self, times: int = 12):
        """(fast, slow) seconds of a pass over all of the decoder's layers: the
        least and the largest of `times` replays after two."""
        import torch
        graph, _ = self.capture()
        took = []
        with torch.cuda.stream(self.stream):
            for i in range(times + 2):
                a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                a.record()
                graph.replay()
                b.record()
                b.synchronize()
                if i >= 2:
                    took.append(a.elapsed_time(b) * 1e-3)
        scale = self.decoder.layers / self.layers
        return min(took) * scale, max(took) * scale


# --------------------------------------------------------------- the cells --
def sum_seconds(decoder: Decoder, tp: int, tokens: int, link_gbs: float, hop_us: float) -> float:
    """The sums over tp ranks after two projections of every layer, exposed:
    a ring's 2 (tp - 1) / tp of the bytes over one link, and its hops."""
    if tp == 1:
        return 0.0
    one = 2.0 * (tp - 1) / tp * tokens * decoder.hidden * 2.0 / (link_gbs * 1e9) + 2.0 * (tp - 1) * hop_us * 1e-6
    return 2.0 * decoder.layers * one


def settle(load: float, answer: int, prefill: float, steps):
    """(capacity, tail) of a replica that load requests a second reach.

    steps: {batch: seconds of a decode step}.  A batch of n answers a request
    in every prefill + answer * step(n) / n seconds of the replica; the cell
    runs with the smallest batch that serves the load.  A request takes its
    own prefill and answer * step(n), longer by the prefills of those that come
    meanwhile: T = (prefill + answer * step(n)) / (1 - load * prefill)."""
    served = 0.0
    for n in sorted(steps):
        rate = 1.0 / (prefill + answer * steps[n] / n)
        served = max(served, rate)
        if rate >= load:
            return rate, min((prefill + answer * steps[n]) / (1.0 - load * prefill) if load * prefill < 1.0 else UNSERVED,
                             UNSERVED)
    return served, UNSERVED


def settle_between(load: float, answer: int, prefill, steps):
    """((least, largest) capacity, (least, largest) tail) of `settle` over all
    times between (fast, slow): prefill a pair, steps {batch: a pair}.

    Between the two sides the cell may run with any batch from the fast side's to
    the slow side's, or, where the slow side does not serve the load, with none.
    A batch that runs serves the load, so its rate lies between the larger of its
    slow rate and the load, and its fast rate."""
    rate = lambda n, side: 1.0 / (prefill[side] + answer * steps[n][side] / n)  # noqa: E731

    def tail(n, side):
        free = 1.0 - load * prefill[side]
        return min((prefill[side] + answer * steps[n][side]) / free, UNSERVED) if free > 0.0 else UNSERVED
    caps, tails = [], []
    for n in sorted(steps):
        if rate(n, 0) >= load:
            caps += [max(rate(n, 1), load), rate(n, 0)]
            tails += [tail(n, 0), tail(n, 1)]
        if rate(n, 1) >= load:  # no larger batch is needed, whatever the times
            break
    else:  # at the slow times no batch serves the load
        caps += [max(rate(n, 1) for n in steps), min(max(rate(n, 0) for n in steps), load)]
        tails.append(UNSERVED)
    return (min(caps), max(caps)), (min(tails), max(tails))


@dataclass
class Times:
    """Seconds by TP degree and class: prefill (fast, slow), and for every
    batch a decode step (fast, slow)."""
    prefill: dict = field(default_factory=dict)  # (tp, class) -> (fast, slow)
    step: dict = field(default_factory=dict)     # (tp, class) -> {batch: (fast, slow)}


def intervals(problem: Problem, classes, times: Times) -> Intervals:
    """Every cell's intervals, one order, none measured: all that `settle` gives
    for times between the fast and the slow ones.  Capacities lie on the 1/64 grid,
    rounded away from the interval's inside (but to one step of it at least)."""
    N = problem.n_cells
    cap, tail = np.zeros((2, N)), np.zeros((2, N))
    for cell in range(N):
        i, t, b = problem.cell_coords(cell)
        key = (int(problem.tp[t]), classes[i].name)
        cap[:, cell], tail[:, cell] = settle_between(float(problem.levels[b]), classes[i].answer, times.prefill[key],
                                                     times.step[key])
    lo, hi = cap
    lo = np.maximum(np.floor(lo / QUANTUM), 1.0) * QUANTUM
    hi = np.maximum(np.ceil(hi / QUANTUM) * QUANTUM, lo)
    one = lambda x: np.ascontiguousarray(x[None], dtype=np.float32)  # noqa: E731
    return Intervals(one(lo), one(hi), one(tail[0]), one(tail[1]), np.zeros((1, N), np.uint8))


def measure(ctx, decoder: Decoder, tps, batches, classes, layers: int = 8, link_gbs: float = 153.0, hop_us: float = 2.0,
            say=None) -> Times:
    """Runs every (TP, class): decode steps of each batch halfway through the
    answers, and a prompt's prefill."""
    import torch
    say = say or (lambda text: None)
    times = Times()
    stream = torch.cuda.Stream(torch.device("cuda", ctx.device))
    for tp in tps:
        for c in classes:
            fast, slow = Shard(ctx, decoder, tp, [c.prompt], [c.prompt], layers, stream).seconds()
            times.prefill[tp, c.name] = fast, slow + sum_seconds(decoder, tp, c.prompt, link_gbs, hop_us)
            say(f"TP{tp} {c.name}: prefill of {c.prompt} tokens {fast * 1e3:.2f} ms")
            steps = times.step[tp, c.name] = {}
            for n in batches:
                fast, slow = Shard(ctx, decoder, tp, [1] * n, [c.prompt + (c.answer + 1) // 2] * n, layers, stream).seconds()
                steps[n] = fast, slow + sum_seconds(decoder, tp, n, link_gbs, hop_us)
                say(f"TP{tp} {c.name}: step of {n} sequences {fast * 1e3:.3f} ms")
    return times


# ---------------------------------------------------------------- the plan --
def plan(ctx, problem: Problem, iv: Intervals, samples: int = 1024, seed: int = 0) -> dict:
    """What the planner says of the intervals: the certificate, the slow and
    the fast side's allocations, and the cell to measure first."""
    import torch
    dev = torch.device("cuda", ctx.device)
    rng = np.random.default_rng(seed)
    steps = np.rint((iv.cap_hi - iv.cap_lo) / QUANTUM).astype(np.int64)[..., None]
    shape = (1, problem.n_cells, samples)
    cap_s = (iv.cap_lo[..., None] + rng.integers(0, steps + 1, size=shape) * QUANTUM).astype(np.float32)
    lo, hi = iv.tail_lo[..., None], iv.tail_hi[..., None]
    tail_s = np.clip(lo + rng.random(shape) * (hi - lo), lo, hi).astype(np.float32)
    d = fs.DeviceIntervals.from_host(iv, dev)
    put = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dev)  # noqa: E731
    says = fs.certify(ctx, problem, d)
    score = fs.score_candidates(ctx, problem, d, put(np.arange(problem.n_cells, dtype=np.int32)), put(cap_s), put(tail_s))
    best = int(score.best[0])

    def fleet(a):
        picks = zip(a["tp_index"][0].tolist(), a["replicas"][0].tolist())
        return dict(fulfilment=float(a["objective"][0]),
                    classes=[None if t == fs.TP_NONE else dict(tp=int(problem.tp[t]), replicas=r & 0xffff) for t, r in picks])

    return dict(state=("undecided", "feasible", "infeasible")[int(says.state[0])], gap=float(says.gap[0]),
                slow=fleet(says.cons), fast=fleet(says.opt),
                measure_next=None if best < 0 else dict(cell=best, score=float(score.score[0, best])))


def main(argv=None):
    p = argparse.ArgumentParser(prog="python -m paper_2608_19659_amd.probe", description=__doc__.split("\n")[0])
    p.add_argument("--tp", type=int, nargs="+", default=[1, 2, 4, 8], help="TP degrees")
    p.add_argument("--batch", type=int, nargs="+", default=[1, 4, 16, 64], help="sequences of a decode step")
    p.add_argument("--budget", type=int, default=16, help="GPUs of the fleet")
    p.add_argument("--layers", type=int, default=8, help="layers that exist at once")
    p.add_argument("--attention", choices=ATTENTIONS, default="cache", help="what the layers keep of earlier tokens")
    p.add_argument("--link-gbs", type=float, default=153.0, help="GB/s between two GPUs")
    p.add_argument("--hop-us", type=float, default=2.0, help="microseconds of a hop between GPUs")
    p.add_argument("--json", action="store_true", help="print one JSON object")
    o = p.parse_args(argv)
    if min(o.batch) < 1 or max(o.batch) > fs.MAX_SEQUENCES or o.layers < 1 or o.link_gbs <= 0.0 or o.hop_us < 0.0:
        p.error("a batch, the layers and the link's rate must be positive, and a batch at most %d" % fs.MAX_SEQUENCES)
    import torch  # before the library, so that both use one HIP runtime
    decoder, classes = Decoder(attention=o.attention), CLASSES
    tps = sorted(set(o.tp))
    try:
        for tp in tps:
            decoder.check(tp)
        problem = Problem(tp=tps, levels=LEVELS, demand=[c.demand for c in classes], slo=[c.slo for c in classes],
                          budget=o.budget)
        fs.validate_problem(problem)
    except (ValueError, fs.FleetSieveError) as e:
        p.error(str(e))
    if not torch.cuda.is_available():
        p.error("a probe needs a GPU")
    ctx = fs.Context(0)
    say = None if o.json else lambda text: print(text, flush=True)
    times = measure(ctx, decoder, tps, sorted(set(o.batch)), classes, o.layers, o.link_gbs, o.hop_us, say)
    iv = intervals(problem, classes, times)
    says = plan(ctx, problem, iv)
    cells = [dict(zip(("class", "tp", "load"), (classes[i].name, int(problem.tp[t]), float(problem.levels[b]))),
                  capacity=[float(iv.cap_lo[0, n]), float(iv.cap_hi[0, n])],
                  tail=[float(iv.tail_lo[0, n]), float(iv.tail_hi[0, n])])
             for n in range(problem.n_cells) for i, t, b in [problem.cell_coords(n)]]
    if o.json:
        print(json.dumps(dict(cells=cells, plan=says)))
        return 0
    print("class  TP   load req/s   capacity req/s      tail s")
    for c in cells:
        tails = ["never" if x >= UNSERVED else f"{x:.3f}" for x in c["tail"]]
        print(f"{c['class']:5}  {c['tp']:2}   {c['load']:10.2f}   {c['capacity'][0]:7.3f} .. {c['capacity'][1]:7.3f}   {tails[0]} .. {tails[1]}")
    for side in ("slow", "fast"):
        picks = ", ".join(f"{c.name} " + (f"{a['replicas']} x TP{a['tp']}" if a else "unserved")
                          for c, a in zip(classes, says[side]["classes"]))
        print(f"{side} side: least fulfilment {says[side]['fulfilment']:.3f}: {picks}")
    nxt = says["measure_next"]
    if nxt is not None:
        c = cells[nxt["cell"]]
        print(f"gap {says['gap']:.3f}, {says['state']}; measure {c['class']} at TP{c['tp']}, {c['load']} req/s first "
              f"(expected gain {nxt['score']:.4f})")
    else:
        print(f"gap {says['gap']:.3f}, {says['state']}")
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
