"""Plain 64-bit statements, on the CPU, of what a decoder layer does around its
products and of state attention, with bounds of the results' errors."""
import math

import torch

TINY = 2.0 ** -100
STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# half the least spacing, which is 2^-149, 2^-24 and 2^-133: what rounding moves a result below the normal numbers
SMALLEST = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def activate(y, name):
    if name == "none":
        return y
    if name == "relu":
        return torch.where(y < 0, torch.zeros_like(y), y)
    if name == "silu":
        return y / (1.0 + torch.exp(-y))
    if name == "gelu":
        return 0.5 * y * torch.special.erfc(-y * math.sqrt(0.5))
    return y / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))


def codes(x, gain=None, eps=None):
    """(codes, row scales): the codes by their definition's binary32 steps, the
    scale in binary64."""
    v = x.float() if gain is None else x.float() * gain
    a = v.abs().amax(dim=1) if v.shape[1] else torch.zeros(v.shape[0])
    live = ~(a < TINY)
    made = torch.where(live[:, None], torch.round(v * (torch.full_like(a, 127.0) / a)[:, None]), torch.zeros_like(v))
    scale = a.double() / 127.0
    if eps is not None:
        scale = scale / torch.sqrt(x.double().pow(2).mean(dim=1) + float(torch.tensor(eps, dtype=torch.float32))) if x.shape[1] else scale
    return made.double(), torch.where(live, scale, torch.zeros_like(scale))


def projection(x, w, w_scale, gain=None, eps=None, bias=None):
    """(y, what its products alone are): the projection behind the norm."""
    c, s = codes(x, gain, eps)
    y = (c @ w.double().t()) * s[:, None] * w_scale.double()[None]
    return (y if bias is None else y + bias.double()), y


def projection_room(y, product, normed):
    """How far binary32 may be from y: the sum's rounding, two scales and what
    multiplies them, the bias, a step each.  Behind a norm the mean of squares: a
    thread adds up to 80 of a row of 20480 elements at most, wavefronts and blocks
    a dozen sums more, all of one sign, and the factor is its root: 46 steps; with
    the root, the quotients and the product under 64."""
    return product.abs() * ((64 if normed else 0) + 6) * 2.0 ** -24 + y.abs() * 2.0 ** -24


def activation_room(y, name, room):
    """An activation moves by at most 1.13 of its argument's error (the largest
    slope, of gelu; silu's is 1.1), beside what the header allows it itself."""
    own = 0.0 if name in ("none", "relu") else 2.0 ** -20 * (1 + y.abs()) * activate(y, name).abs() + 2.0 ** -22 * y.abs()
    return 1.13 * room + own


def stored_room(want, room, dtype):
    """One rounding to the output's type, of a value that is off by `room`, and of
    the sums before it one step of binary32."""
    return room + (want.abs() + room) * (STEP[dtype] + 2.0 ** -23) + SMALLEST[dtype]


def project(x, w, w_scale, norm=None, bias=None, act="none", residual=None, dtype=torch.float32):
    """(result, bound of the error)."""
    gain, eps = norm if norm else (None, None)
    y, product = projection(x, w, w_scale, gain, eps, bias)
    room = activation_room(y, act, projection_room(y, product, norm is not None))
    want = activate(y, act)
    if residual is not None:
        want = want + residual.double()
        room = room + activate(y, act).abs() * 2.0 ** -24
    return want, stored_room(want, room, dtype)


def gated(x, w, w_scale, norm=None, bias=None, act="silu", dtype=torch.float32):
    gain, eps = norm if norm else (None, None)
    y, product = projection(x, w, w_scale, gain, eps, bias)
    room = projection_room(y, product, norm is not None)
    N = w.shape[0] // 2
    g, u = activate(y[:, :N], act), y[:, N:]
    rg, ru = activation_room(y[:, :N], act, room[:, :N]), room[:, N:]
    want = g * u
    return want, stored_room(want, rg * u.abs() + ru * g.abs() + rg * ru, dtype)


# ------------------------------------------------------------ state attention --
def state_attend(q, k, v, state, log_decay, scale):
    """(outputs, state, bound of the outputs' errors, bound of the state's), token
    by token in binary64.  q [n, heads, D], k, v [n, state heads, D], state
    [state heads, D, D], log_decay [state heads].

    The bounds: every decayed product of a key and a value may enter the state with
    2^-17 of itself lost, as if it were held as two bfloat16 values (2^-9 of the first's
    rounding, 2^-9 of that of the rest, half a step each; the states' precision has a
    test of its own); its decay is 2 to a power
    below 128 where anything is left, which is off by 2^-24 of itself: 2^-17 again;
    and each of up to n additions and decays rounds by 2^-24 of the sum of the terms'
    sizes: as long as that sum's own decay counts fewer than n of them.  An output multiplies that by a query and adds the roundings of the
    state (again 2^-17), of the decayed products of queries and keys (2^-17, and 2^-17
    for their decay), and of its own sum."""
    n, heads, D = q.shape
    H = k.shape[1]
    group = heads // H
    lam = torch.exp(log_decay.double())[:, None, None]
    S, size = state.double().clone(), state.double().abs().clone()
    out = torch.zeros(n, heads, D, dtype=torch.float64)
    most = torch.zeros_like(out)
    for t in range(n):
        kv = k[t].double()[:, :, None] * v[t].double()[:, None, :]
        S, size = lam * S + kv, lam * size + kv.abs()
        x = q[t].double().view(H, group, D)
        out[t] = scale * torch.bmm(x, S).reshape(heads, D)
        most[t] = abs(scale) * torch.bmm(x.abs(), size).reshape(heads, D)
    held = 1.0 / max(1e-9, 1.0 - float(lam.max()))  # tokens that count: the sum of a term's decays
    steps = 2 * 2.0 ** -17 + 2.0 ** -24 * (min(n, held) + D)
    return out, S, most * (steps + 3 * 2.0 ** -17), size * steps


def state_attend_at_once(q, k, v, state, log_decay, scale):
    """The same by its closed form, all tokens at once (n^2 products a head; on the
    inputs' device): o_i = scale (l^(i+1) S^T q_i + sum_(j<=i) l^(i-j) <q_i, k_j> v_j)."""
    n, heads, D = q.shape
    H = k.shape[1]
    t = torch.arange(n, device=q.device, dtype=torch.float64)
    rate = log_decay.double()[:, None, None]
    fade = torch.where(t[:, None] >= t[None], torch.exp(rate * (t[:, None] - t[None]).clamp(min=0)), 0.0)  # [H, n, n]
    since, left = torch.exp(rate * (t[:, None] + 1)), torch.exp(rate * (n - 1 - t)[:, None])  # [H, n, 1]
    end = torch.exp(rate * n)

    def values(q, k, v, S):
        q, k, v = (x.transpose(0, 1).contiguous() for x in (q, k, v))  # [heads, n, D]
        q = q.view(H, heads // H, n, D)
        out = (q @ k.transpose(1, 2)[:, None] * fade[:, None]) @ v[:, None] + since[:, None] * (q @ S[:, None])
        return out.reshape(heads, n, D).transpose(0, 1), end * S + (k * left).transpose(1, 2) @ v
    out, S = values(q.double(), k.double(), v.double(), state.double())
    most, size = values(q.double().abs(), k.double().abs(), v.double().abs(), state.double().abs())
    held = 1.0 / max(1e-9, 1.0 - float(torch.exp(rate).max()))
    steps = 2 * 2.0 ** -17 + 2.0 ** -24 * (min(n, held) + D)
    return out * scale, S, most * abs(scale) * (steps + 3 * 2.0 ** -17), size * steps


def state_norm(n, rate):
    """How far the state after n tokens of random keys and values may be from the
    formula's, relative to its norm, where all that is off is off either way: a term's
    value as parts by 2^-22 of itself at most and its decay as much, 2^-22 / sqrt(3) each
    in the root mean square; and the terms that count, 1 / (1 - l) of them, are added to
    a sum of about the state's size, 2^-23 / sqrt(3) each (2^-24 if the matrix units
    round what they add, twice that if they cut it)."""
    terms = min(n, 1.0 / -math.expm1(rate))
    return math.sqrt((2 * 16 + 4 * terms) / 3.0) * 2.0 ** -24


def in_parts(x, dtype, count):
    """x (binary32) as the sum of `count` values of a 16-bit type, each the rest's
    nearest; for binary16 behind a power of two that brings the largest of a column
    (along dim 0) to 2^14."""
    factor = torch.ones_like(x[:1])
    if dtype is torch.float16:
        factor = torch.exp2(14.0 - torch.floor(torch.log2(x.abs().amax(dim=0, keepdim=True).clamp(min=2.0 ** -100))))
    rest, total = x * factor, torch.zeros_like(x)
    for _ in range(count):
        part = rest.to(dtype).float()
        rest, total = rest - part, total + part
    return total / factor
