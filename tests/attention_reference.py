"""The attention operators in 64 bits on the CPU, from their definitions, with what each result may be off by.

Rounding a value v to a type is off by |v| eps / 2 at most (eps: the type's step relative to the value), fp32's half step is U.
The bounds beside the functions count the roundings of a computation in fp32; none is fitted to a measurement."""
import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """Half a step of the smallest values."""
    return {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}[dtype]


def norm(kind, x, w, b, eps):
    """(result, what its fp32 computation is off by): the sum over a head goes over 8 values and then a tree of up to five steps, each of a
    relative U; with mean, difference, quotient, root and two products under 32 U of what they work on."""
    if kind == "none":
        return x, torch.zeros_like(x)
    mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[..., :1])
    c = x - mean
    r = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
    w = torch.ones(x.shape[-1], dtype=torch.float64) if w is None else w
    y = c * r * w
    off = (x.abs() + x.abs().mean(-1, keepdim=True)) * r * w.abs()
    if kind == "layer" and b is not None:
        y = y + b
        off = off + b.abs()
    return y, 32 * U * off


def rotate(x, off, position, freq, rotary, pairs):
    """x [T][heads][D]; the angle is good to 2^-40 turns, sine and cosine to 4 U, the two products and their sum to 3 U."""
    if not rotary:
        return x, off
    half = rotary // 2
    a = position.double()[:, None] * freq.double()[None]
    cos, sin = a.cos()[:, None], a.sin()[:, None]
    first = slice(0, half) if pairs == "halves" else slice(0, rotary, 2)
    second = slice(half, rotary) if pairs == "halves" else slice(1, rotary, 2)
    y, z = x.clone(), off.clone()
    y[..., first] = x[..., first] * cos - x[..., second] * sin
    y[..., second] = x[..., second] * cos + x[..., first] * sin
    both = off[..., first] + off[..., second] + 8 * U * (x[..., first].abs() + x[..., second].abs())
    z[..., first] = z[..., second] = both
    return y, z


def codes_bound(v, off):
    """What scale * code may be off by: half a step of e4m3 (2^-4 of a normal value, 2^-10 of the scale below), and what v was."""
    scale = (v.abs().amax(-1, keepdim=True) + off.amax(-1, keepdim=True)) / 448
    return torch.maximum(v.abs() * 2.0 ** -4, scale * 2.0 ** -10) * (1 + 2.0 ** -20) + 2 * off


def attention(q, k, v, scale, seen, dtype, coarse):
    """One head: q [Lq][D], k, v [Lk][D] in 64 bits, seen [Lq][Lk].  (result, bound).
    A score is off by its sum's roundings, (D + 4) U of the sum of its products' magnitudes; a probability by twice that (its own and its
    row's largest, as parts of the value), 4 U for the exponential and its argument's rounding; the sums over n keys by a chain of n / 32
    additions and 64 more; two-part probabilities by 2^-18, coarse ones by a rounding to dtype; the output by a rounding to dtype."""
    if k.shape[0] == 0:
        o = torch.zeros(q.shape[0], v.shape[1], dtype=torch.float64)
        return o, o
    hidden = ~seen
    s = (q @ k.t() * scale).masked_fill(hidden, -float("inf"))
    size = (q.abs() @ k.abs().t() * abs(scale)).masked_fill(hidden, 0.0).nan_to_num(0.0, 0.0, 0.0).amax(-1, keepdim=True)
    empty = hidden.all(-1, keepdim=True)
    p = torch.softmax(s, -1).masked_fill(hidden, 0.0)
    # (0 for a key that is not seen, whatever its value is)
    terms = torch.where(hidden[..., None], 0.0, p[..., None] * v[None])
    o = torch.where(empty, 0.0, terms.sum(1))
    a = torch.where(empty, 0.0, terms.abs().sum(1))
    n = k.shape[0]
    rel = 2 * (q.shape[1] + 4) * U * size + (4 + 2 * size) * U + (n / 32 + 64) * U + (half_step(dtype) if coarse else 2.0 ** -18)
    return o, o.abs() * half_step(dtype) * (1 + 2 ** -8) + a * 2 * rel + tiny(dtype) + a * tiny(dtype)


def check(got, want, bound, what=""):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), finite), f"{what}: other places are finite"
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: other places are NaN"
    assert torch.equal(got[~finite & ~torch.isnan(want)], want[~finite & ~torch.isnan(want)]), f"{what}: other infinities"
    off = (got - want).abs()[finite]
    worst = (off / bound[finite].clamp(min=1e-300)).max().item() if off.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} of what it may be off by"
