"""Plain 64-bit forms of decayed linear attention and the grouped norm, token by token, and
the tolerances of their tests.

Tolerances (u = 2^-24). Beside each value the reference carries the same sum over absolute
values: S_abs = sum w |k| |v|, y_abs = sum |q| S_abs, which bounds how far any order of
summation can be off per rounding.
 * states: 64 u S_abs per element. A state element of up to 1000 tokens takes two roundings
   a token, of random sign: sqrt(2000) u, or, summed over chunks, fewer.
 * readouts in fp32: 64 u y_abs (the state's error and a sum of 128 terms: about 50 u).
 * readouts in 16 bits: 2^-15 y_abs, a 16-bit split of one factor of each product
   (2^-17 each for the state and the scores, signs open), plus half a unit of the type.
 * normalised readouts: the error of y, e, moves a head's output by at most
   r |w| (e + max_e) (the mean and the root move by no more than the largest e), times |act(z)|,
   plus 2^-20 of the output for the activation, plus half a unit of the type.
"""
import torch

D = 128
U = 2.0 ** -24
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}    # half the subnormal step


def linattn(S, q, k, v, g):
    """S [Hv][128][128] in place, q, k [T][Hk][128], v [T][Hv][128], g [T][Hv] (any types).
    Returns y, y_abs [T][Hv][128] and S_abs, in 64 bits."""
    T, Hv = v.shape[0], v.shape[1]
    grp = Hv // q.shape[1]
    q, k = (x.double().repeat_interleave(grp, 1) for x in (q, k))
    v, g = v.double(), g.double().expand(T, Hv)
    A = S.abs()
    y, ya = torch.empty_like(v), torch.empty_like(v)
    for t in range(T):
        gt = g[t][:, None, None]
        S.copy_(gt * S + k[t][:, :, None] * v[t][:, None, :])
        A = gt * A + k[t].abs()[:, :, None] * v[t].abs()[:, None, :]
        y[t] = (S * q[t][:, :, None]).sum(1)
        ya[t] = (A * q[t].abs()[:, :, None]).sum(1)
    return y, ya, A


def act(x, kind):
    return x * torch.sigmoid(x) if kind == 1 else torch.sigmoid(x) if kind == 2 else x


def norm(x, groups, w=None, b=None, z=None, kind=1, center=True, shared=False, eps=1e-5):
    """x [..., groups * n] in 64 bits -> (out, r |w| |act(z)| per element, out with |.| of its parts)."""
    n = x.shape[-1] // groups
    by = lambda t: t.double().unflatten(-1, (groups, n))  # noqa: E731
    p = lambda t, d: torch.full((1, n), d, dtype=torch.float64, device=x.device) if t is None else \
        (t.double()[None] if shared else by(t))  # noqa: E731
    xg = by(x)
    m = xg.mean(-1, keepdim=True) if center else torch.zeros_like(xg[..., :1])
    r = 1 / torch.sqrt(((xg - m) ** 2).mean(-1, keepdim=True) + eps)
    uw = (xg - m) * r * p(w, 1.0)
    u = uw + p(b, 0.0)
    if z is None:
        out, slope = act(u, kind), 1.1 * torch.ones_like(u)          # |silu'|, |sigmoid'| <= 1.1
    else:
        out, slope = u * act(by(z), kind), act(by(z), kind).abs()
    gain = r * p(w, 1.0).abs() * slope
    part = (uw.abs() + p(b, 0.0).abs()) * slope
    return out.flatten(-2), gain.flatten(-2), part.flatten(-2)


def y_bound(y, ya, dtype):
    return (64 * U if dtype is torch.float32 else 2.0 ** -15) * ya


def rounded(tol, out, dtype):
    """tol plus what rounding a value within tol of `out` to the type adds."""
    return tol + HALF_UNIT[dtype] * (out.abs() + tol) + TINY[dtype]


def norm_bound(e, gain, part, groups):
    worst = e.unflatten(-1, (groups, -1)).amax(-1, keepdim=True).expand(*e.shape[:-1], groups, e.shape[-1] // groups)
    return gain * (e + 2 * worst.flatten(-2)) + 2.0 ** -20 * part


def assert_within(got, want, tol, what):
    d = (got.double() - want).abs()
    over = d > tol
    if bool(over.any()) or bool(torch.isnan(d).any()):
        i = int(torch.where(torch.isnan(d), torch.inf, d / tol.clamp_min(1e-300)).flatten().argmax())
        raise AssertionError(f"{what}: {int(over.sum())} of {d.numel()} outside, {int(torch.isnan(d).sum())} NaN; worst at {i}: "
                             f"{got.flatten()[i].item()} for {want.flatten()[i].item()}, allowed {tol.flatten()[i].item()}")
