"""Plain 64-bit forms of the dense operators (8-bit rows and products, the gated
feed-forward block and its gradients) and the error bounds their kernels keep.

Bounds are per element and follow the arithmetic: an output rounded to type t is off by at
most eps(t) / 2 of its value; a sum of products c_j in fp32 by GAMMA(depth) * sum |c_j| (every
addition and product rounded, a factor two for the order and the last place of the matrix
cores' internal sums); an activation or its derivative in fp32 by ACT_ERR times its scale
(the exponential's argument reaches 88 and is off by 2^-23 of it at most twice, its value
by 2^-22, some operations of 2^-24 each: below 2^-18)."""
import math

import numpy as np
import torch

ACT_ERR = 2.0 ** -18
INT8_MAX_K = 131071


def gamma(depth):
    return (depth + 8) * 2.0 ** -23


def half(t):
    return torch.finfo(t).eps / 2


def floor(t):
    """Half the smallest subnormal: the absolute error of rounding next to zero."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def quantize_ref(x):
    """Codes (int64) and fp32 scales of the rows of x, by the definition."""
    x = x.double()
    s = (x.abs().amax(1).float() * torch.tensor(1 / 127, dtype=torch.float32)).clamp_min(2.0 ** -126)
    ok = torch.isfinite(x).all(1)
    t = x / s.double()[:, None]
    q = torch.where(ok[:, None], torch.round(t), torch.zeros_like(t))   # ties to even
    return q.long(), torch.where(ok, s, torch.full_like(s, math.nan))


def act_ref(g, act):
    """act(g), act'(g) in 64 bits."""
    if act == 0:
        a, da = g, torch.ones_like(g)
    else:
        c = 2.0 * math.sqrt(2.0 / math.pi)
        a, da = c * (g + 0.044715 * g ** 3), c * (1 + 3 * 0.044715 * g ** 2)
    s = torch.sigmoid(a)
    return g * s, s + g * s * torch.sigmoid(-a) * da


def int8_ref(q, sx, wq, sw):
    return (q.double() @ wq.double().t()) * sx.double()[:, None] * sw.double()[None, :]


def gated_ref(x, wg, wu, act):
    """h and the bound of its error before the final rounding."""
    x, wg, wu = x.double(), wg.double(), wu.double()
    g, u = x @ wg.t(), x @ wu.t()
    gm = gamma(x.shape[1])
    return g, u, gm * (x.abs() @ wg.abs().t()), gm * (x.abs() @ wu.abs().t())


def gated_bound(g, u, eg, eu, act, t):
    """h, and how far it may be off when g and u are off by eg and eu: |act'| < 1.2."""
    a, _ = act_ref(g, act)
    h = a * u
    err = 1.2 * eg * (u.abs() + eu) + a.abs() * eu + ACT_ERR * g.abs() * u.abs()
    return h, err + half(t) * (h.abs() + err) + floor(t)


def backward_ref(dh, x, wg, wu, g, u, act, t, base=None):
    """(dx, dgate, dup), each with its bound; g and u are the rounded ones."""
    dh, x, wg, wu, g, u = (v.double() for v in (dh, x, wg, wu, g, u))
    a, da = act_ref(g, act)
    dg, du = dh * u * da, dh * a
    edg = half(t) * dg.abs() * 1.01 + ACT_ERR * 4 * (dh * u).abs() + floor(t)
    edu = half(t) * du.abs() * 1.01 + ACT_ERR * (dh * g).abs() + floor(t)
    adg, adu = dg.abs() + edg, du.abs() + edu

    def out(v, err, old):
        if old is not None:
            v = v + old.double()
        return v, err + half(t) * (v.abs() + err) + floor(t) + 2.0 ** -23 * v.abs()

    dx = dg @ wg + du @ wu
    edx = edg @ wg.abs() + edu @ wu.abs() + gamma(2 * wg.shape[0]) * (adg @ wg.abs() + adu @ wu.abs())
    gm = gamma(x.shape[0])
    edwg = edg.t() @ x.abs() + gm * (adg.t() @ x.abs())
    edwu = edu.t() @ x.abs() + gm * (adu.t() @ x.abs())
    old = (None, None) if base is None else base
    return out(dx, edx, None), out(dg.t() @ x, edwg, old[0]), out(du.t() @ x, edwu, old[1])


def assert_close(y, ref, bound, what=""):
    y = y.detach().cpu().double()
    bad = ~((y - ref).abs() <= bound)
    if bool(bad.any()):
        i = tuple(int(v) for v in torch.nonzero(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: "
                             f"{float(y[i])} against {float(ref[i])} +- {float(bound[i])}")


def rand(seed, *shape, scale=1.0):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape) * scale)
