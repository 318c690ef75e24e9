"""Plain 64-bit forms of the layer operators, on the CPU, and how far a result may be from them.

The bounds are worked out from the arithmetic, not fitted.  u is half a unit in the last place of the arrays' type:
an output is rounded once, |error| <= u |value|; probabilities and score gradients are rounded once more before the
product they enter, which adds u times the product of absolute values.  Everything else happens in 32 bits: a sum of n
products is off by at most (n + 2) 2^-24 times the sum of absolute values, and a probability 2^(c x - l) by its
exponent's error, 2^-22 (|c x| + |l| + 2) relative, with scores |x| of at most `big` and their own products' error.
SLACK below is that 32-bit part, 2^-13, for the sizes tested here (big < 100, n < 2048); it is two hundredths of u for
bfloat16 and a quarter of it for float16.
"""
import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}   # half the least step
SLACK = 2.0 ** -13


def f64(t):
    return t.detach().cpu().double()


def sees(Lq, Lk, causal, nq, nk):
    i, j = torch.arange(Lq).view(-1, 1), torch.arange(Lk).view(1, -1)
    m = (i < nq) & (j < nk)
    return m & (j <= i + nk - nq) if causal else m


def attention(q, k, v, causal=False, scale=None, len_q=None, len_k=None, dout=None, out_given=None):
    """name -> (value, bound) in 64 bits.  out_given: the rounded outputs that the backward pass is given."""
    dtype = q.dtype
    u, tiny = U[dtype], TINY[dtype]
    q, k, v = f64(q), f64(k), f64(v)
    B, Lq, Hq, D = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    z = lambda *s: torch.zeros(*s, dtype=torch.float64)
    res = {n: [z(B, Lq, Hq, D), z(B, Lq, Hq, D)] for n in ("out", "dq")}
    res.update({n: [z(B, Lk, Hk, D), z(B, Lk, Hk, D)] for n in ("dk", "dv")})
    res["lse"] = [torch.full((B, Hq, Lq), -np.inf, dtype=torch.float64), z(B, Hq, Lq)]
    for b in range(B):
        nq = Lq if len_q is None else min(max(int(len_q[b]), 0), Lq)
        nk = Lk if len_k is None else min(max(int(len_k[b]), 0), Lk)
        m = sees(Lq, Lk, causal, nq, nk)[:nq, :nk]
        for h in range(Hq):
            g = h * Hk // Hq
            qq, kk, vv = q[b, :nq, h], k[b, :nk, g], v[b, :nk, g]      # what lies beyond the lengths is not looked at
            x = torch.where(m, scale * (qq @ kk.T), -torch.inf)
            any_ = m.any(1)
            lse = torch.where(any_, torch.logsumexp(torch.where(any_[:, None], x, 0.0), 1) if nk else 0.0, -torch.inf)
            p = torch.where(m, torch.exp(x - torch.where(any_, lse, 0.0)[:, None]), 0.0)
            o = p @ vv
            res["out"][0][b, :nq, h], res["lse"][0][b, h, :nq] = o, lse
            res["out"][1][b, :nq, h] = (u + SLACK) * (p @ vv.abs() + o.abs()) + tiny * (1 + vv.abs().sum(0))
            res["lse"][1][b, h, :nq] = 2.0 ** -18 * (1 + torch.where(any_, lse.abs(), 0.0))
            if dout is None:
                continue
            do, og = f64(dout)[b, :nq, h], o if out_given is None else f64(out_given)[b, :nq, h]
            delta = (do * o).sum(1, keepdim=True)
            ds = p * (do @ vv.T - delta)
            # the given outputs' rounding goes into delta; the products' in 32 bits into both terms
            off = p * (SLACK * (do.abs() @ vv.abs().T + (do.abs() * og.abs()).sum(1, keepdim=True)) +
                       (do * (og - o)).sum(1, keepdim=True).abs())
            e = (u + SLACK) * ds.abs() + off + tiny
            e = torch.where(m, e, 0.0)
            res["dq"][0][b, :nq, h] = scale * (ds @ kk)
            res["dq"][1][b, :nq, h] = scale * (e @ kk.abs()) + (u + SLACK) * scale * (ds @ kk).abs() + tiny
            res["dk"][0][b, :nk, g] += scale * (ds.T @ qq)
            res["dk"][1][b, :nk, g] += scale * (e.T @ qq.abs())
            res["dv"][0][b, :nk, g] += p.T @ do
            res["dv"][1][b, :nk, g] += ((u + SLACK) * p + torch.where(m, tiny, 0.0)).T @ do.abs()
    for n in ("dk", "dv"):
        res[n][1] += (u + SLACK) * res[n][0].abs() + tiny
    return res


def layer_norm(x, w, b, eps, dy=None):
    """name -> value in 64 bits."""
    x, w, b = f64(x), None if w is None else f64(w), None if b is None else f64(b)
    mean = x.mean(-1)
    var = ((x - mean[..., None]) ** 2).mean(-1)
    rstd = 1.0 / torch.sqrt(var + eps)
    xhat = (x - mean[..., None]) * rstd[..., None]
    y = xhat if w is None else xhat * w
    res = dict(y=y if b is None else y + b, mean=mean, rstd=rstd, xhat=xhat)
    if dy is not None:
        dy = f64(dy)
        g = dy if w is None else dy * w
        dx = (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True)) * rstd[..., None]
        axes = tuple(range(x.dim() - 1))
        res.update(dx=dx, dweight=(dy * xhat).sum(axes), dbias=dy.sum(axes))
    return res


def assert_close(name, got, want, bound):
    got = f64(got)
    same_inf = torch.isinf(want) & (got == want)
    bad = ~(((got - want).abs() <= bound) | same_inf)
    if bad.any():
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} values off, first at {at}: {got[at].item()} for "
                             f"{want[at].item()}, {bound[at].item()} allowed")
