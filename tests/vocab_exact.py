"""The softmax losses over a vocabulary from their definition in 64 bits, with bounds on the fp32 kernels' errors.

Bounds, per row i and answer v (u = 2^-24, a rounding of fp32; h = half a step of the 16-bit type, relative):
  logits     a sum of k products and the bias, in any order, an addition off by up to 2u:
             ez = (k + 2) 2u (sum |x w| + |b|)
  exponents  formed as (z log2(e) / T) - (lse log2(e)) with one rounding, of two rounded constants and a rounded
             lse log2(e); the hardware's 2^x is good to 2 ulp:  ep = ez / T + else + 8u (|z / T| + |lse| + 2), relative
  lse        every term's ep (with the maximum in lse's place), V additions of positive terms, a logarithm:
             else = max ez / T + 8u (2 max |z / T| + 2) + V u (at most 64 terms are added up one after another, the
             rest in trees: 2^8 u is plenty) + 8u |lse|
  dz         g T (p (1 + ep) - q (1 + 16u)), rounded to 16 bits: h |dz| + |g T| (p ep + 16u q)
  products   dX and dW add up V or n terms of dz: their errors' sum, (terms) 2u of the sum of magnitudes, and the
             output's own rounding
"""
import torch

U = 2.0 ** -24


def half(dtype):
    return torch.finfo(dtype).eps / 2


def logits(X, W, bias):
    """Logits of CPU tensors and their bound."""
    Xd, Wd = X.double(), W.double()
    z, mag = Xd @ Wd.t(), Xd.abs() @ Wd.abs().t()
    if bias is not None:
        z = z + bias.double()
        mag = mag + torch.where(torch.isfinite(bias), bias.double().abs(), 0.0)
    return z, (X.shape[1] + 2) * 2 * U * mag


def teacher_share(index, teacher, V, T):
    """q of every entry, and the rows that count."""
    held = (index >= 0) & (index < V)
    t = (teacher.double() / T).masked_fill(~held, -torch.inf)
    live = (held & ~(t == -torch.inf)).any(1)
    q = torch.zeros_like(t)
    q[live] = torch.softmax(t[live], 1)
    return q, held, live


def loss(X, W, index, q, held, live, bias=None, T=1.0):
    """(loss, lse, logp) for targets with shares q (cross entropy: one entry of share 1), and a bound of each."""
    z, ez = logits(X, W, bias)
    z, ez = z / T, ez / T
    lse = torch.logsumexp(z, 1)
    fin = torch.where(torch.isfinite(z), z.abs(), 0.0)
    top = fin.max(1)[0]
    else_ = ez.max(1)[0] + 8 * U * (2 * top + 2) + 2 ** 8 * U + 8 * U * lse.abs()
    at = index.clamp(0, W.shape[0] - 1).long()
    logp = torch.where(held & live[:, None], z.gather(1, at) - lse[:, None], 0.0)
    elogp = ez.gather(1, at) + else_[:, None] + 4 * U * (fin.gather(1, at) + lse.abs()[:, None])
    ent = torch.special.entr(q).sum(1)
    logq = torch.where(q > 0, q, 1.0).log()
    eq = 16 * U * (1 + logq.abs())         # of log q: a difference of rounded logits, an expf and a logf
    value = T * T * (-(torch.where(q > 0, q * logp, 0.0)).sum(1) - ent)
    eloss = T * T * ((q * (elogp + eq + eq * (logq.abs() + logp.abs()))).sum(1) + 8 * U * (q * (logq.abs() + logp.abs())).sum(1)) + 4 * U * value.abs()
    zero = torch.zeros_like(lse)
    return {"loss": (torch.where(live, value, zero), torch.where(live, eloss, zero)),
            "lse": (torch.where(live, lse, zero), torch.where(live, else_, zero)),
            "logp": (logp, torch.where(held & live[:, None], elogp, 0.0)), "z": z, "ez": ez, "else": else_}


def gradients(X, W, index, q, held, live, g, bias=None, T=1.0):
    """dX, dW, db and a bound of each."""
    f = loss(X, W, index, q, held, live, bias, T)
    z, lse = f["z"], f["lse"][0]
    p = torch.exp(z - torch.where(live, lse, 0.0)[:, None])
    ep = f["ez"] + f["else"][:, None] + 8 * U * (torch.where(torch.isfinite(z), z.abs(), 0.0) + lse.abs()[:, None] + 2)
    want = torch.zeros_like(p)
    want.scatter_add_(1, index.clamp(0, W.shape[0] - 1).long(), q)
    gt = torch.where(live, g.double() * T, 0.0)[:, None]
    # (a row that is left out has no part, whatever it holds)
    dz = torch.where(live[:, None], gt * (p - want), 0.0)
    e32 = torch.where(live[:, None], gt.abs() * (p * ep + 64 * U * want), 0.0)
    h, tiny = half(X.dtype), 2.0 ** -24 if X.dtype == torch.float16 else 0.0
    top = gt.abs().max()
    e16 = e32 + h * (dz.abs() + e32) + tiny * 2.0 ** -14 * top      # (scaled: |g T| up to 2^14 or more)
    Xl = torch.where(live[:, None], X.double(), 0.0)
    Wd = W.double()
    n, V = p.shape
    out = {}
    for name, a, b, terms in (("dX", dz, Wd, V), ("dW", dz.t(), Xl, n)):
        e = e16 if name == "dX" else e16.t()
        value = a @ b
        err = e @ b.abs() + (terms + 40) * 2 * U * (a.abs() @ b.abs())
        out[name] = (value, err + h * (value.abs() + err) + tiny)
    db = dz.sum(0)
    out["db"] = (db, e32.sum(0) + (n + 8) * 2 * U * ((p * gt.abs()).nan_to_num().sum(0) + (want * gt.abs()).sum(0)) + 2 * U * db.abs() + n * 2.0 ** -40 * top)
    return out


def close(name, got, value, bound):
    d = (got.double().to(value.device) - value).abs()
    bad = ~(d <= bound)
    assert not bad.any(), (f"{name}: {int(bad.sum())} of {bad.numel()} past the bound, the worst "
                           f"{float((d / bound.clamp(min=1e-300)).max()):.3g} times, off by {float(d.max()):.3g}")
