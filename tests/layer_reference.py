"""Plain 64-bit forms of the layer operators for the tests, one sequence and one head at a time, with the sums of absolute values from
which the tests derive their tolerances.  Shares nothing with the library."""
import math

import torch

U32 = 2.0 ** -24          # unit roundoff of fp32
U16 = 2.0 ** -8           # unit roundoff of bf16: 8 significant bits, so half an ulp is up to 2^-8 of the value


def unit(dtype):
    return U16 if dtype == torch.bfloat16 else U32


def norm(x, w, b, eps, center):
    x = x.double()
    mu = x.mean(-1, keepdim=True) if center else torch.zeros_like(x[..., :1])
    c = x - mu
    rstd = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
    y = c * rstd
    if w is not None:
        y = y * w.double()
    if b is not None:
        y = y + b.double()
    return y, mu[..., 0], rstd[..., 0]


def turn(x, inv_freq, pos, layout, amplitude, inverse):
    """x [b, n, h, d], pos [b, n] (int64 or double)."""
    x = x.double()
    f = torch.as_tensor(inv_freq, dtype=torch.float64, device=x.device)
    n = f.numel()
    ang = pos.double()[..., None, None] * f * (-1 if inverse else 1)
    c, s = torch.cos(ang) * amplitude, torch.sin(ang) * amplitude
    y = x.clone()
    ia = torch.arange(n, device=x.device) if layout == "half" else 2 * torch.arange(n, device=x.device)
    ib = ia + n if layout == "half" else ia + 1
    y[..., ia], y[..., ib] = x[..., ia] * c - x[..., ib] * s, x[..., ia] * s + x[..., ib] * c
    return y


def sequences(q, k, q_lens=None, k_lens=None, q_offsets=None, k_offsets=None):
    """[(index of the queries, index of the keys)] into [b, n, ...] tensors; packed tensors have b = 1."""
    if q_offsets is not None:
        qo, ko = q_offsets.tolist(), k_offsets.tolist()
        return [((0, slice(qo[i], qo[i + 1])), (0, slice(ko[i], ko[i + 1]))) for i in range(len(qo) - 1)]
    b = q.shape[0]
    ql = [q.shape[1]] * b if q_lens is None else q_lens.tolist()
    kl = [k.shape[1]] * b if k_lens is None else k_lens.tolist()
    return [((i, slice(0, ql[i])), (i, slice(0, kl[i]))) for i in range(b)]


def seen(nq, nk, causal, window, device):
    i, j = torch.arange(nq, device=device)[:, None] + nk - nq, torch.arange(nk, device=device)[None]
    m = torch.ones((nq, nk), dtype=torch.bool, device=device)
    if causal:
        m &= j <= i
    if window:
        m &= j > i - window
    return m


def attention(q, k, v, causal=True, window=0, scale=None, do=None, o=None, lse=None, **lens):
    """q [b, n, h, d], k, v [b, m, g, d].  Forward: {o, lse, o_abs}.  With do, o, lse: the gradients as functions of these, too, each
    with the sum of absolute values (x_abs) of its last product and, for dq and dk, the same sum before dS is cancelled (x_pre)."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    z = lambda t: torch.zeros(t.shape, dtype=torch.float64, device=t.device)  # noqa: E731
    r = {"o": z(q), "o_abs": z(q), "lse": torch.full((q.shape[0], q.shape[2], q.shape[1]), -math.inf, dtype=torch.float64, device=q.device)}
    for name in ("dq", "dq_abs", "dq_pre"):
        r[name] = z(q)
    for name in ("dk", "dk_abs", "dk_pre", "dv", "dv_abs"):
        r[name] = z(k)
    group = q.shape[2] // k.shape[2]
    for (qb, qs), (kb, ks) in sequences(q, k, **lens):
        for h in range(q.shape[2]):
            g = h // group
            qi, ki, vi = q[qb, qs, h].double(), k[kb, ks, g].double(), v[kb, ks, g].double()
            if qi.shape[0] == 0:
                continue
            m = seen(qi.shape[0], ki.shape[0], causal, window, q.device)
            s = torch.where(m, qi @ ki.T * scale, -math.inf)
            e = torch.logsumexp(s, 1) if ki.shape[0] else torch.full((qi.shape[0],), -math.inf, dtype=torch.float64, device=q.device)
            live = e > -math.inf
            p = torch.where(m & live[:, None], torch.exp(s - torch.where(live, e, 0.0)[:, None]), 0.0)
            r["o"][qb, qs, h], r["o_abs"][qb, qs, h], r["lse"][qb, h, qs] = p @ vi, p @ vi.abs(), e
            if do is None:
                continue
            if lse is not None:
                given = lse[qb, h, qs].double()
                p = torch.where(m & live[:, None], torch.exp(s - torch.where(live, given, 0.0)[:, None]), 0.0)
            gi, oi = do[qb, qs, h].double(), (r["o"] if o is None else o)[qb, qs, h].double()
            gi, oi = torch.where(live[:, None], gi, 0.0), torch.where(live[:, None], oi, 0.0)
            delta = (gi * oi).sum(1, keepdim=True)
            ds = p * (gi @ vi.T - delta)
            pre = p * (gi.abs() @ vi.abs().T + (gi * oi).abs().sum(1, keepdim=True))
            r["dv"][kb, ks, g] += p.T @ gi
            r["dv_abs"][kb, ks, g] += p.T @ gi.abs()
            for name, t in (("", ds), ("_abs", ds.abs()), ("_pre", pre)):
                a = (lambda x: x) if not name else torch.abs
                r["dq" + name][qb, qs, h] = t @ a(ki) * scale
                r["dk" + name][kb, ks, g] += t.T @ a(torch.where(live[:, None], qi, 0.0)) * scale
    return r


def norm_of(x, w, b, eps):
    """Differentiable layer norm in the precision of x."""
    c = x - x.mean(-1, keepdim=True)
    return c / torch.sqrt((c * c).mean(-1, keepdim=True) + eps) * w + b
