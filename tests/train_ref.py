"""What the calls that train the routing compute, in 64 bits from their formulas, with the error that fp32 arithmetic may add.

U is half a step of fp32 relative to a value (2^-24); half(t) that of a storage type.  A sum of n fp32 terms in any order is
off by at most n U times the sum of their magnitudes.  Matrix instructions may cut instead of rounding: twice that."""
import torch

U = 2.0 ** -24
IO = {"f32": torch.float32, "bf16": torch.bfloat16}


def half(t):
    return torch.finfo(t).eps / 2


def d(t):
    return None if t is None else t.detach().double().cpu()


def within(got, want, bound, what):
    """every element of got within bound of want; equal where want is no number"""
    got = d(got)
    assert got.shape == want.shape, what
    off = (got - want).abs()
    fine = (off <= bound + 2.0 ** -120)                       # results near the end of fp32's range may be flushed to zero | (got == want) | (got.isnan() & want.isnan())
    if not fine.all():
        i = (~fine).nonzero()[0].tolist()
        raise AssertionError("%s: %d of %d elements off, the first at %s: %r for %r, bound %r" % (
            what, int((~fine).sum()), got.numel(), i, float(got[tuple(i)]), float(want[tuple(i)]), float(bound.expand_as(off)[tuple(i)])))


# ---- layer norm ---------------------------------------------------------------------------
# A row of D elements is summed in at most LANE elements to a lane, then over 64 lanes and 16 waves: at most 64 terms deep.
DEEP = 64


def norm(x, gamma, beta, eps, residual=None):
    """(u, r, mean, rstd) and the bounds on u, mean, rstd, before u is rounded"""
    r = d(x) if residual is None else (d(x) + d(residual)).to(residual.dtype).double()
    D = r.shape[-1]
    g = torch.ones(D, dtype=torch.float64) if gamma is None else d(gamma)
    b = torch.zeros(D, dtype=torch.float64) if beta is None else d(beta)
    m = r.mean(-1, keepdim=True)
    s = ((r - m).square().mean(-1, keepdim=True) + eps).rsqrt()
    xh = (r - m) * s
    u = xh * g + b
    top = r.abs().amax(-1, keepdim=True)
    dm = DEEP * U * top                                       # of the mean
    ds = (DEEP / 2 + 8) * U + 0.5 * (s * (dm + U * top)) ** 2       # of rstd, relative: its sum and what the mean's error adds
    du = g.abs() * (s * (dm + U * top) + (ds + 4 * U) * xh.abs()) + 4 * U * (g * xh).abs() + 4 * U * b.abs()
    return (u, r, m[..., 0], s[..., 0]), (du, dm[..., 0], (ds * s)[..., 0])


def norm_bwd(du, r, gamma, mean, rstd, d_sum=None):
    """(dx, dgamma, dbeta) and their bounds, before dx is rounded"""
    du, r, m, s = d(du), d(r), d(mean)[..., None], d(rstd)[..., None]
    g = du if gamma is None else du * d(gamma)
    xh = (r - m) * s
    mg, mx = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    dx = s * (g - mg - xh * mx)
    ag, ax = g.abs().mean(-1, keepdim=True), (g * xh).abs().mean(-1, keepdim=True)
    bound = U * s * (8 * g.abs() + (DEEP + 8) * ag + (DEEP + 16) * xh.abs() * ax)
    if d_sum is not None:
        dx = dx + d(d_sum)
    bound = bound + 2 * U * dx.abs()
    lead = tuple(range(du.dim() - 1))
    T = du[..., 0].numel()
    dg, db = (du * xh).sum(lead), du.sum(lead)
    return (dx, dg, db), (bound, (T + 16) * U * (du * xh).abs().sum(lead), (T + 16) * U * du.abs().sum(lead))


# ---- routing ------------------------------------------------------------------------------
def softmax(logits):
    """probabilities over all experts (zeros where every logit is -inf) and their relative error: the exponential's argument is
    a rounded product, its sum one of E terms"""
    z = d(logits)
    none = (z == -torch.inf).all(-1)
    p = torch.where(none[..., None], 0.0, torch.softmax(z, -1))
    reach = torch.where(z.isfinite(), z.amax(-1, keepdim=True) - z, 0.0).nan_to_num(0, 0, 0).amax() if z.numel() else 0.0
    return p, none, (2 * z.shape[-1] + 64 + 4 * min(float(reach), 104.0)) * U      # exp(-104) is nothing in fp32


def picks(logits, k):
    return torch.sort(d(logits), dim=-1, descending=True, stable=True).indices[..., :k]


def balance(logits, k, mask=None, per_sequence=False):
    """loss, counts, prob_mean, n by group, and the relative error of the probabilities' means"""
    p, none, rel = softmax(logits)
    E = p.shape[-1]
    S = p.shape[0] if per_sequence else 1
    on = ~none if mask is None else ~none & mask.cpu().bool()
    p = torch.where(on[..., None], p, 0.0).reshape(S, -1, E)
    idx = picks(logits, k)
    hit = torch.zeros(idx.shape[:-1] + (E,), dtype=torch.float64).scatter_(-1, idx, 1.0)
    counts = torch.where(on[..., None], hit, 0.0).reshape(S, -1, E).sum(1)
    n = on.reshape(S, -1).sum(1).double()
    prob = p.sum(1) / n.clamp(min=1)[:, None]
    loss = E * (counts / (k * n).clamp(min=1)[:, None] * prob).sum(1)
    return loss, counts, prob, n, rel + (p.shape[1] + 8) * U


def routing_bwd(logits, topk_idx, d_topk_w, counts, d_loss, mask=None):
    """d_logits and its bound, before it is rounded"""
    p, none, rel = softmax(logits)
    E = p.shape[-1]
    g = torch.zeros_like(p)
    if counts is not None:
        c = d(counts)
        S = c.shape[0]
        k = topk_idx.shape[-1]
        total = c.sum(1, keepdim=True)
        share = torch.where(total > 0, d(d_loss)[:, None] * E * k * c / total.clamp(min=1) ** 2, 0.0)
        on = torch.ones(p.shape[:-1]) if mask is None else mask.cpu().double()
        g = (share[:, None] * on.double().reshape(S, -1, 1)).reshape(p.shape)
    if d_topk_w is not None:
        g = g.scatter_add(-1, topk_idx.cpu().long(), d(d_topk_w))
    zero = none | (g == 0).all(-1)
    p = torch.where(zero[..., None], 0.0, p)
    s = (p * g).sum(-1, keepdim=True)
    return p * (g - s), 2 * rel * p.abs() * (g.abs() + (p * g).abs().sum(-1, keepdim=True))


def linear_bwd(u, W_g, d_logits, du_add=None):
    D, E = u.shape[-1], W_g.shape[0]
    g, uu, W = d(d_logits).reshape(-1, E), d(u).reshape(-1, D), d(W_g)
    add = torch.zeros_like(uu) if du_add is None else d(du_add).reshape(-1, D)
    du, dW = g @ W + add, g.t() @ uu
    bu = 2 * (E + 2) * U * (g.abs() @ W.abs() + add.abs())
    bw = 2 * (uu.shape[0] + 2) * U * (g.abs().t() @ uu.abs())
    return (du.reshape(u.shape), dW), (bu.reshape(u.shape), bw)
