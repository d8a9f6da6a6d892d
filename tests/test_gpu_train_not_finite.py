"""Infinities and NaN in the calls that train the routing: every output is what its formula gives in 64 bits, NaN where that is
NaN, the same infinity where it is one, and within its bound everywhere else."""
import pytest
import torch

from paper_2603_06938_amd import binding as sw
from train_ref import IO, U, d, half, linear_bwd, norm, norm_bwd, picks, routing_bwd, softmax

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
WIDTHS = [3, 40, 100, 255, 513, 768, 1001, 2047, 4096, 9000, 16384]


def same(got, want, bound, what):
    got, bound = d(got), bound.expand_as(want)
    assert got.shape == want.shape, what
    fine = torch.where(want.isfinite(), got.isfinite() & ((got - want).abs() <= bound), (got == want) | (got.isnan() & want.isnan()))
    if not fine.all():
        i = tuple((~fine).nonzero()[0].tolist())
        raise AssertionError("%s: %d elements, the first at %s: %r for %r, bound %r" % (
            what, int((~fine).sum()), i, float(got[i]), float(want[i]), float(bound[i])))


def normal(*s, io="f32", seed=0, scale=1.0):
    return (scale * torch.randn(*s, generator=torch.Generator().manual_seed(seed))).to(IO[io]).to("cuda:0")


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("io,res", [("f32", None), ("bf16", None), ("bf16", "f32"), ("bf16", "bf16")])
def test_layer_norm(D, io, res):
    x = normal(9, D, io=io, seed=D)
    x[1, 0], x[2, D - 1], x[3, D // 2], x[4, D // 2] = INF, -INF, NAN, INF
    x[4, 0] = -INF
    residual = None if res is None else normal(9, D, io=res, seed=1)
    if res:
        residual[6, 1] = INF
    gamma, beta = 1 + normal(D, seed=2, scale=0.1), normal(D, seed=3, scale=0.1)
    gamma[0], beta[D - 1] = INF, -INF
    out = sw.swimba_layer_norm(x, gamma, beta, 1e-5, residual, want_stats=True)
    (u, r, m, s), (bu, bm, bs) = norm(x, gamma, beta, 1e-5, residual)
    same(out.mean, m, bm, "mean")
    same(out.rstd, s, bs, "rstd")
    same(out.u, u, bu + half(x.dtype) * (u.abs() + bu), "u")
    if res:
        same(out.sum, r, torch.zeros_like(r), "sum")
    # back: a gradient that is not finite, and the rows and statistics from above
    du = normal(9, D, io=io, seed=4)
    du[0, 1], du[5, D - 1], du[7, 0] = INF, NAN, -INF
    rows = x if residual is None else out.sum
    gamma[0] = 1.0
    back = sw.swimba_layer_norm_bwd(du, rows, gamma, out.mean, out.rstd)
    (dx, dg, db), (bx, bg, bb) = norm_bwd(du, rows, gamma, out.mean, out.rstd)
    same(back.dx, dx, bx + half(rows.dtype) * (dx.abs() + bx), "dx")
    same(back.dgamma, dg, bg, "dgamma")
    same(back.dbeta, db, bb, "dbeta")


@pytest.mark.parametrize("E,k", [(3, 1), (8, 2), (16, 4), (40, 3), (100, 4), (256, 8)])
@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_routing(E, k, io):
    B, L = 3, 70
    z = normal(B, L, E, io=io, seed=E)
    z[0, 5, E - 1], z[0, 9] = INF, -INF
    z[1, 7, 1] = -INF
    z[2, 3, 0] = NAN
    out = sw.swimba_router_balance(z, k, per_sequence=True)
    p, none, rel = softmax(z.nan_to_num(0.0, INF, -INF))
    p[2, 3] = NAN
    n = (~none).sum(1).double()
    mean = torch.where(none[..., None], 0.0, p).sum(1) / n[:, None]
    same(out.prob_mean, mean, (rel + 100 * U) * mean, "prob_mean")
    idx = picks(z, k)
    keep = ~none
    keep[2, 3] = False                                          # which experts a token without an order gets is not said
    assert torch.equal(out.topk_idx.cpu().long()[keep], idx[keep])
    w = torch.gather(p, -1, idx)
    same(out.topk_w[keep.to("cuda:0")], w[keep], (rel * w)[keep], "topk_w")
    loss = E * (d(out.counts) / (k * n)[:, None] * mean).sum(1)
    same(out.loss, loss, (rel + 200 * U) * loss, "loss")
    # back, with weights' gradients that are not finite
    z[0, 5, E - 1], z[2, 3, 0] = 1.0, 0.5
    dw = normal(B, L, k, seed=5)
    dw[1, 0, 0], dw[1, 20, k - 1], dw[2, 60, 0] = INF, -INF, NAN
    idx, dl = picks(z, k).int().to("cuda:0"), torch.tensor([1.0, 2.0, 3.0], device="cuda:0")
    got = sw.swimba_router_bwd(z, idx, dw, out.counts, dl)
    ref, bound = routing_bwd(z, idx, dw, out.counts, dl)
    same(got, ref, bound + half(z.dtype) * (ref.abs() + bound) + 2.0 ** -120, "d_logits")


@pytest.mark.parametrize("T,D,E", [(70, 77, 5), (300, 768, 8), (64, 256, 40), (130, 130, 100), (33, 64, 256)])
@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_linear_backward(T, D, E, io):
    u, W, g, add = normal(T, D, io=io, seed=1), normal(E, D, io=io, seed=2), normal(T, E, io=io, seed=3), normal(T, D, io=io, seed=4)
    u[3, 5], u[T - 1, D - 1], W[0, 1], W[E - 1, D - 2], g[7, E // 2], g[9, 0], add[11, 3], add[12, 4] = INF, NAN, -INF, NAN, INF, NAN, INF, NAN
    out = sw.swimba_router_linear_bwd(u, W, g, add)
    (du, dW), (bu, bw) = linear_bwd(u, W, g, add)
    same(out.du, du, bu + half(u.dtype) * (du.abs() + bu), "du")
    same(out.dW_g, dW, bw, "dW_g")
