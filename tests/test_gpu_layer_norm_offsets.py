"""Layer norm of rows whose offset is large beside their deviations, constant ones among them: the mean is rounded, so what a
first mean misses has to be taken out before the squares are summed.  Against 64 bits, with bounds that follow the
deviations and not the offset."""
import pytest
import torch

from paper_2603_06938_amd import binding as sw
from train_ref import DEEP, IO, U, d, half

pytestmark = pytest.mark.gpu

# every number of lanes and waves that a row lies in, with and without a last piece that is moved
WIDTHS = [1, 3, 40, 100, 128, 255, 512, 768, 1000, 1001, 2048, 2047, 4096, 5000, 8192, 8195, 9000, 12288, 12289, 16384]


def bounds(r, eps, gamma, beta):
    """(u, mean, rstd) in 64 bits and what fp32 may be off by, before u is rounded.  e: of a first mean, relative to the largest
    element.  The second is the mean of differences that are rounded to U of themselves; what is left of an element's
    difference is off by `left`."""
    r, g, b = d(r), d(gamma), d(beta)
    m = r.mean(-1, keepdim=True)
    dev = (r - m).abs().amax(-1, keepdim=True)
    var = (r - m).square().mean(-1, keepdim=True)
    s = (var + eps).rsqrt()
    e = (DEEP + 1) * U * r.abs().amax(-1, keepdim=True)
    left = (DEEP + 5) * U * (dev + e)
    ds = (DEEP / 2 + 8) * U + s * s * (dev * left + left * left / 2)       # of rstd, relative
    xh = (r - m) * s
    u = xh * g + b
    return (u, m[..., 0], s[..., 0]), (g.abs() * (s * left + (ds + 4 * U) * xh.abs()) + 4 * U * ((g * xh).abs() + b.abs()),
                                       (left + U * m.abs())[..., 0], (ds * s)[..., 0])


def check(got, want, bound, what):
    off = (d(got) - want).abs()
    assert got.isfinite().all() and (off <= bound).all(), "%s: %r beyond %r" % (what, float(off.max()), float(bound.max()))


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("io,res", [("f32", None), ("bf16", None), ("bf16", "f32"), ("f32", "f32")])
def test_large_offsets(D, io, res):
    gen = torch.Generator().manual_seed(D)
    T, eps = 48, 1e-5
    size = 10.0 ** (torch.rand(T, 1, generator=gen, dtype=torch.float64) * 8 - 2) * torch.where(torch.arange(T)[:, None] % 2 == 0, 1.0, -1.0)
    size[0], size[1] = 12345.678, 0.1
    x = (size * torch.ones(D, dtype=torch.float64)).float()
    ulp = 2.0 ** (torch.log2(size.abs()).floor() - 23)
    x[16:32] += (torch.randint(-3, 4, (16, D), generator=gen) * ulp[16:32]).float()          # a few steps of the type apart
    x[32:] += 0.01 * torch.randn(16, D, generator=gen)                                       # deviations of some size of their own
    residual = None
    if res:
        residual, x = x.to(IO[res]).to("cuda:0"), torch.zeros(T, D)
    x = x.to(IO[io]).to("cuda:0")
    gamma = (1 + 0.1 * torch.randn(D, generator=gen)).to("cuda:0")
    beta = (0.1 * torch.randn(D, generator=gen)).to("cuda:0")
    out = sw.swimba_layer_norm(x, gamma, beta, eps, residual, want_stats=True)
    r = x if residual is None else out.sum
    (u, m, s), (bu, bm, bs) = bounds(r, eps, gamma, beta)
    check(out.mean, m, bm, "mean")
    check(out.rstd, s, bs, "rstd")
    check(out.u, u, bu + half(x.dtype) * (u.abs() + bu), "u")
    # (what a constant row's mean is off by before it is rounded is less than a quarter of a step)
    assert torch.equal(out.mean[:16], r[:16, 0].float())
    # the backward pass from these statistics: a constant row's xh is zero
    du = torch.randn(T, D, generator=gen).to(IO[io]).to("cuda:0")
    back = sw.swimba_layer_norm_bwd(du[:16], r[:16], gamma, out.mean[:16], out.rstd[:16])
    assert (back.dgamma == 0).all()


@pytest.mark.parametrize("D,io", [(1025, "f32"), (1030, "bf16"), (33, "f32")])
def test_more_rows_than_blocks(D, io):
    """2^20 blocks at most: beyond that many rows (times 16, of narrow ones) a block takes another."""
    T = (1 << 20) * (16 if D <= 64 else 1) + 301
    gen = torch.Generator("cuda:0").manual_seed(D)
    x = torch.empty(T, D, dtype=IO[io], device="cuda:0")
    x[:302] = torch.randn(302, D, device="cuda:0", generator=gen) + 100
    x[302:-302] = 1.0
    x[-302:] = torch.randn(302, D, device="cuda:0", generator=gen) - 50
    gamma, beta = torch.randn(D, device="cuda:0", generator=gen), torch.randn(D, device="cuda:0", generator=gen)
    out = sw.swimba_layer_norm(x, gamma, beta, 1e-5, want_stats=True)
    for part in (slice(0, 302), slice(T - 302, T)):
        rows = x[part].clone()
        alone = sw.swimba_layer_norm(rows, gamma, beta, 1e-5, want_stats=True)
        assert torch.equal(out.u[part], alone.u) and torch.equal(out.mean[part], alone.mean) and torch.equal(out.rstd[part], alone.rstd)
        (u, m, s), (bu, bm, bs) = bounds(rows, 1e-5, gamma, beta)
        check(alone.u, u, bu + half(rows.dtype) * (u.abs() + bu), "u")
    assert (out.u[302:-302] == beta.to(x.dtype)).all()
