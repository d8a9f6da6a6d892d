"""swimba_layer_norm and swimba_layer_norm_bwd against their formulas in 64 bits, element by element."""
import pytest
import torch

from paper_2603_06938_amd import binding as sw
from train_ref import IO, half, norm, norm_bwd, within

pytestmark = pytest.mark.gpu

# both sides of every width at which another number of lanes or waves takes a row, and rows that start at any element
WIDTHS = [1, 2, 7, 8, 9, 16, 63, 64, 65, 100, 127, 128, 129, 256, 257, 504, 511, 512, 513, 768, 1001, 1024, 1025, 2047,
          2048, 2056, 4096, 4099, 6144, 6145, 8192, 8200, 12288, 12345, 16384]
TYPES = [("f32", None), ("bf16", None), ("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")]


def rows(T, D, io, seed, offset=0.5, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(T, D, generator=gen) * scale + offset).to(IO[io]).to("cuda:0")


def case(T, D, io, res, seed):
    x = rows(T, D, io, seed)
    residual = None if res is None else rows(T, D, res, seed + 1, -0.25, 2.0)
    return x, residual, 1 + 0.1 * rows(1, D, "f32", seed + 2)[0], rows(1, D, "f32", seed + 3, 0.0, 0.1)[0]


def guarded(T, D, dtype):
    """a (T, D) tensor with values behind it that no call may touch"""
    big = torch.full((T * D + 64,), 7.0, dtype=dtype, device="cuda:0")
    return big[:T * D].view(T, D), big[T * D:]


def check_fwd(x, residual, gamma, beta, eps, out):
    (u, r, m, s), (bu, bm, bs) = norm(x, gamma, beta, eps, residual)
    within(out.u, u, bu + half(x.dtype) * (u.abs() + bu), "u")
    if residual is not None and out.sum is not None:
        assert torch.equal(out.sum.cpu(), r.to(residual.dtype)), "sum"
    if out.mean is not None:
        within(out.mean, m, bm, "mean")
        within(out.rstd, s, bs, "rstd")


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("io,res", TYPES)
def test_forward(D, io, res):
    T = 5
    x, residual, gamma, beta = case(T, D, io, res, D)
    u, behind = guarded(T, D, x.dtype)
    total, behind_sum = guarded(T, D, IO[res]) if res else (None, None)
    out = sw.swimba_layer_norm(x, gamma, beta, 1e-5, residual, u=u, sum=total, want_stats=True)
    assert out.u is u and out.sum is total
    check_fwd(x, residual, gamma, beta, 1e-5, out)
    assert (behind == 7).all() and (behind_sum is None or (behind_sum == 7).all())


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("io,res", TYPES)
def test_backward(D, io, res):
    T = 6
    r = rows(T, D, res or io, D)
    gamma = 1 + 0.1 * rows(1, D, "f32", D + 2)[0]
    du = rows(T, D, io, D + 4, 0.1)
    d_sum = rows(T, D, res, D + 5, 0.0) if res else None
    (_, _, m, s), _ = norm(r, None, None, 1e-5)
    mean, rstd = m.float().to("cuda:0"), s.float().to("cuda:0")
    dx, behind = guarded(T, D, r.dtype)
    got = sw.swimba_layer_norm_bwd(du, r, gamma, mean, rstd, d_sum, dx=dx)
    (rx, rg, rb), (bx, bg, bb) = norm_bwd(du, r, gamma, mean, rstd, d_sum)
    within(got.dx, rx, bx + half(r.dtype) * (rx.abs() + bx), "dx")
    assert (got.dx_io is None) == (r.dtype == du.dtype)
    if got.dx_io is not None:
        assert torch.equal(got.dx_io, got.dx.to(du.dtype)), "dx_io"
    within(got.dgamma, rg, bg, "dgamma")
    within(got.dbeta, rb, bb, "dbeta")
    assert (behind == 7).all()


@pytest.mark.parametrize("T,D", [(1, 768), (2, 8), (3, 513), (64, 768), (65, 1000), (511, 64), (2049, 24), (3000, 130),
                                 (301, 64), (777, 100), (4097, 128), (700, 2048), (600, 9000)])
@pytest.mark.parametrize("io,res", [("bf16", "f32"), ("f32", None)])
def test_numbers_of_rows(T, D, io, res):
    x, residual, gamma, beta = case(T, D, io, res, T)
    out = sw.swimba_layer_norm(x, gamma, beta, 1e-5, residual, want_stats=True)
    check_fwd(x, residual, gamma, beta, 1e-5, out)
    r = x if residual is None else out.sum
    du = rows(T, D, io, T + 9, 0.1)
    got = sw.swimba_layer_norm_bwd(du, r, gamma, out.mean, out.rstd)
    (rx, rg, rb), (bx, bg, bb) = norm_bwd(du, r, gamma, out.mean, out.rstd)
    within(got.dx, rx, bx + half(r.dtype) * (rx.abs() + bx), "dx")
    within(got.dgamma, rg, bg, "dgamma")
    within(got.dbeta, rb, bb, "dbeta")
    again = sw.swimba_layer_norm_bwd(du, r, gamma, out.mean, out.rstd)
    assert all(torch.equal(a, b) for a, b in zip(got, again) if a is not None), "two calls differ"


def test_nothing_but_what_is_wanted():
    x, residual, gamma, beta = case(9, 300, "bf16", "f32", 1)
    out = sw.swimba_layer_norm(x, None, None, 1e-3, residual, want_sum=False)
    assert out.sum is None and out.mean is None and out.rstd is None
    check_fwd(x, residual, None, None, 1e-3, out)
    check_fwd(x, None, None, beta, 1e-3, sw.swimba_layer_norm(x, None, beta, 1e-3))
    check_fwd(x, None, gamma, None, 1e-3, sw.swimba_layer_norm(x, gamma, None, 1e-3))
    full = sw.swimba_layer_norm(x, gamma, beta, 1e-3, residual, want_stats=True)
    a = sw.swimba_layer_norm_bwd(x, full.sum, None, full.mean, full.rstd, want_dx_io=False, want_weights=False)
    assert a.dx_io is None and a.dgamma is None and a.dbeta is None
    b = sw.swimba_layer_norm_bwd(x, full.sum, torch.ones_like(gamma), full.mean, full.rstd)
    assert torch.equal(a.dx, b.dx)
    only = torch.empty_like(gamma)
    c = sw.swimba_layer_norm_bwd(x, full.sum, None, full.mean, full.rstd, dbeta=only, want_weights=False)
    assert c.dgamma is None and torch.equal(only, b.dbeta)


def test_in_place_along_the_residual_stream():
    for io, res in (("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")):
        for D in (768, 1001, 5000, 9000):
            x, residual, gamma, beta = case(37, D, io, res, D)
            want = sw.swimba_layer_norm(x, gamma, beta, 1e-5, residual, want_stats=True)
            stream = residual.clone()
            got = sw.swimba_layer_norm(x, gamma, beta, 1e-5, stream, sum=stream, want_stats=True)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            if io == res:
                stream = x.clone()
                got = sw.swimba_layer_norm(stream, gamma, beta, 1e-5, residual, sum=stream)
                assert torch.equal(got.u, want.u) and torch.equal(stream, want.sum)
            d_sum = rows(37, D, res, 3)
            want = sw.swimba_layer_norm_bwd(x, want.sum, gamma, want.mean, want.rstd, d_sum), want
            got = sw.swimba_layer_norm_bwd(x, want[1].sum, gamma, want[1].mean, want[1].rstd, d_sum, dx=d_sum)
            assert all(torch.equal(a, b) for a, b in zip(got, want[0]) if a is not None)


@pytest.mark.parametrize("io,res", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("D", [5, 67, 130, 515, 771, 1030, 2047, 4099, 5205, 8195, 9001, 12289, 16381])
def test_in_place_where_pieces_overlap(D, io, res):
    """Rows that do not end with a piece, whose last lane reads elements of its neighbour: in place those may be new or old."""
    x, residual, gamma, beta = case(300, D, io, res, D)
    want = sw.swimba_layer_norm(x, gamma, beta, 1e-5, residual, want_stats=True)
    stream = residual.clone()
    got = sw.swimba_layer_norm(x, gamma, beta, 1e-5, stream, sum=stream, want_stats=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    d_sum = rows(300, D, res, 3)
    back = sw.swimba_layer_norm_bwd(x, want.sum, gamma, want.mean, want.rstd, d_sum)
    got = sw.swimba_layer_norm_bwd(x, want.sum, gamma, want.mean, want.rstd, d_sum, dx=d_sum)
    assert all(torch.equal(a, b) for a, b in zip(got, back) if a is not None)
    # a weight that is no number reaches its own column
    for e in {0, D // 2, D - 4, D - 1} & set(range(D)):
        bad, worse = gamma.clone(), beta.clone()
        bad[e], worse[e] = float("inf"), float("nan")
        out = sw.swimba_layer_norm(x, bad, worse, 1e-5, residual, want_sum=False).u
        assert out[:, e].isnan().all()
        out[:, e] = want.u[:, e]
        assert torch.equal(out, want.u)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_rows_apart_from_their_neighbours(io):
    """A row that is not finite, one that is constant, one of large offset: each reaches its own outputs alone."""
    x, _, gamma, beta = case(40, 700, io, None, 4)
    want = sw.swimba_layer_norm(x, gamma, beta, 1e-5, want_stats=True)
    y = x.clone()
    y[3, 5], y[7, 0], y[11, 699] = float("nan"), float("inf"), float("-inf")
    y[13] = 3.0
    y[17] = 0.0
    y[19] = (y[19].float() + 3e4).to(y.dtype)
    y[21] *= 1e-18
    got = sw.swimba_layer_norm(y, gamma, beta, 1e-5, want_stats=True)
    touched = torch.tensor([3, 7, 11, 13, 17, 19, 21], device="cuda:0")
    keep = torch.ones(40, dtype=torch.bool, device="cuda:0")
    keep[touched] = False
    assert torch.equal(got.u[keep], want.u[keep])
    assert got.u[[3, 7, 11]].isnan().all()
    check_fwd(y[[13, 17, 19, 21]], None, gamma, beta, 1e-5, sw.NormOut(got.u[[13, 17, 19, 21]], None, got.mean[[13, 17, 19, 21]],
                                                                        got.rstd[[13, 17, 19, 21]]))
    assert torch.equal(got.u[13], beta.to(x.dtype)) and torch.equal(got.u[17], beta.to(x.dtype))
    g0 = sw.swimba_layer_norm_bwd(x, x, gamma, want.mean, want.rstd)
    g1 = sw.swimba_layer_norm_bwd(x, y, gamma, got.mean, got.rstd)
    assert torch.equal(g0.dx[keep], g1.dx[keep]) and torch.equal(g0.dbeta, g1.dbeta)
    assert g1.dx[[3, 7, 11]].isnan().all()


def test_no_rows():
    for io in ("f32", "bf16"):
        x, ones = torch.zeros(2, 0, 768, dtype=IO[io], device="cuda:0"), torch.ones(768, device="cuda:0")
        out = sw.swimba_layer_norm(x, ones, ones, want_stats=True)
        assert out.u.shape == x.shape and out.mean.shape == (2, 0)
        got = sw.swimba_layer_norm_bwd(x, x, ones, out.mean, out.rstd, dgamma=ones.clone(), dbeta=ones.clone())
        assert (got.dgamma == 0).all() and (got.dbeta == 0).all()


@pytest.mark.parametrize("D", [40, 1500])
def test_backward_against_differences(D):
    """The slope of a random function of u along a random direction, in 64 bits, against the gradients' products with it."""
    T, eps, h = 7, 1e-2, 1e-4
    x, _, gamma, beta = case(T, D, "f32", None, D)
    gen = torch.Generator().manual_seed(5)
    c, vx, vg, vb = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((T, D), (T, D), (D,), (D,)))

    def f(a):
        r = x.double().cpu() + a * vx
        m = r.mean(1, keepdim=True)
        xh = (r - m) / ((r - m).square().mean(1, keepdim=True) + eps).sqrt()
        return (c * (xh * (gamma.double().cpu() + a * vg) + beta.double().cpu() + a * vb)).sum()
    slope = (8 * (f(h) - f(-h)) - (f(2 * h) - f(-2 * h))) / (12 * h)
    out = sw.swimba_layer_norm(x, gamma, beta, eps, want_stats=True)
    got = sw.swimba_layer_norm_bwd(c.float().to("cuda:0"), x, gamma, out.mean, out.rstd)
    parts = [(g.double().cpu() * v) for g, v in ((got.dx, vx), (got.dgamma, vg), (got.dbeta, vb))]
    # fp32 gradients: some ten half steps of each term; the difference itself is exact to h^4
    assert abs(sum(p.sum() for p in parts) - slope) <= sum(p.abs().sum() for p in parts) * 100 * 2.0 ** -24


def test_on_another_stream_and_from_a_graph():
    x, residual, gamma, beta = case(300, 768, "bf16", "f32", 8)
    du = rows(300, 768, "bf16", 9)
    u, total, stream = torch.empty_like(x), torch.empty_like(residual), residual.clone()
    mean, rstd = torch.empty(300, device="cuda:0"), torch.empty(300, device="cuda:0")
    dx, dxio, dg, db = torch.empty_like(residual), torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    ws = torch.empty(sw.swimba_layer_norm_bwd_workspace_bytes(300, 768), dtype=torch.uint8, device="cuda:0")

    def work():
        sw.swimba_layer_norm(x, gamma, beta, 1e-5, residual, u=u, sum=total, mean=mean, rstd=rstd)
        sw.swimba_layer_norm_bwd(du, total, gamma, mean, rstd, residual, dx=dx, dx_io=dxio, dgamma=dg, dbeta=db, workspace=ws)
    outs = (u, total, mean, rstd, dx, dxio, dg, db)
    work()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    assert torch.equal(stream, residual)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]            # two graphs on one workspace
    with torch.cuda.stream(side):
        for t in outs:
            t.zero_()
        work()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        for g in graphs:
            with torch.cuda.graph(g, stream=side):
                work()
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(4):
        for t in outs:
            t.fill_(float("nan"))
        ws.fill_(255)
        assert torch.randn(1 << 12, device="cuda:0").isfinite().all()
        graphs[rep & 1].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), rep


def test_more_than_2_to_the_31_elements():
    """Rows past the 2^31st and the 2^32nd byte are found: the last ones against their formulas, the sums over all of them."""
    T, D = 140000, 16384
    x = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda:0")
    spots = [0, 65535, 131071, 131072, 135000, T - 1]
    gen = torch.Generator("cuda:0").manual_seed(3)
    for t in spots:
        x[t] = torch.randn(D, device="cuda:0", generator=gen) + 1
    gamma, beta = torch.randn(D, device="cuda:0", generator=gen), torch.randn(D, device="cuda:0", generator=gen)
    out = sw.swimba_layer_norm(x, gamma, beta, 1e-5, want_stats=True)
    at = torch.tensor(spots, device="cuda:0")
    check_fwd(x[at], None, gamma, beta, 1e-5, sw.NormOut(out.u[at], None, out.mean[at], out.rstd[at]))
    assert torch.equal(out.u[T - 2], beta.bfloat16())
    du = torch.zeros_like(x)
    du[at] = x[at] * 0.5
    got = sw.swimba_layer_norm_bwd(du, x, gamma, out.mean, out.rstd)
    (rx, rg, rb), (bx, bg, bb) = norm_bwd(du[at], x[at], gamma, out.mean[at], out.rstd[at])
    within(got.dx[at], rx, bx + half(x.dtype) * (rx.abs() + bx), "dx")
    within(got.dgamma, rg, bg, "dgamma")                       # the rows of zeros add nothing
    within(got.dbeta, rb, bb, "dbeta")
    assert (got.dx[T - 2] == 0).all()


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    a, b = [case(3000, 700, "bf16", "f32", s) for s in (1, 2)]
    one = [sw.swimba_layer_norm(x, g, w, 1e-5, r, want_stats=True) for x, r, g, w in (a, b)]
    want = [sw.swimba_layer_norm_bwd(c[0], o.sum, c[2], o.mean, o.rstd, c[1]) for c, o in zip((a, b), one)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(3):
        got = []
        for s, c in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                o = sw.swimba_layer_norm(c[0], c[2], c[3], 1e-5, c[1], want_stats=True)
                got.append((o, sw.swimba_layer_norm_bwd(c[0], o.sum, c[2], o.mean, o.rstd, c[1])))
        torch.cuda.synchronize()
        for (o, g), w, o1 in zip(got, want, one):
            assert torch.equal(o.u, o1.u) and all(torch.equal(p, q) for p, q in zip(g, w))
