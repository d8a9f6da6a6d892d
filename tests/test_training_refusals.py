"""What the calls that train the routing refuse, on the host, before anything is enqueued: no GPU is needed for it."""
import pytest
import torch

from paper_2603_06938_amd import binding as sw

OK, NULL, SHAPE, DTYPE, UNSUPPORTED, WORKSPACE, ALIGNMENT = 0, 1, 2, 3, 4, 5, 7
P = [0x10000 * (i + 1) for i in range(12)]
F32, BF16 = 0, 1


def norm(tokens=4, D=64, io=BF16, res=F32, x=P[0], residual=P[1], gamma=P[2], beta=P[3], eps=1e-5, u=P[4], sum=P[5], mean=P[6], rstd=P[7]):
    return sw._load().swimba_layer_norm(tokens, D, io, res, x, residual, gamma, beta, eps, u, sum, mean, rstd, None)


@pytest.mark.parametrize("kw,status", [
    (dict(io=2), DTYPE), (dict(io=F32, res=BF16), DTYPE), (dict(res=7), DTYPE), (dict(residual=None, sum=None), DTYPE),
    (dict(tokens=-1), SHAPE), (dict(D=0), SHAPE), (dict(D=16385), UNSUPPORTED), (dict(tokens=(1 << 38) + 1), UNSUPPORTED),
    (dict(eps=0.0), SHAPE), (dict(eps=-1e-5), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE),
    (dict(x=None), NULL), (dict(u=None), NULL), (dict(io=F32, residual=None), NULL),
    (dict(x=P[0] + 8), ALIGNMENT), (dict(residual=P[1] + 4), ALIGNMENT), (dict(u=P[4] + 2), ALIGNMENT), (dict(sum=P[5] + 8), ALIGNMENT),
    (dict(gamma=P[2] + 2), ALIGNMENT), (dict(beta=P[3] + 1), ALIGNMENT), (dict(mean=P[6] + 2), ALIGNMENT), (dict(rstd=P[7] + 3), ALIGNMENT),
    (dict(tokens=0, x=None, u=None), OK),
])
def test_layer_norm(kw, status):
    assert norm(**kw) == status


def norm_bwd(tokens=400, D=64, io=BF16, res=F32, du=P[0], r=P[1], gamma=P[2], mean=P[3], rstd=P[4], d_sum=P[5], dx=P[6], dx_io=P[7],
             dgamma=P[8], dbeta=P[9], ws=P[10], size=None):
    lib = sw._load()
    size = lib.swimba_layer_norm_bwd_workspace_bytes(tokens, D) if size is None else size
    return lib.swimba_layer_norm_bwd(tokens, D, io, res, du, r, gamma, mean, rstd, d_sum, dx, dx_io, dgamma, dbeta, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(io=2), DTYPE), (dict(res=2), DTYPE), (dict(io=F32, res=BF16), DTYPE), (dict(res=BF16), DTYPE),     # dx_io of one type
    (dict(tokens=-1), SHAPE), (dict(D=-3), SHAPE), (dict(D=16385), UNSUPPORTED),
    (dict(ws=None), WORKSPACE), (dict(ws=P[10] + 128), WORKSPACE), (dict(size=0), WORKSPACE),
    (dict(du=None), NULL), (dict(r=None), NULL), (dict(mean=None), NULL), (dict(rstd=None), NULL), (dict(dx=None), NULL),
    (dict(du=P[0] + 8), ALIGNMENT), (dict(r=P[1] + 8), ALIGNMENT), (dict(d_sum=P[5] + 4), ALIGNMENT), (dict(dx=P[6] + 4), ALIGNMENT),
    (dict(dx_io=P[7] + 2), ALIGNMENT), (dict(gamma=P[2] + 1), ALIGNMENT), (dict(mean=P[3] + 2), ALIGNMENT), (dict(dgamma=P[8] + 2), ALIGNMENT),
    (dict(dbeta=P[9] + 2), ALIGNMENT), (dict(tokens=0, du=None, dgamma=None, dbeta=None), OK),
])
def test_layer_norm_bwd(kw, status):
    assert norm_bwd(**kw) == status


def balance(groups=2, tokens=50000, E=8, k=2, io=BF16, logits=P[0], mask=P[1], idx=P[2], w=P[3], counts=P[4], prob=P[5], loss=P[6], ws=P[7], size=None):
    lib = sw._load()
    size = lib.swimba_router_balance_workspace_bytes(groups, tokens, E) if size is None else size
    return lib.swimba_router_balance(groups, tokens, E, k, io, logits, mask, idx, w, counts, prob, loss, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(io=2), DTYPE), (dict(groups=-1), SHAPE), (dict(tokens=-1), SHAPE), (dict(E=0, k=1), SHAPE), (dict(k=0), SHAPE), (dict(k=9), SHAPE),
    (dict(E=257), UNSUPPORTED), (dict(E=32, k=17), UNSUPPORTED), (dict(groups=(1 << 20) + 1), UNSUPPORTED), (dict(tokens=1 << 31), UNSUPPORTED),
    (dict(groups=1 << 10, tokens=(1 << 28) + 1), UNSUPPORTED),
    (dict(ws=None), WORKSPACE), (dict(ws=P[7] + 16), WORKSPACE), (dict(size=0), WORKSPACE),
    (dict(logits=None), NULL), (dict(counts=None), NULL), (dict(loss=None), NULL),
    (dict(logits=P[0] + 1), ALIGNMENT), (dict(io=F32, logits=P[0] + 2), ALIGNMENT), (dict(idx=P[2] + 2), ALIGNMENT), (dict(w=P[3] + 2), ALIGNMENT),
    (dict(counts=P[4] + 2), ALIGNMENT), (dict(prob=P[5] + 2), ALIGNMENT), (dict(loss=P[6] + 2), ALIGNMENT), (dict(groups=0, ws=None), OK),
])
def test_router_balance(kw, status):
    assert balance(**kw) == status


def bwd(groups=2, tokens=5, E=8, k=2, io=BF16, logits=P[0], mask=P[1], idx=P[2], dw=P[3], counts=P[4], loss=P[5], out=P[6]):
    return sw._load().swimba_router_bwd(groups, tokens, E, k, io, logits, mask, idx, dw, counts, loss, out, None)


@pytest.mark.parametrize("kw,status", [
    (dict(io=-1), DTYPE), (dict(groups=-1), SHAPE), (dict(k=9), SHAPE), (dict(E=300), UNSUPPORTED), (dict(E=64, k=17), UNSUPPORTED),
    (dict(tokens=1 << 31), UNSUPPORTED), (dict(logits=None), NULL), (dict(out=None), NULL), (dict(idx=None), NULL), (dict(counts=None), NULL),
    (dict(loss=None), NULL), (dict(logits=P[0] + 1), ALIGNMENT), (dict(out=P[6] + 1), ALIGNMENT), (dict(idx=P[2] + 2), ALIGNMENT),
    (dict(dw=P[3] + 1), ALIGNMENT), (dict(counts=P[4] + 2), ALIGNMENT), (dict(loss=P[5] + 2), ALIGNMENT),
    (dict(tokens=0, logits=None, out=None), OK), (dict(groups=0), OK),
])
def test_router_bwd(kw, status):
    assert bwd(**kw) == status


def linear(tokens=500, D=64, E=8, io=BF16, u=P[0], W=P[1], g=P[2], add=P[3], du=P[4], dW=P[5], ws=P[6], size=None):
    lib = sw._load()
    size = lib.swimba_router_linear_bwd_workspace_bytes(tokens, D, E) if size is None else size
    return lib.swimba_router_linear_bwd(tokens, D, E, io, u, W, g, add, du, dW, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(io=2), DTYPE), (dict(tokens=-1), SHAPE), (dict(D=0), SHAPE), (dict(E=0), SHAPE), (dict(E=257), UNSUPPORTED), (dict(D=65537), UNSUPPORTED),
    (dict(tokens=(1 << 38) + 1), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws=P[6] + 8), WORKSPACE), (dict(size=0), WORKSPACE),
    (dict(u=None), NULL), (dict(W=None), NULL), (dict(g=None), NULL), (dict(du=None), NULL),      # du_add without du
    (dict(u=P[0] + 8), ALIGNMENT), (dict(W=P[1] + 4), ALIGNMENT), (dict(add=P[3] + 8), ALIGNMENT), (dict(du=P[4] + 2), ALIGNMENT),
    (dict(g=P[2] + 1), ALIGNMENT), (dict(dW=P[5] + 2), ALIGNMENT), (dict(tokens=0, u=None, W=None, g=None, dW=None), OK),
])
def test_router_linear_bwd(kw, status):
    assert linear(**kw) == status


def test_workspaces_grow_with_the_call_and_end():
    lib = sw._load()
    for f, most in ((lambda t: lib.swimba_layer_norm_bwd_workspace_bytes(t, 768), 1 << 24),
                    (lambda t: lib.swimba_router_balance_workspace_bytes(1, t, 256), 1 << 24),
                    (lambda t: lib.swimba_router_linear_bwd_workspace_bytes(t, 768, 8), 1 << 25)):
        sizes = [f(t) for t in (0, 1, 100, 10000, 1 << 20, 1 << 30)]
        assert sizes == sorted(sizes) and 0 < sizes[0] and sizes[-1] <= most and all(s % 256 == 0 for s in sizes)
    # 256 bytes: nothing is kept there, and no workspace is asked for (but the pointers behind it are)
    assert lib.swimba_layer_norm_bwd_workspace_bytes(16, 768) == lib.swimba_router_balance_workspace_bytes(4, 150, 8) == 256
    assert lib.swimba_router_linear_bwd_workspace_bytes(128, 768, 8) == 256
    assert norm_bwd(tokens=16, D=768, ws=None, size=0, dx=None) == balance(groups=4, tokens=150, ws=None, size=0, loss=None) == NULL
    assert linear(tokens=128, D=768, ws=None, size=0, W=None) == NULL
    assert lib.swimba_router_balance_workspace_bytes(0, 1 << 20, 8) == 256    # no group: nothing to divide the slices among
    assert lib.swimba_layer_norm_bwd_workspace_bytes(17, 768) == 5 * 2 * 768 * 4       # the sums of five blocks of four rows
    assert lib.swimba_layer_norm_bwd_workspace_bytes(-1, 768) == lib.swimba_layer_norm_bwd_workspace_bytes(1, 20000) == 0
    assert lib.swimba_router_balance_workspace_bytes(1, 1 << 31, 8) == lib.swimba_router_balance_workspace_bytes(1, 1, 257) == 0
    assert lib.swimba_router_linear_bwd_workspace_bytes(1, 0, 8) == lib.swimba_router_linear_bwd_workspace_bytes(1, 1 << 17, 8) == 0


@pytest.mark.parametrize("x,kind", [
    (torch.zeros(2, 8), ValueError), (torch.zeros(2, 8, dtype=torch.float64), TypeError), (torch.zeros(()), ValueError), ([[1.0]], TypeError),
], ids=["cpu", "dtype", "rank", "list"])
def test_marshalling(x, kind):
    t = torch.zeros(8)
    for call in (lambda: sw.swimba_layer_norm(x, t, t), lambda: sw.swimba_layer_norm_bwd(x, x, t, t, t),
                 lambda: sw.swimba_router_balance(x, 2), lambda: sw.swimba_router_bwd(x),
                 lambda: sw.swimba_router_linear_bwd(x, torch.zeros(4, 8), t)):
        with pytest.raises(kind):
            call()
