"""The calls that train the routing over tens of thousands of tokens, where every block takes several steps, the last of them
a part: both types, padding, sequences of their own, logits that tie or differ in their last bits."""
import pytest
import torch

from paper_2603_06938_amd import binding as sw
from test_gpu_router_train import check_balance, lengths, logits_of
from train_ref import IO, balance, half, picks, routing_bwd, within

pytestmark = pytest.mark.gpu

# one, two and four pieces of eight experts to a lane, full lanes and others; groups with many blocks, with two, and with one
LONG = [(1, 36011, 256, 8), (1, 34003, 200, 4), (2, 26007, 100, 3), (3, 50021, 64, 6), (1, 90001, 33, 2), (2, 70001, 16, 2), (130, 310, 256, 2),
        (129, 701, 48, 3)]


def near_logits(shape, seed):
    """fp32: whole rows of one value, runs that differ by their lowest bits, equal ones among them"""
    gen = torch.Generator().manual_seed(seed)
    base = 1.0 + torch.randint(0, max(2, shape[-1] // 3), shape, generator=gen) / 16
    base[:, ::5] = 1.0
    step = torch.tensor([1, 40, 300])[torch.arange(shape[1]) % 3][None, :, None]
    bits = base.view(torch.int32) + torch.randint(0, 300, shape, generator=gen, dtype=torch.int32) // step.int()
    z = bits.view(torch.float32)
    z[:, 1::4] *= -1.0
    z[:, 7::9] = 0.0
    return z.to("cuda:0")


@pytest.mark.parametrize("B,L,E,k", LONG)
@pytest.mark.parametrize("kind", ["f32", "bf16", "near"])
def test_balance(B, L, E, k, kind):
    z = near_logits((B, L, E), E) if kind == "near" else logits_of((B, L, E), kind, E)
    mask = lengths(B, L, L)
    mask[0, L // 2:L // 2 + 100] = False                        # and some in the middle
    for m, per_sequence in ((mask, True), (None, False)):
        out = sw.swimba_router_balance(z, k, m, per_sequence=per_sequence)
        check_balance(z, k, m, per_sequence, out)
    again = sw.swimba_router_balance(z, k)
    assert all(torch.equal(a, b) for a, b in zip(out, again)), "two calls differ"


@pytest.mark.parametrize("B,L,E,k", LONG)
@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_every_token_is_counted_once(B, L, E, k, io):
    """One expert has each token's whole probability, so that every sum is a whole number and the mean is rounded once from 64
    bits: a token that is left out or taken twice shows."""
    gen = torch.Generator().manual_seed(L)
    hot = torch.randint(0, E, (B, L, 1), generator=gen)
    z = (-1000.0 - 8 * torch.randint(0, 100, (B, L, E), generator=gen)).scatter_(2, hot, 0.0).to(IO[io]).to("cuda:0")
    mask = lengths(B, L, 3)
    mask[0, 0] = True
    for per_sequence in (True, False):
        out = sw.swimba_router_balance(z, k, mask, per_sequence=per_sequence)
        S = B if per_sequence else 1
        on = mask.cpu().double()
        sums = torch.zeros(B, L, E, dtype=torch.float64).scatter_(2, hot, 1.0).mul_(on[..., None]).reshape(S, -1, E).sum(1)
        n = on.reshape(S, -1).sum(1, keepdim=True)
        want = torch.where(n > 0, sums / n.clamp(min=1), 0.0)
        within(out.prob_mean, want, 2.0 ** -23 * want, "prob_mean")
        assert torch.equal(out.counts.cpu().double(), balance(z, k, mask, per_sequence)[1])
        assert (out.topk_w[..., 0] == 1).all() and (out.topk_w[..., 1:] == 0).all()


# more tokens than 1536 blocks take in one step
STEPS = [(1, 30011, 256, 8), (2, 16001, 200, 4), (1, 60007, 100, 3), (3, 40003, 64, 6), (1, 400001, 8, 2), (300, 130, 256, 2)]


@pytest.mark.parametrize("B,L,E,k", STEPS)
@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_gradient_of_the_logits(B, L, E, k, io):
    z = logits_of((B, L, E), io, E)
    mask = lengths(B, L, L)
    mask[0, L // 2:L // 2 + 50] = False
    dw = torch.randn(B, L, k, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(E))
    idx = picks(z, k)
    counts = balance(z, k, mask, True)[1].int().to("cuda:0")
    idx = idx.int().to("cuda:0")
    dl = torch.linspace(0.5, 2.0, B, device="cuda:0") * 100
    for args, m in (((idx, dw, counts, dl), mask), ((idx, None, counts, dl), mask), ((idx, dw, None, None), None)):
        got = sw.swimba_router_bwd(z, *args, m)
        ref, bound = routing_bwd(z, *args, m)
        within(got, ref, bound + half(z.dtype) * (ref.abs() + bound), "d_logits")
