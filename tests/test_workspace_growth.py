"""A workspace that is enough for a number of tokens is enough for fewer: a program that sizes it for its longest batch passes it
to every other.  Host only."""
import pytest

from paper_2603_06938_amd import binding as sw

COUNTS = list(range(0, 3000)) + list(range(8100, 8400)) + list(range(16300, 16500)) + list(range(32700, 32900)) + [
    n + i for n in (50000, 65536, 98304, 1 << 20, 1 << 24) for i in range(-130, 131)]


def falls(query):
    sizes = [query(t) for t in COUNTS]
    assert min(sizes) >= 256
    return [(a, b) for a, b, s, n in zip(COUNTS, COUNTS[1:], sizes, sizes[1:]) if n < s]


@pytest.mark.parametrize("D,E", [(768, 8), (768, 20), (1024, 16), (2048, 64), (2047, 256), (64, 3), (16384, 8), (65536, 256), (1, 1)])
def test_router_linear_bwd(D, E):
    assert falls(lambda t: sw.swimba_router_linear_bwd_workspace_bytes(t, D, E)) == []


@pytest.mark.parametrize("D", [1, 64, 100, 256, 768, 1001, 4096, 9000, 16384])
def test_layer_norm_bwd(D):
    assert falls(lambda t: sw.swimba_layer_norm_bwd_workspace_bytes(t, D)) == []


@pytest.mark.parametrize("E", [1, 8, 16, 33, 64, 100, 256])
@pytest.mark.parametrize("groups", [1, 2, 7, 100, 128, 129])
def test_router_balance(groups, E):
    assert falls(lambda t: sw.swimba_router_balance_workspace_bytes(groups, t, E)) == []
    # fewer groups of as many tokens, where a group has blocks of its own
    for t in (1, 100, 4097, 70000):
        sizes = [sw.swimba_router_balance_workspace_bytes(g, t, E) for g in range(129)]
        assert sizes == sorted(sizes)
