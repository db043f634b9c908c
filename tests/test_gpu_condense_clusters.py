"""Condensing on either side of every border between launches: a head's candidates go to one CTA up to 2048, to two
up to 4096, to four up to 8192 and to eight beyond, and to no more than two CTAs an SM in all heads together (40
heads to four, 128 to two).  A CTA holds up to 40960 candidates."""
import pytest
import torch

from test_gpu_condense import _cache, _check

pytestmark = pytest.mark.gpu


def _weights(kind, shape, g):
    if kind == "random":
        return torch.exp(2 * torch.randn(shape, generator=g, device="cuda"))
    u = torch.rand(shape, generator=g, device="cuda")
    if kind == "one digit":           # 1 to 1.24: all share the first digit, more than any list takes
        return 1 + 0.24 * u
    return 1 + 0.24 * torch.floor(u * 64) / 64       # "ties": the same with few values


@pytest.mark.parametrize("Hp,Wp,n", [(32, 32, 2), (1, 683, 3), (32, 64, 2), (17, 241, 3), (32, 32, 8), (1, 2731, 3)])
@pytest.mark.parametrize("kind", ["random", "one digit", "ties"])
def test_borders(sva_mod, Hp, Wp, n, kind):
    """2048, 2049, 4096, 12291, 8192 and 8193 candidates."""
    H, T = 2, Hp * Wp
    c, src, dst, g = _cache(sva_mod, 1, Hp, Wp, H, 64, n)
    _check(c, src, dst, _weights(kind, (n + 2, H, T), g), T, H)
    c.close()


@pytest.mark.parametrize("H", [40, 128])
@pytest.mark.parametrize("kind", ["random", "one digit", "ties"])
def test_many_heads(sva_mod, H, kind):
    """11000 candidates of many heads, in clusters of four and two."""
    n, T = 10, 1100
    c, src, dst, g = _cache(sva_mod, 1, 44, 25, H, 64, n)
    _check(c, src, dst, _weights(kind, (n + 2, H, T), g), T, H)
    c.close()


@pytest.mark.parametrize("kind", ["random", "ties"])
def test_many_heads_of_long_ranges(sva_mod, kind):
    """40 heads of 166400 candidates: 41600 a CTA, which are read again for each digit."""
    n, H, T = 16, 40, 10400
    c, src, dst, g = _cache(sva_mod, 1, 104, 100, H, 64, n)
    _check(c, src, dst, _weights(kind, (n + 2, H, T), g), T, H)
    c.close()
