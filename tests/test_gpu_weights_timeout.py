"""Masked launches of sva_attend_weights whose waits run out: a Q tile is withheld in every CTA (a host-armed hook,
0.2 s), so the MMA warps' wait expires while copies, token words and a claim on another unit may be in flight.

Every unit of the first test has two Q tiles or more in the CTA that sums it up, so none ever is: the status is the
timeout, nothing is written, and the next launch gives the bits of the launch before.
"""
import pytest
import torch

from test_gpu_attend_weights import Case, _chain, _pack

pytestmark = pytest.mark.gpu


def _masks(c, n, W, kinds):
    """Masks that leave something of every tile: random tiles of the history only, random bits, a band of bits."""
    T, nt = c.T, -(-c.T // 128)
    m = {}
    if "tile" in kinds:
        tile = torch.rand((n, nt, (1 + W) * nt), generator=c.g, device="cuda") < 0.5
        tile[:, :2] = True                    # every key tile has the first two query tiles
        m["tile_mask"] = _pack(tile)
    if "own" in kinds:
        m["own_mask"] = _pack(torch.rand((n, T, T), generator=c.g, device="cuda") < 0.5)
    if "hist" in kinds:
        m["hist_mask"] = _pack(torch.rand((n, T, max(W, 1), T), generator=c.g, device="cuda") < 0.5)
    return m


@pytest.mark.parametrize("F,Hp,Wp,H,d,n,W,kinds", [
    (4, 5, 55, 20, 64, 2, 3, ("tile",)),             # more units than SMs: CTAs take others' units
    (4, 5, 55, 20, 128, 2, 3, ("tile",)),
    (4, 5, 55, 20, 64, 2, 3, ("own", "hist")),       # the same with token words on their way
    (4, 5, 55, 20, 128, 2, 3, ("tile", "own", "hist")),
    (1, 39, 50, 12, 64, 2, 3, ("own", "hist")),      # long enough for the scan of the masks
    (1, 40, 50, 1, 64, 1, 0, ("own",)),              # a cluster shares a unit's queries, two Q tiles a CTA
    (1, 40, 50, 1, 128, 1, 0, ("tile", "own")),
    (1, 20, 25, 20, 64, 1, 1, ("hist",)),            # a CTA a unit, fewer than SMs
    (1, 20, 25, 3, 64, 1, 1, ("hist",)),             # clusters of two
])
def test_masked(sva_mod, F, Hp, Wp, H, d, n, W, kinds):
    c = Case(sva_mod, F, Hp, Wp, H, d, _chain(n, W))
    masks = _masks(c, n, W, kinds)
    c.attend(masks.get("tile_mask"), masks.get("own_mask"), masks.get("hist_mask"))
    good = torch.full(c.shape, -7.0, device="cuda")
    c.cache.attend_weights(c.nodes, c.q, c.lse, good, **masks)
    assert c.cache.poll() == sva_mod.OK
    assert torch.any(good != -7.0)
    for _ in range(2):
        out = torch.full(c.shape, -7.0, device="cuda")
        c.cache.debug_inject(2, 0.2)
        c.cache.attend_weights(c.nodes, c.q, c.lse, out, **masks)
        assert c.cache.poll() == sva_mod.ERR_DEVICE_TIMEOUT
        assert torch.all(out == -7.0)
        c.cache.debug_inject(0, 1.0)
        c.cache.attend_weights(c.nodes, c.q, c.lse, out, **masks)
        assert c.cache.poll() == sva_mod.OK
        assert torch.equal(out, good)
    c.close()


@pytest.mark.parametrize("H,W", [(20, 3), (2, 1)])
def test_frame_causal(sva_mod, H, W):
    """Units of the own chunk's last keys have few Q tiles and may be whole: every sum is whole or untouched."""
    c = Case(sva_mod, 4, 5, 55, H, 64, _chain(1, W), causal=True)
    c.attend()
    good = torch.full(c.shape, -7.0, device="cuda")
    c.cache.attend_weights(c.nodes, c.q, c.lse, good)
    assert c.cache.poll() == sva_mod.OK
    out = torch.full(c.shape, -7.0, device="cuda")
    c.cache.debug_inject(2, 0.2)
    c.cache.attend_weights(c.nodes, c.q, c.lse, out)
    assert c.cache.poll() == sva_mod.ERR_DEVICE_TIMEOUT
    assert torch.all((out == -7.0) | (out == good))
    assert torch.any(out != good)
    c.cache.debug_inject(0, 1.0)
    c.cache.attend_weights(c.nodes, c.q, c.lse, out)
    assert c.cache.poll() == sva_mod.OK
    assert torch.equal(out, good)
    c.close()
