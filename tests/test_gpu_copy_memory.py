"""sva_cache_copy between caches whose memory overlaps crosswise: the slots of one, the packed slots of the other."""
import pytest
import torch

from tests._packed import make_cache, random_kv, status, write

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("inside", ["source", "destination"])
def test_crosswise_overlaps_are_refused(sva_mod, packed, inside):
    """The packed slots of `inside` lie in the other cache's slots: no state goes from one to the other, whole or
    packed, and nothing is written; with packed slots of its own the same copy is made."""
    sva = sva_mod
    big = make_cache(sva, 1, 5, 7, 2, 64, 8, 2)            # its slots give the memory
    small = make_cache(sva, 1, 5, 7, 2, 64, 2, 2)
    g = torch.Generator(device="cuda").manual_seed(1)
    n = sva.packed_bytes(small.g, 2)
    at = big.nbytes // 2 // 256 * 256
    src, dst = (small, big) if inside == "source" else (big, small)
    a = write(src, (0, 1, 0), random_kv(src, g))
    b = dst.bind(0, 1, 0)
    small.set_packed(big.buf[at:at + n], 2)
    p, q = src.bind_packed(0, 1, 0), dst.bind_packed(0, 1, 0)
    if packed:
        src.pack([a], [p])
    torch.cuda.synchronize()
    before = [x.clone() for x in (big.buf, small.buf, big.packed)]
    for pair in ([([p], [q])] if packed else [([a], [b])]):
        assert status(lambda: src.copy(*pair, to=dst)) == sva.ERR_INVALID_ARGUMENT and "share" in sva.last_error()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(before, (big.buf, small.buf, big.packed)))
    small.release_packed(0, 1, 0)
    small.set_packed(torch.empty(n, dtype=torch.uint8, device="cuda"), 2)
    p, q = (small.bind_packed(0, 1, 0), q) if inside == "source" else (p, small.bind_packed(0, 1, 0))
    if packed:
        src.pack([a], [p])
        src.copy([p], [q], to=dst)
    else:
        src.copy([a], [b], to=dst)
        assert torch.equal(src.slot_pool()[a, :, :, : src.T], dst.slot_pool()[b, :, :, : dst.T])
    assert src.poll() == sva.OK and dst.poll() == sva.OK
    small.close()
    big.close()
