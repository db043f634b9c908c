"""Outputs that share memory with an input are refused, and nothing is launched: the kernels write while other
CTAs still read."""
import pytest
import torch

from test_gpu_attend_weights import Case, _chain, _pack
from test_gpu_condense import _cache

pytestmark = pytest.mark.gpu


def _at(buf, byte, shape, dtype):
    """A tensor of `dtype` that starts at byte `byte` of `buf`."""
    n = 1
    for s in shape:
        n *= s
    size = torch.empty((), dtype=dtype).element_size()
    return buf[byte:byte + n * size].view(dtype).view(shape)


def test_weights_out(sva_mod):
    """330 tokens, 2 heads: out against every input, from its first and from its last bytes; prev itself is allowed."""
    c = Case(sva_mod, 3, 10, 11, 2, 64, _chain(2, 2))
    T, n = c.T, 2
    out_bytes = 4 * c.shape[0] * c.shape[1] * c.shape[2]
    masks = dict(tile_mask=_pack(torch.ones((n, 3, 9), dtype=torch.bool, device="cuda")),
                 own_mask=_pack(torch.ones((n, T, T), dtype=torch.bool, device="cuda")),
                 hist_mask=_pack(torch.ones((n, T, 2, T), dtype=torch.bool, device="cuda")))
    c.attend()
    args = dict(q=c.q, lse=c.lse, prev=torch.rand(c.shape, generator=c.g, device="cuda"), **masks)
    good = torch.full(c.shape, -7.0, device="cuda")
    c.cache.attend_weights(c.nodes, out=good, decay=0.5, **args)
    for name, t in args.items():
        size = t.numel() * t.element_size()
        gap = 16
        for first in (0, 1):        # out before the input, behind it: one row of bytes in common, then none
            for common in (16, 0):
                buf = torch.zeros(out_bytes + size + 2 * gap, dtype=torch.uint8, device="cuda")
                lo, hi = gap, gap + (size if first else out_bytes) - common
                moved = _at(buf, lo if first else hi, t.shape, t.dtype)
                out = _at(buf, hi if first else lo, c.shape, torch.float32)
                out.fill_(-7.0)
                moved.copy_(t)
                before = buf.clone()
                call = dict(args, **{name: moved})
                if common:
                    with pytest.raises(sva_mod.SvaError) as e:
                        c.cache.attend_weights(c.nodes, out=out, decay=0.5, **call)
                    assert e.value.status == sva_mod.ERR_INVALID_ARGUMENT and name in str(e.value)
                    torch.cuda.synchronize()
                    assert torch.equal(buf, before)
                else:
                    c.cache.attend_weights(c.nodes, out=out, decay=0.5, **call)
                    assert torch.equal(out, good)
    acc = args["prev"].clone()
    acc[good == -7.0] = -7.0        # the spare slot, which nothing sees
    c.cache.attend_weights(c.nodes, out=acc, decay=0.5, **dict(args, prev=acc))
    assert torch.equal(acc, good)
    assert c.cache.poll() == sva_mod.OK
    c.close()


def test_condense_index(sva_mod):
    """The index over the first and the last bytes of the weights, and next to them on either side."""
    F, Hp, Wp, H, d, n = 1, 6, 8, 2, 64, 3
    T = F * Hp * Wp
    c, src, dst, g = _cache(sva_mod, F, Hp, Wp, H, d, n)
    w = torch.rand((n + 2, H, T), generator=g, device="cuda")
    good, good_w = torch.empty((H, T), dtype=torch.int32, device="cuda"), w.clone()
    c.condense(src, dst, good_w, good)
    pool = c.slot_pool().view(torch.int16)
    index_bytes, size = 4 * H * T, 4 * w.numel()
    for first in (0, 1):
        for common in (16, 0):
            buf = torch.zeros(index_bytes + size, dtype=torch.uint8, device="cuda")
            hi = (size if first else index_bytes) - common
            weight = _at(buf, 0 if first else hi, w.shape, torch.float32)
            index = _at(buf, hi if first else 0, (H, T), torch.int32)
            index.fill_(-5)
            weight.copy_(w)
            before, before_pool = buf.clone(), pool.clone()
            if common:
                with pytest.raises(sva_mod.SvaError) as e:
                    c.condense(src, dst, weight, index)
                assert e.value.status == sva_mod.ERR_INVALID_ARGUMENT
                torch.cuda.synchronize()
                assert torch.equal(buf, before) and torch.equal(pool, before_pool)
            else:
                c.condense(src, dst, weight, index)
                assert torch.equal(index, good) and torch.equal(weight, good_w)
    c.close()
