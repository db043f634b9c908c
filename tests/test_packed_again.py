"""What was read back, packed again: the same bytes for every largest magnitude of a group but the two just at 2^-120,
whose scale times 7 is below it."""
import pytest
import torch

from tests._packed import held, make_cache, write


def _groups():
    """[n][32]: groups led by every positive bf16 number from 2^-122 to below 2^124, with smaller ones of either sign
    behind it; and whether they may change when packed again."""
    a = torch.arange(0x0280, 0x7D80, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    assert a[0] == 2.0 ** -122 and a[-1] == 2.0 ** 124 * (1 - 2.0 ** -8)
    g = torch.Generator().manual_seed(1)
    x = (a[:, None].double() * (2 * torch.rand((len(a), 32), generator=g) - 1)).bfloat16()
    x[:, 7] = a
    low = (a.double() >= 2.0 ** -120) & (a.double() < 2.0 ** -120 * (1 + 2.0 ** -6))
    assert low.sum() == 2
    return x, low


def test_by_the_definition():
    x, low = _groups()
    once = held(x)
    again = held(once.bfloat16())
    assert torch.equal(again[~low], once[~low])
    assert (again[low] == 0).all() and (once[low, 7] == 0.984375 * 2.0 ** -120).all()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_on_the_gpu(sva_mod, d):
    x, low = _groups()
    T = 256
    H = -(-x.shape[0] // (2 * T * d // 32))
    n = 2 * H * T * d // 32
    c = make_cache(sva_mod, 1, 16, 16, H, d, 2, 2)
    full = torch.zeros((n, 32), dtype=torch.bfloat16)
    full[:x.shape[0]] = x
    s = write(c, (0, 1, 0), full.view(2, H, T, d).cuda())
    p = [c.bind_packed(0, 1, i) for i in range(2)]
    back = c.bind(0, 1, 1)
    pool = c.slot_pool()
    c.pack([s], p[:1])
    c.unpack(p[:1], [back])
    once = pool[back, :, :, :T].reshape(n, 32).double()
    assert torch.equal(once.cpu(), held(full))
    c.pack([back], p[1:])
    c.unpack(p[1:], [back])
    again = pool[back, :, :, :T].reshape(n, 32).double().cpu()
    keep = torch.cat((~low, torch.ones(n - len(low), dtype=torch.bool)))
    assert torch.equal(again[keep], once.cpu()[keep]) and (again[~keep] == 0).all()
    c.close()
