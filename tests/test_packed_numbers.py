"""The arithmetic of packed slots, on the CPU: the kernels' short cuts against fractions, over every pair of bf16
mantissas, and the host side of the calls that needs no GPU."""
import ctypes
from fractions import Fraction

import numpy as np
import torch

from tests._packed import held, pairs


def _scale(a):
    """The kernel's scale of a group with largest magnitude a (fp32 arrays): division by 7, half of the fifth bit
    added, the bits below it cut."""
    b = (a.astype(np.float32) / np.float32(7)).view(np.uint32) + np.uint32(1 << 18)
    return (b & np.uint32(~((1 << 19) - 1) & 0xFFFFFFFF)).view(np.float32)


def _codes(x, s):
    """The kernel's numbers: one fused multiply-add by 1 / s, a little too large (in 64 bits the product of 8 by 24
    bits is exact; what its sum with 2^23 loses is below 2^-28)."""
    inv = (np.float32(1) / s) * np.float32(1 + 2.0 ** -20)
    t = (x.astype(np.float64) * inv.astype(np.float64) + (2.0 ** 23 + 8)).astype(np.float32)
    return (t.view(np.uint32) & 15).astype(np.int64) - 8


def test_scales_of_every_mantissa():
    for e in (-120, -40, 0, 17, 123):
        for m in range(128, 256):
            a = Fraction(m, 128) * Fraction(2) ** e
            got = Fraction(float(_scale(np.array([float(a)], np.float32))[0]))
            t = a / 7
            unit = Fraction(2) ** (e - 3)
            while t / unit >= 32:
                unit *= 2
            while t / unit < 16:
                unit /= 2
            want = (t / unit + Fraction(1, 2)).__floor__() * unit
            assert got == want, (e, m)
            # 7 times the scale is a bf16 number, and so are 24 times and every multiple up to 7
            for k in (1, 2, 3, 4, 5, 6, 7, 24):
                v = np.array([float(want * k)], np.float32)
                assert (v.view(np.uint32) & 0xFFFF)[0] == 0 and np.isfinite(v[0])


def test_numbers_of_every_pair_of_mantissas():
    x = np.concatenate([np.arange(128, 256) * 2.0 ** -e for e in range(0, 13)])
    for m in range(128, 256):
        a = np.float32(m)
        s = _scale(np.array([a]))[0]
        xs = x[x <= a].astype(np.float32)
        s_int = Fraction(float(s))
        want = np.array([(Fraction(float(v)) / s_int + Fraction(1, 2)).__floor__() for v in xs])
        assert want.max() == 7 and np.array_equal(_codes(xs, s), want), m
        assert np.array_equal(_codes(-xs, s), -want), m


def test_reference_is_the_kernels_formula():
    g = torch.Generator().manual_seed(3)
    x = (torch.randn((500, 128), generator=g) * torch.exp(3 * torch.randn((500, 1), generator=g))).bfloat16()
    got = held(x)
    v = x.float().numpy().reshape(-1, 32)
    s = _scale(np.abs(v).max(1, keepdims=True))
    assert np.array_equal(got.numpy().reshape(-1, 32), _codes(v, s) * s.astype(np.float64))
    assert torch.equal(got, got.bfloat16().double())            # bf16 numbers
    assert torch.equal(held(got.bfloat16()), got)               # packed again: the same
    a = x.double().unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True)
    err = (got - x.double()).abs().unflatten(-1, (-1, 32))
    # half a step, or what the largest is above 7 steps: s is a / 7 to 2^-5
    assert (err <= a / 7 * (1 + 2.0 ** -5) / 2).all()


def test_extreme_groups():
    x = torch.zeros((7, 32), dtype=torch.bfloat16)
    x[1, 3] = 2.0 ** -121
    x[2, 3] = -(2.0 ** -120)
    x[3, 3], x[3, 4] = 2.0 ** 124 * (1 - 2.0 ** -8), 1.0
    x[4, 3] = 2.0 ** 124
    x[5, 0], x[5, 31] = float("-inf"), 1.0
    x[6, 31] = float("nan")
    v = held(x)
    assert (v[0] == 0).all() and (v[1] == 0).all() and v[2, 3] < 0 and (v[2, :3] == 0).all()
    assert torch.isfinite(v[3]).all() and v[3, 3] > 2.0 ** 123 and v[4:].isnan().all()


def test_bytes_without_a_gpu(sva_mod):
    lib = sva_mod.load()
    for H, d, F, Hp, Wp in ((12, 128, 3, 30, 52), (2, 64, 1, 8, 8), (1, 64, 1, 1, 1), (128, 128, 1, 256, 256)):
        g = sva_mod.make_geometry(H, d, F, Hp, Wp, 1, pairs(d), 64)
        tiles = -(-F * Hp * Wp // 128)
        one = 2 * H * tiles * 128 * (d // 2 + d // 16)
        assert sva_mod.packed_bytes(g, 1) == one and one % 32 == 0
        assert sva_mod.packed_bytes(g, 1 << 20) == one << 20       # past 32 bits
    g = sva_mod.make_geometry(2, 64, 1, 8, 8, 1, pairs(64), 64)
    for n in (0, -1, (1 << 20) + 1):
        assert lib.sva_packed_bytes(ctypes.byref(g), n) == 0
    bad = sva_mod.make_geometry(2, 96, 1, 8, 8, 1, (16, 16, 16), 64)
    assert lib.sva_packed_bytes(ctypes.byref(bad), 1) == 0 and lib.sva_packed_bytes(None, 1) == 0


def test_null_arguments_without_a_gpu(sva_mod):
    lib = sva_mod.load()
    one = (ctypes.c_int32 * 1)(0)
    bad = sva_mod.ERR_INVALID_ARGUMENT
    assert lib.sva_cache_set_packed(None, None, 0, 1) == bad
    assert lib.sva_cache_bind_packed(None, 0, 1, 0, one) == bad
    assert lib.sva_cache_lookup_packed(None, 0, 1, 0, one) == bad
    assert lib.sva_cache_release_packed(None, 0, 1, 0) == bad
    assert lib.sva_cache_pack(None, one, one, 1, None) == bad
    assert lib.sva_cache_unpack(None, one, one, 1, None) == bad
    assert lib.sva_cache_copy(None, one, None, one, 1, None) == bad
    assert lib.sva_attend_nodes_packed(None, None, 1, None, None, None, 0.125, None, None, 0, None) == bad
    assert lib.sva_attend_packed_space(None, None, 1) == 0
