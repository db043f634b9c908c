"""Which packed slots a node may read, and launches that see none of those they list."""
import pytest
import torch

from tests._packed import make_cache, random_kv, status, write

pytestmark = pytest.mark.gpu


def _packed(c, g, state):
    """A state that is packed and nowhere else."""
    s = write(c, state, random_kv(c, g))
    p = c.bind_packed(*state)
    c.pack([s], [p])
    c.release(*state)
    return p


def test_another_sequences_packed_state_is_refused(sva_mod):
    """A packed state of another sequence, resident and of an earlier chunk: CAUSALITY, visible or hidden, alone or
    beside the same (chunk, level) of the node's own sequence; nothing is written."""
    sva = sva_mod
    c = make_cache(sva, 1, 5, 7, 2, 64, 3, 4)
    g = torch.Generator(device="cuda").manual_seed(1)
    mine, other, later = _packed(c, g, (0, 4, 0)), _packed(c, g, (1, 4, 0)), _packed(c, g, (0, 9, 1))
    own = write(c, (0, 9, 0), random_kv(c, g))
    q = torch.randn((1, c.T, c.H, c.d), generator=g, device="cuda").bfloat16()
    out = torch.full_like(q, 7.0)
    for ctx, visible in (([other], [1]), ([other], [0]), ([mine, other], [1, 1]), ([other, mine], [1, 1]), ([later], [1])):
        node = sva.make_nodes([dict(seq=0, chunk=9, level=0, own_slot=own, ctx=ctx, visible=visible)])
        assert status(lambda: c.attend_nodes_packed(node, q, out)) == sva.ERR_CAUSALITY, ctx
        assert sva.load().sva_attend_packed_space(c.handle, node, 1) == 0
    torch.cuda.synchronize()
    assert (out == 7.0).all()
    c.attend_nodes_packed([dict(seq=0, chunk=9, level=0, own_slot=own, ctx=[mine])], q, out)
    assert not (out == 7.0).all() and c.poll() == sva.OK
    c.close()
