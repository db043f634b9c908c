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


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("masks", [(), ("tile",), ("own", "hist"), ("tile", "own", "hist")])
def test_hidden_packed_states_leave_the_bits_alone(sva_mod, d, masks):
    """Nodes that list whole states and packed ones, all of these hidden: the bits of sva_attend_nodes_masked over the
    whole ones at the same places of the list, with a space (not written) and without."""
    sva = sva_mod
    c = make_cache(sva, 1, 16, 20, 3, d, 7, 2)
    g = torch.Generator(device="cuda").manual_seed(2)
    p = [_packed(c, g, (0, 1 + i, 0)) for i in range(2)]
    twin = [write(c, (0, 1 + i, 0), random_kv(c, g)) for i in range(2)]      # hidden as well, other values
    whole = [write(c, (0, 3 + i, 0), random_kv(c, g)) for i in range(2)]
    own = [write(c, (0, 5 + i, 0), random_kv(c, g)) for i in range(2)]
    visible = [1, 0, 1, 0]

    def nodes(hidden):
        ctx = [whole[0], hidden[0], whole[1], hidden[1]]
        return sva.make_nodes([dict(seq=0, chunk=5 + i, level=0, own_slot=own[i], ctx=ctx, visible=visible) for i in range(2)])

    nt, words = 3, 10
    bits = lambda *s: torch.randint(-2 ** 31, 2 ** 31, s, generator=g, device="cuda", dtype=torch.int64).to(torch.int32)  # noqa: E731
    every = dict(tile=("tile_mask", bits(2, nt, 1)), own=("own_mask", bits(2, c.T, words)),
                 hist=("hist_mask", bits(2, c.T, 4, words)))
    kw = dict(every[m] for m in masks)
    q = torch.randn((2, c.T, c.H, d), generator=g, device="cuda").bfloat16()

    def run(call, hidden, **more):
        out, lse = torch.full_like(q, float("nan")), torch.full((2, c.H, c.T), float("nan"), device="cuda")
        call(nodes(hidden), q, out, lse, **kw, **more)
        return out, lse

    want = run(c.attend_nodes_masked, twin)
    space = torch.full((2 * 2 * c.H * c.Tpad * d * 2,), 255, dtype=torch.uint8, device="cuda")
    for got in (run(c.attend_nodes_packed, p), run(c.attend_nodes_packed, p, space=space)):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert (space == 255).all() and c.poll() == sva.OK
    c.close()
