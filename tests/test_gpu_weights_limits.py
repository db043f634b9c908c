"""sva_attend_weights at the limits with masks: 64 nodes of 16 contexts, so that a unit's bitmaps of (node, Q tile)
run over several words, and contexts hidden under a history mask."""
import pytest
import torch

from test_gpu_attend_weights import Case

pytestmark = pytest.mark.gpu


def _nodes(n, W):
    ctx = [(0, W - r, 0) for r in range(W)]
    return [((0, W + 1, j), ctx) for j in range(n)]


@pytest.mark.parametrize("Hp,Wp,kinds,causal", [
    (5, 9, ("tile",), False),                # one Q tile a node: 64 bits
    (5, 9, ("hist",), False),
    (15, 20, ("tile",), False),              # three: 192 bits, more units than SMs
    (15, 20, ("tile", "own", "hist"), True),
])
def test_nodes_and_contexts(sva_mod, Hp, Wp, kinds, causal):
    n, W = 64, 16
    hidden = {(0, 3), (7, 0), (31, 15), (32, 0), (63, 15)} | {(i, 5) for i in range(n)}    # 5: nobody sees it
    c = Case(sva_mod, 1, Hp, Wp, 5 if Hp > 5 else 1, 64, _nodes(n, W), causal=causal, hidden=hidden)
    T, nt = c.T, -(-c.T // 128)
    tile = own = hist = None
    if "tile" in kinds:
        tile = torch.rand((n, nt, (1 + W) * nt), generator=c.g, device="cuda") < 0.4
        tile[33] = False                     # a node that sees nothing at all
        tile[:, :, 2 * nt] = False           # a key tile that nothing sees
    if "own" in kinds:
        own = torch.rand((n, T, T), generator=c.g, device="cuda") < 0.4
    if "hist" in kinds:
        hist = torch.rand((n, T, W, T), generator=c.g, device="cuda") < 0.4
        hist[:, 11] = False
        hist[40:, :, 2] = False
    c.check(tile=tile, own=own, hist=hist)
    c.close()


def test_hidden_contexts_under_a_history_mask(sva_mod):
    """The mask's states are numbered as listed, hidden ones too; a hidden state's bits say nothing."""
    n, W = 2, 3
    nodes = [((0, 5, 2), [(0, 4, 0), (0, 3, 0), (0, 2, 0)]), ((0, 4, 1), [(0, 3, 0), (0, 2, 0), (0, 1, 0)])]
    c = Case(sva_mod, 1, 13, 27, 3, 128, nodes, hidden={(0, 1), (1, 0), (1, 2)})
    hist = torch.rand((n, c.T, W, c.T), generator=c.g, device="cuda") < 0.5
    first = c.check(hist=hist)
    other = hist.clone()
    other[0, :, 1], other[1, :, 0], other[1, :, 2] = True, ~hist[1, :, 0], False
    again = c.check(hist=other)
    assert torch.equal(first, again)
    c.close()
