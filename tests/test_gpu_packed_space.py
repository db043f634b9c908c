"""What sva_attend_packed_space advises follows the split that the launch gets.

Launches of one node over packed states, each measured both ways (states unpacked by the work units / into a space
first) with the states in L2 and after a flush; only launches where one way wins, or where both are as good and a
neighbour in size must not flip the advice."""
import pytest
import torch

from tests._packed import make_cache, random_kv, write

pytestmark = pytest.mark.gpu

# (tokens as rows x columns of patches, H, d, packed states, workspace) -> unpacked first?
CASES = [
    # no workspace, so no split: each unit walks all tiles.  93.0 / 82.4 us (94.7 / 84.0 after a flush)
    ((16, 20), 12, 128, 16, False, True),
    ((16, 40), 8, 128, 8, False, True),      # 77.6 / 65.5 (80.2 / 67.2)
    ((16, 40), 12, 128, 3, False, True),     # 36.2 / 33.8 (38.1 / 35.4)
    ((32, 40), 8, 64, 8, False, True),       # 103.8 / 93.6 (125.4 / 95.6)
    ((32, 40), 12, 64, 3, False, True),      # 47.5 / 46.1 (55.8 / 47.3)
    # with one, 24 units split over clusters
    ((16, 20), 12, 128, 8, True, False),     # 21.7 / 23.0 (23.1 / 24.6)
    # 72 units in clusters of two; 78 in three ranges through the workspace, two waves
    ((16, 40), 24, 128, 8, True, False),     # 48.3 / 51.0 (50.8 / 52.2)
    ((16, 40), 26, 128, 8, True, False),     # 73.4 / 76.0 (76.7 / 75.1)
    # a full wave and four units behind it, split four ways
    ((16, 40), 52, 64, 8, True, True),       # 70.4 / 69.6 (88.3 / 72.0)
    ((16, 20), 40, 128, 16, True, False),    # 84.0 / 95.5 (86.3 / 95.1)
]


@pytest.mark.parametrize("case", CASES)
def test_advice_follows_the_plan(sva_mod, case):
    (Hp, Wp), H, d, W, workspace, first = case
    c = make_cache(sva_mod, 1, Hp, Wp, H, d, 2, W, workspace)
    g = torch.Generator(device="cuda").manual_seed(1)
    packed = []
    for i in range(W):
        s = write(c, (0, 1 + i, 0), random_kv(c, g))
        packed.append(c.bind_packed(0, 1 + i, 0))
        c.pack([s], [packed[i]])
        c.release(0, 1 + i, 0)
    own = write(c, (0, 30, 0), random_kv(c, g))
    nodes = sva_mod.make_nodes([dict(seq=0, chunk=30, level=0, own_slot=own, ctx=packed)])
    want = W * 2 * H * c.Tpad * d * 2 if first else 0
    assert sva_mod.load().sva_attend_packed_space(c.handle, nodes, 1) == want
    # taken as advised, and the other way: the same bits
    q = torch.randn((1, c.T, H, d), generator=g, device="cuda").bfloat16()
    a, b = torch.empty_like(q), torch.empty_like(q)
    c.attend_nodes_packed(nodes, q, a)
    n = 0 if first else W * 2 * H * c.Tpad * d * 2
    c.attend_nodes_packed(nodes, q, b, space=torch.empty(n, dtype=torch.uint8, device="cuda"))
    assert torch.equal(a, b) and c.poll() == sva_mod.OK
    c.close()
