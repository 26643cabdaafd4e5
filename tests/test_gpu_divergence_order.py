"""The order in which a tile is summed depends on the tile alone, not on what its warp met before."""
import pytest
import torch

from tests import scoring as sc

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NEG = float("-inf")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low", [-2e30, -1e34])
def test_low_entries_behind_masked_tiles(dtype, low):
    """Few pairs have a tile a warp, many have several: behind masked tiles, or not."""
    import paper_2402_14160_b200 as rsd
    V = 30000
    tile = 4 * 32 * (4 if dtype == "f32" else 8)
    draft = sc.random_rows((1, 4, V), torch.float32, 2.0, 1)
    target = (draft + sc.random_rows((1, 4, V), torch.float32, 0.7, 2)).to(DT[dtype])
    draft = draft.to(DT[dtype])
    for rows in (draft, target):
        rows[:, :, :8 * tile:5] = NEG                           # the first eight tiles: masked in both
    draft[:, :2, 8 * tile + 3::tile] = low                      # all others: one entry in one row
    target[:, 2:, 8 * tile + 3::tile] = low
    want = rsd.rsd_row_divergence(draft, target)
    reference = sc.divergences(draft, target, 1.0, 1.0)
    for k in ("kl", "reverse_kl", "overlap"):
        sc.close(want[k], reference[k][0], reference[k][1], k)
    g = torch.ones((1, 4)).cuda()
    grad = rsd.rsd_row_divergence_backward(draft, target, g, g)
    for n in (10, 40, 100, 400):
        d, t = draft.expand(n, 4, V), target.expand(n, 4, V)
        got = rsd.rsd_row_divergence(d, t)
        assert all(torch.equal(got[k], want[k].expand_as(got[k])) for k in got), n
        got = rsd.rsd_row_divergence_backward(d, t, g.expand(n, 4).contiguous(), g.expand(n, 4).contiguous())
        assert all(torch.equal(got[k], grad[k].expand_as(got[k])) for k in got), n
