"""KL(p||q), KL(q||p) and their gradients where one row's logarithms are far below the other's: cold target rows, entries and tiles masked with a finite number in one row only."""
import pytest
import torch

from tests import score_bounds as sb
from tests import scoring as sc

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NEG = float("-inf")


@pytest.fixture(scope="module")
def rsd():
    import paper_2402_14160_b200 as m
    m.lib()
    return m


def _pair(shape, dtype):
    draft = sc.random_rows(shape, torch.float32, 2.0, 1)
    return draft.to(DT[dtype]), (draft + sc.random_rows(shape, torch.float32, 0.7, 2)).to(DT[dtype])


def _check(rsd, draft, target, Td=1.0, Tt=1.0):
    out = rsd.rsd_row_divergence(draft, target, draft_temperature=Td, target_temperature=Tt)
    want = sc.divergences(draft, target, Td, Tt)
    for k in ("kl", "reverse_kl", "overlap"):
        sc.close(out[k], want[k][0], want[k][1], k)
    gen = torch.Generator().manual_seed(4)
    g, h = (torch.randn(draft.shape[:2], generator=gen).cuda() for _ in range(2))
    for a, b in ((g, None), (None, h), (g, h)):
        got = rsd.rsd_row_divergence_backward(draft, target, a, b, draft_temperature=Td, target_temperature=Tt)["grad_draft"]
        sc.check_gradient(got, *sb.divergence_gradient(draft, target, a, b, Td, Tt), "gradient")
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [33, 5003, 32000])
@pytest.mark.parametrize("Tt", [1e-2, 1e-3, 1e-4])
def test_gradient_towards_a_cold_target(rsd, dtype, V, Tt):
    """ln q goes down to -16 / Tt where the draft has mass."""
    assert not _check(rsd, *_pair((2, 3, V), dtype), 1.0, Tt)["status"].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low", [-1e4, -1e5, -1e9, -1e20, -1e29])
def test_gradient_at_low_entries_of_the_target(rsd, dtype, low):
    draft, target = _pair((3, 2, 5003), dtype)
    target[:, :, 17] = low
    target[1, :, 1000:4000:3] = low
    draft[2, :, 17] = low                                       # and where neither has mass
    assert not _check(rsd, draft, target)["status"].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low", [-1e20, -1e30, -5e30, -1e35, -1e38])
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_tiles_of_one_row_masked_with_a_number(rsd, dtype, low, T):
    """Whole tiles: their sums are relative to the mask, and their logarithms count in full."""
    draft, target = _pair((5, 2, 5003), dtype)
    target[0, :, :2048] = low
    draft[1, :, 2048:] = low
    target[2, :, 3000:] = low
    target[2, :, 10:2000:7] = low
    draft[3, :, 1024:4096], target[3, :, 1024:4096] = -1e9, low     # no mass in either, far apart
    target[4, :, 1024:4096], draft[4, :, 1024:4096] = -1e4, low
    assert not _check(rsd, draft, target, T, T)["status"].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tiles_of_the_lowest_value(rsd, dtype):
    """Beyond fp32's range in units of a factor 2 an entry is missing, whether its tile holds others or not."""
    low = torch.finfo(DT[dtype]).min
    zd, zt = rsd.ST_ZERO_DRAFT_PROB, rsd.ST_ZERO_TARGET_PROB
    for places in (slice(0, 2048), slice(0, 5003, 2), slice(17, 18)):
        draft, target = _pair((3, 2, 5003), dtype)
        target[0, :, places] = low
        draft[1, :, places] = low
        draft[2, :, places], target[2, :, places] = low, low
        out = rsd.rsd_row_divergence(draft, target)
        assert out["status"].tolist() == [[zt] * 2, [zd] * 2, [0] * 2]
        assert torch.isinf(out["reverse_kl"][0]).all() and torch.isinf(out["kl"][1]).all()
        want = sc.divergences(draft, target, 1.0, 1.0)
        for k, rows in (("kl", (0, 2)), ("reverse_kl", (1, 2)), ("overlap", (0, 1, 2))):
            for r in rows:
                sc.close(out[k][r], want[k][0][r], want[k][1][r], k)
        g = torch.ones((3, 2)).cuda()
        got = rsd.rsd_row_divergence_backward(draft, target, g, g)
        assert got["status"].tolist() == [[zt] * 2, [0] * 2, [0] * 2]
        sc.check_gradient(got["grad_draft"][:1], *sb.divergence_gradient(draft[:1], target[:1], g[:1], None, 1.0, 1.0), "gradient without KL(p||q)")
        _check(rsd, draft, target, 2.0, 2.0)                    # (within the range)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_finite_entries_below_every_weight_keep_their_logarithm(rsd, dtype):
    """-300 beside ordinary entries has a weight far below 2^-126: as a weight it is 0, its logarithm counts where the other row has mass."""
    draft, target = _pair((2, 2, 5003), dtype)
    draft[0, :, 17] = -300.0
    target[1, :, 17] = -300.0
    draft[:, :, 20], target[:, :, 20] = NEG, -300.0             # no weight: the missing entry does not count
    out = _check(rsd, draft, target)
    assert not out["status"].any() and torch.isfinite(out["kl"]).all() and torch.isfinite(out["reverse_kl"]).all()
