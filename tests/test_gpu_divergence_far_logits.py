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
