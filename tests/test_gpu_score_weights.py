"""Weights of a loss that are no numbers, infinite or large: they reach the gradient as they are."""
import pytest
import torch

from tests import score_bounds as sb
from tests import scoring as sc

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NEG, NAN, INF = float("-inf"), float("nan"), float("inf")
SHAPES = [(2, 3, 1), (2, 3, 700), (2, 3, 9001), (2, 3, 40000)]


@pytest.fixture(scope="module")
def rsd():
    import paper_2402_14160_b200 as m
    m.lib()
    return m


def _rows(shape, dtype, seed):
    rows = sc.random_rows(shape, DT[dtype], 2.0, seed)
    rows[:, :, 5::7] = NEG                                      # masked entries are reached too
    return rows


def _spoilt(clean, got, at):
    """Row `at` holds no finite entry, the others are as they were."""
    assert not torch.isfinite(got[at]).any()
    got = got.clone()
    got[at] = clean[at]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_scores(rsd, dtype, shape, bad):
    rows = _rows(shape, dtype, 1)
    token = torch.randint(0, shape[2], (2, 3, 3), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    token[:, :, 2] = -1
    gen = torch.Generator().manual_seed(3)
    g, h = torch.randn((2, 3, 3), generator=gen).cuda(), torch.randn((2, 3), generator=gen).cuda()
    clean, clean_h = (rsd.rsd_token_logprobs_backward(rows, token, g, x)["grad_rows"] for x in (None, h))
    g_bad, h_bad = g.clone(), h.clone()
    g_bad[0, 1, 1] = bad
    h_bad[1, 2] = bad
    _spoilt(clean, rsd.rsd_token_logprobs_backward(rows, token, g_bad)["grad_rows"], (0, 1))
    _spoilt(clean_h, rsd.rsd_token_logprobs_backward(rows, token, g_bad, h)["grad_rows"], (0, 1))
    _spoilt(clean_h, rsd.rsd_token_logprobs_backward(rows, token, g, h_bad)["grad_rows"], (1, 2))
    got = rsd.rsd_token_logprobs_backward(rows, token, torch.where(token < 0, bad, g), h)["grad_rows"]     # an absent token's weight is not used
    assert torch.equal(got, clean_h)
    rows[0, 1] = NEG                                            # a row without entries has a gradient of 0
    assert not rsd.rsd_token_logprobs_backward(rows, token, g_bad, h_bad)["grad_rows"][0, 1].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_divergences(rsd, dtype, shape, bad):
    draft = _rows(shape, dtype, 1)
    target = (draft.float() + sc.random_rows(shape, torch.float32, 0.7, 2)).to(DT[dtype])
    gen = torch.Generator().manual_seed(3)
    g, h = (torch.randn((2, 3), generator=gen).cuda() for _ in range(2))
    g_bad, h_bad = g.clone(), h.clone()
    g_bad[0, 1] = h_bad[1, 2] = bad

    def gradient(a, b):
        return rsd.rsd_row_divergence_backward(draft, target, a, b)["grad_draft"]

    _spoilt(gradient(g, None), gradient(g_bad, None), (0, 1))
    _spoilt(gradient(g, h), gradient(g_bad, h), (0, 1))
    _spoilt(gradient(None, h), gradient(None, h_bad), (1, 2))
    _spoilt(gradient(g, h), gradient(g, h_bad), (1, 2))
    if shape[2] > 1:
        target[1, 2, 3] = NEG                                   # KL(p||q) is infinite: it has no gradient, whatever its weight
        assert torch.equal(gradient(g, h_bad), gradient(g, h))
    draft[0, 1] = NEG
    assert not gradient(g_bad, h)[0, 1].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e25, 1e31, 1e34, 1e37, 1e38])
@pytest.mark.parametrize("T", [1e-3, 1.0, 1e3])
def test_large_weights(rsd, dtype, size, T):
    """Factors beyond what the fast path takes, and beyond fp32's range once they are divided by the temperature: as large as the formula says, 0 where masked."""
    shape = (2, 3, 9001)
    draft = _rows(shape, dtype, 1)
    target = (draft.float() + sc.random_rows(shape, torch.float32, 0.7, 2)).to(DT[dtype])
    gen = torch.Generator().manual_seed(3)

    def weights(*n):
        return (torch.where(torch.rand(n, generator=gen) < 0.5, -1.0, 1.0) * size * (0.5 + 0.5 * torch.rand(n, generator=gen))).cuda()

    token = torch.randint(-1, shape[2], (2, 3, 3), generator=gen, dtype=torch.int32).cuda()
    g, h = weights(2, 3, 3), weights(2, 3)
    for a, b in ((g, None), (g, h), (g * 0, h)):
        got = rsd.rsd_token_logprobs_backward(draft, token, a, b, temperature=T)["grad_rows"]
        sc.check_gradient(got, *sc.score_gradient(draft, token, a, b, T), "scores")
        assert not got[:, :, 5::7][(draft[:, :, 5::7] == NEG) & ~_given(token, shape)[:, :, 5::7]].any()
    g = weights(2, 3)
    for a, b in ((g, None), (None, h), (g, h)):
        got = rsd.rsd_row_divergence_backward(draft, target, a, b, draft_temperature=T)["grad_draft"]
        sc.check_gradient(got, *sb.divergence_gradient(draft, target, a, b, T, 1.0), "divergences")
        assert not got[:, :, 5::7].any()


def _given(token, shape):
    at = torch.zeros(shape, device=token.device)
    at.scatter_(-1, token.clamp_min(0).long(), (token >= 0).float())
    return at > 0
