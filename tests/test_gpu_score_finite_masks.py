"""Rows masked with a large negative number in place of -inf, and rows that lie far from 0 altogether: whole tiles of them, through all calls."""
import math

import pytest
import torch

from tests import score_bounds as sb
from tests import scoring as sc

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
V = 9001                                                        # five tiles of bf16 entries and more, nine of fp32


@pytest.fixture(scope="module")
def rsd():
    import paper_2402_14160_b200 as m
    m.lib()
    return m


def _tokens(shape, seed):
    return torch.randint(0, V, shape, generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()


def _places():
    """Which entries are masked: tiles in front, behind and between, nearly all, at random, all."""
    x = torch.arange(V)
    g = torch.Generator().manual_seed(3)
    kept = torch.randperm(V, generator=g)[:20]
    few = torch.ones(V, dtype=torch.bool)
    few[kept] = False
    return torch.stack([x >= V // 2, x < 4200, (x >= 2048) & (x < 6200), few, torch.rand(V, generator=g) < 0.9, torch.ones(V, dtype=torch.bool)])[:, None].cuda()


def _check_scores(rsd, rows, T):
    token = _tokens(rows.shape[:2] + (4,), 5)
    out = rsd.rsd_token_logprobs(rows, token, top_k=7, temperature=T)
    sc.check_scores(out, rows, token, 7, T)
    assert not out["status"].any()
    many = rsd.rsd_token_logprobs(rows.repeat(60, 1, 1), token.repeat(60, 1, 1), top_k=7, temperature=T)   # (a block a row)
    assert all(torch.equal(many[k], out[k].repeat((60,) + (1,) * (out[k].dim() - 1))) for k in out)
    gen = torch.Generator().manual_seed(2)
    g, h = torch.randn(token.shape, generator=gen).cuda(), torch.randn(token.shape[:2], generator=gen).cuda()
    for entropy in (None, h):
        got = rsd.rsd_token_logprobs_backward(rows, token, g, entropy, temperature=T)
        assert not got["status"].any()
        sc.check_gradient(got["grad_rows"], *sc.score_gradient(rows, token, g, entropy, T), "gradient")


def _check_pair(rsd, draft, target, Td, Tt, both):
    out = rsd.rsd_row_divergence(draft, target, draft_temperature=Td, target_temperature=Tt)
    want = sc.divergences(draft, target, Td, Tt)
    assert not out["status"].any()
    for k in ("kl", "reverse_kl", "overlap"):
        sc.close(out[k], want[k][0], want[k][1], k)
    many = rsd.rsd_row_divergence(draft.repeat(60, 1, 1), target.repeat(60, 1, 1), draft_temperature=Td, target_temperature=Tt)
    assert all(torch.equal(many[k], out[k].repeat(60, 1)) for k in out)
    gen = torch.Generator().manual_seed(4)
    g, h = (torch.randn(draft.shape[:2], generator=gen).cuda() for _ in range(2))
    for a, b in ((g, None), (None, h), (g, h)) if both else ((g, None),):
        got = rsd.rsd_row_divergence_backward(draft, target, a, b, draft_temperature=Td, target_temperature=Tt)
        assert not got["status"].any()
        sc.check_gradient(got["grad_draft"], *sb.divergence_gradient(draft, target, a, b, Td, Tt), "gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [-1e4, -1e9, -1e10, -1e12, -1e20, -1e27])
@pytest.mark.parametrize("T", [0.1, 0.3, 1.0])
def test_scores_of_rows_masked_with_a_number(rsd, dtype, mask, T):
    where = _places()
    rows = sc.random_rows(where.shape, DT[dtype], 2.0, 1)
    _check_scores(rsd, torch.where(where, torch.full_like(rows, mask), rows), T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [-1e4, -1e9, -1e10, -1e12, -1e20, -1e27])
@pytest.mark.parametrize("T", [0.1, 0.3, 1.0])
def test_divergences_of_rows_masked_with_a_number(rsd, dtype, mask, T):
    where = _places()
    draft = sc.random_rows(where.shape, torch.float32, 2.0, 1)
    target = (draft + sc.random_rows(where.shape, torch.float32, 0.7, 2)).to(DT[dtype])
    draft = draft.to(DT[dtype])
    masked_draft, masked_target = (torch.where(where, torch.full_like(r, mask), r) for r in (draft, target))
    _check_pair(rsd, masked_draft, masked_target, T, T, True)
    _check_pair(rsd, masked_draft, target, T, T, False)
    _check_pair(rsd, draft, masked_target, T, T, False)
    other = torch.where(where, torch.full_like(target, 3 * mask), target)
    _check_pair(rsd, masked_draft, other, T, T, False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("far", [1e9, -1e9, 1e10, -1e10, 1e12, 1e20, -1e27])
def test_rows_that_lie_far_from_zero(rsd, dtype, far):
    """Entries a few steps of their type apart, at a temperature of a few steps."""
    step = 2.0 ** (math.floor(math.log2(abs(far))) - (23 if dtype == "f32" else 7))
    g = torch.Generator().manual_seed(7)
    draft, target = ((far + step * torch.randint(0, 40, (2, 3, V), generator=g).double()).to(DT[dtype]).cuda() for _ in range(2))
    for T in (0.5 * step, 3 * step):
        _check_scores(rsd, draft, T)
        _check_pair(rsd, draft, target, T, T, True)
        near = sc.random_rows(draft.shape, DT[dtype], 2.0, 3)   # beside an ordinary row
        _check_pair(rsd, draft, near, T, 1.0, True)
        _check_pair(rsd, near, draft, 1.0, T, True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_emitted_tokens_of_masked_rows(rsd, dtype):
    where = _places()
    rows = sc.random_rows(where.shape, DT[dtype], 2.0, 1)
    rows = torch.where(where, torch.full_like(rows, -1e10), rows).view(1, 6, V)
    token = _tokens((1, 6), 5)
    walked = dict(accepted_len=torch.tensor([5], dtype=torch.int32).cuda(), accepted_node=torch.arange(1, 6, dtype=torch.int32).cuda()[None],
                  accepted_token=token[:, :5].contiguous(), last_token=token[:, 5].contiguous())
    out = rsd.rsd_emitted_logprobs(rows, walked, top_k=5, temperature=0.3)
    sc.check_scores(out, rows, token, 5, 0.3)
    assert not out["status"].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3.0, 1e3, 1e37, 3e38])
def test_rows_over_the_whole_range(rsd, dtype, T):
    """Differences of two entries beyond the type's range, at temperatures that bring them back into it."""
    most = torch.finfo(DT[dtype]).max
    g = torch.Generator().manual_seed(9)
    draft, target = ((most * (2 * torch.rand((2, 3, V), generator=g).double() - 1)).to(DT[dtype]).cuda() for _ in range(2))
    draft[0, 0, 4500:], draft[0, 0, 4000] = -most, most         # a whole tile and more
    target[0, 1, :4500], target[0, 1, 5000] = -most, most
    draft[1], target[1] = torch.where(draft[1] > 0, most, -most).to(DT[dtype]), torch.where(target[1] > 0, most, -most).to(DT[dtype])
    _check_scores(rsd, draft, T)
    _check_pair(rsd, draft, target, T, T, True)
