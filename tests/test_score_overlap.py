"""Gradients may not lie over the rows that they are taken of: refused by the ranges of memory, before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2402_14160_b200 import api

PTR = 1 << 24    # an address that no check looks behind


def _rows(data=PTR, dtype=api.RSD_F32, seq=256, row=64):
    return C.byref(api.RsdRows(data, dtype, 0, seq, row, 1.0))


def _refused(grad, B=3, R=2, V=64, **rows):
    """As the rows of each call that writes a gradient."""
    lib, other = api.lib(), dict(rows, data=PTR * 1024)
    for code in (lambda: lib.rsd_token_logprobs_backward(_rows(**rows), B, R, V, PTR, 1, PTR, None, grad, PTR, None),
                 lambda: lib.rsd_row_divergence_backward(_rows(**rows), _rows(**other), B, R, V, PTR, None, grad, PTR, None),
                 lambda: lib.rsd_row_divergence_backward(_rows(**other), _rows(**rows), B, R, V, PTR, None, grad, PTR, None)):
        got = code()
        assert got == 1 and b"overlap" in lib.rsd_last_error(), (got, lib.rsd_last_error())


# rows of 64 fp32 entries, two a sequence 256 bytes apart, sequences 1024 bytes apart; a gradient of 3 x 2 x 256 = 1536 bytes
@pytest.mark.parametrize("grad", [PTR, PTR + 4, PTR - 4, PTR - 1532, PTR + 508, PTR + 1024, PTR + 2556, PTR + 2048 + 256])
def test_over_the_rows(grad):
    _refused(grad)


def test_over_rows_with_gaps():
    gap = dict(seq=4096, row=64)                                # 512 bytes of rows every 16 KB
    for grad in (PTR + 508, PTR + 16384 - 1532, PTR + 16384 * 2 + 508):
        _refused(grad, **gap)
    wide = dict(seq=0, row=1024)                                # rows of 256 bytes every 4 KB, one sequence for all
    for grad in (PTR + 252, PTR + 4096 - 1532, PTR + 4096 + 252):
        _refused(grad, **wide)
    half = dict(dtype=api.RSD_BF16)
    for grad in (PTR - 766, PTR + 1278):
        _refused(grad, **half)
    far = dict(seq=1 << 40, row=1 << 33)                        # offsets beyond 32 bits
    _refused(PTR + 4 * ((2 << 40) + (1 << 33)), **far)
    _refused(PTR + 4 * ((2 << 40) + (1 << 33)) + 252, **far)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_beside_and_between_the_rows(dtype):
    """Memory that belongs to no row may hold the gradient: behind, in front, between sequences, between rows, in the target's rows that have no partner."""
    from tests import scoring as sc
    B, R, V = 3, 2, 64
    n = B * R * V
    arena = torch.empty(1 << 16, dtype=dtype, device="cuda")
    token = torch.randint(0, V, (B, R), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    w = torch.ones((B, R)).cuda()
    for seq, row, places in ((R * V, V, (8192 - n, 8192 + n)), (2048, V, (8192 + R * V, 8192 + 2048 - n, 8192 + 2 * 2048 + R * V)), (0, 1024, (8192 + V, 8192 + 1024 - n, 8192 + 1024 + V))):
        rows = arena.as_strided((B, R, V), (seq, row, 1), 8192)
        for at in places:
            arena.copy_(sc.random_rows((1 << 16,), dtype, 2.0, 3))
            other = arena[:n].view(B, R, V) + 1
            want = api.rsd_token_logprobs_backward(rows, token, w)["grad_rows"], api.rsd_row_divergence_backward(rows, other, w)["grad_draft"], api.rsd_row_divergence_backward(other, rows, w)["grad_draft"]
            grad = arena[at:at + n].view(B, R, V)
            out = dict(status=torch.empty_like(token))
            assert torch.equal(api.rsd_token_logprobs_backward(rows, token, w, out=dict(out, grad_rows=grad))["grad_rows"], want[0])
            assert torch.equal(api.rsd_row_divergence_backward(rows, other, w, out=dict(out, grad_draft=grad))["grad_draft"], want[1])
            assert torch.equal(api.rsd_row_divergence_backward(other, rows, w, out=dict(out, grad_draft=grad))["grad_draft"], want[2])
        with pytest.raises(api.RsdError, match="overlap"):
            api.rsd_token_logprobs_backward(rows, token, w, out=dict(out, grad_rows=arena[8192 + V - 1:8192 + V - 1 + n].view(B, R, V)))
    target = arena.as_strided((1, 40, V), (40 * V, V, 1), 8192)
    draft = arena[:R * V].view(1, R, V)
    want = api.rsd_row_divergence_backward(draft, target, w[:1])["grad_draft"]
    grad = arena[8192 + 30 * V:8192 + 32 * V].view(1, R, V)
    assert torch.equal(api.rsd_row_divergence_backward(draft, target, w[:1], out=dict(status=torch.empty_like(token[:1]), grad_draft=grad))["grad_draft"], want)
