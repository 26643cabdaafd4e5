"""The scoring entry points refuse what they cannot take, before anything is launched (no GPU needed: the pointers are never followed)."""
import ctypes as C

import pytest
import torch

from paper_2402_14160_b200 import api

PTR = 1 << 20    # an address that no check looks behind


def _rows(dtype=api.RSD_F32, data=PTR, seq=64, row=64, temp=1.0):
    return C.byref(api.RsdRows(data, dtype, 0, seq, row, temp))


def _refused(call, code, text):
    lib = api.lib()
    got = call(lib)
    message = lib.rsd_last_error()
    assert got == code and text in message, (got, message)


TOKEN_LOGPROBS = dict(rows=None, B=1, R=2, V=64, num_rows=2, row_index=None, token=PTR, T=1, K=1, logprob=PTR, entropy=PTR, top=PTR, top_lp=PTR, status=PTR, stream=None)


@pytest.mark.parametrize("change, code, text", [
    (dict(V=0), 2, b"V = 0"), (dict(V=262145), 2, b"V = 262145"), (dict(B=-1), 1, b"B = -1"), (dict(R=0), 1, b"R = 0"), (dict(R=3), 1, b"R = 3 > num_rows"),
    (dict(num_rows=0), 1, b"num_rows"), (dict(T=-1), 2, b"T = -1"), (dict(T=33), 2, b"T = 33"), (dict(K=33), 2, b"K = 33"), (dict(K=-1), 2, b"K = -1"),
    (dict(token=None), 1, b"null"), (dict(logprob=None), 1, b"null"), (dict(top=None), 1, b"null"), (dict(top_lp=None), 1, b"null"), (dict(status=None), 1, b"null"),
    (dict(B=1 << 16, R=1 << 16, num_rows=1 << 16), 2, b"too large"), (dict(rows=dict(data=None)), 1, b"null rows"), (dict(rows=dict(dtype=5)), 2, b"dtype"),
    (dict(rows=dict(row=63)), 1, b"row_stride"), (dict(rows=dict(temp=-1.0)), 1, b"temperature"), (dict(rows=dict(temp=float("nan"))), 1, b"temperature"),
    (dict(rows=dict(data=PTR + 2)), 1, b"element boundary"), (dict(rows=dict(dtype=api.RSD_BF16, data=PTR + 1)), 1, b"element boundary")])
def test_token_logprobs(change, code, text):
    a = dict(TOKEN_LOGPROBS, **change)
    a["rows"] = _rows(**(a["rows"] or {}))
    _refused(lambda lib: lib.rsd_token_logprobs(*a.values()), code, text)


@pytest.mark.parametrize("change, code, text", [
    (dict(L=-1), 2, b"L = -1"), (dict(nodes=0), 2, b"num_nodes = 0"), (dict(nodes=4097), 2, b"num_nodes = 4097"), (dict(L=4096), 2, b"L = 4096"), (dict(node=None), 1, b"null"),
    (dict(last=None), 1, b"null"), (dict(length=None), 1, b"null"), (dict(K=33), 2, b"K = 33"), (dict(logprob=None), 1, b"null"), (dict(status=None), 1, b"null")])
def test_emitted_logprobs(change, code, text):
    a = dict(rows=_rows(), B=1, nodes=9, V=64, L=2, length=PTR, node=PTR, tok=PTR, last=PTR, K=0, out_token=None, logprob=PTR, entropy=None, top=None, top_lp=None,
             status=PTR, stream=None)
    a.update(change)
    _refused(lambda lib: lib.rsd_emitted_logprobs(*a.values()), code, text)


@pytest.mark.parametrize("change, code, text", [
    (dict(T=0), 2, b"T = 0"), (dict(T=33), 2, b"T = 33"), (dict(token=None), 1, b"null"), (dict(g=None), 1, b"null"), (dict(grad=None), 1, b"null"), (dict(status=None), 1, b"null"),
    (dict(R=0), 1, b"R = 0"), (dict(V=0), 2, b"V = 0"), (dict(), 1, b"overlap")])
def test_token_logprobs_backward(change, code, text):
    a = dict(rows=_rows(), B=1, R=2, V=64, token=PTR, T=1, g=PTR, h=None, grad=PTR, status=PTR, stream=None)
    a.update(change)
    _refused(lambda lib: lib.rsd_token_logprobs_backward(*a.values()), code, text)


@pytest.mark.parametrize("change, code, text", [
    (dict(target=_rows(api.RSD_BF16)), 2, b"same dtype"), (dict(kl=None, reverse=None, overlap=None), 1, b"null"), (dict(status=None), 1, b"null"), (dict(R=0), 1, b"R = 0"),
    (dict(V=0), 2, b"V = 0"), (dict(draft=_rows(data=PTR + 2)), 1, b"draft: not on an element"), (dict(target=_rows(data=PTR + 2)), 1, b"target: not on an element"),
    (dict(target=_rows(row=8)), 1, b"target: row_stride")])
def test_row_divergence(change, code, text):
    a = dict(draft=_rows(), target=_rows(), B=1, R=2, V=64, kl=PTR, reverse=None, overlap=None, status=PTR, stream=None)
    a.update(change)
    _refused(lambda lib: lib.rsd_row_divergence(*a.values()), code, text)


@pytest.mark.parametrize("change, code, text", [
    (dict(g=None, h=None), 1, b"null"), (dict(grad=None), 1, b"null"), (dict(status=None), 1, b"null"), (dict(target=_rows(api.RSD_BF16)), 2, b"same dtype"),
    (dict(), 1, b"overlap"), (dict(draft=_rows(data=2 * PTR)), 1, b"overlap")])
def test_row_divergence_backward(change, code, text):
    a = dict(draft=_rows(), target=_rows(), B=1, R=2, V=64, g=PTR, h=None, grad=PTR, status=PTR, stream=None)
    a.update(change)
    _refused(lambda lib: lib.rsd_row_divergence_backward(*a.values()), code, text)


def test_no_sequences_is_no_work():
    lib = api.lib()
    a = dict(TOKEN_LOGPROBS, B=0, rows=_rows())
    assert lib.rsd_token_logprobs(*a.values()) == 0
    assert lib.rsd_row_divergence(_rows(), _rows(), 0, 2, 64, PTR, None, None, PTR, None) == 0


def test_rows_on_the_host_are_refused():
    rows = torch.zeros((1, 2, 64))
    token = torch.zeros((1, 2), dtype=torch.int32)
    for call in (lambda: api.rsd_token_logprobs(rows, token), lambda: api.rsd_row_divergence(rows, rows),
                 lambda: api.rsd_token_logprobs_backward(rows, token, token.float()), lambda: api.rsd_row_divergence_backward(rows, rows, token.float())):
        with pytest.raises(api.RsdError, match="CUDA"):
            call()
