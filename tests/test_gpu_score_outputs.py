"""Outputs that the binding allocates: tensors of their own, which may be resized, saved and kept without regard to the others."""
import pytest
import torch

from tests import scoring as sc

pytestmark = pytest.mark.gpu


@pytest.fixture()
def rsd(monkeypatch):
    import paper_2402_14160_b200 as m
    from paper_2402_14160_b200 import api
    monkeypatch.setattr(api, "_new", api._plain_new)            # (as outside the tests: no guard words)
    return m


def _calls(rsd):
    rows = sc.random_rows((3, 5, 2000), torch.bfloat16, 2.0, 1)
    token = torch.randint(0, 2000, (3, 5, 3), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    one = torch.ones((3, 5)).cuda()
    return [lambda: rsd.rsd_token_logprobs(rows, token, top_k=4), lambda: rsd.rsd_token_logprobs_backward(rows, token, torch.ones((3, 5, 3)).cuda()),
            lambda: rsd.rsd_row_divergence(rows, rows), lambda: rsd.rsd_row_divergence_backward(rows, rows, one, one)]


def test_outputs_do_not_grow_over_their_neighbours(rsd):
    """An output that is resized, by itself or as the result of another operation, leaves the others alone."""
    for call in _calls(rsd):
        before = {k: v.clone() for k, v in call().items()}
        for k, v in before.items():
            for grow in (lambda t: t.resize_(4096).fill_(7), lambda t: t.resize_(16).fill_(7)):
                out = call()
                grow(out[k])
                assert all(torch.equal(out[o], before[o]) for o in out if o != k), k


def test_outputs_are_ordinary_tensors_otherwise(rsd):
    """Writing in place, views, copies to the host, other streams, use as `out`, in a graph, inside inference_mode."""
    for call in _calls(rsd):
        out = call()
        for k, v in out.items():
            if k.startswith("grad"):
                continue
            w = v.clone()
            v.add_(1)
            assert torch.equal(v, w + 1) and torch.equal(v.view(-1).reshape(v.shape), v) and torch.equal(v.cpu().cuda(), v) and torch.equal(v.detach(), v)
            assert torch.equal(v.unsqueeze(0).squeeze(0), v) and torch.equal(v.transpose(0, 1).contiguous().transpose(0, 1), v)
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                side.wait_stream(torch.cuda.default_stream())
                v.record_stream(side)
                u = v * 2
            torch.cuda.synchronize()
            assert torch.equal(u, v * 2)
        with torch.inference_mode():
            again = call()
            assert all(torch.equal(a, b) for a, b in zip(again.values(), call().values()))


def test_outputs_saved_and_kept(rsd, tmp_path):
    out = _calls(rsd)[0]()
    torch.save({k: v for k, v in out.items()}, tmp_path / "out.pt")
    back = torch.load(tmp_path / "out.pt")
    assert all(torch.equal(back[k], out[k]) for k in out)


def test_outputs_of_no_sequences_and_in_a_captured_graph(rsd):
    rows = sc.random_rows((3, 5, 2000), torch.bfloat16, 2.0, 1)
    token = torch.randint(0, 2000, (3, 5), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    one = torch.ones((3, 5)).cuda()

    def every(r, t, w):
        return [rsd.rsd_token_logprobs(r, t, top_k=3), rsd.rsd_token_logprobs_backward(r, t, w), rsd.rsd_row_divergence(r, r), rsd.rsd_row_divergence_backward(r, r, w, w)]

    for out in every(rows[:0], token[:0], one[:0]):
        assert all(v.shape[:2] == (0, 5) and v.is_cuda for v in out.values())
    want = every(rows, token, one)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = every(rows, token, one)
    for out in got:
        for v in out.values():
            v.fill_(3)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a[k], b[k]) for a, b in zip(got, want) for k in b)
