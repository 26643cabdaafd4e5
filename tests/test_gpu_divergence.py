"""Divergences of draft rows from target rows and their gradients against the definitions in 64 bits."""
import pytest
import torch

from tests import scoring as sc

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NEG = float("-inf")


@pytest.fixture(scope="module")
def rsd():
    import paper_2402_14160_b200 as m
    m.lib()
    return m


def _pair(shape, dtype, seed, noise=0.7, offset=(0, 0), more=1):
    B, R, V = shape
    draft = sc.random_rows((B, R, V), torch.float32, 2.0, seed)
    target = sc.random_rows((B, R + more, V), torch.float32, noise, seed + 1)
    target[:, :R] += draft
    out = []
    for rows, o in ((draft, offset[0]), (target, offset[1])):
        flat = torch.empty(rows.numel() + o, dtype=DT[dtype], device="cuda")
        flat[o:] = rows.reshape(-1).to(DT[dtype])
        out.append(flat[o:].view(rows.shape))
    return out


def _check(rsd, draft, target, Td=1.0, Tt=1.0, gradients=True):
    out = rsd.rsd_row_divergence(draft, target, draft_temperature=Td, target_temperature=Tt)
    want = sc.divergences(draft, target, Td, Tt)
    for k in ("kl", "reverse_kl", "overlap"):
        sc.close(out[k], want[k][0], want[k][1], k)
    if gradients:
        gen = torch.Generator().manual_seed(draft.shape[-1])
        g, h = (torch.randn(draft.shape[:2], generator=gen).cuda() for _ in range(2))
        for a, b in ((g, None), (None, h), (g, h)):
            got = rsd.rsd_row_divergence_backward(draft, target, a, b, draft_temperature=Td, target_temperature=Tt)["grad_draft"]
            grad, bound = sc.divergence_gradient(draft, target, a, b, Td, Tt)
            sc.check_gradient(got, grad, bound, "gradient")
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 33, 511, 512, 513, 1024, 1025, 4099, 12345, 32000, 32001, 50272])
def test_rows_of_every_length(rsd, dtype, V):
    draft, target = _pair((2, 3, V), dtype, V)
    out = _check(rsd, draft, target)
    assert not out["status"].any()
    _check(rsd, draft, target, 0.7, 0.3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [131072, 262144])
def test_long_rows(rsd, dtype, V):
    _check(rsd, *_pair((1, 2, V), dtype, 3))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offsets", [(1, 0), (0, 3), (5, 2), (7, 7), (3, 6)])
def test_rows_off_every_boundary(rsd, dtype, offsets):
    for V in (3, 1000, 4099):
        draft, target = _pair((2, 3, V), dtype, V, offset=offsets)
        a, b = _check(rsd, draft, target), rsd.rsd_row_divergence(draft.clone(), target.clone())
        assert all(torch.equal(a[k], b[k]) for k in a)           # the same bits at other addresses
        g = torch.ones((2, 3)).cuda()
        x, y = (rsd.rsd_row_divergence_backward(d, t, g, g)["grad_draft"] for d, t in ((draft, target), (draft.clone(), target.clone())))
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks(rsd, dtype):
    V = 3000
    low = torch.finfo(DT[dtype]).min
    draft, target = _pair((13, 1, V), dtype, 4)
    for rows in (draft, target):
        rows[0, 0, ::3] = NEG                                   # the same tokens banned in both
        rows[1, 0, 5:] = NEG
        rows[2, 0, :2999] = NEG
        rows[10, 0, 7:] = low
        rows[11, 0, 1000:2500] = NEG                            # whole tiles without an entry
    draft[3, 0, 17] = NEG                                       # target mass where the draft has none
    target[4, 0, 17] = NEG                                      # and the other way round
    draft[5], target[6] = NEG, NEG
    draft[7], target[7] = NEG, NEG
    draft[8, 0, 9] = float("nan")
    target[9, 0, 9] = float("inf")
    draft[12, 0, 100] = NEG
    target[12, 0, 100] = -300.0                                 # mass below 2^-126 of the largest: none
    out = _check(rsd, draft, target)
    nan, none, zd, zt = rsd.ST_NAN_INPUT, rsd.ST_EMPTY_ROW, rsd.ST_ZERO_DRAFT_PROB, rsd.ST_ZERO_TARGET_PROB
    assert out["status"].flatten().tolist() == [0, 0, 0, zd, zt, none, none, none, nan | zd, nan | zt, 0, 0, 0]
    assert torch.isinf(out["kl"][3]) and torch.isinf(out["reverse_kl"][4]) and torch.isfinite(out["kl"][12])
    g = torch.ones((13, 1)).cuda()
    for h in (None, g):
        got = rsd.rsd_row_divergence_backward(draft, target, g, h)
        assert got["status"].flatten().tolist() == [0, 0, 0, 0, zt if h is not None else 0, none, none, none, nan, nan | (zt if h is not None else 0), 0, 0, 0]
        assert not got["grad_draft"][5:8].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_rows_have_no_divergence(rsd, dtype):
    draft, _ = _pair((2, 3, 5000), dtype, 4)
    out = rsd.rsd_row_divergence(draft, draft)
    assert float(out["kl"].max()) < 1e-6 and float(out["reverse_kl"].max()) < 1e-6 and float((out["overlap"] - 1).abs().max()) < 1e-5
    g = torch.ones((2, 3)).cuda()
    assert float(rsd.rsd_row_divergence_backward(draft, draft, g)["grad_draft"].float().abs().max()) == 0


@pytest.mark.parametrize("noise", [0.02, 0.1, 1.5])
def test_small_and_large_differences(rsd, noise):
    draft, target = _pair((2, 4, 32000), "f32", 6, noise)
    out = _check(rsd, draft, target)
    want = sc.divergences(draft, target, 1.0, 1.0)["kl"][0]
    assert float((out["kl"].double() - want).abs().max() / want.min()) < 2e-3      # (1e-5 of what cancels against a divergence of 2e-4 at the least)


def test_gradient_against_differences(rsd):
    V, step = 12, 1e-5
    draft, target = _pair((1, 1, V), "f32", 9)
    g, h, Td, Tt = torch.tensor([[0.75]]).cuda(), torch.tensor([[-1.5]]).cuda(), 0.8, 1.3
    got = rsd.rsd_row_divergence_backward(draft, target, g, h, draft_temperature=Td, target_temperature=Tt)["grad_draft"][0, 0]

    def value(rows):
        d = sc.divergences(rows, target, Td, Tt)
        return float(0.75 * d["kl"][0][0, 0] - 1.5 * d["reverse_kl"][0][0, 0])

    for x in range(V):
        lo, hi = draft.double(), draft.double()
        lo[0, 0, x] -= step
        hi[0, 0, x] += step
        assert abs((value(hi) - value(lo)) / (2 * step) - float(got[x])) < 3e-5


def test_layouts_and_batches(rsd):
    V = 2050
    draft, target = _pair((5, 6, V + 9), "bf16", 2)
    for d, t in ((draft[:, :, 3:3 + V], target[:, :, 3:3 + V]), (draft.transpose(0, 1)[:, :, :V], target[:, :6].transpose(0, 1)[:, :, :V]),
                 (draft[:, :4, :V], target[:, :, 1:1 + V]), (draft[:, :, :V], target[:1, :, :V].expand(5, 7, V)), (draft[:1, :, :V].expand(5, 6, V), target[:, :, :V])):
        whole = _check(rsd, d, t)
        g = torch.randn(d.shape[:2]).cuda()
        grad = rsd.rsd_row_divergence_backward(d, t, g, g)["grad_draft"]
        for a, b in ((0, 1), (2, 5)):
            part = rsd.rsd_row_divergence(d[a:b], t[a:b])
            assert all(torch.equal(part[k], whole[k][a:b]) for k in part)
            pg = g[a:b].contiguous()
            assert torch.equal(rsd.rsd_row_divergence_backward(d[a:b], t[a:b], pg, pg)["grad_draft"], grad[a:b])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_pair_has_the_same_bits_in_every_batch(rsd, dtype):
    draft, target = _pair((200, 3, 20000), dtype, 2)
    g = torch.randn((200, 3)).cuda()
    whole, grad = rsd.rsd_row_divergence(draft, target), rsd.rsd_row_divergence_backward(draft, target, g, g)["grad_draft"]
    for a, b, r in ((0, 1, 1), (5, 20, 2), (100, 200, 3)):
        pg = g[a:b, :r].contiguous()
        part, pgrad = rsd.rsd_row_divergence(draft[a:b, :r], target[a:b]), rsd.rsd_row_divergence_backward(draft[a:b, :r], target[a:b], pg, pg)["grad_draft"]
        for k in ("kl", "reverse_kl", "overlap"):
            assert torch.equal(part[k], whole[k][a:b, :r]), k
        assert torch.equal(pgrad, grad[a:b, :r])


def test_outputs_asked_for_and_refusals(rsd):
    draft, target = _pair((2, 3, 500), "f32", 3)
    whole = rsd.rsd_row_divergence(draft, target)
    for k in ("kl", "reverse_kl", "overlap"):
        out = rsd.rsd_row_divergence(draft, target, **{"want_" + o: o == k for o in ("kl", "reverse_kl", "overlap")})
        assert torch.equal(out[k], whole[k]) and all(out[o] is None for o in ("kl", "reverse_kl", "overlap") if o != k)
    g = torch.zeros((2, 3)).cuda()
    bad_calls = [lambda: rsd.rsd_row_divergence(draft, target[:, :2]), lambda: rsd.rsd_row_divergence(draft, target[:1]), lambda: rsd.rsd_row_divergence(draft, target[:, :, :499]),
                 lambda: rsd.rsd_row_divergence(draft, target.to(torch.bfloat16)), lambda: rsd.rsd_row_divergence(draft, target.cpu()), lambda: rsd.rsd_row_divergence(draft[0], target),
                 lambda: rsd.rsd_row_divergence(draft, target, want_kl=False, want_reverse_kl=False, want_overlap=False), lambda: rsd.rsd_row_divergence_backward(draft, target),
                 lambda: rsd.rsd_row_divergence_backward(draft, target, g[:1]), lambda: rsd.rsd_row_divergence_backward(draft, target, None, g.double()),
                 lambda: rsd.rsd_row_divergence_backward(draft, target, g.cpu()), lambda: rsd.rsd_row_divergence(draft, target, draft_temperature=-1.0),
                 lambda: rsd.rsd_row_divergence(draft, target[:, :1].expand(2, 3, 500))]
    for call in bad_calls:
        with pytest.raises((rsd.RsdError, ValueError)):
            call()
    assert rsd.rsd_row_divergence(draft[:0], target[:0])["kl"].shape == (0, 3)


def test_capture_and_replay(rsd):
    draft, target = _pair((3, 2, 7000), "bf16", 3)
    g = torch.randn((3, 2)).cuda()
    out, grad = rsd.rsd_row_divergence(draft, target), rsd.rsd_row_divergence_backward(draft, target, g, g)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rsd.rsd_row_divergence(draft, target, out=out)
        rsd.rsd_row_divergence_backward(draft, target, g, g, out=grad)
    for seed in (11, 12):
        d, t = _pair((3, 2, 7000), "bf16", seed)
        d[seed - 11, 0, 3] = NEG
        draft.copy_(d), target.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        want, wgrad = rsd.rsd_row_divergence(d, t), rsd.rsd_row_divergence_backward(d, t, g, g)
        assert all(torch.equal(out[k], want[k]) for k in out) and all(torch.equal(grad[k], wgrad[k]) for k in grad)
