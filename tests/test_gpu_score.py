"""Log-probabilities of tokens, entropy, likeliest tokens and their gradient against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import workloads
from tests import scoring as sc

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NEG = float("-inf")


@pytest.fixture(scope="module")
def rsd():
    import paper_2402_14160_b200 as m
    m.lib()
    return m


def _tokens(shape, V, seed):
    return torch.randint(-1, V, shape, generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()


def _score(rsd, rows, token, K, T=1.0):
    out = rsd.rsd_token_logprobs(rows, token, top_k=K, temperature=T)
    sc.check_scores(out, rows, token, K, T)
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 33, 255, 1000, 1024, 2047, 2048, 2049, 4099, 12345, 32000, 32001, 50272])
def test_scores_of_rows_of_every_length(rsd, dtype, V):
    rows = sc.random_rows((3, 4, V), DT[dtype], 2.0, V)
    for T_tokens, K, T in ((1, 5, 1.0), (32, 32, 0.7), (3, 1, 0.3), (0, 20, 1.0), (2, 0, 2.0)):
        token = _tokens((3, 4, T_tokens), V, V + K) if T_tokens else None
        out = _score(rsd, rows, token, K, T)
        few = rsd.ST_FEWER_THAN_K if K > V else 0
        assert out["status"].tolist() == [[few] * 4] * 3


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [1, 2, 3, 5, 7])
@pytest.mark.parametrize("V", [3, 1000, 4099, 32001])
def test_rows_off_every_boundary(rsd, dtype, offset, V):
    rows = sc.random_rows((2, 3, V), DT[dtype], 2.0, offset, offset)
    aligned = rows.clone()
    token = _tokens((2, 3, 2), V, 3)
    a, b = _score(rsd, rows, token, 8), rsd.rsd_token_logprobs(aligned, token, top_k=8)
    for k in a:
        assert torch.equal(a[k], b[k]), k                       # the same bits at another address
    g, h = torch.randn((2, 3, 2)).cuda(), torch.randn((2, 3)).cuda()
    x, y = (rsd.rsd_token_logprobs_backward(r, token, g, h)["grad_rows"] for r in (rows, aligned))
    assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [131072, 200003, 262144])
def test_long_rows(rsd, dtype, V):
    rows = sc.random_rows((1, 2, V), DT[dtype], 3.0, V)
    token = _tokens((1, 2, 4), V, 1)
    _score(rsd, rows, token, 32)
    _check_gradient(rsd, rows, token, True, 0.7, 9)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_that_leave_little_or_nothing(rsd, dtype):
    V = 5000
    low = torch.finfo(DT[dtype]).min
    rows = sc.random_rows((13, 1, V), DT[dtype], 2.0, 5)
    rows[0] = NEG                                              # nothing
    rows[1] = NEG
    rows[1, 0, 4999] = 3.0                                     # one entry
    rows[2, 0, 1:] = NEG
    rows[3, 0, ::2] = NEG
    rows[4] = low                                              # nothing but the type's lowest value: uniform
    rows[5, 0, 7:] = low
    rows[6] = low
    rows[6, 0, 100:] = NEG
    rows[7, 0, :4990] = NEG
    rows[8, 0, 17] = float("nan")
    rows[9, 0, 4000] = float("inf")
    rows[10] = float("nan")
    rows[11] = float("inf")
    rows[12, 0, 10:] = NEG
    rows[12, 0, 3] = float("nan")
    token = torch.tensor([[[0, 4999, 17, 3, 4000]]] * 13, dtype=torch.int32).cuda()
    out = _score(rsd, rows, token, 12)
    nan, few, none = rsd.ST_NAN_INPUT, rsd.ST_FEWER_THAN_K, rsd.ST_EMPTY_ROW
    assert out["status"].flatten().tolist() == [few | none, few, few, 0, 0, 0, 0, few, nan, nan, nan | few | none, nan | few | none, nan | few]
    assert out["entropy"][0].item() == 0 and out["entropy"][1].item() == 0
    for entropy in (False, True):
        grad = _check_gradient(rsd, rows, token, entropy, 1.0, 3)
        assert not grad[0].any() and not grad[10].any() and not grad[11].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [-3e4, -700.0, 600.0, 2e4, 1e30])
def test_rows_far_from_zero(rsd, dtype, shift):
    rows = (sc.random_rows((2, 2, 3001), torch.float32, 2.0, 8) * (abs(shift) / 300 if abs(shift) > 1e4 else 1.0) + shift).to(DT[dtype])
    token = _tokens((2, 2, 3), 3001, 4)
    _score(rsd, rows, token, 10, 1.0)
    _score(rsd, rows, token, 10, 0.3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_temperatures_from_tiny_to_huge(rsd, dtype):
    rows = sc.random_rows((1, 2, 777), DT[dtype], 2.0, 8)
    token = _tokens((1, 2, 3), 777, 4)
    for T in (1e-3, 1e-2, 100.0, 1e6):
        _score(rsd, rows, token, 10, T)
        _check_gradient(rsd, rows, token, True, T, 6)
    out = rsd.rsd_token_logprobs(rows, token, top_k=1, temperature=1e-42)      # only the largest entry is left
    assert out["entropy"].tolist() == [[0.0, 0.0]] and out["top_logprob"].flatten().tolist() == [0.0, 0.0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [64, 700, 40000, 262144])
def test_equal_values_go_to_the_smaller_token(rsd, dtype, V):
    g = torch.Generator().manual_seed(V)
    rows = torch.zeros((6, 2, V))
    rows[1] = torch.randint(-2, 3, (2, V), generator=g).float()
    rows[2, :, V // 2:] = 1.0
    rows[3, :, -5:] = 1.0
    rows[4] = torch.randint(0, 2, (2, V), generator=g).float() * -0.0          # +0 and -0 are one value
    rows[5] = -7.0
    rows[5, 1, V // 3:] = NEG
    rows = rows.to(DT[dtype]).cuda()
    for K in (1, 7, 32):
        _score(rsd, rows, _tokens((6, 2), V, K), K)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_entries_crowded_where_few_threads_look(rsd, dtype):
    """More entries above the bound than the list holds: all of them in the words of a few lanes."""
    V = 262144
    word = 16 // torch.empty((), dtype=DT[dtype]).element_size()
    rows = sc.random_rows((3, 1, V), DT[dtype], 0.1, 3)
    x = torch.arange(V)
    crowd = (x // word) % 32 < 3                                # lanes 0 to 2 of every warp
    values = 10 + torch.randperm(V, generator=torch.Generator().manual_seed(1)).float() / V * 50
    rows[0, 0, crowd] = values[crowd].to(DT[dtype]).cuda()
    crowd = ((x // word) % 32 == 0) & ((x // (word * 256)) % 8 == 0)
    rows[1, 0] = NEG
    rows[1, 0, crowd] = values[crowd].to(DT[dtype]).cuda()
    rows[2, 0, crowd] = 5.0
    for K in (1, 20, 32):
        _score(rsd, rows, _tokens((3, 1), V, K), K)


def test_given_rows_absent_slots_and_indexes_out_of_range(rsd):
    B, N, V, R = 3, 5, 1003, 7
    rows = sc.random_rows((B, N, V), torch.bfloat16, 2.0, 2)
    index = torch.tensor([[0, 4, 4, -1, 2, 1, 0], [3, 3, 3, 3, 3, 3, 3], [-1, -5, 0, 5, 1, 2, 2 ** 31 - 1]], dtype=torch.int32).cuda()
    token = _tokens((B, R, 2), V, 6)
    out = rsd.rsd_token_logprobs(rows, token, row_index=index, top_k=4)
    there = (index >= 0) & (index < N)
    picked = rows[torch.arange(B).cuda()[:, None], torch.where(there, index, 0).long()]
    full = rsd.rsd_token_logprobs(picked.contiguous(), token, top_k=4)
    for key, nothing in (("logprob", 0.0), ("entropy", 0.0), ("top_token", -1), ("top_logprob", NEG)):
        t = there.reshape(there.shape + (1,) * (out[key].dim() - 2))
        assert torch.equal(out[key], torch.where(t, full[key], torch.full_like(full[key], nothing))), key
    assert torch.equal(out["status"], torch.where(index >= N, rsd.ST_BAD_INDEX, 0))
    bad = token.clone()
    bad[1, 2, 0], bad[1, 3, 1] = V, 2 ** 31 - 1
    first = torch.zeros((B, R), dtype=torch.int32).cuda()                       # (a row that all slots share)
    out = rsd.rsd_token_logprobs(rows, bad, row_index=first)
    assert torch.equal(out["status"], torch.where((bad >= V).any(-1), rsd.ST_BAD_INDEX, 0))
    assert out["logprob"][1, 2, 0].item() == 0 and out["logprob"][1, 3, 1].item() == 0
    g = torch.ones((B, R, 2)).cuda()
    wide = rows[:1].repeat(1, 2, 1)[:, :R].expand(B, R, V)                      # (a sequence that all share)
    grads = [rsd.rsd_token_logprobs_backward(wide, t, g) for t in (bad, torch.where(bad >= V, -1, bad))]
    assert torch.equal(grads[0]["grad_rows"], grads[1]["grad_rows"]) and torch.equal(grads[0]["status"], out["status"])


def _check_gradient(rsd, rows, token, entropy, T, seed):
    gen = torch.Generator().manual_seed(seed)
    g = torch.randn(token.shape, generator=gen).cuda()
    h = torch.randn(token.shape[:2], generator=gen).cuda() if entropy else None
    got = rsd.rsd_token_logprobs_backward(rows, token, g, h, temperature=T)["grad_rows"]
    want, bound = sc.score_gradient(rows, token, g, h, T)
    sc.check_gradient(got, want, bound, "gradient")
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 33, 1000, 2048, 2049, 12345, 32000, 50272])
def test_gradient_for_rows_of_every_length(rsd, dtype, V):
    rows = sc.random_rows((2, 5, V), DT[dtype], 2.0, V)
    for T_tokens, entropy, T in ((1, False, 1.0), (1, True, 0.7), (32, True, 1.0), (4, False, 0.3)):
        _check_gradient(rsd, rows, _tokens((2, 5, T_tokens), V, V + T_tokens), entropy, T, V)


@pytest.mark.parametrize("V", [5, 40])
def test_gradient_against_differences(rsd, V):
    rows = sc.random_rows((1, 1, V), torch.float32, 1.5, 4)
    token = torch.tensor([[[2, 2, 0, -1]]], dtype=torch.int32).cuda()
    g, h, T, step = torch.tensor([[[0.5, -1.25, 2.0, 9.0]]]).cuda(), torch.tensor([[0.75]]).cuda(), 0.8, 1e-5
    got = rsd.rsd_token_logprobs_backward(rows, token, g, h, temperature=T)["grad_rows"][0, 0]

    def value(z):
        lp = sc.log_softmax(z, T)
        return float((g[0, 0, :3].double() * lp[0, 0, token[0, 0, :3].long()]).sum() + h[0, 0].double() * sc.entropy(lp)[0, 0])

    for x in range(V):
        lo, hi = rows.double(), rows.double()
        lo[0, 0, x] -= step
        hi[0, 0, x] += step
        assert abs((value(hi) - value(lo)) / (2 * step) - float(got[x])) < 2e-5       # 1e-10 / 1e-5 of cancellation, 1e-5 of the kernel


def test_gradient_of_rows_in_any_layout(rsd):
    """Transposed batches, slices of wider rows, one sequence for a whole batch: the gradient is dense, a row per row."""
    V = 2051
    base = sc.random_rows((4, 6, V + 13), torch.bfloat16, 2.0, 5)
    for rows in (base[:, :, 5:5 + V], base[1:, 2:, :V], base.transpose(0, 1)[:, :, 3:3 + V], base[:1, :, :V].expand(4, 6, V), base[:, ::2, 1:1 + V]):
        token = _tokens(rows.shape[:2] + (2,), V, 8)
        grad = _check_gradient(rsd, rows, token, True, 1.0, 2)
        assert grad.is_contiguous()
        _score(rsd, rows, token, 6)


def test_offsets_beyond_32_bits(rsd):
    V, stride = 1000, (1 << 31) + 8
    flat = torch.empty(2 * stride + 16 * V, dtype=torch.bfloat16, device="cuda")
    rows = flat.as_strided((3, 2, V), (stride, V, 1))
    rows.copy_(sc.random_rows((3, 2, V), torch.bfloat16, 2.0, 3))
    token = _tokens((3, 2), V, 4)
    _score(rsd, rows, token, 5)
    _check_gradient(rsd, rows, token, True, 1.0, 3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [900, 32000, 70001])
def test_a_row_has_the_same_bits_in_every_batch(rsd, dtype, V):
    rows = sc.random_rows((300, 3, V), DT[dtype], 2.0, 7)
    token = _tokens((300, 3, 2), V, 1)
    g, h = torch.randn((300, 3, 2)).cuda(), torch.randn((300, 3)).cuda()
    whole, grad = rsd.rsd_token_logprobs(rows, token, top_k=6), rsd.rsd_token_logprobs_backward(rows, token, g, h)["grad_rows"]
    for a, b, r in ((0, 1, 1), (7, 9, 3), (50, 150, 2), (299, 300, 3)):
        part = rsd.rsd_token_logprobs(rows[a:b, :r], token[a:b, :r].contiguous(), top_k=6)
        for k in ("logprob", "entropy", "top_token", "top_logprob"):
            assert torch.equal(part[k], whole[k][a:b, :r]), (k, a, b)
        part = rsd.rsd_token_logprobs_backward(rows[a:b, :r], token[a:b, :r].contiguous(), g[a:b, :r].contiguous(), h[a:b, :r].contiguous())["grad_rows"]
        assert torch.equal(part, grad[a:b, :r])


def test_binding_refuses_what_does_not_fit(rsd):
    rows = sc.random_rows((2, 3, 100), torch.float32, 1.0, 1)
    token = _tokens((2, 3), 100, 1)
    g = torch.zeros((2, 3)).cuda()
    for bad in (token.long(), token.cpu(), token[:1], token[:, :2].contiguous()[:, :1], token.t().contiguous().t(), token[None]):
        with pytest.raises((rsd.RsdError, ValueError)):
            rsd.rsd_token_logprobs_backward(rows, bad, g)
    with pytest.raises(rsd.RsdError, match="token"):
        rsd.rsd_token_logprobs(rows, token[:1])
    with pytest.raises(rsd.RsdError, match="row_index"):
        rsd.rsd_token_logprobs(rows, token, row_index=token.cpu())
    for bad in (g.double(), g.cpu(), g[:1], g[..., None]):
        with pytest.raises(rsd.RsdError, match="grad_logprob"):
            rsd.rsd_token_logprobs_backward(rows, token, bad)
        with pytest.raises(rsd.RsdError, match="grad_entropy"):
            rsd.rsd_token_logprobs_backward(rows, token, g, bad)
    with pytest.raises(rsd.RsdError, match="grad_rows"):
        rsd.rsd_token_logprobs_backward(rows, token, g, out=dict(grad_rows=rows.to(torch.bfloat16), status=token.clone()))
    with pytest.raises(rsd.RsdError, match="status"):
        rsd.rsd_token_logprobs_backward(rows, token, g, out=dict(grad_rows=rows.clone(), status=token[:, 0].contiguous()))
    with pytest.raises(rsd.RsdError, match="out lacks top_token"):
        rsd.rsd_token_logprobs(rows, token, top_k=2, out=rsd.rsd_token_logprobs(rows, token))
    with pytest.raises(rsd.RsdError, match="K = 33"):
        rsd.rsd_token_logprobs(rows, token, top_k=33)
    with pytest.raises(rsd.RsdError, match="T = 33"):
        rsd.rsd_token_logprobs(rows, token[..., None].expand(2, 3, 33).contiguous())
    with pytest.raises(rsd.RsdError, match="float32 or bfloat16"):
        rsd.rsd_token_logprobs(rows.half(), token)
    with pytest.raises(ValueError):
        rsd.rsd_token_logprobs(rows[0], token[0])
    with pytest.raises(rsd.RsdError, match="row_stride"):
        rsd.rsd_token_logprobs(rows[:, :1].expand(2, 3, 100), token)
    out = rsd.rsd_token_logprobs(rows[:0], token[:0], top_k=3)
    assert out["logprob"].shape == (0, 3) and out["top_token"].shape == (0, 3, 3)
    assert rsd.rsd_token_logprobs_backward(rows[:0], token[:0], g[:0])["grad_rows"].shape == (0, 3, 100)


def test_capture_replay_and_other_streams(rsd):
    rows = sc.random_rows((4, 3, 9000), torch.bfloat16, 2.0, 1)
    token = _tokens((4, 3, 2), 9000, 2)
    g = torch.randn((4, 3, 2)).cuda()
    out, grad = rsd.rsd_token_logprobs(rows, token, top_k=9), rsd.rsd_token_logprobs_backward(rows, token, g)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rsd.rsd_token_logprobs(rows, token, top_k=9, out=out)
        rsd.rsd_token_logprobs_backward(rows, token, g, out=grad)
    for seed in (5, 6):
        fresh = sc.random_rows((4, 3, 9000), torch.bfloat16, 2.0, seed)
        fresh[seed - 5, 1, 7] = float("nan")
        rows.copy_(fresh)
        graph.replay()
        torch.cuda.synchronize()
        want, wgrad = rsd.rsd_token_logprobs(fresh, token, top_k=9), rsd.rsd_token_logprobs_backward(fresh, token, g)
        assert all(torch.equal(out[k], want[k]) for k in out) and all(torch.equal(grad[k], wgrad[k]) for k in grad)
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    torch.cuda.synchronize()
    for s in streams:                                           # the same call on several streams at once
        with torch.cuda.stream(s):
            got.append((rsd.rsd_token_logprobs(rows, token, top_k=9), rsd.rsd_token_logprobs_backward(rows, token, g)))
    torch.cuda.synchronize()
    for o, b in got:
        assert all(torch.equal(o[k], want[k]) for k in o) and all(torch.equal(b[k], wgrad[k]) for k in b)


@pytest.mark.parametrize("L", [0, 1, 4])
def test_what_a_walk_emitted(rsd, L):
    B, V, W = 6, 1201, 3
    rows = sc.random_rows((B, 1 + W * L, V), torch.float32, 2.0, L)
    g = torch.Generator().manual_seed(L)
    length = torch.tensor([min(i, L) for i in range(B)], dtype=torch.int32)
    node = torch.full((B, L), -1, dtype=torch.int32)
    tok = node.clone()
    for b in range(B):
        for i in range(int(length[b])):
            node[b, i], tok[b, i] = 1 + i * W + int(torch.randint(0, W, (1,), generator=g)), int(torch.randint(0, V, (1,), generator=g))
    last = torch.randint(0, V, (B,), generator=g, dtype=torch.int32)
    last[1] = -1                                                # (an abandoned walk)
    verified = {k: v.cuda() for k, v in dict(accepted_len=length, accepted_node=node, accepted_token=tok, last_token=last).items()}
    out = rsd.rsd_emitted_logprobs(rows, verified, top_k=3, temperature=0.9)
    for b in range(B):
        n = int(length[b])
        at = [0] + node[b, :n].tolist()
        want_tok = tok[b, :n].tolist() + [int(last[b])]
        assert out["token"][b].tolist() == want_tok + [-1] * (L - n)
        one = rsd.rsd_token_logprobs(rows[b:b + 1, at].contiguous(), torch.tensor([want_tok], dtype=torch.int32).cuda(), top_k=3, temperature=0.9)
        for k, nothing in (("logprob", 0.0), ("entropy", 0.0), ("top_token", -1), ("top_logprob", NEG)):
            assert torch.equal(out[k][b, :n + 1], one[k][0]), k
            assert (out[k][b, n + 1:] == nothing).all()
    assert not out["status"].any()
    wrong = dict(verified, accepted_len=torch.tensor([-1, L + 1, 2 ** 31 - 1, 0, 0, 0], dtype=torch.int32).cuda())
    out = rsd.rsd_emitted_logprobs(rows, wrong)
    assert (out["token"][:3] == -1).all() and (out["logprob"][:3] == 0).all()
    if L:
        wrong = dict(verified, accepted_len=torch.ones(B, dtype=torch.int32).cuda(), accepted_node=torch.full((B, L), 1 + W * L, dtype=torch.int32).cuda())
        out = rsd.rsd_emitted_logprobs(rows, wrong)
        assert (out["status"][:, 1] == rsd.ST_BAD_INDEX).all() and not out["status"][:, 0].any() and (out["logprob"][:, 1] == 0).all()


@pytest.mark.parametrize("number", [2, 3])
def test_a_step_that_returns_log_probabilities(rsd, number):
    """Draft, walk and score as a server runs them; then the same rows through the divergence and its gradient."""
    from paper_2402_14160_b200 import step as rsd_step
    w = workloads.scaled(workloads.WORKLOADS[number], batch=5, vocab=4096)
    draft, target = workloads.make_logits(w, step=1, device="cuda")
    step = rsd_step.make_step(w, device="cuda")
    out = step.run(draft, target, 3, 1, logprobs=4)
    scored = step.emitted_out
    lp = sc.log_softmax(target, 1.0)
    for b in range(5):
        n = int(out["accepted_len"][b])
        tokens = out["accepted_token"][b, :n].tolist() + [int(out["last_token"][b])]
        assert scored["token"][b, :n + 1].tolist() == tokens
        nodes = [0] + out["accepted_node"][b, :n].tolist()
        want = torch.stack([lp[b, i, t] for i, t in zip(nodes, tokens)])
        sc.close(scored["logprob"][b, :n + 1], want, sc.SUM + 4 * sc.EPS * want.abs(), "emitted")
        assert torch.equal(scored["top_token"][b, :n + 1], sc.top(target[b, nodes], 4)[0])
    again = step.run(draft, target, 3, 2, logprobs=0)
    assert step.emitted_out["top_token"] is None and step.emitted_out["token"][:, 0].ge(0).all() and again is out
    near = rsd.rsd_row_divergence(draft, target)
    assert (near["kl"] > 0).all() and (near["overlap"] < 1).all() and not near["status"].any()
    g = torch.ones(draft.shape[:2]).cuda()
    got = rsd.rsd_row_divergence_backward(draft, target, g)["grad_draft"]
    sc.check_gradient(got, *sc.divergence_gradient(draft, target, g, None, 1.0, 1.0), "gradient of the drafter's rows")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1e-9, 1e-5, 1e10, 1e25, 1e35])
def test_masked_entries_at_extreme_temperatures_and_weights(rsd, dtype, T):
    """Masked entries keep weight 0 however flat the rest is, and get a gradient of 0 however large the factors are."""
    V = 3001
    rows = sc.random_rows((2, 2, V), DT[dtype], 2.0, 5)
    rows[0, 0, ::2] = NEG
    rows[1, 0, 100:] = NEG
    rows[1, 1, 5:2500] = torch.finfo(DT[dtype]).min if T == 1e-5 else NEG
    token = torch.tensor([[[1, 4, 1]] * 2] * 2, dtype=torch.int32).cuda()
    out = rsd.rsd_token_logprobs(rows, token, top_k=3, temperature=T)
    sc.check_scores(out, rows, token, 3, T)
    g = torch.tensor([[[1.0, 2.0, -0.5]] * 2] * 2).cuda()
    for size in (1.0, 1e9):
        h = torch.full((2, 2), size).cuda()
        got = rsd.rsd_token_logprobs_backward(rows, token, g, h, temperature=T)["grad_rows"]
        sc.check_gradient(got, *sc.score_gradient(rows, token, g, h, T), "gradient")
    target = (rows.float() + torch.where(rows > NEG, 1.0, 0.0) * sc.random_rows((2, 2, V), torch.float32, 0.5, 6)).to(DT[dtype])
    near = rsd.rsd_row_divergence(rows, target, draft_temperature=T, target_temperature=T)
    for k, (want, tol) in ((k, sc.divergences(rows, target, T, T)[k]) for k in ("kl", "reverse_kl", "overlap")):
        if T > 1e-4 or k == "overlap":                           # (colder, a divergence is made of differences of 1e5 and more)
            sc.close(near[k], want, tol, k)
    for size in (1.0, 1e9):
        h = torch.full((2, 2), size).cuda()
        assert torch.isfinite(rsd.rsd_row_divergence_backward(rows, target, h, h, draft_temperature=T, target_temperature=T)["grad_draft"][rows == NEG]).all()
