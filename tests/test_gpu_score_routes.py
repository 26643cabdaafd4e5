"""Every launch shape of the scoring kernels: blocks of two to eight warps, clusters of two to eight blocks, one-warp blocks.  A row's results are the same bits in all of them."""
import pytest
import torch

from tests import scoring as sc

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def rsd():
    import paper_2402_14160_b200 as m
    m.lib()
    return m


def _shape(call, kernel):
    """(threads, cluster) of the launch of `kernel` in a call"""
    from cuda.bindings import driver

    def ok(result):
        assert result[0] == driver.CUresult.CUDA_SUCCESS, result[0]
        return result[1:]

    call()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        kept = call()
    handle = driver.CUgraph(graph.raw_cuda_graph())
    _, n = ok(driver.cuGraphGetNodes(handle))
    nodes, n = ok(driver.cuGraphGetNodes(handle, n))
    found = None
    for node in nodes[:n]:
        if ok(driver.cuGraphNodeGetType(node))[0] != driver.CUgraphNodeType.CU_GRAPH_NODE_TYPE_KERNEL:
            continue
        params, = ok(driver.cuGraphKernelNodeGetParams(node))
        if kernel in ok(driver.cuFuncGetName(params.func))[0].decode():
            assert found is None, "one launch a call"
            attribute, = ok(driver.cuGraphKernelNodeGetAttribute(node, driver.CUkernelNodeAttrID.CU_LAUNCH_ATTRIBUTE_CLUSTER_DIMENSION))
            found = (params.blockDimX, max(1, attribute.clusterDim.x))
    graph.instantiate()
    graph.replay()
    torch.cuda.synchronize()
    del kept
    return found


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [0, 3])
def test_scores_are_the_same_in_every_shape(rsd, dtype, offset):
    seen = set()
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for V, most in ((1500, 20 * sms), (9000, 20 * sms), (33000, 20 * sms), (131001, 3 * sms)):
        rows = sc.random_rows((1, 1, V), DT[dtype], 2.0, V, offset).expand(most, 1, V)      # one row, as many times as asked for
        token = torch.full((most, 1, 2), V // 2, dtype=torch.int32).cuda()
        token[:, 0, 1] = -1
        want = rsd.rsd_token_logprobs(rows[:1], token[:1], top_k=7)
        sc.check_scores(want, rows[:1], token[:1], 7, 1.0)
        for n in (1, sms // 4, sms // 2, sms, 3 * sms, 6 * sms, 12 * sms, 20 * sms):
            if n > most:
                continue
            for K in (0, 7):
                shape = _shape(lambda: rsd.rsd_token_logprobs(rows[:n], token[:n], top_k=K), "score_rows_kernel")
                seen.add(shape)
                got = rsd.rsd_token_logprobs(rows[:n], token[:n], top_k=K)
                for k in ("logprob", "entropy", "status") + (("top_token", "top_logprob") if K else ()):
                    assert torch.equal(got[k], want[k].expand_as(got[k])), (V, n, K, shape, k)
    assert seen >= {(32, 1), (64, 1), (128, 1), (256, 1), (256, 2), (256, 4), (256, 8)}, seen


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [0, 3])
def test_gradients_and_divergences_are_the_same_in_every_shape(rsd, dtype, offset):
    seen = {"score_grad_kernel": set(), "divergence_kernel": set(), "divergence_grad_kernel": set()}
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for V, most in ((700, 6 * sms), (5000, 6 * sms), (12000, 6 * sms), (30000, 6 * sms), (131001, sms), (262144, sms // 2)):
        draft = sc.random_rows((1, 1, V), DT[dtype], 2.0, V, offset)
        target = (draft.float() + sc.random_rows((1, 1, V), torch.float32, 0.7, V + 1)).to(DT[dtype])
        draft, target = draft.expand(most, 1, V), target.expand(most, 1, V)
        token = torch.tensor([[[V - 1, 3, V - 1]]], dtype=torch.int32).cuda().expand(most, 1, 3).contiguous()
        g, h = torch.full((most, 1), 0.75).cuda(), torch.full((most, 1), -1.5).cuda()
        w = torch.tensor([[[1.0, -2.0, 0.5]]]).cuda().expand(most, 1, 3).contiguous()
        calls = {"score_grad_kernel": lambda n: rsd.rsd_token_logprobs_backward(draft[:n], token[:n], w[:n], h[:n]),
                 "divergence_kernel": lambda n: rsd.rsd_row_divergence(draft[:n], target[:n]),
                 "divergence_grad_kernel": lambda n: rsd.rsd_row_divergence_backward(draft[:n], target[:n], g[:n], h[:n])}
        for name, call in calls.items():
            want = call(1)
            for n in (1, sms // 8, sms // 4, sms // 2, sms, 3 * sms, 6 * sms):
                if n > most:
                    continue
                shape = _shape(lambda: call(n), name)
                seen[name].add(shape)
                got = call(n)
                for k in got:
                    assert torch.equal(got[k], want[k].expand_as(got[k])), (name, V, n, shape, k)
        sc.check_gradient(calls["score_grad_kernel"](1)["grad_rows"], *sc.score_gradient(draft[:1], token[:1], w[:1], h[:1], 1.0), "gradient")
        sc.check_gradient(calls["divergence_grad_kernel"](1)["grad_draft"], *sc.divergence_gradient(draft[:1], target[:1], g[:1], h[:1], 1.0, 1.0), "gradient")
    for name, shapes in seen.items():
        assert shapes >= {(64, 1), (128, 1), (256, 1), (256, 2), (256, 4), (256, 8)}, (name, shapes)


def test_outputs_over_one_allocation(rsd, monkeypatch):
    """What the binding allocates itself: the same results, each output in a place of its own, small ones over one allocation."""
    from paper_2402_14160_b200 import api
    rows = sc.random_rows((3, 5, 2000), torch.bfloat16, 2.0, 1)
    token = torch.randint(0, 2000, (3, 5, 3), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    g = torch.randn((3, 5, 3)).cuda()
    many = sc.random_rows((300, 200, 40), torch.float32, 2.0, 1)                 # outputs of more than a megabyte
    calls = [lambda: rsd.rsd_token_logprobs(rows, token, top_k=4), lambda: rsd.rsd_token_logprobs(rows, token[..., 0].contiguous(), want_entropy=False),
             lambda: rsd.rsd_token_logprobs_backward(rows, token, g), lambda: rsd.rsd_row_divergence(rows, rows), lambda: rsd.rsd_row_divergence_backward(rows, rows, g[..., 0].contiguous()),
             lambda: rsd.rsd_token_logprobs(many, top_k=4)]
    with_guards = [call() for call in calls]
    monkeypatch.setattr(api, "_new", api._plain_new)
    for call, want in zip(calls, with_guards):
        got = call()
        assert got.keys() == want.keys()
        spans = []
        for k, v in want.items():
            assert (got[k] is None) == (v is None)
            if v is not None:
                assert got[k].dtype == v.dtype and got[k].shape == v.shape and got[k].is_contiguous() and torch.equal(got[k], v), k
                assert got[k].data_ptr() % 16 == 0 and not got[k].requires_grad
                spans.append((got[k].data_ptr(), got[k].data_ptr() + got[k].numel() * got[k].element_size()))
        spans.sort()
        assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
    kept = rsd.rsd_token_logprobs(rows, token, top_k=4)["top_token"]            # one output outlives the others
    clone = kept.clone()
    for _ in range(20):
        rsd.rsd_token_logprobs(rows, token, top_k=4)["logprob"].fill_(7)
    assert torch.equal(kept, clone)
    kept += 1
    assert torch.equal(kept, clone + 1)


def test_clusters_in_a_captured_graph_and_on_two_streams(rsd):
    V = 131072
    rows = [sc.random_rows((2, 2, V), torch.bfloat16, 2.0, s) for s in (1, 2)]
    token = torch.randint(0, V, (2, 2, 4), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    g = torch.randn((2, 2, 4)).cuda()
    h = torch.randn((2, 2)).cuda()

    def every(a, b):
        return [rsd.rsd_token_logprobs(a, token, top_k=20), rsd.rsd_token_logprobs_backward(a, token, g, h), rsd.rsd_row_divergence(a, b), rsd.rsd_row_divergence_backward(a, b, h, h)]

    want = [every(rows[0], rows[1]), every(rows[1], rows[0])]
    a, b = rows[0].clone(), rows[1].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = every(a, b)
    for i in (1, 0, 1):
        a.copy_(rows[i]), b.copy_(rows[1 - i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x[k], y[k]) for x, y in zip(out, want[i]) for k in x)
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for i, s in enumerate(streams * 3):
        with torch.cuda.stream(s):
            got.append((i % 2, every(rows[i % 2], rows[1 - i % 2])))
    torch.cuda.synchronize()
    for i, o in got:
        assert all(torch.equal(x[k], y[k]) for x, y in zip(o, want[i]) for k in x)
