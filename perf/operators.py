"""What the operators that score rows are measured on: log-probabilities of tokens with entropy and alternatives, divergences of
draft rows from target rows, and the gradients of both, as a server or a trainer calls them through
`paper_2402_14160_b200.api`.

A case names a path and its sizes.  Rows are Gaussian logits made on the GPU from the seed (target = draft + noise, as in
`workloads`) in the storage type of the case, a share of them masked with -inf where the case says so (the same tokens in draft and
target rows).  The paths:

  score      rsd_token_logprobs: T given tokens a row, entropy, K alternatives
  emitted    rsd_emitted_logprobs: the tokens that a verification walk emitted, scored on the target rows that it visited
  score_grad rsd_token_logprobs_backward: gradient of weighted log-probabilities and entropies with respect to the rows
  div        rsd_row_divergence: KL both ways and the overlap of draft and target rows
  div_grad   rsd_row_divergence_backward: gradient of weighted divergences with respect to the draft rows
"""
import torch

own = False

ELEM = {"f32": 4, "bf16": 2}
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
NEG = float("-inf")


def listed():
    return [
        # one request after a step with an 8 x 8 beam tree: what was emitted, with five alternatives each
        dict(name="emitted_one_bf16", path="emitted", batch=1, vocab=32000, dtype="bf16", width=8, depth=8, top=5, temp=1.0, masked=0.0, sigma=2.0),
        # the same for a full serving batch: up to nine of 65 target rows a sequence are read
        dict(name="emitted_serving_bf16", path="emitted", batch=512, vocab=32000, dtype="bf16", width=8, depth=8, top=5, temp=1.0, masked=0.0,
             sigma=2.0),
        # a plain sampler's row per request: its token and the 20 likeliest, a large vocabulary
        dict(name="score_large_vocab_bf16", path="score", batch=64, rows=1, vocab=128000, dtype="bf16", tokens=1, top=20, temp=1.0, masked=0.0,
             sigma=3.0),
        # fp32 rows of a vocabulary with one added token (off every vector boundary), tempered, some tokens banned
        dict(name="score_odd_f32", path="score", batch=100, rows=5, vocab=32001, dtype="f32", tokens=3, top=32, temp=0.7, masked=0.3, sigma=2.0),
        # all children of all parents of a batch of 8 x 8 beam trees under their parents' rows: the largest read
        dict(name="score_trees_bf16", path="score", batch=256, rows=57, vocab=32000, dtype="bf16", tokens=8, top=0, temp=1.0, masked=0.0, sigma=2.0),
        # a training batch: one token a position, weighted, with an entropy term
        dict(name="score_grad_bf16", path="score_grad", batch=8, rows=1024, vocab=32000, dtype="bf16", tokens=1, entropy=True, temp=1.0, masked=0.0,
             sigma=2.0),
        # a few rows in fp32 at OPT's vocabulary
        dict(name="score_grad_few_f32", path="score_grad", batch=4, rows=9, vocab=50272, dtype="f32", tokens=4, entropy=False, temp=0.7, masked=0.0,
             sigma=3.0),
        # the parents of one small tree: how near the drafter is, row by row
        dict(name="div_one_f32", path="div", batch=1, rows=7, vocab=32000, dtype="f32", temp_d=1.0, temp_t=1.0, masked=0.0, sigma=2.0, noise=0.5),
        # the parents of a batch of beam trees
        dict(name="div_trees_bf16", path="div", batch=128, rows=57, vocab=32000, dtype="bf16", temp_d=1.0, temp_t=1.0, masked=0.0, sigma=2.0, noise=0.8),
        # rows off every vector boundary, draft and target at different ones
        dict(name="div_odd_bf16", path="div", batch=64, rows=10, vocab=32001, dtype="bf16", temp_d=0.7, temp_t=0.7, masked=0.3, sigma=2.0, noise=0.7),
        # distilling the target into the drafter, a training batch
        dict(name="div_grad_bf16", path="div_grad", batch=8, rows=512, vocab=32000, dtype="bf16", reverse=False, temp_d=1.0, temp_t=1.0, masked=0.0,
             sigma=2.0, noise=0.8),
        # both directions, fp32, a large vocabulary, moderate batch
        dict(name="div_grad_both_f32", path="div_grad", batch=16, rows=12, vocab=128000, dtype="f32", reverse=True, temp_d=1.0, temp_t=1.0, masked=0.3,
             sigma=2.0, noise=0.7),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case: the listed paths at sizes over their whole ranges."""
    path = rng.choice(["emitted", "score", "score", "score_grad", "div", "div_grad"])
    vocab = _log_int(rng, 500, 200000)
    align = rng.choice([1, 1, 8, 16, 64])
    vocab = max(500, vocab // align * align)
    case = dict(path=path, vocab=vocab, dtype=rng.choice(["f32", "bf16"]), sigma=rng.choice([1.5, 2.0, 3.0]), masked=rng.choice([0.0, 0.0, 0.3, 0.9]))
    if path == "emitted":
        case.update(width=rng.randint(1, 8), depth=rng.randint(1, 8), top=rng.choice([0, 1, 5, 20]), temp=rng.choice([0.3, 1.0]))
        per = 1 + case["width"] * case["depth"]
    else:
        case["rows"] = per = _log_int(rng, 1, 1024)
    if path == "score":
        case.update(tokens=rng.randint(0, 10), top=rng.choice([0, 0, 1, 5, 20, 32]), temp=rng.choice([0.3, 0.7, 1.0]))
        if case["top"] == 0:
            case["tokens"] = max(1, case["tokens"])
    if path == "score_grad":
        case.update(tokens=rng.randint(1, 8), entropy=rng.random() < 0.5, temp=rng.choice([0.7, 1.0]))
    if path in ("div", "div_grad"):
        case.update(temp_d=rng.choice([0.7, 1.0]), temp_t=rng.choice([0.7, 1.0]), noise=rng.choice([0.5, 0.7, 1.0]))
    if path == "div_grad":
        case["reverse"] = rng.random() < 0.5
    # at most a quarter of a billion entries (half the largest listed case), fewer where the plain form sorts
    most = 60_000_000 if case.get("top", 0) and path == "score" else 120_000_000 if path.startswith("div") else 250_000_000
    if per * vocab > most:
        case["rows"] = per = most // vocab
    case["batch"] = _log_int(rng, 1, max(1, min(1024, most // (per * vocab))))
    return case


def _rows(case, gen, per, both):
    """Rows [B, per, V], or draft and target rows, of which the target has one more a sequence (a tree's rows and its leaf)."""
    B, V, dt = case["batch"], case["vocab"], DTYPE[case["dtype"]]
    first = torch.empty((B, per, V), dtype=dt, device="cuda")
    second = torch.empty((B, per + 1, V), dtype=dt, device="cuda") if both else None
    seqs = max(1, (1 << 27) // (per * V))
    for b in range(0, B, seqs):
        n = min(seqs, B - b)
        base = torch.randn((n, per + (1 if both else 0), V), generator=gen, device="cuda").mul_(case["sigma"])
        banned = torch.rand((n, 1, V), generator=gen, device="cuda") < case["masked"] if case["masked"] else None
        if banned is not None:
            base.masked_fill_(banned, NEG)
        first[b:b + n].copy_(base[:, :per])
        if both:
            second[b:b + n].copy_(base.add_(torch.randn(base.shape, generator=gen, device="cuda"), alpha=case["noise"]))
    return (first, second) if both else first


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, V, path = case["batch"], case["vocab"], case["path"]
    st = dict(case=case)

    def ints(lo, hi, shape):
        return torch.randint(lo, hi, shape, generator=gen, device="cuda", dtype=torch.int32)

    def floats(shape):
        return torch.randn(shape, generator=gen, device="cuda")

    if path == "emitted":
        W, L = case["width"], case["depth"]
        st["rows"] = _rows(case, gen, 1 + W * L, False)
        length = ints(0, L + 1, (B,))
        slot = torch.arange(L, device="cuda", dtype=torch.int32)
        node = 1 + slot * W + ints(0, W, (B, L))
        inside = slot < length[:, None]
        st["walked"] = dict(accepted_len=length, accepted_node=torch.where(inside, node, -1).to(torch.int32),
                            accepted_token=torch.where(inside, ints(0, V, (B, L)), -1).to(torch.int32), last_token=ints(0, V, (B,)))
        return st
    R = case["rows"]
    if path in ("score", "score_grad"):
        st["rows"] = _rows(case, gen, R, False)
        token = ints(0, V, (B, R, case["tokens"]))
        if case["tokens"] > 1:    # absent children
            token = torch.where(ints(0, 8, token.shape) == 0, -1, token).to(torch.int32)
        st["token"] = token
        if path == "score_grad":
            st["g"] = floats((B, R, case["tokens"]))
            st["h"] = 0.1 * floats((B, R)) if case["entropy"] else None
        return st
    st["draft"], st["target"] = _rows(case, gen, R, True)
    if path == "div_grad":
        st["g"] = floats((B, R)).abs_()
        st["h"] = floats((B, R)).abs_() if case["reverse"] else None
    return st


# ---- plain forms -------------------------------------------------------------------------------------------------------------
def _log_softmax(rows, temp):
    z = rows.float()
    if temp != 1.0:
        z = z / temp
    z = z - z.amax(-1, keepdim=True)
    return z - z.exp().sum(-1, keepdim=True).log()


def _at(logp, token):
    """logp at the tokens, 0 where there is none."""
    got = logp.gather(-1, token.clamp_min(0).long())
    return torch.where(token >= 0, got, 0.0)


def _entropy(logp):
    return -torch.where(logp > NEG, logp.exp() * logp, 0.0).sum(-1)


def _top(rows, logp, k):
    """The k largest entries of each row: equal values go to the smaller token, masked entries to nobody."""
    v = rows.float() + 0.0                                        # (-0 is 0)
    bits = v.view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)     # order of the values
    V = rows.shape[-1]
    key = order * V + torch.arange(V - 1, -1, -1, device=rows.device)
    token = torch.topk(key, min(k, V), dim=-1).indices
    value = logp.gather(-1, token)
    token = torch.where(value > NEG, token, -1).to(torch.int32)
    pad = k - token.shape[-1]
    return torch.nn.functional.pad(token, (0, pad), value=-1), torch.nn.functional.pad(value, (0, pad), value=NEG)


def _plain_score(rows, token, top, temp):
    logp = _log_softmax(rows, temp)
    out = dict(logprob=_at(logp, token), entropy=_entropy(logp))
    if top:
        out["top_token"], out["top_logprob"] = _top(rows, logp, top)
    return out


def _plain_emitted(rows, walked, top, temp):
    B, L = walked["accepted_node"].shape
    slot = torch.arange(L + 1, device=rows.device)
    length = walked["accepted_len"].long()[:, None]
    zero = torch.zeros((B, 1), dtype=torch.int32, device=rows.device)
    node = torch.cat([zero, walked["accepted_node"]], 1)
    token = torch.cat([walked["accepted_token"], zero], 1)
    token = torch.where(slot < length, token, torch.where(slot == length, walked["last_token"][:, None], -1)).to(torch.int32)
    there = slot <= length
    visited = rows[torch.arange(B, device=rows.device)[:, None], node.clamp_min(0).long()]
    out = _plain_score(visited, token[..., None], top, temp)
    out = dict(out, logprob=out["logprob"][..., 0], entropy=torch.where(there, out["entropy"], 0.0))
    if top:
        out["top_token"] = torch.where(there[..., None], out["top_token"], -1)
        out["top_logprob"] = torch.where(there[..., None], out["top_logprob"], NEG)
    return dict(out, token=token)


def _plain_score_grad(rows, token, g, h, temp):
    logp = _log_softmax(rows, temp)
    p = logp.exp()
    g = torch.where(token >= 0, g, 0.0)
    grad = -p * g.sum(-1, keepdim=True)
    if h is not None:
        grad -= torch.where(p > 0, h[..., None] * p * (logp + _entropy(logp)[..., None]), 0.0)
    grad.scatter_add_(-1, token.clamp_min(0).long(), g)
    return (grad / temp).to(rows.dtype)


def _pair(st):
    case = st["case"]
    return _log_softmax(st["draft"], case["temp_d"]), _log_softmax(st["target"][:, :case["rows"]], case["temp_t"])


def _kl(a, b):
    """sum a (log a - log b), terms of little mass first lost in 32 bits: summed in 64"""
    return torch.where(a > NEG, a.exp() * (a - b), 0.0).sum(-1, dtype=torch.float64).float()


def _plain_div(st):
    logp, logq = _pair(st)
    return dict(kl=_kl(logq, logp), reverse_kl=_kl(logp, logq), overlap=torch.minimum(logp, logq).exp().sum(-1))


def _plain_div_grad(st):
    logp, logq = _pair(st)
    p = logp.exp()
    grad = st["g"][..., None] * (p - logq.exp())
    if st["h"] is not None:
        grad += torch.where(p > 0, st["h"][..., None] * p * (logp - logq - _kl(logp, logq)[..., None]), 0.0)
    return (grad / st["case"]["temp_d"]).to(st["draft"].dtype)


def run(st):
    case = st["case"]
    path = case["path"]
    if own:
        from paper_2402_14160_b200 import api
        if path == "score":
            out = api.rsd_token_logprobs(st["rows"], st["token"], top_k=case["top"], temperature=case["temp"])
            return {k: out[k] for k in ("logprob", "entropy", "top_token", "top_logprob") if out.get(k) is not None}
        if path == "emitted":
            out = api.rsd_emitted_logprobs(st["rows"], st["walked"], top_k=case["top"], temperature=case["temp"])
            return {k: out[k] for k in ("token", "logprob", "entropy", "top_token", "top_logprob") if out.get(k) is not None}
        if path == "score_grad":
            return api.rsd_token_logprobs_backward(st["rows"], st["token"], st["g"], st["h"], temperature=case["temp"])["grad_rows"]
        temps = dict(draft_temperature=case["temp_d"], target_temperature=case["temp_t"])
        if path == "div":
            out = api.rsd_row_divergence(st["draft"], st["target"], **temps)
            return {k: out[k] for k in ("kl", "reverse_kl", "overlap")}
        return api.rsd_row_divergence_backward(st["draft"], st["target"], st["g"], st["h"], **temps)["grad_draft"]
    if path == "score":
        return _plain_score(st["rows"], st["token"], case["top"], case["temp"])
    if path == "emitted":
        return _plain_emitted(st["rows"], st["walked"], case["top"], case["temp"])
    if path == "score_grad":
        return _plain_score_grad(st["rows"], st["token"], st["g"], st["h"], case["temp"])
    return _plain_div(st) if path == "div" else _plain_div_grad(st)


# ---- the definitions, in 64 bits ---------------------------------------------------------------------------------------------
def _exact_rows(x, temp):
    z = x.double() / temp
    return z - torch.logsumexp(z, -1, keepdim=True)


def _xlogy(p, q):
    """p (log p - log q) from the logarithms, 0 where p is 0"""
    return torch.nan_to_num(torch.exp(p) * (p - q), nan=0.0)


def _exact_one(rows, token, top, temp):
    logp = _exact_rows(rows, temp)
    out = dict(logprob=torch.stack([torch.where(t < 0, 0.0, logp.gather(-1, t.clamp_min(0).long()[..., None])[..., 0]) for t in token.unbind(-1)], -1)
               if token.shape[-1] else torch.zeros(token.shape, dtype=torch.float64, device=rows.device),
               entropy=-_xlogy(logp, torch.zeros_like(logp)).sum(-1))
    if top:
        # a stable sort keeps equal values in the order of their tokens
        value, index = torch.sort(rows.double(), dim=-1, descending=True, stable=True)
        k = min(top, rows.shape[-1])
        value, index = value[..., :k], index[..., :k]
        token_out = torch.full(rows.shape[:-1] + (top,), -1, dtype=torch.int32, device=rows.device)
        log_out = torch.full(rows.shape[:-1] + (top,), NEG, dtype=torch.float64, device=rows.device)
        token_out[..., :k] = torch.where(value > NEG, index, -1).to(torch.int32)
        log_out[..., :k] = torch.where(value > NEG, logp.gather(-1, index), NEG)
        out["top_token"], out["top_logprob"] = token_out, log_out
    return out


def _joined(parts, at=0):
    return {k: torch.cat([p[k] for p in parts], at) for k in parts[0]}


def exact(case, seed):
    st = prepare(case, seed)
    path, B, V = case["path"], case["batch"], case["vocab"]
    if path == "emitted":
        rows, walked = st["rows"], st["walked"]
        L = case["depth"]
        every = torch.arange(B, device=rows.device)
        slots = []
        for i in range(L + 1):
            there = walked["accepted_len"] >= i
            node = walked["accepted_node"][:, i - 1].long().clamp_min(0) if i else torch.zeros(B, dtype=torch.long, device=rows.device)
            token = walked["last_token"]
            if i < L:
                token = torch.where(walked["accepted_len"] > i, walked["accepted_token"][:, i], token)
            token = torch.where(there, token, -1).to(torch.int32)
            one = _exact_one(rows[every, node], token[:, None], case["top"], case["temp"])
            one = dict(one, logprob=one["logprob"][:, 0], entropy=torch.where(there, one["entropy"], 0.0), token=token)
            if case["top"]:
                one["top_token"] = torch.where(there[:, None], one["top_token"], -1)
                one["top_logprob"] = torch.where(there[:, None], one["top_logprob"], NEG)
            slots.append({k: v[:, None] for k, v in one.items()})
        return _joined(slots, 1)
    R = case["rows"]
    part = max(1, (1 << 27) // V)                                 # rows at a time
    flat = {k: v.reshape((B * R,) + v.shape[2:]) for k, v in st.items() if isinstance(v, torch.Tensor) and k != "target"}
    if "target" in st:
        flat["target"] = st["target"][:, :R].reshape(B * R, V)
    parts = []
    for a in range(0, B * R, part):
        x = {k: v[a:a + part] for k, v in flat.items()}
        if path == "score":
            parts.append(_exact_one(x["rows"], x["token"], case["top"], case["temp"]))
        elif path == "score_grad":
            logp = _exact_rows(x["rows"], case["temp"])
            p = logp.exp()
            grad = torch.zeros_like(p)
            for t, g in zip(x["token"].unbind(-1), x["g"].double().unbind(-1)):
                g = torch.where(t < 0, 0.0, g)[:, None]
                grad -= g * p
                grad.scatter_add_(1, t.clamp_min(0).long()[:, None], g)
            if "h" in x:
                own_term = _xlogy(logp, torch.zeros_like(logp))
                grad -= x["h"].double()[:, None] * (own_term - p * own_term.sum(-1, keepdim=True))
            parts.append({"grad": grad / case["temp"]})
        else:
            logp, logq = _exact_rows(x["draft"], case["temp_d"]), _exact_rows(x["target"], case["temp_t"])
            forward, backward = _xlogy(logq, logp), _xlogy(logp, logq)
            if path == "div":
                parts.append(dict(kl=forward.sum(-1), reverse_kl=backward.sum(-1), overlap=torch.exp(torch.minimum(logp, logq)).sum(-1)))
            else:
                grad = x["g"].double()[:, None] * (logp.exp() - logq.exp())
                if "h" in x:
                    grad += x["h"].double()[:, None] * (backward - logp.exp() * backward.sum(-1, keepdim=True))
                parts.append({"grad": grad / case["temp_d"]})
    whole = {k: v.reshape((B, R) + v.shape[1:]) for k, v in _joined(parts).items()}
    return whole["grad"] if path.endswith("grad") else whole


def work(case):
    """Rows read once, gradients written once, the small outputs once.  Operations: a scale, an exponential and the sums of each entry.  Of a tree
    whose accepted length is uniform over 0 .. L, 1 + L / 2 target rows a sequence are read."""
    B, V, path = case["batch"], case["vocab"], case["path"]
    row = V * ELEM[case["dtype"]]
    if path == "emitted":
        n = B * (1 + case["depth"] / 2)
        return {"bytes": n * row + B * (1 + case["depth"]) * (12 + 8 * case["top"]), "flops": 5 * n * V}
    n = B * case["rows"]
    if path == "score":
        return {"bytes": n * (row + 8 * case["tokens"] + 8 * case["top"] + 4), "flops": 5 * n * V}
    if path == "score_grad":
        return {"bytes": n * (2 * row + 8 * case["tokens"] + 4), "flops": 10 * n * V}
    if path == "div":
        return {"bytes": n * (2 * row + 12), "flops": 12 * n * V}
    return {"bytes": n * (3 * row + 8), "flops": 12 * n * V}
