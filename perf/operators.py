"""A policy's training step as operators that can be timed and compared: scoring, its gradient, the update.

Three operators: the log probabilities of given choices under rows of logits with the rows' entropy and best
alternatives, the gradient of the first two with respect to the logits, and the orthogonalisation of update matrices by
Newton-Schulz products.  `run` computes them in plain torch operations, or, with `own`, through the package.
"""
import math

import torch

own = False

COEFFS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


def _case(name, op, **more):
    c = dict(op=op, **more)
    if name:
        c["name"] = name
    return c


def _rows(name, op, dtype, rows, vocab, pad=0, mask="none", top=0, scale=1.0):
    return _case(name, op, dtype=dtype, rows=rows, vocab=vocab, pad=pad, mask=mask, top=top, scale=scale)


def _update(name, dtype, batch, rows, cols, steps=5):
    return _case(name, "orthogonalise", dtype=dtype, batch=batch, rows=rows, cols=cols, steps=steps)


def listed():
    return [
        # the policy rows of a rollout batch: 64 environments, 128 candidate slots and No-Op, invalid actions masked
        _rows("policy_rows", "logprob", "fp32", 64, 129, mask="rows", top=4),
        # one decoding step of 16 sequences over a large vocabulary, with the alternatives a client asks for
        _rows("next_token", "logprob", "bf16", 16, 128000, top=20, scale=1.25),
        # a training batch of sequences scored under the current policy
        _rows("sequence_scores", "logprob", "bf16", 8192, 32000),
        # constrained choices: an odd vocabulary in rows of a wider buffer, a mask per row, a few alternatives
        _rows("masked_scores", "logprob", "fp32", 1500, 50001, pad=6, mask="rows", top=5, scale=0.7),
        # the gradients of the first, third and fourth
        _rows("policy_grad", "logprob_grad", "fp32", 64, 129, mask="rows"),
        _rows("sequence_grad", "logprob_grad", "bf16", 8192, 32000),
        _rows("masked_grad", "logprob_grad", "fp32", 1500, 50001, pad=6, mask="rows", scale=0.7),
        # the layer matrices of the agent with the paper's hyper-parameters: five layers of hidden 256
        _update("paper_layers", "fp32", 5, 256, 256),
        # the widest layers the agent has, four of them
        _update("wide_layers", "fp32", 4, 512, 512),
        # one matrix of a larger policy, fp32 gradients
        _update("fp32_matrix", "fp32", 1, 2048, 2048),
        # a tall odd matrix
        _update("tall_matrix", "bf16", 1, 4100, 1001),
        # the largest: a square matrix of 4,096
        _update("large_matrix", "bf16", 1, 4096, 4096),
    ]


def _log_range(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logprob", "logprob", "logprob_grad", "orthogonalise", "orthogonalise"])
    dtype = rng.choice(["bf16", "fp32"])
    if op == "orthogonalise":
        most = 4096 ** 3 if dtype == "bf16" else 2048 ** 3
        a, b = _log_range(rng, 32, 4096), _log_range(rng, 32, 8192)
        while a * b * min(a, b) > most:
            a, b = max(32, int(a * 0.8)), max(32, int(b * 0.8))
        batch = min(_log_range(rng, 1, 8), max(1, most // (a * b * min(a, b))))
        return _update(None, dtype, batch, a, b, rng.choice([3, 5, 5, 6]))
    vocab = _log_range(rng, 8, 131072)
    most = 8192 * 32000 // (1 if dtype == "bf16" else 2)
    rows = _log_range(rng, 1, max(1, min(16384, most // vocab)))
    top = rng.choice([0, 1, 5, 20]) if op == "logprob" else 0
    return _rows(None, op, dtype, rows, vocab, pad=rng.choice([0, 0, 1, 8, 13]), mask=rng.choice(["none", "one", "rows"]),
                 top=min(top, vocab), scale=rng.choice([1.0, 1.0, 0.7, 1.5]))


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    if case["op"] == "orthogonalise":
        # a gradient: a few strong directions, the rest small
        b, r, c = case["batch"], case["rows"], case["cols"]
        k = min(16, r, c)
        grad = 0.02 * n(b, r, c) + 0.01 * (n(b, r, k) @ n(b, k, c))
        return dict(case=case, grad=grad.to(_type(case)))
    rows, vocab = case["rows"], case["vocab"]
    x = 3.0 * n(rows, vocab + case["pad"])
    token = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    # a policy in training prefers what it chose
    x.scatter_add_(1, token[:, None], 6.0 * torch.rand(rows, 1, device="cuda", generator=g))
    token[torch.rand(rows, device="cuda", generator=g) < 0.05] = -1          # padding
    s = dict(case=case, logits=x.to(_type(case))[:, :vocab], token=token.to(torch.int32), mask=None)
    if case["mask"] != "none":
        mask = torch.rand(rows if case["mask"] == "rows" else 1, vocab, device="cuda", generator=g) < 0.6
        if case["mask"] == "rows":
            mask.scatter_(1, token.clamp(min=0)[:, None], True)
            mask[torch.rand(rows, device="cuda", generator=g) < 0.02] = False   # rows without a valid choice
        s["mask"] = mask.to(torch.uint8)
    if case["op"] == "logprob_grad":
        # what scoring left, and what an objective sends back
        z = s["logits"].float() if s["mask"] is None else s["logits"].float().masked_fill(s["mask"] == 0, -math.inf)
        m = z.amax(1)
        z = (case["scale"] * (z - m.masked_fill(m == -math.inf, 0)[:, None]))
        total = z.exp().sum(1, dtype=torch.float64)
        weighted = (z.exp() * z.masked_fill(z == -math.inf, 0)).sum(1, dtype=torch.float64)
        s["norm"] = torch.stack((m, total.log().float()), 1)
        s["entropy"] = torch.where(total > 0, total.log() - weighted / total, 0.0 * total).float()
        s["dlogp"] = n(rows) / rows
        s["dentropy"] = 0.01 * (1 + 0.1 * n(rows)) / rows
    return s


def _plain_logprob(case, x, token, mask):
    scale, top, vocab = case["scale"], case["top"], case["vocab"]
    x = x.float()
    if mask is not None:
        x = torch.where(mask != 0, x, -math.inf)
    m = x.amax(1, keepdim=True)
    none = m == -math.inf
    z = scale * (x - torch.where(none, 0.0, m))
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    ln = torch.log(total)
    weighted = torch.where(e > 0, e * z, 0.0).sum(1, keepdim=True)
    out = {"entropy": torch.where(none, 0.0, ln - weighted / total)[:, 0], "norm": torch.cat((m, ln), 1)}
    at = torch.gather(z, 1, token.clamp(min=0).long()[:, None])
    out["logp"] = torch.where(token < 0, 0.0, torch.where(at == -math.inf, -math.inf, at - ln)[:, 0])
    if top:
        # one whole number per entry, ordered by value first and by the lower index then
        bits = (x + 0.0).view(torch.int32).long()
        key = torch.where(bits >= 0, bits, (-1 << 31) - bits) * (1 << 31) + (vocab - 1 - torch.arange(vocab, device=x.device))
        index = torch.topk(key, top, dim=1).indices
        best = torch.gather(z, 1, index)
        out["top_token"] = torch.where(best == -math.inf, -1, index).int()
        out["top_logp"] = torch.where(best == -math.inf, -math.inf, best - ln)
    return out


def _plain_grad(case, x, token, mask, norm, entropy, dlogp, dentropy):
    scale = case["scale"]
    kept = x.float() > -math.inf
    if mask is not None:
        kept &= mask != 0
    lp = scale * (x.float() - norm[:, :1]) - norm[:, 1:]
    p = torch.exp(lp)
    there = torch.arange(case["vocab"], device=x.device) == token[:, None]
    dl = torch.where(token < 0, 0.0, dlogp)[:, None]
    return torch.where(kept, scale * (dl * (there.float() - p) - dentropy[:, None] * p * (lp + entropy[:, None])), 0.0).to(x.dtype)


def _plain_orthogonalise(grad, steps):
    a, b, c = COEFFS
    x = grad.float()
    size = torch.sqrt((x.double() ** 2).sum((1, 2), keepdim=True))
    x = (x.double() / (size + EPS)).float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    for _ in range(steps):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return (x.transpose(1, 2) if tall else x).to(grad.dtype).contiguous()


def run(s):
    c = s["case"]
    if own:
        import paper_2304_14698_b200 as xrl
        if c["op"] == "logprob":
            return xrl.xrl_logprob(s["logits"], s["token"], mask=s["mask"], scale=c["scale"], top=c["top"])
        if c["op"] == "logprob_grad":
            return xrl.xrl_logprob_grad(s["logits"], s["norm"], s["token"], s["dlogp"], s["entropy"], s["dentropy"],
                                        mask=s["mask"], scale=c["scale"])
        return xrl.xrl_orthogonalise(s["grad"], steps=c["steps"])
    if c["op"] == "logprob":
        return _plain_logprob(c, s["logits"], s["token"], s["mask"])
    if c["op"] == "logprob_grad":
        return _plain_grad(c, s["logits"], s["token"], s["mask"], s["norm"], s["entropy"], s["dlogp"], s["dentropy"])
    return _plain_orthogonalise(s["grad"], c["steps"])


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "orthogonalise":
        b, small, large = case["batch"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # the two products that give symmetric matrices need half their entries
        flops = case["steps"] * (small * small * large + small ** 3 + 2 * small * small * large)
        return {"bytes": b * 2 * small * large * size, "flops": b * flops}
    n = case["rows"] * case["vocab"]
    read = n * size + {"none": 0, "one": case["vocab"], "rows": n}[case["mask"]]
    if case["op"] == "logprob":
        return {"bytes": read + case["rows"] * (4 + 16 + 8 * case["top"]), "flops": 6 * n}
    return {"bytes": read + n * size + case["rows"] * 24, "flops": 8 * n}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orthogonalise":
        a, b, c = COEFFS
        outs = []
        for g in s["grad"].double():
            x = g / (torch.linalg.matrix_norm(g) + EPS)
            for _ in range(case["steps"]):
                # X (a + b X'X + c (X'X)^2) = (a + b XX' + c (XX')^2) X
                if x.shape[0] <= x.shape[1]:
                    w = x @ x.T
                    x = (a * torch.eye(len(w), device=w.device, dtype=w.dtype) + b * w + c * w @ w) @ x
                else:
                    w = x.T @ x
                    x = x @ (a * torch.eye(len(w), device=w.device, dtype=w.dtype) + b * w + c * w @ w)
            outs.append(x)
        return torch.stack(outs)
    z = s["logits"].double()
    scale, token = case["scale"], s["token"].long()
    if s["mask"] is not None:
        z = z.masked_fill(s["mask"] == 0, -math.inf)
    if case["op"] == "logprob":
        whole = torch.logsumexp(scale * z, 1)
        lp = scale * z - whole[:, None]
        largest = z.max(1).values
        p = torch.exp(lp)
        empty = largest == -math.inf
        ent = -torch.special.xlogy(p, p).sum(1)
        ent[empty] = 0
        logp = lp.gather(1, token.clamp(min=0)[:, None])[:, 0]
        logp[empty] = -math.inf
        logp[token < 0] = 0
        ln = whole - scale * largest
        ln[empty] = -math.inf
        out = {"entropy": ent, "norm": torch.stack((largest, ln), 1), "logp": logp}
        if case["top"]:
            v, i = torch.sort(z, dim=1, descending=True, stable=True)
            v, i = v[:, :case["top"]], i[:, :case["top"]]
            out["top_token"] = i.masked_fill(v == -math.inf, -1).int()
            out["top_logp"] = (scale * v - whole[:, None]).masked_fill(v == -math.inf, -math.inf)
        return out
    lp = scale * (z - s["norm"][:, :1].double()) - s["norm"][:, 1:].double()
    p = torch.exp(lp).nan_to_num(0.0)
    d = -p * torch.where(token < 0, 0.0, s["dlogp"].double())[:, None]
    d.scatter_add_(1, token.clamp(min=0)[:, None], torch.where(token < 0, 0.0, s["dlogp"].double())[:, None])
    d -= s["dentropy"].double()[:, None] * p * (lp.nan_to_num(0.0, neginf=0.0) + s["entropy"].double()[:, None])
    return (scale * d).masked_fill(z == -math.inf, 0.0)
