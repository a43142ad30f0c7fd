"""The policy calls as a training step uses them: rows of logits scored, their gradient, the weights' update orthogonalised."""
import math

import numpy as np
import pytest
import torch

import paper_2304_14698_b200 as xrl
import gpu_util
from workloads import configs

pytestmark = pytest.mark.gpu


def orthogonal(g, steps=5, eps=1e-7):
    x = g.double() / (g.double().norm() + eps)
    for _ in range(steps):
        a = x @ x.T if x.shape[0] <= x.shape[1] else x.T @ x
        p = -4.7750 * a + 2.0315 * a @ a
        x = 3.4445 * x + (p @ x if x.shape[0] <= x.shape[1] else x @ p)
    return x


def test_a_training_step_of_a_linear_policy():
    """Two steps of: logits = h W; the clipped objective's dlogp with an entropy bonus; dW = h^T dlogits; W -= lr O(dW).  Against
    the same in 64 bits from the same fp32 W: an update's error is that of its parts, 2e-5 of its norm for O (see the tests
    of xrl_orthogonalise) on a dW that is off by the fp32 products' 1e-6 of its own norm, which the map of five steps multiplies
    by 485 at most where dW holds next to nothing and by about 1 where it holds most."""
    g = torch.Generator(device="cuda").manual_seed(3)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    rows, hidden, actions = 700, 96, 130
    h, W = n(rows, hidden), 0.3 * n(hidden, actions)
    mask = (torch.rand(rows, actions, device="cuda", generator=g) < 0.7)
    token = torch.randint(0, actions, (rows,), device="cuda", generator=g, dtype=torch.int32)
    mask.scatter_(1, token[:, None].long(), True)
    token[:30] = -1                                            # padding
    adv, behaviour = n(rows), -3 + 0.3 * n(rows)
    scores = None
    for step in range(2):
        logits = h @ W
        scores = xrl.xrl_logprob(logits, token, mask=mask, top=3, out=scores) if scores else xrl.xrl_logprob(logits, token, mask=mask, top=3)
        ratio = torch.exp((scores["logp"] - behaviour).clamp(-5, 5))
        dlogp = -(adv * ratio) / rows
        dent = torch.full_like(dlogp, -0.01 / rows)
        grad = xrl.xrl_logprob_grad(logits, scores["norm"], token, dlogp, scores["entropy"], dent, mask=mask, grad=logits)
        dW = h.T @ grad
        update = xrl.xrl_orthogonalise(dW)
        # the same in 64 bits
        W8 = W.double().requires_grad_()
        z = (h.double() @ W8).masked_fill(~mask, -math.inf)
        lp = torch.log_softmax(z, 1)
        p = lp.exp()
        logp = torch.where(token < 0, 0.0, lp.gather(1, token.clamp(min=0).long()[:, None])[:, 0])
        ent = -(p * lp.masked_fill(~mask, 0)).sum(1)
        assert float((scores["logp"].double() - logp.detach()).abs().max()) < 2e-5 and float((scores["entropy"].double() - ent.detach()).abs().max()) < 2e-5
        ratio8 = torch.exp((logp - behaviour.double()).clamp(-5, 5)).detach()
        (-(adv.double() * ratio8) / rows * logp - 0.01 / rows * ent).sum().backward()
        assert float((dW.double() - W8.grad).norm() / W8.grad.norm()) < 2e-5
        want = orthogonal(W8.grad)
        assert float((update.double() - want).norm() / want.norm()) < 1e-3
        W = W - 0.02 * update


@pytest.mark.parametrize("cfg", [2, 6])
def test_the_agents_own_layers(cfg):
    """xrl_ppo_grad's blob: the layers' part becomes the orthogonalised update, nothing else changes, and the weights with it
    are a model the agent runs on."""
    batch = configs.make_batch(cfg, candidates=3, envs=2)
    m = batch["model"]
    blob, _ = gpu_util.default_weights(batch, 5)
    agent = gpu_util.make_agent(batch)
    try:
        agent.set_weights(blob)
        agent.pack(batch)
        ne = len(batch["env_off"]) - 1
        mask = torch.from_numpy(batch["mask"]).cuda()
        one = lambda v: torch.full((ne,), v, device="cuda")  # noqa: E731
        loss, grad = torch.empty(4, device="cuda"), torch.empty(len(blob), device="cuda")
        action = torch.full((ne,), m["A_max"], dtype=torch.int32, device="cuda")
        xrl.xrl_ppo_grad(agent.ctx, agent.batch, mask, action, one(-1.0), one(0.7), one(0.3), loss, grad)
        before = grad.clone()
        assert xrl.orthogonalise_layers(m, grad) is grad
        layers, was = xrl.layer_matrices(m, grad), xrl.layer_matrices(m, before)
        for l in range(m["L"]):
            want = orthogonal(was[l])
            assert float((layers[l].double() - want).norm() / want.norm()) < 2e-5
        rest = grad.clone()
        xrl.layer_matrices(m, rest).copy_(was)
        assert torch.equal(rest, before)
        agent.set_weights(blob - 1e-3 * grad.cpu().numpy())
        out = agent.forward(mask)
        torch.cuda.synchronize()
        assert agent.device_status() == 0 and bool(torch.isfinite(out["probs"]).all())
        p = out["probs"]
        assert np.allclose(p.sum(1).cpu().numpy(), 1, atol=1e-5)
        # the agent's own distribution, scored: ln p of its logits' softmax is ln p
        o = xrl.xrl_logprob(p.log().clamp(min=-80), action, mask=torch.cat((mask, torch.ones_like(mask[:, :1])), 1))
        assert torch.allclose(o["logp"], p[torch.arange(ne), action.long()].log(), atol=1e-4)
    finally:
        agent.close()


def test_captured_together_and_replayed_on_new_inputs():
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(300, 2000, device="cuda", generator=g)
    h = torch.randn(300, 64, device="cuda", generator=g)
    token = torch.randint(0, 2000, (300,), device="cuda", generator=g, dtype=torch.int32)
    d = torch.randn(300, device="cuda", generator=g)

    def step():
        o = xrl.xrl_logprob(x, token, top=4)
        gr = xrl.xrl_logprob_grad(x, o["norm"], token, d, o["entropy"], d)
        return o["logp"], gr, xrl.xrl_orthogonalise(h.T @ gr)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    x.mul_(-0.5)
    h.add_(0.1)
    d.neg_()
    for _ in range(3):
        graph.replay()
    want = step()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
