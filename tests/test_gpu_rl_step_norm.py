"""The example's policy with a norm in front of its layer: gradients against torch's autograd in float32
on the CPU, a step in which the host does not wait, and that it runs.

Tolerance, set before any run: that of the example without the norm, 4 % of a gradient's norm (about
ten bf16 roundings in a chain and 8-bit checkpoints); the norm adds two more such roundings.
"""
import pytest

pytestmark = pytest.mark.gpu


def reference(policy, x, ids, token, old, adv, weight):
    import torch
    p = {n: w.detach().cpu().float().requires_grad_() for n, w in policy.p.items()}
    xr = x.cpu().float().requires_grad_()
    ids, token, old, adv, weight = (t.cpu() for t in (ids.long(), token.long(), old, adv, weight))
    n = xr * torch.rsqrt((xr * xr).mean(1, keepdim=True) + 1e-6) * p["w"]
    gate = torch.softmax(torch.gather(n @ p["W_r"], 1, ids), 1)
    y = torch.zeros_like(xr)
    for s in range(policy.k):
        au = torch.bmm(p["W_gu"][ids[:, s]], n.unsqueeze(2)).squeeze(2)
        a, u = au[:, :policy.m], au[:, policy.m:]
        y = y + gate[:, s:s + 1] * torch.bmm(p["W_down"][ids[:, s]],
                                             (torch.nn.functional.silu(a) * u).unsqueeze(2)).squeeze(2)
    logp = torch.log_softmax((xr + y) @ p["W_v"].t(), 1).gather(1, token.unsqueeze(1)).squeeze(1)
    r = torch.exp(logp - old)
    (-(weight * torch.minimum(r * adv, torch.clamp(r, 0.8, 1.28) * adv)).sum()).backward()
    return {**{n: w.grad for n, w in p.items()}, "x": xr.grad}, logp.detach()


@pytest.mark.parametrize("d,m", [(128, 96), (72, 40)])
def test_gradients_of_a_step_against_autograd(d, m):
    import torch
    from examples.rl_step import BF16, MoePolicy
    torch.manual_seed(2)
    T = 200
    policy = MoePolicy(d=d, N=6, k=2, m=m, V=333, seed=4, norm=True)
    policy.p["w"] += 0.2 * torch.randn(d, device="cuda")
    x = (3 * torch.randn((T, d), device="cuda")).to(BF16)
    ids = policy.routes(x)
    token = torch.randint(0, 333, (T,), device="cuda", dtype=torch.int32)
    adv, weight = torch.randn(T, device="cuda"), torch.full((T,), 1 / T, device="cuda")
    _, logp = reference(policy, x, ids, token, torch.zeros(T), adv, weight)
    old = (logp + 0.05).cuda()
    sums, grads = policy.loss_and_grads(x, ids, token, old, adv, weight)
    want, _ = reference(policy, x, ids, token, old, adv, weight)
    assert set(grads) == set(want)
    for n, w in want.items():
        err = (grads[n].cpu() - w).norm() / w.norm()
        assert err < 0.04, f"{n}: {err:.4f}"


def test_a_step_is_captured():
    """Forward, loss and backward as one graph: nothing in them asks the device anything."""
    import torch
    from examples.rl_step import BF16, MoePolicy
    torch.manual_seed(3)
    T = 96
    policy = MoePolicy(d=64, N=4, k=2, m=32, V=64, seed=5, norm=True)
    x = torch.randn((T, 64), device="cuda").to(BF16)
    ids = policy.routes(x)
    token = torch.randint(0, 64, (T,), device="cuda", dtype=torch.int32)
    adv, weight, old = torch.randn(T, device="cuda"), torch.full((T,), 1 / T, device="cuda"), torch.full((T,), -4.0, device="cuda")
    step = lambda: policy.loss_and_grads(x, ids, token, old, adv, weight)
    _, want = step()
    want = {n: g.clone() for n, g in want.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, got = step()
    for rep in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for n, g in want.items():
            # (the library's dense products may take other forms under a capture)
            assert (got[n] - g).norm() <= 0.02 * g.norm(), (rep, n)
        step()
        torch.cuda.synchronize()


def test_it_runs():
    from examples.rl_step import train
    rewards = train(steps=2, T=128, norm=True)
    assert len(rewards) == 2 and all(0 <= r <= 1 for r in rewards)
