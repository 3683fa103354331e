"""The example's training step: its loss and gradients against torch's autograd in float32
on the CPU, and the reward it reaches.

Tolerance, set before any run: the step's products and activations are bf16 (2^-9 relative
rounding each, about ten in a chain) and its checkpoints hold the large values of a group
to 1 part in 128, the small ones to a step of that: a few parts in a thousand of a
gradient's norm each, random, so 4 % of the norm; the loss itself sees no checkpoint."""
import pytest

pytestmark = pytest.mark.gpu


def reference(policy, x, ids, token, old, adv, weight, ref, beta):
    """Loss and gradients with every operation in float32 (weights and x as given)."""
    import torch
    p = {n: w.detach().cpu().float().requires_grad_() for n, w in policy.p.items()}
    xr = x.cpu().float().requires_grad_()
    ids, token, old, adv, weight, ref = (t.cpu() for t in (ids.long(), token.long(), old, adv, weight, ref))
    gate = torch.softmax(torch.gather(xr @ p["W_r"], 1, ids), 1)
    y = torch.zeros_like(xr)
    for s in range(policy.k):
        au = torch.bmm(p["W_gu"][ids[:, s]], xr.unsqueeze(2)).squeeze(2)
        a, u = au[:, :policy.m], au[:, policy.m:]
        h = torch.nn.functional.silu(a) * u
        y = y + gate[:, s:s + 1] * torch.bmm(p["W_down"][ids[:, s]], h.unsqueeze(2)).squeeze(2)
    logp = torch.log_softmax((xr + y) @ p["W_v"].t(), 1).gather(1, token.unsqueeze(1)).squeeze(1)
    r = torch.exp(logp - old)
    surr = torch.minimum(r * adv, torch.clamp(r, 0.8, 1.28) * adv)
    d = ref - logp
    loss = (weight * (-surr + beta * (torch.exp(d) - d - 1))).sum()
    loss.backward()
    return loss.item(), {**{n: w.grad for n, w in p.items()}, "x": xr.grad}, logp.detach()


def test_gradients_of_a_step_against_autograd():
    import torch
    from examples.rl_step import BF16, MoePolicy
    torch.manual_seed(1)
    T = 200
    policy = MoePolicy(d=128, N=6, k=2, m=96, V=333, seed=3)
    x = torch.randn((T, 128), device="cuda").to(BF16)
    ids = policy.routes(x)
    assert torch.equal(ids, torch.sort(torch.topk(x.float() @ policy.p["W_r"], 2).indices, 1).values.short())
    token = torch.randint(0, 333, (T,), device="cuda", dtype=torch.int32)
    adv, weight = torch.randn(T, device="cuda"), torch.full((T,), 1 / T, device="cuda")
    zero = torch.zeros(T, device="cuda")
    _, _, logp = reference(policy, x, ids, token, zero, adv, weight, zero, 0.0)
    old, ref = (logp + 0.05).cuda(), (logp - 0.2).cuda()
    sums, grads = policy.loss_and_grads(x, ids, token, old, adv, weight, ref, 0.1)
    loss, want, _ = reference(policy, x, ids, token, old, adv, weight, ref, 0.1)
    assert abs(sums[0].item() - loss) < 2e-2 * max(abs(loss), adv.abs().mean().item())
    for n, w in want.items():
        err = (grads[n].cpu() - w).norm() / w.norm()
        assert err < 0.04, f"{n}: {err:.4f}"


def test_training_raises_the_reward():
    from examples.rl_step import train
    rewards = train(steps=30)
    assert sum(rewards[:3]) / 3 < 0.25
    assert sum(rewards[-3:]) / 3 > 0.5, rewards
