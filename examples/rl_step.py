"""A policy of one MoE layer trained with routing replay, experts of its own behind the
framework's routes:

    python examples/rl_step.py [--steps 40]

Each step samples one token per prompt position from the current policy, records the
routes (route_predict) and the tokens' log-probabilities (token_logprob), scores them, and
makes two updates on the same samples with the recorded routes replayed: sorted rows
(dispatch_plan, dispatch), the experts' products, SwiGLU kept in 8 bits (swiglu_pack), the
weighted sum back (combine), the loss and the gradient of the logits in one pass
(policy_loss), and the backward pass down to every weight (combine_backward,
swiglu_backward_packed, weight_grad_packed from the 8-bit hidden states, dispatch_backward).
The plain matrix products are the library's.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2606_00395_amd import binding as B  # noqa: E402

BF16 = torch.bfloat16


class MoePolicy:
    """x [T, d] -> logits [T, V]: h = x + sum over the k routed experts of g W_down(SwiGLU(W_gu x)),
    logits = h W_v^T.  fp32 weights, bf16 copies for the products."""

    def __init__(self, d=256, N=8, k=2, m=128, V=512, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)

        def w(*shape, std):
            return torch.randn(shape, generator=g, device=device) * std

        self.d, self.N, self.k, self.m, self.V = d, N, k, m, V
        self.p = {"W_r": w(d, N, std=0.05), "W_gu": w(N, 2 * m, d, std=d ** -0.5),
                  "W_down": w(N, d, m, std=m ** -0.5), "W_v": w(V, d, std=d ** -0.5)}

    def routes(self, x):
        """The recorded route of a rollout step: the k highest logits of the router."""
        ids = torch.empty((x.shape[0], self.k), dtype=torch.int16, device=x.device)
        B.route_predict(x, self.p["W_r"], None, None, None, self.k, ids)
        return ids

    def _per_expert(self, rows, weights, offsets, out):
        """out[rows of e] = rows[rows of e] weights[e]^T (weights [N, n_out, n_in], bf16)."""
        for e in range(self.N):
            a, b = offsets[e], offsets[e + 1]
            if b > a:
                torch.mm(rows[a:b], weights[e].t(), out=out[a:b])

    def forward(self, x, ids):
        """Logits under the replayed routes, and what the backward pass needs."""
        T, dev = x.shape[0], x.device
        R, d, m, N, k = T * self.k, self.d, self.m, self.N, self.k
        i32 = dict(dtype=torch.int32, device=dev)
        plan = (torch.empty(N + 1, **i32), torch.empty((T, k), **i32), torch.empty(R, **i32))
        B.dispatch_plan(ids, N, *plan)
        offsets, row, route = plan
        # replay: the weights come from the current router, over the recorded ids
        logits_r = torch.gather(x.float() @ self.p["W_r"], 1, ids.long())
        gate = torch.softmax(logits_r, dim=1).contiguous()
        new = lambda *s: torch.empty(s, dtype=BF16, device=dev)
        xs, au, h, o, y = new(R, d), new(R, 2 * m), new(R, m), new(R, d), new(T, d)
        B.dispatch(x, offsets, row, xs)
        bounds = offsets.tolist()
        self._per_expert(xs, self.p["W_gu"].to(BF16), bounds, au)
        del xs
        packs = [(torch.empty(s, dtype=torch.int8, device=dev),
                  torch.empty((s[0], -(-s[1] // B.PACK_GROUP)), dtype=torch.uint8, device=dev))
                 for s in ((R, 2 * m), (T, d))]
        B.swiglu_pack(au, h, *packs[0])
        B.act_pack(x, *packs[1])
        del au
        self._per_expert(h, self.p["W_down"].to(BF16), bounds, o)
        B.combine(o, row, gate, y)
        hidden = x + y
        logits = hidden @ self.p["W_v"].to(BF16).t()
        return logits, dict(x=x, ids=ids, offsets=offsets, bounds=bounds, row=row, route=route,
                            gate=gate, o=o, hidden=hidden, au=packs[0], xq=packs[1])

    def backward(self, dlogits, s):
        """Gradients of every weight and of x from that of the logits; overwrites s["o"]."""
        T, dev = dlogits.shape[0], dlogits.device
        R, d, m, N, k = T * self.k, self.d, self.m, self.N, self.k
        new = lambda *sh: torch.empty(sh, dtype=BF16, device=dev)
        grads = {"W_v": dlogits.float().t() @ s["hidden"].float()}
        dy = dlogits @ self.p["W_v"].to(BF16)
        d_o, dgate = s["o"], torch.empty((T, k), device=dev)
        B.combine_backward(dy, s["o"], s["offsets"], s["row"], s["gate"], d_o, dgate)
        dh, dau, h, dxs, dx = new(R, m), new(R, 2 * m), new(R, m), new(R, d), new(T, d)
        self._per_expert(d_o, self.p["W_down"].to(BF16).transpose(1, 2).contiguous(), s["bounds"], dh)
        B.swiglu_backward_packed(*s["au"], dh, dau, h)
        # the down projection's input as the checkpoint gives it, packed for its weight gradient
        hq = (torch.empty((R, m), dtype=torch.int8, device=dev),
              torch.empty((R, -(-m // B.PACK_GROUP)), dtype=torch.uint8, device=dev))
        B.act_pack(h, *hq)
        grads["W_down"] = torch.empty((N, d, m), device=dev)
        B.weight_grad_packed(d_o, *hq, grads["W_down"], offsets=s["offsets"])
        grads["W_gu"] = torch.empty((N, 2 * m, d), device=dev)
        B.weight_grad_packed(dau, *s["xq"], grads["W_gu"], offsets=s["offsets"],
                             route_of_row=s["route"], k=k)
        self._per_expert(dau, self.p["W_gu"].to(BF16).transpose(1, 2).contiguous(), s["bounds"], dxs)
        B.dispatch_backward(dxs, s["row"], dx)
        # through the softmax over the recorded ids
        dp = s["gate"] * (dgate - (s["gate"] * dgate).sum(1, keepdim=True))
        dense = torch.zeros((T, N), device=dev).scatter_(1, s["ids"].long(), dp)
        grads["W_r"] = s["x"].float().t() @ dense
        grads["x"] = dx.float() + dy.float() + dense @ self.p["W_r"].t()
        return grads

    def loss_and_grads(self, x, ids, token, logp_old, adv, weight, logp_ref=None, kl_coef=0.0):
        logits, saved = self.forward(x, ids)
        sums = torch.empty(4, device=x.device)
        # the gradient takes the logits' place
        B.policy_loss(logits, token, logp_old, adv, sums, logp_ref=logp_ref, weight=weight,
                      dlogits=logits, kl_coef=kl_coef)
        return sums, self.backward(logits, saved)


def train(steps=40, T=1024, group=16, lr=1.0, max_norm=0.25, kl_coef=0.01, seed=0, report=None):
    """Mean reward of each step.  T prompt positions in groups of `group` samples of the same
    prompt; a token is worth 1 if it belongs to its prompt's class modulo 8."""
    dev = "cuda"
    torch.manual_seed(seed)
    policy = MoePolicy(seed=seed)
    prompts = torch.randn((T // group, policy.d), device=dev)
    x = prompts.repeat_interleave(group, 0).to(BF16)
    wanted = torch.randint(0, 8, (T // group,), device=dev).repeat_interleave(group)
    weight = torch.full((T,), 1.0 / T, device=dev)
    rewards, ref = [], None
    for step in range(steps):
        # rollout: routes, tokens and their log-probabilities under the current policy
        ids = policy.routes(x)
        logits, _ = policy.forward(x, ids)
        # a sample of the softmax: the largest logit plus Gumbel noise
        noise = -torch.log(-torch.log(torch.rand_like(logits, dtype=torch.float32).clamp_(1e-12, 1 - 1e-6)))
        token = torch.argmax(logits.float() + noise, 1).to(torch.int32)
        logp_old = torch.empty(T, device=dev)
        B.token_logprob(logits, token, logp_old)
        ref = policy.p if ref is None else ref
        reward = (token % 8 == wanted).float()
        per = reward.view(-1, group)
        adv = ((per - per.mean(1, keepdim=True)) / (per.std(1, keepdim=True) + 1e-4)).reshape(-1).contiguous()
        rewards.append(reward.mean().item())
        # the reference policy's log-probabilities of the same tokens, under the same routes
        frozen = MoePolicy.__new__(MoePolicy)
        frozen.__dict__.update({**policy.__dict__, "p": ref})
        logp_ref = torch.empty(T, device=dev)
        B.token_logprob(frozen.forward(x, ids)[0], token, logp_ref)
        for _ in range(2):
            sums, grads = policy.loss_and_grads(x, ids, token, logp_old, adv, weight, logp_ref, kl_coef)
            # a few tokens far from the reference would otherwise carry a step away
            norm = torch.stack([grads[n].square().sum() for n in policy.p]).sum().sqrt()
            scale = lr * torch.clamp(max_norm / norm, max=1.0)
            policy.p = {n: w - scale * grads[n] for n, w in policy.p.items()}
        if report:
            loss, kl, clipped, entropy = sums.tolist()
            report(f"step {step:3d}  reward {rewards[-1]:.3f}  loss {loss:+.4f}  kl {kl:.4f}  "
                   f"clipped {clipped:.3f}  entropy {entropy:.3f}")
    return rewards


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    train(steps=ap.parse_args().steps, report=lambda s: print(s, flush=True))
