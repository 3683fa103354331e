"""A policy of one MoE layer trained with routing replay, experts of its own behind the
framework's routes:

    python examples/rl_step.py [--steps 40] [--norm]

Each step samples one token per prompt position from the current policy, records the
routes (route_predict) and the tokens' log-probabilities (token_logprob), scores them, and
makes two updates on the same samples with the recorded routes replayed: with --norm a norm in
front of the layer (rms_norm), the routes' plan (dispatch_plan), the experts' products
(grouped_mm), SwiGLU kept in 8 bits (swiglu_pack), the weighted sum back (combine), the loss and
the gradient of the logits in one pass (policy_loss), and the backward pass down to every weight
(combine_backward, grouped_mm_backward, swiglu_backward_packed, weight_grad,
weight_grad_packed from the 8-bit hidden states, dispatch_backward, rms_norm_backward).
Nothing in the two passes waits for the device.  The dense matrix products are the library's.
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
    """x [T, d] -> logits [T, V]: h = x + sum over the k routed experts of g W_down(SwiGLU(W_gu n)),
    n = x or (norm) its root-mean-square norm, logits = h W_v^T.  fp32 weights, bf16 copies for the
    products."""

    def __init__(self, d=256, N=8, k=2, m=128, V=512, seed=0, device="cuda", norm=False):
        g = torch.Generator(device=device).manual_seed(seed)

        def w(*shape, std):
            return torch.randn(shape, generator=g, device=device) * std

        self.d, self.N, self.k, self.m, self.V = d, N, k, m, V
        self.p = {"W_r": w(d, N, std=0.05), "W_gu": w(N, 2 * m, d, std=d ** -0.5),
                  "W_down": w(N, d, m, std=m ** -0.5), "W_v": w(V, d, std=d ** -0.5)}
        if norm:
            self.p["w"] = torch.ones(d, device=device)

    def _input(self, x):
        """The layer's input, its 8-bit form and what the norm's backward reads (None without one)."""
        T, d = x.shape
        q = torch.empty((T, d), dtype=torch.int8, device=x.device)
        scale = torch.empty((T, -(-d // B.PACK_GROUP)), dtype=torch.uint8, device=x.device)
        if "w" not in self.p:
            B.act_pack(x, q, scale)
            return x, (q, scale), None
        n, rstd = torch.empty_like(x), torch.empty(T, device=x.device)
        B.rms_norm(x, self.p["w"], n, rstd_out=rstd, q=q, scale=scale)
        return n, (q, scale), rstd

    def routes(self, x):
        """The recorded route of a rollout step: the k highest logits of the router."""
        ids = torch.empty((x.shape[0], self.k), dtype=torch.int16, device=x.device)
        if "w" in self.p:
            n = torch.empty_like(x)
            B.rms_norm(x, self.p["w"], n)
            x = n
        B.route_predict(x, self.p["W_r"], None, None, None, self.k, ids)
        return ids

    def forward(self, x, ids):
        """Logits under the replayed routes, and what the backward pass needs."""
        T, dev = x.shape[0], x.device
        R, d, m, N, k = T * self.k, self.d, self.m, self.N, self.k
        i32 = dict(dtype=torch.int32, device=dev)
        plan = (torch.empty(N + 1, **i32), torch.empty((T, k), **i32), torch.empty(R, **i32))
        B.dispatch_plan(ids, N, *plan)
        offsets, row, route = plan
        n, xq, rstd = self._input(x)
        # replay: the weights come from the current router, over the recorded ids
        logits_r = torch.gather(n.float() @ self.p["W_r"], 1, ids.long())
        gate = torch.softmax(logits_r, dim=1).contiguous()
        new = lambda *s: torch.empty(s, dtype=BF16, device=dev)
        au, h, o, y = new(R, 2 * m), new(R, m), new(R, d), new(T, d)
        B.grouped_mm(n, self.p["W_gu"].to(BF16), au, offsets=offsets, route_of_row=route, k=k)
        aq = (torch.empty((R, 2 * m), dtype=torch.int8, device=dev),
              torch.empty((R, -(-2 * m // B.PACK_GROUP)), dtype=torch.uint8, device=dev))
        B.swiglu_pack(au, h, *aq)
        del au
        B.grouped_mm(h, self.p["W_down"].to(BF16), o, offsets=offsets)
        B.combine(o, row, gate, y)
        hidden = x + y
        logits = hidden @ self.p["W_v"].to(BF16).t()
        return logits, dict(x=x, n=n, rstd=rstd, ids=ids, offsets=offsets, row=row, route=route,
                            gate=gate, o=o, hidden=hidden, au=aq, xq=xq)

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
        B.grouped_mm_backward(d_o, self.p["W_down"].to(BF16), dh, offsets=s["offsets"])
        # h: the down projection's input as the checkpoint gives it
        B.swiglu_backward_packed(*s["au"], dh, dau, h)
        grads["W_down"] = torch.empty((N, d, m), device=dev)
        B.weight_grad(d_o, h, grads["W_down"], offsets=s["offsets"])
        grads["W_gu"] = torch.empty((N, 2 * m, d), device=dev)
        B.weight_grad_packed(dau, *s["xq"], grads["W_gu"], offsets=s["offsets"],
                             route_of_row=s["route"], k=k)
        B.grouped_mm_backward(dau, self.p["W_gu"].to(BF16), dxs, offsets=s["offsets"])
        B.dispatch_backward(dxs, s["row"], dx)
        # through the softmax over the recorded ids
        dp = s["gate"] * (dgate - (s["gate"] * dgate).sum(1, keepdim=True))
        dense = torch.zeros((T, N), device=dev).scatter_(1, s["ids"].long(), dp)
        grads["W_r"] = s["n"].float().t() @ dense
        if s["rstd"] is None:
            grads["x"] = dx.float() + dy.float() + dense @ self.p["W_r"].t()
            return grads
        dn = (dx.float() + dense @ self.p["W_r"].t()).to(BF16)
        grads["w"] = torch.empty(d, device=dev)
        B.rms_norm_backward(dn, s["x"], s["rstd"], self.p["w"], dx, dh=dy, dweight=grads["w"])
        grads["x"] = dx.float()
        return grads

    def loss_and_grads(self, x, ids, token, logp_old, adv, weight, logp_ref=None, kl_coef=0.0):
        logits, saved = self.forward(x, ids)
        sums = torch.empty(4, device=x.device)
        # the gradient takes the logits' place
        B.policy_loss(logits, token, logp_old, adv, sums, logp_ref=logp_ref, weight=weight,
                      dlogits=logits, kl_coef=kl_coef)
        return sums, self.backward(logits, saved)


def train(steps=40, T=1024, group=16, lr=1.0, max_norm=0.25, kl_coef=0.01, seed=0, report=None, norm=False):
    """Mean reward of each step.  T prompt positions in groups of `group` samples of the same
    prompt; a token is worth 1 if it belongs to its prompt's class modulo 8."""
    dev = "cuda"
    torch.manual_seed(seed)
    policy = MoePolicy(seed=seed, norm=norm)
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
    ap.add_argument("--norm", action="store_true")
    args = ap.parse_args()
    train(steps=args.steps, report=lambda s: print(s, flush=True), norm=args.norm)
