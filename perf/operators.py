"""The operators that a training step needs around the layer's own calls, as their speed
is tracked: the policy loss on the sampled tokens, experts of the caller's own behind
the recorded routes, and activations kept in 8 bits for the backward pass.

A case is a dict of plain values; ``op`` names the operator:

* ``logprob``   log-probability and entropy of the sampled tokens (``T`` rows of ``V`` logits);
* ``policy``    clipped policy loss with a KL term and the gradient of the logits, in one
                pass, or (``split``) as a forward and a backward call;
* ``experts``   the routes' plan, tokens sorted by expert, weighted sum back (``T`` tokens of
                width ``d``, ``k`` of ``N`` experts);
* ``experts_backward``  gradients of the weighted sum and of the sorting, the plan given;
* ``experts_both``      both directions;
* ``pack``      8-bit checkpoint of a [``R``, ``C``] activation and its values back;
* ``swiglu``    SwiGLU keeping its input in 8 bits, and its backward from that;
* ``wgrad``     weight gradients from an 8-bit checkpoint of the inputs: of one linear layer
                (``N`` = 0) or of ``N`` experts whose rows are gathered from ``T`` tokens.

Widths are those of the layers that this repository measures (2048/128/8/768, 4096/128/8/1536,
2048/64/8/1024 and 2048/64/6/1408 as d/N/k/m); vocabularies are the 151936 ids of the Qwen3
models they belong to, or generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 32                 # columns that share one power-of-two scale

QWEN30 = dict(d=2048, N=128, k=8, m=768)
QWEN235 = dict(d=4096, N=128, k=8, m=1536)
OLMOE = dict(d=2048, N=64, k=8, m=1024)
MOONLIGHT = dict(d=2048, N=64, k=6, m=1408)
VOCAB = 151936


def _policy(name, op, T, V, act="bf16", pad=0, ref=True, tok="int32", split=False, temp=1.0):
    return dict(name=name, op=op, T=T, V=V, act=act, pad=pad, ref=ref, tok=tok, split=split,
                temp=temp)


def _experts(name, op, T, d, N, k, act="bf16", idx="int32", skew="hot8", drop=0.0):
    return dict(name=name, op=op, T=T, d=d, N=N, k=k, act=act, idx=idx, skew=skew, drop=drop)


def _wgrad(name, T, n_out, n_in, N=0, k=1, act="bf16", skew="none"):
    return dict(name=name, op="wgrad", T=T, n_out=n_out, n_in=n_in, N=N, k=k, act=act, skew=skew)


def listed():
    return [
        # log-probabilities recorded for the eight sequences that still generate
        _policy("logprob_decode_8", "logprob", 8, VOCAB, tok="int64"),
        # one training micro-batch: loss, KL to a reference policy, gradient of the logits
        _policy("policy_4096", "policy", 4096, VOCAB),
        # fp32 logits of an odd vocabulary in padded rows, under a program with its own
        # chain of backward calls, sampled at a temperature, no reference policy
        _policy("policy_split_f32_517", "policy", 517, 50257, act="f32", pad=47, ref=False,
                tok="int64", split=True, temp=0.8),
        # the caller's experts behind the recorded routes of a rollout batch
        _experts("experts_16384", "experts", 16384, 2048, 128, 8),
        # and their backward
        _experts("experts_backward_16384", "experts_backward", 16384, 2048, 128, 8),
        # a decode step of 64 sequences with an int16 record
        _experts("experts_decode_64", "experts", 64, 2048, 64, 8, idx="int16"),
        # fp32 layer of odd sizes, some routes dropped (a capacity limit), both directions
        _experts("experts_f32_1021", "experts_both", 1021, 333, 7, 3, act="f32", drop=0.1),
        # the hidden states of a batch kept in 8 bits
        dict(name="pack_16384", op="pack", R=16384, C=2048, act="bf16"),
        # the experts' pre-activations of that batch: 131072 routes, 768 wide
        dict(name="swiglu_131072", op="swiglu", R=131072, m=768, act="bf16"),
        # gate and up weight gradients of all experts from the packed hidden states
        _wgrad("wgrad_experts_16384", 16384, 1536, 2048, N=128, k=8),
        # weight gradient of one linear layer (an attention or output projection)
        _wgrad("wgrad_linear_8192", 8192, 2048, 2048),
        # odd fp32 experts
        _wgrad("wgrad_f32_613", 613, 135, 203, N=7, k=2, act="f32", skew="hot8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprob", "policy", "policy", "experts", "experts_backward", "experts_both",
                     "pack", "swiglu", "wgrad", "wgrad", "small_f32"])
    if op in ("logprob", "policy"):
        act = rng.choice(["bf16", "bf16", "f32"])
        V = rng.choice([VOCAB, 32000, 50257, _log_int(rng, 1000, 200000)])
        most = 4096 * VOCAB // V // (2 if act == "f32" else 1)
        c = _policy("", op, _log_int(rng, 1, min(16384, most)), V, act=act,
                    pad=rng.choice([0, 0, rng.randint(1, 200)]), ref=rng.random() < 0.7,
                    tok=rng.choice(["int32", "int64"]), split=op == "policy" and rng.random() < 0.4,
                    temp=rng.choice([1.0, 0.7, 1.3]))
    elif op.startswith("experts"):
        layer = rng.choice([QWEN30, OLMOE, MOONLIGHT, QWEN235, None, None])
        if layer is None:
            N = rng.randint(2, 160)
            layer = dict(d=rng.randint(100, 5000), N=N, k=rng.randint(1, min(N, 12)))
        both = 2 if op == "experts_both" else 1
        hi = min(32768, 2 * 16384 * 8 * 2048 // (both * layer["k"] * layer["d"]))
        c = _experts("", op, _log_int(rng, 1, max(1, hi // 2)), layer["d"], layer["N"], layer["k"],
                     idx=rng.choice(["int16", "int32"]), skew=rng.choice(["none", "hot8", "zipf"]),
                     drop=rng.choice([0.0, 0.0, 0.05, 0.3]))
    elif op == "pack":
        C = rng.choice([2048, 4096, rng.randint(1, 6000)])
        c = dict(op=op, R=_log_int(rng, 1, 100_000_000 // C), C=C, act=rng.choice(["bf16", "bf16", "f32"]))
    elif op == "swiglu":
        m = rng.choice([768, 1024, 1408, 1536, rng.randint(1, 3000)])
        c = dict(op=op, R=_log_int(rng, 1, 100_000_000 // m), m=m, act="bf16")
    elif op == "wgrad":
        if rng.random() < 0.35:
            n_out, n_in = (rng.choice([2048, 4096, 1536, 16 * rng.randint(4, 256)]) for _ in range(2))
            T = _log_int(rng, 30, 32768)
            c = _wgrad("", T, n_out, n_in)
        else:
            layer = rng.choice([QWEN30, OLMOE, MOONLIGHT, None, None])
            if layer is None:
                N = rng.randint(2, 128)
                layer = dict(d=32 * rng.randint(8, 80), N=N, k=rng.randint(1, min(N, 8)),
                             m=8 * rng.randint(16, 160))
            most = 16384 * 8 * 1536 * 2048 // (layer["k"] * 2 * layer["m"] * layer["d"])
            c = _wgrad("", _log_int(rng, 30, min(16384, most)), 2 * layer["m"], layer["d"],
                       N=layer["N"], k=layer["k"], skew=rng.choice(["none", "none", "hot8"]))
    else:
        N = rng.randint(2, 32)
        k = rng.randint(1, min(N, 4))
        T = _log_int(rng, 1, 2000)
        c = rng.choice([
            _experts("", "experts_both", T, rng.randint(17, 700), N, k, act="f32",
                     idx=rng.choice(["int16", "int32"]), skew="hot8", drop=0.1),
            _wgrad("", T, rng.randint(1, 400), rng.randint(1, 400), N=N, k=k, act="f32", skew="hot8"),
            dict(op="swiglu", R=T, m=rng.randint(1, 900), act="f32"),
        ])
    c.pop("name", None)
    return c


# ------------------------------------------------------------------ inputs --

def _draws(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 6007 + 29)
    return g


def _dt(case):
    return torch.bfloat16 if case["act"] == "bf16" else torch.float32


def _randn(g, *shape, dt=torch.float32, std=1.0):
    t = torch.randn(shape, generator=g, device="cuda", dtype=dt)
    return t if std == 1.0 else t.mul_(std)


def _routes(case, g, T, N, k, drop, it):
    """Recorded ids [T, k], ascending, under an uneven load; dropped routes are -1."""
    score = _randn(g, T, N)
    order = torch.randperm(N, generator=g, device="cuda")
    if case["skew"] == "hot8":
        score[:, order[:8]] += 1.0
    elif case["skew"] == "zipf":
        score[:, order] += -0.6 * torch.log(torch.arange(1, N + 1, device="cuda").float())
    ids = torch.sort(torch.topk(score, k, dim=1).indices, dim=1).values
    if drop:
        ids = torch.where(torch.rand((T, k), generator=g, device="cuda") < drop, -1, ids)
    return ids.to(it).contiguous()


def _plan(ids, N):
    """Offsets [N+1], row of each route [T, k] (-1: dropped), route of each row [T*k] (-1: none)."""
    flat = ids.reshape(-1).long()
    valid = (flat >= 0) & (flat < N)
    key = torch.where(valid, flat, N)
    order = torch.argsort(key, stable=True)
    ends = torch.cumsum((key.unsqueeze(1) == torch.arange(N, device=key.device)).sum(0), 0)
    offsets = torch.cat([ends.new_zeros(1), ends]).to(torch.int32)
    place = torch.arange(flat.numel(), device=key.device)
    route_of_row = torch.where(place < offsets[N], order, -1).to(torch.int32)
    row_of_route = torch.empty_like(order).index_copy_(0, order, place)
    row_of_route = torch.where(valid, row_of_route, -1).to(torch.int32)
    return offsets, row_of_route.reshape(ids.shape), route_of_row


def _inputs(case, seed):
    g, dt, op = _draws(seed), _dt(case), case["op"]
    s = dict(op=op)
    if op in ("logprob", "policy"):
        T, V = case["T"], case["V"]
        logits = _randn(g, T, V + case["pad"], dt=dt).mul_(2.5)[:, :V]
        logits[:, V - V // 100:] = float("-inf")        # ids that no token may take
        y = torch.randint(0, V - V // 100, (T,), generator=g, device="cuda")
        # the sampled token is a likely one
        rows = torch.arange(T, device="cuda")
        logits[rows, y] = (logits[rows, y].float() + 12 + _randn(g, T)).to(dt)
        s.update(logits=logits, y=y.to(torch.int64 if case["tok"] == "int64" else torch.int32),
                 inv_temp=1.0 / case["temp"], low=0.2, high=0.28, beta=0.02 if case["ref"] else 0.0,
                 split=case["split"])
        if op == "policy":
            logp = torch.empty(T, device="cuda")
            for t0 in range(0, T, 512):
                z = logits[t0:t0 + 512].float() * s["inv_temp"]
                logp[t0:t0 + 512] = (torch.gather(z, 1, y[t0:t0 + 512].unsqueeze(1)).squeeze(1)
                                     - torch.logsumexp(z, 1))
            # the policy has moved since the rollout; no ratio within rounding of a clip bound,
            # where the gradient jumps
            moved = _randn(g, T, std=0.15)
            for b in (0.8, 1.28):
                moved = torch.where((moved.exp() - b).abs() < 1e-3, moved + 0.01, moved)
            s["logp_old"] = logp - moved
            s["logp_ref"] = logp + _randn(g, T, std=0.1) if case["ref"] else None
            # one advantage per response of up to 512 tokens
            seq = torch.arange(T, device="cuda") // 512
            s["adv"] = _randn(g, T // 512 + 1)[seq].contiguous()
            # prompts and padding carry no weight, some of them no token either
            off = torch.rand(T, generator=g, device="cuda")
            off = torch.where(rows == T - 1, 1.0, off)
            s["y"] = torch.where(off < 0.04, -1, s["y"])
            keep = (off >= 0.1).float()
            s["weight"] = keep / keep.sum()
    elif op.startswith("experts"):
        T, d, N, k = case["T"], case["d"], case["N"], case["k"]
        it = torch.int16 if case["idx"] == "int16" else torch.int32
        s.update(N=N, k=k, ids=_routes(case, g, T, N, k, case["drop"], it))
        s["gate"] = torch.softmax(_randn(g, T, k), dim=1)
        s["o"] = _randn(g, T * k, d, dt=dt)
        if op != "experts_backward":
            s["x"] = _randn(g, T, d, dt=dt)
        if op != "experts":
            s["dy"], s["dxs"] = _randn(g, T, d, dt=dt), _randn(g, T * k, d, dt=dt)
            s["offsets"], s["row"], s["route"] = _plan(s["ids"], N)
    elif op == "pack":
        # hidden states: a few columns carry much larger values
        s["x"] = _randn(g, case["R"], case["C"], dt=dt)
        s["x"][:, :: 97] *= 20
    elif op == "swiglu":
        s["au"] = _randn(g, case["R"], 2 * case["m"], dt=dt, std=1.5)
        s["dh"] = _randn(g, case["R"], case["m"], dt=dt)
    else:
        T, N, k = case["T"], case["N"], case["k"]
        s.update(N=N, k=k, x=_randn(g, T, case["n_in"], dt=dt),
                 dy=_randn(g, T * k, case["n_out"], dt=dt, std=0.1))
        if N:
            ids = _routes(case, g, T, N, k, 0.0, torch.int32)
            s["offsets"], _, s["route"] = _plan(ids, N)
            s["most"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op, dt = s["op"], _dt(case)

    def buf(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if op in ("logprob", "policy"):
        T, V = case["T"], case["V"]
        s.update(logp=buf(T), entropy=buf(T), lse=buf(T), coef=buf(T), sums=buf(4))
        if op == "policy":
            s["dlogits"] = buf(T, V, dtype=dt)
    elif op.startswith("experts"):
        T, d, N, k = case["T"], case["d"], case["N"], case["k"]
        if op != "experts_backward":
            s.update(plan=(buf(N + 1, dtype=torch.int32), buf(T, k, dtype=torch.int32),
                           buf(T * k, dtype=torch.int32)),
                     xs=buf(T * k, d, dtype=dt), y=buf(T, d, dtype=dt))
        if op != "experts":
            s.update(do=buf(T * k, d, dtype=dt), dgate=buf(T, k), dx=buf(T, d, dtype=dt))
    elif op == "pack":
        R, C = case["R"], case["C"]
        s.update(q=buf(R, C, dtype=torch.int8), e=buf(R, -(-C // GROUP), dtype=torch.uint8),
                 xh=buf(R, C, dtype=dt))
    elif op == "swiglu":
        R, m = case["R"], case["m"]
        s.update(h=buf(R, m, dtype=dt), q=buf(R, 2 * m, dtype=torch.int8),
                 e=buf(R, -(-2 * m // GROUP), dtype=torch.uint8), dau=buf(R, 2 * m, dtype=dt),
                 hb=buf(R, m, dtype=dt))
    else:
        T, C, N = case["T"], case["n_in"], case["N"]
        s.update(q=buf(T, C, dtype=torch.int8), e=buf(T, -(-C // GROUP), dtype=torch.uint8),
                 dW=buf(max(N, 1), case["n_out"], C))
    return s


# -------------------------------------------------------------- plain forms --

def _policy_rows(s):
    z = s["logits"].float()
    V = z.shape[1]
    y = s["y"].long()
    has = (y >= 0) & (y < V)
    yc = torch.where(has, y, 0).unsqueeze(1)
    t = (z - z.amax(1, keepdim=True)) * s["inv_temp"]
    e = torch.exp(t)
    total = e.sum(1, keepdim=True)
    p = e / total
    log_total = torch.log(total)
    logp = (torch.gather(t, 1, yc) - log_total).squeeze(1)
    entropy = (log_total - torch.where(p > 0, p * t, 0.0).sum(1, keepdim=True)).squeeze(1)
    return p, yc, has, torch.where(has, logp, 0.0), torch.where(has, entropy, 0.0)


def _policy_coef(s, logp, entropy, has):
    w, A = s["weight"], s["adv"]
    on = has & (w != 0)
    r = torch.exp(logp - s["logp_old"])
    surr = torch.minimum(r * A, torch.clamp(r, 1 - s["low"], 1 + s["high"]) * A)
    clipped = ((A > 0) & (r > 1 + s["high"])) | ((A < 0) & (r < 1 - s["low"]))
    coef = torch.where(clipped, 0.0, -A * r)
    loss, kl = -surr, torch.zeros_like(logp)
    if s["logp_ref"] is not None:
        d = s["logp_ref"] - logp
        kl = torch.exp(d) - d - 1
        loss = loss + s["beta"] * kl
        coef = coef + s["beta"] * (1 - torch.exp(d))
    w = torch.where(on, w, 0.0)
    sums = torch.stack([(w * loss).sum(), (w * kl).sum(), (w * clipped).sum(), (w * entropy).sum()])
    return w * coef, sums, torch.where(on, logp, 0.0)


def _pad_groups(x):
    C = x.shape[1]
    n = -(-C // GROUP)
    if C % GROUP:
        full = x.new_zeros((x.shape[0], n * GROUP))
        full[:, :C] = x
        x = full
    return x.reshape(x.shape[0], n, GROUP)


def _kept(x):
    """The values that the 8-bit checkpoint of x stands for (fp32)."""
    v = _pad_groups(x.float())
    exponent = (v.abs().amax(2, keepdim=True).view(torch.int32) >> 23) & 255
    byte = torch.clamp(exponent - 6, min=1)
    step = (byte << 23).view(torch.float32)
    inverse = ((254 - byte) << 23).view(torch.float32)
    q = torch.clamp(torch.round(v * inverse), -127, 127)
    return (q * step).reshape(x.shape[0], -1)[:, :x.shape[1]]


def _swiglu(a, u):
    return a / (1 + torch.exp(-a)) * u


def _plain(s):
    op = s["op"]
    if op == "logprob":
        _, _, _, logp, entropy = _policy_rows(s)
        return logp, entropy
    if op == "policy":
        dt = s["logits"].dtype
        p, yc, has, logp, entropy = _policy_rows(s)
        coef, sums, logp = _policy_coef(s, logp, entropy, has)
        scale = (coef * s["inv_temp"]).unsqueeze(1)
        grad = p.mul_(-scale)
        grad.scatter_add_(1, yc, scale)
        return sums, logp, grad.to(dt)
    if op.startswith("experts"):
        o, gate = s["o"], s["gate"]
        dt = o.dtype
        out = ()
        if op == "experts_backward":
            offsets, row, route = s["offsets"], s["row"], s["route"]
        else:
            offsets, row, route = _plan(s["ids"], s["N"])
        on = (row >= 0).unsqueeze(2)
        rows = torch.clamp(row, min=0).long()
        tokens = torch.clamp(route, min=0).long() // s["k"]
        filled = (route >= 0).unsqueeze(1)
        picked = torch.where(on, o[rows].float(), 0.0)
        if op != "experts_backward":
            xs = torch.where(filled, s["x"][tokens], 0.0)
            y = (gate.unsqueeze(2) * picked).sum(1).to(dt)
            out += (offsets, row, route, xs.to(dt), y)
        if op != "experts":
            dy = s["dy"].float()
            weight = gate.reshape(-1)[torch.clamp(route, min=0).long()].unsqueeze(1)
            do = torch.where(filled, weight * dy[tokens], 0.0).to(dt)
            dgate = (picked * dy.unsqueeze(1)).sum(2)
            dx = torch.where(on, s["dxs"][rows].float(), 0.0).sum(1).to(dt)
            out += (do, dgate, dx)
        return out
    if op == "pack":
        return (_kept(s["x"]).to(s["x"].dtype),)
    if op == "swiglu":
        au, dh = s["au"], s["dh"].float()
        m = dh.shape[1]
        h = _swiglu(au[:, :m].float(), au[:, m:].float()).to(au.dtype)
        kept = _kept(au)
        a, u = kept[:, :m], kept[:, m:]
        sig = 1 / (1 + torch.exp(-a))
        da, du = dh * u * sig * (1 + a * (1 - sig)), dh * a * sig
        return h, torch.cat([da, du], 1).to(au.dtype), (a * sig * u).to(au.dtype)
    kept, dy, N = _kept(s["x"]), s["dy"].float(), s["N"]
    if not N:
        return ((dy.T @ kept).unsqueeze(0),)
    # every expert's rows, padded to the longest
    first, last = s["offsets"][:-1].long().unsqueeze(1), s["offsets"][1:].long().unsqueeze(1)
    at = first + torch.arange(max(s["most"], 1), device=dy.device)
    on = (at < last).unsqueeze(2)
    at = torch.clamp(at, max=dy.shape[0] - 1)
    rows = torch.where(on, dy[at], 0.0).transpose(1, 2).contiguous()
    return (torch.bmm(rows, kept[torch.clamp(s["route"][at], min=0).long() // s["k"]]),)


# ------------------------------------------------------- the framework's calls --

def _own(s):
    from paper_2606_00395_amd import binding as B
    op = s["op"]
    if op == "logprob":
        B.token_logprob(s["logits"], s["y"], s["logp"], entropy_out=s["entropy"],
                        inv_temp=s["inv_temp"])
        return s["logp"], s["entropy"]
    if op == "policy":
        args = (s["logits"], s["y"], s["logp_old"], s["adv"])
        kw = dict(logp_ref=s["logp_ref"], weight=s["weight"], logp_out=s["logp"], clip_low=s["low"],
                  clip_high=s["high"], kl_coef=s["beta"], inv_temp=s["inv_temp"])
        if s["split"]:
            B.policy_loss(*args, s["sums"], lse_out=s["lse"], coef_out=s["coef"], **kw)
            B.policy_loss_backward(s["logits"], s["y"], s["lse"], s["coef"], s["dlogits"],
                                   inv_temp=s["inv_temp"])
        else:
            B.policy_loss(*args, s["sums"], dlogits=s["dlogits"], **kw)
        return s["sums"], s["logp"], s["dlogits"]
    if op.startswith("experts"):
        out = ()
        if op != "experts_backward":
            offsets, row, route = s["plan"]
            B.dispatch_plan(s["ids"], s["N"], offsets, row, route)
            B.dispatch(s["x"], offsets, row, s["xs"])
            B.combine(s["o"], row, s["gate"], s["y"])
            out += (offsets, row, route, s["xs"], s["y"])
        else:
            offsets, row = s["offsets"], s["row"]
        if op != "experts":
            B.combine_backward(s["dy"], s["o"], offsets, row, s["gate"], s["do"], s["dgate"])
            B.dispatch_backward(s["dxs"], row, s["dx"])
            out += (s["do"], s["dgate"], s["dx"])
        return out
    if op == "pack":
        B.act_pack(s["x"], s["q"], s["e"])
        B.act_unpack(s["q"], s["e"], s["xh"])
        return (s["xh"],)
    if op == "swiglu":
        B.swiglu_pack(s["au"], s["h"], s["q"], s["e"])
        B.swiglu_backward_packed(s["q"], s["e"], s["dh"], s["dau"], s["hb"])
        return s["h"], s["dau"], s["hb"]
    B.act_pack(s["x"], s["q"], s["e"])
    if s["N"]:
        B.weight_grad_packed(s["dy"], s["q"], s["e"], s["dW"], offsets=s["offsets"],
                             route_of_row=s["route"], k=s["k"])
    else:
        B.weight_grad_packed(s["dy"], s["q"], s["e"], s["dW"])
    return (s["dW"],)


def run(s):
    return _own(s) if own else _plain(s)


# -------------------------------------------------------------------- work --

def work(case):
    op, a = case["op"], 2 if case["act"] == "bf16" else 4
    if op == "logprob":
        T, V = case["T"], case["V"]
        return {"bytes": T * V * a + T * 16, "flops": 5 * T * V}
    if op == "policy":
        T, V = case["T"], case["V"]
        passes = 3 if case["split"] else 2
        return {"bytes": passes * T * V * a + T * 32, "flops": 9 * T * V}
    if op.startswith("experts"):
        T, d, k = case["T"], case["d"], case["k"]
        token, route = T * d * a, T * k * d * a
        ids = T * k * (2 if case["idx"] == "int16" else 4)
        forward = 2 * token + 2 * route + ids + T * k * 12
        backward = 2 * token + 3 * route + T * k * 12
        both = {"experts": forward, "experts_backward": backward}
        return {"bytes": both.get(op, forward + backward),
                "flops": T * k * d * {"experts": 2, "experts_backward": 4}.get(op, 6)}
    if op == "pack":
        n = case["R"] * case["C"]
        return {"bytes": n * (2 * a + 2 + 2 / GROUP), "flops": 4 * n}
    if op == "swiglu":
        n = case["R"] * case["m"]
        # forward: a, u read, h and their 8-bit form written; backward: that and dh read,
        # da, du and h written
        return {"bytes": n * (7 * a + 4 + 4 / GROUP), "flops": 30 * n}
    T, R, O, C, N = case["T"], case["T"] * case["k"], case["n_out"], case["n_in"], max(case["N"], 1)
    return {"bytes": T * C * (a + 2) + R * O * a + N * O * C * 4, "flops": 2 * R * O * C}


# -------------------------------------------------- the definitions in 64 bits --

def _exact_policy(s):
    logits, y = s["logits"], s["y"].long()
    T, V = logits.shape
    logp = torch.zeros(T, dtype=torch.float64, device="cuda")
    ent, lse = torch.zeros_like(logp), torch.zeros_like(logp)
    for t0 in range(0, T, 256):
        z = logits[t0:t0 + 256].double() * s["inv_temp"]
        l = torch.logsumexp(z, 1)
        lse[t0:t0 + 256] = l
        logp[t0:t0 + 256] = torch.gather(z, 1, y[t0:t0 + 256].clamp(0, V - 1).unsqueeze(1)).squeeze(1) - l
        ls = z - l.unsqueeze(1)
        ent[t0:t0 + 256] = -torch.nan_to_num(ls.exp() * ls, nan=0.0).sum(1)
    return logp, ent, lse


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("logprob", "policy"):
        logp, ent, lse = _exact_policy(s)
        if op == "logprob":
            return logp, ent
        T, V = s["logits"].shape
        y = s["y"].long()
        w = s["weight"].double() * ((y >= 0) & (y < V))
        A, r = s["adv"].double(), torch.exp(logp - s["logp_old"].double())
        lo, hi = 1 - s["low"], 1 + s["high"]
        surr = torch.where(A >= 0, A * torch.clamp(r, max=hi), A * torch.clamp(r, min=lo))
        stops = torch.where(A >= 0, r > hi, r < lo) & (A != 0)
        dl = torch.where(stops, 0.0, -A * r)
        loss, kl = -surr, torch.zeros_like(r)
        if s["logp_ref"] is not None:
            d = s["logp_ref"].double() - logp
            kl = torch.expm1(d) - d
            loss, dl = loss + s["beta"] * kl, dl - s["beta"] * torch.expm1(d)
        c = w * dl * s["inv_temp"]
        sums = torch.stack([(w * loss).sum(), (w * kl).sum(), (w * stops).sum(), (w * ent).sum()])
        grad = torch.empty((T, V), dtype=torch.float64, device="cuda")
        for t0 in range(0, T, 256):
            t1 = min(T, t0 + 256)
            p = torch.exp(s["logits"][t0:t1].double() * s["inv_temp"] - lse[t0:t1].unsqueeze(1))
            p[torch.arange(t1 - t0, device="cuda"), y[t0:t1].clamp(0, V - 1)] -= 1
            grad[t0:t1] = -c[t0:t1].unsqueeze(1) * p
        return sums, torch.where(w != 0, logp, 0.0), grad
    if op.startswith("experts"):
        T, d, N, k = case["T"], case["d"], case["N"], case["k"]
        counts, place, route = [0] * N, [], []
        ids = s["ids"].cpu().tolist()
        per = [[] for _ in range(N)]
        for t in range(T):
            for c in range(k):
                if 0 <= ids[t][c] < N:
                    per[ids[t][c]].append(t * k + c)
        sorted_routes = [q for rows in per for q in rows]
        for e in range(N):
            counts[e] = len(per[e])
        ends = [0]
        for c in counts:
            ends.append(ends[-1] + c)
        place = [-1] * (T * k)
        for r, q in enumerate(sorted_routes):
            place[q] = r
        route = sorted_routes + [-1] * (T * k - len(sorted_routes))
        ints = dict(dtype=torch.int32, device="cuda")
        row = torch.tensor(place, **ints).reshape(T, k)
        n = len(sorted_routes)
        src = torch.tensor(sorted_routes, dtype=torch.int64, device="cuda")
        tok = src // k
        gate = s["gate"].double().reshape(-1)[src].unsqueeze(1)
        o = s["o"][:n].double()
        out = ()
        if op != "experts_backward":
            xs = torch.zeros((T * k, d), dtype=torch.float64, device="cuda")
            xs[:n] = s["x"][tok].double()
            y = torch.zeros((T, d), dtype=torch.float64, device="cuda").index_add_(0, tok, gate * o)
            out += (torch.tensor(ends, **ints), row, torch.tensor(route, **ints), xs, y)
        if op != "experts":
            do = torch.zeros((T * k, d), dtype=torch.float64, device="cuda")
            up = s["dy"][tok].double()
            do[:n] = gate * up
            dgate = torch.zeros(T * k, dtype=torch.float64, device="cuda")
            dgate[src] = (up * o).sum(1)
            dx = torch.zeros((T, d), dtype=torch.float64, device="cuda")
            dx.index_add_(0, tok, s["dxs"][:n].double())
            out += (do, dgate.reshape(T, k), dx)
        return out

    def held(x):
        """int8 multiples of a power of two that brings the group's largest below 128."""
        x = x.double()
        C = x.shape[1]
        out = torch.empty_like(x)
        for c in range(0, C, GROUP):
            part = x[:, c:c + GROUP]
            _, two = torch.frexp(part.abs().amax(1, keepdim=True))
            step = torch.exp2(torch.clamp(two - 7, min=-126).double())
            out[:, c:c + GROUP] = torch.clamp(torch.round(part / step), -127, 127) * step
        return out

    if op == "pack":
        return (held(s["x"]),)
    if op == "swiglu":
        m = case["m"]
        kept, dh = held(s["au"]), s["dh"].double()
        a0, a = s["au"][:, :m].double(), kept[:, :m]
        h = a0 * torch.sigmoid(a0) * s["au"][:, m:].double()
        sig, u = torch.sigmoid(a), kept[:, m:]
        slope = sig + a * sig * (1 - sig)
        return h, torch.cat([dh * u * slope, dh * a * sig], 1), a * sig * u
    kept, N, k = held(s["x"]), case["N"], case["k"]
    if not N:
        return ((s["dy"].double().T @ kept).unsqueeze(0),)
    dW = torch.zeros((N, case["n_out"], case["n_in"]), dtype=torch.float64, device="cuda")
    ends = s["offsets"].cpu().tolist()
    for e in range(N):
        rows = slice(ends[e], ends[e + 1])
        dW[e] = s["dy"][rows].double().T @ kept[s["route"][rows].long() // k]
    return (dW,)
