"""The operators of a block whose experts are the program's own, as their speed is tracked: the
norm in front of the layer with its gradient, the products of rows sorted by expert with both
gradients, and the same products in 8 bits for the rollout.

A case is a dict of plain values; ``op`` names the operator:

* ``norm``           residual added and root-mean-square norm of ``T`` rows of ``d``, with (``pack``)
                     the norm's 8-bit checkpoint and its values back;
* ``norm_backward``  its gradients; ``norm_both`` both directions;
* ``mm``             products of the rows behind ``T`` tokens' routes (``k`` of ``N`` experts) with their
                     experts' [``n_out``, ``n_in``] weights; ``gather``: the rows are read through the
                     plan from the tokens, else they lie sorted already;
* ``mm_backward``    gradients of the rows and of the weights; ``mm_both`` both directions;
* ``quant_mm``       rows brought to 8 bits, then their products with 8-bit weights (``N`` = 0: one
                     linear layer);
* ``quant_layer``    norm with an 8-bit output, gate and up projection, SwiGLU, down projection, the
                     weights in 8 bits.

Widths are those of the layers that this repository measures (2048/128/8/768, 2048/64/8/1024 and
2048/64/6/1408 as d/N/k/m), or generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 32                 # columns that share one power-of-two scale of the packed form
EPS = 1e-6

QWEN30 = dict(d=2048, N=128, k=8, m=768)
OLMOE = dict(d=2048, N=64, k=8, m=1024)
MOONLIGHT = dict(d=2048, N=64, k=6, m=1408)


def _norm(name, op, T, d, act="bf16", res=True, pack=False):
    return dict(name=name, op=op, T=T, d=d, act=act, res=res, pack=pack)


def _mm(name, op, T, n_out, n_in, N, k, act="bf16", gather=True, skew="hot8", drop=0.0):
    return dict(name=name, op=op, T=T, n_out=n_out, n_in=n_in, N=N, k=k, act=act, gather=gather,
                skew=skew, drop=drop)


def _layer8(name, T, d, N, k, m, act="bf16", skew="hot8"):
    return dict(name=name, op="quant_layer", T=T, d=d, N=N, k=k, m=m, act=act, skew=skew)


def listed():
    return [
        # a decode step of eight sequences: residual and norm
        _norm("norm_8", "norm", 8, 2048),
        # a training batch, the norm's output kept in 8 bits for the weight gradients
        _norm("norm_pack_16384", "norm", 16384, 2048, pack=True),
        # and its backward, the residual stream's gradient added
        _norm("norm_backward_16384", "norm_backward", 16384, 2048),
        # fp32 rows of an odd width, first layer (no residual), both directions
        _norm("norm_f32_1021", "norm_both", 1021, 333, act="f32", res=False),
        # gate and up projections of a training batch behind its recorded routes
        _mm("experts_up_16384", "mm", 16384, 1536, 2048, 128, 8),
        # a decode step of 64 sequences: about as many rows as experts
        _mm("experts_up_decode_64", "mm", 64, 2048, 2048, 64, 8),
        # the down projections' gradients: of the rows and of all weights
        _mm("experts_down_backward_16384", "mm_backward", 16384, 2048, 768, 128, 8, gather=False),
        # a short micro-batch whose experts get about a hundred rows each, both directions
        _mm("experts_both_1021", "mm_both", 1021, 2816, 2048, 64, 6),
        # odd fp32 experts, some routes dropped, both directions
        _mm("experts_f32_613", "mm_both", 613, 135, 203, 7, 2, act="f32", drop=0.1),
        # a decode step of 256 sequences through a layer with 8-bit weights
        _layer8("quant_layer_256", 256, 2048, 128, 8, 768),
        # a prompt batch through 8-bit gate and up projections
        _mm("quant_up_16384", "quant_mm", 16384, 2048, 2048, 64, 8),
        # a linear layer of odd sizes from fp32 rows
        _mm("quant_linear_517", "quant_mm", 517, 1001, 999, 0, 1, act="f32", gather=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "norm_both", "mm", "mm", "mm_backward", "mm_both",
                     "quant_mm", "quant_mm", "quant_layer", "small_f32"])
    if op.startswith("norm"):
        d = rng.choice([2048, 4096, rng.randint(64, 9000)])
        act = rng.choice(["bf16", "bf16", "f32"])
        most = 16384 * 2048 // d // (2 if act == "f32" else 1) // (2 if op == "norm_both" else 1)
        c = _norm("", op, _log_int(rng, 1, most), d, act=act, res=rng.random() < 0.7,
                  pack=op == "norm" and rng.random() < 0.4)
    elif op == "quant_layer":
        layer = rng.choice([QWEN30, OLMOE, MOONLIGHT, None])
        if layer is None:
            N = rng.randint(2, 100)
            layer = dict(d=16 * rng.randint(8, 160), N=N, k=rng.randint(1, min(N, 8)), m=rng.randint(60, 1300))
        c = _layer8("", _log_int(rng, 1, 2048), layer["d"], layer["N"], layer["k"], layer["m"],
                    skew=rng.choice(["none", "hot8", "zipf"]))
    elif op == "small_f32":
        N = rng.randint(2, 32)
        c = _mm("", rng.choice(["mm_both", "mm_both", "quant_mm"]), _log_int(rng, 1, 2000), rng.randint(1, 400),
                rng.randint(1, 400), N, rng.randint(1, min(N, 4)), act=rng.choice(["f32", "f32", "bf16"]),
                gather=rng.random() < 0.5, skew="hot8", drop=0.1)
    else:
        if rng.random() < 0.6:
            layer = rng.choice([QWEN30, OLMOE, MOONLIGHT])
            up = rng.random() < 0.5
            n_out, n_in = (2 * layer["m"], layer["d"]) if up else (layer["d"], layer["m"])
            N, k = layer["N"], layer["k"]
        else:
            N = rng.randint(1, 100)
            k = rng.randint(1, min(N, 8))
            n_out, n_in = (rng.choice([8 * rng.randint(16, 300), 64 * rng.randint(2, 40)]) for _ in range(2))
        most = 16384 * 8 * 1536 * 2048 // (k * n_out * n_in) // (3 if op == "mm_both" else 2)
        c = _mm("", op, _log_int(rng, 1, min(16384, most)), n_out, n_in, N, k, gather=rng.random() < 0.5,
                skew=rng.choice(["none", "hot8", "zipf"]), drop=rng.choice([0.0, 0.0, 0.05]))
    c.pop("name", None)
    return c


# ------------------------------------------------------------------ inputs --

def _draws(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7001 + 13)
    return g


def _dt(case):
    return torch.bfloat16 if case["act"] == "bf16" else torch.float32


def _randn(g, *shape, dt=torch.float32, std=1.0):
    t = torch.randn(shape, generator=g, device="cuda", dtype=dt)
    return t if std == 1.0 else t.mul_(std)


def _routes(case, g, T, N, k, drop):
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
    return ids


def _plan(ids, N):
    """Offsets [N + 1] and the route of each row [T * k] (-1: none)."""
    flat = ids.reshape(-1).long()
    key = torch.where(flat >= 0, flat, N)
    order = torch.argsort(key, stable=True)
    ends = torch.cumsum((key.unsqueeze(1) == torch.arange(N, device=key.device)).sum(0), 0)
    offsets = torch.cat([ends.new_zeros(1), ends]).to(torch.int32)
    place = torch.arange(flat.numel(), device=key.device)
    return offsets, torch.where(place < offsets[N], order, -1).to(torch.int32)


def _channels(W):
    """Weights [N, n_out, n_in] in 8 bits with a scale for each output channel."""
    scale = torch.clamp(W.abs().amax(2) / 127, min=1e-30)
    return torch.round(W / scale.unsqueeze(2)).to(torch.int8), scale.contiguous()


def _inputs(case, seed):
    g, dt, op = _draws(seed), _dt(case), case["op"]
    s = dict(op=op)
    if op.startswith("norm"):
        T, d = case["T"], case["d"]
        # the residual stream: a few columns carry much larger values
        s["x"] = _randn(g, T, d, dt=dt)
        s["x"][:, :: 97] *= 20
        s["residual"] = _randn(g, T, d, dt=dt) if case["res"] else None
        s["weight"] = 1 + _randn(g, d, std=0.2)
        if op != "norm":
            s["dy"] = _randn(g, T, d, dt=dt)
            s["dh"] = _randn(g, T, d, dt=dt) if case["res"] else None
        if op == "norm_backward":
            # as the forward pass left it
            s["h"] = s["x"]
            s["rstd"] = torch.rsqrt(s["x"].double().square().mean(1) + EPS).float()
            s["x"] = s["residual"] = None
        return s
    T, N, k = case["T"], case["N"], case["k"]
    s.update(N=N, k=k, T=T)
    if N:
        ids = _routes(case, g, T, N, k, case.get("drop", 0.0))
        s["offsets"], s["route"] = _plan(ids, N)
    n = max(N, 1)
    if op == "quant_layer":
        d, m = case["d"], case["m"]
        s["x"], s["residual"] = _randn(g, T, d, dt=dt), _randn(g, T, d, dt=dt)
        s["x"][:, :: 97] *= 20
        s["weight"] = 1 + _randn(g, d, std=0.2)
        s["Wu"], s["su"] = _channels(_randn(g, n, 2 * m, d, std=d ** -0.5))
        s["Wd"], s["sd"] = _channels(_randn(g, n, d, m, std=m ** -0.5))
        return s
    n_out, n_in = case["n_out"], case["n_in"]
    s["x"] = _randn(g, T if case["gather"] else T * k, n_in, dt=dt)
    if op == "quant_mm":
        s["W"], s["scale"] = _channels(_randn(g, n, n_out, n_in, std=n_in ** -0.5))
    else:
        s["W"] = _randn(g, n, n_out, n_in, dt=dt, std=n_in ** -0.5)
    if op in ("mm_backward", "mm_both"):
        s["dy"] = _randn(g, T * k, n_out, dt=dt)
    if not case["gather"]:
        s["route"] = None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op, dt = s["op"], _dt(case)

    def buf(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if op.startswith("norm"):
        T, d = case["T"], case["d"]
        if op != "norm_backward":
            s.update(h=buf(T, d, dtype=dt) if case["res"] else None, y=buf(T, d, dtype=dt))
            if case["pack"]:
                s.update(q=buf(T, d, dtype=torch.int8), e=buf(T, -(-d // GROUP), dtype=torch.uint8),
                         back=buf(T, d, dtype=dt))
            else:
                s["q"] = None
        if op == "norm_both":
            s["rstd"] = buf(T)
        if op != "norm":
            s.update(dx=buf(T, d, dtype=dt), dweight=buf(d))
        return s
    R = case["T"] * case["k"]
    # a program that runs the experts one by one keeps their bounds on the host
    s["ends"] = s["offsets"].tolist() if s["N"] else [0, R]
    if not s["N"]:
        s["offsets"] = None
    if op == "quant_layer":
        T, d, m = case["T"], case["d"], case["m"]
        s.update(h=buf(T, d, dtype=dt), q=buf(T, d, dtype=torch.int8), e=buf(T), au=buf(R, 2 * m, dtype=dt),
                 hq=buf(R, m, dtype=torch.int8), he=buf(R), o=buf(R, d, dtype=dt))
        return s
    n_out, n_in = case["n_out"], case["n_in"]
    if op != "mm_backward":
        s["out"] = buf(R, n_out, dtype=dt)
    if op == "quant_mm":
        s.update(q=buf(*s["x"].shape, dtype=torch.int8), e=buf(s["x"].shape[0]))
    elif op != "mm":
        s.update(dx=buf(R, n_in, dtype=dt), dW=buf(max(s["N"], 1), n_out, n_in))
    return s


# -------------------------------------------------------------- plain forms --

def _kept(x):
    """The values that the 8-bit checkpoint of x stands for (fp32)."""
    C = x.shape[1]
    n = -(-C // GROUP)
    v = x.new_zeros((x.shape[0], n * GROUP), dtype=torch.float32)
    v[:, :C] = x
    v = v.reshape(x.shape[0], n, GROUP)
    exponent = (v.abs().amax(2, keepdim=True).view(torch.int32) >> 23) & 255
    byte = torch.clamp(exponent - 6, min=1)
    step = (byte << 23).view(torch.float32)
    inverse = ((254 - byte) << 23).view(torch.float32)
    q = torch.clamp(torch.round(v * inverse), -127, 127)
    return (q * step).reshape(x.shape[0], -1)[:, :C]


def _rows8(v):
    """Whole numbers of up to 127 per row and the step (fp32) that they are multiples of."""
    step = v.abs().amax(1, keepdim=True) / 127
    # (in 64 bits: next to a half, 32 decide otherwise)
    return torch.round(v.double() / torch.clamp(step, min=1e-35).double()).float(), step


def _plain_norm(s, dt):
    h = s["x"].float()
    if s["residual"] is not None:
        h = (h + s["residual"].float()).to(dt).float()
    rstd = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    return h, rstd


def _plain_mm(x, W, ends, route, k, R, row=None, channel=None):
    """Row by row with its expert's weights (fp32); zeros behind the last expert's rows."""
    out = x.new_zeros((R, W.shape[1]), dtype=torch.float32)
    for e in range(W.shape[0]):
        a, b = ends[e], ends[e + 1]
        if a == b:
            continue
        src = slice(a, b) if route is None else route[a:b].long() // k
        y = x[src].float() @ W[e].float().T
        out[a:b] = y if row is None else y * row[src] * channel[e]
    return out


def _plain(s):
    op = s["op"]
    if op.startswith("norm"):
        if op == "norm_backward":
            h, rstd, dt, out = s["h"].float(), s["rstd"].unsqueeze(1), s["h"].dtype, ()
        else:
            dt = s["x"].dtype
            h, rstd = _plain_norm(s, dt)
            y = (h * rstd * s["weight"]).to(dt)
            out = (y,) if s["residual"] is None else (h.to(dt), y)
            if s["q"] is not None:
                out += (_kept(y).to(dt),)
        if op != "norm":
            dy = s["dy"].float()
            g = dy * s["weight"]
            dx = rstd * (g - h * rstd * rstd * (g * h).mean(1, keepdim=True))
            if s["dh"] is not None:
                dx = dx + s["dh"].float()
            out += (dx.to(dt), (dy * h * rstd).sum(0))
        return out
    ends, R, k = s["ends"], s["T"] * s["k"], s["k"]
    dt = s["x"].dtype
    if op == "quant_layer":
        h, rstd = _plain_norm(s, dt)
        q, step = _rows8(h * s["weight"])
        au = _plain_mm(q, s["Wu"], ends, s["route"], k, R, step * rstd, s["su"]).to(dt).float()
        m = au.shape[1] // 2
        a, u = au[:, :m], au[:, m:]
        q, step = _rows8(a / (1 + torch.exp(-a)) * u)
        return h.to(dt), _plain_mm(q, s["Wd"], ends, None, k, R, step, s["sd"]).to(dt)
    if op == "quant_mm":
        q, step = _rows8(s["x"].float())
        return (_plain_mm(q, s["W"], ends, s["route"], k, R, step, s["scale"]).to(dt),)
    out = ()
    if op != "mm_backward":
        out += (_plain_mm(s["x"], s["W"], ends, s["route"], k, R).to(dt),)
    if op != "mm":
        x, W, dy = s["x"], s["W"], s["dy"]
        dx, dW = x.new_zeros((R, W.shape[2])), torch.zeros(W.shape, device=W.device)
        for e in range(W.shape[0]):
            a, b = ends[e], ends[e + 1]
            if a == b:
                continue
            g = dy[a:b].float()
            dx[a:b] = (g @ W[e].float()).to(dt)
            dW[e] = g.T @ x[slice(a, b) if s["route"] is None else s["route"][a:b].long() // k].float()
        out += (dx, dW)
    return out


# ------------------------------------------------------- the framework's calls --

def _own(s):
    from paper_2606_00395_amd import binding as B
    op = s["op"]
    if op.startswith("norm"):
        out = ()
        h, rstd = s["h"], s.get("rstd")
        if op != "norm_backward":
            B.rms_norm(s["x"], s["weight"], s["y"], residual=s["residual"], h_out=h, rstd_out=rstd,
                       q=s["q"], scale=s["e"] if s["q"] is not None else None, eps=EPS)
            out = (s["y"],) if h is None else (h, s["y"])
            if s["q"] is not None:
                B.act_unpack(s["q"], s["e"], s["back"])
                out += (s["back"],)
        if op != "norm":
            B.rms_norm_backward(s["dy"], s["x"] if h is None else h, rstd, s["weight"], s["dx"], dh=s["dh"],
                                dweight=s["dweight"])
            out += (s["dx"], s["dweight"])
        return out
    rows = dict(offsets=s["offsets"], route_of_row=s.get("route"), k=s["k"])
    if op == "quant_layer":
        B.rms_norm(s["x"], s["weight"], residual=s["residual"], h_out=s["h"], q=s["q"], row_scale=s["e"], eps=EPS)
        B.grouped_mm_quant(s["q"], s["e"], s["Wu"], s["su"], s["au"], **rows)
        B.swiglu_quant(s["au"], s["hq"], s["he"])
        B.grouped_mm_quant(s["hq"], s["he"], s["Wd"], s["sd"], s["o"], offsets=s["offsets"])
        return s["h"], s["o"]
    if op == "quant_mm":
        B.act_quant(s["x"], s["q"], s["e"])
        B.grouped_mm_quant(s["q"], s["e"], s["W"], s["scale"], s["out"], **rows)
        return (s["out"],)
    out = ()
    if op != "mm_backward":
        B.grouped_mm(s["x"], s["W"], s["out"], **rows)
        out += (s["out"],)
    if op != "mm":
        B.grouped_mm_backward(s["dy"], s["W"], s["dx"], offsets=s["offsets"])
        B.weight_grad(s["dy"], s["x"], s["dW"], **rows)
        out += (s["dx"], s["dW"])
    return out


def run(s):
    return _own(s) if own else _plain(s)


# -------------------------------------------------------------------- work --

def work(case):
    op, a = case["op"], 2 if case["act"] == "bf16" else 4
    T = case["T"]
    if op.startswith("norm"):
        n = T * case["d"]
        forward = n * a * (4 if case["res"] else 2)
        if case["pack"]:
            # the 8-bit form written and read, its values written
            forward += n * (2 + 2 / GROUP + a)
        backward = n * a * (4 if case["res"] else 3)
        return {"bytes": {"norm": forward, "norm_backward": backward}.get(op, forward + backward),
                "flops": n * {"norm": 6, "norm_backward": 10}.get(op, 16)}
    N, k = max(case["N"], 1), case["k"]
    R = T * k
    # experts with rows, as an even load would have them
    E = N * (1 - (1 - k / N) ** T)
    if op == "quant_layer":
        d, m = case["d"], case["m"]
        return {"bytes": 3 * T * d * a + E * 3 * m * d + R * d * a, "flops": 6 * R * m * d}
    n_out, n_in = case["n_out"], case["n_in"]
    x, y, w = (T if case["gather"] else R) * n_in * a, R * n_out * a, E * n_out * n_in
    product = 2 * R * n_out * n_in
    if op == "quant_mm":
        return {"bytes": x + y + w, "flops": product}
    forward = x + y + w * a
    backward = y + w * a + R * n_in * a + x + N * n_out * n_in * 4
    return {"bytes": {"mm": forward, "mm_backward": backward}.get(op, forward + backward),
            "flops": product * {"mm": 1, "mm_backward": 2}.get(op, 3)}


# -------------------------------------------------- the definitions in 64 bits --

def exact(case, seed):
    s = _inputs(case, seed)
    op, dt = case["op"], _dt(case)

    def stored(v):
        """As an intermediate result is kept between two calls."""
        return v.to(dt).double()

    def normed():
        h = s["x"].double()
        if s["residual"] is None:
            return h, h
        h = h + s["residual"].double()
        return h, stored(h)

    def eighths(v):
        """Multiples of a 127th of each row's largest magnitude."""
        step = v.abs().max(1, keepdim=True).values / 127
        return torch.round(v / step.clamp_min(1e-300)) * step

    if op.startswith("norm"):
        w, out = s["weight"].double(), ()
        if op == "norm_backward":
            h, rstd = s["h"].double(), s["rstd"].double().unsqueeze(1)
        else:
            full, h = normed()
            rstd = (h.pow(2).mean(1, keepdim=True) + EPS).pow(-0.5)
            y = h * rstd * w
            out = (y,) if s["residual"] is None else (full, y)
            if case["pack"]:
                out += (_held(stored(y)),)
        if op != "norm":
            dy = s["dy"].double()
            n = h * rstd
            g = dy * w
            dx = rstd * (g - n * (g * n).mean(1, keepdim=True))
            out += (dx if s["dh"] is None else dx + s["dh"].double(), torch.einsum("td,td->d", dy, n))
        return out

    N, k = case["N"], case["k"]
    R = case["T"] * k
    bounds = s["offsets"].cpu().tolist() if N else [0, R]

    def each(fn):
        for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
            if b > a:
                fn(e, a, b)

    def source(a, b, gathered):
        return torch.div(s["route"][a:b].long(), k, rounding_mode="floor") if gathered else torch.arange(
            a, b, device="cuda")

    def products(x, weights, gathered):
        out = torch.zeros((R, weights(0).shape[0]), dtype=torch.float64, device="cuda")

        def one(e, a, b):
            out[a:b] = torch.mm(x[source(a, b, gathered)], weights(e).t())
        each(one)
        return out

    if op == "quant_layer":
        full, h = normed()
        rstd = (h.pow(2).mean(1, keepdim=True) + EPS).pow(-0.5)
        v = eighths(h * s["weight"].double()) * rstd
        au = stored(products(v, lambda e: s["Wu"][e].double() * s["su"][e].double().unsqueeze(1), True))
        a, u = au[:, :case["m"]], au[:, case["m"]:]
        v = eighths(a * torch.sigmoid(a) * u)
        return full, products(v, lambda e: s["Wd"][e].double() * s["sd"][e].double().unsqueeze(1), False)
    gathered = s.get("route") is not None
    x = s["x"].double()
    if op == "quant_mm":
        return (products(eighths(x), lambda e: s["W"][e].double() * s["scale"][e].double().unsqueeze(1), gathered),)
    out = ()
    if op != "mm_backward":
        out += (products(x, lambda e: s["W"][e].double(), gathered),)
    if op != "mm":
        dx = torch.zeros((R, case["n_in"]), dtype=torch.float64, device="cuda")
        dW = torch.zeros((max(N, 1), case["n_out"], case["n_in"]), dtype=torch.float64, device="cuda")

        def gradients(e, a, b):
            g = s["dy"][a:b].double()
            dx[a:b] = torch.mm(g, s["W"][e].double())
            dW[e] = torch.mm(g.t(), x[source(a, b, gathered)])
        each(gradients)
        out += (dx, dW)
    return out


def _held(x):
    """int8 multiples of a power of two that brings each group's largest below 128."""
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], GROUP):
        part = x[:, c:c + GROUP]
        _, two = torch.frexp(part.abs().amax(1, keepdim=True))
        step = torch.exp2(torch.clamp(two - 7, min=-126).double())
        out[:, c:c + GROUP] = torch.clamp(torch.round(part / step), -127, 127) * step
    return out
