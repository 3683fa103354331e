"""pr2_token_logprob, pr2_policy_loss and pr2_policy_loss_backward against the float64
definitions.

Tolerances (set from the arithmetic, before any run): a logp is (z_y - M) / tau - ln S in
fp32; S sums at most V terms, a thread a few hundred of them one after the other, so its
relative error stays below 1e-5 at the sizes here; the exponent of a term of weight p has
relative error 2^-22, which in p is at most 2^-22 |ln p|.  So logp and entropy within
1e-5 + 4e-7 |value| (entropy: times its largest exponent, below 40), p within 3e-5
relatively; coef by its derivative in logp; bf16 outputs within 2^-8 more.
"""
import numpy as np
import pytest

from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu

BF = "bf16"


def make(seed, T, V, act, ld=None, ref=True, banned=0, scale=2.5, offset=0):
    """Inputs on the device (logits a view of rows ld apart, starting `offset` elements in)
    and as float64."""
    import torch
    g = np.random.default_rng([seed, T, V])
    ld = V if ld is None else ld
    flat = torch.from_numpy((scale * g.standard_normal(offset + T * ld)).astype(np.float32))
    flat = flat.to(torch.bfloat16 if act == BF else torch.float32).cuda()
    logits = flat[offset:].view(T, ld)[:, :V]
    y = g.integers(0, max(1, V - banned), T)
    if banned:
        logits[:, V - banned:] = float("-inf")
    z = logits.float().cpu().numpy()
    logp = O.token_stats(z, y)[0]
    f = lambda a: np.asarray(a, dtype=np.float32)
    moved = g.normal(0, 0.2, T)
    for b in (0.8, 1.28):        # no ratio within rounding of a bound, where coef jumps
        moved = np.where(np.abs(np.exp(moved) - b) < 1e-3, moved + 0.01, moved)
    host = dict(logits=z, token=y, logp_old=f(logp - moved), adv=f(g.normal(0, 1, T)),
                logp_ref=f(logp + g.normal(0, 0.3, T)) if ref else None,
                weight=f(g.uniform(0.1, 1, T) / T), kl_coef=0.05 if ref else 0.0, inv_temp=1.0)
    return logits, host


def up(a, dtype=None):
    import torch
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def call(logits, host, split=False, inplace=False, tok="int64", want_grad=True, grad_loss=None):
    import torch
    from paper_2606_00395_amd import binding as B
    T, V = logits.shape
    nan = lambda *s, dt=torch.float32: torch.full(s, float("nan"), device="cuda", dtype=dt)
    out = {n: nan(T) for n in ("logp", "lse", "entropy", "coef")}
    out["sums"] = nan(4)
    tokens = up(host["token"], torch.int64 if tok == "int64" else torch.int32)
    out["dlogits"] = (logits if inplace else nan(T, V, dt=logits.dtype)) if want_grad else None
    B.policy_loss(logits, tokens, up(host["logp_old"]), up(host["adv"]), out["sums"],
                  logp_ref=up(host["logp_ref"]), weight=up(host["weight"]), logp_out=out["logp"],
                  lse_out=out["lse"], entropy_out=out["entropy"], coef_out=out["coef"],
                  dlogits=out["dlogits"] if not split else None, clip_low=0.2, clip_high=0.28,
                  kl_coef=host["kl_coef"], inv_temp=host["inv_temp"])
    if split:
        B.policy_loss_backward(logits, tokens, out["lse"], out["coef"], out["dlogits"],
                               grad_loss=grad_loss, inv_temp=host["inv_temp"])
    torch.cuda.synchronize()
    return {n: None if t is None else t.double().cpu().numpy() for n, t in out.items()}


def compare(got, host, bf16, factor=1.0):
    ref = O.policy_loss(**host, clip_low=np.float32(0.2), clip_high=np.float32(0.28))
    on = ref["lse"] > -np.inf
    tol = 1e-5 + 4e-7 * np.abs(ref["logp"])
    assert np.all(np.abs(got["logp"] - ref["logp"]) <= tol)
    assert np.all(got["lse"][~on] == -np.inf)
    assert np.all(np.abs(got["lse"][on] - ref["lse"][on]) <= 1e-5 + 4e-7 * np.abs(ref["lse"][on]))
    assert np.all(np.abs(got["entropy"] - ref["entropy"]) <= 4e-5 * (1 + ref["entropy"]))
    w = np.ones(len(on)) if host["weight"] is None else host["weight"]
    A, r = np.abs(host["adv"]), np.exp(ref["logp"] - host["logp_old"])
    d = np.zeros(len(on)) if host["logp_ref"] is None else host["logp_ref"] - ref["logp"]
    tc = w * (A * r + host["kl_coef"] * np.exp(d)) * 2e-5 * on
    assert np.all(np.abs(got["coef"] - ref["coef"]) <= tc)
    terms = w * on * (A * np.maximum(r, 1.3) + (host["kl_coef"] + 1) * (np.exp(d) + 1) + ref["entropy"])
    assert np.all(np.abs(got["sums"] - ref["sums"]) <= 4e-5 * np.sum(terms) + 1e-30)
    if got["dlogits"] is None:
        return ref
    it, c = host["inv_temp"], np.abs(ref["coef"])
    share = np.abs(ref["p"])
    share[np.arange(len(on)), np.clip(host["token"], 0, share.shape[1] - 1)] = 1.0
    want = factor * ref["dlogits"]
    tol = abs(factor) * it * (tc + 3e-5 * c)[:, None] * share + 1e-37
    if bf16:
        tol = tol + 2.0 ** -8 * np.abs(want) + 1e-37
    assert np.all(np.abs(got["dlogits"] - want) <= tol)
    return ref


SIZES = [(17, 20001), (16, 9001), (1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (1, 1000), (9, 4097), (2, 33001), (1, 165001),
         (200, 1030), (195, 4200), (193, 33100), (192, 70001), (192, 165000)]


@pytest.mark.parametrize("act", [BF, "f32"])
@pytest.mark.parametrize("T,V", SIZES, ids=[f"{T}x{V}" for T, V in SIZES])
def test_loss_and_gradient(T, V, act):
    logits, host = make(1, T, V, act, banned=V // 10)
    compare(call(logits, host), host, act == BF)


@pytest.mark.parametrize("split", [False, True], ids=["one_call", "two_calls"])
@pytest.mark.parametrize("T", [6, 210])
@pytest.mark.parametrize("ld,offset", [(1003, 0), (1001, 1), (1024, 3), (1040, 8)])
@pytest.mark.parametrize("act", [BF, "f32"])
def test_strides_and_alignment(T, ld, offset, act, split):
    import torch
    logits, host = make(2, T, 1001, act, ld=ld, offset=offset, ref=False)
    host["inv_temp"] = 0.7
    host["logp_old"] = (O.token_stats(host["logits"], host["token"], 0.7)[0] + 0.05).astype(np.float32)
    tok = "int32" if offset else "int64"
    compare(call(logits, host, split=split, tok=tok), host, act == BF)
    # in place: the padding between the rows stays as it was
    whole = logits.as_strided((T - 1, ld), (ld, 1), logits.storage_offset())
    pad = whole[:, 1001:].clone()
    got = call(logits, host, split=split, inplace=True, tok=tok)
    compare(got, host, act == BF)
    assert torch.equal(whole[:, 1001:], pad)


@pytest.mark.parametrize("T", [5, 230])
def test_rows_that_do_not_count(T):
    """Weight 0, a token out of range, every logit -inf: zeros, whatever else stands there."""
    import torch
    logits, host = make(3, T, 2051, BF)
    host["weight"][0] = 0.0
    host["token"][1] = -1
    host["token"][2] = 2051
    logits[0] = float("nan")
    logits[1, 5] = float("inf")
    logits[3] = float("-inf")
    for n in ("logp_old", "adv", "logp_ref"):
        host[n][:3] = np.nan
    host["logits"] = logits.float().cpu().numpy()
    for split in (False, True):
        got = call(logits, host, split=split)
        clean = {n: (np.nan_to_num(v) if isinstance(v, np.ndarray) and v.dtype == np.float32
                     and v.ndim == 1 else v) for n, v in host.items()}
        compare(got, clean, True)
        assert np.all(got["dlogits"][:4] == 0) and np.all(got["coef"][:4] == 0)
    torch.cuda.synchronize()


def test_a_nan_in_a_row_that_counts_is_seen():
    for T in (4, 220):
        logits, host = make(4, T, 1500, BF)
        logits[1, 700] = float("nan")
        logits[2, 3] = float("inf")
        host["logits"] = logits.float().cpu().numpy()
        for split in (False, True):
            got = call(logits, host, split=split)
            assert np.isnan(got["logp"][1:3]).all() and np.isnan(got["sums"][0])
            assert np.isnan(got["dlogits"][1:3]).all()
            assert np.isfinite(got["dlogits"][3:]).all() and np.isfinite(got["logp"][3:]).all()


def test_lowest_numbers_and_far_logits():
    import torch
    logits, host = make(5, 200, 1100, "f32")
    low = torch.finfo(torch.float32).min
    logits[0] = low                       # uniform
    logits[1, 100:] = low                 # masked by the lowest number
    logits[2] = logits[2] * 1000
    logits[3] = logits[3] - 3e38          # far below the running maximum's start
    host["token"][1] = 7
    host["logits"] = logits.cpu().numpy()
    lp = O.token_stats(host["logits"], host["token"], 2.0)[0]
    host["inv_temp"] = 2.0
    host["logp_old"] = lp.astype(np.float32)
    host["logp_ref"] = (lp + 0.1).astype(np.float32)
    host["weight"][2] = 0.0               # a token of probability 0 is not this test's
    for split in (False, True):
        got = call(logits, host, split=split)
        assert abs(got["logp"][0] + np.log(1100)) < 1e-5
        assert np.abs(got["entropy"][0] - np.log(1100)) < 1e-4
        assert np.all(got["dlogits"][1, 100:] == 0)
        keep = [i for i in range(200) if i not in (0, 3)]
        sub = {n: (v[keep] if isinstance(v, np.ndarray) else v) for n, v in host.items()}
        one = {n: v[keep] for n, v in got.items() if n != "sums"}
        # (rows 0 and 3 apart: lse itself has no digits left at 3e38)
        ref = O.policy_loss(**sub)
        assert np.all(np.abs(one["logp"] - ref["logp"]) <= 1e-5 + 4e-7 * np.abs(ref["logp"]))
        assert np.abs(one["dlogits"] - ref["dlogits"]).max() <= 1e-4 * np.abs(ref["coef"]).max()


def test_log_probabilities_alone():
    import torch
    from paper_2606_00395_amd import binding as B
    for T, V, act in ((1, 50257, BF), (7, 151936, BF), (300, 1003, "f32"), (2500, 520, BF)):
        logits, host = make(6, T, V, act, banned=V // 50)
        host["token"][0] = -1 if T > 1 else host["token"][0]
        logp, lse, ent = (torch.full((T,), float("nan"), device="cuda") for _ in range(3))
        B.token_logprob(logits, up(host["token"]), logp, lse, ent, inv_temp=1.25)
        ref = O.token_stats(host["logits"], host["token"], 1.25)
        on = ref[1] > -np.inf
        assert np.all(np.abs(logp.cpu().numpy() - ref[0]) <= 1e-5 + 4e-7 * np.abs(ref[0]))
        assert np.all(lse.cpu().numpy()[~on] == -np.inf)
        assert np.all(np.abs(lse.cpu().numpy()[on] - ref[1][on]) <= 2e-5)
        assert np.all(np.abs(ent.cpu().numpy() - ref[2]) <= 4e-5 * (1 + ref[2]))
        # the rollout's record and the training pass agree bit for bit where the same kernel runs
        again = torch.empty_like(logp)
        B.token_logprob(logits, up(host["token"]), again, inv_temp=1.25)
        assert torch.equal(again, logp)


def test_clip_kl_and_weights_at_their_edges():
    logits, host = make(7, 200, 600, "f32")
    lp = O.token_stats(host["logits"], host["token"])[0]
    g = np.random.default_rng(1)
    host["logp_old"] = (lp - np.where(g.random(200) < 0.5, 1.0, -1.0)).astype(np.float32)
    host["adv"][::5] = 0.0
    ref = compare(call(logits, host), host, False)
    assert 0 < ref["sums"][2]
    host["adv"][:] = 0.0
    host["logp_old"][:] = -1e30            # a ratio of infinity under an advantage of 0
    got = call(logits, host)
    assert np.isfinite(got["dlogits"]).all() and np.isfinite(got["sums"]).all()
    host["weight"] = None
    host["logp_old"] = lp.astype(np.float32)
    host["adv"][:] = 1.0
    compare(call(logits, host), host, False)


def test_gradient_against_differences_of_the_loss():
    """The gradient along random directions is the loss's slope (differences of the
    float64 loss)."""
    for T, split in ((40, True), (40, False), (220, False)):
        logits, host = make(8, T, 300, "f32")
        got = call(logits, host, split=split)
        g = np.random.default_rng(2)
        for _ in range(3):
            v = g.standard_normal(host["logits"].shape)
            f = [O.policy_loss(**{**host, "logits": host["logits"] + s * 1e-5 * v})["sums"][0]
                 for s in (1, -1)]
            slope = (f[0] - f[1]) / 2e-5
            dot = np.sum(got["dlogits"] * v)
            # rounding: 3e-5 of the gradient's norm along a random direction
            assert abs(dot - slope) <= 1e-4 * np.linalg.norm(got["dlogits"]) + 1e-9


def test_backward_scaled_by_the_loss_gradient():
    import torch
    logits, host = make(9, 12, 900, "f32")
    got = call(logits, host, split=True, grad_loss=torch.tensor([-2.5], device="cuda"))
    compare(got, host, False, factor=-2.5)


def test_no_rows():
    import torch
    from paper_2606_00395_amd import binding as B
    z = torch.empty((0, 50), device="cuda")
    e = torch.empty(0, device="cuda")
    sums = torch.full((4,), 3.0, device="cuda")
    B.policy_loss(z, e.long(), e, e, sums, dlogits=torch.empty_like(z))
    B.token_logprob(z, e.long(), e)
    B.policy_loss_backward(z, e.long(), e, e, torch.empty_like(z))
    assert torch.all(sums == 0)


def test_offsets_past_two_to_the_31():
    """Logits of 2.2e9 elements: the last rows' results are those of the rows alone."""
    import torch
    from paper_2606_00395_amd import binding as B
    T, V = 16500, 131100
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.zeros((T, V), dtype=torch.bfloat16, device="cuda")
    assert T * V > 2 ** 31
    tail = torch.randn((300, V), generator=g, device="cuda").mul_(3).to(torch.bfloat16)
    z[-300:] = tail
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    old = torch.full((T,), -12.0, device="cuda")
    adv = torch.randn(T, generator=g, device="cuda")
    w = torch.zeros(T, device="cuda")
    w[-300:] = 0.01
    out = []
    for zz, sl in ((z, slice(None)), (tail, slice(-300, None))):
        n = zz.shape[0]
        logp, sums = torch.empty(n, device="cuda"), torch.empty(4, device="cuda")
        keep = zz.clone()
        B.policy_loss(keep, y[sl], old[sl].contiguous(), adv[sl].contiguous(), sums,
                      weight=w[sl].contiguous(), logp_out=logp, dlogits=keep)
        lp = torch.empty(n, device="cuda")
        B.token_logprob(zz, y[sl], lp)
        out.append((logp[-300:].clone(), sums, keep[-300:].clone(), lp[-300:].clone()))
        assert torch.all(keep[:n - 300] == 0)
        del keep
    for a, b in zip(out[0][:3], out[1][:3]):
        assert torch.equal(a, b)
    # (the two calls split their rows differently)
    assert torch.all((out[0][3] - out[1][3]).abs() <= 2e-5 + 8e-7 * out[1][3].abs())


def test_another_stream_and_graph_replays():
    import torch
    from paper_2606_00395_amd import binding as B
    for T in (16, 256):
        logits, host = make(10, T, 8192, BF)
        args = [up(host[n]) for n in ("token", "logp_old", "adv")]
        w, ref = up(host["weight"]), up(host["logp_ref"])
        ws = B.policy_workspace(logits)
        sums, grad = torch.empty(4, device="cuda"), torch.empty_like(logits)

        def step(stream=None):
            B.policy_loss(logits, *args, sums, logp_ref=ref, weight=w, dlogits=grad, kl_coef=0.1,
                          ws=ws, stream=stream)

        step()
        torch.cuda.synchronize()
        want = (sums.clone(), grad.clone())
        side = torch.cuda.Stream()
        for t in (sums, grad):
            t.fill_(float("nan"))
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        torch.cuda.synchronize()
        assert torch.equal(sums, want[0]) and torch.equal(grad, want[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for rep in range(4):
            for t in (sums, grad):
                t.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(sums, want[0]) and torch.equal(grad, want[1]), rep
            junk = torch.empty_like(logits)
            B.policy_loss(torch.roll(logits, 1, 0), *args, torch.empty(4, device="cuda"), weight=w,
                          dlogits=junk, ws=ws)
            torch.cuda.synchronize()


def test_refusals_of_the_binding():
    import torch
    from paper_2606_00395_amd import binding as B
    z = torch.zeros((4, 10), device="cuda")
    y = torch.zeros(4, dtype=torch.int64, device="cuda")
    f = torch.zeros(4, device="cuda")
    with pytest.raises(TypeError):
        B.token_logprob(z.half(), y, f)
    with pytest.raises(TypeError):
        B.token_logprob(z, y.float(), f)
    with pytest.raises(ValueError):
        B.token_logprob(z.t(), torch.zeros(10, dtype=torch.int64, device="cuda"), torch.zeros(10, device="cuda"))
    with pytest.raises(ValueError):
        B.token_logprob(z[:1].expand(4, 10), y, f)
    with pytest.raises(ValueError):
        B.token_logprob(z, y[:3], f)
    with pytest.raises(ValueError):
        B.token_logprob(z, y.cpu(), f)
    with pytest.raises(TypeError):
        B.policy_loss(z, y, f, f, f, dlogits=z.bfloat16())
    with pytest.raises(B.Pr2Error, match="inv_temp"):
        B.token_logprob(z, y, f, inv_temp=0.0)
    with pytest.raises(B.Pr2Error, match="overlaps"):
        wide = torch.zeros((4, 20), device="cuda")
        B.policy_loss(wide[:, :10], y, f, f, torch.zeros(4, device="cuda"), dlogits=wide[:, 5:15])


def test_many_long_rows_taken_in_turns():
    """2300 rows that take a CU each, a third of them without weight: the rows' results are
    those of the same rows in batches too small for turns, bit for bit, whatever order the
    turns came in; and rows of a sample against the definition."""
    import torch
    from paper_2606_00395_amd import binding as B
    T, V = 2300, 80003
    g = torch.Generator(device="cuda").manual_seed(11)
    z = torch.empty((T, V), dtype=torch.bfloat16, device="cuda")
    for t0 in range(0, T, 100):
        z[t0:t0 + 100] = torch.randn((100, V), generator=g, device="cuda").mul_(3).to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    old = torch.full((T,), -12.0, device="cuda")
    adv = torch.randn(T, generator=g, device="cuda")
    w = (torch.rand(T, generator=g, device="cuda") > 0.33).float() / T
    logp, coef, sums = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(4, device="cuda")
    grad = torch.empty_like(z)
    for _ in range(3):
        for t in (logp, coef, sums, grad):
            t.fill_(float("nan"))
        B.policy_loss(z, y, old, adv, sums, weight=w, logp_out=logp, coef_out=coef, dlogits=grad)
    for t0 in range(0, T, 575):
        sl = slice(t0, t0 + 575)
        lp, cf, gr = torch.empty(575, device="cuda"), torch.empty(575, device="cuda"), torch.empty_like(grad[sl])
        B.policy_loss(z[sl], y[sl], old[sl], adv[sl], torch.empty(4, device="cuda"), weight=w[sl], logp_out=lp,
                      coef_out=cf, dlogits=gr)
        assert torch.equal(lp, logp[sl]) and torch.equal(cf, coef[sl]) and torch.equal(gr, grad[sl])
    pick = torch.cat([torch.arange(6, device="cuda"), torch.arange(T - 6, T, device="cuda")])
    host = dict(logits=z[pick].float().cpu().numpy(), token=y[pick].cpu().numpy(), logp_old=old[pick].cpu().numpy(),
                adv=adv[pick].cpu().numpy(), logp_ref=None, weight=w[pick].cpu().numpy(), kl_coef=0.0, inv_temp=1.0)
    ref = O.policy_loss(**host, clip_low=np.float32(0.2), clip_high=np.float32(0.28))
    got = grad[pick].double().cpu().numpy()
    assert np.all(np.abs(logp[pick].cpu().numpy() - ref["logp"]) <= 1e-5 + 4e-7 * np.abs(ref["logp"]))
    assert np.all(np.abs(got - ref["dlogits"]) <= 2.0 ** -7 * np.abs(ref["dlogits"]) + 1e-37)
    in_place = z
    B.policy_loss(in_place, y, old, adv, sums, weight=w, dlogits=in_place)
    assert torch.equal(in_place, grad)


# the widths at which a row's threads and pieces change
@pytest.mark.parametrize("act", [BF, "f32"])
@pytest.mark.parametrize("T,V", [(3, 2041), (5, 2048), (2, 2049), (3, 4089), (1, 4096), (300, 1017), (2, 8192), (3, 8193)])
def test_loss_and_gradient_of_short_rows(T, V, act):
    test_loss_and_gradient(T, V, act)


def test_more_rows_than_a_grid_of_one_dimension_holds():
    """2^24 rows and more, as many workgroups of 256: the first and last rows' results are those
    of the rows alone."""
    import torch
    from paper_2606_00395_amd import binding as B
    T, V, n = 2 ** 24 + 5, 3, 1000
    g = torch.Generator(device="cuda").manual_seed(4)
    z = torch.randn((T, V), generator=g, device="cuda").to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    old = torch.full((T,), -1.0, device="cuda")
    adv = torch.randn(T, generator=g, device="cuda")
    nan = lambda *s, dt=torch.float32: torch.full(s, float("nan"), device="cuda", dtype=dt)

    def run(z, y, old, adv):
        T = len(y)
        out = [nan(T) for _ in range(5)] + [nan(T, V, dt=z.dtype) for _ in range(2)]
        lp, logp, lse, ent, coef, once, twice = out
        sums = nan(4)
        B.token_logprob(z, y, lp)
        B.policy_loss(z, y, old, adv, sums, logp_out=logp, lse_out=lse, entropy_out=ent, coef_out=coef)
        B.policy_loss_backward(z, y, lse, coef, twice)
        B.policy_loss(z, y, old, adv, nan(4), dlogits=once)
        return out, sums

    whole, sums = run(z, y, old, adv)
    for sl in (slice(0, n), slice(T - n, T)):
        for a, b in zip(whole, run(z[sl], y[sl], old[sl], adv[sl])[0]):
            assert torch.equal(a[sl], b)
    lp, _, _, _, _, once, twice = whole
    assert torch.isfinite(lp).all() and torch.isfinite(once).all() and torch.isfinite(twice).all()
    want = torch.log_softmax(z.double(), 1).gather(1, y.long()[:, None])[:, 0]
    assert torch.all((lp.double() - want).abs() <= 1e-5 + 4e-7 * want.abs())
    assert torch.isfinite(sums).all()


# Levels of the logits: p and 1 - p_y depend on differences alone, however far from zero the row
# lies (None: every logit the lowest finite number).
LEVELS = (0.0, 1e3, -1e3, 1e4, -1e4, 1e6, -1e6, None)


def far_rows(T, V, act):
    """Rows at every level; every third row's token takes nearly all of the probability."""
    import torch
    g = np.random.default_rng([12, T, V])
    z = 2.5 * g.standard_normal((T, V))
    y = g.integers(0, V, T)
    z[np.arange(0, T, 3), y[::3]] = 28.0
    for t in range(T):
        level = LEVELS[t % len(LEVELS)]
        z[t] = np.finfo(np.float32).min if level is None else z[t] + level
    logits = torch.from_numpy(z).to(torch.float32)
    if act == BF:
        low = logits == torch.finfo(torch.float32).min
        logits = logits.to(torch.bfloat16)
        logits[low] = torch.finfo(torch.bfloat16).min
    host_z = logits.float().numpy()
    logp = O.token_stats(host_z, y)[0]
    f = lambda a: np.asarray(a, dtype=np.float32)
    host = dict(logits=host_z, token=y, logp_old=f(logp - 0.05), adv=f(g.choice([-1.5, 0.7], T)),
                logp_ref=f(logp + g.normal(0, 0.3, T)), weight=f(g.uniform(0.1, 1, T) / T), kl_coef=0.05,
                inv_temp=1.0)
    return logits.cuda(), host


def check_far_gradient(got, host, bf16, log_p_error=0.0):
    """Every entry to its own size: an error e of a log-probability moves p by e p and 1 - p_y by
    e p_y.  logp is within 1e-5 (see above), the other terms' exponents within 3e-5."""
    ref = O.policy_loss(**host, clip_low=np.float32(0.2), clip_high=np.float32(0.28))
    rows = np.arange(len(host["token"]))
    r, d = np.exp(ref["logp"] - host["logp_old"]), host["logp_ref"] - ref["logp"]
    tc = host["weight"] * (np.abs(host["adv"]) * r + host["kl_coef"] * np.exp(d)) * 2e-5
    c, p = np.abs(ref["coef"]), ref["p"]
    py = p[rows, host["token"]]
    e = np.broadcast_to(np.asarray(log_p_error, dtype=np.float64), py.shape)
    e = np.expm1(np.minimum(e, 50.0))
    tol = (tc + (3e-5 + e) * c)[:, None] * p
    tol[rows, host["token"]] = (tc + 3e-5 * c) * (1 - py) + (1.02e-5 + e) * c * py
    want = ref["dlogits"]
    if bf16:
        tol = tol + 2.0 ** -8 * np.abs(want)
    assert np.all(np.abs(got["dlogits"] - want) <= host["inv_temp"] * tol + 1e-37)


# (T rows of V: both sides of the number of long rows from which on a row is one workgroup's)
@pytest.mark.parametrize("act,V", [(BF, 80000), ("f32", 40000)])
@pytest.mark.parametrize("T", [1, 9, 48, 195])
def test_gradient_of_logits_far_from_zero(T, act, V):
    logits, host = far_rows(T, V, act)
    got = call(logits, host)
    compare(dict(got, dlogits=None), host, act == BF)
    check_far_gradient(got, host, act == BF)


@pytest.mark.parametrize("act,V", [(BF, 80000), ("f32", 40000)])
@pytest.mark.parametrize("T", [9, 48, 195])
def test_gradient_from_lse_far_from_zero(T, act, V):
    """Two calls: log p within the rounding of lse, |lse| 2^-23, as the header states."""
    logits, host = far_rows(T, V, act)
    got = call(logits, host, split=True)
    compare(dict(got, dlogits=None), host, act == BF)
    check_far_gradient(got, host, act == BF, log_p_error=np.abs(got["lse"]) * 2.0 ** -23)


@pytest.mark.parametrize("act", [BF, "f32"])
@pytest.mark.parametrize("T", [7, 210])
def test_logits_and_gradient_as_column_halves_of_one_buffer(T, act):
    """Each in its half, at odd starts; the gradient is that of a buffer of its own."""
    import torch
    from paper_2606_00395_amd import binding as B
    logits, host = make(13, T, 1001, act)
    both = torch.full((T, 2051), 7.0, dtype=logits.dtype, device="cuda")
    z, g = both[:, 1:1002], both[:, 1003:2004]
    z.copy_(logits)
    args = [up(host[n]) for n in ("token", "logp_old", "adv")]
    want = torch.full_like(logits, float("nan"))
    sums = [torch.empty(4, device="cuda") for _ in range(2)]
    B.policy_loss(logits, *args, sums[0], dlogits=want)
    B.policy_loss(z, *args, sums[1], dlogits=g)
    assert torch.equal(g, want) and torch.equal(z, logits) and torch.equal(*sums)
    for c in (0, 1002, 2004, 2050):
        assert torch.all(both[:, c] == 7)


@pytest.mark.parametrize("split", [False, True], ids=["one_call", "two_calls"])
@pytest.mark.parametrize("T,V", [(4, 1500), (220, 1500), (4, 80003)])
def test_nan_logits_under_an_advantage_of_zero(T, V, split):
    """Neither loss nor gradient depends on the row then, and neither is NaN; what does is."""
    logits, host = make(14, T, V, BF)
    logits[1, 700], logits[2, 3] = float("nan"), float("inf")
    host["adv"][1:3] = 0.0
    for ref, beta in ((None, 0.0), (host["logp_ref"], 0.0)):
        host.update(logp_ref=ref, kl_coef=beta)
        got = call(logits, host, split=split)
        assert np.isnan(got["logp"][1:3]).all() and np.isnan(got["lse"][1:3]).all()
        assert np.isnan(got["entropy"][1:3]).all() and np.isnan(got["sums"][3])
        assert np.all(got["coef"][1:3] == 0) and np.all(got["dlogits"][1:3] == 0)
        assert np.isfinite(got["sums"][0]) and np.isnan(got["sums"][1]) == (ref is not None)
        assert np.isfinite(got["dlogits"]).all()
    host["kl_coef"] = 0.1
    got = call(logits, host, split=split)
    assert np.isnan(got["coef"][1:3]).all() and np.isnan(got["dlogits"][1:3]).all() and np.isnan(got["sums"][0])
