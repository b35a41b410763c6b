"""The clipped policy loss and its gradient on the GPU against float64."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

EPS32, STEP16 = 2.0 ** -24, 2.0 ** -8  # half a step of float32 / bf16, relative


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available()
    import paper_2505_22296_amd as m
    m.load()
    return m


def make(T, V, cu, seed, per_token=False, spread=2.0, ignored=0.2):
    """Inputs in float64 on the CPU (bf16 / float32 values): likely labels, some
    ignored, ratios on both sides of the clip and none within 1e-3 of its borders."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(T, V, generator=g) * spread).bfloat16().double()
    label = torch.randint(0, V, (T,), generator=g)
    x[torch.arange(T), label] = (math.log(V) + torch.randn(T, generator=g)).bfloat16().double()
    logp = torch.log_softmax(x, 1)[torch.arange(T), label]
    ratio = 0.3 * torch.randn(T, generator=g).double()
    for edge in (math.log(0.8), math.log(1.3)):
        ratio = torch.where((ratio - edge).abs() < 2e-3, ratio + 5e-3, ratio)
    lab = torch.where(torch.rand(T, generator=g) < ignored, torch.full_like(label, -100), label)
    n = len(cu) - 1
    return dict(x=x, labels=lab, old=(logp - ratio).float().double(),
                ref=(logp + 0.3 * torch.randn(T, generator=g).double()).float().double(),
                adv=torch.randn(T if per_token else n, generator=g).double(),
                grad=torch.randn(n, generator=g).double(), cu=list(cu), per_token=per_token)


def reference(d, kl=0.1, ent_coef=0.01, use_ref=True, clip=(0.2, 0.3)):
    """Every value and the gradient (autograd) of the definition, in float64."""
    T, V = d["x"].shape
    n = len(d["cu"]) - 1
    seq = torch.full((T,), -1)
    for s in range(n):
        seq[d["cu"][s]:d["cu"][s + 1]] = s
    live = (seq >= 0) & (d["labels"] >= 0) & (d["labels"] < V)
    x = d["x"].clone().requires_grad_()
    rows = torch.nonzero(live)[:, 0]
    z, lab, of = x[rows], d["labels"][rows], seq[rows]
    A = d["adv"][rows] if d["per_token"] else d["adv"][of]
    q = torch.log_softmax(z, 1)
    lp = q.gather(1, lab[:, None])[:, 0]
    p = q.exp()
    ent = -(p * torch.where(p > 0, q, torch.zeros_like(q))).sum(1)
    r = torch.exp(lp - d["old"][rows])
    held = r.clamp(1 - clip[0], 1 + clip[1])
    term = -torch.minimum(r * A, held * A) - ent_coef * ent
    klv = torch.zeros_like(term)
    if use_ref:
        dd = d["ref"][rows] - lp
        klv = torch.expm1(dd) - dd
        term = term + kl * klv
    G = d["grad"][of]
    (G * term).sum().backward()

    def per_seq(v):
        return torch.zeros(n, dtype=torch.float64).index_add_(0, of, v.detach())

    def per_tok(v):
        return torch.zeros(T, dtype=torch.float64).index_copy_(0, rows, v.detach())
    return dict(logp=per_tok(lp), lse=per_tok(torch.logsumexp(z, 1)), ent=per_tok(ent), sums=per_seq(term),
                stats=torch.stack([per_seq(klv), per_seq(ent), per_seq((r * A > held * A).double()),
                                   per_seq(torch.ones_like(term))], 1),
                dx=x.grad, live=live, size=per_seq(term.abs() + klv.abs() + r * A.abs() + 1))


def device(d):
    f = lambda k, t: d[k].to(t).cuda()  # noqa: E731
    return dict(x=f("x", torch.bfloat16), labels=f("labels", torch.int32), old=f("old", torch.float32),
                ref=f("ref", torch.float32), adv=f("adv", torch.float32), grad=f("grad", torch.float32))


def check(name, got, want, tol):
    off = (got.double().cpu() - want).abs() - tol
    assert torch.isfinite(got).all() and (off <= 0).all(), f"{name}: {off.max().item():.3e} past its tolerance"


def lse_tol(d, want):
    # a thread sums V / 256 terms one by one, each rounded by at most half a step
    # (the reference's own are not), their exponents by half a step of at most 2^6;
    # the joins add 14 roundings; storing rounds once
    V = d["x"].shape[1]
    return EPS32 * (V / 256 + 32 + 64 + 14) + EPS32 * want.abs()


CASES = [  # T, V, cu, per_token
    (1, 8, [0, 1], False), (5, 8, [0, 2, 5], True), (3, 1000, [0, 3], False), (40, 1000, [2, 2, 17, 33], False),
    (300, 2056, [0, 100, 101, 260], True), (2100, 264, [0, 700, 2100], False), (7, 152064, [0, 7], False),
    (1500, 4104, [0] + [1500], True), (64, 8200, list(range(0, 65)), False),
]


@pytest.mark.parametrize("T,V,cu,per_token", CASES)
@pytest.mark.parametrize("kl,ent", [(0.1, 0.01), (0.0, 0.0)])
def test_policy_loss_matches_definition(sp, T, V, cu, per_token, kl, ent):
    d = make(T, V, cu, seed=T + V, per_token=per_token)
    want, x = reference(d, kl, ent), device(d)
    p = sp.PolicyParams(0.2, 0.3, kl, ent, adv_per_token=per_token)
    logp, lse, e, sums, stats = sp.sp_policy_loss(p, x["x"], x["labels"], x["old"], x["ref"], x["adv"], cu)
    tol = lse_tol(d, want["lse"])
    check("lse", lse, want["lse"], tol)
    check("logp", logp, want["logp"], tol)
    # u / s: the entropy is a mean of exponents of at most 2^6, each rounded
    check("entropy", e, want["ent"], 64 * tol)
    # a term moves with logp by less than its size in `size`, and is rounded once
    # more when it waits in float32 for the sum
    size = want["size"][:, None]
    check("seq_sum", sums, want["sums"], (2 * tol.max() * (1 + 64 * ent) + EPS32 * 4) * size[:, 0])
    check("stats", stats[:, :2], want["stats"][:, :2],
          (64 * tol.max() + EPS32 * 4) * size + EPS32 * want["stats"][:, :2].abs())
    assert torch.equal(stats[:, 2:].cpu().double(), want["stats"][:, 2:])
    dl = sp.sp_policy_loss_bwd(p, x["x"], x["labels"], logp, lse, e, x["old"], x["ref"], x["adv"], cu, x["grad"])
    dx = want["dx"]
    # g = O(G (|A| r + kl e^d)); p and r carry logp's error and an exponent's
    big = dx.abs().amax(1, keepdim=True)
    check("dlogits", dl, dx, STEP16 * dx.abs() + 64 * (tol.max() + EPS32 * 64) * (big + dx.abs()) + 2.0 ** -126)
    assert not dl[~want["live"].cuda()].view(torch.int16).any()  # +0 in rows that do not count
    # without entropy and reference, and again: the same bits
    q = sp.PolicyParams(0.2, 0.3, adv_per_token=per_token)
    a = sp.sp_policy_loss(q, x["x"], x["labels"], x["old"], None, x["adv"], cu, with_entropy=False)
    plain = reference(d, 0.0, 0.0, use_ref=False)
    assert a[2] is None and not a[4][:, :2].any()
    check("seq_sum without", a[3], plain["sums"], (2 * tol.max() + EPS32 * 4) * size[:, 0])
    b = sp.sp_policy_loss(q, x["x"], x["labels"], x["old"], None, x["adv"], cu, with_entropy=False)
    assert all(torch.equal(u, w) for u, w in zip(a[:2] + a[3:], b[:2] + b[3:]))


def test_policy_gradient_against_differences(sp):
    """(sum(x + h u) - sum(x - h u)) / 2h along one direction: h is a power of two
    that moves every logit by whole bf16 steps, so no input is rounded."""
    T, V, cu = 24, 64, [0, 10, 24]
    d = make(T, V, cu, seed=5, spread=1.0, ignored=0.0)
    d["x"] = torch.round(d["x"] * 16) / 16  # multiples of 1/16 below 8: steps of 1/32 at most
    d["x"].clamp_(-3.9, 3.9)
    d["x"] = (d["x"] * 16).round() / 16
    g = torch.Generator().manual_seed(1)
    u, h = torch.randint(-1, 2, (T, V), generator=g).double(), 1 / 64
    p = sp.PolicyParams(0.2, 0.3, 0.1, 0.05)
    d["old"] = torch.log_softmax(d["x"], 1).gather(1, d["labels"][:, None])[:, 0].float().double()  # ratios near 1

    def value(x):
        y = device(dict(d, x=x))
        out = sp.sp_policy_loss(p, y["x"], y["labels"], y["old"], y["ref"], y["adv"], cu)
        return out, y
    out, y = value(d["x"])
    dl = sp.sp_policy_loss_bwd(p, y["x"], y["labels"], *out[:3], y["old"], y["ref"], y["adv"], cu, y["grad"])
    up, dn = value(d["x"] + h * u)[0][3].double().cpu(), value(d["x"] - h * u)[0][3].double().cpu()
    slope = ((up - dn) / (2 * h) * d["grad"]).sum()
    along = (dl.double().cpu() * u).sum()
    # bf16 rounding of every entry; h^2 / 6 times a third derivative of at most
    # 8 |G| (|A| r + kl e^d + ent) a token, whose logits move by at most h; float32 sums
    third = 8 * d["grad"].abs().max() * (2 * d["adv"].abs().max() + 1) * T
    tol = STEP16 * (dl.double().cpu().abs() * u.abs()).sum() + h * h / 6 * third + 1e-5 * T / h * 2
    assert abs(slope - along) <= tol, (slope, along, tol)


def test_policy_masked_logits_and_edges(sp):
    """Banned tokens (-inf, the type's lowest value) have probability 0; rows of
    nothing else, infinite ratios beside A = 0, and NaN in rows that do not count."""
    T, V, cu = 8, 2048, [0, 3, 8]
    d = make(T, V, cu, seed=9, ignored=0.0)
    keep = torch.zeros(T, V, dtype=torch.bool)
    keep[torch.arange(T), d["labels"]] = True
    ban = (torch.rand(T, V, generator=torch.Generator().manual_seed(2)) < 0.7) & ~keep
    ban[:, :256] = ~keep[:, :256]  # whole vectors of them, at the row's start
    d["x"][ban] = -math.inf
    d["x"][1][ban[1]] = torch.finfo(torch.bfloat16).min
    lp = torch.log_softmax(d["x"], 1).gather(1, d["labels"][:, None])[:, 0]
    d["old"], d["ref"] = (lp - 0.1).float().double(), (lp + 0.2).float().double()
    finite = dict(d, x=torch.where(ban, torch.full_like(d["x"], -1e4), d["x"]))  # e^-1e4 = 0 in float64
    want, x = reference(finite), device(d)
    p = sp.PolicyParams(0.2, 0.3, 0.1, 0.01)
    out = sp.sp_policy_loss(p, x["x"], x["labels"], x["old"], x["ref"], x["adv"], cu)
    tol = lse_tol(d, want["lse"])
    check("logp", out[0], want["logp"], tol)
    check("entropy", out[2], want["ent"], 64 * tol)
    dl = sp.sp_policy_loss_bwd(p, x["x"], x["labels"], *out[:3], x["old"], x["ref"], x["adv"], cu, x["grad"])
    big = want["dx"].abs().amax(1, keepdim=True)
    check("dlogits", dl, want["dx"], STEP16 * want["dx"].abs() + 64 * (tol.max() + EPS32 * 64) * big + 2.0 ** -126)
    assert not dl[ban.cuda()].any()
    # row 0: nothing but -inf; row 1: ignored NaN; row 2: an infinite ratio, A = 0
    x["x"][0] = -math.inf
    x["x"][1] = math.nan
    x["labels"][1] = -100
    x["old"][2] = -1e9
    x["adv"][0] = 0.0
    q = sp.PolicyParams(0.2, 0.3)
    logp, lse, ent, sums, _ = sp.sp_policy_loss(q, x["x"], x["labels"], x["old"], None, x["adv"], cu)
    assert logp[0] == -math.inf and lse[0] == -math.inf and ent[0] == 0 and logp[1] == 0 and lse[1] == 0
    assert sums[0] == 0 and torch.isfinite(sums).all()
    dl = sp.sp_policy_loss_bwd(q, x["x"], x["labels"], logp, lse, None, x["old"], None, x["adv"], cu, x["grad"])
    assert not dl[:3].any() and torch.isfinite(dl).all() and dl[3:].any()


def test_policy_gradient_over_the_logits(sp):
    for T, V in ((33, 8200), (600, 520)):
        cu = [0, T // 2, T - 1]
        d = make(T, V, cu, seed=T)
        x, p = device(d), sp.PolicyParams(0.2, 0.3, 0.1, 0.01)
        out = sp.sp_policy_loss(p, x["x"], x["labels"], x["old"], x["ref"], x["adv"], cu)
        args = (x["labels"], *out[:3], x["old"], x["ref"], x["adv"], cu, x["grad"])
        apart = sp.sp_policy_loss_bwd(p, x["x"], *args)
        over = sp.sp_policy_loss_bwd(p, x["x"], *args, dlogits=x["x"])
        assert over is x["x"] and torch.equal(over.view(torch.int16), apart.view(torch.int16))


def test_policy_without_tokens_or_sequences(sp):
    p = sp.PolicyParams()
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    out = sp.sp_policy_loss(p, z(0, 64, t=torch.bfloat16), z(0, t=torch.int32), z(0), None, z(2), [0, 0, 0])
    assert out[3].tolist() == [0, 0] and not out[4].any()
    for T, V in ((3, 64), (1200, 64), (3, 20000)):  # no sequence holds a token
        x = torch.full((T, V), math.nan, dtype=torch.bfloat16, device="cuda")
        out = sp.sp_policy_loss(p, x, z(T, t=torch.int32), z(T), None, z(0), [], logp=z(T) + 7, lse=z(T) + 7)
        assert not out[0].any() and not out[1].any() and not out[2].any()
        dl = sp.sp_policy_loss_bwd(p, x, z(T, t=torch.int32), *out[:3], z(T), None, z(0), [], z(0))
        assert not dl.any()


def test_policy_in_a_graph_and_on_a_stream(sp):
    """A captured forward and backward, replayed over other inputs with eager calls
    in between, gives the eager results bit for bit; so does another stream."""
    T, V, cu = 700, 4104, [0, 300, 690]
    p = sp.PolicyParams(0.2, 0.3, 0.1, 0.01)
    sets = [device(make(T, V, cu, seed=s)) for s in (1, 2, 3)]

    def step(x, **kw):
        out = sp.sp_policy_loss(p, x["x"], x["labels"], x["old"], x["ref"], x["adv"], cu, **kw)
        return (*out, sp.sp_policy_loss_bwd(p, x["x"], x["labels"], *out[:3], x["old"], x["ref"], x["adv"], cu,
                                            x["grad"], **kw))
    eager = [step(x) for x in sets]
    held = {k: v.clone() for k, v in sets[0].items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(held)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(held)
    for i in (1, 2, 0, 1):
        for k in held:
            held[k].copy_(sets[i][k])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager[i]))
        step(sets[(i + 1) % 3])
    on_side = step(sets[1], stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(on_side, eager[1]))


def test_policy_sums_feed_the_loss_reduction(sp):
    """Two ranks' sums through sp_loss_reduce and back: the gradient of the mean
    over all tokens of both."""
    T, V, cu = 50, 1000, [0, 20, 50]
    ranks = [make(T, V, cu, seed=s) for s in (11, 12)]
    p = sp.PolicyParams(0.2, 0.3, 0.1)
    xs = [device(r) for r in ranks]
    outs = [sp.sp_policy_loss(p, x["x"], x["labels"], x["old"], x["ref"], x["adv"], cu) for x in xs]
    n = sum(int(o[4][:, 3].sum()) for o in outs)
    loss, grad = sp.sp_loss_reduce(torch.stack([o[3] for o in outs]), sp.SP_LOSS_SFT, -1.0 / n)
    want = [reference(dict(r, grad=torch.full((2,), 2.0 / n).double()), 0.1, 0.0) for r in ranks]
    total = sum(w["sums"].sum() for w in want) / n
    tol = max(lse_tol(r, w["lse"]).max() for r, w in zip(ranks, want))
    assert abs(loss.item() - total) <= 8 * (tol + EPS32 * 16) * sum(w["size"].sum() for w in want) / n
    for i, (x, o, w) in enumerate(zip(xs, outs, want)):
        dl = sp.sp_policy_loss_bwd(p, x["x"], x["labels"], *o[:3], x["old"], x["ref"], x["adv"], cu, grad[i].contiguous())
        big = w["dx"].abs().amax(1, keepdim=True)
        check("dlogits", dl, w["dx"], STEP16 * w["dx"].abs() + 64 * (tol + EPS32 * 64) * big + 2.0 ** -126)


def test_policy_labels_that_do_not_count(sp):
    """Labels outside [0, V), an ignored label inside it, tokens outside the
    sequences: zero, and their logits are not looked at."""
    T, V, cu = 12, 64, [1, 6, 11]
    d = make(T, V, cu, seed=21, ignored=0.0)
    d["labels"][2], d["labels"][3], d["labels"][7], d["labels"][8] = V, -1, 2 ** 31 - 1, -2 ** 31
    d["labels"][4] = d["labels"][9] = 5  # the ignored one here
    x = device(d)
    out = [0, 2, 3, 4, 7, 8, 9, 11]
    x["x"][out] = math.nan
    p = sp.PolicyParams(0.2, 0.3, 0.1, 0.01, ignore_index=5)
    logp, lse, ent, sums, stats = sp.sp_policy_loss(p, x["x"], x["labels"], x["old"], x["ref"], x["adv"], cu)
    dl = sp.sp_policy_loss_bwd(p, x["x"], x["labels"], logp, lse, ent, x["old"], x["ref"], x["adv"], cu, x["grad"])
    keep = [i for i in range(T) if i not in out]
    for t in (logp, lse, ent, dl):
        assert not t[out].any() and torch.isfinite(t).all() and t[keep].any()
    d["labels"][out] = -100
    d["x"][out] = 0.0
    want = reference(d, 0.1, 0.01)
    assert stats[:, 3].tolist() == [2.0, 2.0]
    tol = lse_tol(d, want["lse"])
    check("seq_sum", sums, want["sums"], 4 * tol.max() * want["size"])


def test_policy_offsets_past_32_bits(sp):
    """The last rows of 15000 x 152064 logits (2.3e9 of them): the same bits as in a
    call of their own."""
    T, V, n = 15000, 152064, 40
    x = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    x[-n:] = torch.randn(n, V, generator=g, device="cuda").bfloat16()
    lab = torch.full((T,), -100, dtype=torch.int32, device="cuda")
    lab[-n:] = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    f = [torch.randn(T, generator=g, device="cuda") - 12 for _ in range(2)]
    adv, up = torch.ones(1, device="cuda"), torch.ones(1, device="cuda")
    p = sp.PolicyParams(0.2, 0.3, 0.1, 0.01)
    tail = slice(T - n, T)
    # (a row of the small call is summed in more parts: its logp differs by roundings)
    out = sp.sp_policy_loss(p, x, lab, *f, adv, [0, T])
    few = sp.sp_policy_loss(p, x[tail], lab[tail], f[0][tail], f[1][tail], adv, [0, n])
    assert (out[0][tail] - few[0]).abs().max() <= 64 * EPS32 * 16 and not out[0][:-n].any()
    own = [t[tail].contiguous() for t in out[:3]]
    want = sp.sp_policy_loss_bwd(p, x[tail], lab[tail], *own, f[0][tail], f[1][tail], adv, [0, n], up)
    dl = sp.sp_policy_loss_bwd(p, x, lab, *out[:3], *f, adv, [0, T], up, dlogits=x)
    assert torch.equal(dl[tail], want) and want.any()
    assert not dl[:-n].any()


def test_policy_kl_of_banned_labels(sp):
    """A label of probability 0, and rows without a distribution, beside a reference
    model: finite wherever both models ban the token, and infinite where one does."""
    T, V, cu = 6, 1000, [0, 3, 4, 6]
    d = make(T, V, cu, seed=21, ignored=0.0)
    d["x"][0] = -math.inf                    # no distribution, a finite reference
    for t in (1, 3):
        d["x"][t, d["labels"][t]] = -math.inf  # the label alone
    d["x"][2] = -math.inf
    d["ref"][1:3] = d["old"][2] = -math.inf    # banned in all models
    d["adv"][:] = 1.0
    x = device(d)
    p = sp.PolicyParams(0.2, 0.3, 0.5)
    logp, lse, _, sums, stats = sp.sp_policy_loss(p, x["x"], x["labels"], x["old"], x["ref"], x["adv"], cu,
                                                  with_entropy=False)
    assert (logp[:4] == -math.inf).all() and torch.isfinite(lse[[1, 3]]).all()
    # ratios 0, 0 and 1 (nothing differs), no divergence: -(0 + 0 + 1)
    assert sums[0] == -1.0 and stats[0].tolist() == [0.0, 0.0, 0.0, 3.0]
    assert sums[1] == math.inf and stats[1][0] == math.inf
    want = reference({k: v[4:] if k in ("x", "labels", "old", "ref") else v for k, v in
                      dict(d, adv=d["adv"][2:], grad=d["grad"][2:], cu=[0, 2]).items()}, kl=0.5, ent_coef=0.0)
    tol = lse_tol(d, want["lse"]).max() * (2 * want["size"] + 2)
    check("sums", sums[2:], want["sums"], tol)
    dl = sp.sp_policy_loss_bwd(p, x["x"], x["labels"], logp, lse, None, x["old"], x["ref"], x["adv"], cu, x["grad"])
    assert not dl[:3].any() and torch.isfinite(dl[4:]).all() and dl[4:].any()
