"""Norm, rotation and pack of query and key heads, and the backward, on the GPU
against float64 (pairs as complex numbers)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

STEP16, EPS32 = 2.0 ** -8, 2.0 ** -24  # half a step of bf16 / float32, relative


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available()
    import paper_2505_22296_amd as m
    m.load()
    return m


def freqs(rot, theta=1e6):
    return theta ** (-2.0 * np.arange(rot // 2) / rot)


def turned(y, angle, rot, neigh, scale, back=False):
    """Rotation of the first rot dims of y [T, H, D] float64 by angle [T, rot/2]."""
    if rot == 0:
        return y
    z = y[..., :rot].unflatten(-1, (rot // 2, 2)) if neigh else y[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    u = torch.polar(torch.full_like(angle, scale), -angle if back else angle)[:, None]
    z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * u)
    return torch.cat([(z if neigh else z.transpose(-1, -2)).flatten(-2), y[..., rot:]], -1)


def slots(m, n):
    return [(i // (len(m) // n), i % (len(m) // n), h) for i, h in enumerate(m)]


def packed(y, m, n):
    out = torch.zeros(n, y.shape[0], len(m) // n, y.shape[2], dtype=torch.float64)
    for j, h, g in slots(m, n):
        if g >= 0:
            out[j, :, h] = y[:, g]
    return out


def gathered(d, m, n, H):
    out = torch.zeros(d.shape[1], H, d.shape[3], dtype=torch.float64)
    for j, h, g in slots(m, n):
        if g >= 0:
            out[:, g] += d[j, :, h].double()
    return out


MHA7 = ([0, 1, 2, 3, 4, 5, 6, -1],) * 2
GQA = (list(range(28)) + [-1] * 4, [0, -1, 0, 1, 1, -1, 1, 2, 2, -1, 2, 3, 3, -1, 3, -1])
CASES = [  # T, D, Hq, Hkv, sp, maps, rot, neighbours, norm, positions
    (1, 64, 7, 7, 2, MHA7, 64, False, True, "ramp"),
    (3, 128, 1, 1, 1, ([0], [0]), 128, False, True, "far"),
    (129, 128, 28, 4, 8, GQA, 128, False, True, "far"),
    (67, 128, 28, 4, 8, GQA, 64, False, False, "ramp"),
    (50, 64, 7, 7, 2, MHA7, 32, True, True, "any"),
    (33, 128, 28, 4, 8, GQA, 112, True, True, "any"),
    (40, 64, 7, 7, 2, MHA7, 0, False, True, "ramp"),
    (5000, 64, 2, 1, 1, ([0, 1], [0]), 64, False, True, "ramp"),  # more tokens than the backward has wavefronts
    (17, 128, 3, 2, 1, ([2, 0, 2], [-1, 1]), 16, False, True, "none"),  # heads twice, and in no slot
    (9, 64, 100, 70, 4, (list(range(100)) + [-1] * 4, list(range(70)) + [3, -1]), 64, False, True, "ramp"),  # large maps
    (20, 64, 2, 2, 2, ([-1, 0, -1, 1], [1, -1, -1, -1]), 48, True, True, "ramp"),  # slots without heads first
]


def make(case, seed):
    T, D, Hq, Hkv, n, maps, rot, neigh, norm, pos = case
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g).bfloat16()  # noqa: E731
    x = dict(qkv=r(T, Hq + 2 * Hkv + 1, D), wq=1 + 0.3 * r(D), wk=1 + 0.3 * r(D),
             dq=r(n, T, len(maps[0]) // n, D), dk=r(n, T, len(maps[1]) // n, D), dv=r(n, T, len(maps[1]) // n, D))
    p = {"ramp": torch.arange(T), "far": 2 ** 31 - 1 - 7919 * torch.arange(T), "none": 1000 + torch.arange(T),
         "any": torch.randint(-2 ** 31, 2 ** 31, (T,), generator=g)}[pos]
    return x, p


def desc(sp, case, **over):
    T, D, Hq, Hkv, n, maps, rot, neigh, norm, pos = case
    kw = dict(T=T, head_dim=D, H_q=Hq, H_kv=Hkv, sp=n, q_map=maps[0], kv_map=maps[1], rotary_dim=rot,
              inv_freq=freqs(rot) if rot else None, interleaved=neigh, rope_scale=1.25, eps=1e-5, weight_offset=0.5,
              position_base=1000)
    kw.update(over)
    return sp.QkDesc(**kw)


def parts(qkv, Hq, Hkv):
    return qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:Hq + 2 * Hkv]


def reference(case, x, pos, scale=1.25, eps=1e-5, off=0.5):
    T, D, Hq, Hkv, n, maps, rot, neigh, norm, _ = case
    angle = torch.outer(pos.double(), torch.from_numpy(freqs(rot))) if rot else None
    out = {}
    q, k, v = (t.double() for t in parts(x["qkv"], Hq, Hkv))
    for name, y, w, m, d in (("q", q, x["wq"], maps[0], x["dq"]), ("k", k, x["wk"], maps[1], x["dk"])):
        y, w = y.clone().requires_grad_(), (w.double() + off).requires_grad_()
        z = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * w if norm else y * 1.0
        z = turned(z, angle, rot, neigh, scale)
        G = gathered(d, m, n, y.shape[1])
        (z * G).sum().backward()
        out.update({name: packed(z.detach(), m, n), "d" + name: y.grad, "dw" + name: w.grad, "g" + name: G,
                    "r" + name: 1 / (y.detach().square().mean(-1, keepdim=True) + eps).sqrt() * w.detach().abs().max()
                    if norm else torch.ones(T, y.shape[1], 1).double()})
    out.update(v=packed(v, maps[1], n), dv=gathered(x["dv"], maps[1], n, Hkv))
    return out


def check(name, got, want, tol):
    off = (got.double().cpu() - want).abs() - tol
    assert torch.isfinite(got).all() and (off <= 0).all(), f"{name}: {off.max().item():.3e} past its tolerance"


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"T{c[0]}_D{c[1]}_q{c[2]}kv{c[3]}_sp{c[4]}_rot{c[6]}_{c[9]}")
def test_qk_norm_rope_and_backward(sp, case):
    T, D, Hq, Hkv, n, maps, rot, neigh, norm, posk = case
    x, pos = make(case, seed=T + D)
    want, d = reference(case, x, pos), desc(sp, case)
    g = {k: v.cuda() for k, v in x.items()}
    q, k, v = parts(g["qkv"], Hq, Hkv)  # heads of one projection: their tokens lie further apart
    w = (g["wq"], g["wk"]) if norm else (None, None)
    p = None if posk == "none" else pos.to(torch.int32).cuda()
    oq, ok, ov = sp.sp_qk_norm_rope(d, q, k, v, p, *w)
    # float32: some 20 roundings of a norm, a frequency's 2^-32 turns and a sine of
    # 4 units in the last place, of the pair's size; then one rounding to bf16
    for name, got in (("q", oq), ("k", ok)):
        size = want[name].norm(dim=-1, keepdim=True)
        check(name, got, want[name], STEP16 * want[name].abs() + 32 * EPS32 * size)
    assert torch.equal(ov.cpu().double(), want["v"])
    zero = [(j, h) for j, h, s in slots(maps[0], n) if s < 0]
    assert not any(oq[j, :, h].view(torch.int16).any() for j, h in zero)

    dq, dk, dv, dwq, dwk = sp.sp_qk_norm_rope_bwd(d, q, k, g["dq"], g["dk"], g["dv"], p, *w)
    check("dv", dv, want["dv"], STEP16 * want["dv"].abs() + 8 * EPS32 * 10)
    for name, got in (("q", dq), ("k", dk)):
        # a sum over D of products of the row: D / 16 + 8 additions and some 24 roundings
        size = 1.25 * want["g" + name].norm(dim=-1, keepdim=True) * want["r" + name]
        check("d" + name, got, want["d" + name], STEP16 * want["d" + name].abs() + 64 * EPS32 * size)
    if not norm:
        assert dwq is None and dwk is None
        return
    for name, got, H in (("q", dwq, Hq), ("k", dwk, Hkv)):
        # T H terms of at most |g| |n|, in partial sums of at most T H / 2^10 + 200
        # additions; each term off by some 40 roundings of the row's size
        gr = want["g" + name].norm(dim=-1).max() * 1.25
        xr = want["r" + name].max() * x["qkv"].double().abs().max()
        check("dw" + name, got, want["dw" + name],
              EPS32 * (40 + T * H / 1024 + 200) * gr * xr * (T * H) ** 0.5 * 4)
    again = sp.sp_qk_norm_rope_bwd(d, q, k, g["dq"], g["dk"], g["dv"], p, *w)
    assert all(torch.equal(a, b) for a, b in zip(again, (dq, dk, dv, dwq, dwk)))


def test_qk_backward_against_differences(sp):
    """Central differences of sum(G * dst) along a direction of q; h moves x by
    whole bf16 steps and dst is taken in bf16, whose rounding bounds the check."""
    case = (6, 64, 2, 2, 1, ([0, 1], [0, 1]), 64, False, True, "ramp")
    x, pos = make(case, 3)
    x["qkv"] = (x["qkv"].double().clamp(-3.5, 3.5) * 4).round().div(4).bfloat16()
    d, g = desc(sp, case), {k: v.cuda() for k, v in x.items()}
    u = torch.randint(-1, 2, (6, 2, 64), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    h = 0.0625

    def value(s):
        q, k, v = parts(g["qkv"], 2, 2)
        out = sp.sp_qk_norm_rope(d, q + s * u, k, v, None, g["wq"], g["wk"])[0]
        return (out.double() * g["dq"].double()).sum().item(), (out.double().abs() * g["dq"].double().abs()).sum().item()
    q, k, v = parts(g["qkv"], 2, 2)
    dq = sp.sp_qk_norm_rope_bwd(d, q, k, g["dq"], g["dk"], g["dv"], None, g["wq"], g["wk"])[0]
    (up, size), (dn, _) = value(h), value(-h)
    along = (dq.double() * u.double()).sum().item()
    # independent roundings of dst (12 rows of 64) add up as a random walk, 6 of
    # its deviations allowed; the third derivative along u of a row of norm 8 moved by
    # 8 h is below |G| (8 / 8)^3
    n = 6 * 2 * 64
    tol = 6 * STEP16 * size / n ** 0.5 / h + h * h / 6 * 1.25 * 1.5 * g["dq"].double().norm(dim=-1).sum().item() \
        + STEP16 * (dq.double() * u.double()).abs().sum().item()
    assert abs((up - dn) / (2 * h) - along) <= tol, ((up - dn) / (2 * h), along, tol)


def test_qk_equals_pack_without_norm_and_rotation(sp):
    """With nothing to do to the heads, the pass is the pack, and its backward the
    summing unpack, bit for bit."""
    case = (100, 128, 28, 4, 8, GQA, 0, False, False, "ramp")
    x, _ = make(case, 8)
    d, g = desc(sp, case, rotary_dim=0), {k: v.cuda() for k, v in x.items()}
    q, k, v = (t.contiguous() for t in parts(g["qkv"], 28, 4))
    oq, ok, ov = sp.sp_qk_norm_rope(d, q, k, v)
    assert torch.equal(oq, sp.sp_ulysses_pack(q, 8, 4, GQA[0]))
    assert torch.equal(ok, sp.sp_ulysses_pack(k, 8, 2, GQA[1])) and torch.equal(ov, sp.sp_ulysses_pack(v, 8, 2, GQA[1]))
    dq, dk, dv, _, _ = sp.sp_qk_norm_rope_bwd(d, None, None, g["dq"], g["dk"], g["dv"])
    assert torch.equal(dq, sp.sp_ulysses_unpack(g["dq"], GQA[0], 28))
    assert torch.equal(dk, sp.sp_ulysses_unpack_add(g["dk"], GQA[1], 4))
    assert torch.equal(dv, sp.sp_ulysses_unpack_add(g["dv"], GQA[1], 4))


def test_qk_outputs_inside_a_projection_and_over_q_and_k(sp):
    """Gradients written into one [T, heads, D] buffer, and dq, dk over q, k; what
    lies behind the heads stays as it was."""
    case = (77, 128, 28, 4, 8, GQA, 128, False, True, "ramp")
    x, pos = make(case, 9)
    d, g = desc(sp, case), {k: v.cuda() for k, v in x.items()}
    p = pos.to(torch.int32).cuda()
    q, k, v = parts(g["qkv"], 28, 4)
    args = (g["dq"], g["dk"], g["dv"], p, g["wq"], g["wk"])
    want = sp.sp_qk_norm_rope_bwd(d, q, k, *args)
    buf = torch.full_like(g["qkv"], 7.0)
    bq, bk, bv = parts(buf, 28, 4)
    sp.sp_qk_norm_rope_bwd(d, q, k, *args, dq=bq, dk=bk, dv=bv)
    assert torch.equal(bq, want[0]) and torch.equal(bk, want[1]) and torch.equal(bv, want[2])
    assert (buf[:, -1] == 7).all()
    sp.sp_qk_norm_rope_bwd(d, q, k, *args, dq=q, dk=k, dv=v)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, want[2])
    assert torch.equal(g["qkv"][:, -1].cpu(), x["qkv"][:, -1])


def test_qk_edges(sp):
    """No tokens; rows of zeros without eps's help; values whose squares are large;
    wrong tensors."""
    case = (4, 64, 2, 1, 1, ([0, 1], [0]), 64, False, True, "ramp")
    x, pos = make(case, 1)
    g = {k: v.cuda() for k, v in x.items()}
    z = desc(sp, case, T=0)
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    out = sp.sp_qk_norm_rope(z, e(0, 2, 64), e(0, 1, 64), e(0, 1, 64), None, g["wq"], g["wk"])
    assert out[0].shape == (1, 0, 2, 64)
    dw = torch.full((64,), 5.0, device="cuda")
    sp.sp_qk_norm_rope_bwd(z, e(0, 2, 64), e(0, 1, 64), e(1, 0, 2, 64), e(1, 0, 1, 64), e(1, 0, 1, 64), None, g["wq"],
                           g["wk"], dw_q=dw)
    assert not dw.any()
    q, k, v = parts(g["qkv"], 2, 1)
    g["qkv"][0] = 0
    g["qkv"][1] *= 1e15
    x["qkv"] = g["qkv"].cpu()
    want = reference(case, x, pos)
    d, p = desc(sp, case), pos.to(torch.int32).cuda()
    oq = sp.sp_qk_norm_rope(d, q, k, v, p, g["wq"], g["wk"])[0]
    check("q", oq, want["q"], STEP16 * want["q"].abs() + 32 * EPS32 * want["q"].norm(dim=-1, keepdim=True))
    dq = sp.sp_qk_norm_rope_bwd(d, q, k, g["dq"], g["dk"], g["dv"], p, g["wq"], g["wk"])[0]
    size = 1.25 * want["gq"].norm(dim=-1, keepdim=True) * want["rq"]
    check("dq", dq, want["dq"], STEP16 * want["dq"].abs() + 64 * EPS32 * size)
    with pytest.raises(ValueError, match="shape"):
        sp.sp_qk_norm_rope(d, q[:3], k, v, p)
    with pytest.raises(ValueError, match="torch.int32"):
        sp.sp_qk_norm_rope(d, q, k, v, p.long())
    with pytest.raises(ValueError, match="contiguous within a token"):
        sp.sp_qk_norm_rope(d, g["qkv"].transpose(0, 1)[:4, :2], k, v, p) if g["qkv"].shape[1] >= 4 else sp.sp_qk_norm_rope(
            d, q.transpose(1, 2).contiguous().transpose(1, 2), k, v, p)
    with pytest.raises(ValueError, match="without its weight"):
        sp.sp_qk_norm_rope_bwd(d, q, k, g["dq"], g["dk"], g["dv"], p, dw_q=dw)


def test_qk_in_a_graph(sp):
    case = (130, 128, 28, 4, 8, GQA, 128, False, True, "ramp")
    d = desc(sp, case)
    sets = [{k: v.cuda() for k, v in make(case, s)[0].items()} for s in (1, 2, 3)]

    def step(g, **kw):
        q, k, v = parts(g["qkv"], 28, 4)
        out = sp.sp_qk_norm_rope(d, q, k, v, None, g["wq"], g["wk"], **kw)
        return (*out, *sp.sp_qk_norm_rope_bwd(d, q, k, g["dq"], g["dk"], g["dv"], None, g["wq"], g["wk"], **kw))
    eager = [step(g) for g in sets]
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


def test_qk_offsets_past_32_bits(sp):
    """Tokens 8192 elements apart whose last one lies past 2^31 elements."""
    T, D, n = 263000, 64, 50
    buf = torch.empty(T, 8192, dtype=torch.bfloat16, device="cuda")
    rows = torch.randn(T, 3, D, device="cuda").bfloat16()
    buf[:, :192] = rows.view(T, 192)
    q, k, v = (buf[:, i * D:(i + 1) * D].view(T, 1, D) for i in range(3))
    w = torch.randn(2, D, device="cuda").bfloat16()
    kw = dict(head_dim=D, H_q=1, H_kv=1, sp=1, q_map=[0], kv_map=[0], inv_freq=freqs(D))
    far = sp.sp_qk_norm_rope(sp.QkDesc(T=T, **kw), q, k, v, None, w[0], w[1])
    near = sp.sp_qk_norm_rope(sp.QkDesc(T=n, position_base=T - n, **kw),
                              *(rows[T - n:, i:i + 1].contiguous() for i in range(3)), None, w[0], w[1])
    assert all(torch.equal(a[:, T - n:], b) for a, b in zip(far, near))
    up = [torch.randn(1, T, 1, D, device="cuda").bfloat16() for _ in range(3)]
    want = sp.sp_qk_norm_rope_bwd(sp.QkDesc(T=n, position_base=T - n, **kw), rows[T - n:, :1].contiguous(),
                                  rows[T - n:, 1:2].contiguous(), *(u[:, T - n:].contiguous() for u in up), None, w[0], w[1])
    got = sp.sp_qk_norm_rope_bwd(sp.QkDesc(T=T, **kw), q, k, *up, None, w[0], w[1], dq=q, dk=k, dv=v)
    assert all(torch.equal(a[T - n:], b) for a, b in zip(got[:3], want[:3]))
    assert not torch.isnan(got[3]).any()
