"""Attention of segments that share a prefix (SP_DESC_SHARED_PREFIX) on the GPU:
against float64 from the definition's mask, against the unpacked sequences, over
every launch shape, and inside a step of a group of answers."""
import math

import numpy as np
import pytest
import torch

from tests.test_prefix_host import desc, mask_of

pytestmark = pytest.mark.gpu

STEP16, EPS32 = 2.0 ** -8, 2.0 ** -24  # half a step of bf16 / float32, relative


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available()
    import paper_2505_22296_amd as m
    m.load()
    return m


def inputs(d, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    c = d.c
    r = lambda T, H: (scale * torch.randn(T, H, c.head_dim, generator=g)).bfloat16().cuda()  # noqa: E731
    return r(c.T_q, c.H_loc), r(c.T_k, c.Hkv_loc), r(c.T_k, c.Hkv_loc), r(c.T_q, c.H_loc)


def visible(p):
    """The definition's mask [T_q, T_k], built segment by segment."""
    m = torch.zeros(p["T_q"], p["T_k"], dtype=torch.bool)
    pos_q, pos_k = torch.from_numpy(p["pos_q"]), torch.from_numpy(p["pos_k"])
    for s, f in enumerate(p["prefix_of"]):
        q, k = slice(p["cu_q"][s], p["cu_q"][s + 1]), slice(p["cu_k"][s], p["cu_k"][s + 1])
        m[q, k] = (pos_k[None, k] <= pos_q[q, None]) if p["causal"] else True
        if f >= 0:
            m[q, p["cu_k"][f]:p["cu_k"][f + 1]] = True
    return m.cuda()


def check(name, got, want, tol):
    got = got.double()
    same = (got == want)  # (-inf rows)
    off = torch.where(same, torch.zeros_like(want), (got - want).abs() - tol)
    assert (off <= 0).all(), f"{name}: {off.max().item():.3e} past its tolerance"


def compare(sp, d, p, seed=0, scale=1.0, static=False, real=None):
    """Forward and backward against float64, head by head, with the bounds that the
    roundings of bf16 operands give."""
    q, k, v, do = inputs(d, seed, scale)
    c = d.c
    real = min(c.H_loc, c.num_real_heads - c.head_offset)
    o, lse = sp.sp_attn_fwd(d, q, k, v)
    dq, dk, dv = sp.sp_attn_bwd(d, q, k, v, o, lse, do)
    m, D, sc = visible(p), c.head_dim, c.softmax_scale
    wk, wv = (torch.zeros(c.T_k, c.Hkv_loc, D, dtype=torch.float64, device="cuda") for _ in range(2))
    tk, tv = torch.zeros_like(wk), torch.zeros_like(wk)
    for h in range(real):
        kv = (c.head_offset + h) // c.gqa_group - c.kv_head_offset
        Q, K, V, G = (t.double() for t in (q[:, h], k[:, kv], v[:, kv], do[:, h]))
        z = torch.where(m, Q @ K.T * sc, -math.inf)
        L = torch.logsumexp(z, 1)
        w = torch.where(m, torch.exp(z - torch.where(L > -math.inf, L, torch.zeros_like(L))[:, None]), 0.0)
        # a score off by D float32 roundings of |q| |k|, its exponent by half a step of
        # at most 2^7; P rounded to bf16 beside an unrounded sum
        es = EPS32 * (D * sc * Q.norm(dim=1).max() * K.norm(dim=1).max() + 128 + 64) if c.T_k else 0.0
        check("lse", lse[h], L, 4 * es + EPS32 * c.T_k / 32 + 4 * EPS32 * L.abs())
        check("o", o[:, h], w @ V, STEP16 * (w @ V).abs() + (STEP16 + 4 * es) * (w @ V.abs()) + 1e-30)
        # the backward's own inputs are o and lse as they were written
        w = torch.where(m, torch.exp(z - torch.where(L > -math.inf, lse[h].double(), torch.zeros_like(L))[:, None]), 0.0)
        dp = G @ V.T
        dd = (G * o[:, h].double()).sum(1, keepdim=True)
        dz = w * (dp - dd)
        # dS is rounded to bf16 (in dK from P in fp16: 2^-11, and 2^-25 where it is
        # smallest); dP - D off by D roundings of |dO| |V|
        ed = 4 * EPS32 * D * (G.norm(dim=1).max() * V.norm(dim=1).max() if c.T_k else 0.0)
        size = dz.abs() * (STEP16 + 8 * es) + w * ed
        want = sc * (dz @ K)
        check("dq", dq[:, h], want, STEP16 * want.abs() + sc * (size @ K.abs()) + 1e-30)
        size = size + dz.abs() * 2.0 ** -11 + torch.where(m, 2.0 ** -25 * (dp - dd).abs(), 0.0)
        wk[:, kv] += sc * (dz.T @ Q)
        tk[:, kv] += sc * (size.T @ Q.abs())
        wv[:, kv] += w.T @ G
        tv[:, kv] += (STEP16 + 8 * es) * (w.T @ G.abs())
    check("dk", dk, wk, STEP16 * wk.abs() + tk + 1e-30)
    check("dv", dv, wv, STEP16 * wv.abs() + tv + 1e-30)
    for t in (o[:, real:], dq[:, real:]):
        assert not t.contiguous().view(torch.int16).any()
    assert (lse[real:] == -math.inf).all()
    if static:
        o2, l2 = torch.empty_like(o), torch.empty_like(lse)
        sp.sp_attn_fwd_static(d, q, k, v, o2, l2)
        assert torch.equal(o2, o) and torch.equal(l2, lse)
    again = (*sp.sp_attn_fwd(d, q, k, v), *sp.sp_attn_bwd(d, q, k, v, o, lse, do))
    assert all(torch.equal(a, b) for a, b in zip(again, (o, lse, dq, dk, dv)))
    return o, lse, dq, dk, dv


SMALL = [  # rows, keys (None: the same), prefixes
    ([5, 3], None, [-1, 0]), ([1, 1], None, [-1, 0]), ([70, 1, 1, 2], None, [-1, 0, 0, 0]),
    ([33, 40, 0, 31], None, [-1, 0, 0, 0]), ([0, 40, 31], None, [-1, 0, 0]),
    ([300, 17, 200, 90, 5, 260, 64], None, [-1, 0, 0, -1, 3, 3, 3]), ([50, 20, 30], None, [-1, 0, -1]),
    ([0, 1, 1, 1], [129, 40, 1, 200], [-1, 0, 0, 0]),      # one row an answer, the prompt's keys alone
    ([0, 3, 2, 9], [500, 64, 2, 9], [-1, 0, 0, 0]), ([4, 3], [100, 0], [-1, 0]),  # and an answer without keys
    ([0, 5, 2], [0, 5, 2], [-1, 0, 0]),                    # an empty prompt
]


@pytest.mark.parametrize("D,hq,hkv,dummies", [(128, 4, 1, 0), (64, 3, 3, 1), (64, 4, 2, 0), (128, 2, 2, 0)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nk,pre", SMALL)
def test_prefix_matches_definition(sp, nq, nk, pre, causal, D, hq, hkv, dummies):
    d, p = desc(nq, nq if nk is None else nk, pre, D=D, hq=hq, hkv=hkv, dummies=dummies, causal=causal,
                pad_q=2 if D == 64 else 0, pad_k=3 if D == 64 else 0)
    assert np.array_equal(visible(p).cpu().numpy(), mask_of(**p))
    compare(sp, d, p, seed=sum(nq), static=True)


LARGE = [  # rows, prefixes, hq, hkv, D; what the plan of forward and backward then is
    ([700, 300, 180, 90, 40, 400], [-1, 0, 0, 0, 0, 0], 4, 1, 128),
    ([1500, 600, 513, 700, 60], [-1, 0, 0, 0, 0], 14, 2, 128),
    ([2100] + [300] * 8, [-1] + [0] * 8, 28, 4, 128),
    ([900, 200, 300, 800, 100, 300], [-1, 0, 0, -1, 3, 3], 28, 4, 64),
    ([1000] + [130] * 20, [-1] + [0] * 20, 40, 8, 64),
    ([300, 200] * 40, [-1, -1] * 2 + [-1, 4] + [-1, 6] + [-1, 8] + [-1, -1] * 35, 8, 8, 64),
    ([260] + [1] * 300, [-1] + [0] * 300, 4, 1, 128),
    ([2500, 1300, 900], [-1, 0, 0], 16, 16, 64), ([2500, 900, 700], [-1, 0, 0], 7, 1, 128),
    ([2500, 900, 700], [-1, 0, 0], 8, 8, 64),
]


@pytest.mark.parametrize("nq,pre,hq,hkv,D", LARGE, ids=lambda x: str(len(x)) if isinstance(x, list) else str(x))
def test_prefix_larger_batches(sp, nq, pre, hq, hkv, D):
    d, p = desc(nq, nq, pre, D=D, hq=hq, hkv=hkv)
    compare(sp, d, p, seed=len(nq))


def test_large_batches_reach_every_launch_shape(sp):
    """What the cases above are for: split and unsplit row items, one and two
    workgroups a CU, one launch and two, lists in the arguments and in memory."""
    seen = {k: set() for k in ("fwd", "bwd", "list")}
    for nq, pre, hq, hkv, D in LARGE:
        d, _ = desc(nq, nq, pre, D=D, hq=hq, hkv=hkv)
        f, b = sp.sp_attn_plan(d, sp.SP_OP_FWD), sp.sp_attn_plan(d, sp.SP_OP_BWD)
        seen["fwd"].add((D, f["row_split"], f["row_two"]))
        seen["bwd"].add((D, b["row_split"], b["row_two"], b["one_launch"]))
        seen["list"].add(sp.sp_attn_workspace_size(d, sp.SP_OP_FWD) > 32 * 700)
    assert {s[1] for s in seen["fwd"]} == {1, 2, 4} and any(s[2] for s in seen["fwd"])
    assert {s[3] for s in seen["bwd"]} == {0, 1} and {s[1] for s in seen["bwd"]} == {1, 2, 4}
    assert seen["list"] == {True, False}


FEW = [  # rows, keys, prefixes, hq, hkv, dummies, D, causal: a long prompt's keys and few rows
    ([0] + [1] * 16, [20000] + [100 + 7 * i for i in range(16)], [-1] + [0] * 16, 7, 1, 0, 128, True),
    ([0] + [1] * 16, [20000] + [100 + 7 * i for i in range(16)], [-1] + [0] * 16, 7, 1, 0, 128, False),
    ([0, 1, 5, 40], [12001, 9, 300, 40], [-1, 0, 0, 0], 4, 2, 0, 64, True),
    ([0, 1, 1, 0, 1, 1, 2], [9000, 300, 0, 7001, 1, 33, 2], [-1, 0, 0, -1, 3, 3, 3], 3, 3, 1, 64, True),
    ([0, 1, 3], [16000, 50, 3], [-1, 0, 0], 40, 1, 0, 128, True),   # more query heads than a slot has lanes
    ([30, 20, 7], [12000, 20, 90], [-1, 0, 0], 28, 4, 0, 128, True),  # the prompt's last rows too
    ([0] + [1] * 100, [8192] + [1] * 100, [-1] + [0] * 100, 4, 1, 0, 128, True),
    ([2, 0, 1], [30000, 8000, 1], [-1, -1, 1], 4, 1, 0, 128, True),  # rows without a prefix beside them
]


@pytest.mark.parametrize("nq,nk,pre,hq,hkv,dummies,D,causal", FEW)
def test_prefix_of_few_rows(sp, nq, nk, pre, hq, hkv, dummies, D, causal):
    """Keys cut into parts over workgroups, and the parts merged."""
    d, p = desc(nq, nk, pre, D=D, hq=hq, hkv=hkv, dummies=dummies, causal=causal, pad_q=3 if D == 64 else 0)
    assert sp.sp_attn_plan(d, sp.SP_OP_FWD)["key_split"] > 1
    o, lse, *_ = compare(sp, d, p, seed=len(nq))
    # the same in whole walks (the allocation-free forward never cuts the keys): both
    # are within P's rounding of each other
    q, k, v, _ = inputs(d, len(nq))
    o2, l2 = torch.empty_like(o), torch.empty_like(lse)
    sp.sp_attn_fwd_static(d, q, k, v, o2, l2)
    assert (o.float() - o2.float()).abs().max() <= 4 * STEP16 * v.float().abs().max()
    fin = lse > -math.inf
    assert torch.equal(fin, l2 > -math.inf) and (lse - l2)[fin].abs().max() <= 1e-4


def test_prefix_large_scores(sp):
    """Scores of a few hundred: the running maximum is raised between the prefix's
    keys and the answer's, in either order."""
    d, p = desc([200, 100, 130], [200, 100, 130], [-1, 0, 0], D=64, hq=2, hkv=2)
    compare(sp, d, p, seed=3, scale=4.0)


def test_prefix_equals_unpacked_sequences(sp):
    """The same as a batch in which every answer has its own copy of the prompt:
    bounds of two roundings of the outputs, as both sides round their P."""
    nq, pre = [333, 150, 64, 290], [-1, 0, 0, 0]
    d, p = desc(nq, nq, pre, D=128, hq=4, hkv=1)
    q, k, v, do = inputs(d, 5)
    o, lse = sp.sp_attn_fwd(d, q, k, v)
    dq, dk, dv = sp.sp_attn_bwd(d, q, k, v, o, lse, do)
    cu = np.cumsum([0] + nq)
    idx = [np.r_[0:333]] + [np.r_[0:333, cu[s]:cu[s + 1]] for s in (1, 2, 3)]
    flat = torch.from_numpy(np.concatenate(idx)).cuda()
    lens = [len(i) for i in idx]
    u, _ = desc(lens, lens, [-1] * 4, D=128, hq=4, hkv=1)
    own = torch.cat([torch.arange(333)] + [333 + torch.arange(n - 333) + sum(lens[:s + 1])
                                           for s, n in enumerate(lens[1:])]).cuda()
    uo, ul = sp.sp_attn_fwd(u, q[flat].contiguous(), k[flat].contiguous(), v[flat].contiguous())
    assert (uo[own].double() - o.double()).abs().max() <= 4 * STEP16 * v.double().abs().max()
    assert (ul[:, own] - lse).abs().max() <= 1e-4
    # gradients: rows of the copied prompts carry none
    ud = torch.zeros_like(uo)
    ud[own] = do
    udq, udk, udv = sp.sp_attn_bwd(u, q[flat].contiguous(), k[flat].contiguous(), v[flat].contiguous(), uo, ul, ud)
    for name, a, b, parts in (("dq", dq, udq, 1), ("dk", dk, udk, 4), ("dv", dv, udv, 4)):
        s = torch.zeros(a.shape, dtype=torch.float64, device="cuda").index_add_(0, flat, b.double())
        # (each side's own error is below 3 steps of the row's size: see compare)
        assert ((a.double() - s).norm() / s.norm()).item() <= 3 * STEP16, name


def test_prefix_on_a_stream_and_in_a_capture(sp):
    d, p = desc([200, 100], [200, 100], [-1, 0], D=64, hq=2, hkv=2)
    q, k, v, do = inputs(d, 1)
    o, lse = sp.sp_attn_fwd(d, q, k, v)
    want = sp.sp_attn_bwd(d, q, k, v, o, lse, do)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2, l2 = sp.sp_attn_fwd(d, q, k, v, stream=side)
    got = sp.sp_attn_bwd(d, q, k, v, o2, l2, do, stream=side)
    side.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, l2) and all(torch.equal(a, b) for a, b in zip(want, got))
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(sp.SpError):  # as every attention call
            sp.sp_attn_fwd(d, q, k, v, o=o, lse=lse, workspace=ws)
        q.add_(0)


def test_prefix_dq_accumulator_and_gradients_over_inputs(sp):
    """A float32 dQ that is added to, and dK, dV written over K and V."""
    d, p = desc([300, 200, 90], [300, 200, 90], [-1, 0, 0], D=128, hq=4, hkv=1)
    q, k, v, do = inputs(d, 2)
    o, lse = sp.sp_attn_fwd(d, q, k, v)
    dq, dk, dv = sp.sp_attn_bwd(d, q, k, v, o, lse, do)
    acc = torch.ones(q.shape, device="cuda")
    k2, v2 = k.clone(), v.clone()
    sp.sp_attn_bwd(d, q, k2, v2, o, lse, do, dq_acc=acc, dk=k2, dv=v2)
    assert torch.equal(k2, dk) and torch.equal(v2, dv)
    assert torch.equal((acc - 1).bfloat16(), dq) or ((acc - 1) - dq.float()).abs().max() <= STEP16 * dq.abs().max() + 1e-6


def test_prefix_on_a_rank_of_dummy_slots_and_empty_inputs(sp):
    """No real query head, no rows, no keys."""
    cu = np.array([0, 40, 60], np.int32)
    kw = dict(head_dim=64, H_loc=1, head_offset=3, num_real_heads=3, num_padded_heads=4, gqa_group=1, Hkv_loc=1,
              kv_head_offset=3, prefix_of=[-1, 0])
    d = sp.Desc(T_q=60, T_k=60, cu_seqlens_q=cu, cu_seqlens_k=cu, **kw)
    q, k, v, do = inputs(d, 1)
    o, lse = sp.sp_attn_fwd(d, q, k, v)
    grads = sp.sp_attn_bwd(d, q, k, v, o, lse, do)
    assert not any(t.view(torch.int16).any() for t in (o, *grads)) and (lse == -math.inf).all()
    zero = np.zeros(3, np.int32)
    d = sp.Desc(T_q=0, T_k=60, cu_seqlens_q=zero, cu_seqlens_k=cu, **dict(kw, head_offset=0, kv_head_offset=0))
    q, k, v, do = inputs(d, 1)
    o, lse = sp.sp_attn_fwd(d, q, k, v)
    dq, dk, dv = sp.sp_attn_bwd(d, q, k, v, o, lse, do)
    assert not dk.view(torch.int16).any() and not dv.view(torch.int16).any()
    d = sp.Desc(T_q=60, T_k=0, cu_seqlens_q=cu, cu_seqlens_k=zero, causal=False,
                **dict(kw, head_offset=0, kv_head_offset=0))
    q, k, v, do = inputs(d, 1)
    o, lse = sp.sp_attn_fwd(d, q, k, v)
    dq, _, _ = sp.sp_attn_bwd(d, q, k, v, o, lse, do)
    assert not o.view(torch.int16).any() and not dq.view(torch.int16).any() and (lse == -math.inf).all()


def test_prefix_row_statistics_are_kept(sp):
    """A second backward on the same workspace with SP_DESC_ROWSTATS_READY."""
    nq, pre = [260, 90, 70], [-1, 0, 0]
    d, p = desc(nq, nq, pre, D=128, hq=4, hkv=1)
    q, k, v, do = inputs(d, 4)
    o, lse = sp.sp_attn_fwd(d, q, k, v)
    ws = torch.empty(sp.sp_attn_workspace_size(d, sp.SP_OP_BWD), dtype=torch.uint8, device="cuda")
    want = sp.sp_attn_bwd(d, q, k, v, o, lse, do, workspace=ws)
    d.c.flags |= sp.SP_DESC_ROWSTATS_READY
    got = sp.sp_attn_bwd(d, q, k, v, o, lse, do, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_prefix_offsets_past_32_bits(sp):
    """A group at the end of 2.1 million keys of 8 heads (2.2e9 elements a tensor), whose
    other keys no row sees: the bits of the group alone, and no gradient before it."""
    n, H, D = 2100000, 8, 128
    for nq, nk in (([300, 120, 40], [300, 120, 40]), ([0, 1, 1], [9000, 40, 1])):
        d, _ = desc([0] + nq, [n] + nk, [-1, -1, 1, 1], D=D, hq=H, hkv=H)
        e, _ = desc(nq, nk, [-1, 0, 0], D=D, hq=H, hkv=H)
        q, k, v, do = inputs(e, 6)
        K, V = (torch.zeros(d.c.T_k, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        K[n:], V[n:] = k, v
        assert list(sp.sp_attn_plan(d, sp.SP_OP_FWD).values()) == list(sp.sp_attn_plan(e, sp.SP_OP_FWD).values())
        o, lse = sp.sp_attn_fwd(d, q, K, V)
        o2, l2 = sp.sp_attn_fwd(e, q, k, v)
        assert torch.equal(o, o2) and torch.equal(lse, l2)
        dq, dk, dv = sp.sp_attn_bwd(d, q, K, V, o, lse, do, dk=K, dv=V)
        dq2, dk2, dv2 = sp.sp_attn_bwd(e, q, k, v, o, lse, do)
        for a, b in ((dq, dq2), (dk[n:], dk2), (dv[n:], dv2)):  # (another plan sums in another order)
            assert (a.float() - b.float()).abs().max() <= 8 * STEP16 * b.float().abs().max()
        assert not dk[:n].any() and not dv[:n].any()
        del K, V, dk, dv


MANY = [  # rows (and keys) of the groups, prefixes, query and KV heads, dummies, D, causal
    ([130] + [300] * 6, [-1] + [0] * 6, 1, 1, 0, 128, True),
    ([40] + [217] * 9, [-1] + [0] * 9, 4, 2, 0, 64, True),           # one tile of keys
    ([301, 1, 0] + [300] * 13, [-1] + [0] * 15, 3, 3, 1, 64, True),   # an odd last tile, a dummy
    ([70, 800, 400, 900, 33, 700, 9, 1100], [-1, 0, 0, 0, -1, 4, 4, 4], 2, 1, 0, 128, True),  # two groups
    ([129, 513, 640, 511], [-1, 0, 0, 0], 2, 1, 0, 128, False),
    ([64, 600] + [310] * 16, [-1] + [0] * 17, 7, 1, 0, 64, True),
    ([0, 2500, 1900], [-1, 0, 0], 2, 2, 0, 128, True),                 # the prefix's keys alone
    ([130] + [20] * 200, [-1] + [0] * 200, 4, 1, 0, 128, True),       # both kinds of items in one list
    ([70] + [33] * 150, [-1] + [0] * 150, 7, 1, 0, 64, True),         # and two workgroups a CU
]


@pytest.mark.parametrize("nq,pre,hq,hkv,dummies,D,causal", MANY)
def test_prefix_of_many_rows(sp, nq, pre, hq, hkv, dummies, D, causal):
    """A short prompt, whose few key tiles see every answer's rows: those are cut into
    parts, and their sums joined."""
    nk = [n if n or i else 200 for i, n in enumerate(nq)]
    d, p = desc(nq, nk, pre, D=D, hq=hq, hkv=hkv, dummies=dummies, causal=causal, pad_k=5 if D == 64 else 0)
    alone, _ = desc(nq, nk, [-1] * len(nq), D=D, hq=hq, hkv=hkv, dummies=dummies, causal=causal, pad_k=5 if D == 64 else 0)
    sizes = [sp.sp_attn_workspace_size(x, sp.SP_OP_BWD) for x in (d, alone)]
    assert sizes[0] - sizes[1] >= 1.5 * 2 * nk[0] * hq * D * 4  # (two parts at least, and fewer items)
    o, lse, dq, dk, dv = compare(sp, d, p, seed=len(nq))
    # over K and V, in two launches
    q, k, v, do = inputs(d, len(nq))
    sp.sp_attn_bwd(d, q, k, v, o, lse, do, dk=k, dv=v)
    assert torch.equal(k, dk) and torch.equal(v, dv)


def test_prefix_of_many_rows_over_a_spoiled_workspace(sp):
    """Parts without rows are written too: nothing of the workspace's old content shows."""
    nq, pre = [257, 2600, 1, 2000], [-1, 0, 0, 0]
    d, _ = desc(nq, nq, pre, D=64, hq=2, hkv=2)
    q, k, v, do = inputs(d, 8)
    o, lse = sp.sp_attn_fwd(d, q, k, v)
    n = sp.sp_attn_workspace_size(d, sp.SP_OP_BWD)
    grads = [sp.sp_attn_bwd(d, q, k, v, o, lse, do, workspace=torch.full((n,), x, dtype=torch.uint8, device="cuda"))
             for x in (0, 255)]
    assert all(torch.equal(a, b) for a, b in zip(*grads))
