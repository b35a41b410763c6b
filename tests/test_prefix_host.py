"""CPU-only checks of SP_DESC_SHARED_PREFIX: refusals, and that the work lists
cover exactly the pairs the definition allows."""
import ctypes

import numpy as np
import pytest
from hypothesis import given, settings, strategies as st

import paper_2505_22296_amd as sp


def mask_of(cu_q, cu_k, pos_q, pos_k, prefix_of, T_q, T_k, causal):
    """[T_q, T_k]: which key a row sees, from the definition alone."""
    m = np.zeros((T_q, T_k), bool)
    for s, f in enumerate(prefix_of):
        for i in range(cu_q[s], cu_q[s + 1]):
            for j in range(cu_k[s], cu_k[s + 1]):
                m[i, j] = not causal or pos_k[j] <= pos_q[i]
            if f >= 0:
                m[i, cu_k[f]:cu_k[f + 1]] = True
    return m


def ramps(cu, T, first):
    p = np.zeros(T, np.int32)
    for s in range(len(cu) - 1):
        p[cu[s]:cu[s + 1]] = first[s] + np.arange(cu[s + 1] - cu[s])
    return p


def desc(nq, nk, pre, D=128, hq=4, hkv=1, dummies=0, causal=True, pad_q=0, pad_k=0, first_q=None, first_k=None):
    """Segments of nq rows and nk keys; positions so that a segment's last row is
    at its last key's position, answers continuing their prefix."""
    cu_q, cu_k = (np.concatenate([[0], np.cumsum(n)]).astype(np.int32) for n in (nq, nk))
    T_q, T_k = int(cu_q[-1]) + pad_q, int(cu_k[-1]) + pad_k
    fk = [0 if f < 0 else nk[f] for f in pre] if first_k is None else first_k
    fq = [k + b - a for k, a, b in zip(fk, nq, nk)] if first_q is None else first_q
    fq = [max(0, x) for x in fq]
    pos_q, pos_k = ramps(cu_q, T_q, fq), ramps(cu_k, T_k, fk)
    H = hq + dummies
    heads = dict(H_loc=H, head_offset=0, num_real_heads=hq, num_padded_heads=H, gqa_group=hq // hkv, Hkv_loc=hkv,
                 kv_head_offset=0)
    if dummies:
        heads = dict(H_loc=H, head_offset=H, num_real_heads=H + hq, num_padded_heads=2 * H,
                     gqa_group=1 if hq == hkv else H + hq, Hkv_loc=H if hq == hkv else 1,
                     kv_head_offset=H if hq == hkv else 0)
    d = sp.Desc(T_q=T_q, T_k=T_k, head_dim=D, cu_seqlens_q=cu_q, cu_seqlens_k=cu_k, position_ids_q=pos_q,
                position_ids_k=pos_k, causal=causal, prefix_of=pre, **heads)
    return d, dict(cu_q=cu_q, cu_k=cu_k, pos_q=pos_q, pos_k=pos_k, prefix_of=pre, T_q=T_q, T_k=T_k, causal=causal)


def status(d, op=sp.SP_OP_FWD):
    return sp.load().sp_attn_workspace_size(d.ref, op, ctypes.byref(ctypes.c_size_t(0)))


@pytest.mark.parametrize("pre,expect", [
    ([-1, 0, 0, -1, 3], sp.SP_OK), ([-1, -1, -1, -1, -1], sp.SP_OK), ([-1, 0, -1, -1, -1], sp.SP_OK),
    ([0, -1, -1, -1, -1], sp.SP_ERR_INVALID_ARG),   # its own prefix
    ([-1, 2, -1, -1, -1], sp.SP_ERR_INVALID_ARG),   # a prefix behind it
    ([-1, 0, 1, -1, -1], sp.SP_ERR_INVALID_ARG),    # a prefix with a prefix
    ([-1, 0, -1, 0, -1], sp.SP_ERR_INVALID_ARG),    # a group torn apart
    ([-1, -1, 0, -1, -1], sp.SP_ERR_INVALID_ARG),
    ([-1, -2, -1, -1, -1], sp.SP_ERR_INVALID_ARG),
    ([-1, 5, -1, -1, -1], sp.SP_ERR_INVALID_ARG),
])
def test_which_prefixes_are_refused(pre, expect):
    d, _ = desc([10] * 5, [10] * 5, [-1] * 5)
    a = np.asarray(pre, np.int32)
    d.c.prefix_of = a.ctypes.data_as(sp._lib._i32p)
    assert status(d) == expect and status(d, sp.SP_OP_BWD) == expect
    d.c.flags = 0  # without the flag nobody reads it
    assert status(d) == sp.SP_OK


def test_other_refusals():
    d, _ = desc([10, 5, 5], [10, 5, 5], [-1, 0, 0])
    assert status(d, sp.SP_OP_RING_STEP) == sp.SP_ERR_UNSUPPORTED
    fake, lib = 1 << 20, sp.load()
    assert lib.sp_ring_step(d.ref, fake, fake, fake, fake, fake, 1, None, fake, 1 << 40, None) == sp.SP_ERR_UNSUPPORTED
    with pytest.raises(sp.SpError):
        sp.sp_attn_schedule(d, sp.SP_OP_RING_STEP)
    with pytest.raises(sp.SpError):
        sp.sp_attn_plan(d, sp.SP_OP_RING_STEP)
    assert lib.sp_attn_fwd(d.ref, fake, fake, fake, fake, fake, None, 0, None) == sp.SP_ERR_WORKSPACE
    d.c.flags |= sp.SP_DESC_SINGLE_SEQUENCE
    assert status(d) == sp.SP_ERR_INVALID_ARG
    d.c.flags = sp.SP_DESC_SHARED_PREFIX
    d.c.prefix_of = None
    assert status(d) == sp.SP_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        desc([10, 5], [10, 5], [-1, 0, 0])
    # a prefix whose last row does not see its last key
    d, _ = desc([10, 5], [10, 5], [-1, 0], first_q=[8, 10], first_k=[9, 10])
    assert status(d) == sp.SP_ERR_INVALID_ARG
    d, _ = desc([10, 5], [10, 5], [-1, 0], first_q=[8, 10], first_k=[9, 10], causal=False)
    assert status(d) == sp.SP_OK
    d, _ = desc([0, 5], [10, 5], [-1, 0])  # a prefix without rows
    assert status(d) == sp.SP_OK


def covered(items, T_q, T_k, causal, rows):
    cov, seen = {}, {}
    for it in items:
        a, b, c, e, delta, head = (int(v) for v in it[:6])
        q0, q1, k0, k1 = (a, b, c, e) if rows else (c, e, a, b)
        m = cov.setdefault(head, np.zeros((T_q, T_k), np.int32))
        i, j = np.arange(q0, q1)[:, None], np.arange(k0, k1)[None]
        m[q0:q1, k0:k1] += (j <= i + delta) if causal or (rows and delta == 1 << 30) else np.ones((q1 - q0, k1 - k0), bool)
        if rows and delta == 1 << 30:
            continue
        n = seen.setdefault(head, np.zeros(T_q if rows else T_k, np.int32))
        n[a:b] += 1
    return cov, seen


def check_lists(d, p, real):
    want = mask_of(p["cu_q"], p["cu_k"], p["pos_q"], p["pos_k"], p["prefix_of"], p["T_q"], p["T_k"], p["causal"])
    for op, rows in ((sp.SP_OP_FWD, True), (sp.SP_OP_BWD, False)):
        cov, seen = covered(sp.sp_attn_schedule(d, op), p["T_q"], p["T_k"], p["causal"], rows)
        n = p["T_q"] if rows else p["T_k"]
        assert set(seen) == (set(range(real)) if n else set())
        for h in seen:
            assert (seen[h] == 1).all()
            assert np.array_equal(cov[h], want.astype(np.int32)), (op, h)


@settings(max_examples=60, deadline=None)
@given(data=st.data())
def test_lists_cover_exactly_the_mask(data):
    draw = data.draw
    nq, nk, pre = [], [], []
    causal, train = draw(st.booleans()), draw(st.booleans())
    for _ in range(draw(st.integers(1, 3))):
        at = len(nq)
        n = draw(st.sampled_from([0, 1, 7, 31, 33, 130, 300]))
        nk.append(n)
        nq.append(n if train else draw(st.sampled_from([0, n // 2])))
        pre.append(-1)
        for _ in range(draw(st.integers(0, 5))):
            n = draw(st.sampled_from([0, 1, 2, 31, 32, 40, 257]))
            nk.append(n)
            nq.append(n if train else draw(st.sampled_from([min(n, 1), n, 1])))
            pre.append(at)
    dummies = draw(st.integers(0, 1))
    hq, hkv = draw(st.sampled_from([(1, 1), (2, 1), (2, 2)]))
    if hq != hkv:
        dummies = 0
    d, p = desc(nq, nk, pre, D=draw(st.sampled_from([64, 128])), hq=hq, hkv=hkv, dummies=dummies, causal=causal,
                pad_q=draw(st.sampled_from([0, 3, 270])), pad_k=draw(st.sampled_from([0, 5])))
    check_lists(d, p, hq)


def test_plans_of_calls_without_rows_heads_or_keys():
    """Sizes and plans of shared-prefix calls with nothing to do."""
    for nq, nk in (([0, 0], [50, 3]), ([50, 3], [0, 0]), ([0, 0], [0, 0])):
        d, _ = desc(nq, nk, [-1, 0], causal=False)
        for op in (sp.SP_OP_FWD, sp.SP_OP_BWD):
            assert status(d, op) == sp.SP_OK
            assert len(sp.sp_attn_plan(d, op)) == 6
    d = sp.Desc(T_q=8, T_k=8, head_dim=64, H_loc=1, head_offset=3, num_real_heads=3, num_padded_heads=4, gqa_group=1,
                Hkv_loc=1, kv_head_offset=3, cu_seqlens_q=[0, 4, 8], cu_seqlens_k=[0, 4, 8], prefix_of=[-1, 0])
    assert status(d) == sp.SP_OK and sp.sp_attn_plan(d, sp.SP_OP_FWD)["key_split"] == 0
    assert len(sp.sp_attn_schedule(d, sp.SP_OP_FWD)) == 0


def test_few_rows_take_parts_of_the_keys():
    """Many keys and few rows; not where the rows alone fill the launch, or their
    windows do not fit its arguments."""
    for nq, nk, split in (([0, 1, 1], [20000, 30, 40], True), ([0, 1, 1], [300, 30, 40], False),
                          ([2000, 40, 40], [2000, 40, 40], False), ([0, 2100], [20000, 2100], False)):
        d, _ = desc(nq, nk, [-1] + [0] * (len(nq) - 1))
        parts = sp.sp_attn_plan(d, sp.SP_OP_FWD)["key_split"]
        assert (parts >= 2) == split and parts <= 256
        small = sp.sp_attn_workspace_size(d, sp.SP_OP_FWD)
        assert small >= parts * d.c.T_q * d.c.H_loc * (d.c.head_dim + 1) * 4


def test_rests_of_answers_share_tiles():
    """Sixteen answers of 600 rows to a prompt: 2 full tiles an answer, and 88 rows
    left, three groups of rows, of all answers in 6 tiles; the prompt has 3."""
    d, p = desc([600] * 17, [600] * 17, [-1] + [0] * 16, hq=1, hkv=1)
    items = sp.sp_attn_schedule(d, sp.SP_OP_FWD)
    rows = [tuple(it[:2]) for it in items if it[4] != 1 << 30]
    assert len(rows) == 17 * (8 * 2 + 3)
    n = sp.sp_attn_workspace_size(d, sp.SP_OP_FWD) // 32
    tiles = 3 + 16 * 2 + 6
    assert tiles <= n <= tiles * 13 + 8  # items, and at most 12 items' room of records each
    check_lists(d, p, 1)
