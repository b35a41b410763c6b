"""CPU-only checks of the policy loss and of norm / rotation / pack: what the
library and its wrappers refuse before anything is launched (fake pointers are
never dereferenced), and the sizes they report."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2505_22296_amd as sp

FAKE = 1 << 20
BIG = 1 << 40


def _cu(*v):
    a = np.array(v, dtype=np.int32)
    return a, a.ctypes.data


def _policy(lib, p, **over):
    """Status of a forward with fake device pointers."""
    a, cu = _cu(*over.pop("cu", (0, 4, 8)))
    kw = dict(logits=FAKE, labels=FAKE, old=FAKE, ref=FAKE, adv=FAKE, T=8, V=64, n=len(a) - 1, logp=FAKE, lse=FAKE,
              ent=FAKE, sums=FAKE, stats=FAKE, ws=FAKE, nb=BIG)
    kw.update(over)
    return lib.sp_policy_loss(p, kw["logits"], kw["labels"], kw["old"], kw["ref"], kw["adv"], kw["T"], kw["V"], cu,
                              kw["n"], kw["logp"], kw["lse"], kw["ent"], kw["sums"], kw["stats"], kw["ws"], kw["nb"],
                              None)


def _policy_bwd(lib, p, **over):
    a, cu = _cu(*over.pop("cu", (0, 4, 8)))
    kw = dict(logits=FAKE, labels=FAKE, logp=FAKE, lse=FAKE, ent=FAKE, old=FAKE, ref=FAKE, adv=FAKE, T=8, V=64,
              n=len(a) - 1, grad=FAKE, out=FAKE)
    kw.update(over)
    return lib.sp_policy_loss_bwd(p, kw["logits"], kw["labels"], kw["logp"], kw["lse"], kw["ent"], kw["old"], kw["ref"],
                                  kw["adv"], kw["T"], kw["V"], cu, kw["n"], kw["grad"], kw["out"], None)


@pytest.mark.parametrize("over,expect", [
    (dict(V=60), sp.SP_ERR_INVALID_ARG), (dict(V=0), sp.SP_ERR_INVALID_ARG), (dict(T=-1), sp.SP_ERR_INVALID_ARG),
    (dict(logits=FAKE + 8), sp.SP_ERR_INVALID_ARG), (dict(logits=None), sp.SP_ERR_INVALID_ARG),
    (dict(labels=None), sp.SP_ERR_INVALID_ARG), (dict(old=None), sp.SP_ERR_INVALID_ARG),
    (dict(adv=None), sp.SP_ERR_INVALID_ARG), (dict(logp=None), sp.SP_ERR_INVALID_ARG),
    (dict(cu=(0, 6, 4)), sp.SP_ERR_INVALID_ARG), (dict(cu=(0, 4, 9)), sp.SP_ERR_INVALID_ARG),
    (dict(cu=(-1, 4, 8)), sp.SP_ERR_INVALID_ARG), (dict(ref=None), sp.SP_ERR_INVALID_ARG),
    (dict(ent=None), sp.SP_ERR_INVALID_ARG), (dict(T=1 << 24, cu=(0, 4)), sp.SP_ERR_UNSUPPORTED),
    (dict(T=300, cu=tuple(range(258))), sp.SP_ERR_UNSUPPORTED),
])
def test_policy_refusals(over, expect):
    lib, p = sp.load(), sp.PolicyParams(kl_coef=0.1, entropy_coef=0.1)
    assert _policy(lib, p.ref, **dict(over)) == expect
    assert _policy_bwd(lib, p.ref, **dict(over)) == expect


def test_policy_refusals_of_one_direction():
    lib, p = sp.load(), sp.PolicyParams(kl_coef=0.1, entropy_coef=0.1)
    for over in (dict(ws=None), dict(nb=255), dict(ws=FAKE + 64)):
        assert _policy(lib, p.ref, **over) == sp.SP_ERR_WORKSPACE
    for over in (dict(sums=None), dict(stats=None)):
        assert _policy(lib, p.ref, **over) == sp.SP_ERR_INVALID_ARG
    for over in (dict(grad=None), dict(out=None), dict(out=FAKE + 2), dict(lse=None)):
        assert _policy_bwd(lib, p.ref, **over) == sp.SP_ERR_INVALID_ARG
    assert _policy(lib, None) == sp.SP_ERR_INVALID_ARG
    assert _policy_bwd(lib, p.ref, T=0, cu=(0, 0), logits=None, out=None) == sp.SP_OK  # no tokens: nothing to write


@pytest.mark.parametrize("over", [dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-0.1),
                                  dict(clip_high=float("inf")), dict(kl_coef=float("nan")),
                                  dict(entropy_coef=float("inf")), dict(clip_low=float("nan"))])
def test_policy_constants_refused(over):
    lib, p = sp.load(), sp.PolicyParams(**over)
    assert _policy(lib, p.ref) == sp.SP_ERR_INVALID_ARG
    assert _policy_bwd(lib, p.ref) == sp.SP_ERR_INVALID_ARG


def test_policy_workspace_sizes():
    n = ctypes.c_size_t(0)
    lib = sp.load()
    assert lib.sp_policy_workspace_size(4, 60, ctypes.byref(n)) == sp.SP_ERR_INVALID_ARG
    assert lib.sp_policy_workspace_size(4, 64, None) == sp.SP_ERR_INVALID_ARG
    for T, V in ((0, 8), (1, 8), (1, 152064), (48, 152064), (4096, 152064), (100000, 8)):
        need = sp.sp_policy_workspace_size(T, V)
        assert need >= 256 and need % 256 == 0 and need >= 16 * T and need <= (1 << 20) + 16 * T


def test_policy_wrapper_refuses_wrong_tensors(monkeypatch):
    """Types, shapes and devices are looked at before the library is called."""
    from paper_2505_22296_amd import _lib
    monkeypatch.setattr(_lib, "_device_of", lambda s: 0)
    p, x = sp.PolicyParams(), torch.zeros(4, 64, dtype=torch.bfloat16)
    lab, f, cu = torch.zeros(4, dtype=torch.int32), torch.zeros(4), [0, 4]
    with pytest.raises(ValueError, match="must be on GPU 0"):
        sp.sp_policy_loss(p, x, lab, f, None, f[:1], cu)
    with pytest.raises(ValueError, match="logits must be a torch.bfloat16"):
        sp.sp_policy_loss(p, x.float(), lab, f, None, f[:1], cu)


# ------------------------------------------------------- norm, rotation, pack
def _qk(**over):
    kw = dict(T=4, head_dim=64, H_q=3, H_kv=3, sp=2, q_map=[0, 1, 2, -1], kv_map=[0, 1, 2, -1],
              inv_freq=np.ones(64))
    kw.update(over)
    return sp.QkDesc(**kw)


def _size_status(d):
    n = ctypes.c_size_t(0)
    return sp.load().sp_qk_workspace_size(d.ref, ctypes.byref(n)), n.value


@pytest.mark.parametrize("over,expect", [
    (dict(), sp.SP_OK), (dict(head_dim=128), sp.SP_OK), (dict(rotary_dim=0), sp.SP_OK), (dict(rotary_dim=16), sp.SP_OK),
    (dict(T=0), sp.SP_OK), (dict(inv_freq=None), sp.SP_OK),
    (dict(head_dim=96), sp.SP_ERR_UNSUPPORTED), (dict(T=-1), sp.SP_ERR_INVALID_ARG),
    (dict(T=1 << 24), sp.SP_ERR_UNSUPPORTED), (dict(rotary_dim=24), sp.SP_ERR_INVALID_ARG),
    (dict(rotary_dim=80), sp.SP_ERR_INVALID_ARG), (dict(q_map=[0, 1, 3, -1]), sp.SP_ERR_INVALID_ARG),
    (dict(kv_map=[0, 1, 2, -2]), sp.SP_ERR_INVALID_ARG), (dict(eps=-1.0), sp.SP_ERR_INVALID_ARG),
    (dict(eps=float("nan")), sp.SP_ERR_INVALID_ARG), (dict(rope_scale=float("inf")), sp.SP_ERR_INVALID_ARG),
    (dict(weight_offset=float("nan")), sp.SP_ERR_INVALID_ARG),
    (dict(inv_freq=np.full(64, np.inf)), sp.SP_ERR_INVALID_ARG), (dict(H_q=0), sp.SP_ERR_INVALID_ARG),
    (dict(H_q=257), sp.SP_ERR_UNSUPPORTED), (dict(q_map=[0] * 514), sp.SP_ERR_UNSUPPORTED),
])
def test_qk_descriptor_refusals(over, expect):
    st, n = _size_status(_qk(**over))
    assert st == expect
    if st == sp.SP_OK:
        assert n >= 256 and n % 256 == 0


def test_qk_wrapper_refusals():
    with pytest.raises(ValueError):
        _qk(q_map=[0, 1, 2])            # three slots over two ranks
    with pytest.raises(ValueError):
        _qk(inv_freq=np.ones(8), rotary_dim=64)
    assert _size_status(_qk())[0] == sp.SP_OK
    assert sp.load().sp_qk_workspace_size(None, ctypes.byref(ctypes.c_size_t(0))) == sp.SP_ERR_INVALID_ARG


def test_qk_calls_refuse_before_launch():
    lib, d = sp.load(), _qk()
    ok = [FAKE, 192, FAKE, 192, FAKE, 192, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None]

    def fwd(**at):
        a = list(ok)
        for i, v in at.items():
            a[int(i[1:])] = v
        return lib.sp_qk_norm_rope(d.ref, *a)
    for i in (0, 2, 4, 9, 10, 11):
        assert fwd(**{f"_{i}": None}) == sp.SP_ERR_INVALID_ARG      # a missing tensor
        assert fwd(**{f"_{i}": FAKE + 8}) == sp.SP_ERR_INVALID_ARG  # a misaligned one
    for i in (1, 3, 5):
        assert fwd(**{f"_{i}": 184}) == sp.SP_ERR_INVALID_ARG       # the heads do not fit
        assert fwd(**{f"_{i}": 196}) == sp.SP_ERR_INVALID_ARG       # not a multiple of 8
        assert fwd(**{f"_{i}": 1 << 26}) == sp.SP_ERR_INVALID_ARG   # past 32-bit offsets
    for i in (7, 8):
        assert fwd(**{f"_{i}": FAKE + 2}) == sp.SP_ERR_INVALID_ARG
    bwd_ok = [FAKE, 192, FAKE, 192, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 192, FAKE, 192, FAKE, 192, FAKE, FAKE,
              FAKE, BIG, None]

    def bwd(**at):
        a = list(bwd_ok)
        for i, v in at.items():
            a[int(i[1:])] = v
        return lib.sp_qk_norm_rope_bwd(d.ref, *a)
    for i in (0, 2, 4, 5, 6, 10, 12, 14, 16, 17):
        assert bwd(**{f"_{i}": None}) == sp.SP_ERR_INVALID_ARG
    for i in (1, 3, 11, 13, 15):
        assert bwd(**{f"_{i}": 184}) == sp.SP_ERR_INVALID_ARG
    assert bwd(_8=None) == sp.SP_ERR_INVALID_ARG                     # dw_q without w_q
    for at in (dict(_18=None), dict(_18=FAKE + 16), dict(_19=255)):
        assert bwd(**at) == sp.SP_ERR_WORKSPACE
    z = _qk(T=0)
    assert lib.sp_qk_norm_rope(z.ref, None, 192, None, 192, None, 192, None, None, None, None, None, None,
                               None) == sp.SP_OK
