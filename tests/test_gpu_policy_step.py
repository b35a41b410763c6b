"""One attention layer and the policy loss over a group of answers, on two
sequence-parallel ranks that share this GPU (the all-to-alls are copies between
their buffers): norm, rotation and pack -> attention with a shared prompt -> unpack
-> logits -> clipped policy loss, and back to the projection, the norms' weights
and the output matrix -- against float64 autograd of the unpacked sequences."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def reference(x, cu, pre, pos, labels, old, ref, adv, hs, hkv, D, V, freq, n):
    """Loss and gradients of the definition in float64: every answer attends to its
    own concatenation [prompt, answer]."""
    qkv, wq, wk, wo = (x[k].double().requires_grad_() for k in ("qkv", "wq", "wk", "wo"))
    T = qkv.shape[0]
    ang = torch.outer(pos.double(), freq)[:, None]
    c, s = ang.cos(), ang.sin()

    def head(y, w):
        y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
        a, b = y[..., :D // 2], y[..., D // 2:]
        return torch.cat([a * c - b * s, a * s + b * c], -1)
    q, k, v = head(qkv[:, :hs], wq), head(qkv[:, hs:hs + hkv], wk), qkv[:, hs + hkv:]
    k, v = (t.repeat_interleave(hs // hkv, 1) for t in (k, v))
    rows = []
    for i, f in enumerate(pre):
        own = torch.arange(cu[i], cu[i + 1])
        keys = own if f < 0 else torch.cat([torch.arange(cu[f], cu[f + 1]), own])
        z = torch.einsum("qhd,khd->hqk", q[own], k[keys]) / math.sqrt(D)
        z = z.masked_fill((keys[None] > own[:, None])[None], -math.inf)
        rows.append(torch.einsum("hqk,khd->qhd", z.softmax(-1), v[keys]))
    o = torch.cat(rows)
    logits = o.flatten(1) @ wo
    lp = torch.log_softmax(logits, 1)
    total = 0.0
    for i in range(len(pre)):
        t = torch.arange(cu[i], cu[i + 1])
        t = t[labels[t] >= 0]
        if not len(t):
            continue
        l = lp[t, labels[t]]
        r = torch.exp(l - old[t])
        d = ref[t] - l
        ent = -(lp[t].exp() * lp[t]).sum(1)
        total = total + (-torch.minimum(r * adv[i], r.clamp(0.8, 1.28) * adv[i]) + 0.05 * (torch.exp(d) - d - 1)
                         - 0.01 * ent).sum()
    loss = total / n
    loss.backward()
    return loss.detach(), dict(qkv=qkv.grad, wq=wq.grad, wk=wk.grad, wo=wo.grad), lp.detach()


@pytest.mark.parametrize("hs,hkv,D,lens,pre", [
    (7, 7, 64, [90, 40, 61, 33], [-1, 0, 0, 0]),
    (6, 2, 128, [100, 30, 30, 64, 17, 9], [-1, 0, 0, -1, 3, 3]),
])
def test_policy_step_of_two_ranks(hs, hkv, D, lens, pre):
    import paper_2505_22296_amd as sp
    n, V = 2, 512
    cu = np.cumsum([0] + lens).astype(np.int32)
    T = int(cu[-1])
    C = T // n
    assert T % n == 0
    g = torch.Generator().manual_seed(T)
    x = dict(qkv=torch.randn(T, hs + 2 * hkv, D, generator=g).bfloat16(), wq=(1 + 0.2 * torch.randn(D, generator=g)).bfloat16(),
             wk=(1 + 0.2 * torch.randn(D, generator=g)).bfloat16(),
             wo=(torch.randn(hs * D, V, generator=g) * 2 / math.sqrt(hs * D)).bfloat16())
    pos = torch.cat([torch.arange(m) + (0 if f < 0 else lens[f]) for m, f in zip(lens, pre)])
    labels = torch.randint(0, V, (T,), generator=g)
    for i, f in enumerate(pre):
        if f < 0:
            labels[cu[i]:cu[i + 1]] = -100  # prompts do not count
    counted = int((labels >= 0).sum())
    adv = torch.randn(len(pre), generator=g)
    freq = 1e4 ** (-2.0 * np.arange(D // 2) / D)
    ratio, away = 0.05 * torch.randn(T, generator=g).double(), 0.3 * torch.randn(T, generator=g).double()
    zero = torch.zeros(T, dtype=torch.float64)
    _, _, lp = reference(x, cu, pre, pos, labels, zero, zero, adv.double(), hs, hkv, D, V, torch.from_numpy(freq), counted)
    at = lp.gather(1, labels.clamp(min=0)[:, None])[:, 0]
    # (|ratio| < 0.2 = -log 0.82: this batch's bf16 logits do not reach the clip)
    old, ref = (at - ratio.clamp(-0.1, 0.1)).float(), (at + away).float()
    loss, want, _ = reference(x, cu, pre, pos, labels, old.double(), ref.double(), adv.double(), hs, hkv, D, V,
                              torch.from_numpy(freq), counted)

    # ---- the ranks
    loc = -(-hs // n)
    qm = np.arange(loc * n)
    qm[qm >= hs] = -1
    if hs == hkv:
        km, koff, kloc = qm, [0, loc], loc
    else:
        kloc = 1
        km, koff = np.arange(hkv), [0, 1]
    dev = {k: t.cuda() for k, t in x.items()}
    qkv, p = dev["qkv"], pos.to(torch.int32).cuda()
    sl = [slice(r * C, (r + 1) * C) for r in range(n)]
    qk = sp.QkDesc(T=C, head_dim=D, H_q=hs, H_kv=hkv, sp=n, q_map=qm, kv_map=km, inv_freq=freq)
    heads = (slice(0, hs), slice(hs, hs + hkv), slice(hs + hkv, None))
    packed = [sp.sp_qk_norm_rope(qk, *(qkv[s, h] for h in heads), p[s], dev["wq"], dev["wk"]) for s in sl]
    desc, kept = [], []
    for r in range(n):
        desc.append(sp.Desc(T_q=T, T_k=T, head_dim=D, H_loc=loc, head_offset=r * loc, num_real_heads=hs,
                            num_padded_heads=loc * n, gqa_group=hs // hkv, Hkv_loc=kloc, kv_head_offset=koff[r],
                            cu_seqlens_q=cu, cu_seqlens_k=cu, position_ids_q=pos, position_ids_k=pos, prefix_of=pre))
        q, k, v = (torch.cat([packed[j][i][r] for j in range(n)]) for i in range(3))  # all-to-all
        kept.append((q, k, v, *sp.sp_attn_fwd(desc[r], q, k, v)))
    acts, logits, outs = [], [], []
    params = sp.PolicyParams(0.2, 0.28, 0.05, 0.01)
    tok = dict(labels=labels.to(torch.int32).cuda(), old=old.cuda(), ref=ref.cuda())
    cus = [np.clip(cu - r * C, 0, C) for r in range(n)]
    for r, s in enumerate(sl):
        recv = torch.stack([kept[j][3][s] for j in range(n)])
        acts.append(sp.sp_ulysses_unpack(recv, qm, hs).flatten(1))
        logits.append((acts[r].float() @ dev["wo"].float()).bfloat16())
        outs.append(sp.sp_policy_loss(params, logits[r], tok["labels"][s], tok["old"][s], tok["ref"][s], adv.cuda(), cus[r]))
    got_loss, grad = sp.sp_loss_reduce(torch.stack([o[3] for o in outs]), sp.SP_LOSS_SFT, -1.0 / counted)
    assert sum(int(o[4][:, 3].sum()) for o in outs) == counted

    # ---- back; sp_loss_reduce gives each rank sp times its gradient (parameter
    # gradients are averaged over the ranks), activations take their own share
    dwo, dact = 0.0, []
    for r, s in enumerate(sl):
        dl = sp.sp_policy_loss_bwd(params, logits[r], tok["labels"][s], *outs[r][:3], tok["old"][s], tok["ref"][s],
                                   adv.cuda(), cus[r], grad[r].contiguous() / n)
        dwo = dwo + acts[r].float().t() @ dl.float()
        dact.append((dl.float() @ dev["wo"].float().t().contiguous()).bfloat16().view(C, hs, D))
    sent = [sp.sp_ulysses_pack(d, n, loc, qm) for d in dact]
    grads = [sp.sp_attn_bwd(desc[r], *kept[r], torch.cat([sent[j][r] for j in range(n)])) for r in range(n)]
    dqkv, dwq, dwk = torch.empty_like(qkv), 0.0, 0.0
    for s in sl:
        recv = [torch.stack([grads[j][i][s] for j in range(n)]) for i in range(3)]
        _, _, _, a, b = sp.sp_qk_norm_rope_bwd(qk, qkv[s, heads[0]], qkv[s, heads[1]], *recv, p[s], dev["wq"], dev["wk"],
                                               **{k: dqkv[s, h] for k, h in zip(("dq", "dk", "dv"), heads)})
        dwq, dwk = dwq + a, dwk + b
    # Logits of size 2 rounded to bf16 (2^-8) move a log-probability by 2^-7 and a
    # token's gradient by that part; each of the five bf16 stages on the way back
    # (logits' gradient, its product, attention, norm) adds two roundings or less.
    tol = 2.0 ** -7 + 10 * 2.0 ** -8
    assert abs(got_loss.item() - loss.item()) <= 4 * 2.0 ** -7 * (1 + adv.abs().max().item())
    for name, v in (("qkv", dqkv), ("wq", dwq), ("wk", dwk), ("wo", dwo)):
        w = want[name]
        rel = ((v.double().cpu() - w).norm() / w.norm()).item()
        assert rel <= tol, (name, rel)
