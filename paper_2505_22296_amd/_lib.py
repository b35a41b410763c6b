"""ctypes binding of libspattn.so (argument marshalling only).

Every computation happens in the HIP library; this module only turns torch
tensors into device pointers, the current torch stream into a hipStream_t,
and allocates outputs/workspaces with torch's caching allocator.  If the
compiled library is missing, loading fails loudly: there is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
from typing import Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libspattn.so")

SP_OK, SP_ERR_INVALID_ARG, SP_ERR_UNSUPPORTED, SP_ERR_WORKSPACE, SP_ERR_HIP = range(5)
SP_OP_FWD, SP_OP_BWD, SP_OP_RING_STEP = 0, 1, 2
SP_DESC_SINGLE_SEQUENCE = 1
SP_DESC_ROWSTATS_READY = 4
SP_DESC_DQ_ACC_INIT = 8
SP_DESC_SHARED_PREFIX = 32
SCHED_ITEM_INTS = 8
PLAN_INTS = 6

_i32p = ctypes.POINTER(ctypes.c_int32)


class SpAttnDesc(ctypes.Structure):
    _fields_ = [
        ("T_q", ctypes.c_int32), ("T_k", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("H_loc", ctypes.c_int32), ("head_offset", ctypes.c_int32),
        ("num_real_heads", ctypes.c_int32), ("num_padded_heads", ctypes.c_int32),
        ("gqa_group", ctypes.c_int32), ("Hkv_loc", ctypes.c_int32),
        ("kv_head_offset", ctypes.c_int32), ("num_seqs", ctypes.c_int32),
        ("causal", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
        ("flags", ctypes.c_int32),
        ("cu_seqlens_q", _i32p), ("cu_seqlens_k", _i32p),
        ("position_ids_q", _i32p), ("position_ids_k", _i32p), ("prefix_of", _i32p),
    ]


class SpPolicyParams(ctypes.Structure):
    _fields_ = [("clip_low", ctypes.c_float), ("clip_high", ctypes.c_float), ("kl_coef", ctypes.c_float),
                ("entropy_coef", ctypes.c_float), ("adv_per_token", ctypes.c_int32),
                ("ignore_index", ctypes.c_int32)]


class SpQkDesc(ctypes.Structure):
    _fields_ = [
        ("T", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("H_q", ctypes.c_int32), ("H_kv", ctypes.c_int32),
        ("sp", ctypes.c_int32), ("Hq_loc", ctypes.c_int32), ("Hkv_loc", ctypes.c_int32),
        ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("position_base", ctypes.c_int32),
        ("rope_scale", ctypes.c_float), ("eps", ctypes.c_float), ("weight_offset", ctypes.c_float),
        ("q_map", _i32p), ("kv_map", _i32p), ("inv_freq", ctypes.POINTER(ctypes.c_double)),
    ]


class SpError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = None


def load() -> ctypes.CDLL:
    """Load libspattn.so (after torch, so the library binds to the HIP
    runtime torch already loaded)."""
    global _lib
    if _lib is not None:
        return _lib
    import torch  # noqa: F401  (HIP runtime first)
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} not built; run `python -m paper_2505_22296_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    i64 = ctypes.c_int64
    D, P, Q = ctypes.POINTER(SpAttnDesc), ctypes.POINTER(SpPolicyParams), ctypes.POINTER(SpQkDesc)
    sig = {
        "sp_status_string": (ctypes.c_char_p, [i32]),
        "sp_version": (i32, []),
        # (host int32 arrays as addresses: see _i32)
        "sp_ulysses_pack": (i32, [vp, i32, i32, i32, i32, i32, vp, vp, vp]),
        "sp_ulysses_unpack": (i32, [vp, i32, i32, i32, i32, vp, i32, vp, vp]),
        "sp_ulysses_unpack_add": (i32, [vp, i32, i32, i32, i32, vp, i32, vp, vp]),
        "sp_token_logprob": (i32, [vp, vp, i32, i32, i32, vp, i32, vp, vp, vp, vp]),
        "sp_token_logprob_bwd": (i32, [vp, vp, vp, i32, i32, i32, vp, i32, vp, vp, vp]),
        "sp_loss_reduce": (i32, [vp, vp, i32, i32, i32, ctypes.c_float, vp, vp, vp]),
        "sp_policy_workspace_size": (i32, [i32, i32, ctypes.POINTER(sz)]),
        "sp_policy_loss": (i32, [P, vp, vp, vp, vp, vp, i32, i32, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]),
        "sp_policy_loss_bwd": (i32, [P, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, i32, vp, vp, vp]),
        "sp_qk_norm_rope": (i32, [Q, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, vp]),
        "sp_qk_workspace_size": (i32, [Q, ctypes.POINTER(sz)]),
        "sp_qk_norm_rope_bwd": (i32, [Q, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, vp, i64, vp, i64, vp, i64, vp, vp,
                                      vp, sz, vp]),
        "sp_attn_workspace_size": (i32, [D, i32, ctypes.POINTER(sz)]),
        "sp_attn_fwd": (i32, [D, vp, vp, vp, vp, vp, vp, sz, vp]),
        "sp_attn_fwd_static": (i32, [D, vp, vp, vp, vp, vp, vp]),
        "sp_attn_bwd": (i32, [D, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
        "sp_ring_step": (i32, [D, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp]),
        "sp_lse_merge": (i32, [vp, vp, vp, i32, vp, i32, i32, i32, vp, vp]),
        "sp_f32_to_bf16": (i32, [vp, vp, ctypes.c_int64, vp]),
        "sp_attn_schedule": (i32, [D, i32, _i32p, i32, _i32p]),
        "sp_attn_plan": (i32, [D, i32, _i32p]),
        "sp_profile_events": (i32, [i32, vp, vp]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    return lib


EXPORTED = ["sp_status_string", "sp_version", "sp_ulysses_pack", "sp_ulysses_unpack",
            "sp_ulysses_unpack_add", "sp_token_logprob", "sp_token_logprob_bwd", "sp_loss_reduce",
            "sp_policy_workspace_size", "sp_policy_loss", "sp_policy_loss_bwd",
            "sp_qk_norm_rope", "sp_qk_workspace_size", "sp_qk_norm_rope_bwd",
            "sp_attn_workspace_size", "sp_attn_fwd", "sp_attn_fwd_static", "sp_attn_bwd", "sp_ring_step",
            "sp_lse_merge", "sp_f32_to_bf16", "sp_attn_schedule", "sp_attn_plan",
            "sp_profile_events"]

SP_KERNEL_ATTN_FWD, SP_KERNEL_ATTN_DQ, SP_KERNEL_ATTN_DKDV = 1, 2, 3
SP_KERNEL_PACK, SP_KERNEL_UNPACK, SP_KERNEL_LSE_MERGE, SP_KERNEL_UNPACK_ADD = 4, 5, 6, 7
SP_KERNEL_TOKEN_LOGPROB, SP_KERNEL_TOKEN_LOGPROB_BWD = 8, 9
SP_KERNEL_POLICY, SP_KERNEL_POLICY_BWD, SP_KERNEL_QK_ROPE, SP_KERNEL_QK_ROPE_BWD = 10, 11, 12, 13
SP_LOSS_SFT, SP_LOSS_DPO = 0, 1


def status_string(s: int) -> str:
    return load().sp_status_string(int(s)).decode()


def _check(status: int, where: str):
    if status != SP_OK:
        raise SpError(status, where)


class Desc:
    """Owns an sp_attn_desc and the host arrays it points to."""

    def __init__(self, *, T_q, T_k, head_dim, H_loc, head_offset, num_real_heads,
                 num_padded_heads, gqa_group, Hkv_loc, kv_head_offset, cu_seqlens_q,
                 cu_seqlens_k, position_ids_q=None, position_ids_k=None, causal=True,
                 softmax_scale=None, single_sequence=False, rowstats_ready=False,
                 dq_acc_init=False, prefix_of=None):
        self._keep = []

        def arr(x):
            if x is None:
                return None
            a = np.ascontiguousarray(np.asarray(x, dtype=np.int32))
            self._keep.append(a)
            return a.ctypes.data_as(_i32p)

        cq = np.asarray(cu_seqlens_q, dtype=np.int32)
        # the C ABI reads these host arrays by the counts in the descriptor
        if len(np.asarray(cu_seqlens_k)) != len(cq):
            raise ValueError("cu_seqlens_q and cu_seqlens_k need the same length (num_seqs + 1)")
        for name, pos, T in (("position_ids_q", position_ids_q, T_q),
                             ("position_ids_k", position_ids_k, T_k)):
            if pos is not None and len(np.asarray(pos)) < T:
                raise ValueError(f"{name} has fewer than {T} entries")
        if prefix_of is not None and len(np.asarray(prefix_of)) != max(0, len(cq) - 1):
            raise ValueError("prefix_of needs one entry per segment")
        self.c = SpAttnDesc(
            T_q=T_q, T_k=T_k, head_dim=head_dim, H_loc=H_loc, head_offset=head_offset,
            num_real_heads=num_real_heads, num_padded_heads=num_padded_heads,
            gqa_group=gqa_group, Hkv_loc=Hkv_loc, kv_head_offset=kv_head_offset,
            num_seqs=max(0, len(cq) - 1), causal=1 if causal else 0,
            softmax_scale=(1.0 / math.sqrt(head_dim)) if softmax_scale is None else softmax_scale,
            flags=((SP_DESC_SINGLE_SEQUENCE if single_sequence else 0)
                   | (SP_DESC_ROWSTATS_READY if rowstats_ready else 0)
                   | (SP_DESC_DQ_ACC_INIT if dq_acc_init else 0)
                   | (SP_DESC_SHARED_PREFIX if prefix_of is not None else 0)),
            cu_seqlens_q=arr(cu_seqlens_q), cu_seqlens_k=arr(cu_seqlens_k),
            position_ids_q=arr(position_ids_q), position_ids_k=arr(position_ids_k),
            prefix_of=arr(prefix_of))

    @property
    def ref(self):
        return ctypes.byref(self.c)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream=None) -> int:
    """hipStream_t of `stream` or of the current device's current stream (its
    raw handle: building a Stream object cost 2.7 us of the 9 us of a small
    call's host time)."""
    if stream is not None:
        return stream.cuda_stream
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _i32(x):
    """Host int32 array of `x` and its address (valid while the array lives)."""
    a = np.ascontiguousarray(x, dtype=np.int32)
    return a, a.__array_interface__["data"][0]


_no_context = contextlib.nullcontext()


def _alloc_on(stream=None):
    """Context for the wrapper's own allocations (outputs, workspace): on the
    stream the kernels are launched on.  torch's caching allocator ties a
    block to the stream current at allocation and, once the tensor is
    dropped, hands it to the next allocation on that stream without waiting
    for other streams; a workspace allocated on the current stream but read
    by kernels queued on `stream` could be reused while they still run."""
    if stream is None:
        return _no_context
    import torch
    return torch.cuda.stream(stream)


def sp_attn_workspace_size(desc: Desc, op: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load().sp_attn_workspace_size(desc.ref, op, ctypes.byref(n)), "sp_attn_workspace_size")
    return n.value


def _with_workspace(desc: Desc, op: int, device, ws, call, where: str):
    """call(pointer, bytes) with the caller's workspace, or one allocated here
    if there is none or it is too small.  The library checks the size, so a
    workspace that fits costs no call of its own (which validates the
    descriptor, O(T) host work, once more)."""
    if ws is not None:
        status = call(ws.data_ptr(), ws.numel())
        if status != SP_ERR_WORKSPACE or ws.numel() >= sp_attn_workspace_size(desc, op):
            return _check(status, where)
    import torch
    need = sp_attn_workspace_size(desc, op)
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    _check(call(ws.data_ptr(), need), where)


def sp_attn_schedule(desc: Desc, op: int) -> np.ndarray:
    """Host-side work list: [n_items, 8] int32 (see include/sp_attn.h)."""
    lib = load()
    n = ctypes.c_int32(0)
    _check(lib.sp_attn_schedule(desc.ref, op, None, 0, ctypes.byref(n)), "sp_attn_schedule")
    out = np.zeros((max(1, n.value), SCHED_ITEM_INTS), dtype=np.int32)
    _check(lib.sp_attn_schedule(desc.ref, op, out.ctypes.data_as(_i32p), n.value, ctypes.byref(n)),
           "sp_attn_schedule")
    return out[: n.value]


def sp_attn_plan(desc: Desc, op: int) -> dict:
    """Host-side launch shapes: row_split, row_two, key_split, key_two,
    one_launch, dq_first (see include/sp_attn.h)."""
    out = (ctypes.c_int32 * PLAN_INTS)()
    _check(load().sp_attn_plan(desc.ref, op, out), "sp_attn_plan")
    return dict(zip(("row_split", "row_two", "key_split", "key_two", "one_launch", "dq_first"), out))


def sp_ulysses_pack(src, sp: int, H_dst_loc: int, head_map: Sequence[int], dst=None, stream=None):
    """src [T_loc, H_src, D] bf16 -> dst [sp, T_loc, H_dst_loc, D] bf16."""
    import torch
    T, Hs, D = src.shape
    if dst is None:
        with _alloc_on(stream):
            dst = torch.empty((sp, T, H_dst_loc, D), dtype=src.dtype, device=src.device)
    m, mp = _i32(head_map)
    _check(load().sp_ulysses_pack(_ptr(src), T, Hs, D, sp, H_dst_loc, mp, _ptr(dst),
                                  _stream(stream)), "sp_ulysses_pack")
    return dst


def sp_ulysses_unpack(src, head_map: Sequence[int], H_dst: int, dst=None, stream=None):
    """src [sp, T_loc, H_src_loc, D] bf16 -> dst [T_loc, H_dst, D] bf16."""
    import torch
    sp, T, Hs, D = src.shape
    if dst is None:
        with _alloc_on(stream):
            dst = torch.empty((T, H_dst, D), dtype=src.dtype, device=src.device)
    m, mp = _i32(head_map)
    _check(load().sp_ulysses_unpack(_ptr(src), T, Hs, D, sp, mp, H_dst, _ptr(dst),
                                    _stream(stream)), "sp_ulysses_unpack")
    return dst


def sp_ulysses_unpack_add(src, head_map: Sequence[int], H_dst: int, dst=None, stream=None):
    """src [sp, T_loc, H_src_loc, D] bf16 -> dst [T_loc, H_dst, D] bf16: the
    copies of a head that several slots name are summed (float32, ascending
    slot order, one rounding to bf16)."""
    import torch
    sp, T, Hs, D = src.shape
    if dst is None:
        with _alloc_on(stream):
            dst = torch.empty((T, H_dst, D), dtype=src.dtype, device=src.device)
    m, mp = _i32(head_map)
    _check(load().sp_ulysses_unpack_add(_ptr(src), T, Hs, D, sp, mp, H_dst, _ptr(dst),
                                        _stream(stream)), "sp_ulysses_unpack_add")
    return dst


def _cu(cu_seqlens):
    cu, p = _i32(cu_seqlens)
    return cu, p, len(cu) - 1


def sp_token_logprob(logits, labels, cu_seqlens, ignore_index: int = -100, logp=None, lse=None,
                     seq_sum=None, stream=None):
    """logits [T, V] bf16, labels [T] int32 (device) -> (logp [T], lse [T],
    seq_sum [num_seqs]) float32."""
    import torch
    T, V = logits.shape
    cu, cup, n = _cu(cu_seqlens)
    dev = logits.device
    with _alloc_on(stream):
        logp = torch.empty(T, dtype=torch.float32, device=dev) if logp is None else logp
        lse = torch.empty(T, dtype=torch.float32, device=dev) if lse is None else lse
        if seq_sum is None:
            seq_sum = torch.empty(max(n, 0), dtype=torch.float32, device=dev)
    _check(load().sp_token_logprob(_ptr(logits), _ptr(labels), T, V, ignore_index, cup, n,
                                   _ptr(logp), _ptr(lse), _ptr(seq_sum) if n > 0 else None, _stream(stream)),
           "sp_token_logprob")
    return logp, lse, seq_sum


def sp_token_logprob_bwd(logits, labels, lse, cu_seqlens, grad_seq, ignore_index: int = -100,
                         dlogits=None, stream=None):
    """-> dlogits [T, V] bf16 = g (onehot(label) - softmax(logits)) per
    counted token, g = grad_seq[its sequence]."""
    import torch
    T, V = logits.shape
    cu, cup, n = _cu(cu_seqlens)
    if dlogits is None:
        with _alloc_on(stream):
            dlogits = torch.empty_like(logits)
    _check(load().sp_token_logprob_bwd(_ptr(logits), _ptr(labels), _ptr(lse), T, V, ignore_index,
                                       cup, n, _ptr(grad_seq), _ptr(dlogits), _stream(stream)),
           "sp_token_logprob_bwd")
    return dlogits


def sp_loss_reduce(partial_sums, kind: int, coef: float, ref_partial_sums=None, loss=None,
                   grad=None, stream=None):
    """partial_sums [sp, n] float32 -> (loss [1], grad [sp, n]): the loss over
    the ranks' all-reduced sums and each rank's upstream gradient."""
    import torch
    spn, n = partial_sums.shape
    dev = partial_sums.device
    with _alloc_on(stream):
        loss = torch.empty(1, dtype=torch.float32, device=dev) if loss is None else loss
        grad = torch.empty((spn, n), dtype=torch.float32, device=dev) if grad is None else grad
    _check(load().sp_loss_reduce(_ptr(partial_sums), _ptr(ref_partial_sums), spn, n, kind,
                                 float(coef), _ptr(loss), _ptr(grad), _stream(stream)),
           "sp_loss_reduce")
    return loss, grad


def _device_of(stream) -> int:
    import torch
    return torch.cuda.current_device() if stream is None else stream.device.index


def _arg(t, name: str, dtype, shape: tuple, device: int, optional: bool = False):
    """Device pointer of a contiguous tensor argument.  The library reads memory
    by the sizes it is told, so type, shape, device and layout are checked here."""
    if t is None and optional:
        return None
    if t is None or t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {list(shape)}, got "
                         + ("none" if t is None else f"{t.dtype} {list(t.shape)}"))
    if t.get_device() != device:
        raise ValueError(f"{name} must be on GPU {device}, where its stream is: it is on {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


class PolicyParams:
    """The constants of a clipped policy loss (see include/sp_attn.h): a ratio
    counts inside [1 - clip_low, 1 + clip_high]; advantages are [num_seqs] or,
    with adv_per_token, [T]."""

    def __init__(self, clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0,
                 entropy_coef: float = 0.0, adv_per_token: bool = False, ignore_index: int = -100):
        self.c = SpPolicyParams(clip_low=clip_low, clip_high=clip_high, kl_coef=kl_coef, entropy_coef=entropy_coef,
                                adv_per_token=1 if adv_per_token else 0, ignore_index=ignore_index)

    @property
    def ref(self):
        return ctypes.byref(self.c)


def sp_policy_workspace_size(T: int, V: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load().sp_policy_workspace_size(T, V, ctypes.byref(n)), "sp_policy_workspace_size")
    return n.value


def _outs(given, dtype, device, dev):
    """Outputs and their pointers: each (tensor or None, name, shape), allocated
    here where it is None (one that is given is checked)."""
    import torch
    ts = [torch.empty(s, dtype=dtype, device=device) if t is None else t for t, _, s in given]
    return ts, [t.data_ptr() if g is None else _arg(g, n, dtype, s, dev) for t, (g, n, s) in zip(ts, given)]


def _workspace(need: int, workspace, device, dev: int):
    """The caller's workspace, or one allocated here if there is none or it is
    too small."""
    import torch
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        return torch.empty(need, dtype=torch.uint8, device=device)
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous on GPU {dev}")
    return workspace


def sp_policy_loss(params: PolicyParams, logits, labels, old_logp, ref_logp, advantages, cu_seqlens,
                   with_entropy: bool = True, logp=None, lse=None, entropy=None, seq_sum=None, seq_stats=None,
                   workspace=None, stream=None):
    """logits [T, V] bf16, labels [T] int32, old_logp and ref_logp (or None) [T]
    float32, advantages [num_seqs] or [T] float32 -> (logp, lse, entropy [T] --
    None without entropy --, seq_sum [num_seqs], seq_stats [num_seqs, 4]: sums of
    KL and entropy, clipped and counted tokens) float32."""
    import torch
    T, V = logits.shape
    cu, cup, n = _cu(cu_seqlens)
    n = max(n, 0)
    f, dev = torch.float32, _device_of(stream)
    per = T if params.c.adv_per_token else n
    args = (_arg(logits, "logits", torch.bfloat16, (T, V), dev), _arg(labels, "labels", torch.int32, (T,), dev),
            _arg(old_logp, "old_logp", f, (T,), dev), _arg(ref_logp, "ref_logp", f, (T,), dev, True),
            _arg(advantages, "advantages", f, (per,), dev))
    given = [(logp, "logp", (T,)), (lse, "lse", (T,)), (seq_sum, "seq_sum", (n,)), (seq_stats, "seq_stats", (n, 4))]
    if with_entropy:
        given.append((entropy, "entropy", (T,)))
    with _alloc_on(stream):
        ts, ps = _outs(given, f, logits.device, dev)
        ws = _workspace(sp_policy_workspace_size(T, V), workspace, logits.device, dev)
        _check(load().sp_policy_loss(params.ref, *args, T, V, cup, n, ps[0], ps[1], ps[4] if with_entropy else None,
                                     ps[2], ps[3], ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream)),
               "sp_policy_loss")
    return ts[0], ts[1], ts[4] if with_entropy else None, ts[2], ts[3]


def sp_policy_loss_bwd(params: PolicyParams, logits, labels, logp, lse, entropy, old_logp, ref_logp, advantages,
                       cu_seqlens, grad_seq, dlogits=None, stream=None):
    """-> dlogits [T, V] bf16 (which may be the logits): the gradient of
    sum(grad_seq * seq_sum), from what sp_policy_loss returned."""
    import torch
    T, V = logits.shape
    cu, cup, n = _cu(cu_seqlens)
    n = max(n, 0)
    f, bf, dev = torch.float32, torch.bfloat16, _device_of(stream)
    per = T if params.c.adv_per_token else n
    args = (_arg(logits, "logits", bf, (T, V), dev), _arg(labels, "labels", torch.int32, (T,), dev),
            _arg(logp, "logp", f, (T,), dev), _arg(lse, "lse", f, (T,), dev), _arg(entropy, "entropy", f, (T,), dev, True),
            _arg(old_logp, "old_logp", f, (T,), dev), _arg(ref_logp, "ref_logp", f, (T,), dev, True),
            _arg(advantages, "advantages", f, (per,), dev))
    grad = _arg(grad_seq, "grad_seq", f, (n,), dev)
    with _alloc_on(stream):
        (out,), (p,) = _outs([(dlogits, "dlogits", (T, V))], bf, logits.device, dev)
        _check(load().sp_policy_loss_bwd(params.ref, *args, T, V, cup, n, grad, p, _stream(stream)),
               "sp_policy_loss_bwd")
    return out


class QkDesc:
    """Owns an sp_qk_desc and the host arrays it points to."""

    def __init__(self, *, T, head_dim, H_q, H_kv, sp, q_map, kv_map, rotary_dim=None, inv_freq=None,
                 interleaved=False, position_base=0, rope_scale=1.0, eps=1e-6, weight_offset=0.0):
        qm, km = (np.ascontiguousarray(np.asarray(m, dtype=np.int32)) for m in (q_map, kv_map))
        if sp < 1 or qm.size % sp or km.size % sp or not qm.size or not km.size:
            raise ValueError("q_map and kv_map need the same number of slots for each of the sp ranks")
        rot = (head_dim if rotary_dim is None else rotary_dim) if inv_freq is not None else (rotary_dim or 0)
        f = np.ascontiguousarray(np.asarray([] if inv_freq is None else inv_freq, dtype=np.float64))
        if f.size < rot // 2:
            raise ValueError(f"inv_freq has fewer than {rot // 2} entries")
        self._keep = (qm, km, f)
        self.c = SpQkDesc(T=T, head_dim=head_dim, H_q=H_q, H_kv=H_kv, sp=sp, Hq_loc=qm.size // sp,
                          Hkv_loc=km.size // sp, rotary_dim=rot, interleaved=1 if interleaved else 0,
                          position_base=position_base, rope_scale=rope_scale, eps=eps, weight_offset=weight_offset,
                          q_map=qm.ctypes.data_as(_i32p), kv_map=km.ctypes.data_as(_i32p),
                          inv_freq=f.ctypes.data_as(ctypes.POINTER(ctypes.c_double)) if rot else None)

    @property
    def ref(self):
        return ctypes.byref(self.c)


def sp_qk_workspace_size(desc: QkDesc) -> int:
    n = ctypes.c_size_t(0)
    _check(load().sp_qk_workspace_size(desc.ref, ctypes.byref(n)), "sp_qk_workspace_size")
    return n.value


def _heads(t, name, shape, dev):
    """Pointer and token stride of a [T, H, D] bf16 tensor whose tokens may lie
    further apart than their heads need."""
    import torch
    T, H, D = shape
    if t is None or t.dtype is not torch.bfloat16 or t.shape != shape or t.get_device() != dev or T < 2:
        return _arg(t, name, torch.bfloat16, shape, dev), H * D
    st, sh, sd = t.stride()
    if sd != 1 or (sh != D and H > 1):
        raise ValueError(f"{name} must be contiguous within a token")
    return t.data_ptr(), st


def sp_qk_norm_rope(desc: QkDesc, q, k, v, positions=None, w_q=None, w_k=None, q_dst=None, k_dst=None, v_dst=None,
                    stream=None):
    """q [T, H_q, D], k, v [T, H_kv, D] bf16 (any token stride) -> (q_dst [sp, T,
    Hq_loc, D], k_dst, v_dst [sp, T, Hkv_loc, D]): normed (by w_q, w_k [D] bf16),
    rotated by positions [T] int32 (None: position_base + t) and packed."""
    import torch
    c, dev, bf = desc.c, _device_of(stream), torch.bfloat16
    T, D, Hq, Hkv = c.T, c.head_dim, c.H_q, c.H_kv
    args = (*_heads(q, "q", (T, Hq, D), dev), *_heads(k, "k", (T, Hkv, D), dev), *_heads(v, "v", (T, Hkv, D), dev),
            _arg(positions, "positions", torch.int32, (T,), dev, True), _arg(w_q, "w_q", bf, (D,), dev, True),
            _arg(w_k, "w_k", bf, (D,), dev, True))
    sq, sk = (c.sp, T, c.Hq_loc, D), (c.sp, T, c.Hkv_loc, D)
    with _alloc_on(stream):
        ts, ps = _outs([(q_dst, "q_dst", sq), (k_dst, "k_dst", sk), (v_dst, "v_dst", sk)], bf, q.device, dev)
        _check(load().sp_qk_norm_rope(desc.ref, *args, *ps, _stream(stream)), "sp_qk_norm_rope")
    return tuple(ts)


def sp_qk_norm_rope_bwd(desc: QkDesc, q, k, dq_src, dk_src, dv_src, positions=None, w_q=None, w_k=None, dq=None,
                        dk=None, dv=None, dw_q=None, dw_k=None, workspace=None, stream=None):
    """dq_src [sp, T, Hq_loc, D], dk_src, dv_src [sp, T, Hkv_loc, D] bf16 -> (dq
    [T, H_q, D], dk, dv [T, H_kv, D] bf16, dw_q, dw_k [D] float32 -- None without
    the weight).  q and k are needed where their weight is given."""
    import torch
    c, dev, bf, f = desc.c, _device_of(stream), torch.bfloat16, torch.float32
    T, D, Hq, Hkv = c.T, c.head_dim, c.H_q, c.H_kv
    sq, sk = (c.sp, T, c.Hq_loc, D), (c.sp, T, c.Hkv_loc, D)
    hq, hk = (T, Hq, D), (T, Hkv, D)
    args = (*(_heads(q, "q", hq, dev) if w_q is not None else (None, 0)),
            *(_heads(k, "k", hk, dev) if w_k is not None else (None, 0)),
            _arg(dq_src, "dq_src", bf, sq, dev), _arg(dk_src, "dk_src", bf, sk, dev),
            _arg(dv_src, "dv_src", bf, sk, dev), _arg(positions, "positions", torch.int32, (T,), dev, True),
            _arg(w_q, "w_q", bf, (D,), dev, True), _arg(w_k, "w_k", bf, (D,), dev, True))
    for w, dw, name in ((w_q, dw_q, "dw_q"), (w_k, dw_k, "dw_k")):
        if w is None and dw is not None:
            raise ValueError(f"{name} is given without its weight")
    device = dq_src.device
    with _alloc_on(stream):
        dq, dk, dv = (torch.empty(s, dtype=bf, device=device) if t is None else t for t, s in ((dq, hq), (dk, hk), (dv, hk)))
        dws, pws = _outs([(dw, n, (D,)) for w, dw, n in ((w_q, dw_q, "dw_q"), (w_k, dw_k, "dw_k")) if w is not None], f,
                         device, dev)
        ws = _workspace(sp_qk_workspace_size(desc), workspace, device, dev)
        _check(load().sp_qk_norm_rope_bwd(desc.ref, *args, *_heads(dq, "dq", hq, dev), *_heads(dk, "dk", hk, dev),
                                          *_heads(dv, "dv", hk, dev), pws[0] if w_q is not None else None,
                                          pws[-1] if w_k is not None else None, ws.data_ptr(),
                                          ws.numel() * ws.element_size(), _stream(stream)), "sp_qk_norm_rope_bwd")
    return dq, dk, dv, dws[0] if w_q is not None else None, dws[-1] if w_k is not None else None


def sp_attn_fwd(desc: Desc, q, k, v, o=None, lse=None, workspace=None, stream=None):
    import torch
    c = desc.c
    with _alloc_on(stream):
        if o is None:
            o = torch.empty((c.T_q, c.H_loc, c.head_dim), dtype=q.dtype, device=q.device)
        if lse is None:
            lse = torch.empty((c.H_loc, c.T_q), dtype=torch.float32, device=q.device)
        f, st = load().sp_attn_fwd, _stream(stream)
        _with_workspace(desc, SP_OP_FWD, q.device, workspace,
                        lambda ws, nb: f(desc.ref, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
                                         ws, nb, st), "sp_attn_fwd")
    return o, lse


STATIC_SCRATCH_BYTES = 1 << 20


def sp_attn_fwd_static(desc: Desc, q, k, v, o, lse, stream=None):
    """Allocation-free forward: outputs must be given (o [T_q, H_loc, D]
    bf16, lse [H_loc, T_q] float32); the work list lives in the library's
    fixed device array (STATIC_SCRATCH_BYTES per GPU)."""
    _check(load().sp_attn_fwd_static(desc.ref, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
                                     _stream(stream)), "sp_attn_fwd_static")
    return o, lse


def sp_attn_bwd(desc: Desc, q, k, v, o, lse, dout, dq=None, dq_acc=None, dk=None, dv=None,
                workspace=None, stream=None):
    import torch
    with _alloc_on(stream):
        if dq is None and dq_acc is None:
            dq = torch.empty_like(q)
        if dk is None:
            dk = torch.empty_like(k)
        if dv is None:
            dv = torch.empty_like(v)
        f, st = load().sp_attn_bwd, _stream(stream)
        _with_workspace(desc, SP_OP_BWD, q.device, workspace,
                        lambda ws, nb: f(desc.ref, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse),
                                         _ptr(dout), _ptr(dq), _ptr(dq_acc), _ptr(dk), _ptr(dv),
                                         ws, nb, st), "sp_attn_bwd")
    return (dq if dq is not None else dq_acc), dk, dv


def sp_ring_step(desc: Desc, q, k_chunk, v_chunk, o_acc, lse_acc, init: bool, o_out=None,
                 workspace=None, stream=None):
    with _alloc_on(stream):
        f, st = load().sp_ring_step, _stream(stream)
        _with_workspace(desc, SP_OP_RING_STEP, q.device, workspace,
                        lambda ws, nb: f(desc.ref, _ptr(q), _ptr(k_chunk), _ptr(v_chunk),
                                         _ptr(o_acc), _ptr(lse_acc), 1 if init else 0,
                                         _ptr(o_out), ws, nb, st), "sp_ring_step")
    return o_acc, lse_acc


def sp_lse_merge(o_acc, lse_acc, o_part, lse_part, o_out=None, stream=None):
    import torch
    T, H, D = o_acc.shape
    is_bf16 = 1 if o_part.dtype == torch.bfloat16 else 0
    _check(load().sp_lse_merge(_ptr(o_acc), _ptr(lse_acc), _ptr(o_part), is_bf16, _ptr(lse_part),
                               T, H, D, _ptr(o_out), _stream(stream)), "sp_lse_merge")
    return o_acc, lse_acc


def sp_f32_to_bf16(src, dst=None, stream=None):
    import torch
    if dst is None:
        with _alloc_on(stream):
            dst = torch.empty(src.shape, dtype=torch.bfloat16, device=src.device)
    _check(load().sp_f32_to_bf16(_ptr(src), _ptr(dst), src.numel(), _stream(stream)),
           "sp_f32_to_bf16")
    return dst


def sp_profile_events(kernel_id: int, start=None, stop=None):
    """Arm (or with None, disarm) the per-thread timer of one kernel with
    torch.cuda.Event objects (enable_timing=True; recorded once beforehand so
    the underlying hipEvent exists)."""
    _check(load().sp_profile_events(kernel_id, None if start is None else start.cuda_event,
                                    None if stop is None else stop.cuda_event),
           "sp_profile_events")
