"""Thin binding of libtppo.so (see include/tppo.h for the contract): ctypes, and for the calls of a training step a native
half (csrc/marshal.cpp), which checks, allocates and calls in half to four fifths of the time (figures there).

Argument marshalling only: every step of the path runs in the HIP kernels.
PyTorch provides device memory and the current HIP stream.  There is no CPU
fallback: if the shared library is missing, every call raises.
"""
import ctypes
import importlib.machinery
import importlib.util
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtppo.so")
NATIVE_PATH = os.path.join(_HERE, "_marshal.so")

TPPO_F32, TPPO_BF16 = 0, 1
ERRORS = {-1: "TPPO_ERR_NULL", -2: "TPPO_ERR_SIZE", -3: "TPPO_ERR_PARAM", -4: "TPPO_ERR_DTYPE",
          -5: "TPPO_ERR_WORKSPACE", -6: "TPPO_ERR_LAUNCH"}
STATUS_BAD_TARGET, STATUS_BAD_LAYOUT, STATUS_CAPACITY, STATUS_BAD_ROW, STATUS_TIMEOUT = 1, 2, 4, 8, 16

_c_i64, _c_i32, _c_f32, _c_ptr, _c_size = (ctypes.c_int64, ctypes.c_int32, ctypes.c_float,
                                            ctypes.c_void_p, ctypes.c_size_t)
_SIGNATURES = {
    "tppo_version": (ctypes.c_int, []),
    "tppo_select_workspace_bytes": (_c_size, [_c_i64, _c_i64]),
    "tppo_select": (ctypes.c_int, [_c_ptr] * 4 + [_c_i64, _c_i64, _c_i32] + [_c_ptr] * 6 +
                    [_c_i64, _c_ptr, _c_ptr, _c_size, _c_ptr, _c_size, _c_ptr, _c_ptr]),
    "tppo_plan_bytes": (_c_size, [_c_i64, _c_i64]),
    "tppo_plan_build": (ctypes.c_int, [_c_ptr] * 3 + [_c_i64, _c_i64, _c_ptr, _c_size, _c_ptr, _c_ptr]),
    "tppo_token_logprobs_workspace_bytes": (_c_size, [_c_i64, _c_i64, _c_i64, ctypes.c_int]),
    "tppo_token_logprobs": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_i64, _c_ptr, _c_i64, _c_i64,
                                           ctypes.c_int, _c_ptr, _c_ptr, _c_i64, _c_ptr, _c_ptr,
                                           _c_ptr, _c_ptr, _c_ptr, _c_size, _c_ptr, _c_ptr]),
    "tppo_egae_workspace_bytes": (_c_size, [_c_i64, _c_i64]),
    "tppo_egae": (ctypes.c_int, [_c_ptr] * 5 + [_c_i64, _c_i64, _c_f32, _c_f32, _c_ptr, _c_ptr,
                                                _c_ptr, _c_size, _c_ptr, _c_ptr, _c_ptr]),
    "tppo_egae_terminal": (ctypes.c_int, [_c_ptr] * 5 + [_c_i64, _c_i64, _c_f32, _c_f32, _c_ptr, _c_ptr,
                                                         _c_ptr, _c_size, _c_ptr, _c_ptr, _c_ptr]),
    "tppo_egae_static_max_tiles": (_c_i64, []),
    "tppo_egae_static": (ctypes.c_int, [_c_ptr] * 5 + [_c_i64, _c_i64, _c_f32, _c_f32, _c_ptr, _c_ptr,
                                                       _c_ptr, _c_ptr]),
    "tppo_ppo_losses_workspace_bytes": (_c_size, [_c_i64, _c_i64]),
    "tppo_ppo_losses": (ctypes.c_int, [_c_ptr] * 9 + [_c_i64, _c_i64] + [_c_f32] * 4 +
                        [_c_ptr, _c_ptr, _c_size, _c_ptr, _c_ptr, _c_ptr]),
    "tppo_ppo_losses_backward_workspace_bytes": (_c_size, [_c_i64, _c_i64]),
    "tppo_ppo_losses_backward": (ctypes.c_int, [_c_ptr] * 9 + [_c_i64, _c_i64] + [_c_f32] * 6 +
                                 [_c_i64, _c_i64] + [_c_ptr] * 5 + [_c_size, _c_ptr, _c_ptr, _c_ptr]),
    "tppo_token_logprobs_backward_workspace_bytes": (_c_size, [_c_i64, _c_i64, _c_i64, ctypes.c_int]),
    "tppo_token_logprobs_backward": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_i64, _c_ptr, _c_i64, _c_i64,
                                                    ctypes.c_int, _c_ptr, _c_ptr, _c_i64, _c_ptr, _c_ptr,
                                                    _c_ptr, _c_ptr, _c_ptr, _c_i32, _c_ptr, _c_size, _c_ptr,
                                                    _c_ptr]),
    "tppo_batcher_create": (_c_ptr, [_c_i64, _c_i32, _c_i32]),
    "tppo_batcher_destroy": (None, [_c_ptr]),
    "tppo_batcher_refill": (ctypes.c_int, [_c_ptr, _c_ptr, _c_i64, ctypes.POINTER(ctypes.c_int64)]),
    "tppo_batcher_advance": (ctypes.c_int, [_c_ptr, _c_ptr, _c_ptr]),
    "tppo_batcher_layout": (ctypes.c_int, [_c_ptr] * 6),
    "tppo_value_head": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_i64, _c_ptr, _c_f32, ctypes.c_int, _c_ptr,
                                       _c_ptr, _c_i64, _c_ptr, _c_ptr, _c_ptr, _c_ptr]),
    "tppo_layer_norm": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_i64, ctypes.c_int, _c_ptr, _c_ptr, ctypes.c_int, _c_f32,
                                       _c_ptr, _c_i64, _c_ptr, _c_ptr, _c_i64, _c_ptr, _c_ptr, _c_ptr, _c_ptr]),
    "tppo_layer_norm_backward_workspace_bytes": (_c_size, [_c_i64, _c_i64]),
    "tppo_layer_norm_backward": (ctypes.c_int, [_c_ptr, _c_i64, ctypes.c_int, _c_ptr, _c_i64, _c_i64, _c_i64, ctypes.c_int,
                                                _c_ptr, ctypes.c_int, _c_ptr, _c_ptr, _c_ptr, _c_i64, _c_ptr, _c_ptr, _c_i64,
                                                ctypes.c_int, _c_ptr, _c_i64, _c_ptr, _c_ptr, _c_i32, _c_ptr, _c_size,
                                                _c_ptr, _c_ptr]),
    "tppo_balance_loss_workspace_bytes": (_c_size, [_c_i64, _c_i64]),
    "tppo_balance_loss": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_i64, ctypes.c_int, _c_ptr, _c_i64, _c_i64, _c_ptr, _c_i64,
                                         _c_ptr, _c_f32, _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_size, _c_ptr, _c_ptr]),
    "tppo_balance_loss_backward": (ctypes.c_int, [_c_ptr, _c_i64, _c_i64, _c_i64, ctypes.c_int, _c_ptr, _c_i64, _c_i64, _c_ptr,
                                                  _c_i64, _c_ptr, _c_f32, _c_f32, _c_ptr, _c_i64, _c_ptr, _c_i64, _c_ptr, _c_i64,
                                                  _c_ptr, _c_ptr, _c_ptr, _c_ptr, _c_size, _c_ptr, _c_ptr]),
    "tppo_orthogonalize_workspace_bytes": (_c_size, [_c_i64] * 3),
    "tppo_orthogonalize": (ctypes.c_int, [_c_ptr] + [_c_i64] * 5 + [ctypes.c_int, _c_i32] + [_c_f32] * 5 +
                           [_c_ptr, _c_i64, _c_i64, _c_ptr, _c_size, _c_ptr]),
    "tppo_diag_streams": (ctypes.c_int, [_c_ptr, _c_ptr, _c_i64, _c_i64, _c_i32, _c_i32, _c_ptr]),
    "tppo_diag_mfma_rate": (ctypes.c_int, [_c_ptr, _c_ptr, _c_i64, ctypes.POINTER(ctypes.c_double), _c_ptr]),
}
EXPORTS = tuple(_SIGNATURES)
_lib = None


def load():
    """Load libtppo.so (built by ``python -m paper_2506_15050_amd.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2506_15050_amd.build`; there is no fallback path")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


_native_module = None


def _native():
    """The native half of the binding (built with the library)."""
    global _native_module
    if _native_module is None:
        load()
        if not os.path.exists(NATIVE_PATH):
            raise RuntimeError(f"{NATIVE_PATH} is missing: build it with "
                               "`python -m paper_2506_15050_amd.build`; there is no fallback path")
        loader = importlib.machinery.ExtensionFileLoader("_marshal", NATIVE_PATH)
        _native_module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_marshal", loader))
        loader.exec_module(_native_module)
    return _native_module


def _check(rc, what):
    if rc != 0:
        raise RuntimeError(f"{what} failed: {ERRORS.get(rc, rc)}")


def _ptr(t):
    return None if t is None else t.data_ptr()          # the argument types turn it into a pointer


# The current stream of the current device.  torch's way to the raw handle has private names; a torch without them gets
# the public way, a Stream object that costs 2.8 us to make (the smallest calls are bound by what happens here).
if hasattr(torch._C, "_cuda_getCurrentRawStream") and hasattr(torch._C, "_cuda_getDevice"):
    _raw_stream, _device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice

    def _stream():
        return _raw_stream(_device())
else:
    def _stream():
        return torch.cuda.current_stream().cuda_stream


def _dev_i32(t):
    assert t.is_cuda and t.dtype == torch.int32 and t.is_contiguous()
    return t


def _dev_f32(t):
    assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()
    return t


def _workspace(nbytes, device):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def new_status(device):
    return torch.zeros(1, dtype=torch.int32, device=device)


def tppo_select(cu_seqlens, ctx_len, done, input_ids, tail_drop, capacity=None, status=None,
                want_indices=True, n_tok=None, workspace=None, want_plan=False, plan=None):
    """Token filter.  Returns a dict of device tensors: resp_off, sel_off, keep_len,
    sel_rows, sel_targets, sel_resp_idx (capacity-sized) and counts (int64[3] =
    M, n_resp, N_val); with ``want_plan`` (or a ``plan`` buffer) also ``plan``, the
    work plan that tppo_egae* and the loss calls take."""
    native = _native()
    B = ctx_len.numel()
    if input_ids is not None:
        n_tok = input_ids.numel()
    assert n_tok is not None, "n_tok is required when input_ids is None"
    cap = n_tok if capacity is None else int(capacity)
    kinds, sizes = "iiil", [B + 1, B + 1, B, 3]
    if want_indices:
        kinds += "iii" if input_ids is not None else "ii"
        sizes += [cap] * (len(kinds) - 4)
    if workspace is None and want_indices:
        kinds += "b"
        sizes.append(max(native.select_workspace_bytes(B, max(cap, n_tok)), 256))
    if plan is None and want_plan:
        kinds += "b"
        sizes.append(max(native.plan_bytes(n_tok, B), 256))
    made = iter(native.empties(cu_seqlens, kinds, *sizes))
    resp_off, sel_off, keep_len, counts = next(made), next(made), next(made), next(made)
    out = dict(resp_off=resp_off, sel_off=sel_off, keep_len=keep_len, counts=counts)
    rows = targets = resp_idx = None
    ws = workspace
    if want_indices:
        rows, resp_idx = next(made), next(made)
        targets = next(made) if input_ids is not None else None
        out.update(sel_rows=rows, sel_targets=targets, sel_resp_idx=resp_idx)
        if ws is None:
            ws = next(made)
    if plan is None and want_plan:
        plan = next(made)
    out["plan"] = plan
    rc = native.select(cu_seqlens, ctx_len, done, input_ids, B, n_tok, int(tail_drop), resp_off, sel_off, keep_len, rows,
                       targets, resp_idx, cap, counts, ws, plan, status, _stream())
    _check(rc, "tppo_select")
    return out


def tppo_plan_build(resp_off, keep_len, done, n_resp, status=None, plan=None):
    """Work plan of a batch layout (keep_len may be None: such a plan serves tppo_egae* only)."""
    lib = load()
    B = done.numel()
    if plan is None:
        plan = _workspace(lib.tppo_plan_bytes(int(n_resp), B), resp_off.device)
    rc = lib.tppo_plan_build(_ptr(_dev_i32(resp_off)), _ptr(keep_len), _ptr(_dev_i32(done)), B, int(n_resp),
                             _ptr(plan), plan.numel(), _ptr(status), _stream())
    _check(rc, "tppo_plan_build")
    return plan


def tppo_token_logprobs(hidden, w_head, sel_rows, sel_targets, M=None, m_actual=None,
                        out_index=None, out_size=None, want_lse=True, status=None, workspace=None):
    """log pi(a_t|s_t) of the kept tokens.  hidden [n_rows, H], w_head [V, H], both
    bf16 or both fp32.  Returns (logp, lse)."""
    lib = load()
    assert hidden.is_cuda and w_head.is_cuda and hidden.dtype == w_head.dtype
    assert hidden.dim() == 2 and w_head.dim() == 2 and hidden.stride(1) == 1 and w_head.stride(1) == 1
    dt = {torch.float32: TPPO_F32, torch.bfloat16: TPPO_BF16}[hidden.dtype]
    n_rows, H = hidden.shape
    V = w_head.shape[0]
    M = sel_rows.numel() if M is None else int(M)
    n_out = M if out_size is None else int(out_size)
    native = _native()
    made = native.empties(hidden, "ff" if want_lse else "f", *([n_out] * (2 if want_lse else 1)))
    logp, lse = made if want_lse else (made[0], None)
    ws = workspace
    if ws is None:
        ws = _workspace(lib.tppo_token_logprobs_workspace_bytes(M, H, V, dt), hidden.device)
    rc = native.token_logprobs(hidden, n_rows, H, hidden.stride(0), w_head, V, w_head.stride(0), dt, sel_rows, sel_targets, M,
                               m_actual, out_index, logp, lse, ws, status, _stream())
    _check(rc, "tppo_token_logprobs")
    return logp, lse


def _scratch(lib_bytes, n_resp, B, workspace, plan, device):
    """The workspace of a call that may have been given a plan instead."""
    if plan is not None or workspace is not None:
        return workspace
    return _workspace(lib_bytes(n_resp, B), device)


def tppo_egae(rewards, values, resp_off, done, gamma, lam, bootstrap=None, status=None,
              workspace=None, out=None, plan=None):
    """Extended GAE advantages and Monte-Carlo returns.  Returns (adv, ret)."""
    lib = load()
    n_resp, B = rewards.numel(), done.numel()
    adv, ret = out if out is not None else (torch.empty_like(rewards), torch.empty_like(rewards))
    ws = _scratch(lib.tppo_egae_workspace_bytes, n_resp, B, workspace, plan, rewards.device)
    rc = _native().egae(rewards, values, resp_off, done, bootstrap, B, n_resp, float(gamma), float(lam), adv, ret, ws, plan,
                        status, _stream())
    _check(rc, "tppo_egae")
    return adv, ret


def tppo_egae_static(rewards, values, resp_off, done, gamma, lam, bootstrap=None, status=None, out=None):
    """``tppo_egae`` without a workspace: the library's own fixed array holds the plan.  The binding
    still allocates the outputs unless ``out=(adv, ret)`` is given.  Returns (adv, ret)."""
    lib = load()
    n_resp, B = rewards.numel(), done.numel()
    adv, ret = out if out is not None else (torch.empty_like(rewards), torch.empty_like(rewards))
    rc = lib.tppo_egae_static(_ptr(_dev_f32(rewards)), _ptr(_dev_f32(values)), _ptr(_dev_i32(resp_off)),
                              _ptr(_dev_i32(done)), _ptr(bootstrap), B, n_resp, float(gamma), float(lam),
                              _ptr(adv), _ptr(ret), _ptr(status), _stream())
    _check(rc, "tppo_egae_static")
    return adv, ret


def tppo_egae_terminal(terminal_reward, values, resp_off, done, gamma, lam, bootstrap=None, status=None,
                       workspace=None, out=None, plan=None):
    """Extended GAE with one terminal reward per finished sequence instead of a
    dense reward array.  Returns (adv, ret)."""
    lib = load()
    n_resp, B = values.numel(), done.numel()
    adv, ret = out if out is not None else (torch.empty_like(values), torch.empty_like(values))
    ws = _scratch(lib.tppo_egae_workspace_bytes, n_resp, B, workspace, plan, values.device)
    rc = _native().egae_terminal(terminal_reward, values, resp_off, done, bootstrap, B, n_resp, float(gamma), float(lam), adv,
                                 ret, ws, plan, status, _stream())
    _check(rc, "tppo_egae_terminal")
    return adv, ret


class LossOut(ctypes.Structure):
    _fields_ = [("policy_loss", ctypes.c_float), ("value_loss", ctypes.c_float),
                ("policy_sum", ctypes.c_float), ("value_sum", ctypes.c_float),
                ("n_policy", ctypes.c_int64), ("n_value", ctypes.c_int64)]


def tppo_ppo_losses(logp_new, logp_old, adv, v_new, v_old, ret, resp_off, keep_len, done,
                    eps_low, eps_high, xi_low, xi_high, status=None, workspace=None, out=None, plan=None):
    """Clipped policy / value losses.  Returns a 32-byte device tensor holding a
    ``tppo_loss_out``; ``read_loss_out`` copies it to the host."""
    lib = load()
    dev = resp_off.device
    B = done.numel()
    n_resp = (logp_new if logp_new is not None else v_new).numel()
    res = torch.empty(ctypes.sizeof(LossOut), dtype=torch.uint8, device=dev) if out is None else out
    ws = _scratch(lib.tppo_ppo_losses_workspace_bytes, n_resp, B, workspace, plan, dev)
    rc = _native().ppo_losses(logp_new, logp_old, adv, v_new, v_old, ret, resp_off, keep_len, done, B, n_resp, float(eps_low),
                              float(eps_high), float(xi_low), float(xi_high), res, ws, plan, status, _stream())
    _check(rc, "tppo_ppo_losses")
    return res


def read_loss_out(res):
    """Device ``tppo_loss_out`` -> dict (synchronises)."""
    raw = bytes(res.cpu().numpy().tobytes())
    s = LossOut.from_buffer_copy(raw)
    return {name: getattr(s, name) for name, _ in LossOut._fields_}


def tppo_token_logprobs_backward(hidden, w_head, sel_rows, sel_targets, lse, grad_logp, M=None,
                                 in_index=None, want_hidden=True, want_w=True, grad_w=None,
                                 accumulate_w=False, status=None, workspace=None):
    """Derivatives of the kept tokens' log-probs with respect to the hidden rows
    ([M, H] fp32, compact order) and the head matrix ([V, H] fp32)."""
    lib = load()
    assert hidden.is_cuda and w_head.is_cuda and hidden.dtype == w_head.dtype == torch.bfloat16
    assert hidden.stride(1) == 1 and w_head.stride(1) == 1
    n_rows, H = hidden.shape
    V = w_head.shape[0]
    M = sel_rows.numel() if M is None else int(M)
    dev = hidden.device
    g_h = torch.empty(M, H, dtype=torch.float32, device=dev) if want_hidden else None
    if want_w and grad_w is None:
        grad_w = torch.empty(V, H, dtype=torch.float32, device=dev)
    if not want_w:
        grad_w = None
    ws = workspace
    if ws is None:
        ws = _workspace(lib.tppo_token_logprobs_backward_workspace_bytes(M, H, V, TPPO_BF16), dev)
    rc = lib.tppo_token_logprobs_backward(_ptr(hidden), n_rows, H, hidden.stride(0), _ptr(w_head), V,
                                          w_head.stride(0), TPPO_BF16, _ptr(_dev_i32(sel_rows)),
                                          _ptr(_dev_i32(sel_targets)), M, _ptr(_dev_f32(lse)),
                                          _ptr(_dev_f32(grad_logp)), _ptr(in_index), _ptr(g_h), _ptr(grad_w),
                                          1 if accumulate_w else 0, _ptr(ws), ws.numel(), _ptr(status),
                                          _stream())
    _check(rc, "tppo_token_logprobs_backward")
    return g_h, grad_w


def tppo_value_head(hidden, w_value, bias=0.0, rows=None, M=None, m_actual=None, out_index=None,
                    out_size=None, status=None, out=None):
    """V(s_t) = w_value . hidden[rows[t]] + bias.  Returns the fp32 values."""
    lib = load()
    assert hidden.is_cuda and hidden.dtype == w_value.dtype == torch.bfloat16 and hidden.stride(1) == 1
    n_rows, H = hidden.shape
    if M is None:
        M = n_rows if rows is None else rows.numel()
    n_out = int(M) if out_size is None else int(out_size)
    v = torch.empty(n_out, dtype=torch.float32, device=hidden.device) if out is None else out
    rc = _native().value_head(hidden, n_rows, H, hidden.stride(0), w_value, float(bias), TPPO_BF16, rows, out_index, int(M),
                              m_actual, v, status, _stream())
    _check(rc, "tppo_value_head")
    return v


_DTYPES = {torch.float32: TPPO_F32, torch.bfloat16: TPPO_BF16}


def _rows_like(t, what):
    """A device matrix whose rows lie whole in memory, for a call that takes their stride."""
    if not (t.is_cuda and t.dim() == 2 and t.dtype in _DTYPES and (t.stride(1) == 1 or t.shape[1] == 1)):
        raise ValueError(f"{what}: a device matrix of fp32 or bf16 with rows contiguous in memory is required")
    return t, (t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1]))


def _vector_like(t, n, dtypes, what):
    """A contiguous device tensor of n elements (None passes)."""
    if t is None:
        return None
    if not (t.is_cuda and t.is_contiguous() and t.numel() == n and t.dtype in dtypes):
        raise ValueError(f"{what}: a contiguous device tensor of {n} elements of the documented type is required")
    return t


def _count_rows(rows, M, n_rows, what):
    """The number of rows a call is about, and its list checked against it."""
    if rows is not None:
        if not (rows.is_cuda and rows.dtype == torch.int32 and rows.is_contiguous()):
            raise ValueError(f"{what}: rows must be a contiguous int32 device tensor")
        if M is not None and int(M) > rows.numel():
            raise ValueError(f"{what}: M = {int(M)} is more than the {rows.numel()} rows listed")
        return rows.numel() if M is None else int(M)
    return n_rows if M is None else int(M)


def _same_device(what, first, *others):
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError(f"{what}: tensors on {first.device} and {t.device}")


def _m_actual(t, what):
    if t is not None and not (t.is_cuda and t.dtype == torch.int64 and t.numel() >= 1):
        raise ValueError(f"{what}: m_actual must be an int64 device tensor")
    return t


def tppo_layer_norm(x, weight, bias=None, eps=1e-5, rows=None, M=None, m_actual=None, want_stats=True, status=None, out=None):
    """Layer norm of the rows x[rows] (rows None: all), compact.  x [n_rows, H] bf16 or fp32; weight, bias [H] fp32, or bf16
    with bf16 x.  ``out``: (y, mean, rstd) to write to.  Returns (y, mean, rstd); the statistics are None without ``want_stats``."""
    what = "tppo_layer_norm"
    lib = load()
    x, ld_x = _rows_like(x, what)
    n_rows, H = x.shape
    M = _count_rows(rows, M, n_rows, what)
    _vector_like(weight, H, _DTYPES, what)
    _vector_like(bias, H, (weight.dtype,), what)
    if out is None:
        y = torch.empty(M, H, dtype=x.dtype, device=x.device)
        mean, rstd = (torch.empty(M, dtype=torch.float32, device=x.device) for _ in range(2)) if want_stats else (None, None)
    else:
        y, mean, rstd = out
        for t in (mean, rstd):
            _vector_like(t, t.numel() if t is not None and t.numel() >= M else M, (torch.float32,), what)
    y, ld_y = _rows_like(y, what)
    if y.dtype != x.dtype or y.shape[0] < M or y.shape[1] != H:
        raise ValueError(f"{what}: y must be [M, H] of x's type")
    _same_device(what, x, weight, bias, rows, y, mean, rstd, _m_actual(m_actual, what), status)
    with torch.cuda.device(x.device):
        rc = lib.tppo_layer_norm(_ptr(x), n_rows, H, ld_x, _DTYPES[x.dtype], _ptr(weight), _ptr(bias), _DTYPES[weight.dtype],
                                 float(eps), _ptr(rows), M, _ptr(m_actual), _ptr(y), ld_y, _ptr(mean), _ptr(rstd), _ptr(status),
                                 _stream())
    _check(rc, what)
    return y, mean, rstd


def tppo_layer_norm_backward(grad_y, x, weight, mean, rstd, rows=None, M=None, m_actual=None, out_index=None, out=None,
                             grad_dtype=None, want_x=True, want_w=True, want_bias=True, grad_w=None, accumulate_w=False,
                             status=None, workspace=None):
    """Derivatives of ``tppo_layer_norm``.  grad_y [M, H] fp32 or bf16 (fp32 with fp32 x).  ``out``: the grad_x tensor to
    write to, whose rows ``out_index`` names (None: 0 .. M-1); otherwise a new [M, H] one of ``grad_dtype`` (x's by default).
    ``grad_w``: (grad_weight, grad_bias) fp32 to write, or with ``accumulate_w`` to add, to.  Returns (grad_x, grad_weight,
    grad_bias), None where not wanted."""
    what = "tppo_layer_norm_backward"
    lib = load()
    x, ld_x = _rows_like(x, what)
    grad_y, ld_gy = _rows_like(grad_y, what)
    n_rows, H = x.shape
    M = _count_rows(rows, M, n_rows, what)
    if grad_y.shape[0] < M or grad_y.shape[1] != H:
        raise ValueError(f"{what}: grad_y must be [M, H]")
    _vector_like(weight, H, _DTYPES, what)
    for t in (mean, rstd):
        if t.numel() < M:
            raise ValueError(f"{what}: statistics of {M} rows are required")
        _vector_like(t, t.numel(), (torch.float32,), what)
    if out_index is not None and not (out_index.is_cuda and out_index.dtype == torch.int32 and out_index.is_contiguous() and
                                      out_index.numel() >= M):
        raise ValueError(f"{what}: out_index must be a contiguous int32 device tensor of M entries")
    if out_index is not None and out is None and want_x:
        raise ValueError(f"{what}: out_index needs the tensor that it points into (out)")
    gx, ld_gx = None, H
    if want_x:
        gx = torch.empty(M, H, dtype=grad_dtype or x.dtype, device=x.device) if out is None else out
        gx, ld_gx = _rows_like(gx, what)
        if gx.shape[1] != H or (out_index is None and gx.shape[0] < M):
            raise ValueError(f"{what}: grad_x must be [M, H]")
    if not want_w:
        grad_w = (None, None)
    elif grad_w is None:
        if accumulate_w:
            raise ValueError(f"{what}: accumulate_w needs the tensors to add to (grad_w)")
        grad_w = (torch.empty(H, dtype=torch.float32, device=x.device),
                  torch.empty(H, dtype=torch.float32, device=x.device) if want_bias else None)
    g_w, g_b = (_vector_like(t, H, (torch.float32,), what) for t in grad_w)
    if not want_bias:
        g_b = None
    ws = workspace
    if ws is None and (g_w is not None or g_b is not None):
        ws = _workspace(lib.tppo_layer_norm_backward_workspace_bytes(M, H), x.device)
    _same_device(what, x, grad_y, weight, mean, rstd, rows, out_index, gx, g_w, g_b, ws, _m_actual(m_actual, what), status)
    with torch.cuda.device(x.device):
        rc = lib.tppo_layer_norm_backward(_ptr(grad_y), ld_gy, _DTYPES[grad_y.dtype], _ptr(x), n_rows, H, ld_x, _DTYPES[x.dtype],
                                          _ptr(weight), _DTYPES[weight.dtype], _ptr(mean), _ptr(rstd), _ptr(rows), M,
                                          _ptr(m_actual), _ptr(gx), ld_gx, _DTYPES[gx.dtype if want_x else x.dtype],
                                          _ptr(out_index), gx.shape[0] if want_x else 0, _ptr(g_w), _ptr(g_b),
                                          1 if accumulate_w else 0, _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                          _ptr(status), _stream())
    _check(rc, what)
    return gx, g_w, g_b


def _balance_arguments(logits, experts, rows, M, m_actual, workspace, out, status, what):
    lib = load()
    logits, ld = _rows_like(logits, what)
    n_rows, E = logits.shape
    if not (experts.is_cuda and experts.dtype == torch.int32 and experts.dim() == 2 and experts.shape[0] == n_rows and
            (experts.stride(1) == 1 or experts.shape[1] == 1)):
        raise ValueError(f"{what}: experts must be an int32 device matrix [n_rows, k] with rows contiguous in memory")
    M = _count_rows(rows, M, n_rows, what)
    if out is None:
        loss, mean_prob = (torch.empty(n, dtype=torch.float32, device=logits.device) for n in (1, E))
        counts = torch.empty(E, dtype=torch.int64, device=logits.device)
    else:
        loss, counts, mean_prob = out
        _vector_like(loss, 1, (torch.float32,), what)
        _vector_like(counts, E, (torch.int64,), what)
        _vector_like(mean_prob, E, (torch.float32,), what)
    ws = _workspace(lib.tppo_balance_loss_workspace_bytes(M, E), logits.device) if workspace is None else workspace
    _same_device(what, logits, experts, rows, loss, counts, mean_prob, ws, _m_actual(m_actual, what), status)
    k = experts.shape[1]
    return lib, logits, ld, n_rows, E, max(experts.stride(0), k), k, M, loss, counts, mean_prob, ws


def tppo_balance_loss(logits, experts, rows=None, M=None, m_actual=None, coefficient=1.0, status=None, workspace=None, out=None):
    """Balance loss of a mixture-of-experts router over the tokens ``rows`` (None: all).  logits [n_rows, E] bf16 or fp32;
    experts [n_rows, k] int32, -1 where none was chosen.  ``out``: (loss, counts, mean_prob) to write to.  Returns (loss [1]
    fp32, counts [E] int64, mean_prob [E] fp32)."""
    what = "tppo_balance_loss"
    lib, logits, ld, n_rows, E, ld_e, k, M, loss, counts, mean_prob, ws = _balance_arguments(
        logits, experts, rows, M, m_actual, workspace, out, status, what)
    with torch.cuda.device(logits.device):
        rc = lib.tppo_balance_loss(_ptr(logits), n_rows, E, ld, _DTYPES[logits.dtype], _ptr(experts), k, ld_e, _ptr(rows), M,
                                   _ptr(m_actual), float(coefficient), _ptr(loss), _ptr(counts), _ptr(mean_prob), _ptr(ws),
                                   ws.numel() * ws.element_size(), _ptr(status), _stream())
    _check(rc, what)
    return loss, counts, mean_prob


def tppo_balance_loss_backward(logits, experts, rows=None, M=None, m_actual=None, coefficient=1.0, scale=1.0, counts_in=None,
                               token_denominator=0, out_index=None, grad=None, status=None, workspace=None, out=None):
    """Derivative of ``tppo_balance_loss`` with respect to the logits, and the loss with it.  ``grad``: the tensor to write
    the derivatives to, whose rows ``out_index`` names (None: 0 .. M-1); otherwise a new [M, E] one of the logits' type.
    ``counts_in`` [E] int64 and ``token_denominator`` stand for a batch of which this call has a part.  Returns (grad_logits,
    loss, counts, mean_prob)."""
    what = "tppo_balance_loss_backward"
    lib, logits, ld, n_rows, E, ld_e, k, M, loss, counts, mean_prob, ws = _balance_arguments(
        logits, experts, rows, M, m_actual, workspace, out, status, what)
    _vector_like(counts_in, E, (torch.int64,), what)
    if out_index is not None and not (out_index.is_cuda and out_index.dtype == torch.int32 and out_index.is_contiguous() and
                                      out_index.numel() >= M):
        raise ValueError(f"{what}: out_index must be a contiguous int32 device tensor of M entries")
    if out_index is not None and grad is None:
        raise ValueError(f"{what}: out_index needs the tensor that it points into (grad)")
    g = torch.empty(M, E, dtype=logits.dtype, device=logits.device) if grad is None else grad
    g, ld_g = _rows_like(g, what)
    if g.dtype != logits.dtype or g.shape[1] != E or (out_index is None and g.shape[0] < M):
        raise ValueError(f"{what}: grad must be [M, E] of the logits' type")
    _same_device(what, logits, g, counts_in, out_index)
    with torch.cuda.device(logits.device):
        rc = lib.tppo_balance_loss_backward(_ptr(logits), n_rows, E, ld, _DTYPES[logits.dtype], _ptr(experts), k, ld_e, _ptr(rows),
                                            M, _ptr(m_actual), float(coefficient), float(scale), _ptr(counts_in),
                                            int(token_denominator), _ptr(g), ld_g, _ptr(out_index), g.shape[0], _ptr(loss),
                                            _ptr(counts), _ptr(mean_prob), _ptr(ws), ws.numel() * ws.element_size(),
                                            _ptr(status), _stream())
    _check(rc, what)
    return g, loss, counts, mean_prob


def tppo_orthogonalize(g, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, scale=1.0, workspace=None, out=None):
    """An update made nearly orthogonal by Newton-Schulz products.  g [rows, cols] or [count, rows, cols], bf16 or fp32, rows
    contiguous in memory.  Returns the bf16 result in g's shape (``out``, if given)."""
    what = "tppo_orthogonalize"
    lib = load()

    def stack(t, types):
        if not (t.is_cuda and t.dim() in (2, 3) and t.dtype in types and (t.stride(-1) == 1 or t.shape[-1] == 1)):
            raise ValueError(f"{what}: matrices on the device with rows contiguous in memory are required")
        rows, cols = t.shape[-2:]
        ld = t.stride(-2) if rows > 1 else max(t.stride(-2), cols)
        count = t.shape[0] if t.dim() == 3 else 1
        return count, rows, cols, ld, t.stride(0) if t.dim() == 3 else rows * ld

    count, rows, cols, ld_g, each_g = stack(g, _DTYPES)
    if out is None:
        out = torch.empty(g.shape, dtype=torch.bfloat16, device=g.device)
    elif out.shape != g.shape:
        raise ValueError(f"{what}: out must have g's shape")
    _, _, _, ld_out, each_out = stack(out, (torch.bfloat16,))
    a, b, c = coefficients
    ws = _workspace(lib.tppo_orthogonalize_workspace_bytes(count, rows, cols), g.device) if workspace is None else workspace
    _same_device(what, g, out, ws)
    with torch.cuda.device(g.device):
        rc = lib.tppo_orthogonalize(_ptr(g), count, rows, cols, ld_g, each_g, _DTYPES[g.dtype], int(steps), float(a), float(b),
                                    float(c), float(eps), float(scale), _ptr(out), ld_out, each_out, _ptr(ws),
                                    ws.numel() * ws.element_size(), _stream())
    _check(rc, what)
    return out


class Batcher:
    """Successive-batching slot bookkeeping (host side, numpy int32 arrays in and out)."""

    def __init__(self, slots, window, max_response):
        self._lib = load()
        self.slots = int(slots)
        self._h = self._lib.tppo_batcher_create(self.slots, int(window), int(max_response))
        if not self._h:
            raise ValueError("tppo_batcher_create: bad sizes")

    def close(self):
        if self._h:
            self._lib.tppo_batcher_destroy(self._h)
            self._h = None

    __del__ = close

    @staticmethod
    def _i32(a):
        import numpy as np
        return np.ascontiguousarray(a, dtype=np.int32)

    def refill(self, prompt_len):
        p = self._i32(prompt_len)
        taken = ctypes.c_int64(0)
        _check(self._lib.tppo_batcher_refill(self._h, p.ctypes.data, p.size, ctypes.byref(taken)),
               "tppo_batcher_refill")
        return taken.value

    def advance(self, gen_len, eos):
        g, e = self._i32(gen_len), self._i32(eos)
        assert g.size == self.slots and e.size == self.slots
        _check(self._lib.tppo_batcher_advance(self._h, g.ctypes.data, e.ctypes.data), "tppo_batcher_advance")

    def layout(self):
        import numpy as np
        cu = np.empty(self.slots + 1, np.int32)
        ctx, prompt, done = (np.empty(self.slots, np.int32) for _ in range(3))
        ids = np.empty(self.slots, np.int64)
        _check(self._lib.tppo_batcher_layout(self._h, cu.ctypes.data, ctx.ctypes.data, prompt.ctypes.data,
                                             done.ctypes.data, ids.ctypes.data), "tppo_batcher_layout")
        return cu, ctx, prompt, done, ids


class LossStats(ctypes.Structure):
    _fields_ = [("ratio_mean", ctypes.c_float), ("policy_clip_frac", ctypes.c_float),
                ("value_clip_frac", ctypes.c_float), ("reserved", ctypes.c_float),
                ("n_policy_clipped", ctypes.c_int64), ("n_value_clipped", ctypes.c_int64)]


def tppo_ppo_losses_backward(logp_new, logp_old, adv, v_new, v_old, ret, resp_off, keep_len, done,
                             eps_low, eps_high, xi_low, xi_high, policy_scale=1.0, value_scale=1.0,
                             policy_denominator=0, value_denominator=0, status=None, workspace=None,
                             out=None, stats=None, grads=None, plan=None):
    """Derivatives of the two losses (plus the losses and clip statistics) in one
    pass.  Returns (grad_logp, grad_v, loss_out tensor, stats tensor)."""
    lib = load()
    dev = resp_off.device
    B = done.numel()
    n_resp = (logp_new if logp_new is not None else v_new).numel()
    if grads is None:
        g_lp = torch.empty(n_resp, dtype=torch.float32, device=dev) if logp_new is not None else None
        g_v = torch.empty(n_resp, dtype=torch.float32, device=dev) if v_new is not None else None
    else:
        g_lp, g_v = grads
    res = torch.empty(ctypes.sizeof(LossOut), dtype=torch.uint8, device=dev) if out is None else out
    st = torch.empty(ctypes.sizeof(LossStats), dtype=torch.uint8, device=dev) if stats is None else stats
    ws = _scratch(lib.tppo_ppo_losses_backward_workspace_bytes, n_resp, B, workspace, plan, dev)
    rc = _native().ppo_losses_backward(
        logp_new, logp_old, adv, v_new, v_old, ret, resp_off, keep_len, done, B, n_resp, float(eps_low), float(eps_high),
        float(xi_low), float(xi_high), float(policy_scale), float(value_scale), int(policy_denominator),
        int(value_denominator), g_lp, g_v, res, st, ws, plan, status, _stream())
    _check(rc, "tppo_ppo_losses_backward")
    return g_lp, g_v, res, st


def read_loss_stats(st):
    """Device ``tppo_loss_stats`` -> dict (synchronises)."""
    s = LossStats.from_buffer_copy(bytes(st.cpu().numpy().tobytes()))
    return {name: getattr(s, name) for name, _ in LossStats._fields_ if name != "reserved"}


def tppo_diag_mfma_rate(operands, out, iters):
    """Launch the register-resident MFMA loop; returns the flop count of the launch."""
    lib = load()
    flop = ctypes.c_double(0.0)
    rc = lib.tppo_diag_mfma_rate(_ptr(operands), _ptr(out), int(iters), ctypes.byref(flop), _stream())
    _check(rc, "tppo_diag_mfma_rate")
    return flop.value


def tppo_diag_streams(src, dst, bytes_per_stream, stride_bytes, n_read, n_write):
    """Elementwise pass over n_read input and n_write output streams; returns the bytes moved."""
    lib = load()
    _check(lib.tppo_diag_streams(_ptr(src), _ptr(dst), int(bytes_per_stream), int(stride_bytes), int(n_read),
                                 int(n_write), _stream()), "tppo_diag_streams")
    return int(bytes_per_stream) * (n_read + n_write)
