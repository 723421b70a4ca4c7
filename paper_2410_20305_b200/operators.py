"""Calls of the operators that complete a training step on the shared layout, beside those of binding.py and in its manner:
log-probabilities straight from the hidden states (for dpo_logp, whose logits are stored), rotary positions in their
various forms (for psa_rope, which has one), and the norms around a block whose output is normalised or gated before it joins the
residual stream (for psa_norm, which adds it as it is)."""
from __future__ import annotations

import ctypes as C

from . import binding as B


def _want_linear_logp(hidden, table, targets, segment_ids, forks):
    """(n_rows, vocab, width, number of forks), the checked operands, and the fork arrays as they are handed over."""
    import torch
    if hidden.dim() != 2 or table.dim() != 2:
        raise ValueError("hidden: [rows, width], table: [vocab, width]")
    (n_rows, D), V = hidden.shape, table.shape[0]
    given = [("hidden", hidden, (n_rows, D), torch.bfloat16), ("table", table, (V, D), torch.bfloat16),
             ("targets", targets, (n_rows,), torch.int32), ("segment_ids", segment_ids, (n_rows,), torch.int32)]
    missing = [t is None for t in forks]
    if any(missing) and not all(missing):
        raise ValueError("fork_rows, fork_targets and fork_segments go together")
    n_forks = 0 if missing[0] else forks[0].numel()
    if n_forks:
        given += [(name, t, (n_forks,), torch.int32) for name, t in zip(("fork_rows", "fork_targets", "fork_segments"), forks)]
    else:
        forks = (None, None, None)
    return n_rows, V, D, n_forks, given, forks


def dpo_linear_logp(hidden, table, targets, segment_ids, n_segments, fork_rows=None, fork_targets=None, fork_segments=None,
                    scale=1.0, out=None, lse=None, workspace=None, status=None, stream=None):
    """dpo_logp of the logits scale * hidden @ table.T, which are never stored: hidden [n_rows, width] and table [vocab, width]
    bf16 (width a multiple of 8), labels as dpo_logp takes them.  Returns (out fp32 [n_segments], lse fp32 [n_rows]); lse is
    what dpo_linear_logp_bwd needs: log sum exp of the logits of every row that scores a label, 0 of the others."""
    fast = B._fast(stream) if out is None and lse is None else None
    if fast:
        got = fast.linear_logp(hidden, table, targets, segment_ids, fork_rows, fork_targets, fork_segments, n_segments, float(scale),
                               workspace, status)
        if type(got) is tuple:
            return got
        if got is not None:
            B._check("dpo_linear_logp", got)
    import torch
    n_rows, V, D, n_forks, given, forks = _want_linear_logp(hidden, table, targets, segment_ids,
                                                           (fork_rows, fork_targets, fork_segments))
    n_segments = int(n_segments)
    B._want_given(given)
    B._want_status_here(status)
    B._want_widths("dpo_linear_logp", D, n_forks, n_segments)
    if n_segments < 0:
        raise ValueError("n_segments: %d" % n_segments)
    new = lambda n: B._result(hidden, stream, lambda: torch.empty(n, dtype=torch.float32, device=hidden.device))  # noqa: E731
    out, lse = new(n_segments) if out is None else out, new(n_rows) if lse is None else lse
    outputs = [("out", out, (n_segments,), torch.float32), ("lse", lse, (n_rows,), torch.float32)]
    B._want_given(outputs)
    B._want_apart([(n, t) for n, t, _, _ in outputs], [(n, t) for n, t, _, _ in given])
    lib = B.load_library()
    need = lib.dpo_linear_logp_workspace_bytes(n_rows, n_forks, n_segments, V, D, 0)
    workspace = B._scratch(workspace, need, hidden, stream)
    B._check("dpo_linear_logp", lib.dpo_linear_logp(B._ptr(hidden), B._ptr(table), n_rows, V, D, float(scale), B._ptr(targets), B._ptr(segment_ids),
                                                  *map(B._ptr, forks), n_forks, n_segments, B._ptr(out), B._ptr(lse), B._ptr(workspace),
                                                  B._ptr(status), B._stream(stream)))
    return out, lse


def dpo_linear_logp_bwd(coef, hidden, table, lse, targets, segment_ids, fork_rows=None, fork_targets=None, fork_segments=None,
                        scale=1.0, with_table=True, d_hidden=None, d_table=None, workspace=None, status=None, stream=None):
    """Gradient of sum_g coef[g] * dpo_linear_logp(...)[0][g] for coef fp32 [n_segments]; lse as dpo_linear_logp returned it.
    Returns (d_hidden [n_rows, width], d_table [vocab, width]), bf16; with_table=False leaves d_table out (None), for a table
    that is not trained."""
    fast = B._fast(stream) if d_hidden is None and d_table is None else None
    if fast:
        got = fast.linear_logp_bwd(coef, hidden, table, lse, targets, segment_ids, fork_rows, fork_targets, fork_segments, float(scale),
                                   with_table, workspace, status)
        if type(got) is tuple:
            return got
        if got is not None:
            B._check("dpo_linear_logp_bwd", got)
    import torch
    n_rows, V, D, n_forks, given, forks = _want_linear_logp(hidden, table, targets, segment_ids,
                                                           (fork_rows, fork_targets, fork_segments))
    if coef.dim() != 1:
        raise ValueError("coef: [n_segments]")
    n_segments = coef.shape[0]
    given += [("coef", coef, (n_segments,), torch.float32), ("lse", lse, (n_rows,), torch.float32)]
    B._want_given(given)
    B._want_status_here(status)
    B._want_widths("dpo_linear_logp_bwd", D, n_forks, n_segments)
    d_hidden = B._result(hidden, stream) if d_hidden is None else d_hidden
    outputs = [("d_hidden", d_hidden, (n_rows, D), torch.bfloat16)]
    if with_table:
        d_table = B._result(table, stream) if d_table is None else d_table
        outputs.append(("d_table", d_table, (V, D), torch.bfloat16))
    elif d_table is not None:
        raise ValueError("d_table: not written with with_table=False")
    B._want_given(outputs)
    B._want_apart([(n, t) for n, t, _, _ in outputs], [(n, t) for n, t, _, _ in given])
    lib = B.load_library()
    need = lib.dpo_linear_logp_workspace_bytes(n_rows, n_forks, n_segments, V, D, 1)
    workspace = B._scratch(workspace, need, hidden, stream)
    B._check("dpo_linear_logp_bwd", lib.dpo_linear_logp_bwd(
        B._ptr(coef), B._ptr(hidden), B._ptr(table), B._ptr(lse), n_rows, V, D, float(scale), B._ptr(targets), B._ptr(segment_ids), *map(B._ptr, forks),
        n_forks, n_segments, B._ptr(d_hidden), B._ptr(d_table), B._ptr(workspace), B._ptr(status), B._stream(stream)))
    return d_hidden, d_table


ROTARY_SCALINGS = {None: 0, "linear": 1, "base": 2, "wavelength": 3, "ramp": 4}


def psa_rotary_frequencies(rotary_dim, theta=10000.0, scaling=None, factor=1.0, original_length=0, low=1.0, high=None, device=None):
    """The table of frequencies for psa_rotary: (turns int64 [rotary_dim / 2], on `device` where one is named, and the factor
    `magnitude` of the rotated part).  `scaling` for contexts longer than original_length: None, "linear" (positions divided by
    factor), "base" (theta raised), "wavelength" (frequencies divided by factor where a pair turns fewer than `low` times over the
    original length, kept from `high` times on, 4 where it is not given), or "ramp" (the same along the pairs' numbers, `high` 32,
    with a magnitude that grows with factor)."""
    import torch
    if scaling not in ROTARY_SCALINGS:
        raise ValueError("scaling: %r, one of %s is needed" % (scaling, ", ".join(map(repr, ROTARY_SCALINGS))))
    if not 0 < rotary_dim <= 0x7fffffff:
        raise ValueError("rotary_dim: %d" % rotary_dim)
    if high is None:
        high = 32.0 if scaling == "ramp" else 4.0
    turns, magnitude = torch.empty(max(int(rotary_dim) // 2, 1), dtype=torch.int64), C.c_float()
    B._check("psa_rotary_frequencies", B.load_library().psa_rotary_frequencies(
        int(rotary_dim), float(theta), ROTARY_SCALINGS[scaling], float(factor), float(original_length), float(low), float(high),
        turns.data_ptr(), C.byref(magnitude)))
    return (turns if device is None else turns.to(device)), magnitude.value


def _extent(t):
    """First byte and the one behind the last of a strided tensor (strides are not negative)."""
    size = t.element_size()
    last = sum((n - 1) * s for n, s in zip(t.shape, t.stride())) if t.numel() else -1
    return t.data_ptr(), t.data_ptr() + (last + 1) * size


def _disjoint(a, b):
    """Whether two [tokens, heads, head_dim] views share no element: their extents lie apart, or tokens are equally far from one
    another in both and the parts of a token do not meet."""
    (a0, a1), (b0, b1) = _extent(a), _extent(b)
    if a1 <= b0 or b1 <= a0:
        return True
    size, pitch = a.element_size(), a.stride(0) * a.element_size()
    if a.element_size() != b.element_size() or a.stride(0) != b.stride(0) or pitch <= 0:
        return False
    part = lambda t: ((t.shape[1] - 1) * t.stride(1) + t.shape[2]) * size  # noqa: E731
    ahead = (b0 - a0) % pitch
    return part(a) <= ahead and ahead + part(b) <= pitch


def _want_heads(name, t, shape, dtype):
    """Raises ValueError unless `t` is a CUDA tensor of this shape and type whose heads' elements are neighbours."""
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError("%s: %s %s, %s %s is needed" % (name, tuple(t.shape), t.dtype, tuple(shape), dtype))
    if t.numel() and (t.stride(2) != 1 and t.shape[2] > 1):
        raise ValueError("%s: the elements of a head have to be neighbours" % name)
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % name)


def _same_place(a, b):
    return a.data_ptr() == b.data_ptr() and a.stride()[:2] == b.stride()[:2] and a.shape == b.shape


def psa_rotary(q, k, position_ids, turns, magnitude=1.0, interleaved=False, inverse=False, q_out=None, k_out=None, stream=None):
    """Rotary embedding of q [T, Hq, d] and k [T, Hkv, d] (or None), bf16 or fp32, in one launch; views of any token and head
    stride.  turns, magnitude: as psa_rotary_frequencies gave them (turns on the device; its length says how much of a head
    is turned); position_ids int32 [T].  interleaved: pairs are neighbours, else halves of the rotated part.  inverse=True is the
    gradient of the call without it.  Returns (q_out, k_out), contiguous unless given; q_out may be q, k_out may be k."""
    fast = B._fast(stream) if q_out is None and k_out is None else None
    if fast:
        got = fast.rotary(q, k, position_ids, turns, float(magnitude), interleaved, inverse)
        if type(got) is tuple:
            return got
        if got is not None:
            B._check("psa_rotary", got)
    import torch
    if q.dim() != 3 or (k is not None and k.dim() != 3) or turns.dim() != 1:
        raise ValueError("q, k: [tokens, heads, head_dim], turns: [rotary_dim / 2]")
    dtype = B._dtype_code(q, "q")
    T, Hq, d = q.shape
    Hk = 0 if k is None else k.shape[1]
    _want_heads("q", q, (T, Hq, d), q.dtype)
    ins = [("q", q)]
    if k is None:
        if k_out is not None:
            raise ValueError("k_out: there is none without k")
    else:
        _want_heads("k", k, (T, Hk, d), q.dtype)
        ins.append(("k", k))
    B._want_given([("position_ids", position_ids, (T,), torch.int32), ("turns", turns, (turns.shape[0],), torch.int64)])
    here = torch.device("cuda", torch.cuda.current_device()) if q.device.type == "cuda" else q.device
    rotary_dim = 2 * turns.shape[0]
    if rotary_dim > d:
        raise ValueError("turns: %d pairs, a head has %d elements" % (turns.shape[0], d))
    B._want_widths("psa_rotary", Hq, Hk, d)
    new = lambda t: B._result(t, stream, lambda: torch.empty(t.shape, dtype=t.dtype, device=t.device))  # noqa: E731
    q_out = new(q) if q_out is None else q_out
    outs = [("q_out", q_out)]
    _want_heads("q_out", q_out, (T, Hq, d), q.dtype)
    if k is not None:
        k_out = new(k) if k_out is None else k_out
        _want_heads("k_out", k_out, (T, Hk, d), q.dtype)
        outs.append(("k_out", k_out))
    for name, t in ins + outs:
        if t.device.type == "cuda" and t.device != here or t.device != q.device:
            raise ValueError("%s: on %s, all have to be on the current device" % (name, t.device))
    for i, (name, t) in enumerate(outs):
        room = d
        for s, n in sorted((s, n) for s, n in zip(t.stride(), t.shape[:2]) if n > 1):
            if s < room:
                raise ValueError("%s: its heads share memory" % name)
            room += s * (n - 1)
        source = ins[i][1]
        for other, u in ins + outs[i + 1:]:
            if u is source and _same_place(t, u):
                continue
            if t.numel() and u.numel() and not _disjoint(t, u):
                raise ValueError("%s and %s share memory" % (name, other))
        for other, u in (("position_ids", position_ids), ("turns", turns)):
            (a0, a1), (b0, b1) = _extent(t), _extent(u)
            if a0 < b1 and b0 < a1:
                raise ValueError("%s and %s share memory" % (name, other))
    strides = [s for x, y in ((q, q_out), (k, k_out)) if x is not None for s in (*x.stride()[:2], *y.stride()[:2])]
    strides += [0] * (8 - len(strides))
    B._check("psa_rotary", B.load_library().psa_rotary(B._ptr(q), B._ptr(k), B._ptr(q_out), B._ptr(k_out), B._ptr(position_ids), B._ptr(turns), dtype, T, Hq,
                                                   Hk, d, rotary_dim, (C.c_int64 * 8)(*strides), 1 if interleaved else 0,
                                                   1 if inverse else 0, float(magnitude), B._stream(stream)))
    return q_out, k_out


def _want_block(x, weight, bias, post_weight, post_bias, gate, rms):
    """(n_tokens, hidden, type of x, type of weight, parameters as (name, tensor, shape, dtype)) of a block's norms."""
    T, D, dtype, wtype = B._want_norm(x, weight, "x")
    if rms and (bias is not None or post_bias is not None):
        raise ValueError("bias, post_bias: the root-mean-square form has none")
    if post_bias is not None and post_weight is None:
        raise ValueError("post_bias: there is none without post_weight")
    params = [(name, t, (D,), weight.dtype) for name, t in (("weight", weight), ("bias", bias), ("post_weight", post_weight),
                                                            ("post_bias", post_bias), ("gate", gate)) if t is not None]
    return T, D, dtype, wtype, params


def psa_block_norm(x, residual, weight, bias=None, post_weight=None, post_bias=None, gate=None, residual_scale=1.0, eps=1e-5,
                   rms=False, out=None, total=None, stats=None, stream=None):
    """The step between two sublayers whose output x [T, hidden] is normalised (post_weight, post_bias [hidden]) or scaled by
    a gate [hidden], or both, before it joins the residual stream [T, hidden]:
        total = residual_scale * residual + gate * (norm(x) * post_weight + post_bias),   out = norm(total) * weight + bias
    with what is None left out; layer norms, or with rms=True the root-mean-square form (without biases).  x in bf16 or fp32,
    parameters in x's type or fp32.  Returns (out, total, stats); stats, fp32 [4, T], is what psa_block_norm_bwd needs.  out and
    total may be x or residual."""
    fast = B._fast(stream) if out is None and total is None and stats is None else None
    if fast:
        got = fast.block_norm(x, residual, weight, bias, post_weight, post_bias, gate, float(residual_scale), float(eps), rms)
        if type(got) is tuple:
            return got
        if got is not None:
            B._check("psa_block_norm", got)
    import torch
    T, D, dtype, wtype, params = _want_block(x, weight, bias, post_weight, post_bias, gate, rms)
    if residual is None:
        raise ValueError("residual: needed")
    given = [("x", x, (T, D), x.dtype), ("residual", residual, (T, D), x.dtype)] + params
    B._want_given(given)
    B._want_widths("psa_block_norm", D)
    out, total = B._result(x, stream) if out is None else out, B._result(x, stream) if total is None else total
    if stats is None:
        stats = B._result(x, stream, lambda: torch.empty((4, T), dtype=torch.float32, device=x.device))
    outputs = [("out", out, (T, D), x.dtype), ("total", total, (T, D), x.dtype), ("stats", stats, (4, T), torch.float32)]
    B._want_given(outputs)
    B._want_in_place([(n, t) for n, t, _, _ in outputs], [(n, t) for n, t, _, _ in given], {"out": ("x", "residual"),
                                                                                      "total": ("x", "residual")})
    B._check("psa_block_norm", B.load_library().psa_block_norm(
        B._ptr(x), B._ptr(residual), B._ptr(weight), B._ptr(bias), B._ptr(post_weight), B._ptr(post_bias), B._ptr(gate), float(residual_scale), dtype,
        wtype, T, D, float(eps), 1 if rms else 0, B._ptr(out), B._ptr(total), B._ptr(stats), B._stream(stream)))
    return out, total, stats


def psa_block_norm_bwd(d_out, x, total, weight, stats, post_weight=None, post_bias=None, gate=None, residual_scale=1.0, rms=False,
                       d_total=None, with_bias=False, dx=None, d_residual=None, workspace=None, status=None, stream=None):
    """Gradient of psa_block_norm for d_out and, if given, d_total, the gradient that reaches the sum by the residual stream.
    Returns (dx, d_residual, d_weight, d_bias, d_post_weight, d_post_bias, d_gate), None for parameters that the forward pass
    had not (d_bias: unless with_bias).  dx and d_residual may be d_out, total or d_total, dx may be x."""
    fast = B._fast(stream) if dx is None and d_residual is None else None
    if fast:
        got = fast.block_norm_bwd(d_out, x, total, weight, None, post_weight, post_bias, gate, stats, float(residual_scale), rms, d_total,
                                  with_bias, workspace, status)
        if type(got) is tuple:
            return got
        if got is not None:
            B._check("psa_block_norm_bwd", got)
    import torch
    T, D, dtype, wtype, params = _want_block(x, weight, None, post_weight, post_bias, gate, rms)
    if rms and with_bias:
        raise ValueError("d_bias: the root-mean-square form has none")
    given = [("d_out", d_out, (T, D), x.dtype), ("x", x, (T, D), x.dtype), ("total", total, (T, D), x.dtype),
             ("stats", stats, (4, T), torch.float32)] + params
    if d_total is not None:
        given.append(("d_total", d_total, (T, D), x.dtype))
    B._want_given(given)
    B._want_status_here(status)
    B._want_widths("psa_block_norm_bwd", D)
    dx, d_residual = B._result(x, stream) if dx is None else dx, B._result(x, stream) if d_residual is None else d_residual
    outputs = [("dx", dx, (T, D), x.dtype), ("d_residual", d_residual, (T, D), x.dtype)]
    B._want_given(outputs)
    B._want_in_place([(n, t) for n, t, _, _ in outputs], [(n, t) for n, t, _, _ in given],
                   {"dx": ("d_out", "x", "total", "d_total"), "d_residual": ("d_out", "total", "d_total")})
    grads = [B._result(weight, stream) if there else None
             for there in (True, with_bias, post_weight is not None, post_bias is not None, gate is not None)]
    lib = B.load_library()
    need = lib.psa_block_norm_bwd_workspace_bytes(T, D)
    workspace = B._scratch(workspace, need, x, stream)
    B._check("psa_block_norm_bwd", lib.psa_block_norm_bwd(
        B._ptr(d_out), B._ptr(x), B._ptr(total), B._ptr(weight), B._ptr(post_weight), B._ptr(post_bias), B._ptr(gate), float(residual_scale), B._ptr(stats),
        B._ptr(d_total), dtype, wtype, T, D, 1 if rms else 0, B._ptr(dx), B._ptr(d_residual), *map(B._ptr, grads), B._ptr(workspace), B._ptr(status),
        B._stream(stream)))
    return (dx, d_residual, *grads)
