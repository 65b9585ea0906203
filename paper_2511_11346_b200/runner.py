"""Moves a synthetic workload onto the device and drives the head through the C-ABI binding.
Used by the GPU tests, the smoke check and the benchmark; holds no arithmetic of the method."""
from __future__ import annotations

import numpy as np

from . import binding as B
from . import inputs as I


def to_device_bf16(x_q: np.ndarray, device="cuda"):
    """fp32 array of bf16-representable values -> torch.bfloat16 tensor with the same bit patterns."""
    import torch
    return torch.from_numpy(I.bf16_bits(x_q).view(np.int16)).to(device).view(torch.bfloat16).reshape(x_q.shape)


def to_host_bf16(x_q: np.ndarray, pinned: bool = True):
    import torch
    t = torch.from_numpy(I.bf16_bits(x_q).view(np.int16)).view(torch.bfloat16).reshape(x_q.shape)
    return t.pin_memory() if pinned else t


def lowrank_compose(W_base, lora_A, lora_B):
    """Device bf16 tensors W_base [n, v, d], lora_A [n, r, v, k], lora_B [n, r, k, d] -> composed W_emit [n, r, v, d] (bf16)."""
    import torch
    n, r, v, k = lora_A.shape
    d = lora_B.shape[-1]
    out = torch.empty((n, r, v, d), dtype=torch.bfloat16, device=lora_A.device)
    B.mtpc_lowrank_compose(n, r, v, d, k, W_base.data_ptr(), lora_A.data_ptr(), lora_B.data_ptr(), out.data_ptr(),
                           torch.cuda.current_stream().cuda_stream)
    return out


def lowrank_backward(lora_A, lora_B, dW_emit):
    """Device tensors lora_A, lora_B (bf16) and dW_emit [n, r, v, d] (fp32) -> (dW_base, dA, dB) as fp32 device tensors."""
    import torch
    n, r, v, k = lora_A.shape
    d = lora_B.shape[-1]
    f32 = dict(dtype=torch.float32, device=lora_A.device)
    dW, dA, dB = torch.empty((n, v, d), **f32), torch.empty((n, r, v, k), **f32), torch.empty((n, r, k, d), **f32)
    B.mtpc_lowrank_backward(n, r, v, d, k, lora_A.data_ptr(), lora_B.data_ptr(), dW_emit.data_ptr(), dW.data_ptr(),
                            dA.data_ptr(), dB.data_ptr(), torch.cuda.current_stream().cuda_stream)
    return dW, dA, dB


def embed(tokens, table, scale: float = 1.0, dtype=None):
    """Device tensors tokens [T] int32 (negative: padding) and table [v, d] (fp32 or bf16) -> rows scale * table[token] [T, d]
    (dtype: the table's)."""
    import torch
    out = torch.empty((tokens.shape[0], table.shape[1]), dtype=dtype or table.dtype, device=table.device)
    B.mtpc_embed(tokens, table, out, scale=scale)
    return out


def embed_backward(tokens, d_out, v: int, scale: float = 1.0, into=None):
    """Gradient of `embed` with respect to the table [v, d] (fp32). into: added to that tensor (a table tied to the unembeddings: the gradient
    dW_base[0] of a factored head)."""
    import torch
    d_table = torch.empty((v, d_out.shape[1]), dtype=torch.float32, device=d_out.device) if into is None else into
    B.mtpc_embed_backward(tokens, d_out, d_table, scale=scale, accumulate=into is not None)
    return d_table


def residual_rmsnorm(x, residual, weight, eps: float = 1e-5):
    """Device tensors x, residual (or None) [T, d] -> (hidden states, x + residual): the residual stream's last addition and the norm whose output a
    head reads."""
    import torch
    hidden, total = torch.empty_like(x), torch.empty_like(x)
    B.mtpc_residual_rmsnorm(x, residual, weight, eps, hidden, out_sum=total)
    return hidden, total


def residual_rmsnorm_backward(total, weight, d_hidden, d_total=None, eps: float = 1e-5, dtype=None):
    """-> (gradient of x and of residual [T, d] (dtype: total's), gradient of weight [d] fp32) from the head's d_hidden and what reaches the sum along
    the residual stream."""
    import torch
    d_x = torch.empty(total.shape, dtype=dtype or total.dtype, device=total.device)
    d_weight = torch.empty(total.shape[1], dtype=torch.float32, device=total.device)
    B.mtpc_residual_rmsnorm_backward(total, weight, eps, d_hidden, d_total, d_x, d_weight)
    return d_x, d_weight


def adapted_projection(x, W, A, B_, scale=None, row_adaptor=None, x_low=None, keep_low=True, out_status=None):
    """Device bf16 tensors x [T, d], W [m, d] and the adaptors' factors A [S, m, k], B_ [S, k, d] -> (out [T, m], low [T, k] fp32 or None): W x and, for rows
    with an adaptor, A low, low = scale B_ x (or B_ x_low). out_status: int32 [1], into which the status bits are or-ed (a wait that expired shows nowhere else)."""
    import torch
    out = torch.empty((x.shape[0], W.shape[0]), dtype=x.dtype, device=x.device)
    low = torch.empty((x.shape[0], A.shape[2]), dtype=torch.float32, device=x.device) if keep_low else None
    B.mtpc_adapted_projection(x, W, A, B_, scale, row_adaptor, out, out_low=low, x_low=x_low, out_status=out_status)
    return out, low


def adapted_projection_backward(x, W, A, B_, low, d_out, scale=None, row_adaptor=None, x_low=None, out_status=None):
    """-> dict(d_x, dA, dB, d_x_low): gradients of adapted_projection from d_out [T, m] bf16; with x_low, d_x_low is its gradient (None otherwise).
    out_status as above."""
    import torch
    f32 = dict(dtype=torch.float32, device=x.device)
    out = dict(d_x=torch.empty(x.shape, dtype=x.dtype, device=x.device), dA=torch.empty(A.shape, **f32), dB=torch.empty(B_.shape, **f32),
               d_x_low=None if x_low is None else torch.empty(x.shape, dtype=x.dtype, device=x.device))
    B.mtpc_adapted_projection_backward(x if x_low is None else x_low, W, A, B_, scale, row_adaptor, low, d_out, out["d_x"], out["dA"], out["dB"],
                                       d_x_low=out["d_x_low"], out_status=out_status)
    return out


def dropout(x, p: float, rng, offset: int = 0, residual=None, dtype=None):
    """Device tensors x, residual (or None) [T, d] -> residual + dropout of x (dtype: the residual's, or x's). On the gradient of that, without residual:
    the gradient of x, while rng [2] int64 (seed, step) holds the same values."""
    import torch
    out = torch.empty(x.shape, dtype=dtype or (x if residual is None else residual).dtype, device=x.device)
    B.mtpc_dropout(x, out, p, rng, offset=offset, residual=residual)
    return out


def policy_loss(logp, old_logp, ref_logp, advantage, offsets, clip_low: float = 0.2, clip_high: float = 0.2, beta: float = 0.0, mask=None, by_sequence=False,
                by_position=False):
    """-> dict(loss [1], stats [3], d_logp [T]) of packed sequences; d_logp is the `weight` of DeviceHead.window_logprob_backward."""
    import torch
    f32 = dict(dtype=torch.float32, device=logp.device)
    out = dict(loss=torch.empty(1, **f32), stats=torch.empty(3, **f32), d_logp=torch.zeros(logp.shape, **f32))
    B.mtpc_policy_loss(logp, old_logp, ref_logp, advantage, offsets, clip_low, clip_high, beta, out["loss"], out["d_logp"], mask=mask,
                       by_sequence=by_sequence, by_position=by_position, out_stats=out["stats"])
    return out


def preference_loss(logp, ref_logp, offsets, beta: float = 0.1, smoothing: float = 0.0, mask=None):
    """-> dict(loss [1], h [S / 2], d_logp [T]) of packed pairs of sequences; d_logp as for policy_loss."""
    import torch
    f32 = dict(dtype=torch.float32, device=logp.device)
    out = dict(loss=torch.empty(1, **f32), h=torch.empty((offsets.numel() - 1) // 2, **f32), d_logp=torch.zeros(logp.shape, **f32))
    B.mtpc_preference_loss(logp, ref_logp, offsets, beta, out["loss"], out["d_logp"], mask=mask, smoothing=smoothing, out_h=out["h"])
    return out


def _written_again(what, shapes, device, out):
    """The dict of an earlier call, if its tensors are what the call writes: adjacent fp32 elements of these shapes (None: absent) on that device."""
    import torch
    for key, shape in shapes.items():
        t = out.get(key)
        if shape is None and t is None:
            continue
        if (not isinstance(t, torch.Tensor) or shape is None or t.shape != shape or t.dtype is not torch.float32 or t.device != device or
                not t.is_contiguous()):
            is_now = f"{t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}" if isinstance(t, torch.Tensor) else repr(t)
            raise B.MtpcError(B.ERR_SHAPE, f"{what}: out[{key!r}] is {is_now} where fp32 {shape} on {device} is written")
    return out


class DeviceHead:
    """Weights of a workload resident in HBM plus a head created on them."""

    def __init__(self, wl: I.Workload, max_positions: int | None = None, max_wpp: int | None = None, device="cuda",
                 lowrank=None):
        """lowrank = (W_base, A, B) as fp32 arrays of bf16-representable values: a head that keeps the shared
        unembeddings factored (wl.W_emit_q is then not uploaded)."""
        import torch
        s = wl.shape
        self.wl = wl
        self.device = device
        self.lowrank = None
        if lowrank is not None:
            self.lowrank = tuple(to_device_bf16(np.ascontiguousarray(x), device) for x in lowrank)
            self.W_emit = None
            self.W_sum = to_device_bf16(wl.W_sum_q, device)
        elif s.io_dtype == I.F32:
            self.W_emit = torch.from_numpy(wl.W_emit_raw).to(device)
            self.W_sum = torch.from_numpy(wl.W_sum_raw).to(device)
        else:
            self.W_emit = to_device_bf16(wl.W_emit_q if wl.W_emit_dev_q is None else wl.W_emit_dev_q, device)
            self.W_sum = to_device_bf16(wl.W_sum_q, device)
        self.T_static = torch.from_numpy(np.ascontiguousarray(wl.T_static)).to(device) if wl.T_static is not None else None
        ctx = s.family == I.HMM_CTX
        self.head = B.MtpcHead(B.MTPC_HMM if ctx else s.family, s.n, s.r, s.v, s.d, s.io_dtype,
                               max_positions or max(wl.T, 1), max_wpp or max(wl.wpp, 1), self.W_emit, self.W_sum,
                               self.T_static, flags=B.MTPC_FLAG_HMM_CONTEXTUAL if ctx else 0, v_valid=s.v_valid,
                               lowrank=self.lowrank)

    def hidden_device(self, rows=None):
        import torch
        wl = self.wl
        sl = slice(None) if rows is None else rows
        if wl.shape.io_dtype == I.F32:
            return torch.from_numpy(np.ascontiguousarray(wl.hidden_raw[sl])).to(self.device)
        return to_device_bf16(np.ascontiguousarray(wl.hidden_q[sl]), self.device)

    def hidden_host(self, rows=None):
        import torch
        wl = self.wl
        sl = slice(None) if rows is None else rows
        if wl.shape.io_dtype == I.F32:
            return torch.from_numpy(np.ascontiguousarray(wl.hidden_raw[sl])).pin_memory()
        return to_host_bf16(np.ascontiguousarray(wl.hidden_q[sl]))

    def window_logprob(self, hidden=None, targets=None):
        """Device-buffer call on the workload's own hidden states / targets (or the given device tensors)."""
        import torch
        h = self.hidden_device() if hidden is None else hidden
        t = torch.from_numpy(self.wl.targets).to(self.device) if targets is None else targets
        out = torch.empty(h.shape[0], dtype=torch.float32, device=self.device)
        self.head.mtpc_window_logprob(h, t, out)
        return out

    def draft_sample(self, wpp=None, hidden=None, uniforms=None):
        import torch
        wpp = wpp or self.wl.wpp
        h = self.hidden_device() if hidden is None else hidden
        u = torch.from_numpy(self.wl.uniforms).to(self.device) if uniforms is None else uniforms
        W = h.shape[0] * wpp
        out_bytes = torch.empty((W, self.wl.shape.n), dtype=torch.int32, device=self.device)
        out_lp = torch.empty(W, dtype=torch.float32, device=self.device)
        self.head.mtpc_draft_sample(h, wpp, u, out_bytes, out_lp)
        return out_bytes, out_lp

    def window_prefix_logprob(self, hidden=None, targets=None):
        import torch
        h = self.hidden_device() if hidden is None else hidden
        t = torch.from_numpy(self.wl.targets).to(self.device) if targets is None else targets
        out = torch.empty((h.shape[0], self.wl.shape.n), dtype=torch.float32, device=self.device)
        self.head.mtpc_window_prefix_logprob(h, t, out)
        return out

    def draft_sample_prefix(self, wpp=None, hidden=None, uniforms=None):
        import torch
        wpp = wpp or self.wl.wpp
        h = self.hidden_device() if hidden is None else hidden
        u = torch.from_numpy(self.wl.uniforms).to(self.device) if uniforms is None else uniforms
        W = h.shape[0] * wpp
        out_bytes = torch.empty((W, self.wl.shape.n), dtype=torch.int32, device=self.device)
        out_prefix = torch.empty((W, self.wl.shape.n), dtype=torch.float32, device=self.device)
        self.head.mtpc_draft_sample_prefix(h, wpp, u, out_bytes, out_prefix)
        return out_bytes, out_prefix

    def speculative_accept(self, P, wpp, draft_bytes, prefix_logprob, target_probs, accept_uniforms):
        import torch
        W = P * wpp
        accepted = torch.empty(W, dtype=torch.int32, device=self.device)
        next_byte = torch.empty(W, dtype=torch.int32, device=self.device)
        self.head.mtpc_speculative_accept(P, wpp, draft_bytes, prefix_logprob, target_probs, accept_uniforms, accepted,
                                          next_byte)
        return accepted, next_byte

    def window_loss(self, num_sequences, sequence_length, gamma, hidden=None, targets=None):
        import torch
        h = self.hidden_device() if hidden is None else hidden
        t = torch.from_numpy(self.wl.targets).to(self.device) if targets is None else targets
        slot = torch.empty(self.wl.shape.n, dtype=torch.float32, device=self.device)
        loss = torch.empty(1, dtype=torch.float32, device=self.device)
        self.head.mtpc_window_loss(h, t, num_sequences, sequence_length, gamma, slot, loss)
        return slot, loss

    def window_logprob_backward(self, weight, hidden=None, targets=None):
        """-> dict(logprob [T], dh [T, d], dW_emit, dW_sum, dT_static or None) as fp32 device tensors."""
        import torch
        s = self.wl.shape
        h = self.hidden_device() if hidden is None else hidden
        t = torch.from_numpy(self.wl.targets).to(self.device) if targets is None else targets
        T = h.shape[0]
        f32 = dict(dtype=torch.float32, device=self.device)
        out = dict(logprob=torch.empty(T, **f32), dh=torch.empty((T, s.d), **f32),
                   dW_emit=torch.empty((s.n, s.r, s.v, s.d), **f32), dW_sum=torch.empty((s.sum_rows, s.d), **f32),
                   dT_static=torch.empty((max(s.n - 1, 1), s.r, s.r), **f32) if s.family == I.HMM else None)
        self.head.mtpc_window_logprob_backward(h, t, weight, out["logprob"], out["dh"], out["dW_emit"], out["dW_sum"],
                                               out["dT_static"])
        return out

    def window_policy_backward(self, old_logp, ref_logp, advantage, offsets, clip_low=0.2, clip_high=0.2, beta=0.0, mask=None, by_sequence=False, hidden=None,
                               targets=None, by_position=False):
        """The clipped policy loss of the windows' log-likelihoods (positions of packed sequences) and its gradients -> the dicts of policy_loss and of
        window_logprob_backward together. by_position: an advantage for every position."""
        logp = self.window_logprob(hidden=hidden, targets=targets)
        out = policy_loss(logp, old_logp, ref_logp, advantage, offsets, clip_low, clip_high, beta, mask=mask, by_sequence=by_sequence, by_position=by_position)
        return dict(self.window_logprob_backward(out["d_logp"], hidden=hidden, targets=targets), **out)

    def window_preference_backward(self, ref_logp, offsets, beta=0.1, smoothing=0.0, mask=None, hidden=None, targets=None):
        """The same of the preference loss of pairs of sequences."""
        logp = self.window_logprob(hidden=hidden, targets=targets)
        out = preference_loss(logp, ref_logp, offsets, beta, smoothing, mask=mask)
        return dict(self.window_logprob_backward(out["d_logp"], hidden=hidden, targets=targets), **out)

    def window_loss_backward(self, num_sequences, sequence_length, gamma, hidden=None, targets=None, out=None, max_norm=None):
        """-> dict(slot_loss [n], loss [1], dh, dW_emit, dW_sum, dT_static or None) as fp32 device tensors. out: the dict of an earlier call, whose
        buffers are written again. max_norm: the gradients of the head's parameters together are clipped to that norm, in place, and
        `grad_norm` [1] is what it was before; `gradients` is the list for that, of these very buffers, made by the first such call (not while a graph is
        captured). dh is not scaled: what is behind the head gets the gradient of the loss itself (for a norm over a whole model: `GradientList`)."""
        import torch
        s = self.wl.shape
        h = self.hidden_device() if hidden is None else hidden
        t = torch.from_numpy(self.wl.targets).to(self.device) if targets is None else targets
        T = h.shape[0]
        f32 = dict(dtype=torch.float32, device=h.device)
        shapes = dict(slot_loss=(s.n,), loss=(1,), dh=(T, s.d), dW_emit=(s.n, s.r, s.v, s.d), dW_sum=(s.sum_rows, s.d),
                      dT_static=(max(s.n - 1, 1), s.r, s.r) if s.family == I.HMM else None)
        if out is None:
            out = {k: None if shape is None else torch.empty(shape, **f32) for k, shape in shapes.items()}
        else:
            _written_again("window_loss_backward", shapes, h.device, out)
        grads = [out["dW_emit"], out["dW_sum"]] + ([out["dT_static"]] if s.family == I.HMM and s.n > 1 else [])
        if max_norm is not None and "gradients" in out and not out["gradients"].is_of(grads):
            raise B.MtpcError(B.ERR_SHAPE, "window_loss_backward: out['gradients'] is a list of other buffers (without it, a call makes one of these)")
        self.head.mtpc_window_loss_backward(h, t, num_sequences, sequence_length, gamma, out["slot_loss"], out["loss"],
                                            out["dh"], out["dW_emit"], out["dW_sum"], out["dT_static"])
        if max_norm is None:
            out.pop("grad_norm", None)                       # (an earlier step's)
            return out
        if "gradients" not in out:
            out["gradients"] = B.GradientList(grads)
        clip = out["gradients"]
        if "grad_norm" not in out:                           # where the list's calls write it: kept with the list, for graphs that hold them
            clip.norm = torch.empty(1, **f32) if clip.norm is None else clip.norm
            out["grad_norm"] = clip.norm
        clip.mtpc_clip_gradients(max_norm, out["grad_norm"])
        return out

    def close(self):
        self.head.mtpc_destroy()
