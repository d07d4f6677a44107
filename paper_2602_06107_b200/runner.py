"""Output allocation around the libjackpot calls (no arithmetic of the method here)."""
from __future__ import annotations

import torch

from . import binding as B

AUX_F32 = ("accept_prob", "uniform", "z_approx", "lse_actor", "lse_policy")


def _alloc_outputs(T, dev):
    return dict(accept=torch.empty(T, dtype=torch.uint8, device=dev),
                weight=torch.empty(T, dtype=torch.float32, device=dev),
                logp_actor=torch.empty(T, dtype=torch.float32, device=dev),
                logp_policy=torch.empty(T, dtype=torch.float32, device=dev),
                stats_buf=B.new_stats_buffer(dev))


def _alloc_aux(T, k, V, dev, want_exact):
    aux = {n: torch.empty(T, dtype=torch.float32, device=dev) for n in AUX_F32}
    if k < V:
        aux["topk_idx_actor"] = torch.empty((T, k), dtype=torch.int32, device=dev)
        aux["topk_idx_policy"] = torch.empty((T, k), dtype=torch.int32, device=dev)
        aux["topk_val_actor"] = torch.empty((T, k), dtype=torch.float32, device=dev)
        aux["topk_val_policy"] = torch.empty((T, k), dtype=torch.float32, device=dev)
    if want_exact:
        aux["z_exact"] = torch.empty(T, dtype=torch.float32, device=dev)
    return aux


def forward(ctx: B.Context, za, zp, tokens, mask=None, *, lam=None, budget=None, k=20, seed=0,
            token_offset=0, c1=0.0, aux=True, want_exact=False, sync=True):
    """One jp_obrs_forward call; returns a dict of device tensors plus ``stats``."""
    assert (lam is None) != (budget is None)
    T, V = za.shape
    dev = za.device
    out = _alloc_outputs(T, dev)
    auxd = _alloc_aux(T, k, V, dev, want_exact) if aux else {}
    mode = B.JP_LAMBDA_FIXED if budget is None else B.JP_LAMBDA_FROM_BUDGET
    desc = B.make_desc(za, lambda_mode=mode, c1=c1, token_offset=token_offset, aux=auxd)
    B.jp_obrs_forward(ctx, desc, za, zp, tokens, mask, lam if budget is None else budget, k, seed,
                      out["accept"], out["weight"], out["logp_actor"], out["logp_policy"], out["stats_buf"])
    out.update(auxd)
    if sync:
        torch.cuda.synchronize(dev)
        out["stats"] = B.read_stats(out["stats_buf"])
    return out


def forward_chunked(ctx: B.Context, chunks, T_total, V, dtype_code, *, lam=None, budget=None, k=20, seed=0,
                    c1=0.0, device="cuda", aux=False):
    """``chunks`` yields (token_offset, za, zp, tokens, mask_or_None) blocks of rows."""
    assert (lam is None) != (budget is None)
    exact = k >= V
    B.jp_batch_begin(ctx, T_total, V, dtype_code, k, lam if (exact and lam is not None) else 0.0)
    for off, za, zp, tok, m in chunks:
        d = B.make_desc(za, token_offset=off)
        B.jp_batch_chunk(ctx, d, za, zp, tok, m)
    out = _alloc_outputs(T_total, device)
    auxd = {}
    d = B.jp_obrs_desc()
    d.c1 = c1
    if aux:
        auxd = _alloc_aux(T_total, k, V, device, False)
        for n, t in auxd.items():
            setattr(d, n, t.data_ptr())
    mode = B.JP_LAMBDA_FIXED if budget is None else B.JP_LAMBDA_FROM_BUDGET
    B.jp_batch_finalize(ctx, d, lam if budget is None else budget, mode, seed, out["accept"], out["weight"],
                        out["logp_actor"], out["logp_policy"], out["stats_buf"])
    out.update(auxd)
    torch.cuda.synchronize()
    out["stats"] = B.read_stats(out["stats_buf"])
    return out


def backward(ctx: B.Context, za, zp, tokens, mask, accept, weight, *, advantages=None, lambda_distill=0.0,
             grad_out=1.0, n_valid=0, record_offset=0, d_actor=None, d_policy=None, vocab_offset=None, **general):
    """``general``: the optional fields of jp_obrs_bwd_desc (logp_ref, logp_actor_ref, logp_inf, eps_lo,
    eps_hi, c2, tis_cap, out_obj_policy, out_obj_actor, out_kl, out_loss).  ``vocab_offset``: the logits are
    the columns from there on of rows whose records a vocabulary-parallel forward left (jp_vshard_backward)."""
    T, V = za.shape
    if d_actor is None:
        d_actor = torch.empty((T, za.stride(0)), dtype=torch.bfloat16, device=za.device)[:, :V]
    if d_policy is None:
        d_policy = torch.empty((T, zp.stride(0)), dtype=torch.bfloat16, device=za.device)[:, :V]
    desc = B.make_desc(za)
    bwd = B.make_bwd_desc(advantages, lambda_distill, grad_out, n_valid, record_offset, **general)
    if vocab_offset is None:
        B.jp_obrs_backward(ctx, desc, bwd, za, zp, tokens, mask, accept, weight, d_actor, d_policy)
    else:
        B.jp_vshard_backward(ctx, desc, bwd, za, zp, tokens, mask, vocab_offset, accept, weight, d_actor, d_policy)
    return d_actor, d_policy


def forward_sparse_actor(ctx: B.Context, zp, tokens, mask, logp_inf_token, topk_inf_idx, topk_inf_logp, *, lam=None,
                         budget=None, k=20, seed=0, token_offset=0, c1=0.0, cap=False, aux=True):
    """One jp_obrs_forward_sparse_actor call; returns a dict of device tensors plus ``stats``."""
    assert (lam is None) != (budget is None)
    T, V = zp.shape
    dev = zp.device
    out = _alloc_outputs(T, dev)
    del out["logp_actor"]
    out["z_lower"] = torch.empty(T, dtype=torch.float32, device=dev)
    out["z_upper"] = torch.empty(T, dtype=torch.float32, device=dev)
    auxd = {}
    if aux:
        auxd = {n: torch.empty(T, dtype=torch.float32, device=dev) for n in ("accept_prob", "uniform", "z_approx",
                                                                              "lse_policy")}
        auxd["topk_idx_policy"] = torch.empty((T, k), dtype=torch.int32, device=dev)
        auxd["topk_val_policy"] = torch.empty((T, k), dtype=torch.float32, device=dev)
    mode = B.JP_LAMBDA_FIXED if budget is None else B.JP_LAMBDA_FROM_BUDGET
    desc = B.make_desc(zp, lambda_mode=mode, c1=c1, token_offset=token_offset, aux=auxd,
                       flags=B.JP_DESC_SPARSE_CAP if cap else 0)
    B.jp_obrs_forward_sparse_actor(ctx, desc, zp, tokens, mask, logp_inf_token, topk_inf_idx, topk_inf_logp,
                                   topk_inf_idx.shape[1], lam if budget is None else budget, k, seed, out["accept"],
                                   out["weight"], out["logp_policy"], out["z_lower"], out["z_upper"], out["stats_buf"])
    out.update(auxd)
    torch.cuda.synchronize(dev)
    out["stats"] = B.read_stats(out["stats_buf"])
    return out


def _final_norm(ctx, h, norm):
    """The model's last norm on its hidden states, ready for the context's stream."""
    weight, bias, eps, rms = norm
    y, _, _ = layer_norm(ctx, h, weight, bias, eps=eps, rms=rms)
    current = torch.cuda.current_stream(ctx.device)
    if current.cuda_stream != ctx.stream:
        own = torch.cuda.ExternalStream(ctx.stream, device=ctx.device)
        own.wait_stream(current)
        y.record_stream(own)
    return y


def forward_lmhead(ctx: B.Context, h_actor, w_actor, h_policy, w_policy, tokens, mask=None, *, lam=None, budget=None, k=20,
                   seed=0, token_offset=0, c1=0.0, norm_actor=None, norm_policy=None):
    """One jp_obrs_forward_lmhead call; returns a dict of device tensors plus ``stats``.  ``norm_actor`` /
    ``norm_policy``: a model's last norm, ``(weight, bias or None, eps, rms)``, when ``h_*`` are the hidden states in
    front of it (jp_layer_norm_forward runs first)."""
    assert (lam is None) != (budget is None)
    if norm_actor is not None:
        h_actor = _final_norm(ctx, h_actor, norm_actor)
    if norm_policy is not None:
        h_policy = _final_norm(ctx, h_policy, norm_policy)
    T, V = h_actor.shape[0], w_actor.shape[0]
    dev = h_actor.device
    out = _alloc_outputs(T, dev)
    auxd = _alloc_aux(T, k, V, dev, False)
    d = B.jp_obrs_desc()
    d.T, d.V = T, V
    d.lambda_mode = B.JP_LAMBDA_FIXED if budget is None else B.JP_LAMBDA_FROM_BUDGET
    d.c1, d.token_offset = c1, token_offset
    for n, t in auxd.items():
        setattr(d, n, t.data_ptr())
    B.jp_obrs_forward_lmhead(ctx, d, h_actor, w_actor, h_policy, w_policy, tokens, mask,
                             lam if budget is None else budget, k, seed, out["accept"], out["weight"],
                             out["logp_actor"], out["logp_policy"], out["stats_buf"])
    out.update(auxd)
    torch.cuda.synchronize(dev)
    out["stats"] = B.read_stats(out["stats_buf"])
    return out


def _rows(t, name):
    """[T, H] matrix with contiguous rows -> its row pitch in elements."""
    shape = t.shape
    if len(shape) == 2:
        if t.is_contiguous() or shape[0] <= 1 and (shape[1] <= 1 or t.stride(1) == 1):
            return shape[1]
        pitch, one = t.stride()
        if one == 1 or shape[1] <= 1:
            if pitch < shape[1]:
                raise B.JackpotError(f"{name}: rows overlap")
            return pitch
    raise B.JackpotError(f"{name} must be a matrix with contiguous rows")


def _dense(t, shape, dtype, name):
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        raise B.JackpotError(f"{name} must be a contiguous {dtype} tensor of shape {list(shape)}")


def _like(x):
    return torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)


def _norm_desc(ctx, x, weight, bias, eps, rms, out, name, dy=None):
    """Checks and fills what both passes share; ``out`` is y or dx."""
    ld_x, shape, dtype, param = _rows(x, "x"), x.shape, x.dtype, weight.dtype
    _dense(weight, shape[1:], param, "weight")
    if bias is not None:
        _dense(bias, shape[1:], param, "bias")
    if out.shape != shape or out.dtype is not dtype:
        raise B.JackpotError(f"{name} must have x's shape and dtype")
    ld_out, ld_y, ld_dy, ld_dx = _rows(out, name), 0, 0, 0
    if dy is None:
        ld_y = ld_out
    else:
        if dy.shape != shape or dy.dtype is not dtype:
            raise B.JackpotError("dy must have x's shape and dtype")
        ld_dx, ld_dy = ld_out, _rows(dy, "dy")
    return B._desc(ctx, B.jp_norm_desc, shape[0], shape[1], ld_x, ld_y, ld_dy, ld_dx, B._dtype_code(x, "x"), B._dtype_code(weight, "weight"),
                   B.JP_NORM_RMS if rms else 0, float(eps))


def layer_norm(ctx: B.Context, x, weight, bias=None, *, eps=1e-6, rms=False, out=None):
    """One jp_layer_norm_forward call on torch's current stream: ``(y, mean, rstd)`` (mean None with ``rms``).
    ``out``: where y goes (may be ``x``)."""
    y = _like(x) if out is None else out
    d = _norm_desc(ctx, x, weight, bias, eps, rms, y, "out")
    mean = None if rms else x.new_empty(d.T, dtype=torch.float32)
    rstd = x.new_empty(d.T, dtype=torch.float32)
    B.jp_layer_norm_forward(ctx, d, x, weight, bias, y, mean, rstd)
    return y, mean, rstd


def layer_norm_backward(ctx: B.Context, dy, x, weight, mean, rstd, *, rms=False, bias=True, dx=None):
    """One jp_layer_norm_backward call on torch's current stream: ``(dx, dweight, dbias)`` with fp32 dweight and dbias
    (dbias None without ``bias``).  ``mean`` and ``rstd`` are the forward's; ``dx``: where dx goes (may be ``dy`` or ``x``)."""
    if dx is None:
        dx = _like(x)
    d = _norm_desc(ctx, x, weight, None, 0.0, rms, dx, "dx", dy)
    T, H = x.shape
    if not rms:
        _dense(mean, (T,), torch.float32, "mean")
    _dense(rstd, (T,), torch.float32, "rstd")
    dweight = x.new_empty(H, dtype=torch.float32)
    dbias = x.new_empty(H, dtype=torch.float32) if bias else None
    need = B.jp_layer_norm_workspace_bytes(ctx, T, H, d.dtype)
    ws = x.new_empty(need, dtype=torch.uint8) if need else None
    B.jp_layer_norm_backward(ctx, d, dy, x, weight, None if rms else mean, rstd, dx, dweight, dbias, ws)
    return dx, dweight, dbias


class W4Weight:
    """4-bit weights laid out by jp_w4_pack: what jp_w4_linear takes."""

    def __init__(self, packed, N, K, group):
        self.packed = packed
        self.desc = B.jp_w4_desc(N=N, K=K, group=group)
        self.N, self.K, self.group = N, K, group


def quantize_w4(weight, group=128, *, symmetric=True, scale_dtype=torch.bfloat16):
    """Rounds a [N, K] weight to 4 bits, each ``group`` of a row by its own largest magnitude (``symmetric``) or range:
    ``(q [N, (K + 1) // 2] uint8, scales [N, groups], zeros [N, groups] uint8 or None)`` for :func:`pack_w4`."""
    N, K = weight.shape
    G = (K + group - 1) // group
    w = torch.nn.functional.pad(weight.float(), (0, G * group - K)).view(N, G, group)
    if symmetric:
        scales = (w.abs().amax(2) / 7.0).to(scale_dtype)
        zeros, z = None, 8.0
    else:
        lo, hi = w.amin(2).clamp(max=0.0), w.amax(2).clamp(min=0.0)
        scales = ((hi - lo) / 15.0).to(scale_dtype)
        s = scales.float()
        z = torch.where(s > 0, -lo / s, torch.zeros_like(s)).round().clamp(0, 15)
        zeros, z = z.to(torch.uint8), z[..., None]
    s = scales.float()[..., None]
    v = torch.where(s > 0, w / s, torch.zeros_like(w)).round()
    v = (v + z).clamp(0, 15).to(torch.uint8).view(N, G * group)
    v = v[:, :K + K % 2] if G * group >= K + K % 2 else torch.nn.functional.pad(v, (0, 1))
    return (v[:, 0::2] | v[:, 1::2] << 4).contiguous(), scales, zeros


def pack_w4(ctx: B.Context, q, scales, zeros=None, *, K, group=128):
    """One jp_w4_pack call on torch's current stream: lays ``q`` [N, (K + 1) // 2] uint8 (two values a byte, the lower
    index in the low half), ``scales`` [N, groups] bf16 or fp16 and ``zeros`` [N, groups] uint8 (None: 8) out once."""
    N, bytes_, G = q.shape[0], (K + 1) // 2, (K + group - 1) // group
    d = B.jp_w4_desc(N=N, K=K, group=group)
    need = B.jp_w4_packed_bytes(N, K, group)
    if need == 0:
        raise B.JackpotError(f"no layout for N = {N}, K = {K}, group = {group} (1 <= K <= 65536; group 32, 64 or 128)")
    codes = {torch.bfloat16: B.JP_BF16, torch.float16: B.JP_F16}
    if q.dtype != torch.uint8 or scales.dtype not in codes or (zeros is not None and zeros.dtype != torch.uint8):
        raise B.JackpotError("q and zeros must be uint8, scales bfloat16 or float16")
    if q.shape != (N, bytes_) or scales.shape != (N, G) or (zeros is not None and zeros.shape != (N, G)):
        raise B.JackpotError(f"for K = {K} and group = {group}: q must be [N, {bytes_}], scales and zeros [N, {G}]")
    d.scale_dtype = codes[scales.dtype]
    d.ld_q, d.ld_scales = _rows(q, "q"), _rows(scales, "scales")
    if zeros is not None:
        d.ld_zeros = _rows(zeros, "zeros")
    packed = torch.empty(need, dtype=torch.uint8, device=q.device)
    B.jp_w4_pack(ctx, d, q, scales, zeros, packed)
    return W4Weight(packed, N, K, group)


def linear_w4(ctx: B.Context, x, w: W4Weight, *, out_dtype=torch.bfloat16, out=None):
    """One jp_w4_linear call on torch's current stream: x [M, K] bf16, M <= 32, times the packed weight: [M, N], contiguous or
    in ``out``.  :func:`verify_draft` takes logits with rows a multiple of 16 bytes apart only: for an N that is no multiple of 8 (bf16)
    or 4 (fp32), pass ``out = torch.empty((M, (N + 7) // 8 * 8), ...)[:, :N]``."""
    if x.dtype != torch.bfloat16:
        raise B.JackpotError(f"x must be bfloat16, got {x.dtype}")
    ld_x = _rows(x, "x")
    M = x.shape[0]
    if x.shape[1] != w.K:
        raise B.JackpotError(f"x has {x.shape[1]} columns, the weight {w.K}")
    if out is None:
        out = x.new_empty((M, w.N), dtype=out_dtype)
    elif out.shape != (M, w.N):
        raise B.JackpotError(f"out must be [{M}, {w.N}]")
    B.jp_w4_linear(ctx, w.desc, w.packed, x, ld_x, M, out, _rows(out, "out"), B._dtype_code(out, "out"))
    return out


def _positions(t, shape, name):
    """[B, rows, V] logits with contiguous rows -> the pitches of rows and sequences in elements."""
    stride = t.stride()
    if t.shape != shape or (stride[2] != 1 and shape[2] > 1):
        raise B.JackpotError(f"{name} must be {list(shape)} with contiguous rows")
    n_seq, rows, V = shape
    ld = stride[1] if rows > 1 else (V + 7) // 8 * 8         # a single row has no pitch of its own: any that is allowed
    seq = stride[0] if n_seq > 1 else rows * ld
    if ld < V or seq < (rows - 1) * ld + V:
        raise B.JackpotError(f"{name}: rows or sequences overlap")
    return ld, seq


def verify_draft(ctx: B.Context, target_logits, draft_logits, draft_tokens, u_accept, u_sample, *, n_draft=None,
                 temperature=None, accept_prob=True, logp=True):
    """One jp_verify_draft call on torch's current stream.  target_logits [B, N + 1, V], draft_logits [B, N, V] or None
    (drafts without a distribution), draft_tokens [B, N] int32, u_accept [B, N] and u_sample [B] fp32, n_draft [B] int32
    or None, temperature [B] fp32 or None.  The logits start on 16 bytes and their rows and sequences are multiples of 16 bytes
    apart: those of an odd vocabulary are a slice of wider rows.  Returns ``n_accepted`` [B], ``tokens`` [B, N + 1] and,
    unless turned off, ``accept_prob`` [B, N] and ``logp`` [B, N + 1]."""
    if target_logits.dim() != 3 or target_logits.shape[1] < 1:
        raise B.JackpotError("target_logits must be [B, N + 1, V]")
    n_seq, rows, V = target_logits.shape
    N = rows - 1
    ld, seq = _positions(target_logits, (n_seq, rows, V), "target_logits")
    dtype, ld_d, seq_d = B._dtype_code(target_logits), 0, 0
    if draft_logits is not None:
        if draft_logits.dtype is not target_logits.dtype:
            raise B.JackpotError("draft_logits must have target_logits' dtype")
        if draft_logits.dim() != 3:
            raise B.JackpotError("draft_logits must be [B, N, V]")
        ld_d, seq_d = _positions(draft_logits, (n_seq, N, V), "draft_logits")
    d = B._desc(ctx, B.jp_verify_desc, n_seq, V, ld, seq, ld_d, seq_d, N, dtype)
    _dense(draft_tokens, (n_seq, N), torch.int32, "draft_tokens")
    _dense(u_accept, (n_seq, N), torch.float32, "u_accept")
    _dense(u_sample, (n_seq,), torch.float32, "u_sample")
    if n_draft is not None:
        _dense(n_draft, (n_seq,), torch.int32, "n_draft")
    if temperature is not None:
        _dense(temperature, (n_seq,), torch.float32, "temperature")
    dev = u_sample.device                                    # (empty_strided: the cheapest call that makes a matrix)
    out = dict(n_accepted=torch.empty_like(u_sample, dtype=torch.int32),
               tokens=torch.empty_strided((n_seq, rows), (rows, 1), dtype=torch.int32, device=dev))
    if accept_prob:
        out["accept_prob"] = torch.empty_like(u_accept)
    if logp:
        out["logp"] = torch.empty_strided((n_seq, rows), (rows, 1), dtype=torch.float32, device=dev)
    need = B.jp_verify_workspace_bytes(ctx, n_seq, N, V, d.dtype, draft_logits is not None and N > 0)
    ws = u_sample.new_empty(need, dtype=torch.uint8) if need else None
    B.jp_verify_draft(ctx, d, target_logits, draft_logits, draft_tokens, n_draft, temperature, u_accept, u_sample,
                      out["n_accepted"], out["tokens"], out.get("accept_prob"), out.get("logp"), ws)
    return out
