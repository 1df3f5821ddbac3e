"""The sequence operators in double precision on the CPU, from their formulas, and the sums of absolute values that the
error bounds of the tests are multiples of."""
import torch


def heads_for(x, H):
    return x if x.shape[2] == H else x.repeat_interleave(H // x.shape[2], 2)


def decay_attention(q, k, v, log_decay, lengths=None, state=None, scale=1.0):
    """(o, last state) row by row; q [B,N,H,D], k and v [B,N,Hkv,D], all double."""
    B, N, H, D = q.shape
    k, v = heads_for(k, H), heads_for(v, H)
    g = torch.exp(log_decay)[None, :, None, None]
    S = torch.zeros(B, H, D, D, dtype=q.dtype) if state is None else state
    n = torch.full((B,), N) if lengths is None else lengths.long()
    rows = []
    zero = torch.zeros((), dtype=q.dtype)
    for t in range(N):
        on = (t < n)[:, None, None, None]
        # rows past the length are left out before any product: they may hold anything
        kt, vt, qt = (torch.where(on[..., 0], x[:, t], zero) for x in (k, v, q))
        S = torch.where(on, g * S + kt[..., :, None] * vt[..., None, :], S)
        rows.append(torch.where(on[..., 0], scale * (qt[..., :, None] * S).sum(-2), zero))
    return torch.stack(rows, 1), S


def decay_bound(q, k, v, log_decay, lengths=None, state=None, scale=1.0):
    """The same with absolute values: what the rounding errors of any order of the sums are relative to."""
    return decay_attention(q.abs(), k.abs(), v.abs(), log_decay, lengths, None if state is None else state.abs(), abs(scale))


def rotary(x, positions, freq, interleaved=False, inverse=False, amplitude=1.0, lengths=None):
    """x [B,N,H,D] double, positions [B,N], freq [rot/2] double."""
    n = freq.numel()
    angle = (positions.double()[:, :, None] * freq)[:, :, None, :]
    if inverse:
        angle = -angle
    c, s = amplitude * torch.cos(angle), amplitude * torch.sin(angle)
    y = x.clone()
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    if lengths is not None:
        past = torch.arange(x.shape[1])[None, :] >= lengths[:, None]
        y[past] = 0.0
    return y


def layer_norm(x, weight, bias, eps):
    """x [rows, groups, d] double; (y, mean, rstd)."""
    mean = x.mean(-1)
    diff = x - mean[..., None]
    rstd = 1 / torch.sqrt((diff * diff).mean(-1) + eps)
    y = diff * rstd[..., None]
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return y, mean, rstd
