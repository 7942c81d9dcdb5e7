"""Plain 64-bit implementations of the training attention and of the norm + rotation of queries and keys, and how far a kernel with
bf16 products and fp32 sums may be from them, element by element.

A rounding to bf16 moves a value by at most u = 2^-8 of itself, one to fp32 by at most 2^-24.  A dot product of n terms in fp32
moves by at most n 2^-23 times the sum of the terms' magnitudes (each addition may round or truncate).
"""
import math

import torch

U = 2.0 ** -8
F = 2.0 ** -23


def heads_of(x, Nb, heads):
    return x.double().reshape(Nb, -1, heads, x.shape[1] // heads).permute(0, 2, 1, 3)


def rows_of(x):
    return x.permute(0, 2, 1, 3).flatten(0, 1).flatten(1)


def visible(Nb, Lq, Lk, causal, q_lens, k_lens, device):
    ql = torch.full((Nb,), Lq, device=device) if q_lens is None else q_lens.long().clamp(0, Lq)
    kl = torch.full((Nb,), Lk, device=device) if k_lens is None else k_lens.long().clamp(0, Lk)
    i, j = torch.arange(Lq, device=device)[None, :, None], torch.arange(Lk, device=device)[None, None]
    see = (i < ql[:, None, None]) & (j < kl[:, None, None])
    if causal:
        see &= j <= i + (kl - ql)[:, None, None]
    return see[:, None]


def scores(q, k, Nb, H, G, scale, see):
    qd, kd = heads_of(q, Nb, H), heads_of(k, Nb, G).repeat_interleave(H // G, 1)
    # what no query sees has no part, whatever it holds
    qd = torch.where(see.any(-1, keepdim=True), qd, 0.0)
    kd = torch.where(see.any(-2)[..., None], kd, 0.0)
    S = (qd @ kd.transpose(-1, -2)) * scale
    slack = qd.shape[-1] * F * scale * (qd.abs() @ kd.abs().transpose(-1, -2)) + 4 * F * S.abs()
    return qd, kd, S.masked_fill(~see, -math.inf), slack.masked_fill(~see, 0.0)


def forward(q, k, v, Nb, H, G, scale, causal=False, q_lens=None, k_lens=None):
    """out, lse and their bounds."""
    Lq, Lk = q.shape[0] // Nb, k.shape[0] // Nb
    see = visible(Nb, Lq, Lk, causal, q_lens, k_lens, q.device)
    _, _, S, slack = scores(q, k, Nb, H, G, scale, see)
    vd = torch.where(see.any(-2)[..., None], heads_of(v, Nb, G).repeat_interleave(H // G, 1), 0.0)
    lse = torch.logsumexp(S, -1)
    P = (S - lse[..., None]).exp().nan_to_num(0.0)
    out, A = P @ vd, P @ vd.abs()
    # relative error of a weight: its score's, exp2 and the sums (a few units of fp32 each; the sum of Lk weights adds up 2^-23 each)
    w = slack.amax(-1, keepdim=True) * 2 + (16 + Lk / 64) * F
    bound = A * (U + 2 * w) * (1 + U) + U * out.abs() + 1e-30
    lse_bound = w[..., 0] + 8 * F * (lse.abs().nan_to_num(0.0, posinf=0.0) + S.abs().nan_to_num(0.0, posinf=0.0).amax(-1))
    return rows_of(out), lse, rows_of(bound), lse_bound


def backward(q, k, v, out, lse, dout, Nb, H, G, scale, causal=False, q_lens=None, k_lens=None):
    """dq, dk, dv and their bounds, from the given out and lse."""
    Lq, Lk = q.shape[0] // Nb, k.shape[0] // Nb
    see = visible(Nb, Lq, Lk, causal, q_lens, k_lens, q.device)
    qd, kd, S, slack = scores(q, k, Nb, H, G, scale, see)
    alive = see.any(-1, keepdim=True)
    vd = torch.where(see.any(-2)[..., None], heads_of(v, Nb, G).repeat_interleave(H // G, 1), 0.0)
    do, o = (torch.where(alive, heads_of(t, Nb, H), 0.0) for t in (dout, out))
    l = torch.where(alive, lse.double()[..., None], 0.0)
    P = (S - l).exp().nan_to_num(0.0)
    wP = 2 * slack + (16 + 8 * l.abs()) * F                                    # relative error of P
    dP, D = do @ vd.transpose(-1, -2), (do * o).sum(-1, keepdim=True)
    n = qd.shape[-1]
    eP = n * F * (do.abs() @ vd.abs().transpose(-1, -2)) + n * F * (do * o).abs().sum(-1, keepdim=True) + 2 * F * (dP.abs() + D.abs())
    dS = P * (dP - D)
    eS = (wP + U + 4 * F) * dS.abs() + 2 * P * eP
    fold = lambda x: x.unflatten(1, (G, H // G)).sum(2)  # noqa: E731
    dq, dk, dv = scale * dS @ kd, scale * fold(dS.transpose(-1, -2) @ qd), fold(P.transpose(-1, -2) @ do)
    sums = F * (8 + (Lk + Lq * (H // G)) / 64)                                 # the accumulations
    bq = scale * (eS + sums * dS.abs()) @ kd.abs()
    bk = scale * fold((eS + sums * dS.abs()).transpose(-1, -2) @ qd.abs())
    bv = fold((P * (U + 2 * wP + sums)).transpose(-1, -2) @ do.abs())
    return [rows_of(t) for t in (dq, dk, dv)], [rows_of((1 + U) * b + U * t.abs() + 1e-30) for t, b in ((dq, bq), (dk, bk), (dv, bv))]


def rope(x, heads, gamma, eps, cos, sin, positions, interleaved):
    """The norm and rotation in 64 bits: [rows, heads * dh]; differentiable."""
    y = x.double().reshape(x.shape[0], heads, -1)
    y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt()
    if gamma is not None:
        y = y * gamma.double()
    if cos is None:
        return y.flatten(1)
    half, rot = cos.shape[1], 2 * cos.shape[1]
    at = torch.arange(x.shape[0], device=x.device) % cos.shape[0] if positions is None else positions.long().clamp(0, cos.shape[0] - 1)
    c, s = cos.double()[at][:, None], sin.double()[at][:, None]
    a, b = (y[..., :rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :half], y[..., half:rot])
    a, b = a * c - b * s, b * c + a * s
    r = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((r, y[..., rot:]), -1).flatten(1)
