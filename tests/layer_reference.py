"""Plain float64 forms (torch, CPU) of the linear attention, the rotary positions and the norms around a block, written
from their definitions for the tests."""
import math

import torch


def length_mask(lengths, B, n):
    """[B, n] bool: the tokens inside each sequence."""
    t = torch.arange(n)
    return t[None, :] < (torch.full((B,), n) if lengths is None else lengths.clamp(0, n))[:, None]


def f64(t):
    return None if t is None else t.detach().cpu().double()


def decay_powers(log_decay, x):
    """exp(log_decay * x) with 0^0 = 1; log_decay [H], x any shape -> [H, *x.shape]."""
    lam = log_decay.double().exp()
    return lam.view(-1, *[1] * x.dim()) ** x.double()


def linear(Q, K, V, log_decay, scale, lengths=None, state=None):
    """(O, final state, absolute sums): O_i = scale (sum_{j <= i} l^(i-j) (q_i . k_j) v_j + l^(i+1) q_i S).  The
    absolute sums are O's with every factor's magnitude: what rounding errors are measured against."""
    B, H, n, d = Q.shape
    G = H // K.shape[1]
    live = length_mask(lengths, B, n)[:, None, :, None].double()
    # rows behind the end are not part of the inputs (they may hold anything)
    q, k, v = (torch.where(live > 0, f64(x).repeat_interleave(r, 1), 0.0) for x, r in ((Q, 1), (K, G), (V, G)))
    g = f64(log_decay)
    t = torch.arange(n)
    gap = t[:, None] - t[None, :]
    W = torch.where(gap >= 0, decay_powers(g, gap.clamp(min=0)), 0.0)[None]
    S = torch.zeros(B, H, d, d, dtype=torch.float64) if state is None else f64(state)
    since = decay_powers(g, t + 1)[None, ..., None]
    length = live.sum((1, 2, 3)).long()
    until = torch.stack([decay_powers(g, (m - 1 - t).clamp(min=0)) for m in length])[..., None]
    whole = torch.stack([decay_powers(g, m) for m in length])[..., None, None]
    O = scale * (((q @ k.transpose(-1, -2)) * W) @ v + since * (q @ S)) * live
    A = abs(scale) * (((q.abs() @ k.abs().transpose(-1, -2)) * W) @ v.abs() + since * (q.abs() @ S.abs())) * live
    return O, (k * until).transpose(-1, -2) @ v + whole * S, A


def linear_grad(Q, K, V, dO, log_decay, scale, lengths=None, state=None, dstate=None):
    """dict of dQ, dK, dV, dS and their absolute sums (keys with a leading 'a')."""
    B, H, n, d = Q.shape
    G = H // K.shape[1]
    live = length_mask(lengths, B, n)[:, None, :, None].double()
    q, k, v, o = (torch.where(live > 0, f64(x).repeat_interleave(r, 1), 0.0)
                  for x, r in ((Q, 1), (K, G), (V, G), (dO, 1)))
    g = f64(log_decay)
    t = torch.arange(n)
    gap = t[:, None] - t[None, :]
    W = torch.where(gap >= 0, decay_powers(g, gap.clamp(min=0)), 0.0)[None]
    zero = torch.zeros(B, H, d, d, dtype=torch.float64)
    S, R = (zero if x is None else f64(x) for x in (state, dstate))
    since = decay_powers(g, t + 1)[None, ..., None]
    length = live.sum((1, 2, 3)).long()
    until = torch.stack([decay_powers(g, (m - 1 - t).clamp(min=0)) for m in length])[..., None]
    whole = torch.stack([decay_powers(g, m) for m in length])[..., None, None]

    def grads(q, k, v, o, S, R, s):
        back = lambda x: x.transpose(-1, -2)  # noqa: E731
        dQ = s * (((o @ back(v)) * W) @ k + since * (o @ back(S))) * live
        dK = (s * (back((o @ back(v)) * W) @ q) + until * (v @ back(R))) * live
        dV = (s * (back((q @ back(k)) * W) @ o) + until * (k @ R)) * live
        dK, dV = (x.view(B, H // G, G, n, d).sum(2) for x in (dK, dV))
        return dict(dQ=dQ, dK=dK, dV=dV, dS=s * (back(q * since) @ o) + whole * R)

    got = grads(q, k, v, o, S, R, scale)
    got.update({"a" + x: y for x, y in grads(*(x.abs() for x in (q, k, v, o, S, R)), abs(scale)).items()})
    return got


def rotary(x, pos, pairs, base=10000.0, interleaved=False, shared=False, inverse=False):
    """x [B, H, n, 64], pos [axes, B or 1, n]."""
    x, pos = f64(x), f64(pos)
    a, b = (x[..., 0::2].clone(), x[..., 1::2].clone()) if interleaved else (x[..., :32].clone(), x[..., 32:].clone())
    i = 0
    for axis, many in enumerate(pairs):
        for m in range(many):
            angle = pos[axis] * math.pow(base, -i / 32 if shared else -m / many) * (-1 if inverse else 1)
            c, s = angle.cos()[:, None], angle.sin()[:, None]
            a[..., i], b[..., i] = a[..., i] * c - b[..., i] * s, b[..., i] * c + a[..., i] * s
            i += 1
    return torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)


def norm(z, kind, eps, w, b):
    if kind == "layer":
        z = z - z.mean(-1, keepdim=True)
    z = z / (z.square().mean(-1, keepdim=True) + eps).sqrt() * w
    return z if b is None else z + b


def norm_residual(p, kind, eps, residual_scale, branch_scale):
    """p: dict of float64 X, F, post_w, post_b, gate, pre_w, pre_b (each None or a tensor); (Y, H or None)."""
    Y = residual_scale * p["X"]
    if p["F"] is not None:
        u = p["F"] if p["post_w"] is None else norm(p["F"], kind, eps, p["post_w"], p["post_b"])
        if p["gate"] is not None:
            u = u * (p["gate"] if p["gate"].dim() == 1 else p["gate"][:, None])
        Y = Y + branch_scale * u
    return Y, None if p["pre_w"] is None else norm(Y, kind, eps, p["pre_w"], p["pre_b"])
