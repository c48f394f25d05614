"""The objectives beside the PPO step written out in float64 torch (CPU or GPU), for the tests: one function per objective
that takes logits as float64 and returns the loss terms and the gradient from its formula.  Shares no code with the
library."""
from __future__ import annotations

import torch


def valid_mask(lengths, T):
    return torch.arange(T, device=lengths.device)[None] < lengths.clamp(0, T)[:, None]


def label_logprobs(z, ids, lengths):
    """(log softmax of every row, log-prob of each generated token; 0 at padding and at ids out of range, and that mask)."""
    V = z.shape[2]
    lq = torch.log_softmax(z, dim=2)
    ok = valid_mask(lengths, z.shape[1]) & (ids >= 0) & (ids < V)
    y = ids.clamp(0, V - 1)
    lp = torch.where(ok, lq.gather(2, y[..., None])[..., 0], 0.0)
    return lq, lp, ok


def label_gradient(lq, ids, g):
    V = lq.shape[2]
    d = -lq.exp()
    y = ids.clamp(0, V - 1)[..., None]
    d.scatter_(2, y, -torch.expm1(lq.gather(2, y)))
    return torch.where(g[..., None] != 0, g[..., None] * d, 0.0)


def policy_kl(z, ids, lengths, lp_old, lp_ref, adv, clip_low, clip_high, kl_coef, reduction, grad_scale):
    """loss_pg, loss_kl, dlogits, lp and, per token, the sum of the absolute parts of the gradient factor."""
    B, T, _ = z.shape
    lq, lp, ok = label_logprobs(z, ids, lengths)
    n = lengths.clamp(0, T).double()
    if reduction == 0:
        w = torch.ones((B, T), dtype=torch.float64, device=z.device) / n.sum().clamp(min=1)
    else:
        w = (1 / (n.clamp(min=1) * (n > 0).sum().clamp(min=1)))[:, None].expand(B, T)
    A = (adv[:, None].expand(B, T) if adv.dim() == 1 else adv).double()
    rho = torch.exp(lp - lp_old.double())
    free, held = -A * rho, -A * rho.clamp(1 - clip_low, 1 + clip_high)
    d = (lp_ref.double() - lp) if lp_ref is not None else torch.zeros_like(lp)
    zero = torch.zeros_like(lp)
    d_pg = torch.where(free >= held, free, zero)
    g = torch.where(ok, grad_scale * w * (d_pg - kl_coef * torch.expm1(d)), zero)
    size = torch.where(ok, abs(grad_scale) * w * (d_pg.abs() + kl_coef * (1 + torch.exp(d))), zero)
    pg = torch.where(ok, w * torch.maximum(free, held), zero).sum()
    kl = torch.where(ok, w * (torch.expm1(d) - d), zero).sum()
    return pg, kl, label_gradient(lq, ids, g), lp, size


def preference(z, ids, lengths, lp_ref, kind, beta, margin, smoothing, length_mean, grad_scale):
    """loss, rewards, dlogits, lp, factor of every sequence."""
    B, T, _ = z.shape
    lq, lp, ok = label_logprobs(z, ids, lengths)
    ref = lp_ref.double() if lp_ref is not None else torch.zeros_like(lp)
    n = lengths.clamp(0, T).double()
    c = 1 / n.clamp(min=1) if length_mean else torch.ones_like(n)
    s = c * torch.where(ok, lp - ref, 0.0).sum(dim=1)
    half = B // 2
    h = beta * (s[:half] - s[half:]) - margin
    if kind == 0:
        up, down = torch.nn.functional.logsigmoid(h), torch.nn.functional.logsigmoid(-h)
        loss = -(1 - smoothing) * up - smoothing * down
        dh = smoothing * up.exp() - (1 - smoothing) * down.exp()
    elif kind == 1:
        loss, dh = (1 - h).clamp(min=0), -(h < 1).double()
    else:
        loss, dh = ((h - 0.5) / beta) ** 2, 2 * (h - 0.5) / beta ** 2
    f = torch.cat([dh, -dh]) * beta * c * (grad_scale / half)
    g = torch.where(ok, f[:, None].expand(B, T), 0.0)
    return loss.mean(), beta * s, label_gradient(lq, ids, g), lp, f


def row_logits(B, T, V, dtype, gen, device, sigma=3.0, prompt=0, offset=0, pitch=0):
    """Random 16-bit logits as a [B,T,V] view: `prompt` rows before each sequence's, `offset` entries before the first row,
    `pitch` entries between rows beyond V."""
    row = V + pitch
    store = torch.full((offset + B * (prompt + T) * row + 8,), float("nan"), dtype=dtype, device=device)
    full = store[offset:offset + B * (prompt + T) * row].view(B, prompt + T, row)
    z = full[:, prompt:, :V]
    z.copy_(sigma * torch.randn((B, T, V), generator=gen, device=device))
    return z, store


def topk(z, lengths, K, temperature):
    """ids (int64) and log-probs of the K largest entries: value descending, then entry ascending; -1 / -inf left over."""
    B, T, V = z.shape
    lq = torch.log_softmax(z / temperature, dim=2)
    top, at = z.sort(dim=2, descending=True, stable=True)
    k = min(K, V)
    ids = torch.full((B, T, K), -1, dtype=torch.int64, device=z.device)
    lp = torch.full((B, T, K), float("-inf"), dtype=torch.float64, device=z.device)
    keep = top[..., :k] > float("-inf")
    ids[..., :k] = torch.where(keep, at[..., :k], -1)
    lp[..., :k] = torch.where(keep, lq.gather(2, at[..., :k]), float("-inf"))
    pad = ~valid_mask(lengths, T)
    ids[pad], lp[pad] = 0, 0.0
    return ids, lp


def distill(z, topk_ids, topk_logprobs, lengths, mode, temperature, grad_scale):
    """loss, row losses, dlogits and, entry by entry, the absolute parts of the gradient."""
    B, T, V = z.shape
    valid = valid_mask(lengths, T)
    ids = topk_ids.long()
    used = (ids >= 0) & (ids < V)
    at = torch.where(used, ids, 0)
    lt = torch.where(used, topk_logprobs.double(), float("-inf"))
    if mode == 1:
        norm = torch.logsumexp(lt, dim=2, keepdim=True)
        lt = torch.where(torch.isinf(norm), float("-inf"), lt - norm)
    p = torch.exp(lt)
    lq = torch.log_softmax(z / temperature, dim=2)
    named = torch.zeros_like(lq).scatter_add_(2, at, used.double()) > 0
    target = torch.zeros_like(lq).scatter_add_(2, at, p)
    P = p.sum(dim=2, keepdim=True)
    L = torch.where(p > 0, p * (lt - lq.gather(2, at)), 0.0).sum(dim=2)
    q = lq.exp()
    W, out = P, P
    if mode == 2:
        p0 = (1 - P).clamp(min=0)
        l0 = torch.logsumexp(lq.masked_fill(named, float("-inf")), dim=2, keepdim=True)
        there = (p0 > 0) & (l0 > float("-inf"))
        L = L + torch.where(there, p0 * (torch.log(p0) - l0), 0.0)[..., 0]
        W = torch.where(there, P + p0, P)
        out = torch.where(there, W - p0 * torch.exp(-l0), P)
        size = torch.where(there, W + p0 * torch.exp(-l0), P)
    else:
        size = P
    N = valid.sum().clamp(min=1)
    k = grad_scale * temperature / N
    d = k * (torch.where(named, W, out) * q - target)
    parts = abs(k) * (torch.where(named, W, size) * q + target)
    d = torch.where(valid[..., None], d, 0.0)
    rows = torch.where(valid, temperature ** 2 * L, 0.0)
    return rows.sum() / N, rows, d, torch.where(valid[..., None], parts, 0.0)
