"""The operators on shaped logits and the router's balance loss written out in float64 torch, row by row, for the tests.
Shares no code with the library."""
from __future__ import annotations

import torch


class Settings:
    """Random settings of a rollout for B sequences, T rows and V entries; `parts` names what is given."""

    def __init__(self, B, T, V, gen, device, parts, P=0, S0=0, repeat=8, mask_density=0.5):
        u = lambda *n: torch.rand(n, generator=gen, device=device)  # noqa: E731
        few = torch.randint(0, V, (B, repeat), generator=gen, device=device)
        some = lambda n: few.gather(1, (u(B, n) * repeat).long().clamp(max=repeat - 1))  # noqa: E731
        kw = self.kw = {}
        if "tokens" in parts:
            kw["tokens"] = some(S0 + T)
            if S0:
                kw["start"] = (u(B) * (S0 + 1)).int().clamp(max=S0)
                kw["start"][0] = S0
        if "prompt" in parts and P:
            kw["prompt"] = some(P)
            kw["prompt"][:, ::3] = -1
            kw["prompt_lengths"] = (u(B) * (P + 1)).int().clamp(max=P)
            kw["prompt_lengths"][0] = P
        for name, lo, hi in (("repetition", 0.7, 1.6), ("frequency", -0.3, 0.6), ("presence", -0.3, 0.6), ("temperature", 0.5, 2.0)):
            if name in parts:
                kw[name] = lo + (hi - lo) * u(B)
        if "bias" in parts or "bias_own" in parts:
            n = (V,) if "bias" in parts else (B, V)
            kw["bias"] = torch.where(u(*n) < 0.3, 2 * torch.randn(n, generator=gen, device=device), 0.0)
        if "mask" in parts or "mask_rows" in parts:
            W = (V + 31) // 32
            allowed = u(B, T if "mask_rows" in parts else 1, W * 32) < mask_density
            kw["mask"] = pack_mask(allowed)


def pack_mask(allowed):
    bits = allowed.long().unflatten(-1, (-1, 32)) << torch.arange(32, device=allowed.device)
    words = bits.sum(dim=-1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()


ALL = ("tokens", "prompt", "repetition", "frequency", "presence", "temperature")


def shaped(z, lengths, kw):
    """x, dx/dz, and a bound of the absolute parts that x is summed from (0 where x is z itself), [B,T,V] float64; x is 0 at
    padding."""
    z = z.double()
    B, T, V = z.shape
    dev = z.device
    x, scale, parts = torch.zeros_like(z), torch.zeros_like(z), torch.zeros_like(z)
    value = lambda n, b, d: float(kw[n][b].double()) if n in kw else d  # noqa: E731
    for b in range(B):
        n = max(0, min(T, int(lengths[b])))
        start = max(0, int(kw["start"][b])) if "start" in kw else 0
        asked = set()
        if "prompt" in kw:
            m = int(kw["prompt_lengths"][b]) if "prompt_lengths" in kw else kw["prompt"].shape[1]
            asked = {v for v in kw["prompt"][b, :max(0, m)].tolist() if 0 <= v < V}
        tokens = kw["tokens"][b].tolist() if "tokens" in kw else []
        r, f, p, tau = (value(k, b, d) for k, d in (("repetition", 1.0), ("frequency", 0.0), ("presence", 0.0), ("temperature", 1.0)))
        for t in range(n):
            count = torch.zeros(V, dtype=torch.float64, device=dev)
            before = [v for v in tokens[:start + t] if 0 <= v < V]
            if before:
                count = torch.bincount(torch.tensor(before, device=dev), minlength=V).double()
            seen = count > 0
            if asked:
                seen[torch.tensor(sorted(asked), device=dev)] = True
            row = z[b, t]
            by = torch.where(seen, torch.where(row < 0, r, 1 / r), torch.ones_like(row)) if "repetition" in kw else torch.ones_like(row)
            a = row * by - f * count - p * (count > 0)
            size = (row * by).abs() + abs(f) * count + abs(p) * (count > 0)
            moved = seen.clone()
            if "bias" in kw:
                bias = (kw["bias"] if kw["bias"].dim() == 1 else kw["bias"][b]).double()
                a, size, moved = a + bias, size + bias.abs(), moved | (bias != 0)
            a, size = a / tau, size / tau
            if "temperature" in kw:
                moved = torch.ones_like(moved)
            d = by / tau
            if "mask" in kw:
                words = kw["mask"][b if kw["mask"].shape[0] > 1 else 0]
                words = words if words.dim() == 1 else words[t if words.shape[0] > 1 else 0]
                ok = ((words[:, None] >> torch.arange(32, device=dev)) & 1).bool().flatten()[:V]
                a, d = torch.where(ok, a, float("-inf")), torch.where(ok, d, 0.0)
                size = torch.where(ok, size, 0.0)
            x[b, t], scale[b, t] = a, d
            parts[b, t] = torch.where(moved, size, 0.0)
    return x, scale, parts


def logprobs(x, ids, lengths):
    """Log-probs, entropy and log p of every entry; a row without mass: -inf, 0, -inf."""
    B, T, V = x.shape
    valid = torch.arange(T, device=x.device)[None] < lengths.clamp(0, T)[:, None]
    some = (x > float("-inf")).any(dim=2)
    lq = torch.where(some[..., None], torch.log_softmax(torch.where(some[..., None], x, 0.0), dim=2), float("-inf"))
    known = valid & (ids >= 0) & (ids < V)
    lp = torch.where(known, lq.gather(2, ids.clamp(0, V - 1)[..., None])[..., 0], 0.0)
    entropy = torch.where(valid, torch.special.entr(lq.exp()).sum(dim=2), 0.0)
    return lp, entropy, lq, valid, known


def logprobs_grad(x, scale, ids, lengths, g, h):
    """The gradient of sum g lp + sum h entropy with respect to the logits and, entry by entry, its absolute parts."""
    B, T, V = x.shape
    lp, entropy, lq, valid, known = logprobs(x, ids, lengths)
    p = lq.exp()
    one = torch.nn.functional.one_hot(ids.clamp(0, V - 1), V).double() * known[..., None]
    g = torch.where(known, g.double(), 0.0)[..., None]
    own = torch.where(one > 0, -torch.expm1(lq), -p)
    d, parts = g * own, g.abs() * (one + p)
    if h is not None:
        h = torch.where(valid, h.double(), 0.0)[..., None]
        ent = -torch.special.entr(p) + p * entropy[..., None]
        d = d - h * ent
        parts = parts + h.abs() * (torch.special.entr(p).abs() + p * entropy[..., None])
    live = (x > float("-inf")) & valid[..., None]
    return torch.where(live, d * scale, 0.0), torch.where(live, parts * scale.abs(), 0.0)


def router(z, lengths, k, scoring, per_sequence, balance_coef, z_coef, grad_scale, expert_ids=None):
    """losses [L,2], counts, ids, dlogits and, entry by entry, the absolute parts of the gradient."""
    z = z.double()
    L, B, T, E = z.shape
    n = [max(0, min(T, int(v))) for v in lengths]
    N, filled = sum(n), sum(v > 0 for v in n)
    loss = torch.zeros((L, 2), dtype=torch.float64, device=z.device)
    counts = torch.zeros((L, B, E), dtype=torch.int64, device=z.device)
    ids = torch.zeros((L, B, T, k), dtype=torch.int32, device=z.device)
    d, parts = torch.zeros_like(z), torch.zeros_like(z)
    for b in range(B):
        pick = z[:, b, :n[b]].sort(dim=2, descending=True, stable=True).indices[..., :k].int() if expert_ids is None else expert_ids[:, b, :n[b]]
        ids[:, b, :n[b]] = pick
        for l in range(L):
            v = pick[l].flatten().long()
            counts[l, b] = torch.bincount(v[(v >= 0) & (v < E)], minlength=E)
    total = counts.sum(dim=1)
    for b in range(B):
        if n[b] == 0:
            continue
        c = counts[:, b] if per_sequence else total
        m = n[b] if per_sequence else N
        f = (c.double() * E / (k * m))[:, None]
        w = 1 / (m * filled) if per_sequence else 1 / m
        y = z[:, b, :n[b]]
        if scoring == 0:
            none = (y == float("-inf")).all(dim=2, keepdim=True)
            y = torch.where(none, 0.0, y)
            p, rise = torch.where(none, 0.0, torch.softmax(y, dim=2)), torch.ones_like(y)
        else:
            s = torch.sigmoid(y)
            p, rise = s / s.sum(dim=2, keepdim=True), torch.sigmoid(-y)
        dot = (p * f).sum(dim=2, keepdim=True)
        loss[:, 0] += w * dot.sum(dim=(1, 2))
        g = balance_coef * w * rise * p * (f - dot)
        a = abs(balance_coef) * w * rise * p * (1 + f.abs() + dot.abs())
        if z_coef:
            lse = torch.logsumexp(y, dim=2, keepdim=True)
            loss[:, 1] += (lse ** 2).sum(dim=(1, 2)) / N
            g = g + z_coef * 2 / N * lse * p
            a = a + (z_coef * 2 / N * lse * p).abs()
        d[:, b, :n[b]], parts[:, b, :n[b]] = grad_scale * g, abs(grad_scale) * a
    return loss, (counts if per_sequence else total).int(), ids, d, parts
