"""Cases of the training objectives over a [B,T,V] logits tensor that stand beside the PPO loss: the teacher's top-K
log-probs, distillation from them, the clipped policy loss with its KL term, and the preference loss over pairs of
sequences.  `run` computes a case in elementary torch operations, or through the library where `own` is set.

A case:  op, B, T, V, K (teacher entries per row; 0 where there are none), dtype ("bf16" | "fp16"), lengths ("full" |
"uniform" | "mixture"), P (prompt rows that precede the responses in memory: the logits are a view of [B,P+T,V]),
deleted (share of the vocabulary at -inf on a quarter of the rows), and what the operator takes beside them.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------- the cases
def _topk(name, **kw):
    return dict(dict(name=name, op="topk", dtype="bf16", lengths="uniform", P=0, deleted=0.0, temperature=1.0), **kw)


def _distill(name, **kw):
    return dict(dict(name=name, op="distill", dtype="bf16", lengths="uniform", P=0, deleted=0.0, temperature=1.0,
                     mode="plain"), **kw)


def _policy(name, **kw):
    return dict(dict(name=name, op="policy", K=0, dtype="bf16", lengths="uniform", P=0, deleted=0.0, clip_low=0.2,
                     clip_high=0.28, kl_coef=0.04, reduction="tokens", adv="sequence"), **kw)


def _preference(name, **kw):
    return dict(dict(name=name, op="preference", K=0, dtype="bf16", lengths="uniform", P=0, deleted=0.0, kind="sigmoid",
                     beta=0.1, margin=0.0, smoothing=0.0, length_mean=False), **kw)


def listed():
    return [
        # one scored position of an OPT-shaped teacher: latency
        _topk("topk_one_row", B=1, T=1, V=50272, K=20, lengths="full"),
        # a teacher's pass over an OPT-shaped batch of responses
        _topk("topk_opt", B=16, T=256, V=50272, K=64),
        # large vocabulary, many entries kept, behind a prompt
        _topk("topk_large_vocab", B=8, T=512, V=128256, K=128, P=16, temperature=2.0),
        # a toy student: latency
        _distill("distill_tiny", B=2, T=16, V=1000, K=8, mode="normalised"),
        # GPT-2 vocabulary (rows off 16-byte boundaries) in fp16, an odd number of entries
        _distill("distill_gpt2_fp16", B=16, T=256, V=50257, K=50, dtype="fp16", temperature=2.0),
        # large vocabulary, the mass outside the teacher's entries as one more class
        _distill("distill_large_vocab", B=16, T=512, V=128256, K=64, mode="tail", lengths="full"),
        # a policy step on a toy model: latency
        _policy("policy_tiny", B=2, T=16, V=1000),
        # Llama-2-shaped batch, every sequence of the same weight
        _policy("policy_llama2_fp16", B=32, T=512, V=32000, dtype="fp16", reduction="sequences"),
        # large vocabulary, ragged responses (empty ones among them), advantages per token
        _policy("policy_large_vocab", B=16, T=512, V=128256, lengths="mixture", adv="token"),
        # one pair of short answers
        _preference("preference_one_pair", B=2, T=32, V=32000, lengths="full"),
        # a batch of pairs, OPT shape
        _preference("preference_opt", B=16, T=256, V=50272, smoothing=0.1),
        # pairs over a large vocabulary, log ratios averaged over the answer's length
        _preference("preference_large_vocab", B=8, T=512, V=128256, kind="squared", length_mean=True, beta=0.5),
    ]


# logits of the largest listed case of each operator: no drawn case has more
_MOST = {"topk": 8 * 512 * 128256, "distill": 16 * 512 * 128256, "policy": 16 * 512 * 128256, "preference": 8 * 512 * 128256}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["topk", "distill", "policy", "preference"])
    V = rng.choice([32000, 50257, 50272, 128256, _log(rng, 500, 160000), _log(rng, 500, 160000)])
    T = _log(rng, 1, 1024)
    B = _log(rng, 1, 64)
    if op == "preference":
        B = max(2, B // 2 * 2)
    while B * T * V > _MOST[op]:
        if T > 1 and (rng.random() < 0.5 or B <= 2):
            T = max(1, T // 2)
        else:
            B = max(2 if op == "preference" else 1, B // 4 * 2)
    P = rng.choice([0, 0, 1, min(T, 64)])
    while B * (P + T) * V > 1.25 * _MOST[op]:
        P //= 2
    case = dict(B=B, T=T, V=V, P=P, dtype=rng.choice(["bf16", "bf16", "fp16"]),
                lengths=rng.choice(["full", "uniform", "mixture"]), deleted=rng.choice([0.0, 0.0, 0.02]))
    if op == "topk":
        c = _topk("", K=_log(rng, 1, 256), temperature=rng.choice([1.0, 1.0, 0.7, 2.0]))
    elif op == "distill":
        c = _distill("", K=min(V, _log(rng, 1, 256)), temperature=rng.choice([1.0, 1.0, 2.0, 1.5]),
                     mode=rng.choice(["plain", "normalised", "tail"]))
    elif op == "policy":
        c = _policy("", kl_coef=rng.choice([0.0, 0.04, 0.2]), reduction=rng.choice(["tokens", "sequences"]),
                    adv=rng.choice(["token", "sequence"]), clip_high=rng.choice([0.2, 0.28]))
    else:
        kind = rng.choice(["sigmoid", "hinge", "squared"])
        c = _preference("", kind=kind, beta=rng.choice([0.1, 0.5]), margin=rng.choice([0.0, 0.5]),
                        smoothing=rng.choice([0.0, 0.1]) if kind == "sigmoid" else 0.0, length_mean=rng.random() < 0.5)
    c.update(case)
    del c["name"]
    return c


def _mean_length(case):
    T = case["T"]
    if case["lengths"] == "full":
        return T
    if case["lengths"] == "uniform":
        return ((T + 1) // 2 + T) / 2
    return 0.65 * (min(3, T) + T) / 2 + 0.15 * min(2, T) + 0.15


def work(case):
    rows, valid, V, K = case["B"] * case["T"], case["B"] * _mean_length(case), case["V"], case["K"]
    if case["op"] == "topk":
        return {"bytes": 2 * V * valid + 8 * K * rows, "flops": 4.0 * V * valid}
    return {"bytes": 2 * V * (valid + rows) + 8 * K * valid + 24 * rows, "flops": 6.0 * V * valid}


# ---------------------------------------------------------------- the inputs
def _lengths(case, gen):
    B, T = case["B"], case["T"]
    full = torch.full((B,), T, dtype=torch.int32)
    if case["lengths"] == "full":
        return full
    if case["lengths"] == "uniform":
        return torch.randint((T + 1) // 2, T + 1, (B,), generator=gen, dtype=torch.int32)
    u = torch.rand((B,), generator=gen)
    out = torch.randint(min(3, T), T + 1, (B,), generator=gen, dtype=torch.int32)
    out[u < 0.35] = min(2, T)
    out[u < 0.20] = 1
    out[u < 0.05] = 0
    out[0] = T                                        # at least one whole answer
    return out


def prepare(case, seed):
    """The logits of a batch, the generated tokens (or the teacher's entries for them) and the per-token arrays of the
    objective, as the passes before it leave them on the device."""
    dev = "cuda"
    B, T, V, P, K, op = (case[k] for k in ("B", "T", "V", "P", "K", "op"))
    cpu = torch.Generator().manual_seed(seed * 7919 + 11)
    gen = torch.Generator(device=dev).manual_seed(seed * 7919 + 13)
    lengths = _lengths(case, cpu)
    # rows of one tensor; the rows before a sequence's responses are the prompt's, which no operator reads
    full = torch.empty((B, P + T, V), dtype=DTYPES[case["dtype"]], device=dev)
    logits = full[:, P:]
    s = {"case": dict(case), "logits": logits, "lengths": lengths.to(dev)}
    r = lambda *n: torch.randn(n, generator=gen, device=dev)  # noqa: E731
    if op == "distill":
        s["topk_ids"] = torch.empty((B, T, K), dtype=torch.int32, device=dev)
        s["topk_logprobs"] = torch.empty((B, T, K), dtype=torch.float32, device=dev)
    if op in ("policy", "preference"):
        s["ids"] = torch.empty((B, T), dtype=torch.int64, device=dev)
        lp = torch.empty((B, T), device=dev)
    step = max(1, (1 << 27) // ((P + T) * V))
    for b in range(0, B, step):
        z = 3.0 * r(min(B, b + step) - b, P + T, V)
        if case["deleted"]:
            hit = torch.rand(z.shape[:2] + (1,), generator=gen, device=dev) < 0.25
            cut = torch.rand(z.shape, generator=gen, device=dev) < case["deleted"]
            cut[..., 0] = False
            z = z.masked_fill(cut & hit, float("-inf"))
        full[b:b + step] = z
        x = full[b:b + step, P:].float()
        if op == "distill":
            # a teacher about a nat away from the student; its log-probs at the loss's temperature
            t = (x + 1.5 * r(*x.shape)) / case["temperature"]
            top, at = t.topk(K, dim=2)
            top = top - torch.logsumexp(t, dim=2, keepdim=True)
            s["topk_logprobs"][b:b + step] = top
            s["topk_ids"][b:b + step] = torch.where(top > float("-inf"), at, -1).int()
        elif op in ("policy", "preference"):
            # tokens sampled from the model; no deleted entry among them
            e = -torch.log(torch.rand(x.shape, generator=gen, device=dev).clamp_(1e-12, 1 - 1e-7))
            y = (x - torch.log(e)).argmax(dim=2, keepdim=True)
            s["ids"][b:b + step] = y[..., 0]
            lp[b:b + step] = (x.gather(2, y) - torch.logsumexp(x, dim=2, keepdim=True))[..., 0]
    valid = torch.arange(T, device=dev)[None] < s["lengths"][:, None]
    if op == "policy":
        s["lp_old"] = (lp + 0.1 * r(B, T)) * valid
        s["lp_ref"] = (lp + 0.3 * r(B, T)) * valid
        s["adv"] = r(B) if case["adv"] == "sequence" else r(B, T)
    if op == "preference":
        s["lp_ref"] = (lp + 0.3 * r(B, T)) * valid
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    if own:
        return _own(s)
    return {"topk": _plain_topk, "distill": _plain_distill, "policy": _plain_policy, "preference": _plain_preference}[s["case"]["op"]](s)


def _own(s):
    from paper_2410_15651_b200 import binding as lib
    c, z, n = s["case"], s["logits"], s["lengths"]
    if "ws" not in s:
        s["ws"] = lib.workspace(c["B"], c["T"], z.device)
    ws = s["ws"]
    if c["op"] == "topk":
        o = lib.topk_logprobs(z, n, c["K"], c["temperature"], ws)
        return {"ids": o.ids, "logprobs": o.logprobs}
    if c["op"] == "distill":
        mode = {"plain": lib.DISTILL_PLAIN, "normalised": lib.DISTILL_NORMALISED, "tail": lib.DISTILL_TAIL}[c["mode"]]
        o = lib.distill_loss_fwd_bwd(z, s["topk_ids"], s["topk_logprobs"], n, mode, c["temperature"], 1000.0, ws)
        return {"loss": o.loss, "dlogits": o.dlogits, "row_loss": o.row_loss}
    if c["op"] == "policy":
        red = {"tokens": lib.MEAN_TOKENS, "sequences": lib.MEAN_SEQUENCES}[c["reduction"]]
        o = lib.policy_kl_loss_fwd_bwd(z, s["ids"], n, s["lp_old"], s["lp_ref"], s["adv"], c["clip_low"], c["clip_high"],
                                       c["kl_coef"], red, 1000.0, ws)
        return {"loss": o.loss, "dlogits": o.dlogits, "lp_new": o.lp_new}
    kind = {"sigmoid": lib.PREF_SIGMOID, "hinge": lib.PREF_HINGE, "squared": lib.PREF_SQUARED}[c["kind"]]
    o = lib.preference_loss_fwd_bwd(z, s["ids"], n, s["lp_ref"], kind, c["beta"], c["margin"], c["smoothing"],
                                    c["length_mean"], 1000.0, ws)
    return {"loss": o.loss, "dlogits": o.dlogits, "rewards": o.rewards, "lp_new": o.lp_new}


# Gradients are scaled by 1000, as with loss scaling, so that fp16 holds them.
_SCALE = 1000.0


def _valid(s):
    c = s["case"]
    return torch.arange(c["T"], device=s["lengths"].device)[None] < s["lengths"][:, None]


def _log_softmax(z):
    m = z.amax(dim=2, keepdim=True)
    return z - (m + torch.log(torch.exp(z - m).sum(dim=2, keepdim=True)))


def _plain_topk(s):
    c, z, valid = s["case"], s["logits"], _valid(s)[..., None]
    K, k = c["K"], min(c["K"], c["V"])
    lq = _log_softmax(z.float() / c["temperature"])
    # one whole number per entry: its value's order, then the lower index first
    b = z.contiguous().view(torch.int16).long()
    key = torch.where(b >= 0, b, -32768 - b) * (1 << 32) - torch.arange(c["V"], device=z.device)
    at = key.topk(k, dim=2).indices
    lp = lq.gather(2, at)
    ids = torch.where(lp > float("-inf"), at, -1).int()
    ids = torch.nn.functional.pad(ids, (0, K - k), value=-1)
    lp = torch.nn.functional.pad(lp, (0, K - k), value=float("-inf"))
    return {"ids": torch.where(valid, ids, 0), "logprobs": torch.where(valid, lp, 0.0)}


def _plain_distill(s):
    c, valid = s["case"], _valid(s)
    tau, ids, lt = c["temperature"], s["topk_ids"].long(), s["topk_logprobs"]
    used = ids >= 0
    at = ids.clamp(min=0)
    # a row's loss is a small difference of log-probs: those of the teacher's entries are held in 64 bits
    z = s["logits"].float() / tau
    m = z.amax(dim=2, keepdim=True)
    q = torch.exp(z - m)
    sums = q.sum(dim=2, keepdim=True, dtype=torch.float64)
    lq = s["logits"].gather(2, at).double() / tau - (m.double() + torch.log(sums))
    q = q / sums.float()
    lt = lt.double()
    p = torch.where(used, torch.exp(lt), 0.0)
    total = p.sum(dim=2, keepdim=True)
    if c["mode"] == "normalised":
        lt = lt - torch.log(total)
        p = p / total
        total = torch.ones_like(total)
    row = torch.where(p > 0, p * (lt - lq), 0.0).sum(dim=2)
    d = total.float() * q
    if c["mode"] == "tail":
        p0 = (1 - total).clamp(min=0)
        inside = torch.zeros_like(q).scatter_reduce_(2, at, used.float(), "amax") > 0
        q0 = torch.where(inside, 0.0, q).sum(dim=2, keepdim=True, dtype=torch.float64)
        row = row + torch.where(p0 > 0, p0 * (torch.log(p0) - torch.log(q0)), 0.0)[..., 0]
        whole = (total + p0).float()
        d = torch.where(inside, whole, whole - torch.where(p0 > 0, p0 / q0, 0.0).float()) * q
    d = d.scatter_add_(2, at, -p.float())
    n = valid.sum().clamp(min=1)
    row = torch.where(valid, row * tau * tau, 0.0).float()
    d = torch.where(valid[..., None], d * (_SCALE * tau / n), 0.0)
    return {"loss": (row.double().sum() / n).float().reshape(1), "dlogits": d.to(s["logits"].dtype), "row_loss": row}


def _label_grad(s, q, g):
    """g * ([v == y] - q_v) for every row, in the logits' type."""
    y = s["ids"][..., None]
    d = -q
    d.scatter_(2, y, 1.0 - q.gather(2, y))
    return torch.where(_valid(s)[..., None], d * g[..., None], 0.0).to(s["logits"].dtype)


def _plain_policy(s):
    c, valid = s["case"], _valid(s)
    A = s["adv"] if s["adv"].dim() == 2 else s["adv"][:, None]
    lq = _log_softmax(s["logits"].float())
    lp = torch.where(valid, lq.gather(2, s["ids"][..., None])[..., 0], 0.0)
    rho = torch.exp(lp - s["lp_old"])
    plain, clipped = -A * rho, -A * rho.clamp(1 - c["clip_low"], 1 + c["clip_high"])
    d = (s["lp_ref"] - lp).double()
    pg, kl = torch.maximum(plain, clipped), (torch.expm1(d) - d).float()
    n = s["lengths"].float()[:, None]
    if c["reduction"] == "tokens":
        w = valid / n.sum().clamp(min=1)
    else:
        w = valid / (n.clamp(min=1) * (n > 0).sum().clamp(min=1))
    g = _SCALE * w * (torch.where(plain >= clipped, plain, 0.0) - c["kl_coef"] * torch.expm1(d).float())
    loss = torch.stack([(pg * w).double().sum(), (kl * w).double().sum()]).float()
    return {"loss": loss, "dlogits": _label_grad(s, torch.exp(lq), g), "lp_new": lp}


def _plain_preference(s):
    c, valid = s["case"], _valid(s)
    half, beta = c["B"] // 2, c["beta"]
    lq = _log_softmax(s["logits"].float())
    lp = torch.where(valid, lq.gather(2, s["ids"][..., None])[..., 0], 0.0)
    n = s["lengths"].double()
    w = 1 / n.clamp(min=1) if c["length_mean"] else torch.ones_like(n)
    ratio = (torch.where(valid, lp.double() - s["lp_ref"].double(), 0.0)).sum(dim=1) * w
    h = beta * (ratio[:half] - ratio[half:]) - c["margin"]
    if c["kind"] == "sigmoid":
        e = c["smoothing"]
        loss = (1 - e) * torch.log1p(torch.exp(-h.abs())) + (1 - e) * (-h).clamp(min=0) + e * (torch.log1p(torch.exp(-h.abs())) + h.clamp(min=0))
        dh = e - torch.sigmoid(-h)
    elif c["kind"] == "hinge":
        loss = (1 - h).clamp(min=0)
        dh = -(h < 1).double()
    else:
        loss = (h - 0.5) ** 2 / beta ** 2
        dh = 2 * (h - 0.5) / beta ** 2
    g = (_SCALE / half) * beta * torch.cat([dh, -dh]) * w
    return {"loss": loss.mean().float().reshape(1), "dlogits": _label_grad(s, torch.exp(lq), g.float()[:, None].expand(-1, c["T"])),
            "rewards": (beta * ratio).float(), "lp_new": lp}


# ---------------------------------------------------------------- the definitions in 64 bits, a sequence at a time
def exact(case, seed):
    s = prepare(case, seed)
    B, T, V, K, op = case["B"], case["T"], case["V"], case["K"], case["op"]
    dev = s["logits"].device
    lens = s["lengths"].tolist()
    N = max(1, sum(lens))
    if op == "topk":
        ids = torch.zeros((B, T, K), dtype=torch.int32, device=dev)
        out = torch.zeros((B, T, K), dtype=torch.float64, device=dev)
        for b, n in enumerate(lens):
            z = s["logits"][b, :n].double()
            top, at = z.sort(dim=1, descending=True, stable=True)
            top, at = top[:, :K] / case["temperature"], at[:, :K]
            k = top.shape[1]
            ids[b, :n], out[b, :n] = -1, float("-inf")
            out[b, :n, :k] = top - torch.logsumexp(z / case["temperature"], dim=1, keepdim=True)
            ids[b, :n, :k] = torch.where(top.isfinite(), at, -1).int()
        return {"ids": ids, "logprobs": out}
    grad = torch.zeros((B, T, V), dtype=torch.float64, device=dev)
    if op == "distill":
        tau = case["temperature"]
        row = torch.zeros((B, T), dtype=torch.float64, device=dev)
        for b, n in enumerate(lens):
            lq = torch.log_softmax(s["logits"][b, :n].double() / tau, dim=1)
            ids, lt = s["topk_ids"][b, :n].long(), s["topk_logprobs"][b, :n].double()
            lt = torch.where(ids >= 0, lt, float("-inf"))
            if case["mode"] == "normalised":
                lt = torch.log_softmax(lt, dim=1)
            p = lt.exp()
            # targets over the whole vocabulary; unused entries add 0 to column 0
            target = torch.zeros_like(lq).scatter_add_(1, ids.clamp(min=0), p)
            ent = torch.where(p > 0, p * lt, 0.0).sum(dim=1)
            loss = ent - torch.where(target > 0, target * lq, 0.0).sum(dim=1)
            d = p.sum(dim=1, keepdim=True) * lq.exp() - target
            if case["mode"] == "tail":
                rest = (1 - p.sum(dim=1)).clamp(min=0)
                names = torch.zeros_like(lq)
                names.scatter_add_(1, ids.clamp(min=0), (ids >= 0).double())
                lr = lq.masked_fill(names > 0, float("-inf"))
                l0 = torch.logsumexp(lr, dim=1)
                loss = loss + torch.where(rest > 0, rest * (rest.log() - l0), 0.0)
                d = d + rest[:, None] * (lq.exp() - torch.where(names > 0, 0.0, (lr - l0[:, None]).exp()))
            row[b, :n] = tau * tau * loss
            grad[b, :n] = d * (1000.0 * tau / N)
        return {"loss": row.sum().reshape(1) / N, "dlogits": grad, "row_loss": row}
    lp = torch.zeros((B, T), dtype=torch.float64, device=dev)
    for b, n in enumerate(lens):
        lq = torch.log_softmax(s["logits"][b, :n].double(), dim=1)
        y = s["ids"][b, :n, None]
        lp[b, :n] = lq.gather(1, y)[:, 0]
        grad[b, :n] = lq.exp_().neg_().scatter_add_(1, y, torch.ones_like(y, dtype=torch.float64))
    if op == "policy":
        filled = sum(n > 0 for n in lens)
        losses, coef = [0.0, 0.0], torch.zeros_like(lp)
        for b, n in enumerate(lens):
            if n == 0:
                continue
            w = 1 / N if case["reduction"] == "tokens" else 1 / (n * filled)
            A = s["adv"][b].double() if case["adv"] == "sequence" else s["adv"][b, :n].double()
            rho = (lp[b, :n] - s["lp_old"][b, :n].double()).exp()
            d = s["lp_ref"][b, :n].double() - lp[b, :n]
            bound = rho.clamp(1 - case["clip_low"], 1 + case["clip_high"])
            free = rho * A <= bound * A
            losses[0] += -(torch.minimum(rho * A, bound * A)).sum() * w
            losses[1] += (d.expm1() - d).sum() * w
            coef[b, :n] = 1000.0 * w * (-(A * rho * free) + case["kl_coef"] * (1 - d.exp()))
        return {"loss": torch.stack([torch.as_tensor(x, dtype=torch.float64, device=dev) for x in losses]),
                "dlogits": grad.mul_(coef[..., None]), "lp_new": lp}
    half, beta = B // 2, case["beta"]
    w = [1 / max(1, n) if case["length_mean"] else 1.0 for n in lens]
    rewards = torch.stack([beta * w[b] * (lp[b, :n] - s["lp_ref"][b, :n].double()).sum() for b, n in enumerate(lens)])
    loss = torch.zeros((), dtype=torch.float64, device=dev)
    coef = torch.zeros((B,), dtype=torch.float64, device=dev)
    for i in range(half):
        h = rewards[i] - rewards[half + i] - case["margin"]
        if case["kind"] == "sigmoid":
            e, up, down = case["smoothing"], torch.nn.functional.logsigmoid(h), torch.nn.functional.logsigmoid(-h)
            loss, dh = loss - (1 - e) * up - e * down, -(1 - e) * down.exp() + e * up.exp()
        elif case["kind"] == "hinge":
            loss, dh = loss + (1 - h).clamp(min=0), torch.where(h < 1, -1.0, 0.0)
        else:
            loss, dh = loss + ((h - 0.5) / beta) ** 2, 2 * (h - 0.5) / beta ** 2
        coef[i], coef[half + i] = dh * beta * w[i], -dh * beta * w[half + i]
    return {"loss": loss.reshape(1) / half, "dlogits": grad.mul_(coef[:, None, None] * (1000.0 / half)), "rewards": rewards,
            "lp_new": lp}
