"""Cases of the operators on shaped logits (penalties for repeated tokens, bias, grammar mask and temperature between a
model's logits and the distribution its tokens are drawn from) and of the balance loss of a policy's expert router.  `run`
computes a case in elementary torch operations, or through the library where `own` is set.

A case on logits:  op, B, T, V, pitch (entries between the rows beyond V: a padded vocabulary), P (prompt tokens), S0 (most
response tokens before the first row), dtype ("bf16" | "fp16"), lengths ("full" | "uniform" | "mixture"), repetition,
frequency, presence, temperature (truth values: per-sequence settings are given), bias ("none" | "shared" | "own"), mask
("none" | "sequence" | "row"), out32 (shaped logits in fp32), entropy (with the entropy, or its gradient).
A case of the router:  op, L, B, T, E, K, dtype ("bf16" | "fp16" | "fp32"), lengths, scoring ("softmax" | "sigmoid"), scope ("batch" |
"sequence"), z (with the z-loss), given (the chosen experts are inputs).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---------------------------------------------------------------- the cases
def _logits(op, name, **kw):
    return dict(dict(name=name, op=op, pitch=0, P=0, S0=0, dtype="bf16", lengths="uniform", repetition=True, frequency=False,
                     presence=False, temperature=True, bias="none", mask="none", out32=False, entropy=False), **kw)


def _router(name, **kw):
    return dict(dict(name=name, op="router", dtype="bf16", lengths="uniform", scoring="softmax", scope="batch", z=False,
                     given=False), **kw)


def listed():
    return [
        # one step of one rollout: latency
        _logits("shape", "shape_one_token", B=1, T=1, V=50272, P=64, S0=32, lengths="full", frequency=True, presence=True),
        # a step of a batch of rollouts over a large vocabulary, a grammar per sequence, fp32 for the sampler
        _logits("shape", "shape_decode", B=128, T=1, V=128256, P=2048, S0=512, lengths="full", frequency=True,
                presence=True, mask="sequence", out32=True),
        # all positions of the answers of a batch at once, for a loss: GPT-2 vocabulary (rows off 16-byte boundaries) in fp16
        _logits("shape", "shape_gpt2_fp16", B=16, T=256, V=50257, P=128, dtype="fp16", presence=True, bias="shared"),
        # the gradient through the shaping: a toy model, latency
        _logits("shape_bwd", "shape_bwd_tiny", B=2, T=16, V=1000, P=8),
        # the gradient of a Llama-2-shaped batch
        _logits("shape_bwd", "shape_bwd_llama2", B=32, T=512, V=32000, P=256, mask="sequence"),
        # log-probs of one pair of short answers
        _logits("logprobs", "logprobs_one_pair", B=2, T=32, V=32000, P=32, lengths="full", frequency=True),
        # the experience pass over a large vocabulary, a grammar mask per row, with the entropy
        _logits("logprobs", "logprobs_large_vocab", B=16, T=512, V=128256, P=512, mask="row", entropy=True),
        # the update of an OPT-shaped batch, frequency and presence penalties
        _logits("logprobs_bwd", "logprobs_bwd_opt", B=16, T=256, V=50272, P=256, frequency=True, presence=True),
        # the update over a large vocabulary, ragged answers (empty ones among them), with an entropy bonus
        _logits("logprobs_bwd", "logprobs_bwd_large_vocab", B=16, T=512, V=128256, P=512, lengths="mixture", entropy=True),
        # the router of one layer of a toy model: latency
        _router("router_tiny", L=1, B=2, T=16, E=8, K=2, dtype="fp32"),
        # one layer's router, fp32 logits, normalised sigmoid scores, a loss per sequence, experts chosen elsewhere
        _router("router_layer_fp32", L=1, B=16, T=1024, E=256, K=8, dtype="fp32", scoring="sigmoid", scope="sequence",
                given=True),
        # all layers of a model at once, with the z-loss
        _router("router_model", L=24, B=16, T=1024, E=128, K=8, z=True),
    ]


# logits of the largest listed case of each operator: no drawn case has more
_MOST = {"shape": 16 * 256 * 50257, "shape_bwd": 32 * 512 * 32000, "logprobs": 16 * 512 * 128256,
         "logprobs_bwd": 16 * 512 * 128256, "router": 24 * 16 * 1024 * 128}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["shape", "shape", "shape_bwd", "logprobs", "logprobs_bwd", "router", "router"])
    lengths = rng.choice(["full", "uniform", "mixture"])
    if op == "router":
        E = rng.choice([8, 64, 128, 256, _log(rng, 4, 512)])
        c = _router("", E=E, K=min(E, rng.choice([1, 2, 6, 8, 8])), L=_log(rng, 1, 32), B=_log(rng, 1, 64), T=_log(rng, 1, 4096),
                    dtype=rng.choice(["bf16", "fp16", "fp32"]), lengths=lengths, scoring=rng.choice(["softmax", "sigmoid"]),
                    scope=rng.choice(["batch", "sequence"]), given=rng.random() < 0.4)
        c["z"] = c["scoring"] == "softmax" and rng.random() < 0.5
        while c["L"] * c["B"] * c["T"] * E > _MOST[op]:
            k = rng.choice([n for n in "LBT" if c[n] > 1])
            c[k] //= 2
        del c["name"]
        return c
    V = rng.choice([32000, 50257, 50272, 128256, _log(rng, 500, 160000), _log(rng, 500, 160000)])
    decode = op == "shape" and rng.random() < 0.5
    T = rng.choice([1, 1, 1, 4]) if decode else _log(rng, 1, 1024)
    B = _log(rng, 1, 256 if decode else 64)
    while B * T * V > _MOST[op]:
        if T > 1 and (rng.random() < 0.5 or B == 1):
            T //= 2
        else:
            B //= 2
    c = _logits(op, "", B=B, T=T, V=V, pitch=rng.choice([0, 0, -V % 64, 7]) if B * T * V < 0.9 * _MOST[op] else 0,
                P=_log(rng, 1, 8192 if decode else 1024) if rng.random() < 0.8 else 0, S0=_log(rng, 1, 4096) if decode else 0,
                dtype=rng.choice(["bf16", "bf16", "fp16"]), lengths=lengths, repetition=rng.random() < 0.8,
                frequency=rng.random() < 0.4, presence=rng.random() < 0.4, temperature=rng.random() < 0.7,
                bias=rng.choice(["none", "none", "shared", "own"]), mask=rng.choice(["none", "sequence", "row"]))
    if op == "shape":
        c["out32"] = rng.random() < 0.5 and 2 * B * T * V <= _MOST[op]
    if op in ("logprobs", "logprobs_bwd"):
        c["entropy"] = rng.random() < 0.5
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
    rows, valid = case["B"] * case["T"], case["B"] * _mean_length(case)
    if case["op"] == "router":
        L, E, K = case["L"], case["E"], case["K"]
        size = 4 if case["dtype"] == "fp32" else 2
        groups = L * (case["B"] if case["scope"] == "sequence" else 1)
        return {"bytes": size * L * E * (valid + rows) + 4 * K * L * (valid if case["given"] else rows) + 4 * E * groups,
                "flops": 8.0 * L * E * valid}
    V, op = case["V"], case["op"]
    # the history is read once per sequence, a bias once, a mask once per sequence or row
    more = 8 * case["B"] * (case["P"] + case["S0"] + case["T"])
    more += {"none": 0, "shared": 4 * V, "own": 4 * V * case["B"]}[case["bias"]]
    more += {"none": 0, "sequence": V / 8 * case["B"], "row": V / 8 * valid}[case["mask"]]
    if op == "shape":
        return {"bytes": 2 * V * valid + (4 if case["out32"] else 2) * V * rows + more, "flops": 2.0 * V * valid}
    if op == "logprobs":
        return {"bytes": 2 * V * valid + 12 * rows + more, "flops": (6.0 if case["entropy"] else 4.0) * V * valid}
    return {"bytes": 2 * V * (valid + rows) + (20 * valid if op == "logprobs_bwd" else 0) + more, "flops": 6.0 * V * valid}


# ---------------------------------------------------------------- the inputs
def _lengths(case, gen):
    B, T = case["B"], case["T"]
    if case["lengths"] == "full":
        return torch.full((B,), T, dtype=torch.int32)
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
    """The logits of a batch with the tokens and settings that its distribution was shaped by, or the router logits of a
    forward pass, as they are on the device before the call."""
    cpu = torch.Generator().manual_seed(seed * 7919 + 17)
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 19)
    s = {"case": dict(case), "lengths": _lengths(case, cpu).cuda()}
    if case["op"] == "router":
        _prepare_router(s, case, gen)
    else:
        _prepare_logits(s, case, gen)
    return s


def _prepare_router(s, case, gen):
    L, B, T, E, K = (case[k] for k in ("L", "B", "T", "E", "K"))
    # some experts are liked better than others
    liked = 0.5 * torch.randn((L, 1, 1, E), generator=gen, device="cuda")
    s["logits"] = (torch.randn((L, B, T, E), generator=gen, device="cuda") + liked).to(DTYPES[case["dtype"]])
    if case["given"]:
        # chosen by biased scores, a few tokens dropped by their experts
        bias = 0.3 * torch.randn((L, 1, 1, E), generator=gen, device="cuda")
        ids = (s["logits"].float() + bias).topk(K, dim=3).indices.int()
        drop = torch.rand(ids.shape, generator=gen, device="cuda") < 0.01
        s["expert_ids"] = ids.masked_fill(drop, -1)


def _prepare_logits(s, case, gen):
    dev = "cuda"
    B, T, V, P, S0, op = (case[k] for k in ("B", "T", "V", "P", "S0", "op"))
    r = lambda *n: torch.randn(n, generator=gen, device=dev)  # noqa: E731
    u = lambda *n: torch.rand(n, generator=gen, device=dev)  # noqa: E731
    pad = V + case["pitch"]
    z = s["logits"] = torch.empty((B, T, pad), dtype=DTYPES[case["dtype"]], device=dev)[:, :, :V]
    # text repeats itself: tokens of the prompt and of earlier parts of the answer come from a few hundred of the vocabulary
    often = torch.randint(0, V, (B, min(V, 400)), generator=gen, device=dev)
    some = lambda n: often.gather(1, (u(B, n) ** 2 * often.shape[1]).long().clamp(max=often.shape[1] - 1))  # noqa: E731
    if P:
        s["prompt"] = some(P)
        s["prompt_lengths"] = (P - (u(B) * (P // 2 + 1)).int()).int()
        s["prompt"][:, : P // 8].masked_fill_((u(B, 1) < 0.25).expand(B, P // 8), -1)      # padded on the left
    S = S0 + T
    tokens = s["tokens"] = some(S)
    if S0:
        s["start"] = (u(B) * (S0 + 1)).int().clamp(max=S0)
    start = s.get("start", torch.zeros(B, dtype=torch.int32, device=dev))
    if case["repetition"]:
        s["repetition"] = 1 + 0.3 * u(B)
    if case["frequency"]:
        s["frequency"] = 0.5 * u(B)
    if case["presence"]:
        s["presence"] = 0.5 * u(B)
    if case["temperature"]:
        s["temperature"] = 0.6 + 0.8 * u(B)
    if case["bias"] != "none":
        hit = u(V) < 0.05 if case["bias"] == "shared" else u(B, V) < 0.05
        s["bias"] = torch.where(hit, 2 * r(*hit.shape), 0.0)
    if op in ("logprobs", "logprobs_bwd"):
        s["ids"] = torch.empty((B, T), dtype=torch.int64, device=dev)
    step = max(1, (1 << 27) // (T * V))
    at = start.long()[:, None] + torch.arange(T, device=dev)
    for b in range(0, B, step):
        e = min(B, b + step)
        z[b:e] = 3.0 * r(e - b, T, V)
        x = z[b:e].float()
        y = (x - torch.log(-torch.log(u(*x.shape).clamp_(1e-12, 1 - 1e-7)))).argmax(dim=2)
        y = torch.where(u(*y.shape) < 0.5, y, tokens[b:e].gather(1, at[b:e].clamp(max=S - 1)))
        tokens[b:e].scatter_(1, at[b:e].clamp(max=S - 1), y)
        if "ids" in s:
            s["ids"][b:e] = y
    if case["mask"] != "none":
        rows, W = (T if case["mask"] == "row" else 1), (V + 31) // 32
        # an eighth of the sequences may say anything, the others what a grammar leaves; what was said was allowed
        words = torch.randint(-2 ** 31, 2 ** 31, (B, rows, W), generator=gen, device=dev, dtype=torch.int64)
        words = words & torch.randint(-2 ** 31, 2 ** 31, (B, rows, W), generator=gen, device=dev, dtype=torch.int64)
        words[u(B) < 0.125] = -1
        if "ids" in s:
            for k in range(T):
                w, bit = (s["ids"][:, k, None] // 32), 1 << (s["ids"][:, k, None] % 32)
                row = words[:, k if rows > 1 else 0]
                row.scatter_(1, w, row.gather(1, w) | bit)
        elif B > 1:
            words[1, 0] = 0                           # a grammar that has come to its end
        s["mask"] = torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()
    if op == "shape_bwd":
        # the gradient of a loss with respect to the shaped logits
        d = s["dshaped"] = torch.empty((B, T, V), dtype=DTYPES[case["dtype"]], device=dev)
        for b in range(0, B, step):
            e = min(B, b + step)
            p = torch.softmax(z[b:e].float(), dim=2)
            d[b:e] = -30.0 * r(e - b, T, 1) * p
    if op == "logprobs_bwd":
        # what the forward pass left, and the gradient of the objective
        s["logprobs"], s["entropy"] = torch.empty((B, T), device=dev), torch.empty((B, T), device=dev)
        s["lse"] = torch.empty((B, T, 2), device=dev)
        for b in range(0, B, step):
            e = min(B, b + step)
            x = _shape(s, b, e)
            hi = x.amax(dim=2)
            x -= hi[..., None]
            lo = torch.log(torch.exp(x).sum(dim=2))
            lp = x.gather(2, s["ids"][b:e, :, None])[..., 0] - lo
            x -= lo[..., None]
            ent = -torch.where(x > float("-inf"), x * torch.exp(x), 0.0).sum(dim=2)
            ok = _valid(s)[b:e]
            s["lse"][b:e, :, 0], s["lse"][b:e, :, 1] = torch.where(ok, hi, 0.0), torch.where(ok, lo, 0.0)
            s["logprobs"][b:e], s["entropy"][b:e] = torch.where(ok, lp, 0.0), torch.where(ok, ent, 0.0)
        ok = _valid(s)
        s["grad_logprobs"] = torch.where(ok, r(B, T), 0.0)
        if case["entropy"]:
            s["grad_entropy"] = torch.where(ok, -0.01 * torch.ones((B, T), device=dev), 0.0)


# ---------------------------------------------------------------- one pass
def run(s):
    if own:
        return _own(s)
    return {"shape": _plain_shape, "shape_bwd": _plain_shape_bwd, "logprobs": _plain_logprobs, "logprobs_bwd": _plain_logprobs_bwd,
            "router": _plain_router}[s["case"]["op"]](s)


_SETTINGS = ("tokens", "start", "prompt", "prompt_lengths", "repetition", "frequency", "presence", "temperature", "bias", "mask")


def _own(s):
    from paper_2410_15651_b200 import binding as lib
    c, z, n = s["case"], s["logits"], s["lengths"]
    if c["op"] == "router":
        if "ws" not in s:
            s["ws"] = lib.router_workspace(c["L"], c["B"], c["T"], c["E"], z.device)
        scoring = {"softmax": lib.ROUTER_SOFTMAX, "sigmoid": lib.ROUTER_SIGMOID}[c["scoring"]]
        scope = {"batch": lib.ROUTER_BATCH, "sequence": lib.ROUTER_SEQUENCE}[c["scope"]]
        o = lib.router_loss_fwd_bwd(z, n, c["K"], scoring, scope, _BALANCE, _Z if c["z"] else 0.0, _SCALE, s["ws"],
                                    expert_ids=s.get("expert_ids"))
        out = {"loss": o.loss, "counts": o.counts, "dlogits": o.dlogits}
        if not c["given"]:
            out["ids"] = o.ids
        return out
    if "ws" not in s:
        s["ws"] = lib.workspace(c["B"], c["T"], z.device)
        s["shaping"] = lib.Shaping(c["B"], c["V"], **{k: s[k] for k in _SETTINGS if k in s})
        if c["op"] == "logprobs_bwd":
            s["forward"] = lib.ShapedLogprobs(z, logprobs=s["logprobs"], lse=s["lse"], entropy=s["entropy"])
    ws, sh = s["ws"], s["shaping"]
    if c["op"] == "shape":
        return lib.shape_logits(z, n, sh, ws, dtype=torch.float32 if c["out32"] else z.dtype)
    if c["op"] == "shape_bwd":
        return lib.shape_logits_bwd(s["dshaped"], z, n, sh, ws)
    if c["op"] == "logprobs":
        o = lib.shaped_logprobs(z, s["ids"], n, sh, ws, want_entropy=c["entropy"])
        return {"logprobs": o.logprobs, "entropy": o.entropy} if c["entropy"] else {"logprobs": o.logprobs}
    return lib.shaped_logprobs_bwd(z, s["ids"], n, sh, s["forward"], s["grad_logprobs"], s.get("grad_entropy"), ws)


# The coefficients of the router's losses; its gradient is scaled by 1000, as with loss scaling, so that fp16 holds it.
_BALANCE, _Z, _SCALE = 0.01, 0.001, 1000.0


def _valid(s):
    c = s["case"]
    return torch.arange(c["T"], device=s["lengths"].device)[None] < s["lengths"][:, None]


def _one(s, name, b, e, neutral):
    return s[name][b:e, None, None] if name in s else neutral


def _history(s, b, e):
    """Of every row: whether an entry is among the tokens before it, and how often the answer has it so far."""
    c, dev = s["case"], s["logits"].device
    T, V, n = c["T"], c["V"], e - b
    tok = s["tokens"][b:e]
    S = tok.shape[1]
    start = s["start"][b:e].long() if "start" in s else torch.zeros(n, dtype=torch.int64, device=dev)
    count = torch.zeros((n, T, V), dtype=torch.int32, device=dev)
    before = torch.arange(S, device=dev)[None] < start[:, None]
    count[:, 0].scatter_add_(1, tok, before.int())
    if T > 1:
        at = (start[:, None] + torch.arange(T - 1, device=dev)).clamp(max=S - 1)
        count[:, 1:].scatter_(2, tok.gather(1, at)[..., None], 1)
        count = count.cumsum(dim=1, dtype=torch.int32)
    seen = count > 0
    if "prompt" in s:
        p = s["prompt"][b:e]
        use = (torch.arange(p.shape[1], device=dev)[None] < s["prompt_lengths"][b:e, None]) & (p >= 0)
        asked = torch.zeros((n, V), dtype=torch.int32, device=dev).scatter_add_(1, p.clamp(min=0), use.int()) > 0
        seen |= asked[:, None]
    return seen, count


def _allowed(s, b, e):
    if "mask" not in s:
        return None
    bits = (s["mask"][b:e][..., None] >> torch.arange(32, device=s["mask"].device, dtype=torch.int32)) & 1
    return bits.bool().flatten(2)[..., : s["case"]["V"]]


def _shape(s, b, e):
    """The shaped logits of sequences b..e-1 in fp32."""
    x = s["logits"][b:e].float()
    if "repetition" in s or "frequency" in s or "presence" in s:
        seen, count = _history(s, b, e)
        if "repetition" in s:
            rep = _one(s, "repetition", b, e, 1.0)
            x = torch.where(seen, torch.where(x < 0, x * rep, x / rep), x)
        if "frequency" in s:
            x = x - _one(s, "frequency", b, e, 0.0) * count
        if "presence" in s:
            x = x - _one(s, "presence", b, e, 0.0) * (count > 0)
        del seen, count
    if "bias" in s:
        x = x + (s["bias"] if s["bias"].dim() == 1 else s["bias"][b:e, None])
    if "temperature" in s:
        x = x / _one(s, "temperature", b, e, 1.0)
    ok = _allowed(s, b, e)
    return x if ok is None else torch.where(ok, x, float("-inf"))


def _through(s, d):
    """The gradient with respect to the logits, from the one with respect to the shaped logits."""
    B = s["case"]["B"]
    if "repetition" in s:
        seen, _ = _history(s, 0, B)
        rep = _one(s, "repetition", 0, B, 1.0)
        d = torch.where(seen, torch.where(s["logits"] < 0, d * rep, d / rep), d)
    if "temperature" in s:
        d = d / _one(s, "temperature", 0, B, 1.0)
    ok = _allowed(s, 0, B)
    ok = _valid(s)[..., None] if ok is None else ok & _valid(s)[..., None]
    return torch.where(ok, d, 0.0).to(s["logits"].dtype)


def _plain_shape(s):
    x = torch.where(_valid(s)[..., None], _shape(s, 0, s["case"]["B"]), 0.0)
    return x if s["case"]["out32"] else x.to(s["logits"].dtype)


def _plain_shape_bwd(s):
    return _through(s, s["dshaped"].float())


def _plain_logprobs(s):
    x = _shape(s, 0, s["case"]["B"])
    x = x - x.amax(dim=2, keepdim=True)
    x = x - torch.log(torch.exp(x).sum(dim=2, keepdim=True))
    out = {"logprobs": torch.where(_valid(s), x.gather(2, s["ids"][..., None])[..., 0], 0.0)}
    if s["case"]["entropy"]:
        h = -torch.where(x > float("-inf"), x * torch.exp(x), 0.0).sum(dim=2)
        out["entropy"] = torch.where(_valid(s), h, 0.0)
    return out


def _plain_logprobs_bwd(s):
    x = _shape(s, 0, s["case"]["B"])
    x = (x - s["lse"][..., :1]) - s["lse"][..., 1:]
    p = torch.exp(x)
    d = -s["grad_logprobs"][..., None] * p
    y = s["ids"][..., None]
    d.scatter_(2, y, -s["grad_logprobs"][..., None] * torch.expm1(s["logprobs"][..., None]))
    if "grad_entropy" in s:
        d = d - s["grad_entropy"][..., None] * torch.where(p > 0, p * (x + s["entropy"][..., None]), 0.0)
    return _through(s, d)


def _plain_router(s):
    c = s["case"]
    L, B, T, E, K = (c[k] for k in ("L", "B", "T", "E", "K"))
    z, ok = s["logits"].float(), _valid(s)[None, :, :, None]
    if c["given"]:
        ids = s["expert_ids"]
    else:
        ids = torch.where(ok, z.sort(dim=3, descending=True, stable=True).indices[..., :K].int(), 0)
    count = torch.zeros((L, B, E), dtype=torch.int32, device=z.device)
    count.scatter_add_(2, ids.clamp(min=0).long().flatten(2), (ok & (ids >= 0)).int().flatten(2))
    m = z.amax(dim=3, keepdim=True)
    if c["scoring"] == "softmax":
        e = torch.exp(z - m)
        total = e.sum(dim=3, keepdim=True)
        p, slope = e / total, 1.0
        lse = m + torch.log(total)
    else:
        e = 1 / (1 + torch.exp(-z))
        p = e / e.sum(dim=3, keepdim=True)
        slope = 1 / (1 + torch.exp(z))
    n = s["lengths"].double()
    N = n.sum().clamp(min=1)
    if c["scope"] == "batch":
        count = count.sum(dim=1, dtype=torch.int32)
        f = (count.double() * (E / (K * N)))[:, None, None]
        w = (ok / N)
    else:
        f = (count.double() * (E / (K * n.clamp(min=1)))[None, :, None])[:, :, None]
        w = ok / (n.clamp(min=1) * (n > 0).sum().clamp(min=1))[None, :, None, None]
    f = f.float()
    dot = (p * f).sum(dim=3, keepdim=True)
    balance = (dot.double() * w).sum(dim=(1, 2, 3))
    d = _BALANCE * w.float() * slope * p * (f - dot)
    zl = torch.zeros_like(balance)
    if c["z"]:
        zl = (torch.where(ok, lse.double() ** 2, 0.0) / N).sum(dim=(1, 2, 3))
        d = d + (_Z * 2 / N).float() * lse * p
    d = torch.where(ok, _SCALE * d, 0.0)
    out = {"loss": torch.stack([balance, zl], dim=1).float(), "counts": count, "dlogits": d.to(s["logits"].dtype)}
    if not c["given"]:
        out["ids"] = ids
    return out


# ---------------------------------------------------------------- the definitions in 64 bits, a sequence (and a row) at a time
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "router":
        return _exact_router(s)
    B, T, V, op = case["B"], case["T"], case["V"], case["op"]
    if B * T > 20000:
        return None
    dev, lens = s["logits"].device, s["lengths"].tolist()
    start = s["start"].tolist() if "start" in s else [0] * B
    tokens = s["tokens"].tolist()
    value = {k: s[k].double().tolist() if k in s else [d] * B
             for k, d in (("repetition", 1.0), ("frequency", 0.0), ("presence", 0.0), ("temperature", 1.0))}
    wide = op != "logprobs"
    out = torch.zeros((B, T, V) if wide else (B, T), dtype=torch.float64, device=dev)
    entropy = torch.zeros((B, T), dtype=torch.float64, device=dev)
    bit = torch.arange(V, device=dev) % 32
    for b in range(B):
        n = lens[b]
        if n == 0:
            continue
        rep, tau = value["repetition"][b], value["temperature"][b]
        seen = torch.zeros(V, dtype=torch.bool, device=dev)
        count = torch.zeros(V, dtype=torch.float64, device=dev)
        if "prompt" in s:
            told = s["prompt"][b, : int(s["prompt_lengths"][b])]
            seen[told[told >= 0]] = True
        for v in tokens[b][: start[b]]:
            seen[v] = True
            count[v] += 1
        z = s["logits"][b, :n].double()
        x, scale = torch.empty_like(z), torch.empty_like(z)
        for t in range(n):
            if t > 0:
                v = tokens[b][start[b] + t - 1]
                seen[v] = True
                count[v] += 1
            by = torch.where(seen, torch.where(z[t] < 0, rep, 1 / rep), 1.0)
            x[t] = z[t] * by - value["frequency"][b] * count - value["presence"][b] * (count > 0)
            scale[t] = by / tau
        if "bias" in s:
            x += s["bias"].double() if s["bias"].dim() == 1 else s["bias"][b].double()
        x /= tau
        if "mask" in s:
            words = s["mask"][b, :n] if s["mask"].shape[1] > 1 else s["mask"][b]
            cut = (words.repeat_interleave(32, dim=1)[:, :V] >> bit) & 1 == 0
            x.masked_fill_(cut, float("-inf"))
            scale.masked_fill_(cut.expand_as(scale), 0.0)
        if op == "shape":
            out[b, :n] = x
            continue
        if op == "shape_bwd":
            out[b, :n] = s["dshaped"][b, :n].double() * scale
            continue
        lq = torch.log_softmax(x, dim=1)
        q = lq.exp()
        h = torch.special.entr(q).sum(dim=1)
        y = s["ids"][b, :n, None]
        if op == "logprobs":
            out[b, :n], entropy[b, :n] = lq.gather(1, y)[:, 0], h
            continue
        g = s["grad_logprobs"][b, :n, None].double()
        d = torch.zeros_like(q).scatter_(1, y, 1.0).sub_(q).mul_(g)
        if case["entropy"]:
            d -= s["grad_entropy"][b, :n, None].double() * (h[:, None] * q - torch.special.entr(q))
        out[b, :n] = d * scale
    if op == "logprobs":
        return {"logprobs": out, "entropy": entropy} if case["entropy"] else {"logprobs": out}
    return out


def _exact_router(s):
    c = s["case"]
    L, B, E, K = (c[k] for k in ("L", "B", "E", "K"))
    lens = s["lengths"].tolist()
    N, filled = max(1, sum(lens)), max(1, sum(n > 0 for n in lens))
    dev = s["logits"].device
    grad = torch.zeros(s["logits"].shape, dtype=torch.float64, device=dev)
    ids = torch.zeros(s["logits"].shape[:3] + (K,), dtype=torch.int32, device=dev)
    counts = torch.zeros((L, B, E), dtype=torch.int32, device=dev)
    loss = torch.zeros((L, 2), dtype=torch.float64, device=dev)
    for b, n in enumerate(lens):
        pick = s["expert_ids"][:, b, :n] if c["given"] else s["logits"][:, b, :n].float().argsort(dim=2, descending=True, stable=True)[..., :K]
        ids[:, b, :n] = pick
        for layer in range(L):
            got = pick[layer].flatten()
            counts[layer, b] = torch.bincount(got[got >= 0].long(), minlength=E)[:E]
    totals = counts.sum(dim=1)
    for b, n in enumerate(lens):
        if n == 0:
            continue
        z = s["logits"][:, b, :n].double()
        share, w = (totals / (N * K), 1 / N) if c["scope"] == "batch" else (counts[:, b] / (n * K), 1 / (n * filled))
        share = E * share.double()[:, None]
        if c["scoring"] == "softmax":
            p, rise = torch.softmax(z, dim=2), 1.0
        else:
            p = torch.sigmoid(z)
            p = p / p.sum(dim=2, keepdim=True)
            rise = torch.sigmoid(-z)
        mean = (p * share).sum(dim=2, keepdim=True)
        loss[:, 0] += w * mean.sum(dim=(1, 2))
        d = _BALANCE * w * rise * p * (share - mean)
        if c["z"]:
            lse = torch.logsumexp(z, dim=2, keepdim=True)
            loss[:, 1] += (lse ** 2).sum(dim=(1, 2)) / N
            d = d + _Z * 2 / N * lse * p
        grad[:, b, :n] = _SCALE * d
    out = {"loss": loss, "counts": totals.int() if c["scope"] == "batch" else counts, "dlogits": grad}
    if not c["given"]:
        out["ids"] = ids
    return out
