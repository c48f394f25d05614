"""The objectives beside the PPO step on the GPU against their float64 definitions (objectives64.py).

Tolerances.  A log-prob lp is formed in fp32 as ln2 * (fma(z_y, log2e, -M) - log2(sum)): with |x_y - M| <= 64 the first
term is rounded by at most 2^-24 * 64, the terms of the sum carry 2^-24 * 64 * ln2 from their exponent and 2^-22 from the
exponential, log2 adds 2^-23 of a value below 32: together below 1.3e-5, and 2e-5 is allowed (LP).  A gradient entry is a
product of such quantities, rounded once to its type: half a step of the value (finfo.eps / 2), plus 2e-5 of the absolute
parts it is summed from (a KL part may cancel a policy part), plus half of the type's smallest step (fp16) or the fp32
flush bound (bf16).  Sums and means of fp32 terms are formed in double: a loss is off by at most the terms' own errors,
their mean absolute size times 2e-5, and one final rounding to fp32."""
import pytest
import torch

import objectives64 as ref
from paper_2410_15651_b200 import binding as lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
LP = 2e-5
BF, HF = torch.bfloat16, torch.float16


def tiny(dtype):
    return 2.0 ** -25 if dtype == HF else 2.0 ** -120


def check_gradient(got, want, parts):
    """|got - want| within half a step of want, 2e-5 of `parts`, and the smallest step."""
    tol = torch.finfo(got.dtype).eps / 2 * want.abs() + LP * parts + tiny(got.dtype)
    bad = (got.double() - want).abs() - tol
    assert not torch.isnan(got).any()
    assert (bad <= 0).all(), (bad.max().item(), want.abs().max().item())


def mixed_lengths(B, T):
    pattern = [T, 0, 1, max(1, T - 1), T // 2, T]
    return torch.tensor([pattern[b % len(pattern)] for b in range(B)], dtype=torch.int32, device=DEV)


def labels(B, T, V, gen):
    return torch.randint(0, V, (B, T), generator=gen, device=DEV)


# sizes around the kernels' borders: single entries, vectors off and on 16-byte boundaries, the chunk ring, clusters of two
# to four blocks, rows streamed twice
SIZES = [(2, 1, 1), (4, 3, 7), (4, 5, 1000), (4, 5, 1001), (2, 3, 8192), (6, 4, 8200), (6, 4, 32000), (4, 3, 50257),
         (4, 3, 50272), (2, 3, 57344), (4, 3, 128256), (2, 2, 163840), (2, 2, 230000), (2, 2, 300000), (2, 2, 100003)]


def policy_inputs(z, ids, lengths, gen, per_sequence):
    B, T, _ = z.shape
    _, lp, _ = ref.label_logprobs(z.double(), ids, lengths)
    # ratios away from the clip's edges, where either branch would be a right answer
    rho = torch.tensor([0.5, 0.9, 1.0, 1.1, 1.6], device=DEV)[torch.randint(0, 5, (B, T), generator=gen, device=DEV)]
    lp_old = (lp - rho.double().log()).float()
    lp_ref = (lp + 0.5 * torch.randn((B, T), generator=gen, device=DEV)).float()
    adv = torch.randn((B,) if per_sequence else (B, T), generator=gen, device=DEV)
    return lp_old, lp_ref, adv


def check_policy(z, ids, lengths, lp_old, lp_ref, adv, kl_coef, reduction, scale, out=None, z64=None):
    B, T, V = z.shape
    z64 = z.double() if z64 is None else z64
    ws = lib.workspace(B, T, DEV)
    got = lib.policy_kl_loss_fwd_bwd(z, ids, lengths, lp_old, lp_ref, adv, 0.2, 0.3, kl_coef, reduction, scale, ws, out)
    pg, kl, d, lp, size = ref.policy_kl(z64, ids, lengths, lp_old, lp_ref, adv, 0.2, 0.3, kl_coef, reduction, scale)
    if got.lp_new is not None:
        assert (got.lp_new.double() - lp).abs().max() <= LP
    part = torch.softmax(z64, dim=2) + torch.nn.functional.one_hot(ids.clamp(0, V - 1), V)
    check_gradient(got.dlogits, d, size[..., None] * part)
    n = lengths.clamp(0, T).double()
    # every term |A| rho <= 4.3 * 1.6 and its error LP of that; KL terms: d exp(d) per unit of lp
    assert abs(got.loss[0].item() - pg.item()) <= 8 * LP + 2 ** -23 * abs(pg.item())
    assert abs(got.loss[1].item() - kl.item()) <= 8 * LP + 2 ** -23 * abs(kl.item())
    if n.sum() == 0:
        assert (got.loss == 0).all()
    return got, ws


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("B,T,V", SIZES)
def test_policy_kl_sizes(B, T, V, dtype):
    gen = torch.Generator(device=DEV).manual_seed(V + T)
    z, _ = ref.row_logits(B, T, V, dtype, gen, DEV)
    ids, lengths = labels(B, T, V, gen), mixed_lengths(B, T)
    lp_old, lp_ref, adv = policy_inputs(z, ids, lengths, gen, per_sequence=V % 2 == 0)
    got, ws = check_policy(z, ids, lengths, lp_old, lp_ref, adv, 0.1, V % 3 % 2, 100.0)
    assert lib.poll_status(ws) == 0
    pads = ~ref.valid_mask(lengths, T)
    assert (got.dlogits[pads] == 0).all() and (got.lp_new[pads] == 0).all()


@pytest.mark.parametrize("reduction", [lib.MEAN_TOKENS, lib.MEAN_SEQUENCES])
@pytest.mark.parametrize("layout", ["prompt", "pitch", "offset", "in_place", "other_offset", "strided_adv"])
def test_policy_kl_layouts(layout, reduction):
    gen = torch.Generator(device=DEV).manual_seed(7)
    B, T, V = 5, 6, 8200
    kw = {"prompt": dict(prompt=3), "pitch": dict(pitch=5), "offset": dict(offset=3), "in_place": dict(prompt=2, offset=1, pitch=3)}
    z, store = ref.row_logits(B, T, V, BF, gen, DEV, **kw.get(layout, {}))
    ids_full = labels(B, T + 4, V, gen)
    ids, lengths = ids_full[:, 2:2 + T], mixed_lengths(B, T)
    lp_old, lp_ref, adv = policy_inputs(z, ids, lengths, gen, False)
    out, z64 = None, z.double()
    if layout == "in_place":
        before = store.clone()
        out = lib.PolicyKlOutputs(z, in_place=True)
    elif layout == "other_offset":                       # gradient rows off the logits' alignment: element-wise kernel
        out = lib.PolicyKlOutputs(z)
        out.dlogits = torch.full((B * T * V + 3,), 7.0, dtype=BF, device=DEV)[3:].view(B, T, V)
    elif layout == "strided_adv":
        adv = torch.randn((T, B), generator=gen, device=DEV).t()
    check_policy(z, ids, lengths, lp_old, lp_ref, adv, 0.05, reduction, 30.0, out, z64)
    if layout == "in_place":                             # nothing but the rows was written
        keep = torch.ones_like(store, dtype=torch.bool)
        keep.as_strided(z.shape, z.stride(), z.storage_offset())[...] = False
        assert torch.equal(store.view(torch.int16)[keep], before.view(torch.int16)[keep])


def test_policy_kl_without_reference_and_without_tokens():
    gen = torch.Generator(device=DEV).manual_seed(8)
    B, T, V = 3, 4, 32000
    z, _ = ref.row_logits(B, T, V, BF, gen, DEV)
    ids, lengths = labels(B, T, V, gen), mixed_lengths(B, T)
    lp_old, _, adv = policy_inputs(z, ids, lengths, gen, True)
    got, _ = check_policy(z, ids, lengths, lp_old, None, adv, 0.3, 0, 1.0)
    assert got.loss[1].item() == 0
    for reduction in (0, 1):
        got, ws = check_policy(z, ids, torch.zeros_like(lengths), lp_old, None, adv, 0.3, reduction, 1.0)
        assert (got.dlogits == 0).all() and lib.poll_status(ws) == 0


@pytest.mark.parametrize("V", [1000, 8200, 50257, 128256])
def test_policy_kl_bad_ids_lengths_and_deleted_entries(V):
    gen = torch.Generator(device=DEV).manual_seed(9)
    B, T = 4, 4
    z, _ = ref.row_logits(B, T, V, BF, gen, DEV)
    z[..., 5:V - 3:7] = float("-inf")
    ids, lengths = torch.full((B, T), 3, device=DEV), torch.tensor([T + 9, -2, 2, T], dtype=torch.int32, device=DEV)
    ids[0, 1], ids[3, 2] = V, -1
    lp_old, lp_ref, adv = policy_inputs(z, ids, lengths, gen, False)
    got, ws = check_policy(z, ids, lengths, lp_old, lp_ref, adv, 0.1, 1, 10.0)
    assert lib.poll_status(ws) == 16 | 32
    assert (got.dlogits[0, 1] == 0).all() and (got.dlogits[3, 2] == 0).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("V", [32000, 128256])
def test_policy_kl_far_logits(V, dtype):
    """Peaked rows and logits far above the first ones of their row."""
    gen = torch.Generator(device=DEV).manual_seed(10)
    B, T = 2, 4
    z, _ = ref.row_logits(B, T, V, dtype, gen, DEV, sigma=1.0)
    z[0, 0, V - 1] = 300.0
    z[0, 1, :8] = -2000.0
    z[1, 0] = 0.0
    ids, lengths = labels(B, T, V, gen), torch.full((B,), T, dtype=torch.int32, device=DEV)
    ids[0, 0] = V - 1
    z[0, 2, ids[0, 2]] = 30.0
    z64 = z.double()
    lp_old, lp_ref, adv = policy_inputs(z, ids, lengths, gen, False)
    got, _ = check_policy(z, ids, lengths, lp_old, lp_ref, adv, 0.1, 0, 8.0)
    assert torch.isfinite(got.loss).all()


def check_preference(z, ids, lengths, lp_ref, kind, beta, margin, smoothing, length_mean, scale, out=None, z64=None):
    B, T, V = z.shape
    z64 = z.double() if z64 is None else z64
    ws = lib.workspace(B, T, DEV)
    got = lib.preference_loss_fwd_bwd(z, ids, lengths, lp_ref, kind, beta, margin, smoothing, length_mean, scale, ws, out)
    loss, rewards, d, lp, f = ref.preference(z64, ids, lengths, lp_ref, kind, beta, margin, smoothing, length_mean, scale)
    # a sequence's sum is off by at most LP per token (LP in all where it is a mean over the tokens)
    per_seq = beta * LP * (torch.ones(B, device=DEV) if length_mean else lengths.clamp(0, T).double())
    if got.lp_new is not None:
        assert (got.lp_new.double() - lp).abs().max() <= LP
    assert ((got.rewards.double() - rewards).abs() <= per_seq + 2 ** -23 * rewards.abs()).all()
    dh = 2 * per_seq.max().item()                        # error of h
    slope = 1.0 if kind < 2 else 2 * ((rewards[:B // 2] - rewards[B // 2:] - margin - 0.5).abs().max().item() + dh) / beta ** 2
    assert abs(got.loss.item() - loss.item()) <= slope * dh + 2 ** -23 * abs(loss.item())
    # the factor changes by at most max|loss''| per unit of h: 1/4, 0 (away from the kink), 2 / beta^2
    curve = {0: 0.25, 1: 0.0, 2: 2 / beta ** 2}[kind]
    c = 1 / lengths.clamp(1, T).double() if length_mean else torch.ones(B, device=DEV).double()
    df = curve * dh * beta * c * scale * 2 / B
    part = torch.softmax(z64, dim=2) + torch.nn.functional.one_hot(ids.clamp(0, V - 1), V)
    check_gradient(got.dlogits, d, (f.abs() + df / LP)[:, None, None] * part)
    return got, ws


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("B,T,V", SIZES)
def test_preference_sizes(B, T, V, dtype):
    gen = torch.Generator(device=DEV).manual_seed(V + T)
    z, _ = ref.row_logits(B, T, V, dtype, gen, DEV)
    ids, lengths = labels(B, T, V, gen), mixed_lengths(B, T)
    _, lp, _ = ref.label_logprobs(z.double(), ids, lengths)
    lp_ref = (lp + 0.5 * torch.randn((B, T), generator=gen, device=DEV)).float()
    got, ws = check_preference(z, ids, lengths, lp_ref, V % 3, 0.3, 0.1, 0.1 if V % 3 == 0 else 0.0, T % 2 == 0, 100.0)
    assert lib.poll_status(ws) == 0
    pads = ~ref.valid_mask(lengths, T)
    assert (got.dlogits[pads] == 0).all() and (got.lp_new[pads] == 0).all()


@pytest.mark.parametrize("kind", [lib.PREF_SIGMOID, lib.PREF_HINGE, lib.PREF_SQUARED])
@pytest.mark.parametrize("layout", ["prompt", "in_place", "other_offset", "no_reference", "no_lp"])
def test_preference_layouts(layout, kind):
    gen = torch.Generator(device=DEV).manual_seed(17)
    B, T, V = 6, 5, 16001 if layout == "in_place" else 16000
    kw = {"prompt": dict(prompt=3), "in_place": dict(prompt=1, offset=1)}
    z, store = ref.row_logits(B, T, V, BF, gen, DEV, **kw.get(layout, {}))
    ids, lengths = labels(B, T + 2, V, gen)[:, 1:1 + T], mixed_lengths(B, T)
    _, lp, _ = ref.label_logprobs(z.double(), ids, lengths)
    lp_ref = None if layout == "no_reference" else (lp + 0.2 * torch.randn((B, T), generator=gen, device=DEV)).float()
    out, z64 = lib.PreferenceOutputs(z, in_place=layout == "in_place", want_lp_new=layout != "no_lp"), z.double()
    if layout == "other_offset":
        out.dlogits = torch.full((B * T * V + 3,), 7.0, dtype=BF, device=DEV)[3:].view(B, T, V)
    check_preference(z, ids, lengths, lp_ref, kind, 0.2 if layout != "no_reference" else 0.01, -0.3, 0.0, kind == 2, 50.0, out, z64)


def test_preference_saturated_pairs_and_bad_ids():
    """Ratios of hundreds of nats (no overflow), empty responses, ids out of range."""
    gen = torch.Generator(device=DEV).manual_seed(18)
    B, T, V = 8, 6, 8200
    z, _ = ref.row_logits(B, T, V, BF, gen, DEV)
    ids = labels(B, T, V, gen)
    lengths = torch.tensor([T, T, 0, 0, T, 2, 0, T + 1], dtype=torch.int32, device=DEV)
    _, lp, _ = ref.label_logprobs(z.double(), ids, lengths)
    lp_ref = lp.float()
    lp_ref[0] -= 100.0
    lp_ref[1] += 100.0
    ids[5, 1], ids[4, 0] = V + 5, -7
    for kind in (0, 1, 2):
        got, ws = check_preference(z, ids, lengths, lp_ref, kind, 1.0, 0.0, 0.0, False, 1.0)
        assert lib.poll_status(ws) == 16 | 32
        assert torch.isfinite(got.loss).all()
        assert (got.dlogits[4, 0] == 0).all() and (got.dlogits[5, 1] == 0).all()


def test_repeated_calls_give_the_same_bits_and_leave_the_workspace_usable():
    gen = torch.Generator(device=DEV).manual_seed(19)
    for V in (1000, 32000, 50257, 128256):
        B, T = 6, 37
        z, _ = ref.row_logits(B, T, V, BF, gen, DEV)
        ids, lengths = labels(B, T, V, gen), mixed_lengths(B, T)
        lp_old, lp_ref, adv = policy_inputs(z, ids, lengths, gen, False)
        ws = lib.workspace(B, T, DEV)
        runs = []
        for _ in range(3):
            a = lib.policy_kl_loss_fwd_bwd(z, ids, lengths, lp_old, lp_ref, adv, 0.2, 0.3, 0.1, 1, 1.0, ws)
            b = lib.preference_loss_fwd_bwd(z, ids, lengths, lp_ref, 0, 0.1, 0.0, 0.0, False, 1.0, ws)
            runs.append([a.loss, a.dlogits, a.lp_new, b.loss, b.dlogits, b.rewards, b.lp_new])
        for r in runs[1:]:
            assert all(torch.equal(x, y) for x, y in zip(runs[0], r))
        assert lib.poll_status(ws) == 0


# ---------------------------------------------------------------- the teacher's top log-probs
def check_topk(z, lengths, K, temperature):
    B, T, V = z.shape
    ws = lib.workspace(B, T, DEV)
    got = lib.topk_logprobs(z, lengths, K, temperature, ws)
    ids, lp = ref.topk(z.double(), lengths, K, temperature)
    assert torch.equal(got.ids.long(), ids)
    assert torch.equal(torch.isinf(got.logprobs), torch.isinf(lp))
    fine = torch.isfinite(lp)
    # LP bounds the log of the sum.  The entry itself, ln2 * ((z - maximum) * log2(e) / temperature - log2(sum)), takes four
    # roundings that are relative to its size (the factor, the fused product, ln2, the result; 2^-24 each): 2^-22 |lp|,
    # which exceeds LP at the -60000 of a row with one entry of 60000, where half a step of fp32 alone is 0.002.
    assert ((got.logprobs.double() - lp).abs()[fine] <= LP * max(1.0, 1 / temperature) + 2.0 ** -22 * lp[fine].abs()).all()
    return got, ws


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("B,T,V,K", [(1, 1, 1, 1), (2, 3, 7, 9), (1, 1, 50272, 20), (3, 5, 1000, 256), (3, 5, 1001, 1), (2, 9, 2047, 100),
                                     (3, 70, 8200, 33), (4, 60, 32000, 64), (2, 3, 50257, 50), (2, 200, 50257, 7),
                                     (2, 3, 128256, 256), (3, 101, 128256, 128), (1, 2, 300001, 256),
                                     # enough rows for a row per warp
                                     (8, 90, 1, 3), (8, 90, 7, 5), (8, 90, 1000, 256), (8, 90, 1001, 1), (6, 120, 8200, 100), (5, 160, 32000, 64),
                                     (5, 160, 50257, 256), (3, 210, 128256, 128)])
def test_topk_sizes(B, T, V, K, dtype):
    gen = torch.Generator(device=DEV).manual_seed(V + K)
    z, _ = ref.row_logits(B, T, V, dtype, gen, DEV, prompt=1 if V < 60000 else 0, pitch=3 if V % 2 else 0)
    lengths = mixed_lengths(B, T)
    _, ws = check_topk(z, lengths, K, 1.0 if V % 2 else 2.0)
    assert lib.poll_status(ws) == 0


@pytest.mark.parametrize("T", [2, 55])                       # a row per block, a row per warp
def test_topk_ties_runs_and_deleted_entries(T):
    gen = torch.Generator(device=DEV).manual_seed(31)
    B, V = 12, 20003
    for dtype in (BF, HF):
        z, _ = ref.row_logits(B, T, V, dtype, gen, DEV, pitch=2)
        z[0] = 0.0                                           # all entries equal
        z[1] = -0.0
        z[1, :, 1::2] = 0.0                                  # the two zeros are the same value
        z[2] = z[2].round()                                  # a few values, each many times
        z[3] = torch.linspace(-4, 4, V, device=DEV)          # ascending: the top sits in neighbouring vectors
        z[4] = torch.linspace(4, -4, V, device=DEV)
        z[5] = float("-inf")
        z[5, :, V - 3:] = 1.0                                # three entries left
        z[6, :, ::3] = float("-inf")
        z[7, :, 8:16] = 50.0                                 # one vector far above the rest
        z[8] = -3.0
        z[8, :, -300:] = -2.0                                # more equal entries than K, at the end
        z[9, :, 0] = 60000.0 if dtype == HF else 1e30
        z[10] = -1000.0
        z[10, 1, 77] = 900.0
        z[11, :, 5::1024] = 20.0                             # the top in one thread's vectors
        lengths = torch.full((B,), T, dtype=torch.int32, device=DEV)
        for K in (1, 5, 64, 256):
            check_topk(z, lengths, K, 1.0)


@pytest.mark.parametrize("T", [3, 210])
def test_topk_lengths_out_of_range_and_non_finite_logits(T):
    gen = torch.Generator(device=DEV).manual_seed(32)
    B, V, K = 3, 9000, 16
    z, _ = ref.row_logits(B, T, V, BF, gen, DEV)
    lengths = torch.tensor([T + 4, -1, 2], dtype=torch.int32, device=DEV)
    _, ws = check_topk(z, lengths, K, 0.7)
    assert lib.poll_status(ws) == 32
    # rows with NaN or +inf give NaN in their own outputs, never a fault, and leave the other rows alone
    z[0, 0, 7] = float("nan")
    z[0, 1, 8] = float("inf")
    lengths = torch.full((B,), T, dtype=torch.int32, device=DEV)
    got = lib.topk_logprobs(z, lengths, K, 1.0, ws)
    ids, lp = ref.topk(z.double(), lengths, K, 1.0)
    clean = torch.ones((B, T), dtype=torch.bool, device=DEV)
    clean[0, :2] = False
    assert torch.equal(got.ids.long()[clean], ids[clean])
    assert torch.isnan(got.logprobs[0, :2]).any()
    assert lib.poll_status(ws) == 0


# ---------------------------------------------------------------- distillation
def teacher_entries(z, K, temperature, gen, noise=1.0):
    t = (z.float() + noise * torch.randn(z.shape, generator=gen, device=DEV)) / temperature
    k = min(K, z.shape[2])
    top, at = t.topk(k, dim=2)
    top = top - torch.logsumexp(t, dim=2, keepdim=True)
    ids = torch.full(z.shape[:2] + (K,), -1, dtype=torch.int32, device=DEV)
    lt = torch.zeros(z.shape[:2] + (K,), device=DEV)
    ids[..., :k] = torch.where(top > float("-inf"), at, -1).int()
    lt[..., :k] = top
    return ids, lt


def check_distill(z, ids, lt, lengths, mode, temperature, scale, out=None, z64=None, reach=64):
    B, T, V = z.shape
    z64 = z.double() if z64 is None else z64
    ws = lib.workspace(B, T, DEV)
    got = lib.distill_loss_fwd_bwd(z, ids, lt, lengths, mode, temperature, scale, ws, out)
    loss, rows, d, parts = ref.distill(z64, ids, lt, lengths, mode, temperature, scale)
    # a row's loss is a sum of p (log p - log q) with sum p <= 1 (+ p_0 of the same kind): every log is off by LP at most,
    # and the weights' relative errors (2^-22) meet logs below 64.  Where |x - M| reaches further, every rounding of it, and
    # the logs that the weights meet, grow in proportion.
    each = temperature ** 2 * (2 * LP + 2 ** -22 * 64) * reach / 64
    if got.row_loss is not None:
        off = (got.row_loss.double() - rows).abs()
        assert (off <= each + 2 ** -23 * rows.abs()).all(), off.max().item()
    assert abs(got.loss.item() - loss.item()) <= each + 2 ** -23 * abs(loss.item())
    if reach > 64:
        # An entry outside the list is e * mag with e = 2^(x - M) and mag = |g| 2^(M - Mmax) / sum; a thread's M is such that
        # e <= 2^64, and fp32 flushes below 2^-126: mag's flush loses at most 2^64 * 2^-126 = 2^-62, that of e at most |g| * 2^-126.
        q = torch.softmax(z64 / temperature, dim=2)
        outside = torch.ones_like(q).scatter_(2, ids.long().clamp(min=0), 0.0).bool() & (q > 0)
        g = torch.where(outside, parts / q.clamp(min=1e-300), 0.0).amax(dim=2, keepdim=True)
        lost = (2.0 ** -62 + g * 2.0 ** -126).expand_as(d)
        parts = parts + lost / LP
    check_gradient(got.dlogits, d, parts)
    return got, ws


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("B,T,V", [s for s in SIZES if s[2] > 1])
def test_distill_sizes(B, T, V, dtype):
    gen = torch.Generator(device=DEV).manual_seed(V + T)
    z, _ = ref.row_logits(B, T, V, dtype, gen, DEV)
    lengths = mixed_lengths(B, T)
    for mode, K, temperature in ((0, 1, 1.0), (1, 50, 2.0), (2, 256, 1.0), (2, 33, 1.5)):
        ids, lt = teacher_entries(z, K, temperature, gen)
        got, ws = check_distill(z, ids, lt, lengths, mode, temperature, 1000.0)
        assert lib.poll_status(ws) == 0
        pads = ~ref.valid_mask(lengths, T)
        assert (got.dlogits[pads] == 0).all() and (got.row_loss[pads] == 0).all()


@pytest.mark.parametrize("mode", [lib.DISTILL_PLAIN, lib.DISTILL_NORMALISED, lib.DISTILL_TAIL])
@pytest.mark.parametrize("layout", ["prompt", "pitch", "in_place", "other_offset", "strided_entries", "no_rows"])
@pytest.mark.parametrize("V", [1001, 20008])
def test_distill_layouts(layout, mode, V):
    gen = torch.Generator(device=DEV).manual_seed(41)
    B, T, K = 5, 6, 20
    kw = {"prompt": dict(prompt=3), "pitch": dict(pitch=5), "in_place": dict(prompt=2, offset=1, pitch=3)}
    z, store = ref.row_logits(B, T, V, BF, gen, DEV, **kw.get(layout, {}))
    lengths = mixed_lengths(B, T)
    ids, lt = teacher_entries(z, K, 1.0, gen)
    before, z64 = store.clone(), z.double()
    out = lib.DistillOutputs(z, in_place=layout == "in_place", want_row_loss=layout != "no_rows")
    if layout == "other_offset":
        out.dlogits = torch.full((B * T * V + 3,), 7.0, dtype=BF, device=DEV)[3:].view(B, T, V)
    if layout == "strided_entries":
        wide_i, wide_l = torch.zeros((T, B, K + 9), dtype=torch.int32, device=DEV), torch.zeros((T, B, K + 9), device=DEV)
        wide_i[..., 3:3 + K], wide_l[..., 3:3 + K] = ids.transpose(0, 1), lt.transpose(0, 1)
        ids, lt = wide_i[..., 3:3 + K].transpose(0, 1), wide_l[..., 3:3 + K].transpose(0, 1)
    check_distill(z, ids, lt, lengths, mode, 1.0, 100.0, out, z64)
    if layout == "in_place":
        keep = torch.ones_like(store, dtype=torch.bool)
        keep.as_strided(z.shape, z.stride(), z.storage_offset())[...] = False
        assert torch.equal(store.view(torch.int16)[keep], before.view(torch.int16)[keep])


@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("V", [1000, 20000, 50257, 128256])
def test_distill_entries_that_are_unused_out_of_range_or_repeated(V, mode):
    gen = torch.Generator(device=DEV).manual_seed(42)
    B, T, K = 3, 4, 70
    z, _ = ref.row_logits(B, T, V, BF, gen, DEV)
    ids, lt = teacher_entries(z, K, 1.0, gen)
    lt = lt - 0.5
    lengths = torch.full((B,), T, dtype=torch.int32, device=DEV)
    ids[0, 0] = -1                                       # a token without entries
    ids[0, 1, 1:] = -1
    ids[0, 2, 40:] = ids[0, 2, :30]                      # the same index twice
    ids[0, 3, 1::2] = ids[0, 3, 0]                       # the same index many times
    lt[0, 3] = -5.0
    lt[1, 0, 10:] = float("-inf")                        # entries of no weight
    z[1, 1, ids[1, 1, 5].long()] = float("-inf")         # deleted by the student, no weight in the teacher
    lt[1, 1, 5] = float("-inf")
    z[1, 2, :V // 2] = float("-inf")
    ids[1, 2], lt[1, 2] = torch.arange(V - K, V, device=DEV).int(), -5.0
    ids[2, 0] = torch.arange(K, device=DEV).int()        # neighbours, the row's first vectors
    lt[2, 0] = -4.5
    runs = [check_distill(z, ids, lt, lengths, mode, 1.0, 1.0) for _ in range(2)]
    assert lib.poll_status(runs[0][1]) == 0
    assert torch.equal(runs[0][0].dlogits, runs[1][0].dlogits) and torch.equal(runs[0][0].row_loss, runs[1][0].row_loss)
    ids[2, 1, 3], ids[2, 1, 4] = V, -2
    _, ws = check_distill(z, ids, lt, lengths, mode, 1.0, 1.0)
    assert lib.poll_status(ws) == 16


@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("V", [1000, 20000, 128256])
def test_distill_peaked_rows(V, mode):
    """A student with almost all of its mass on, or off, the teacher's entries: the sums must not be differences."""
    gen = torch.Generator(device=DEV).manual_seed(43)
    B, T, K = 2, 4, 16
    z, _ = ref.row_logits(B, T, V, BF, gen, DEV, sigma=0.5)
    ids, lt = teacher_entries(z, K, 1.0, gen)
    lt = torch.log_softmax(lt, dim=2) - 0.1
    for b, t, lift in ((0, 0, 25.0), (0, 1, -40.0), (0, 2, 60.0), (1, 0, 200.0)):
        z[b, t, ids[b, t].long()] += lift
    z[1, 1, :8] = 250.0                                  # far above the entries, in the row's first vector
    lengths = torch.full((B,), T, dtype=torch.int32, device=DEV)
    if mode == 2:                                        # 200 above: the mass outside leaves the range of fp32
        lengths[1] = 0
    got, _ = check_distill(z, ids, lt, lengths, mode, 1.0, 10.0)
    assert torch.isfinite(got.loss).all()


def test_distill_whole_vocabulary_named():
    """No entry outside the teacher's: the tail term is left out."""
    gen = torch.Generator(device=DEV).manual_seed(44)
    B, T, V = 2, 3, 100
    z, _ = ref.row_logits(B, T, V, BF, gen, DEV)
    ids, lt = teacher_entries(z, 120, 1.0, gen)
    lengths = torch.full((B,), T, dtype=torch.int32, device=DEV)
    for mode in (0, 1, 2):
        got, ws = check_distill(z, ids, lt - 0.2, lengths, mode, 1.0, 10.0)
        assert torch.isfinite(got.loss).all() and lib.poll_status(ws) == 0
    # the same where a deleted vocabulary leaves nothing else, on the kernel of long rows
    z, _ = ref.row_logits(B, T, 20000, BF, gen, DEV)
    ids, lt = teacher_entries(z, 64, 1.0, gen)
    keep = torch.zeros(z.shape, dtype=torch.bool, device=DEV).scatter_(2, ids.long(), True)
    z[~keep] = float("-inf")
    for mode in (0, 1, 2):
        got, ws = check_distill(z, ids, lt, lengths, mode, 1.0, 10.0)
        assert torch.isfinite(got.loss).all() and lib.poll_status(ws) == 0


def test_distill_without_tokens_and_lengths_out_of_range():
    gen = torch.Generator(device=DEV).manual_seed(45)
    for V in (1000, 20000):
        z, _ = ref.row_logits(3, 4, V, BF, gen, DEV)
        ids, lt = teacher_entries(z, 8, 1.0, gen)
        got, ws = check_distill(z, ids, lt, torch.zeros(3, dtype=torch.int32, device=DEV), 2, 1.0, 1.0)
        assert (got.loss == 0).all() and (got.dlogits == 0).all() and lib.poll_status(ws) == 0
        _, ws = check_distill(z, ids, lt, torch.tensor([9, -1, 2], dtype=torch.int32, device=DEV), 2, 1.0, 1.0)
        assert lib.poll_status(ws) == 32


def test_preference_with_deleted_tokens():
    """A response that holds a token its row deletes has log-prob -inf.  Where it is the rejected one, h = +inf: the pair is won
    (loss 0, no gradient).  Where it is the chosen one the loss is infinite and the gradient that of h -> -inf: f = -beta."""
    gen = torch.Generator(device=DEV).manual_seed(51)
    for T, V in ((3, 1000), (3, 20000), (700, 8200)):
        B = 4
        z, _ = ref.row_logits(B, T, V, BF, gen, DEV)
        ids, lengths = labels(B, T, V, gen), torch.full((B,), T, dtype=torch.int32, device=DEV)
        z[2, 1, ids[2, 1]] = float("-inf")               # pair 0: the rejected response
        ws = lib.workspace(B, T, DEV)
        for kind in (lib.PREF_SIGMOID, lib.PREF_HINGE):
            got = lib.preference_loss_fwd_bwd(z, ids, lengths, None, kind, 0.01, 0.0, 0.0, False, 1.0, ws)
            _, lp, _ = ref.label_logprobs(z.double(), ids, lengths)
            h = 0.01 * (lp[1].sum() - lp[3].sum())
            want = (torch.nn.functional.softplus(-h) if kind == 0 else (1 - h).clamp(min=0)) / 2
            # T log-probs of LP each, twice, times beta; both losses' slope in h is at most 1
            assert abs(got.loss.item() - want.item()) <= 0.01 * T * LP + 2.0 ** -23 * want.item()
            assert got.rewards[2].item() == float("-inf") and torch.isfinite(got.rewards[[0, 1, 3]]).all()
            assert (got.dlogits[0] == 0).all() and (got.dlogits[2] == 0).all() and not torch.isnan(got.dlogits).any()
        z[0], ids[0], z[2], ids[2] = z[2].clone(), ids[2].clone(), z[0].clone(), ids[0].clone()
        got = lib.preference_loss_fwd_bwd(z, ids, lengths, None, lib.PREF_SIGMOID, 0.01, 0.0, 0.0, False, 1.0, ws)
        assert got.loss.item() == float("inf") and got.rewards[0].item() == float("-inf")
        assert not torch.isnan(got.dlogits).any() and (got.dlogits[0] != 0).any()
        assert lib.poll_status(ws) == 0


@pytest.mark.parametrize("dtype,base", [(HF, 20000.0), (HF, -20000.0), (BF, 2.0 ** 20)])
@pytest.mark.parametrize("V", [1000, 1001, 8200, 20000, 20001, 50272, 128256])
def test_distill_far_logits(V, dtype, base):
    """Rows far from 0: differences to the row's maximum are what counts, and they are exact."""
    gen = torch.Generator(device=DEV).manual_seed(52)
    B, T, K = 2, 3, 20
    step = 16.0 if dtype == HF else 2.0 ** 13            # spacing of the type there
    z = torch.full((B, T, V), base, dtype=dtype, device=DEV)
    z[:, 1] -= step * torch.randint(0, 2, (B, V), generator=gen, device=DEV).to(dtype)
    lengths = torch.full((B,), T, dtype=torch.int32, device=DEV)
    ids, lt = teacher_entries(torch.zeros_like(z), K, 1.0, gen)
    for mode in (0, 1, 2):
        for temperature in (1.0, 0.5) if dtype == HF else (float(step), ):
            check_distill(z, ids, lt, lengths, mode, temperature, 1000.0)


@pytest.mark.parametrize("temperature", [0.05, 20.0, 1000.0])
@pytest.mark.parametrize("V", [1000, 20000, 50257, 128256])
def test_small_and_large_temperatures(V, temperature):
    gen = torch.Generator(device=DEV).manual_seed(53)
    B, T = 2, 4
    z, _ = ref.row_logits(B, T, V, BF, gen, DEV)
    lengths = torch.full((B,), T, dtype=torch.int32, device=DEV)
    assert z.float().abs().max().item() * 2 * 1.45 / 0.05 <= 1024
    check_topk(z, lengths, 30, temperature)
    ids, lt = teacher_entries(z, 30, temperature, gen)
    for mode in (0, 1, 2):
        check_distill(z, ids, lt, lengths, mode, temperature, 100.0, reach=1024 if temperature < 1 else 64)


@pytest.mark.parametrize("K", [1, 64, 65, 256])
@pytest.mark.parametrize("V", [8184, 8192, 8193, 32768, 52000, 53760, 57344, 57352, 61440, 65528, 65536, 65544, 106496, 114688,
                               114696, 131072, 212992, 229376, 229384, 262144])
def test_distill_at_the_borders_of_the_kernels(V, K):
    gen = torch.Generator(device=DEV).manual_seed(V + K)
    B, T = 2, 3
    z, _ = ref.row_logits(B, T, V, BF, gen, DEV)
    ids, lt = teacher_entries(z, K, 1.0, gen)
    lengths = torch.tensor([T, 1], dtype=torch.int32, device=DEV)
    _, ws = check_distill(z, ids, lt, lengths, 2, 1.0, 100.0)
    assert lib.poll_status(ws) == 0


def test_distill_strides_of_single_positions():
    """The stride of an axis with one position says nothing."""
    gen = torch.Generator(device=DEV).manual_seed(54)
    z, _ = ref.row_logits(1, 1, 1000, BF, gen, DEV)
    lengths = torch.ones(1, dtype=torch.int32, device=DEV)
    for K in (1, 8):
        ids, lt = teacher_entries(z, K, 1.0, gen)
        got, _ = check_distill(z, ids.as_strided((1, 1, K), (40, 3, 1)), lt.as_strided((1, 1, K), (0, 77, 1)), lengths, 2, 1.0, 1.0)
    one = lt[:, :, :1].as_strided((1, 1, 1), (5, 5, 9))
    check_distill(z, ids[:, :, :1], one, lengths, 0, 1.0, 1.0)
    z, _ = ref.row_logits(2, 3, 1000, BF, gen, DEV)
    ids, lt = teacher_entries(z, 8, 1.0, gen)
    with pytest.raises(ValueError, match="strides"):
        lib.distill_loss_fwd_bwd(z, ids, lt.transpose(0, 1).contiguous().transpose(0, 1), torch.ones(2, dtype=torch.int32, device=DEV),
                                 0, 1.0, 1.0, lib.workspace(2, 3, DEV))


@pytest.mark.parametrize("dtype,base", [(HF, 20000.0), (HF, -20000.0), (BF, 2.0 ** 20)])
@pytest.mark.parametrize("V", [1000, 1001, 8200, 20000, 20001, 50272, 128256, 300000])
def test_policy_and_preference_far_logits(V, dtype, base):
    """As above for the objectives of one token per row; a row's entries are one, two or more steps of their type apart."""
    gen = torch.Generator(device=DEV).manual_seed(55)
    B, T = 2, 3
    step = 16.0 if dtype == HF else 2.0 ** 13
    z = torch.full((B, T, V), base, dtype=dtype, device=DEV)
    few = torch.randint(0, V, (B, 5), generator=gen, device=DEV)
    z[:, 1].scatter_(1, few, base - step)
    ids, lengths = labels(B, T, V, gen), torch.full((B,), T, dtype=torch.int32, device=DEV)
    ids[:, 1] = torch.where((few == ids[:, 1:2]).any(dim=1), (few.max(dim=1).values + 1) % V, ids[:, 1])
    lp_old, lp_ref, adv = policy_inputs(z, ids, lengths, gen, False)
    check_policy(z, ids, lengths, lp_old, lp_ref, adv, 0.1, 0, 1000.0)
    check_preference(z, ids, lengths, lp_ref, 0, 0.3, 0.1, 0.0, False, 1000.0)


def test_log_probs_of_few_rows_have_no_bias():
    """A reward adds a sequence's log-probs, so that an error of the same sign in each counts.  Of 2048 log-probs near -10 (fp32
    spacing 2^-20, rounded to the nearest: standard deviation 2^-20 / sqrt(12) = 2.8e-7, and 2e-7 for that of the sum behind it)
    the mean is off by chance by 3.4e-7 / sqrt(2048) = 7.6e-9; five times that is allowed."""
    gen = torch.Generator(device=DEV).manual_seed(56)
    total, count = 0.0, 0
    for _ in range(32):
        z, _ = ref.row_logits(2, 32, 32000, BF, gen, DEV)
        ids, lengths = labels(2, 32, 32000, gen), torch.full((2,), 32, dtype=torch.int32, device=DEV)
        got = lib.preference_loss_fwd_bwd(z, ids, lengths, None, 0, 0.1, 0.0, 0.0, False, 1.0, lib.workspace(2, 32, DEV))
        _, lp, _ = ref.label_logprobs(z.double(), ids, lengths)
        total += (got.lp_new.double() - lp).sum().item()
        count += lp.numel()
    assert abs(total / count) <= 5 * 7.6e-9
