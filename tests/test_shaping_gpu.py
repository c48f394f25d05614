"""The operators on shaped logits on the GPU against their float64 definitions (shaping64.py).

Tolerances.  x is formed from z by at most six fp32 operations (a product with r or a rounded 1/r, a fused multiply-add of the
count, two sums, a product with a rounded 1/tau): each is off by 2^-24 of a value that is at most `parts`, the sum of the
absolute parts, so eight steps of it are allowed (X); entries that nothing moves are exact.  A 16-bit output adds half a step of
the value.  A log-prob adds the errors of exp, of the sums and of the logarithm: below 2e-5 (LP) as for the other objectives, and
the largest error of an x of its row, twice.  The entropy sums p |x - m| with relative errors of 2^-23 |x - m| + 2^-22 and of the
sums (twenty fp32 additions): with |x - m| of 15 in the mean and 225 in the mean square below 6e-5; 1e-4 is allowed
(ENT), and the rows' x errors times 40.  A gradient entry is a product of such quantities, rounded once: half a step of the
value plus LP (and, of the entropy's part, ENT) of the absolute parts, and half of the type's smallest step."""
import pytest
import torch

import shaping64 as ref
from objectives64 import row_logits
from paper_2410_15651_b200 import binding as lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, HF = torch.bfloat16, torch.float16
X, LP, ENT = 8 * 2.0 ** -24, 2e-5, 1e-4
ALL = ref.ALL


def tiny(dtype):
    return 2.0 ** -25 if dtype == HF else 2.0 ** -120


def mixed_lengths(B, T):
    pattern = [T, 0, 1, max(1, T - 1), T // 2, T]
    return torch.tensor([pattern[b % len(pattern)] for b in range(B)], dtype=torch.int32, device=DEV)


def same_but(got, want, tol, what):
    """Equal infinities, no NaN, and the rest within tol."""
    assert not torch.isnan(got).any(), what
    far = torch.isinf(want)
    assert torch.equal(got.double()[far], want[far]), what
    assert torch.isfinite(got[~far]).all(), what
    bad = ((got.double() - want).abs() - tol)[~far]
    assert (bad <= 0).all(), (what, bad.max().item())


def check_shape(z, lengths, kw, ws, out=None, dtype=None, store=None, z64=None):
    B, T, V = z.shape
    x, _, parts = ref.shaped(z if z64 is None else z64, lengths, kw)
    got = lib.shape_logits(z, lengths, lib.Shaping(B, V, **kw), ws, out=out, dtype=dtype)
    tol = X * parts
    if got.dtype != torch.float32:
        big = torch.finfo(got.dtype).max
        x = torch.where(x.abs() > big, torch.sign(x) * float("inf"), x)
        tol = tol + torch.finfo(got.dtype).eps / 2 * x.abs().clamp(max=big) + tiny(got.dtype)
    same_but(got, x, tol, "shape")
    return got


def row_error(parts):
    return X * parts.amax(dim=2)


def check_logprobs(z, ids, lengths, kw, ws, entropy=True):
    B, T, V = z.shape
    x, scale, parts = ref.shaped(z, lengths, kw)
    lp, ent, _, valid, _ = ref.logprobs(x, ids, lengths)
    got = lib.shaped_logprobs(z, ids, lengths, lib.Shaping(B, V, **kw), ws, want_entropy=entropy)
    err = row_error(parts)
    same_but(got.logprobs, lp, LP + 2 * err, "logprobs")
    if entropy:
        same_but(got.entropy, ent, ENT + 40 * err, "entropy")
    lse = got.lse.double().sum(dim=2)
    want = torch.where(valid, torch.logsumexp(x, dim=2), 0.0)
    some = want > float("-inf")
    assert ((lse - want).abs() <= LP + 2 * err + 2.0 ** -24 * want.abs())[some].all()
    return got


def check_logprobs_bwd(z, ids, lengths, kw, ws, forward, gen, with_entropy, out=None, z64=None):
    B, T, V = z.shape
    x, scale, parts = ref.shaped(z if z64 is None else z64, lengths, kw)
    g = torch.randn((B, T), generator=gen, device=DEV)
    h = 0.3 * torch.randn((B, T), generator=gen, device=DEV) if with_entropy else None
    want, size = ref.logprobs_grad(x, scale, ids, lengths, g, h)
    got = lib.shaped_logprobs_bwd(z, ids, lengths, lib.Shaping(B, V, **kw), forward, g, h, ws, out=out)
    rel = (ENT if with_entropy else LP) + (40 if with_entropy else 4) * row_error(parts)
    same_but(got, want, torch.finfo(z.dtype).eps / 2 * want.abs() + rel[..., None] * size + tiny(z.dtype), "logprobs_bwd")
    return got


def check_shape_bwd(z, lengths, kw, ws, gen, out=None, d=None, d64=None):
    B, T, V = z.shape
    _, scale, _ = ref.shaped(z, lengths, kw)
    d = torch.randn((B, T, V), generator=gen, device=DEV).to(z.dtype) if d is None else d
    valid = torch.arange(T, device=DEV)[None] < lengths.clamp(0, T)[:, None]
    want = torch.where(valid[..., None], (d.double() if d64 is None else d64) * scale, 0.0)
    got = lib.shape_logits_bwd(d, z, lengths, lib.Shaping(B, V, **kw), ws, out=out)
    same_but(got, want, (torch.finfo(z.dtype).eps / 2 + X) * want.abs() + tiny(z.dtype), "shape_bwd")
    return got


def labels(B, T, V, kw, gen):
    """Generated tokens: the history's own where there is one, some of them masked."""
    ids = torch.randint(0, V, (B, T), generator=gen, device=DEV)
    if "tokens" in kw and "start" not in kw:
        ids = torch.where(torch.rand((B, T), generator=gen, device=DEV) < 0.5, ids, kw["tokens"][:, :T])
    return ids


def everything(B, T, V, dtype, parts, seed, P=0, S0=0, repeat=8, layout=None, density=0.5):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    z, store = row_logits(B, T, V, dtype, gen, DEV, **(layout or {}))
    kw = ref.Settings(B, T, V, gen, DEV, parts, P=P, S0=S0, repeat=min(repeat, V), mask_density=density).kw
    lengths, ws = mixed_lengths(B, T), lib.workspace(B, T, DEV)
    ids = labels(B, T, V, kw, gen)
    check_shape(z, lengths, kw, ws)
    check_shape(z, lengths, kw, ws, dtype=torch.float32)
    check_shape_bwd(z, lengths, kw, ws, gen)
    forward = check_logprobs(z, ids, lengths, kw, ws)
    check_logprobs_bwd(z, ids, lengths, kw, ws, forward, gen, True)
    check_logprobs_bwd(z, ids, lengths, kw, ws, forward, gen, False)
    assert lib.poll_status(ws) == 0
    return z, store, kw, lengths, ids, ws, gen


# sizes around the kernels' borders: single entries, vectors, words of the mask, slices of 16384 entries, clusters of up to eight
# blocks and rows that need them twice
SIZES = [(1, 1, 1), (2, 3, 7), (3, 4, 8), (2, 2, 33), (4, 5, 1000), (3, 4, 1001), (2, 3, 16384), (2, 3, 16385), (2, 3, 16391),
         (3, 3, 32000), (3, 3, 50257), (2, 2, 131072), (2, 2, 131073), (1, 2, 140001), (2, 2, 151643), (1, 2, 300000)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("B,T,V", SIZES)
def test_sizes(B, T, V, dtype):
    everything(B, T, V, dtype, ALL + ("mask_rows", "bias"), V + T, P=9, S0=5)


# batches that are walked down sequence by sequence: several rows per block, several slices per row, rows that a cluster takes in
# turns, more than 32 rows between two tokens' tables, many listed entries
WALKS = [(6, 64, 50272, ALL, {}), (6, 64, 50272, ALL + ("mask_rows",), {}), (5, 70, 50257, ALL + ("mask",), {}),
         (4, 80, 32000, ("repetition", "tokens", "prompt"), {}), (3, 50, 128256, ALL + ("bias_own",), {}), (3, 40, 151643, ALL, {}),
         (2, 40, 400000, ALL, {}), (30, 40, 6000, ALL + ("mask_rows", "bias"), {}), (4, 40, 50257, ALL, dict(pitch=47)),
         (4, 40, 40003, ALL + ("mask_rows",), dict(pitch=5, offset=3)), (40, 40, 1000, ("presence", "tokens", "mask"), {}), (4, 100, 20000, (), {})]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("B,T,V,parts,layout", WALKS)
def test_walks(B, T, V, parts, layout, dtype):
    if V == 400000 and dtype == HF:
        B, V = 1, 280000
    everything(B, T, V, dtype, parts, V + T, P=200, S0=100 if V % 2 else 0, repeat=300, layout=layout, density=0.9)


@pytest.mark.parametrize("parts", [(), ("temperature",), ("bias",), ("bias_own",), ("mask",), ("mask_rows",), ("repetition", "prompt"),
                                   ("repetition", "tokens"), ("frequency", "tokens"), ("presence", "tokens"), ("repetition",),
                                   ("tokens", "prompt"), ("presence", "prompt"), ("frequency", "tokens", "prompt", "mask"),
                                   ("repetition", "tokens", "prompt", "bias_own")], ids=lambda p: "+".join(p) or "nothing")
@pytest.mark.parametrize("V", [4000, 4003])
def test_parts(V, parts):
    z, _, kw, lengths, _, ws, _ = everything(4, 6, V, BF, parts, 11, P=7)
    if not parts:                                        # nothing is moved: the rows themselves, bit by bit
        got = lib.shape_logits(z, lengths, lib.Shaping(4, V), ws)
        valid = torch.arange(6, device=DEV)[None] < lengths[:, None]
        assert torch.equal(got[valid].view(torch.int16), z[valid].view(torch.int16))


@pytest.mark.parametrize("layout", [dict(prompt=2), dict(pitch=5), dict(pitch=48), dict(offset=3), dict(offset=1, pitch=3, prompt=1)],
                         ids=lambda d: "+".join(f"{k}{v}" for k, v in d.items()))
@pytest.mark.parametrize("dtype", [BF, HF])
def test_layouts(layout, dtype):
    everything(3, 5, 20001, dtype, ALL + ("mask_rows", "bias_own"), 5, P=4, layout=layout)


@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 70])
def test_long_segments_and_long_histories(T):
    everything(2, T, 5000, BF, ALL, T, P=300, S0=700, repeat=40)


def test_long_answers_of_one_token():
    """A token that the answer has 70000 times."""
    B, T, V, S0 = 1, 2, 1000, 70000
    gen = torch.Generator(device=DEV).manual_seed(3)
    z, _ = row_logits(B, T, V, BF, gen, DEV)
    kw = dict(tokens=torch.full((B, S0 + T), 5, device=DEV), start=torch.full((B,), S0, dtype=torch.int32, device=DEV),
              frequency=torch.full((B,), 1e-4, device=DEV))
    ws = lib.workspace(B, T, DEV)
    got = check_shape(z, torch.full((B,), T, dtype=torch.int32, device=DEV), kw, ws, dtype=torch.float32)
    B2, T2 = 40, 40                                      # the same in a batch that is walked down
    y, _ = row_logits(B2, T2, V, BF, gen, DEV)
    many = dict(tokens=torch.full((B2, S0 + T2), 5, device=DEV), start=torch.full((B2,), S0, dtype=torch.int32, device=DEV),
                frequency=torch.full((B2,), 1e-4, device=DEV))
    check_shape(y, torch.full((B2,), T2, dtype=torch.int32, device=DEV), many, lib.workspace(B2, T2, DEV), dtype=torch.float32)
    check_logprobs(y, torch.full((B2, T2), 5, device=DEV), torch.full((B2,), T2, dtype=torch.int32, device=DEV), many, lib.workspace(B2, T2, DEV))
    assert abs(got[0, 0, 5].item() - (z[0, 0, 5].item() - 7.0)) < 1e-4 and lib.poll_status(ws) == 0


@pytest.mark.parametrize("B,T", [(4, 5), (40, 40)])
@pytest.mark.parametrize("V", [2000, 2001])
@pytest.mark.parametrize("parts", [ALL[:-1], ALL + ("mask",)], ids=["penalties", "dense"])
def test_in_place(V, parts, B, T):
    """Everything that may be written over its input, with nothing else touched."""
    gen = torch.Generator(device=DEV).manual_seed(V)
    kw = ref.Settings(B, T, V, gen, DEV, parts, P=6).kw
    lengths, ws = mixed_lengths(B, T), lib.workspace(B, T, DEV)
    z, store = row_logits(B, T, V, BF, gen, DEV, prompt=1, offset=1, pitch=3)
    keep = torch.ones_like(store, dtype=torch.bool)
    keep.as_strided(z.shape, z.stride(), z.storage_offset())[...] = False
    before, z0 = store.clone(), z.clone()
    ids = labels(B, T, V, kw, gen)
    d0 = torch.randn((B, T, V), generator=gen, device=DEV).to(BF)
    d = d0.clone()
    assert check_shape_bwd(z, lengths, kw, ws, gen, out=d, d=d, d64=d0.double()) is d
    forward = check_logprobs(z, ids, lengths, kw, ws)
    z64 = z.double()
    check_logprobs_bwd(z, ids, lengths, kw, ws, forward, gen, False, out=z, z64=z64)
    assert torch.equal(store.view(torch.int16)[keep], before.view(torch.int16)[keep])
    z.copy_(z0)
    assert check_shape(z, lengths, kw, ws, out=z, z64=z64) is z
    assert torch.equal(store.view(torch.int16)[keep], before.view(torch.int16)[keep]) and lib.poll_status(ws) == 0


@pytest.mark.parametrize("V", [4096, 4099])
def test_masks_that_leave_little_or_nothing(V):
    B, T = 4, 3
    gen = torch.Generator(device=DEV).manual_seed(21)
    z, _ = row_logits(B, T, V, BF, gen, DEV)
    allowed = torch.zeros((B, T, (V + 31) // 32 * 32), dtype=torch.bool, device=DEV)
    allowed[0, :, V - 1] = True                          # one entry
    allowed[1, 0] = True                                 # all of a row, nothing of the next
    allowed[2, :, 5:9] = True
    allowed[3, 2, V:] = True                             # only bits behind the vocabulary
    ids = torch.tensor([[V - 1, V - 1, 0], [7, 7, 7], [5, 8, 9], [0, 1, 2]], device=DEV)
    z[2, :, 9:12] = float("nan")                         # what is masked says nothing
    z[2, :, 20], z[2, :, 21] = float("inf"), float("-inf")
    z[0, :, 0] = torch.finfo(BF).min
    kw = dict(mask=ref.pack_mask(allowed), temperature=torch.full((B,), 0.7, device=DEV))
    lengths, ws = torch.full((B,), T, dtype=torch.int32, device=DEV), lib.workspace(B, T, DEV)
    clean = torch.where(torch.isfinite(z), z, 0.0)
    x, _, _ = ref.shaped(clean, lengths, kw)
    got = lib.shape_logits(z, lengths, lib.Shaping(B, V, **kw), ws, dtype=torch.float32)
    same_but(got, x, 1e-5 + 0 * x, "shape")
    f = lib.shaped_logprobs(z, ids, lengths, lib.Shaping(B, V, **kw), ws, want_entropy=True)
    lp, ent, _, _, _ = ref.logprobs(x, ids, lengths)
    same_but(f.logprobs, lp, LP + 1e-5 + 0 * lp, "logprobs")
    same_but(f.entropy, ent, ENT + 0 * ent, "entropy")
    assert f.logprobs[0].tolist() == [0, 0, float("-inf")] and (f.logprobs[3] == float("-inf")).all() and (f.entropy[3] == 0).all()
    for d in (lib.shaped_logprobs_bwd(z, ids, lengths, lib.Shaping(B, V, **kw), f, torch.ones_like(lp, dtype=torch.float32),
                                      torch.ones_like(lp, dtype=torch.float32), ws),
              lib.shape_logits_bwd(torch.full_like(z, float("nan")).masked_fill(allowed[..., :V], 1.0), z, lengths, lib.Shaping(B, V, **kw), ws)):
        assert torch.isfinite(d).all() and (d[~allowed[..., :V]] == 0).all()


@pytest.mark.parametrize("V", [2048, 40000])
def test_deleted_entries_and_rows_far_from_zero(V):
    B, T = 3, 4
    gen = torch.Generator(device=DEV).manual_seed(8)
    for dtype, far in ((BF, 0.0), (HF, 20000.0), (HF, -20000.0), (BF, 1e30)):
        z, _ = row_logits(B, T, V, dtype, gen, DEV)
        z += far
        z[..., 3::5] = float("-inf")
        kw = dict(tokens=torch.randint(0, 5, (B, T), generator=gen, device=DEV) * 5, presence=torch.full((B,), 0.5, device=DEV))
        lengths, ws = mixed_lengths(B, T), lib.workspace(B, T, DEV)
        ids = kw["tokens"].clone()
        check_shape(z, lengths, kw, ws, dtype=torch.float32)
        if abs(far) <= 20000:
            f = check_logprobs(z, ids, lengths, kw, ws)
            d = check_logprobs_bwd(z, ids, lengths, kw, ws, f, gen, True)
            assert (d[..., 3::5] == 0).all()


def test_one_token_far_above_the_others():
    """A sure token: its log-prob is far below one step of 1, and so is the gradient."""
    B, T, V = 1, 2, 30000
    gen = torch.Generator(device=DEV).manual_seed(4)
    for gap in (12.0, 30.0, 80.0, 3000.0):
        z = torch.randn((B, T, V), generator=gen, device=DEV).to(BF)
        z[..., 17] = gap
        z[0, 1, 29999] = gap + (4 if gap < 100 else 64)
        ids = torch.tensor([[17, 17]], device=DEV)
        n, ws = torch.full((B,), T, dtype=torch.int32, device=DEV), lib.workspace(B, T, DEV)
        f = check_logprobs(z, ids, n, {}, ws)
        # (the mass beside the token is 1e-30 of it: lost in a sum of all, even in 64 bits)
        others = torch.cat([z[0, 0, :17], z[0, 0, 18:]]).double()
        lp = -torch.log1p(torch.exp(others - gap).sum())
        assert abs(f.logprobs[0, 0].item() - lp.item()) <= 1e-5 * abs(lp.item()) + 2.0 ** -126
        d = check_logprobs_bwd(z, ids, n, {}, ws, f, gen, False)
        got = lib.shaped_logprobs_bwd(z, ids, n, lib.Shaping(B, V), f, torch.ones((B, T), device=DEV), None, ws)
        want = -torch.expm1(lp).item()
        # (bf16 has 8 significant bits: half a step is up to 2^-8 of the value)
        assert abs(got[0, 0, 17].item() - want) <= (2.0 ** -8 + 1e-5) * want + 2.0 ** -126 and d.shape == z.shape


def test_bad_tokens_lengths_and_settings():
    B, T, V = 5, 4, 1000
    gen = torch.Generator(device=DEV).manual_seed(2)
    z, _ = row_logits(B, T, V, BF, gen, DEV)
    ws = lib.workspace(B, T, DEV)
    full = torch.full((B,), T, dtype=torch.int32, device=DEV)
    tokens, prompt = torch.randint(0, V, (B, T), generator=gen, device=DEV), torch.randint(0, V, (B, 3), generator=gen, device=DEV)
    rep = torch.full((B,), 1.3, device=DEV)
    ids = torch.randint(0, V, (B, T), generator=gen, device=DEV)

    def flags(lengths=full, ids=ids, **kw):
        settings = dict(dict(tokens=tokens, prompt=prompt, repetition=rep), **kw)
        sh = lib.Shaping(B, V, **settings)
        out = []
        lib.shape_logits(z, lengths, sh, ws)
        out.append(lib.poll_status(ws))
        lib.shape_logits_bwd(z, z, lengths, sh, ws)
        out.append(lib.poll_status(ws))
        f = lib.shaped_logprobs(z, ids, lengths, sh, ws, want_entropy=True)
        out.append(lib.poll_status(ws))
        lib.shaped_logprobs_bwd(z, ids, lengths, sh, f, f.logprobs, None, ws)
        out.append(lib.poll_status(ws))
        return out

    assert flags() == [0] * 4
    bad = tokens.clone()
    bad[1, 0] = V
    assert flags(tokens=bad) == [16] * 4
    bad[1, 0], bad[2, 3] = -1, -7                        # -1 is no token, and the last token is nobody's history
    assert flags(tokens=bad) == [0] * 4
    check_shape(z, full, dict(tokens=bad, repetition=rep), ws)
    bad = prompt.clone()
    bad[4, 2] = -2
    assert flags(prompt=bad) == [16] * 4
    n = full.clone()
    n[0], n[1] = T + 1, -3
    assert flags(lengths=n) == [32] * 4
    check_shape(z, n, dict(tokens=tokens, repetition=rep), ws)
    lib.poll_status(ws)
    start = torch.zeros(B, dtype=torch.int32, device=DEV)
    start[3] = 1                                         # the last row's history is all tokens: enough
    assert flags(start=start) == [0] * 4
    start[3] = 2
    assert flags(start=start) == [32] * 4
    start[3] = -1
    assert flags(start=start) == [32] * 4
    assert flags(prompt_lengths=torch.full((B,), 4, dtype=torch.int32, device=DEV)) == [32] * 4
    assert flags(prompt_lengths=torch.full((B,), -1, dtype=torch.int32, device=DEV)) == [32] * 4
    for name, values in (("repetition", (0.0, -1.0, float("nan"), float("inf"))), ("temperature", (0.0, -1.0, float("nan"), float("inf"))),
                         ("frequency", (float("nan"), float("inf"))), ("presence", (float("nan"), float("-inf")))):
        neutral = torch.full((B,), 1.0 if name in ("repetition", "temperature") else 0.0, device=DEV)
        want = lib.shape_logits(z, full, lib.Shaping(B, V, **dict(dict(tokens=tokens, repetition=rep), **{name: neutral})), ws)
        for v in values:
            s = neutral.clone()
            s[2] = v
            assert flags(**{name: s}) == [128] * 4, (name, v)
            got = lib.shape_logits(z, full, lib.Shaping(B, V, **dict(dict(tokens=tokens, repetition=rep), **{name: s})), ws)
            assert torch.equal(got, want) and lib.poll_status(ws) == 128
    wrong = ids.clone()
    wrong[0, 0], wrong[4, 3] = V, -1
    assert flags(ids=wrong) == [0, 0, 16, 16]
    sh = lib.Shaping(B, V, tokens=tokens, repetition=rep)
    f = lib.shaped_logprobs(z, wrong, full, sh, ws, want_entropy=True)
    assert f.logprobs[0, 0] == 0 and f.logprobs[4, 3] == 0
    g = torch.randn((B, T), generator=gen, device=DEV)
    d = lib.shaped_logprobs_bwd(z, wrong, full, sh, f, g, None, ws)
    assert (d[0, 0] == 0).all() and (d[4, 3] == 0).all() and (d[0, 1] != 0).any()
    lib.poll_status(ws)


def test_equal_to_the_plain_log_probs_where_nothing_is_shaped():
    B, T, V = 4, 6, 50272
    gen = torch.Generator(device=DEV).manual_seed(6)
    z, _ = row_logits(B, T, V, BF, gen, DEV)
    ids, lengths, ws = torch.randint(0, V, (B, T), generator=gen, device=DEV), mixed_lengths(B, T), lib.workspace(B, T, DEV)
    ent = torch.empty((B, T), device=DEV)
    lp = lib.gather_logprobs(z, ids, lengths, ws, out_entropy=ent)
    f = lib.shaped_logprobs(z, ids, lengths, lib.Shaping(B, V), ws, want_entropy=True)
    assert (f.logprobs - lp).abs().max() <= 2 * LP and (f.entropy - ent).abs().max() <= 2 * ENT


def test_gradients_against_differences():
    """The float64 loss along random directions, and the gradients of both backward passes."""
    B, T, V = 2, 4, 600
    gen = torch.Generator(device=DEV).manual_seed(12)
    z, _ = row_logits(B, T, V, HF, gen, DEV)
    z = torch.where(z.abs() < 0.05, 0.1, z).to(HF)       # away from 0, where the penalty has a kink
    kw = ref.Settings(B, T, V, gen, DEV, ALL + ("mask_rows", "bias"), P=5).kw
    lengths, ws = mixed_lengths(B, T), lib.workspace(B, T, DEV)
    lengths[1] = 3
    ids = torch.randint(0, V, (B, T), generator=gen, device=DEV)
    allowed = ((kw["mask"][..., None] >> torch.arange(32, device=DEV)) & 1).bool().flatten(2)
    allowed.scatter_(2, ids[..., None], True)
    kw["mask"] = ref.pack_mask(allowed)
    g, h = torch.randn((B, T), generator=gen, device=DEV), torch.randn((B, T), generator=gen, device=DEV)
    sh = lib.Shaping(B, V, **kw)
    f = lib.shaped_logprobs(z, ids, lengths, sh, ws, want_entropy=True)
    d = lib.shaped_logprobs_bwd(z, ids, lengths, sh, f, g, h, ws).double()
    w = torch.randn((B, T, V), generator=gen, device=DEV).to(HF)
    ds = lib.shape_logits_bwd(w, z, lengths, sh, ws).double()

    def loss(y):
        x, _, _ = ref.shaped(y, lengths, kw)
        lp, ent, _, valid, _ = ref.logprobs(x, ids, lengths)
        linear = torch.where(valid[..., None] & (x > float("-inf")), w.double() * x, 0.0).sum()
        return (g.double() * lp + h.double() * ent)[valid].sum(), linear

    for seed in range(4):
        v = torch.randn(z.shape, generator=gen, device=DEV).double()
        up, down = loss(z.double() + 1e-6 * v), loss(z.double() - 1e-6 * v)
        for got, a, b in ((d, up[0], down[0]), (ds, up[1], down[1])):
            # every entry is rounded by up to half a step of fp16; the direction adds them up at random: their root sum of squares, five-fold
            noise = 5 * (2.0 ** -11 * (got * v)).square().sum().sqrt() + 5 * 2.0 ** -25 * v.norm()
            assert abs((got * v).sum() - (a - b) / 2e-6) <= noise + 1e-4 * (got * v).abs().sum(), seed


def test_offsets_beyond_32_bits():
    """Rows whose elements lie more than 2^32 bytes (and 2^31 elements) apart."""
    B, T, V = 2, 2, 5000
    gen = torch.Generator(device=DEV).manual_seed(30)
    store = torch.empty((2 ** 31 + 4 * V,), dtype=BF, device=DEV)
    out = torch.empty_like(store)
    z, o = (s.as_strided((B, T, V), (2 ** 31, V + 8, 1)) for s in (store, out))
    z.copy_(3 * torch.randn((B, T, V), generator=gen, device=DEV))
    kw = ref.Settings(B, T, V, gen, DEV, ALL, P=4).kw
    lengths, ws = torch.full((B,), T, dtype=torch.int32, device=DEV), lib.workspace(B, T, DEV)
    ids = labels(B, T, V, kw, gen)
    check_shape(z, lengths, kw, ws, out=o)
    check_shape_bwd(z, lengths, kw, ws, gen, out=o)
    f = check_logprobs(z, ids, lengths, kw, ws)
    check_logprobs_bwd(z, ids, lengths, kw, ws, f, gen, True, out=o)


def test_repeated_calls_are_bit_identical():
    B, T, V = 8, 40, 20000
    gen = torch.Generator(device=DEV).manual_seed(9)
    z, _ = row_logits(B, T, V, BF, gen, DEV)
    kw = ref.Settings(B, T, V, gen, DEV, ALL + ("mask_rows", "bias"), P=50, repeat=30).kw
    lengths, ws, sh = mixed_lengths(B, T), lib.workspace(B, T, DEV), lib.Shaping(B, V, **kw)
    ids = labels(B, T, V, kw, gen)

    def once():
        f = lib.shaped_logprobs(z, ids, lengths, sh, ws, want_entropy=True)
        x = lib.shape_logits(z, lengths, sh, ws)
        return [x, f.logprobs, f.lse, f.entropy, lib.shaped_logprobs_bwd(z, ids, lengths, sh, f, f.entropy, f.entropy, ws),
                lib.shape_logits_bwd(x.masked_fill(torch.isinf(x), 0.0), z, lengths, sh, ws)]

    first = once()
    for _ in range(3):
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(once(), first))
