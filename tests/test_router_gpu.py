"""The router's balance loss on the GPU against its float64 definition (shaping64.py).

Tolerances.  A probability is formed in fp32 as a quotient of hardware exponentials: with exponents up to 64 it is off by 64 *
2^-23 * ln 2 from the exponent, 2^-22 from the exponential and 2^-22 from sum and quotient: 2e-5 (REL) of its value is allowed.  The dot
product and f are sums of such and of one rounding, so a gradient entry is off by REL of its absolute parts, half a step of
its type, and half of the type's smallest step.  The losses are means of REL-exact terms summed in double and rounded once:
REL of the mean absolute term.  Counts and chosen experts are whole numbers and equal."""
import pytest
import torch

import shaping64 as ref
from paper_2410_15651_b200 import binding as lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, HF, FF = torch.bfloat16, torch.float16, torch.float32
REL = 2e-5


def tiny(dtype):
    return 2.0 ** -25 if dtype == HF else 2.0 ** -120


def mixed_lengths(B, T):
    pattern = [T, 0, 1, max(1, T - 1), T // 2, T]
    return torch.tensor([pattern[b % len(pattern)] for b in range(B)], dtype=torch.int32, device=DEV)


def logits(L, B, T, E, dtype, gen, sigma=1.0, lead=0, pitch=0):
    store = torch.full((L * B * T * (E + pitch) + lead + 8,), float("nan"), dtype=dtype, device=DEV)
    z = store[lead:lead + L * B * T * (E + pitch)].view(L, B, T, E + pitch)[..., :E]
    z.copy_(sigma * torch.randn((L, B, T, E), generator=gen, device=DEV))
    return z, store


def choose(z, k, gen):
    """Experts chosen elsewhere: some none, some twice by a token."""
    ids = torch.randint(0, z.shape[3], z.shape[:3] + (k,), generator=gen, device=DEV, dtype=torch.int32)
    return ids.masked_fill(torch.rand(ids.shape, generator=gen, device=DEV) < 0.1, -1)


def check(z, lengths, k, scoring, scope, balance, zc, scale, ws, expert_ids=None, out=None, z64=None):
    got = lib.router_loss_fwd_bwd(z, lengths, k, scoring, scope, balance, zc, scale, ws, expert_ids=expert_ids, out=out)
    loss, counts, ids, d, parts = ref.router(z if z64 is None else z64, lengths, k, scoring, scope == lib.ROUTER_SEQUENCE, balance, zc,
                                             scale, expert_ids)
    assert torch.equal(got.counts, counts)
    if expert_ids is None and got.ids is not None:
        assert torch.equal(got.ids, ids)
    assert ((got.loss.double() - loss).abs() <= REL * loss.abs().clamp(min=1e-30) + 1e-30).all(), (got.loss, loss)
    tol = torch.finfo(z.dtype).eps / 2 * d.abs() + REL * parts + tiny(z.dtype)
    assert torch.isfinite(got.dlogits).all()
    bad = (got.dlogits.double() - d).abs() - tol
    assert (bad <= 0).all(), (bad.max().item(), d.abs().max().item())
    pad = torch.arange(z.shape[2], device=DEV)[None] >= lengths.clamp(0, z.shape[2])[:, None]
    assert (got.dlogits[:, pad] == 0).all()
    return got


# lanes per token 1 .. 32 with one vector each, two and four vectors, experts off a multiple of 8, one token, many chunks
SIZES = [(1, 1, 1, 1, 1), (1, 2, 3, 3, 2), (2, 3, 5, 8, 2), (1, 4, 33, 16, 4), (3, 2, 40, 60, 6), (2, 6, 50, 64, 6), (1, 6, 100, 128, 8),
         (2, 3, 17, 250, 8), (1, 6, 64, 256, 8), (2, 2, 9, 264, 3), (1, 3, 20, 512, 8), (1, 2, 11, 1024, 16), (1, 2, 11, 1001, 5),
         (1, 40, 300, 8, 2), (1, 700, 1, 32, 4), (40, 2, 3, 12, 12)]


@pytest.mark.parametrize("dtype", [BF, HF, FF])
@pytest.mark.parametrize("L,B,T,E,K", SIZES)
def test_sizes(L, B, T, E, K, dtype):
    gen = torch.Generator(device=DEV).manual_seed(E + T)
    z, _ = logits(L, B, T, E, dtype, gen)
    lengths, ws = mixed_lengths(B, T), lib.router_workspace(L, B, T, E, DEV)
    for scope in (lib.ROUTER_BATCH, lib.ROUTER_SEQUENCE):
        check(z, lengths, K, lib.ROUTER_SOFTMAX, scope, 0.5, 0.1, 100.0, ws)
        check(z, lengths, K, lib.ROUTER_SIGMOID, scope, 0.5, 0.0, 100.0, ws, choose(z, K, gen))
    assert lib.poll_status(ws) == 0


@pytest.mark.parametrize("dtype", [BF, FF])
@pytest.mark.parametrize("layout", ["pitch", "lead", "pitch_and_lead", "layers_last", "in_place", "other_out", "strided_ids"])
def test_layouts(layout, dtype):
    L, B, T, E, K = 2, 4, 9, 64, 4
    gen = torch.Generator(device=DEV).manual_seed(3)
    kw = {"pitch": dict(pitch=3), "lead": dict(lead=1), "pitch_and_lead": dict(pitch=8, lead=8), "in_place": dict(pitch=2, lead=5)}
    z, store = logits(L, B, T, E, dtype, gen, **kw.get(layout, {}))
    lengths, ws = mixed_lengths(B, T), lib.router_workspace(L, B, T, E, DEV)
    out, ids, z64 = None, None, z.double()
    if layout == "layers_last":                          # [B,T,L,E] in memory
        z = z.permute(1, 2, 0, 3).contiguous().permute(2, 0, 1, 3)
        out = lib.RouterOutputs(z, K, lib.ROUTER_BATCH)
        out.dlogits = torch.empty_strided(z.shape, z.stride(), dtype=dtype, device=DEV)
    elif layout == "in_place":
        before = store.clone()
        out = lib.RouterOutputs(z, K, lib.ROUTER_BATCH, in_place=True)
    elif layout == "other_out":
        out = lib.RouterOutputs(z, K, lib.ROUTER_BATCH)
        out.dlogits = torch.full((L * B * T * (E + 1) + 1,), 7.0, dtype=dtype, device=DEV)[1:].view(L, B, T, E + 1)[..., :E]
    elif layout == "strided_ids":
        ids = choose(z, 2 * K, gen)[..., 3:3 + K]
    check(z, lengths, K, lib.ROUTER_SOFTMAX, lib.ROUTER_BATCH, 1.0, 0.01, 10.0, ws, ids, out, z64)
    if layout == "in_place":
        keep = torch.ones_like(store, dtype=torch.bool)
        keep.as_strided(z.shape, z.stride(), z.storage_offset())[...] = False
        assert torch.equal(store.view(torch.uint8).view(store.numel(), -1)[keep], before.view(torch.uint8).view(store.numel(), -1)[keep])


def test_ties_go_to_the_lowest_expert():
    gen = torch.Generator(device=DEV).manual_seed(5)
    for E in (8, 48, 256, 512):
        z = torch.randint(-2, 3, (1, 3, 50, E), generator=gen, device=DEV).to(BF)
        z = torch.where(torch.rand(z.shape, generator=gen, device=DEV) < 0.5, -z, z)       # zeros of both signs
        ws = lib.router_workspace(1, 3, 50, E, DEV)
        check(z, torch.tensor([50, 50, 7], dtype=torch.int32, device=DEV), 6, 0, 0, 1.0, 0.0, 1.0, ws)


def test_deleted_experts_and_extreme_logits():
    gen = torch.Generator(device=DEV).manual_seed(6)
    for dtype in (BF, FF):
        z, _ = logits(1, 2, 20, 32, dtype, gen)
        z[..., 5:9] = float("-inf")
        z[0, 0, 3] = float("-inf")
        z[0, 0, 4] = 1e30
        z[0, 0, 5, 11] = -1e38
        ws = lib.router_workspace(1, 2, 20, 32, DEV)
        n = torch.full((2,), 20, dtype=torch.int32, device=DEV)
        got = check(z, n, 2, lib.ROUTER_SOFTMAX, lib.ROUTER_BATCH, 1.0, 0.0, 1.0, ws, torch.zeros((1, 2, 20, 2), dtype=torch.int32, device=DEV))
        assert (got.dlogits[z == float("-inf")] == 0).all()
        z[0, 0, 3] = 0
        for sigma in (30.0, 1e4):                        # probabilities of 0 and 1
            y = torch.where(torch.isinf(z), z, (sigma * z.clamp(-3, 3).float()).to(dtype))
            check(y, n, 3, lib.ROUTER_SIGMOID, lib.ROUTER_SEQUENCE, 1.0, 0.0, 1.0, ws)


def test_no_tokens_and_bad_inputs():
    gen = torch.Generator(device=DEV).manual_seed(7)
    L, B, T, E, K = 2, 3, 6, 24, 3
    z, _ = logits(L, B, T, E, BF, gen)
    ws = lib.router_workspace(L, B, T, E, DEV)
    none = torch.zeros(B, dtype=torch.int32, device=DEV)
    for scope in (0, 1):
        got = check(z, none, K, 0, scope, 1.0, 1.0, 1.0, ws)
        assert (got.loss == 0).all() and (got.counts == 0).all() and (got.dlogits == 0).all() and (got.ids == 0).all()
    assert lib.poll_status(ws) == 0
    check(z, torch.tensor([T + 4, -1, 2], dtype=torch.int32, device=DEV), K, 0, 0, 1.0, 1.0, 1.0, ws)
    assert lib.poll_status(ws) == 32
    ids = choose(z, K, gen)
    ids[0, 0, 1, 0], ids[1, 0, 0, 2] = E, -2
    n = torch.tensor([T, 2, 1], dtype=torch.int32, device=DEV)
    check(z, n, K, 0, 1, 1.0, 0.0, 1.0, ws, ids)
    assert lib.poll_status(ws) == 16
    ids[0, 0, 1, 0], ids[1, 0, 0, 2], ids[0, 2, 5, 0] = 0, -1, 99        # the last one is padding
    check(z, n, K, 0, 1, 1.0, 0.0, 1.0, ws, ids)
    assert lib.poll_status(ws) == 0
    with pytest.raises(lib.RlhfError, match="WORKSPACE"):
        lib.router_loss_fwd_bwd(z, n, K, 0, 0, 1.0, 0.0, 1.0, ws[:1024])


def test_balanced_experts():
    """Experts that are chosen equally often: the loss is 1 and the gradient 0 to rounding, however peaked the tokens are."""
    E, K = 16, 2
    z = torch.zeros((1, 1, E, E), device=DEV)
    for t in range(E):
        z[0, 0, t, t], z[0, 0, t, (t + 1) % E] = 6.0, 5.0
    ws = lib.router_workspace(1, 1, E, E, DEV)
    got = check(z, torch.full((1,), E, dtype=torch.int32, device=DEV), K, 0, 0, 1.0, 0.0, 1.0, ws)
    assert got.loss[0, 0].item() == 1.0 and got.dlogits.abs().max().item() == 0.0


@pytest.mark.parametrize("scoring,scope", [(0, 0), (0, 1), (1, 0), (1, 1)])
def test_gradient_against_differences(scoring, scope):
    gen = torch.Generator(device=DEV).manual_seed(9)
    L, B, T, E, K = 2, 3, 5, 12, 2
    z, _ = logits(L, B, T, E, FF, gen)
    ids, n = choose(z, K, gen), torch.tensor([5, 0, 3], dtype=torch.int32, device=DEV)
    ws, zc = lib.router_workspace(L, B, T, E, DEV), 0.2 if scoring == 0 else 0.0
    got = lib.router_loss_fwd_bwd(z, n, K, scoring, scope, 0.7, zc, 3.0, ws, expert_ids=ids)

    def loss(y):
        v = ref.router(y, n, K, scoring, scope == 1, 0.7, zc, 3.0, ids)[0]
        return 3.0 * (0.7 * v[:, 0] + zc * v[:, 1]).sum()

    for _ in range(3):
        v = torch.randn(z.shape, generator=gen, device=DEV).double()
        slope = (loss(z.double() + 1e-5 * v) - loss(z.double() - 1e-5 * v)) / 2e-5
        terms = (got.dlogits.double() * v)
        assert abs(terms.sum() - slope) <= 1e-4 * terms.abs().sum()


def test_repeated_calls_are_bit_identical_and_leave_the_workspace_ready():
    gen = torch.Generator(device=DEV).manual_seed(10)
    ws = lib.router_workspace(4, 8, 512, 128, DEV)
    cases = []
    for L, B, T, E, K, scope in ((4, 8, 512, 128, 8, 0), (1, 2, 7, 8, 2, 1), (2, 8, 100, 64, 4, 1), (1, 8, 512, 128, 8, 0)):
        z, _ = logits(L, B, T, E, BF, gen)
        cases.append((z, mixed_lengths(B, T), K, 0, scope, 0.1, 0.01, 100.0, ws))
    first = [lib.router_loss_fwd_bwd(*c) for c in cases]
    for _ in range(3):
        for c, f in zip(cases, first):
            o = lib.router_loss_fwd_bwd(*c)
            assert torch.equal(o.loss, f.loss) and torch.equal(o.counts, f.counts) and torch.equal(o.ids, f.ids)
            assert torch.equal(o.dlogits.view(torch.int16), f.dlogits.view(torch.int16))


def test_offsets_beyond_32_bits():
    L, B, T, E, K = 2, 2, 3, 40, 4
    gen = torch.Generator(device=DEV).manual_seed(11)
    store = torch.empty((2 ** 31 + 4096,), dtype=FF, device=DEV)
    z = store.as_strided((L, B, T, E), (2 ** 31, 1024, E, 1))
    z.copy_(torch.randn((L, B, T, E), generator=gen, device=DEV))
    out = lib.RouterOutputs(z, K, 0)
    out.dlogits = torch.empty_like(store).as_strided(z.shape, z.stride())
    check(z, mixed_lengths(B, T), K, 0, 0, 1.0, 0.1, 1.0, lib.router_workspace(L, B, T, E, DEV), None, out)
