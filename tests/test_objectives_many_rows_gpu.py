"""The objectives with many rows per block: their buffers, entry sets, announcements, counters and candidate lists are used again
and again, and every row is still compared with its float64 definition.  The definition is formed a sequence at a time."""
import pytest
import torch

import objectives64 as ref
from paper_2410_15651_b200 import binding as lib
from test_objectives_gpu import BF, DEV, HF, LP, check_gradient, labels, policy_inputs, teacher_entries

pytestmark = pytest.mark.gpu


def ragged(B, T, gen):
    """Whole, empty, nearly empty and any lengths; more than half of the rows are valid."""
    n = torch.randint(T // 2, T + 1, (B,), generator=gen, device=DEV).int()
    n[1], n[2], n[3] = 0, 1, T
    return n


def batch(B, T, V, dtype, gen):
    z = torch.empty((B, T, V), dtype=dtype, device=DEV)
    for b in range(B):
        z[b] = 3.0 * torch.randn((T, V), generator=gen, device=DEV)
    return z


def gradient_shares(lengths, T, scale):
    """What a sequence alone has to be scaled by, so that its mean is its share of the batch's."""
    n = lengths.clamp(0, T).double()
    return (scale * n / n.sum().clamp(min=1)).tolist()


# rows per block or cluster: at least ten of valid ones.  One block with the exponentials in registers; with tensor memory; rows
# off 16-byte boundaries; a cluster of two with whole-slice buffers; the chunk ring in one block and in two; the kernel of short
# rows, three rows per block of eight per SM
@pytest.mark.parametrize("B,T,V,dtype", [(16, 190, 8200, BF), (16, 190, 20000, BF), (16, 190, 8201, HF), (16, 190, 20003, BF),
                                         (10, 120, 80000, BF), (16, 150, 57344, HF), (10, 120, 128256, BF), (20, 250, 1000, BF),
                                         (20, 250, 1001, HF)])
@pytest.mark.parametrize("K", [8, 64, 65, 96, 97, 200])
def test_distill(B, T, V, dtype, K):
    gen = torch.Generator(device=DEV).manual_seed(V + K)
    z, lengths = batch(B, T, V, dtype, gen), ragged(B, T, gen)
    ids = torch.empty((B, T, K), dtype=torch.int32, device=DEV)
    lt = torch.empty((B, T, K), device=DEV)
    for b in range(B):
        ids[b:b + 1], lt[b:b + 1] = teacher_entries(z[b:b + 1], K, 1.0, gen)
    ids[:, ::7, 1] = ids[:, ::7, 0]                      # the same entry twice in some rows
    ids[:, 3::11, K // 2:] = -1
    mode = (V + K) % 3
    ws = lib.workspace(B, T, DEV)
    got = lib.distill_loss_fwd_bwd(z, ids, lt, lengths, mode, 1.0, 1000.0, ws)
    again = lib.distill_loss_fwd_bwd(z, ids, lt, lengths, mode, 1.0, 1000.0, ws)
    assert torch.equal(got.dlogits, again.dlogits) and torch.equal(got.row_loss, again.row_loss) and torch.equal(got.loss, again.loss)
    assert lib.poll_status(ws) == 0
    each, total = 2 * LP + 2 ** -22 * 64, 0.0
    for b, scale in enumerate(gradient_shares(lengths, T, 1000.0)):
        s = slice(b, b + 1)
        _, rows, d, parts = ref.distill(z[s].double(), ids[s], lt[s], lengths[s], mode, 1.0, scale)
        off = (got.row_loss[s].double() - rows).abs()
        assert (off <= each + 2 ** -23 * rows.abs()).all(), (b, off.max().item())
        check_gradient(got.dlogits[s], d, parts)
        total += rows.sum().item()
    total /= lengths.sum().item()
    assert abs(got.loss.item() - total) <= each + 2 ** -23 * abs(total)


# several rows per block of each of the three block sizes (16, 8 and 4 blocks per SM), with rows that many equal values send to the
# bisection between ordinary ones
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("B,T,V,K", [(20, 300, 1000, 32), (12, 500, 7, 9), (14, 300, 8192, 200), (12, 250, 8200, 64),
                                     (12, 250, 20003, 64), (12, 250, 32000, 7), (12, 250, 50257, 256), (10, 250, 100003, 100)])
def test_topk(B, T, V, K, dtype):
    gen = torch.Generator(device=DEV).manual_seed(V + K)
    z, lengths = batch(B, T, V, dtype, gen), ragged(B, T, gen)
    z[:, 1::5] = z[:, 1::5].round()
    z[0, ::3] = 0.0
    z[3, ::4] = torch.linspace(-4, 4, V, device=DEV).to(dtype)
    z[3, 1::4, V // 3:] = float("-inf")
    ws = lib.workspace(B, T, DEV)
    for temperature in (1.0, 0.5):                       # twice on one workspace
        got = lib.topk_logprobs(z, lengths, K, temperature, ws)
        for b in range(B):
            s = slice(b, b + 1)
            ids, lp = ref.topk(z[s].double(), lengths[s], K, temperature)
            assert torch.equal(got.ids[s].long(), ids), b
            assert torch.equal(torch.isinf(got.logprobs[s]), torch.isinf(lp)), b
            fine = torch.isfinite(lp)
            off = (got.logprobs[s].double() - lp).abs()[fine]
            assert (off <= LP / temperature + 2.0 ** -22 * lp[fine].abs()).all(), (b, off.max().item())
    assert lib.poll_status(ws) == 0


@pytest.mark.parametrize("B,T,V,dtype", [(16, 190, 8200, BF), (16, 190, 20003, BF), (10, 120, 80000, HF), (16, 150, 57344, BF),
                                         (10, 120, 128256, BF), (16, 150, 1000, HF)])
def test_policy_and_preference(B, T, V, dtype):
    gen = torch.Generator(device=DEV).manual_seed(V)
    z, lengths = batch(B, T, V, dtype, gen), ragged(B, T, gen)
    ids = labels(B, T, V, gen)
    lp_old, lp_ref = torch.empty((B, T), device=DEV), torch.empty((B, T), device=DEV)
    adv = torch.empty((B, T), device=DEV)
    for b in range(B):
        s = slice(b, b + 1)
        lp_old[s], lp_ref[s], adv[s] = policy_inputs(z[s], ids[s], lengths[s], gen, False)
    ws = lib.workspace(B, T, DEV)
    pol = lib.policy_kl_loss_fwd_bwd(z, ids, lengths, lp_old, lp_ref, adv, 0.2, 0.3, 0.1, lib.MEAN_TOKENS, 1000.0, ws)
    pre = lib.preference_loss_fwd_bwd(z, ids, lengths, lp_ref, lib.PREF_SQUARED, 0.5, 0.0, 0.0, True, 10.0, ws)
    assert lib.poll_status(ws) == 0
    sums, rewards = [0.0, 0.0], []
    n = lengths.double()
    for b, scale in enumerate(gradient_shares(lengths, T, 1000.0)):
        s = slice(b, b + 1)
        z64 = z[s].double()
        pg, kl, d, lp, size = ref.policy_kl(z64, ids[s], lengths[s], lp_old[s], lp_ref[s], adv[s], 0.2, 0.3, 0.1, 0, scale)
        part = torch.softmax(z64, dim=2) + torch.nn.functional.one_hot(ids[s], V)
        check_gradient(pol.dlogits[s], d, size[..., None] * part)
        assert (pol.lp_new[s].double() - lp).abs().max() <= LP and (pre.lp_new[s].double() - lp).abs().max() <= LP
        share = (n[b] / n.sum()).item()
        sums = [sums[0] + share * pg.item(), sums[1] + share * kl.item()]
        rewards.append(0.5 * torch.where(ref.valid_mask(lengths[s], T), lp - lp_ref[s].double(), 0.0).sum() / n[b].clamp(min=1))
    assert abs(pol.loss[0].item() - sums[0]) <= 8 * LP + 2 ** -23 * abs(sums[0])
    assert abs(pol.loss[1].item() - sums[1]) <= 8 * LP + 2 ** -23 * abs(sums[1])
    # the preference loss: its own rewards (off by 0.5 LP), and the rows' gradients with the factor that these rewards give
    rewards = torch.stack(rewards)
    assert ((pre.rewards.double() - rewards).abs() <= 0.5 * LP + 2 ** -23 * rewards.abs()).all()
    h = rewards[:B // 2] - rewards[B // 2:]
    df = 2 / 0.25 * LP * 0.5 * 10.0 * 2 / B              # 2 / beta^2 per unit of h, off by LP; times beta, grad_scale, 2 / B
    f = 2 * (h - 0.5) / 0.25 * 0.5 * 10.0 * 2 / B
    f = torch.cat([f, -f]) / n.clamp(min=1)
    for b in range(B):
        s = slice(b, b + 1)
        lq, _, ok = ref.label_logprobs(z[s].double(), ids[s], lengths[s])
        d = ref.label_gradient(lq, ids[s], torch.where(ok, f[b], 0.0))
        part = torch.where(ok[..., None], lq.exp() + torch.nn.functional.one_hot(ids[s], V), 0.0)
        check_gradient(pre.dlogits[s], d, (f[b].abs() + df / n[b].clamp(min=1) / LP) * part)
