"""The policy loss with KL where one of its two parts is switched off and the other's exponentials leave the range of fp32."""
import pytest
import torch

import objectives64 as ref
from paper_2410_15651_b200 import binding as lib
from test_objectives_gpu import BF, DEV, HF, LP, check_gradient, labels, policy_inputs

pytestmark = pytest.mark.gpu

# generic row kernel, streamed chunks, one block, off 16-byte boundaries, chunk ring (one block, two), streamed twice
VOCABULARIES = [1000, 1001, 8200, 20001, 32000, 57344, 128256, 300000]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("V", VOCABULARIES)
def test_kl_reported_but_not_trained_on(V, dtype):
    """kl_coef = 0: the gradient is that of the policy part, however far the reference is, and where the row deletes its token; the
    KL is reported all the same, and is infinite there."""
    gen = torch.Generator(device=DEV).manual_seed(V)
    B, T = 4, 3
    z, _ = ref.row_logits(B, T, V, dtype, gen, DEV)
    ids, lengths = labels(B, T, V, gen), torch.tensor([T, T, 0, 1], dtype=torch.int32, device=DEV)
    lp_old, lp_ref, adv = policy_inputs(z, ids, lengths, gen, True)
    lp_ref[0, 1] += 100.0
    lp_ref[1, 2] += 1e4
    ws = lib.workspace(B, T, DEV)
    got = lib.policy_kl_loss_fwd_bwd(z, ids, lengths, lp_old, lp_ref, adv, 0.2, 0.3, 0.0, 0, 100.0, ws)
    pg, _, d, lp, size = ref.policy_kl(z.double(), ids, lengths, lp_old, None, adv, 0.2, 0.3, 0.0, 0, 100.0)
    part = torch.softmax(z.double(), dim=2) + torch.nn.functional.one_hot(ids, V)
    check_gradient(got.dlogits, d, size[..., None] * part)
    assert abs(got.loss[0].item() - pg.item()) <= 8 * LP + 2 ** -23 * abs(pg.item())
    assert got.loss[1].item() == float("inf")            # exp(1e4)
    # a token that its row deletes: ratio 0
    z[0, 0, ids[0, 0]] = float("-inf")
    lp_ref[0, 1] -= 100.0
    lp_ref[1, 2] -= 1e4
    got = lib.policy_kl_loss_fwd_bwd(z, ids, lengths, lp_old, lp_ref, adv, 0.2, 0.3, 0.0, 0, 100.0, ws)
    pg, _, d, lp, size = ref.policy_kl(z.double(), ids, lengths, lp_old, None, adv, 0.2, 0.3, 0.0, 0, 100.0)
    part = torch.softmax(z.double(), dim=2) + torch.nn.functional.one_hot(ids, V)
    check_gradient(got.dlogits, d, size[..., None] * part)
    assert abs(got.loss[0].item() - pg.item()) <= 8 * LP + 2 ** -23 * abs(pg.item())
    assert got.loss[1].item() == float("inf") and got.lp_new[0, 0].item() == float("-inf")
    assert lib.poll_status(ws) == 0


@pytest.mark.parametrize("V", VOCABULARIES)
def test_no_advantage_and_a_ratio_beyond_fp32(V):
    """An advantage of 0 (a group of equal scores) leaves the policy part out, at any ratio: exp(lp - lp_old) = exp(190)."""
    gen = torch.Generator(device=DEV).manual_seed(V + 1)
    B, T = 2, 3
    z, _ = ref.row_logits(B, T, V, BF, gen, DEV)
    ids, lengths = labels(B, T, V, gen), torch.full((B,), T, dtype=torch.int32, device=DEV)
    lp_old, lp_ref, adv = policy_inputs(z, ids, lengths, gen, False)
    adv[0], lp_old[0, 1] = 0.0, -200.0
    adv[1, 0], lp_old[1, 0] = 1.0, -200.0                # clipped: the loss is -1.3, no gradient
    for kl_coef in (0.1, 0.0):
        ws = lib.workspace(B, T, DEV)
        got = lib.policy_kl_loss_fwd_bwd(z, ids, lengths, lp_old, lp_ref, adv, 0.2, 0.3, kl_coef, 0, 100.0, ws)
        pg, kl, d, lp, size = ref.policy_kl(z.double(), ids, lengths, lp_old, lp_ref, adv, 0.2, 0.3, kl_coef, 0, 100.0)
        part = torch.softmax(z.double(), dim=2) + torch.nn.functional.one_hot(ids, V)
        check_gradient(got.dlogits, d, size[..., None] * part)
        assert abs(got.loss[0].item() - pg.item()) <= 8 * LP + 2 ** -23 * abs(pg.item())
        assert abs(got.loss[1].item() - kl.item()) <= 8 * LP + 2 ** -23 * abs(kl.item())
