"""Distillation with the tail class where the student leaves little or nothing outside the teacher's entries, on every kernel that
takes such rows, against the float64 definition.  Tolerances as in test_objectives_gpu.py."""
import pytest
import torch

import objectives64 as ref
from paper_2410_15651_b200 import binding as lib
from test_objectives_gpu import BF, DEV, HF, LP, check_distill, check_gradient

pytestmark = pytest.mark.gpu

# rows below 16 KB, off 16-byte boundaries, in one block (registers alone, and with tensor memory), beyond one block and off a
# boundary, in the chunk ring (one block, two, four), in clusters of two to four with whole-slice buffers, beyond every cluster
VOCABULARIES = [1000, 1001, 8200, 20000, 50257, 57353, 57344, 80000, 128256, 150000, 212992, 230000, 300000]


def entries_of(V, K, shape, gen, first):
    """K different entries per row (with the row's first 16 among them if `first`), weights that sum to about 0.7."""
    ids = torch.stack([torch.randperm(V - 16, generator=gen, device=DEV)[:K] + 16 for _ in range(shape[0] * shape[1])])
    if first:
        ids[:, :16] = torch.arange(16, device=DEV)
    lt = torch.log_softmax(torch.randn((shape[0] * shape[1], K), generator=gen, device=DEV), dim=1) - 0.36
    return ids.view(*shape, K).int(), lt.view(*shape, K)


@pytest.mark.parametrize("K", [20, 100])
@pytest.mark.parametrize("V", VOCABULARIES)
def test_nothing_outside(V, K):
    """The student has deleted all but the teacher's entries: the tail term is left out of the loss and of its gradient."""
    gen = torch.Generator(device=DEV).manual_seed(V + K)
    B, T = 2, 2
    for dtype in (BF, HF):
        z, _ = ref.row_logits(B, T, V, dtype, gen, DEV)
        ids, lt = entries_of(V, K, (B, T), gen, first=True)
        keep = torch.zeros(z.shape, dtype=torch.bool, device=DEV).scatter_(2, ids.long(), True)
        z[~keep] = float("-inf")
        lengths = torch.full((B,), T, dtype=torch.int32, device=DEV)
        got, ws = check_distill(z, ids, lt, lengths, lib.DISTILL_TAIL, 1.0, 10.0)
        assert lib.poll_status(ws) == 0


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("K", [20, 100])
@pytest.mark.parametrize("V", VOCABULARIES)
def test_little_outside(V, K, dtype):
    """Entries 35 to 210 nats above all others (a mass outside of 2^-33 to 2^-290), and rows whose first vectors lie 40 nats below
    the others that are outside, or are the teacher's, or with few others left.  Every entry's gradient is p_0 q_v / q_0 at most
    beside W q_v, and no part of it is lost."""
    gen = torch.Generator(device=DEV).manual_seed(V + K + 1)
    lifts = [35.0, 60.0, 70.0, 78.0, 84.0, 87.0, 90.0, 104.0, 128.0, 210.0]
    B, T = len(lifts), 4
    z, _ = ref.row_logits(B, T, V, dtype, gen, DEV, sigma=0.5)
    ids, lt = entries_of(V, K, (B, T), gen, first=False)
    ids[:, 2, :16] = torch.arange(16, device=DEV).int()
    z[:, 1, :16] -= 40.0
    few = torch.randint(16, V, (B, 5), generator=gen, device=DEV)
    left = torch.zeros((B, V), dtype=torch.bool, device=DEV).scatter_(1, few, True).scatter_(1, ids[:, 3].long(), True)
    z[:, 3] = torch.where(left, z[:, 3], float("-inf"))
    for b, lift in enumerate(lifts):
        z[b].scatter_add_(1, ids[b].long(), torch.full((T, K), lift, dtype=dtype, device=DEV))
    lengths = torch.full((B,), T, dtype=torch.int32, device=DEV)
    scale = 100.0 if dtype == HF else 1e6                # (fp16 holds gradients up to 65504)
    got = lib.distill_loss_fwd_bwd(z, ids, lt, lengths, lib.DISTILL_TAIL, 1.0, scale, lib.workspace(B, T, DEV))
    for b in range(B):
        part = slice(b, b + 1)
        _, rows, d, parts = ref.distill(z[part].double(), ids[part], lt[part], lengths[part], 2, 1.0, scale / B)
        # the logs of masses down to 2^-310 are off by LP and a rounding of theirs (2^-22 of 215 nats)
        off = (got.row_loss[part].double() - rows).abs()
        assert (off <= 2 * LP + 2 ** -22 * 215 + 2 ** -23 * rows.abs()).all(), (lifts[b], off)
        check_gradient(got.dlogits[part], d, parts)
    assert abs(got.loss.item() - got.row_loss.double().mean().item()) <= 2 ** -23 * abs(got.loss.item())


@pytest.mark.parametrize("V", VOCABULARIES)
def test_outside_far_above_the_entries(V):
    """The other end: entries 35 to 210 nats below the rest."""
    gen = torch.Generator(device=DEV).manual_seed(V + 2)
    lifts = [-35.0, -90.0, -210.0]
    B, T, K = 3, 2, 20
    z, _ = ref.row_logits(B, T, V, BF, gen, DEV, sigma=0.5)
    ids, lt = entries_of(V, K, (B, T), gen, first=True)
    for b, lift in enumerate(lifts):
        z[b].scatter_add_(1, ids[b].long(), torch.full((T, K), lift, dtype=BF, device=DEV))
    lengths = torch.full((B,), T, dtype=torch.int32, device=DEV)
    for mode in (0, 1, 2):
        check_distill(z, ids, lt, lengths, mode, 1.0, 1000.0, reach=512)
