"""Distillation with the tail class where the student leaves little or nothing outside the teacher's entries, on every kernel that
takes such rows, against the float64 definition.  Tolerances as in test_objectives_gpu.py."""
import pytest
import torch

import objectives64 as ref
from paper_2410_15651_b200 import binding as lib
from test_objectives_gpu import BF, DEV, HF, check_distill

pytestmark = pytest.mark.gpu

# rows below 16 KB, off 16-byte boundaries, in one block (registers alone, and with tensor memory), beyond one block and off a
# boundary, in the chunk ring (one block, two), in clusters of two and four with whole-slice buffers, beyond every cluster
VOCABULARIES = [1000, 1001, 8200, 20000, 50257, 57353, 57344, 80000, 128256, 212992, 300000]


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
