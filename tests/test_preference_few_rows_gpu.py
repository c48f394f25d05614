"""Log-probs of the preference loss on batches of at most eight rows per SM, which a block per row forms, with padded rows between a
block's valid ones."""
import pytest
import torch

import objectives64 as ref
from paper_2410_15651_b200 import binding as lib
from test_objectives_gpu import BF, DEV, HF, LP, labels

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("per_sm", [1, 6, 8])
@pytest.mark.parametrize("V", [1001, 20000])
def test_padded_rows_between_valid_ones(V, per_sm, dtype):
    gen = torch.Generator(device=DEV).manual_seed(V + per_sm)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    B, T = {1: (sms // 2 * 2, 1), 6: (2 * sms, 3), 8: (2 * sms, 4)}[per_sm]
    z, _ = ref.row_logits(B, T, V, dtype, gen, DEV)
    ids, lengths = labels(B, T, V, gen), torch.randint(0, T + 1, (B,), generator=gen, device=DEV).int()
    ws = lib.workspace(B, T, DEV)
    got = lib.preference_loss_fwd_bwd(z, ids, lengths, None, lib.PREF_SIGMOID, 0.1, 0.0, 0.0, False, 1.0, ws)
    _, lp, _ = ref.label_logprobs(z.double(), ids, lengths)
    assert (got.lp_new.double() - lp).abs().max() <= LP
    for _ in range(20):
        again = lib.preference_loss_fwd_bwd(z, ids, lengths, None, lib.PREF_SIGMOID, 0.1, 0.0, 0.0, False, 1.0, ws)
        assert torch.equal(again.lp_new, got.lp_new) and torch.equal(again.dlogits, got.dlogits)
    assert lib.poll_status(ws) == 0
