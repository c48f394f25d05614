"""The tail class of the distillation loss where the student leaves little or nothing outside the teacher's entries: the float64
definition's gradient against central differences of its own loss (CPU)."""
import pytest
import torch

import objectives64 as ref


@pytest.mark.parametrize("lift", [0.0, 30.0, 90.0, float("inf")])
@pytest.mark.parametrize("mode", [0, 1, 2])
def test_gradient_with_little_or_nothing_outside(mode, lift):
    """`lift` nats between the entries and the others; inf: the others are deleted, and the tail term is left out."""
    gen = torch.Generator().manual_seed(4)
    V, K = 20, 4
    z = 2.0 * torch.randn((1, 1, V), generator=gen, dtype=torch.float64)
    ids = torch.tensor([[[3, 11, 0, 19]]], dtype=torch.int32)
    lt = (torch.log_softmax(torch.randn((1, 1, K), generator=gen, dtype=torch.float64), dim=2) + torch.log(torch.tensor(0.7))).float()
    named = torch.zeros(V, dtype=torch.bool)
    named[ids[0, 0].long()] = True
    z[..., ~named] -= lift
    lengths = torch.ones(1, dtype=torch.int32)
    f = lambda x: ref.distill(x, ids, lt, lengths, mode, 1.3, 1.0)  # noqa: E731
    _, _, d, _ = f(z)
    h = 1e-5
    for v in range(V):
        up, down = z.clone(), z.clone()
        up[..., v] += h
        down[..., v] -= h
        want = (f(up)[0] - f(down)[0]) / (2 * h)
        # truncation h^2 |f'''| / 6 <= 1e-10; rounding 2^-52 |f| / h with |f| <= 200: 5e-9 where the others are far below; the
        # definition's factor temperature / N is a quotient by a whole-number tensor, which torch rounds to fp32: 2^-24 of the value
        assert abs(d[0, 0, v] - want) <= 1e-8 + 2.0 ** -24 * abs(want), (v, d[0, 0, v].item(), want.item())
    # a softmax does not change when all logits do by the same amount
    assert abs(d.sum()) <= 1e-12
