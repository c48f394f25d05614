"""The float64 definitions that the objective kernels are checked against: their gradients against central differences of
their own losses (CPU)."""
import pytest
import torch

import objectives64 as ref


def _batch(seed, B=4, T=5, V=11):
    g = torch.Generator().manual_seed(seed)
    z = 2.0 * torch.randn((B, T, V), generator=g, dtype=torch.float64)
    ids = torch.randint(0, V, (B, T), generator=g)
    lengths = torch.tensor([5, 0, 1, 3], dtype=torch.int32)
    _, lp, _ = ref.label_logprobs(z, ids, lengths)
    r = lambda *n: torch.randn(n, generator=g, dtype=torch.float64)  # noqa: E731
    return g, z, ids, lengths, lp, r


def _differences(loss, z, lengths, h=1e-5):
    """d loss / d z by central differences, entry by entry.  Truncation h^2 |f'''| / 6 <= 1e-10 and rounding
    2^-52 |f| / h <= 1e-10 for the losses of order one used here: 1e-8 is allowed."""
    d = torch.zeros_like(z)
    for b in range(z.shape[0]):
        for t in range(int(lengths[b])):
            for v in range(z.shape[2]):
                up, down = z.clone(), z.clone()
                up[b, t, v] += h
                down[b, t, v] -= h
                d[b, t, v] = (loss(up) - loss(down)) / (2 * h)
    return d


@pytest.mark.parametrize("reduction", [0, 1])
def test_policy_kl_gradient(reduction):
    g, z, ids, lengths, lp, r = _batch(1)
    rho = torch.tensor([0.5, 0.9, 1.1, 1.5])[torch.randint(0, 4, lp.shape, generator=g)].double()
    lp_old, lp_ref, adv = lp - rho.log(), lp + 0.5 * r(4, 5), r(4, 5)
    f = lambda x: ref.policy_kl(x, ids, lengths, lp_old, lp_ref, adv, 0.2, 0.3, 0.1, reduction, 1.0)  # noqa: E731
    want = _differences(lambda x: f(x)[0] + 0.1 * f(x)[1], z, lengths)
    assert (f(z)[2] - want).abs().max() < 1e-8


@pytest.mark.parametrize("kind,smoothing,length_mean", [(0, 0.0, False), (0, 0.1, True), (1, 0.0, False), (2, 0.0, True)])
def test_preference_gradient(kind, smoothing, length_mean):
    g, z, ids, lengths, lp, r = _batch(2)
    lp_ref = lp + 0.5 * r(4, 5)
    f = lambda x: ref.preference(x, ids, lengths, lp_ref, kind, 0.7, 0.2, smoothing, length_mean, 1.0)  # noqa: E731
    want = _differences(lambda x: f(x)[0], z, lengths)
    assert (f(z)[2] - want).abs().max() < 1e-8


@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("temperature", [1.0, 2.5])
def test_distill_gradient(mode, temperature):
    g, z, _, lengths, _, r = _batch(3)
    teacher = torch.log_softmax((z + r(4, 5, 11)) / temperature, dim=2)
    lt, ids = teacher.topk(4, dim=2)
    ids[0, 0, 2] = -1                                    # unused
    ids[0, 1, 3] = ids[0, 1, 1]                          # named twice
    f = lambda x: ref.distill(x, ids, lt, lengths, mode, temperature, 1.0)  # noqa: E731
    want = _differences(lambda x: f(x)[0], z, lengths)
    assert (f(z)[2] - want).abs().max() < 1e-8
