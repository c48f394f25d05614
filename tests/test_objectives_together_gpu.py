"""The objectives as they are used: one after the other on one workspace, on other streams, in captured graphs, on views whose
offsets pass 32 bits; and their gradients against differences of the float64 losses."""
import pytest
import torch

import objectives64 as ref
from paper_2410_15651_b200 import binding as lib
from test_objectives_gpu import BF, DEV, HF, LP, labels, mixed_lengths, policy_inputs, teacher_entries, tiny

pytestmark = pytest.mark.gpu


class Batch:
    """A student, its teacher and what the objectives need beside them."""

    def __init__(self, B, T, V, seed, dtype=BF, **layout):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.z, _ = ref.row_logits(B, T, V, dtype, gen, DEV, **layout)
        self.teacher, _ = ref.row_logits(B, T, V, dtype, gen, DEV)
        self.ids, self.lengths = labels(B, T, V, gen), mixed_lengths(B, T)
        self.lp_old, self.lp_ref, self.adv = policy_inputs(self.z, self.ids, self.lengths, gen, True)


def whole_step(b, ws, K=32):
    """Every objective of one batch; returns everything that was written."""
    t = lib.topk_logprobs(b.teacher, b.lengths, K, 2.0, ws)
    d = lib.distill_loss_fwd_bwd(b.z, t.ids, t.logprobs, b.lengths, lib.DISTILL_TAIL, 2.0, 10.0, ws)
    lp = lib.gather_logprobs(b.z, b.ids, b.lengths, ws)
    p = lib.policy_kl_loss_fwd_bwd(b.z, b.ids, b.lengths, b.lp_old, b.lp_ref, b.adv, 0.2, 0.3, 0.1, 1, 10.0, ws)
    r = lib.preference_loss_fwd_bwd(b.z, b.ids, b.lengths, b.lp_ref, lib.PREF_SIGMOID, 0.2, 0.0, 0.1, True, 10.0, ws)
    s = lib.ppo_stats(p.lp_new, b.lp_old, b.lp_ref, b.lengths, 0.2, ws)
    return [t.ids, t.logprobs, d.loss, d.dlogits, d.row_loss, lp, p.loss, p.dlogits, p.lp_new, r.loss, r.dlogits, r.rewards,
            r.lp_new, s]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("V", [1000, 20000, 50257, 128256])
def test_one_step_of_everything(V):
    """Distillation from the teacher's own entries agrees with the definition, and the log-probs of the objectives agree."""
    b = Batch(4, 9, V, seed=V)
    ws = lib.workspace(4, 9, DEV)
    out = whole_step(b, ws)
    assert lib.poll_status(ws) == 0
    ids, lt = ref.topk(b.teacher.double(), b.lengths, 32, 2.0)
    assert torch.equal(out[0].long(), ids)
    loss, rows, _, _ = ref.distill(b.z.double(), out[0], out[1], b.lengths, 2, 2.0, 10.0)
    each = 4.0 * (2 * LP + 2 ** -22 * 64)
    assert ((out[4].double() - rows).abs() <= each + 2 ** -23 * rows.abs()).all()
    assert (out[5] - out[8]).abs().max() <= 2 * LP and (out[8] - out[12]).abs().max() <= 2 * LP


def test_workspace_of_another_shape_and_after_other_calls():
    """A workspace for the largest batch serves smaller ones, whatever the calls before left in it."""
    ws = lib.workspace(16, 40, DEV)
    shapes = [(16, 40, 1000), (2, 3, 128256), (6, 11, 20000), (16, 40, 8200), (2, 1, 50257), (4, 4, 20000)]
    fresh = [whole_step(Batch(B, T, V, seed=B + T), lib.workspace(B, T, DEV)) for B, T, V in shapes]
    for _ in range(2):
        for (B, T, V), want in zip(shapes, fresh):
            assert same(whole_step(Batch(B, T, V, seed=B + T), ws), want), (B, T, V)
    assert lib.poll_status(ws) == 0


def test_other_streams():
    """Calls on a stream of their own, two at once with a workspace each, and tensors made on another stream."""
    a, b = Batch(6, 33, 20000, 1), Batch(6, 33, 50257, 2)
    wa, wb = lib.workspace(6, 33, DEV), lib.workspace(6, 33, DEV)
    want = whole_step(a, wa), whole_step(b, wb)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(sa):
            ga = whole_step(a, wa)
        with torch.cuda.stream(sb):
            gb = whole_step(b, wb)
        torch.cuda.synchronize()
        assert same(ga, want[0]) and same(gb, want[1])
    assert lib.poll_status(wa) == 0 and lib.poll_status(wb) == 0


@pytest.mark.parametrize("V", [1000, 20000, 128256])
def test_captured_and_replayed(V):
    """Two graphs that share a workspace, replayed in turn with new inputs in place, and an eager call between them."""
    a, b, other = Batch(4, 17, V, 3), Batch(4, 17, V, 4), Batch(4, 17, V, 5)
    ws = lib.workspace(4, 17, DEV)
    side = torch.cuda.Stream()
    graphs, outs = [], []
    with torch.cuda.stream(side):
        for x in (a, b):
            whole_step(x, ws)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                outs.append(whole_step(x, ws))
            graphs.append(g)
        for x in (a, b):                                  # the same addresses, other values
            for name in ("z", "teacher", "ids", "lengths", "lp_old", "lp_ref", "adv"):
                getattr(x, name).copy_(getattr(other, name))
        want = [t.clone() for t in whole_step(other, ws)]
        for _ in range(3):
            for g in graphs:
                g.replay()
            whole_step(other, ws)
        torch.cuda.synchronize()
    assert same(outs[0], want) and same(outs[1], want)
    assert lib.poll_status(ws) == 0


@pytest.mark.parametrize("V", [1000, 20000, 20001])
def test_offsets_beyond_32_bits(V):
    """Sequences more than 2^32 elements apart, in place."""
    B, T = 2, 3
    far = (1 << 32) + 8 * 1001
    store = torch.zeros(far + T * V + 8, dtype=BF, device=DEV)
    z = store.as_strided((B, T, V), (far, V, 1))
    b = Batch(B, T, V, 6)
    z.copy_(b.z)
    ws = lib.workspace(B, T, DEV)
    want = whole_step(b, ws)
    b.teacher = z.clone()
    t = lib.topk_logprobs(z, b.lengths, 20, 1.0, ws)
    t2 = lib.topk_logprobs(b.teacher, b.lengths, 20, 1.0, ws)
    assert torch.equal(t.ids, t2.ids) and torch.equal(t.logprobs, t2.logprobs)
    tw = lib.topk_logprobs(Batch(B, T, V, 6).teacher, b.lengths, 32, 2.0, ws)

    def in_place(make, call):
        z.copy_(b.z)
        return call(make(z, in_place=True))
    d = in_place(lib.DistillOutputs, lambda o: lib.distill_loss_fwd_bwd(z, tw.ids, tw.logprobs, b.lengths, lib.DISTILL_TAIL, 2.0, 10.0, ws, o))
    assert torch.equal(d.loss, want[2]) and torch.equal(z, want[3])
    p = in_place(lib.PolicyKlOutputs, lambda o: lib.policy_kl_loss_fwd_bwd(z, b.ids, b.lengths, b.lp_old, b.lp_ref, b.adv, 0.2, 0.3, 0.1, 1, 10.0, ws, o))
    assert torch.equal(p.loss, want[6]) and torch.equal(z, want[7])
    r = in_place(lib.PreferenceOutputs, lambda o: lib.preference_loss_fwd_bwd(z, b.ids, b.lengths, b.lp_ref, lib.PREF_SIGMOID, 0.2, 0.0, 0.1, True, 10.0, ws, o))
    assert torch.equal(r.loss, want[9]) and torch.equal(z, want[10])
    assert store[T * V:far].count_nonzero() == 0           # nothing between the sequences was written
    assert lib.poll_status(ws) == 0


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("V", [40, 9000])
def test_gradients_against_differences(V, dtype):
    """The written gradient along random directions against central differences of the float64 losses."""
    b = Batch(4, 3, V, 7, dtype)
    ws = lib.workspace(4, 3, DEV)
    t = lib.topk_logprobs(b.teacher, b.lengths, 8, 1.5, ws)
    z64 = b.z.double()
    cases = [
        (lib.distill_loss_fwd_bwd(b.z, t.ids, t.logprobs, b.lengths, 2, 1.5, 1.0, ws).dlogits,
         lambda z: ref.distill(z, t.ids, t.logprobs, b.lengths, 2, 1.5, 1.0)[0],
         ref.distill(z64, t.ids, t.logprobs, b.lengths, 2, 1.5, 1.0)[3]),
        (lib.policy_kl_loss_fwd_bwd(b.z, b.ids, b.lengths, b.lp_old, b.lp_ref, b.adv, 0.2, 0.3, 0.1, 0, 1.0, ws).dlogits,
         lambda z: sum(w * x for w, x in zip((1.0, 0.1), ref.policy_kl(z, b.ids, b.lengths, b.lp_old, b.lp_ref, b.adv, 0.2, 0.3, 0.1, 0, 1.0)[:2])),
         None),
        (lib.preference_loss_fwd_bwd(b.z, b.ids, b.lengths, b.lp_ref, 2, 0.5, 0.1, 0.0, False, 1.0, ws).dlogits,
         lambda z: ref.preference(z, b.ids, b.lengths, b.lp_ref, 2, 0.5, 0.1, 0.0, False, 1.0)[0], None)]
    gen = torch.Generator(device=DEV).manual_seed(8)
    h = 1e-4
    for grad, loss, parts in cases:
        for _ in range(3):
            u = torch.randn(z64.shape, generator=gen, device=DEV, dtype=torch.float64)
            want = ((loss(z64 + h * u) - loss(z64 - h * u)) / (2 * h)).item()
            got = (grad.double() * u).sum().item()
            # entry by entry: half a step of the gradient's type and 1e-3 of its size for what is formed of fp32 parts
            # (log-probs off by 2e-5 against slopes of at most 40); the difference itself is good to h^2 times third
            # derivatives of order |u|^3 per row, below 1e-5
            size = grad.double().abs() if parts is None else parts.maximum(grad.double().abs())
            tol = ((torch.finfo(dtype).eps / 2 + 1e-3) * size + tiny(dtype)).mul(u.abs()).sum().item() + 1e-4
            assert abs(got - want) <= tol, (got, want, tol)


def test_many_short_pairs():
    """More pairs than blocks, tokens of a small vocabulary, empty responses among them."""
    B, T, V = 4096, 3, 16
    b = Batch(B, T, V, 9)
    ws = lib.workspace(B, T, DEV)
    got = lib.preference_loss_fwd_bwd(b.z, b.ids, b.lengths, b.lp_ref, 0, 0.3, 0.0, 0.0, False, 1000.0, ws)
    loss, rewards, d, _, _ = ref.preference(b.z.double(), b.ids, b.lengths, b.lp_ref, 0, 0.3, 0.0, 0.0, False, 1000.0)
    assert abs(got.loss.item() - loss.item()) <= 2 * T * 0.3 * LP + 2 ** -23 * loss.item()
    assert ((got.rewards.double() - rewards).abs() <= T * 0.3 * LP + 2 ** -23 * rewards.abs()).all()
    # the factor is off by at most 1/4 of h's error, 2 * 3 * 0.3 LP, times beta * scale * 2 / B; the entries by half a step:
    # bf16 has 8 significant bits, a step of 2^-7 at 1, so half a step is 2^-8 of a value just above a power of two
    half_step = torch.finfo(BF).eps / 2
    assert ((got.dlogits.double() - d).abs() <= (half_step + LP) * d.abs() + 0.25 * 1.8 * LP * 0.3 * 1000.0 * 2 / B + tiny(BF)).all()
