"""The operators on shaped logits and the router's loss as they are used: a decoding loop and the training step after it, one
workspace for batches of every shape, other streams, captured graphs; and what the binding refuses.  The tolerances are those
that test_shaping_gpu.py and test_router_gpu.py derive."""
import pytest
import torch

import shaping64 as ref
from objectives64 import row_logits
from paper_2410_15651_b200 import binding as lib
from test_router_gpu import check as check_router
from test_shaping_gpu import (ALL, BF, DEV, ENT, HF, LP, X, check_logprobs, check_shape, check_shape_bwd, labels, mixed_lengths, row_error,
                              same_but, tiny)

pytestmark = pytest.mark.gpu


class Batch:
    """Logits of an actor and a reference, a rollout's settings and its answers, and a router's logits."""

    def __init__(self, B, T, V, seed, dtype=BF, parts=ALL + ("bias", "mask_rows"), L=2, E=16, **layout):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.z, _ = row_logits(B, T, V, dtype, gen, DEV, **layout)
        self.z_ref, _ = row_logits(B, T, V, dtype, gen, DEV)
        self.kw = ref.Settings(B, T, V, gen, DEV, parts, P=9, S0=5, repeat=min(8, V)).kw
        self.shaping = lib.Shaping(B, V, **self.kw)
        self.lengths, self.ids = mixed_lengths(B, T), labels(B, T, V, self.kw, gen)
        self.g, self.h = torch.randn((B, T), generator=gen, device=DEV), 0.1 * torch.randn((B, T), generator=gen, device=DEV)
        self.d = torch.randn((B, T, V), generator=gen, device=DEV).to(dtype)
        self.router = torch.randn((L, B, T, E), generator=gen, device=DEV).to(dtype)

    def fields(self):
        return [self.z, self.z_ref, self.lengths, self.ids, self.g, self.h, self.d, self.router] + [self.kw[k] for k in sorted(self.kw)]


def workspaces(B, T, L=2, E=16):
    return lib.workspace(B, T, DEV), lib.router_workspace(L, B, T, E, DEV)


def whole_step(b, ws, rws):
    """Every operator once; returns everything that was written."""
    x = lib.shape_logits(b.z, b.lengths, b.shaping, ws)
    x32 = lib.shape_logits(b.z, b.lengths, b.shaping, ws, dtype=torch.float32)
    dz = lib.shape_logits_bwd(b.d, b.z, b.lengths, b.shaping, ws)
    f = lib.shaped_logprobs(b.z, b.ids, b.lengths, b.shaping, ws, want_entropy=True)
    r = lib.shaped_logprobs(b.z_ref, b.ids, b.lengths, b.shaping, ws)
    dl = lib.shaped_logprobs_bwd(b.z, b.ids, b.lengths, b.shaping, f, b.g, b.h, ws)
    o = lib.router_loss_fwd_bwd(b.router, b.lengths, 4, lib.ROUTER_SOFTMAX, lib.ROUTER_BATCH, 0.01, 0.001, 10.0, rws)
    s = lib.router_loss_fwd_bwd(b.router, b.lengths, 4, lib.ROUTER_SIGMOID, lib.ROUTER_SEQUENCE, 0.01, 0.0, 10.0, rws, expert_ids=o.ids)
    return [x, x32, dz, f.logprobs, f.lse, f.entropy, r.logprobs, dl, o.loss, o.counts, o.ids, o.dlogits, s.loss, s.counts, s.dlogits]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("V,dtype", [(1000, BF), (4003, HF), (32000, BF)])
def test_a_decoding_loop_and_the_same_rows_at_once(V, dtype):
    """Greedy decoding with the history kept on the device: the shaped rows of the loop are those of one call over the answers."""
    B, T = 5, 40
    gen = torch.Generator(device=DEV).manual_seed(V)
    z, _ = row_logits(B, T, V, dtype, gen, DEV)
    z[:, :, 7] = z.amax(dim=2) + 1                        # a token that would be chosen again and again
    kw = ref.Settings(B, T, V, gen, DEV, ("prompt", "repetition", "frequency", "presence", "temperature", "bias", "mask"), P=20).kw
    kw["mask"][:] |= 1 << 7
    kw["frequency"] = kw["frequency"].abs() + 0.5
    tokens = torch.full((B, T), -1, dtype=torch.int64, device=DEV)
    start = torch.zeros(B, dtype=torch.int32, device=DEV)
    ws, wide = lib.workspace(B, 1, DEV), lib.workspace(B, T, DEV)
    one = torch.ones(B, dtype=torch.int32, device=DEV)
    shaping = lib.Shaping(B, V, tokens=tokens, start=start, **kw)
    steps = torch.empty((B, T, V), dtype=torch.float32, device=DEV)
    for t in range(T):
        lib.shape_logits(z[:, t:t + 1], one, shaping, ws, out=steps[:, t:t + 1])
        tokens[:, t] = steps[:, t].argmax(dim=1)
        start += 1
    assert lib.poll_status(ws) == 0
    full = torch.full((B,), T, dtype=torch.int32, device=DEV)
    x, _, parts = ref.shaped(z, full, dict(kw, tokens=tokens))
    same_but(steps, x, X * parts, "steps")
    check_shape(z, full, dict(kw, tokens=tokens), wide, dtype=torch.float32)
    assert any(len(set(row.tolist())) > 1 for row in tokens)
    lp = lib.shaped_logprobs(z, tokens, full, lib.Shaping(B, V, tokens=tokens, **kw), wide).logprobs
    want = torch.log_softmax(x, dim=2).gather(2, tokens[..., None])[..., 0]
    assert ((lp.double() - want).abs() <= LP + 2 * row_error(parts)).all()


@pytest.mark.parametrize("V", [1000, 20000])
def test_a_policy_step_under_the_rollouts_settings(V):
    """Log-probs of actor and reference, rewards, advantages, the gradient of the policy's log-probs, the router's beside it."""
    B, T = 6, 12
    b, (ws, rws) = Batch(B, T, V, seed=V, parts=ALL), workspaces(6, 12)
    f = check_logprobs(b.z, b.ids, b.lengths, b.kw, ws)
    r = check_logprobs(b.z_ref, b.ids, b.lengths, b.kw, ws, entropy=False)
    rewards = lib.kl_reward(f.logprobs, r.logprobs, b.g[:, 0].contiguous(), b.lengths, 0.1, 5.0)
    adv, _ = lib.gae(rewards, b.h, b.lengths, 0.99, 0.95)
    adv = lib.whiten_advantages(adv, b.lengths, 1e-8, ws)
    g, h = -adv / B, torch.full_like(adv, -0.01)
    d = lib.shaped_logprobs_bwd(b.z, b.ids, b.lengths, b.shaping, f, g, h, ws)
    x, scale, parts = ref.shaped(b.z, b.lengths, b.kw)
    want, size = ref.logprobs_grad(x, scale, b.ids, b.lengths, g, h)
    rel = ENT + 40 * row_error(parts)
    same_but(d, want, torch.finfo(BF).eps / 2 * want.abs() + rel[..., None] * size + tiny(BF), "gradient")
    check_router(b.router, b.lengths, 4, lib.ROUTER_SOFTMAX, lib.ROUTER_BATCH, 0.01, 0.001, 10.0, rws)
    assert lib.poll_status(ws) == 0 and lib.poll_status(rws) == 0


@pytest.mark.parametrize("V", [1000, 20000])
def test_the_objective_on_shaped_logits(V):
    """Shaped logits in place of the logits, the library's loss on them in place, its gradient back through the shaping in place."""
    B, T = 6, 12
    b, (ws, _) = Batch(B, T, V, seed=V + 1, parts=ALL), workspaces(6, 12)
    x = lib.shape_logits(b.z, b.lengths, b.shaping, ws)
    lp = lib.gather_logprobs(x, b.ids, b.lengths, ws)
    # (the shaped logits are rounded to bf16 here, so the log-prob moves by up to a half step of the two largest)
    f = lib.shaped_logprobs(b.z, b.ids, b.lengths, b.shaping, ws)
    step = torch.finfo(BF).eps / 2 * x.double().abs().amax(dim=2)
    assert ((lp - f.logprobs).abs().double() <= 2 * step + 2 * LP).all()
    out = lib.PPOOutputs(x, in_place=True)
    lib.ppo_loss_fwd_bwd(x, b.ids, b.lengths, f.logprobs, b.g, b.h, b.h, b.g, 0.2, 0.2, 10.0, ws, out)
    d64 = x.double().clone()
    check_shape_bwd(b.z, b.lengths, b.kw, ws, None, out=x, d=x, d64=d64)
    assert lib.poll_status(ws) == 0


def test_workspace_of_another_shape_and_after_other_calls():
    ws, rws = workspaces(16, 40)
    shapes = [(16, 40, 1000), (2, 3, 128256), (6, 11, 20000), (16, 40, 8200), (2, 1, 50257), (16, 1, 4001), (4, 4, 20000)]
    fresh = [whole_step(Batch(B, T, V, seed=B + T), *workspaces(B, T)) for B, T, V in shapes]
    for _ in range(2):
        for (B, T, V), want in zip(shapes, fresh):
            assert same(whole_step(Batch(B, T, V, seed=B + T), ws, rws), want), (B, T, V)
    assert lib.poll_status(ws) == 0 and lib.poll_status(rws) == 0


def test_other_streams():
    """Calls on a stream of their own, two at once with workspaces of their own."""
    a, b = Batch(6, 33, 20000, 1), Batch(6, 33, 50257, 2)
    wa, wb = workspaces(6, 33), workspaces(6, 33)
    want = whole_step(a, *wa), whole_step(b, *wb)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(sa):
            ga = whole_step(a, *wa)
        with torch.cuda.stream(sb):
            gb = whole_step(b, *wb)
        torch.cuda.synchronize()
        assert same(ga, want[0]) and same(gb, want[1])
    assert all(lib.poll_status(w) == 0 for w in wa + wb)


@pytest.mark.parametrize("B,T,V", [(4, 1, 1000), (4, 17, 20000), (12, 40, 4003), (4, 17, 128256)])
def test_captured_and_replayed(B, T, V):
    """Two graphs that share their workspaces, replayed in turn with new inputs in place, and eager calls between them."""
    a, b, other = Batch(B, T, V, 3), Batch(B, T, V, 4), Batch(B, T, V, 5)
    ws, rws = workspaces(B, T)
    side = torch.cuda.Stream()
    graphs, outs = [], []
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for x in (a, b):
            whole_step(x, ws, rws)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                outs.append(whole_step(x, ws, rws))
            graphs.append(g)
        for x in (a, b):                                  # the same addresses, other values
            for mine, its in zip(x.fields(), other.fields()):
                mine.copy_(its)
        want = [t.clone() for t in whole_step(other, ws, rws)]
        for _ in range(3):
            for g in graphs:
                g.replay()
            whole_step(other, ws, rws)
        torch.cuda.synchronize()
    assert same(outs[0], want) and same(outs[1], want)
    assert lib.poll_status(ws) == 0 and lib.poll_status(rws) == 0


def test_what_the_binding_refuses():
    B, T, V = 2, 3, 40
    b, (ws, rws) = Batch(B, T, V, 6), workspaces(2, 3)
    i64, i32, f32 = (dict(dtype=t, device=DEV) for t in (torch.int64, torch.int32, torch.float32))
    wrong = [dict(tokens=torch.zeros((B, 4), **i32)), dict(tokens=torch.zeros((B + 1, 4), **i64)), dict(tokens=torch.zeros((4, B), **i64).t()),
             dict(start=torch.zeros(B, **i64)), dict(start=torch.zeros(B + 1, **i32)), dict(prompt=torch.zeros(B, **i64)),
             dict(prompt_lengths=torch.zeros((B, 1), **i32)), dict(repetition=torch.ones(2 * B, **f32)[::2]),
             dict(temperature=torch.ones(B, dtype=torch.float64, device=DEV)), dict(frequency=torch.ones(1, **f32)),
             dict(bias=torch.zeros(V + 1, **f32)), dict(bias=torch.zeros((V, B), **f32).t()), dict(bias=torch.zeros(V, dtype=BF, device=DEV)),
             dict(mask=torch.zeros((B, 1), **i32)), dict(mask=torch.zeros((B + 1, 2), **i32)), dict(mask=torch.zeros(2, **i32)),
             dict(mask=torch.zeros((B, 2), **i64)), dict(mask=torch.zeros((B, T, 4), **i32)[..., ::2])]
    for kw in wrong:
        with pytest.raises((ValueError, TypeError)):
            lib.Shaping(B, V, **kw)
    sh, f = lib.Shaping(B, V), lib.ShapedLogprobs(b.z, True)
    rows = lib.Shaping(B, V, mask=torch.zeros((B, T + 1, 2), **i32))
    calls = [lambda: lib.shape_logits(b.z, b.lengths, lib.Shaping(B, V + 1), ws), lambda: lib.shape_logits(b.z, b.lengths, rows, ws),
             lambda: lib.shape_logits(b.z, b.lengths, lib.Shaping(B + 1, V), ws), lambda: lib.shape_logits(b.z, b.lengths.long(), sh, ws),
             lambda: lib.shape_logits(b.z.float(), b.lengths, sh, ws), lambda: lib.shape_logits(b.z, b.lengths, sh, ws, dtype=HF),
             lambda: lib.shape_logits(b.z, b.lengths, sh, ws, out=torch.empty((B, T, V + 1), **f32)),
             lambda: lib.shape_logits(b.z, b.lengths, sh, ws, out=torch.empty((B, T, 2 * V), **f32)[..., ::2]),
             lambda: lib.shape_logits_bwd(b.d.float(), b.z, b.lengths, sh, ws), lambda: lib.shape_logits_bwd(b.d[:, :2], b.z, b.lengths, sh, ws),
             lambda: lib.shaped_logprobs(b.z, b.ids.int(), b.lengths, sh, ws), lambda: lib.shaped_logprobs(b.z, b.ids[:, :2], b.lengths, sh, ws),
             lambda: lib.shaped_logprobs(b.z, b.ids, b.lengths, sh, ws, out=lib.ShapedLogprobs(b.z, lse=torch.empty((B, T), **f32))),
             lambda: lib.shaped_logprobs_bwd(b.z, b.ids, b.lengths, sh, f, b.g[:, :2], None, ws),
             lambda: lib.shaped_logprobs_bwd(b.z, b.ids, b.lengths, sh, f, b.g, b.h.double(), ws),
             lambda: lib.shaped_logprobs_bwd(b.z, b.ids, b.lengths, sh, f, b.g, None, ws, out=torch.empty_like(b.z, dtype=torch.float32))]
    k = dict(k=4, scoring=0, scope=0, balance_coef=0.1, z_coef=0.0, grad_scale=1.0, ws=rws)
    calls += [lambda: lib.router_loss_fwd_bwd(b.router[0], b.lengths, **k), lambda: lib.router_loss_fwd_bwd(b.router.double(), b.lengths, **k),
              lambda: lib.router_loss_fwd_bwd(b.router.transpose(2, 3), b.lengths, **k), lambda: lib.router_loss_fwd_bwd(b.router, b.lengths[:1], **k),
              lambda: lib.router_loss_fwd_bwd(b.router, b.lengths, expert_ids=torch.zeros((2, B, T, 3), **i32), **k),
              lambda: lib.router_loss_fwd_bwd(b.router, b.lengths, expert_ids=torch.zeros((2, B, T, 4), **i64), **k),
              lambda: lib.router_loss_fwd_bwd(b.router, b.lengths, out=lib.RouterOutputs(b.router.float(), 4, 0), **k),
              lambda: lib.router_loss_fwd_bwd(b.router, b.lengths, out=lib.RouterOutputs(b.router, 4, 1), **k)]
    for i, call in enumerate(calls):
        with pytest.raises((ValueError, TypeError)):
            call()
            pytest.fail(f"call {i} was let through")
    for call in (lambda: lib.router_loss_fwd_bwd(b.router, b.lengths, **dict(k, k=17)), lambda: lib.router_loss_fwd_bwd(b.router, b.lengths, **dict(k, k=0)),
                 lambda: lib.router_loss_fwd_bwd(b.router, b.lengths, **dict(k, scoring=1, z_coef=0.1)),
                 lambda: lib.router_loss_fwd_bwd(b.router, b.lengths, **dict(k, ws=rws[:64])),
                 lambda: lib.shaped_logprobs_bwd(b.z, b.ids, b.lengths, sh, lib.ShapedLogprobs(b.z), b.g, b.h, ws),
                 lambda: lib.shape_logits(b.z, b.lengths, sh, ws[:64])):
        with pytest.raises((lib.RlhfError, ValueError)):
            call()
    torch.cuda.synchronize()
    assert lib.poll_status(ws) == 0 and lib.poll_status(rws) == 0
