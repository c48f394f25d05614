"""Argument checks of the objectives beside the PPO step: made on the host before the device is touched, so they run without
a GPU (pointers are never dereferenced)."""
import ctypes

import pytest
import torch

from paper_2410_15651_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


@pytest.fixture(scope="module")
def p():
    buf = (ctypes.c_char * 65536)()
    test_pointer = (ctypes.addressof(buf) + 255) // 256 * 256
    yield test_pointer
    del buf


NULL, SHAPE, ALIGN, STRIDE, WORKSPACE, SCALAR = 1, 2, 3, 4, 5, 6
BAD = float("nan"), float("inf")


def caller(lib, fn, names, defaults):
    def call(**kw):
        unknown = set(kw) - set(names)
        assert not unknown, unknown
        return getattr(lib, fn)(*[kw.get(n, defaults[n]) for n in names])
    return call


def rows(p, ws):
    return dict(logits=p, dtype=0, sb=32, st=8, ids=p, isb=4, lengths=p, B=2, T=4, V=8, dl=p + 1024, dsb=32, dst=8, ws=p,
                wsn=ws, stream=None)


def check_rows(call, p):
    """What all of them check of logits, gradient and workspace."""
    for name in ("logits", "lengths", "dl", "ws"):
        assert call(**{name: None}) == NULL, name
    assert call(dtype=2) == SCALAR and call(dtype=-1) == SCALAR
    for kw in (dict(B=0), dict(T=0), dict(V=0), dict(B=-2), dict(B=1 << 16, T=1 << 14)):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(st=7), dict(dst=7), dict(sb=-1), dict(dsb=-1), dict(dsb=24), dict(dl=p, dsb=64)):
        assert call(**kw) == STRIDE, kw
    for kw in (dict(logits=p + 1), dict(dl=p + 1025), dict(lengths=p + 2), dict(ws=p + 16)):
        assert call(**kw) == ALIGN, kw
    assert call(wsn=100) == WORKSPACE


def test_policy_kl(lib, p):
    names = "logits dtype sb st ids isb lengths lp_old lp_ref adv asb ast B T V lo hi kl red gs lpg lkl dl dsb dst lpn ws wsn stream".split()
    d = dict(rows(p, lib.rlhf_workspace_bytes(2, 4)), lp_old=p, lp_ref=p, adv=p, asb=4, ast=1, lo=0.2, hi=0.3, kl=0.1, red=0,
             gs=1.0, lpg=p, lkl=p + 4, lpn=None)
    call = caller(lib, "rlhf_policy_kl_loss_fwd_bwd", names, d)
    check_rows(call, p)
    for name in ("ids", "lp_old", "adv", "lpg", "lkl"):
        assert call(**{name: None}) == NULL, name
    for kw in [dict(lo=x) for x in (0.0, 1.0, -0.1) + BAD] + [dict(hi=x) for x in (0.0, -1.0) + BAD] + \
            [dict(kl=x) for x in (-0.1,) + BAD] + [dict(gs=x) for x in BAD] + [dict(red=2), dict(red=-1)]:
        assert call(**kw) == SCALAR, kw
    assert call(asb=-1) == STRIDE and call(ast=-1) == STRIDE and call(isb=-1) == STRIDE
    for name in ("ids", "lp_old", "lp_ref", "adv", "lpg", "lkl", "lpn"):
        assert call(**{name: p + 2}) == ALIGN, name


def test_preference(lib, p):
    names = "logits dtype sb st ids isb lengths lp_ref B T V kind beta margin eps mean gs loss rew dl dsb dst lpn ws wsn stream".split()
    d = dict(rows(p, lib.rlhf_workspace_bytes(2, 4)), lp_ref=p, kind=0, beta=0.1, margin=0.0, eps=0.0, mean=0, gs=1.0, loss=p,
             rew=p, lpn=None)
    call = caller(lib, "rlhf_preference_loss_fwd_bwd", names, d)
    check_rows(call, p)
    for name in ("ids", "loss", "rew"):
        assert call(**{name: None}) == NULL, name
    assert call(B=3) == SHAPE and call(B=1) == SHAPE
    for kw in [dict(kind=3), dict(kind=-1), dict(mean=2), dict(eps=0.5), dict(eps=-0.1), dict(kind=1, eps=0.1),
               dict(kind=2, eps=0.1)] + [dict(beta=x) for x in (0.0, -1.0) + BAD] + [dict(margin=x) for x in BAD] + \
            [dict(gs=x) for x in BAD] + [dict(eps=BAD[0])]:
        assert call(**kw) == SCALAR, kw
    for name in ("ids", "lp_ref", "loss", "rew", "lpn"):
        assert call(**{name: p + 2}) == ALIGN, name


def test_distill(lib, p):
    names = "logits dtype sb st tid tlp ksb kst K lengths B T V mode tau gs loss row dl dsb dst ws wsn stream".split()
    d = dict(rows(p, lib.rlhf_workspace_bytes(2, 4)), tid=p, tlp=p, ksb=16, kst=4, K=4, mode=0, tau=1.0, gs=1.0, loss=p, row=None)
    call = caller(lib, "rlhf_distill_loss_fwd_bwd", names, d)
    check_rows(call, p)
    for name in ("tid", "tlp", "loss"):
        assert call(**{name: None}) == NULL, name
    assert call(K=0) == SHAPE and call(K=257) == SHAPE and call(K=-1) == SHAPE
    assert call(ksb=-1) == STRIDE and call(kst=-1) == STRIDE
    for kw in [dict(mode=3), dict(mode=-1)] + [dict(tau=x) for x in (0.0, -1.0) + BAD] + [dict(gs=x) for x in BAD]:
        assert call(**kw) == SCALAR, kw
    for name in ("tid", "tlp", "loss", "row"):
        assert call(**{name: p + 2}) == ALIGN, name


def test_topk(lib, p):
    names = "logits dtype sb st lengths B T V K tau oid olp ws wsn stream".split()
    d = dict(rows(p, lib.rlhf_workspace_bytes(2, 4)), K=4, tau=1.0, oid=p, olp=p)
    call = caller(lib, "rlhf_topk_logprobs", names, d)
    for name in ("logits", "lengths", "oid", "olp", "ws"):
        assert call(**{name: None}) == NULL, name
    for kw in (dict(K=0), dict(K=257), dict(K=-3), dict(B=0), dict(T=-1), dict(V=0), dict(B=1 << 16, T=1 << 14)):
        assert call(**kw) == SHAPE, kw
    assert call(st=7) == STRIDE and call(sb=-1) == STRIDE
    for kw in [dict(dtype=2)] + [dict(tau=x) for x in (0.0, -1.0) + BAD]:
        assert call(**kw) == SCALAR, kw
    for name, off in (("logits", 1), ("lengths", 2), ("oid", 2), ("olp", 2), ("ws", 16)):
        assert call(**{name: p + off}) == ALIGN, name
    assert call(wsn=100) == WORKSPACE


def test_binding_says_what_is_wrong_with_cpu_tensors():
    z = torch.zeros((2, 3, 8), dtype=torch.bfloat16)
    n, ws = torch.ones(2, dtype=torch.int32), torch.zeros(8192, dtype=torch.uint8)
    f, ids = torch.zeros((2, 3)), torch.zeros((2, 3), dtype=torch.int64)
    k = torch.zeros((2, 3, 4))
    for call in (lambda: binding.topk_logprobs(z, n, 4, 1.0, ws), lambda: binding.distill_loss_fwd_bwd(z, k.int(), k, n, 0, 1.0, 1.0, ws),
                 lambda: binding.policy_kl_loss_fwd_bwd(z, ids, n, f, f, f, 0.2, 0.2, 0.1, 0, 1.0, ws),
                 lambda: binding.preference_loss_fwd_bwd(z, ids, n, f, 0, 0.1, 0.0, 0.0, False, 1.0, ws)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()


def test_temperatures_whose_scale_or_square_leaves_fp32(lib, p):
    names = "logits dtype sb st lengths B T V K tau oid olp ws wsn stream".split()
    topk = caller(lib, "rlhf_topk_logprobs", names, dict(rows(p, lib.rlhf_workspace_bytes(2, 4)), K=4, tau=1.0, oid=p, olp=p))
    names = "logits dtype sb st tid tlp ksb kst K lengths B T V mode tau gs loss row dl dsb dst ws wsn stream".split()
    d = dict(rows(p, lib.rlhf_workspace_bytes(2, 4)), tid=p, tlp=p, ksb=16, kst=4, K=4, mode=0, tau=1.0, gs=1.0, loss=p, row=None)
    distill = caller(lib, "rlhf_distill_loss_fwd_bwd", names, d)
    for tau in (1e-45, 1e-39, 1e-30, 0.9e-3, 1.1e18, 1e20, 3e38):
        assert topk(tau=tau) == SCALAR and distill(tau=tau) == SCALAR, tau
    for tau in (1e-3, 1e18):                             # accepted: the next check answers
        assert topk(tau=tau, wsn=100) == WORKSPACE and distill(tau=tau, wsn=100) == WORKSPACE


def test_log_probs_written_over_an_input(lib, p):
    names = "logits dtype sb st ids isb lengths lp_ref B T V kind beta margin eps mean gs loss rew dl dsb dst lpn ws wsn stream".split()
    d = dict(rows(p, lib.rlhf_workspace_bytes(2, 4)), lp_ref=p + 256, kind=0, beta=0.1, margin=0.0, eps=0.0, mean=0, gs=1.0,
             loss=p, rew=p, lpn=p + 512)
    call = caller(lib, "rlhf_preference_loss_fwd_bwd", names, d)
    assert call(lpn=p + 256) == STRIDE and call(lpn=p + 256 + 4) == STRIDE and call(lpn=p + 256 - 4) == STRIDE
    assert call(wsn=100) == WORKSPACE and call(wsn=100, lpn=p + 256 + 32) == WORKSPACE
    names = "logits dtype sb st ids isb lengths lp_old lp_ref adv asb ast B T V lo hi kl red gs lpg lkl dl dsb dst lpn ws wsn stream".split()
    d = dict(rows(p, lib.rlhf_workspace_bytes(2, 4)), lp_old=p + 256, lp_ref=p + 512, adv=p + 768, asb=4, ast=1, lo=0.2, hi=0.3,
             kl=0.1, red=0, gs=1.0, lpg=p, lkl=p + 4, lpn=p + 2048)
    call = caller(lib, "rlhf_policy_kl_loss_fwd_bwd", names, d)
    for at in (256, 512, 768):
        assert call(lpn=p + at) == STRIDE and call(lpn=p + at + 4) == STRIDE, at
    assert call(wsn=100) == WORKSPACE
