"""Argument checks of the operators on shaped logits and of the router's loss: made on the host before the device is touched,
so they run without a GPU (pointers are never dereferenced)."""
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
    yield (ctypes.addressof(buf) + 255) // 256 * 256
    del buf


NULL, SHAPE, ALIGN, STRIDE, WORKSPACE, SCALAR = 1, 2, 3, 4, 5, 6
BAD = float("nan"), float("inf")


def caller(lib, fn, names, defaults):
    def call(**kw):
        assert not set(kw) - set(names), kw
        return getattr(lib, fn)(*[kw.get(n, defaults[n]) for n in names])
    return call


def shaping(p, **kw):
    s = binding.ShapingStruct(prompt=p, prompt_stride_b=4, prompt_len=4, tokens=p, tokens_stride_b=4, tokens_len=4, start=p,
                              repetition=p, frequency=p, presence=p, temperature=p, bias=p, mask=p, mask_stride_b=4, mask_stride_t=1)
    for k, v in kw.items():
        setattr(s, k, v)
    return ctypes.pointer(s)


def calls(lib, p):
    rows = dict(logits=p, dtype=0, sb=32, st=8, sh=shaping(p), lengths=p, B=2, T=4, V=8, ws=p, wsn=lib.rlhf_workspace_bytes(2, 4), stream=None)
    yield "shape", caller(lib, "rlhf_shape_logits", "logits dtype sb st sh lengths B T V out odt osb ost ws wsn stream".split(),
                          dict(rows, out=p + 1024, odt=0, osb=32, ost=8))
    yield "shape_bwd", caller(lib, "rlhf_shape_logits_bwd", "ds dtype dsb dst logits sb st sh lengths B T V out osb ost ws wsn stream".split(),
                              dict(rows, ds=p + 2048, dsb=32, dst=8, out=p + 1024, osb=32, ost=8))
    yield "logprobs", caller(lib, "rlhf_shaped_logprobs", "logits dtype sb st ids isb sh lengths B T V lp lse ent ws wsn stream".split(),
                             dict(rows, ids=p, isb=4, lp=p, lse=p, ent=p))
    yield "logprobs_bwd", caller(lib, "rlhf_shaped_logprobs_bwd",
                                 "logits dtype sb st ids isb sh lengths B T V lp lse ent g h out osb ost ws wsn stream".split(),
                                 dict(rows, ids=p, isb=4, lp=p, lse=p, ent=p, g=p, h=p, out=p + 1024, osb=32, ost=8))


def test_what_all_of_them_check(lib, p):
    for name, call in calls(lib, p):
        writes = name != "logprobs"
        for arg in ("logits", "lengths", "ws", "sh") + (("out",) if writes else ("lp", "lse", "ids")):
            assert call(**{arg: None}) == NULL, (name, arg)
        assert call(dtype=2) == SCALAR and call(dtype=-1) == SCALAR
        for kw in (dict(B=0), dict(T=0), dict(V=0), dict(B=-2), dict(B=1 << 16, T=1 << 14)):
            assert call(**kw) == SHAPE, (name, kw)
        for kw in (dict(st=7), dict(sb=-1), dict(st=-8)):
            assert call(**kw) == STRIDE, (name, kw)
        if writes:
            for kw in (dict(ost=7), dict(osb=-1), dict(osb=31), dict(ost=9, osb=34)):
                assert call(**kw) == STRIDE, (name, kw)
            assert call(out=p + 1025) == ALIGN
        assert call(logits=p + 1) == ALIGN and call(lengths=p + 2) == ALIGN and call(ws=p + 16) == ALIGN
        assert call(wsn=100) == WORKSPACE


def test_the_shaping(lib, p):
    for name, call in calls(lib, p):
        ok = dict(wsn=100)                               # accepted: the next check answers
        assert call(sh=shaping(p), **ok) == WORKSPACE
        assert call(sh=ctypes.pointer(binding.ShapingStruct()), **ok) == WORKSPACE
        for kw in (dict(prompt=None), dict(tokens=None)):
            assert call(sh=shaping(p, **kw), **ok) == NULL, (name, kw)
        for kw in (dict(prompt_len=-1), dict(tokens_len=-1)):
            assert call(sh=shaping(p, **kw), **ok) == SHAPE, (name, kw)
        for k in ("prompt_stride_b", "tokens_stride_b", "bias_stride_b", "mask_stride_b", "mask_stride_t"):
            assert call(sh=shaping(p, **{k: -1}), **ok) == STRIDE, (name, k)
        for k in ("prompt", "tokens"):
            assert call(sh=shaping(p, **{k: p + 4}), **ok) == ALIGN, (name, k)
        for k in ("prompt_lengths", "start", "repetition", "frequency", "presence", "temperature", "bias", "mask"):
            assert call(sh=shaping(p, **{k: p + 2}), **ok) == ALIGN, (name, k)


def test_sizes_beyond_what_is_counted(lib, p):
    most = 1 << 30
    for name, call in calls(lib, p):
        assert call(V=most + 1) == SHAPE, name
        for k in ("prompt_len", "tokens_len"):
            assert call(sh=shaping(p, **{k: most}), wsn=100) == WORKSPACE, (name, k)
            assert call(sh=shaping(p, **{k: most + 1}), wsn=100) == SHAPE, (name, k)


def test_what_each_of_them_checks(lib, p):
    c = dict(calls(lib, p))
    for odt in (1, 3, -1):
        assert c["shape"](odt=odt) == SCALAR
    assert c["shape"](odt=2, wsn=100) == WORKSPACE and c["shape"](odt=2, out=p + 1026) == ALIGN
    assert c["shape"](out=p, osb=64) == STRIDE and c["shape"](out=p, odt=2) == STRIDE
    assert c["shape_bwd"](ds=None) == NULL and c["shape_bwd"](ds=p + 1) == ALIGN
    assert c["shape_bwd"](dst=7) == STRIDE and c["shape_bwd"](dsb=-1) == STRIDE
    assert c["shape_bwd"](out=p) == STRIDE               # the logits
    assert c["shape_bwd"](out=p + 2048, osb=64) == STRIDE
    for name in ("logprobs", "logprobs_bwd"):
        assert c[name](isb=-1) == STRIDE and c[name](ids=p + 4) == ALIGN and c[name](lse=p + 4) == ALIGN
        assert c[name](lp=p + 2) == ALIGN and c[name](ent=p + 2) == ALIGN
    assert c["logprobs_bwd"](out=p, osb=64) == STRIDE
    for arg in ("ids", "lp", "lse", "g", "ent"):
        assert c["logprobs_bwd"](**{arg: None}) == NULL, arg
    assert c["logprobs_bwd"](h=None, ent=None, wsn=100) == WORKSPACE
    assert c["logprobs_bwd"](g=p + 2) == ALIGN and c["logprobs_bwd"](h=p + 2) == ALIGN


def test_router(lib, p):
    names = "z dtype sl sb st ids isl isb ist lengths L B T E K scoring scope bc zc gs loss counts oids d dl db dt ws wsn stream".split()
    d = dict(z=p, dtype=0, sl=64, sb=32, st=8, ids=p, isl=16, isb=8, ist=2, lengths=p, L=3, B=2, T=4, E=8, K=2, scoring=0, scope=0,
             bc=0.01, zc=0.0, gs=1.0, loss=p, counts=p, oids=p, d=p + 4096, dl=64, db=32, dt=8, ws=p,
             wsn=lib.rlhf_router_workspace_bytes(3, 2, 4, 8), stream=None)
    call = caller(lib, "rlhf_router_loss_fwd_bwd", names, d)
    for name in ("z", "lengths", "loss", "counts", "d", "ws"):
        assert call(**{name: None}) == NULL, name
    for kw in (dict(L=0), dict(B=0), dict(T=0), dict(E=0), dict(E=1025), dict(K=0), dict(K=9), dict(K=-1), dict(L=1 << 10, B=1 << 10, T=1 << 10)):
        assert call(**kw) == SHAPE, kw
    for kw in [dict(dtype=3), dict(dtype=-1), dict(scoring=2), dict(scoring=-1), dict(scope=2), dict(scope=-1), dict(scoring=1, zc=0.1)] + \
            [{k: x} for k in ("bc", "zc", "gs") for x in BAD]:
        assert call(**kw) == SCALAR, kw
    for kw in [{k: -1} for k in ("sl", "sb", "st", "isl", "isb", "ist", "dl", "db", "dt")] + \
            [dict(dt=7), dict(db=31), dict(dl=63), dict(d=p, dl=128), dict(dl=0), dict(dt=0)]:
        assert call(**kw) == STRIDE, kw
    for name, off in (("z", 1), ("d", 4097), ("ids", 2), ("lengths", 2), ("loss", 2), ("counts", 2), ("oids", 2), ("ws", 16)):
        assert call(**{name: p + off}) == ALIGN, name
    assert call(dtype=2, z=p + 2) == ALIGN
    assert call(wsn=100) == WORKSPACE
    # axes of the gradient in any order, and axes of one position with any stride, are accepted: the next check answers
    for kw in (dict(dt=24, dl=8, db=96), dict(dl=8, db=24, dt=48), dict(L=1, dl=0), dict(B=1, T=1, db=0, dt=0), dict(ids=None), dict(oids=None)):
        assert call(wsn=100, **kw) == WORKSPACE, kw
    assert lib.rlhf_router_workspace_bytes(1, 0, 1, 8) == 0 and lib.rlhf_router_workspace_bytes(1, 1, 1, 1025) == 0
    for shape in ((1, 1, 1, 1), (24, 16, 1024, 128), (61, 1024, 1, 256)):
        n = lib.rlhf_router_workspace_bytes(*shape)
        assert n % 256 == 0 and n <= (1 << 16) + 16 * (1184 + shape[0] * shape[1]) + 4 * shape[3] * (1184 + shape[0] * shape[1])


def test_status_of_a_setting_out_of_range(lib):
    assert lib.rlhf_status_string(128) == b"RLHF_ERR_VALUE_RANGE"
    assert lib.rlhf_status_string(16 | 128) == b"RLHF_ERR_ID_RANGE|RLHF_ERR_VALUE_RANGE"
    assert lib.rlhf_status_string(240) == b"RLHF_ERR_ID_RANGE|RLHF_ERR_LENGTH_RANGE|RLHF_ERR_TIMEOUT|RLHF_ERR_VALUE_RANGE"
    assert lib.rlhf_status_string(256) == b"RLHF_ERR_UNKNOWN"


def test_binding_says_what_is_wrong_with_cpu_tensors():
    z = torch.zeros((2, 3, 8), dtype=torch.bfloat16)
    n, ws = torch.ones(2, dtype=torch.int32), torch.zeros(8192, dtype=torch.uint8)
    ids, sh = torch.zeros((2, 3), dtype=torch.int64), binding.Shaping(2, 8)
    f = binding.ShapedLogprobs(z)
    for call in (lambda: binding.shape_logits(z, n, sh, ws), lambda: binding.shape_logits_bwd(z, z, n, sh, ws),
                 lambda: binding.shaped_logprobs(z, ids, n, sh, ws), lambda: binding.shaped_logprobs_bwd(z, ids, n, sh, f, f.logprobs, None, ws),
                 lambda: binding.Shaping(2, 8, tokens=ids), lambda: binding.Shaping(2, 8, temperature=torch.ones(2)),
                 lambda: binding.router_loss_fwd_bwd(z[None], n, 2, 0, 0, 0.1, 0.0, 1.0, ws)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
