"""Refusals of the group-normalisation and optimiser entry points (CPU: every
call fails, or has nothing to do, before any HIP call)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2003_06513_amd import binding as B

FAKE, FAR = 0x10000, 0x400000000       # never dereferenced


@pytest.fixture(scope="module")
def L():
    return B.lib()


def _says(rc, status, text):
    assert rc == status and text in B.last_error(), (rc, B.last_error())


FWD = dict(dtype=0, layout=0, x=FAKE, n=2, c=6, h=4, w=5, groups=3, gamma=None, beta=None, eps=1e-5, act=0, y=FAR,
           mean=None, rstd=None, ws=FAKE, ws_bytes=1 << 20, stream=None)
BWD = dict(dtype=0, layout=0, x=FAKE, dy=FAKE, n=2, c=6, h=4, w=5, groups=3, gamma=None, beta=None, mean=FAKE,
           rstd=FAKE, act=0, dx=FAR, dgamma=None, dbeta=None, ws=FAKE, ws_bytes=1 << 20, stream=None)
SHARED = [
    (dict(dtype=2), "dtype"), (dict(layout=2), "layout"), (dict(n=-1), "shape"), (dict(n=65536), "shape"),
    (dict(c=0), "shape"), (dict(h=0), "shape"), (dict(w=32769), "shape"), (dict(groups=0), "groups"),
    (dict(groups=4), "groups"), (dict(groups=12), "groups"), (dict(act=3), "act"), (dict(act=-1), "act"),
    (dict(n=60000, c=60000, groups=1), "2^31-1"), (dict(n=60000, c=1, h=32768, w=32768, groups=1), "2^31-1"),
    (dict(x=None), "non-NULL"), (dict(x=FAKE + 2), "aligned"),
]


@pytest.mark.parametrize("change,text", SHARED + [
    (dict(eps=0.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"),
    (dict(mean=FAKE), "both"), (dict(rstd=FAKE), "both"), (dict(y=None), "non-NULL"), (dict(y=FAKE + 4), "overlaps"),
    (dict(y=FAKE), "overlaps"),
])
def test_forward_refuses(L, change, text):
    _says(L.psc_group_norm_fwd(*{**FWD, **change}.values()), B.PSC_ERR_ARG, text)


@pytest.mark.parametrize("change,text", SHARED + [
    (dict(dy=None), "non-NULL"), (dict(dx=None), "non-NULL"), (dict(mean=None), "non-NULL"),
    (dict(rstd=None), "non-NULL"), (dict(dx=FAKE), "overlaps"), (dict(dy=FAR + 100), "overlaps"),
])
def test_backward_refuses(L, change, text):
    _says(L.psc_group_norm_bwd(*{**BWD, **change}.values()), B.PSC_ERR_ARG, text)


def test_group_norm_workspace(L):
    big = dict(c=64, h=56, w=56, groups=2)
    need = B.group_norm_workspace(0, 0, 2, 64, 56, 56, 2, True)
    assert need >= B.group_norm_workspace(0, 0, 2, 64, 56, 56, 2, True, aligned=True) > 0
    need = B.group_norm_workspace(0, 0, 2, 64, 56, 56, 2, True, aligned=True)
    for ws, size in ((None, need), (FAKE, need - 1), (FAKE + 8, need)):
        assert L.psc_group_norm_bwd(*{**BWD, **big, "ws": ws, "ws_bytes": size}.values()) == B.PSC_ERR_WORKSPACE
    need = B.group_norm_workspace(0, 0, 1, 8, 300, 300, 1, aligned=True)
    if need:
        args = {**FWD, "n": 1, "c": 8, "h": 300, "w": 300, "groups": 1, "ws": FAKE, "ws_bytes": need - 1}
        assert L.psc_group_norm_fwd(*args.values()) == B.PSC_ERR_WORKSPACE
    assert B.group_norm_workspace(0, 0, 0, 64, 56, 56, 2, True) >= 0
    out = ctypes.c_size_t(0)
    _says(L.psc_group_norm_workspace(0, 0, 1, 6, 4, 4, 5, 0, 0, ctypes.byref(out)), B.PSC_ERR_ARG, "groups")
    _says(L.psc_group_norm_workspace(0, 0, 1, 6, 4, 4, 3, 0, 0, None), B.PSC_ERR_ARG, "NULL")
    # no images: nothing to do, whatever the pointers are
    assert L.psc_group_norm_fwd(*{**FWD, "n": 0, "x": None, "y": None, "ws": None}.values()) == B.PSC_OK


def _param(**k):
    q = B.CParam(FAKE, FAKE, None, FAKE, FAKE, FAKE, 10, 0.0, B.PSC_F32, 32, 0)
    for name, v in k.items():
        setattr(q, name, v)
    return q


@pytest.mark.parametrize("change,text", [
    (dict(numel=-1), "numel"), (dict(numel=1 << 31), "numel"), (dict(grad_dtype=5), "grad_dtype"),
    (dict(grad=None), "grad is NULL"), (dict(grad=FAKE + 2), "aligned"), (dict(grad=FAKE + 1, grad_dtype=1), "aligned"),
])
def test_lists_are_refused(L, change, text):
    q = (B.CParam * 2)(_param(), _param(**change))
    _says(L.psc_grad_norm(q, 2, 1.0, 1.0, FAKE, FAKE, 8192, None), B.PSC_ERR_ARG, text)
    opt = B.CAdamW(0.1, 0.9, 0.99, 1e-8, None)
    _says(L.psc_adamw_step(q, 2, ctypes.byref(opt), None, FAKE, None), B.PSC_ERR_ARG, text)
    assert "params[1]" in B.last_error()


@pytest.mark.parametrize("change,text", [
    (dict(state_bits=16), "state_bits"), (dict(reserved=1), "reserved"), (dict(weight_decay=-0.1), "weight_decay"),
    (dict(weight_decay=float("nan")), "weight_decay"), (dict(param=None), "non-NULL"), (dict(m=None), "non-NULL"),
    (dict(v=None), "non-NULL"), (dict(param=FAKE + 2), "aligned"), (dict(m=FAKE + 1), "aligned"),
    (dict(copy=FAKE + 1), "aligned"), (dict(state_bits=8, scale=None), "scale"), (dict(state_bits=8, scale=FAKE + 4), "scale"),
    (dict(param=1 << 48), "48 bits"), (dict(grad=1 << 63), "48 bits"), (dict(copy=1 << 50), "48 bits"),
    (dict(m=1 << 48), "48 bits"), (dict(v=1 << 48), "48 bits"), (dict(state_bits=8, scale=1 << 48), "48 bits"),
])
def test_step_refuses_tensors(L, change, text):
    q, opt = (B.CParam * 1)(_param(**change)), B.CAdamW(0.1, 0.9, 0.99, 1e-8, None)
    _says(L.psc_adamw_step(q, 1, ctypes.byref(opt), None, FAKE, None), B.PSC_ERR_ARG, text)


def test_step_refuses_settings(L):
    q = (B.CParam * 1)(_param())
    for opt, text in ((B.CAdamW(float("nan"), 0.9, 0.99, 1e-8, None), "lr"), (B.CAdamW(0.1, 1.0, 0.99, 1e-8, None), "beta"),
                      (B.CAdamW(0.1, -0.1, 0.99, 1e-8, None), "beta"), (B.CAdamW(0.1, 0.9, 1.0, 1e-8, None), "beta"),
                      (B.CAdamW(0.1, 0.9, 0.99, 0.0, None), "eps"), (B.CAdamW(0.1, 0.9, 0.99, float("inf"), None), "eps")):
        _says(L.psc_adamw_step(q, 1, ctypes.byref(opt), None, FAKE, None), B.PSC_ERR_ARG, text)
    opt = B.CAdamW(0.1, 0.9, 0.99, 1e-8, None)
    _says(L.psc_adamw_step(q, 1, None, None, FAKE, None), B.PSC_ERR_ARG, "opt")
    _says(L.psc_adamw_step(q, 1, ctypes.byref(opt), None, None, None), B.PSC_ERR_ARG, "d_state")
    _says(L.psc_adamw_step(q, 1, ctypes.byref(opt), None, FAKE + 8, None), B.PSC_ERR_ARG, "d_state")
    _says(L.psc_adamw_step(q, -1, ctypes.byref(opt), None, FAKE, None), B.PSC_ERR_ARG, "count")
    _says(L.psc_adamw_step(None, 1, ctypes.byref(opt), None, FAKE, None), B.PSC_ERR_ARG, "h_params")


def test_norm_refuses(L):
    q = (B.CParam * 1)(_param())
    _says(L.psc_grad_norm(q, 1, 0.0, 1.0, FAKE, FAKE, 8192, None), B.PSC_ERR_ARG, "scale")
    _says(L.psc_grad_norm(q, 1, float("inf"), 1.0, FAKE, FAKE, 8192, None), B.PSC_ERR_ARG, "scale")
    _says(L.psc_grad_norm(q, 1, 1.0, 0.0, FAKE, FAKE, 8192, None), B.PSC_ERR_ARG, "max_norm")
    _says(L.psc_grad_norm(q, 1, 1.0, float("nan"), FAKE, FAKE, 8192, None), B.PSC_ERR_ARG, "max_norm")
    _says(L.psc_grad_norm(q, 1, 1.0, 1.0, None, FAKE, 8192, None), B.PSC_ERR_ARG, "d_out")
    for ws, size in ((None, 8192), (FAKE, 8191), (FAKE + 4, 8192)):
        assert L.psc_grad_norm(q, 1, 1.0, 1.0, FAKE, ws, size, None) == B.PSC_ERR_WORKSPACE


def test_moments_refuse(L):
    _says(L.psc_adamw_moments(FAKE, FAKE, FAKE, -1, FAKE, FAKE, None), B.PSC_ERR_ARG, "numel")
    _says(L.psc_adamw_moments(FAKE, None, FAKE, 5, FAKE, FAKE, None), B.PSC_ERR_ARG, "non-NULL")
    _says(L.psc_adamw_moments(FAKE, FAKE, FAKE + 4, 5, FAKE, FAKE, None), B.PSC_ERR_ARG, "aligned")
    assert L.psc_adamw_moments(None, None, None, 0, None, None, None) == B.PSC_OK


def test_structs_match_the_header():
    assert ctypes.sizeof(B.CParam) == 72 and ctypes.sizeof(B.CAdamW) == 24


class _Fake(torch.Tensor):
    """A host tensor that says it lies on a device, for the binding's own checks."""

    is_cuda = property(lambda self: True)


def _t(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(_Fake)


def test_lists_of_the_binding():
    p, g = [_t(300), _t(5)], [_t(300), _t(5)]
    m, v = [_t(300), _t(5)], [_t(300), _t(5)]
    ok = B.ParamList(p, g, m, v, weight_decay=[0.1, 0.0])
    assert ok.c[0].numel == 300 and ok.c[1].state_bits == 32 and abs(ok.c[0].weight_decay - 0.1) < 1e-7
    whole = _t(10)
    for args, text in (
            ((p, g[:1], m, v), "one entry"), ((p, g, m, [v[0], _t(6)]), "v[1]"), ((p, g, [m[0], None], v), "m[1]"),
            (([p[0], _t(5, dtype=torch.float16)], g, m, v), "params[1]"), (([p[0], p[0][:5]], g, m, v), "overlap"),
            ((p, g, m, [v[0], m[1]]), "overlap"), ((p, [g[0], p[0][295:]], m, v), "overlaps"),
            ((p, g, [_t(300, dtype=torch.int8), m[1]], [_t(300, dtype=torch.uint8), v[1]]), "scale[0]"),
            ((p, [g[0], _t(5, dtype=torch.float64)], m, v), "float32 and float16"),
            ((p, [g[0], _t(5, 2)[:, 0]], m, v), "contiguous"),
            (([whole[:5], whole[3:8]], [_t(5), _t(5)], [_t(5), _t(5)], [_t(5), _t(5)]), "overlap")):
        with pytest.raises((ValueError, TypeError)) as e:
            B.ParamList(*args)
        assert text in str(e.value), (text, str(e.value))
    with pytest.raises(ValueError):
        ok.set_grads([g[0]])
    with pytest.raises(ValueError):
        ok.set_grads([g[0], _t(6)])
    with pytest.raises(ValueError):
        ok.set_grads([g[0], v[1]])
    ok.set_grads([_t(300, dtype=torch.float16), g[1]])
    assert ok.c[0].grad_dtype == B.PSC_F16


def test_layouts_of_the_binding():
    x = _t(2, 6, 4, 5)
    assert B._layout(x) == B.PSC_NCHW
    last = torch.zeros(2, 4, 5, 6).permute(0, 3, 1, 2).as_subclass(_Fake)
    assert B._layout(last) == B.PSC_NHWC
    with pytest.raises(ValueError):
        B._like(x, last, B.PSC_NHWC, "y")
    for bad in (_t(2, 6, 4), _t(2, 6, 4, 10)[..., ::2], _t(2, 6, 5, 4).transpose(2, 3), torch.zeros(2, 6, 4, 5)):
        with pytest.raises(ValueError):
            B._layout(bad)
    with pytest.raises(ValueError):
        B._act_code("gelu")
