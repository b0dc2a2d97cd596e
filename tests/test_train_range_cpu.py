"""Refusals of the group-normalisation and optimiser entry points at the ends of
what they accept (CPU: every call fails before any HIP call)."""
import ctypes

import pytest
import torch

from paper_2003_06513_amd import binding as B
from test_train_abi_cpu import BWD, FAKE, FWD, _param, _says


@pytest.fixture(scope="module")
def L():
    return B.lib()


@pytest.mark.parametrize("name", ["gamma", "beta", "mean", "rstd", "dgamma", "dbeta"])
@pytest.mark.parametrize("off", [1, 2, 3])
def test_norm_parameters_and_statistics_that_are_not_aligned(L, name, off):
    """A load that a wave has in common rounds such an address down: it would read other values."""
    if name in FWD:
        args = {**FWD, "mean": FAKE, "rstd": FAKE, name: FAKE + off}
        _says(L.psc_group_norm_fwd(*args.values()), B.PSC_ERR_ARG, "aligned")
    _says(L.psc_group_norm_bwd(*{**BWD, name: FAKE + off}.values()), B.PSC_ERR_ARG, "aligned")


@pytest.mark.parametrize("off", [1, 2, 3])
def test_optimiser_values_that_are_not_aligned(L, off):
    q, bad = (B.CParam * 1)(_param()), FAKE + off
    _says(L.psc_grad_norm(q, 1, 1.0, 1.0, bad, FAKE, 8192, None), B.PSC_ERR_ARG, "aligned")
    opt = B.CAdamW(0.1, 0.9, 0.99, 1e-8, None)
    _says(L.psc_adamw_step(q, 1, ctypes.byref(opt), bad, FAKE, None), B.PSC_ERR_ARG, "aligned")
    opt = B.CAdamW(0.1, 0.9, 0.99, 1e-8, bad)
    _says(L.psc_adamw_step(q, 1, ctypes.byref(opt), None, FAKE, None), B.PSC_ERR_ARG, "aligned")
    for m_out, v_out in ((bad, FAKE), (FAKE, bad)):
        _says(L.psc_adamw_moments(FAKE, FAKE, FAKE, 5, m_out, v_out, None), B.PSC_ERR_ARG, "aligned")


@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1.1754942e-38])
def test_eps_of_the_norm_below_the_least_normal(L, eps):
    """Squares of about eps would be lost in fp32: rstd would be that of a group without spread."""
    _says(L.psc_group_norm_fwd(*{**FWD, "eps": eps}.values()), B.PSC_ERR_ARG, "eps")


def test_current_stream_without_the_short_way(monkeypatch):
    """A torch that lacks the entry point for a stream's bare handle has the same streams by its public ones."""
    class Stream:
        cuda_stream = 1234

    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    for name in ("_TORCH", "_CURRENT", "_DEVICE"):
        monkeypatch.setattr(B, name, None)
    assert B._same_device() == 3
    assert B._stream(None) == B._stream(None, 0) == B._stream(Stream) == 1234


def test_optimiser_memory_is_held_for_the_stream_that_works_on_it(monkeypatch):
    """Also where that stream is the current one, not named: dropped early, the buffers would be given out while
    its step still writes them."""
    held = []

    class Buffer:
        def record_stream(self, s):
            held.append(s)

    opt = B.AdamW.__new__(B.AdamW)
    opt.m, opt.v, opt.scale, opt._state, opt._out, opt._ws = Buffer(), Buffer(), None, Buffer(), Buffer(), Buffer()
    opt._at, opt._streams = 0, {10}
    now, capturing = [10], [False]
    B._torch()
    monkeypatch.setattr(B, "_CURRENT", lambda device: now[0])
    monkeypatch.setattr(B, "_torch_stream", lambda stream: now[0] if stream is None else stream.cuda_stream)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])

    class Stream:
        def __init__(self, handle):
            self.cuda_stream = handle

    opt._hold(None)
    assert held == []
    now[0], capturing[0] = 11, True
    opt._hold(None)
    assert held == []
    capturing[0] = False
    opt._hold(None)
    assert held == [11] * 5
    for s in (None, Stream(10), Stream(11)):        # its own, and what it is held for already
        opt._hold(s)
    assert held == [11] * 5
    opt._hold(Stream(12))
    assert held[5:] == [12] * 5
