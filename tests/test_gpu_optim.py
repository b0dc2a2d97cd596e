"""The gradient norm and the AdamW step against the fp64 oracle.

Bounds (u = 2^-24): the norm sums in fp64 and is rounded once, its factor
rounded once after a quotient in fp64: 2 u each, relatively.  m takes two
products and a sum of rounded constants: 4 u of |b1 m| + |(1-b1) g|; v one
product more: 5 u of itself (its terms are positive).  The parameter: two
roundings of p and the decay, and of the update rounded constants, v's error
halved, a root and a reciprocal within one unit in the last place each, and
three products: 16 u of it, the decay's product 2 u; besides, the update is m
times lr / (1-b1^t) / (sqrt(v / (1-b2^t)) + eps), so that m's error of up to
4 u (|b1 m| + |(1-b1) g|), which is more than a rounding of m where the two
terms cancel, reaches it times that quotient.  8-bit moments are computed in fp64: their scales are
within one rounding, the codes those of the oracle exactly."""
import numpy as np
import pytest

from oracle import train
from paper_2003_06513_amd import binding as B
from gpu_cases import U16, U32, dev, note, torch_mod

pytestmark = pytest.mark.gpu
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8)


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    B.lib()


def _h(t):
    return t.detach().cpu().numpy()


def _flat(arrays, shift, guard, dtype=None):
    """Device tensors in one buffer, ``shift`` elements past a multiple of 256
    each, guard values around them."""
    torch = torch_mod()
    at, end = [], 0
    for a in arrays:
        at.append(end + shift)
        end += -(-(a.size + shift + 8) // 256) * 256
    buf = torch.full((end,), guard, dtype=dtype or torch.float32, device="cuda")
    views = [buf[i:i + a.size] for i, a in zip(at, arrays)]
    for t, a in zip(views, arrays):
        t.copy_(torch.from_numpy(a.copy()))
    mask = torch.ones(end, dtype=torch.bool, device="cuda")
    for i, a in zip(at, arrays):
        mask[i:i + a.size] = False
    return views, buf, mask


LISTS = [[1], [5, 0, 256, 257, 3], [1024, 1023, 4097, 64], [70001, 12], list(range(1, 120)), [300_000, 5, 262_144],
         [7] * 400, [1024] * 16, [1000] * 17, [16384], [300] * 83, [300] * 84]


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: "%dx%d" % (len(s), max(s)))
def test_norm(sizes, half):
    torch = torch_mod()
    rng = np.random.default_rng(len(sizes))
    grads = [rng.standard_normal(k).astype(np.float16 if half else np.float32) for k in sizes]
    for shift in (0, 1, 4):
        views, _, _ = _flat(grads, shift, 1e30 if not half else 1e4, torch.float16 if half else None)
        out = torch.full((2,), 7.0, device="cuda")
        for max_norm, scale in ((np.inf, 1.0), (0.5, 1.0), (3.0, 0.25)):
            note("norm of %d tensors" % len(sizes))
            B.grad_norm(B.ParamList(None, views), out, max_norm=max_norm, scale=scale)
            got = _h(out)
            want = train.grad_norm(grads, scale, max_norm)
            assert np.abs(got - want).max() <= 2 * U32 * max(want), (got, want)


@pytest.mark.parametrize("half", [False, True])
def test_norm_rounds_once(half):
    """Squares and sums in 64 bits (2^-53 of the sum each, far below 2^-10 of a
    rounding of 32): norm and factor are those of 64 bits rounded once.  The
    last bit of the factor decides codes of 8-bit moments."""
    torch = torch_mod()
    rng = np.random.default_rng(77)
    out = torch.zeros(2, device="cuda")
    most = float(np.float32(1e-3))      # the argument has 32 bits: 1e-3 itself is 4.7e-8 of it away
    for k in list(range(1, 40)) + [100, 333, 1000, 5000, 20_000, 70_001] * 5:
        g = (10.0 ** rng.uniform(-4, 2) * rng.standard_normal(k)).astype(np.float16 if half else np.float32)
        if not g.any():
            continue
        note("norm of %d values" % k)
        B.grad_norm(B.ParamList(None, [torch.from_numpy(g).cuda()]), out, max_norm=1e-3)
        want = np.array(train.grad_norm([g], 1.0, most))
        assert (np.abs(_h(out) - want) <= U32 * (1 + 2.0 ** -10) * want).all(), (k, _h(out), want)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_norm_of_half_precision_that_is_not_finite(bad):
    torch = torch_mod()
    out = torch.zeros(2, device="cuda")
    for n, at in ((1, 0), (5000, 4999), (70000, 31), (70000, 69999)):
        g = torch.full((n,), 65504.0, dtype=torch.float16, device="cuda")
        B.grad_norm(B.ParamList(None, [g]), out)
        assert abs(float(out[0]) / (65504 * np.sqrt(n)) - 1) < 1e-6 and float(out[1]) == 1.0
        g[at] = bad
        B.grad_norm(B.ParamList(None, [g]), out)
        assert (np.isnan(_h(out)[0]) if np.isnan(bad) else _h(out)[0] == np.inf) and np.isnan(_h(out)[1])
    least = torch.full((3,), 2.0 ** -24, dtype=torch.float16, device="cuda")
    B.grad_norm(B.ParamList(None, [least]), out)
    assert abs(float(out[0]) / (2.0 ** -24 * np.sqrt(3)) - 1) < 1e-6
    B.grad_norm(B.ParamList(None, [torch.zeros(5000, dtype=torch.float16, device="cuda")]), out, max_norm=1.0)
    assert np.array_equal(_h(out), [0, 1])


def test_norm_extremes():
    torch = torch_mod()
    out = torch.zeros(2, device="cuda")
    run = lambda *g, **k: (B.grad_norm(B.ParamList(None, list(g)), out, **k), _h(out))[1]      # noqa: E731
    big = torch.full((1000,), 1e30, device="cuda")        # the squares pass fp32, the norm does not
    assert abs(run(big, max_norm=1.0)[0] / (1e30 * np.sqrt(1000)) - 1) < 1e-6
    small = torch.full((1000,), 1e-38, device="cuda")
    assert abs(run(small)[0] / (1e-38 * np.sqrt(1000)) - 1) < 1e-6
    for bad in (np.inf, np.nan):
        t = torch.ones(70000, device="cuda")
        t[69999] = bad
        got = run(big, t, max_norm=1.0)
        assert not np.isfinite(got[0]) and np.isnan(got[1])
    assert np.array_equal(run(torch.zeros(10, device="cuda"), max_norm=1.0), [0, 1])
    assert np.array_equal(run(torch.zeros(0, device="cuda"), max_norm=1.0), [0, 1])


def _check_step(p0, g, m0, v0, p, m, v, t, decay, factor, what, hyper=HYPER):
    rp, rm, rv = train.adamw(p0, g, m0, v0, t, weight_decay=decay, factor=factor, **hyper)
    g = np.abs(g.astype(np.float64) * np.float32(factor))
    e_m = 4 * U32 * (hyper["beta1"] * np.abs(m0) + (1 - hyper["beta1"]) * g)
    assert (np.abs(m - rm) <= e_m + 1e-44).all(), what + " m"
    assert (np.abs(v - rv) <= 5 * U32 * rv + 1e-44).all(), what + " v"
    quotient = hyper["lr"] / (1 - hyper["beta1"] ** t) / (np.sqrt(rv / (1 - hyper["beta2"] ** t)) + hyper["eps"])
    _check_param(p0, p, rp, decay, hyper, what, e_m * quotient)


def _check_param(p0, p, rp, decay, hyper, what, from_m=0.0):
    p0 = p0.astype(np.float64)
    kept = p0 - float(np.float32(hyper["lr"])) * float(np.float32(decay)) * p0
    update = np.abs(rp - kept)
    bound = 2 * U32 * (np.abs(rp) + np.abs(kept)) + 4 * U32 * hyper["lr"] * decay * np.abs(p0) + 16 * U32 * update + from_m
    assert (np.abs(p - rp) <= bound + 1e-44).all(), "%s: p off by %.3g bounds" % (
        what, (np.abs(p - rp) / (bound + 1e-44)).max())


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: "%dx%d" % (len(s), max(s)))
def test_adamw32(sizes, half):
    torch = torch_mod()
    rng = np.random.default_rng(3 + len(sizes))
    for shift in (0, 1):
        p0 = [rng.standard_normal(k).astype(np.float32) for k in sizes]
        decay = [0.1 * (i % 3) for i in range(len(sizes))]
        p, buf, outside = _flat(p0, shift, 77.0)
        cp, cbuf, _ = _flat([a.astype(np.float16) for a in p0], shift, 77.0, torch.float16)
        grads = [torch.empty(k, dtype=torch.float16 if half else torch.float32, device="cuda") for k in sizes]
        opt = B.AdamW(p, grads, lr=HYPER["lr"], weight_decay=decay, copies=[c if i % 2 == 0 else None
                                                                           for i, c in enumerate(cp)])
        factor = torch.tensor([0.37], device="cuda")
        for t in (1, 2, 3):
            g = [(10.0 ** rng.uniform(-3, 1, k) * rng.standard_normal(k)).astype(np.float16 if half else np.float32)
                 for k in sizes]
            for d, a in zip(grads, g):
                d.copy_(torch.from_numpy(a))
            before = [[_h(x).copy() for x in (p[i], m, v)] for i, (m, v) in enumerate(_moments(opt, sizes))]
            note("adamw 32 step %d of %d tensors" % (t, len(sizes)))
            opt.step(factor=factor if t == 2 else None)
            torch.cuda.synchronize()
            for i, (m, v) in enumerate(_moments(opt, sizes)):
                b = before[i]
                _check_step(b[0], g[i], b[1], b[2], _h(p[i]), _h(m), _h(v), t, decay[i], 0.37 if t == 2 else 1.0,
                            "tensor %d step %d" % (i, t))
                if i % 2 == 0:
                    assert _h(cp[i]).tobytes() == _h(p[i]).astype(np.float16).tobytes()
                else:
                    assert _h(cp[i]).tobytes() == p0[i].astype(np.float16).tobytes()
        assert int(opt.steps) == 3
        assert bool((buf[outside] == 77).all()) and bool((cbuf[outside] == 77).all()), "written outside the tensors"


def _moments(opt, sizes):
    at = 0
    for k in sizes:
        yield opt.m[at:at + k], opt.v[at:at + k]
        at += -(-k // 256) * 256


def _scales(opt, sizes):
    at = 0
    for k in sizes:
        n = -(-k // 256)
        yield opt.scale[at:at + n]
        at += n


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: "%dx%d" % (len(s), max(s)))
def test_adamw8(sizes, half):
    torch = torch_mod()
    rng = np.random.default_rng(5 + len(sizes))
    for shift in (0, 3):
        p0 = [rng.standard_normal(k).astype(np.float32) for k in sizes]
        p, buf, outside = _flat(p0, shift, 77.0)
        grads = [torch.empty(k, dtype=torch.float16 if half else torch.float32, device="cuda") for k in sizes]
        opt = B.AdamW(p, grads, lr=HYPER["lr"], weight_decay=0.1, state_bits=8)
        factor = torch.tensor([0.37], device="cuda")
        for t in (1, 2, 3, 4):
            f = 0.37 if t == 2 else 1.0
            g = [(10.0 ** rng.uniform(-3, 1, k) * rng.standard_normal(k)).astype(np.float16 if half else np.float32)
                 for k in sizes]
            if t == 3:
                g = [np.zeros_like(a) for a in g]
            for d, a in zip(grads, g):
                d.copy_(torch.from_numpy(a))
            before = [[_h(x).copy() for x in (p[i], m, v, s)]
                      for i, ((m, v), s) in enumerate(zip(_moments(opt, sizes), _scales(opt, sizes)))]
            note("adamw 8 step %d of %d tensors" % (t, len(sizes)))
            opt.step(factor=factor if t == 2 else None)
            torch.cuda.synchronize()
            fm, fv = opt.moments()
            at = 0
            for i, ((m, v), s) in enumerate(zip(_moments(opt, sizes), _scales(opt, sizes))):
                k, what = sizes[i], "tensor %d step %d" % (i, t)
                bp, bm, bv, bs = before[i]
                rp, rm, rv = train.adamw(bp, g[i], train.decode_m(bm, bs), train.decode_v(bv, bs), t, weight_decay=0.1,
                                         factor=f, **HYPER)
                qm, qv, qs = train.encode(rm, rv)
                assert (np.abs(_h(s).astype(np.float64) - qs) <= 2 * U32 * qs).all(), what + " scales"
                assert np.array_equal(_h(m), qm) and np.array_equal(_h(v), qv), what + " codes"
                _check_param(bp, _h(p[i]), rp, 0.1, HYPER, what)
                dm, dv = train.decode_m(qm, _h(s)), train.decode_v(qv, _h(s))
                assert (np.abs(_h(fm)[at:at + k] - dm) <= U32 * np.abs(dm) + 1e-44).all(), what + " values of m"
                assert (np.abs(_h(fv)[at:at + k] - dv) <= U32 * dv + 1e-44).all(), what + " values of v"
                at += -(-k // 256) * 256
        assert bool((buf[outside] == 77).all()), "written outside the tensors"


@pytest.mark.parametrize("bits", [32, 8])
def test_tiny_large_and_zero_moments(bits):
    """Gradients whose squares leave fp32's range at both ends stay in their own groups."""
    torch = torch_mod()
    g = torch.zeros(5 * 256, device="cuda")
    g[256:512] = 1e-15
    g[512:768] = 1e-22        # its square is below every fp32
    g[768:1024] = 1e15
    g[1024] = 1.0             # the rest of this group: zero
    p = torch.zeros(5 * 256, device="cuda")
    opt = B.AdamW([p], [g], lr=0.1, state_bits=bits)
    for _ in range(3):
        opt.step()
    m, v = opt.moments()
    torch.cuda.synchronize()
    assert not p[:256].any() and not m[:256].any() and not v[:256].any()
    assert bool(torch.isfinite(p).all()) and bool((v >= 0).all())
    # equal gradients: the step is lr in size, three times, where eps does not count
    assert abs(float(p[800]) + 0.3) < 1e-3 and abs(float(p[1024]) + 0.3) < 1e-3
    assert not p[1025:].any()
    # (1 - b1) g = 1e-16 against eps = 1e-8
    assert float(p[300]) == pytest.approx(-0.3 * 1e-15 / 1e-8, rel=1e-2)


@pytest.mark.parametrize("bits", [32, 8])
def test_not_finite(bits):
    """A factor that is not finite: nothing changes.  Without one, a gradient that is not finite spoils its own
    element, or the 256 that share its scales."""
    torch = torch_mod()
    rng = np.random.default_rng(8)
    p0 = rng.standard_normal(1000).astype(np.float32)
    p, g = dev(p0), dev(rng.standard_normal(1000).astype(np.float32))
    copy = torch.zeros(1000, dtype=torch.float16, device="cuda")
    opt = B.AdamW([p], [g], state_bits=bits, copies=[copy])
    opt.step()
    held = [t.clone() for t in (p, opt.m, opt.v, copy, opt.steps)]
    g[300] = np.inf
    opt.grad_norm(1.0)
    opt.step(factor=opt.factor)
    torch.cuda.synchronize()
    assert np.isinf(float(opt.norm)) and np.isnan(float(opt.factor))
    assert all(torch.equal(a, b) for a, b in zip(held, (p, opt.m, opt.v, copy, opt.steps)))
    opt.step()
    m, v = opt.moments()
    spoilt = torch.zeros(1000, dtype=torch.bool, device="cuda")
    spoilt[300] = True
    assert torch.equal(torch.isnan(p), spoilt)
    if bits == 8:
        spoilt[256:512] = True
    assert torch.equal(~torch.isfinite(m[:1000]), spoilt)
    assert int(opt.steps) == 2


def test_clip_and_mixed_list():
    """The factor from the norm's call, and moments of both widths in one list."""
    torch = torch_mod()
    rng = np.random.default_rng(11)
    sizes = [3000, 700, 64]
    p0 = [rng.standard_normal(k).astype(np.float32) for k in sizes]
    g0 = [rng.standard_normal(k).astype(np.float32) for k in sizes]
    p, g = [dev(a) for a in p0], [dev(a) for a in g0]
    bits = [8, 32, 8]
    z = lambda k, dt: torch.zeros(k, dtype=dt, device="cuda")      # noqa: E731
    m = [z(k, torch.int8 if b == 8 else torch.float32) for k, b in zip(sizes, bits)]
    v = [z(k, torch.uint8 if b == 8 else torch.float32) for k, b in zip(sizes, bits)]
    s = [z((-(-k // 256), 2), torch.float32) if b == 8 else None for k, b in zip(sizes, bits)]
    plist = B.ParamList(p, g, m, v, s, weight_decay=[0.1, 0.0, 0.0])
    out, state = z(2, torch.float32), z(B.ADAMW_STATE_BYTES // 8, torch.int64)
    lr = torch.tensor([0.02], device="cuda")
    B.grad_norm(plist, out, max_norm=2.0)
    B.adamw_step(plist, state, lr, factor=out[1:])
    torch.cuda.synchronize()
    norm, factor = train.grad_norm(g0, 1.0, 2.0)
    assert abs(float(out[0]) / norm - 1) <= 2 * U32 and factor < 1
    hyper = dict(HYPER, lr=0.02)
    for i, k in enumerate(sizes):
        rp, rm, rv = train.adamw(p0[i], g0[i], np.zeros(k), np.zeros(k), 1, weight_decay=[0.1, 0, 0][i],
                                 factor=float(out[1]), **hyper)
        _check_param(p0[i], _h(p[i]), rp, [0.1, 0, 0][i], hyper, "tensor %d" % i)
        if bits[i] == 8:
            qm, qv, _ = train.encode(rm, rv)
            assert np.array_equal(_h(m[i]), qm) and np.array_equal(_h(v[i]), qv)
    assert int(state[0]) == 1


@pytest.mark.parametrize("bits", [32, 8])
def test_graph_replays_count_steps(bits):
    """A captured clip and step: the count, the learning rate and the gradients are read on the device, so
    replays equal eager steps."""
    torch = torch_mod()
    rng = np.random.default_rng(21)
    sizes = [5000, 33, 300]
    p0 = [rng.standard_normal(k).astype(np.float32) for k in sizes]
    g0 = [[rng.standard_normal(k).astype(np.float32) for k in sizes] for _ in range(4)]

    def make():
        p, g = [dev(a) for a in p0], [torch.zeros(k, device="cuda") for k in sizes]
        lr = torch.tensor([0.1], device="cuda")
        return p, g, lr, B.AdamW(p, g, lr=lr, weight_decay=0.01, state_bits=bits)

    def fill(g, lr, t):
        for d, a in zip(g, g0[t]):
            d.copy_(torch.from_numpy(a))
        lr.fill_(0.1 / (t + 1))

    def step(opt, stream=None):
        opt.grad_norm(1.0, stream=stream)
        opt.step(factor=opt.factor, stream=stream)

    want, replayed, aside = make(), make(), make()
    note("adamw graph %d" % bits)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(replayed[3])
    side = torch.cuda.Stream()
    for t in range(4):
        for q in (want, replayed, aside):
            fill(q[1], q[2], t)
        torch.cuda.synchronize()
        step(want[3])
        graph.replay()
        step(aside[3], side)
        torch.cuda.synchronize()
        for other in (replayed, aside):
            assert all(torch.equal(a, b) for a, b in zip(want[0], other[0])), "parameters of step %d" % t
            for name in ("m", "v", "steps", "_out"):
                assert torch.equal(getattr(want[3], name), getattr(other[3], name)), name
    assert int(want[3].steps) == 4
