"""AdamW over the whole range of arguments that it accepts: eps down to
FLT_MIN, betas from 0 to the last number below 1, moments and gradients at
both ends of fp32.

Bounds (u = 2^-24, s = 2^-150, half of the least subnormal).  m takes two
products and a sum of rounded constants: 4 u of |b1 m| + |(1-b1) g| + 3 s.  v:
5 u + 3 s.  The update is compared with the formula at the moments that the
step left (32 bits: its own new m and v; 8 bits: the fp64 ones, rounded to
fp32 on the way, 2 u + s each before the quotient), so that what is checked is
the root and the quotient: lr / (1-b1^t) and 1 / sqrt(1-b2^t) take a logarithm
rounded to fp32, a product, an exponential of at most two units in the last
place and a division or a root and a reciprocal (8 u and 6 u), the root of v
and the reciprocal one unit each (4 u), three more roundings: 21 u, with the
rounded lr and eps 23 u; 24 u are allowed, and a rounding of the parameter."""
import numpy as np
import pytest

from oracle import train
from paper_2003_06513_amd import binding as B
from gpu_cases import U32, dev, note, torch_mod

pytestmark = pytest.mark.gpu
SUB = 2.0 ** -150
LEAST = float(np.finfo(np.float32).tiny)
LAST = 1.0 - 2.0 ** -24         # the last fp32 below 1


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    B.lib()


def _f(x):
    return float(np.float32(x))


def _update(m, v, t, lr, b1, b2, eps):
    """lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps) in fp64."""
    return _f(lr) * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + _f(eps))


def _near(p, want, update, what, more=0.0):
    bound = 24 * U32 * np.abs(update) + U32 * np.abs(want) + SUB + more
    err = np.abs(p - want)
    assert (err <= bound).all(), "%s: p off by %.3g bounds" % (what, (err / bound).max())


@pytest.mark.parametrize("eps", [LEAST, 1e-30, 1e-20, 1e-12, 1e-8])
@pytest.mark.parametrize("betas", [(0.9, 0.999), (0.0, 0.0), (0.0, 0.999), (0.5, 0.0), (0.99, LAST)])
@pytest.mark.parametrize("shift", [0, 1])
def test_small_second_moments(betas, eps, shift):
    """Second moments from 0 and the least subnormal up, with parameters of 0 whose whole value is the update."""
    torch = torch_mod()
    rng = np.random.default_rng(5)
    b1, b2 = (_f(b) for b in betas)
    n, t, lr = 5000, 7, 1e-3
    # the moment that a gradient's square leaves, or less, or nothing at all
    g = (10.0 ** rng.uniform(-23, -6, n) * rng.choice([-1.0, 1.0], n)).astype(np.float32)
    v0 = (g.astype(np.float64) ** 2 * 10.0 ** rng.uniform(-2, 2, n)).astype(np.float32)
    m0 = (np.sqrt(v0.astype(np.float64)) * rng.uniform(-1, 1, n)).astype(np.float32)
    v0[:64] = np.float32(2.0 ** -149) * np.arange(64)
    g[:128], m0[:128] = 0, 1e-25
    buf = torch.zeros(n + shift, device="cuda")
    p = buf[shift:]
    opt = B.AdamW([p], [dev(g)], lr=lr, betas=betas, eps=eps)
    opt.m[:n], opt.v[:n] = dev(m0), dev(v0)
    opt.steps.fill_(t - 1)
    note("small second moments, betas %s eps %g" % (betas, eps))
    opt.step()
    torch.cuda.synchronize()
    m, v, p = (x[:n].cpu().numpy().astype(np.float64) for x in (opt.m, opt.v, p))
    _, rm, rv = train.adamw(np.zeros(n), g, m0, v0, t, lr, b1, b2, eps, 0.0)
    g = np.abs(g.astype(np.float64))
    assert (np.abs(m - rm) <= 4 * U32 * (b1 * np.abs(m0) + (1 - b1) * g) + 3 * SUB).all()
    assert (np.abs(v - rv) <= 5 * U32 * rv + 3 * SUB).all()
    assert ((v > 0) & (v < LEAST)).any() or b2 == 0
    update = _update(m, v, t, lr, b1, b2, eps)
    _near(p, -update, update, "eps %g" % eps)
    assert int(opt.steps) == t


@pytest.mark.parametrize("eps", [LEAST, 1e-30, 1e-20, 1e-8])
@pytest.mark.parametrize("betas", [(0.9, 0.999), (0.0, 0.0), (0.0, 0.999), (0.5, 0.0), (0.99, LAST)])
def test_small_second_moments_of_8_bits(betas, eps):
    """Codes far below their group's largest stand for values that fp32 does not hold."""
    torch = torch_mod()
    rng = np.random.default_rng(6)
    b1, b2 = (_f(b) for b in betas)
    n, t, lr = 4096, 7, 1e-3
    scale = np.stack([10.0 ** rng.uniform(-20, -15, n // 256), 10.0 ** rng.uniform(-37, -30, n // 256)], 1)
    scale = scale.astype(np.float32)
    # gradients that leave the groups' scales where they are, or about there
    g = (10.0 ** rng.uniform(-26, -19, n) * rng.choice([-1.0, 1.0], n)).astype(np.float32)
    g[rng.random(n) < 0.3] = 0
    qm, qv = rng.integers(-127, 128, n).astype(np.int8), rng.integers(0, 256, n).astype(np.uint8)
    few = rng.random(n) < 0.5
    qv[few] = rng.integers(0, 4, int(few.sum()))
    qm[::256], qv[::256] = 127, 255
    p = torch.zeros(n, device="cuda")
    opt = B.AdamW([p], [dev(g)], lr=lr, betas=betas, eps=eps, state_bits=8)
    opt.m.copy_(dev(qm)), opt.v.copy_(dev(qv)), opt.scale.copy_(dev(scale))
    opt.steps.fill_(t - 1)
    note("small second moments of 8 bits, betas %s eps %g" % (betas, eps))
    opt.step()
    torch.cuda.synchronize()
    _, rm, rv = train.adamw(np.zeros(n), g, train.decode_m(qm, scale), train.decode_v(qv, scale), t, lr, b1, b2, eps, 0.0)
    update = _update(rm, rv, t, lr, b1, b2, eps)
    from_m = SUB * lr / (1 - b1 ** t) / (np.sqrt(rv / (1 - b2 ** t)) + _f(eps))
    _near(p.cpu().numpy().astype(np.float64), -update, update, "eps %g" % eps, 2 * U32 * np.abs(update) + from_m)
    assert ((rv > 0) & (rv < 2.0 ** -149)).any() or b2 == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_large_gradients(bits):
    """A gradient whose square passes fp32, while (1 - beta2) times it does not, is like any other."""
    torch = torch_mod()
    rng = np.random.default_rng(7)
    n, lr = 1500, 1e-2
    g = (10.0 ** rng.uniform(17, 20.6, n) * rng.choice([-1.0, 1.0], n)).astype(np.float32)
    p = torch.zeros(n, device="cuda")
    opt = B.AdamW([p], [dev(g)], lr=lr, state_bits=bits)
    note("large gradients, %d bits" % bits)
    opt.step()
    m, v = opt.moments()
    torch.cuda.synchronize()
    _, rm, rv = train.adamw(np.zeros(n), g, np.zeros(n), np.zeros(n), 1, lr, 0.9, 0.999, 1e-8, 0.0)
    update = _update(rm, rv, 1, lr, _f(0.9), _f(0.999), 1e-8)
    # at the formula's own moments: 4 u of m, half of 5 u of v
    _near(p.cpu().numpy().astype(np.float64), -update, update, "large", 7 * U32 * np.abs(update))
    if bits == 32:
        assert (np.abs(v[:n].cpu().numpy() - rv) <= 5 * U32 * rv).all()
    else:
        assert bool(torch.isfinite(v).all()) and bool(torch.isfinite(m).all())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_learning_rate_on_the_device_that_is_not_finite(bad, bits):
    """Nothing is changed and no step counted, as with a factor that is not finite."""
    torch = torch_mod()
    rng = np.random.default_rng(8)
    p, g = dev(rng.standard_normal(1000).astype(np.float32)), dev(rng.standard_normal(1000).astype(np.float32))
    copy = torch.zeros(1000, dtype=torch.float16, device="cuda")
    lr = torch.tensor([0.1], device="cuda")
    opt = B.AdamW([p], [g], lr=lr, state_bits=bits, copies=[copy], weight_decay=0.1)
    opt.step()
    held = [t.clone() for t in (p, opt.m, opt.v, copy, opt.steps)]
    lr.fill_(bad)
    note("learning rate %s" % bad)
    opt.step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, (p, opt.m, opt.v, copy, opt.steps)))
    none = B.ParamList([], [], [], [])
    B.adamw_step(none, opt._state, lr)
    torch.cuda.synchronize()
    assert int(opt.steps) == 1
    lr.fill_(0.1)
    opt.step()
    B.adamw_step(none, opt._state, lr)
    torch.cuda.synchronize()
    assert int(opt.steps) == 3 and bool(torch.isfinite(p).all()) and not torch.equal(p, held[0])


def test_current_stream_that_is_not_the_buffers_own():
    """Steps under another current stream, the optimiser dropped at once: its memory is not given out before they are
    done, and they are done right."""
    torch = torch_mod()
    rng = np.random.default_rng(9)
    p0, g0 = rng.standard_normal(300_000).astype(np.float32), rng.standard_normal(300_000).astype(np.float32)
    want, p, g = dev(p0), dev(p0), dev(g0)
    B.AdamW([want], [g], lr=0.1).step()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    note("step on another current stream")
    opt = B.AdamW([p], [g], lr=0.1)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            opt.grad_norm(1.0)
        opt.step()
    del opt
    others = [torch.full((300_000,), 7.0, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(p, want) and all(bool((t == 7).all()) for t in others)


def _codes_of_whole_numbers(x, peak, top, power):
    """How many borders (k - 1/2)^power, k = 1 .. top, lie at or below x top^power / peak, in whole numbers."""
    borders = (2 * np.arange(1, top + 1) - 1) ** power * peak
    return np.searchsorted(borders, x * (2 * top) ** power, side="right")


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("unit", [1.0, 2.0 ** -7, 2.0 ** 5])
def test_codes_of_values_on_borders(unit, half):
    """Whole gradients and betas of 0: m and v are they and their squares, and many lie on a border between two codes
    (1/4 of the largest m; 1/16, 1/1296 or 1/10000 of the largest v), where the code is the upper one."""
    torch = torch_mod()
    peaks = np.concatenate([np.arange(4, 1204, 4), [100 * k for k in range(1, 13)], [36 * k for k in range(1, 30)]])
    g = np.stack([np.linspace(0, k, 256).astype(np.int64) for k in peaks])
    g[:, 1], g[:, 2], g[:, 3] = peaks // 4, peaks // 10, peaks // 6
    sign = np.where(np.arange(g.size) % 3 == 1, -1, 1)
    p = torch.zeros(g.size, device="cuda")
    grad = dev((unit * sign * g.reshape(-1)).astype(np.float16 if half else np.float32))
    opt = B.AdamW([p], [grad], betas=(0.0, 0.0), state_bits=8)
    note("codes on borders, unit %g" % unit)
    opt.step()
    torch.cuda.synchronize()
    m = np.stack([_codes_of_whole_numbers(r, k, 127, 2) for r, k in zip(g, peaks)])
    v = np.stack([np.maximum(_codes_of_whole_numbers(r * r, k * k, 255, 4), r > 0) for r, k in zip(g, peaks)])
    assert np.array_equal(opt.m.cpu().numpy(), sign * m.reshape(-1))
    assert np.array_equal(opt.v.cpu().numpy(), v.reshape(-1))
    assert (4 * g == peaks[:, None]).sum() >= 300 and (10 * g == peaks[:, None]).sum() > 10 and \
        (6 * g == peaks[:, None]).sum() > 10
