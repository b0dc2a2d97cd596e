"""Group normalisation with an activation, forward and backward, against the
fp64 oracle.

Bounds (u = 2^-24; every output element by element).  No thread of the kernels
adds more than M/64 + 64 values of a sum of M in a row before the partial sums
meet in trees, so a sum is off by at most k u times the sum of magnitudes with
k = M/64 + 64 (the classical bound; the trees' few levels are in the 64).
With e_mu = k u mean|x|, relative errors of rstd k u + (rstd e_mu)^2 and a few
roundings, the forward's u is off by
    e_u = |gamma| (rstd e_mu + |xhat| ((k + 8) u + (rstd e_mu)^2)) + 3 u (|gamma xhat| + |beta|)
and y by at most 1.1 e_u (the SiLU's slope) + (|u| + 8) u |y| (its sigmoid:
an exponential whose argument is rounded) + one rounding to the type.  The
backward has its own sums, bounded the same way, below."""
import numpy as np
import pytest

from oracle import train
from paper_2003_06513_amd import binding as B
from gpu_cases import U16, U32, dev, note, torch_mod

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    B.lib()


def _data(shape, dtype, seed):
    n, c, h, w = shape
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * (0.5 + rng.random((1, c, 1, 1))) + rng.standard_normal((1, c, 1, 1))
    return (x.astype(dtype), (0.1 * rng.standard_normal(shape)).astype(dtype),
            (1 + 0.3 * rng.standard_normal(c)).astype(np.float32), (0.3 * rng.standard_normal(c)).astype(np.float32))


def _place(a, layout, shift=0):
    """The array on the device in a layout, ``shift`` elements into an
    allocation that ends with it, guard elements on both sides."""
    torch = torch_mod()
    n, c, h, w = a.shape
    buf = torch.full((a.size + shift + 64,), 77.0, dtype=torch.float16 if a.dtype == np.float16 else torch.float32,
                     device="cuda")
    flat = buf[shift:shift + a.size]
    t = flat.view(n, h, w, c).permute(0, 3, 1, 2) if layout == "nhwc" else flat.view(n, c, h, w)
    t.copy_(torch.from_numpy(a))
    return t, buf


def _guards_hold(t, buf, shift):
    size = t.numel()
    assert bool((buf[:shift] == 77).all()) and bool((buf[shift + size:] == 77).all()), "written outside the tensor"


def _group(t, groups):
    n, c, h, w = t.shape
    return np.asarray(t, dtype=np.float64).reshape(n, groups, c // groups, h * w)


def _bounds(x, groups, gamma, beta, mean, rstd):
    n, c, h, w = x.shape
    m = (c // groups) * h * w
    k = m / 64 + 64
    ga = np.abs(np.asarray(gamma, dtype=np.float64)).reshape(1, groups, -1, 1)
    be = np.abs(np.asarray(beta, dtype=np.float64)).reshape(1, groups, -1, 1)
    xg = _group(x, groups)
    r = np.asarray(rstd, dtype=np.float64)[:, :, None, None]
    e_mu = k * U32 * np.abs(xg).mean(axis=(2, 3), keepdims=True) + U32 * np.abs(mean)[:, :, None, None]
    xh = np.abs(xg - mean[:, :, None, None]) * r
    return k, ga, be, r, e_mu, xh


def _round_off(y, dtype):
    return np.abs(y) * U16 + 2.0 ** -25 if dtype == np.float16 else np.abs(y) * U32 + 1e-38


def check_forward(x, groups, gamma, beta, act, y, mean, rstd, what, eps=EPS):
    ry, rmean, rrstd = train.group_norm(x, groups, gamma, beta, eps, act)
    k, ga, be, r, e_mu, xh = _bounds(x, groups, gamma, beta, rmean, rrstd)
    rel = (k + 8) * U32 + (r * e_mu) ** 2
    e_u = ga * (r * e_mu + xh * rel) + 3 * U32 * (ga * xh + be)
    yg = np.abs(_group(ry, groups))
    bound = 1.1 * e_u + (8 + ga * xh + be) * U32 * yg
    bound = bound.reshape(x.shape) * (1 + U16) + _round_off(ry, x.dtype.type)
    err = np.abs(y.astype(np.float64) - ry)
    assert (err <= bound).all(), "%s: y off by %.3g bounds" % (what, (err / bound).max())
    if mean is not None:
        assert (np.abs(mean - rmean) <= e_mu[:, :, 0, 0]).all(), what + " mean"
        assert (np.abs(rstd - rrstd) <= rrstd * rel[:, :, 0, 0]).all(), what + " rstd"


def check_backward(x, dy, groups, gamma, beta, mean, rstd, act, dx, dgamma, dbeta, what):
    n, c, h, w = x.shape
    rdx, rdg, rdb = train.group_norm_back(x, dy, groups, gamma, beta, mean, rstd, act)
    m = (c // groups) * h * w
    ga = np.abs(gamma.astype(np.float64)).reshape(1, groups, -1, 1)
    be = np.abs(beta.astype(np.float64)).reshape(1, groups, -1, 1)
    r = rstd.astype(np.float64)[:, :, None, None]
    xh = np.abs(_group(x, groups) - mean.astype(np.float64)[:, :, None, None]) * r
    u = ga * xh + be
    g = np.abs(_group(dy, groups))
    # du = dy act'(u); |act'| <= 1.1, |act''| <= 0.5 for the SiLU; u off by 6 roundings of its terms
    du = 1.1 * g
    e_du = g * (0.5 * 6 * U32 * u + 8 * U32 * (2 + u)) if act == "silu" else 0 * g
    # of a channel's sums over h w (k additions in a row), and over the images (n more)
    k = h * w / 64 + 64
    e_a = (k * U32 * du + e_du).sum(axis=3, keepdims=True)
    e_b = ((k + 4) * U32 * du * xh + e_du * xh).sum(axis=3, keepdims=True)
    terms = lambda t: t.sum(axis=(0, 3)).reshape(c)        # noqa: E731
    bound = terms(e_a) + n * U32 * terms(du)
    assert (np.abs(dbeta - rdb) <= bound + 1e-38).all(), what + " dbeta"
    bound = terms(e_b) + n * U32 * terms(du * xh)
    assert (np.abs(dgamma - rdg) <= bound + 1e-38).all(), what + " dgamma"
    kc = c // groups / 64 + 64
    s1, s2 = ((ga * t).sum(axis=(2, 3), keepdims=True) / m for t in (du, du * xh))
    e1 = (ga * e_a).sum(axis=2, keepdims=True) / m + (kc + 4) * U32 * s1
    e2 = (ga * e_b).sum(axis=2, keepdims=True) / m + (kc + 4) * U32 * s2
    bound = r * (ga * e_du + e1 + xh * e2 + 8 * U32 * (ga * du + s1 + xh * s2))
    bound = bound.reshape(x.shape) * (1 + U16) + _round_off(rdx, x.dtype.type)
    err = np.abs(dx.astype(np.float64) - rdx)
    assert (err <= bound).all(), "%s: dx off by %.3g bounds" % (what, (err / bound).max())


SHAPES = [
    # (n, c, h, w), groups
    ((1, 1, 1, 1), 1),                  # one value: its group has no spread
    ((2, 6, 1, 1), 3), ((5, 4, 1, 1), 4),
    ((3, 8, 1, 3), 1), ((2, 12, 5, 7), 3),
    ((2, 93, 9, 11), 31),               # nothing a multiple of anything
    ((2, 64, 14, 14), 32),              # two channels a group
    ((3, 40, 7, 7), 8), ((2, 512, 7, 7), 32),
    ((2, 24, 3, 130), 2), ((1, 7, 33, 65), 7),
    ((300, 16, 4, 4), 4),               # many images
    ((1, 2048, 2, 2), 8), ((1, 1500, 1, 1), 1), ((2, 4100, 1, 2), 2),     # many channels a group
    ((2, 32, 64, 64), 1),               # one large group an image
    ((1, 16, 112, 112), 4), ((1, 8, 224, 224), 4), ((2, 6, 181, 193), 2),   # large planes
    ((3, 128, 28, 28), 32), ((40, 64, 16, 16), 32), ((2, 256, 56, 56), 32),
    ((9, 512, 14, 14), 32), ((20, 96, 40, 40), 24), ((40, 64, 40, 40), 32),     # between one and a few blocks a CU
    ((16, 32, 20, 20), 8), ((24, 48, 9, 10), 4),                                # whole images on a die
    ((4, 771, 12, 12), 1), ((3, 778, 11, 11), 2), ((2, 512, 14, 14), 1),        # many short rows of a group
]


@pytest.mark.parametrize("dtype", [np.float32, np.float16])
@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("shape,groups", SHAPES)
def test_forward_and_backward(shape, groups, layout, dtype):
    torch = torch_mod()
    n, c, h, w = shape
    for i, act in enumerate(("none", "relu", "silu")):
        if act == "none" and n * c * h * w > 300_000:
            continue
        # elements into the allocation: aligned for wide accesses, or for single elements only; input and output
        # not always alike
        sx, sy = ((0, 0), (1, 1), (16, 3))[i]
        x, dy, gamma, beta = _data(shape, dtype, 17 * c + h + i)
        note("group norm %s G=%d %s %s %s" % (shape, groups, layout, np.dtype(dtype).name, act))
        (tx, _), (ty, by) = _place(x, layout, sx), _place(np.zeros_like(x), layout, sy)
        mean, rstd = (torch.full((n, groups), 7.0, device="cuda") for _ in range(2))
        B.group_norm_fwd(tx, groups, dev(gamma), dev(beta), ty, eps=EPS, act=act, mean=mean, rstd=rstd)
        torch.cuda.synchronize()
        _guards_hold(ty, by, sy)
        hm, hr = mean.cpu().numpy(), rstd.cpu().numpy()
        what = "%s G=%d %s %s" % (shape, groups, layout, act)
        check_forward(x, groups, gamma, beta, act, ty.cpu().numpy(), hm, hr, what)
        (tdy, _), (tdx, bx) = _place(dy, layout, sx), _place(np.zeros_like(x), layout, sy)
        dgamma, dbeta = (torch.full((c,), 7.0, device="cuda") for _ in range(2))
        run = lambda: B.group_norm_bwd(tx, tdy, groups, dev(gamma), dev(beta), mean, rstd, tdx, dgamma, dbeta,   # noqa: E731
                                       act=act)
        run()
        torch.cuda.synchronize()
        _guards_hold(tdx, bx, sy)
        check_backward(x, dy, groups, gamma, beta, hm, hr, act, tdx.cpu().numpy(), dgamma.cpu().numpy(),
                       dbeta.cpu().numpy(), what)
        first = [t.clone() for t in (tdx, dgamma, dbeta)]
        run()
        assert all(torch.equal(a, b) for a, b in zip(first, (tdx, dgamma, dbeta))), what + ": another result"


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("shape,groups", [((2, 8, 6, 6), 2), ((1, 4, 120, 150), 2), ((2, 32, 64, 64), 1)])
def test_without_what_is_optional(shape, groups, layout):
    """gamma, beta, the statistics and the parameters' gradients may be left out."""
    torch = torch_mod()
    x, dy, _, _ = _data(shape, np.float32, 9)
    tx, _ = _place(x, layout)
    ty, tdx, tdx2 = (_place(np.zeros_like(x), layout)[0] for _ in range(3))
    tdy, _ = _place(dy, layout)
    one, zero = np.ones(shape[1], np.float32), np.zeros(shape[1], np.float32)
    note("group norm without parameters %s %s" % (shape, layout))
    B.group_norm_fwd(tx, groups, None, None, ty)
    mean, rstd = (torch.empty((shape[0], groups), device="cuda") for _ in range(2))
    ty2 = torch.empty_like(ty)
    B.group_norm_fwd(tx, groups, dev(one), None, ty2, mean=mean, rstd=rstd)
    B.group_norm_bwd(tx, tdy, groups, None, None, mean, rstd, tdx)
    dbeta, dgamma = (torch.empty(shape[1], device="cuda") for _ in range(2))
    B.group_norm_bwd(tx, tdy, groups, None, dev(zero), mean, rstd, tdx2, dbeta=dbeta)
    torch.cuda.synchronize()
    assert torch.equal(ty, ty2) and torch.equal(tdx, tdx2)
    B.group_norm_bwd(tx, tdy, groups, None, dev(zero), mean, rstd, tdx2, dgamma=dgamma)
    check_forward(x, groups, one, zero, "none", ty.cpu().numpy(), None, None, "plain")
    check_backward(x, dy, groups, one, zero, mean.cpu().numpy(), rstd.cpu().numpy(), "none", tdx.cpu().numpy(),
                   dgamma.cpu().numpy(), dbeta.cpu().numpy(), "plain")


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("shape,groups", [((2, 8, 6, 6), 2), ((1, 4, 130, 140), 1), ((64, 64, 16, 16), 8)])
def test_level_far_from_zero(shape, groups, layout):
    """A mean of a thousand spreads: the variance is taken about the mean."""
    torch = torch_mod()
    x, _, gamma, beta = _data(shape, np.float32, 31)
    x = (x + 1000).astype(np.float32)
    tx, _ = _place(x, layout)
    ty = torch.empty_like(tx)
    mean, rstd = (torch.empty((shape[0], groups), device="cuda") for _ in range(2))
    note("group norm far from zero %s %s" % (shape, layout))
    B.group_norm_fwd(tx, groups, dev(gamma), dev(beta), ty, mean=mean, rstd=rstd)
    torch.cuda.synchronize()
    check_forward(x, groups, gamma, beta, "none", ty.cpu().numpy(), mean.cpu().numpy(), rstd.cpu().numpy(), "far")
    # the bound above allows an error of the mean; that of the spread has to stay far below one
    assert np.abs(rstd.cpu().numpy() / train.statistics(x, groups, EPS)[1] - 1).max() < 1e-4


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("shape,groups", [((2, 8, 6, 6), 2), ((2, 8, 130, 140), 2)])
def test_not_finite_and_constant_groups(shape, groups, layout):
    torch = torch_mod()
    x, dy, gamma, beta = _data(shape, np.float16, 33)
    x[0, 1, 2, 3], x[1, 6, 0, 1] = np.nan, np.inf      # groups (0, 0) and (1, 1)
    x[1, :4] = 2.5                                     # group (1, 0): no spread
    tx, _ = _place(x, layout)
    ty = torch.empty_like(tx)
    mean, rstd = (torch.empty((2, 2), device="cuda") for _ in range(2))
    note("group norm with values that are not finite %s %s" % (shape, layout))
    B.group_norm_fwd(tx, 2, dev(gamma), dev(beta), ty, act="relu", mean=mean, rstd=rstd)
    tdy, _ = _place(dy, layout)
    tdx = torch.empty_like(tx)
    B.group_norm_bwd(tx, tdy, 2, dev(gamma), dev(beta), mean, rstd, tdx, act="relu")
    torch.cuda.synchronize()
    y, dx = ty.cpu().numpy(), tdx.cpu().numpy()
    for img, ch in ((0, slice(0, 4)), (1, slice(4, 8))):
        assert np.isnan(y[img, ch]).all() and np.isnan(dx[img, ch]).all()
    ok_x = x.copy()
    ok_x[0, :4], ok_x[1, 4:] = 0, 0
    hm, hr = mean.cpu().numpy(), rstd.cpu().numpy()
    for img, g in ((0, 1), (1, 0)):
        ch = slice(4 * g, 4 * g + 4)
        one = (slice(img, img + 1), ch)
        check_forward(x[one], 1, gamma[ch], beta[ch], "relu", y[one], hm[img:img + 1, g:g + 1], hr[img:img + 1, g:g + 1],
                      "beside a group that is not finite")
        assert np.isfinite(dx[one]).all()
    assert abs(hr[1, 0] * np.sqrt(EPS) - 1) < 1e-6


def test_no_images():
    torch = torch_mod()
    x = torch.empty((0, 6, 4, 4), device="cuda")
    dgamma, dbeta = (torch.full((6,), 7.0, device="cuda") for _ in range(2))
    stats = torch.empty((0, 3), device="cuda")
    B.group_norm_fwd(x, 3, None, None, torch.empty_like(x), mean=stats, rstd=stats.clone())
    B.group_norm_bwd(x, x, 3, None, None, stats, stats, torch.empty_like(x), dgamma, dbeta)
    torch.cuda.synchronize()
    assert not dgamma.any() and not dbeta.any()


@pytest.mark.parametrize("shape,groups", [((2, 64, 14, 14), 32), ((1, 8, 150, 160), 2)])
@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
def test_graph_and_other_stream(shape, groups, layout):
    """Replays between eager calls on other data, and calls on a side stream."""
    torch = torch_mod()
    x, dy, gamma, beta = _data(shape, np.float16, 41)
    tx, tdy = _place(x, layout)[0], _place(dy, layout)[0]
    ga, be = dev(gamma), dev(beta)
    out = lambda: dict(y=torch.zeros_like(tx), dx=torch.zeros_like(tx), mean=torch.zeros(shape[0], groups, device="cuda"),   # noqa: E731
                       rstd=torch.zeros(shape[0], groups, device="cuda"), dg=torch.zeros_like(ga), db=torch.zeros_like(ga))

    def step(x, o, stream=None):
        B.group_norm_fwd(x, groups, ga, be, o["y"], act="silu", mean=o["mean"], rstd=o["rstd"], stream=stream)
        B.group_norm_bwd(x, tdy, groups, ga, be, o["mean"], o["rstd"], o["dx"], o["dg"], o["db"], act="silu",
                         stream=stream)

    want, got, other = out(), out(), out()
    note("group norm graph %s %s" % (shape, layout))
    step(tx, want)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(tx, got)
    for _ in range(3):
        for t in got.values():
            t.fill_(9)
        step(2 * tx, other)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], want[k]) for k in want)
    side = torch.cuda.Stream()
    for t in got.values():
        t.fill_(9)
    torch.cuda.synchronize()
    for _ in range(5):
        step(tx, got, side)
        step(2 * tx, other)
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
def test_more_groups_than_a_launch_has_threads(layout):
    """134 million groups of one value each: y = act(beta), dx = 0, dbeta = the sums of dy."""
    torch = torch_mod()
    n, c = 65535, 2048
    fmt = torch.channels_last if layout == "nhwc" else torch.contiguous_format
    note("group norm, 2^27 groups, %s" % layout)
    x = torch.ones((n, c, 1, 2), dtype=torch.float16, device="cuda")[:, :, :, :1].contiguous(memory_format=fmt)
    if layout == "nhwc":        # one pixel is in both layouts: two of them are not, with two values a group
        x = torch.ones((n // 2, c, 1, 2), dtype=torch.float16, device="cuda").contiguous(memory_format=fmt)
    n = x.shape[0]
    y, beta = torch.zeros_like(x), torch.linspace(-1, 1, c, device="cuda")
    mean, rstd = (torch.empty((n, c), device="cuda") for _ in range(2))
    B.group_norm_fwd(x, c, None, beta, y, act="relu", mean=mean, rstd=rstd)
    torch.cuda.synchronize()
    want = beta.clamp(min=0).half().view(1, c, 1, 1)
    assert bool((y == want).all()) and bool((mean == 1).all())
    del mean
    mean = torch.ones((n, c), device="cuda")
    dgamma, dbeta = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    B.group_norm_bwd(x, x, c, None, beta, mean, rstd, y, dgamma, dbeta)
    torch.cuda.synchronize()
    assert not y.any() and not dgamma.any()
    assert bool((dbeta == n * x.shape[3]).all())


@pytest.mark.parametrize("shift", [0, 1])
def test_row_of_four_gigabytes(shift):
    """A channel of 2^30 values: offsets beyond 32 bits, aligned for wide accesses and not."""
    torch = torch_mod()
    side = 32768
    buf = torch.empty(side * side + shift, device="cuda")
    x = buf[shift:].view(1, 1, side, side)
    x.normal_(3.0, 2.0)
    out = torch.empty(side * side + shift, device="cuda")
    y = out[shift:].view(1, 1, side, side)
    mean, rstd = (torch.empty((1, 1), device="cuda") for _ in range(2))
    note("group norm, 2^30 values, shift %d" % shift)
    B.group_norm_fwd(x, 1, None, None, y, act="silu", mean=mean, rstd=rstd)
    torch.cuda.synchronize()
    rows = x.view(64, -1)
    mu = sum(float(r.double().sum()) for r in rows) / x.numel()
    var = sum(float((r.double() - mu).square().sum()) for r in rows) / x.numel()
    # sums of 2^30 values by 2^20 partial ones: their roundings average out far below these
    assert abs(float(mean) - mu) < 1e-5 and abs(float(rstd) * np.sqrt(var + 1e-5) - 1) < 1e-5
    for r, o in zip(rows, y.view(64, -1)):
        u = (r - mean.view(())) * rstd.view(())
        assert float((o - u * torch.sigmoid(u)).abs().max()) < 1e-5
    dx = torch.empty_like(out)[shift:].view(1, 1, side, side)
    dbeta = torch.empty(1, device="cuda")
    B.group_norm_bwd(x, y, 1, None, None, mean, rstd, dx, dbeta=dbeta)
    torch.cuda.synchronize()
    s1 = sum(float(o.double().sum()) for o in y.view(64, -1))
    s2 = sum(float((o.double() * ((r - mean.view(())) * rstd.view(())).double()).sum())
             for r, o in zip(rows, y.view(64, -1)))
    assert abs(float(dbeta) / s1 - 1) < 1e-5
    for r, o, d in zip(rows, y.view(64, -1), dx.view(64, -1)):
        u = (r - mean.view(())) * rstd.view(())
        want = rstd.view(()) * (o - s1 / x.numel() - u * (s2 / x.numel()))
        assert float((d - want).abs().max()) < 1e-5
