"""Group normalisation: what the first file's sweep over shapes leaves out."""
import numpy as np
import pytest

from oracle import train
from paper_2003_06513_amd import binding as B
from gpu_cases import U32, dev, note, torch_mod
from test_gpu_group_norm import (EPS, _data, _guards_hold, _need_gpu, _place, check_backward,        # noqa: F401
                                 check_forward)

pytestmark = pytest.mark.gpu


# held, joined and combined sums of both layouts
@pytest.mark.parametrize("dtype", [np.float32, np.float16])
@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("shape", [(2, 8, 6, 6), (2, 8, 130, 140), (1, 64, 300, 300)])
def test_statistics_of_groups_that_are_not_finite(shape, layout, dtype):
    """One infinity, infinities of one sign or of both, a NaN, values whose squares or whose sum pass fp32: mean and
    rstd are NaN, and nothing else is."""
    torch = torch_mod()
    n, c, h, w = shape
    for case, put in enumerate(((np.inf,), (-np.inf, -np.inf), (np.inf, -np.inf), (np.nan,), (1e25,), (3e38, 3e38))):
        if dtype == np.float16 and np.isfinite(put[0]):
            continue
        x, dy, gamma, beta = _data(shape, dtype, 35)
        for i, value in enumerate(put):
            x[0, 0, i, h - 1 - i] = value
        for groups in (1, 2):
            tx, _ = _place(x, layout)
            ty, tdx = torch.empty_like(tx), torch.empty_like(tx)
            mean, rstd = (torch.zeros((n, groups), device="cuda") for _ in range(2))
            note("statistics of a group that is not finite %s %s %s G=%d" % (shape, layout, put, groups))
            B.group_norm_fwd(tx, groups, dev(gamma), dev(beta), ty, mean=mean, rstd=rstd)
            B.group_norm_bwd(tx, _place(dy, layout)[0], groups, dev(gamma), dev(beta), mean, rstd, tdx)
            torch.cuda.synchronize()
            want = torch.zeros((n, groups), dtype=torch.bool, device="cuda")
            want[0, 0] = True
            assert torch.equal(torch.isnan(mean), want) and torch.equal(torch.isnan(rstd), want), (case, groups)
            assert bool(torch.isfinite(mean[~want]).all()) and bool(torch.isfinite(rstd[~want]).all())
            for t in (ty, tdx):
                spoilt = torch.isnan(t).view(n, groups, -1) if layout == "nchw" else \
                    torch.isnan(t).contiguous().view(n, groups, -1)
                assert torch.equal(spoilt.all(2), want) and torch.equal(spoilt.any(2), want)


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("shape,groups", [((2, 8, 6, 6), 2), ((1, 4, 120, 150), 2), ((1, 64, 300, 300), 1)])
def test_least_eps(shape, groups, layout):
    """FLT_MIN, and spreads whose squares lie about it: a square is off by 2^-150, which is 2^-24 of eps."""
    torch = torch_mod()
    least = float(np.finfo(np.float32).tiny)
    for spread in (1e-22, 1e-20, 1e-19, 1e-17):
        x, _, gamma, beta = _data(shape, np.float64, 37)
        x = (spread * (x - x.mean(axis=(2, 3), keepdims=True))).astype(np.float32)
        gamma, beta = gamma.astype(np.float32), beta.astype(np.float32)
        tx, _ = _place(x, layout)
        ty = torch.empty_like(tx)
        mean, rstd = (torch.empty((shape[0], groups), device="cuda") for _ in range(2))
        note("group norm, eps %g, spread %g %s %s" % (least, spread, shape, layout))
        B.group_norm_fwd(tx, groups, dev(gamma), dev(beta), ty, eps=least, mean=mean, rstd=rstd)
        torch.cuda.synchronize()
        check_forward(x, groups, gamma, beta, "none", ty.cpu().numpy(), mean.cpu().numpy(), rstd.cpu().numpy(),
                      "spread %g" % spread, eps=least)


# A shape for every compiled form that a call can take: whole groups in a block's registers or pieces that the writers
# or a launch of its own join, each count of vectors per thread, 16-byte vectors, vectors with windows or single
# elements, and what goes past the caches.
FORMS = [
    # NCHW, fp32: (n, c, h, w), groups, elements into the allocation
    *[("nchw", np.float32) + t for t in (((2, 4, 1, 1), 2, 0), ((2, 4, 1, 4), 2, 0), ((2, 527, 2, 7), 1, 0),
        ((2, 604, 5, 3), 2, 0), ((2, 261, 6, 6), 1, 0), ((2, 78, 12, 12), 2, 0), ((2, 148, 12, 12), 2, 0),
        ((2, 863, 10, 3), 1, 0), ((2, 17, 40, 40), 1, 0), ((2, 426, 2, 34), 1, 0), ((2, 151, 14, 14), 1, 0),
        ((2, 53, 113, 5), 1, 0), ((2, 53, 24, 24), 1, 0), ((2, 101, 18, 18), 1, 0), ((2, 272, 30, 7), 2, 0),
        ((2, 359, 20, 13), 1, 0), ((2, 307, 25, 25), 1, 0), ((2, 281, 33, 33), 1, 0), ((2, 149, 8, 314), 1, 0),
        ((2, 628, 302, 2), 2, 0), ((40, 897, 6, 6), 13, 0), ((2, 130, 8, 8), 1, 1), ((2, 97, 16, 16), 1, 1),
        ((2, 17, 40, 40), 1, 1), ((2, 267, 16, 16), 1, 1), ((40, 897, 6, 6), 13, 1))],
    # NCHW, fp16: (n, c, h, w), groups, elements into the allocation
    *[("nchw", np.float16) + t for t in (((2, 4, 1, 1), 2, 0), ((2, 4, 1, 8), 2, 0), ((2, 269, 2, 13), 1, 0),
        ((2, 9, 54, 38), 1, 0), ((2, 36, 23, 23), 1, 0), ((2, 709, 9, 3), 1, 0), ((2, 133, 12, 12), 1, 0),
        ((2, 148, 12, 12), 2, 0), ((2, 23, 138, 8), 1, 0), ((2, 65, 28, 28), 1, 0), ((2, 524, 10, 10), 1, 0),
        ((1, 266, 20, 20), 2, 0), ((2, 17, 56, 56), 1, 0), ((2, 184, 18, 18), 1, 0), ((2, 55, 220, 5), 1, 0),
        ((2, 33, 44, 44), 1, 0), ((2, 571, 16, 7), 1, 0), ((2, 307, 25, 25), 1, 0), ((3, 267, 24, 24), 1, 0),
        ((2, 281, 33, 33), 1, 0), ((2, 286, 40, 40), 1, 0), ((2, 136, 334, 13), 1, 0), ((2, 139, 278, 16), 1, 0),
        ((11, 235, 13, 80), 47, 0), ((2, 67, 16, 16), 1, 1), ((2, 34, 32, 32), 2, 1), ((2, 65, 28, 28), 1, 1),
        ((2, 17, 56, 56), 1, 1), ((11, 235, 13, 80), 47, 1))],
    # channels last, fp32: (n, c, h, w), groups, elements into the allocation
    *[("nhwc", np.float32) + t for t in (((2, 4, 1, 2), 2, 0), ((2, 32, 1, 2), 2, 0), ((2, 52, 1, 2), 2, 0),
        ((2, 515, 3, 3), 1, 0), ((2, 36, 1, 148), 2, 0), ((2, 20, 17, 17), 4, 0), ((2, 12, 23, 23), 4, 0),
        ((2, 12, 117, 9), 4, 0), ((2, 6, 48, 48), 2, 0), ((2, 180, 9, 9), 2, 0), ((2, 44, 2, 184), 4, 0),
        ((2, 148, 12, 12), 2, 0), ((2, 28, 33, 33), 4, 0), ((2, 4, 91, 91), 2, 0), ((2, 24, 81, 296), 12, 0),
        ((18, 528, 12, 12), 44, 0), ((52, 40, 132, 8), 20, 0), ((49, 140, 18, 18), 28, 0),
        ((2, 12, 320, 320), 4, 0), ((2, 4, 1, 2), 2, 1), ((2, 4, 70, 30), 2, 1))],
    # channels last, fp16: (n, c, h, w), groups, elements into the allocation
    *[("nhwc", np.float16) + t for t in (((2, 4, 1, 2), 2, 0), ((2, 6, 1, 2), 2, 0), ((2, 8, 1, 2), 2, 0),
        ((2, 64, 1, 2), 2, 0), ((2, 128, 1, 2), 2, 0), ((2, 515, 3, 3), 1, 0), ((2, 9, 27, 27), 3, 0),
        ((2, 9, 34, 34), 3, 0), ((2, 12, 117, 9), 4, 0), ((2, 56, 67, 4), 1, 0), ((2, 8, 10, 210), 2, 0),
        ((2, 552, 6, 6), 4, 0), ((2, 8, 138, 30), 4, 0), ((2, 64, 262, 2), 1, 0), ((2, 136, 19, 19), 8, 0),
        ((2, 56, 33, 33), 2, 0), ((2, 8, 75, 110), 2, 0), ((2, 36, 114, 132), 2, 0), ((2, 24, 240, 240), 8, 0),
        ((100, 156, 31, 6), 13, 0), ((51, 216, 2, 141), 24, 0), ((18, 348, 11, 47), 116, 0),
        ((109, 760, 5, 8), 20, 0))],
]


@pytest.mark.parametrize("layout,dtype,shape,groups,shift", FORMS)
def test_every_form(layout, dtype, shape, groups, shift):
    torch = torch_mod()
    n, c, h, w = shape
    # the largest with one activation each: the oracle takes a second for them
    acts = ("none", "relu", "silu") if n * c * h * w < 500_000 else (("relu", "silu")[(c + h) % 2],)
    for act in acts:
        x, dy, gamma, beta = _data(shape, dtype, 3 * c + h)
        what = "%s G=%d %s %s %s +%d" % (shape, groups, layout, np.dtype(dtype).name, act, shift)
        note("group norm form " + what)
        (tx, _), (ty, by) = _place(x, layout, shift), _place(np.zeros_like(x), layout, shift)
        mean, rstd = (torch.full((n, groups), 7.0, device="cuda") for _ in range(2))
        B.group_norm_fwd(tx, groups, dev(gamma), dev(beta), ty, eps=EPS, act=act, mean=mean, rstd=rstd)
        torch.cuda.synchronize()
        _guards_hold(ty, by, shift)
        hm, hr = mean.cpu().numpy(), rstd.cpu().numpy()
        check_forward(x, groups, gamma, beta, act, ty.cpu().numpy(), hm, hr, what)
        (tdy, _), (tdx, bx) = _place(dy, layout, shift), _place(np.zeros_like(x), layout, shift)
        dgamma, dbeta = (torch.full((c,), 7.0, device="cuda") for _ in range(2))
        B.group_norm_bwd(tx, tdy, groups, dev(gamma), dev(beta), mean, rstd, tdx, dgamma, dbeta, act=act)
        torch.cuda.synchronize()
        _guards_hold(tdx, bx, shift)
        check_backward(x, dy, groups, gamma, beta, hm, hr, act, tdx.cpu().numpy(), dgamma.cpu().numpy(),
                       dbeta.cpu().numpy(), what)


# In pieces: joined by those who write them, or by a launch of its own; single elements (shift 1 of one tensor alone).
@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("shape,groups,shift", [((2, 32, 64, 64), 1, 0), ((1, 64, 300, 300), 1, 0), ((1, 4, 120, 150), 2, 0),
                                                ((30, 64, 9, 9), 32, 1), ((3, 24, 50, 50), 2, 1)])
def test_spread_far_from_zero(shape, groups, shift, layout):
    """Levels of up to 10^4 spreads, and channels that differ: rstd is off by the square of the mean's error (in spreads)
    and the roundings of sums of at most 64 values a lane, 64 a lane of the join and the trees: 160 u."""
    torch = torch_mod()
    for level in (0, 30, 100, 1000, 10000):
        x, _, _, _ = _data(shape, np.float32, 39)
        x = (x + np.float32(level)).astype(np.float32)
        (tx, _), (ty, _) = _place(x, layout), _place(np.zeros_like(x), layout, shift)
        mean, rstd = (torch.empty((shape[0], groups), device="cuda") for _ in range(2))
        note("spread far from zero %s %s level %g" % (shape, layout, level))
        B.group_norm_fwd(tx, groups, None, None, ty, mean=mean, rstd=rstd)
        torch.cuda.synchronize()
        rmean, rrstd = train.statistics(x, groups, 1e-5)
        off = np.abs(mean.cpu().numpy() - rmean) * rrstd
        err = np.abs(rstd.cpu().numpy() / rrstd - 1)
        assert (err <= 160 * U32 + off ** 2).all(), (level, err.max(), off.max())


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("shape,groups,shift", [((3000, 3, 7, 11), 1, 1), ((300, 6, 37, 41), 2, 1), ((200, 12, 9, 5), 3, 0),
                                                ((30, 32, 61, 67), 1, 0), ((20, 64, 300, 30), 1, 0)])
def test_constant_groups_with_the_least_eps(shape, groups, shift, layout):
    """No spread, and an eps far below the square of a rounding of the mean: a variance that rounds below zero would
    make NaN of it.  The mean is the constant to within the roundings of the sums (and of the pieces' own means)."""
    torch = torch_mod()
    rng = np.random.default_rng(40)
    value = (10.0 ** rng.uniform(-12, 7, shape[0]) * rng.choice([-1.0, 1.0], shape[0])).astype(np.float32)
    value[:3] = 0, 1e-20, 0.1
    x = np.broadcast_to(value[:, None, None, None], shape).copy()
    (tx, _), (ty, _) = _place(x, layout), _place(np.zeros_like(x), layout, shift)
    mean, rstd = (torch.empty((shape[0], groups), device="cuda") for _ in range(2))
    note("constant groups %s %s" % (shape, layout))
    B.group_norm_fwd(tx, groups, None, None, ty, eps=1.2e-38, mean=mean, rstd=rstd)
    torch.cuda.synchronize()
    assert (np.abs(mean.cpu().numpy() - value[:, None]) <= 160 * U32 * np.abs(value[:, None])).all()
    assert bool(torch.isfinite(rstd).all()) and bool((rstd > 0).all()) and bool(torch.isfinite(ty).all())
