"""Group normalisation: what the first file's sweep over shapes leaves out."""
import numpy as np
import pytest

from paper_2003_06513_amd import binding as B
from gpu_cases import dev, note, torch_mod
from test_gpu_group_norm import _data, _need_gpu, _place, check_forward       # noqa: F401 (the fixture)

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
