"""The gradient norm over lists of many chunks of 1024 elements: blocks that
load several of them before they add the first, that go on from one tensor to
the next, and lists of more tensors than a launch takes.  Squares and sums in
64 bits: norm and factor are those of 64 bits rounded once (2^-53 of the sum
for each of its terms, far below 2^-10 of a rounding of 32)."""
import numpy as np
import pytest

from oracle import train
from paper_2003_06513_amd import binding as B
from gpu_cases import U32, note, torch_mod

pytestmark = pytest.mark.gpu
# sizes, and how many elements into its buffer each tensor begins, in turn
LISTS = {
    "one": ([9_000_001], [0]),
    "whole chunks": ([10_240 * 1024], [0]),
    "ends inside a block's run": ([3_000_001, 2_500_003, 5, 4_194_309], [0]),
    "some not aligned": ([2_900_000, 3_100_001, 2_999_999, 1023], [0, 1, 0, 2]),
    "none aligned": ([9_437_184], [1]),
    "few chunks a block": ([1_100_000, 70_000, 1_500_001], [0, 0, 3]),
    "more than a launch takes": ([40_000 + 17 * i for i in range(250)], [0]),
    "many that end early": ([8 * 1024 + 1, 1] * 600 + [5_000_000], [0, 4]),
}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    B.lib()


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("name", LISTS)
def test_long_lists(name, half):
    torch = torch_mod()
    sizes, shifts = LISTS[name]
    rng = np.random.default_rng(len(name))
    views, host = [], []
    for i, k in enumerate(sizes):
        shift = shifts[i % len(shifts)]
        g = (rng.standard_normal(k, dtype=np.float32) * np.float32(10.0 ** rng.uniform(-2, 1)))
        g = g.astype(np.float16) if half else g
        # values beside the tensor that a read outside it would add
        buf = torch.full((k + shift + 64,), 1e4 if half else 1e30, dtype=torch.float16 if half else torch.float32,
                         device="cuda")
        buf[shift:shift + k] = torch.from_numpy(g)
        views.append(buf[shift:shift + k]), host.append(g)
    plist = B.ParamList(None, views)
    out = torch.empty(2, device="cuda")
    most = float(np.float32(0.3))
    note("norm of %s, %s" % (name, "fp16" if half else "fp32"))
    B.grad_norm(plist, out, max_norm=most, scale=0.5)
    torch.cuda.synchronize()
    first = out.cpu().numpy()
    want = np.array(train.grad_norm(host, 0.5, most))
    assert (np.abs(first - want) <= U32 * (1 + 2.0 ** -10) * want).all(), (first, want)
    B.grad_norm(plist, out, max_norm=most, scale=0.5)
    assert out.cpu().numpy().tobytes() == first.tobytes()
    # one element that is not finite, the last, is seen
    views[-1][-1] = np.nan
    B.grad_norm(plist, out, max_norm=most)
    assert np.isnan(out.cpu().numpy()).all()
