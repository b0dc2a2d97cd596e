"""A retraining step of a small pruned network, put together from the library's
calls as a program would: two pruned convolutions, each with group
normalisation and an activation, a mean-square loss, the backward through both
(transposed packing, masked weight gradient, normalisation), the clip over all
gradients and AdamW on the stored values and the norm parameters, and the new
values in both packings.  Several steps against the same in fp64 on the CPU,
eager and replayed from a graph."""
import numpy as np
import pytest

import oracle
from oracle import train
from paper_2003_06513_amd import binding as B
from synthetic import inputs
from gpu_cases import dev, note, torch_mod

pytestmark = pytest.mark.gpu
EPS, LR, CLIP = 1e-5, 1e-2, 0.5
SHAPE = (4, 6, 14, 14)                     # the batch
LAYERS = [(6, 16, 4, "silu"), (16, 24, 8, "relu")]     # cin, cout, groups, act


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    B.lib()


def _start(seed):
    """Host weights, library, keeps, norm parameters, batch and target."""
    rng = np.random.default_rng(seed)
    ws = [inputs.he_weights(seed + i, co, ci) for i, (ci, co, _, _) in enumerate(LAYERS)]
    masks = oracle.select_library(np.concatenate([w.reshape(-1, 3, 3) for w in ws]), 8)
    keeps = [inputs.keep_after_drop(ci * co, 30) for ci, co, _, _ in LAYERS]
    norm = [((1 + 0.1 * rng.standard_normal(co)).astype(np.float32), (0.1 * rng.standard_normal(co)).astype(np.float32))
            for _, co, _, _ in LAYERS]
    n, _, h, w = SHAPE
    x = rng.standard_normal(SHAPE).astype(np.float32)
    target = rng.standard_normal((n, LAYERS[-1][1], h, w)).astype(np.float32)
    return ws, masks, keeps, norm, x, target


class Net:
    """The network on the GPU; step() makes one retraining step."""

    def __init__(self, start, bits):
        torch = torch_mod()
        ws, masks, keeps, norm, x, target = start
        n, _, h, w = SHAPE
        self.x, self.target = dev(x), dev(target)
        self.prep = [B.prepare(dev(a), masks, k) for a, k in zip(ws, keeps)]
        self.dense = [torch.empty(a.shape, device="cuda") for a in ws]
        self.prep_t = []
        for p, d in zip(self.prep, self.dense):
            B.unpack_dense(p.layer, p.packed, d)
            self.prep_t.append(B.prepare_transposed(p, d))
        self.gamma, self.beta = [dev(g) for g, _ in norm], [dev(b) for _, b in norm]
        like = lambda co: torch.empty((n, co, h, w), device="cuda")        # noqa: E731
        self.z, self.y, self.dz, self.dy = ([like(co) for _, co, _, _ in LAYERS] for _ in range(4))
        self.stats = [[torch.empty((n, g), device="cuda") for _ in range(2)] for _, _, g, _ in LAYERS]
        self.grads = [[torch.empty(4 * k, device="cuda"), torch.empty(co, device="cuda"), torch.empty(co, device="cuda")]
                      for k, (_, co, _, _) in zip(keeps, LAYERS)]
        self.ws = [B.conv3x3_bwd_weight_workspace(p.layer, B.PSC_F32, n, h, w) for p in self.prep]
        params = [t for p, g, b in zip(self.prep, self.gamma, self.beta) for t in (p.packed.values, g, b)]
        self.opt = B.AdamW(params, [g for layer in self.grads for g in layer], lr=LR,
                           weight_decay=[0.01, 0.0, 0.0] * len(LAYERS), state_bits=bits)

    def step(self):
        h = self.x
        for i, (_, _, g, act) in enumerate(LAYERS):
            p = self.prep[i]
            B.conv3x3_fwd(p.layer, p.packed, h, self.z[i])
            B.group_norm_fwd(self.z[i], g, self.gamma[i], self.beta[i], self.y[i], EPS, act, *self.stats[i])
            h = self.y[i]
        torch_mod().sub(h, self.target, out=self.dy[-1])
        self.dy[-1].mul_(2.0 / h.numel())           # of the mean of the squares
        for i in reversed(range(len(LAYERS))):
            _, _, g, act = LAYERS[i]
            p, (dv, dgamma, dbeta) = self.prep[i], self.grads[i]
            B.group_norm_bwd(self.z[i], self.dy[i], g, self.gamma[i], self.beta[i], *self.stats[i], self.dz[i], dgamma,
                             dbeta, act=act)
            B.conv3x3_bwd_weight(p.layer, p.packed, self.y[i - 1] if i else self.x, self.dz[i], dv, ws=self.ws[i])
            if i:
                B.conv(self.prep_t[i], self.dz[i], out=self.dy[i - 1])
        self.opt.grad_norm(CLIP)
        self.opt.step(factor=self.opt.factor)
        for p, t, d in zip(self.prep, self.prep_t, self.dense):     # the new values in the transposed packing
            B.unpack_dense(p.layer, p.packed, d)
            B.transpose_prep(p.layer, d, p.pat, p.keep_mask, t.w, t.pat, t.keep_mask)
            B.pack(t.layer, t.w, t.pat, t.keep_mask, t.packed, t.workspaces[0])

    def params(self):
        return [t.cpu().numpy() for p, g, b in zip(self.prep, self.gamma, self.beta) for t in (p.packed.values, g, b)]


def _reference(start, packed, steps):
    """The same in fp64: dense masked weights, the stored values' gradients."""
    ws, masks, keeps, norm, x, target = start
    where = []          # (filter, channel, row, column) of each stored value
    bits = [[q for q in range(9) if (int(c) >> q) & 1] for c in masks]
    for pk in packed:
        idx = []
        for i in range(len(pk["filter_perm"])):
            for k in range(pk["filter_ptr"][i], pk["filter_ptr"][i + 1]):
                idx += [(pk["filter_perm"][i], pk["cin_idx"][k], q // 3, q % 3) for q in bits[pk["pat_id"][k]]]
        where.append(tuple(np.array(idx).T))
    values = [pk["values"].astype(np.float64) for pk in packed]
    gamma, beta = [g.astype(np.float64) for g, _ in norm], [b.astype(np.float64) for _, b in norm]
    params = [t for i in range(len(LAYERS)) for t in (values[i], gamma[i], beta[i])]
    moments = [(np.zeros(p.size), np.zeros(p.size)) for p in params]
    taps = [(r, s) for r in range(3) for s in range(3)]

    def shifted(t, r, s):
        p = np.pad(t, ((0, 0), (0, 0), (1, 1), (1, 1)))
        return p[:, :, r:r + t.shape[2], s:s + t.shape[3]]

    for step in range(1, steps + 1):
        h, zs, ys, stats, dense = x.astype(np.float64), [], [], [], []
        for i, (ci, co, g, act) in enumerate(LAYERS):
            d = np.zeros((co, ci, 3, 3))
            d[where[i]] = params[3 * i]
            dense.append(d)
            z = sum(np.einsum("oi,nihw->nohw", d[:, :, r, s], shifted(h, r, s)) for r, s in taps)
            y, mean, rstd = train.group_norm(z, g, params[3 * i + 1], params[3 * i + 2], EPS, act)
            zs.append(z), ys.append(y), stats.append((mean, rstd))
            h = y
        dy = 2.0 / h.size * (h - target)
        grads = [None] * len(params)
        for i in reversed(range(len(LAYERS))):
            _, _, g, act = LAYERS[i]
            dz, dgamma, dbeta = train.group_norm_back(zs[i], dy, g, params[3 * i + 1], params[3 * i + 2], *stats[i], act)
            below = ys[i - 1] if i else x.astype(np.float64)
            dw = np.stack([np.einsum("nohw,nihw->oi", dz, shifted(below, r, s)) for r, s in taps], axis=-1)
            dw = dw.reshape(dense[i].shape)
            grads[3 * i:3 * i + 3] = [dw[where[i]], dgamma, dbeta]
            # the input's gradient: the taps of the rotated, transposed weights
            dy = sum(np.einsum("oi,nohw->nihw", dense[i][:, :, r, s], shifted(dz, 2 - r, 2 - s)) for r, s in taps)
        norm_, factor = train.grad_norm(grads, 1.0, CLIP)
        for k, g in enumerate(grads):
            params[k], m, v = train.adamw(params[k], g, *moments[k], step, LR, 0.9, 0.999, 1e-8,
                                          0.01 if k % 3 == 0 else 0.0, factor)
            moments[k] = (m, v)
        yield norm_, grads, params


# An AdamW step has the size lr in every element, whatever the gradient's: an element whose gradient is all rounding
# may go either way.  So gradients and norms are compared (a convolution of 64 terms in 2^-24 steps, twice forward and
# back, leaves them well below 1e-4 of their largest), and parameters where the gradient is above 1e-3 of its largest:
# there a relative gradient error of 1e-4 / 1e-3 moves the update by at most 0.1 lr in each of the steps.
TOL_G, TOL_P = 1e-4, 0.1


@pytest.mark.parametrize("bits", [32, 8])
def test_step_follows_the_formulas(bits):
    torch = torch_mod()
    start = _start(70)
    net = Net(start, bits)
    packed = [p.packed.to_host() for p in net.prep]
    steps = 3
    ref = _reference(start, packed, steps)
    clear = None
    for t in range(steps):
        note("retraining step %d, %d bits" % (t, bits))
        net.step()
        torch.cuda.synchronize()
        norm, grads, params = next(ref)
        if bits == 8 and t:
            # rounded moments take the parameters elsewhere, within their steps
            for a, b in zip(net.params(), params):
                assert np.abs(a - b).max() <= 2.0 * LR * (t + 1)
            continue
        assert abs(float(net.opt.norm) / norm - 1) < TOL_G
        flat = [g.cpu().numpy() for layer in net.grads for g in layer]
        for a, b in zip(flat, grads):
            assert np.abs(a - b).max() <= TOL_G * np.abs(b).max()
        sure = [np.abs(g) > 1e-3 * np.abs(g).max() for g in grads]
        clear = sure if clear is None else [a & b for a, b in zip(clear, sure)]
        for a, b, s in zip(net.params(), params, clear):
            assert np.abs(a - b)[s].max() <= TOL_P * LR * (t + 1)
            assert s.mean() > 0.9
    # the transposed packing has the new values too
    for p, tr, d in zip(net.prep, net.prep_t, net.dense):
        want = torch.empty_like(tr.w)
        B.unpack_dense(tr.layer, tr.packed, want)
        torch.cuda.synchronize()
        assert torch.equal(want, d.flip(2, 3).transpose(0, 1))
    assert int(net.opt.steps) == steps


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_replayed_from_a_graph(bits):
    torch = torch_mod()
    start = _start(71)
    eager, replayed = Net(start, bits), Net(start, bits)
    note("retraining graph %d bits" % bits)
    eager.step()
    replayed.step()                                   # first calls, outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed.step()
    for _ in range(3):
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.params(), replayed.params()):
            assert a.tobytes() == b.tobytes()
    assert int(replayed.opt.steps) == 4
