"""The retraining step, each of its steps from the state that the one before
left on the device: with moments in 8 bits, whose codes the reference takes up
and has to give back, and of an fp16 network, whose packed values are the fp16
copies of fp32 parameters and whose loss is scaled."""
import numpy as np
import pytest

from oracle import train
from paper_2003_06513_amd import binding as B
import test_gpu_retrain_step as R
from test_gpu_retrain_step import _need_gpu        # noqa: F401 (the fixture)
from gpu_cases import U32, dev, note, torch_mod

pytestmark = pytest.mark.gpu
LOSS_SCALE = 1024.0
SILU = [(ci, co, g, "silu") for ci, co, g, _ in R.LAYERS]


class HalfNet(R.Net):
    """The network in fp16: fp32 parameters, whose fp16 copies are the packed values."""

    def __init__(self, start, bits):
        torch = torch_mod()
        ws, masks, keeps, norm, x, target = start
        n, _, h, w = R.SHAPE
        self.x, self.target = dev(x).half(), dev(target).half()
        self.prep = [B.prepare(dev(a).half(), masks, k) for a, k in zip(ws, keeps)]
        self.dense = [torch.empty(a.shape, dtype=torch.float16, device="cuda") for a in ws]
        self.prep_t = []
        for p, d in zip(self.prep, self.dense):
            B.unpack_dense(p.layer, p.packed, d)
            self.prep_t.append(B.prepare_transposed(p, d))
        self.gamma, self.beta = [dev(g) for g, _ in norm], [dev(b) for _, b in norm]
        like = lambda co: torch.empty((n, co, h, w), dtype=torch.float16, device="cuda")        # noqa: E731
        self.z, self.y, self.dz, self.dy = ([like(co) for _, co, _, _ in SILU] for _ in range(4))
        self.stats = [[torch.empty((n, g), device="cuda") for _ in range(2)] for _, _, g, _ in SILU]
        self.grads = [[torch.empty(4 * k, device="cuda"), torch.empty(co, device="cuda"), torch.empty(co, device="cuda")]
                      for k, (_, co, _, _) in zip(keeps, SILU)]
        self.ws = [B.conv3x3_bwd_weight_workspace(p.layer, B.PSC_F16, n, h, w) for p in self.prep]
        self.values = [p.packed.values.float() for p in self.prep]
        self.list = [t for v, g, b in zip(self.values, self.gamma, self.beta) for t in (v, g, b)]
        copies = [t for p in self.prep for t in (p.packed.values, None, None)]
        self.opt = B.AdamW(self.list, [g for layer in self.grads for g in layer], lr=R.LR,
                           weight_decay=[0.01, 0.0, 0.0] * len(SILU), state_bits=bits, copies=copies)

    def step(self):
        h = self.x
        for i, (_, _, g, act) in enumerate(SILU):
            p = self.prep[i]
            B.conv3x3_fwd(p.layer, p.packed, h, self.z[i])
            B.group_norm_fwd(self.z[i], g, self.gamma[i], self.beta[i], self.y[i], R.EPS, act, *self.stats[i])
            h = self.y[i]
        torch_mod().sub(h, self.target, out=self.dy[-1])
        self.dy[-1].mul_(2.0 * LOSS_SCALE / h.numel())
        for i in reversed(range(len(SILU))):
            _, _, g, act = SILU[i]
            p, (dv, dgamma, dbeta) = self.prep[i], self.grads[i]
            B.group_norm_bwd(self.z[i], self.dy[i], g, self.gamma[i], self.beta[i], *self.stats[i], self.dz[i], dgamma,
                             dbeta, act=act)
            B.conv3x3_bwd_weight(p.layer, p.packed, self.y[i - 1] if i else self.x, self.dz[i], dv, ws=self.ws[i])
            if i:
                B.conv(self.prep_t[i], self.dz[i], out=self.dy[i - 1])
        self.opt.grad_norm(R.CLIP, scale=1.0 / LOSS_SCALE)
        self.opt.step(factor=self.opt.factor)
        for p, t, d in zip(self.prep, self.prep_t, self.dense):
            B.unpack_dense(p.layer, p.packed, d)
            B.transpose_prep(p.layer, d, p.pat, p.keep_mask, t.w, t.pat, t.keep_mask)
            B.pack(t.layer, t.w, t.pat, t.keep_mask, t.packed, t.workspaces[0])


def _h(t):
    return t.cpu().numpy().copy()


def _state(net):
    """Parameters, moments and scales on the host, one entry for each tensor."""
    params = getattr(net, "list", None) or [t for p, g, b in zip(net.prep, net.gamma, net.beta)
                                            for t in (p.packed.values, g, b)]
    at, out = 0, []
    for p in params:
        k, end = p.numel(), at - (-p.numel() // 256) * 256
        out.append((_h(p), _h(net.opt.m[at:at + k]), _h(net.opt.v[at:at + k]),
                    None if net.opt.scale is None else _h(net.opt.scale[at // 256:end // 256])))
        at = end
    return out


def _check_update(before, after, grads, factor, t, bits, what):
    """The optimiser's part from the device's own gradients, factor and state.  Bounds as derived beside the tests of
    the step alone: m's error by the quotient it meets, 24 u of the update, two roundings of the parameter, four of
    the decay."""
    b1, b2, eps = (float(np.float32(k)) for k in (0.9, 0.999, 1e-8))
    for i, ((p0, m0, v0, s0), (p1, m1, v1, s1), g) in enumerate(zip(before, after, grads)):
        decay = 0.01 if i % 3 == 0 else 0.0
        if bits == 8:
            m0, v0 = train.decode_m(m0, s0), train.decode_v(v0, s0)
        rp, rm, rv = train.adamw(p0, g, m0, v0, t, R.LR, 0.9, 0.999, 1e-8, decay, factor)
        e_m = 4 * U32 * (b1 * np.abs(m0) + (1 - b1) * np.abs(g.astype(np.float64) * np.float32(factor)))
        quotient = R.LR / (1 - b1 ** t) / (np.sqrt(rv / (1 - b2 ** t)) + eps)
        kept = p0 * (1 - float(np.float32(R.LR)) * float(np.float32(decay)))
        bound = 24 * U32 * np.abs(rp - kept) + 2 * U32 * (np.abs(rp) + np.abs(kept)) + 4 * U32 * R.LR * decay * np.abs(p0) + \
            e_m * quotient
        assert (np.abs(p1 - rp) <= bound + 1e-44).all(), "%s: parameter %d off by %.3g bounds" % (
            what, i, (np.abs(p1 - rp) / (bound + 1e-44)).max())
        if bits == 8:
            qm, qv, scale = train.encode(rm, rv)
            assert np.array_equal(m1, qm) and np.array_equal(v1, qv), "%s: codes of %d" % (what, i)
            assert (np.abs(s1.astype(np.float64) - scale) <= 2 * U32 * scale).all()
        else:
            assert (np.abs(m1 - rm) <= e_m + 1e-44).all() and (np.abs(v1 - rv) <= 5 * U32 * rv + 1e-44).all()


def _reference(start, packed, state):
    """Norm and gradients in fp64 of the network with the device's parameters."""
    ws, masks, keeps, _, x, target = start
    norm = [(state[3 * i + 1][0], state[3 * i + 2][0]) for i in range(len(packed))]
    now = [dict(pk, values=state[3 * i][0]) for i, pk in enumerate(packed)]
    return next(R._reference((ws, masks, keeps, norm, x, target), now, 1))[:2]


@pytest.mark.parametrize("bits", [8, 32])
def test_every_step_from_the_state_before(bits):
    torch = torch_mod()
    start = R._start(72)
    net = R.Net(start, bits)
    packed = [p.packed.to_host() for p in net.prep]
    for t in range(1, 6):
        before = _state(net)
        norm, grads = _reference(start, packed, before)
        note("retraining step %d from the state before, %d bits" % (t, bits))
        net.step()
        torch.cuda.synchronize()
        flat = [_h(g) for layer in net.grads for g in layer]
        what = "step %d" % t
        assert abs(float(net.opt.norm) / norm - 1) < R.TOL_G, what
        for a, b in zip(flat, grads):
            assert np.abs(a - b).max() <= R.TOL_G * np.abs(b).max(), what
        _check_update(before, _state(net), flat, float(net.opt.factor), t, bits, what)
    assert int(net.opt.steps) == 5


# Of the largest gradient of a tensor: z, y, dz and dy of both layers and the loss's gradient are rounded to fp16, 2^-11
# of each value, and a value is at most a few times what the sums take of it on average (4 covers the norm's reciprocal
# spread too): 9 roundings, 4 * 9 * 2^-11 = 1.8e-2.  (The SiLU has no step that a rounding could pass.)
TOL_HALF = 2e-2


@pytest.mark.parametrize("bits", [8, 32])
def test_half_precision_network(bits, monkeypatch):
    torch = torch_mod()
    monkeypatch.setattr(R, "LAYERS", SILU)
    ws, masks, keeps, norm, x, target = R._start(73)
    start = ([w.astype(np.float16).astype(np.float32) for w in ws], masks, keeps, norm,
             *(t.astype(np.float16).astype(np.float32) for t in (x, target)))
    net = HalfNet(start, bits)
    packed = [p.packed.to_host() for p in net.prep]
    stale = None
    for t in range(1, 5):
        before = _state(net)
        for p, v in zip(net.prep, net.values):
            assert torch.equal(p.packed.values, v.half()), "the copy of step %d" % (t - 1)
        now = [(b[0].astype(np.float16).astype(np.float32) if i % 3 == 0 else b[0],) for i, b in enumerate(before)]
        norm, grads = _reference(start, packed, now)
        note("fp16 retraining step %d, %d bits" % (t, bits))
        net.step()
        torch.cuda.synchronize()
        flat = [_h(g) for layer in net.grads for g in layer]
        what = "step %d" % t
        assert abs(float(net.opt.norm) / norm - 1) < TOL_HALF, what
        for a, b in zip(flat, grads):
            assert np.abs(a / LOSS_SCALE - b).max() <= TOL_HALF * np.abs(b).max(), what
        if stale is not None:       # the convolutions read the copies: with the values before them it would show
            assert any(np.abs(a - b).max() > 2 * TOL_HALF * np.abs(b).max() for a, b in zip(stale, grads))
        stale = grads
        _check_update(before, _state(net), flat, float(net.opt.factor), t, bits, what)
    for p, tr, d in zip(net.prep, net.prep_t, net.dense):
        want = torch.empty_like(tr.w)
        B.unpack_dense(tr.layer, tr.packed, want)
        torch.cuda.synchronize()
        assert torch.equal(want, d.flip(2, 3).transpose(0, 1))
    assert int(net.opt.steps) == 4
