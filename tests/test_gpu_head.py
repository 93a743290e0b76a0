"""The classification head against 64-bit numpy: forward and every gradient."""
import numpy as np
import pytest

import operator_reference as R

pytestmark = pytest.mark.gpu

SIZES = [  # n, c, h, w, classes
    (2, 3, 2, 2, 2), (1, 5, 4, 4, 1), (4, 16, 8, 8, 10), (17, 33, 7, 7, 21), (5, 8, 1, 5, 300), (128, 112, 8, 8, 10), (32, 130, 7, 7, 1000),
    (3, 70, 15, 17, 33), (200, 20, 3, 3, 40), (6, 9, 56, 56, 12), (70, 12, 32, 32, 5), (33, 2050, 1, 1, 65), (2, 4, 90, 91, 7),
    (8, 512, 3, 3, 1000), (37, 700, 2, 2, 610), (24, 2050, 7, 7, 501), (100, 2049, 7, 7, 3),
]
BORDER = 1e-4


def problem(rng, n, c, h, w, classes):
    x = (rng.standard_normal((n, c, h, w)) * rng.uniform(0.5, 2, (c, 1, 1)) + rng.standard_normal((c, 1, 1))).astype(np.float32)
    gamma, beta = rng.uniform(0.5, 1.5, c).astype(np.float32), (rng.standard_normal(c) * 0.1).astype(np.float32)
    # no pixel nearer to the ReLU's border than rounding can decide
    x64 = x.astype(np.float64)
    scale = gamma / np.sqrt(x64.var((0, 2, 3)) + 1e-5)
    z = (x64 - x64.mean((0, 2, 3), keepdims=True)) * scale[:, None, None] + beta[:, None, None]
    x += np.where(np.abs(z) < BORDER, 4 * BORDER / scale[:, None, None], 0).astype(np.float32)
    wt = (rng.standard_normal((classes, c)) / np.sqrt(c)).astype(np.float32)
    return x, gamma, beta, wt, (rng.standard_normal(classes) * 0.1).astype(np.float32), (rng.standard_normal((n, classes)) / n).astype(np.float32)


def tolerances(x, gamma, beta, w, b, dl):
    """Elementwise bounds on a float32 evaluation.  z and xh: the mean is a sum of at most a few dozen terms a thread and a
    tree, rounded relative to mean |x|; with it 8 roundings.  A pooled value adds at most 64 of them a lane and a tree.  A
    product adds K / 16 / wavefronts + 16 terms: K / 16 + 24 bounds it."""
    n, c, h, wd = x.shape
    x = x.astype(np.float64)
    mean, rstd = x.mean((0, 2, 3), keepdims=True), 1 / np.sqrt(x.var((0, 2, 3), keepdims=True) + 1e-5)
    g, be = gamma.astype(np.float64)[:, None, None], beta.astype(np.float64)[:, None, None]
    e_mean = R.EPS * 128 * np.abs(x).mean((0, 2, 3), keepdims=True)
    xh = (x - mean) * rstd
    z = xh * g + be
    e_rstd = 128 * R.EPS                                         # relative
    e_xh = rstd * (e_mean + 4 * R.EPS * (np.abs(x) + np.abs(mean))) + e_rstd * np.abs(xh)
    e_z = np.abs(g) * e_xh + 4 * R.EPS * (np.abs(z) + np.abs(be) + np.abs(g * rstd * x) + np.abs(g * rstd * mean))
    pooled = np.maximum(z, 0).mean((2, 3))
    e_pool = np.where(z > 0, e_z, 0).mean((2, 3)) + 80 * R.EPS * pooled
    w, dl, b = w.astype(np.float64), dl.astype(np.float64), b.astype(np.float64)
    aw, adl = np.abs(w), np.abs(dl)
    terms = lambda k: (k / 16 + 24) * R.EPS
    t = dict(logits=e_pool @ aw.T + terms(c) * (pooled @ aw.T) + 2 * R.EPS * (pooled @ aw.T + np.abs(b)),
             w=adl.T @ e_pool + terms(n) * (adl.T @ pooled), b=terms(n) * adl.sum(0))
    e_dp = terms(len(w)) * (adl @ aw)
    dp = dl @ w
    hw = h * wd
    dz = np.where(z > 0, dp[:, :, None, None] / hw, 0)
    e_dz = np.where(z > 0, (e_dp + 4 * R.EPS * np.abs(dp))[:, :, None, None] / hw, 0)
    sums = (n / 256 + 80) * R.EPS                                # images a thread, pixels a lane, trees
    t["beta"] = e_dz.sum((0, 2, 3)) + sums * np.abs(dz).sum((0, 2, 3))
    t["gamma"] = (e_dz * np.abs(xh) + np.abs(dz) * e_xh).sum((0, 2, 3)) + sums * np.abs(dz * xh).sum((0, 2, 3))
    m = n * hw
    c1, c2 = dz.sum((0, 2, 3))[:, None, None] / m, (dz * xh).sum((0, 2, 3))[:, None, None] / m
    size = np.abs(dz) + np.abs(c1) + np.abs(xh * c2)
    t["dx"] = np.abs(g * rstd) * (e_dz + t["beta"][:, None, None] / m + np.abs(xh) * t["gamma"][:, None, None] / m + e_xh * np.abs(c2) +
                                  (8 * R.EPS + e_rstd) * size)
    return t


class Head:
    def __init__(self, n, c, h, w, classes, arrays, layout="dense"):
        import torch
        import paper_1707_04585_amd as rv
        dev = lambda a: torch.as_tensor(a).cuda()
        x, gamma, beta, wt, b, dl = arrays
        self.rv, self.d, self.shape = rv, rv.HeadDesc(c, classes), (n, c, h, w)
        full = torch.full((n, 2 * c, h, w), 7.0, device="cuda")
        self.x = dev(x) if layout == "dense" else full[:, c:].copy_(dev(x))
        self.dx = torch.zeros(n, c, h, w, device="cuda") if layout == "dense" else torch.full((n, 2 * c, h, w), 7.0, device="cuda")[:, c:]
        wide = 0 if layout == "dense" else 3
        self.logits = torch.full((n, classes + wide), 7.0, device="cuda")[:, :classes]
        self.dl = torch.full((n, classes + wide), 7.0, device="cuda")[:, :classes]
        self.dl.copy_(dev(dl))
        self.p = dict(gamma=dev(gamma), beta=dev(beta), w=dev(wt), b=dev(b))
        self.g = {k: torch.full_like(v, 5.0) for k, v in self.p.items()}
        saved, bwd = rv.revnet_head_workspace_bytes(self.d, n, h, w)
        self.saved = torch.full((saved,), 0xFF, dtype=torch.uint8, device="cuda")
        self.ws = torch.full((bwd,), 0xFF, dtype=torch.uint8, device="cuda")

    def step(self, stream=None, accumulate=0):
        self.rv.revnet_head_fwd(self.d, self.x, self.p, self.logits, self.saved, stream)
        self.rv.revnet_head_bwd(self.d, self.x, self.saved, self.dl, self.p, self.dx, self.g, accumulate, self.ws, stream)


@pytest.mark.parametrize("layout", ["dense", "half"])
@pytest.mark.parametrize("n,c,h,w,classes", SIZES)
def test_forward_and_gradients(n, c, h, w, classes, layout):
    import torch
    rng = np.random.default_rng(n + c + h + classes)
    arrays = problem(rng, n, c, h, w, classes)
    x, gamma, beta, wt, b, dl = arrays
    logits, ref = R.head(x, gamma, beta, wt, b, dl)
    ref["logits"] = logits
    tol = tolerances(*arrays)
    k = Head(n, c, h, w, classes, arrays, layout)
    k.step()
    torch.cuda.synchronize()
    got = dict(k.g, logits=k.logits, dx=k.dx)
    for name in ("logits", "w", "b", "gamma", "beta", "dx"):
        off = np.abs(got[name].cpu().numpy().astype(np.float64) - ref[name])
        assert np.all(off <= tol[name] + 1e-30), (name, float((off / (tol[name] + 1e-30)).max()))
    if layout == "half":
        assert (k.dx._base[:, :c] == 7).all() and (k.logits._base[:, classes:] == 7).all()
    first = {name: t.clone() for name, t in got.items()}
    k.step(accumulate=1)          # added to, and the same bits
    torch.cuda.synchronize()
    for name, t in k.g.items():
        assert torch.equal(t, first[name] + first[name]), name
    assert torch.equal(k.dx, first["dx"]) and torch.equal(k.logits, first["logits"])


def test_channels_that_are_constant_or_never_positive():
    import torch
    rng = np.random.default_rng(1)
    n, c, h, w, classes = 4, 6, 5, 5, 9
    arrays = list(problem(rng, n, c, h, w, classes))
    arrays[0][:, 1] = 2.5            # no variance: xhat is 0, z is beta
    arrays[2][1] = 0.25
    arrays[2][2] = -50.0             # never positive
    arrays[1][3], arrays[2][3] = 0.0, -1.0
    logits, ref = R.head(*arrays)
    k = Head(n, c, h, w, classes, arrays)
    k.step()
    torch.cuda.synchronize()
    # z = x * scale + shift with shift = beta - mean * scale rounded to 24 bits: where the variance is 0, mean * scale is
    # 2.5 * gamma * 316, and z = beta carries that rounding, half a step, and scale's own (in x * scale and in shift, once each)
    off = 3 * R.EPS * 2.5 * arrays[1][1] * 1e-5 ** -0.5
    assert np.all(np.abs(k.logits.cpu().numpy() - logits) < 1e-5 + off * np.abs(arrays[3][:, 1]))
    dx = k.dx.cpu().numpy()
    # (the constant channel's scale is 1 / sqrt(eps), 316 times the others': its derivative is a sum that cancels)
    for ch, bar in ((0, 1e-5), (1, 1e-3), (4, 1e-5), (5, 1e-5)):
        assert np.abs(dx[:, ch] - ref["dx"][:, ch]).max() <= bar * max(1.0, np.abs(ref["dx"][:, ch]).max()), ch
    assert (dx[:, 2] == 0).all() and (dx[:, 3] == 0).all()
    assert k.g["gamma"][2] == 0 and k.g["beta"][2] == 0


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("n,c,h,w", [(4, 6, 5, 5), (20, 3, 8, 8), (70, 3, 32, 32)])
def test_a_value_that_is_no_number_is_not_hidden(n, c, h, w, bad):
    import torch
    arrays = list(problem(np.random.default_rng(3), n, c, h, w, 9))
    arrays[0][n - 2, 1, h - 1, w - 1] = bad
    k = Head(n, c, h, w, 9, arrays)
    k.step()
    torch.cuda.synchronize()
    assert torch.isnan(k.logits).all() and torch.isnan(k.dx[:, 1]).all() and torch.isnan(k.g["w"][:, 1]).all() and torch.isnan(k.g["gamma"][1])
    assert torch.isfinite(k.dx[:, 0]).all() and torch.isfinite(k.g["w"][:, 0]).all() and torch.isfinite(k.g["gamma"][0])


def test_graph():
    import torch
    rng = np.random.default_rng(2)
    size = (32, 130, 7, 7, 100)
    a, b = (Head(*size, problem(np.random.default_rng(2), *size)) for _ in range(2))
    a.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(torch.cuda.current_stream())
    for k in range(4):
        for t in (a, b):
            t.x.mul_(1.0 + 0.5 * k)
            t.dl.mul_(-2.0)
        a.dx.zero_()
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        assert torch.equal(a.dx, b.dx) and torch.equal(a.logits, b.logits)
        for name in a.g:
            assert torch.equal(a.g[name], b.g[name]), name
