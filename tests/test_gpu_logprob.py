"""Log probabilities of labels with entropy and top classes, and their gradient,
against 64-bit numpy at the sizes and values where they can go wrong."""
import numpy as np
import pytest

import operator_reference as R

pytestmark = pytest.mark.gpu

# rows, classes, top_k: one class to long rows; a wavefront, a workgroup and several workgroups a row
SIZES = [
    (1, 1, 1), (7, 2, 2), (5, 3, 0), (130, 10, 5), (3, 63, 32), (4, 64, 1), (6, 255, 32), (5, 256, 3), (33, 1000, 5), (2, 2047, 20),
    (3, 2048, 5), (3, 2049, 5), (9, 4095, 4), (3, 4097, 32), (300, 4111, 3), (260, 9001, 2), (1, 20011, 32), (5, 33000, 20), (40, 16400, 8),
    (1, 131072, 32), (2, 262147, 5), (600, 2100, 1), (193, 33001, 3), (70, 29001, 6),
]


def logits(rng, rows, classes, bf16, pad=0, offset=0):
    """-> (tensor [rows, classes] with `pad` columns behind each row and its base off alignment by `offset` elements, float64 values)"""
    import torch
    x = (rng.standard_normal((rows, classes)) * 3).astype(np.float32)
    dtype = torch.bfloat16 if bf16 else torch.float32
    ld = classes + pad
    flat = torch.full((rows * ld + offset + 8,), 99.0, dtype=dtype, device="cuda")
    t = flat[offset:offset + rows * ld].view(rows, ld)[:, :classes]
    t.copy_(torch.as_tensor(x))
    return t, t.float().cpu().numpy().astype(np.float64)


def labels_of(rng, rows, classes, odd=False):
    lab = rng.integers(0, classes, rows)
    if odd and rows > 3:
        lab[1], lab[2], lab[3] = -1, classes, -7
    return lab.astype(np.int64)


class Out:
    def __init__(self, rows, top_k):
        import torch
        f = lambda *s: torch.full(s, 55.0, device="cuda")
        self.logprob, self.entropy, self.lse, self.top = f(rows), f(rows), f(rows), f(rows, top_k)
        self.ids = torch.full((rows, top_k), 55, dtype=torch.int64, device="cuda")

    def host(self):
        return {k: getattr(self, k).cpu().numpy() for k in ("logprob", "entropy", "lse", "ids", "top")}


def forward(t, labels, top_k, out=None, stream=None):
    import torch
    import paper_1707_04585_amd as rv
    rows, classes = t.shape
    out = out or Out(rows, top_k)
    need = rv.revnet_logprob_workspace_bytes(rows, classes, top_k)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") if need else None
    rv.revnet_logprob_fwd(t, labels, top_k, out.logprob, out.entropy, out.lse, out.ids, out.top, ws, stream)
    return out


def near(got, ref, tol):
    got = got.astype(np.float64)
    same = (got == ref) | (np.isnan(got) & np.isnan(ref))
    with np.errstate(invalid="ignore"):
        ok = same | (np.isfinite(ref) & (np.abs(got - ref) <= tol))
    return bool(ok.all())


def check(got, ref):
    assert near(got["lse"], ref["lse"], ref["tol"]), "lse"
    assert near(got["logprob"], ref["logprob"], ref["tol"] + 4 * R.EPS * np.abs(np.nan_to_num(ref["logprob"], neginf=0))), "logprob"
    assert near(got["entropy"], ref["entropy"], ref["tol_entropy"]), "entropy"
    assert np.array_equal(got["ids"], ref["ids"]), "ids"
    with np.errstate(invalid="ignore"):
        assert near(got["top"], ref["top"], ref["tol"][:, None] + 4 * R.EPS * np.abs(np.nan_to_num(ref["top"], neginf=0))), "top"


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,classes,top_k", SIZES)
def test_forward(rows, classes, top_k, bf16):
    import torch
    rng = np.random.default_rng(rows * 7 + classes)
    for pad, offset in ((0, 0), (3, 1)):
        t, x = logits(rng, rows, classes, bf16, pad, offset)
        lab = labels_of(rng, rows, classes, odd=True)
        out = forward(t, torch.as_tensor(lab).cuda(), top_k)
        torch.cuda.synchronize()
        check(out.host(), R.logprob(x, lab, top_k))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("classes", [10, 700, 2500, 5000, 40000])
def test_masks_ties_and_values_that_are_no_numbers(classes, bf16):
    import torch
    rng = np.random.default_rng(classes)
    top_k = min(classes, 12)
    t, _ = logits(rng, 16, classes, bf16)
    lowest = torch.finfo(t.dtype).min
    t[0] = -torch.inf                                   # no class left
    t[1] = lowest                                       # masked by the type's lowest value: uniform
    t[2, : classes - 1] = -torch.inf                    # one class left, the last
    t[3, ::2] = -torch.inf
    t[4, 1::2] = lowest
    t[5] = 1.25                                         # all equal: the lower index first
    t[6] = torch.as_tensor(rng.integers(0, 3, classes).astype(np.float32)).cuda()    # many ties
    t[7, classes // 2] = torch.nan
    t[8, classes - 1] = torch.inf
    t[9, 0], t[9, classes - 1] = torch.nan, torch.nan
    t[10] = 0.0
    t[10, ::3] = -0.0                                   # -0 and 0 tie
    t[11] *= 100                                        # one class takes all
    t[12, : classes // 2] = lowest
    t[13, 3:] = -torch.inf                              # fewer classes than top_k
    lab = labels_of(rng, 16, classes)
    lab[0], lab[2], lab[3], lab[7] = 4, classes - 1, 0, -1
    out = forward(t, torch.as_tensor(lab).cuda(), top_k)
    torch.cuda.synchronize()
    got, ref = out.host(), R.logprob(t.float().cpu().numpy(), lab, top_k)
    check(got, ref)
    assert got["entropy"][0] == 0 and got["lse"][0] == -np.inf and got["logprob"][3] == -np.inf and got["logprob"][7] == 0


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("classes", [2600, 5001, 8191])
def test_many_rows_of_middle_length(classes, bf16):
    """So many rows that each of these goes to one wavefront, or (13 top classes) to a workgroup: the values that can go wrong
    among the first and last rows, and both ways agree on the classes of all."""
    import torch
    rng = np.random.default_rng(classes)
    rows, some = 2051, 12
    t, _ = logits(rng, rows, classes, bf16, pad=1, offset=1)
    lowest = torch.finfo(t.dtype).min
    t[0] = -torch.inf
    t[1] = lowest
    t[2, : classes - 1] = -torch.inf
    t[3] = 1.25
    t[4] = torch.as_tensor(rng.integers(0, 3, classes).astype(np.float32)).cuda()
    t[5, classes // 2] = torch.nan
    t[6, classes - 1] = torch.inf
    t[7, 1::2] = lowest
    t[8] *= 100
    t[rows - 1, : classes - 5] = -torch.inf
    t[rows - 2, 5] = torch.nan
    lab = labels_of(rng, rows, classes)
    lab[2], lab[9] = classes - 1, -1
    out, wide = (forward(t, torch.as_tensor(lab).cuda(), k) for k in (12, 13))
    torch.cuda.synchronize()
    for part in (slice(0, some), slice(rows - some, rows)):
        check({k: v[part] for k, v in out.host().items()}, R.logprob(t[part].float().cpu().numpy(), lab[part], 12))
        check({k: v[part] for k, v in wide.host().items()}, R.logprob(t[part].float().cpu().numpy(), lab[part], 13))
    assert torch.equal(out.ids, wide.ids[:, :12])


def test_outputs_that_are_not_asked_for():
    import torch
    import paper_1707_04585_amd as rv
    rng = np.random.default_rng(4)
    for rows, classes in ((9, 300), (2, 50000)):
        t, x = logits(rng, rows, classes, False)
        ref = R.logprob(x, np.full(rows, -1), 3)
        need = rv.revnet_logprob_workspace_bytes(rows, classes, 3)
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        o = Out(rows, 3)
        rv.revnet_logprob_fwd(t, None, 3, None, None, None, o.ids, None, ws)
        rv.revnet_logprob_fwd(t, None, 0, None, o.entropy, None, None, None, ws)
        assert np.array_equal(o.ids.cpu().numpy(), ref["ids"]) and near(o.entropy.cpu().numpy(), ref["entropy"], ref["tol_entropy"])
        assert (o.lse == 55).all() and (o.top == 55).all()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,classes,_", SIZES)
def test_gradient(rows, classes, _, bf16):
    """Every combination of weights, in place and with padded rows, whose padding stays as it was."""
    import torch
    import paper_1707_04585_amd as rv
    rng = np.random.default_rng(rows + classes * 3)
    gl, ge = rng.uniform(-1, 1, rows).astype(np.float32), rng.uniform(-1, 1, rows).astype(np.float32)
    gl[rows // 2] = 0
    for pad, offset, weights, entropies in ((0, 0, False, False), (3, 1, True, True), (0, 1, True, False), (1, 0, False, True)):
        t, x = logits(rng, rows, classes, bf16, pad, offset)
        lab = labels_of(rng, rows, classes, odd=True)
        r = R.logprob(x, lab, 0)
        lse, ent = r["lse"].astype(np.float32), r["entropy"].astype(np.float32)
        scale = np.float32(-1.0 / rows)
        ref = R.logprob_bwd(x, lab, lse, ent, gl if weights else None, ge if entropies else None, scale)
        dev = lambda a: torch.as_tensor(a).cuda()
        args = (dev(lab), dev(lse), dev(ent), dev(gl) if weights else None, dev(ge) if entropies else None, float(scale))
        out = torch.full((rows, classes + 2), 42.0, dtype=t.dtype, device="cuda")
        rv.revnet_logprob_bwd(t, *args, out[:, :classes])
        rv.revnet_logprob_bwd(t, *args, t)     # in place
        torch.cuda.synchronize()
        assert (out[:, classes:] == 42).all()
        if pad:
            assert (t._base.view(-1)[offset + classes:offset + classes + pad] == 99).all()
        assert torch.equal(torch.nan_to_num(t, nan=77.0), torch.nan_to_num(out[:, :classes], nan=77.0))
        got = out[:, :classes].float().cpu().numpy().astype(np.float64)
        # p is off by 6 roundings and those of its exponent (3 per unit); four terms of an element; the result's own rounding
        logp = np.abs(x - lse[:, None].astype(np.float64))
        p = np.exp(x - lse[:, None])
        wl = np.abs(scale) * (np.abs(gl) if weights else np.ones(rows))[:, None]
        we = np.abs(scale) * (np.abs(ge) if entropies else np.zeros(rows))[:, None]
        tol = R.EPS * (8 + 4 * logp) * p * (wl + we * (logp + np.abs(ent)[:, None])) + 4 * R.EPS * np.abs(np.nan_to_num(ref))
        if bf16:
            tol = tol + 2.0 ** -8 * (np.abs(np.nan_to_num(ref)) + tol) + 2.0 ** -134
        tol = tol + 2.0 ** -149
        ok = (np.isnan(got) & np.isnan(ref)) | (np.abs(got - ref) <= tol)
        assert ok.all(), (pad, weights, entropies, int((~ok).sum()))


def test_gradient_of_rows_without_a_label_or_a_class():
    """A row that takes no part has a gradient of zeros whatever it holds; one with a label out of range has NaN."""
    import torch
    import paper_1707_04585_amd as rv
    for bf16 in (False, True):
        t, _ = logits(np.random.default_rng(8), 6, 1003, bf16)
        t[0], t[1, 5], t[2] = torch.nan, torch.inf, -torch.inf
        lab = torch.tensor([-1, -1, 3, 1003, 4, 5]).cuda()
        o = forward(t, lab, 0)
        weight = torch.tensor([1.0, 1.0, 1.0, 1.0, 0.0, 1.0]).cuda()
        t[4, 7] = torch.nan                               # weight 0: absent
        out = torch.full_like(t, 3.0)
        rv.revnet_logprob_bwd(t, lab, o.lse, o.entropy, weight, None, 1.0, out)
        torch.cuda.synchronize()
        assert (out[[0, 1, 2, 4]] == 0).all() and torch.isnan(out[3]).all() and torch.isfinite(out[5]).all()
        assert float(o.logprob[0]) == 0 and float(o.logprob[2]) == -np.inf and np.isnan(float(o.logprob[3]))
        t[3:5] = torch.where(torch.isnan(t[3:5]), 0, t[3:5])
        rv.revnet_logprob_bwd(t, None, o.lse, o.entropy, None, torch.tensor([0.0, 0, 1, 1, 1, 1]).cuda(), 1.0, out)
        assert (out[:3] == 0).all() and torch.isfinite(out[3:]).all()


def test_rows_beyond_32_bit_offsets():
    """A matrix of more than 2^32 bytes: its last rows against the reference, their gradient in place.  (Not against the bits
    of the same rows elsewhere: rows of an odd length start at any alignment, and the order of the sums goes by that.)"""
    import torch
    import paper_1707_04585_amd as rv
    rows, classes = 17000, 131073
    t = torch.empty((rows, classes), dtype=torch.bfloat16, device="cuda")      # 4.46 GB, more than 2^31 elements
    tail, x = logits(np.random.default_rng(6), 5, classes, True)
    t[:-5] = 1.0
    t[-5:] = tail
    lab = torch.arange(rows, device="cuda") % classes
    big, last = forward(t, lab, 4), lab[-5:].cpu().numpy()
    ref = R.logprob(x, last, 4)
    check({k: v[-5:] for k, v in big.host().items()}, ref)
    lse = big.lse[-5:].cpu().numpy()
    rv.revnet_logprob_bwd(t, lab, big.lse, None, None, None, 1.0, t)
    want = R.logprob_bwd(x, last, lse, None, None, None, 1.0)
    p, logp = np.exp(x - lse[:, None]), np.abs(x - lse[:, None])
    tol = R.EPS * (8 + 4 * logp) * p + (2.0 ** -8 + 4 * R.EPS) * np.abs(want) + 2.0 ** -134      # as in test_gradient
    assert np.all(np.abs(t[-5:].float().cpu().numpy() - want) <= tol)


def test_two_streams_and_a_graph():
    import torch
    import paper_1707_04585_amd as rv
    rng = np.random.default_rng(12)
    cases = []
    for rows, classes in ((3, 60001), (70, 1000), (300, 5000)):
        t, _ = logits(rng, rows, classes, True)
        need = rv.revnet_logprob_workspace_bytes(rows, classes, 6)
        cases.append(dict(t=t, lab=torch.as_tensor(labels_of(rng, rows, classes)).cuda(), ws=torch.empty(max(need, 1), dtype=torch.uint8, device="cuda"),
                          o=Out(rows, 6), g=torch.empty_like(t)))

    def step(c, o, g, stream):
        rv.revnet_logprob_fwd(c["t"], c["lab"], 6, o.logprob, o.entropy, o.lse, o.ids, o.top, c["ws"], stream)
        rv.revnet_logprob_bwd(c["t"], c["lab"], o.lse, o.entropy, None, o.entropy, 0.5, g, stream)

    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for c, s in zip(cases, streams):
        step(c, c["o"], c["g"], s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for c in cases:
            step(c, c["o"], c["g"], torch.cuda.current_stream())
    for k in range(4):
        for c in cases:
            c["t"].add_(0.125 * k)
            c["t"][:, k] += 1.0
            c["o"].ids.zero_()
            c["g"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for c in cases:
            o, g = Out(c["t"].shape[0], 6), torch.empty_like(c["g"])
            step(c, o, g, None)
            torch.cuda.synchronize()
            for name in ("logprob", "entropy", "lse", "ids", "top"):
                assert torch.equal(getattr(o, name), getattr(c["o"], name)), name
            assert torch.equal(g, c["g"])


def test_more_rows_than_one_launch_has_threads_for():
    """2^26 + 5 rows, a wavefront each: the rows where one launch ends and the next begins, and the last."""
    import torch
    import paper_1707_04585_amd as rv
    rows, classes, step = 2 ** 26 + 5, 3, 2 ** 23
    t = torch.ones((rows, classes), dtype=torch.bfloat16, device="cuda")
    some, x = logits(np.random.default_rng(8), 12, classes, True)
    at = torch.as_tensor([0, 1, step - 2, step - 1, step, step + 1, 3 * step - 1, 3 * step, 8 * step - 1, 8 * step, rows - 2, rows - 1], device="cuda")
    t[at] = some
    lab = torch.arange(rows, device="cuda") % classes
    out = forward(t, lab, 2)
    part = at.cpu().numpy()
    check({k: v[part] for k, v in out.host().items()}, R.logprob(x, lab[at].cpu().numpy(), 2))
    flat = R.logprob(np.ones((1, classes)), np.zeros(1, np.int64), 2)
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    for name, bar in (("lse", flat["tol"][0]), ("logprob", flat["tol"][0] + 4 * R.EPS * np.log(3)), ("entropy", flat["tol_entropy"][0])):
        got = getattr(out, name)[rest].double()
        assert float((got - float(flat[name][0])).abs().max()) <= float(bar), name
    assert int((out.ids[rest] != torch.tensor([0, 1], device="cuda")).sum()) == 0
