"""Every class of a row counts once, wherever it lies: at the borders of the vectors, of a thread's groups of vectors, of the
parts that workgroups take and of the row itself."""
import numpy as np
import pytest

import operator_reference as R
from test_gpu_logprob import Out, check, forward, labels_of, logits

pytestmark = pytest.mark.gpu

# rows, classes, top_k: a wavefront a row (short, and long ones in numbers), a workgroup, several of them, on rows of odd length
SHAPES = [
    (37, 255, 1), (300, 1000, 3), (2050, 5001, 2), (64, 6011, 1), (40, 9001, 13), (1, 20011, 2), (5, 33000, 2), (3, 65537, 1),
    (70, 29001, 2), (193, 33001, 1), (200, 131073, 1),
]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,classes,top_k", SHAPES)
def test_one_class_or_two_neighbours_at_every_place_of_a_row(rows, classes, top_k, bf16):
    """All other classes are -infinity.  One class: lse is its value, log probability and entropy are 0, exactly (the sum is 1
    and its logarithm 0).  Two neighbours of one value: the sum is 2; lse adds one rounding to that of its logarithm (an ulp)."""
    import torch
    import paper_1707_04585_amd as rv
    value = 0.75
    for pad, offset, count in ((0, 0, 1), (3, 1, 2)):
        dtype = torch.bfloat16 if bf16 else torch.float32
        ld = classes + pad
        flat = torch.full((rows * ld + offset + 8,), 99.0, dtype=dtype, device="cuda")
        t = flat[offset:offset + rows * ld].view(rows, ld)[:, :classes]
        t.fill_(-torch.inf)
        batches = -(-classes // rows)
        out, need = Out(batches * rows, top_k), rv.revnet_logprob_workspace_bytes(rows, classes, top_k)
        ws = torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device="cuda")
        place = torch.arange(batches * rows, device="cuda").remainder_(classes)
        both = torch.stack([place, (place + 1) % classes], 1)[:, :count].contiguous()
        for b in range(batches):
            s = slice(b * rows, (b + 1) * rows)
            t.scatter_(1, both[s], value)
            rv.revnet_logprob_fwd(t, place[s], top_k, out.logprob[s], out.entropy[s], out.lse[s], out.ids[s], out.top[s], ws)
            t.scatter_(1, both[s], -torch.inf)
        torch.cuda.synchronize()
        log = float(np.log(count))
        off = lambda name, want: float((getattr(out, name).double() - want).abs().max())  # noqa: E731
        bar = 0.0 if count == 1 else 2 * R.EPS
        assert off("lse", value + log) <= bar * (value + 2 * log) and off("logprob", -log) <= bar * log and off("entropy", log) <= bar * log
        # the largest classes in order, then the lowest of the others
        first = torch.sort(both, 1).values
        want = first[:, :top_k]
        if top_k > count:
            rest = torch.arange(top_k, device="cuda").expand(len(place), -1)     # skips the classes that came first
            for k in range(count):
                rest = rest + (rest >= first[:, k:k + 1]).long()
            want = torch.cat([first, rest[:, :top_k - count]], 1)
        assert torch.equal(out.ids, want)
        top = torch.where(torch.arange(top_k, device="cuda") < count, -log, -torch.inf)
        assert bool(((out.top.double() - top).abs() <= bar * log).logical_or(out.top.double() == top).all())
        if pad:
            assert (flat[offset:offset + rows * ld].view(rows, ld)[:, classes:] == 99).all()


# rows, classes, top_k, workgroups a row (0: a wavefront) for fp32 and bf16 at these sizes.  test_gpu_logprob.py allows for the
# terms that a thread adds where a wavefront has the whole row; here for those that it has.
TERMS = [
    (1, 40000, 5, 20, 10), (8, 65537, 5, 33, 17), (1, 131072, 32, 32, 16), (70, 50000, 5, 13, 7), (200, 131072, 1, 6, 4), (1, 262147, 5, 64, 64),
    (40, 9001, 5, 1, 1), (2100, 4001, 5, 0, 0),
]


@pytest.mark.parametrize("uniform", [False, True])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,classes,top_k,many32,many16", TERMS)
def test_sums_within_the_terms_that_a_thread_adds(rows, classes, top_k, many32, many16, bf16, uniform):
    """Drawn rows, and rows of one value but for a thousandth of the classes, in which a lost vector would show."""
    import torch
    many = many16 if bf16 else many32
    rng = np.random.default_rng(rows + classes)
    t, x = logits(rng, rows, classes, bf16, pad=1, offset=1)
    if uniform:
        x = np.where(rng.random((rows, classes)) < 1e-3, x, 0.5)
        t.copy_(torch.as_tensor(x))
    lab = labels_of(rng, rows, classes)
    ref = R.logprob(x, lab, top_k)
    # a part of at most classes / many + 16, split over 256 threads (64) in vectors of up to 8, begun up to a cache line early
    terms = (classes / max(many, 1) + 16 + 64) / (256 if many else 64) + 16
    less = classes / 64 - terms
    ref["tol_entropy"] = ref["tol_entropy"] - R.EPS * less * (1 + 2 * ref["spread"])
    ref["tol"] = ref["tol"] - R.EPS * less
    out = forward(t, torch.as_tensor(lab).cuda(), top_k)
    torch.cuda.synchronize()
    check(out.host(), ref)


@pytest.mark.parametrize("base,step", [(10.0, 1), (-11.0, 1), (10.0, 8), (-11.0, 5), (0.7, 3)])
@pytest.mark.parametrize("rows,classes,top_k", [(2, 600, 32), (2050, 2500, 5), (3, 5000, 5), (4, 9001, 13), (2, 40000, 12), (1, 65537, 32)])
def test_distinct_values_in_a_narrow_band(rows, classes, top_k, base, step):
    """fp32 logits a few units in the last place apart: many share the upper half of their bits with the bound that the search
    for the top classes ends at, more than its list holds."""
    import torch
    rng = np.random.default_rng(classes + step)
    first = np.float32(base).view(np.int32)
    x = (first + step * np.stack([rng.permutation(classes) for _ in range(min(rows, 20))])).astype(np.int32).view(np.float32)
    x = np.resize(x, (rows, classes))
    t, _ = logits(rng, rows, classes, False, pad=1, offset=1)
    t.copy_(torch.as_tensor(x))
    lab = labels_of(rng, rows, classes)
    out = forward(t, torch.as_tensor(lab).cuda(), top_k)
    torch.cuda.synchronize()
    some = slice(0, 40)
    ref = R.logprob(x[some], lab[some], top_k)
    check({k: v[some] for k, v in out.host().items()}, ref)
    ids = out.host()["ids"]
    assert np.array_equal(ids, ids[np.arange(rows) % 20 if rows > 20 else np.arange(rows)])
