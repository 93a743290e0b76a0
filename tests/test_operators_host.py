"""Checks without a GPU of the 8-bit checkpoints, the stored stacks and bodies,
the classification head and the log probabilities: refusals come before the
first device call, sizes are what the header says, and the references that the
GPU tests use agree with differences of their own forward passes."""
import os
import subprocess

import numpy as np
import pytest

import operator_reference as R
import paper_1707_04585_amd as rv
from paper_1707_04585_amd.binding import rvn_head_ptrs, rvn_matrix
from test_abi_host import BASE, fake, fake_params, halves, status_of

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, STRIDE, DTYPE, WS, ALIAS = -1, -2, -3, -4, -5, -6
FAR = BASE + 0x10000000


@pytest.mark.parametrize("n,c,h,w", [(1, 1, 1, 1), (2, 3, 7, 9), (4, 8, 16, 8), (3, 5, 1, 129), (64, 128, 56, 56)])
def test_checkpoint_size(n, c, h, w):
    codes = -(-n * c * h * w // 256) * 256
    assert rv.revnet_ckpt_bytes(n, c, h, w) == codes + 4 * n * c * -(-h * w // rv.CKPT_GROUP)


def test_checkpoint_refusals():
    x = fake(BASE)
    size = rv.revnet_ckpt_bytes(2, 4, 4, 4)
    k = (FAR, size)
    assert status_of(rv.revnet_ckpt_bytes, 2, 0, 4, 4)[0] == SHAPE
    assert status_of(rv.revnet_ckpt_bytes, 0, 4, 4, 4)[0] == SHAPE
    assert status_of(rv.revnet_ckpt_bytes, 2, 65536, 4, 4)[0] == SHAPE
    for call in (lambda t, p: rv.revnet_ckpt_save(t, None, p), lambda t, p: rv.revnet_ckpt_load(p, t)):
        assert status_of(call, fake(0), k)[0] == NULL
        assert status_of(call, fake(BASE, sw=2), k)[0] == STRIDE
        assert status_of(call, fake(BASE, n=0), k)[0] == SHAPE
        assert status_of(call, x, None)[0] == NULL
        assert status_of(call, x, (FAR + 4, size))[0] == STRIDE
        assert status_of(call, x, (FAR, size - 1))[0] == SHAPE
        assert status_of(call, x, (BASE, size))[0] == ALIAS
    da, dx, skip = fake(BASE), fake(BASE + 0x100000), fake(BASE + 0x200000)
    need = rv.revnet_ckpt_bn_relu_workspace_bytes(2, 4, 4, 4)
    ws = (FAR + 0x1000000, need)
    bwd = rv.revnet_ckpt_bn_relu_bwd
    assert status_of(bwd, k, None, da, skip, dx, 16, 16, 0, ws)[0] == NULL
    assert status_of(bwd, k, 16, da, skip, dx, None, 16, 0, ws)[0] == NULL
    assert status_of(bwd, k, 16, da, skip, dx, 16, None, 0, ws)[0] == NULL
    assert status_of(bwd, None, 16, da, skip, dx, 16, 16, 0, ws)[0] == NULL
    assert status_of(bwd, k, 16, da, skip, fake(BASE + 0x100000, c=3), 16, 16, 0, ws)[0] == SHAPE
    assert status_of(bwd, k, 16, da, fake(BASE + 0x200000, h=5), dx, 16, 16, 0, ws)[0] == SHAPE
    assert status_of(bwd, k, 16, da, skip, dx, 16, 16, 0, (ws[0], need - 1))[0] == WS
    assert status_of(bwd, k, 16, da, skip, dx, 16, 16, 0, None)[0] == WS
    assert status_of(bwd, k, 16, da, skip, fake(BASE + 64), 16, 16, 0, ws)[0] == ALIAS      # dx off da by a row
    assert status_of(bwd, k, 16, da, skip, fake(BASE + 0x200000 + 64), 16, 16, 0, ws)[0] == ALIAS
    assert status_of(bwd, (BASE + 0x100000, size), 16, da, skip, dx, 16, 16, 0, ws)[0] == ALIAS
    assert status_of(bwd, k, 16, da, skip, dx, 16, 16, 0, (BASE, need))[0] == ALIAS
    assert status_of(bwd, k, 16, da, skip, dx, 16, 16, 0, (FAR, need))[0] == ALIAS


def test_arrays_of_the_wrong_type_or_length_are_refused_by_the_binding():
    import torch
    x = torch.zeros(2, 4, 4, 4)
    k = (FAR, rv.revnet_ckpt_bytes(2, 4, 4, 4))
    for stats in (torch.zeros(4, 4, dtype=torch.float64), torch.zeros(4, 3), torch.zeros(4, 8)[:, ::2]):
        with pytest.raises(ValueError):
            rv.revnet_ckpt_save(x, stats, k)
    for dtype in (torch.bfloat16, torch.float64, torch.int32):
        y = torch.zeros(2, 4, 4, 4, dtype=dtype)
        for call in (lambda: rv.revnet_ckpt_save(y, None, k), lambda: rv.revnet_ckpt_load(k, y),
                     lambda: rv.revnet_body_fwd_stored(rv.BodyDesc([rv.BlockDesc("basic", 4)], [1], []), x, [[fake_params(rv.BlockDesc("basic", 4))]], [], [y], k, k),
                     lambda: rv.revnet_stack_fwd_stored(rv.BlockDesc("basic", 4), 1, x, y, [fake_params(rv.BlockDesc("basic", 4))], x, x, k, k),
                     lambda: rv.revnet_stack_bwd_stored(rv.BlockDesc("basic", 4), 1, x, x, [fake_params(rv.BlockDesc("basic", 4))], y, x,
                                                        [fake_params(rv.BlockDesc("basic", 4))], 0, k, k)):
            with pytest.raises(ValueError):
                call()
    logits, out = torch.zeros(3, 5), torch.zeros(3)
    for labels in (torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int64), torch.zeros(6, dtype=torch.int64)[::2]):
        with pytest.raises(ValueError):
            rv.revnet_logprob_fwd(logits, labels, 0, out, None, None, None, None, None)
    with pytest.raises(ValueError):
        rv.revnet_logprob_fwd(logits, None, 2, None, None, None, torch.zeros(3, 1, dtype=torch.int64), None, None)
    with pytest.raises(ValueError):
        rv.revnet_logprob_fwd(torch.zeros(5, 3).t(), None, 0, None, out, None, None, None, None)


def test_stored_stack_refusals():
    d = rv.BlockDesc("basic", 4)
    x1, x2 = halves(BASE)
    y1, y2 = halves(BASE + 0x100000)
    p = fake_params(d)
    store, fwd, bwd = rv.revnet_stack_stored_bytes(d, 2, 2, 4, 4)
    assert rv.revnet_stack_stored_bytes(d, 4, 2, 4, 4) == (2 * store, fwd, bwd)      # only the store grows with the depth
    assert fwd == rv.revnet_workspace_bytes(d, 2, 4, 4)[0]
    ws, st = (BASE + 0x800000, fwd), (FAR, store)
    call = rv.revnet_stack_fwd_stored
    assert status_of(rv.revnet_stack_stored_bytes, d, 0, 2, 4, 4)[0] == SHAPE
    assert status_of(call, d, 0, x1, x2, [p], y1, y2, st, ws)[0] == SHAPE
    assert status_of(call, d, 2, x1, x2, [p] * 2, y1, y2, None, ws)[0] == NULL
    assert status_of(call, d, 2, x1, x2, [p] * 2, y1, y2, (FAR, store - 1), ws)[0] == SHAPE
    assert status_of(call, d, 2, x1, x2, [p] * 2, y1, y2, (FAR + 8, store), ws)[0] == STRIDE
    assert status_of(call, d, 2, x1, x2, [p] * 2, y1, y2, (BASE, store), ws)[0] == ALIAS
    assert status_of(call, d, 2, x1, x2, [p] * 2, y1, y2, (ws[0], store), ws)[0] == ALIAS
    assert status_of(call, d, 2, x1, x2, [p] * 2, y1, y2, st, (ws[0], fwd - 1))[0] == WS
    assert status_of(call, d, 2, x1, x1, [p] * 2, y1, y2, st, ws)[0] == ALIAS
    dy1, dy2 = halves(BASE)
    dx1, dx2 = halves(BASE + 0x100000)
    ws = (BASE + 0x800000, bwd)
    call = rv.revnet_stack_bwd_stored
    assert status_of(call, d, 2, dy1, dy2, [p] * 2, dx2, dx1, [p] * 2, 0, st, (ws[0], bwd - 1))[0] == WS
    assert status_of(call, d, 2, dy1, dy2, [p] * 2, dy2, dx2, [p] * 2, 0, st, ws)[0] == ALIAS
    assert status_of(call, d, 2, dy1, dy2, [p] * 2, dx1, dx2, [p] * 2, 0, (FAR, store - 1), ws)[0] == SHAPE
    assert status_of(call, d, 2, dy1, dy2, [p] * 2, dx1, dx2, [p] * 2, 0, (BASE + 0x100000, store), ws)[0] == ALIAS
    bad = dict(F=p["F"], G=[dict(w=0x10, gamma=None, beta=0x30)] * 2)
    assert status_of(call, d, 2, dy1, dy2, [p] * 2, dx1, dx2, [p, bad], 0, st, ws)[0] == NULL
    assert status_of(call, rv.BlockDesc(7, 4), 2, dy1, dy2, [p] * 2, dx1, dx2, [p] * 2, 0, st, ws)[0] == DTYPE


def test_stored_body_refusals():
    layer = dict(w=0x10, gamma=0x20, beta=0x30)
    body = rv.BodyDesc([rv.BlockDesc("basic", 4), rv.BlockDesc("basic", 8)], [2, 3], [rv.DownDesc("basic", 8, 16)])
    bp, dp = dict(F=[layer] * 2, G=[layer] * 2), dict(R=[layer] * 2, S=dict(w=0x40))
    store, f, b = rv.revnet_body_stored_bytes(body, 2, 4, 4)
    assert store == rv.revnet_stack_stored_bytes(body.stages[0], 2, 2, 4, 4)[0] + rv.revnet_stack_stored_bytes(body.stages[1], 3, 2, 2, 2)[0]
    x = fake(BASE, n=2, c=8, h=4, w=4, sn=8 * 16)
    tops = [fake(BASE + 0x100000, n=2, c=8, h=4, w=4, sn=8 * 16), fake(BASE + 0x200000, n=2, c=16, h=2, w=2, sn=16 * 4)]
    dtops = [fake(BASE + 0x300000, n=2, c=8, h=4, w=4, sn=8 * 16), fake(BASE + 0x400000, n=2, c=16, h=2, w=2, sn=16 * 4)]
    st, ws = (FAR, store), (BASE + 0x800000, max(f, b))
    sp = [[bp] * 2, [bp] * 3]
    assert status_of(rv.revnet_body_fwd_stored, body, x, sp, [dp], tops, (FAR, store - 1), ws)[0] == SHAPE
    assert status_of(rv.revnet_body_fwd_stored, body, x, sp, [dp], tops, None, ws)[0] == NULL
    assert status_of(rv.revnet_body_fwd_stored, body, x, sp, [dp], tops, (BASE + 0x200000, store), ws)[0] == ALIAS
    assert status_of(rv.revnet_body_fwd_stored, body, x, sp, [dp], tops, st, (ws[0], f - 1))[0] == WS
    assert status_of(rv.revnet_body_bwd_stored, body, tops, dtops, sp, [dp], sp, [dp], 0, (BASE + 0x400000, store), ws)[0] == ALIAS
    assert status_of(rv.revnet_body_bwd_stored, body, tops, dtops, sp, [dp], sp, [dp], 0, st, (ws[0], b - 1))[0] == WS
    assert status_of(rv.revnet_body_bwd_stored, body, tops, [dtops[0], tops[1]], sp, [dp], sp, [dp], 0, st, ws)[0] == ALIAS


def matrix(ptr, rows, cols, ld=None, dtype=0):
    return rvn_matrix(ptr, dtype, rows, cols, cols if ld is None else ld)


def test_head_refusals():
    d = rv.HeadDesc(8, 5)
    x, dx = fake(BASE, c=8), fake(BASE + 0x100000, c=8)
    p = rvn_head_ptrs(16, 16, 16, 16)
    saved, need = rv.revnet_head_workspace_bytes(d, 2, 4, 4)
    s, ws, l = (FAR, saved), (FAR + 0x100000, need), matrix(BASE + 0x400000, 2, 5)
    assert status_of(rv.revnet_head_workspace_bytes, rv.HeadDesc(0, 5), 2, 4, 4)[0] == SHAPE
    assert status_of(rv.revnet_head_workspace_bytes, rv.HeadDesc(8, 0), 2, 4, 4)[0] == SHAPE
    assert status_of(rv.revnet_head_workspace_bytes, rv.HeadDesc(8, 5, 0.0), 2, 4, 4)[0] == SHAPE
    assert status_of(rv.revnet_head_workspace_bytes, d, 65536, 1, 1)[0] == SHAPE
    f = rv.revnet_head_fwd
    assert status_of(f, d, fake(BASE, c=7), p, l, s)[0] == SHAPE
    assert status_of(f, d, fake(0, c=8), p, l, s)[0] == NULL
    assert status_of(f, d, x, rvn_head_ptrs(16, 16, None, 16), l, s)[0] == NULL
    assert status_of(f, d, x, p, None, s)[0] == NULL
    assert status_of(f, d, x, p, matrix(BASE + 0x400000, 2, 6), s)[0] == SHAPE
    assert status_of(f, d, x, p, matrix(BASE + 0x400000, 2, 5, ld=4), s)[0] == STRIDE
    assert status_of(f, d, x, p, matrix(BASE + 0x400002, 2, 5), s)[0] == STRIDE
    assert status_of(f, d, x, p, matrix(BASE + 0x400000, 2, 5, dtype=1), s)[0] == DTYPE
    assert status_of(f, d, x, p, l, (FAR, saved - 1))[0] == SHAPE
    assert status_of(f, d, x, p, matrix(FAR, 2, 5), s)[0] == ALIAS
    assert status_of(f, d, x, p, matrix(BASE + 64, 2, 5), s)[0] == ALIAS
    b = rv.revnet_head_bwd
    assert status_of(b, d, x, s, l, p, x, p, 0, ws)[0] == ALIAS
    assert status_of(b, d, x, s, l, p, dx, rvn_head_ptrs(16, 16, 16, None), 0, ws)[0] == NULL
    assert status_of(b, d, x, s, l, p, dx, p, 0, (ws[0], need - 1))[0] == WS
    assert status_of(b, d, x, None, l, p, dx, p, 0, ws)[0] == NULL
    assert status_of(b, d, x, s, matrix(BASE + 0x100000, 2, 5), p, dx, p, 0, ws)[0] == ALIAS
    assert status_of(b, d, x, s, l, p, dx, p, 0, (FAR, need))[0] == ALIAS


def test_logprob_refusals():
    l, g = matrix(BASE, 3, 7), matrix(BASE + 0x1000, 3, 7)
    f, b = rv.revnet_logprob_fwd, rv.revnet_logprob_bwd
    assert status_of(rv.revnet_logprob_workspace_bytes, 0, 7, 0)[0] == SHAPE
    assert status_of(rv.revnet_logprob_workspace_bytes, 3, 7, 8)[0] == SHAPE
    assert status_of(rv.revnet_logprob_workspace_bytes, 3, 100, 33)[0] == SHAPE
    assert status_of(f, None, 16, 0, 16, 16, 16, None, None, None)[0] == NULL
    assert status_of(f, matrix(0, 3, 7), 16, 0, 16, 16, 16, None, None, None)[0] == NULL
    assert status_of(f, matrix(BASE, 0, 7), 16, 0, 16, 16, 16, None, None, None)[0] == SHAPE
    assert status_of(f, matrix(BASE, 3, (1 << 30) + 1), 16, 0, 16, 16, 16, None, None, None)[0] == SHAPE
    assert status_of(f, matrix(BASE, 3, 7, ld=6), 16, 0, 16, 16, 16, None, None, None)[0] == STRIDE
    assert status_of(f, matrix(BASE, 3, 7, dtype=5), 16, 0, 16, 16, 16, None, None, None)[0] == DTYPE
    assert status_of(f, matrix(BASE + 1, 3, 7, dtype=1), 16, 0, 16, 16, 16, None, None, None)[0] == STRIDE
    assert status_of(f, l, 16, 8, 16, 16, 16, 16, 16, None)[0] == SHAPE
    assert status_of(f, l, 16, 0, None, 16, 16, None, None, None)[0] == NULL     # labels without logprob
    assert status_of(f, l, None, 0, 16, 16, 16, None, None, None)[0] == NULL
    assert status_of(f, l, 16, 3, 16, 16, 16, None, None, None)[0] == NULL       # top_k without top_ids
    assert status_of(f, l, None, 0, None, None, None, None, None, None)[0] == NULL
    need = rv.revnet_logprob_workspace_bytes(1, 1 << 20, 20)                      # few long rows: parts in the workspace
    assert need > 0 and rv.revnet_logprob_workspace_bytes(4096, 1 << 20, 20) == 0
    long = matrix(BASE, 1, 1 << 20)
    assert status_of(f, long, 16, 20, 16, 16, 16, 16, 16, (FAR, need - 1))[0] == WS
    assert status_of(f, long, 16, 20, 16, 16, 16, 16, 16, None)[0] == WS
    assert status_of(f, long, 16, 20, 16, 16, 16, 16, 16, (BASE, need))[0] == ALIAS
    assert status_of(b, l, 16, None, 16, None, None, 1.0, g)[0] == NULL
    assert status_of(b, l, None, 16, 16, None, None, 1.0, g)[0] == NULL
    assert status_of(b, l, None, 16, 16, 16, 16, 1.0, g)[0] == NULL              # d_logprob without labels
    assert status_of(b, l, 16, 16, None, None, 16, 1.0, g)[0] == NULL            # d_entropy without entropy
    assert status_of(b, l, 16, 16, 16, None, None, 1.0, matrix(BASE + 0x1000, 3, 6))[0] == SHAPE
    assert status_of(b, l, 16, 16, 16, None, None, 1.0, matrix(BASE + 0x1000, 3, 7, dtype=1))[0] == DTYPE
    assert status_of(b, l, 16, 16, 16, None, None, 1.0, matrix(BASE + 4, 3, 7))[0] == ALIAS
    assert status_of(b, l, 16, 16, 16, None, None, 1.0, matrix(BASE, 3, 7, ld=8))[0] == ALIAS


def test_division_by_a_known_number_is_exact(tmp_path):
    src = tmp_path / "div.cpp"
    src.write_text("""
#include "fast_div.h"
int main() {
    uint64_t r = 88172645463325252ull;
    auto next = [&] { r ^= r << 13; r ^= r >> 7; r ^= r << 17; return r; };
    for (int i = 0; i < 4000; ++i) {
        const int d = i < 1000 ? i + 1 : i < 1031 ? 1 << (i - 1000) : (int)(next() >> (33 + next() % 30)) + 1;
        const rvn::FastDiv f = rvn::fast_div(d);
        for (int j = 0; j < 64; ++j) {
            const int64_t k = (int64_t)(next() >> 33) / d * d;   // a multiple of d and its neighbours
            const int64_t e[4] = {k, k - 1, k + d - 1, (int64_t)(next() >> 33)};
            for (int64_t v : e)
                if (v >= 0 && v <= 0x7fffffff && rvn::quotient((int)v, f) != (int)(v / d)) return 1;
        }
        if (rvn::quotient(0x7fffffff, f) != 0x7fffffff / d) return 2;
    }
    return 0;
}
""")
    exe = tmp_path / "div"
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_1707_04585_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    subprocess.run([str(exe)], check=True)


# ---- the references ------------------------------------------------------------------------------


def differences(f, x, at, step=1e-5):
    out = []
    for i in at:
        hi, lo = x.copy(), x.copy()
        hi.flat[i] += step
        lo.flat[i] -= step
        out.append((f(hi) - f(lo)) / (2 * step))
    return np.array(out)


def test_reference_gradient_of_log_probabilities_is_that_of_differences():
    rng = np.random.default_rng(1)
    x, labels = rng.standard_normal((4, 9)) * 2, np.array([3, 0, -1, 8])
    gl, ge = rng.uniform(0.5, 1.5, 4), rng.uniform(-1, 1, 4)

    def f(v):
        r = R.logprob(v, labels, 0)
        return -0.25 * (gl @ r["logprob"] + ge @ r["entropy"])

    r = R.logprob(x, labels, 0)
    got = R.logprob_bwd(x, labels, r["lse"], r["entropy"], gl, ge, -0.25)
    assert np.abs(got.ravel() - differences(f, x, range(x.size))).max() < 1e-8


def test_reference_gradient_of_the_head_is_that_of_differences():
    rng = np.random.default_rng(2)
    x, w = rng.standard_normal((3, 4, 3, 2)), rng.standard_normal((5, 4))
    gamma, beta, b, dl = rng.uniform(0.5, 1.5, 4), rng.standard_normal(4) * 0.1, rng.standard_normal(5), rng.standard_normal((3, 5))
    _, g = R.head(x, gamma, beta, w, b, dl)
    at = range(x.size)
    assert np.abs(g["dx"].ravel() - differences(lambda v: (R.head(v, gamma, beta, w, b) * dl).sum(), x, at)).max() < 1e-7
    assert np.abs(g["gamma"] - differences(lambda v: (R.head(x, v, beta, w, b) * dl).sum(), gamma, range(4))).max() < 1e-7
    assert np.abs(g["beta"] - differences(lambda v: (R.head(x, gamma, v, w, b) * dl).sum(), beta, range(4))).max() < 1e-7
    assert np.abs(g["w"].ravel() - differences(lambda v: (R.head(x, gamma, beta, v, b) * dl).sum(), w, range(20))).max() < 1e-7


@pytest.mark.parametrize("h,w", [(1, 1), (7, 7), (8, 16), (3, 43), (20, 13)])
def test_reference_codes_keep_the_decisions_and_stay_within_a_scale(h, w):
    rng = np.random.default_rng(h * 100 + w)
    x = (rng.standard_normal((3, 6, h, w)) * 2 + rng.standard_normal((6, 1, 1))).astype(np.float32)
    gamma = rng.uniform(0.5, 1.5, 6) * np.array([1, 1, -1, 1, 0, 1])
    stats = R.statistics(x, gamma, rng.standard_normal(6) * 0.1)
    for st, steps in ((None, 0.5), (stats, 1.0)):
        q, s = R.encode(x, st)
        v = R.decode(q, s)
        each = np.repeat(s, R.GROUP, axis=2)[:, :, :h * w].reshape(x.shape)
        assert np.all(np.abs(v.astype(np.float64) - x) <= steps * each * (1 + 1e-4))
        assert np.abs(q.astype(int)).max() <= (126 if st is None else 127)
    assert np.array_equal(R.positive(v, stats), R.positive(x, stats))


def test_sizes_that_the_launches_cannot_count_are_refused():
    assert rv.revnet_ckpt_bytes(1, 64, 8192, 8192) > 0                               # 2^30 quads, the most
    assert status_of(rv.revnet_ckpt_bytes, 1, 65, 8192, 8192)[0] == SHAPE
    assert status_of(rv.revnet_ckpt_bn_relu_workspace_bytes, 1, 65, 8192, 8192)[0] == SHAPE
    assert rv.revnet_ckpt_bytes(1 << 18, 32768, 1, 1) > 0                            # 2^33 in all
    assert status_of(rv.revnet_ckpt_bytes, (1 << 18) + 1, 32768, 1, 1)[0] == SHAPE
    big = fake(BASE, n=1, c=65, h=8192, w=8192)
    assert status_of(rv.revnet_ckpt_save, big, None, (FAR, 1 << 50))[0] == SHAPE
    assert status_of(rv.revnet_ckpt_load, (FAR, 1 << 50), big)[0] == SHAPE
    assert rv.revnet_stack_stored_bytes(rv.BlockDesc("basic", 64), 1, 1, 8192, 8192)[0] > 0
    assert status_of(rv.revnet_stack_stored_bytes, rv.BlockDesc("basic", 65), 1, 1, 8192, 8192)[0] == SHAPE
    body = rv.BodyDesc([rv.BlockDesc("basic", 65), rv.BlockDesc("basic", 8)], [2, 3], [rv.DownDesc("basic", 130, 16)])
    assert status_of(rv.revnet_body_stored_bytes, body, 1, 8192, 8192)[0] == SHAPE
    assert rv.revnet_head_workspace_bytes(rv.HeadDesc(16384, 5), 65535, 1, 1)[0] > 0
    assert status_of(rv.revnet_head_workspace_bytes, rv.HeadDesc(16385, 5), 65535, 1, 1)[0] == SHAPE
    assert status_of(rv.revnet_head_workspace_bytes, rv.HeadDesc(2048, 1 << 20), 1, 1, 1)[0] == SHAPE


@pytest.mark.parametrize("rows,classes", [(1, 65537), (3, 40000), (70, 131072), (300, 131072), (2048, 12000)])
def test_log_probability_workspace_suffices_for_fewer_top_classes(rows, classes):
    sizes = [rv.revnet_logprob_workspace_bytes(rows, classes, k) for k in range(rv.MAX_TOP_K + 1)]
    assert sizes == sorted(sizes)
