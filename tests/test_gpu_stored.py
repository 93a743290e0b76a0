"""Stacks and bodies that store every layer's input in 8 bits instead of
recomputing it: forward bits equal to the reversible ones, gradients against
ordinary backprop of the oracle with its stored activations put through the
same 8 bits, and a whole network's training step from image to loss."""
import numpy as np
import pytest

import operator_reference as R
import synth_inputs as S

pytestmark = pytest.mark.gpu

# Against the oracle's own 8 bits.  The GPU's layer inputs differ from the oracle's by about 1e-6 of their deviation; a
# scale is about 0.024 deviations, so about 1e-4 of the codes fall to the neighbour, each a change by a scale: 1e-2 * 0.024,
# about 3e-4 of an activation's norm.  A gradient sums such changes with random signs: the same share at each of a few layers.
CODES = 2e-3
# bf16 operands: the bar of the other bf16 tests or, where two correct summation orders are further apart than that (a
# difference of 1e-7 moves a share of the operands by a whole bf16 step, and some ReLU decisions with them), 1.5 times what
# the oracle in float32 is off the oracle in float64.
BF16, FLOOR_FACTOR = 2e-2, 1.5
# Against unrounded activations: a uniform rounding error of a scale's 1/sqrt(12) is 0.7 % of the deviation, at most twice
# that where codes step over the border, and a layer's share of it adds to those above in quadrature (at most 8 layers).
ROUNDED = 2.5e-2

CASES = [
    dict(kind="basic", n=4, c=16, h=8, w=8, depth=1, width=None, conv="f32", affine="random"),
    dict(kind="basic", n=6, c=32, h=16, w=16, depth=2, width=None, conv="f32", affine="random"),
    dict(kind="basic", n=5, c=14, h=9, w=11, depth=2, width=None, conv="f32", affine="random"),
    dict(kind="basic", n=40, c=64, h=16, w=16, depth=1, width=None, conv="f32", affine="random"),
    dict(kind="bottleneck", n=4, c=32, h=8, w=8, depth=2, width=12, conv="f32", affine="random"),
    dict(kind="bottleneck", n=3, c=128, h=14, w=14, depth=1, width=16, conv="f32", affine="random"),
    dict(kind="basic", n=6, c=32, h=16, w=16, depth=2, width=None, conv="bf16", affine="random"),
    dict(kind="basic", n=8, c=112, h=8, w=8, depth=1, width=None, conv="bf16", affine="random"),
    dict(kind="bottleneck", n=8, c=128, h=16, w=16, depth=2, width=32, conv="bf16", affine="random"),
    dict(kind="bottleneck", n=5, c=200, h=13, w=11, depth=1, width=44, conv="bf16", affine="random"),
    dict(kind="bottleneck", n=4, c=512, h=7, w=7, depth=1, width=128, conv="bf16", affine="random"),
]


def eight_bits(stored, params):
    """The oracle's stored state with every layer's input rounded to a checkpoint (statistics and decisions as they were)."""
    out = []
    for block, P in zip(stored, params):
        new = {}
        for fn in ("F", "G"):
            layers = []
            for st, L in zip(block[fn], P[fn]):
                x = st["x"].astype(np.float32)
                stats = R.statistics(st["x"], L["gamma"], L["beta"])
                v = R.decode(*R.encode(x, stats)).astype(np.float64)
                mean, rstd, scale, shift = (s.astype(np.float64)[:, None, None] for s in stats)
                u = v * scale + shift
                layers.append(dict(st, x=v, xhat=(v - mean) * rstd, u=u, a=np.maximum(u, 0)))
            new[fn] = layers
        out.append(new)
    return out


# float32 sums of a few hundred terms leave u = x * scale + shift off by 1e-6 at most: where the oracle's |u| is below this,
# the ReLU's decision may be either.
UNDECIDED = 2e-6


def either_way(stored):
    """Copies of the stored state, each with one undecided ReLU decision the other way: what that one decision moves bounds
    how far a correct result may be off beside the rounding."""
    for k, block in enumerate(stored):
        for fn in ("F", "G"):
            for l, st in enumerate(block[fn]):
                for i in np.flatnonzero(np.abs(st["u"]) < UNDECIDED):
                    u = st["u"].copy()
                    u.flat[i] = -1e-30 if u.flat[i] > 0 else 1e-30
                    layers = list(block[fn])
                    layers[l] = dict(st, u=u, a=np.maximum(u, 0))
                    yield stored[:k] + [dict(block, **{fn: layers})] + stored[k + 1:]


def grads_of(r):
    from paper_1707_04585_amd.torch_harness import download_grads
    return download_grads(r.grads)


@pytest.mark.parametrize("cfg", CASES, ids=lambda c: "%s_%s_c%d_%dx%d_d%d" % (c["kind"], c["conv"], c["c"], c["h"], c["w"], c["depth"]))
def test_stack(oracle, cfg):
    import torch
    from paper_1707_04585_amd.torch_harness import StackRunner
    x, params, dy = S.draw_stack(cfg["n"] * 100 + cfg["c"], **cfg)
    c = cfg["c"] // 2
    plain, r = StackRunner(**cfg), StackRunner(stored=True, **cfg)
    plain.set_params(params)
    r.set_params(params)
    r.store.fill_(0xFF)
    r.ws.fill_(0xFF)
    Y, Z = plain.new_pair(x), r.new_pair(x)
    plain.forward(Y, Y)
    r.forward(Z, Z)
    torch.cuda.synchronize()
    assert torch.equal(Y[0], Z[0])                       # the forward pass is the same one
    kept = r.store.clone()
    DY, DX = r.new_pair(dy), r.new_pair()
    r.ws.fill_(0xFF)
    r.backward(None, DY, None, DX)
    torch.cuda.synchronize()
    assert torch.equal(r.store, kept)
    dx, grads = r.to_host(DX[0]), grads_of(r)
    first = {k: v.clone() for k, v in zip("ab", (DX[0], r.grads[0]["F"][0]["w"]))}
    r.backward(None, DY, None, DY, accumulate=True)      # in place, added to: the same bits
    torch.cuda.synchronize()
    assert torch.equal(DY[0], first["a"]) and torch.equal(r.grads[0]["F"][0]["w"], first["b"] + first["b"])

    split = lambda t: (np.ascontiguousarray(t[:, :c]), np.ascontiguousarray(t[:, c:]))
    dy1, dy2 = split(dy.astype(np.float32).astype(np.float64))
    bar = CODES if cfg["conv"] == "f32" else BF16
    with oracle.conv_operands(cfg["conv"]):
        _, _, _, stored = oracle.stack_fwd(*split(x.astype(np.float32).astype(np.float64)), params, keep=True)
        grad = oracle.flatten_grads(grads)

        def backprop(state):
            a, b, ref = oracle.stack_bwd_stored(state, params, dy1, dy2)
            return dict(dx=np.concatenate([a, b], 1), grads=oracle.flatten_grads(ref))

        exact, rounded = backprop(stored), backprop(eight_bits(stored, params))
        floor = dict(dx=0.0, grads=0.0)
        if cfg["conv"] == "bf16":
            single = [np.ascontiguousarray(t, dtype=np.float32) for t in split(x)]
            _, _, _, other = oracle.stack_fwd(*single, S.cast_params(params, np.float32), eps=np.float32(1e-5), keep=True)
            other = [{fn: [{k: v if k == "in_hw" else v.astype(np.float64) for k, v in st.items()} for st in b[fn]] for fn in ("F", "G")}
                     for b in other]
            second = backprop(eight_bits(other, params))
            floor = {k: FLOOR_FACTOR * oracle.rel_l2(second[k], rounded[k]) for k in floor}
        moved = dict(dx=0.0, grads=0.0)
        for state in either_way(stored):
            other = backprop(state)
            for key in moved:
                moved[key] += oracle.rel_l2(other[key], exact[key])
        for ref, limit in ((rounded, bar), (exact, ROUNDED if cfg["conv"] == "f32" else ROUNDED + BF16)):
            off = dict(dx=oracle.rel_l2(dx, ref["dx"]), grads=oracle.rel_l2(grad, ref["grads"]))
            print(cfg, "limit %.1e" % limit, {k: "%.2e, undecided %.2e, floor %.2e" % (v, moved[k], floor[k]) for k, v in off.items()},
                  flush=True)
            assert all(v < max(limit, floor[k]) + moved[k] for k, v in off.items()), (off, limit, floor, moved)


def net(stored, conv="f32", head_classes=10):
    from paper_1707_04585_amd.torch_harness import NetRunner
    rng = np.random.default_rng(77)
    cfg = dict(kind="basic", n=6, h=16, w=16, channels=(16, 32), depths=(2, 1), widths=(None, None), conv=conv)
    stages, downs = [], []
    for s, (ch, depth) in enumerate(zip(cfg["channels"], cfg["depths"])):
        stages.append(S.draw_stack(50 + s, kind="basic", n=1, c=ch, h=2, w=2, depth=depth, width=None, affine="random")[1])
    layer = lambda ci, co, k: dict(w=rng.standard_normal((co, ci, k, k)) * np.sqrt(2 / (ci * k * k)), gamma=rng.uniform(0.5, 1.5, ci),
                                   beta=rng.standard_normal(ci) * 0.1)
    downs.append(dict(R=[dict(layer(16, 32, 3), stride=2), layer(32, 32, 3)], S=dict(w=rng.standard_normal((32, 16, 1, 1)) * 0.3)))
    stem = dict(w=rng.standard_normal((16, 3, 3, 3)) * 0.3, stride=1, pool=False)
    head = dict(gamma=rng.uniform(0.5, 1.5, 32), beta=rng.standard_normal(32) * 0.1, w=rng.standard_normal((head_classes, 32)) * 0.2,
                b=rng.standard_normal(head_classes) * 0.1)
    r = NetRunner(dict(cfg, stored=stored), stem, head=head)
    r.set_params(stages, downs)
    img = rng.standard_normal((6, 3, 16, 16)).astype(np.float32)
    return r, img, (stages, downs, stem, head), rng.integers(0, head_classes, 6)


def grad_list(r):
    """Every gradient of the network, in one order."""
    out = [r.stem_dw]
    for st in r.body.stage_grads:
        out += [t for P in st for fn in ("F", "G") for L in P[fn] for t in L.values()]
    for D in r.body.down_grads:
        out += [t for L in D["R"] for t in L.values()] + [D["S"]["w"]]
    return out + list(r.head.grads.values())


def oracle_step(oracle, img, model, labels):
    """Log probabilities and the image filter's gradient of the mean negative log likelihood, ordinary backprop in 64 bits."""
    stages, downs, stem, head = model
    x, stem_kept = oracle.stem_fwd(img.astype(np.float64), dict(w=stem["w"].astype(np.float32).astype(np.float64), stride=1, pool=False))
    single = lambda v: v.astype(np.float32).astype(np.float64)
    stages = [[{fn: [{k: single(v) for k, v in L.items()} for L in P[fn]] for fn in ("F", "G")} for P in st] for st in stages]
    downs = [dict(R=[{k: single(v) if isinstance(v, np.ndarray) else v for k, v in L.items()} for L in D["R"]], S=dict(w=single(D["S"]["w"])))
             for D in downs]
    h = {k: single(v) for k, v in head.items()}
    tops, kept = oracle.body_fwd(x, stages, downs, keep=True)
    top = tops[-1]
    logits = R.head(top, h["gamma"], h["beta"], h["w"], h["b"])
    r = R.logprob(logits, labels, 3)
    dl = R.logprob_bwd(logits, labels, r["lse"], r["entropy"], None, None, -1.0 / len(labels))
    _, g = R.head(top, h["gamma"], h["beta"], h["w"], h["b"], dl)
    dx = oracle.body_bwd_stored(kept, stages, downs, g["dx"])
    return r, g, oracle.stem_bwd(stem_kept, dict(w=stem["w"], stride=1, pool=False), dx[0])


@pytest.mark.parametrize("stored", [False, True])
def test_training_step_of_a_network_from_image_to_loss(oracle, stored):
    import torch
    r, img, model, labels = net(stored)
    dev, lab = torch.as_tensor(img).cuda(), torch.as_tensor(labels).cuda()
    r.forward(dev, labels=lab)
    r.backward(labels=lab)
    torch.cuda.synchronize()
    ref, head_grads, stem_grad = oracle_step(oracle, img, model, labels)
    h = r.head
    assert np.abs(h.logprob.cpu().numpy() - ref["logprob"]).max() < 1e-4      # the forward bar of 1e-5 on logits of a few units
    assert np.array_equal(h.top_ids.cpu().numpy()[:, :3], ref["ids"])
    bar = ROUNDED if stored else 1e-3
    for k in ("w", "b", "gamma", "beta"):
        assert oracle.rel_l2(h.grads[k].cpu().numpy(), head_grads[k]) < 1e-4, k
    assert oracle.rel_l2(r.stem_dw.cpu().numpy(), stem_grad) < bar


@pytest.mark.parametrize("conv", ["f32", "bf16"])
def test_training_step_captured_and_replayed(conv):
    """Stem, stored body, head, loss and back in one graph, replayed with other images and labels: the eager step's bits."""
    import torch
    a, img, _, labels = net(True, conv)
    b = net(True, conv)[0]
    dev, lab = torch.as_tensor(img).cuda(), torch.as_tensor(labels).cuda()

    def step(r, stream=None):
        r.forward(dev, stream, lab)
        r.backward(stream, lab)

    step(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, torch.cuda.current_stream())
    for k in range(4):
        dev.mul_(-0.75).add_(0.1 * k)
        lab.add_(1).remainder_(10)
        for t in grad_list(a):
            t.zero_()
        graph.replay()
        step(b)
        torch.cuda.synchronize()
        for t, u in zip(grad_list(a), grad_list(b)):
            assert torch.equal(t, u)
        assert torch.equal(a.head.logprob, b.head.logprob) and torch.equal(a.head.top_ids, b.head.top_ids)


def test_stored_body_agrees_with_the_reversible_one(oracle):
    """A three-stage body: the forward bits, the tops left as they were, and gradients within the codes' rounding."""
    import torch
    from paper_1707_04585_amd.torch_harness import BodyRunner
    rng = np.random.default_rng(5)
    cfg = dict(kind="bottleneck", n=4, h=16, w=16, channels=(32, 64, 128), depths=(1, 2, 1), widths=(8, 16, 32), conv="f32")
    stages = [S.draw_stack(60 + s, kind="bottleneck", n=1, c=ch, h=2, w=2, depth=d, width=wd, affine="random")[1]
              for s, (ch, d, wd) in enumerate(zip(cfg["channels"], cfg["depths"], cfg["widths"]))]
    downs = []
    for ci, co in ((32, 64), (64, 128)):
        shapes = [(ci, co // 4, 1, 1), (co // 4, co // 4, 3, 2), (co // 4, co, 1, 1)]
        downs.append(dict(R=[dict(w=rng.standard_normal((o, i, k, k)) * np.sqrt(2 / (i * k * k)), gamma=rng.uniform(0.5, 1.5, i),
                                  beta=rng.standard_normal(i) * 0.1, stride=st) for i, o, k, st in shapes],
                          S=dict(w=rng.standard_normal((co, ci, 1, 1)) * np.sqrt(2 / ci))))
    x = torch.as_tensor(rng.standard_normal((4, 32, 16, 16)).astype(np.float32)).cuda()
    dy = torch.as_tensor(rng.standard_normal((4, 128, 4, 4)).astype(np.float32)).cuda()
    runs = []
    for stored in (False, True):
        r = BodyRunner(stored=stored, **cfg)
        r.set_params(stages, downs)
        r.forward(x)
        torch.cuda.synchronize()
        tops = [t.clone() for t in r.tops]
        r.dtops[-1].copy_(dy)
        r.backward()
        torch.cuda.synchronize()
        runs.append((r, tops))
    (a, tops_a), (b, tops_b) = runs
    for u, v, w in zip(tops_a, tops_b, b.tops):
        assert torch.equal(u, v) and torch.equal(v, w)
    flat = lambda r: torch.cat([t.flatten() for st in r.stage_grads for P in st for fn in ("F", "G") for L in P[fn] for t in L.values()] +
                               [t.flatten() for D in r.down_grads for L in D["R"] for t in L.values()])
    off = float((flat(a) - flat(b)).norm() / flat(a).norm())
    print("stored against reversible gradients: %.2e" % off, "at the input: %.2e" % float((a.dtops[0] - b.dtops[0]).norm() / a.dtops[0].norm()), flush=True)
    assert off < ROUNDED
    assert float((a.dtops[0] - b.dtops[0]).norm() / a.dtops[0].norm()) < ROUNDED
