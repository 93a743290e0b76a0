"""What is timed for the operators of a training step's ends: activation checkpoints in 8 bits (saved, read back,
and used by the backward pass of BatchNorm + ReLU), the classification head, the log probabilities of given labels
with entropy and top alternatives, and their gradient.

``run`` computes a case in elementary torch operations while ``own`` is false, and through the public entry points
(``paper_1707_04585_amd``) where it is true.
"""
from __future__ import annotations

import torch

own = False

DEVICE = "cuda:0"
GROUP = 128           # pixels that share a scale in a checkpoint
TOP = 126             # the largest code that rounding alone gives
TINY = 2.0 ** -126    # the smallest scale
# A pixel whose normalised value lies nearer to the ReLU's border than this is moved off it: which side it is on
# is then the same for every order in which the batch statistics are summed.
BORDER = 1e-4


def listed():
    return [
        # One half of the single block of the tests (N=4, 8 + 8 channels, 8x8): launches and latency.
        dict(name="ckpt_block_tiny", op="ckpt", n=4, c=8, h=8, w=8, half=True, bn=True),
        # One half of the benchmark's bottleneck stage (56x56): throughput of saving and reading back.
        dict(name="ckpt_bottleneck", op="ckpt", n=64, c=128, h=56, w=56, half=True, bn=True),
        # BatchNorm backward in a basic block of the 32x32 networks, added to the residual stream's derivative.
        dict(name="bnbwd_cifar", op="bnbwd", n=128, c=16, h=32, w=32, half=True, skip=True),
        # An inner layer of the 7x7 stage of the 224x224 networks: planes that no vector access divides.
        dict(name="bnbwd_7x7", op="bnbwd", n=32, c=512, h=7, w=7, half=False, skip=False),
        # The first layer of the benchmark's bottleneck function.
        dict(name="bnbwd_bottleneck", op="bnbwd", n=64, c=128, h=56, w=56, half=True, skip=True),
        # Evaluation on ten classes: the label's log probability, entropy and the first five.
        dict(name="logprob_ten", op="logprob", rows=128, classes=10, top=5, bf16=False, masked=0, unlabelled=False),
        # One position of a large vocabulary, as a sampler scores it.
        dict(name="logprob_single", op="logprob", rows=1, classes=65537, top=20, bf16=True, masked=0, unlabelled=False),
        # Scoring sequences over a vocabulary whose tail is padding and masked; some positions carry no label.
        dict(name="logprob_vocabulary", op="logprob", rows=4096, classes=50021, top=8, bf16=True, masked=21, unlabelled=True),
        # The training gradient at the batch of the 224x224 networks, mean loss.
        dict(name="grad_thousand", op="grad", rows=32, classes=1000, bf16=False, masked=0, unlabelled=False, entropy=False),
        # The gradient over a vocabulary with a weight for each position and an entropy term.
        dict(name="grad_vocabulary", op="grad", rows=4096, classes=32003, bf16=True, masked=3, unlabelled=True, entropy=True),
        # Head of the three-stage network for 32x32 images: forward and backward.
        dict(name="head_cifar", op="head", n=128, c=112, h=8, w=8, classes=10),
        # Head of the four-stage network for 224x224 images: forward and backward.
        dict(name="head_imagenet", op="head", n=32, c=2048, h=7, w=7, classes=1000),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case of the same ranges: every operator, planes from one pixel to 64x64, classes from two to a large
    vocabulary, rows from one to thousands, both types."""
    while True:
        op = rng.choice(["ckpt", "bnbwd", "logprob", "grad", "head"])
        case = dict(op=op)
        if op in ("ckpt", "bnbwd"):
            side = _log(rng, 1, 64)
            case.update(n=_log(rng, 1, 128), c=_log(rng, 1, 512), h=side, w=max(1, side + rng.choice([0, 0, -3, 2])),
                        half=rng.random() < 0.5)
            case.update(bn=rng.random() < 0.8) if op == "ckpt" else case.update(skip=rng.random() < 0.5)
            if op == "bnbwd" and case["n"] * case["h"] * case["w"] < 16:
                continue   # a batch's statistics want a batch
        elif op == "head":
            side = rng.randint(1, 14)
            case.update(n=_log(rng, 2, 256), c=_log(rng, 8, 2048), h=side, w=side, classes=_log(rng, 2, 4096))
            if case["n"] * side * side < 16:
                continue
        else:
            case.update(rows=_log(rng, 1, 8192), classes=_log(rng, 2, 131072), bf16=rng.random() < 0.5, unlabelled=rng.random() < 0.3)
            case["masked"] = rng.choice([0, 0, case["classes"] // 10])
            case.update(top=min(rng.choice([0, 1, 5, 20, 32]), case["classes"])) if op == "logprob" else case.update(entropy=rng.random() < 0.5)
        if all(work(case)[k] <= max(work(c)[k] for c in listed()) for k in ("bytes", "flops")):
            return case


def work(case):
    """Every input read once, every output written once; arithmetic of the products and, roughly, of the elements."""
    op = case["op"]
    if op in ("ckpt", "bnbwd"):
        plane = case["h"] * case["w"]
        items, planes = case["n"] * case["c"] * plane, case["n"] * case["c"]
        scales = 4 * planes * -(-plane // GROUP)
        if op == "ckpt":   # save: values in, codes out; load: codes in, values out
            return {"bytes": 10 * items + 2 * scales + (16 * case["c"] if case["bn"] else 0), "flops": 8 * items}
        return {"bytes": (9 + 4 * case["skip"]) * items + scales + 24 * case["c"], "flops": 12 * items}
    if op == "head":
        items, pooled = case["n"] * case["c"] * case["h"] * case["w"], case["n"] * case["c"]
        weights = case["classes"] * case["c"]
        return {"bytes": 12 * items + 12 * weights + 8 * case["n"] * case["classes"] + 16 * case["c"] + 8 * case["classes"],
                "flops": 6 * pooled * case["classes"] + 16 * items}
    rows, classes, size = case["rows"], case["classes"], 2 if case["bf16"] else 4
    if op == "logprob":
        return {"bytes": rows * (classes * size + 20 + 12 * case["top"]), "flops": 5 * rows * classes}
    return {"bytes": rows * (2 * classes * size + 16 + 8 * case["entropy"]), "flops": 8 * rows * classes}


# ---- inputs -------------------------------------------------------------------------------------------


def _normal(shape, gen):
    return torch.empty(shape, dtype=torch.float32, device=DEVICE).normal_(generator=gen)


def _uniform(shape, lo, hi, gen):
    return torch.empty(shape, dtype=torch.float32, device=DEVICE).uniform_(lo, hi, generator=gen)


def _activations(case, gen):
    """[n, c, h, w] with a mean and a deviation of its own for each channel; `half`: the second half of a tensor with twice the channels."""
    n, c, h, w = (case[k] for k in "nchw")
    whole = _normal((n, 2 * c if case.get("half") else c, h, w), gen)
    x = whole[:, -c:]
    return x.mul_(_uniform((c, 1, 1), 0.5, 2.0, gen)).add_(_normal((c, 1, 1), gen))


def _statistics(x, gamma, beta, eps=1e-5):
    """Rows mean, rstd, scale and shift of BatchNorm over the batch."""
    x = x.double()
    var, mean = torch.var_mean(x, (0, 2, 3), unbiased=False)
    mean, rstd = mean.float(), (var + eps).rsqrt().float()
    scale = gamma * rstd
    return torch.stack([mean, rstd, scale, (beta.double() - mean.double() * scale.double()).float()])


def _labels(case, gen):
    labels = torch.randint(0, case["classes"] - case["masked"], (case["rows"],), generator=gen, device=DEVICE)
    if case["unlabelled"]:
        labels = torch.where(_uniform((case["rows"],), 0.0, 1.0, gen) < 0.1, -1, labels)
    return labels


def _logits(case, gen):
    """Deviation 3, and the label's own raised by 4: a model that has learned something."""
    rows, classes = case["rows"], case["classes"]
    x, labels = _normal((rows, classes), gen).mul_(3.0), _labels(case, gen)
    x.scatter_add_(1, labels.clamp_min(0)[:, None], torch.full((rows, 1), 4.0, device=DEVICE))
    if case["masked"]:
        x[:, classes - case["masked"]:] = -torch.inf
    return x.to(torch.bfloat16) if case["bf16"] else x, labels


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    op, s = case["op"], dict(case=case)
    empty = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=DEVICE)  # noqa: E731
    if op in ("ckpt", "bnbwd"):
        n, c, h, w = (case[k] for k in "nchw")
        x = _activations(case, gen)
        stats = _statistics(x, _uniform((c,), 0.5, 1.5, gen) * torch.sign(_normal((c,), gen) + 1.0), _normal((c,), gen).mul_(0.1))
        groups = -(-h * w // GROUP)
        codes = -(-n * c * h * w // 256) * 256
        s.update(ckpt=torch.zeros(codes + 4 * n * c * groups, dtype=torch.uint8, device=DEVICE), shape=(n, c, h, w))
        if op == "ckpt":
            s.update(x=x, stats=stats if case["bn"] else None, y=empty(n, c, h, w))
            return s
        q, scales = _quantise(x, stats)
        s["ckpt"][:q.numel()] = q.reshape(-1).view(torch.uint8)
        s["ckpt"][codes:] = scales.reshape(-1).view(torch.uint8)
        s.update(stats=stats, da=_normal((n, c, h, w), gen), dx=empty(n, c, h, w), d_gamma=empty(c), d_beta=empty(c),
                 skip=_normal((n, 2 * c if case["half"] else c, h, w), gen)[:, -c:] if case["skip"] else None)
    elif op == "head":
        n, c, h, w, classes = (case[k] for k in ("n", "c", "h", "w", "classes"))
        x = _activations(case, gen)
        gamma, beta = _uniform((c,), 0.5, 1.5, gen), _normal((c,), gen).mul_(0.1)
        stats = _statistics(x, gamma, beta)
        z = x * stats[2, :, None, None] + stats[3, :, None, None]
        x += torch.where(z.abs() < BORDER, 4 * BORDER / stats[2, :, None, None], 0.0)
        s.update(x=x, gamma=gamma, beta=beta, weight=_normal((classes, c), gen).mul_(c ** -0.5), bias=_normal((classes,), gen).mul_(0.1),
                 dlogits=_normal((n, classes), gen).div_(n), logits=empty(n, classes), dx=empty(n, c, h, w),
                 d_gamma=empty(c), d_beta=empty(c), d_weight=empty(classes, c), d_bias=empty(classes))
    else:
        rows, classes = case["rows"], case["classes"]
        s["logits"], s["labels"] = _logits(case, gen)
        if op == "logprob":
            top = case["top"]
            s.update(logprob=empty(rows), entropy=empty(rows), lse=empty(rows), top_ids=empty(rows, top, dtype=torch.int64), top_logprob=empty(rows, top))
        else:
            x = s["logits"].float()
            s["lse"] = torch.logsumexp(x, 1)
            p = torch.softmax(x, 1)
            s["entropy"] = -(p * torch.where(p > 0, x - s["lse"][:, None], 0.0)).sum(1) if case["entropy"] else None
            s["d_logprob"] = _uniform((rows,), 0.5, 1.5, gen) if case["entropy"] else None
            s["d_entropy"] = _uniform((rows,), 0.0, 0.1, gen) if case["entropy"] else None
            s.update(scale=-1.0 / rows, d_logits=torch.empty_like(s["logits"]))
    return s


# ---- the operators, plain -------------------------------------------------------------------------------


def _quantise(x, stats):
    """Codes [n, c, h*w] (int8) and scales [n, c, groups]: the largest magnitude of GROUP pixels becomes TOP; with `stats`
    a code whose value fell on the other side of the ReLU's border moves one step back over it."""
    n, c, h, w = x.shape
    plane, groups = h * w, -(-h * w // GROUP)
    x = torch.nn.functional.pad(x.reshape(n, c, plane), (0, groups * GROUP - plane)).view(n, c, groups, GROUP)
    most = x.abs().amax(3, keepdim=True).clamp_min(TOP * TINY).double()
    step, inverse = (most / TOP).float(), (TOP / most).float()
    q = torch.round(x * inverse)
    if stats is not None:
        scale, shift = stats[2, :, None, None].double(), stats[3, :, None, None].double()
        over = lambda v: v.double() * scale + shift > 0  # noqa: E731
        want = over(x)
        q = torch.where(want != over(q * step), q + torch.sign(scale).float() * torch.where(want, 1.0, -1.0), q)
    return q.to(torch.int8).view(n, c, -1)[..., :plane].contiguous(), step.view(n, c, groups)


def _values(ckpt, shape):
    """The values that a checkpoint's codes stand for."""
    n, c, h, w = shape
    plane, groups = h * w, -(-h * w // GROUP)
    codes = -(-n * c * plane // 256) * 256
    q = ckpt[:n * c * plane].view(torch.int8).view(n, c, plane).float()
    scales = ckpt[codes:].view(torch.float32).view(n, c, groups)
    return (q * scales.repeat_interleave(GROUP, 2)[..., :plane]).view(shape), scales


def _plain_bnbwd(s):
    v, _ = _values(s["ckpt"], s["shape"])
    mean, rstd, scale, shift = (t[:, None, None] for t in s["stats"])
    dz = torch.where(v.double() * scale + shift > 0, s["da"], 0.0)
    xh = (v - mean) * rstd
    d_beta, d_gamma = dz.sum((0, 2, 3)), (dz * xh).sum((0, 2, 3))
    count = v.numel() // v.shape[1]
    dx = scale * (dz - (d_beta / count)[:, None, None] - xh * (d_gamma / count)[:, None, None])
    return [dx if s["skip"] is None else s["skip"] + dx, d_gamma, d_beta]


def _plain_logprob(s):
    x, labels, top = s["logits"].float(), s["labels"], s["case"]["top"]
    most = x.amax(1, keepdim=True)
    d = x - most
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    lse = most + log_total
    entropy = log_total - (e * torch.where(e > 0, d, 0.0)).sum(1, keepdim=True) / total
    logprob = torch.where(labels < 0, 0.0, d.gather(1, labels.clamp_min(0)[:, None])[:, 0] - log_total[:, 0])
    # larger values first, the lower index among equals: one 64-bit key
    bits = (x + 0.0).view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7fffffff)).long() * 2 ** 32 + (2 ** 32 - 1 - torch.arange(x.shape[1], device=x.device))
    ids = 2 ** 32 - 1 - (key.topk(top, 1).values & (2 ** 32 - 1))
    return [logprob, entropy[:, 0], lse[:, 0], ids, d.gather(1, ids) - log_total]


def _plain_grad(s):
    x, labels, scale = s["logits"].float(), s["labels"], s["scale"]
    logp = x - s["lse"][:, None]
    p = torch.exp(logp)
    given = torch.where(labels < 0, 0.0, scale if s["d_logprob"] is None else scale * s["d_logprob"])[:, None]
    d = -given * p
    d.scatter_add_(1, labels.clamp_min(0)[:, None], given)
    if s["d_entropy"] is not None:
        d -= (scale * s["d_entropy"])[:, None] * p * torch.where(p > 0, logp + s["entropy"][:, None], 0.0)
    return d.to(s["logits"].dtype)


def _plain_head(s):
    x, weight, dlogits = s["x"], s["weight"], s["dlogits"]
    plane, count = x.shape[2] * x.shape[3], x.numel() // x.shape[1]
    mean = x.mean((0, 2, 3), keepdim=True)
    rstd = ((x - mean).square().mean((0, 2, 3), keepdim=True) + 1e-5).rsqrt()
    xh = (x - mean) * rstd
    gamma, beta = s["gamma"][:, None, None], s["beta"][:, None, None]
    z = xh * gamma + beta
    pooled = z.clamp_min(0).mean((2, 3))
    logits = pooled @ weight.t() + s["bias"]
    dz = torch.where(z > 0, (dlogits @ weight / plane)[:, :, None, None], 0.0)
    d_beta, d_gamma = dz.sum((0, 2, 3)), (dz * xh).sum((0, 2, 3))
    dx = gamma * rstd * (dz - (d_beta / count)[:, None, None] - xh * (d_gamma / count)[:, None, None])
    return [logits, dx, d_gamma, d_beta, dlogits.t() @ pooled, dlogits.sum(0)]


def _plain(s):
    op = s["case"]["op"]
    if op == "ckpt":
        q, scales = _quantise(s["x"], s["stats"])
        return [(q.float() * scales.repeat_interleave(GROUP, 2)[..., :q.shape[2]]).view(s["shape"]), scales]
    return {"bnbwd": _plain_bnbwd, "logprob": _plain_logprob, "grad": _plain_grad, "head": _plain_head}[op](s)


# ---- the operators, through the framework ----------------------------------------------------------------


def _workspace(s, nbytes):
    if "ws" not in s:
        s["ws"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEVICE)
    return s["ws"]


def _own(s):
    import paper_1707_04585_amd as rv
    op, case, stream = s["case"]["op"], s["case"], torch.cuda.current_stream()
    if op == "ckpt":
        n, c, h, w = s["shape"]
        rv.revnet_ckpt_save(s["x"], s["stats"], s["ckpt"], stream)
        rv.revnet_ckpt_load(s["ckpt"], s["y"], stream)
        return [s["y"], s["ckpt"][-(-n * c * h * w // 256) * 256:].view(torch.float32).view(n, c, -1)]
    if op == "bnbwd":
        ws = s["ws"] if "ws" in s else _workspace(s, rv.revnet_ckpt_bn_relu_workspace_bytes(*s["shape"]))
        rv.revnet_ckpt_bn_relu_bwd(s["ckpt"], s["stats"], s["da"], s["skip"], s["dx"], s["d_gamma"], s["d_beta"], 0, ws, stream)
        return [s["dx"], s["d_gamma"], s["d_beta"]]
    if op == "logprob":
        ws = s["ws"] if "ws" in s else _workspace(s, rv.revnet_logprob_workspace_bytes(case["rows"], case["classes"], case["top"]))
        rv.revnet_logprob_fwd(s["logits"], s["labels"], case["top"], s["logprob"], s["entropy"], s["lse"], s["top_ids"], s["top_logprob"], ws, stream)
        return [s["logprob"], s["entropy"], s["lse"], s["top_ids"], s["top_logprob"]]
    if op == "grad":
        rv.revnet_logprob_bwd(s["logits"], s["labels"], s["lse"], s["entropy"], s["d_logprob"], s["d_entropy"], s["scale"], s["d_logits"], stream)
        return s["d_logits"]
    if "desc" not in s:
        s["desc"] = rv.HeadDesc(case["c"], case["classes"])
        saved, nbytes = rv.revnet_head_workspace_bytes(s["desc"], case["n"], case["h"], case["w"])
        s["saved"] = torch.empty(saved, dtype=torch.uint8, device=DEVICE)
        _workspace(s, nbytes)
        s["params"] = rv.pack_head(dict(gamma=s["gamma"], beta=s["beta"], w=s["weight"], b=s["bias"]))
        s["grads"] = rv.pack_head(dict(gamma=s["d_gamma"], beta=s["d_beta"], w=s["d_weight"], b=s["d_bias"]))
    rv.revnet_head_fwd(s["desc"], s["x"], s["params"], s["logits"], s["saved"], stream)
    rv.revnet_head_bwd(s["desc"], s["x"], s["saved"], s["dlogits"], s["params"], s["dx"], s["grads"], 0, s["ws"], stream)
    return [s["logits"], s["dx"], s["d_gamma"], s["d_beta"], s["d_weight"], s["d_bias"]]


def run(state):
    return _own(state) if own else _plain(state)


# ---- the same from the definitions, in 64 bits --------------------------------------------------------------


def _exact_values(x, stats):
    """A checkpoint's values and scales: its scales, the products with their inverses and the values are single-precision
    numbers by definition, everything between is 64 bits wide."""
    n, c, h, w = x.shape
    single = lambda t: t.to(torch.float32).to(torch.float64)  # noqa: E731
    flat = x.reshape(n * c, h * w).double()
    group = torch.arange(h * w, device=x.device).div(GROUP, rounding_mode="floor").expand(n * c, -1)
    most = torch.full((n * c, -(-h * w // GROUP)), TOP * TINY, dtype=torch.float64, device=x.device).scatter_reduce(1, group, flat.abs(), "amax")
    step = single(most / TOP)
    q = torch.round(single(flat * single(TOP / most).gather(1, group)))
    each = step.gather(1, group)
    if stats is not None:
        scale, shift = (t.double().repeat(n)[:, None] for t in stats[2:])
        side = torch.sign(torch.clamp_min(flat * scale + shift, 0)) - torch.sign(torch.clamp_min(single(q * each) * scale + shift, 0))
        q = q + side * torch.sign(scale)
    return single(q * each).view(x.shape), step.view(n, c, -1)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "ckpt":
        return list(_exact_values(s["x"], s["stats"]))
    if op == "bnbwd":
        n, c, h, w = s["shape"]
        gen = torch.Generator(device=DEVICE)
        gen.manual_seed(seed)
        v = _exact_values(_activations(case, gen), s["stats"])[0].transpose(0, 1).reshape(c, -1)
        mean, rstd, scale, shift = (t.double()[:, None] for t in s["stats"])
        dz = s["da"].double().transpose(0, 1).reshape(c, -1) * (v * scale + shift).gt(0)
        xh = (v - mean) * rstd
        dx = scale * (dz - dz.mean(1, keepdim=True) - xh * (dz * xh).mean(1, keepdim=True))
        dx = dx.view(c, n, h, w).transpose(0, 1)
        return [dx if s["skip"] is None else dx + s["skip"].double(), (dz * xh).sum(1), dz.sum(1)]
    if op == "head":
        x, weight, dl = s["x"].double(), s["weight"].double(), s["dlogits"].double()
        plane = x.shape[2] * x.shape[3]
        x = x.transpose(0, 1).flatten(1)                                  # [c, n * plane]
        var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
        rstd = (var + 1e-5) ** -0.5
        gamma, beta = s["gamma"].double()[:, None], s["beta"].double()[:, None]
        xh = (x - mean) * rstd
        z = (gamma * xh + beta).view(case["c"], case["n"], plane)
        pooled = torch.relu(z).sum(2) / plane                             # [c, n]
        logits = (weight @ pooled).t() + s["bias"].double()
        dz = ((weight.t() @ dl.t() / plane)[:, :, None] * z.gt(0)).flatten(1)
        dx = gamma * rstd * (dz - dz.mean(1, keepdim=True) - xh * (dz * xh).mean(1, keepdim=True))
        dx = dx.view(case["c"], case["n"], case["h"], case["w"]).transpose(0, 1)
        return [logits, dx, (dz * xh).sum(1), dz.sum(1), (pooled @ dl).t(), dl.sum(0)]
    x, labels = s["logits"].double(), s["labels"]
    at = torch.where(labels < 0, 0, labels)[:, None]
    if op == "logprob":
        lse = torch.logsumexp(x, 1)
        logp = x - lse[:, None]
        entropy = -torch.special.xlogy(logp.exp(), logp.exp()).sum(1)
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
        logprob = logp.gather(1, at)[:, 0] * (labels >= 0)
        return [logprob, entropy, lse, order, logp.gather(1, order)]
    logp = x - s["lse"].double()[:, None]
    p = logp.exp()
    given = each = torch.full((case["rows"],), s["scale"], dtype=torch.float64, device=DEVICE)
    if s["d_logprob"] is not None:
        given = given * s["d_logprob"].double()
    d = -(given * (labels >= 0))[:, None] * p
    d[torch.arange(case["rows"], device=DEVICE), at[:, 0]] += given * (labels >= 0)
    if s["d_entropy"] is not None:
        d += (each * s["d_entropy"].double())[:, None] * (-torch.special.xlogy(p, p) - p * s["entropy"].double()[:, None])
    return d
