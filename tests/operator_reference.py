"""Plain references of the 8-bit checkpoints, the classification head and the
log probabilities: numpy, 64 bits wherever the definition does not name a
single-precision number."""
import numpy as np

GROUP, TOP = 128, 126
EPS = 2.0 ** -24   # half a unit in the last place of a float32, relative
f32 = np.float32


def statistics(x, gamma, beta, eps=1e-5):
    """float32 [4, c] (mean, rstd, scale, shift) of an [n, c, h, w] array."""
    x = np.asarray(x, np.float64)
    mean = x.mean((0, 2, 3)).astype(f32)
    rstd = (1.0 / np.sqrt(x.var((0, 2, 3)) + eps)).astype(f32)
    scale = np.asarray(gamma, f32) * rstd
    shift = (np.asarray(beta, np.float64) - mean.astype(np.float64) * scale).astype(f32)
    return np.stack([mean, rstd, scale, shift])


def positive(v, stats):
    """Whether v * scale + shift > 0, decided on the exact value (what one fused multiply-add rounds keeps its sign)."""
    scale, shift = (stats[i].astype(np.float64)[:, None, None] for i in (2, 3))
    with np.errstate(invalid="ignore"):
        return np.asarray(v, np.float64) * scale + shift > 0


def encode(x, stats=None):
    """(codes int8 [n, c, h, w], scales float32 [n, c, groups]) of a float32 array."""
    x = np.asarray(x, f32)
    n, c, h, w = x.shape
    groups = -(-h * w // GROUP)
    flat = x.reshape(n, c, h * w)
    q = np.zeros_like(flat)
    scales = np.empty((n, c, groups), f32)
    over = None if stats is None else positive(x, stats).reshape(flat.shape)
    for g in range(groups):
        part = flat[:, :, g * GROUP:(g + 1) * GROUP]
        most = np.abs(part).max(2)
        fine = np.isfinite(most)
        a = np.maximum(np.where(fine, most, 1), f32(TOP * 2.0 ** -126)).astype(f32)
        step, inverse = a / f32(TOP), f32(TOP) / a
        with np.errstate(invalid="ignore"):
            codes = np.rint(np.where(fine[:, :, None], part, 0) * inverse[:, :, None])
        if stats is not None:
            got = positive((codes * step[:, :, None])[..., None], stats)[..., 0]
            want = over[:, :, g * GROUP:(g + 1) * GROUP] & fine[:, :, None]
            got &= fine[:, :, None]
            codes = codes + (want.astype(f32) - got.astype(f32)) * np.sign(stats[2])[:, None]
        q[:, :, g * GROUP:(g + 1) * GROUP] = codes
        scales[:, :, g] = np.where(fine, step, np.nan)
    return q.astype(np.int8).reshape(x.shape), scales


def decode(q, scales):
    n, c, h, w = q.shape
    each = np.repeat(scales, GROUP, axis=2)[:, :, :h * w].reshape(q.shape)
    return q.astype(f32) * each


def bn_relu_bwd(v, stats, da, skip=None):
    """-> dx, d_gamma, d_beta and, for tolerances, the sums of magnitudes that the two sums have."""
    mean, rstd, scale, _ = (s.astype(np.float64)[:, None, None] for s in stats)
    dz = np.where(positive(v, stats), np.asarray(da, np.float64), 0.0)
    xh = (np.asarray(v, np.float64) - mean) * rstd
    count = v.size // v.shape[1]
    db, dg = dz.sum((0, 2, 3)), (dz * xh).sum((0, 2, 3))
    ab, ag = np.abs(dz).sum((0, 2, 3)), np.abs(dz * xh).sum((0, 2, 3))
    c1, c2 = (db / count)[:, None, None], (dg / count)[:, None, None]
    dx = scale * (dz - c1 - xh * c2) + (0 if skip is None else np.asarray(skip, np.float64))
    # How far a float32 evaluation may be off.  Sums: a thread adds at most 256 terms, each rounded three times, then a
    # tree in double.  dx: some ten roundings of quantities of these magnitudes, and the sums' own errors.
    ts = 264 * EPS
    size = np.abs(scale) * (np.abs(dz) + np.abs(c1) + np.abs(xh * c2)) + (0 if skip is None else np.abs(skip))
    tol = 10 * EPS * size + np.abs(scale) * ts * ((ab / count)[:, None, None] + np.abs(xh) * (ag / count)[:, None, None])
    return dx, dg, db, dict(dx=tol, dg=ts * ag, db=ts * ab)


def logprob(x, labels, top_k):
    """x [rows, classes] -> dict of the outputs in 64 bits and `tol`, how far float32 sums of a row may be off."""
    x = np.asarray(x, np.float64)
    rows, classes = x.shape
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        m = x.max(1, keepdims=True)
        d = np.where(np.isneginf(x), -np.inf, x - np.where(np.isneginf(m), 0, m))
        e = np.exp(d)
        s = e.sum(1, keepdims=True)
        log_s = np.log(s)
        p = e / s
        finite = np.where(np.isneginf(d), 0, d)
        entropy = (log_s - (p * finite).sum(1, keepdims=True))[:, 0]
        lse = (m + log_s)[:, 0]
        logp = np.where(np.isneginf(x), -np.inf, d - log_s)
    empty = np.isneginf(m[:, 0])
    bad = np.isnan(x).any(1) | np.isposinf(x).any(1)
    entropy = np.where(bad, np.nan, np.where(empty, 0.0, entropy))
    lse = np.where(bad, np.nan, np.where(empty, -np.inf, lse))
    logp = np.where(bad[:, None], np.nan, np.where(empty[:, None], -np.inf, logp))
    order = np.argsort(-np.where(np.isnan(x), np.inf, x), axis=1, kind="stable")   # a stable sort keeps the lower index first
    if np.isnan(x).any():
        order = np.stack([np.lexsort((np.arange(classes), -np.where(np.isnan(r), 0, r), ~np.isnan(r))) for r in x])
    ids = order[:, :top_k]
    inside = (labels >= 0) & (labels < classes)
    given = np.take_along_axis(logp, np.where(inside, labels, 0)[:, None], 1)[:, 0]
    given = np.where(labels == -1, 0.0, np.where(inside, given, np.nan))
    # A term exp(x - m) is off by the rounding of its exponent (relative 2 eps per unit of it) and of the exponential (4 eps);
    # a thread adds at most classes / 64 + 32 of them; the results add roundings of m, x - m and log s themselves.
    with np.errstate(invalid="ignore"):
        spread = np.nan_to_num((p * np.abs(finite)).sum(1))
        tol = EPS * (classes / 64 + 48 + 4 * spread + 2 * np.abs(np.nan_to_num(m[:, 0], neginf=0, posinf=0)) + 4 * np.nan_to_num(np.abs(log_s[:, 0]), posinf=0))
        second = np.nan_to_num((p * np.abs(finite) * (2 + 2 * np.abs(finite))).sum(1))
    return dict(logprob=given, entropy=entropy, lse=lse, ids=ids, top=np.take_along_axis(logp, ids, 1), tol=tol, spread=spread,
                tol_entropy=tol * (1 + spread) + EPS * (second + (classes / 64 + 48) * spread))


def logprob_bwd(x, labels, lse, entropy, d_logprob, d_entropy, scale):
    x, lse = np.asarray(x, np.float64), np.asarray(lse, np.float64)[:, None]
    rows, classes = x.shape
    with np.errstate(invalid="ignore", over="ignore"):
        logp = x - lse
        p = np.exp(logp)
    given = np.full(rows, float(scale)) if d_logprob is None else scale * np.asarray(d_logprob, np.float64)
    given = np.where(labels == -1, 0.0, given)
    given = np.where((labels < -1) | (labels >= classes), np.nan, given)
    out = np.zeros((rows, classes))
    for r in range(rows):
        if np.isneginf(lse[r, 0]):
            continue
        ge = 0.0 if d_entropy is None else float(scale) * float(d_entropy[r])
        if given[r] != 0:
            out[r] -= given[r] * p[r]
            if 0 <= labels[r] < classes:
                out[r, labels[r]] += given[r]
        if ge != 0:
            out[r] -= ge * p[r] * (np.where(np.isneginf(logp[r]), 0, logp[r]) + float(entropy[r]))
    return out


def head(x, gamma, beta, w, b, dl=None, eps=1e-5):
    """logits and, with dl, dict(dx, gamma, beta, w, b)."""
    x = np.asarray(x, np.float64)
    n, c, h, wd = x.shape
    mean = x.mean((0, 2, 3), keepdims=True)
    rstd = 1.0 / np.sqrt(x.var((0, 2, 3), keepdims=True) + eps)
    g, be = np.reshape(gamma, (c, 1, 1)).astype(np.float64), np.reshape(beta, (c, 1, 1)).astype(np.float64)
    xh = (x - mean) * rstd
    z = xh * g + be
    pooled = np.maximum(z, 0).mean((2, 3))
    logits = pooled @ np.asarray(w, np.float64).T + b
    if dl is None:
        return logits
    dl = np.asarray(dl, np.float64)
    dz = np.where(z > 0, (dl @ np.asarray(w, np.float64))[:, :, None, None] / (h * wd), 0.0)
    dbeta, dgamma = dz.sum((0, 2, 3)), (dz * xh).sum((0, 2, 3))
    count = n * h * wd
    dx = g * rstd * (dz - dbeta[:, None, None] / count - xh * dgamma[:, None, None] / count)
    return logits, dict(dx=dx, gamma=dgamma, beta=dbeta, w=dl.T @ pooled, b=dl.sum(0))
