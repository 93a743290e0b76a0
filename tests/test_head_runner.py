"""Order of the calls that the head's runner makes, without a GPU: the entry points are replaced by records of their names."""
import numpy as np
import pytest
import torch

from paper_1707_04585_amd import torch_harness as H


def head(c=32, classes=4):
    return dict(gamma=np.ones(c), beta=np.zeros(c), w=np.zeros((classes, c)), b=np.zeros(classes))


def network(monkeypatch, calls, **cfg):
    for name in ("stem_fwd", "stem_bwd", "body_fwd", "body_bwd", "head_fwd", "head_bwd", "logprob_fwd", "logprob_bwd"):
        monkeypatch.setattr(H.B, "revnet_" + name, lambda *a, name=name: calls.append((name, a)))
    cfg = dict(dict(kind="basic", n=2, h=8, w=8, channels=(16, 32), depths=(1, 1), widths=(None, None)), **cfg)
    r = H.NetRunner(cfg, dict(w=np.zeros((16, 3, 3, 3)), stride=1, pool=False), device="cpu", head=head())
    r.body._sp = r.body._dp = r.body._sg = r.body._dg = None
    return r


def names(calls):
    out = [name for name, _ in calls]
    calls.clear()
    return out


def test_the_gradient_is_formed_from_scores_of_the_same_forward_pass(monkeypatch):
    calls = []
    r = network(monkeypatch, calls)
    img, lab = torch.zeros(2, 3, 8, 8), torch.zeros(2, dtype=torch.int64)
    there, back = ["stem_fwd", "body_fwd", "head_fwd"], ["logprob_bwd", "head_bwd", "body_bwd", "stem_bwd"]
    r.forward(img)                     # no labels: nothing is scored yet
    r.backward(labels=lab)
    assert names(calls) == there + ["logprob_fwd"] + back
    r.forward(img, labels=lab)
    r.backward(labels=lab)             # (the scores are those of this pass)
    assert names(calls) == there + ["logprob_fwd"] + back
    r.forward(img)                     # those of the pass before are of other logits
    r.backward(labels=lab)
    assert names(calls) == there + ["logprob_fwd"] + back
    r.forward(img)
    r.head.score(lab)
    r.backward(labels=lab)
    assert names(calls) == there + ["logprob_fwd"] + back
    r.backward(labels=lab)             # what came between may have been a replayed graph: scored again
    assert names(calls) == ["logprob_fwd"] + back


def test_a_head_on_a_stream_in_fixed_point_is_refused():
    """The head reads floats; the top of such a body holds codes."""
    cfg = dict(kind="basic", n=2, h=8, w=8, channels=(16, 32), depths=(1, 1), widths=(None, None), frac_bits=16)
    stem = dict(w=np.zeros((16, 3, 3, 3)), stride=1, pool=False)
    with pytest.raises(ValueError):
        H.NetRunner(cfg, stem, device="cpu", head=head())
    assert H.NetRunner(cfg, stem, device="cpu").head is None


def test_the_head_of_a_network_has_the_networks_epsilon(monkeypatch):
    calls = []
    assert network(monkeypatch, calls).head.desc.bn_eps == 1e-5
    r = network(monkeypatch, calls, eps=1e-3)
    assert r.head.desc.bn_eps == 1e-3 and all(st.bn_eps == 1e-3 for st in r.body.desc.stages)


def test_labels_for_a_network_without_a_head_are_refused(monkeypatch):
    calls = []
    r = network(monkeypatch, calls)
    r.head = None
    img, lab = torch.zeros(2, 3, 8, 8), torch.zeros(2, dtype=torch.int64)
    for call in (lambda: r.forward(img, labels=lab), lambda: r.backward(labels=lab)):
        with pytest.raises(ValueError):
            call()
    assert calls == []
    r.forward(img)
    r.backward()
    assert names(calls) == ["stem_fwd", "body_fwd", "body_bwd", "stem_bwd"]
