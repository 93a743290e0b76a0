"""Arguments of the classification head and of the log probabilities, without a GPU: what the binding has to refuse
because a kernel would read it wrongly or beyond its end, and what it must not refuse."""
import pytest
import torch

import paper_1707_04585_amd as rv
from paper_1707_04585_amd.binding import rvn_head_desc, rvn_head_ptrs
from test_abi_host import BASE, fake, status_of
from test_operators_host import ALIAS, FAR, NULL, matrix

C, CLASSES = 8, 5
SHAPES = dict(gamma=(C,), beta=(C,), w=(CLASSES, C), b=(CLASSES,))


def head_arrays(**other):
    return {k: other.get(k, torch.zeros(SHAPES[k])) for k in SHAPES}


def head_calls(desc):
    """Calls of the head with the arrays given in each place that takes such a set; every other argument is in order."""
    x, dx, logits = fake(BASE, c=C), fake(BASE + 0x100000, c=C), matrix(BASE + 0x400000, 2, CLASSES)
    raw, far = rvn_head_ptrs(16, 16, 16, 16), (FAR, 1 << 20)
    return [lambda P: rv.revnet_head_fwd(desc, x, P, logits, far),
            lambda P: rv.revnet_head_bwd(desc, x, far, logits, P, dx, raw, 0, (FAR + (1 << 21), 1 << 20)),
            lambda P: rv.revnet_head_bwd(desc, x, far, logits, raw, dx, P, 0, (FAR + (1 << 21), 1 << 20))]


@pytest.mark.parametrize("bad", [
    dict(gamma=torch.zeros(C, dtype=torch.float64)), dict(beta=torch.zeros(C, dtype=torch.int32)),
    dict(w=torch.zeros(CLASSES, C, dtype=torch.bfloat16)), dict(b=torch.zeros(CLASSES, dtype=torch.float16)),
    dict(w=torch.zeros(C, CLASSES).t()),
], ids=lambda b: next(iter(b)))
def test_head_arrays_of_another_type_or_with_gaps_are_refused_when_packed(bad):
    with pytest.raises(ValueError):
        rv.pack_head(head_arrays(**bad))


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("desc", [rv.HeadDesc(C, CLASSES), rvn_head_desc(C, CLASSES, 1e-5)], ids=["HeadDesc", "rvn_head_desc"])
@pytest.mark.parametrize("bad", [
    dict(gamma=torch.zeros(C - 1)), dict(beta=torch.zeros(C + 1)), dict(w=torch.zeros(CLASSES - 1, C)), dict(w=torch.zeros(CLASSES, C - 1)),
    dict(w=torch.zeros(C, CLASSES)), dict(b=torch.zeros(1)),
], ids=lambda b: "%s%s" % next((k, list(v.shape)) for k, v in b.items()))
def test_head_arrays_of_another_size_are_refused(bad, desc, packed):
    arrays = head_arrays(**bad)
    if packed:
        arrays = rv.pack_head(arrays)
    for call in head_calls(desc):
        with pytest.raises(ValueError):
            call(arrays)


def test_head_arrays_that_fit_reach_the_library():
    """Arrays in order, packed or not, and raw pointers get past the binding: what is refused next is refused by the library."""
    desc, x, far = rv.HeadDesc(C, CLASSES), fake(BASE, c=C), (FAR, 1 << 20)
    wide = {k: v.view(1, -1, 1, 1) if v.dim() == 1 else v.view(CLASSES, C, 1, 1) for k, v in head_arrays().items()}
    for P in (head_arrays(), rv.pack_head(head_arrays()), wide, rv.pack_head(dict(gamma=16, beta=16, w=16, b=16)), rvn_head_ptrs(16, 16, 16, 16)):
        assert status_of(rv.revnet_head_fwd, desc, x, P, None, far)[0] == NULL
    missing = rv.pack_head(dict(head_arrays(), b=None))
    assert status_of(rv.revnet_head_fwd, desc, x, missing, matrix(BASE + 0x400000, 2, CLASSES), far)[0] == NULL
