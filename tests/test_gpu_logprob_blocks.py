"""Logits and their gradient as column blocks of one matrix."""
import numpy as np
import pytest

from test_gpu_logprob import forward, labels_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,classes", [(1, 5), (7, 3), (33, 64), (600, 1001), (70, 29001), (4100, 258)])
@pytest.mark.parametrize("first", [True, False])
def test_gradient_beside_the_logits_in_one_matrix(rows, classes, bf16, first):
    """Neither block's bytes reach the other, on either side, nor the columns around both; the bits are those of matrices of
    their own at the same alignment."""
    import torch
    import paper_1707_04585_amd as rv
    rng = np.random.default_rng(rows + classes)
    dtype = torch.bfloat16 if bf16 else torch.float32
    gap, ld = 3, 2 * classes + 9
    both = torch.full((rows, ld), 99.0, dtype=dtype, device="cuda")
    a, b = both[:, 2:2 + classes], both[:, 2 + classes + gap:2 + 2 * classes + gap]
    x, out = (a, b) if first else (b, a)
    x.copy_(torch.as_tensor((rng.standard_normal((rows, classes)) * 3).astype(np.float32)))
    lab = torch.as_tensor(labels_of(rng, rows, classes, odd=True)).cuda()
    apart, alone = both.clone(), both.clone()
    same = lambda whole, t: whole.as_strided(t.shape, t.stride(), t.storage_offset())  # noqa: E731
    o = forward(x, lab, 0)
    rv.revnet_logprob_bwd(same(apart, x), lab, o.lse, o.entropy, None, o.entropy, -0.5, same(alone, out))
    rv.revnet_logprob_bwd(x, lab, o.lse, o.entropy, None, o.entropy, -0.5, out)
    torch.cuda.synchronize()
    # (alone differs from what `both` was in the gradient's block alone)
    assert torch.equal(torch.nan_to_num(both, nan=77.0), torch.nan_to_num(alone, nan=77.0))
    assert not torch.equal(torch.nan_to_num(both, nan=77.0), torch.nan_to_num(apart, nan=77.0))
