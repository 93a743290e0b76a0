"""A network's backward pass after a forward pass that scored nothing."""
import pytest

from test_gpu_stored import grad_list, net

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stored", [False, True])
def test_gradients_after_a_forward_pass_without_labels(oracle, stored):
    """Of the first step of a runner, and behind a pass that scored other images: the bits of a pass with labels."""
    import torch
    (a, img, _, labels), b, first = net(stored), net(stored)[0], net(stored)[0]
    dev, lab = torch.as_tensor(img).cuda(), torch.as_tensor(labels).cuda()
    a.forward(dev, labels=lab)
    a.backward(labels=lab)
    first.head.lse.fill_(5.0)
    first.forward(dev)
    first.backward(labels=lab)
    b.forward(-2 * dev, labels=lab)
    b.forward(dev)
    b.backward(labels=lab)
    torch.cuda.synchronize()
    for t, u, v in zip(grad_list(a), grad_list(first), grad_list(b)):
        assert torch.equal(t, u) and torch.equal(t, v)


def test_gradients_behind_a_replayed_forward_pass_without_labels(oracle):
    """The forward pass in a graph, replayed with other images, the backward pass by itself: the bits of an eager step."""
    import torch
    (a, img, _, labels), b = net(True), net(True)[0]
    dev, lab = torch.as_tensor(img).cuda(), torch.as_tensor(labels).cuda()
    a.forward(dev)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.forward(dev, torch.cuda.current_stream())
    for k in range(3):
        dev.mul_(-0.75).add_(0.1 * k)
        graph.replay()
        a.backward(labels=lab)
        b.forward(dev, labels=lab)
        b.backward(labels=lab)
        torch.cuda.synchronize()
        for t, u in zip(grad_list(a), grad_list(b)):
            assert torch.equal(t, u)
