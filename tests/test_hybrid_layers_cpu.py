"""The example model's layers without a GPU: what their autograd functions refuse, which heads a width gives."""
import types

import pytest
import torch

from paper_2507_01652_amd import hybrid


@pytest.fixture
def plain(monkeypatch):
    """In the place of the kernels: calls of the same form, each gradient twice its input."""
    double = lambda *t: tuple(2 * x for x in t)
    monkeypatch.setattr(hybrid, "lasad", types.SimpleNamespace(
        lasad_forward_qk=lambda q, k, *a: (q * q, k * k), lasad_backward_qk=lambda q, k, dq, dk, h, w, wq, wk: double(q * dq, k * dk, wq, wk),
        lasad_forward_window=lambda q, k, v, *a, **kw: (q * q, q[..., 0].transpose(1, 2)),
        lasad_backward_window=lambda q, k, v, o, lse, do, *a: double(q * do, k, v),
        lasad_forward_layer=lambda q, z, v, *a, **kw: q * q, lasad_backward_layer=lambda q, z, v, do, *a, norm_weight: double(q * do, z, v, norm_weight)))


@pytest.mark.parametrize("function", ["norms", "window", "linear"])
def test_a_second_derivative_is_refused(plain, function):
    x = torch.randn(1, 4, 2, 64).requires_grad_()
    w = torch.ones(64).requires_grad_()
    if function == "norms":
        y = hybrid._HeadNorms.apply(x, x, w, w, (2, 2))[0]
    elif function == "window":
        y = hybrid._Window.apply(x, x, x, 2, 1)
    else:
        y = hybrid._Linear.apply(x, x, x, w, (2, 2))
    # (a second path, so that the sum has a second derivative of its own: the missing part would go unnoticed)
    loss = (y ** 2).sum() + (x ** 3).sum()
    g, = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.sum().backward()


@pytest.mark.parametrize("width,group,heads,key_heads", [(256, 2, 4, 2), (320, 2, 5, 1), (384, 2, 6, 3), (384, 4, 6, 1), (576, 4, 9, 1), (576, 2, 9, 3),
                                                         (640, 4, 10, 2), (64, 2, 1, 1), (256, 8, 4, 1)])
def test_key_heads_divide_the_heads(width, group, heads, key_heads):
    layer = hybrid.SoftmaxLayer(width, (4, 4), 5, group=group)
    assert (layer.hq, layer.hk) == (heads, key_heads)
    assert layer.project.out_features == (heads + 2 * key_heads) * hybrid.HEAD


@pytest.mark.parametrize("width", (0, 32, 100, 250))
def test_a_width_that_is_no_number_of_heads(width):
    for make in (lambda: hybrid.SoftmaxLayer(width, (4, 4), 5), lambda: hybrid.LinearLayer(width, (4, 4))):
        with pytest.raises(ValueError, match="heads of 64"):
            make()
