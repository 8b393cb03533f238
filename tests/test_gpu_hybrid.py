"""The model of linear and softmax layers: it learns, its token-by-token pass gives what the whole pass gives, and its gradient
is the loss's slope."""
import pytest
import torch

pytestmark = pytest.mark.gpu

GRID, VOCABULARY, CLASSES = (6, 7), 64, 8


def small(window, **kw):
    from paper_2507_01652_amd import hybrid
    torch.manual_seed(3)
    return hybrid.Model(256, 4, GRID, VOCABULARY, CLASSES, window=window, **kw).cuda()


def batch(n):
    from paper_2507_01652_amd import hybrid
    return tuple(t.cuda() for t in hybrid.images(n, GRID, CLASSES, VOCABULARY, torch.Generator().manual_seed(4)))


# Windows of one position, of less than an image (the cache of a step goes round) and of more than one.
# fp32: sums of some 1000 terms a layer, 2^-24 sqrt(1000) each, a few tens of them in a row: 1e-4 is an order above.
# bf16: two passes of some 40 roundings in a row, each 2^-8 / sqrt(3) of its value in the root mean square: 2 sqrt(2 * 40) of
# these is 0.04 for a chain that keeps its errors; the bound is that.
@pytest.mark.parametrize("window", (1, 11, 64))
@pytest.mark.parametrize("half,bound", ((False, 1e-4), (True, 0.04)))
def test_token_by_token_is_the_whole_pass(window, half, bound):
    model = small(window)
    label, tokens = batch(3)
    with torch.no_grad(), torch.autocast("cuda", torch.bfloat16, enabled=half):
        whole = model(label, tokens).double()
        _, stepped = model.sample(label, given=tokens)
    apart = (stepped.double() - whole).norm() / whole.norm()
    assert apart <= bound, float(apart)


# The slope along the gradient: differences of +-h with a change of the loss of 2e-2, whose own error is 1e-5 (fp32 sums of a
# mean of some hundred logarithms near 4); what h leaves of the third derivative is a per cent or so.
def test_gradient_is_the_slope():
    model = small(11)
    label, tokens = batch(4)

    def loss():
        return torch.nn.functional.cross_entropy(model(label, tokens).double().flatten(0, 1), tokens.flatten())

    loss().backward()
    grads = [p.grad.clone() for p in model.parameters()]
    assert all(g.abs().max() > 0 for g in grads)
    size = sum(g.double().pow(2).sum() for g in grads).sqrt().item()
    h = 1e-2 / size ** 2                                    # (of the gradient itself: the loss moves by 2 h size^2)
    values = []
    with torch.no_grad():
        for sign in (1, -2):
            for p, g in zip(model.parameters(), grads):
                p.add_(g, alpha=sign * h)
            values.append(loss().item())
    slope = (values[0] - values[1]) / (2 * h)
    assert abs(slope / size ** 2 - 1) < 0.03, (slope, size ** 2)


def test_it_learns():
    from paper_2507_01652_amd import hybrid
    losses, apart, _ = hybrid.main(["--steps", "30", "--grid", "8", "--batch", "16"])
    assert losses[-1] < 0.7 * losses[0]
    assert apart <= 0.04
