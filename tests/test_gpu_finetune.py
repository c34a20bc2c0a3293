"""The adapters, the layer norm and AdamW together on a two-bit network:
gradients of the whole stack against the same network in 64 bits, training,
and serving single tokens."""
import pytest
import torch

import paper_1701_00485_gb300 as tbn
from paper_1701_00485_gb300 import finetune, inputs

pytestmark = pytest.mark.gpu


def _plain(net, x, ids, leaves):
    """The stack in 64 bits on the kernels' own weights; leaves: gamma, beta,
    a, b by block."""
    x = x.double()
    none = torch.zeros((1, net.r, net.width), dtype=torch.float64, device=x.device)
    for l in range(net.depth):
        gamma, beta, a, b = leaves[4 * l:4 * l + 4]
        h = torch.nn.functional.layer_norm(x, (net.width,), gamma, beta, 1e-5)
        W = tbn.tbn_unpack(net.codes[l], None, net.width).double() * net.alpha[l].double()[:, None]
        at, bt = torch.cat([a, none])[ids.long()], torch.cat([b, none])[ids.long()]
        low = torch.einsum("trk,tk->tr", at, h)
        x = x + h @ W.T + 2.0 * torch.einsum("tr,trk->tk", low, bt)
    return x


@pytest.mark.parametrize("width,depth,n,r,T", [(256, 2, 3, 8, 300), (512, 2, 5, 16, 700), (128, 1, 1, 4, 9)])
def test_gradients_of_the_stack(width, depth, n, r, T):
    """Every tensor between the calls is rounded to bf16, which moves it by at
    most 2^-8 of itself: per block h, the projection's sum and y forward, and the
    two branches' sum and dx backward, so five roundings a block and one of dy.
    A block's norm passes an error of x on with a gain of about one, the residual
    branch beside it with one, so the relative error of a gradient, as a norm, is
    at most (5 depth + 1) 2^-8 2^depth."""
    g = inputs.generator(width + T)
    net = finetune.AdaptedStack(width, depth, n, r, seed=3)
    for p, c in zip(net.params, net.copies):
        if p.dim() == 3:
            p.copy_(torch.randn(p.shape, generator=g) * width ** -0.5)
            c.copy_(p)
        else:
            p.add_(torch.randn(p.shape, generator=g).cuda() * 0.1)
    x = torch.randn((T, width), generator=g).to(torch.bfloat16).cuda()
    ids = torch.randint(-1, n, (T,), generator=g, dtype=torch.int32).cuda()
    dy = torch.randn((T, width), generator=g).to(torch.bfloat16).cuda()
    y = net.forward(x, ids)
    dx = net.backward(dy)
    assert tbn.tbn_device_error() == 0
    leaves = [(p if c is None else c).double().requires_grad_() for p, c in zip(net.params, net.copies)]
    xd = x.double().requires_grad_()
    want = _plain(net, xd, ids, leaves)
    want.backward(dy.double())
    bound = (5 * depth + 1) * 2.0 ** -8 * 2 ** depth
    for got, exact in [(y, want.detach()), (dx, xd.grad)] + list(zip(net.grads, [t.grad for t in leaves])):
        assert float((got.double() - exact).norm()) <= bound * float(exact.norm())


def test_training_and_serving():
    """Thirty steps of the command's network at a smaller size take most of the
    loss off, and tokens served one at a time see what was learnt."""
    losses = finetune.main(["--width", "256", "--depth", "2", "--adapters", "3", "--tokens", "512",
                            "--rank", "8", "--lr", "0.01"])
    assert tbn.tbn_device_error() == 0
    assert losses[-2] < 0.5 * losses[0] and losses[-1] < 0.75 * losses[0]


def test_an_adapter_learns_only_from_its_own_tokens():
    """A step leaves the adapters without tokens as they were but for weight
    decay, which is zero here."""
    net = finetune.AdaptedStack(128, 1, 4, 8, seed=5)
    g = inputs.generator(9)
    x = torch.randn((40, 128), generator=g).to(torch.bfloat16).cuda()
    ids = torch.full((40,), 2, dtype=torch.int32, device="cuda")
    before = [p.clone() for p in net.params]
    net.forward(x, ids)
    net.backward(torch.randn((40, 128), generator=g).to(torch.bfloat16).cuda())
    net.step(1e-2)
    a, b = net.params[2:4]
    assert not torch.equal(b[2], before[3][2])
    for i in (0, 1, 3):
        assert torch.equal(a[i], before[2][i]) and torch.equal(b[i], before[3][i])
    assert torch.equal(net.copies[3], b.to(torch.bfloat16))
