"""A masked layer under a head of words, retrained by both losses (masked_layer.py), against the same in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def means(head, state, ids, top, targets, temperature):
    """Mean divergence (times the square of the temperature) and mean cross entropy in 64 bits."""
    z = state @ head.t()
    q = torch.softmax(top.double() / temperature, 1)
    log_p = torch.log_softmax(z / temperature, 1).gather(1, ids)
    divergence = (q * (q.log() - log_p)).sum(1).mean() * temperature ** 2
    return divergence, torch.nn.functional.cross_entropy(z, targets, ignore_index=-100)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,vocab,width,k", [(1, 50, 64, 3), (70, 1001, 128, 16), (300, 700, 256, 40)])
def test_head_against_autograd(tokens, vocab, width, k, dtype):
    from paper_2505_23949_amd.masked_layer import Head

    gen = torch.Generator().manual_seed(tokens)
    h, w = torch.randn(tokens, width, generator=gen).to(dtype), (2.0 / width ** 0.5 * torch.randn(vocab, width, generator=gen)).to(dtype)
    ids, top = torch.stack([torch.randperm(vocab, generator=gen)[:k] for _ in range(tokens)]), 3.0 * torch.randn(tokens, k, generator=gen)
    targets = torch.randint(0, vocab, (tokens,), generator=gen)
    targets[1::3] = -100
    head = Head(w.cuda(), trained=True)
    for name, temperature, args in (("cross_entropy", 1.0, (targets.cuda(),)), ("distill", 1.7, (ids.cuda(), top.cuda()))):
        more = {"temperature": temperature} if name == "distill" else {}
        only, none = getattr(head, name)(h.cuda(), *args, **more)
        assert none is None
        losses, dh = getattr(head, name)(h.cuda(), *args, training=True, **more)
        # (what a token's loss is does not depend on what else is wanted, but for the order of sums: a score of few tokens has other kernels)
        assert torch.allclose(only, losses, rtol=1e-5, atol=1e-5)
        x, y = h.double().requires_grad_(), w.double().requires_grad_()
        want = means(y, x, ids, top, targets, temperature)[name == "cross_entropy"]
        want.backward()
        want = want.item()
        counts = (targets >= 0).sum() if name == "cross_entropy" else tokens
        # losses in single precision: 2^-24 of the sums of up to 256 products of a size of 2 or less, and as much for exponentials and sums
        assert abs(float(losses.double().sum()) / int(counts) * temperature ** 2 - want) < 1e-4 * (1 + want)
        # gradients: rounded to their type, of gradients of logits that bf16 rounds too: twice 2^-9 on average
        off = 2.0 ** -7.5 if dtype == torch.bfloat16 else 2.0 ** -17
        assert (dh.double().cpu() - x.grad).norm() <= off * x.grad.norm()
        assert (head.dweight.double().cpu() - y.grad).norm() <= off * y.grad.norm()


def test_gradient_of_the_layer_below():
    """dL/dx through head, masked layer and residual, and the layer's own gradients."""
    from paper_2505_23949_amd.masked_layer import Head, MaskedLayer

    gen = torch.Generator().manual_seed(3)
    tokens, vocab, width, k, temperature = 200, 900, 256, 24, 2.0

    def rand(*shape):
        return torch.randn(*shape, generator=gen)

    one = MaskedLayer((rand(width, width) / width ** 0.5).cuda(), (1 + 0.2 * rand(width)).cuda(), 8, 16, iters=50, tau=0.01)
    head = Head((2.0 / width ** 0.5 * rand(vocab, width)).bfloat16().cuda())
    x, top = rand(tokens, width).bfloat16().cuda(), 3.0 * rand(tokens, k).cuda()
    ids = torch.stack([torch.randperm(vocab, generator=gen)[:k] for _ in range(tokens)]).cuda()
    targets = torch.randint(0, vocab, (tokens,), generator=gen).cuda()
    targets[::5] = -100
    out, h = one.forward(x, training=True)
    state = h + out
    _, dstate = head.distill(state, ids, top, temperature=temperature, training=True)
    _, more = head.cross_entropy(state, targets, training=True)
    dstate = dstate + more
    dx = one.backward(dstate, dstate)

    w = torch.where(one.mask != 0, one.weight, 0.0).double().cpu().requires_grad_()
    gain, deep = one.gain.double().cpu().requires_grad_(), x.double().cpu().requires_grad_()
    y = deep * torch.rsqrt(deep.square().mean(1, keepdim=True) + one.eps) * gain
    sum(means(head.weight.double().cpu(), deep + y @ w.t(), ids.cpu(), top.cpu(), targets.cpu(), temperature)).backward()
    # The products of the layer take 8-bit operands, 2^-4 off at most each and of either sign, and the state that the losses see carries those of the
    # forward pass: as of the layer alone, 6 % of a gradient's norm.
    assert (dx.double().cpu() - deep.grad).norm() <= 0.06 * deep.grad.norm()
    assert (one.dgain.double().cpu() - gain.grad).norm() <= 0.06 * gain.grad.norm()
    kept = one.mask.cpu() != 0
    assert (one.dweight.double().cpu() - w.grad)[kept].norm() <= 0.06 * w.grad[kept].norm()
    assert not one.dweight.cpu()[~kept].any()


def test_nothing_counts():
    from paper_2505_23949_amd.masked_layer import Head

    head = Head(torch.randn(100, 64, device="cuda"), trained=True)
    h = torch.randn(9, 64, device="cuda")
    losses, dh = head.cross_entropy(h, torch.full((9,), -100, device="cuda"), training=True)
    assert not losses.any() and not dh.any() and not head.dweight.any()


def test_the_demonstration_runs():
    from paper_2505_23949_amd import masked_layer

    losses = masked_layer.words(tokens=96, vocab=500, width=128, steps=4, k=8)
    assert len(losses) == 4 and all(x >= 0 and y > 0 for x, y in losses)


def test_a_trained_head_is_clipped_and_updated():
    from paper_2505_23949_amd.masked_layer import Head, clip_gradients

    head = Head(torch.randn(300, 64, device="cuda"), trained=True)
    before = head.weight.clone()
    head.cross_entropy(torch.randn(40, 64, device="cuda"), torch.arange(40, device="cuda"), training=True)
    gradient = head.dweight.clone()
    norm, factor = clip_gradients([head], 0.01).tolist()
    assert abs(norm - float(gradient.norm())) < 1e-4 * norm and factor < 1
    head.update(2.0)
    assert torch.allclose(head.weight, before - 2.0 * factor * gradient, atol=1e-6)
