"""Forward and backward passes of a masked layer in other orders than one after the other."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_serving_pass_between_a_training_pass_and_its_gradients():
    from paper_2505_23949_amd.masked_layer import MaskedLayer

    gen = torch.Generator("cuda").manual_seed(4)

    def rand(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    one = MaskedLayer(rand(256, 128) / 128 ** 0.5, 1 + 0.2 * rand(128), 2, 4, iters=20, tau=0.01)
    x, residual, dout = rand(40, 128).bfloat16(), rand(40, 128).bfloat16(), rand(40, 256).bfloat16()
    one.forward(x, residual, training=True)
    want = [one.backward(dout).clone(), one.dweight.clone(), one.dgain.clone()]
    one.forward(x, residual, training=True)
    one.forward(rand(1, 128).bfloat16())
    got = [one.backward(dout), one.dweight, one.dgain]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(ValueError, match="40 x 256"):
        one.backward(dout[:39])
