"""A layer with a transposable mask, found, run and retrained in 8-bit floating point: the mask finder and the layer operators as
a program uses them together.

    python -m paper_2505_23949_amd.masked_layer        # a layer learns to do what a dense one does

``MaskedLayer`` is residual addition, root-mean-square norm and a linear map whose weights carry an N:M mask that holds in the
rows and in the columns of every block, so that its forward pass and its input gradient both read masked weights:

    forward    h = x + residual;  y = norm(h) gain;  out = y (W . S)^T             norm and product in 8 bits
    backward   dy = dout (W . S);  dW = (dout^T y) . S;  dh, dgain from dy          products in 8 bits, operands along their sums
    step       all gradients scaled down to a largest norm, masters updated, weights into 8 bits again, both ways
"""
from __future__ import annotations

from . import binding, layer


def _scratch(size: int, device):
    import torch

    return torch.empty(max(size, 1), dtype=torch.uint8, device=device)


class MaskedLayer:
    """Weights W (out, in) and gain (in), float32 masters; activations and gradients are bfloat16.

    The mask keeps N of every M, by importance |W| (times ``col_scale`` of the input columns if given)."""

    def __init__(self, weight, gain, N: int, M: int, *, eps: float = 1e-5, tau: float = 0.005, iters: int = 300, col_scale=None):
        import torch

        self.weight, self.gain, self.eps = weight, gain, eps
        with torch.cuda.device(weight.device):  # (the mask finder goes to the current GPU)
            self.mask = binding.solve(weight, N, M, tau, iters, col_scale=col_scale, tau_mode=binding.TSENOR_TAU_REL_MATRIX_MAX)["mask"]
        rows, cols = weight.shape
        device = weight.device
        self.weights8 = layer.empty_scaled(rows, cols, device)
        self.weights8_t = layer.empty_scaled(cols, rows, device)
        self._quantize_weights = layer.make_quantize(weight, mask=self.mask, square=True, out=self.weights8, out_t=self.weights8_t)
        self.refresh()
        self.dweight = torch.empty((rows, cols), dtype=torch.bfloat16, device=device)
        self.dgain = torch.empty(cols, dtype=torch.float32, device=device)
        self._kept = None

    def refresh(self) -> None:
        """Masked weights into 8 bits, for both directions; after every change of the masters."""
        layer.tsenor_quantize(self._quantize_weights)

    def forward(self, x, residual=None, *, training: bool = False):
        """(out, h): the layer's output and the residual stream behind the addition (x itself without residual).  A training pass
        keeps h and the norm's output for ``backward``, in the place of the last one's; other passes leave them alone."""
        import torch

        tokens, cols = x.shape
        h = x if residual is None else torch.empty_like(x, memory_format=torch.contiguous_format)
        y = torch.empty((tokens, cols), dtype=x.dtype, device=x.device) if training else None
        y8 = layer.empty_scaled(tokens, cols, x.device)
        layer.tsenor_norm(layer.make_norm(x, self.gain, self.eps, residual=residual, out=y8, y_out=y, sum_out=None if residual is None else h))
        out = torch.empty((tokens, self.weight.shape[0]), dtype=torch.bfloat16, device=x.device)
        self._product(y8, self.weights8, out)
        if training:
            self._kept = (h, y)
        return out, h

    def backward(self, dout, dsum=None):
        """dL/dh of the last training forward pass (the gradient of x and of the residual alike), from dL/dout and what reaches h
        past this layer; writes ``dweight`` and ``dgain`` (they are not added to)."""
        import torch

        if self._kept is None:
            raise RuntimeError("backward needs a forward pass with training=True before it")
        h, y = self._kept
        tokens, cols = h.shape
        rows = self.weight.shape[0]
        if dout.shape != (tokens, rows):
            raise ValueError(f"dout must be {tokens} x {rows}, as the output of the last training pass")
        d8, d8_t = layer.empty_scaled(tokens, rows, h.device), layer.empty_scaled(rows, tokens, h.device)
        y8_t = layer.empty_scaled(cols, tokens, h.device)
        layer.tsenor_quantize(layer.make_quantize(dout, out=d8, out_t=d8_t))
        layer.tsenor_quantize(layer.make_quantize(y, out_t=y8_t))
        dy = torch.empty((tokens, cols), dtype=torch.bfloat16, device=h.device)
        self._product(d8, self.weights8_t, dy)
        self._product(d8_t, y8_t, self.dweight, self.mask)
        dh = torch.empty((tokens, cols), dtype=torch.bfloat16, device=h.device)
        p = layer.make_norm_backward(h, self.gain, self.eps, dy, dh=dh, dgain=self.dgain, dsum=dsum)
        layer.tsenor_norm_backward(p, _scratch(layer.tsenor_norm_backward_workspace_bytes(p), h.device))
        return dh

    @staticmethod
    def _product(a, b, out, mask=None) -> None:
        p = layer.make_product(a, b, out=out, mask=mask)
        layer.tsenor_product(p, _scratch(layer.tsenor_product_workspace_bytes(p), out.device))

    def gradients(self):
        return [self.dweight, self.dgain]

    def update(self, rate: float) -> None:
        """A plain gradient step on the masters; dropped weights have no gradient and stay as they are."""
        self.weight.add_(self.dweight, alpha=-rate)
        self.gain.add_(self.dgain, alpha=-rate)
        self.refresh()


def clip_gradients(layers, max_norm: float):
    """The gradients of all layers scaled down, in place, to ``max_norm``; returns (norm, factor) on the GPU."""
    import torch

    gradients = [g for one in layers for g in one.gradients()]
    norm = torch.empty(2, device=gradients[0].device)
    p = layer.make_clip(gradients, max_norm, norm_out=norm)
    layer.tsenor_clip(p, _scratch(layer.tsenor_clip_workspace_bytes(p), norm.device))
    return norm


def main(tokens: int = 1024, rows: int = 768, cols: int = 512, steps: int = 30, rate: float = 30.0) -> list[float]:
    """A masked 8:16 layer, its weights pruned from a dense one's, learns what the dense one does; returns the losses.
    The columns of its inputs are mixtures of fewer sources: kept weights can make up for dropped ones."""
    import torch

    gen = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    dense = normal(rows, cols) / cols ** 0.5
    mixture = normal(cols // 4, cols) / (cols // 4) ** 0.5

    def inputs(count):
        return (normal(count, cols // 4) @ mixture).bfloat16()

    one = MaskedLayer(dense.clone(), torch.ones(cols, device="cuda"), 8, 16)
    losses = []
    for step in range(steps):
        x, residual = inputs(tokens), inputs(tokens)
        out, h = one.forward(x, residual, training=True)
        wide = h.float()
        target = (wide * torch.rsqrt(wide.square().mean(1, keepdim=True) + one.eps)) @ dense.t()
        error = out.float() - target
        losses.append(float(error.square().mean()))
        one.backward((error * (2.0 / error.numel())).bfloat16())
        norm, factor = clip_gradients([one], 0.02).tolist()
        one.update(rate)
        if step % 5 == 0 or step == steps - 1:
            print(f"step {step}: loss {losses[-1]:.5f}, gradient norm {norm:.5f}, scaled by {factor:.3f}", flush=True)
    token, _ = one.forward(inputs(1))      # serving: one token
    print(f"one token: {tuple(token.shape)}, kept {int(one.mask.sum())} of {one.mask.numel()} weights", flush=True)
    return losses


if __name__ == "__main__":
    main()
