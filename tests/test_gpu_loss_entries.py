"""Distillation with one entry to a token and with several, by each of the ways that their logits come."""
import pytest
import torch

from test_gpu_loss import Case, loss  # noqa: F401  (loss: a fixture)

pytestmark = pytest.mark.gpu

# (tokens, vocab, width, dtype, k): so much to read again that the entries' logits come from the tiles, of one entry and of several; rows by 64, by 256
# and by 1024 threads
FROM_TILES = [(4096, 2500, 4096, "bf16", 1), (2100, 130, 8192, "bf16", 1), (1000, 600, 8192, "f32", 1), (1500, 2500, 4096, "bf16", 3), (2100, 1500, 8192, "bf16", 16),
              (400, 900, 2048, "f32", 40)]


@pytest.mark.parametrize("tokens,vocab,width,dtype,k", FROM_TILES)
def test_entries_from_the_tiles(loss, tokens, vocab, width, dtype, k):  # noqa: F811
    case = Case(tokens, vocab, width, dtype, k=k, left_out=0.1, temperature=1.5).reference("cuda")
    case.run(loss).check()
