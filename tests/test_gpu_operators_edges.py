"""Rotary positions, norm and loss where test_gpu_operators.py does not reach: logits far from zero, weights of infinities beside rows that fill
a tile, gradients that come in unaligned, gradients of gradients, and the loops, pieces and tiles that larger calls take.  The 64-bit forms and their
tolerances are that file's."""
import pytest
import torch

from test_gpu_operators import _check_loss, _loss_case

pytestmark = pytest.mark.gpu


# ---- loss: an offset that all logits of a row have --------------------------------------------------------------------

# Tiles of 64 words x 64 rows, 256 x 64, x 128 and x 256; a last strip (of 32 words in the first, of 128 in the others) of 1 to 12 words, so that some of
# its lanes have none; fewer strips than the 64 that share a row's sums, and more.
OFFSET_SIZES = [(3, 64, 5), (37, 64, 300), (1000, 64, 129), (64, 72, 4099), (500, 136, 4099), (9000, 64, 129), (100, 64, 70019), (1100, 200, 19971), (33100, 64, 130)]


@pytest.mark.parametrize("offset", [-100.0, -1000.0, 1000.0])
@pytest.mark.parametrize("rows,hidden,vocab", OFFSET_SIZES)
def test_loss_of_logits_with_a_common_offset(rows, hidden, vocab, offset):
    """Softmax does not see it: x has a component along a direction that all words share."""
    x, w, target, d = _loss_case(rows, hidden, vocab, 0.25)
    target[0] = vocab - 1
    x[:, 0], w[:, 0] = offset / 8, 8.0
    _check_loss(x, w, target, d)
