"""The column sums of layer norm's gradient: how many additions a term passes."""
import pytest
import torch

from layer_ref import U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(4099, 1138), (4099, 1136), (20000, 64), (9000, 4096), (5000, 9000)])
def test_a_large_term_among_small_ones(lrc, cuda, rows, cols):
    """One row has 2^24, the first rows 1, the others 0: a one that is added to 2^24
    on its own is lost, so the error counts the additions on one path.  A block adds
    its own rows in order (rows are dealt to as many blocks of all columns as there
    are multiprocessors at least), the blocks' sums pass a 64th of their number and
    twelve more; each addition is within U of the sum."""
    dev = cuda
    gamma = torch.ones(cols, device=dev)
    x = torch.randn((rows, cols), generator=torch.Generator(device=dev).manual_seed(1), device=dev)
    mean, rstd = x.mean(1), torch.ones(rows, device=dev)
    sms = torch.cuda.get_device_properties(dev).multi_processor_count
    ones = min(rows, sms // -(-cols // 8192))
    for first in (ones, min(rows, 3 * ones), min(rows, 6 * ones)):
        dy = torch.zeros((rows, cols), device=dev)
        dy[:first] = 1
        dy[0] = 2.0 ** 24
        db, dg = torch.empty(cols, device=dev), torch.empty(cols, device=dev)
        lrc.lrc_layer_norm_grad(dy, x, gamma, mean, rstd, None, dg, db, rows, cols, cols, cols, cols, "f32", "f32")
        want = dy.double().sum(0)
        # rows with a one that a block has at most; a 64th of at most six blocks a multiprocessor
        own, most = -(-first // ones) + 1, 6 * sms
        assert float((db.double() - want).abs().max()) <= (own + most / 64 + 12) * U * float(want.max())
