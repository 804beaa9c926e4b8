"""Gradients that share a launch whose last product (of few slots: dx) has divided tiles behind a round of whole ones that some workgroups have no tile of:
wide, small and tiny tiles, with the products before it beginning at different workgroups."""
import pytest
import torch

import test_ffn_gpu
import test_linear_gpu
from test_linear_gpu import spread

pytestmark = pytest.mark.gpu


def twice(op, run):
    first, second = run(), run()
    assert all(torch.equal(a, b) for a, b in zip(first, second))


@pytest.mark.parametrize("padding", [0, 300])
@pytest.mark.parametrize("n,hidden,inner", [(5376, 1024, 4096), (1736, 3736, 792), (1527, 1096, 1912), (1971, 912, 64)])
def test_feed_forward(n, hidden, inner, padding):
    q_idx = spread(n + padding, n, n) if padding else n
    ffn, (x, w_in, w_out, _, dy, kept), _ = test_ffn_gpu.check_both(q_idx, hidden, inner, "silu", False)
    twice(ffn, lambda: ffn.backward(x, w_in, w_out, dy, kept=kept))


@pytest.mark.parametrize("padding", [0, 300])
@pytest.mark.parametrize("n,n_in,n_out", [(1854, 3848, 2184), (3524, 1440, 1832), (1475, 592, 1752), (100, 38408, 776)])
def test_product(n, n_in, n_out, padding):
    q_idx = spread(n + padding, n, n) if padding else n
    linear, (x, w, b, _, dy, kept), _ = test_linear_gpu.check_both(q_idx, n_in, n_out, "none", True, False)
    twice(linear, lambda: linear.backward(x, w, dy, bias=b, kept=kept))
