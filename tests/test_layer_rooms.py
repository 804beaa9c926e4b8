"""Workspaces of the product and of the feed-forward block: of the sizes that the calls need, and not written past their end."""
import pytest
import torch

from paper_2503_17924_amd import binding as B

MB = 1 << 20


def test_small_calls_take_little():
    for n, a, b, most in ((1, 64, 64, MB // 16), (65, 1024, 1024, 8 * MB), (300, 512, 512, 8 * MB)):
        _, fwd, bwd = B.wlb_linear_workspace_size(B.linear_desc(n, n, a, b, 3))
        assert fwd <= most and bwd <= most + 8 * n * (a + b)
        _, fwd, bwd = B.wlb_ffn_workspace_size(B.ffn_desc(n, n, a, b))
        assert fwd <= most and bwd <= most + 16 * n * (a + b)


def values(*shape, seed):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) / 16).bfloat16().cuda()


class Room:
    """A workspace of a number of bytes, of values that no part is left with, and what lies behind it."""

    def __init__(self, nbytes):
        self.all = torch.full((nbytes + 65536,), 0xff, dtype=torch.uint8, device="cuda")
        self.t = self.all[:nbytes]

    def check(self, name):
        assert (self.all[self.t.numel():] == 0xff).all(), name


SIZES = [(1, 64, 64), (1, 4096, 8192), (5, 4096, 4096), (20, 264, 8200), (33, 1024, 4096), (65, 1024, 1024), (100, 4096, 8200), (129, 8200, 264), (300, 512, 512), (300, 264, 16392),
         (1000, 1024, 4096), (1527, 1096, 1912), (1736, 3736, 792), (1971, 912, 64), (2000, 2048, 2048), (4189, 1544, 5000), (5376, 1024, 4096)]


@pytest.mark.gpu
@pytest.mark.parametrize("n,n_in,n_out", SIZES)
def test_product(n, n_in, n_out):
    x, w, b, dy = values(n, n_in, seed=1), values(n_out, n_in, seed=2), values(n_out, seed=3), values(n, n_out, seed=4)
    for act in (0, 3):
        desc = B.linear_desc(n, n, n_in, n_out, act)
        kept, fwd, bwd = B.wlb_linear_workspace_size(desc)
        fwd, bwd = Room(fwd), Room(bwd + kept)
        want = None
        for dx, dw in ((True, True), (True, False), (False, True)):
            out = torch.empty_like(dy), torch.empty_like(x) if dx else None, torch.empty_like(w) if dw else None, torch.empty_like(b)
            B.wlb_linear_fwd(desc, x, None, w, b, dy, out[0], None, fwd.t)
            fwd.check("forward")
            B.wlb_linear_bwd(desc, x, None, w, b, None, dy, *out[1:], bwd.t)
            bwd.check("backward")
            assert all(torch.isfinite(t).all() for t in out if t is not None)
            want = want or out
            # by itself a product may be divided otherwise: its sums are the same but for their order
            assert torch.equal(out[0], want[0]) and torch.equal(out[3], want[3])
            assert all(torch.allclose(t.float(), s.float(), rtol=2.0 ** -7, atol=2.0 ** -7) for t, s in zip(out[1:3], want[1:3]) if t is not None)


@pytest.mark.gpu
@pytest.mark.parametrize("n,hidden,inner", SIZES)
def test_feed_forward(n, hidden, inner):
    x, w_in, w_out, dy = values(n, hidden, seed=1), values(2 * inner, hidden, seed=2), values(hidden, inner, seed=3), values(n, hidden, seed=4)
    desc = B.ffn_desc(n, n, hidden, inner)
    kept, fwd, bwd = B.wlb_ffn_workspace_size(desc)
    fwd, bwd = Room(fwd), Room(bwd + kept)
    want = None
    for which in (7, 1, 2, 3, 4, 5, 6):
        y, grads = torch.empty_like(x), [torch.empty_like(t) if which >> k & 1 else None for k, t in enumerate((x, w_in, w_out))]
        B.wlb_ffn_fwd(desc, x, None, w_in, w_out, None, y, None, fwd.t)
        fwd.check("forward")
        B.wlb_ffn_bwd(desc, x, None, w_in, w_out, None, dy, *grads, bwd.t)
        bwd.check("backward")
        assert torch.isfinite(y).all() and all(torch.isfinite(t).all() for t in grads if t is not None)
        want = want or grads
        assert all(torch.allclose(t.float(), s.float(), rtol=2.0 ** -7, atol=2.0 ** -7) for t, s in zip(grads, want) if t is not None)
