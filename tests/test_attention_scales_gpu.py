"""Attention over pages whose value scales are far apart, tiny, or not the row's to see."""
import pytest

torch = pytest.importorskip("torch")

import _serve_util as su
from test_attention_gpu import make

pytestmark = pytest.mark.gpu


def tight(dtype, lengths, n, H, G, D, page, edit, window=0, seed=0):
    """As check(), with the bound's absolute part no more than a few of fp32's least steps: it is results of tiny values that count.
    (One step for each of the result's last factors and its rounding, and for each of the pieces that are joined.)"""
    op, freq = make(H, D, page, dtype, rotary=0, q_heads=H * G, window=window)
    pages = su.Pages(lengths, H, D, page, seed=seed)
    q = torch.randn((sum(n), H * G * D), device="cuda", generator=su.gen(seed + 1)).to(su.T[dtype])
    edit(pages, q)
    y = su.attend(op, pages, n, q, H * G, dtype)
    want, bound = su.attention(pages, n, q, H * G, dtype, freq, window=window)
    if dtype == "f32":
        bound = bound - 1e-37 + 8 * 2.0 ** -149
    su.close(y.t, want, bound)
    op.sync(su.stream())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("D", [32, 128, 256])
@pytest.mark.parametrize("n", [1, 5, 40, 150])
@pytest.mark.parametrize("size", [2.0 ** -126, 1e-37, 1e-30])
def test_tiny_values(dtype, D, n, size):
    """Value scales down to the least that appending makes, in all pages, and in the first ones, larger ones behind them."""
    def alone(pages, q):
        pages.scale[1].fill_(size)

    def ahead(pages, q):
        pages.scale[1][pages.table[0, :6].long()] = size
    tight(dtype, [300, 90], [n, min(n, 90)], 2, 4, D, 16, alone)
    tight(dtype, [300, 90], [n, min(n, 90)], 2, 4, D, 16, ahead)
