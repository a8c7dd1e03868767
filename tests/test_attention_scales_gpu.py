"""Attention over pages whose value scales are far apart, tiny, or not the row's to see."""
import pytest

torch = pytest.importorskip("torch")

import _serve_util as su
from test_attention_gpu import check, make

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
@pytest.mark.parametrize("size", [1e-40, 2.0 ** -126, 1e-37, 1e-30])
def test_tiny_values(dtype, D, n, size):
    """Value scales down to the least that appending makes, and below, in all pages, and in the first ones, larger ones behind them."""
    def alone(pages, q):
        pages.scale[1].fill_(size)

    def ahead(pages, q):
        pages.scale[1][pages.table[0, :6].long()] = size
    tight(dtype, [300, 90], [n, min(n, 90)], 2, 4, D, 16, alone)
    tight(dtype, [300, 90], [n, min(n, 90)], 2, 4, D, 16, ahead)


def far_pages(pages, q, H, G, D, seqs, ratio, low):
    """Values of the pages `seqs` (sequence, page) times `ratio`; queries all alike up to noise, so that keys of those pages, which point
    the other way, have a score of about -low (natural) relative to the others."""
    g = su.gen(77)
    u = torch.sign(torch.randn(D, device="cuda", generator=g))
    q.copy_((u.repeat(H * G) + 0.01 * torch.randn(q.shape, device="cuda", generator=g)).to(q.dtype))
    for w in seqs:
        at = int(pages.table[w])
        pages.codes[0][at] = (-127 * u).to(torch.int8)
        pages.scale[0][at] = low / (127 * D ** 0.5)
        pages.scale[1][at] *= ratio
    return u


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("n", [3, 100])
@pytest.mark.parametrize("ratio,low", [(1e3, 20.0), (1e5, 25.0), (1e8, 30.0), (1e12, 40.0), (1e25, 70.0)])
def test_the_weight_on_the_small_values(dtype, n, ratio, low):
    """Pages of large values that hardly count: probabilities keep their bits relative to what they contribute."""
    if dtype == "f16" and ratio > 1e5:
        scale = 1e5 / ratio                                 # (results within fp16)
    else:
        scale = 1.0
    H, G, D, page = 2, 4, 64, 16

    def edit(pages, q):
        far_pages(pages, q, H, G, D, [(0, 1), (0, 7), (1, 0)], ratio, low)
        pages.scale[1] *= scale
    if dtype == "f32":
        tight(dtype, [400, 150], [n, min(n, 150)], H, G, D, page, edit)
    else:
        check(dtype, [400, 150], [n, min(n, 150)], H, G, D, page, rotary=0, edit=edit)


@pytest.mark.parametrize("n", [8, 16, 100, 140])
@pytest.mark.parametrize("dtype,ratio", [("f16", 1e4), ("f32", 1e4), ("f32", 1e6), ("f32", 1e9), ("f32", 1e14), ("f32", 1e30)])      # (results within fp16)
@pytest.mark.parametrize("window", [0, 96])
def test_pages_that_a_row_does_not_see(dtype, n, ratio, window):
    """Large values behind a row, or before its window, in steps that other rows see: the row is as exact as without them."""
    H, G, D, page, L = 1, 2, 64, 16, 304
    op, freq = make(H, D, page, dtype, rotary=0, q_heads=H * G, window=window)
    pages = su.Pages([L], H, D, page, seed=5)
    q = torch.randn((n, H * G * D), device="cuda", generator=su.gen(6)).to(su.T[dtype])
    plain = pages.scale[1].clone()
    small = torch.ones(n, dtype=torch.bool, device="cuda")
    position = torch.arange(L - n, L, device="cuda")
    # pages that some rows see and others do not: the last ones (later rows), and those at the windows' ends
    where = [L - 16] if not window else [L - 16 - window - 16 * i for i in range(0, 6, 2)]
    for first in where:
        if first < 0:
            continue
        pages.scale[1][int(pages.table[0, first // page])] = plain[int(pages.table[0, first // page])] * ratio
        sees = position >= first
        if window:
            sees &= position - window < first + 15
        small &= ~sees
    assert n <= 16 and not window or small.any()
    y = su.attend(op, pages, [n], q, H * G, dtype)
    want, bound = su.attention(pages, [n], q, H * G, dtype, freq, window=window)
    su.close(y.t[small], want[small], bound[small])
    su.close(y.t, want, bound)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("n", [2, 100])
@pytest.mark.parametrize("size", [1e3, 1e6, 1e9, 1e13])
def test_scores_far_from_zero(dtype, n, size):
    """Scores far beyond where fp32 tells units apart, values of scales far apart: an average of values that some row sees, no more than the
    largest of them (and its rounding)."""
    H, G, D, page, L = 1, 2, 64, 16, 200
    op, _ = make(H, D, page, dtype, rotary=0, q_heads=H * G, scale=size)
    pages = su.Pages([L], H, D, page, seed=8)
    g = su.gen(9)
    pages.scale[1] *= torch.exp(torch.randn(pages.scale[1].shape, device="cuda", generator=g) * 4).clamp(max=100.0)
    q = torch.randn((n, H * G * D), device="cuda", generator=g).to(su.T[dtype])
    y = su.attend(op, pages, [n], q, H * G, dtype).t.double()
    assert torch.isfinite(y).all()
    most = pages.values(1, 0, L).abs().amax()
    assert y.abs().max() <= most * 1.001 and (y != 0).any(1).all()
