"""Sums over long contexts: what the matrix unit cuts off each time must not add up."""
import pytest

torch = pytest.importorskip("torch")

import _serve_util as su
from paper_2206_10620_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,copies,L", [(130, 160, 1 << 18), (1, 512, 1 << 18), (1, 512, 1 << 20)])
def test_equal_values_over_a_long_context(rows, copies, L):
    """fp16, all values the same number of fp16: the average is that number, whatever the probabilities.

    Their roundings (2^-11 each, in no direction) leave less than 2^-11 / sqrt(L / 8) of it, fp32 sums with rounding less than
    2^-24 sqrt(L), both far below the half step (2^-11.7 of 0.78) at which another number is the nearest."""
    D, page = 32, 128
    op = binding.Attention(1, 1, D, page, "f16")
    pages = su.Pages([L], 1, D, page, seed=1)
    pages.codes[1].fill_(100)
    pages.scale[1].fill_(2.0 ** -7)
    q = torch.randn((rows * copies, D), device="cuda", generator=su.gen(2)).half()
    start, length = su.starts([rows] * copies), su.ints([L] * copies)
    table = pages.table.expand(copies, -1).contiguous()     # (pages that are only read may be shared)
    batch = binding.Batch(copies, rows * copies, rows, start.data_ptr(), length.data_ptr(), table.data_ptr(), table.shape[1])
    y = torch.zeros_like(q)
    work = torch.empty(op.workspace(batch), dtype=torch.uint8, device="cuda")
    op.run(q.data_ptr(), D, batch, pages.handle, y.data_ptr(), D, work.data_ptr(), su.stream())
    op.sync(su.stream())
    assert (y == 100 * 2.0 ** -7).all(), "off by %.3g" % float((y.double() / 0.78125 - 1).abs().max())


def below_the_steps(pages, rows, q, q_heads, window):
    """What products of probability and scale below the least step of fp16 are off by: a row's largest such product becomes 2^6 at least
    (its reference is at most twice it, and lifted by 2^7), half the least step is 2^-25, so 2^-31 of that largest one, and no more
    than the product itself.  It counts where the token with the weight has a code of 0."""
    H, D, L = pages.H, pages.D, pages.lengths[0]
    k, v = pages.values(0, 0, L), pages.values(1, 0, L)
    at = pages.table[0].long()[torch.arange(L, device="cuda") // pages.page]
    j = torch.arange(L, device="cuda")
    out = torch.zeros((rows, q_heads, D), dtype=torch.float64, device="cuda")
    for h in range(q_heads):
        s = q.double().view(rows, q_heads, D)[:, h] @ k[:, h // (q_heads // H)].T * D ** -0.5
        pos = torch.arange(L - rows, L, device="cuda")[:, None]
        p = torch.softmax(s.masked_fill((j > pos) | ((j <= pos - window) if window else False), float("-inf")), 1)
        product = p * pages.scale[1][at, h // (q_heads // H)].double()
        least = torch.minimum(product, product.amax(1, keepdim=True) * 2.0 ** -31)
        share = torch.where(product > 0, least / torch.where(product > 0, product, 1.0), 0.0) * p
        out[:, h] = share @ v[:, h // (q_heads // H)].abs()
    return out.flatten(1)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("rows,copies", [(1, 40), (3, 24), (40, 4)])
def test_long_contexts_of_values_of_all_sizes(dtype, rows, copies):
    """Sums that are put aside on the way: references that go up and down between, pages of small and large values, windows that leave
    some of the pieces without anything to see; checked on the first and the last sequence of those that share the pages."""
    H, G, D, page, L = 1, 4, 32, 64, 150_000
    for window in (0, 100_000):
        op = binding.Attention(H * G, H, D, page, dtype, window=window)
        pages = su.Pages([L], H, D, page, seed=4)
        g = su.gen(5)
        for w in range(2):
            pages.scale[w] *= torch.exp(torch.randn(pages.scale[w].shape, device="cuda", generator=g) * (0.7 if w == 0 else 2.0))
        pages.scale[1][pages.table[0, 700:900].long()] = 0
        one = torch.randn((rows, H * G * D), device="cuda", generator=g).to(su.T[dtype])
        q = one.repeat(copies, 1)
        start, length = su.starts([rows] * copies), su.ints([L] * copies)
        table = pages.table.expand(copies, -1).contiguous()
        batch = binding.Batch(copies, rows * copies, rows, start.data_ptr(), length.data_ptr(), table.data_ptr(), table.shape[1])
        y = torch.zeros_like(q)
        work = torch.full((op.workspace(batch) // 4 + 1,), float("nan"), device="cuda")
        op.run(q.data_ptr(), H * G * D, batch, pages.handle, y.data_ptr(), H * G * D, work.data_ptr(), su.stream())
        op.sync(su.stream())
        want, bound = su.attention(pages, [rows], one, H * G, dtype, window=window)
        bound = bound + below_the_steps(pages, rows, one, H * G, window)
        for i in (0, copies // 2, copies - 1):
            su.close(y[i * rows:(i + 1) * rows], want, bound)


@pytest.mark.parametrize("dtype,rows,copies,L,D,page", [
    ("f16", 1, 256, 150_000, 32, 64), ("f16", 3, 256, 150_000, 32, 128), ("f32", 1, 256, 150_000, 32, 64),       # a piece: some 1300 units
    ("f16", 40, 60, 30_000, 128, 64), ("f16", 40, 60, 30_000, 64, 16), ("f16", 40, 60, 30_000, 96, 32), ("f16", 40, 40, 30_000, 256, 64),
    ("f32", 40, 60, 30_000, 64, 16)])                       # a piece: some 190 units
@pytest.mark.parametrize("window", [0, 20_000])
def test_sums_put_aside_at_every_place(dtype, rows, copies, L, D, page, window):
    """So many sequences over the same pages that a block goes on with a tile for long, and that pieces begin anywhere in it; pages of small and
    large values and of zeros, a row that is not finite: every sequence's rows are as those of one."""
    H, G = 1, 4
    op = binding.Attention(H * G, H, D, page, dtype, window=window)
    pages = su.Pages([L], H, D, page, seed=D)
    g = su.gen(6)
    for w in range(2):
        pages.scale[w] *= torch.exp(torch.randn(pages.scale[w].shape, device="cuda", generator=g) * (0.4 if w == 0 else 2.0))
    pages.scale[1][pages.table[0, 100:160].long()] = 0
    one = torch.randn((rows, H * G * D), device="cuda", generator=g).to(su.T[dtype])
    want, bound = su.attention(pages, [rows], one, H * G, dtype, window=window)
    bound = bound + below_the_steps(pages, rows, one, H * G, window)
    one[-1, D:2 * D] = float("nan")
    want[-1, D:2 * D] = float("nan")
    q = one.repeat(copies, 1)
    start, length = su.starts([rows] * copies), su.ints([L] * copies)
    table = pages.table.expand(copies, -1).contiguous()
    batch = binding.Batch(copies, rows * copies, rows, start.data_ptr(), length.data_ptr(), table.data_ptr(), table.shape[1])
    y = torch.zeros_like(q)
    work = torch.full((op.workspace(batch) // 4 + 1,), float("nan"), device="cuda")
    op.run(q.data_ptr(), H * G * D, batch, pages.handle, y.data_ptr(), H * G * D, work.data_ptr(), su.stream())
    op.sync(su.stream())
    su.close(y, want.repeat(copies, 1), bound.repeat(copies, 1))
