"""The paged cache of 8 bits (appending, reading back) and attention over it against their definitions in 64 bits."""
import math
from fractions import Fraction

import pytest

torch = pytest.importorskip("torch")

import _serve_util as su
from paper_2206_10620_b200 import binding

pytestmark = pytest.mark.gpu


# --- append, read ------------------------------------------------------------------------------------------
def make(H, D, page, dtype, rotary=None, interleaved=False, q_heads=None, window=0, scale=0.0):
    freq = su.frequencies(D if rotary is None else rotary)
    return binding.Attention(q_heads or H, H, D, page, dtype, freq=freq, interleaved=interleaved, window=window, softmax_scale=scale), freq


def append(op, pages, n, kv, dtype, rows=None, longest=None, stride=None, shift=0):
    width = pages.H * pages.D
    g = su.guard(kv, stride, shift)
    op.append(g.ptr(), g.ptr() + width * g.buf.element_size(), g.stride, pages.batch(n, rows=rows, longest=longest), pages.handle, su.stream())
    torch.cuda.synchronize()


def read(op, pages, n, dtype, stride=None, shift=0):
    width = pages.H * pages.D
    k, v = (su.Guarded(sum(n), width, su.T[dtype], stride, shift) for _ in range(2))
    op.read(pages.batch(n), pages.handle, k.ptr(), v.ptr(), k.stride, dtype, su.stream())
    torch.cuda.synchronize()
    assert k.rest_is_untouched() and v.rest_is_untouched()
    return k.t.view(sum(n), pages.H, pages.D), v.t.view(sum(n), pages.H, pages.D)


def check_append(pages, before, n, new, exact_turn):
    """The cache's bytes after an append, page by page.

    new: [keys, values], each [rows, heads, dim] in 64 bits (keys turned).  A scale is amax/127 or the old one doubled; entries
    are off by half a step and what fp32 turning (4 roundings of the larger of a pair) and the product by the reciprocal
    (2^-23 of up to 127) add; older codes are exactly the halved ones, rounded to even."""
    at = 0
    touched = torch.zeros((pages.pages, pages.page), dtype=torch.bool, device="cuda")
    scaled = torch.zeros(pages.pages, dtype=torch.bool, device="cuda")
    for i, m in enumerate(n):
        length = pages.lengths[i]
        lo, p = max(length - m, 0), max(length - m, 0)
        row0 = at - (length - m)
        while p < length:
            page, slot = p // pages.page, p % pages.page
            end = min(length, (page + 1) * pages.page)
            where = int(pages.table[i, page]) if page < pages.table.shape[1] else -1
            if 0 <= where < pages.pages:
                touched[where, slot:slot + end - p] = True
                scaled[where] = True
                for w in range(2):
                    x = new[w][row0 + p:row0 + end].transpose(0, 1)                       # [head, token, dim]
                    old_codes, old_scale = before[w][0][where, :, :slot].double(), before[w][1][where].double()
                    scale, codes = pages.scale[w][where].double(), pages.codes[w][where].double()
                    amax = x.abs().amax((1, 2))
                    lost = ~torch.isfinite(x).all(2).all(1) | (torch.isnan(old_scale) & (slot > 0))
                    assert torch.equal(torch.isnan(scale), lost)
                    fresh = (torch.tensor(slot == 0, device="cuda") | (old_scale == 0)) & ~lost
                    least = torch.where(amax > 0, torch.clamp(amax / 127, min=2.0 ** -126), torch.zeros_like(amax))
                    assert (((scale - least).abs() <= least * 2.0 ** -21) | ~fresh).all()
                    grown = ~fresh & ~lost
                    ratio = torch.where(grown, scale / torch.where(grown, old_scale, 1.0), 1.0)
                    mantissa, up = torch.frexp(ratio)
                    up = up - 1
                    assert (mantissa == 0.5).all() and (up >= 0).all()
                    slack = 1 + 2.0 ** -20
                    assert ((amax <= 127.5 * scale * slack) | ~grown).all()
                    assert ((up == 0) | (amax * slack > 127.5 * scale / 2)).all()
                    halved = torch.round(old_codes / ratio[:, None, None])
                    halved[fresh] = 0
                    keep = ~lost
                    assert torch.equal(codes[keep, :slot], halved[keep])
                    s = torch.where(scale > 0, scale, 1.0)[:, None, None]
                    off = (codes[:, slot:slot + end - p] * s - x).abs()
                    most = 127.5 * s if exact_turn else x.abs().amax((1, 2), keepdim=True)
                    limit = 0.5 * s + most * 2.0 ** -20 + 127 * s * 2.0 ** -22
                    assert (off <= limit)[keep & (scale > 0)].all()
                    assert (codes[:, slot:slot + end - p][scale == 0] == 0).all()
                    assert codes[:, slot:slot + end - p].abs().max() <= 127
            p = end
        at += m
    for w in range(2):                                       # nothing else was written
        same = pages.codes[w] == before[w][0]
        same = same | touched[:, None, :, None] | scaled[:, None, None, None]
        assert same.all()
        assert torch.equal(pages.scale[w][~scaled], before[w][1][~scaled])


def stale_slots_unchanged(pages, before, n):
    for i, m in enumerate(n):
        length = pages.lengths[i]
        if m and length % pages.page:
            where = int(pages.table[i, length // pages.page])
            for w in range(2):
                assert torch.equal(pages.codes[w][where, :, length % pages.page:], before[w][0][where, :, length % pages.page:])


def snapshot(pages):
    return [(pages.codes[w].clone(), pages.scale[w].clone()) for w in range(2)]


def new_entries(kv, pages, n, freq, interleaved):
    x = kv.double().view(kv.shape[0], 2, pages.H, pages.D)
    pos = torch.cat([torch.arange(l - m, l, device="cuda") for l, m in zip(pages.lengths, n)] + [torch.zeros(kv.shape[0] - sum(n), device="cuda")])
    return [su.turned(x[:, 0], pos, freq, interleaved), x[:, 1]]


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("D,page", [(32, 16), (64, 128), (96, 32), (128, 64), (192, 16), (256, 128)])
@pytest.mark.parametrize("rotary,interleaved", [(None, False), (None, True), (0, False), (10, False), (6, True)])
def test_append(dtype, D, page, rotary, interleaved):
    """Pages begun, gone on with, filled; empty sequences; rows behind the last; small and large entries against the old scale."""
    H = 3
    n = [1, 1, 0, page, 2 * page + 3, 5, page - 1]
    lengths = [1, page * 3 + 7, 9, page, 5 * page + 2, page + 2, page * 2]
    op, freq = make(H, D, page, dtype, rotary, interleaved)
    pages = su.Pages(lengths, H, D, page, seed=D + page)
    rows = sum(n) + 4
    g = su.gen(D)
    kv = torch.randn((rows, 2 * H * D), device="cuda", generator=g) * torch.exp(torch.randn((rows, 1), device="cuda", generator=g) * 2)
    kv = kv.to(su.T[dtype])
    before = snapshot(pages)
    append(op, pages, n, kv, dtype, rows=sum(n))
    op.sync(su.stream())
    check_append(pages, before, n, new_entries(kv, pages, n, freq, interleaved), False)
    stale_slots_unchanged(pages, before, n)
    for out in ("f32", "f16"):                              # and back, every row of every sequence
        k, v = read(op, pages, lengths, out, stride=H * D + 8, shift=out == "f16")
        at = 0
        for i, length in enumerate(lengths):
            for w, got in ((0, k), (1, v)):
                want = pages.values(w, i, length)
                su.close(got[at:at + length], want, su.HALF_STEP[out] * want.abs() + 2.0 ** -25)
            at += length


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_append_token_by_token(dtype):
    """However often a page is appended to, an entry is off by less than one step of the page's scale."""
    H, D, page = 2, 64, 32
    op, freq = make(H, D, page, dtype, rotary=0)
    pages = su.Pages([0], H, D, page, capacity=[80])
    g = su.gen(5)
    size = torch.exp(torch.linspace(-6, 3, 80, device="cuda"))[:, None]
    kv = (torch.randn((80, 2 * H * D), device="cuda", generator=g) * size).to(su.T[dtype])
    for i in range(80):
        pages.lengths[0] = i + 1
        pages.length.fill_(i + 1)
        append(op, pages, [1], kv[i:i + 1], dtype)
    for w in range(2):
        got, want = pages.values(w, 0, 80), kv.double().view(80, 2, H, D)[:, w]
        step = torch.stack([pages.scale[w][int(pages.table[0, p // page])] for p in range(80)])[:, :, None].double()
        assert ((got - want).abs() <= step * 1.0001).all()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_append_in_chunks(dtype):
    """Chunks that end where pages end leave the same cache as one call."""
    op, freq = make(2, 64, 16, dtype)
    one, two = (su.Pages([70], 2, 64, 16, seed=1) for _ in range(2))
    kv = torch.randn((70, 256), device="cuda", generator=su.gen(9)).to(su.T[dtype])
    append(op, one, [70], kv, dtype)
    for lo, hi in ((0, 16), (16, 48), (48, 70)):
        two.lengths = [hi]
        two.length.fill_(hi)
        append(op, two, [hi - lo], kv[lo:hi].contiguous(), dtype)
    for w in range(2):
        assert torch.equal(one.codes[w], two.codes[w]) and torch.equal(one.scale[w], two.scale[w])


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("stride,shift", [(2 * 128 + 8, 0), (2 * 128 + 1, 0), (2 * 128 + 3, 1)])
def test_append_strides(dtype, stride, shift):
    op, freq = make(2, 64, 16, dtype)
    n, lengths = [3, 20, 1], [10, 33, 17]
    pages = su.Pages(lengths, 2, 64, 16)
    kv = torch.randn((24, 256), device="cuda", generator=su.gen(stride)).to(su.T[dtype])
    before = snapshot(pages)
    append(op, pages, n, kv, dtype, stride=stride, shift=shift)
    check_append(pages, before, n, new_entries(kv, pages, n, freq, False), False)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_append_zeros_infinities_nan(dtype):
    """Zeros make a scale of 0, which the next entries set; what is not finite loses the page's head until slot 0 is written."""
    H, D, page = 3, 32, 16
    op, freq = make(H, D, page, dtype, rotary=0)
    pages = su.Pages([4], H, D, page)
    t = su.T[dtype]
    zero = torch.zeros((4, 2 * H * D), device="cuda", dtype=t)
    before = snapshot(pages)
    append(op, pages, [4], zero, dtype)
    check_append(pages, before, [4], new_entries(zero, pages, [4], None, False), True)
    assert all((s[int(pages.table[0, 0])] == 0).all() for s in pages.scale)

    def more(length, m, kv):
        pages.lengths[0] = length
        pages.length.fill_(length)
        before = snapshot(pages)
        append(op, pages, [m], kv, dtype)
        check_append(pages, before, [m], new_entries(kv, pages, [m], None, False), True)

    kv = torch.randn((2, 2 * H * D), device="cuda", generator=su.gen(6)).to(t)
    more(6, 2, kv)
    bad = kv.clone()
    bad[0, 5] = math.nan                                    # keys of head 0
    bad[1, H * D + D + 1] = -math.inf                       # values of head 1
    more(8, 2, bad)
    more(10, 2, kv)                                         # still lost
    more(page, 6, kv.repeat(3, 1))
    more(page, page, torch.randn((page, 2 * H * D), device="cuda").to(t))      # begun anew
    assert all(torch.isfinite(s[int(pages.table[0, 0])]).all() for s in pages.scale)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("multiple", [1, 3, 5, 7, 9, 15])
def test_append_entries_halfway_between_codes(dtype, multiple):
    """They go to the even one: scales of few bits, whose halves an entry can hold."""
    H, D, page = 1, 128, 64
    op, freq = make(H, D, page, dtype, rotary=0)
    pages = su.Pages([page], H, D, page)
    scale = multiple * 2.0 ** -7
    x = (torch.arange(page * D, device="cuda") % 253 - 126 + 0.5) * scale
    x = torch.where((x / 2.0 ** -8).abs() < 2048, x, 0.0)   # (11 bits hold them)
    x[5] = 127 * scale
    kv = x.view(page, 1, D).expand(page, 2, D).reshape(page, 2 * D).to(su.T[dtype])
    append(op, pages, [page], kv, dtype)
    where = int(pages.table[0, 0])
    for w in range(2):
        assert float(pages.scale[w][where, 0]) == scale
        assert torch.equal(pages.codes[w][where, 0].double(), torch.round(kv[:, :D].double() / scale))


def test_append_smallest_and_largest():
    """Entries at the edges of fp32 and of what is normal."""
    op, freq = make(1, 32, 16, "f32", rotary=0)
    for size in (3e38, 1e-37, 1e-40, 1e-44):
        pages = su.Pages([8], 1, 32, 16)
        kv = (torch.rand((8, 64), device="cuda", generator=su.gen(7)) * 2 - 1) * size
        before = snapshot(pages)
        append(op, pages, [8], kv, "f32")
        got = pages.values(0, 0, 8)
        step = float(pages.scale[0][int(pages.table[0, 0])].double())
        assert step >= 2.0 ** -126 and ((got[:, 0] - kv[:, :32].double()).abs() <= 0.5001 * step).all()


def test_positions_far_out():
    """Angles of positions past 2^24 are those of the exact position."""
    page, D, far = 128, 64, 200_000_123
    freq = su.frequencies(D)
    op, _ = make(1, D, page, "f32")
    kv = torch.randn((1, 2 * D), device="cuda", generator=su.gen(8))
    table = torch.full((1, far // page + 2), -1, dtype=torch.int32, device="cuda")
    table[0, far // page] = 1
    codes = [torch.zeros((2, 1, page, D), dtype=torch.int8, device="cuda") for _ in range(2)]
    scale = [torch.zeros((2, 1), device="cuda") for _ in range(2)]
    cache = binding.Cache(codes[0].data_ptr(), codes[1].data_ptr(), scale[0].data_ptr(), scale[1].data_ptr(), 2)
    start, length = su.starts([1]), su.ints([far + 1])
    batch = binding.Batch(1, 1, 1, start.data_ptr(), length.data_ptr(), table.data_ptr(), table.shape[1])
    op.append(kv.data_ptr(), kv.data_ptr() + 4 * D, 2 * D, batch, cache, su.stream())
    op.sync(su.stream())
    # the angle in rational arithmetic: position times the float64 frequency, modulo a turn
    pi2 = Fraction("6.28318530717958647692528676655900576839433879875021")
    want = kv[0, :D].double().clone()
    for u in range(D // 2):
        a = Fraction(float(freq[u])) * far
        angle = float(a - pi2 * int(a / pi2))
        x, y = float(kv[0, u]), float(kv[0, u + D // 2])
        want[u], want[u + D // 2] = x * math.cos(angle) - y * math.sin(angle), x * math.sin(angle) + y * math.cos(angle)
    got = codes[0][1, 0, far % page].double() * scale[0][1].double()
    step = float(scale[0][1])
    assert ((got - want).abs() <= 0.5 * step + 3e-6).all()


def test_pages_that_are_not_there():
    """Appending to them is left out, they read as zeros and are seen by nobody; all of it is reported, once."""
    H, D, page = 2, 64, 16
    op, freq = make(H, D, page, "f16")
    lengths, n = [40, 20], [40, 1]
    pages = su.Pages(lengths, H, D, page)
    kept = int(pages.table[0, 1])
    pages.table[0, 1] = pages.pages                         # one past the last
    pages.table[1, 1] = -5
    kv = torch.randn((41, 2 * H * D), device="cuda", generator=su.gen(9)).half()
    before = snapshot(pages)
    append(op, pages, n, kv, "f16")
    with pytest.raises(binding.PatconvError) as e:
        op.sync(su.stream())
    assert e.value.status == 1
    op.sync(su.stream())
    check_append(pages, before, n, new_entries(kv, pages, n, freq, False), False)
    assert torch.equal(pages.codes[0][kept], before[0][0][kept])
    k, v = read(op, pages, [40, 20], "f16")
    assert (k[16:32] == 0).all() and (v[56:60] == 0).all() and (k[:16] != 0).any()
    with pytest.raises(binding.PatconvError):
        op.sync(su.stream())
    q = torch.randn((3, H * D), device="cuda", generator=su.gen(10)).half()
    y = su.attend(op, pages, [2, 1], q, H, "f16")
    want, bound = su.attention(pages, [2, 1], q, H, "f16", freq)
    su.close(y.t, want, bound)
    with pytest.raises(binding.PatconvError):
        op.sync(su.stream())
    op.sync(su.stream())


# --- attention -------------------------------------------------------------------------------------------------
def check(dtype, lengths, n, H, G, D, page, rotary=None, interleaved=False, window=0, scale=0.0, strides=(None, 0), spare=0, seed=0, edit=None,
          longest=None, size=1.0):
    op, freq = make(H, D, page, dtype, rotary, interleaved, q_heads=H * G, window=window, scale=scale)
    pages = su.Pages(lengths, H, D, page, seed=seed)
    q = (torch.randn((sum(n) + spare, H * G * D), device="cuda", generator=su.gen(seed + 1)) * size).to(su.T[dtype])
    if edit:
        edit(pages, q)
    y = su.attend(op, pages, n, q, H * G, dtype, rows=sum(n), stride=strides[0], shift=strides[1], longest=longest)
    assert y.rest_is_untouched(sum(n))
    want, bound = su.attention(pages, n, q, H * G, dtype, freq, interleaved, window, scale or None)
    su.close(y.t[:sum(n)], want, bound)
    op.sync(su.stream())
    return y.t


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 192, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_decode(dtype, D, page):
    check(dtype, [1, 15, 16, 17, 63, 64, 65, 300, 1000], [1] * 9, 2, 4, D, page, seed=D + page)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("G", [1, 2, 3, 5, 7, 8, 16, 17, 32])
def test_heads(dtype, G):
    check(dtype, [1, 130, 700], [1, 1, 1], 2, G, 64, 16, seed=G)
    check(dtype, [5, 130, 700], [5, 3, 2], 1, G, 64, 32, seed=G)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("window", [0, 1, 7, 16, 100, 1000])
def test_prompts_and_windows(dtype, window):
    """Rows from the first token on, chunks behind a cache, a sequence without rows; rows that see one token."""
    check(dtype, [200, 333, 50, 1, 129], [200, 70, 0, 1, 129], 2, 3, 64, 32, window=window, seed=window)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("rotary,interleaved", [(0, False), (16, False), (64, True), (30, True), (2, False)])
def test_rotations(dtype, rotary, interleaved):
    check(dtype, [77, 1000], [4, 1], 2, 2, 64, 16, rotary=rotary, interleaved=interleaved)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("strides", [(520, 0), (513, 1), (515, 3)])
def test_strides(dtype, strides):
    check(dtype, [100, 40], [3, 40], 2, 4, 64, 16, strides=strides, spare=3)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_long_and_short_together(dtype):
    check(dtype, [20000, 3, 1, 500, 7], [1, 1, 1, 1, 1], 1, 4, 128, 64)
    check(dtype, [5000], [1], 1, 1, 128, 16)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_many_sequences(dtype):
    lengths = [1 + (i * 37) % 90 for i in range(300)]
    check(dtype, lengths, [1 - (i % 5 == 4) for i in range(300)], 1, 2, 32, 16)


def test_rows_of_a_longer_sequence_than_the_cache_holds_positions():
    """More rows than tokens: the first ones have no position, see nothing and give zeros; a length of 0 likewise."""
    y = check("f32", [3, 0, 10], [5, 2, 1], 1, 2, 32, 16)
    assert (y[:2] == 0).all() and (y[5:7] == 0).all() and (y[2:5] != 0).any()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_sharp_and_flat(dtype):
    """Softmaxes of one winner among large scores, and of equal ones."""
    check(dtype, [500], [2], 1, 2, 64, 16, size=60.0 if dtype == "f16" else 30.0, scale=0.5)
    check(dtype, [500], [2], 1, 2, 64, 16, size=0.0)
    check(dtype, [500], [2], 1, 2, 64, 16, scale=1e-3)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_scales_far_apart(dtype):
    """Pages whose values differ by orders of magnitude, the largest probabilities on the smallest."""
    def edit(pages, q):
        g = su.gen(20)
        for w in range(2):
            pages.scale[w] *= torch.exp(torch.randn(pages.scale[w].shape, device="cuda", generator=g) * (0.5 if w == 0 else 4))
    check(dtype, [900, 333], [1, 5], 2, 4, 64, 16, edit=edit)

    def zeros(pages, q):
        pages.scale[1][pages.table[0, :3].long()] = 0
        pages.scale[1][pages.table[1, :].clamp(min=0).long()] = 0
        pages.scale[0][pages.table[0, 5].long()] = 0
    check(dtype, [900, 60], [1, 5], 2, 4, 64, 16, edit=zeros)


def test_query_magnitudes():
    for size in (1e-30, 1e-6, 1e6):
        check("f32", [200], [3], 1, 2, 64, 16, size=size, scale=1e-6 if size > 1 else 0.0)
    check("f16", [200], [3], 1, 2, 64, 16, size=2e4, scale=1e-6)
    check("f16", [200], [3], 1, 2, 64, 16, size=1e-7)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_what_is_not_finite_stays_with_those_who_see_it(dtype):
    """A query row of NaN or infinity; a page lost in one head: rows that see it are NaN, the others not; stale pages may hold anything."""
    H, G, D, page = 2, 2, 64, 16
    op, freq = make(H, D, page, dtype, q_heads=H * G)
    lengths, n = [100, 60, 200], [20, 3, 1]
    for what in ("k", "v"):
        pages = su.Pages(lengths, H, D, page, seed=3)
        w = "kv".index(what)
        lost = int(pages.table[0, 5])                       # tokens 80..95 of sequence 0, whose rows are at 80..99
        pages.scale[w][lost, 1] = math.nan
        used = pages.table[pages.table >= 0].long()
        spare = torch.ones(pages.pages, dtype=torch.bool, device="cuda")
        spare[used] = False
        pages.scale[0][spare] = math.nan
        pages.scale[1][spare] = math.inf
        q = torch.randn((24, H * G * D), device="cuda", generator=su.gen(4)).to(su.T[dtype])
        q[21, 3] = math.nan
        q[22, 2 * D + 1] = math.inf
        y = su.attend(op, pages, n, q, H * G, dtype).t.view(24, H * G, D)
        bad = torch.zeros((24, H * G), dtype=torch.bool, device="cuda")
        bad[:20, 2:] = True
        bad[21, 0] = True
        bad[22, 2] = True
        assert torch.equal(torch.isnan(y).all(2), bad) and torch.equal(torch.isnan(y).any(2), bad)
        pages.scale[w][lost, 1] = 0.01
        q = q.nan_to_num(0, 0, 0)
        want, bound = su.attention(pages, n, q, H * G, dtype, freq)
        ok = ~bad.repeat_interleave(D, 1)
        su.close(torch.where(ok, y.flatten(1).double(), 0.0), torch.where(ok, want, 0.0), bound)


def test_a_loose_bound_on_the_rows():
    check("f16", [300, 40, 10], [3, 1, 2], 2, 4, 64, 16, longest=5000)


def test_captured_and_replayed_with_other_lengths():
    """One graph, sequences that grow and shrink between replays, beside another graph with a workspace of its own."""
    H, G, D, page, dtype = 2, 4, 128, 64, "f16"
    op, freq = make(H, D, page, dtype, q_heads=H * G)
    pages = su.Pages([900, 900, 900], H, D, page)
    q = torch.randn((3, H * G * D), device="cuda", generator=su.gen(5)).half()
    kv = torch.randn((3, 2 * H * D), device="cuda", generator=su.gen(6)).half()
    y = torch.zeros_like(q)
    batch = pages.batch([1, 1, 1])
    work = torch.zeros(op.workspace(batch), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream().cuda_stream
        op.append(kv.data_ptr(), kv.data_ptr() + 2 * H * D, 2 * H * D, batch, pages.handle, s)
        op.run(q.data_ptr(), H * G * D, batch, pages.handle, y.data_ptr(), H * G * D, work.data_ptr(), s)
    for lengths in ([900, 1, 64], [2, 899, 500], [900, 900, 900], [1, 1, 1]):
        pages.lengths = lengths
        pages.length.copy_(su.ints(lengths))
        q.copy_(torch.randn(q.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want, bound = su.attention(pages, [1, 1, 1], q, H * G, dtype, freq)
        su.close(y, want, bound)


def test_two_streams_at_once():
    H, G, D, page, dtype = 2, 4, 64, 16, "f32"
    op, freq = make(H, D, page, dtype, q_heads=H * G)
    jobs = []
    for seed in range(2):
        pages = su.Pages([3000, 500], H, D, page, seed=seed)
        q = torch.randn((2, H * G * D), device="cuda", generator=su.gen(seed))
        batch = pages.batch([1, 1])
        jobs.append((pages, q, torch.zeros_like(q), batch, torch.empty(op.workspace(batch), dtype=torch.uint8, device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for pages, q, y, batch, work, s in jobs:
            op.run(q.data_ptr(), H * G * D, batch, pages.handle, y.data_ptr(), H * G * D, work.data_ptr(), s.cuda_stream)
    torch.cuda.synchronize()
    for pages, q, y, *_ in jobs:
        want, bound = su.attention(pages, [1, 1], q, H * G, dtype, freq)
        su.close(y, want, bound)


def test_offsets_past_32_bits():
    """Pages beyond the first 4 GB of codes."""
    H, D, page = 8, 256, 128
    pages = 17000                                           # 4.46 GB of keys, the same of values
    codes = [torch.zeros((pages, H, page, D), dtype=torch.int8, device="cuda") for _ in range(2)]
    scale = [torch.zeros((pages, H), device="cuda") for _ in range(2)]
    op, freq = make(H, D, page, "f16")
    p = object.__new__(su.Pages)
    p.lengths, p.H, p.D, p.page, p.pages, p.codes, p.scale = [300], H, D, page, pages, codes, scale
    p.table = su.ints([pages - 1, 3, pages - 2])[None]
    p.length = su.ints([300])
    p.handle = binding.Cache(codes[0].data_ptr(), codes[1].data_ptr(), scale[0].data_ptr(), scale[1].data_ptr(), pages)
    kv = torch.randn((300, 2 * H * D), device="cuda", generator=su.gen(11)).half()
    append(op, p, [300], kv, "f16")
    for w, x in enumerate(new_entries(kv, p, [300], freq, False)):
        got = p.values(w, 0, 300)
        step = torch.stack([scale[w][int(p.table[0, t // page])] for t in range(300)])[:, :, None].double()
        assert ((got - x).abs() <= 0.501 * step).all()
    q = torch.randn((2, H * D), device="cuda", generator=su.gen(12)).half()
    y = su.attend(op, p, [2], q, H, "f16")
    want, bound = su.attention(p, [2], q, H, "f16", freq)
    su.close(y.t, want, bound)
    k, v = read(op, p, [300], "f16")
    su.close(k, p.values(0, 0, 300), 2.0 ** -11 * p.values(0, 0, 300).abs() + 2.0 ** -25)


# --- many rows -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 192, 256])
@pytest.mark.parametrize("page", [16, 64, 128])
def test_prompts_beside_decoding(dtype, D, page):
    """Sequences of one row, of a few and of many in one call, over caches that end inside a page and a unit."""
    check(dtype, [1, 700, 150, 333, 40, 64, 90], [1, 1, 150, 40, 40, 3, 17], 2, 4, D, page, seed=D + page)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("G,n", [(1, [64]), (1, [65]), (1, [127]), (1, [128]), (1, [129]), (1, [257, 1]), (3, [43]), (5, [26, 13]),
                                 (16, [5, 9]), (32, [3, 2]), (64, [2])])
def test_tiles_that_rows_just_fill(dtype, G, n):
    check(dtype, [x + 70 for x in n], n, 1, G, 64, 32, seed=G)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("D", [32, 64, 128, 192])
def test_chunks_over_a_long_cache(dtype, D):
    """So many rows that no block's piece ends within thousands of tokens; entries that differ by orders of magnitude along the cache."""
    def edit(pages, q):
        for w in range(2):
            grow = 2.0 ** torch.linspace(-3, 3 - 2 * w, pages.table.shape[1], device="cuda")
            pages.scale[w][pages.table[0].long()] *= grow[:, None]
    check(dtype, [4500], [2200], 2, 8, D, 64, size=0.3, edit=edit, seed=D)


def test_long_sums_are_not_short_of_their_values():
    """fp32: sums rounded toward zero lose half a step (2^-24 at most) with every product, and no more than 16 products may
    come before they are added up with rounding: 16 * 2^-24 of a running sum that is half of the last one on average."""
    H, G, D, page, L, n = 1, 4, 128, 64, 5000, 1200
    op, freq = make(H, D, page, "f32", q_heads=H * G)
    pages = su.Pages([L], H, D, page, seed=1)
    q = torch.randn((n, H * G * D), device="cuda", generator=su.gen(2))
    y = su.attend(op, pages, [n], q, H * G, "f32").t.double()
    want, _ = su.attention(pages, [n], q, H * G, "f32", freq)
    assert abs(((y - want) * want.sign()).mean() / want.abs().mean()) < 5e-7


@pytest.mark.parametrize("window", [1, 3, 63, 64, 65, 200])
def test_windows_of_chunks(window):
    check("f16", [1000, 333], [300, 90], 2, 4, 128, 64, window=window, seed=window)
    check("f32", [1000, 333], [300, 90], 1, 4, 64, 16, window=window, seed=window)


@pytest.mark.parametrize("sequences", [1023, 1024, 1025])
def test_more_sequences_than_one_kernel_sorts(sequences):
    n = [1] * sequences
    n[5], n[-1] = 40, 17
    check("f16", [x + (7 * i) % 30 for i, x in enumerate(n)], n, 1, 4, 32, 16, longest=40)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("strides", [(1024, 0), (1032, 0), (1025, 1), (1027, 3)])
def test_strides_of_chunks(dtype, strides):
    check(dtype, [100, 240, 7], [90, 70, 0], 2, 8, 64, 16, strides=strides, spare=3)


def test_chunks_with_more_rows_than_positions():
    y = check("f16", [30, 0, 200], [60, 70, 65], 1, 2, 64, 16)
    assert (y[:30] == 0).all() and (y[60:130] == 0).all() and (y[30:60] != 0).any()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_chunks_with_lost_pages(dtype):
    """Pages that are not there are seen by nobody, a page's lost scale by those who see it, and stale pages may hold anything."""
    H, G, D, page = 2, 4, 64, 16
    op, freq = make(H, D, page, dtype, q_heads=H * G)
    lengths, n = [200, 90], [100, 40]
    for what in ("there", "k", "v"):
        pages = su.Pages(lengths, H, D, page, seed=3)
        spare = torch.ones(pages.pages, dtype=torch.bool, device="cuda")
        spare[pages.table[pages.table >= 0].long()] = False
        pages.scale[0][spare] = math.nan
        pages.scale[1][spare] = math.inf
        q = torch.randn((sum(n), H * G * D), device="cuda", generator=su.gen(4)).to(su.T[dtype])
        bad = torch.zeros((sum(n), H * G), dtype=torch.bool, device="cuda")
        if what == "there":
            pages.table[0, 2] = pages.pages
            pages.table[0, 9] = -1
            pages.table[1, 5] = -7
        else:
            w = "kv".index(what)
            lost = int(pages.table[0, 8])                    # tokens 128 .. 143 of sequence 0, whose rows are at 100 .. 199
            keep = float(pages.scale[w][lost, 1])
            pages.scale[w][lost, 1] = math.nan
            q[110, 3] = math.nan
            q[120, 5 * D + 1] = math.inf
            bad[28:100, G:] = True
            bad[110, 0] = True
            bad[120, 5] = True
        y = su.attend(op, pages, n, q, H * G, dtype).t.view(sum(n), H * G, D)
        assert torch.equal(torch.isnan(y).all(2), bad) and torch.equal(torch.isnan(y).any(2), bad)
        if what == "there":
            with pytest.raises(binding.PatconvError) as e:
                op.sync(su.stream())
            assert e.value.status == 1
        else:
            pages.scale[w][lost, 1] = keep
        op.sync(su.stream())
        want, bound = su.attention(pages, n, q.nan_to_num(0, 0, 0), H * G, dtype, freq)
        ok = ~bad.repeat_interleave(D, 1)
        su.close(torch.where(ok, y.flatten(1).double(), 0.0), torch.where(ok, want, 0.0), bound)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_chunks_captured_and_on_two_streams(dtype):
    """Two graphs, each with its own workspace, replayed side by side with other rows and lengths than they were captured with."""
    H, G, D, page = 2, 4, 64, 16
    op, freq = make(H, D, page, dtype, q_heads=H * G)
    jobs = []
    for seed in range(2):
        pages = su.Pages([900, 500, 300], H, D, page, seed=seed)
        q = torch.randn((200, H * G * D), device="cuda", generator=su.gen(seed)).to(su.T[dtype])
        y = torch.zeros_like(q)
        batch = pages.batch([100, 1, 60], rows=200, longest=190)
        work = torch.full((op.workspace(batch) // 4 + 1,), float("nan"), device="cuda")
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            op.run(q.data_ptr(), H * G * D, batch, pages.handle, y.data_ptr(), H * G * D, work.data_ptr(), torch.cuda.current_stream().cuda_stream)
        jobs.append((pages, q, y, batch, work, stream, graph))
    for n, lengths in [([100, 1, 60], [900, 500, 300]), ([5, 190, 0], [9, 500, 300]), ([1, 1, 180], [900, 1, 200]), ([0, 0, 0], [0, 0, 0])]:
        for (pages, q, y, batch, work, stream, graph) in jobs:
            pages.lengths = lengths
            pages.length.copy_(su.ints(lengths))
            pages._starts[-1].copy_(su.starts(n))
            y.fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(3):
            for (pages, q, y, batch, work, stream, graph) in jobs:
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for (pages, q, y, batch, work, stream, graph) in jobs:
            want, bound = su.attention(pages, n, q, H * G, dtype, freq)
            su.close(y[:sum(n)], want, bound)
            assert (y[sum(n):] == 7.0).all()
    op.sync(su.stream())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_workspace_does_for_smaller_batches(dtype):
    op, _ = make(2, 64, 16, dtype, q_heads=8)
    def size(sequences, rows, longest):
        return op.workspace(binding.Batch(sequences, rows, longest, 256, 256, 256, 4))
    sizes = [size(s, r, l) for s in (1, 2, 1024, 1025) for r, l in ((1, 1), (3, 2), (40, 5), (40, 16), (40, 17), (200, 17), (200, 190))]
    per = len(sizes) // 4
    assert all(sizes[i] <= sizes[i + 1] for i in range(len(sizes) - 1) if (i + 1) % per)
    assert all(sizes[i] <= sizes[i + per] for i in range(len(sizes) - per))


def test_long_sums_of_single_rows_are_not_short_of_their_values():
    """As for chunks: at most the 2 products of 16 tokens come before they are added up with rounding."""
    H, G, D, page, L = 256, 4, 128, 64, 8000
    op, freq = make(H, D, page, "f32", q_heads=H * G)
    pages = su.Pages([L], H, D, page, seed=1)
    q = torch.randn((1, H * G * D), device="cuda", generator=su.gen(2))
    y = su.attend(op, pages, [1], q, H * G, "f32").t.double()
    want, _ = su.attention(pages, [1], q, H * G, "f32", freq)
    assert abs(((y - want) * want.sign()).mean() / want.abs().mean()) < 2.0 ** -23
