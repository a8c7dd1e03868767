"""Low-rank adapters of many requests against their definition in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

import _serve_util as su
from paper_2206_10620_b200 import binding

pytestmark = pytest.mark.gpu


def make(dtype, k, c_out, rank, count, seed=0):
    g = su.gen(seed)
    t = su.T[dtype]
    a = (torch.randn((count, rank, k), device="cuda", generator=g) * k ** -0.5).to(t)
    b = (torch.randn((count, c_out, rank), device="cuda", generator=g) * rank ** -0.5).to(t)
    scale = torch.rand(count, device="cuda", generator=g) + 0.5
    return a, b, scale, binding.Adapters(k, c_out, dtype, a.cpu().numpy(), b.cpu().numpy(), scale.cpu().numpy())


def check(dtype, n, which, k, c_out, rank, count=4, in_place=False, strides=(None, None, None), shift=0, spare=0, edit=None, seed=0):
    a, b, scale, op = make(dtype, k, c_out, rank, count, seed)
    g = su.gen(seed + 1)
    rows = sum(n) + spare
    x = su.guard(torch.randn((rows, k), device="cuda", generator=g).to(su.T[dtype]), strides[0], shift)
    y = su.guard(torch.randn((rows, c_out), device="cuda", generator=g).to(su.T[dtype]), strides[1], shift)
    if edit:
        edit(x.t, y.t)
    before = y.t.clone()
    out = y if in_place else su.Guarded(rows, c_out, su.T[dtype], strides[2], shift)
    want, bound = su.adapters(x.t, before, n, which, a, b, scale, dtype)
    start, adapter = su.starts(n), su.ints(which)
    op.run(x.ptr(), rows, x.stride, start.data_ptr(), adapter.data_ptr(), len(n), y.ptr(), y.stride, out.ptr(), out.stride, su.stream())
    torch.cuda.synchronize()
    own = sum(n)
    su.close(out.t[:own], want[:own], bound[:own])
    if in_place:
        assert torch.equal(out.t[own:], before[own:])
    else:
        assert out.rest_is_untouched(own)
        assert torch.equal(y.t.view(torch.int16 if dtype == "f16" else torch.int32), before.view(torch.int16 if dtype == "f16" else torch.int32))
    return op


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("rank", [1, 8, 12, 16, 17, 32, 40, 64, 100, 128])
def test_ranks(dtype, rank):
    check(dtype, [1, 5, 16, 33], [0, 3, -1, 2], 264, 200, rank, seed=rank)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("k,c_out", [(1, 1), (3, 40), (31, 33), (64, 7), (500, 1000), (1000, 333), (2048, 4096), (4097, 257)])
def test_sizes(dtype, k, c_out):
    check(dtype, [1, 2, 17], [1, 0, 2], k, c_out, 16, seed=k)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("n", [[1] * 70, [0, 1, 0, 0, 15, 64, 0], [200, 1, 63, 65], [64], [1], [300, 100]])
@pytest.mark.parametrize("in_place", [False, True])
def test_mixtures(dtype, n, in_place):
    """Decoding rows, empty requests, prompts; more requests than a warp has lanes; adapters shared, missing."""
    check(dtype, n, [(i * 5) % 7 - 1 if i % 7 < 5 else i % 4 for i in range(len(n))], 136, 96, 24, count=6, in_place=in_place, spare=9)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("strides,shift", [((200, 128, 136), 0), ((137, 101, 103), 1), ((144, 104, 112), 3)])
@pytest.mark.parametrize("n", [[3, 30], [90, 70]])
def test_strides_and_alignment(dtype, strides, shift, n):
    check(dtype, n, [0, 1], 136, 100, 16, strides=strides, shift=shift)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("strides,shift", [((136, 104, 104), 0), ((137, 101, 103), 1)])
@pytest.mark.parametrize("n", [[1, 3, 1, 16], [90, 70, 130, 64]])
def test_rows_of_no_adapter(dtype, strides, shift, n):
    """Copied as they are, a bit pattern for a bit pattern, whatever the alignment."""
    check(dtype, n, [-1, 0, -1, -1], 136, 100, 16, strides=strides, shift=shift)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("rank", [16, 64, 128])
@pytest.mark.parametrize("n", [[1] * 180, [1, 2] * 300, [70] * 70, [64, 65] * 120])
def test_many_requests(dtype, rank, n):
    """More tiles than the device holds as clusters of eight: they become clusters of four, of two."""
    check(dtype, n, [i % 5 - 1 for i in range(len(n))], 200, 104, rank, count=4)


@pytest.mark.parametrize("n", [[1] * 8, [200] * 200])
@pytest.mark.parametrize("k", [1000, 4096])
def test_long_sums_are_not_short_of_their_values(n, k):
    """fp32: a matrix unit's sums are rounded toward zero, by half a step of at most 2^-23 on average.  Two of them in each of the two
    products may lose that, the others are a thousand times smaller: 2^-22 in all, however long the sum."""
    a, b, scale, op = make("f32", k, 256, 64, 2)
    rows, which = sum(n), [i % 2 for i in range(len(n))]
    x = torch.randn((rows, k), device="cuda", generator=su.gen(1))
    y = torch.zeros((rows, 256), device="cuda")
    want, _ = su.adapters(x, y, n, which, a, b, scale, "f32")
    start, adapter = su.starts(n), su.ints(which)
    op.run(x.data_ptr(), rows, k, start.data_ptr(), adapter.data_ptr(), len(n), y.data_ptr(), 256, y.data_ptr(), 256, su.stream())
    torch.cuda.synchronize()
    assert abs(((y - want) * want.sign()).mean() / want.abs().mean()) < 2.0 ** -22


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_infinities_and_nan_stay_in_their_rows(dtype):
    """A row of x with a NaN is lost, its neighbours are not; rows of no adapter and result rows keep what they hold."""
    def edit(x, y):
        x[1, 3] = math.nan
        x[7, 0] = math.nan
        y[2, 5] = math.inf
        y[9, 1] = -math.inf
        y[20, 2] = math.nan
    a, b, scale, op = make(dtype, 96, 64, 8, 2)
    check(dtype, [8, 4, 10], [0, 1, -1], 96, 64, 8, count=2, edit=edit)


def test_magnitudes_beyond_fp16():
    """Inner sums far above and below fp16's range reach the result: a row's power of two."""
    a, b, scale, op = make("f16", 256, 64, 16, 1)
    for size in (6e4, 1e-6):
        x = (torch.rand((4, 256), device="cuda", generator=su.gen(3)) * size).half()
        a1 = torch.full((1, 16, 256), 30.0 if size > 1 else 1e-3, device="cuda").half()
        b1 = (torch.rand((1, 64, 16), device="cuda", generator=su.gen(4)) * (1e-5 if size > 1 else 1.0)).half()
        s = torch.tensor([1e-2 if size > 1 else 1e6], device="cuda")
        op = binding.Adapters(256, 64, "f16", a1.cpu().numpy(), b1.cpu().numpy(), s.cpu().numpy())
        y, out = torch.zeros((4, 64), device="cuda").half(), torch.zeros((4, 64), device="cuda").half()
        want, bound = su.adapters(x, y, [4], [0], a1, b1, s, "f16")
        start, which = su.starts([4]), su.ints([0])
        op.run(x.data_ptr(), 4, 256, start.data_ptr(), which.data_ptr(), 1, y.data_ptr(), 64, out.data_ptr(), 64, su.stream())
        assert float(want.abs().max()) > 1e-4
        su.close(out, want, bound)


def test_an_adapter_that_is_not_there():
    """Counts as none, and is reported once."""
    a, b, scale, op = make("f32", 32, 32, 4, 2)
    x, y = torch.randn((6, 32), device="cuda"), torch.randn((6, 32), device="cuda")
    out = torch.zeros_like(y)
    start, which = su.starts([2, 2, 2]), su.ints([0, 2, 1])
    op.run(x.data_ptr(), 6, 32, start.data_ptr(), which.data_ptr(), 3, y.data_ptr(), 32, out.data_ptr(), 32, su.stream())
    assert torch.equal(out[2:4], y[2:4])
    want, bound = su.adapters(x, y, [2, 2, 2], [0, -1, 1], a, b, scale, "f32")
    su.close(out[:2], want[:2], bound[:2])
    with pytest.raises(binding.PatconvError) as e:
        op.sync(su.stream())
    assert e.value.status == 1
    op.sync(su.stream())


def test_row_starts_beyond_the_rows_are_cut():
    a, b, scale, op = make("f32", 32, 32, 4, 2)
    x, y = torch.randn((5, 32), device="cuda"), torch.randn((5, 32), device="cuda")
    out = su.Guarded(5, 32, torch.float32)
    start, which = su.ints([-3, 2, 9]), su.ints([0, 1])
    op.run(x.data_ptr(), 5, 32, start.data_ptr(), which.data_ptr(), 2, y.data_ptr(), 32, out.ptr(), 32, su.stream())
    want, bound = su.adapters(x, y, [2, 3], [0, 1], a, b, scale, "f32")
    su.close(out.t, want, bound)
    assert out.rest_is_untouched()


def test_captured_and_replayed_with_other_requests():
    a, b, scale, op = make("f16", 512, 512, 16, 5)
    x, y = torch.randn((40, 512), device="cuda").half(), torch.randn((40, 512), device="cuda").half()
    out = torch.zeros_like(y)
    start, which = su.starts([10] * 4), su.ints([0, 1, 2, 3])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.run(x.data_ptr(), 40, 512, start.data_ptr(), which.data_ptr(), 4, y.data_ptr(), 512, out.data_ptr(), 512, torch.cuda.current_stream().cuda_stream)
    for n, w in (([10] * 4, [0, 1, 2, 3]), ([1, 0, 35, 4], [4, 1, -1, 2])):
        start.copy_(su.starts(n))
        which.copy_(su.ints(w))
        graph.replay()
        torch.cuda.synchronize()
        want, bound = su.adapters(x, y, n, w, a, b, scale, "f16")
        su.close(out, want, bound)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("rows", [40, 400])
def test_captured_and_on_two_streams(dtype, rows):
    """Two graphs of one handle, replayed side by side with other requests than they were captured with; rows behind the last are left.
    An adapter that is not there is reported where its request has rows."""
    a, b, scale, op = make(dtype, 264, 200, 24, 4)
    jobs = []
    for seed in range(2):
        x = torch.randn((rows, 264), device="cuda", generator=su.gen(seed)).to(su.T[dtype])
        y = torch.randn((rows, 200), device="cuda", generator=su.gen(seed + 2)).to(su.T[dtype])
        out = torch.zeros_like(y)
        start, which = su.starts([rows - 3, 1, 2]), su.ints([0, 1, 2])
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            op.run(x.data_ptr(), rows, 264, start.data_ptr(), which.data_ptr(), 3, y.data_ptr(), 200, out.data_ptr(), 200, torch.cuda.current_stream().cuda_stream)
        jobs.append((x, y, out, start, which, stream, graph))
    for n, who in [([rows // 2, 0, rows // 2], [3, 0, -1]), ([1, 1, 1], [2, 1, 0]), ([0, rows, 0], [0, 3, 9]), ([0, 0, 0], [0, 0, 0]), ([2, 3, 4], [0, 9, 3])]:
        op.sync(su.stream())
        for x, y, out, start, which, stream, graph in jobs:
            start.copy_(su.starts(n))
            which.copy_(su.ints(who))
            out.fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(3):
            for job in jobs:
                with torch.cuda.stream(job[5]):
                    job[6].replay()
        torch.cuda.synchronize()
        for x, y, out, *_ in jobs:
            want, bound = su.adapters(x, y, n, [w if w < 4 else -1 for w in who], a, b, scale, dtype)
            su.close(out[:sum(n)], want[:sum(n)], bound[:sum(n)])
            assert (out[sum(n):] == 7.0).all()
    with pytest.raises(binding.PatconvError) as e:
        op.sync(su.stream())
    assert e.value.status == 1
    op.sync(su.stream())
