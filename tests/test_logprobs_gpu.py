"""Log probabilities, entropy and top alternatives against their definition in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

import _serve_util as su
from paper_2206_10620_b200 import binding

pytestmark = pytest.mark.gpu


def run(x, token, top, stride=None, shift=0, dtype="f32"):
    rows, vocab = x.shape
    op = binding.LogProbs(vocab, dtype, top)
    g = su.guard(x, stride, shift)
    lp, en = su.Guarded(rows, 1, torch.float32), su.Guarded(rows, 1, torch.float32)
    ti, tl = su.Guarded(rows, max(top, 1), torch.int32, fill=7), su.Guarded(rows, max(top, 1), torch.float32)
    op.run(g.ptr(), rows, g.stride, token.data_ptr() if token is not None else 0, lp.ptr() if token is not None else 0, en.ptr(), ti.ptr(),
           tl.ptr(), su.stream())
    torch.cuda.synchronize()
    for o in (lp, en, ti, tl):
        assert o.rest_is_untouched()
    got = {"entropy": en.t[:, 0]}
    if token is not None:
        got["logprob"] = lp.t[:, 0]
    if top:
        got["top"], got["top_logprob"] = ti.t, tl.t
    return got


def check(x, token, top, **kw):
    got, want = run(x, token, top, **kw), su.logprobs(x, token, top)
    assert set(got) == set(want)
    for name, (value, bound) in want.items():
        if bound is None:
            assert torch.equal(got[name].long(), value.long()), name
        else:
            su.close(got[name], value, bound)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (3, 2, 0), (2, 7, 7), (1, 33, 5), (5, 255, 32), (4, 256, 20), (2, 1000, 1), (1, 4099, 32),
                                            (3, 50001, 20), (150, 5003, 5), (1, 130001, 32), (333, 1001, 3)])
def test_sizes(dtype, rows, vocab, top):
    g = su.gen(rows * 7 + vocab)
    x = (torch.randn((rows, vocab), device="cuda", generator=g) * 3).to(su.T[dtype])
    token = torch.randint(0, vocab, (rows,), dtype=torch.int32, device="cuda", generator=g)
    check(x, token, top, dtype=dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("stride,shift", [(1000, 0), (1001, 1), (1003, 3), (1024, 5)])
def test_rows_at_any_alignment(dtype, stride, shift):
    x = (torch.randn((9, 997), device="cuda", generator=su.gen(stride)) * 4).to(su.T[dtype])
    check(x, su.ints(range(9)), 11, stride=stride, shift=shift, dtype=dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("rows,vocab", [(1, 40000), (200, 3000)])
def test_equal_logits(dtype, rows, vocab):
    """Of equal logits the lowest index is first: all equal, two levels, and an order that puts all of the largest in one lane's pieces."""
    base = torch.full((rows, vocab), 1.5, device="cuda")
    check(base.to(su.T[dtype]), None, 32, dtype=dtype)
    base[:, ::3] = 2.0
    check(base.to(su.T[dtype]), None, 20, dtype=dtype)
    lane = torch.arange(vocab, device="cuda") // (8 if dtype == "f16" else 4) % 32
    check(torch.where(lane == 5, 4.0, base).to(su.T[dtype]), None, 32, dtype=dtype)
    check(torch.arange(vocab, 0, -1, device="cuda").float().expand(rows, vocab).div(64).floor().to(su.T[dtype]), None, 32, dtype=dtype)
    zero = torch.zeros((rows, vocab), device="cuda")
    zero[:, 1::2] = -0.0
    check(zero.to(su.T[dtype]), None, 9, dtype=dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("vocab", [50, 9000, 70001])
def test_what_is_banned(dtype, vocab):
    """Rows of -infinity in part, but for few, altogether; the type's lowest value as a mask; a row all at that value."""
    g = su.gen(vocab)
    x = torch.randn((6, vocab), device="cuda", generator=g).to(su.T[dtype])
    low = torch.finfo(su.T[dtype]).min
    x[0, torch.rand(vocab, device="cuda", generator=g) < 0.5] = -math.inf
    x[1] = -math.inf
    x[2] = -math.inf
    x[2, [3, vocab - 1]] = x[0, 1].nan_to_num(neginf=0.25)
    x[3, 5:] = low
    x[4] = low
    check(x, su.ints([0, 1, 3, 7, 2, vocab - 1]), 4 if vocab < 4 else 20, dtype=dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_infinities_and_nan(dtype):
    x = torch.randn((6, 5000), device="cuda", generator=su.gen(1)).to(su.T[dtype])
    x[0, 4321] = math.inf
    x[2, 0] = math.nan
    x[3, 4999] = math.nan
    x[4] = math.nan
    check(x, su.ints([0, 1, 2, 3, 4, 4999]), 5, dtype=dtype)


def test_largest_numbers():
    x = torch.zeros((3, 3000), device="cuda")
    x[0, 7] = 3.4e38
    x[0, 9] = -3.4e38
    x[1] = 3.3e38
    x[2] = torch.linspace(-1e38, 1e38, 3000, device="cuda")
    check(x, su.ints([7, 5, 2999]), 3)


def test_tokens_out_of_range():
    x = torch.randn((5, 100), device="cuda", generator=su.gen(2))
    check(x, su.ints([-1, 99, 100, -2, 2 ** 31 - 1]), 0)


def test_nothing_but_the_entropy():
    x = torch.randn((4, 3001), device="cuda", generator=su.gen(3))
    check(x, None, 0)


def test_no_rows():
    op = binding.LogProbs(10, "f32", 0)
    op.run(0, 0, 10, 0, 0, 16, 0, 0, su.stream())


def test_captured_and_replayed():
    x = torch.randn((20, 40000), device="cuda", generator=su.gen(4)).half()
    op = binding.LogProbs(40000, "f16", 8)
    token = su.ints(range(20))
    lp, en = (torch.zeros(20, device="cuda") for _ in range(2))
    ti, tl = torch.zeros((20, 8), dtype=torch.int32, device="cuda"), torch.zeros((20, 8), device="cuda")
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        op.run(x.data_ptr(), 20, 40000, token.data_ptr(), lp.data_ptr(), en.data_ptr(), ti.data_ptr(), tl.data_ptr(), torch.cuda.current_stream().cuda_stream)
    for seed in (5, 6):
        x.copy_(torch.randn((20, 40000), device="cuda", generator=su.gen(seed)))
        graph.replay()
        torch.cuda.synchronize()
        want = su.logprobs(x, token, 8)
        assert torch.equal(ti.long(), want["top"][0].long())
        su.close(lp, *want["logprob"])
        su.close(en, *want["entropy"])
        su.close(tl, *want["top_logprob"])
