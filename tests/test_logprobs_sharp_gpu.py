"""Rows with nearly all of the probability on one token."""
import pytest

torch = pytest.importorskip("torch")

import _serve_util as su
from test_logprobs_gpu import check, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("rest", [-float("inf"), -30.0])
@pytest.mark.parametrize("rows", [3, 400])
def test_no_probability_above_one_and_no_entropy_below_zero(dtype, rest, rows):
    """The largest logit comes late and up to 8 above one before it in the same thread's pieces, so that sums are of numbers up to e^8."""
    V = 9000
    x = torch.full((rows, V), rest, device="cuda")
    x[:, 0] = 0.0
    x[:, 4096] = torch.linspace(0.01, 7.99, rows, device="cuda")
    x[:, 8192] = -1.0
    x[rows // 2:, 0] = rest                                 # all but nothing on one
    x[rows // 2:, 8192] = rest
    x = x.to(su.T[dtype])
    token = torch.full((rows,), 4096, dtype=torch.int32, device="cuda")
    check(x, token, 3, dtype=dtype)
    got = run(x, token, 3, dtype=dtype)
    assert (got["entropy"] >= 0).all(), float(got["entropy"].min())
    assert (got["logprob"] <= 0).all(), float(got["logprob"].max())
    assert (got["top_logprob"] <= 0).all()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_sharp_rows_of_all_kinds(dtype):
    """Few tokens that may be given, all in one thread's pieces, the best 5 to 8 above the first and the others far below."""
    V, rows = 13000, 4000
    g = su.gen(3)
    x = torch.full((rows, V), -float("inf"), device="cuda")
    x[:, 0] = torch.randn(rows, device="cuda", generator=g) * 3
    x[:, 4096] = x[:, 0] + 5 + 2.9 * torch.rand(rows, device="cuda", generator=g)
    x[:, 8192] = x[:, 0] - 20 * torch.rand(rows, device="cuda", generator=g) - 4
    x[rows // 2:, 0] -= 20.0
    x = x.to(su.T[dtype])
    token = torch.full((rows,), 4096, dtype=torch.int32, device="cuda")
    check(x, token, 2, dtype=dtype)
    got = run(x, token, 2, dtype=dtype)
    assert (got["entropy"] >= 0).all(), float(got["entropy"].min())
    assert (got["logprob"] <= 0).all(), float(got["logprob"].max())
    assert (got["top_logprob"] <= 0).all()
