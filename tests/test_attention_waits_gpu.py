"""A wait of the attention kernel for many rows that runs out."""
import pytest

torch = pytest.importorskip("torch")

import _serve_util as su
from paper_2206_10620_b200 import binding
from test_attention_gpu import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [("f32", 64), ("f32", 128), ("f16", 64), ("f16", 128), ("f16", 256)])
@pytest.mark.parametrize("n,lengths", [([70], [70]), ([40], [40]), ([700, 3, 90], [5000, 900, 90])])
def test_a_wait_that_runs_out_is_reported(dtype, D, n, lengths):
    """Products told to wait for an arrival that never comes, with matrix instructions under way: the call ends by itself at its
    (shortened) limit and stays inside its tensors, the timeout is reported once, and the next run is as the one before."""
    H, G, page = 2, 4, 64
    op, _ = make(H, D, page, dtype, q_heads=H * G)
    pages = su.Pages(lengths, H, D, page, seed=D)
    q = torch.randn((sum(n), H * G * D), device="cuda", generator=su.gen(D)).to(su.T[dtype])
    before = su.attend(op, pages, n, q, H * G, dtype)
    op.sync(su.stream())
    kept = [t.clone() for t in pages.codes + pages.scale]
    op.test_expect_arrivals(1)
    y = su.attend(op, pages, n, q, H * G, dtype)            # only enqueues: OK
    assert y.rest_is_untouched()
    with pytest.raises(binding.PatconvError) as e:
        op.sync(su.stream())
    assert e.value.status == 7
    op.sync(su.stream())                                    # reported once
    assert all(torch.equal(a, b) for a, b in zip(kept, pages.codes + pages.scale))
    op.test_expect_arrivals(0)
    assert torch.equal(su.attend(op, pages, n, q, H * G, dtype).t, before.t)
    op.sync(su.stream())
