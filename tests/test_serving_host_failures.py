"""Handles of the operators between the products when an allocation fails, and what their calls launch (a stand-in for the CUDA
runtime; no device)."""
import pytest

from test_host_failures import _run, fake_lib  # noqa: F401  (the fixture)

MAKE = """
def status(f, *a, **kw):
    try:
        f(*a, **kw)
    except binding.PatconvError as e:
        return e.status
    return 0
X, Y, Z = 1 << 20, 1 << 30, 1 << 36
makers = [lambda: binding.Adapters(100, 50, "f16", np.ones((3, 5, 100)), np.ones((3, 50, 5)), device=1),
          lambda: binding.Attention(4, 2, 64, 16, "f32", freq=np.ones(32), device=1),
          lambda: binding.LogProbs(100, "f32", 5, device=1)]
"""


def test_a_failed_allocation_leaves_nothing(fake_lib):      # noqa: F811
    _run(fake_lib, MAKE + """
for make, allocations in zip(makers, (4, 2, 0)):
    before = fake.fake_live_bytes()
    for n in range(1, allocations + 1):
        fake.fake_fail_alloc(n)
        assert status(make) == 5
        assert fake.fake_live_bytes() == before and fake.fake_device() == 0
    fake.fake_fail_alloc(0)
    op = make()
    assert (fake.fake_live_bytes() > before) == (allocations > 0) and fake.fake_device() == 0
    if allocations:
        assert fake.fake_alloc_device() == 1
    op.close()
    assert fake.fake_live_bytes() == before
""")


def test_launches_are_on_the_handles_device_and_leave_the_callers(fake_lib):     # noqa: F811
    """Sizes of the launches: clusters of eight for adapters, a page each for appending, the workers and their cuts for
    attention, a cluster for each row of a few logits rows."""
    _run(fake_lib, MAKE + """
ad, at, lp = (m() for m in makers)
n = fake.fake_launches()
assert status(ad.run, X, 48, 100, Z, Z + 4096, 48, Y, 50, Y, 50) == 0
assert fake.fake_launches() == n + 1 and fake.fake_launch(3) == 8 and fake.fake_launch(0) == 8 * 51 and fake.fake_device() == 0
assert status(ad.run, X, 2000, 100, Z, Z + 4096, 2, Y, 50, Y, 50) == 0
assert fake.fake_launch(0) == 8 * (2000 // 64 + 2)
b, c = binding.Batch(3, 100, 60, Z, Z + 64, Z + 128, 9), binding.Cache(X, X + (1 << 22), X + (1 << 24), X + (1 << 25), 40)
assert status(at.append, Y, Y + 512, 256, b, c) == 0
assert fake.fake_launch(0) == 100 // 16 + 6 and fake.fake_launch(1) == 32 and fake.fake_device() == 0
assert status(at.read, b, c, Y, Y + (1 << 20), 128, "f16") == 0
assert fake.fake_launch(0) == 100 // 16 + 6
assert at.workspace(b) > 0
n = fake.fake_launches()
assert status(at.run, Y, 256, b, c, Y + (1 << 20), 256, Z * 2) == 0
assert fake.fake_launches() > n and fake.fake_device() == 0
assert status(lp.run, X, 3, 100, Z, Z + 64, Z + 128, Z + 192, Z + 256) == 0
assert fake.fake_launch(0) == 3 and fake.fake_launch(3) == 1
big = binding.LogProbs(128000, "f16", 0)
assert status(big.run, X, 2, 128000, 0, 0, Z, 0, 0) == 0
assert fake.fake_launch(3) == 16 and fake.fake_launch(0) == 32
""")
