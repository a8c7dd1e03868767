"""Further checks of the operators between the products, made before anything reaches a device (host-only handles)."""
import ctypes


from paper_2206_10620_b200 import binding
from test_serving_refusals import INVALID, attention, refused


def test_a_wait_cannot_be_told_to_expect_fewer_arrivals():
    op = attention()
    op.test_expect_arrivals(1)
    op.test_expect_arrivals(0)
    refused(INVALID, op.test_expect_arrivals, -1)
    refused(INVALID, op.test_expect_arrivals, 1001)
    assert binding.lib().xgen_attention_test_expect_arrivals(ctypes.c_void_p(), 1) == INVALID
