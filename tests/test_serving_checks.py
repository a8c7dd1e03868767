"""Further checks of the operators between the products, made before anything reaches a device (host-only handles)."""
import ctypes


from paper_2206_10620_b200 import binding
from test_host_failures import _run, fake_lib  # noqa: F401  (the fixture)
from test_serving_host_failures import MAKE
from test_serving_refusals import A, CUDA, INVALID, SHAPE, adapters, attention, batch, cache, calls, logprobs, refused


def test_a_wait_cannot_be_told_to_expect_fewer_arrivals():
    op = attention()
    op.test_expect_arrivals(1)
    op.test_expect_arrivals(0)
    refused(INVALID, op.test_expect_arrivals, -1)
    refused(INVALID, op.test_expect_arrivals, 1001)
    assert binding.lib().xgen_attention_test_expect_arrivals(ctypes.c_void_p(), 1) == INVALID


# --- memory that must not overlap ---------------------------------------------------------------------
def test_attention_results_lie_outside_what_the_call_reads():
    """Row starts at 2 A (3 numbers), lengths at 3 A (2), the page table at 4 A (2 rows of 4); three rows of 256 elements."""
    op = attention()
    append, read, run = calls(op)
    for first, size in ((2 * A, 12), (3 * A, 8), (4 * A, 32)):
        for at in (first, first + size - 4, first - 4 * 3 * 256 + 4):
            refused(INVALID, run, y=at)
        for at in (first, first + size - 4, first - 4 * 3 * 128 + 4):
            refused(INVALID, read, k=at)
            refused(INVALID, read, v=at)
        refused(CUDA, run, y=first + size)
        refused(CUDA, run, y=first - 4 * 3 * 256)
        refused(CUDA, read, k=first + size)
        refused(CUDA, read, v=first - 4 * 3 * 128)


def test_attention_read_does_not_write_twice_to_a_place():
    op = attention()
    _, read, _ = calls(op)
    refused(INVALID, read, k=A, v=A)
    refused(INVALID, read, k=A, v=A + 4 * 127)
    refused(INVALID, read, k=A + 4 * 127, v=A)
    refused(INVALID, read, k=A, v=A + 4 * (2 * 300 + 127), stride=300)            # the last row of one, the first of the other
    refused(INVALID, read, k=A, v=A + 4 * 200, stride=300)                        # v's rows reach into k's next ones
    refused(CUDA, read, k=A, v=A + 4 * 3 * 128)
    refused(CUDA, read, k=A, v=A + 4 * 128, stride=256)                           # parts of the same rows
    refused(CUDA, read, k=A + 4 * 172, v=A, stride=300)
    refused(CUDA, read, k=A, v=A + 4 * (2 * 300 + 128), stride=300)


def test_attention_append_writes_to_a_cache_apart():
    """Five pages of 2 heads of 16 tokens: 10 scales, 10240 codes, keys and values each."""
    op = attention()
    append, read, run = calls(op)
    K, V, KS, VS = 16 * A, 17 * A, 18 * A, 19 * A
    for kw in (dict(v=K), dict(v=K + 10240 - 16), dict(ks=K), dict(vs=V + 10240 - 4), dict(vs=KS), dict(vs=KS + 36), dict(ks=2 * A), dict(k=3 * A),
               dict(v=4 * A)):
        refused(INVALID, append, c=cache(**kw))
    for kw in (dict(v=K + 10240), dict(vs=KS + 40), dict(ks=2 * A + 12)):
        refused(CUDA, append, c=cache(**kw))
    refused(CUDA, read, c=cache(v=K))                                             # what is only read may be shared
    refused(CUDA, run, c=cache(v=K, vs=KS))


def test_attention_workspace_lies_apart(fake_lib):         # noqa: F811
    _run(fake_lib, MAKE + """
at = makers[1]()
H = 1 << 20
b, c = binding.Batch(2, 100, 60, 2 * Z, 3 * Z, 4 * Z, 9), binding.Cache(5 * Z, 6 * Z, 7 * Z, 8 * Z, 40)
run = lambda **kw: status(at.run, *{**dict(q=10 * Z, qs=256, b=b, c=c, y=11 * Z, ys=256, w=9 * Z), **kw}.values())
assert run() == 0
size = at.workspace(b)
for first, n in ((10 * Z, 100 * 1024), (2 * Z, 12), (3 * Z, 8), (4 * Z, 72), (11 * Z, 100 * 1024), (5 * Z, 40 * 2 * 16 * 64)):
    for w in (first, first + (n - 1) // 16 * 16, first - size + 16):
        assert run(w=w // 16 * 16) == 1, (first, w)
    assert run(w=first + (n + 15) // 16 * 16) == 0 and run(w=(first - size) // 16 * 16) == 0
""")


# --- sizes ----------------------------------------------------------------------------------------------
ROWS, STRIDE = (1 << 31) - 1, 1 << 31                       # fp32: all but 2^34 of the 2^64 bytes that addresses reach


def test_spans_that_reach_past_the_last_address_overlap_what_is_behind_them():
    op = adapters()
    good = dict(x_ptr=A, rows=4, x_stride=8, row_start_ptr=2 * A, adapter_ptr=3 * A, requests=2, y_ptr=4 * A, y_stride=8, out_ptr=5 * A, out_stride=8)
    far = 1 << 36
    refused(INVALID, op.run, **{**good, "rows": ROWS, "x_stride": STRIDE, "x_ptr": far, "out_ptr": 1 << 45, "y_ptr": 1 << 50})
    refused(INVALID, op.run, **{**good, "rows": ROWS, "y_ptr": far, "y_stride": STRIDE, "x_ptr": 1 << 58, "out_ptr": 1 << 45})
    refused(INVALID, op.run, **{**good, "rows": ROWS, "out_ptr": far, "out_stride": STRIDE, "y_ptr": 1 << 45})
    _, read, run = calls(attention(q=1, kv=1))
    near = cache(1 << 30, 1 << 31, 1 << 32, 1 << 33)
    refused(INVALID, run, b=batch(rows=ROWS - 256), q=far, q_stride=STRIDE, c=near, y=1 << 45)
    refused(INVALID, read, b=batch(rows=ROWS), stride=STRIDE, k=far, v=far + (1 << 30), c=cache(1 << 30, 1 << 31, 1 << 32, 1 << 60))


def test_logits_of_more_bytes_than_there_are():
    op = logprobs()
    run = lambda rows, **kw: op.run(**{**dict(x_ptr=8 * A, rows=rows, row_stride=STRIDE, token_ptr=2 * A, logprob_ptr=0, entropy_ptr=4 * A,      # noqa: E731
                                              top_ptr=5 * A, top_logprob_ptr=6 * A), **kw})
    refused(SHAPE, run, ROWS, token_ptr=0)
    refused(SHAPE, run, (1 << 29) + 1, token_ptr=0)         # 2^62 + 40
    refused(CUDA, run, 4, token_ptr=0)
    refused(INVALID, run, 1 << 29, token_ptr=0, entropy_ptr=1 << 50)


def test_adapters_of_more_bytes_than_a_number_holds():
    """2^30 adapters of 2^33 bytes on either side: 2^64 in all."""
    desc = binding.AdaptersDesc(1 << 24, 1 << 24, 128, 1 << 30, binding.F32)
    h = ctypes.c_void_p()
    pack = lambda: binding.lib().xgen_adapters_pack(ctypes.byref(desc), A, A, A, -1, ctypes.byref(h))      # noqa: E731  (nothing reads them)
    assert pack() == SHAPE and not h
    desc.adapters = (1 << 31) - 1
    assert pack() == SHAPE and not h
    desc.adapters = 64                                      # 2^40 in all
    assert pack() == 0 and h
    binding.lib().xgen_adapters_free(h)


def test_attention_counts_query_rows_in_32_bits():
    """Tiles of rows (of all query heads of a key head) are rounded up, to 128 at most."""
    op = attention(q=64, kv=1)
    run = lambda rows: op.run(1 << 50, 4096, batch(rows=rows, longest=rows), cache(), 1 << 55, 4096, 6 * A)      # noqa: E731
    refused(SHAPE, run, (1 << 25) - 3)                      # 2^31 - 192
    refused(CUDA, run, (1 << 25) - 5)                       # 2^31 - 320
