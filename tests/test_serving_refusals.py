"""What the operators between the products refuse, checked before anything reaches a device (host-only handles)."""
import numpy as np
import pytest

from paper_2206_10620_b200 import binding

INVALID, SHAPE, UNSUPPORTED, CUDA = 1, 3, 4, 6
A = 1 << 20                     # an address; nothing reads it


def refused(status, f, *a, **kw):
    with pytest.raises(binding.PatconvError) as e:
        f(*a, **kw)
    assert e.value.status == status


# --- adapters ---------------------------------------------------------------------------------------
def adapters(k=8, c_out=8, rank=4, count=2, dtype="f32"):
    return binding.Adapters(k, c_out, dtype, np.zeros((count, rank, k)), np.zeros((count, c_out, rank)), device=-1)


def test_adapters_pack():
    adapters(rank=128)
    refused(UNSUPPORTED, adapters, rank=129)
    refused(UNSUPPORTED, adapters, dtype="i8")
    refused(INVALID, adapters, count=0)
    refused(INVALID, adapters, rank=0)
    with pytest.raises(ValueError):
        binding.Adapters(8, 8, "f32", np.zeros((2, 4, 8)), np.zeros((2, 8, 3)), device=-1)
    with pytest.raises(ValueError):
        binding.Adapters(8, 8, "f32", np.zeros((2, 4, 8)), np.zeros((2, 8, 4)), np.ones(3), device=-1)


def test_adapters_run():
    op = adapters()
    good = dict(x_ptr=A, rows=4, x_stride=8, row_start_ptr=2 * A, adapter_ptr=3 * A, requests=2, y_ptr=4 * A, y_stride=8, out_ptr=5 * A, out_stride=8)
    run = lambda **kw: op.run(**{**good, **kw})                                     # noqa: E731
    refused(CUDA, run)                                                            # host-only
    refused(CUDA, run, out_ptr=4 * A)                                             # in place is allowed
    op.run(**{**good, "rows": 0, "x_ptr": 0})                                     # nothing to do
    op.run(**{**good, "requests": 0, "row_start_ptr": 0})
    for name in ("x_ptr", "row_start_ptr", "adapter_ptr", "y_ptr", "out_ptr"):
        refused(INVALID, run, **{name: 0})
        refused(INVALID, run, **{name: good[name] + 2})
    for name in ("x_stride", "y_stride", "out_stride"):
        refused(SHAPE, run, **{name: 7})
        refused(SHAPE, run, **{name: 1 << 40})
    refused(SHAPE, run, rows=-1)
    refused(SHAPE, run, requests=-1)
    refused(SHAPE, run, rows=1 << 31)
    refused(SHAPE, run, requests=(1 << 31) - 1)
    refused(INVALID, run, out_ptr=4 * A, out_stride=9)                            # in place with another stride
    refused(INVALID, run, out_ptr=4 * A + 32)                                     # half over y
    refused(INVALID, run, out_ptr=A)                                              # over x
    refused(INVALID, run, out_ptr=A + 4 * 31)
    refused(INVALID, run, out_ptr=2 * A - 64)                                     # over the row starts
    refused(INVALID, run, out_ptr=3 * A)
    refused(CUDA, op.sync)


# --- attention --------------------------------------------------------------------------------------
def attention(q=4, kv=2, D=64, page=16, dtype="f32", freq=(1.0,), **kw):
    return binding.Attention(q, kv, D, page, dtype, freq=None if freq is None else np.asarray(freq, np.float64), device=-1, **kw)


def test_attention_pack():
    attention(freq=np.ones(32))
    attention(freq=None, window=5, softmax_scale=2.0)
    for bad in (dict(q=3), dict(q=0), dict(kv=0), dict(window=-1), dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")),
                dict(softmax_scale=float("inf")), dict(freq=[float("inf")]), dict(freq=[1.0, float("nan")])):
        refused(INVALID, attention, **bad)
    for bad in (dict(D=48), dict(D=0), dict(D=512), dict(page=8), dict(page=48), dict(page=256), dict(dtype="i8"), dict(freq=np.ones(33)),
                dict(window=(1 << 30) + 1)):
        refused(UNSUPPORTED, attention, **bad)
    refused(SHAPE, attention, q=65536, kv=65536)


def batch(sequences=2, rows=3, longest=2, start=2 * A, length=3 * A, table=4 * A, stride=4):
    return binding.Batch(sequences, rows, longest, start, length, table, stride)


def cache(k=16 * A, v=17 * A, ks=18 * A, vs=19 * A, pages=5):
    return binding.Cache(k, v, ks, vs, pages)


BAD_BATCHES = [(SHAPE, dict(sequences=-1)), (SHAPE, dict(rows=-1)), (SHAPE, dict(rows=1 << 31)), (SHAPE, dict(longest=0)), (SHAPE, dict(longest=-1)),
               (SHAPE, dict(stride=0)), (SHAPE, dict(stride=1 << 32)), (SHAPE, dict(sequences=(1 << 31) - 1)),
               (INVALID, dict(start=0)), (INVALID, dict(length=0)), (INVALID, dict(table=0)), (INVALID, dict(start=2 * A + 1)),
               (INVALID, dict(length=3 * A + 2)), (INVALID, dict(table=4 * A + 3))]
BAD_CACHES = [(INVALID, dict(k=0)), (INVALID, dict(v=0)), (INVALID, dict(ks=0)), (INVALID, dict(vs=0)), (INVALID, dict(k=16 * A + 8)),
              (INVALID, dict(v=17 * A + 4)), (INVALID, dict(ks=18 * A + 2)), (SHAPE, dict(pages=0)), (SHAPE, dict(pages=1 << 31))]


def calls(op):
    """The three calls with good arguments, each to be changed in part."""
    def append(b=None, c=None, k=A, v=A + 512, stride=256):
        op.append(k, v, stride, b or batch(), c or cache())

    def read(b=None, c=None, k=A, v=5 * A, stride=128, dtype="f32"):
        op.read(b or batch(), c or cache(), k, v, stride, dtype)

    def run(b=None, c=None, q=A, q_stride=256, y=5 * A, y_stride=256, work=6 * A):
        op.run(q, q_stride, b or batch(), c or cache(), y, y_stride, work)
    return append, read, run


def test_attention_calls():
    op = attention()
    append, read, run = calls(op)
    for f in (append, read, run):
        refused(CUDA, f)                                                          # host-only
        f(b=batch(rows=0))                                                        # nothing to do
        f(b=batch(sequences=0, start=0))
        for status, kw in BAD_BATCHES:
            refused(status, f, b=batch(**kw))
        for status, kw in BAD_CACHES:
            refused(status, f, c=cache(**kw))
    for f in (append, read):
        for kw in (dict(k=0), dict(v=0), dict(k=A + 1), dict(v=A + 2), dict(k=16 * A), dict(v=19 * A)):
            refused(INVALID, f, **kw)
        refused(SHAPE, f, stride=127)
        refused(SHAPE, f, stride=1 << 40)
    refused(UNSUPPORTED, read, dtype="i8")
    for kw in (dict(q=0), dict(y=0), dict(work=0), dict(q=A + 2), dict(y=5 * A + 1), dict(work=6 * A + 8), dict(y=A), dict(y=A + 1024),
               dict(y=17 * A), dict(y=18 * A)):
        refused(INVALID, run, **kw)
    refused(SHAPE, run, q_stride=255)
    refused(SHAPE, run, y_stride=255)
    refused(SHAPE, attention_run_of_too_many_rows)
    refused(CUDA, op.sync)
    refused(CUDA, op.workspace, batch())
    refused(SHAPE, op.workspace, batch(rows=-1))


def attention_run_of_too_many_rows():
    op = attention(q=64, kv=1)
    op.run(A, 4096, batch(rows=1 << 26, longest=1 << 26), cache(), 1 << 50, 4096, 6 * A)


# --- log probabilities --------------------------------------------------------------------------------
def logprobs(vocab=10, dtype="f32", top=3):
    return binding.LogProbs(vocab, dtype, top, device=-1)


def test_logprobs():
    logprobs(top=0)
    logprobs(vocab=32, top=32)
    for bad in (dict(vocab=0), dict(top=-1), dict(top=11), dict(vocab=100, top=33)):
        refused(INVALID, logprobs, **bad)
    refused(UNSUPPORTED, logprobs, dtype="i8")
    op = logprobs()
    good = dict(x_ptr=A, rows=4, row_stride=10, token_ptr=2 * A, logprob_ptr=3 * A, entropy_ptr=4 * A, top_ptr=5 * A, top_logprob_ptr=6 * A)
    run = lambda **kw: op.run(**{**good, **kw})                                     # noqa: E731
    refused(CUDA, run)
    run(rows=0, x_ptr=0)
    refused(SHAPE, run, row_stride=9)
    refused(SHAPE, run, row_stride=1 << 40)
    refused(SHAPE, run, rows=-1)
    refused(SHAPE, run, rows=1 << 31)
    for name in good:
        if name.endswith("_ptr"):
            refused(INVALID, run, **{name: good[name] + 2})
    for name in ("x_ptr", "token_ptr", "logprob_ptr", "top_ptr", "top_logprob_ptr"):
        refused(INVALID, run, **{name: 0})
    refused(CUDA, run, entropy_ptr=0)
    refused(CUDA, run, token_ptr=0, logprob_ptr=0)
    for a, b in (("logprob_ptr", "x_ptr"), ("entropy_ptr", "logprob_ptr"), ("top_ptr", "token_ptr"), ("top_logprob_ptr", "top_ptr")):
        refused(INVALID, run, **{a: good[b] + 4})
    op = logprobs(top=0)
    refused(INVALID, op.run, A, 4, 10, 0, 0, 0, 0, 0)                             # nothing asked for
