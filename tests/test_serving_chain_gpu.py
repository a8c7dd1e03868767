"""A layer's step as one chain of launches that may overlap: products, adapters, appending, attention, products, log probabilities
one behind the other, captured and replayed and not, against the same calls waited for one by one."""
import re
from pathlib import Path

import pytest

torch = pytest.importorskip("torch")

import _serve_util as su
from test_serving_step_gpu import DIM, HEADS, KV_HEADS, VOCAB, WIDTH, Layer

TOP = 5


class Chain:
    """A layer with buffers for a step of `n` rows to a sequence."""

    def __init__(self, dtype, n, lengths, capacity, which):
        self.n, self.dtype, self.layer = n, dtype, Layer(dtype, lengths, capacity)
        rows, t = sum(n), su.T[dtype]
        make = lambda width, type=t: torch.zeros((rows, width), dtype=type, device="cuda")      # noqa: E731
        self.rows, self.x, self.qkv, self.y, self.z, self.logits = rows, make(WIDTH), make(self.layer.width), make(HEADS * DIM), make(WIDTH), make(VOCAB)
        self.start, self.which, self.token = su.starts(n), su.ints(which), torch.arange(rows, dtype=torch.int32, device="cuda")
        self.lp, self.en, self.ti, self.tl = make(1, torch.float32), make(1, torch.float32), make(TOP, torch.int32), make(TOP, torch.float32)
        self.batch = self.layer.pages.batch(n)
        self.work = torch.empty(self.layer.attention.workspace(self.batch), dtype=torch.uint8, device="cuda")

    def step(self, wait=lambda: None):
        l, rows, width, s = self.layer, self.rows, self.layer.width, torch.cuda.current_stream().cuda_stream
        at = self.qkv.data_ptr() + HEADS * DIM * self.x.element_size()
        pages = l.pages.handle
        for call in (
                lambda: l.project.op.run(self.x.data_ptr(), rows, 0, False, self.qkv.data_ptr(), s),
                lambda: l.adapters.run(self.x.data_ptr(), rows, WIDTH, self.start.data_ptr(), self.which.data_ptr(), len(self.n),
                                       self.qkv.data_ptr(), width, self.qkv.data_ptr(), width, s),
                lambda: l.attention.append(at, at + KV_HEADS * DIM * self.x.element_size(), width, self.batch, pages, s),
                lambda: l.attention.run(self.qkv.data_ptr(), width, self.batch, pages, self.y.data_ptr(), HEADS * DIM, self.work.data_ptr(), s),
                lambda: l.out.op.run(self.y.data_ptr(), rows, 0, False, self.z.data_ptr(), s),
                lambda: l.head.op.run(self.z.data_ptr(), rows, 0, False, self.logits.data_ptr(), s),
                lambda: l.logprobs.run(self.logits.data_ptr(), rows, VOCAB, self.token.data_ptr(), self.lp.data_ptr(), self.en.data_ptr(),
                                       self.ti.data_ptr(), self.tl.data_ptr(), s)):
            call()
            wait()

    def grow(self, more):
        self.layer.pages.length += torch.tensor(more, dtype=torch.int32, device="cuda")

    def outcome(self):
        p = self.layer.pages
        return [t.clone() for t in (self.qkv, self.y, self.logits, self.lp, self.en, self.ti, self.tl, *p.codes, *p.scale)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("n", [[1, 1, 1], [70, 1, 20], [1, 150, 33]])
def test_a_captured_step_is_the_one_waited_for(dtype, n):
    """Two graphs on two streams, each with its own cache and workspace, replayed step by step; and the same without capture."""
    steps, which = 5, [0, -1, 2]
    lengths = [40 + a for a in n]
    capacity = [l + steps * a for l, a in zip(lengths, n)]
    chains = [Chain(dtype, n, lengths, capacity, which) for _ in range(4)]        # (alike: made from the same seeds)
    plain, eager, *captured = chains
    graphs = []
    for c in captured:
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        kept = [t.clone() for t in c.layer.pages.codes + c.layer.pages.scale]
        with torch.cuda.graph(graph, stream=stream):
            c.step()
        assert all(torch.equal(a, b) for a, b in zip(kept, c.layer.pages.codes + c.layer.pages.scale))     # only recorded
        graphs.append((c, stream, graph))
    g = su.gen(21)
    for i in range(steps):
        x = torch.randn((sum(n), WIDTH), device="cuda", generator=g).to(su.T[dtype])
        for c in chains:
            c.x.copy_(x)
            if i:
                c.grow(n)
        torch.cuda.synchronize()
        plain.step(torch.cuda.synchronize)
        want = plain.outcome()
        eager.step()
        for c, stream, graph in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        assert torch.isfinite(want[2]).all() and (want[5] >= 0).all()
        for c in chains[1:]:
            assert all(torch.equal(a, b) for a, b in zip(c.outcome(), want))


def test_what_a_predecessor_writes_is_not_read_by_read_only_loads():
    """A kernel of these operators may start while the one before it still writes: such loads are for what was laid out with the handle."""
    csrc = Path(__file__).resolve().parent.parent / "paper_2206_10620_b200" / "csrc"
    handles_own = {"adapters.cu": {"w", "B"}, "attention.cu": {"by_slot"}, "attention_wide.cu": set(), "logprobs.cu": set(), "attention.cuh": set(),
                   "serve.cuh": set()}
    for name, own in handles_own.items():
        code = re.sub(r"//[^\n]*", "", (csrc / name).read_text())
        assert "ld.global.nc" not in code
        for what in re.findall(r"__ldg\(([^;]*)", code):
            assert re.match(r"\(?(?:%s)\b" % "|".join(own or {"nothing"}), what.strip()), (name, what)
