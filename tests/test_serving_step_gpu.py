"""One transformer layer and the answers behind it, as a serving program runs them: block-pruned products with adapters beside
them, keys and values into the cache, attention over it, the head's logits, log probabilities.  Every step is checked
against its definition in 64 bits on what the step before it gave."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import _serve_util as su
from paper_2206_10620_b200 import binding

pytestmark = pytest.mark.gpu

VOCAB, WIDTH, HEADS, KV_HEADS, DIM, PAGE, RANK = 1000, 256, 8, 2, 32, 16, 8


class Product:
    """A block-pruned product: half of the rows and of the columns of every block kept."""

    def __init__(self, k, c_out, dtype, seed):
        rng = np.random.default_rng(seed)
        nr, nc = -(-c_out // 32), -(-k // 32)
        rows, cols = rng.random((nr, nc, 32)) < 0.5, rng.random((nr, nc, 32)) < 0.5
        w = (rng.standard_normal((c_out, k)) * (k / 4) ** -0.5).astype(np.float32 if dtype == "f32" else np.float16)
        keep = (rows[:, :, :, None] & cols[:, :, None, :]).transpose(0, 2, 1, 3).reshape(nr * 32, nc * 32)[:c_out, :k]
        self.w = torch.from_numpy(np.where(keep, w, 0).astype(np.float64)).cuda()
        self.op = binding.BlockGemm(k, c_out, 32, 32, dtype, w, rows, cols)
        self.dtype, self.c_out = dtype, c_out

    def __call__(self, x, checked=True):
        y = torch.empty((x.shape[0], self.c_out), dtype=x.dtype, device="cuda")
        self.op.run(x.data_ptr(), x.shape[0], 0, False, y.data_ptr(), torch.cuda.current_stream().cuda_stream)
        if checked:
            want, size = x.double() @ self.w.T, x.double().abs() @ self.w.abs().T
            tol = 1e-4 if self.dtype == "f32" else 2e-3
            su.close(y, want, tol * torch.maximum(want.abs(), 0.01 * size) + 1e-30)
        return y


class Layer:
    def __init__(self, dtype, lengths, capacity, count=3):
        self.dtype, t = dtype, su.T[dtype]
        self.width = (HEADS + 2 * KV_HEADS) * DIM
        self.project, self.out, self.head = (Product(*s, dtype, i) for i, s in enumerate([(WIDTH, self.width), (HEADS * DIM, WIDTH), (WIDTH, VOCAB)]))
        g = su.gen(7)
        self.a = (torch.randn((count, RANK, WIDTH), device="cuda", generator=g) * WIDTH ** -0.5).to(t)
        self.b = (torch.randn((count, self.width, RANK), device="cuda", generator=g) * 0.3).to(t)
        self.scale = torch.tensor([0.5, 1.0, 2.0], device="cuda")
        self.adapters = binding.Adapters(WIDTH, self.width, dtype, self.a.cpu().numpy(), self.b.cpu().numpy(), self.scale.cpu().numpy())
        self.freq = su.frequencies(DIM)
        self.attention = binding.Attention(HEADS, KV_HEADS, DIM, PAGE, dtype, freq=self.freq)
        self.pages = su.Pages(lengths, KV_HEADS, DIM, PAGE, capacity=capacity)
        self.logprobs = binding.LogProbs(VOCAB, dtype, 5)

    def step(self, x, n, which, checked=True):
        """One step over the rows x [sum n, WIDTH]; the answers of every row."""
        rows, width, eb, s = x.shape[0], self.width, x.element_size(), torch.cuda.current_stream().cuda_stream
        start, adapter = su.starts(n), su.ints(which)
        qkv = self.project(x, checked)
        base = qkv.clone() if checked else None
        self.adapters.run(x.data_ptr(), rows, WIDTH, start.data_ptr(), adapter.data_ptr(), len(n), qkv.data_ptr(), width, qkv.data_ptr(), width, s)
        batch = self.pages.batch(n)
        at = qkv.data_ptr() + HEADS * DIM * eb
        self.attention.append(at, at + KV_HEADS * DIM * eb, width, batch, self.pages.handle, s)
        y = torch.empty((rows, HEADS * DIM), dtype=x.dtype, device="cuda")
        work = torch.empty(self.attention.workspace(batch), dtype=torch.uint8, device="cuda")
        self.attention.run(qkv.data_ptr(), width, batch, self.pages.handle, y.data_ptr(), HEADS * DIM, work.data_ptr(), s)
        logits = self.head(self.out(y, checked), checked)
        token = torch.arange(rows, dtype=torch.int32, device="cuda")
        lp, en = (torch.empty(rows, device="cuda") for _ in range(2))
        ti, tl = torch.empty((rows, 5), dtype=torch.int32, device="cuda"), torch.empty((rows, 5), device="cuda")
        self.logprobs.run(logits.data_ptr(), rows, VOCAB, token.data_ptr(), lp.data_ptr(), en.data_ptr(), ti.data_ptr(), tl.data_ptr(), s)
        if checked:
            torch.cuda.synchronize()
            su.close(qkv, *su.adapters(x, base, n, which, self.a, self.b, self.scale, self.dtype))
            su.close(y, *su.attention(self.pages, n, qkv[:, :HEADS * DIM], HEADS, self.dtype, self.freq))
            want = su.logprobs(logits, token, 5)
            assert torch.equal(ti.long(), want["top"][0].long())
            for got, name in ((lp, "logprob"), (en, "entropy"), (tl, "top_logprob")):
                su.close(got, *want[name])
            # what was appended: the page's scale holds every new entry to within a step
            kv, first = qkv[:, HEADS * DIM:].double().view(rows, 2, KV_HEADS, DIM), 0
            for i, m in enumerate(n):
                length = self.pages.lengths[i]
                pos = torch.arange(length - m, length, device="cuda")
                for w in range(2):
                    new = kv[first:first + m, w]
                    new = su.turned(new, pos, self.freq, False) if w == 0 else new
                    step = torch.stack([self.pages.scale[w][int(self.pages.table[i, p // PAGE])] for p in range(length - m, length)]).double()[:, :, None]
                    assert ((self.pages.values(w, i, length)[length - m:] - new).abs() <= 0.51 * step).all()
                first += m
        return lp, ti


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_prompts_then_tokens(dtype):
    """Prompts of three requests go in, then each decodes some tokens, with and without adapters."""
    prompts, more = [40, 3, 17], 12
    layer = Layer(dtype, prompts, [p + more for p in prompts])
    g = su.gen(8)
    layer.step((torch.randn((60, WIDTH), device="cuda", generator=g)).to(su.T[dtype]), prompts, [0, -1, 2])
    for i in range(more):
        layer.pages.lengths = [p + i + 1 for p in prompts]
        layer.pages.length.copy_(su.ints(layer.pages.lengths))
        layer.step((torch.randn((3, WIDTH), device="cuda", generator=g)).to(su.T[dtype]), [1, 1, 1], [0, -1, 2])
