"""Plain 64-bit forms of the operators between the products, with the bounds that their kernels' roundings give, and helpers
that call the kernels.  Everything is torch on the GPU; nothing here uses the library's arithmetic."""
import math

import numpy as np
import torch

from paper_2206_10620_b200 import binding

T = {"f32": torch.float32, "f16": torch.float16}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11}       # relative rounding of a stored result
GUARD = 32


def stream():
    return torch.cuda.current_stream().cuda_stream


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def starts(n):
    return ints([0] + list(np.cumsum(n)))


class Guarded:
    """A poisoned tensor [rows, width] with its rows `stride` apart (offset by `shift` elements), between guard bands."""

    def __init__(self, rows, width, dtype, stride=None, shift=0, fill=77.0):
        self.stride = stride or width
        self.n = (rows - 1) * self.stride + width if rows else 0
        self.buf = torch.full((self.n + 2 * GUARD + shift,), fill, dtype=dtype, device="cuda")
        self.lo = GUARD + shift
        self.t = self.buf.as_strided((rows, width), (self.stride, 1), self.lo) if rows else self.buf[:0].view(0, width)
        self.fill = fill

    def ptr(self):
        return self.buf.data_ptr() + self.lo * self.buf.element_size()

    def rest_is_untouched(self, rows=None):
        """Nothing but the first `rows` rows (all of them by default) was written."""
        keep = torch.ones_like(self.buf, dtype=torch.bool)
        inner = keep.as_strided(self.t.shape, (self.stride, 1), self.lo)
        inner[:self.t.shape[0] if rows is None else rows] = False
        return bool((self.buf[keep] == self.fill).all())


def close(got, want, bound):
    """|got - want| <= bound, infinities and NaN in the same places."""
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN in other places"
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    err = (got - want).abs()[fine]
    bound = (torch.as_tensor(bound, dtype=torch.float64, device="cuda") + torch.zeros_like(want))[fine]
    worst = float((err / bound.clamp(min=1e-300)).max()) if err.numel() else 0.0
    assert worst <= 1.0, "%.3g of the bound, largest error %.3g" % (worst, float(err.max()))
    return worst


# --- rotation, the cache -------------------------------------------------------------------------
def frequencies(rotary, base=10000.0):
    return base ** (-np.arange(rotary // 2) * 2.0 / rotary) if rotary else None


def turned(x, positions, freq, interleaved):
    """x [rows, heads, dim] float64 turned by its positions."""
    if freq is None:
        return x.clone()
    r = 2 * len(freq)
    angle = positions.double()[:, None] * torch.tensor(freq, device="cuda")
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    y = x.clone()
    i, j = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., i] * s + x[..., j] * c
    return y


class Pages:
    """A cache with its sequences: pages dealt out at random, a few spare."""

    def __init__(self, lengths, kv_heads, dim, page, seed=0, capacity=None, spare=2):
        g = gen(1000 + seed)
        self.lengths, self.H, self.D, self.page = list(lengths), kv_heads, dim, page
        need = [-(-max(x, 1) // page) for x in (capacity or lengths)]
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, device="cuda", generator=g).to(torch.int32)
        self.table = torch.full((len(need), max(need) + 1), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = order[at:at + n]
            at += n
        shape = (self.pages, kv_heads, page, dim)
        self.codes = [torch.randint(-127, 128, shape, dtype=torch.int8, device="cuda", generator=g) for _ in range(2)]
        self.scale = [(torch.rand(shape[:2], device="cuda", generator=g) + 0.5) / 64 for _ in range(2)]
        self.length = ints(lengths)
        self.handle = binding.Cache(self.codes[0].data_ptr(), self.codes[1].data_ptr(), self.scale[0].data_ptr(), self.scale[1].data_ptr(),
                                    self.pages)

    def batch(self, n, rows=None, longest=None):
        self._starts = getattr(self, "_starts", []) + [starts(n)]
        return binding.Batch(len(n), sum(n) if rows is None else rows, max(list(n) + [1]) if longest is None else longest,
                             self._starts[-1].data_ptr(), self.length.data_ptr(), self.table.data_ptr(), self.table.shape[1])

    def values(self, which, seq, upto):
        """What the cache holds of a sequence: [tokens, heads, dim] float64 (0 in pages that are not there)."""
        out = torch.zeros((upto, self.H, self.D), dtype=torch.float64, device="cuda")
        for p in range(-(-upto // self.page)):
            at = int(self.table[seq, p]) if p < self.table.shape[1] else -1
            if 0 <= at < self.pages:
                n = min(self.page, upto - p * self.page)
                v = self.codes[which][at, :, :n].double() * self.scale[which][at].double()[:, None, None]
                out[p * self.page:p * self.page + n] = v.transpose(0, 1)
        return out

    def there(self, seq, upto):
        """Which tokens of a sequence are in pages that are there."""
        p = torch.arange(upto, device="cuda") // self.page
        at = torch.where(p < self.table.shape[1], self.table[seq, p.clamp(max=self.table.shape[1] - 1)], torch.full_like(p, -1, dtype=torch.int32))
        return (at >= 0) & (at < self.pages)


def attention(pages, n, q, q_heads, dtype, freq=None, interleaved=False, window=0, scale=None):
    """(result, bound) [rows, q_heads * dim] in 64 bits for q [rows, q_heads * dim].

    The bound: queries rounded with relative error e_q (2^-11 or, as two parts, 2^-22) and fp32 sums of dim products, each
    matrix instruction cutting its sum (2^-23), move a score by at most d = (e_q + (dim + 8) 2^-23) sum |q k| scale, and its
    own roundings (times a factor, minus the maximum: 2^-22) by |s| 2^-21; exp2 by 2^-21; a probability is rounded
    by e_q again; sums over n tokens by (n/16 + 16) 2^-23.  Numerator and denominator both move: twice the sum, times
    sum p |v|; the result's own rounding on top (and fp16's least step)."""
    H, D = pages.H, pages.D
    G = q_heads // H
    scale = D ** -0.5 if scale is None else scale
    eq = 2.0 ** -11 if dtype == "f16" else 2.0 ** -22
    out, bound, at = [], [], 0
    for i, m in enumerate(n):
        length = pages.lengths[i]
        pos = torch.arange(length - m, length, device="cuda")
        x = turned(q[at:at + m].double().view(m, q_heads, D), pos, freq, interleaved)
        k, v = pages.values(0, i, length), pages.values(1, i, length)
        j = torch.arange(length, device="cuda")
        sees = (j <= pos[:, None]) & pages.there(i, length)
        if window:
            sees &= j > pos[:, None] - window
        y = torch.zeros((m, q_heads, D), dtype=torch.float64, device="cuda")
        b = torch.zeros_like(y)
        for h in range(q_heads):
            if length == 0:
                continue
            s = (x[:, h] @ k[:, h // G].T * scale).masked_fill(~sees, -math.inf)
            top = s.amax(1, keepdim=True)
            p = torch.where(sees, torch.exp(s - torch.where(top == -math.inf, 0.0, top)), 0.0)
            total = p.sum(1, keepdim=True)
            p = p / torch.where(total == 0, 1.0, total)
            vv = torch.where(sees.any(0)[:, None], v[:, h // G], 0.0)
            y[:, h] = p @ vv
            moved = (eq + (D + 8) * 2.0 ** -23) * (x[:, h].abs() @ k[:, h // G].abs().T * scale).masked_fill(~sees, 0).amax(1, keepdim=True)
            moved = moved + s.masked_fill(~sees, 0).abs().amax(1, keepdim=True) * 2.0 ** -20 + 2.0 ** -21 + eq + (length / 16 + 16) * 2.0 ** -23
            b[:, h] = 2 * moved * (p @ vv.abs()) + HALF_STEP[dtype] * y[:, h].abs() + (2.0 ** -25 if dtype == "f16" else 1e-37)
        out.append(y.flatten(1))
        bound.append(b.flatten(1))
        at += m
    return torch.cat(out), torch.cat(bound)


def attend(op, pages, n, q, q_heads, dtype, rows=None, longest=None, stride=None, shift=0):
    """Runs the kernel; the result with its guards."""
    q = q if isinstance(q, Guarded) else _guard(q, stride, shift)
    batch = pages.batch(n, rows=rows, longest=longest)
    y = Guarded(q.t.shape[0], q.t.shape[1], T[dtype], stride, shift)
    work = torch.full((op.workspace(batch) // 4 + 1,), float("nan"), device="cuda")     # nothing in it may count
    op.run(q.ptr(), q.stride, batch, pages.handle, y.ptr(), y.stride, work.data_ptr(), stream())
    torch.cuda.synchronize()
    return y


def _guard(t, stride=None, shift=0):
    g = Guarded(t.shape[0], t.shape[1], t.dtype, stride, shift)
    g.t.copy_(t)
    return g


guard = _guard


# --- adapters -------------------------------------------------------------------------------------
def adapters(x, y, n, which, a, b, scale, dtype):
    """(result, bound): inner sums of k products in fp32 (each matrix instruction cuts: (k/8 + 16) 2^-23), kept to 2^-11 of
    the row's largest in fp16 or split in two (2^-21 for both operands' rests) in fp32; outer sums of rank products; one rounding."""
    out, bound, at = y.double().clone(), torch.zeros(y.shape, dtype=torch.float64, device="cuda"), 0
    for m, w in zip(n, which):
        r = slice(at, at + m)
        if 0 <= w < a.shape[0]:
            xa, A, B, s = x[r].double(), a[w].double(), b[w].double(), float(scale[w])
            h, size = xa @ A.T, xa.abs() @ A.abs().T
            split = 2.0 ** -20 if dtype == "f32" else 0.0
            moved = size * ((x.shape[1] / 8 + 16) * 2.0 ** -23 + split) + (2.0 ** -11 * h.abs().amax(1, keepdim=True) if dtype == "f16" else 0.0)
            out[r] += s * (h @ B.T)
            bound[r] = abs(s) * (moved @ B.abs().T + h.abs() @ B.abs().T * ((a.shape[1] / 8 + 8) * 2.0 ** -23 + split))
            bound[r] += (HALF_STEP[dtype] + 2.0 ** -23) * (out[r].abs() + bound[r]) + (2.0 ** -25 if dtype == "f16" else 1e-37)
        at += m
    return out, bound


# --- log probabilities ------------------------------------------------------------------------------
def logprobs(x, token, top):
    """{name: (value, bound)} for x [rows, vocab].  A term e^(x-m) is off by 2^-22 (exp2) and 2^-23 |x - m| (its argument), where it counts
    (|x - m| < 25); sums of vocab/512 terms in a thread and 9 + 4 joins: 2^-24 each, so lse moves by d = 2^-22 + 25 2^-23 + (vocab/512 + 32)
    2^-24; an answer x - m - log s by d and the roundings of two subtractions; the entropy log s - w/s by d (1 + mean |x - m|) twice."""
    x = x.double()
    V = x.shape[1]
    m = x.amax(1, keepdim=True)
    bad = torch.isnan(x).any(1) | (m[:, 0] == math.inf)
    empty = ~bad & (m[:, 0] == -math.inf)
    shifted = x - torch.where((bad | empty)[:, None], 0.0, m)
    logp = torch.where(x == -math.inf, -math.inf, shifted - torch.log(torch.exp(shifted).sum(1, keepdim=True)))
    logp[empty] = -math.inf
    logp[bad] = math.nan
    p = torch.exp(logp)
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
    entropy[bad] = math.nan
    entropy[empty] = 0.0
    d = 2.0 ** -22 + 25 * 2.0 ** -23 + (V / 512 + 32) * 2.0 ** -24
    bound = lambda v: d + 3 * 2.0 ** -24 * (v.abs().nan_to_num(0, 0, 0) + 20)      # noqa: E731
    got = {"entropy": (entropy, 2 * d * (2 + entropy.nan_to_num(0).abs()) + 2.0 ** -22)}
    if token is not None:
        t = token.long()
        asked = logp.gather(1, t.clamp(0, V - 1)[:, None])[:, 0]
        asked = torch.where((t < 0) | (t >= V), math.nan, asked)
        asked[t == -1] = 0.0
        got["logprob"] = (asked, bound(asked))
    if top:
        order = torch.sort(torch.where(torch.isnan(x), -math.inf, x), dim=1, descending=True, stable=True).indices[:, :top]
        values = logp.gather(1, order)
        order = torch.where((x.gather(1, order) == -math.inf) | bad[:, None], -1, order)
        values = torch.where(bad[:, None], math.nan, torch.where(order < 0, -math.inf, values))
        got["top"] = (order, None)
        got["top_logprob"] = (values, bound(values))
    return got
