"""What is measured of the operators that serve language models with pruned projections.

A step of such a model runs its block-pruned products (`BlockGemm`) and, between and behind them, these four:

  adapters  low-rank adapters of many requests beside a shared product:  y[r] += s_a (x[r] A_a^T) B_a^T
  append    new keys (rotated by their position) and values into a paged cache held in 8 bits, a scale for each page and head;
            the values that the touched pages then stand for are read back (`read`, which exports cached tokens)
  attend    attention of new rows over that cache: softmax(rot(q) k^T / sqrt(d)) v, causal, optionally in a window
  logprobs  log probability of a given token, entropy and top alternatives of rows of logits
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_T = {"f32": torch.float32, "f16": torch.float16}
_EB = {"f32": 4, "f16": 2}


# --- cases -------------------------------------------------------------------
def _adapters(name, requests, longest, k, c_out, rank, adapters, dtype, seed):
    return {"name": name, "kind": "adapters", "requests": requests, "longest": longest, "k": k, "c_out": c_out, "rank": rank,
            "adapters": adapters, "dtype": dtype, "ragged": seed}


def _append(name, seqs, longest, cached, heads, dim, page, dtype, seed, *, rotary=None, interleaved=False):
    return {"name": name, "kind": "append", "seqs": seqs, "longest": longest, "cached": cached, "heads": heads, "dim": dim, "page": page,
            "dtype": dtype, "ragged": seed, "rotary": dim if rotary is None else rotary, "interleaved": interleaved}


def _attend(name, seqs, longest, cached, group, heads, dim, page, dtype, seed, *, rotary=None, interleaved=False, window=0):
    return {"name": name, "kind": "attend", "seqs": seqs, "longest": longest, "cached": cached, "group": group, "heads": heads, "dim": dim,
            "page": page, "dtype": dtype, "ragged": seed, "rotary": dim if rotary is None else rotary, "interleaved": interleaved,
            "window": window}


def _logprobs(name, rows, vocab, top, dtype, *, banned=0.0):
    return {"name": name, "kind": "logprobs", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "banned": banned}


def listed():
    return [
        # a decoding step of a busy server: every request one token, its adapter any of the resident ones
        _adapters("adapters_decode_f16", 48, 1, 4096, 4096, 16, 32, "f16", 1),
        # prompts of four tenants in one step, adapters of a high rank
        _adapters("adapters_prompt_f16", 4, 2048, 4096, 4096, 64, 8, "f16", 2),
        # a classifier's fully connected layer (1000 to 1000), fp32, odd rank, mixed lengths
        _adapters("adapters_ragged_f32", 11, 17, 1000, 1000, 12, 5, "f32", 3),
        # a decoding step: one token of each of 64 requests, anywhere in their pages
        _append("append_decode_f16", 64, 1, 4000, 8, 128, 64, "f16", 4),
        # prompts going in, most pages begun anew
        _append("append_prompt_f16", 4, 4096, 500, 8, 128, 64, "f16", 5),
        # odd lengths, small pages, part of a head rotated, pairs side by side
        _append("append_ragged_f32", 7, 300, 100, 12, 64, 16, "f32", 6, rotary=32, interleaved=True),
        # one interactive request: latency counts
        _attend("attend_single_f16", 1, 1, 1000, 4, 8, 128, 64, "f16", 7),
        # a decoding step of a busy server over long contexts: the cache's bytes count
        _attend("attend_decode_f16", 64, 1, 8192, 4, 8, 128, 64, "f16", 8),
        # a chunk of two prompts behind what is cached of them: products count
        _attend("attend_chunk_f16", 2, 1024, 5000, 4, 8, 128, 64, "f16", 9),
        # a few proposed tokens to check for each request, as many key heads as query heads, fp32, a window
        _attend("attend_ragged_f32", 9, 8, 1500, 1, 12, 64, 16, "f32", 10, window=1024),
        # the answers of a decoding step: a large vocabulary, banned tokens, twenty alternatives
        _logprobs("logprobs_decode_f16", 16, 128000, 20, "f16", banned=0.1),
        # scoring prompts
        _logprobs("logprobs_prompt_f32", 2048, 32000, 5, "f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _positions(rng, dim):
    """How a model turns its heads: all of the head, or a part; halves or neighbours paired."""
    return {"rotary": rng.choice([dim, dim, dim // 2, 0]), "interleaved": rng.random() < 0.3}


# A drawn case moves and computes no more than the largest listed ones.
_MOST = {"adapters": (1.5e8, 5e9), "append": (1.6e8, 1e12), "attend": (6.8e8, 1.2e11), "logprobs": (2.6e8, 1e12)}


def draw(rng):
    while True:
        kind = rng.choice(["adapters", "append", "attend", "logprobs"])
        dtype = rng.choice(["f16", "f16", "f32"])
        seed = rng.randrange(1 << 30)
        # lengths: decoding, a few tokens each, prompts
        longest = rng.choice([1, 1, _log(rng, 2, 32), _log(rng, 32, 2048)])
        if kind == "adapters":
            k, c_out = (_log(rng, 64, 8192) // q * q or q for q in (rng.choice([1, 8, 64]), rng.choice([1, 8, 64])))
            c = _adapters("", _log(rng, 1, 128), longest, k, c_out, rng.choice([4, 8, 16, 32, 64, _log(rng, 1, 64)]), _log(rng, 1, 64),
                          dtype, seed)
            if c["adapters"] * c["rank"] * (k + c_out) > 3e7:
                continue
        elif kind == "append":
            dim = rng.choice([32, 64, 96, 128, 256])
            c = _append("", _log(rng, 1, 128), longest, _log(rng, 1, 8000), rng.choice([1, 2, 4, 8, 12]), dim, rng.choice([16, 32, 64, 128]),
                        dtype, seed, **_positions(rng, dim))
        elif kind == "attend":
            dim = rng.choice([32, 64, 96, 128, 256])
            c = _attend("", _log(rng, 1, 128), longest, _log(rng, 1, 16000), rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), rng.choice([1, 2, 4, 8, 12]),
                        dim, rng.choice([16, 32, 64, 128]), dtype, seed, window=rng.choice([0, 0, _log(rng, 16, 4096)]), **_positions(rng, dim))
            n, total = _lengths(c)
            # the plain form's padded scores and keys
            if len(n) * max(n) * max(total) * c["group"] * c["heads"] > 5e8 or len(n) * max(total) * c["heads"] * dim > 6e8:
                continue
        else:
            c = _logprobs("", _log(rng, 1, 2048), _log(rng, 1000, 160000), rng.choice([0, 1, 5, 20, 32]), dtype,
                          banned=rng.choice([0.0, 0.0, 0.3]))
        w = work(c)
        if w["bytes"] <= _MOST[kind][0] and w["flops"] <= _MOST[kind][1]:
            del c["name"]
            return c


# --- sizes -------------------------------------------------------------------
def _lengths(c):
    """(new rows of each sequence or request, tokens of each behind them): one case, one set."""
    rng = random.Random(c["ragged"])
    n = [c["longest"]] + [max(1, rng.randint(c["longest"] // 3, c["longest"])) for _ in range(c.get("seqs", c.get("requests")) - 1)]
    return n, [x + rng.randint(c["cached"] // 3, c["cached"]) for x in n] if "cached" in c else n


def _choice(c):
    """The adapter of each request; one request in eight has none."""
    rng = random.Random(c["ragged"] + 1)
    return [-1 if rng.random() < 1 / 8 else rng.randrange(c["adapters"]) for _ in range(c["requests"])]


def _visible(c):
    """(pairs of a row and a token that it sees, tokens that some row sees), over all sequences."""
    n, total = _lengths(c)
    pairs = tokens = 0
    for m, length in zip(n, total):
        seen = [min(length - m + i + 1, c["window"] or 1 << 40) for i in range(m)]
        pairs += sum(seen)
        tokens += min(length, seen[0] + m - 1)
    return pairs, tokens


def work(case):
    """Inputs read once and outputs written once; two operations a multiply-add."""
    c = case
    if c["kind"] == "logprobs":
        return {"bytes": c["rows"] * (c["vocab"] * _EB[c["dtype"]] + 12 + 8 * c["top"]), "flops": 6 * c["rows"] * c["vocab"]}
    b = _EB[c["dtype"]]
    n, total = _lengths(c)
    if c["kind"] == "adapters":
        a = _choice(c)
        rows = sum(m for m, x in zip(n, a) if x >= 0)
        per_row = c["rank"] * (c["k"] + c["c_out"])
        return {"bytes": (rows * c["k"] + 2 * sum(n) * c["c_out"] + len({x for x in a if x >= 0}) * per_row) * b, "flops": 2 * rows * per_row}
    hd = c["heads"] * c["dim"]
    if c["kind"] == "append":
        rows = sum(n)
        back = sum(t - (t - m) // c["page"] * c["page"] for m, t in zip(n, total))      # tokens of the touched pages
        # new rows in, their codes out; older codes of the pages in; all of them read back out in fp16
        return {"bytes": 2 * hd * (rows * (b + 1) + (back - rows) + back * (1 + 2)), "flops": 10 * rows * hd}
    pairs, tokens = _visible(c)
    return {"bytes": 2 * hd * tokens + 8 * c["heads"] * (tokens // c["page"] + 1) + 2 * sum(n) * c["group"] * hd * b,
            "flops": 4 * pairs * c["group"] * hd}


# --- inputs ------------------------------------------------------------------
def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(n):
    return _ints([0] + list(np.cumsum(n)))


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    t = _T[c["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, device="cuda", generator=g) * std).to(t)

    if c["kind"] == "logprobs":
        x = normal(c["rows"], c["vocab"], std=3.0)
        if c["banned"]:                                     # what a grammar or a stop list leaves out
            x.masked_fill_(torch.rand(x.shape, device="cuda", generator=g) < c["banned"], -math.inf)
        return {"case": c, "x": x, "token": torch.randint(0, c["vocab"], (c["rows"],), dtype=torch.int32, device="cuda", generator=g)}
    n, total = _lengths(c)
    s = {"case": c, "n": _starts(n)}
    rows = sum(n)
    if c["kind"] == "adapters":
        s["a"] = normal(c["adapters"], c["rank"], c["k"], std=c["k"] ** -0.5)
        s["b"] = normal(c["adapters"], c["c_out"], c["rank"], std=c["rank"] ** -0.5)
        s["scale"] = torch.rand(c["adapters"], device="cuda", generator=g) + 0.5
        s["x"], s["y"], s["adapter"] = normal(rows, c["k"]), normal(rows, c["c_out"]), _ints(_choice(c))
        return s
    # the cache as earlier steps left it: pages in any order, codes about normal, scales of about 1/32
    need = [-(-x // c["page"]) for x in total]
    pages = sum(need) + 3
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table, at = torch.zeros((len(n), max(need)), dtype=torch.int32, device="cuda"), 0
    for i, x in enumerate(need):
        table[i, :x] = order[at:at + x]
        at += x
    s["table"], s["length"], s["pages"] = table, _ints(total), pages
    for w in "kv":
        codes = torch.empty((pages, c["heads"], c["page"], c["dim"]), dtype=torch.int8, device="cuda")
        for i in range(0, pages, 4096):
            codes[i:i + 4096] = (torch.randn(codes[i:i + 4096].shape, device="cuda", generator=g) * 32).round_().clamp_(-127, 127).to(torch.int8)
        s[w + "_codes"] = codes
        s[w + "_scale"] = (torch.rand((pages, c["heads"]), device="cuda", generator=g) + 0.5) / 32
    s["freq"] = 10000.0 ** (-np.arange(c["rotary"] // 2) * 2.0 / c["rotary"]) if c["rotary"] else None
    if c["kind"] == "append":
        hd = c["heads"] * c["dim"]
        kv = normal(rows, 2 * hd)                            # the product's output: keys, then values
        s["kv"], s["stride"] = kv, 2 * hd
        back = [t - (t - m) // c["page"] * c["page"] for m, t in zip(n, total)]
        s["back"] = _starts(back)
        s["rows_back"], s["longest_back"] = sum(back), max(back)
    else:
        s["q"] = normal(rows, c["group"] * c["heads"] * c["dim"])
    return s


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    if own:
        from paper_2206_10620_b200 import binding
    if c["kind"] == "logprobs":
        r, k = c["rows"], c["top"]
        s["logprob"], s["entropy"] = (torch.empty(r, device="cuda") for _ in range(2))
        s["top"], s["top_logprob"] = torch.empty((r, k), dtype=torch.int32, device="cuda"), torch.empty((r, k), device="cuda")
        if own:
            s["op"] = binding.LogProbs(c["vocab"], c["dtype"], c["top"])
    elif c["kind"] == "adapters":
        s["out"] = torch.empty_like(s["y"])
        if own:
            s["op"] = binding.Adapters(c["k"], c["c_out"], c["dtype"], s["a"].cpu().numpy(), s["b"].cpu().numpy(), s["scale"].cpu().numpy())
    else:
        if own:
            s["op"] = binding.Attention(c["heads"] * c.get("group", 1), c["heads"], c["dim"], c["page"], c["dtype"], freq=s["freq"],
                                        interleaved=c["interleaved"], window=c.get("window", 0))
            s["cache"] = binding.Cache(s["k_codes"].data_ptr(), s["v_codes"].data_ptr(), s["k_scale"].data_ptr(), s["v_scale"].data_ptr(),
                                       s["pages"])

            def batch(start, rows, longest):
                return binding.Batch(len(s["length"]), rows, longest, start.data_ptr(), s["length"].data_ptr(), s["table"].data_ptr(),
                                     s["table"].shape[1])

            s["batch"] = batch(s["n"], sum(_lengths(c)[0]), c["longest"])
        if c["kind"] == "append":
            s["k_out"], s["v_out"] = (torch.empty((s["rows_back"], c["heads"] * c["dim"]), dtype=torch.float16, device="cuda") for _ in range(2))
            if own:
                s["batch_back"] = batch(s["back"], s["rows_back"], s["longest_back"])
        else:
            s["y"] = torch.empty_like(s["q"])
            if own:
                s["work"] = torch.empty(s["op"].workspace(s["batch"]), dtype=torch.uint8, device="cuda")
    return s


# --- one pass ----------------------------------------------------------------
def run(state):
    s = state
    c = s["case"]
    if not own:
        return _PLAIN[c["kind"]](s)
    op, stream = s["op"], torch.cuda.current_stream().cuda_stream
    if c["kind"] == "logprobs":
        op.run(s["x"].data_ptr(), c["rows"], c["vocab"], s["token"].data_ptr(), s["logprob"].data_ptr(), s["entropy"].data_ptr(),
               s["top"].data_ptr(), s["top_logprob"].data_ptr(), stream)
        return {"logprob": s["logprob"], "entropy": s["entropy"], "top": s["top"], "top_logprob": s["top_logprob"]}
    if c["kind"] == "adapters":
        op.run(s["x"].data_ptr(), s["x"].shape[0], c["k"], s["n"].data_ptr(), s["adapter"].data_ptr(), c["requests"], s["y"].data_ptr(),
               c["c_out"], s["out"].data_ptr(), c["c_out"], stream)
        return s["out"]
    if c["kind"] == "append":
        kv = s["kv"].data_ptr()
        op.append(kv, kv + s["stride"] // 2 * _EB[c["dtype"]], s["stride"], s["batch"], s["cache"], stream)
        op.read(s["batch_back"], s["cache"], s["k_out"].data_ptr(), s["v_out"].data_ptr(), c["heads"] * c["dim"], "f16", stream)
        return {"k": s["k_out"], "v": s["v_out"]}
    width = s["q"].shape[1]
    op.run(s["q"].data_ptr(), width, s["batch"], s["cache"], s["y"].data_ptr(), width, s["work"].data_ptr(), stream)
    return s["y"]


def _plain_logprobs(s):
    x = s["x"].float()
    top = x.amax(1, keepdim=True)
    shifted = x - top
    e = torch.exp(shifted)
    total = e.sum(1, keepdim=True)
    logp = shifted - torch.log(total)
    p = e / total
    entropy = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :s["case"]["top"]]
    return {"logprob": logp.gather(1, s["token"].long()[:, None])[:, 0], "entropy": entropy, "top": order.to(torch.int32),
            "top_logprob": logp.gather(1, order)}


def _owners(start, rows):
    """The sequence that each of `rows` rows belongs to."""
    return torch.searchsorted(start, torch.arange(rows, dtype=torch.int32, device="cuda"), right=True) - 1


def _plain_adapters(s):
    # every row through all adapters, the others' columns taken out between the two products
    x, a, b = s["x"].float(), s["a"].float(), s["b"].float()
    mine = s["adapter"].long()[_owners(s["n"], x.shape[0])]
    keep = (mine[:, None] == torch.arange(a.shape[0], device="cuda")) * s["scale"]
    h = (x @ a.flatten(0, 1).T).view(x.shape[0], *a.shape[:2]) * keep[:, :, None]
    return (s["y"].float() + h.flatten(1) @ b.transpose(1, 2).flatten(0, 1)).to(s["y"].dtype)


def _turned(x, position, s):
    """x [rows, heads, dim] in fp32, its leading `rotary` components turned by position times frequency."""
    c, r = s["case"], s["case"]["rotary"]
    if not r:
        return x
    angle = position.double()[:, None] * torch.from_numpy(s["freq"]).cuda()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    head, tail = x[..., :r], x[..., r:]
    u, v = (head[..., 0::2], head[..., 1::2]) if c["interleaved"] else (head[..., :r // 2], head[..., r // 2:])
    a, b = u * cos - v * sin, u * sin + v * cos
    both = torch.stack((a, b), -1).flatten(-2) if c["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((both, tail), -1)


def _places(s, start, rows):
    """(sequence, position, page, slot) of each row: the last ones of its sequence."""
    who = _owners(start, rows)
    position = s["length"].long()[who] - (start.long()[who + 1] - torch.arange(rows, device="cuda"))
    page = s["table"].long()[who, position // s["case"]["page"]]
    return who, position, page, position % s["case"]["page"]


def _plain_append(s):
    c = s["case"]
    heads, dim = c["heads"], c["dim"]
    rows = s["kv"].shape[0]
    who, position, page, slot = _places(s, s["n"], rows)
    first = (slot == 0) | (torch.arange(rows, device="cuda") == s["n"].long()[who])   # the first new row of a page
    item = torch.cumsum(first, 0) - 1
    pages, begun = page[first], slot[first]
    both = s["kv"].float().view(rows, 2, heads, dim)
    new = torch.zeros((len(pages), c["page"], 2, heads, dim), device="cuda")
    new[item, slot] = torch.stack((_turned(both[:, 0], position, s), both[:, 1]), 1)
    fresh = torch.zeros((len(pages), c["page"]), dtype=torch.bool, device="cuda")
    fresh[item, slot] = True
    old = torch.arange(c["page"], device="cuda") < begun[:, None]
    out = []
    _, _, page_back, slot_back = _places(s, s["back"], s["rows_back"])
    for i, w in enumerate("kv"):
        codes, scales = s[w + "_codes"], s[w + "_scale"]
        x = new[:, :, i].transpose(1, 2)                                              # [page, head, slot, dim]
        most = x.abs().amax((2, 3))
        was = torch.where(begun[:, None] > 0, scales[pages], torch.zeros_like(most))
        m, e = torch.frexp(most / (127.5 * was))                                      # 2^e >= the ratio, 2^(e-1) is not
        up = torch.where(was > 0, torch.clamp(e - (m == 0.5).int(), min=0), torch.zeros_like(e)).float()
        scale = torch.where(was > 0, was * torch.exp2(up), most / 127)
        kept = torch.round(codes[pages].float() * torch.exp2(-up)[:, :, None, None])
        q = torch.clamp(torch.round(x / torch.where(scale > 0, scale, torch.ones_like(scale))[:, :, None, None]), -127, 127)
        stays = codes[pages].float()
        codes[pages] = torch.where(fresh[:, None, :, None], q, torch.where(old[:, None, :, None], kept, stays)).to(torch.int8)
        scales[pages] = scale
        back = codes[page_back, :, slot_back].float() * scales[page_back][:, :, None]
        out.append(back.flatten(1).to(torch.float16))
    return {"k": out[0], "v": out[1]}


def _plain_attend(s):
    c = s["case"]
    heads, dim, group = c["heads"], c["dim"], c["group"]
    rows, longest, seqs = s["q"].shape[0], c["longest"], len(s["length"])
    who, position, _, _ = _places(s, s["n"], rows)
    within = torch.arange(rows, device="cuda") - s["n"].long()[who]
    q = torch.zeros((seqs, longest, heads, group, dim), device="cuda")
    q[who, within] = _turned(s["q"].float().view(rows, heads * group, dim), position, s).view(rows, heads, group, dim)
    at = torch.full((seqs, longest), -1, device="cuda")
    at[who, within] = position
    table = s["table"].long()
    tokens = table.shape[1] * c["page"]

    def cached(w):                                                                    # [seq, head, token, dim]
        x = s[w + "_codes"][table].float() * s[w + "_scale"][table][..., None, None]
        return x.transpose(1, 2).reshape(seqs, heads, tokens, dim)

    scores = q.permute(0, 2, 1, 3, 4).reshape(seqs, heads, longest * group, dim) @ cached("k").transpose(2, 3) * dim ** -0.5
    j = torch.arange(tokens, device="cuda")
    sees = (j <= at[..., None]) & (j > at[..., None] - (c["window"] or tokens))
    sees = sees.repeat_interleave(group, 1)[:, None]
    scores = scores.masked_fill_(~sees, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores.sub_(torch.where(top > -math.inf, top, torch.zeros_like(top))))
    total = e.sum(-1, keepdim=True)
    y = (e @ cached("v")) / torch.where(total > 0, total, torch.ones_like(total))
    y = y.view(seqs, heads, longest, group, dim).permute(0, 2, 1, 3, 4)[who, within]
    return y.reshape(rows, -1).to(s["q"].dtype)


_PLAIN = {"logprobs": _plain_logprobs, "adapters": _plain_adapters, "append": _plain_append, "attend": _plain_attend}


# --- the definitions in 64 bits ------------------------------------------------
def exact(case, seed):
    c, s = case, _inputs(case, seed)
    return {"logprobs": _exact_logprobs, "adapters": _exact_adapters, "append": _exact_append, "attend": _exact_attend}[c["kind"]](c, s)


def _exact_logprobs(c, s):
    logprob, entropy, top, values = [], [], [], []
    for i in range(0, c["rows"], 64):
        logp = torch.log_softmax(s["x"][i:i + 64].double(), 1)
        logprob.append(logp.gather(1, s["token"][i:i + 64].long()[:, None])[:, 0])
        entropy.append(torch.special.entr(logp.exp()).sum(1))
        v, k = torch.sort(s["x"][i:i + 64].double(), dim=1, descending=True, stable=True)
        top.append(k[:, :c["top"]].to(torch.int32))
        values.append(logp.gather(1, k[:, :c["top"]]))
    return {"logprob": torch.cat(logprob), "entropy": torch.cat(entropy), "top": torch.cat(top), "top_logprob": torch.cat(values)}


def _exact_adapters(c, s):
    y, start = s["y"].double(), s["n"].tolist()
    for i, a in enumerate(s["adapter"].tolist()):
        if a >= 0:
            r = slice(start[i], start[i + 1])
            y[r] += s["scale"][a].double() * (s["x"][r].double() @ s["a"][a].double().T @ s["b"][a].double().T)
    return y


def _exact_turn(x, first, s):
    """x [rows, heads, dim] in 64 bits, row i at position first + i: each pair as a complex number times e^(i angle)."""
    c, r = s["case"], s["case"]["rotary"]
    if not r:
        return x
    angle = torch.arange(first, first + len(x), device=x.device).double()[:, None] * torch.tensor(s["freq"], device=x.device)
    by = torch.polar(torch.ones_like(angle), angle)[:, None]
    y = x.clone()
    even, odd = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    z = torch.complex(x[..., even], x[..., odd]) * by
    y[..., even], y[..., odd] = z.real, z.imag
    return y


def _exact_append(c, s):
    heads, dim, page = c["heads"], c["dim"], c["page"]
    start, out = s["n"].tolist(), {"k": [], "v": []}
    for i, length in enumerate(s["length"].tolist()):
        n = start[i + 1] - start[i]
        x = s["kv"][start[i]:start[i + 1]].double().view(n, 2, heads, dim)
        new = {"k": _exact_turn(x[:, 0], length - n, s), "v": x[:, 1]}
        for w in "kv":
            for p in range((length - n) // page, (length - 1) // page + 1):
                lo, hi = max(p * page, length - n), min((p + 1) * page, length)
                y = new[w][lo - (length - n):hi - (length - n)].transpose(0, 1)      # [head, token, dim]
                most, at = y.abs().amax((1, 2)), int(s["table"][i, p])
                if lo == p * page:
                    scale, old = most / 127, y[:, :0]
                else:
                    was = s[w + "_scale"][at].double()
                    up = torch.ceil(torch.log2(most / (127.5 * was))).clamp(min=0)
                    scale = was * 2 ** up
                    old = torch.round(s[w + "_codes"][at, :, :lo - p * page].double() * (2 ** -up)[:, None, None])
                codes = torch.round(y / scale[:, None, None]).clamp(-127, 127)
                out[w].append((torch.cat((old, codes), 1) * scale[:, None, None]).transpose(0, 1).flatten(1))
    return {w: torch.cat(x) for w, x in out.items()}


def _exact_attend(c, s):
    heads, dim, group, page = c["heads"], c["dim"], c["group"], c["page"]
    start, out = s["n"].tolist(), []
    for i, length in enumerate(s["length"].tolist()):
        n = start[i + 1] - start[i]
        q = _exact_turn(s["q"][start[i]:start[i + 1]].double().view(n, heads * group, dim), length - n, s)
        at = s["table"][i, :-(-length // page)].long()
        position = torch.arange(length - n, length, device="cuda")[:, None]
        j = torch.arange(length, device="cuda")
        hidden = (j > position) | ((position - j >= c["window"]) if c["window"] else (j < 0))
        y = torch.empty_like(q)
        for h in range(heads):
            k, v = ((s[w + "_codes"][at, h].double() * s[w + "_scale"][at, h].double()[:, None, None]).flatten(0, 1)[:length] for w in "kv")
            for m in range(h * group, (h + 1) * group):
                y[:, m] = torch.softmax((q[:, m] @ k.T / math.sqrt(dim)).masked_fill(hidden, -math.inf), 1) @ v
        out.append(y.flatten(1))
    return torch.cat(out)
