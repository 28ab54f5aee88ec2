"""What is measured: the operators of prompts, through the public binding.

A serving program lets whole prompts attend to themselves, packed one after the other, or brings them to a paged cache in chunks
whose queries attend to all tokens of their sequence so far; it copies pages where sequences fork or a cache is compacted.  A training
program runs the attention of packed sequences forward and backward.  Every case below is one such call (training: the two passes).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # one short question, where the call's own latency is what counts
        {"name": "prompt_short", "op": "prompt", "seqs": 1, "longest": 33, "heads": 32, "kv_heads": 8, "dim": 128,
         "causal": True, "dtype": "bf16", "padding": 0},
        # requests of all lengths, packed, the batch padded to a fixed number of rows
        {"name": "prompt_packed", "op": "prompt", "seqs": 24, "longest": 1999, "heads": 32, "kv_heads": 8, "dim": 128,
         "causal": True, "dtype": "bf16", "padding": 40},
        # an encoder's sentences: every token sees every other one, a head of 64, as many key heads as query heads
        {"name": "prompt_encoder", "op": "prompt", "seqs": 48, "longest": 1021, "heads": 12, "kv_heads": 12, "dim": 64,
         "causal": False, "dtype": "f16", "padding": 0},
        # one long document
        {"name": "prompt_long", "op": "prompt", "seqs": 1, "longest": 16384, "heads": 32, "kv_heads": 8, "dim": 128,
         "causal": True, "dtype": "bf16", "padding": 0},
        # training: a small batch of short sequences in 16-bit floats, groups of seven heads
        {"name": "train_small", "op": "train", "seqs": 3, "longest": 257, "heads": 14, "kv_heads": 2, "dim": 64,
         "causal": True, "dtype": "f16", "padding": 1},
        # a batch of packed sequences as a training step has them
        {"name": "train_batch", "op": "train", "seqs": 8, "longest": 4096, "heads": 32, "kv_heads": 8, "dim": 128,
         "causal": True, "dtype": "bf16", "padding": 0},
        # one sequence of a long context, an odd length
        {"name": "train_long", "op": "train", "seqs": 1, "longest": 12289, "heads": 16, "kv_heads": 2, "dim": 128,
         "causal": True, "dtype": "bf16", "padding": 0},
        # a short turn of one dialogue
        {"name": "chunk_turn", "op": "chunk", "seqs": 1, "new": 17, "context": 1000, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 16, "order": "tokens", "dtype": "bf16"},
        # a server's step: chunks and single tokens of many sequences, pages that end inside a tile
        {"name": "chunk_mixed", "op": "chunk", "seqs": 40, "new": 256, "context": 6000, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 48, "order": "heads", "dtype": "bf16"},
        # the last chunk of a book, a head of 64
        {"name": "chunk_long", "op": "chunk", "seqs": 1, "new": 2048, "context": 63488, "heads": 32, "kv_heads": 4, "dim": 64,
         "page": 64, "order": "tokens", "dtype": "f16"},
        # a sequence forks into eight samples: each gets its own copy of the page that is being filled
        {"name": "copy_fork", "op": "copy", "sources": 4, "times": 8, "part": True, "kv_heads": 8, "dim": 128, "page": 64,
         "order": "tokens", "dtype": "bf16"},
        # a cache is compacted
        {"name": "copy_compact", "op": "copy", "sources": 4001, "times": 1, "part": False, "kv_heads": 8, "dim": 128, "page": 64,
         "order": "heads", "dtype": "bf16"},
    ]


HEADS = [(32, 8), (32, 32), (32, 4), (16, 2), (24, 8), (8, 1), (14, 2), (12, 12)]
MOST = {"prompt": (5.1e8, 2.19e12), "train": (7.5e8, 2.16e12), "chunk": (6.1e8, 1.08e12), "copy": (2.09e9, 1.0)}  # bytes, flops of a drawn case
MOST_SCORES = 1 << 33                                                # of all heads, hidden ones too


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["prompt", "prompt", "train", "train", "chunk", "chunk", "copy"])
        heads, kv_heads = rng.choice(HEADS)
        case = {"op": op}
        if op == "copy":
            case.update(sources=_log(rng, 1, 8000), times=rng.choice([1, 1, 1, 2, 4, 16]), part=rng.random() < 0.5, kv_heads=kv_heads,
                        dim=rng.choice([64, 128, 128, 128, 256]), page=rng.choice([16, 16, 32, 48, 64, 100, 128, 256]),
                        order=rng.choice(["tokens", "heads"]), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
        else:
            case.update(heads=heads, kv_heads=kv_heads, dim=rng.choice([64, 128, 128]), dtype=rng.choice(["bf16", "bf16", "f16"]),
                        seqs=_log(rng, 1, 64))
            if op == "chunk":
                case.update(new=_log(rng, 1, 4096), context=0 if rng.random() < 0.1 else _log(rng, 1, 65536),
                            page=rng.choice([16, 16, 32, 48, 64, 100, 128, 256]), order=rng.choice(["tokens", "heads"]))
            else:
                case.update(longest=_log(rng, 1, 16384), causal=rng.random() < 0.8, padding=rng.choice([0, 0, 1, 77]))
        w = work(case)
        if w["bytes"] <= MOST[op][0] and w["flops"] <= MOST[op][1]:
            if op == "copy" or case["heads"] * sum(n * m for n, m in _lengths(case)) <= MOST_SCORES:
                return case


def _lengths(case):
    """(queries, keys) of each sequence: spread evenly up to the longest, whatever the seed."""
    b = case["seqs"]

    def spread(i, least, most):
        return least + ((i + 1) * (most - least)) // b

    if case["op"] != "chunk":
        return [(n, n) for n in (spread(i, min(1, case["longest"]), case["longest"]) for i in range(b))]
    new = [spread(i, 1, case["new"]) for i in range(b)]
    return [(n, n + spread((7 * i + b // 2) % b, 0, case["context"])) for i, n in enumerate(new)]


# ---------------------------------------------------------------- inputs
def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _cache(case, pages, dtype, g, scale_k=1.0):
    kv, d, page = case["kv_heads"], case["dim"], case["page"]
    got = []
    for scale in (scale_k, 1.0):
        if case["order"] == "tokens":
            got.append(_normal(g, (pages, page, kv, d), dtype, scale))
        else:
            got.append(_normal(g, (pages, kv, page, d), dtype, scale).transpose(1, 2))
    return got


def _copies(case):
    """Tokens of each copied page: all, or the filled part of a page."""
    n = case["sources"] * case["times"]
    return [1 + (17 * (i // case["times"])) % case["page"] if case["part"] else case["page"] for i in range(n)]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = {"case": case}
    dt = DTYPES[case["dtype"]]
    if case["op"] == "copy":
        n, times = case["sources"], case["times"]
        ids = rng.permutation(n * (1 + times) + 3).astype(np.int32)
        tokens = np.array(_copies(case), np.int32)
        s["kc"], s["vc"] = _cache(case, len(ids), dt, g)
        s["src"] = torch.from_numpy(np.repeat(ids[:n], times)).cuda()
        s["dst"] = torch.from_numpy(ids[n:n + n * times].copy()).cuda()
        s["tokens"] = torch.from_numpy(tokens).cuda() if case["part"] else None
        if own:
            from paper_2607_11262_gb300 import serving
            s["cache"] = serving.PagedCache(s["kc"], s["vc"])
        return s
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    lengths = [_lengths(case)[i] for i in rng.permutation(case["seqs"])]
    at = np.concatenate([[0], np.cumsum([n for n, _ in lengths])])
    s["lengths"], s["scale"] = lengths, 1.0 / math.sqrt(d)
    s["starts"] = torch.from_numpy(at.astype(np.int32)).cuda()
    if case["op"] == "chunk":
        page = case["page"]
        lens = np.array([m for _, m in lengths], np.int64)
        held = -(-lens // page)
        ids = rng.permutation(int(held.sum()) + 2).astype(np.int32)
        table = np.full((case["seqs"], int(held.max())), -1, np.int32)
        table[np.arange(table.shape[1])[None, :] < held[:, None]] = ids[:int(held.sum())]
        s["q"] = _normal(g, (int(at[-1]), h, d), dt)
        s["kc"], s["vc"] = _cache(case, len(ids), dt, g, 1.5)        # scores of a spread that makes some keys count
        s["table"], s["lens"] = torch.from_numpy(table).cuda(), torch.from_numpy(lens.astype(np.int32)).cuda()
        if own:
            from paper_2607_11262_gb300 import serving
            s["cache"] = serving.PagedCache(s["kc"], s["vc"])
            s["workspace"] = serving.chunk_workspace(s["q"], s["starts"], s["cache"], s["table"])
        return s
    # views of one projection's rows, as a model has them
    rows = _normal(g, (int(at[-1]) + case["padding"], h + 2 * kv, d), dt)
    rows[:, h:h + kv] *= 1.5
    s["q"], s["k"], s["v"] = torch.split(rows, [h, kv, kv], dim=1)
    if case["op"] == "train":
        s["dout"] = _normal(g, s["q"].shape, dt)
        if own:
            for n in ("q", "k", "v"):
                s[n] = s[n].detach().requires_grad_()
    elif own:
        from paper_2607_11262_gb300 import serving
        s["workspace"] = serving.prompt_workspace(s["q"], s["k"], s["starts"])
    return s


# ---------------------------------------------------------------- one pass
MOST_AT_ONCE = 1 << 28                                               # scores of a piece of the plain form


def _attend(q, k, v, scale, causal, dout=None):
    """One sequence in 32 bits: queries [n, heads, dim] against keys [m, kv_heads, dim], the last query beside the last key:
    (out, lse), or (out, dq, dk, dv)."""
    n, h, d = q.shape
    m, kv = k.shape[:2]
    kt, vt = k.to(torch.float32).permute(1, 0, 2), v.to(torch.float32).permute(1, 0, 2)      # [kv, m, d]
    out = torch.empty((n, h, d), dtype=torch.float32, device="cuda")
    lse = torch.empty((n, h), dtype=torch.float32, device="cuda")
    if dout is not None:
        dq, dk, dv = torch.empty_like(out), torch.zeros_like(kt), torch.zeros_like(vt)
    step = max(1, MOST_AT_ONCE // max(1, m * h))
    for a in range(0, n, step):
        c = min(n, a + step) - a
        qt = q[a:a + c].to(torch.float32).view(c, kv, h // kv, d).permute(1, 2, 0, 3).reshape(kv, -1, d)   # [kv, group * c, d]
        x = torch.matmul(qt, kt.transpose(1, 2)) * scale
        if causal:
            last = torch.arange(a, a + c, device="cuda") + (m - n)
            hidden = torch.arange(m, device="cuda")[None, :] > last[:, None]
            x.view(kv, h // kv, c, m).masked_fill_(hidden, -math.inf)
        top = x.amax(-1, keepdim=True)
        x = torch.exp(x - top)
        total = x.sum(-1, keepdim=True)
        x = x / total
        o = torch.matmul(x, vt)

        def rows(y):
            return y.view(kv, h // kv, c, -1).permute(2, 0, 1, 3).reshape(c, h, -1)
        out[a:a + c] = rows(o)
        lse[a:a + c] = rows(top + torch.log(total))[..., 0]
        if dout is not None:
            g = dout[a:a + c].to(torch.float32).view(c, kv, h // kv, d).permute(1, 2, 0, 3).reshape(kv, -1, d)
            dv += torch.matmul(x.transpose(1, 2), g)
            y = torch.matmul(g, vt.transpose(1, 2)) - (g * o).sum(-1, keepdim=True)
            x = x * y * scale
            dq[a:a + c] = rows(torch.matmul(x, kt))
            dk += torch.matmul(x.transpose(1, 2), qt)
    if dout is None:
        return out, lse
    return out, dq, dk.permute(1, 0, 2), dv.permute(1, 0, 2)


def _plain(s):
    case, q = s["case"], s.get("q")
    if case["op"] == "copy":
        src, dst, page = s["src"].long(), s["dst"].long(), case["page"]
        tokens = s["tokens"]
        for c in (s["kc"], s["vc"]):
            if tokens is None:
                c[dst] = c[src]
            else:
                copied = (torch.arange(page, device="cuda")[None, :] < tokens[:, None])[..., None, None]
                c[dst] = torch.where(copied, c[src], c[dst])
        return [s["kc"], s["vc"]]
    train = case["op"] == "train"
    shapes = [q.shape, q.shape, s["k"].shape, s["v"].shape] if train else [q.shape]
    got = [torch.zeros(x, dtype=q.dtype, device="cuda") for x in shapes]
    if not train:
        got.append(torch.full(q.shape[:2], -math.inf, device="cuda"))
    a = 0
    for i, (n, m) in enumerate(s["lengths"]):
        if case["op"] == "chunk":
            pages = s["table"][i, :-(-m // case["page"])].long()
            k, v = (c[pages].flatten(0, 1)[:m] for c in (s["kc"], s["vc"]))
        else:
            k, v = s["k"][a:a + n], s["v"][a:a + n]
        parts = _attend(q[a:a + n], k, v, s["scale"], case.get("causal", True), s["dout"][a:a + n] if train else None)
        for to, x in zip(got, parts):
            to[a:a + n] = x.to(to.dtype)
        a += n
    return got


def run(state):
    s = state
    if not own:
        return _plain(s)
    from paper_2607_11262_gb300 import serving
    case = s["case"]
    if case["op"] == "copy":
        serving.copy_pages(s["cache"], s["src"], s["dst"], s["tokens"])
        return [s["kc"], s["vc"]]
    if case["op"] == "chunk":
        return list(serving.chunk_attention(s["q"], s["starts"], s["cache"], s["table"], s["lens"], scale=s["scale"],
                                            workspace=s["workspace"]))
    if case["op"] == "prompt":
        return list(serving.prompt_attention(s["q"], s["k"], s["v"], s["starts"], causal=case["causal"], scale=s["scale"],
                                             workspace=s["workspace"]))
    out, _ = serving.prompt_attention(s["q"], s["k"], s["v"], s["starts"], causal=case["causal"], scale=s["scale"])
    return [out.detach(), *torch.autograd.grad(out, [s["q"], s["k"], s["v"]], s["dout"])]


def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "copy":
        row, tokens = 2 * case["kv_heads"] * case["dim"] * e, _copies(case)
        return {"bytes": row * (sum(tokens) + sum(tokens[::case["times"]])) + 12 * len(tokens), "flops": 0}
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    lengths = _lengths(case)
    n, m = sum(x for x, _ in lengths), sum(y for _, y in lengths)
    seen = sum(x * y - (x * (x - 1) // 2 if case.get("causal", True) else 0) for x, y in lengths)
    size = e * d * (2 * n * h + 2 * m * kv)                          # q, out, k, v
    if case["op"] == "train":                                        # and dout, dq, dk, dv
        return {"bytes": 2 * size, "flops": 14 * seen * h * d}
    return {"bytes": size + 4 * n * h, "flops": 4 * seen * h * d}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "copy":
        old = [c.double() for c in (s["kc"], s["vc"])]
        new = [c.clone() for c in old]
        count = _copies(case)
        if len(count) > 5000:
            return None
        for src, dst, n in zip(s["src"].tolist(), s["dst"].tolist(), count):
            for x, y in zip(old, new):
                y[dst, :n] = x[src, :n]
        return new
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    train = case["op"] == "train"
    if sum(n * m for n, m in s["lengths"]) * h * d * (14 if train else 4) > 8e12:
        return None
    # a head at a time, with the derivatives of 64-bit arithmetic
    q = s["q"].detach().double()
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    if train:
        k0, v0 = s["k"].detach().double(), s["v"].detach().double()
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k0), torch.zeros_like(v0)
    a = 0
    for i, (n, m) in enumerate(s["lengths"]):
        rows = slice(a, a + n)
        a += n
        if case["op"] == "chunk":
            j = torch.arange(m, device="cuda")
            page, at = s["table"][i].long()[j // case["page"]], j % case["page"]
            ks, vs = s["kc"][page, at].double(), s["vc"][page, at].double()
        else:
            ks, vs = s["k"][rows].detach().double(), s["v"][rows].detach().double()
        mask = torch.ones(n, m, dtype=torch.bool, device="cuda")
        if case.get("causal", True):
            mask = mask.tril(m - n)
        for x in range(h):
            y = x // (h // kv)
            with torch.set_grad_enabled(train):
                a1, a2, a3 = (t.clone().requires_grad_(train) for t in (q[rows, x], ks[:, y], vs[:, y]))
                w = torch.where(mask, (a1 @ a2.T) * s["scale"], -math.inf)
                o = torch.softmax(w, -1) @ a3
                out[rows, x], lse[rows, x] = o.detach(), torch.logsumexp(w.detach(), -1)
                if train:
                    g = torch.autograd.grad(o, [a1, a2, a3], s["dout"][rows, x].double())
                    dq[rows, x] = g[0]
                    dk[rows, y] += g[1]
                    dv[rows, y] += g[2]
    return [out, dq, dk, dv] if train else [out, lse]
