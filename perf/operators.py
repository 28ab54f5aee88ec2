"""What is measured: the operators of a decode step, through the public binding.

A serving program appends the new tokens' keys and values to a paged cache, rotated to their positions on the way, and
lets their queries attend to a prefix that the whole batch shares and to each sequence's own tokens; a training program
rotates queries and keys, and rotates their gradients back.  Every case below is one call of one of the three.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # rotary positions: one decoded token, where the call's own latency is what counts
        {"name": "rope_one_token", "op": "rope", "dir": "fwd", "tokens": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "rot": 128, "layout": "half", "scaling": "none", "dtype": "bf16", "fused": True, "start": 2000},
        # a training batch of eight sequences, queries and keys as views of one projection's output
        {"name": "rope_train", "op": "rope", "dir": "fwd", "tokens": 16384, "heads": 32, "kv_heads": 8, "dim": 128,
         "rot": 128, "layout": "half", "scaling": "none", "dtype": "bf16", "fused": True, "start": 0},
        # the gradients of a long context's positions: interleaved pairs, part of the head, an odd token count
        {"name": "rope_train_grad", "op": "rope", "dir": "grad", "tokens": 8191, "heads": 32, "kv_heads": 8, "dim": 128,
         "rot": 64, "layout": "interleaved", "scaling": "by_parts", "dtype": "f32", "fused": False, "start": 120000},
        # append: one sequence decodes one token
        {"name": "append_one_token", "op": "append", "seqs": 1, "new": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "rot": 128, "layout": "half", "scaling": "none", "dtype": "bf16", "page": 16, "order": "tokens", "start": 900,
         "padding": 0},
        # a decode batch, padded to a fixed number of rows
        {"name": "append_batch", "op": "append", "seqs": 256, "new": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "rot": 128, "layout": "half", "scaling": "linear", "dtype": "bf16", "page": 64, "order": "tokens",
         "start": 32768, "padding": 13},
        # prompts of an odd length into pages that keep a head's tokens together
        {"name": "append_prompts", "op": "append", "seqs": 4, "new": 4093, "heads": 32, "kv_heads": 8, "dim": 128,
         "rot": 96, "layout": "interleaved", "scaling": "by_parts", "dtype": "f16", "page": 48, "order": "heads",
         "start": 7, "padding": 0},
        # attention: one user on a short prompt
        {"name": "attend_one_token", "op": "attend", "seqs": 1, "new": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "prefix": 512, "longest": 128, "page": 16, "order": "tokens", "dtype": "bf16"},
        # five drafted tokens a sequence, pages that end inside a tile, a head of 64
        {"name": "attend_drafts", "op": "attend", "seqs": 48, "new": 5, "heads": 32, "kv_heads": 4, "dim": 64,
         "prefix": 4093, "longest": 777, "page": 48, "order": "tokens", "dtype": "f16"},
        # a decode batch on a common system prompt
        {"name": "attend_batch", "op": "attend", "seqs": 64, "new": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "prefix": 8192, "longest": 512, "page": 64, "order": "tokens", "dtype": "bf16"},
        # no prefix at all: ordinary decoding of ragged sequences
        {"name": "attend_no_prefix", "op": "attend", "seqs": 128, "new": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "prefix": 0, "longest": 4096, "page": 16, "order": "heads", "dtype": "bf16"},
        # many users of one document, each with a dialogue of their own
        {"name": "attend_document", "op": "attend", "seqs": 256, "new": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "prefix": 32768, "longest": 1024, "page": 128, "order": "tokens", "dtype": "bf16"},
        # samples drawn in parallel from one long context
        {"name": "attend_long", "op": "attend", "seqs": 128, "new": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "prefix": 131072, "longest": 256, "page": 64, "order": "heads", "dtype": "bf16"},
    ]


HEADS = [(32, 8), (32, 32), (32, 4), (16, 2), (24, 8), (8, 1), (14, 2), (12, 12)]
MOST = {"rope": (6e8, 1e12), "append": (6e8, 1e12), "attend": (1.1e9, 2.7e11)}  # bytes, flops of a drawn case
MOST_SCORES = 1 << 29


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["rope", "append", "attend", "attend"])
        heads, kv_heads = rng.choice(HEADS)
        case = {"op": op, "heads": heads, "kv_heads": kv_heads}
        if op == "attend":
            new = rng.choice([1, 1, 1, 2, 3, 5, 8, 16])
            case.update(seqs=_log(rng, 1, 256), new=new, dim=rng.choice([64, 128, 128, 128, 256]),
                        prefix=0 if rng.random() < 0.15 else _log(rng, 16, 131072),
                        longest=max(new, _log(rng, 1, 4096)), page=rng.choice([16, 16, 32, 48, 64, 100, 128, 256]),
                        order=rng.choice(["tokens", "heads"]), dtype=rng.choice(["bf16", "bf16", "f16"]))
        else:
            dim = rng.choice([64, 128, 128, 128, 256])
            case.update(dim=dim, rot=rng.choice([dim, dim, dim // 2, dim // 4, dim - 32]),
                        layout=rng.choice(["half", "interleaved"]),
                        scaling=rng.choice(["none", "linear", "ntk", "by_parts"]),
                        dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), start=rng.randrange(0, 131072))
            if op == "rope":
                case.update(tokens=_log(rng, 1, 16384), dir=rng.choice(["fwd", "grad"]), fused=rng.choice([True, False]))
            else:
                new = _log(rng, 1, 8192)
                case.update(seqs=max(1, _log(rng, 1, 16384) // new), new=new, order=rng.choice(["tokens", "heads"]),
                            page=rng.choice([16, 16, 32, 48, 64, 100, 128, 256]), padding=rng.choice([0, 0, 1, 7]))
        w = work(case)
        if w["bytes"] <= MOST[op][0] and w["flops"] <= MOST[op][1]:
            if op != "attend" or case["seqs"] * case["new"] * heads * (case["prefix"] + case["longest"]) <= MOST_SCORES:
                return case


# ---------------------------------------------------------------- rotary frequencies
BASE, FACTOR, ORIGINAL = 10000.0, 8.0, 16384


def frequencies(rot, scaling):
    """Radians a position of each of the rot / 2 pairs, in 64 bits, and the factor of the rotated values."""
    i = np.arange(rot // 2, dtype=np.float64)
    base = BASE * FACTOR ** (rot / (rot - 2)) if scaling == "ntk" and rot > 2 else BASE
    theta = base ** (-2.0 * i / rot)
    if scaling == "linear":
        return theta / FACTOR, 1.0
    if scaling == "by_parts":
        turns = ORIGINAL * theta / (2 * np.pi)                       # of the pair over the original context
        keep = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)       # 1: as it is, 0: stretched by the factor
        return theta * keep + theta / FACTOR * (1.0 - keep), 0.1 * math.log(FACTOR) + 1.0
    return theta, 1.0


def _scaling(case):
    """The framework's own words for it."""
    return {"none": None, "linear": {"kind": "linear", "factor": FACTOR}, "ntk": {"kind": "ntk", "factor": FACTOR},
            "by_parts": {"kind": "by_parts", "factor": FACTOR, "original_len": ORIGINAL, "low": 1.0, "high": 32.0}}[
                case["scaling"]]


def _rotary_state(case, s):
    theta, s["factor"] = frequencies(case["rot"], case["scaling"])
    # turns a position in units of 2^-64, so that the phase of any position is exact in wrapping integers
    units = [round(float(t) / (2 * math.pi) * 2.0 ** 64) for t in theta]
    s["units"] = torch.tensor(units, dtype=torch.int64, device="cuda")
    if own:
        from paper_2607_11262_gb300 import serving
        s["rotary"] = serving.Rotary(case["dim"], rot_dim=case["rot"], base=BASE, layout=case["layout"],
                                     scaling=_scaling(case), device="cuda")


def _cos_sin(positions, units, factor):
    """cos and sin of each pair's angle, [tokens, 1, rot / 2] in 32 bits."""
    phase = positions.to(torch.int64)[:, None] * units             # modulo one turn
    angle = (phase >> 32).to(torch.float32) * (2 * math.pi / 2.0 ** 32)
    return (torch.cos(angle) * factor)[:, None], (torch.sin(angle) * factor)[:, None]


def _rotate(x, cos, sin, layout):
    n = cos.shape[-1]
    y = x.to(torch.float32)
    if layout == "half":
        a, b, rest = y[..., :n], y[..., n:2 * n], y[..., 2 * n:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1).to(x.dtype)
    a, b, rest = y[..., 0:2 * n:2], y[..., 1:2 * n:2], y[..., 2 * n:]
    turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, rest], -1).to(x.dtype)


def _rotate_exact(x, positions, case, back=False):
    theta, factor = frequencies(case["rot"], case["scaling"])
    pos = np.asarray(positions.cpu().numpy(), np.float64)
    z = np.exp((-1j if back else 1j) * (pos[:, None] * theta[None, :]))[:, None, :] * factor
    y = x.double().cpu().numpy().copy()
    r, n = case["rot"], case["rot"] // 2
    lo, hi = (slice(0, n), slice(n, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    w = (y[..., lo] + 1j * y[..., hi]) * z
    y[..., lo], y[..., hi] = w.real, w.imag
    return torch.from_numpy(y)


# ---------------------------------------------------------------- inputs
def _normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _projected(g, case, tokens, parts):
    """q, k (and v): views of one projection's rows, some channels much larger than the others, as keys have them."""
    h, kv, d, dt = case["heads"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]]
    counts = [h, kv, kv][:parts]
    if case.get("fused", True):
        rows = _normal(g, (tokens, sum(counts), d), dt)
        out = list(torch.split(rows, counts, dim=1))
    else:
        out = [_normal(g, (tokens, c, d), dt) for c in counts]
    out[1][..., ::17] *= 6.0
    return out


def _lengths(case):
    """Each sequence's own tokens, new ones included: spread evenly up to the longest, whatever the seed."""
    b, new, most = case["seqs"], case["new"], case["longest"]
    return [new + ((i + 1) * (most - new)) // b for i in range(b)]


def _cache(case, pages, dtype, g, scale_k=1.0):
    kv, d, page = case["kv_heads"], case["dim"], case["page"]
    got = []
    for scale in (scale_k, 1.0):
        if case["order"] == "tokens":
            got.append(_normal(g, (pages, page, kv, d), dtype, scale))
        else:
            got.append(_normal(g, (pages, kv, page, d), dtype, scale).transpose(1, 2))
    return got


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = {"case": case}
    if case["op"] == "rope":
        t = case["tokens"]
        _rotary_state(case, s)
        s["q"], s["k"] = _projected(g, case, t, 2)
        s["pos"] = torch.arange(case["start"], case["start"] + t, dtype=torch.int32, device="cuda")
        return s
    dt, page = DTYPES[case["dtype"]], case["page"]
    if case["op"] == "append":
        b, new = case["seqs"], case["new"]
        t = b * new + case["padding"]
        _rotary_state(case, s)
        s["q"], s["k"], s["v"] = _projected(g, case, t, 3)
        first = case["start"] + rng.integers(0, 4 * page, b)         # each sequence's length so far
        at = (first[:, None] + np.arange(new)).reshape(-1)
        per = (new + page - 1) // page + 1                           # pages a sequence's new tokens may touch
        table = rng.permutation(b * per + 3)[:b * per].reshape(b, per)
        seq = np.repeat(np.arange(b), new)
        which = at // page - np.repeat(first // page, new)
        slots = table[seq, which].astype(np.int64) * page + at % page
        pad = np.full(case["padding"], -1, np.int64)                 # rows of no sequence
        s["slots"] = torch.from_numpy(np.concatenate([slots, pad])).cuda()
        s["pos"] = torch.from_numpy(np.concatenate([at, 0 * pad]).astype(np.int32)).cuda()
        s["kc"], s["vc"] = _cache(case, b * per + 3, dt, g)
        if own:
            from paper_2607_11262_gb300 import serving
            s["cache"] = serving.PagedCache(s["kc"], s["vc"])
        return s
    b, new, h, d = case["seqs"], case["new"], case["heads"], case["dim"]
    lens = np.array(_lengths(case), np.int64)[rng.permutation(b)]
    n_prefix, per = -(-case["prefix"] // page), -(-case["longest"] // page)
    held = -(-lens // page)
    ids = rng.permutation(n_prefix + int(held.sum()) + 2).astype(np.int32)
    table = np.full((b, per), -1, np.int32)
    table[np.arange(per)[None, :] < held[:, None]] = ids[n_prefix:n_prefix + int(held.sum())]
    s["q"] = _normal(g, (b, new, h, d), dt)
    s["kc"], s["vc"] = _cache(case, len(ids), dt, g, 1.5)            # scores of a spread that makes some keys count
    s["prefix_pages"] = torch.from_numpy(ids[:n_prefix].copy()).cuda()
    s["table"] = torch.from_numpy(table).cuda()
    s["lens"] = torch.from_numpy(lens.astype(np.int32)).cuda()
    s["prefix"] = case["prefix"]
    s["scale"] = 1.0 / math.sqrt(d)
    if own:
        from paper_2607_11262_gb300 import serving
        s["cache"] = serving.PagedCache(s["kc"], s["vc"])
        s["workspace"] = serving.attention_workspace(s["cache"], s["q"], s["prefix"], s["table"])
    return s


# ---------------------------------------------------------------- one pass
def _rope_plain(s):
    case = s["case"]
    cos, sin = _cos_sin(s["pos"], s["units"], s["factor"])
    if case["dir"] == "grad":                                        # the transposed rotation
        sin = -sin
    return [_rotate(s["q"], cos, sin, case["layout"]), _rotate(s["k"], cos, sin, case["layout"])]


def _append_plain(s):
    case = s["case"]
    cos, sin = _cos_sin(s["pos"], s["units"], s["factor"])
    q, k = (_rotate(s[n], cos, sin, case["layout"]) for n in ("q", "k"))
    live = s["slots"].numel() - case["padding"]                      # padding rows come last
    page, at = s["slots"][:live] // case["page"], s["slots"][:live] % case["page"]
    s["kc"][page, at] = k[:live]
    s["vc"][page, at] = s["v"][:live]
    return [q, s["kc"], s["vc"]]


def _attend_plain(s):
    case = s["case"]
    b, new, h, d = s["q"].shape
    kv, page = case["kv_heads"], case["page"]
    q = s["q"].to(torch.float32).view(b, new, kv, h // kv, d) * s["scale"]
    n = s["prefix"]
    kp = s["kc"][s["prefix_pages"].long()].reshape(-1, kv, d)[:n].to(torch.float32)
    vp = s["vc"][s["prefix_pages"].long()].reshape(-1, kv, d)[:n].to(torch.float32)
    pages = s["table"].long().clamp(min=0)
    m = pages.shape[1] * page
    ks = s["kc"][pages].reshape(b, m, kv, d).to(torch.float32)
    vs = s["vc"][pages].reshape(b, m, kv, d).to(torch.float32)
    sp = torch.einsum("bnkgd,skd->bnkgs", q, kp)
    ss = torch.einsum("bnkgd,bskd->bnkgs", q, ks)
    i = torch.arange(new, device="cuda")
    sees = s["lens"].long()[:, None] - (new - 1 - i)[None, :]        # own keys that each query sees
    hidden = torch.arange(m, device="cuda")[None, None, :] >= sees[:, :, None]
    ss = ss.masked_fill(hidden[:, :, None, None, :], -math.inf)
    top = ss.amax(-1, keepdim=True)
    if n:
        top = torch.maximum(top, sp.amax(-1, keepdim=True))
    top = torch.where(top == -math.inf, 0.0, top)
    pp, ps = torch.exp(sp - top), torch.exp(ss - top)
    total = pp.sum(-1) + ps.sum(-1)
    out = torch.einsum("bnkgs,skd->bnkgd", pp, vp) + torch.einsum("bnkgs,bskd->bnkgd", ps, vs)
    out = torch.where(total[..., None] > 0, out / total[..., None], 0.0)
    lse = top[..., 0] + torch.log(total)
    return [out.view(b, new, h, d).to(s["q"].dtype), lse.view(b, new, h)]


def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return {"rope": _rope_plain, "append": _append_plain, "attend": _attend_plain}[op](s)
    from paper_2607_11262_gb300 import serving
    if op == "rope":
        call = serving.rope_grad if s["case"]["dir"] == "grad" else serving.rope
        return list(call(s["q"], s["k"], s["pos"], s["rotary"]))
    if op == "append":
        q = serving.append_kv(s["q"], s["k"], s["v"], s["pos"], s["slots"], s["rotary"], s["cache"])
        return [q, s["kc"], s["vc"]]
    return list(serving.prefix_attention(s["q"], s["cache"], s["prefix_pages"], s["prefix"], s["table"], s["lens"],
                                         scale=s["scale"], workspace=s["workspace"]))


def work(case):
    e, d, h, kv = SIZE[case["dtype"]], case["dim"], case["heads"], case["kv_heads"]
    if case["op"] == "rope":
        t = case["tokens"]
        return {"bytes": 2 * t * (h + kv) * d * e + 4 * t, "flops": 3 * t * (h + kv) * case["rot"]}
    if case["op"] == "append":
        t = case["seqs"] * case["new"] + case["padding"]
        return {"bytes": 2 * t * (h + 2 * kv) * d * e + 12 * t, "flops": 3 * t * (h + kv) * case["rot"]}
    b, new, lens = case["seqs"], case["new"], _lengths(case)
    keys = case["prefix"] + sum(lens)
    seen = sum(new * (case["prefix"] + n) - new * (new - 1) // 2 for n in lens)
    return {"bytes": 2 * keys * kv * d * e + 2 * b * new * h * d * e + 4 * b * new * h + 4 * b + 4 * (keys // case["page"]),
            "flops": 4 * seen * h * d}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return [_rotate_exact(s[n], s["pos"], case, case["dir"] == "grad") for n in ("q", "k")]
    if case["op"] == "append":
        q, k = (_rotate_exact(s[n], s["pos"], case) for n in ("q", "k"))
        kc, vc = s["kc"].double().cpu().numpy().copy(), s["vc"].double().cpu().numpy().copy()
        for t, slot in enumerate(s["slots"].tolist()):
            if slot >= 0:
                kc[slot // case["page"], slot % case["page"]] = k[t].numpy()
                vc[slot // case["page"], slot % case["page"]] = s["v"][t].double().cpu().numpy()
        return [q, torch.from_numpy(kc), torch.from_numpy(vc)]
    # one sequence and key head at a time, its keys in order, the visible ones alone
    b, new, h, d = s["q"].shape
    kv, n = case["kv_heads"], case["prefix"]
    q = s["q"].double()
    out = torch.zeros(b, new, h, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, new, h), -math.inf, dtype=torch.float64, device="cuda")

    def rows(cache, pages, count):
        return cache[pages.long()].flatten(0, 1)[:count].transpose(0, 1).double()   # [kv, count, d]

    kp, vp = rows(s["kc"], s["prefix_pages"], n), rows(s["vc"], s["prefix_pages"], n)
    lens = s["lens"].tolist()
    for i in range(b):
        pages = s["table"][i, :-(-lens[i] // case["page"])]
        ks, vs = rows(s["kc"], pages, lens[i]), rows(s["vc"], pages, lens[i])
        for j in range(new):
            own_keys = max(0, lens[i] - (new - 1 - j))
            if n + own_keys == 0:
                continue
            x = q[i, j].view(kv, h // kv, d) * s["scale"]
            x = torch.cat([x @ kp.transpose(1, 2), x @ ks[:, :own_keys].transpose(1, 2)], -1)
            lse[i, j] = torch.logsumexp(x, -1).view(h)
            p = torch.softmax(x, -1)
            out[i, j] = (p[..., :n] @ vp + p[..., n:] @ vs[:, :own_keys]).reshape(h, d)
    return [out, lse]
