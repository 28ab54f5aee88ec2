"""A decode step of one attention layer, run on the GPU and simulated.

``Step`` is the step as a serving program runs it: a batch of sequences that share a prompt, whose keys and values are
appended to a paged cache with the rotation on the way, and attention of the new tokens over the shared prompt and each
sequence's own tokens.  ``Step.check`` compares it with the same attention worked out without a cache, from rotated queries and
keys as a training program has them.

``graph`` is the step's attention as a tile graph: the blocks, tiles and rings of the kernels that run, so that the
simulated cycles of a GB300-like row (``gb300_params``) can be set beside the measured time, as Section 6.2 does for
Flash-Decoding.  Input plumbing only: graphs and parameter rows, no scheduling arithmetic.
"""
from __future__ import annotations

import numpy as np

from . import workloads as W

SMS = 152
GHZ = 1.92                       # SM clock that measured times are compared at
ROWS, PREFIX_KEYS = 256, 128     # query rows of a block and keys of its tiles, on the prefix
OWN_TILE_KEYS = 64               # keys of a tile of a sequence's own (of one head, or 16 of each of four)
PAGE = 64                        # tokens of a page in Step

CASES = (dict(seqs=64, prefix=8192, own=256), dict(seqs=128, prefix=32768, own=128), dict(seqs=256, prefix=32768, own=512))


def gb300_params():
    """One row for a GB300: 152 SMs, 6.78 TB/s of memory (measured copy rate), 4096 FMA a cycle and SM, at 1.92 GHz; the
    latencies are the framework's defaults."""
    p = W.default_params()
    p[W.P_NUM_SMS] = SMS
    p[W.P_HBM_BPC] = int(6780 / GHZ)
    p[W.P_DRAM_LAT] = 900
    p[W.P_TMA_BPC] = 100
    p[W.P_MMA_FMA_PC] = 4096
    return p


def own_cta(tiles, stages=3, tile_bytes=32768, fma=2 * 16 * 64 * 128, softmax_ops=16 * 64 * 8):
    """An SM's two streaming blocks: per block (consumers 1 and 2) ``tiles`` tiles of keys and values through a ring."""
    t = W.CtaTemplate(3)
    ring = ([], [])
    for j in range(tiles):
        for i, c in enumerate((1, 2)):
            free = t.node(W.BAR, 0)
            if j >= stages:
                t.edge(ring[i][j - stages], free)
            load = t.node(W.LOAD, 0, tile_bytes)
            t.edge(free, load)
            full = t.node(W.BAR, c)
            t.edge(load, full)
            soft = t.node(W.EW, c, softmax_ops)
            t.edge(full, soft)
            pv = t.node(W.MMA, c, fma)
            t.edge(soft, pv)
            ring[i].append(pv)
    for i, c in enumerate((1, 2)):
        st = t.node(W.STORE, c, 16 * 128 * 4)
        t.edge(ring[i][-1], st)
    return t


def prefix_blocks(prefix_tiles, kv_heads, row_tiles, own_rows, own_tiles, own_pairs):
    """SMs that the prefix gets at a head of 128, as the kernels work it out from the lengths (``prefix_sms`` in
    csrc/attention.cu, which has the reasons and where the costs come from): in units of an own tile's time on an SM."""
    if own_tiles == 0:
        return SMS
    f = np.float32                                     # in 32 bits, like the kernels
    tile, pair = f(2.2), f(8)
    p = (tile * f(prefix_tiles) + pair) * f(kv_heads) * f(row_tiles)
    o = (f(own_tiles) + f(3) * f(own_pairs)) * f({16: 0.8, 32: 1.1}.get(own_rows, 2.1))
    memory = f(own_tiles) / f(104)
    even = max(1, min(SMS - 1, int(p / max((p + o) / f(SMS), memory) + f(0.5))))
    side = row_tiles if even >= row_tiles else 1       # row tiles that pass along the keys side by side
    units = prefix_tiles * kv_heads * (row_tiles if side == 1 else 1)
    per = -(-units // (even // side))
    best, least = even, f(np.inf)
    for x in range(max(1, per - 1), per + 2):          # whole numbers of tiles to a block
        sms = -(-units // x) * side
        if sms < SMS:
            time = max((tile + pair / f(prefix_tiles)) * f(x), o / f(SMS - sms), memory)
            if time < least:
                best, least = sms, time
    return best


def deal(seqs, prefix, own, heads=32, kv_heads=8):
    """(tiles of each prefix block, SMs that stream own keys, own tiles of each of their two blocks) of a step at a head of 128."""
    group = heads // kv_heads
    row_tiles, tiles = -(-seqs * group // ROWS), -(-prefix // PREFIX_KEYS)
    rows = 16 if group <= 16 else 32 if group <= 32 else 64
    # by fours: a unit is 16 keys of four heads, else 64 of one
    at_once = 4 if rows == 16 and kv_heads % 4 == 0 and -(-own // PAGE) * PAGE <= 2048 else 1
    pairs = kv_heads // at_once * -(-group // rows)    # of a sequence
    own_tiles = seqs * -(-own // (OWN_TILE_KEYS // at_once)) * pairs
    blocks = prefix_blocks(tiles, kv_heads, row_tiles, rows, own_tiles, seqs * pairs)
    side = row_tiles if blocks >= row_tiles else 1
    units = tiles * kv_heads * (row_tiles if side == 1 else 1)
    per = -(-units // (blocks // side))
    counts = [min(per, units - at) for at in range(0, units, per) for _ in range(side)]
    streams = max(1, SMS - blocks)
    return counts, streams, -(-own_tiles // (2 * streams))


def graph(seqs, prefix, own, heads=32, kv_heads=8):
    """The step's attention: blocks on the prefix (256 rows, tiles of 128 keys, two halves in turn) beside SMs that stream the
    sequences' own keys, dealt out as the kernels do it (``deal``)."""
    counts, streams, rest = deal(seqs, prefix, own, heads, kv_heads)
    tpls, kind = [], {}

    def template(key, make):
        if key not in kind:
            kind[key] = len(tpls)
            tpls.append(make())
        return kind[key]
    fma = 128 * 128 * 128
    ct = [template(("prefix", n), lambda n=n: W.fa_fwd_cta(n, q_bytes=ROWS * 256, kv_bytes=32768, qk_fma=fma, softmax_ops=128 * 128 * 4,
                                                           pv_fma=fma, norm_ops=0, o_bytes=128 * 128 * 4)) for n in counts]
    ct += [template(("own", rest), lambda: own_cta(rest))] * streams
    return W.template_set("decode_step", 3, tpls, np.array(ct), np.zeros(len(ct), np.uint32))


class Step:
    """One decode step of ``seqs`` sequences with ``own`` tokens of their own (the newest included) after a shared prompt of
    ``prefix`` tokens."""

    def __init__(self, seqs, prefix, own, heads=32, kv_heads=8, head_dim=128, page=PAGE, dtype=None, seed=0, device="cuda"):
        import torch

        from . import serving as S
        self.S, self.torch = S, torch
        g = torch.Generator(device=device).manual_seed(seed)
        dtype = dtype or torch.bfloat16
        self.seqs, self.prefix, self.own = seqs, prefix, own
        self.shape = heads, kv_heads, head_dim
        held, shared = -(-own // page), -(-prefix // page)
        ids = torch.randperm(shared + seqs * held, generator=g, device=device).to(torch.int32)
        self.pages, self.table = ids[:shared].contiguous(), ids[shared:].view(seqs, held).contiguous()
        self.cache = S.PagedCache.empty(ids.numel(), page, kv_heads, head_dim, dtype, device=device)
        self.rotary = S.Rotary(head_dim, device=device)
        self.lens = torch.full((seqs,), own, dtype=torch.int32, device=device)

        def rows(n):
            x = torch.randn((n, heads + 2 * kv_heads, head_dim), generator=g, device=device).to(dtype)
            return x.split([heads, kv_heads, kv_heads], 1)

        def places(pages, first, count):
            at = torch.arange(first, first + count, device=device)
            return pages.long()[..., at // page] * page + at % page
        # the prompt once, each sequence's earlier tokens, and the step's own inputs
        self.before = rows(prefix), rows(seqs * (own - 1))
        pos = torch.arange(prefix, dtype=torch.int32, device=device)
        S.append_kv(*self.before[0], pos, places(self.pages, 0, prefix), self.rotary, self.cache)
        pos = (prefix + torch.arange(own - 1, dtype=torch.int32, device=device)).repeat(seqs)
        S.append_kv(*self.before[1], pos, places(self.table, 0, own - 1).reshape(-1).contiguous(), self.rotary, self.cache)
        self.q, self.k, self.v = rows(seqs)
        self.pos = torch.full((seqs,), prefix + own - 1, dtype=torch.int32, device=device)
        self.slots = places(self.table, own - 1, 1).reshape(-1).contiguous()
        self.workspace = S.attention_workspace(self.cache, self.q[:, None], prefix, self.table)

    def append(self):
        return self.S.append_kv(self.q, self.k, self.v, self.pos, self.slots, self.rotary, self.cache)

    def attend(self, q):
        return self.S.prefix_attention(q[:, None], self.cache, self.pages, self.prefix, self.table, self.lens,
                                       workspace=self.workspace)

    def run(self):
        """The step: (out [seqs, 1, heads, head_dim], lse)."""
        return self.attend(self.append())

    def check(self):
        """Largest difference of the step's results to attention without a cache, relative to their root mean square."""
        torch, S = self.torch, self.S
        heads, kv_heads, dim = self.shape
        out = self.run()[0]
        worst = 0.0
        dev = self.q.device
        pos = torch.arange(self.prefix + self.own, dtype=torch.int32, device=dev)
        for b in range(0, self.seqs, max(1, self.seqs // 4)):
            mine = slice(b * (self.own - 1), (b + 1) * (self.own - 1))
            k, v = (torch.cat([self.before[0][i], self.before[1][i][mine], x[b:b + 1]]) for i, x in ((1, self.k), (2, self.v)))
            q = self.q[b:b + 1].expand(len(pos), -1, -1)
            q, k = S.rope(q, k, pos, self.rotary)                  # as in training: queries and keys of all positions
            q = q[-1].float().view(kv_heads, heads // kv_heads, dim)
            p = torch.softmax(torch.einsum("hgd,shd->hgs", q, k.float()) * dim ** -0.5, -1)
            want = torch.einsum("hgs,shd->hgd", p, v.float()).reshape(heads, dim)
            worst = max(worst, float((out[b, 0].float() - want).abs().max() / want.square().mean().sqrt()))
        return worst

    def time_us(self, call, reps=20):
        torch = self.torch
        for _ in range(3):
            call()
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(reps):
            call()
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b) / reps * 1e3
