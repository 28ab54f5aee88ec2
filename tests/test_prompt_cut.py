"""How the attention of prompts divides its work among the blocks, the kernels' own code compiled for the host from csrc/prompt.cu:
every tile of every item is some block's, exactly once, and what the joining kernel is told of the items that are cut is so."""
import ctypes
import os
import random
import re
import shutil
import subprocess

import numpy as np
import pytest

from paper_2607_11262_gb300 import build as B

SHIM = r"""
#include <algorithm>
#include <cstdint>
using std::min;
using std::max;
#define __device__
#define __forceinline__ inline
struct int4 { int x, y, z, w; };
static int4 make_int4(int x, int y, int z, int w) { return {x, y, z, w}; }
static int64_t quotient(int64_t x, int64_t y) { return x / y; }
static struct { int x; } blockIdx;
struct Args { const int32_t *starts, *lens; int n_seqs, n_tokens, kv_heads, paged, max_pages, page_size, causal; int32_t *status; };
#define GTS_ERR_INVALID_PARAMS (-3)
"""
ENTRY = r"""
template <bool K> static int64_t go(const Args &a, int q, int blocks, int *out, int64_t room, int *ends) {
  const Items<K> items = {q, a.causal};
  Stretch whole = {};
  for (int b = 0; b < a.n_seqs; b++) { const Seq s = sequence(a, b); whole.head += items.before(s, items.count(s)); }
  whole.all = whole.head * a.kv_heads;
  whole.per = max((int64_t)items.lead(), (whole.all + blocks - 1) / blocks);
  int64_t n = 0;
  for (int c = 0; c < blocks; c++) {
    blockIdx.x = c;
    ends[4 * c] = -1;
    Stretch s = whole;
    s.x0 = min(s.all, s.per * c), s.x1 = min(s.all, s.x0 + s.per);
    if (s.x0 >= s.x1) continue;
    s.kh = (int)(s.x0 / s.head);
    int64_t at = s.kh * s.head;
    for (int b = 0; b < a.n_seqs; b++) {
      const Seq x = sequence(a, b);
      const int64_t w = items.before(x, items.count(x));
      if (s.x0 < at + w) {
        int lo = 0, hi = items.count(x) - 1;
        while (lo < hi) {
          const int mid = (lo + hi + 1) / 2;
          if (at + items.before(x, mid) <= s.x0) lo = mid; else hi = mid - 1;
        }
        s.b = b, s.t = lo, s.pos = at + items.before(x, lo);
        break;
      }
      at += w;
    }
    Seq x;
    Item i;
    i.b = -1;
    while (next_item(a, items, s, x, i, (int4 *)(ends + 4 * c))) {
      if (n < room) { const int row[] = {c, i.b, i.kh, i.t, i.tile0, i.tile1, i.tiles, i.n}; std::copy(row, row + 8, out + 8 * n); }
      n++;
    }
  }
  return n;
}
extern "C" int64_t cut(int by_keys, const int32_t *starts, const int32_t *lens, int n_seqs, int n_tokens, int kv_heads, int paged, int most,
                       int causal, int q, int blocks, int *out, int64_t room, int *ends) {
  const Args a = {starts, lens, n_seqs, n_tokens, kv_heads, paged, most, 1, causal, nullptr};
  return by_keys ? go<true>(a, q, blocks, out, room, ends) : go<false>(a, q, blocks, out, room, ends);
}
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    with open(os.path.join(B.CSRC, "prompt.cu")) as f:
        text = f.read()
    parts = [re.search(p, text, re.M | re.S).group(0) for p in (
        r"^constexpr int SMS = .*?;\n", r"^struct Seq \{.*?\n", r"^__device__ __forceinline__ Seq sequence\(.*?^}\n", r"^template <bool BY_KEYS> struct Items \{.*?^};\n",
        r"^struct Stretch \{.*?\n", r"^struct Item \{.*?\n", r"^template <bool BY_KEYS>\n__device__ __forceinline__ bool next_item\(.*?^}\n")]
    path = str(tmp_path_factory.mktemp("cut"))
    src, lib = os.path.join(path, "cut.cpp"), os.path.join(path, "cut.so")
    with open(src, "w") as f:
        f.write(SHIM + "".join(parts) + ENTRY)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wno-unknown-pragmas", "-o", lib, src])
    f = ctypes.CDLL(lib).cut
    f.restype = ctypes.c_int64

    def run(by_keys, starts, lens, kv_heads, causal, q, blocks=152, n_tokens=None):
        s = np.array(starts, np.int32)
        k = None if lens is None else np.array(lens, np.int32)
        room = 4 * blocks + kv_heads * sum(int(n) // min(q, 128) + 2 for n in np.clip(np.diff(s.astype(np.int64)), 0, s.max()))
        out, ends = np.zeros((room, 8), np.int32), np.zeros((blocks, 4), np.int32)
        p = [x.ctypes.data_as(ctypes.c_void_p) if x is not None else None for x in (s, k, out, ends)]
        n = f(int(by_keys), p[0], p[1], len(s) - 1, int(s[-1]) if n_tokens is None else n_tokens, kv_heads, int(lens is not None), 1 << 28, int(causal), q, blocks, p[2],
              ctypes.c_int64(room), p[3])
        assert n <= room
        return out[:n], ends
    return run


def items_of(by_keys, starts, lens, kv_heads, causal, q):
    """{(sequence, key head, item): its tiles}, from the definition."""
    got = {}
    for b, (x, y) in enumerate(zip(starts[:-1], starts[1:])):
        n = max(0, y - x)
        keys = n if lens is None else max(0, lens[b])
        for h in range(kv_heads):
            if by_keys:                                    # 128 keys; tiles of q queries, from that of the first that sees the first key
                for t in range(-(-keys // 128)):
                    got[b, h, t] = -(-n // q) - (t * 128 // q if causal else 0)
            else:                                          # q queries; tiles of 128 keys up to the last that the last query sees
                for t in range(-(-n // q)):
                    seen = max(0, keys - n + min(n, (t + 1) * q)) if causal else keys
                    got[b, h, t] = max(1, -(-seen // 128))
    return got


def cases():
    rng = random.Random(1)
    for _ in range(250):
        by_keys = rng.random() < 0.4
        n = rng.choice([1, 1, 2, 7, 40])
        group = rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16, 100, 128])
        most = int(2 ** rng.uniform(0, 13 if n * group < 30 else 9)) + 1
        new = [rng.randrange(0, most) for _ in range(n)]
        starts = [rng.randrange(0, 4)]
        for x in new:
            starts.append(starts[-1] + x)
        lens = None if by_keys or rng.random() < 0.5 else [rng.choice([x, x + rng.randrange(0, 20000), rng.randrange(-2, x + 1)]) for x in new]
        q = (128 // group) * (1 if by_keys else rng.choice([1, 2]))
        yield by_keys, starts, lens, rng.choice([1, 2, 8]), lens is not None or rng.random() < 0.7, q, rng.choice([152, 152, 7, 1])


def test_every_tile_is_one_blocks(cut):
    for case in cases():
        want = items_of(*case[:6])
        got, ends = cut(*case[:6], blocks=case[6])
        at = {}
        for block, b, h, t, tile0, tile1, tiles, _ in got.tolist():
            assert want[b, h, t] == tiles and 0 <= tile0 < tile1 <= tiles, case
            parts = at.setdefault((b, h, t), [])
            assert tile0 == (parts[-1][2] if parts else 0) and (not parts or block == parts[-1][0] + 1), case   # the next block goes on
            parts.append((block, tile0, tile1))
        assert {k: v[-1][2] for k, v in at.items()} == want, case
        # records: the item that begins in a block and goes on, and how many blocks more it takes
        told = {c: tuple(e) for c, e in enumerate(ends.tolist()) if e[0] >= 0}
        assert told == {v[0][0]: (*k, len(v) - 1) for k, v in at.items() if len(v) > 1}, case
        later = got[got[:, 4] > 0, 0]                      # items that began in an earlier block: one at most
        assert len(set(later.tolist())) == len(later), case
        # work is shared evenly: no block has more than its share, its items' begins and two tiles more
        load = np.bincount(got[:, 0], got[:, 5] - got[:, 4], minlength=case[6])
        total = sum(want.values()) + 2 * len(want)
        assert load.max(initial=0) <= total / case[6] + 4, case


def test_starts_at_the_ends_of_their_type(cut):
    """What lies between starts that are far out of range has no rows beyond the call's."""
    low, high = -2**31, 2**31 - 1
    for by_keys in (False, True):
        for starts, want in (([0, 30, low, 40], {0: 30, 2: 40}), ([low, 30, 80], {0: 30, 1: 50}), ([0, high, low, high], {0: 80, 2: 80}),
                             ([high, low, 80], {1: 80}), ([30, low, low], {})):
            got, _ = cut(by_keys, starts, None, 2, True, 64, n_tokens=80)
            assert {int(b): int(n) for b, n in got[:, [1, 7]]} == want, starts
