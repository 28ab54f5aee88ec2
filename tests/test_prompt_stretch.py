"""Where a block of prompts' attention begins (find_stretch), and the division of the work that follows from it, the kernels' own code
compiled for the host from csrc/prompt.cu: a block's threads run as fibers that meet at each of its collectives.  For items of every
cost beside their tiles that the kernels have."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

from paper_2607_11262_gb300 import build as B
from tests.test_prompt_cut import SHIM, cases, items_of

FIBERS = r"""
#include <ucontext.h>
#include <vector>
constexpr int THREADS = 96, WARPS_OF_BLOCK = THREADS / 32;
static struct { int x; } threadIdx;
static ucontext_t main_context, context[THREADS];
static std::vector<char> stack[THREADS];
static int64_t left[2][THREADS];
static int meetings[THREADS], ended;
static bool apart;
static void (*body)();
// Leaves x for the others, who all come to the same call, and returns what every thread has left.
static const int64_t *meet(int64_t x) {
  const int me = threadIdx.x, phase = meetings[me]++ & 1;
  left[phase][me] = x;
  swapcontext(&context[me], &main_context);
  return left[phase];
}
static void run() { body(); ended++; swapcontext(&context[threadIdx.x], &main_context); }
static void block(void (*f)()) {
  body = f, ended = 0;
  for (int t = 0; t < THREADS; t++) {
    stack[t].resize(1 << 16), meetings[t] = 0;
    getcontext(&context[t]);
    context[t].uc_stack.ss_sp = stack[t].data(), context[t].uc_stack.ss_size = stack[t].size(), context[t].uc_link = nullptr;
    makecontext(&context[t], run, 0);
  }
  while (ended == 0) {
    for (int t = 0; t < THREADS; t++) threadIdx.x = t, swapcontext(&main_context, &context[t]);
    if (ended && ended != THREADS) apart = true;               // some have left while others meet
  }
}
static void __syncthreads() { meet(0); }
static int64_t __shfl_up_sync(unsigned, int64_t x, int n) {
  const int me = threadIdx.x;
  const int64_t *const all = meet(x);
  return all[me % 32 >= n ? me - n : me];
}
static int reduced(int x, bool most) {
  const int me = threadIdx.x;
  const int64_t *const all = meet(x);
  int64_t y = all[me / 32 * 32];
  for (int i = 0; i < 32; i++) y = most ? max(y, all[me / 32 * 32 + i]) : min(y, all[me / 32 * 32 + i]);
  return (int)y;
}
static int __reduce_min_sync(unsigned, int x) { return reduced(x, false); }
static int __reduce_max_sync(unsigned, int x) { return reduced(x, true); }
"""
ENTRY = r"""
static Args call;
static int of_items, beside_of, blocks_of, by_keys_of;
static int64_t scratch[SCRATCH / 8];
static Stretch found_by[THREADS];
static void find() {
  found_by[threadIdx.x] = by_keys_of ? find_stretch<true, THREADS>(call, {of_items, call.causal, beside_of}, blocks_of, scratch)
                                     : find_stretch<false, THREADS>(call, {of_items, call.causal, beside_of}, blocks_of, scratch);
}
template <bool K> static int64_t go(int *out, int64_t room, int *ends, int *rest) {
  const Items<K> items = {of_items, call.causal, beside_of};
  int64_t n = 0;
  for (int c = 0; c < blocks_of; c++) {
    blockIdx.x = c, ends[4 * c] = -1;
    block(find);
    for (int t = 1; t < THREADS; t++)
      if (found_by[t].x0 != found_by[0].x0 || found_by[t].x1 != found_by[0].x1 ||
          (found_by[t].x0 < found_by[t].x1 && (found_by[t].b != found_by[0].b || found_by[t].t != found_by[0].t || found_by[t].pos != found_by[0].pos))) return -1;
    if (apart) return -2;
    Stretch s = found_by[0];
    rest[0] = s.rest_from, rest[1] = s.rest_to;
    if (s.x0 >= s.x1) continue;
    Seq x;
    Item i;
    i.b = -1;
    while (next_item(call, items, s, x, i, (int4 *)(ends + 4 * c))) {
      if (n < room) { const int row[] = {c, i.b, i.kh, i.t, i.tile0, i.tile1, i.tiles, i.n}; std::copy(row, row + 8, out + 8 * n); }
      n++;
    }
  }
  return n;
}
extern "C" int64_t cut(int by_keys, const int32_t *starts, const int32_t *lens, int n_seqs, int n_tokens, int kv_heads, int most, int causal, int q,
                       int beside, int blocks, int *out, int64_t room, int *ends, int *rest) {
  call = {starts, lens, n_seqs, n_tokens, kv_heads, lens != nullptr, most, 1, causal, nullptr};
  of_items = q, beside_of = beside, blocks_of = blocks, by_keys_of = by_keys, apart = false;
  return by_keys ? go<true>(out, room, ends, rest) : go<false>(out, room, ends, rest);
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
        r"^struct Stretch \{.*?\n", r"^constexpr int SCRATCH = .*?\n", r"^template <bool BY_KEYS, int THREADS>\n__device__ __forceinline__ Stretch find_stretch\(.*?^}\n",
        r"^struct Item \{.*?\n", r"^template <bool BY_KEYS>\n__device__ __forceinline__ bool next_item\(.*?^}\n")]
    path = str(tmp_path_factory.mktemp("stretch"))
    src, lib = os.path.join(path, "stretch.cpp"), os.path.join(path, "stretch.so")
    with open(src, "w") as f:
        f.write(SHIM + FIBERS + "".join(parts) + ENTRY)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wno-unknown-pragmas", "-o", lib, src])
    f = ctypes.CDLL(lib).cut
    f.restype = ctypes.c_int64

    def run(by_keys, starts, lens, kv_heads, causal, q, blocks, beside, n_tokens=None):
        s = np.array(starts, np.int32)
        k = None if lens is None else np.array(lens, np.int32)
        room = 4 * blocks + kv_heads * sum(int(n) // min(q, 128) + 2 for n in np.clip(np.diff(s.astype(np.int64)), 0, s.max(initial=0)))
        out, ends, rest = np.zeros((room, 8), np.int32), np.zeros((blocks, 4), np.int32), np.zeros(2, np.int32)
        p = [x.ctypes.data_as(ctypes.c_void_p) if x is not None else None for x in (s, k, out, ends, rest)]
        n = f(int(by_keys), p[0], p[1], len(s) - 1, int(s[-1]) if n_tokens is None else n_tokens, kv_heads, 1 << 28, int(causal), q, beside, blocks, p[2],
              ctypes.c_int64(room), p[3], p[4])
        assert 0 <= n <= room, n
        return out[:n], ends, tuple(rest.tolist())
    return run


@pytest.mark.parametrize("beside", [2, 3])
def test_every_tile_is_one_blocks(cut, beside):
    """As in tests/test_prompt_cut.py, from what the block's threads find together; items by rows at both costs."""
    for n, (by_keys, starts, lens, kv_heads, causal, q, blocks) in enumerate(cases()):
        if (by_keys and beside != 2) or n % 3:
            continue
        case = by_keys, starts, lens, kv_heads, causal, q, blocks
        want = items_of(*case[:6])
        got, ends, rest = cut(*case, beside, n_tokens=starts[-1] + 7)
        at = {}
        for block, b, h, t, tile0, tile1, tiles, _ in got.tolist():
            assert want[b, h, t] == tiles and 0 <= tile0 < tile1 <= tiles, case
            parts = at.setdefault((b, h, t), [])
            assert tile0 == (parts[-1][2] if parts else 0) and (not parts or block == parts[-1][0] + 1), case
            parts.append((block, tile0, tile1))
        assert {k: v[-1][2] for k, v in at.items()} == want, case
        told = {c: tuple(e) for c, e in enumerate(ends.tolist()) if e[0] >= 0}
        assert told == {v[0][0]: (*k, len(v) - 1) for k, v in at.items() if len(v) > 1}, case
        later = got[got[:, 4] > 0, 0]
        assert len(set(later.tolist())) == len(later), case
        # A block's stretch is its share of the weights, or what an item costs beside its tiles where that is more.  Its first and last item add a
        # tile each by rounding; the others have no more tiles than their weight.
        load = np.bincount(got[:, 0], got[:, 5] - got[:, 4], minlength=blocks)
        assert load.max(initial=0) <= (sum(want.values()) + beside * len(want)) / blocks + beside + 2, case
        # rows of no sequence: those before the first row of one and after the last
        rows = [(x, y) for x, y in zip(starts[:-1], starts[1:]) if y > x]
        assert rest == ((rows[0][0], rows[-1][1]) if rows else (0, 0)), case


def test_more_sequences_than_threads(cut):
    lens = [(7 * i) % 5 for i in range(500)]
    starts = np.concatenate([[2], 2 + np.cumsum(lens)]).tolist()
    for by_keys in (False, True):
        got, _, rest = cut(by_keys, starts, None, 2, True, 128, 152, 2, n_tokens=starts[-1] + 3)
        assert sorted(map(tuple, got[:, [2, 1]].tolist())) == [(h, b) for h in range(2) for b in range(500) if lens[b]]
        first, last = min(b for b in range(500) if lens[b]), max(b for b in range(500) if lens[b])
        assert rest == (starts[first], starts[last + 1])
