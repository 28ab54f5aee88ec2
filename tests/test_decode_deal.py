"""The decode step's graph divides the machine as the kernels do: decode.prefix_blocks against the device's own function, compiled
for the host from csrc/attention.cu."""
import ctypes
import itertools
import os
import random
import re
import shutil
import subprocess

import pytest

from paper_2607_11262_gb300 import build as B
from paper_2607_11262_gb300 import decode

SHIM = """
#include <algorithm>
#include <cmath>
#include <cstdint>
using std::max;
using std::min;
#define __device__
#define __host__
#define __forceinline__ inline
constexpr int SMS = 152;
struct Args { int prefix_len, kv_heads; };
struct Line { int keys, prefix_tiles; };
inline int tiles_of(int keys, int tile) { return (keys + tile - 1) / tile; }
inline int64_t quotient(int64_t x, int64_t y) { return x / y; }
"""
ENTRY = """
extern "C" int deal(int prefix_len, int kv_heads, int row_tiles, int own_rows, int64_t own_tiles, int64_t own_pairs) {
  return prefix_sms<128>(Args{prefix_len, kv_heads}, Line{128, row_tiles}, own_rows, own_tiles, own_pairs);
}
"""


@pytest.fixture(scope="module")
def device(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    with open(os.path.join(B.CSRC, "attention.cu")) as f:
        text = f.read()
    assert "constexpr int SMS = 152;" in text
    body = re.search(r"^template <int D>\n__device__ __forceinline__ int prefix_sms\(.*?^}\n", text, re.M | re.S).group(0)
    path = str(tmp_path_factory.mktemp("deal"))
    src, lib = os.path.join(path, "deal.cpp"), os.path.join(path, "deal.so")
    with open(src, "w") as f:
        f.write(SHIM + body + ENTRY)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-ffp-contract=off", "-shared", "-fPIC", "-Wno-unknown-pragmas", "-o", lib, src])
    got = ctypes.CDLL(lib).deal
    got.argtypes = [ctypes.c_int] * 4 + [ctypes.c_int64] * 2
    return got


def test_the_deal_is_the_kernels(device):
    rng = random.Random(5)
    cases = [(prefix, kv, tiles, rows, own, pairs) for prefix, kv, tiles, rows, own, pairs in itertools.product(
        (256, 8192, 32768, 131072), (1, 8), (1, 4, 160), (16, 32, 64), (0, 1, 2000), (1, 512))]
    for _ in range(3000):
        pairs = int(2 ** rng.uniform(0, 12))
        cases.append((int(2 ** rng.uniform(8, 18)), rng.choice([1, 2, 4, 8, 12, 32]), int(2 ** rng.uniform(0, 7)), rng.choice([16, 32, 64]),
                      int(pairs * 2 ** rng.uniform(0, 7)), pairs))
    for prefix, kv, tiles, rows, own, pairs in cases:
        want = device(prefix, kv, tiles, rows, own, pairs)
        assert decode.prefix_blocks(-(-prefix // 128), kv, tiles, rows, own, pairs) == want, (prefix, kv, tiles, rows, own, pairs)


@pytest.mark.parametrize("case", decode.CASES)
def test_the_graph_follows_it(case, device):
    """The study's steps: 32 heads over 8 key heads, own keys by fours (16 keys of four heads to a tile)."""
    row_tiles = -(-case["seqs"] * 4 // 256)
    want = device(case["prefix"], 8, row_tiles, 16, case["seqs"] * 2 * (case["own"] // 16), case["seqs"] * 2)
    counts, streams, rest = decode.deal(**case)
    units = case["prefix"] // 128 * 8 * row_tiles
    assert len(counts) <= want and streams == decode.SMS - want and sum(counts) == units and max(counts) == -(-units // want)
    g = decode.graph(**case)
    assert g.n_ctas == len(counts) + streams
    assert rest == -(-case["seqs"] * 2 * (case["own"] // 16) // (2 * streams))
