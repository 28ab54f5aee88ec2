"""attention.cu with waits that run out: a copy whose waits give up after a number of tries that a test sets, instead of after
two seconds.  What a block does from there on (the ends of its copies and products, its status) is the source's own."""
import ctypes
import os
import subprocess

from paper_2607_11262_gb300 import build as B
from paper_2607_11262_gb300 import serving

EDITS = (
    ("constexpr uint64_t LIMIT_NS = 2000000000ull, DRAIN_NS", "constexpr uint64_t LIMIT_NS = 0, DRAIN_NS"),
    ("constexpr int TRIES = 1024, BETWEEN = 64;", "__constant__ int TRIES;\nconstexpr int BETWEEN = 1;"),
    ("mbarrier.try_wait.parity", "mbarrier.test_wait.parity"),   # at once, where try_wait may stand for a while
    # fewer instances to compile: bfloat16, heads of 128 and 256
    ("head_dim == 64    ? run<T, 64>(a, p, maps, own_maps, s)\n         : ", ""),
    (": launch<__half>(a,", ": launch<__nv_bfloat16>(a,"),
)
APPENDED = """
namespace gts {
gts_status fail(gts_status s, const char *) { return s; }
gts_status cuda_fail(cudaError_t, const char *) { return GTS_ERR_CUDA; }
void clear_error() {}
}  // namespace gts
extern "C" int set_tries(int n) { return (int)cudaMemcpyToSymbol(TRIES, &n, sizeof(n)); }
"""


def build(path):
    """The copy as a library with serving.py's entries for attention, and set_tries."""
    with open(os.path.join(B.CSRC, "attention.cu")) as f:
        text = f.read()
    for old, new in EDITS:
        assert text.count(old) == 1, old
        text = text.replace(old, new)
    src, lib = os.path.join(path, "short_waits.cu"), os.path.join(path, "short_waits.so")
    with open(src, "w") as f:
        f.write(text + APPENDED)
    subprocess.check_call([B.nvcc()] + B.NVCC_FLAGS + ["-shared", "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC, "-o", lib, src])
    got = ctypes.CDLL(lib)
    for name in ("gts_prefix_attention", "gts_attention_workspace_bytes"):
        whole = getattr(serving._load(), name)
        getattr(got, name).argtypes, getattr(got, name).restype = whole.argtypes, whole.restype
    got.set_tries.argtypes, got.set_tries.restype = [ctypes.c_int], ctypes.c_int
    return got
