"""prompt.cu with waits that run out: a copy whose waits give up after a number of tries that a test sets, instead of after two
seconds.  What a block does from there on is the source's own."""
import ctypes
import os
import subprocess

from paper_2607_11262_gb300 import build as B
from paper_2607_11262_gb300 import serving

EDITS = (
    ("constexpr uint64_t LIMIT_NS = 2000000000ull, DRAIN_NS", "constexpr uint64_t LIMIT_NS = 0, DRAIN_NS"),
    ("constexpr int TRIES = 1024, BETWEEN = 64;", "__constant__ int TRIES;\nconstexpr int BETWEEN = 1;"),
    ("mbarrier.try_wait.parity", "mbarrier.test_wait.parity"),   # at once, where try_wait may stand for a while
    # fewer instances to compile: bfloat16
    ("return dim == 64 ? forward<__half, 64>(a, maps, most, w, s) : forward<__half, 128>(a, maps, most, w, s);", "return cudaErrorInvalidValue;"),
    (": run_grad<__half>(a, p, maps, *d, (cudaStream_t)stream)", ": cudaErrorInvalidValue"),
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
    """The copy as a library with serving.py's entries for prompts, and set_tries."""
    with open(os.path.join(B.CSRC, "prompt.cu")) as f:
        text = f.read()
    for old, new in EDITS:
        assert text.count(old) == 1, old
        text = text.replace(old, new)
    src, lib = os.path.join(path, "short_waits_prompt.cu"), os.path.join(path, "short_waits_prompt.so")
    with open(src, "w") as f:
        f.write(text + APPENDED)
    subprocess.check_call([B.nvcc()] + B.NVCC_FLAGS + ["-shared", "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC, "-o", lib, src])
    got = ctypes.CDLL(lib)
    for name in ("gts_prompt_attention", "gts_prompt_attention_grad", "gts_chunk_attention", "gts_prompt_workspace_bytes",
                 "gts_prompt_grad_workspace_bytes", "gts_chunk_workspace_bytes"):
        whole = getattr(serving._load(), name)
        getattr(got, name).argtypes, getattr(got, name).restype = whole.argtypes, whole.restype
    got.set_tries.argtypes, got.set_tries.restype = [ctypes.c_int], ctypes.c_int
    return got
