// What the attention kernels share: types, barriers, asynchronous copies, tcgen05 products and tensor memory, and on the host the
// launches and the maps of a cache's pages.
#ifndef GTS_TENSOR_CUH
#define GTS_TENSOR_CUH

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "internal.h"

namespace {

// x / d for 0 <= x < 2^31 by a multiplication: m = floor(2^(31 + l) / d) + 1 with 2^(l-1) < d <= 2^l, so m d exceeds 2^(31 + l) by
// at most d <= 2^l, and x times that is below 2^(31 + l).
struct Divisor {
  uint32_t m;
  int shift;           // l - 1; -1 for d = 1
  int d;
};
Divisor divisor(int d) {
  int l = 0;
  while ((1ll << l) < d) l++;
  return {l ? (uint32_t)(((1ull << (31 + l)) / (uint32_t)d) + 1) : 0u, l - 1, d};
}
__device__ __forceinline__ int operator/(int x, const Divisor &d) { return d.shift < 0 ? x : (int)(__umulhi((uint32_t)x, d.m) >> d.shift); }
__device__ __forceinline__ int operator%(int x, const Divisor &d) { return x - x / d * d.d; }

template <typename T> __device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ __half narrow(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow(float x) { return __float2bfloat16_rn(x); }

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool live) {  // zeros where not live
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}

__device__ __forceinline__ float exp2_fast(float x) {  // ex2.approx: 2 ulp, 0 for -infinity
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void bar_init(uint32_t bar, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("{\n.reg .b64 t;\nmbarrier.arrive.shared::cta.b64 t, [%0];\n}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("{\n.reg .b64 t;\nmbarrier.arrive.expect_tx.shared::cta.b64 t, [%0], %1;\n}" ::"r"(bar), "r"(bytes) : "memory");
}

__device__ __forceinline__ uint64_t now_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}

__device__ __forceinline__ void tile_load(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int page, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(page), "r"(bar) : "memory");
}
// the barrier's next arrival comes when this thread's copies so far have landed
__device__ __forceinline__ void bar_arrive_copies(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// two 32-bit values in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 y;
  asm("{\n.reg .b64 a, b, c;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 a, a, b, c;\nmov.b64 {%0, %1}, a;\n}"
      : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return y;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 y;
  asm("{\n.reg .b64 a, b;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}"
      : "=f"(y.x), "=f"(y.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return y;
}
template <typename T> __device__ __forceinline__ uint32_t pack(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <> __device__ __forceinline__ uint32_t pack<__half>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// A page number of a table: a negative one becomes the largest, which no cache has (-1 stands for "no page" in the kernels).
__device__ __forceinline__ int page_number(int32_t x) { return (int)min((uint32_t)x, 0x7FFFFFFFu); }

__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
  return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

__device__ __forceinline__ void dependents_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_kernels_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

struct Pages {
  CUtensorMap k, v;    // pages x heads x tokens (or tokens x heads) x D, boxes of `box` tokens of a head x 64 values (0: no maps)
  int box, k_heads_first, v_heads_first;
};

__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
// d [128 rows][N] (+)= a [128][16] b [16][N]; a from shared memory, or from tensor memory.  Operands in shared memory are
// described by two words; the upper one is the same for all of them here.
__device__ __forceinline__ void tc_mma(uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t shape, bool add) {
  asm volatile("{\n.reg .pred p;\n.reg .b64 x, y;\nmov.b64 x, {%1, %3};\nmov.b64 y, {%2, %3};\nsetp.ne.u32 p, %5, 0;\n"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %4, p;\n}"
               ::"r"(d), "r"(a), "r"(b), "r"(hi), "r"(shape), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void tc_mma_t(uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t shape, bool add) {
  asm volatile("{\n.reg .pred p;\n.reg .b64 y;\nmov.b64 y, {%2, %3};\nsetp.ne.u32 p, %5, 0;\n"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %4, p;\n}"
               ::"r"(d), "r"(a), "r"(b), "r"(hi), "r"(shape), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ bool elected() {  // one lane of a converged warp
  uint32_t is;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(is));
  return is;
}
#define R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define W8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 columns of the warp's 32 rows, one row a lane
__device__ __forceinline__ void tc_ld(uint32_t *r, uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : R8(r, 0), R8(r, 8), R8(r, 16), R8(r, 24) : "r"(at) : "memory");
}
__device__ __forceinline__ void tc_st(uint32_t at, const uint32_t *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
               ::W8(r, 0), W8(r, 8), W8(r, 16), W8(r, 24), "r"(at) : "memory");
}
#undef R8
#undef W8
__device__ __forceinline__ void tc_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Operands in shared memory are rows of 128 bytes, eight rows to a swizzled group of 1024 bytes, groups one after the other.
// Lower word: address, and the bytes from one 128-byte column of groups to the next (for operands that are wider and not
// summed over); upper word: bytes from group to group, version, swizzle.
__device__ __forceinline__ uint32_t operand(uint32_t at, uint32_t blocks) { return at >> 4 | (blocks >> 4) << 16; }
constexpr uint32_t OPERAND_HI = 1024 >> 4 | 1u << 14 | 2u << 29;

// ---------------------------------------------------------------- host side
// A kernel's shared memory above 48 KB is granted once per device.
template <typename K> cudaError_t grant(K kernel, int bytes, std::atomic<uint64_t> &granted) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && (granted.load(std::memory_order_relaxed) >> dev & 1))) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev < 64) granted.fetch_or(1ull << dev, std::memory_order_relaxed);
  return e;
}

size_t up(size_t x) { return (x + 255) / 256 * 256; }

int box_of(int page_size, int most) {  // tokens of a TMA box: the largest power of two that divides both the page and a tile
  int box = 1;
  while (box < most && page_size % (box * 2) == 0) box *= 2;
  return box;
}

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static std::atomic<void *> found{nullptr};
  void *f = found.load(std::memory_order_relaxed);
  if (!f) {
    cudaDriverEntryPointQueryResult got;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &got) != cudaSuccess ||
        got != cudaDriverEntryPointSuccess)
      return nullptr;
    found.store(f, std::memory_order_relaxed);
  }
  return (EncodeTiled)f;
}

// A map of the cache's pages for the tensor cores' kernel.  False where strides or alignment do not fit one: each dimension's
// stride has to be a multiple of 16 bytes and of the one before it.
bool tile_map(CUtensorMap &map, int &heads_first, int box, const gts_cache &c, void *base, int64_t page, int64_t token, int64_t head) {
  const int64_t D = c.head_dim;
  heads_first = c.page_size > 1 && (c.kv_heads == 1 || head < token);
  if (c.kv_heads == 1) head = heads_first ? D : token * c.page_size;
  if (c.page_size == 1) token = D;
  const int64_t lo = heads_first ? head : token, hi = heads_first ? token : head;
  if (c.n_pages == 1) page = hi * (heads_first ? c.page_size : c.kv_heads);
  if ((uintptr_t)base % 16 || lo % 8 || lo < D || hi < lo || hi % lo || page < hi || page % hi || page >= 1ll << 38) return false;
  const EncodeTiled encode = encode_tiled();
  if (!encode) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)D, heads_first ? c.kv_heads : c.page_size, heads_first ? c.page_size : c.kv_heads, c.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)lo * 2, (cuuint64_t)hi * 2, (cuuint64_t)page * 2};
  const cuuint32_t boxes[4] = {64, heads_first ? 1u : (cuuint32_t)box, heads_first ? (cuuint32_t)box : 1u, 1}, ones[4] = {1, 1, 1, 1};
  return encode(&map, c.dtype == GTS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, base, dims, strides,
                boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool tile_maps(Pages &p, const gts_cache &c, int most) {
  const int box = box_of((int)c.page_size, most);
  if (box < 8 || !c.n_pages) return false;   // a box is whole groups of eight rows
  p.box = box;
  const bool ok = tile_map(p.k, p.k_heads_first, p.box, c, c.k, c.k_page_stride, c.k_token_stride, c.k_head_stride) &&
                  tile_map(p.v, p.v_heads_first, p.box, c, c.v, c.v_page_stride, c.v_token_stride, c.v_head_stride);
  if (!ok) p.box = 0;
  return ok;
}

// A launch that may start as soon as the kernel before it allows (`early`): the kernels above wait for each other themselves.
template <typename... P, typename... A>
cudaError_t launch_kernel(void (*kernel)(P...), unsigned blocks, unsigned threads, int shared, cudaStream_t s, bool early, const A &...args) {
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3(blocks), c.blockDim = dim3(threads), c.dynamicSmemBytes = (size_t)shared, c.stream = s;
  c.attrs = &attr, c.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&c, kernel, args...);
}

}  // namespace

#endif
