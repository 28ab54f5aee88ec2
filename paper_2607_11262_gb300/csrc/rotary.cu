// Rotary positions, and appending keys and values to a paged cache with the rotation on the way (gts_rope,
// gts_append_kv).
//
// Mathematics.  Pair i of a head at position p turns by 2 pi frac(p * t_i), t_i turns a position.  t_i is held as an
// integer in units of 2^-64 turns, so p * t_i modulo one turn is one wrapping 64-bit product: exact for every 32-bit
// position, with no large argument ever given to sine and cosine.  The upper 32 bits, as a signed fraction of a turn,
// go to sincospif.  All arithmetic is in 32 bits; a value is rounded to its type once, when it is stored.
//
// Bound by memory traffic: each value is read once and written once.  A block takes a few tokens and all their heads: the
// angles are computed once per block into shared memory, and the values move as 16-byte vectors.  What counts beside that is
// that many blocks stand on an SM (32 registers a thread): several vectors of a thread in flight, which take registers, and
// angles kept in registers over the heads were slower by 5 to 60%, and the packed conversions gained 5%.  Under that limit 8 of the 24
// instances spill 4 to 24 bytes a thread.
// Measured: 16384 tokens of 32 + 8 heads of 128 in 16 bits, 336 MB, 59 us, 85% of the rate of a copy; 8191 in 32 bits 54 us,
// 92%; 16372 appended in 16 bits, 403 MB, 69 us, 87%.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

#include "internal.h"

namespace {

constexpr int THREADS = 256;

struct Part {          // one [tokens][heads][head_dim] tensor of the call
  const void *src;
  void *dst;
  int64_t s_tok, s_head, d_tok, d_head, d_page;  // d_page: for a part that goes to the cache
};

struct Args {
  Part part[3];        // q, k, v
  int end[3];          // heads up to the end of each part
  int n_tokens, head_dim, half;   // half = rot_dim / 2
  int tile;            // tokens of a block; a power of two, at most its rows of threads
  const int32_t *positions;
  const uint64_t *units;
  float factor, sine_factor;      // sine_factor: negative where the map is transposed
  const int64_t *slots;           // append: where tokens go
  int64_t n_slots;
  uint32_t page_size;
  int32_t *status;
};

template <typename T> __device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen(float x) { return x; }
template <> __device__ __forceinline__ float widen(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow(float x) { return x; }
template <> __device__ __forceinline__ __half narrow(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow(float x) { return __float2bfloat16_rn(x); }

// V values of a head as one access: V * sizeof(T) is 16, or V is 1
template <typename T> __device__ __forceinline__ float2 widen2(uint32_t x) {
  if constexpr (std::is_same<T, __half>::value) return __half22float2(*(const __half2 *)&x);
  else return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
}
template <typename T> __device__ __forceinline__ uint32_t narrow2(float x, float y) {
  uint32_t r;
  if constexpr (std::is_same<T, __half>::value) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  return r;
}

// the pair (x, y) turned by f = (cos, sin): one rounding order in every variant, whatever the alignment
__device__ __forceinline__ float turn_x(float x, float y, float2 f) { return __fmaf_rn(x, f.x, -__fmul_rn(y, f.y)); }
__device__ __forceinline__ float turn_y(float x, float y, float2 f) { return __fmaf_rn(y, f.x, __fmul_rn(x, f.y)); }

template <typename T, int V> struct alignas(sizeof(T) * V) Vec { T v[V]; };

// The unit of work is 2 V values of a head: V pairs of the rotated part, or 2 V values that are copied.  Unit u < half /
// V holds pairs u V ...: two runs of V values half apart, or 2 V neighbours (interleaved).  The units after that copy.
template <typename T, int V, bool INTERLEAVED, bool APPEND>
__global__ void __launch_bounds__(THREADS, 8) k_rotary(const Args a) {
  extern __shared__ float2 angles[];  // [tile][half]: factor * (cos, sin)
  using X = Vec<T, V>;
  const int units = (a.head_dim + 2 * V - 1) / (2 * V);
  const int lanes = min(units, THREADS);              // threads along a head; heads with more units take turns
  const int rows = THREADS / lanes;
  const int row = threadIdx.x / lanes, lane = threadIdx.x - row * lanes;
  const int per = rows / a.tile;                      // rows of one token
  const int first = blockIdx.x * a.tile;
  const int which = row / per;                        // the row's token within the tile
  const int token = first + which;
  const bool live = which < a.tile && token < a.n_tokens;
  const int heads = a.end[2];
  const int h0 = row - which * per;
  int64_t page = 0, at = 0;
  bool kept = true;                                   // append: the token has a place in the cache
  if (APPEND && live) {
    const int64_t slot = a.slots[token];
    kept = slot >= 0 && slot < a.n_slots;
    if (slot >= a.n_slots && a.status && lane == 0) *a.status = GTS_ERR_INVALID_PARAMS;
    if (kept) {
      page = (slot >> 32) == 0 ? (int64_t)((uint32_t)slot / a.page_size) : slot / a.page_size;
      at = slot - page * a.page_size;
    }
  }
  X lo, hi;
  T *dst = nullptr;
  int u = lane, x = 0, y = 0;
  bool turned = false, second = false;
  auto place = [&] {                                  // where unit u is in a head
    turned = u * V < a.half;
    x = !turned ? 2 * V * u : INTERLEAVED ? 2 * V * u : V * u;
    y = !turned || INTERLEAVED ? x + V : V * u + a.half;
    second = V > 1 || y < a.head_dim;                 // an odd head's last copied value has no neighbour
  };
  auto load = [&](int h) {
    const int p = h < a.end[0] ? 0 : h < a.end[1] ? 1 : 2;
    dst = nullptr;
    if (h < heads && (!APPEND || p == 0 || kept)) {
      const int head = p == 0 ? h : h - a.end[p - 1];
      const Part &t = a.part[p];
      const T *src = (const T *)t.src + token * t.s_tok + head * t.s_head;
      dst = (T *)t.dst + head * t.d_head + (APPEND && p > 0 ? page * t.d_page + at * t.d_tok : token * t.d_tok);
      lo = *(const X *)(src + x);
      if (second) hi = *(const X *)(src + y);
    }
  };
  place();
  if (live) load(h0);                                 // on its way while the angles are worked out
  for (int i = threadIdx.x; i < a.tile * a.half; i += THREADS) {
    const int w = i / a.half, pair = i - w * a.half;
    if (first + w < a.n_tokens) {
      const uint64_t phase = (uint64_t)(int64_t)a.positions[first + w] * a.units[pair];
      float s, c;
      sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &s, &c);
      angles[i] = make_float2(c * a.factor, s * a.sine_factor);
    }
  }
  __syncthreads();
  if (!live) return;
  bool have = true;                                   // the first unit's values, loaded above
  for (; u < units; u += lanes) {
    place();
#pragma unroll 1
    for (int h = h0; h < heads; h += per) {
      if (!have) load(h);
      have = false;
      if (!dst) continue;
      if (turned && h < a.end[1]) {
        const float2 *const f = angles + which * a.half + u * V;   // read from shared memory each time: fewer registers
        if constexpr (V > 1 && sizeof(T) == 2) {
          // two values at a time through the packed conversions
          uint32_t *const l = (uint32_t *)&lo, *const h2 = (uint32_t *)&hi;
#pragma unroll
          for (int j = 0; j < V / 2; j++) {
            if (INTERLEAVED) {
              const float2 p = widen2<T>(l[j]), q = widen2<T>(h2[j]);
              l[j] = narrow2<T>(turn_x(p.x, p.y, f[j]), turn_y(p.x, p.y, f[j]));
              h2[j] = narrow2<T>(turn_x(q.x, q.y, f[V / 2 + j]), turn_y(q.x, q.y, f[V / 2 + j]));
            } else {
              const float2 e = widen2<T>(l[j]), o = widen2<T>(h2[j]);
              l[j] = narrow2<T>(turn_x(e.x, o.x, f[2 * j]), turn_x(e.y, o.y, f[2 * j + 1]));
              h2[j] = narrow2<T>(turn_y(e.x, o.x, f[2 * j]), turn_y(e.y, o.y, f[2 * j + 1]));
            }
          }
        } else {
          T both[2 * V];
#pragma unroll
          for (int j = 0; j < V; j++) both[j] = lo.v[j], both[V + j] = hi.v[j];
#pragma unroll
          for (int j = 0; j < V; j++) {
            const int e_at = INTERLEAVED ? 2 * j : j, o_at = INTERLEAVED ? 2 * j + 1 : V + j;
            const float e = widen(both[e_at]), o = widen(both[o_at]);
            both[e_at] = narrow<T>(turn_x(e, o, f[j]));
            both[o_at] = narrow<T>(turn_y(e, o, f[j]));
          }
#pragma unroll
          for (int j = 0; j < V; j++) lo.v[j] = both[j], hi.v[j] = both[V + j];
        }
      }
      *(X *)(dst + x) = lo;
      if (second) *(X *)(dst + y) = hi;
    }
  }
}

template <typename T, int V>
cudaError_t launch(const Args &a, bool interleaved, bool append, cudaStream_t stream) {
  const int units = (a.head_dim + 2 * V - 1) / (2 * V);
  const int rows = THREADS / std::min(units, THREADS);
  Args b = a;
  // Tokens of a block: eight rows of threads to a token where that leaves blocks enough for four to an SM.  At a head of 128, 16384
  // tokens: 2 a block take 62 us in 16 bits, 4 take 59; in 32 bits, where a head has twice the units, 2 take 54 and 4 take 58.
  b.tile = 1;
  while (b.tile * 2 * 8 <= rows && (int64_t)a.n_tokens >= (int64_t)b.tile * 2 * 608) b.tile *= 2;
  const int tiles = (a.n_tokens + b.tile - 1) / b.tile;
  const size_t shared = (size_t)b.tile * a.half * sizeof(float2);
  auto k = interleaved ? (append ? k_rotary<T, V, true, true> : k_rotary<T, V, true, false>)
                       : (append ? k_rotary<T, V, false, true> : k_rotary<T, V, false, false>);
  k<<<tiles, THREADS, shared, stream>>>(b);
  return cudaGetLastError();
}

// A part moves as 16-byte vectors if its base and every stride used are multiples of 16 bytes.
bool aligned(const void *p, std::initializer_list<int64_t> strides, int size) {
  uintptr_t bits = (uintptr_t)p;
  for (int64_t s : strides) bits |= (uintptr_t)(s * size);
  return bits % 16 == 0;
}

cudaError_t dispatch(const Args &a, int dtype, bool interleaved, bool append, bool vectors, cudaStream_t stream) {
  switch (dtype) {
    case GTS_BF16:
      return vectors ? launch<__nv_bfloat16, 8>(a, interleaved, append, stream)
                     : launch<__nv_bfloat16, 1>(a, interleaved, append, stream);
    case GTS_F16:
      return vectors ? launch<__half, 8>(a, interleaved, append, stream)
                     : launch<__half, 1>(a, interleaved, append, stream);
    default:
      return vectors ? launch<float, 4>(a, interleaved, append, stream) : launch<float, 1>(a, interleaved, append, stream);
  }
}

int size_of(int dtype) { return dtype == GTS_F32 ? 4 : 2; }

constexpr uint32_t MAX_TOKENS = 1u << 30, MAX_HEADS = 1u << 16, MAX_DIM = 4096;

// What both calls refuse; null where nothing is wrong.
const char *refuse(uint32_t n_tokens, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim, int32_t dtype,
                   const int32_t *positions, const gts_rotary &r) {
  if (dtype != GTS_BF16 && dtype != GTS_F16 && dtype != GTS_F32) return "dtype must be GTS_BF16, GTS_F16 or GTS_F32";
  if (n_tokens > MAX_TOKENS || q_heads > MAX_HEADS || kv_heads > MAX_HEADS || head_dim < 1 || head_dim > MAX_DIM)
    return "size out of range (tokens <= 2^30, heads <= 2^16, 1 <= head_dim <= 4096)";
  if (r.rot_dim % 2 || r.rot_dim > head_dim) return "rot_dim must be even and at most head_dim";
  if (r.layout != GTS_ROTARY_HALF && r.layout != GTS_ROTARY_INTERLEAVED) return "unknown rotary layout";
  if (r.transposed > 1) return "transposed must be 0 or 1";
  if (n_tokens && !positions) return "null positions";
  if (n_tokens && r.rot_dim && !r.units) return "null units";
  if ((uintptr_t)positions % 4 || (uintptr_t)r.units % 8) return "positions or units misaligned";
  return nullptr;
}

const char *refuse_heads(const gts_heads &t, uint32_t heads, uint32_t n_tokens, int size) {
  if (heads && n_tokens && !t.data) return "null tensor";
  if ((uintptr_t)t.data % size) return "tensor misaligned for its type";
  return nullptr;
}

void rotary_args(Args &a, const gts_rotary &r) {
  a.half = (int)(r.rot_dim / 2);
  a.units = r.units;
  a.factor = r.factor;
  a.sine_factor = r.transposed ? -r.factor : r.factor;
}

// Vectors hold whole units only if the rotated part and the head are whole numbers of units.
bool whole_units(uint32_t head_dim, uint32_t rot_dim, int size) {
  return (head_dim * size) % 32 == 0 && (rot_dim * size) % 32 == 0;
}

}  // namespace

extern "C" gts_status gts_rope(const gts_rope_desc *d, void *stream) {
  gts::clear_error();
  if (!d) return gts::fail(GTS_ERR_INVALID_ARG, "rope: null desc");
  const uint32_t kv_heads = d->k.data ? d->kv_heads : 0;
  if (!d->k.data && d->kv_heads && d->n_tokens) return gts::fail(GTS_ERR_INVALID_ARG, "rope: kv_heads without k");
  if (const char *why = refuse(d->n_tokens, d->q_heads, kv_heads, d->head_dim, d->dtype, d->positions, d->rotary))
    return gts::fail(GTS_ERR_INVALID_ARG, why);
  const int size = size_of(d->dtype);
  const gts_heads *t[4] = {&d->q, &d->q_out, &d->k, &d->k_out};
  for (int i = 0; i < 4; i++)
    if (const char *why = refuse_heads(*t[i], i < 2 ? d->q_heads : kv_heads, d->n_tokens, size))
      return gts::fail(GTS_ERR_INVALID_ARG, why);
  if (d->n_tokens == 0 || d->q_heads + kv_heads == 0) return GTS_OK;
  Args a = {};
  a.n_tokens = (int)d->n_tokens;
  a.head_dim = (int)d->head_dim;
  a.positions = d->positions;
  rotary_args(a, d->rotary);
  a.end[0] = (int)d->q_heads;
  a.end[1] = a.end[2] = (int)(d->q_heads + kv_heads);
  a.part[0] = {d->q.data, d->q_out.data, d->q.token_stride, d->q.head_stride, d->q_out.token_stride,
               d->q_out.head_stride, 0};
  a.part[1] = {d->k.data, d->k_out.data, d->k.token_stride, d->k.head_stride, d->k_out.token_stride,
               d->k_out.head_stride, 0};
  bool vectors = whole_units(d->head_dim, d->rotary.rot_dim, size);
  for (int i = 0; i < 4; i++)
    if (i < 2 ? d->q_heads : kv_heads) vectors &= aligned(t[i]->data, {t[i]->token_stride, t[i]->head_stride}, size);
  const cudaError_t e =
      dispatch(a, d->dtype, d->rotary.layout == GTS_ROTARY_INTERLEAVED, false, vectors, (cudaStream_t)stream);
  return e == cudaSuccess ? GTS_OK : gts::cuda_fail(e, "rope: launch");
}

extern "C" gts_status gts_append_kv(const gts_append_desc *d, void *stream) {
  gts::clear_error();
  if (!d) return gts::fail(GTS_ERR_INVALID_ARG, "append_kv: null desc");
  const gts_cache &c = d->cache;
  if (const char *why =
          refuse(d->n_tokens, d->q_heads, c.kv_heads, c.head_dim, c.dtype, d->positions, d->rotary))
    return gts::fail(GTS_ERR_INVALID_ARG, why);
  if (d->rotary.transposed) return gts::fail(GTS_ERR_INVALID_ARG, "append_kv: transposed must be 0");
  const int size = size_of(c.dtype);
  const gts_heads *t[4] = {&d->q, &d->q_out, &d->k, &d->v};
  for (int i = 0; i < 4; i++)
    if (const char *why = refuse_heads(*t[i], i < 2 ? d->q_heads : c.kv_heads, d->n_tokens, size))
      return gts::fail(GTS_ERR_INVALID_ARG, why);
  if (c.page_size < 1 || c.page_size > 1u << 30 || c.n_pages > 1u << 30)
    return gts::fail(GTS_ERR_INVALID_ARG, "append_kv: 1 <= page_size <= 2^30, n_pages <= 2^30");
  if (d->n_tokens == 0) return GTS_OK;
  if (!d->slots || (c.n_pages && c.kv_heads && (!c.k || !c.v)))
    return gts::fail(GTS_ERR_INVALID_ARG, "append_kv: null slots or cache");
  if ((uintptr_t)d->slots % 8 || (uintptr_t)c.k % size || (uintptr_t)c.v % size || (uintptr_t)d->d_status % 4)
    return gts::fail(GTS_ERR_INVALID_ARG, "append_kv: misaligned slots, cache or status");
  Args a = {};
  a.n_tokens = (int)d->n_tokens;
  a.head_dim = (int)c.head_dim;
  a.positions = d->positions;
  rotary_args(a, d->rotary);
  a.end[0] = (int)d->q_heads;
  a.end[1] = (int)(d->q_heads + c.kv_heads);
  a.end[2] = (int)(d->q_heads + 2 * c.kv_heads);
  a.part[0] = {d->q.data, d->q_out.data, d->q.token_stride, d->q.head_stride, d->q_out.token_stride,
               d->q_out.head_stride, 0};
  a.part[1] = {d->k.data, c.k, d->k.token_stride, d->k.head_stride, c.k_token_stride, c.k_head_stride, c.k_page_stride};
  a.part[2] = {d->v.data, c.v, d->v.token_stride, d->v.head_stride, c.v_token_stride, c.v_head_stride, c.v_page_stride};
  a.slots = d->slots;
  a.n_slots = (int64_t)c.n_pages * c.page_size;
  a.page_size = c.page_size;
  a.status = d->d_status;
  if (a.end[2] == 0) return GTS_OK;
  bool vectors = whole_units(c.head_dim, d->rotary.rot_dim, size);
  for (int i = 0; i < 4; i++)
    if (i < 2 ? d->q_heads : c.kv_heads) vectors &= aligned(t[i]->data, {t[i]->token_stride, t[i]->head_stride}, size);
  vectors &= aligned(c.k, {c.k_page_stride, c.k_token_stride, c.k_head_stride}, size) &&
             aligned(c.v, {c.v_page_stride, c.v_token_stride, c.v_head_stride}, size);
  const cudaError_t e =
      dispatch(a, c.dtype, d->rotary.layout == GTS_ROTARY_INTERLEAVED, true, vectors, (cudaStream_t)stream);
  return e == cudaSuccess ? GTS_OK : gts::cuda_fail(e, "append_kv: launch");
}
