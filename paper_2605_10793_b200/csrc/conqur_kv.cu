// The paged key/value cache: writing rows into it (4-bit zero-point codes of Appendix B or bf16), reading values back, and the attention of
// drafted tokens over it (conqur_attention.cuh).
//
// Writing and reading move every byte once and are bound by memory.  A row of head_dim elements lies in head_dim / 8 lanes, 16 bytes (bf16) each;
// a lane's eight elements make one 32-bit word of codes.  Key and value row of a (token, head) are worked on together, two of them a lane, so that
// 64 bytes a lane are in flight.
// Measured, 32768 tokens of 8 heads of 128 into 4-bit codes and back: 69 us (51.7 at memory's rate); writing takes 39 of them under a profiler, where it issues 3.2 of 4
// instructions a cycle.  With each lane dividing for itself and codes one by one: 87 us.
// Codes are the ones that exact arithmetic gives: the step is rounded to bf16 BEFORE it divides, so y / step is a quotient of two 8-bit significands.
// Such a quotient is a tie (k + 1/2) or at least 2^-9 away from one; y * (1 / step) in fp32 is off by 2^-19 at most, so rounding it to a
// multiple of 2^-11 first restores the ties and disturbs nothing else, and no division per element is needed.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <mutex>

#include "../../include/conqur.h"
#include "conqur_attention.cuh"
#include "conqur_attention_tc.cuh"

using namespace conqur;
using bf16 = __nv_bfloat16;

namespace {

constexpr int KV_ANSWERS = 64;
__device__ int g_kv_flags[1 + KV_ANSWERS];   // the conditions latched on this device; answers of conqur_kv_status

struct RowsArgs {
  uint8_t* cache;
  const bf16 *k, *v;
  int64_t k_t, k_h, v_t, v_h;
  void *k_out, *v_out;
  const int64_t* slots;
  int64_t items, slots_total;              // (token, head) pairs; places of the cache
  int64_t block_bytes;
  uint32_t heads, head_mul, head_shift;    // item / heads = item * head_mul >> head_shift for item < 2^31
  int log_page;
  float clip;
  int* flags;
};

constexpr int ROWS_THREADS = 256;

// max and -min of a lane's eight elements as a pair of bf16, NaN kept
__device__ __forceinline__ uint32_t range_of(const uint4 raw) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  __nv_bfloat162 h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = *reinterpret_cast<const __nv_bfloat162*>(&w[i]);
  const __nv_bfloat162 mx = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  const __nv_bfloat162 mn = __hmin2_nan(__hmin2_nan(h[0], h[1]), __hmin2_nan(h[2], h[3]));
  const __nv_bfloat162 both = __halves2bfloat162(__hmax_nan(__low2bfloat16(mx), __high2bfloat16(mx)),
                                                 __hneg(__hmin_nan(__low2bfloat16(mn), __high2bfloat16(mn))));
  return *reinterpret_cast<const uint32_t*>(&both);
}
__device__ __forceinline__ uint32_t wider(uint32_t x, uint32_t y) {
  const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&x), *reinterpret_cast<const __nv_bfloat162*>(&y));
  return *reinterpret_cast<const uint32_t*>(&m);
}
// Record (step, zero-point code) and 1 / step (0: all codes are zero) of a row with this range.
template <bool CLIP>
__device__ __forceinline__ uint32_t row_record(uint32_t range, float clip, float& inv) {
  const float top = __uint_as_float(range << 16), low = -__uint_as_float(range & 0xFFFF0000u);
  float step, zero = 0.f;
  inv = 0.f;
  if (!(top < 1.7014118346046923e38f && low > -1.7014118346046923e38f)) {      // 2^127: a code's value may lie 1/15 beyond the range
    step = __uint_as_float(0x7FC00000u);
  } else {
    const float hi = fmaxf(top, 0.f), lo = fminf(low, 0.f);
    // c = 1: every quantity below is what 64-bit arithmetic rounds to (hi - lo has at most 17 bits or a part below 2^-16 of it)
    if (CLIP) {
      const double c = (double)clip;
      step = __bfloat162float(__float2bfloat16_rn((float)((c * hi - c * lo) / 15.0)));
    } else {
      step = __bfloat162float(__float2bfloat16_rn((hi - lo) / 15.f));
    }
    if (step < 7.888609052210118e-31f) step = 0.f;             // 2^-100
    if (step > 0.f) {
      zero = CLIP ? (float)-rint((double)clip * lo / (double)step) : -rintf(lo / step);
      zero = fminf(fmaxf(zero, 0.f), 15.f);
      inv = 1.f / step;
    }
  }
  return (__float_as_uint(step) >> 16) | ((uint32_t)zero << 16);
}
// A lane's eight codes.
template <bool CLIP>
__device__ __forceinline__ uint32_t row_codes(const uint4 raw, uint32_t record, float inv) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w}, zeros = (record >> 16) * 0x10001u;
  const uint64_t inv2 = kv::two(inv, inv), up = kv::two(6144.f, 6144.f), down = kv::two(-6144.f, -6144.f), magic = kv::two(12582912.f, 12582912.f);
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint64_t q = kv::two(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
    if (CLIP) {                                                // (beyond the range by any factor)
      const float2 y = kv::apart(kv::two_mul(q, inv2));
      q = kv::two_add(kv::two(fminf(fmaxf(y.x, -64.f), 64.f), fminf(fmaxf(y.y, -64.f), 64.f)), up);
    } else {
      q = kv::two_fma(q, inv2, up);                            // 1.5 * 2^12: multiples of 2^-11
    }
    const float2 r = kv::apart(kv::two_add(kv::two_add(q, down), magic));      // 1.5 * 2^23: half to even, the integer in the low bits
    c[i] = __viaddmin_s16x2_relu(__byte_perm(__float_as_uint(r.x), __float_as_uint(r.y), 0x5410), zeros, 0x000F000Fu);
  }
  return inv > 0.f ? c[0] | (c[1] << 4) | (c[2] << 8) | (c[3] << 12) : 0u;
}
// Four rows, L lanes each with eight elements of every one.  The ranges are reduced so that a lane ends with that of row lane % 4: the divisions of a row
// are made by L / 4 lanes, not L, and handed round.
template <int L, bool CLIP>
__device__ __forceinline__ void quantise4(const uint4 (&raw)[4], float clip, int l, uint32_t (&word)[4], uint32_t (&record)[4]) {
  const uint32_t r0 = range_of(raw[0]), r1 = range_of(raw[1]), r2 = range_of(raw[2]), r3 = range_of(raw[3]);
  const bool b0 = l & 1, b1 = l & 2;
  const uint32_t x = wider(b0 ? r1 : r0, __shfl_xor_sync(0xffffffffu, b0 ? r0 : r1, 1));
  const uint32_t y = wider(b0 ? r3 : r2, __shfl_xor_sync(0xffffffffu, b0 ? r2 : r3, 1));
  uint32_t range = wider(b1 ? y : x, __shfl_xor_sync(0xffffffffu, b1 ? x : y, 2));
#pragma unroll
  for (int m = 4; m < L; m <<= 1) range = wider(range, __shfl_xor_sync(0xffffffffu, range, m));
  float inv;
  const uint32_t rec = row_record<CLIP>(range, clip, inv);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    record[r] = __shfl_sync(0xffffffffu, rec, r, 4);
    word[r] = row_codes<CLIP>(raw[r], record[r], __shfl_sync(0xffffffffu, inv, r, 4));
  }
}

template <bool VEC>
__device__ __forceinline__ uint4 load8(const bf16* p) {
  if (VEC) return *reinterpret_cast<const uint4*>(p);
  const unsigned short* u = reinterpret_cast<const unsigned short*>(p);
  return make_uint4(u[0] | ((uint32_t)u[1] << 16), u[2] | ((uint32_t)u[3] << 16), u[4] | ((uint32_t)u[5] << 16), u[6] | ((uint32_t)u[7] << 16));
}

__device__ __forceinline__ void split_item(const RowsArgs& a, int64_t item, int64_t& token, int& head) {
  const uint32_t t = (uint32_t)(((uint64_t)(uint32_t)item * a.head_mul) >> a.head_shift);
  token = t;
  head = (int)((uint32_t)item - t * a.heads);
}

template <int BITS, int D, bool VEC, bool CLIP>
__global__ void __launch_bounds__(ROWS_THREADS) kv_append_kernel(const RowsArgs a) {
  constexpr int L = D / 8, PER_BLOCK = ROWS_THREADS / L;
  const int l = threadIdx.x % L;
  const int64_t first = (int64_t)blockIdx.x * PER_BLOCK * 2 + threadIdx.x / L;
  uint4 rows[4];                                               // key and value of both items
  int64_t slot[2];
  int head[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int64_t item = first + u * PER_BLOCK;
    slot[u] = -1;
    rows[2 * u] = rows[2 * u + 1] = make_uint4(0u, 0u, 0u, 0u);
    if (item < a.items) {
      int64_t token;
      split_item(a, item, token, head[u]);
      slot[u] = a.slots[token];
      rows[2 * u] = load8<VEC>(a.k + token * a.k_t + head[u] * a.k_h + 8 * l);
      rows[2 * u + 1] = load8<VEC>(a.v + token * a.v_t + head[u] * a.v_h + 8 * l);
    }
  }
  uint32_t word[4], record[4];
  if (BITS == 4) quantise4<L, CLIP>(rows, a.clip, l, word, record);      // all lanes: there are shuffles
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    if (slot[u] < 0) continue;
    if (slot[u] >= a.slots_total) {
      if (l == 0) atomicOr(a.flags, kv::KV_FLAG_BAD_INDEX);
      continue;
    }
    const int64_t page = slot[u] >> a.log_page;
    const int ps = 1 << a.log_page, t = (int)(slot[u] & (ps - 1));
    uint8_t* block = a.cache + (page * a.heads + head[u]) * a.block_bytes;
    if (BITS == 4) {
      *reinterpret_cast<uint32_t*>(block + t * (D / 2) + 4 * l) = word[2 * u];
      *reinterpret_cast<uint32_t*>(block + (ps + t) * (D / 2) + 4 * l) = word[2 * u + 1];
      if (l < 2) *reinterpret_cast<uint32_t*>(block + ps * D + (l * ps + t) * 4) = l ? record[2 * u + 1] : record[2 * u];
    } else {
      const int at = ((l >> 3) * ps + t) * 128 + (((l & 7) ^ (t & 7)) << 4);
      *reinterpret_cast<uint4*>(block + at) = rows[2 * u];
      *reinterpret_cast<uint4*>(block + ps * D * 2 + at) = rows[2 * u + 1];
    }
  }
}

__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(bf16* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(kv::bf16x2(x[0], x[1]), kv::bf16x2(x[2], x[3]), kv::bf16x2(x[4], x[5]), kv::bf16x2(x[6], x[7]));
}

// (code - zero-point) * step: a code masked where it lies, with the bits of 2^23 above it, is 2^23 + c 16^i; every step but the last product is exact.
__device__ __forceinline__ void unpack(uint32_t w, uint32_t record, float (&x)[8]) {
  const float step = kv::step_of(record), z = (float)kv::zero_of(record);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float p = (float)(1 << (4 * i)), down = -fmaf(z, p, 8388608.f), scaled = step * (1.f / p);
    const uint32_t m = 15u << (4 * i);
    const float2 v = kv::apart(kv::two_mul(
        kv::two_add(kv::two(__uint_as_float((w & m) | 0x4B000000u), __uint_as_float(((w >> 16) & m) | 0x4B000000u)), kv::two(down, down)),
        kv::two(scaled, scaled)));
    x[2 * i] = v.x;
    x[2 * i + 1] = v.y;
  }
}

template <int BITS, int D, typename T>
__global__ void __launch_bounds__(ROWS_THREADS) kv_read_kernel(const RowsArgs a) {
  constexpr int L = D / 8, PER_BLOCK = ROWS_THREADS / L;
  const int l = threadIdx.x % L;
  const int64_t first = (int64_t)blockIdx.x * PER_BLOCK * 2 + threadIdx.x / L;
  uint4 kr[2], vr[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int64_t item = first + u * PER_BLOCK;
    kr[u] = vr[u] = make_uint4(0u, 0u, 0u, 0u);
    if (item >= a.items) continue;
    int64_t token;
    int head;
    split_item(a, item, token, head);
    const int64_t slot = a.slots[token];
    if (slot >= a.slots_total && l == 0) atomicOr(a.flags, kv::KV_FLAG_BAD_INDEX);
    if (slot < 0 || slot >= a.slots_total) continue;
    const int64_t page = slot >> a.log_page;
    const int ps = 1 << a.log_page, t = (int)(slot & (ps - 1));
    const uint8_t* block = a.cache + (page * a.heads + head) * a.block_bytes;
    if (BITS == 4) {
      kr[u].x = *reinterpret_cast<const uint32_t*>(block + t * (D / 2) + 4 * l);
      vr[u].x = *reinterpret_cast<const uint32_t*>(block + (ps + t) * (D / 2) + 4 * l);
      kr[u].y = *reinterpret_cast<const uint32_t*>(block + ps * D + t * 4);
      vr[u].y = *reinterpret_cast<const uint32_t*>(block + ps * D + (ps + t) * 4);
    } else {
      const int at = ((l >> 3) * ps + t) * 128 + (((l & 7) ^ (t & 7)) << 4);
      kr[u] = *reinterpret_cast<const uint4*>(block + at);
      vr[u] = *reinterpret_cast<const uint4*>(block + ps * D * 2 + at);
    }
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int64_t item = first + u * PER_BLOCK;
    if (item >= a.items) continue;
    T* ko = static_cast<T*>(a.k_out) + item * D + 8 * l;
    T* vo = static_cast<T*>(a.v_out) + item * D + 8 * l;
    float x[8], y[8];
    if (BITS == 4) {
      unpack(kr[u].x, kr[u].y, x);
      unpack(vr[u].x, vr[u].y, y);
    } else {
      const uint32_t kw[4] = {kr[u].x, kr[u].y, kr[u].z, kr[u].w}, vw[4] = {vr[u].x, vr[u].y, vr[u].z, vr[u].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = __uint_as_float((i & 1) ? (kw[i >> 1] & 0xFFFF0000u) : (kw[i >> 1] << 16));
        y[i] = __uint_as_float((i & 1) ? (vw[i >> 1] & 0xFFFF0000u) : (vw[i >> 1] << 16));
      }
    }
    store8(ko, x);
    store8(vo, y);
  }
}

// Takes one condition out of the flags: each is seen and cleared in one step, and the other one, or what another stream latches meanwhile, stays.
__global__ void kv_status_kernel(int* flags, int* answer) {
  int told = atomicAnd(flags, ~kv::KV_FLAG_TIMEOUT) & kv::KV_FLAG_TIMEOUT;
  if (!told) told = atomicAnd(flags, ~kv::KV_FLAG_BAD_INDEX) & kv::KV_FLAG_BAD_INDEX;
  *answer = told;
}

// ---------------------------------------------------------------------------------------------------- host

bool cache_ok(const conqur_kv_cache* c) {
  if (!c || c->struct_size != sizeof(conqur_kv_cache)) return false;
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64) return false;
  if (c->kv_heads < 1 || c->kv_heads > 65535 || (c->head_dim != 64 && c->head_dim != 128) || (c->bits != 4 && c->bits != 16)) return false;
  if (!(c->clip_ratio >= 0.f && c->clip_ratio <= 1.f)) return false;
  return c->pages >= 1 && c->pages <= ((int64_t)1 << 31) / c->page_size;
}
int64_t block_bytes(const conqur_kv_cache* c) { return (int64_t)c->page_size * (c->bits == 4 ? c->head_dim + 8 : 4 * c->head_dim); }
int log2_of(int x) { return x == 16 ? 4 : x == 32 ? 5 : 6; }
int launched() { return cudaGetLastError() == cudaSuccess ? CONQUR_OK : CONQUR_ERR_CUDA; }

// The flag word's address on the current device (looked up once per device).
int* flags_here(int* device = nullptr) {
  static std::mutex mu;
  static int* known[64] = {nullptr};
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
  if (device) *device = dev;
  std::lock_guard<std::mutex> lock(mu);
  if (!known[dev]) {
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_kv_flags) != cudaSuccess) return nullptr;
    known[dev] = static_cast<int*>(p);
  }
  return known[dev];
}

int rows_args(const conqur_kv_cache* c, int64_t n, const int64_t* slots, RowsArgs& a) {
  if (!cache_ok(c) || n < 0) return CONQUR_ERR_INVALID_ARG;
  if (n > 0 && (!c->cache_dev || (reinterpret_cast<uintptr_t>(c->cache_dev) & 15) || !slots || (reinterpret_cast<uintptr_t>(slots) & 7))) return CONQUR_ERR_INVALID_ARG;
  if (n > (int64_t)0x7fffffff / c->kv_heads) return CONQUR_ERR_INVALID_ARG;
  a = RowsArgs{};
  a.cache = static_cast<uint8_t*>(c->cache_dev);
  a.slots = slots;
  a.items = n * c->kv_heads;
  a.slots_total = c->pages * c->page_size;
  a.block_bytes = block_bytes(c);
  a.heads = (uint32_t)c->kv_heads;
  int s = 0;
  while ((1u << s) < a.heads) ++s;
  a.head_shift = 31 + s;
  a.head_mul = (uint32_t)((((uint64_t)1 << a.head_shift) + a.heads - 1) / a.heads);
  a.log_page = log2_of(c->page_size);
  a.clip = c->clip_ratio;
  a.flags = nullptr;
  return CONQUR_OK;
}

// ---- attention: variants by bits, head_dim and rows of a block

struct AttnVariant {
  void (*kernel)(const kv::AttnArgs);
  int rows, threads, smem, slot_floats, ctas_max;
  float code_scale;                       // 4 bits: what the scores' units ask for
};
template <typename C>
AttnVariant variant() {
  return {kv::attn_kernel<C>, C::ROWS, C::THREADS, C::SMEM, C::PART * 32, 592, C::BITS == 4 ? kv::ATTN_Q_BACK : 1.f};
}
template <typename C>
AttnVariant tree_variant() {
  return {kv::attn_tree_kernel<C>, C::ROWS, C::THREADS, C::SMEM, C::SLOT, 160, C::BITS == 4 ? 64.f : 1.f};
}
constexpr int ATTN_VARIANTS = 3;
constexpr int ATTN_CTAS_MAX = 592;        // runs of work: 4 per SM (the tensor cores' variant: 1, and larger parts)
constexpr size_t ATTN_COUNTER_BYTES = (ATTN_CTAS_MAX * sizeof(unsigned) + 255) / 256 * 256;      // at the workspace's start in every call

template <int BITS, int D>
AttnVariant by_rows(int i) {
  // chunks of codes are a quarter of those of bf16: two blocks an SM
  constexpr bool small = BITS == 4;
  constexpr int halves = 128 / D;
  switch (i) {
    case 0: return variant<kv::AttnCfg<BITS, D, 1, small ? 8 : 4, (small ? 2 : 3) * halves, small ? 2 : 1>>();
    case 1: return variant<kv::AttnCfg<BITS, D, 2, small ? 8 : 4, (small ? 4 : 2) * halves, 1>>();
    default: return tree_variant<kv::TreeCfg<BITS, D>>();
  }
}
// Eight or sixteen rows on the warps' own products, more on the tcgen05 tensor cores in blocks of 128.
int rows_class(int rows) { return rows <= 8 ? 0 : rows <= 16 ? 1 : 2; }
AttnVariant pick(int bits, int d, int cls) {
  if (bits == 4) return d == 64 ? by_rows<4, 64>(cls) : by_rows<4, 128>(cls);
  return d == 64 ? by_rows<16, 64>(cls) : by_rows<16, 128>(cls);
}

bool attn_sizes_ok(const conqur_kv_cache* c, int batch, int group, int max_nodes) {
  return cache_ok(c) && batch >= 0 && batch <= 65535 && group >= 1 && group <= 64 && max_nodes >= 1 && max_nodes <= 64 &&
         (int64_t)c->kv_heads * group <= 65536;
}

}  // namespace

extern "C" size_t conqur_kv_cache_bytes(const conqur_kv_cache* c) { return cache_ok(c) ? (size_t)(c->pages * c->kv_heads * block_bytes(c)) : 0; }

extern "C" int conqur_kv_append(const conqur_kv_cache* cache, const void* K_dev, int64_t k_token_stride, int64_t k_head_stride, const void* V_dev,
                                int64_t v_token_stride, int64_t v_head_stride, int64_t n, const int64_t* slots_dev, void* cuda_stream) {
  RowsArgs a;
  const int rc = rows_args(cache, n, slots_dev, a);
  if (rc != CONQUR_OK) return rc;
  if (n > 0 && (!K_dev || !V_dev || ((reinterpret_cast<uintptr_t>(K_dev) | reinterpret_cast<uintptr_t>(V_dev)) & 1))) return CONQUR_ERR_INVALID_ARG;
  if (n == 0) return CONQUR_OK;
  a.flags = flags_here();
  if (!a.flags) return CONQUR_ERR_CUDA;
  a.k = static_cast<const bf16*>(K_dev); a.v = static_cast<const bf16*>(V_dev);
  a.k_t = k_token_stride; a.k_h = k_head_stride; a.v_t = v_token_stride; a.v_h = v_head_stride;
  const bool vec = ((reinterpret_cast<uintptr_t>(K_dev) | reinterpret_cast<uintptr_t>(V_dev)) & 15) == 0 &&
                   ((k_token_stride | k_head_stride | v_token_stride | v_head_stride) & 7) == 0;
  const bool clip = cache->clip_ratio != 0.f && cache->clip_ratio != 1.f;
  const int per_block = 2 * ROWS_THREADS / (cache->head_dim / 8);
  const unsigned blocks = (unsigned)((a.items + per_block - 1) / per_block);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  auto go = [&](auto bits, auto d, auto v, auto c) {
    kv_append_kernel<decltype(bits)::value, decltype(d)::value, decltype(v)::value, decltype(c)::value><<<blocks, ROWS_THREADS, 0, s>>>(a);
  };
  using std::integral_constant;
  auto with_vec = [&](auto bits, auto d, auto c) {
    if (vec) go(bits, d, std::true_type(), c);
    else go(bits, d, std::false_type(), c);
  };
  auto with_clip = [&](auto bits, auto d) {
    if (decltype(bits)::value == 4 && clip) with_vec(bits, d, std::true_type());
    else with_vec(bits, d, std::false_type());
  };
  auto with_bits = [&](auto d) {
    if (cache->bits == 4) with_clip(integral_constant<int, 4>(), d);
    else with_clip(integral_constant<int, 16>(), d);
  };
  if (cache->head_dim == 64) with_bits(integral_constant<int, 64>());
  else with_bits(integral_constant<int, 128>());
  return launched();
}

extern "C" int conqur_kv_read(const conqur_kv_cache* cache, const int64_t* slots_dev, int64_t n, void* K_out_dev, void* V_out_dev, int32_t out_dtype,
                              void* cuda_stream) {
  RowsArgs a;
  const int rc = rows_args(cache, n, slots_dev, a);
  if (rc != CONQUR_OK) return rc;
  if (out_dtype != CONQUR_F32 && out_dtype != CONQUR_BF16) return CONQUR_ERR_INVALID_ARG;
  if (n > 0 && (!K_out_dev || !V_out_dev || ((reinterpret_cast<uintptr_t>(K_out_dev) | reinterpret_cast<uintptr_t>(V_out_dev)) & 15))) return CONQUR_ERR_INVALID_ARG;
  if (n == 0) return CONQUR_OK;
  a.flags = flags_here();
  if (!a.flags) return CONQUR_ERR_CUDA;
  a.k_out = K_out_dev; a.v_out = V_out_dev;
  const int per_block = 2 * ROWS_THREADS / (cache->head_dim / 8);
  const unsigned blocks = (unsigned)((a.items + per_block - 1) / per_block);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  auto go = [&](auto bits, auto d) {
    if (out_dtype == CONQUR_F32) kv_read_kernel<decltype(bits)::value, decltype(d)::value, float><<<blocks, ROWS_THREADS, 0, s>>>(a);
    else kv_read_kernel<decltype(bits)::value, decltype(d)::value, bf16><<<blocks, ROWS_THREADS, 0, s>>>(a);
  };
  using std::integral_constant;
  if (cache->bits == 4) {
    if (cache->head_dim == 64) go(integral_constant<int, 4>(), integral_constant<int, 64>());
    else go(integral_constant<int, 4>(), integral_constant<int, 128>());
  } else {
    if (cache->head_dim == 64) go(integral_constant<int, 16>(), integral_constant<int, 64>());
    else go(integral_constant<int, 16>(), integral_constant<int, 128>());
  }
  return launched();
}

extern "C" int conqur_kv_status(void* cuda_stream) {
  static std::atomic<unsigned> calls{0};                       // callers on several threads get their answers in words of their own
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  int* flags = flags_here();
  int told = 0;
  if (!flags) return CONQUR_ERR_CUDA;
  int* answer = flags + 1 + calls.fetch_add(1u) % KV_ANSWERS;
  kv_status_kernel<<<1, 1, 0, s>>>(flags, answer);
  if (cudaGetLastError() != cudaSuccess || cudaMemcpyAsync(&told, answer, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess)
    return CONQUR_ERR_CUDA;
  return told == kv::KV_FLAG_TIMEOUT ? CONQUR_ERR_TIMEOUT : told == kv::KV_FLAG_BAD_INDEX ? CONQUR_ERR_BAD_INDEX : CONQUR_OK;
}

extern "C" size_t conqur_tree_attention_workspace_bytes(const conqur_kv_cache* cache, int32_t group, int32_t max_nodes) {
  if (!attn_sizes_ok(cache, 0, group, max_nodes)) return 0;
  size_t most = 0;                         // the variants of fewer rows may have the larger slots
  for (int i = 0; i <= rows_class(group * max_nodes); ++i) {
    const AttnVariant v = pick(cache->bits, cache->head_dim, i);
    const size_t n = (size_t)2 * v.ctas_max * v.slot_floats;
    if (n > most) most = n;
  }
  return ATTN_COUNTER_BYTES + most * sizeof(float);
}

namespace {

// The wait that a test asks for (conqur_debug_tree_attention); site 0: none.
struct LostWait { int block, site, index; };

int tree_attention(const conqur_kv_cache* cache, const conqur_tree_call* c, const LostWait& lost, void* cuda_stream) {
  if (!c || c->struct_size != sizeof(conqur_tree_call) || !attn_sizes_ok(cache, c->batch, c->group, c->max_nodes)) return CONQUR_ERR_INVALID_ARG;
  if (!std::isfinite(c->scale) || c->table_width < 0 || c->rows < 0 || c->rows > 0x7fffffff || c->table_stride < 0) return CONQUR_ERR_INVALID_ARG;
  if (c->batch == 0 || c->rows == 0) return CONQUR_OK;
  if (!cache->cache_dev || (reinterpret_cast<uintptr_t>(cache->cache_dev) & 15)) return CONQUR_ERR_INVALID_ARG;
  if (!c->q_dev || !c->out_dev || !c->starts_dev || !c->contexts_dev || (!c->table_dev && c->table_width > 0) || !c->workspace_dev) return CONQUR_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(c->q_dev) | reinterpret_cast<uintptr_t>(c->out_dev)) & 15) ||
      ((c->q_token_stride | c->q_head_stride | c->out_token_stride | c->out_head_stride) & 7))
    return CONQUR_ERR_INVALID_ARG;
  const int64_t heads = (int64_t)cache->kv_heads * c->group;
  if (c->lse_dev && c->rows > 1 && c->lse_token_stride < heads && c->lse_token_stride > -heads) return CONQUR_ERR_INVALID_ARG;
  if ((c->rows > 1 && c->out_token_stride == 0) || (heads > 1 && c->out_head_stride == 0)) return CONQUR_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(c->starts_dev) | reinterpret_cast<uintptr_t>(c->contexts_dev) | reinterpret_cast<uintptr_t>(c->table_dev) |
       reinterpret_cast<uintptr_t>(c->lse_dev)) & 3)
    return CONQUR_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(c->mask_dev) & 7) || (reinterpret_cast<uintptr_t>(c->workspace_dev) & 255)) return CONQUR_ERR_INVALID_ARG;
  if (c->workspace_bytes < conqur_tree_attention_workspace_bytes(cache, c->group, c->max_nodes)) return CONQUR_ERR_WORKSPACE_TOO_SMALL;

  const int cls = rows_class(c->group * c->max_nodes);
  if (lost.site != 0 && cls != 2) return CONQUR_ERR_UNSUPPORTED;
  const AttnVariant v = pick(cache->bits, cache->head_dim, cls);
  kv::AttnArgs a = {};
  a.cache = static_cast<const uint8_t*>(cache->cache_dev);
  a.pages = (int)cache->pages; a.page_size = cache->page_size; a.log_page = log2_of(cache->page_size); a.kv_heads = cache->kv_heads;
  a.group = c->group; a.max_nodes = c->max_nodes; a.batch = c->batch; a.table_width = c->table_width;
  a.block_bytes = block_bytes(cache); a.page_bytes = a.block_bytes * cache->kv_heads;
  a.codes_bytes = cache->page_size * cache->head_dim / 2; a.plane_bytes = cache->page_size * 128;
  a.rows = c->rows;
  a.scale = (float)((double)c->scale * 1.4426950408889634) * v.code_scale;
  a.q = static_cast<const bf16*>(c->q_dev); a.q_t = c->q_token_stride; a.q_h = c->q_head_stride;
  a.out = static_cast<bf16*>(c->out_dev); a.o_t = c->out_token_stride; a.o_h = c->out_head_stride;
  a.lse = c->lse_dev; a.lse_t = c->lse_token_stride;
  a.starts = c->starts_dev; a.contexts = c->contexts_dev; a.table = c->table_dev; a.table_stride = c->table_stride;
  a.mask = reinterpret_cast<const unsigned long long*>(c->mask_dev);
  a.lose_block = lost.block; a.lose_site = lost.site; a.lose_index = lost.index;
  a.counters = static_cast<unsigned*>(c->workspace_dev);
  a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(c->workspace_dev) + ATTN_COUNTER_BYTES);

  // per device and variant: shared-memory limit set and resident blocks counted once
  struct Facts { int known, ctas; };
  static std::mutex mu;
  static Facts facts[64][2][2][ATTN_VARIANTS] = {};
  int dev = -1;
  a.flags = flags_here(&dev);
  if (!a.flags) return CONQUR_ERR_CUDA;
  int ctas = 0;
  {
    std::lock_guard<std::mutex> lock(mu);
    Facts& f = facts[dev][cache->bits == 16][cache->head_dim == 128][cls];
    if (!f.known) {
      int per_sm = 0, sms = 0;
      if (cudaFuncSetAttribute(v.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, v.smem) != cudaSuccess ||
          cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, v.kernel, v.threads, v.smem) != cudaSuccess ||
          cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return CONQUR_ERR_CUDA;
      if (per_sm < 1) return CONQUR_ERR_UNSUPPORTED;
      f.ctas = per_sm * sms < v.ctas_max ? per_sm * sms : v.ctas_max;
      f.known = 1;
    }
    ctas = f.ctas;
  }
  v.kernel<<<ctas, v.threads, v.smem, static_cast<cudaStream_t>(cuda_stream)>>>(a);
  return launched();
}

}  // namespace

extern "C" int conqur_tree_attention(const conqur_kv_cache* cache, const conqur_tree_call* call, void* cuda_stream) {
  return tree_attention(cache, call, LostWait{0, 0, 0}, cuda_stream);
}

extern "C" int conqur_debug_tree_attention(const conqur_kv_cache* cache, const conqur_tree_call* call, int32_t block, int32_t site, int32_t index, void* cuda_stream) {
  if (block < 0 || site < CONQUR_TREE_WAIT_STAGE || site > CONQUR_TREE_WAIT_OUTPUT || index < 0 || index >= (site <= CONQUR_TREE_WAIT_TILE ? 4 : 2)) return CONQUR_ERR_INVALID_ARG;
  return tree_attention(cache, call, LostWait{block, site, index}, cuda_stream);
}
