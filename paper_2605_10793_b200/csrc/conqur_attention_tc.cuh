// The attention of conqur_attention.cuh for more than 16 query rows a key head (trees of drafted tokens): there the products set the pace, and they go to
// the tcgen05 tensor cores.  One CTA an SM works on blocks of 128 rows, 64 tokens at a time:
//   S = Q K^T (128 x 64) and O += P V (128 x D) with accumulators in TMEM; S and P have two buffers, so that the products of one tile run
//   while the exponentials of the other are taken.
//   warps 0-3   one row a thread: scores from TMEM, bound, exponentials (no exchange between threads), P as bf16 to shared memory
//   warps 4-7   bring keys and values: bf16 as they lie (the cache's planes are the operands' swizzled layout), codes turned into the bf16 integers
//               (code - zero-point) / 64, exactly; the steps go to the scores and the probabilities
//   warp 8      issues the products
// The bound of a row is raised only when a score exceeds it by 2^8; then its accumulators are read, scaled and written back.  Work is cut into runs and parts
// are joined as in conqur_attention.cuh.  Every wait between the warps is bounded: when one runs out the CTA latches TIMEOUT, writes nothing more and ends.
// Floor of the exponentials: 8192 a tile at 16 a cycle, 512 cycles; the products take about the same.
#pragma once
#include "conqur_attention.cuh"

namespace conqur {
namespace kv {

template <int BITS_, int D_>
struct TreeCfg {
  static constexpr int BITS = BITS_, D = D_;
  static constexpr int ROWS = 128, THREADS = 288, PLANES = D / 64;
  static constexpr int Q_BYTES = PLANES * 16384;               // 128 rows x 128 bytes a plane
  static constexpr int T_BYTES = PLANES * 8192;                // keys or values of a tile
  static constexpr int P_BYTES = 16384;
  static constexpr int AUX_BYTES = 2048;
  static constexpr int SMEM = 1024 + Q_BYTES + 4 * T_BYTES + 2 * P_BYTES + AUX_BYTES;
  static constexpr int SLOT = (D + 2) * 128;                   // floats of a part: columns of 128 rows; then bounds, sums
};

template <typename C>
struct TreeAux {
  uint64_t full[2], scored[2], ready[2], done[2];              // tile brought; S complete; P written; P V complete
  float kstep[2][64], vstep[2][64];
  uint32_t bad[2][2];                                          // tokens of a tile whose page could not be read
  Walk<C> w;
  uint32_t tmem;
  int abort_flag, last, odd;                                   // odd: some value near the end of the sequence is not finite
};

// 32 lanes x 16 consecutive columns: thread t of the warp holds row (lane base + t).
__device__ __forceinline__ void tmem_read16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_write16(uint32_t taddr, const uint32_t (&w)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "r"(w[8]), "r"(w[9]), "r"(w[10]), "r"(w[11]),
        "r"(w[12]), "r"(w[13]), "r"(w[14]), "r"(w[15])
      : "memory");
}
__device__ __forceinline__ void tmem_write_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
// Eight codes of a word as (code - zero-point) / 64, in the order of their elements: nibbles at bits 0 and 4 of both halves are c 2^-133 and 16 c 2^-133 as bf16.
__device__ __forceinline__ uint4 codes8(uint32_t w, uint32_t bias) {
  const uint32_t h = w >> 8;
  return make_uint4(fma_bf16x2(codes_even(w), 0x7F007F00u, bias), fma_bf16x2(codes_odd(w), 0x7D007D00u, bias),
                    fma_bf16x2(codes_even(h), 0x7F007F00u, bias), fma_bf16x2(codes_odd(h), 0x7D007D00u, bias));
}
__device__ __forceinline__ uint32_t zero_bias(uint32_t rec) { return fma_bf16x2(zero_of(rec) * 0x10001u, 0xFF00FF00u, 0x80008000u); }   // -z / 64
__device__ __forceinline__ bool not_finite2(uint32_t w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; }

// ---- warps 4-7: a thread takes a token's 64 dimensions of one plane, of keys and values (D = 64: threads 0-63 the keys, 64-127 the values)
template <typename C>
struct Bring {
  int tok, plane;
  bool keys, values;
  const int* table;
  const uint8_t* head;
  int len;
  int page, cur;                     // of the tile after next (asked for ahead), of the next tile
  uint4 k[2], v[2];                  // 4 bits: the next tile's codes and records
  uint32_t kr, vr;
  bool good;

  __device__ __forceinline__ void item(const AttnArgs& a, const Walk<C>& w, int tid) {
    tok = tid & 63;
    const int half = tid >> 6;
    plane = C::D == 128 ? half : 0;
    keys = C::D == 128 || half == 0;
    values = C::D == 128 || half == 1;
    table = a.table + (long long)w.b * a.table_stride;
    head = a.cache + (long long)(w.item % a.kv_heads) * a.block_bytes;
    len = w.s.context + w.s.nodes;
  }
  __device__ __forceinline__ void ask(const AttnArgs& a, int tile, int end) {
    const int pos = tile * ATTN_UNIT + tok;
    page = -1;
    if (tile < end && pos < len && (pos >> a.log_page) < a.table_width) page = table[pos >> a.log_page];
  }
  __device__ __forceinline__ const uint8_t* block(const AttnArgs& a) const { return head + (long long)cur * a.page_bytes; }
  // 4 bits: the codes of the tile whose page was asked for
  __device__ __forceinline__ void load(const AttnArgs& a, int tile) {
    cur = page;
    good = (unsigned)cur < (unsigned)a.pages;
    kr = vr = 0u;
    k[0] = k[1] = v[0] = v[1] = make_uint4(0u, 0u, 0u, 0u);
    if (C::BITS == 4 && good) {
      const int at = (tile * ATTN_UNIT + tok) & (a.page_size - 1);
      const uint8_t* p = block(a);
      const uint8_t* c = p + at * (C::D / 2) + plane * 32;
      if (keys) {
        k[0] = *reinterpret_cast<const uint4*>(c);
        k[1] = *reinterpret_cast<const uint4*>(c + 16);
        kr = *reinterpret_cast<const uint32_t*>(p + 2 * a.codes_bytes + at * 4);
      }
      if (values) {
        v[0] = *reinterpret_cast<const uint4*>(c + a.codes_bytes);
        v[1] = *reinterpret_cast<const uint4*>(c + a.codes_bytes + 16);
        vr = *reinterpret_cast<const uint32_t*>(p + 2 * a.codes_bytes + (a.page_size + at) * 4);
      }
    }
  }
  static __device__ __forceinline__ void spread(uint8_t* row, const uint4 (&c)[2], uint32_t bias, int t) {
    const uint32_t w[8] = {c[0].x, c[0].y, c[0].z, c[0].w, c[1].x, c[1].y, c[1].z, c[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(row + ((i ^ (t & 7)) << 4)) = codes8(w[i], bias);
  }
  __device__ __forceinline__ void put(const AttnArgs& a, TreeAux<C>* aux, uint8_t* tile_mem, int buf, int tile, int context) {
    const int pos = tile * ATTN_UNIT + tok;
    uint8_t* kd = tile_mem + plane * 8192 + tok * 128;
    uint8_t* vd = kd + C::T_BYTES;
    const unsigned lost = __ballot_sync(0xffffffffu, !good && pos < len);
    const int tid = threadIdx.x - 128;
    if (tid < 64 && (tid & 31) == 0) {
      aux->bad[buf][tid >> 5] = lost;
      if (lost) atomicOr(a.flags, KV_FLAG_BAD_INDEX);
    }
    if (C::BITS == 4) {
      // (a record that says NaN: the step carries it; its codes are codes)
      if (keys) spread(kd, k, zero_bias(kr), tok);
      if (values) spread(vd, v, zero_bias(vr), tok);
      if (tid < 64) aux->kstep[buf][tok] = step_of(kr) * a.scale;               // the scale has the 64 of the codes
      if (values && (C::D == 64 || tid >= 64)) aux->vstep[buf][tok] = step_of(vr) * 64.f;
    } else {
      const int at = pos & (a.page_size - 1), bytes = good ? 16 : 0;
      const uint8_t* p = good ? block(a) + plane * a.plane_bytes + at * 128 : a.cache;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (keys) copy16(ptx::smem_u32(kd + i * 16), p + i * 16, bytes);
        if (values) copy16(ptx::smem_u32(vd + i * 16), good ? p + C::PLANES * a.plane_bytes + i * 16 : p, bytes);
      }
      asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
      if (values && (tile + 1) * ATTN_UNIT > context) {
        // what is not finite must not meet the zeros of rows that do not see it: left out here, added at the end
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint4 x = *reinterpret_cast<uint4*>(vd + i * 16);
          uint32_t* e = &x.x;
          bool hit = false;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (not_finite2(e[j])) {
              hit = true;
              if ((e[j] & 0x7F80u) == 0x7F80u) e[j] &= 0xFFFF0000u;
              if ((e[j] & 0x7F800000u) == 0x7F800000u) e[j] &= 0x0000FFFFu;
            }
          if (hit) {
            *reinterpret_cast<uint4*>(vd + i * 16) = x;
            *reinterpret_cast<volatile int*>(&aux->odd) = 1;
          }
        }
      }
    }
  }
};

// ---- a row of the block, as its thread (warps 0-3) sees it
struct TreeRow {
  bool real;
  long long row;                     // of q and out
  int head;                          // query head
  unsigned long long mask;
};
template <typename C>
__device__ __forceinline__ TreeRow tree_row(const AttnArgs& a, const Seq& s, int item, int r) {
  const int kh = item % a.kv_heads;
  r += (item / a.kv_heads) * C::ROWS;
  TreeRow t;
  const int node = r / a.group;
  t.real = r < s.nodes * a.group;
  t.row = s.start + node;
  t.head = kh * a.group + r - node * a.group;
  t.mask = 0ull;
  if (t.real) {
    t.mask = a.mask ? a.mask[t.row] : (2ull << node) - 1ull;
    if (s.nodes < 64) t.mask &= (1ull << s.nodes) - 1ull;
  }
  return t;
}
// Bits of the 64 positions from `first` on that a row sees: the context and its drafted tokens.
__device__ __forceinline__ unsigned long long seen64(unsigned long long mask, int context, int first) {
  const int n = context - first;
  if (n >= 64) return ~0ull;
  if (n > 0) return ((1ull << n) - 1ull) | (mask << n);
  return -n < 64 ? mask >> -n : 0ull;
}

template <typename C>
__global__ void __launch_bounds__(C::THREADS, 1) attn_tree_kernel(const AttnArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  constexpr int D = C::D, PL = C::PLANES;
  uint8_t* sQ = smem;
  uint8_t* sT = smem + C::Q_BYTES;                             // keys, values; keys, values
  uint8_t* sP = sT + 4 * C::T_BYTES;
  TreeAux<C>* aux = reinterpret_cast<TreeAux<C>*>(sP + 2 * C::P_BYTES);
  static_assert(sizeof(TreeAux<C>) <= C::AUX_BYTES, "TreeCfg::AUX_BYTES");
  const int warp = warp_index(), lane = threadIdx.x & 31, tid = threadIdx.x;
  volatile int* abort_flag = &aux->abort_flag;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&aux->full[i], 128);
      ptx::mbar_init(&aux->scored[i], 1);
      ptx::mbar_init(&aux->ready[i], 128);
      ptx::mbar_init(&aux->done[i], 1);
    }
    aux->abort_flag = 0;
    ptx::fence_barrier_init();
    ptx::fence_proxy_async();
  }
  if (warp == 0) {
    Walk<C> b;
    b.begin(a);
    if (lane == 0) aux->w = b;
  }
  if (warp == 8) {
    ptx::tmem_alloc(&aux->tmem, 256);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = aux->tmem, tO = tmem + 128;            // S: two buffers of 64 columns; O: D columns
  Walk<C> w = aux->w;
  int cnt = 0;                                                 // tiles so far: buffer cnt & 1, phase (cnt >> 1) & 1
  bool head_of_run = true, more = w.left > 0;

  while (more) {
    // ---- the item's rows
    if (warp < 8) {
      const int kh = w.item % a.kv_heads, first = (w.item / a.kv_heads) * C::ROWS, rows = w.s.nodes * a.group;
      for (int i = tid; i < 128 * (D / 8); i += 256) {
        const int r = i / (D / 8), ch = i % (D / 8);
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (first + r < rows) {
          const int node = (first + r) / a.group;
          x = *reinterpret_cast<const uint4*>(a.q + (long long)(w.s.start + node) * a.q_t + (long long)(kh * a.group + first + r - node * a.group) * a.q_h + ch * 8);
        }
        *reinterpret_cast<uint4*>(sQ + (ch >> 3) * 16384 + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = x;
      }
      if (tid == 0) aux->odd = 0;
      ptx::fence_proxy_async();
    }
    __syncthreads();
    const int tiles = w.end - w.tile;
    const int len = w.s.context + w.s.nodes;

    if (warp >= 4 && warp < 8) {
      // ------------------------------------------------------------ keys and values
      Bring<C> in;
      in.item(a, w, tid - 128);
      in.ask(a, w.tile, w.end);
      in.load(a, w.tile);
      in.ask(a, w.tile + 1, w.end);
      for (int i = 0; i < tiles; ++i) {
        const int n = cnt + i, buf = n & 1;
        if (!tc_wait_warp(&aux->done[buf], ((n >> 1) & 1) ^ 1, abort_flag)) break;
        in.put(a, aux, sT + buf * 2 * C::T_BYTES, buf, w.tile + i, w.s.context);
        ptx::fence_proxy_async();
        ptx::mbar_arrive(&aux->full[buf]);
        in.load(a, w.tile + i + 1);
        in.ask(a, w.tile + i + 2, w.end);
      }
    } else if (warp == 8) {
      // ------------------------------------------------------------ products
      const uint32_t leader = ptx::elect_one();
      const uint32_t base = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 4) << 24);
      const uint32_t id_s = base | ((uint32_t)(64 >> 3) << 17), id_o = base | (1u << 16) | ((uint32_t)(D >> 3) << 17);
      const uint32_t q0 = ptx::smem_u32(sQ), t0 = ptx::smem_u32(sT), p0 = ptx::smem_u32(sP);
      auto scores = [&](int n) {
        const int buf = n & 1;
        if (!tc_wait_warp(&aux->full[buf], (n >> 1) & 1, abort_flag)) return false;
        ptx::tc_fence_after();
        const uint32_t k0 = t0 + buf * 2 * C::T_BYTES;
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
          ptx::umma_bf16_by<false>(leader, tmem + buf * 64, tc_smem_desc(q0 + (j >> 2) * 16384 + (j & 3) * 32, 16, 1024),
                                   tc_smem_desc(k0 + (j >> 2) * 8192 + (j & 3) * 32, 16, 1024), id_s, j > 0 ? 1u : 0u);
        ptx::umma_commit_by<false>(leader, ptx::smem_u32(&aux->scored[buf]));
        return true;
      };
      bool ok = scores(cnt);
      for (int i = 0; ok && i < tiles; ++i) {
        const int n = cnt + i, buf = n & 1;
        // the buffer of the next scores was read before P of the tile before this one was written
        if (i + 1 < tiles && !(ok = scores(n + 1))) break;
        if (!(ok = tc_wait_warp(&aux->ready[buf], (n >> 1) & 1, abort_flag))) break;
        ptx::tc_fence_after();
        const uint32_t v0 = t0 + buf * 2 * C::T_BYTES + C::T_BYTES;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          ptx::umma_bf16_by<false>(leader, tO, tc_smem_desc(p0 + buf * C::P_BYTES + j * 32, 16, 1024), tc_smem_desc(v0 + j * 2048, 8192, 1024), id_o,
                                   (i > 0 || j > 0) ? 1u : 0u);
        ptx::umma_commit_by<false>(leader, ptx::smem_u32(&aux->done[buf]));
      }
    } else {
      // ------------------------------------------------------------ a row a thread
      const TreeRow row = tree_row<C>(a, w.s, w.item, tid);
      const uint32_t lanes = (uint32_t)(warp * 32) << 16;
      float m = -INFINITY, l = 0.f;
      bool ok = true;
      for (int i = 0; i < tiles; ++i) {
        const int n = cnt + i, buf = n & 1, first = (w.tile + i) * ATTN_UNIT;
        // (the steps come with the tile, the scores with its product)
        if (!(ok = tc_wait_warp(&aux->full[buf], (n >> 1) & 1, abort_flag) && tc_wait_warp(&aux->scored[buf], (n >> 1) & 1, abort_flag))) break;
        ptx::tc_fence_after();
        float s[2][32];
        ptx::tmem_ld32(tmem + lanes + buf * 64, s[0]);
        ptx::tmem_ld32(tmem + lanes + buf * 64 + 32, s[1]);
        const unsigned long long bad = (unsigned long long)aux->bad[buf][0] | ((unsigned long long)aux->bad[buf][1] << 32);
        const bool edge = first + ATTN_UNIT > w.s.context || bad != 0ull;
        const unsigned long long see = edge ? seen64(row.mask, w.s.context, first) & ~bad : ~0ull;
        float top = -INFINITY;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            float4 k = make_float4(a.scale, a.scale, a.scale, a.scale);
            if (C::BITS == 4) k = *reinterpret_cast<const float4*>(&aux->kstep[buf][h * 32 + j]);
            s[h][j] *= k.x; s[h][j + 1] *= k.y; s[h][j + 2] *= k.z; s[h][j + 3] *= k.w;
          }
        if (edge) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (!((see >> (h * 32 + j)) & 1ull)) s[h][j] = -INFINITY;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 32; ++j) top = fmaxf(top, s[h][j]);
        const bool up = top > m + 8.f;                         // (no bound yet: m = -inf, and any score exceeds it)
        if (__any_sync(0xffffffffu, up)) {
          const float f = up ? ex2(m - top) : 1.f;
          if (up) m = top;
          l *= f;
          if (i > 0) {                                         // (the first tile's product overwrites O)
            if (!(ok = tc_wait_warp(&aux->done[(n - 1) & 1], ((n - 1) >> 1) & 1, abort_flag))) break;
            ptx::tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {
              uint32_t o[16];
              tmem_read16(tO + lanes + c, o);
#pragma unroll
              for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
              tmem_write16(tO + lanes + c, o);
            }
            tmem_write_wait();
          }
        }
        const float bound = m == -INFINITY ? 0.f : m;
        // P of two tiles ago has been read when its product is complete
        if (!(ok = tc_wait_warp(&aux->done[buf], ((n >> 1) & 1) ^ 1, abort_flag))) break;
        uint8_t* prow = sP + buf * C::P_BYTES + tid * 128;
        float sum = 0.f;                                       // a tile's probabilities by themselves: fewer roundings of a long sum
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 32; j += 8) {
            float p[8];
            float4 v0 = make_float4(1.f, 1.f, 1.f, 1.f), v1 = v0;
            if (C::BITS == 4) {
              v0 = *reinterpret_cast<const float4*>(&aux->vstep[buf][h * 32 + j]);
              v1 = *reinterpret_cast<const float4*>(&aux->vstep[buf][h * 32 + j + 4]);
            }
            const float vs[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float q = ex2(s[h][j + e] - bound);
              sum += q;
              p[e] = C::BITS == 4 ? q * vs[e] : q;
              if (C::BITS == 4 && edge && s[h][j + e] == -INFINITY) p[e] = 0.f;      // an unseen record may say NaN
            }
            *reinterpret_cast<uint4*>(prow + (((h * 4 + j / 8) ^ (tid & 7)) << 4)) =
                make_uint4(bf16x2(p[0], p[1]), bf16x2(p[2], p[3]), bf16x2(p[4], p[5]), bf16x2(p[6], p[7]));
          }
        l += sum;
        ptx::fence_proxy_async();
        ptx::tc_fence_before();
        ptx::mbar_arrive(&aux->ready[buf]);
      }
      const int last = cnt + tiles - 1;
      if (ok) ok = tc_wait_warp(&aux->done[last & 1], (last >> 1) & 1, abort_flag);
      ptx::tc_fence_after();
      bar_sync(BAR_ALL, 128);
      if (!*abort_flag) {
        const bool whole = w.tile == 0 && w.end == w.s.tiles;
        const bool none = l == 0.f && m == -INFINITY;
        float* part = a.parts + (2 * (size_t)blockIdx.x + (head_of_run ? 0 : 1)) * C::SLOT + tid;
        const float inv = none ? 0.f : 1.f / l;
        const int odd = C::BITS == 16 ? *reinterpret_cast<volatile int*>(&aux->odd) : 0;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          float o[32];
          ptx::tmem_ld32(tO + lanes + c, o);
          if (whole) {
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] *= inv;
          }
          if (C::BITS == 16 && odd && row.real) {
            // values that are not finite, of the tokens that the row sees (rare)
            for (int pos = max(w.tile * ATTN_UNIT, w.s.context & ~(ATTN_UNIT - 1)); pos < min(len, w.end * ATTN_UNIT); ++pos) {
              const int d = pos - w.s.context;
              if (d >= 0 && !((row.mask >> d) & 1ull)) continue;
              const int page = (pos >> a.log_page) < a.table_width ? a.table[(long long)w.b * a.table_stride + (pos >> a.log_page)] : -1;
              if ((unsigned)page >= (unsigned)a.pages) continue;
              const int at = pos & (a.page_size - 1);
              const uint8_t* v = a.cache + (long long)page * a.page_bytes + (long long)(w.item % a.kv_heads) * a.block_bytes + (PL + c / 64) * a.plane_bytes + at * 128;
#pragma unroll
              for (int j = 0; j < 32; ++j) {
                const int e = (c & 63) + j;
                const uint32_t x = *reinterpret_cast<const unsigned short*>(v + (((e >> 3) ^ (at & 7)) << 4) + (e & 7) * 2);
                if ((x & 0x7F80u) == 0x7F80u) o[j] += __uint_as_float(x << 16);
              }
            }
          }
          if (!whole) {
#pragma unroll
            for (int j = 0; j < 32; ++j) __stcg(part + (c + j) * 128, o[j]);
          } else if (row.real) {
            __nv_bfloat16* out = a.out + row.row * a.o_t + row.head * a.o_h + c;
#pragma unroll
            for (int j = 0; j < 32; j += 8)
              *reinterpret_cast<uint4*>(out + j) = make_uint4(bf16x2(o[j], o[j + 1]), bf16x2(o[j + 2], o[j + 3]), bf16x2(o[j + 4], o[j + 5]), bf16x2(o[j + 6], o[j + 7]));
          }
        }
        if (whole) {
          if (row.real && a.lse) a.lse[row.row * a.lse_t + row.head] = none ? -INFINITY : (m == -INFINITY ? 0.f : m) * 0.6931471805599453f + logf(l);
        } else {
          __stcg(part + D * 128, m);
          __stcg(part + (D + 1) * 128, l);
          __threadfence();
          bar_sync(BAR_ALL, 128);
          const int c0 = w.owner(w.item_at), c1 = w.owner(w.item_at + w.s.tiles - 1);
          if (tid == 0) {
            const unsigned n = (unsigned)(c1 - c0);
            aux->last = atomicInc(a.counters + c0, n) == n;
            __threadfence();
          }
          bar_sync(BAR_ALL, 128);
          if (aux->last) {
            auto slot = [&](int k) { return a.parts + (2 * (size_t)k + (w.run_begin(k) < w.item_at ? 1 : 0)) * C::SLOT + tid; };
            float tm = -INFINITY, tl = 0.f;
            for (int k = c0; k <= c1; ++k) {
              const float* p = slot(k);
              const float om = __ldcg(p + D * 128), ol = __ldcg(p + (D + 1) * 128);
              const float to = om > tm ? om : tm;
              tl = tl * (to == -INFINITY ? 1.f : ex2(tm - to)) + ol * (to == -INFINITY ? 1.f : ex2(om - to));
              tm = to;
            }
            const bool zero = tl == 0.f && tm == -INFINITY;
            const float ti = zero ? 0.f : 1.f / tl;
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              float o[32];
#pragma unroll
              for (int j = 0; j < 32; ++j) o[j] = 0.f;
              for (int k = c0; k <= c1; ++k) {
                const float* p = slot(k);
                const float om = __ldcg(p + D * 128), f = (tm == -INFINITY ? 1.f : ex2(om - tm)) * ti;
#pragma unroll
                for (int j = 0; j < 32; ++j) o[j] = fmaf(__ldcg(p + (c + j) * 128), f, o[j]);
              }
              if (row.real) {
                __nv_bfloat16* out = a.out + row.row * a.o_t + row.head * a.o_h + c;
#pragma unroll
                for (int j = 0; j < 32; j += 8)
                  *reinterpret_cast<uint4*>(out + j) = make_uint4(bf16x2(o[j], o[j + 1]), bf16x2(o[j + 2], o[j + 3]), bf16x2(o[j + 4], o[j + 5]), bf16x2(o[j + 6], o[j + 7]));
              }
            }
            if (row.real && a.lse) a.lse[row.row * a.lse_t + row.head] = zero ? -INFINITY : (tm == -INFINITY ? 0.f : tm) * 0.6931471805599453f + logf(tl);
          }
        }
      }
      ptx::tc_fence_before();
    }
    __syncthreads();                                           // rows, tiles and accumulators may be replaced
    ptx::tc_fence_after();
    if (*abort_flag) break;
    cnt += tiles;
    head_of_run = false;
    more = w.next(a);
  }
  if (tid == 0 && *abort_flag) atomicOr(a.flags, KV_FLAG_TIMEOUT);
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 8) ptx::tmem_dealloc(tmem, 256);
}

}  // namespace kv
}  // namespace conqur
