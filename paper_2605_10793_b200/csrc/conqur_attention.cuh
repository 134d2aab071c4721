// Attention of a few query rows per sequence (one drafted token or a tree of them, times the query heads that share a key head)
// over a paged cache of keys and values, 4-bit codes or bf16.
//
//   s_l = scale q . k_l,  o = sum_l 2^(s_l log2 e - m) v_l / sum_l 2^(s_l log2 e - m),  m a running bound of the row's scores
//
// What bounds it: the cache is read once and every byte of it meets at most a few hundred rows, so with few rows memory sets the
// pace, with a tree of some dozen rows the unpacking and the products do.
//   - The tokens, not the rows, are the 16-row side of the warps' products (m16n8k16): S^T = K Q^T and O^T = V^T P^T.  Eight
//     rows fill an instruction, and a fragment of K or V that was unpacked from codes is used for all rows of the warp.  The codes go from shared memory to the
//     fragments in registers, in an order of dimensions (and of output dimensions) that lets every lane read whole words of a token's row;
//     a product does not depend on the order of what it sums over.
//   - P^T goes from the accumulator layout of the first product to the operand layout of the second with movmatrix, two per eight rows.
//   - The running maximum is only a bound: rows are rescaled when a score exceeds it by 2^8, one vote per 16 tokens instead of a
//     reduction (P is rounded relatively, a common factor changes nothing).
//   - The work, in tiles of tokens of one sequence, key head and block of rows, is laid end to end and cut into equal runs, one per
//     resident CTA, whatever the lengths.  A piece of work that is cut leaves its parts (accumulators, maximum, sum) in the workspace; the
//     last CTA to finish one of its parts adds them up in their order.  No CTA waits for another.
//   - A producer warp brings pages with bulk copies into a ring of stages; pages are contiguous per head, one copy each.
// Every wait is bounded; a warp whose wait ran out goes on without reading or writing results, so that the block's barriers match, and the call latches TIMEOUT.
#pragma once
#include "conqur_tc.cuh"

namespace conqur {
namespace kv {

struct AttnArgs {
  const uint8_t* cache;
  long long pages;
  int page_size, log_page, kv_heads, group, max_nodes, batch, table_width;
  long long block_bytes, rows;
  float scale;                       // times log2 e
  const __nv_bfloat16* q; long long q_t, q_h;
  __nv_bfloat16* out; long long o_t, o_h;
  float* lse; long long lse_t;
  const int* starts; const int* contexts; const int* table; long long table_stride;
  const unsigned long long* mask;
  unsigned* counters;                // one per CTA, for the item that its run ends in the middle of: parts finished, wraps to 0
  float* parts;                      // two slots per CTA
  int* flags;
};

enum { KV_FLAG_BAD_INDEX = 1, KV_FLAG_TIMEOUT = 2 };

// BITS of the cache, D, and how a block of 8 NT WM rows and TILE tokens is shared out: WM warps over the rows, WN over the tokens.
template <int BITS_, int D_, int NT_, int WM_, int WN_, int STAGES_, int MINB_>
struct AttnCfg {
  static constexpr int BITS = BITS_, D = D_, NT = NT_, WM = WM_, WN = WN_, STAGES = STAGES_, MINB = MINB_;
  static constexpr int WARPS = WM * WN, CONSUMERS = 32 * WARPS, THREADS = CONSUMERS + 32;
  static constexpr int ROWS = 8 * NT * WM;                       // query rows of a block
  static constexpr int TILE = WN * 16 < 64 ? 64 : WN * 16;       // tokens of a stage: a multiple of the largest page
  static constexpr int SUBS = TILE / (16 * WN);                  // groups of 16 tokens of a warp
  static constexpr int TOKEN_BYTES = BITS == 4 ? D + 8 : 4 * D;
  static constexpr int STAGE_BYTES = TILE * TOKEN_BYTES;
  static constexpr int KS = D / 16;                              // k steps of the first product, 16-dimension tiles of the second
  static constexpr int QFRAG_BYTES = KS * (ROWS / 8) * 32 * 8;
  static constexpr int ACC = NT * KS * 4;                        // accumulators a lane
  static constexpr int PART = ACC + 4 * NT;                      // and its maxima and sums
  static constexpr int MERGE_BYTES = WN > 1 ? WM * (WN / 2) * PART * 32 * 4 : 0;
  static constexpr int AUX_BYTES = 512;
  static constexpr int SMEM = STAGES * STAGE_BYTES + QFRAG_BYTES + MERGE_BYTES + ROWS * 8 + AUX_BYTES;
  static_assert(SMEM * MINB <= 227 * 1024, "shared memory of an SM");
  static_assert(TILE % 64 == 0 && SUBS * 16 * WN == TILE, "a stage holds whole pages");
  static_assert((WN & (WN - 1)) == 0, "the warps' parts are added in halves");
};

struct AttnAux {
  uint64_t full[8], empty[8];
  uint32_t bad[8];                   // per stage: pages (in order) that could not be read
  int abort_flag, last;
};
static_assert(sizeof(AttnAux) <= 512, "AttnCfg::AUX_BYTES");

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t movmatrix(uint32_t a) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
  return r;
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void named_sync(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }
// codes c in the low nibbles of both halves of w >> shift, less (128 + z) once 128 is added by the exponent: c - z as bf16, exactly
__device__ __forceinline__ uint32_t codes2(uint32_t w, int shift, uint32_t bias) {
  const uint32_t v = ((w >> shift) & 0x000F000Fu) | 0x43004300u;
  uint32_t r;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(bias));
  return r;
}
__device__ __forceinline__ float step_of(uint32_t rec) { return __uint_as_float(rec << 16); }
__device__ __forceinline__ uint32_t zero_of(uint32_t rec) { return (rec >> 16) & 15u; }       // whatever the bytes are, a code

// The drafted tokens and context of a sequence, and what its work comes to.
struct Seq {
  int start, nodes, context;
  int tiles, blocks;                 // tiles of tokens, blocks of rows
};
template <typename C>
__device__ __forceinline__ Seq sequence(const AttnArgs& a, int b) {
  Seq s;
  const long long s0 = a.starts[b], s1 = a.starts[b + 1];
  long long n = s1 - s0;
  int c = a.contexts[b];
  bool bad = false;
  if (s0 < 0 || n < 0 || s1 > a.rows) { n = 0; bad = true; }
  if (n > a.max_nodes) { n = a.max_nodes; bad = true; }
  if (c < 0) { c = 0; bad = true; }
  if (c > 0x7fffff00) { c = 0x7fffff00; bad = true; }       // positions stay below 2^31
  if (bad && blockIdx.x == 0 && threadIdx.x < 32) atomicOr(a.flags, KV_FLAG_BAD_INDEX);
  s.start = (int)s0;
  s.nodes = (int)n;
  s.context = c;
  s.tiles = n > 0 ? (int)(((long long)c + n + C::TILE - 1) / C::TILE) : 0;
  s.blocks = (int)((n * a.group + C::ROWS - 1) / C::ROWS);
  return s;
}

// A CTA's run of tiles, item after item; an item is one (sequence, block of rows, key head).
template <typename C>
struct Walk {
  long long left, total, at;         // tiles of the run still to come; of all work; the next tile's place in all work
  int ctas;                          // CTAs with a run: no more than there are tiles, so that none is empty
  Seq s;
  int b, item, tile;                 // the item's sequence, its number there (block of rows * kv_heads + key head), and its next tile
  int end;                           // the run's last tile of the item, plus one
  long long item_at;                 // place of the item's first tile

  // Every warp works this out for itself: a sum over the sequences, then the one in which the run begins.
  __device__ void begin(const AttnArgs& a) {
    const int lane = threadIdx.x & 31;
    total = 0;
    for (int i = lane; i < a.batch; i += 32) {
      const Seq q = sequence<C>(a, i);
      total += (long long)q.tiles * q.blocks * a.kv_heads;
    }
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) total += __shfl_xor_sync(0xffffffffu, total, m);
    ctas = total < (long long)gridDim.x ? (int)total : (int)gridDim.x;
    b = 0;
    left = 0;
    if ((int)blockIdx.x >= ctas) return;
    at = run_begin(blockIdx.x);
    left = run_begin(blockIdx.x + 1) - at;
    long long before = 0;
    for (int base = 0; base < a.batch; base += 32) {
      long long mine = 0;
      if (base + lane < a.batch) {
        const Seq q = sequence<C>(a, base + lane);
        mine = (long long)q.tiles * q.blocks * a.kv_heads;
      }
      long long upto = mine;
#pragma unroll
      for (int m = 1; m < 32; m <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, upto, m);
        if (lane >= m) upto += o;
      }
      const unsigned in = __ballot_sync(0xffffffffu, at < before + upto);
      if (in) {
        const int k = __ffs(in) - 1;
        b = base + k;
        before += __shfl_sync(0xffffffffu, upto - mine, k);
        break;
      }
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    s = sequence<C>(a, b);
    const long long in_seq = at - before;
    item = (int)(in_seq / s.tiles);
    tile = (int)(in_seq - (long long)item * s.tiles);
    item_at = at - tile;
    cut();
  }
  __device__ void cut() { end = (long long)(s.tiles - tile) <= left ? s.tiles : tile + (int)left; }
  // To the next item; false at the end of the run.
  __device__ bool next(const AttnArgs& a) {
    left -= end - tile;
    at += end - tile;
    if (left <= 0) return false;
    if (++item == s.blocks * a.kv_heads) {
      item = 0;
      do s = sequence<C>(a, ++b);
      while (s.tiles == 0 && b + 1 < a.batch);
    }
    tile = 0;
    item_at = at;
    cut();
    return true;
  }
  // CTA whose run holds a tile
  __device__ int owner(long long t) const { return (int)(((t + 1) * ctas - 1) / total); }
  __device__ long long run_begin(int cta) const { return total * cta / ctas; }
};

// ---------------------------------------------------------------------------------------------- the producer warp
template <typename C>
__device__ void attn_produce(const AttnArgs& a, uint8_t* stages, AttnAux* aux) {
  const int lane = threadIdx.x & 31;
  const int pages_per_tile = C::TILE >> a.log_page;              // at most 8
  Walk<C> w;
  w.begin(a);
  if (w.left <= 0) return;
  int st = 0;
  uint32_t phase = 1;                                            // a fresh barrier's previous phase counts as complete
  bool ok = true, any = false;
  do {
    const int head = w.item % a.kv_heads;
    const long long len = (long long)w.s.context + w.s.nodes;
    const int* row = a.table + (long long)w.b * a.table_stride;
    for (int tile = w.tile; ok && tile < w.end; ++tile) {
      const long long first = ((long long)tile * C::TILE >> a.log_page) + lane;      // this lane's page of the sequence
      const bool mine = lane < pages_per_tile && (first << a.log_page) < len;
      long long page = -1;
      if (mine && first < a.table_width) page = row[first];
      const bool good = mine && page >= 0 && page < a.pages;
      const unsigned have = __ballot_sync(0xffffffffu, good), want = __ballot_sync(0xffffffffu, mine);
      ok = tc_wait_warp(&aux->empty[st], phase, &aux->abort_flag);
      if (!ok) break;
      const uint32_t bytes = (uint32_t)a.block_bytes;
      if (lane == 0) {
        aux->bad[st] = want & ~have;
        if (want & ~have) atomicOr(a.flags, KV_FLAG_BAD_INDEX);
        if (have) ptx::mbar_expect_tx(&aux->full[st], bytes * __popc(have));
        else ptx::mbar_arrive(&aux->full[st]);
      }
      __syncwarp();
      if (good) {
        any = true;
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     ::"r"(ptx::smem_u32(stages + (size_t)st * C::STAGE_BYTES + (size_t)lane * bytes)),
                       "l"(a.cache + (page * a.kv_heads + head) * a.block_bytes), "r"(bytes), "r"(ptx::smem_u32(&aux->full[st]))
                     : "memory");
      }
      if (++st == C::STAGES) { st = 0; phase ^= 1u; }
    }
  } while (ok && w.next(a));
  if (!ok && __any_sync(0xffffffffu, any)) {                     // copies in flight land before the block's shared memory goes
    const long long t0 = clock64();
    while (clock64() - t0 < 4000000ll) {}
  }
}

// ---------------------------------------------------------------------------------------------- the consumer warps
template <typename C>
struct Acc {
  float o[C::NT][C::KS][4];          // O^T: 16-dimension tile x 8 rows; [0], [1] and [2], [3]: dimensions lane / 4 and + 8, rows 2 (lane & 3) and + 1
  float m[C::NT][2], l[C::NT][2];    // bound and sum (this lane's tokens only) of rows 2 (lane & 3) and + 1
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int n = 0; n < C::NT; ++n) {
#pragma unroll
      for (int t = 0; t < C::KS; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][t][i] = 0.f;
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
    }
  }
  // The factor that takes sums under bound `from` to bound `to` >= from.
  static __device__ __forceinline__ float shrink(float from, float to) { return to == -INFINITY ? 1.f : ex2(from - to); }
  __device__ __forceinline__ void rescale(int n, int j, float to) {
    const float f = shrink(m[n][j], to);
    m[n][j] = to;
    l[n][j] *= f;
#pragma unroll
    for (int t = 0; t < C::KS; ++t) {
      o[n][t][j] *= f;
      o[n][t][2 + j] *= f;
    }
  }
  // Adds a part stored by the same lane of another warp or CTA, PART values `stride` apart.
  template <bool GLOBAL>
  __device__ __forceinline__ void add(const float* p, int stride) {
    auto get = [&](int i) { return GLOBAL ? __ldcg(p + (size_t)i * stride) : p[i * stride]; };
#pragma unroll
    for (int n = 0; n < C::NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float om = get(C::ACC + n * 4 + j), ol = get(C::ACC + n * 4 + 2 + j);
        // (a bound that is not a number: neither comparison holds, the sums carry it)
        const float to = om > m[n][j] ? om : m[n][j];
        rescale(n, j, to);
        const float f = shrink(om, to);
        l[n][j] = fmaf(ol, f, l[n][j]);
#pragma unroll
        for (int t = 0; t < C::KS; ++t) {
          o[n][t][j] = fmaf(get((n * C::KS + t) * 4 + j), f, o[n][t][j]);
          o[n][t][2 + j] = fmaf(get((n * C::KS + t) * 4 + 2 + j), f, o[n][t][2 + j]);
        }
      }
  }
  template <bool GLOBAL>
  __device__ __forceinline__ void store(float* p, int stride) const {
    auto put = [&](int i, float v) {
      if (GLOBAL) __stcg(p + (size_t)i * stride, v);
      else p[i * stride] = v;
    };
#pragma unroll
    for (int n = 0; n < C::NT; ++n) {
#pragma unroll
      for (int t = 0; t < C::KS; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) put((n * C::KS + t) * 4 + i, o[n][t][i]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        put(C::ACC + n * 4 + j, m[n][j]);
        put(C::ACC + n * 4 + 2 + j, l[n][j]);
      }
    }
  }
};

// The warps' parts of a block of rows into those of wn = 0, by halves (every consumer warp comes here).
template <typename C>
__device__ __forceinline__ void attn_merge(Acc<C>& acc, float* buf, int wm, int wn, int lane) {
  if (C::WN == 1) return;
#pragma unroll 1
  for (int h = C::WN / 2; h >= 1; h >>= 1) {
    float* p = buf + ((size_t)(wm * (C::WN / 2) + (wn & (h - 1)) ) * C::PART) * 32 + lane;
    if (wn >= h && wn < 2 * h) acc.template store<false>(p, 32);
    named_sync(C::CONSUMERS);
    if (wn < h) acc.template add<false>(p, 32);
    named_sync(C::CONSUMERS);
  }
}

// Query rows of an item in the fragment order of the first product's second operand, and their masks.
template <typename C>
__device__ void attn_load_q(const AttnArgs& a, const Seq& s, int item, uint2* frag, unsigned long long* mask) {
  const int head = item % a.kv_heads, first = (item / a.kv_heads) * C::ROWS;
  const int rows = s.nodes * a.group;
  for (int i = threadIdx.x; i < C::KS * (C::ROWS / 8) * 32; i += C::CONSUMERS) {
    const int lane = i & 31, n = (i >> 5) % (C::ROWS / 8), ks = (i >> 5) / (C::ROWS / 8);
    const int r = first + n * 8 + (lane >> 2), c = lane & 3;
    uint2 v = make_uint2(0u, 0u);
    if (r < rows) {
      const int node = r / a.group;
      const __nv_bfloat16* p = a.q + (long long)(s.start + node) * a.q_t + (long long)(head * a.group + r - node * a.group) * a.q_h;
      if (C::BITS == 4) {
        v = *reinterpret_cast<const uint2*>(p + c * (C::D / 4) + ks * 4);
      } else {
        v.x = *reinterpret_cast<const uint32_t*>(p + ks * 16 + 2 * c);
        v.y = *reinterpret_cast<const uint32_t*>(p + ks * 16 + 8 + 2 * c);
      }
    }
    frag[i] = v;
  }
  for (int i = threadIdx.x; i < C::ROWS; i += C::CONSUMERS) {
    const int r = first + i;
    unsigned long long m = 0;
    if (r < rows) {
      const int node = r / a.group;
      m = a.mask ? a.mask[s.start + node] : (2ull << node) - 1ull;
      if (s.nodes < 64) m &= (1ull << s.nodes) - 1ull;
    }
    mask[i] = m;
  }
}

// 16 tokens of a stage against the warp's rows.  `token`: the first one's place in the stage; `pos`: its position in the sequence.
// EDGE: some position is not seen by some row (drafted tokens, the end of the sequence, a page that could not be read).
template <typename C, bool EDGE>
__device__ __forceinline__ void attn_tokens(const AttnArgs& a, Acc<C>& acc, uint32_t stage, int token, long long pos, const Seq& s, uint32_t bad,
                                            const uint2* frag, const unsigned long long* mask, int lane) {
  const int g = lane >> 2, c = lane & 3;
  const int page = token >> a.log_page, at = token & (a.page_size - 1);        // 16 tokens lie in one page
  const uint32_t block = stage + (uint32_t)page * (uint32_t)a.block_bytes;
  constexpr int D = C::D, KS = C::KS, NT = C::NT;
  float sc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) sc[n][i] = 0.f;

  // ---- S^T = K Q^T: rows (tokens) g and g + 8, columns (query rows) 2c and 2c + 1
  float k0 = a.scale, k1 = a.scale;
  if (C::BITS == 4) {
    const uint32_t kr = block + (uint32_t)(a.page_size * D) + (uint32_t)(at + g) * 4;
    const uint32_t r0 = lds32(kr), r1 = lds32(kr + 32);
    const uint32_t z0 = 0x43004300u | zero_of(r0) * 0x10001u, z1 = 0x43004300u | zero_of(r1) * 0x10001u;
    k0 *= step_of(r0);
    k1 *= step_of(r1);
    const uint32_t kc = block + (uint32_t)(at + g) * (D / 2) + c * (D / 8);
    uint32_t w0[D / 32], w1[D / 32];
    if (D == 128) {
      const uint4 u = lds128(kc), v = lds128(kc + 8 * (D / 2));
      w0[0] = u.x; w0[1] = u.y; w0[D / 32 - 2] = u.z; w0[D / 32 - 1] = u.w;
      w1[0] = v.x; w1[1] = v.y; w1[D / 32 - 2] = v.z; w1[D / 32 - 1] = v.w;
    } else {
      const uint2 u = lds64(kc), v = lds64(kc + 8 * (D / 2));
      w0[0] = u.x; w0[1] = u.y;
      w1[0] = v.x; w1[1] = v.y;
    }
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int sh = (k & 1) * 8;
      const uint32_t f[4] = {codes2(w0[k >> 1], sh, z0), codes2(w1[k >> 1], sh, z1), codes2(w0[k >> 1], sh + 4, z0), codes2(w1[k >> 1], sh + 4, z1)};
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uint2 q = frag[(k * (C::ROWS / 8) + n) * 32 + lane];
        mma16816(sc[n], f, q.x, q.y);
      }
    }
  } else {
    // lanes 0-7, 8-15, 16-23, 24-31 give the rows of: tokens 0-7 and 8-15 of the first 8 dimensions, then of the second
    const int t = at + (lane & 15);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      uint32_t f[4];
      const int piece = 2 * (k & 3) + (lane >> 4);
      ldmatrix4(f, block + (uint32_t)((k >> 2) * a.page_size + t) * 128 + ((piece ^ (t & 7)) << 4));
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uint2 q = frag[(k * (C::ROWS / 8) + n) * 32 + lane];
        mma16816(sc[n], f, q.x, q.y);
      }
    }
  }

  // ---- scores, bound, probabilities
  bool up = false;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v = sc[n][i] * ((i & 2) ? k1 : k0);
      if (EDGE) {
        const long long p = pos + g + ((i & 2) ? 8 : 0), j = p - s.context;
        const unsigned long long m = mask[n * 8 + 2 * c + (i & 1)];
        const bool see = (j < 0 || (j < 64 && ((m >> (j & 63)) & 1ull))) && !((bad >> page) & 1u);
        if (!see) v = -INFINITY;
      }
      sc[n][i] = v;
      up = up || v > acc.m[n][i & 1] + 8.f;
    }
  }
  if (__any_sync(0xffffffffu, up)) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float t = fmaxf(fmaxf(sc[n][j], sc[n][2 + j]), acc.m[n][j]);
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, k));
        acc.rescale(n, j, t);
      }
  }
  float v0 = 1.f, v1 = 1.f;
  uint32_t rec_v = 0;
  if (C::BITS == 4) {
    rec_v = block + (uint32_t)(a.page_size * D) + (uint32_t)(a.page_size + at) * 4;
    v0 = step_of(lds32(rec_v + g * 4));
    v1 = step_of(lds32(rec_v + g * 4 + 32));
  }
  uint32_t pf[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float m = acc.m[n][i & 1];
      p[i] = ex2(sc[n][i] - (m == -INFINITY ? 0.f : m));
      acc.l[n][i & 1] += p[i];
      if (C::BITS == 4) {
        p[i] *= (i & 2) ? v1 : v0;                            // the value's step joins its probability
        if (EDGE && sc[n][i] == -INFINITY) p[i] = 0.f;        // an unseen record may say NaN
      }
    }
    pf[n][0] = movmatrix(bf16x2(p[0], p[1]));
    pf[n][1] = movmatrix(bf16x2(p[2], p[3]));
  }

  // ---- O^T += V^T P^T
  if (C::BITS == 4) {
    // the pairs of tokens (2c, 2c + 1) and (2c + 8, 2c + 9); dimensions g * D/8 ... of each
    const uint32_t vr = rec_v + 8 * c;
    const uint2 ra = lds64(vr), rb = lds64(vr + 32);
    const uint32_t za = 0x43004300u | zero_of(ra.x) | (zero_of(ra.y) << 16), zb = 0x43004300u | zero_of(rb.x) | (zero_of(rb.y) << 16);
    const uint32_t vc = block + (uint32_t)(a.page_size * (D / 2)) + (uint32_t)(at + 2 * c) * (D / 2) + g * (D / 16);
    uint32_t w[4][D / 64];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t p = vc + ((i & 1) + (i >> 1) * 8) * (D / 2);
      if (D == 128) {
        const uint2 u = lds64(p);
        w[i][0] = u.x;
        w[i][D / 64 - 1] = u.y;
      } else {
        w[i][0] = lds32(p);
      }
    }
#pragma unroll
    for (int h = 0; h < D / 64; ++h) {
      // low halves: elements 0, 2, 4, 6 of the word's eight; high halves: 1, 3, 5, 7
      const uint32_t al = __byte_perm(w[0][h], w[1][h], 0x5410), ah = __byte_perm(w[0][h], w[1][h], 0x7632);
      const uint32_t bl = __byte_perm(w[2][h], w[3][h], 0x5410), bh = __byte_perm(w[2][h], w[3][h], 0x7632);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t f[4] = {codes2(al, 4 * e, za), codes2(ah, 4 * e, za), codes2(bl, 4 * e, zb), codes2(bh, 4 * e, zb)};
#pragma unroll
        for (int n = 0; n < NT; ++n) mma16816(acc.o[n][h * 4 + e], f, pf[n][0], pf[n][1]);
      }
    }
  } else {
    const uint32_t vb = block + (uint32_t)(a.page_size * D * 2);
    const int t = at + (lane & 7) + ((lane >> 4) << 3);       // lanes 0-7, 8-15: tokens 0-7 of the first and second 8 dimensions; 16-31: tokens 8-15
    uint32_t odd = 0;                                         // tokens some of whose values are not finite
    if (EDGE) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t q = lds32(vb + (uint32_t)(at + i) * 128 + lane * 4);
        const uint32_t q2 = D == 128 ? lds32(vb + (uint32_t)(a.page_size + at + i) * 128 + lane * 4) : 0u;
        const bool nf = (q & 0x7F80u) == 0x7F80u || (q & 0x7F800000u) == 0x7F800000u || (q2 & 0x7F80u) == 0x7F80u || (q2 & 0x7F800000u) == 0x7F800000u;
        if (__any_sync(0xffffffffu, nf)) odd |= 1u << i;
      }
    }
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      uint32_t f[4];
      const int piece = 2 * (k & 3) + ((lane >> 3) & 1);
      ldmatrix4t(f, vb + (uint32_t)((k >> 2) * a.page_size + t) * 128 + ((piece ^ (t & 7)) << 4));
      if (EDGE && odd) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if ((f[i] & 0x7F80u) == 0x7F80u) f[i] &= 0xFFFF0000u;
          if ((f[i] & 0x7F800000u) == 0x7F800000u) f[i] &= 0x0000FFFFu;
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) mma16816(acc.o[n][k], f, pf[n][0], pf[n][1]);
    }
    if (EDGE && odd) {
      // what was left out above, for the rows that see the token: the product of a probability and a value that is not finite
#pragma unroll 1
      for (int i = 0; i < 16; ++i) {
        if (!((odd >> i) & 1u)) continue;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float mine = (i & 8) ? sc[n][2 + j] : sc[n][j];
            const float v = __shfl_sync(0xffffffffu, mine, (i & 7) * 4 + c);
            const float m = acc.m[n][j];
            if (v == -INFINITY) continue;
            const float p = ex2(v - (m == -INFINITY ? 0.f : m));
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int e = k * 16 + g + 8 * h, tt = at + i;
                const uint32_t q = lds32(vb + (uint32_t)((e >> 6) * a.page_size + tt) * 128 + (((((e & 63) >> 3) ^ (tt & 7)) << 4) | ((e & 6) << 1)));
                const float x = (e & 1) ? __uint_as_float(q & 0xFFFF0000u) : __uint_as_float(q << 16);
                if (!(fabsf(x) <= 3.4028234663852886e38f)) acc.o[n][k][2 * h + j] += p * x;
              }
          }
      }
    }
  }
}

// Rows of an item that is complete: normalised, rounded, written.
template <typename C>
__device__ void attn_write(const AttnArgs& a, Acc<C>& acc, const Seq& s, int item, int wm, int lane) {
  const int g = lane >> 2, c = lane & 3;
  const int head = item % a.kv_heads, first = (item / a.kv_heads) * C::ROWS + wm * 8 * C::NT;
  const int rows = s.nodes * a.group;
#pragma unroll
  for (int n = 0; n < C::NT; ++n)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float l = acc.l[n][j];
#pragma unroll
      for (int k = 4; k < 32; k <<= 1) l += __shfl_xor_sync(0xffffffffu, l, k);
      const int r = first + n * 8 + 2 * c + j;
      if (r >= rows) continue;
      const bool none = acc.m[n][j] == -INFINITY && l == 0.f;         // nothing seen
      const float inv = none ? 0.f : 1.f / l;
      const int node = r / a.group, h = head * a.group + r - node * a.group;
      const long long row = s.start + node;
      __nv_bfloat16* o = a.out + row * a.o_t + h * a.o_h;
      if (C::BITS == 4) {
        // dimensions g * D/8 + 2t and + 1 of tile t
        uint32_t v[C::KS];
#pragma unroll
        for (int t = 0; t < C::KS; ++t) v[t] = bf16x2(acc.o[n][t][j] * inv, acc.o[n][t][2 + j] * inv);
        uint4* p = reinterpret_cast<uint4*>(o + g * (C::D / 8));
#pragma unroll
        for (int t = 0; t < C::KS / 4; ++t) p[t] = make_uint4(v[4 * t], v[4 * t + 1], v[4 * t + 2], v[4 * t + 3]);
      } else {
#pragma unroll
        for (int t = 0; t < C::KS; ++t) {
          o[t * 16 + g] = __float2bfloat16_rn(acc.o[n][t][j] * inv);
          o[t * 16 + g + 8] = __float2bfloat16_rn(acc.o[n][t][2 + j] * inv);
        }
      }
      if (a.lse && g == 0) a.lse[row * a.lse_t + h] = none ? -INFINITY : (acc.m[n][j] == -INFINITY ? 0.f : acc.m[n][j]) * 0.6931471805599453f + logf(l);
    }
}

template <typename C>
__global__ void __launch_bounds__(C::THREADS, C::MINB) attn_kernel(const AttnArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t* stages = smem;
  uint2* frag = reinterpret_cast<uint2*>(smem + C::STAGES * C::STAGE_BYTES);
  float* merge = reinterpret_cast<float*>(smem + C::STAGES * C::STAGE_BYTES + C::QFRAG_BYTES);
  unsigned long long* mask = reinterpret_cast<unsigned long long*>(smem + C::STAGES * C::STAGE_BYTES + C::QFRAG_BYTES + C::MERGE_BYTES);
  AttnAux* aux = reinterpret_cast<AttnAux*>(smem + C::SMEM - C::AUX_BYTES);
  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::STAGES; ++i) {
      ptx::mbar_init(&aux->full[i], 1);
      ptx::mbar_init(&aux->empty[i], C::WARPS);
    }
    aux->abort_flag = 0;
    ptx::fence_barrier_init();
    ptx::fence_proxy_async();
  }
  __syncthreads();
  if (warp == C::WARPS) {
    attn_produce<C>(a, stages, aux);
    return;
  }
  const int wm = warp / C::WN, wn = warp % C::WN;
  Walk<C> w;
  w.begin(a);
  if (w.left <= 0) return;
  bool dead = false, head_of_run = true;
  int st = 0;
  uint32_t phase = 0;
  Acc<C> acc;
  do {
    attn_load_q<C>(a, w.s, w.item, frag, mask);
    acc.clear();
    named_sync(C::CONSUMERS);
    const long long len = (long long)w.s.context + w.s.nodes;
    for (int tile = w.tile; tile < w.end; ++tile) {
      if (!dead) dead = !tc_wait_warp(&aux->full[st], phase, &aux->abort_flag);
      if (!dead) {
        const uint32_t stage = ptx::smem_u32(stages + (size_t)st * C::STAGE_BYTES);
        const uint32_t bad = *reinterpret_cast<volatile uint32_t*>(&aux->bad[st]);
        const long long pos0 = (long long)tile * C::TILE;
#pragma unroll 1
        for (int sub = 0; sub < C::SUBS; ++sub) {
          const int token = (sub * C::WN + wn) * 16;
          const long long pos = pos0 + token;
          if (pos >= len) break;
          if (pos + 16 <= w.s.context && bad == 0) attn_tokens<C, false>(a, acc, stage, token, pos, w.s, bad, frag + wm * C::NT * 32, mask + wm * C::NT * 8, lane);
          else attn_tokens<C, true>(a, acc, stage, token, pos, w.s, bad, frag + wm * C::NT * 32, mask + wm * C::NT * 8, lane);
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&aux->empty[st]);
      }
      if (++st == C::STAGES) { st = 0; phase ^= 1u; }
    }
    attn_merge<C>(acc, merge, wm, wn, lane);
    if (*reinterpret_cast<volatile int*>(&aux->abort_flag)) dead = true;      // some warp's tokens are missing
    const bool whole = w.tile == 0 && w.end == w.s.tiles;
    if (whole) {
      if (wn == 0 && !dead) attn_write<C>(a, acc, w.s, w.item, wm, lane);
    } else {
      // this CTA's part; its first one of the run goes to its first slot
      constexpr size_t SLOT = (size_t)C::PART * 32 * C::WM;
      if (wn == 0 && !dead) {
        acc.template store<true>(a.parts + (2 * (size_t)blockIdx.x + (head_of_run ? 0 : 1)) * SLOT + (size_t)wm * C::PART * 32 + lane, 32);
        __threadfence();
      }
      const int c0 = w.owner(w.item_at), c1 = w.owner(w.item_at + w.s.tiles - 1);
      named_sync(C::CONSUMERS);
      if (threadIdx.x == 0) {
        const unsigned n = (unsigned)(c1 - c0);
        aux->last = !aux->abort_flag && atomicInc(a.counters + c0, n) == n;
        __threadfence();
      }
      named_sync(C::CONSUMERS);
      if (aux->last) {
        acc.clear();
        for (int k = c0 + wn; k <= c1; k += C::WN) {
          // the part of CTA k: its run begins with it unless the item began inside the run
          acc.template add<true>(a.parts + (2 * (size_t)k + (w.run_begin(k) < w.item_at ? 1 : 0)) * SLOT + (size_t)wm * C::PART * 32 + lane, 32);
        }
        attn_merge<C>(acc, merge, wm, wn, lane);
        if (wn == 0 && !dead) attn_write<C>(a, acc, w.s, w.item, wm, lane);
      }
    }
    head_of_run = false;
    named_sync(C::CONSUMERS);                                  // the fragments may be replaced
  } while (w.next(a));
  if (dead && lane == 0) atomicOr(a.flags, KV_FLAG_TIMEOUT);
}

}  // namespace kv
}  // namespace conqur
