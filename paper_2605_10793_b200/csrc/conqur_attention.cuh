// Attention of a few query rows per sequence (one drafted token or a tree of them, times the query heads that share a key head)
// over a paged cache of keys and values, 4-bit codes or bf16.
//
//   s_l = scale q . k_l,  o = sum_l 2^(s_l log2 e - m) v_l / sum_l 2^(s_l log2 e - m),  m a running bound of the row's scores
//
// This file: at most 16 rows a key head.  The cache is read once, so memory sets the pace; over 4-bit codes the unpacking of a byte into two operands comes
// close to it.  Measured on one row of 8 key heads of 4 query heads each, 64 sequences of 8192: bf16 325 us (6.6 TB/s, a copy's rate), 4 bits 123 us (4.6 TB/s:
// about 1.1 instructions a code, 2.15 of 4 a cycle and the ALU 57 % busy: 16 warps an SM whose chains of score, exponential and product, and ends of items, do
// not overlap any further); one sequence of 200: 9 us, of which 3 are a launch.
//   - The tokens, not the rows, are the 16-row side of the warps' products (m16n8k16): S^T = K Q^T and O^T = V^T P^T.  Eight
//     rows fill an instruction, and a fragment of K or V that was unpacked from codes is used for all rows of the warp.  The codes go from shared memory to the
//     fragments in registers, in an order of dimensions (and of output dimensions) that lets every lane read whole words of a token's row;
//     a product does not depend on the order of what it sums over.
//   - P is rounded to bf16, the values' type, which is what the products take: 2^-8 of a probability at most, either way, so that an output is off by 1.9 to
//     2.4e-3 of itself (root mean square) where rounding it alone makes 1.6 to 1.7e-3.
//   - P^T goes from the accumulator layout of the first product to the operand layout of the second with movmatrix, two per eight rows.
//   - The running maximum is only a bound: rows are rescaled when a score exceeds it by 2^8, one vote per 32 tokens instead of a
//     reduction (P is rounded relatively, a common factor changes nothing).  It starts at the lowest finite number, not at -inf: a token whose score is
//     -inf then has the weight 0 that it is due also where no other has been met.
//   - The work, in tiles of tokens of one sequence, key head and block of rows, is laid end to end and cut into equal runs, one per
//     resident CTA, whatever the lengths (Walk has the exception for few items).  A piece of work that is cut leaves its parts (accumulators, maximum, sum) in the workspace; the
//     last CTA to finish one of its parts adds them up in their order.  No CTA waits for another.
//   - A warp takes groups of 32 tokens of its own and brings them with asynchronous 16-byte copies into a ring of its own: no warp waits for another
//     but the one that adds up an item's parts: the warps take turns at that, the others go on with the next item.
#pragma once
#include <cuda_bf16.h>

#include "../../include/conqur.h"
#include "conqur_ptx.cuh"

namespace conqur {
namespace kv {

struct AttnArgs {
  const uint8_t* cache;
  int pages, page_size, log_page, kv_heads, group, max_nodes, batch, table_width;
  long long block_bytes, page_bytes, rows;   // of a page of one head, of all heads
  int codes_bytes, plane_bytes;      // of a page's codes of one kind; of a plane
  float scale;                       // times log2 e
  const __nv_bfloat16* q; long long q_t, q_h;
  __nv_bfloat16* out; long long o_t, o_h;
  float* lse; long long lse_t;
  const int* starts; const int* contexts; const int* table; long long table_stride;
  const unsigned long long* mask;
  unsigned* counters;                // one per CTA, for the item that its run ends in the middle of: parts finished, wraps to 0
  float* parts;                      // two slots per CTA
  int* flags;
  // conqur_attention_tc.cuh, test support: the barrier of one CTA that expects one arrival more than it gets, a CONQUR_TREE_WAIT_* and its number
  int lose_block, lose_site, lose_index;
};

enum { KV_FLAG_BAD_INDEX = 1, KV_FLAG_TIMEOUT = 2 };

constexpr int ATTN_UNIT = 64;                                    // tokens: what the work is counted and cut in, a multiple of the largest page

constexpr int ATTN_CHUNK = 32;                                   // tokens a warp takes at a time: each half lies in one page

// BITS of the cache, D; a block works on 8 NT query rows with WN warps, each with a ring of STAGES chunks.  MIN_RUN: tiles a CTA takes at least, one for each pair
// of its warps (one sequence of 200 over 4 bits: with 1 11.2 us, with 4 8.7; eight are better for some short batches, worse by as much for others).
template <int BITS_, int D_, int NT_, int WN_, int STAGES_, int PER_SM_>
struct AttnCfg {
  static constexpr int BITS = BITS_, D = D_, NT = NT_, WN = WN_, STAGES = STAGES_, PER_SM = PER_SM_;
  static constexpr int MIN_RUN = 4;
  static constexpr int THREADS = 32 * WN;
  static constexpr int ROWS = 8 * NT;                            // query rows of a block
  static constexpr int STAGE_BYTES = ATTN_CHUNK * (BITS == 4 ? D + 8 : 4 * D);
  static constexpr int KS = D / 16;                              // k steps of the first product, 16-dimension tiles of the second
  static constexpr int ACC = NT * KS * 4;                        // accumulators a lane
  static constexpr int PART = ACC + 6 * NT;                      // and its maxima, sums and sums of p z
  static constexpr int MERGE_BYTES = (WN - 1) * PART * 32 * 4;
  static constexpr int AUX_BYTES = 1024;
  static constexpr int SMEM = WN * STAGES * STAGE_BYTES + MERGE_BYTES + AUX_BYTES;
  static_assert((SMEM + 1024) * PER_SM <= 228 * 1024, "shared memory of an SM");
  static_assert(NT <= 2, "the rows' fragments and sums stay in registers");
  static_assert(STAGES <= 16 && (WN & (WN - 1)) == 0, "two bits for every stage; the warps' parts are added in halves");
};

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
__device__ __forceinline__ void bar_sync(int bar, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int bar, int threads) { asm volatile("bar.arrive %0, %1;" ::"r"(bar), "r"(threads) : "memory"); }
enum { BAR_ALL = 1, BAR_STORED = 2, BAR_ADDED = 3 };      // BAR_ADDED and the one behind it, in turn
// Codes enter the products as they lie: a bf16 whose upper byte is 0 is its lower byte times 2^-133, below and above the smallest
// normal number alike, and the products take such numbers exactly.  So the nibbles at bits 0 and 4 of both halves, masked where they are, are c 2^-133 and
// 16 c 2^-133; one mask a pair is all the unpacking.  The other operand carries 2^96 (rows) or 2^90 (probabilities), the rows also the 1/16 of their
// dimensions in odd nibbles, and the sums come back with 2^37 or 2^43.  Zero-points come off the sums: q . (c - z) = q . c - z sum q, and for the values
// one more tile of the product holds sum p z.
constexpr float ATTN_Q_UP = 7.922816251426434e28f, ATTN_Q_BACK = 1.37438953472e11f;        // 2^96, 2^(133 - 96)
constexpr float ATTN_P_UP = 1.2379400392853803e27f, ATTN_P_BACK = 8.796093022208e12f;      // 2^90, 2^(133 - 90)
__device__ __forceinline__ uint32_t codes_even(uint32_t w) { return w & 0x000F000Fu; }
__device__ __forceinline__ uint32_t codes_odd(uint32_t w) { return w & 0x00F000F0u; }
__device__ __forceinline__ float step_of(uint32_t rec) { return __uint_as_float(rec << 16); }
__device__ __forceinline__ uint32_t zero_of(uint32_t rec) { return (rec >> 16) & 15u; }
__device__ __forceinline__ float zero_float(uint32_t rec) { return __uint_as_float(zero_of(rec) | 0x4B000000u) - 8388608.f; }
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

constexpr float ATTN_NO_BOUND = -3.4028234663852886e38f;       // before the first score

// The drafted tokens and context of a sequence, and what its work comes to.
struct Seq {
  int start, nodes, context;
  int tiles, blocks;                 // units of tokens, blocks of rows
};
// over (where asked for): set if the sequence has more than max_nodes tokens.
template <typename C>
__device__ __forceinline__ Seq sequence(const AttnArgs& a, int b, bool* over = nullptr) {
  Seq s;
  const long long s0 = a.starts[b], s1 = a.starts[b + 1];
  long long n = s1 - s0;
  int c = a.contexts[b];
  bool bad = false;
  if (s0 < 0 || n < 0 || s1 > a.rows) { n = 0; bad = true; }
  if (n > a.max_nodes) {
    n = a.max_nodes;
    bad = true;
    if (over) *over = true;
  }
  if (c < 0) { c = 0; bad = true; }
  if (c > 0x7fff0000) { c = 0x7fff0000; bad = true; }       // positions stay below 2^31
  // Positions that have no place in the table are not seen: no work for them, whatever the context says (one tile for rows that see nothing).
  const long long reach = (long long)a.table_width << a.log_page;
  if (n > 0 && c + n > reach) bad = true;
  if (bad && blockIdx.x == 0 && threadIdx.x < 32) atomicOr(a.flags, KV_FLAG_BAD_INDEX);
  s.start = (int)s0;
  s.nodes = (int)n;
  s.context = c;
  s.tiles = n > 0 ? max(1, (int)((min(c + n, reach) + ATTN_UNIT - 1) / ATTN_UNIT)) : 0;
  s.blocks = (int)((n * a.group + C::ROWS - 1) / C::ROWS);
  return s;
}

// Tokens behind the first max_nodes of their sequence get NaN, by one warp of every CTA (rare: the call was given too small a max_nodes).
template <typename C>
__device__ void blank_rows(const AttnArgs& a) {
  const int lane = threadIdx.x & 31, heads = a.kv_heads * a.group;
  const uint4 nan = make_uint4(0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u);
  for (int b = 0; b < a.batch; ++b) {
    const long long s0 = a.starts[b], s1 = a.starts[b + 1];
    if (s0 < 0 || s1 > a.rows) continue;
    for (long long row = s0 + a.max_nodes + blockIdx.x; row < s1; row += gridDim.x)
      for (int h = 0; h < heads; ++h) {
        if (lane < C::D / 8) *reinterpret_cast<uint4*>(a.out + row * a.o_t + h * a.o_h + 8 * lane) = nan;
        if (a.lse && lane == 0) a.lse[row * a.lse_t + h] = __uint_as_float(0x7FC00000u);
      }
  }
}

// A CTA's run of tiles, item after item; an item is one (sequence, block of rows, key head).
template <typename C>
struct Walk {
  long long left, total, at;         // tiles of the run still to come; places of all work; the next tile's place
  int ctas;                          // CTAs with a run: none is empty
  Seq s;
  int b, item, tile;                 // the item's sequence, its number there (block of rows * kv_heads + key head), and its next tile
  int end;                           // the run's last tile of the item, plus one
  long long item_at;                 // place of the item's first tile

  int pad;                           // 1, or the length of the runs, of which each item takes a whole number of places

  __device__ int places(int tiles) const { return pad == 1 ? tiles : (int)((unsigned)(tiles + pad - 1) / (unsigned)pad) * pad; }
  // One warp: a sum over the sequences, then the one in which the run begins.
  __device__ void begin(const AttnArgs& a) {
    const int lane = threadIdx.x & 31;
    total = 0;
    long long items = 0;
    Seq own = {};                                              // of the first 32 sequences: read once
    bool over = false;
    if (lane < a.batch) own = sequence<C>(a, lane, &over);
    for (int i = lane; i < a.batch; i += 32) {
      const Seq q = i < 32 ? own : sequence<C>(a, i, &over);
      total += (long long)q.tiles * q.blocks * a.kv_heads;
      items += q.tiles ? (long long)q.blocks * a.kv_heads : 0;
    }
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) {
      total += __shfl_xor_sync(0xffffffffu, total, m);
      items += __shfl_xor_sync(0xffffffffu, items, m);
    }
    if (__any_sync(0xffffffffu, over)) blank_rows<C>(a);
    const int grid = (int)gridDim.x;
    ctas = (int)min((long long)grid, (total + C::MIN_RUN - 1) / C::MIN_RUN);
    pad = 1;
    if (items > 0 && items <= grid) {
      // Runs that end with their item, if the grid has enough for it with up to four tiles more each than it would take otherwise: a run over two items
      // costs its CTA about 6 us, four tiles 2; and no item is cut that needs no cutting.  (One sequence of 8192, 8 key heads: 22.5 to 16.0 us over 4 bits, 22.7 to 17.4 over bf16.)
      constexpr int TRY = 2;
      const int run = max(C::MIN_RUN, (int)ratio(total + grid - 1, grid));
      int pieces[TRY] = {};
      for (int i = lane; i < a.batch; i += 32) {
        const Seq q = i < 32 ? own : sequence<C>(a, i);
#pragma unroll
        for (int j = 0; j < TRY; ++j) pieces[j] += min((int)((unsigned)(q.tiles + run + 4 * j - 1) / (unsigned)(run + 4 * j)) * q.blocks * a.kv_heads, grid + 1);
      }
#pragma unroll
      for (int j = TRY - 1; j >= 0; --j) {
        const int n = __reduce_add_sync(0xffffffffu, min(pieces[j], grid + 1));
        if (n > grid) continue;
        pad = run + 4 * j;
        ctas = n;
      }
      if (pad > 1) total = (long long)ctas * pad;
    }
    b = 0;
    left = 0;
    if ((int)blockIdx.x >= ctas) return;
    at = run_begin(blockIdx.x);
    left = run_begin(blockIdx.x + 1) - at;
    long long before = 0;
    for (int base = 0; base < a.batch; base += 32) {
      long long mine = 0;
      if (base + lane < a.batch) {
        const Seq q = base == 0 ? own : sequence<C>(a, base + lane);
        mine = (long long)places(q.tiles) * q.blocks * a.kv_heads;
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
    if (b < 32) {
      s.start = __shfl_sync(0xffffffffu, own.start, b);
      s.nodes = __shfl_sync(0xffffffffu, own.nodes, b);
      s.context = __shfl_sync(0xffffffffu, own.context, b);
      s.tiles = __shfl_sync(0xffffffffu, own.tiles, b);
      s.blocks = __shfl_sync(0xffffffffu, own.blocks, b);
    } else {
      s = sequence<C>(a, b);
    }
    const long long in_seq = at - before;
    item = (int)ratio(in_seq, places(s.tiles));
    tile = (int)(in_seq - (long long)item * places(s.tiles));
    item_at = at - tile;
    if (pad > 1) left = min(left, (long long)(s.tiles - tile));
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
  __device__ int owner(long long t) const { return (int)(pad > 1 ? ratio(t, pad) : ratio((t + 1) * ctas - 1, total)); }
  __device__ long long run_begin(int cta) const { return pad > 1 ? (long long)pad * cta : ratio(total * cta, ctas); }
  // (64-bit divisions cost several times those of 32 bits: a few of them were 1 us of a call)
  static __device__ long long ratio(long long x, long long y) {
    return (((unsigned long long)x | (unsigned long long)y) >> 32) == 0 ? (long long)((unsigned)x / (unsigned)y) : x / y;
  }
};

// ---------------------------------------------------------------------------------------------- copies
template <typename C>
struct AttnAux {
  Walk<C> ahead[C::WN];              // per warp: the item whose chunks are fetched (the one that is worked on, or a later one)
  // cut items of which this CTA finished the last part (at most the first and the last of its run): added up when the run is done
  struct { Seq s; int item, c0, c1; long long item_at; } todo[2];
  int todos;
};

// `bytes`: 16, or 0: nothing is read and zeros are stored.
__device__ __forceinline__ void copy16(uint32_t to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}

// A warp's chunks, fetched in the order in which they are worked on, up to STAGES ahead.  A stage holds, of 32 tokens: key codes, value codes, key and
// value records; or the planes of the keys, then of the values.
template <typename C>
struct Fetch {
  const int* table;                  // the sequence's row
  const uint8_t* head;               // the key head's block of page 0
  uint32_t ring;
  int token, end;                    // the warp's next chunk; end of the item's tokens in this run
  int page[2];                       // the cache's pages of that chunk's halves, asked for one chunk ahead
  uint32_t bad;                      // two bits a stage: halves that could not be read
  int stage;
  bool more;

  __device__ __forceinline__ void begin(const AttnArgs& a, const Walk<C>& w, uint8_t* smem_ring, Walk<C>* ahead, int wn, int lane) {
    ring = ptx::smem_u32(smem_ring);
    bad = 0;
    stage = 0;
    more = true;
    if (lane == 0) *ahead = w;
    __syncwarp();
    item(a, w, wn);
    if (token >= end) settle(a, ahead, wn, lane);
    ask(a);
  }
  __device__ __forceinline__ void item(const AttnArgs& a, const Walk<C>& w, int wn) {
    table = a.table + (long long)w.b * a.table_stride;
    head = a.cache + (long long)(w.item % a.kv_heads) * a.block_bytes;
    token = w.tile * ATTN_UNIT + wn * ATTN_CHUNK;
    end = min(w.end * ATTN_UNIT, w.s.context + w.s.nodes);
  }
  // To the next item that has a chunk for this warp.
  __device__ __forceinline__ void settle(const AttnArgs& a, Walk<C>* ahead, int wn, int lane) {
    Walk<C> w = *ahead;
    while (more && token >= end) {
      more = w.next(a);
      if (more) item(a, w, wn);
    }
    if (!more) token = end = 0;
    __syncwarp();
    if (lane == 0) *ahead = w;
    __syncwarp();
  }
  __device__ __forceinline__ void ask(const AttnArgs& a) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = token + 16 * i;
      page[i] = -1;
      if (t < end && (t >> a.log_page) < a.table_width) page[i] = table[t >> a.log_page];
    }
  }
  __device__ __forceinline__ void issue(const AttnArgs& a, Walk<C>* ahead, int wn, int lane) {
    const uint8_t* block[2];
    int at[2], bytes[2];
    bad &= ~(3u << (2 * stage));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool good = (unsigned)page[i] < (unsigned)a.pages; // (behind the item's end: -1)
      bytes[i] = good ? 16 : 0;
      bad |= (good ? 0u : 1u) << (2 * stage + i);
      at[i] = (token + 16 * i) & (a.page_size - 1);
      block[i] = head + (good ? (long long)page[i] * a.page_bytes : 0);
    }
    const uint32_t to = ring + stage * C::STAGE_BYTES + lane * 16;
    if (C::BITS == 4) {
      constexpr int CODES = 16 * C::D / 2;                     // bytes of 16 tokens: 512 or 1024
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint8_t* p = block[i] + at[i] * (C::D / 2) + lane * 16;
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int j = 0; j < CODES / 512; ++j) copy16(to + (2 * part + i) * CODES + j * 512, p + part * a.codes_bytes + j * 512, bytes[i]);
      }
      // records of 16 tokens are 64 bytes: lanes 0-3 and 4-7 the keys' of the two halves, 8-11 and 12-15 the values'
      const int i = (lane >> 2) & 1;
      if (lane < 16) copy16(to + 4 * CODES, (i ? block[1] : block[0]) + 2 * a.codes_bytes + ((i ? at[1] : at[0]) + (lane >> 3) * a.page_size) * 4 + (lane & 3) * 16, i ? bytes[1] : bytes[0]);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint8_t* p = block[i] + at[i] * 128 + lane * 16;
#pragma unroll
        for (int part = 0; part < C::D / 32; ++part)
#pragma unroll
          for (int j = 0; j < 4; ++j) copy16(to + (2 * part + i) * 2048 + j * 512, p + part * a.plane_bytes + j * 512, bytes[i]);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");       // one group a chunk, of zeros at the end of the run
    stage = stage + 1 == C::STAGES ? 0 : stage + 1;
    if (more) token += C::WN * ATTN_CHUNK;
    if (token >= end && more) settle(a, ahead, wn, lane);
    ask(a);
  }
};

// ---------------------------------------------------------------------------------------------- the consumer warps
template <typename C>
struct Acc {
  float o[C::NT][C::KS][4];          // O^T: 16-dimension tile x 8 rows; [0], [1] and [2], [3]: dimensions lane / 4 and + 8, rows 2 (lane & 3) and + 1
  float m[C::NT][2], l[C::NT][2];    // bound and sum (this lane's tokens only) of rows 2 (lane & 3) and + 1
  float z[C::NT][4];                 // sum p z, 4 bits: [0] and [1] of rows 2 (lane & 3) and + 1
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int n = 0; n < C::NT; ++n) {
#pragma unroll
      for (int t = 0; t < C::KS; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][t][i] = 0.f;
      m[n][0] = m[n][1] = ATTN_NO_BOUND;
      l[n][0] = l[n][1] = 0.f;
      z[n][0] = z[n][1] = z[n][2] = z[n][3] = 0.f;
    }
  }
  // The factor that takes sums under bound `from` to bound `to` >= from.
  static __device__ __forceinline__ float shrink(float from, float to) { return ex2(from - to); }
  __device__ __forceinline__ void rescale(int n, int j, float to) {
    const float f = shrink(m[n][j], to);
    m[n][j] = to;
    l[n][j] *= f;
    z[n][j] *= f;
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
        const float om = get(C::ACC + n * 6 + j), ol = get(C::ACC + n * 6 + 2 + j), oz = C::BITS == 4 ? get(C::ACC + n * 6 + 4 + j) : 0.f;
        const float to = om > m[n][j] ? om : m[n][j];
        rescale(n, j, to);
        const float f = shrink(om, to);
        l[n][j] = fmaf(ol, f, l[n][j]);
        z[n][j] = fmaf(oz, f, z[n][j]);
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
        put(C::ACC + n * 6 + j, m[n][j]);
        put(C::ACC + n * 6 + 2 + j, l[n][j]);
        if (C::BITS == 4) put(C::ACC + n * 6 + 4 + j, z[n][j]);
      }
    }
  }
};

// The parts of `warps` warps, by halves, into those of the first (every warp of the CTA comes here).
template <typename C>
__device__ __forceinline__ void attn_merge(Acc<C>& acc, float* buf, int me, int warps, int lane) {
#pragma unroll 1
  for (int h = warps / 2; h >= 1; h >>= 1) {
    float* p = buf + (size_t)(me & (h - 1)) * C::PART * 32 + lane;
    if (me >= h && me < 2 * h) acc.template store<false>(p, 32);
    bar_sync(BAR_ALL, C::THREADS);
    if (me < h) acc.template add<false>(p, 32);
    bar_sync(BAR_ALL, C::THREADS);
  }
}

// The query rows of an item as a lane meets them in the first product's second operand: row g = lane / 4 of each eight, a quarter of its dimensions.
template <typename C>
struct Query {
  const __nv_bfloat16* p[C::NT];     // NULL: no such row
  uint2 f[C::KS][C::NT];
  float sum[C::NT][2];               // 4 bits: sums of rows 2 (lane & 3) and + 1, in the units of the products
  int first, rows;                   // the block's first row; rows of the sequence

  __device__ __forceinline__ uint2 load(int k, int n, int c) const {
    uint2 v = make_uint2(0u, 0u);
    if (p[n]) {
      if (C::BITS == 4) {
        v = *reinterpret_cast<const uint2*>(p[n] + c * (C::D / 4) + k * 4);
      } else {
        v.x = *reinterpret_cast<const uint32_t*>(p[n] + k * 16 + 2 * c);
        v.y = *reinterpret_cast<const uint32_t*>(p[n] + k * 16 + 8 + 2 * c);
      }
    }
    return v;
  }
  static __device__ __forceinline__ uint2 scaled(uint2 v) {
    // even nibbles meet the first two of four dimensions with 2^96, odd ones the others with 2^92
    return C::BITS == 4 ? make_uint2(mul2(v.x, 0x6F806F80u), mul2(v.y, 0x6D806D80u)) : v;
  }
  __device__ __forceinline__ void begin(const AttnArgs& a, const Seq& s, int item, int lane) {
    const int g = lane >> 2, c = lane & 3;
    const int head = item % a.kv_heads;
    first = (item / a.kv_heads) * C::ROWS;
    rows = s.nodes * a.group;
#pragma unroll
    for (int n = 0; n < C::NT; ++n) {
      const int r = first + n * 8 + g, node = r / a.group;
      p[n] = r < rows ? a.q + (long long)(s.start + node) * a.q_t + (long long)(head * a.group + r - node * a.group) * a.q_h : nullptr;
    }
#pragma unroll
    for (int n = 0; n < C::NT; ++n) {
      float part = 0.f;
#pragma unroll
      for (int k = 0; k < C::KS; ++k) {
        const uint2 v = load(k, n, c);
        if (C::BITS == 4) {
          const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v.x)), y = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v.y));
          part += (x.x + x.y) + (y.x + y.y);
        }
        f[k][n] = scaled(v);
      }
      if (C::BITS == 4) {
        part += __shfl_xor_sync(0xffffffffu, part, 1);
        part += __shfl_xor_sync(0xffffffffu, part, 2);
        sum[n][0] = __shfl_sync(0xffffffffu, part, 8 * c) * (1.f / ATTN_Q_BACK);
        sum[n][1] = __shfl_sync(0xffffffffu, part, 8 * c + 4) * (1.f / ATTN_Q_BACK);
      }
    }
  }
  // The drafted tokens that row n * 8 + 2 (lane & 3) + j sees.
  __device__ __forceinline__ unsigned long long mask(const AttnArgs& a, const Seq& s, int n, int j, int c) const {
    const int r = first + n * 8 + 2 * c + j;
    if (r >= rows) return 0ull;
    const int node = r / a.group;
    unsigned long long m = a.mask ? a.mask[s.start + node] : (2ull << node) - 1ull;
    if (s.nodes < 64) m &= (1ull << s.nodes) - 1ull;
    return m;
  }
};

// A chunk of twice 16 tokens against the rows.  `pos`: the first one's position in the sequence; `bad`: halves that could not be read.
// EDGE: some position is not seen by some row (drafted tokens, the end of the sequence, a page that could not be read).  Both halves go through
// each stage of the computation together: what one waits for (products, exponentials) the other fills.
template <typename C, bool EDGE>
__device__ __forceinline__ void attn_tokens(const AttnArgs& a, Acc<C>& acc, uint32_t stage, int pos, const Seq& s, uint32_t bad,
                                            const Query<C>& query, int lane) {
  constexpr int H = 2;
  const int g = lane >> 2, c = lane & 3;
  constexpr int D = C::D, KS = C::KS, NT = C::NT, CT = ATTN_CHUNK;
  float sc[H][NT][4], ks[H][2];

  // ---- S^T = K Q^T: rows (tokens) g and g + 8, columns (query rows) 2c and 2c + 1
#pragma unroll
  for (int u = 0; u < H; ++u) {
    const int au = 16 * u;
    float sd[NT][4];                   // (the k steps alternate between two sums: a product that waits for the one before it takes several times its issue)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[u][n][i] = sd[n][i] = 0.f;
    ks[u][0] = ks[u][1] = a.scale;
    if (C::BITS == 4) {
      const uint32_t kr = stage + CT * D + au * 4 + g * 4;
      const uint32_t r0 = lds32(kr), r1 = lds32(kr + 32);
      const uint32_t kc = stage + au * (D / 2) + lane * (D / 8);         // token g, the c-th quarter of its row
      uint32_t w0[D / 32], w1[D / 32];
      if (D == 128) {
        const uint4 x = lds128(kc), y = lds128(kc + 8 * (D / 2));
        w0[0] = x.x; w0[1] = x.y; w0[D / 32 - 2] = x.z; w0[D / 32 - 1] = x.w;
        w1[0] = y.x; w1[1] = y.y; w1[D / 32 - 2] = y.z; w1[D / 32 - 1] = y.w;
      } else {
        const uint2 x = lds64(kc), y = lds64(kc + 8 * (D / 2));
        w0[0] = x.x; w0[1] = x.y;
        w1[0] = y.x; w1[1] = y.y;
      }
      ks[u][0] *= step_of(r0);
      ks[u][1] *= step_of(r1);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const uint32_t x0 = (k & 1) ? w0[k >> 1] >> 8 : w0[k >> 1], x1 = (k & 1) ? w1[k >> 1] >> 8 : w1[k >> 1];
        const uint32_t f[4] = {codes_even(x0), codes_even(x1), codes_odd(x0), codes_odd(x1)};
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint2 q = query.f[k][n];
          mma16816((k & 1) ? sd[n] : sc[u][n], f, q.x, q.y);
        }
      }
      const float z0 = zero_float(r0), z1 = zero_float(r1);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        sd[n][0] = fmaf(-z0, query.sum[n][0], sd[n][0]);
        sd[n][1] = fmaf(-z0, query.sum[n][1], sd[n][1]);
        sd[n][2] = fmaf(-z1, query.sum[n][0], sd[n][2]);
        sd[n][3] = fmaf(-z1, query.sum[n][1], sd[n][3]);
      }
    } else {
      // lanes 0-7, 8-15, 16-23, 24-31 give the rows of: tokens 0-7 and 8-15 of the first 8 dimensions, then of the second
      const int t = lane & 15;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t f[4];
        const int piece = 2 * (k & 3) + (lane >> 4);
        ldmatrix4(f, stage + (uint32_t)((k >> 2) * CT + au + t) * 128 + ((piece ^ (t & 7)) << 4));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint2 q = query.f[k][n];
          mma16816((k & 1) ? sd[n] : sc[u][n], f, q.x, q.y);
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[u][n][i] += sd[n][i];
  }

  // ---- exponents against the rows' bounds (none yet: any finite score is above it)
  float x[H][NT][4], top = -INFINITY;
  unsigned long long mask[NT][2];
  if (EDGE)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      mask[n][0] = query.mask(a, s, n, 0, c);
      mask[n][1] = query.mask(a, s, n, 1, c);
    }
#pragma unroll
  for (int u = 0; u < H; ++u)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float k = ks[u][i >> 1];
        if (EDGE) {
          const int j = pos + 16 * u + g + ((i & 2) ? 8 : 0) - s.context;
          const unsigned long long m = mask[n][i & 1];
          const bool see = (j < 0 || (j < 64 && ((m >> (j & 63)) & 1ull))) && !((bad >> u) & 1u);
          sc[u][n][i] = see ? sc[u][n][i] * k : -INFINITY;
          x[u][n][i] = sc[u][n][i] - acc.m[n][i & 1];
        } else {
          x[u][n][i] = fmaf(sc[u][n][i], k, -acc.m[n][i & 1]);
        }
        top = fmaxf(top, x[u][n][i]);
      }
  if (__any_sync(0xffffffffu, top > 8.f)) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float y[H][2], t = acc.m[n][j];
#pragma unroll
        for (int u = 0; u < H; ++u) {
          y[u][0] = EDGE ? sc[u][n][j] : sc[u][n][j] * ks[u][0];
          y[u][1] = EDGE ? sc[u][n][2 + j] : sc[u][n][2 + j] * ks[u][1];
          t = fmaxf(t, fmaxf(y[u][0], y[u][1]));
        }
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, k));
        acc.rescale(n, j, t);
#pragma unroll
        for (int u = 0; u < H; ++u) {
          x[u][n][j] = y[u][0] - t;
          x[u][n][2 + j] = y[u][1] - t;
        }
      }
  }
  // ---- probabilities; with codes, the value's step joins them
  uint32_t pf[H][NT][2];
#pragma unroll
  for (int u = 0; u < H; ++u) {
    float v0 = 1.f, v1 = 1.f;
    if (C::BITS == 4) {
      const uint32_t vr = stage + CT * (D + 4) + (16 * u) * 4 + g * 4;
      v0 = step_of(lds32(vr)) * ATTN_P_UP;
      v1 = step_of(lds32(vr + 32)) * ATTN_P_UP;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[i] = ex2(x[u][n][i]);
        acc.l[n][i & 1] += p[i];
        if (C::BITS == 4) {
          p[i] *= (i & 2) ? v1 : v0;
          if (EDGE && sc[u][n][i] == -INFINITY) p[i] = 0.f;        // an unseen record may say NaN
        }
      }
      pf[u][n][0] = movmatrix(bf16x2(p[0], p[1]));
      pf[u][n][1] = movmatrix(bf16x2(p[2], p[3]));
    }
  }

  // ---- O^T += V^T P^T
#pragma unroll
  for (int u = 0; u < H; ++u) {
    const int au = 16 * u;
    if (C::BITS == 4) {
      // the pairs of tokens (2c, 2c + 1) and (2c + 8, 2c + 9); dimensions g * D/8 ... of each
      const uint32_t vr = stage + CT * (D + 4) + au * 4 + 2 * c * 4;
      const uint2 ra = lds64(vr), rb = lds64(vr + 32);
      const uint32_t z[4] = {codes_even(__byte_perm(ra.x, ra.y, 0x7632)), 0u, codes_even(__byte_perm(rb.x, rb.y, 0x7632)), 0u};
#pragma unroll
      for (int n = 0; n < NT; ++n) mma16816(acc.z[n], z, pf[u][n][0], pf[u][n][1]);
      const uint32_t vc = stage + CT * (D / 2) + au * (D / 2) + 2 * c * (D / 2) + g * (D / 16);
      uint32_t w[4][D / 64];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t p = vc + ((i & 1) + (i >> 1) * 8) * (D / 2);
        if (D == 128) {
          const uint2 y = lds64(p);
          w[i][0] = y.x;
          w[i][D / 64 - 1] = y.y;
        } else {
          w[i][0] = lds32(p);
        }
      }
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {
        // low halves: elements 0, 2, 4, 6 of the word's eight; high halves: 1, 3, 5, 7
        uint32_t al = __byte_perm(w[0][h], w[1][h], 0x5410), ah = __byte_perm(w[0][h], w[1][h], 0x7632);
        uint32_t bl = __byte_perm(w[2][h], w[3][h], 0x5410), bh = __byte_perm(w[2][h], w[3][h], 0x7632);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (e == 2) { al >>= 8; ah >>= 8; bl >>= 8; bh >>= 8; }
          uint32_t f[4];
          if (e & 1) { f[0] = codes_odd(al); f[1] = codes_odd(ah); f[2] = codes_odd(bl); f[3] = codes_odd(bh); }
          else { f[0] = codes_even(al); f[1] = codes_even(ah); f[2] = codes_even(bl); f[3] = codes_even(bh); }
#pragma unroll
          for (int n = 0; n < NT; ++n) mma16816(acc.o[n][h * 4 + e], f, pf[u][n][0], pf[u][n][1]);
        }
      }
    } else {
      const uint32_t vb = stage + CT * D * 2;
      const int t = (lane & 7) + ((lane >> 4) << 3);       // lanes 0-7, 8-15: tokens 0-7 of the first and second 8 dimensions; 16-31: tokens 8-15
      uint32_t odd = 0;                                         // tokens some of whose values are not finite
      if (EDGE) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t q = lds32(vb + (uint32_t)(au + i) * 128 + lane * 4);
          const uint32_t q2 = D == 128 ? lds32(vb + (uint32_t)(CT + au + i) * 128 + lane * 4) : 0u;
          const bool nf = (q & 0x7F80u) == 0x7F80u || (q & 0x7F800000u) == 0x7F800000u || (q2 & 0x7F80u) == 0x7F80u || (q2 & 0x7F800000u) == 0x7F800000u;
          if (__any_sync(0xffffffffu, nf)) odd |= 1u << i;
        }
      }
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t f[4];
        const int piece = 2 * (k & 3) + ((lane >> 3) & 1);
        ldmatrix4t(f, vb + (uint32_t)((k >> 2) * CT + au + t) * 128 + ((piece ^ (t & 7)) << 4));
        if (EDGE && odd) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if ((f[i] & 0x7F80u) == 0x7F80u) f[i] &= 0xFFFF0000u;
            if ((f[i] & 0x7F800000u) == 0x7F800000u) f[i] &= 0x0000FFFFu;
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) mma16816(acc.o[n][k], f, pf[u][n][0], pf[u][n][1]);
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
              const float mine = (i & 8) ? sc[u][n][2 + j] : sc[u][n][j];
              const float v = __shfl_sync(0xffffffffu, mine, (i & 7) * 4 + c);
              if (v == -INFINITY) continue;
              const float p = ex2(v - acc.m[n][j]);
#pragma unroll
              for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  const int e = k * 16 + g + 8 * h, tt = au + i;
                  const uint32_t q = lds32(vb + (uint32_t)((e >> 6) * CT + tt) * 128 + (((((e & 63) >> 3) ^ (tt & 7)) << 4) | ((e & 6) << 1)));
                  const float y = (e & 1) ? __uint_as_float(q & 0xFFFF0000u) : __uint_as_float(q << 16);
                  if (!(fabsf(y) <= 3.4028234663852886e38f)) acc.o[n][k][2 * h + j] += p * y;
                }
            }
        }
      }
    }
  }
}

// Rows of an item that is complete: normalised, rounded, written.
template <typename C>
__device__ void attn_write(const AttnArgs& a, Acc<C>& acc, const Seq& s, int item, int lane) {
  const int g = lane >> 2, c = lane & 3;
  const int head = item % a.kv_heads, first = (item / a.kv_heads) * C::ROWS;
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
      const bool none = l == 0.f;                                     // nothing seen, or nothing but scores of -inf
      const float inv = none ? 0.f : 1.f / l;
      const int node = r / a.group, h = head * a.group + r - node * a.group;
      const long long row = s.start + node;
      __nv_bfloat16* o = a.out + row * a.o_t + h * a.o_h;
      if (C::BITS == 4) {
        // dimensions g * D/8 + 2t and + 1 of tile t
        uint32_t v[C::KS];
#pragma unroll
        for (int t = 0; t < C::KS; ++t) {
          const float up = (t & 1) ? 0.0625f : 1.f, f = inv * ATTN_P_BACK, z = acc.z[n][j];
          v[t] = bf16x2(fmaf(acc.o[n][t][j], up, -z) * f, fmaf(acc.o[n][t][2 + j], up, -z) * f);
        }
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
      if (a.lse && g == 0) a.lse[row * a.lse_t + h] = none ? -INFINITY : acc.m[n][j] * 0.6931471805599453f + logf(l);
    }
}

template <typename C>
__global__ void __launch_bounds__(C::THREADS, C::PER_SM) attn_kernel(const AttnArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  constexpr int RINGS = C::WN * C::STAGES * C::STAGE_BYTES;
  constexpr size_t SLOT = (size_t)C::PART * 32;
  float* merge = reinterpret_cast<float*>(smem + RINGS);
  AttnAux<C>* aux = reinterpret_cast<AttnAux<C>*>(smem + RINGS + C::MERGE_BYTES);
  static_assert(sizeof(AttnAux<C>) <= C::AUX_BYTES, "AttnCfg::AUX_BYTES");
  const int wn = warp_index(), lane = threadIdx.x & 31;
  Walk<C> w;
  if (wn == 0) {
    w.begin(a);
    if (lane == 0) {
      aux->ahead[0] = w;
      aux->todos = 0;
    }
  }
  __syncthreads();
  w = aux->ahead[0];
  if (w.left <= 0) return;
  __syncthreads();
  uint8_t* ring = smem + wn * C::STAGES * C::STAGE_BYTES;
  Fetch<C> fetch;
  fetch.begin(a, w, ring, &aux->ahead[wn], wn, lane);
  for (int i = 0; i < C::STAGES; ++i) fetch.issue(a, &aux->ahead[wn], wn, lane);

  bool head_of_run = true;
  int st = 0, adder = 0, turn = 0;                             // the warp that adds up the present item's parts; items so far, modulo 2
  Acc<C> acc;
  bool more;
  do {
    Query<C> query;
    query.begin(a, w.s, w.item, lane);
    acc.clear();
    const int end = min(w.end * ATTN_UNIT, w.s.context + w.s.nodes);
    for (int first = w.tile * ATTN_UNIT + wn * ATTN_CHUNK; first < end; first += C::WN * ATTN_CHUNK) {
      asm volatile("cp.async.wait_group %0;" ::"n"(C::STAGES - 1) : "memory");
      __syncwarp();
      const uint32_t stage = ptx::smem_u32(ring + st * C::STAGE_BYTES);
      const uint32_t bad = (fetch.bad >> (2 * st)) & 3u;
      const uint32_t lost = first + 16 < end ? bad : bad & 1u;           // (a second half behind the end is not fetched)
      if (lost && lane == 0) atomicOr(a.flags, KV_FLAG_BAD_INDEX);
      const bool edge = first + ATTN_CHUNK > w.s.context || lost;
      if (!edge) attn_tokens<C, false>(a, acc, stage, 0, w.s, 0u, query, lane);
      else attn_tokens<C, true>(a, acc, stage, first, w.s, bad, query, lane);
      __syncwarp();
      fetch.issue(a, &aux->ahead[wn], wn, lane);               // into the stage that is free now
      st = st + 1 == C::STAGES ? 0 : st + 1;
    }
    // Parts are stored once those of the item before are added up; its adder knows that, and may be an item ahead of the warps that still ask: hence
    // two barriers in turn.
    if (!head_of_run && wn != (adder + C::WN - 1) % C::WN) bar_sync(BAR_ADDED + (turn ^ 1), C::THREADS);
    if (wn != adder) {
      acc.template store<false>(merge + (size_t)(wn < adder ? wn : wn - 1) * SLOT + lane, 32);
      bar_arrive(BAR_STORED, C::THREADS);
    } else {
      bar_sync(BAR_STORED, C::THREADS);
#pragma unroll 1
      for (int k = 0; k < C::WN - 1; ++k) acc.template add<false>(merge + (size_t)k * SLOT + lane, 32);
      if (w.tile == 0 && w.end == w.s.tiles) {
        attn_write<C>(a, acc, w.s, w.item, lane);
      } else {
        // this CTA's part; its first one of the run goes to its first slot
        acc.template store<true>(a.parts + (2 * (size_t)blockIdx.x + (head_of_run ? 0 : 1)) * SLOT + lane, 32);
        __threadfence();
        __syncwarp();
        if (lane == 0) {
          const int c0 = w.owner(w.item_at), c1 = w.owner(w.item_at + w.s.tiles - 1);
          const unsigned n = (unsigned)(c1 - c0);
          if (atomicInc(a.counters + c0, n) == n) {
            auto& d = aux->todo[aux->todos++];
            d.s = w.s;
            d.item = w.item;
            d.c0 = c0;
            d.c1 = c1;
            d.item_at = w.item_at;
          }
          __threadfence();
        }
        __syncwarp();
      }
      bar_arrive(BAR_ADDED + turn, C::THREADS);
    }
    head_of_run = false;
    more = w.next(a);
    adder = adder + 1 == C::WN ? 0 : adder + 1;
    turn ^= 1;
  } while (more);
  if (wn != (adder + C::WN - 1) % C::WN) bar_sync(BAR_ADDED + (turn ^ 1), C::THREADS);
  bar_sync(BAR_ALL, C::THREADS);
  // Cut items whose last part was this CTA's: with two of them half of the warps each.
  const int todos = aux->todos;
  if (todos > 0) {
    const int warps = C::WN / todos, which = wn / warps, me = wn - which * warps;
    const auto& d = aux->todo[which];
    acc.clear();
    for (int k = d.c0 + me; k <= d.c1; k += warps)
      // the part of CTA k: its run begins with it unless the item began inside the run
      acc.template add<true>(a.parts + (2 * (size_t)k + (w.run_begin(k) < d.item_at ? 1 : 0)) * SLOT + lane, 32);
    attn_merge<C>(acc, merge + which * (warps / 2) * SLOT, me, warps, lane);
    if (me == 0) attn_write<C>(a, acc, d.s, d.item, lane);
  }
}

}  // namespace kv
}  // namespace conqur
