// The attention of conqur_attention.cuh for more than 16 query rows a key head (trees of drafted tokens): there the products set the pace, and they go to
// the tcgen05 tensor cores.  One CTA an SM works on blocks of 128 rows, 64 tokens at a time:
//   S = Q K^T (128 x 64) and O += P V (128 x D) with accumulators in TMEM, and so are Q and P: shared memory, which the products read their other operand
//   from, is what is scarce here.  Tiles of even and odd number are two streams, each with its own S, P, O, bounds and sums, joined at the end of an
//   item, so that two groups of warps take exponentials while the products of the other's tile run:
//   warps 0-3, 4-7   one row a thread: scores from TMEM, bound, exponentials (no exchange between threads), P as bf16 to TMEM
//   warps 8-11, 12-15  bring the keys and values of every other tile into four stages: bf16 as they lie (the cache's planes are the operands' swizzled
//                    layout), codes turned into the bf16 integers (code - zero-point) / 64, exactly; the steps go to the scores and the probabilities
//   warp 16          issues the products: the scores of a stream's next tile as soon as those of the present one are read
// The bound of a row is raised only when a score exceeds it by 2^8; then its accumulators are read, scaled and written back.  Values that are not finite meet
// zeros of rows that do not see them only among the drafted tokens; there they are left out of the product and added at the item's end.  Work is cut into runs and
// parts are joined as in conqur_attention.cuh.  Every wait between the warps is bounded: when one runs out the CTA latches TIMEOUT,
// leaves the item that it is at and all later ones unwritten, waits for its products under way and ends.
// Floor: 8192 exponentials a tile at 16 a cycle are 512 cycles, and the products take as long.  Measured, 37 sequences of 6000, 8 key heads, 128 rows: 161 us over
// 4 bits, about 1500 cycles a tile (a half-used issue rate: the chain score - exponential - product of two streams is what is left), 222 to 226 us over bf16 (two
// thirds of it the cache's bytes).  Sixteen rows in the kernel of conqur_attention.cuh take 79 us there, 32 rows would take two passes of it: 158, and here 155.
#pragma once
#include "conqur_attention.cuh"

namespace conqur {
namespace kv {

enum { BAR_ITEM = 5 };
constexpr long long TREE_LOST_LIMIT = 10000000ll;              // some 5 ms

template <int BITS_, int D_>
struct TreeCfg {
  static constexpr int BITS = BITS_, D = D_;
  static constexpr int ROWS = 128, THREADS = 640, PLANES = D / 64, STAGES = 4;
  static constexpr int T_BYTES = PLANES * 8192;                // keys or values of a tile
  static constexpr int RAW = 2, RAW_BYTES = 9728;   // tiles of codes on their way: 64 bytes and two records a thread; page numbers
  static constexpr int AUX_BYTES = 5120;
  static constexpr int SMEM = 1024 + 2 * STAGES * T_BYTES + (BITS == 4 ? 2 * RAW * RAW_BYTES : 0) + AUX_BYTES;
  // TMEM columns: scores 2 x 64, accumulators 2 x 128, the rows D / 2 (two bf16 a column), probabilities 2 x 32
  static constexpr int T_O = 128, T_Q = 384, T_P = 448;
  static_assert(SMEM <= 227 * 1024, "shared memory of an SM");
  static constexpr int MIN_RUN = 4;                            // tiles a CTA takes at least
  static constexpr int SLOT = (D + 2) * 128;                   // floats of a part: columns of 128 rows; then bounds, sums
};

template <typename C>
struct TreeAux {
  uint64_t full[C::STAGES], empty[C::STAGES], scored[2], read[2], ready[2], done[2];   // tile brought, free again; S complete, read; P written; P V complete
  uint64_t drained;                                            // all products of the CTA complete
  alignas(16) float kstep[C::STAGES][64];                      // (read four at a time)
  alignas(16) float vstep[C::STAGES][64];
  uint32_t bad[C::STAGES][2];                                  // tokens of a tile whose page could not be read
  float bound[2][128], sum[2][128];                            // of the two streams
  Walk<C> w;
  uint32_t tmem;
  int abort_flag, ended, last;
  int odd;                                                     // some value or step of a drafted token was not finite (never taken back: it only asks for a look)
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
// 64 columns with one wait.
__device__ __forceinline__ void tmem_read64(uint32_t taddr, float (&v)[64]) {
  uint32_t r[4][16];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[i][0]), "=r"(r[i][1]), "=r"(r[i][2]), "=r"(r[i][3]), "=r"(r[i][4]), "=r"(r[i][5]), "=r"(r[i][6]), "=r"(r[i][7]), "=r"(r[i][8]),
          "=r"(r[i][9]), "=r"(r[i][10]), "=r"(r[i][11]), "=r"(r[i][12]), "=r"(r[i][13]), "=r"(r[i][14]), "=r"(r[i][15])
        : "r"(taddr + 16 * i)
        : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 64; ++i) v[i] = __uint_as_float(r[i >> 4][i & 15]);
}
// D(tmem) (+)= A(tmem: lane = row, two consecutive k a column) B(smem)
__device__ __forceinline__ void umma_from_tmem(uint32_t leader, uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(leader)
      : "memory");
}
// Two fp32 in one instruction.
__device__ __forceinline__ uint64_t two(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 apart(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t two_mul(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t two_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t two_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
// One look at a barrier, without the hardware's suspension of a waiting thread; the whole warp agrees.
__device__ __forceinline__ bool arrived(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.b32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(ptx::smem_u32(bar)), "r"(parity)
      : "memory");
  return __all_sync(0xffffffffu, ok != 0u);
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

// A barrier that tells all of its threads whether any of them brought `mine`.
__device__ __forceinline__ bool bar_any(int bar, int threads, bool mine) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %3, 0;\n\t"
      "bar.red.or.pred q, %1, %2, p;\n\t"
      "selp.b32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"(bar), "r"(threads), "r"((uint32_t)mine)
      : "memory");
  return any != 0u;
}

// ---- warps 8-11: a thread takes a token's 64 dimensions of one plane, of keys and values (D = 64: threads 0-63 the keys, 64-127 the values)
template <typename C>
struct Bring {
  int tok, plane;
  bool keys, values;
  const int* table;
  const uint8_t* head;
  int len;
  int page;                          // 4 bits: of the next tile to fetch
  int now[2], next[2];               // 16 bits: of tokens lane and lane + 32 of the tile being brought and of the group's next
  uint32_t goods, ahead;             // a bit a slot of the ring: the page could be read; a page number comes with it
  int last;                          // end of the item's tiles in this run

  __device__ __forceinline__ void item(const AttnArgs& a, const Walk<C>& w, int tid) {
    tok = tid & 63;
    const int half = tid >> 6;
    plane = C::D == 128 ? half : 0;
    keys = C::D == 128 || half == 0;
    values = C::D == 128 || half == 1;
    table = a.table + (long long)w.b * a.table_stride;
    head = a.cache + (long long)(w.item % a.kv_heads) * a.block_bytes;
    len = w.s.context + w.s.nodes;
    last = w.end;
    goods = ahead = 0u;
  }
  __device__ __forceinline__ int look(const AttnArgs& a, int tile, int at) const {
    const int pos = tile * ATTN_UNIT + at;
    return tile < last && pos < len && (pos >> a.log_page) < a.table_width ? table[pos >> a.log_page] : -1;
  }
  __device__ __forceinline__ void ask(const AttnArgs& a, int tile, int lane) {
    next[0] = look(a, tile, lane);
    next[1] = look(a, tile, lane + 32);
  }
  // 4 bits: the codes of the tile whose page was asked for, into this thread's places of a slot (zeros where there is no page)
  __device__ __forceinline__ void fetch(const AttnArgs& a, uint8_t* raw, int slot, int tile, int tid) {
    const bool good = (unsigned)page < (unsigned)a.pages;
    goods = (goods & ~(1u << slot)) | ((good ? 1u : 0u) << slot);
    const int at = (tile * ATTN_UNIT + tok) & (a.page_size - 1), n = good ? 16 : 0;
    const uint8_t* p = head + (good ? (long long)page * a.page_bytes : 0);
    const uint8_t* c = p + at * (C::D / 2) + plane * 32;
    const uint32_t to = ptx::smem_u32(raw + slot * C::RAW_BYTES) + tid * 16;
    if (keys) {
      copy16(to, c, n);
      copy16(to + 2048, c + 16, n);
    }
    if (values) {
      copy16(to + 4096, c + a.codes_bytes, n);
      copy16(to + 6144, c + a.codes_bytes + 16, n);
    }
    // the page number of the tile that takes this slot next comes along
    const int next = tile + 2 * C::RAW, npos = next * ATTN_UNIT + tok;
    const bool have = next < last && npos < len && (npos >> a.log_page) < a.table_width;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(ptx::smem_u32(raw + slot * C::RAW_BYTES) + 9216 + tid * 4), "l"(have ? table + (npos >> a.log_page) : a.starts), "r"(have ? 4 : 0) : "memory");
    ahead = (ahead & ~(1u << slot)) | ((have ? 1u : 0u) << slot);
    const uint32_t rec = ptx::smem_u32(raw + slot * C::RAW_BYTES) + 8192 + tid * 8;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(rec), "l"(p + 2 * a.codes_bytes + at * 4), "r"(n / 4) : "memory");
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(rec + 4), "l"(p + 2 * a.codes_bytes + (a.page_size + at) * 4), "r"(n / 4) : "memory");
  }
  static __device__ __forceinline__ void spread(uint8_t* row, const uint4 c0, const uint4 c1, uint32_t bias, int t) {
    const uint32_t w[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(row + ((i ^ (t & 7)) << 4)) = codes8(w[i], bias);
  }
  // Tokens of the tile whose page cannot be read, 32 a warp.
  __device__ __forceinline__ void lost(const AttnArgs& a, TreeAux<C>* aux, int st, int tile, bool good, int half, int at) {
    const unsigned x = __ballot_sync(0xffffffffu, !good && tile * ATTN_UNIT + at < len);
    if ((at & 31) == 0) {
      aux->bad[st][half] = x;
      if (x) atomicOr(a.flags, KV_FLAG_BAD_INDEX);
    }
  }
  __device__ __forceinline__ void put(const AttnArgs& a, TreeAux<C>* aux, uint8_t* tile_mem, const uint8_t* raw, int slot, int st, int tid, bool drafted) {
    uint8_t* kd = tile_mem + plane * 8192 + tok * 128;
    uint8_t* vd = kd + C::T_BYTES;
    const uint8_t* from = raw + slot * C::RAW_BYTES + tid * 16;
    const uint2 rec = *reinterpret_cast<const uint2*>(raw + slot * C::RAW_BYTES + 8192 + tid * 8);
    // (a record that says NaN: the step carries it; its codes are codes)
    if (keys) spread(kd, *reinterpret_cast<const uint4*>(from), *reinterpret_cast<const uint4*>(from + 2048), zero_bias(rec.x), tok);
    if (values) spread(vd, *reinterpret_cast<const uint4*>(from + 4096), *reinterpret_cast<const uint4*>(from + 6144), zero_bias(rec.y), tok);
    if (tid < 64) aux->kstep[st][tok] = step_of(rec.x) * a.scale;                // the scale has the 64 of the codes
    else {
      // a step that is not finite must not meet the zeros of rows that do not see it: left out here, added at the end
      float step = step_of(rec.y) * 64.f;
      if (drafted && !(fabsf(step) < INFINITY)) {
        step = 0.f;
        *reinterpret_cast<volatile int*>(&aux->odd) = 1;
      }
      aux->vstep[st][tok] = step;
    }
  }
  // 16 bits: the copies of a tile (one group of copies): eight threads a row of 128 bytes, sixteen rows at a time
  __device__ __forceinline__ void copy(const AttnArgs& a, uint8_t* tile_mem, int tile, int tid) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int row = 16 * k + (tid >> 3), page = __shfl_sync(0xffffffffu, now[k >> 1], row & 31);
      const bool good = (unsigned)page < (unsigned)a.pages;
      const int bytes = good ? 16 : 0;
      const uint8_t* p = good ? head + (long long)page * a.page_bytes + ((tile * ATTN_UNIT + row) & (a.page_size - 1)) * 128 + (tid & 7) * 16 : a.cache;
      const long long step = good ? a.plane_bytes : 0;
      const uint32_t to = ptx::smem_u32(tile_mem) + row * 128 + (tid & 7) * 16;
#pragma unroll
      for (int i = 0; i < 2 * C::PLANES; ++i) copy16(to + i * 8192, p + i * step, bytes);
    }
  }
  // What is left to do when this thread's copies are there: values that are not finite must not meet the zeros of rows that do not see them.  They are
  // left out here and added at the end.
  __device__ __forceinline__ void finish(TreeAux<C>* aux, uint8_t* tile_mem, int tile, int context, int tid) {
    if ((tile + 1) * ATTN_UNIT <= context) return;
#pragma unroll 1
    for (int i = 0; i < 4 * C::PLANES; ++i) {
      uint8_t* v = tile_mem + C::T_BYTES + i * 2048 + tid * 16;
      const uint4 x = *reinterpret_cast<uint4*>(v);
      uint32_t e[4] = {x.x, x.y, x.z, x.w};
      bool hit = false;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (not_finite2(e[j])) {
          hit = true;
          if ((e[j] & 0x7F80u) == 0x7F80u) e[j] &= 0xFFFF0000u;
          if ((e[j] & 0x7F800000u) == 0x7F800000u) e[j] &= 0x0000FFFFu;
        }
      if (hit) {
        *reinterpret_cast<uint4*>(v) = make_uint4(e[0], e[1], e[2], e[3]);
        *reinterpret_cast<volatile int*>(&aux->odd) = 1;
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

// One of the three roles' warps through all items of the CTA.
enum TreeRole { TREE_ROWS, TREE_BRING, TREE_PRODUCTS };
template <typename C, TreeRole ROLE>
__device__ __forceinline__ void tree_role(const AttnArgs& a, TreeAux<C>* aux, uint8_t* sT, uint8_t* sRaw, int warp) {
  constexpr int D = C::D, PL = C::PLANES, S = C::STAGES, STAGE = 2 * C::T_BYTES;
  const int tid = threadIdx.x;
  volatile int* abort_flag = &aux->abort_flag;
  const uint32_t tmem = aux->tmem, tO = tmem + C::T_O, tQ = tmem + C::T_Q, tP = tmem + C::T_P;
  Walk<C> w = aux->w;
  int cnt = 0;                                                 // tiles so far: stream and buffers cnt & 1, phase (cnt >> 1) & 1; stage cnt % S
  bool head_of_run = true, more = w.left > 0;

  while (more) {
    // ---- the item's rows
    if (ROLE == TREE_ROWS && warp < 4) {
      const TreeRow row = tree_row<C>(a, w.s, w.item, tid);
      const __nv_bfloat16* q = a.q + row.row * a.q_t + row.head * a.q_h;
#pragma unroll
      for (int c = 0; c < D / 2; c += 16) {
        uint32_t x[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 y = row.real ? *reinterpret_cast<const uint4*>(q + 2 * c + 8 * j) : make_uint4(0u, 0u, 0u, 0u);
          x[4 * j] = y.x; x[4 * j + 1] = y.y; x[4 * j + 2] = y.z; x[4 * j + 3] = y.w;
        }
        tmem_write16(tQ + ((uint32_t)(warp * 32) << 16) + c, x);
      }
      tmem_write_wait();
      ptx::tc_fence_before();
    }
    if constexpr (ROLE != TREE_BRING) {                        // (keys and values run ahead into the next item)
      bar_sync(BAR_ITEM, 288);
      ptx::tc_fence_after();
    }
    const int tiles = w.end - w.tile;
    const int len = w.s.context + w.s.nodes;
    bool ok = true;                                            // no wait of this warp's has run out in this item

    if constexpr (ROLE == TREE_BRING) {
      // ------------------------------------------------------------ keys and values
      // two groups of warps take the tiles of even and odd number
      Bring<C> in;
      const int id = tid & 127, group = (warp >> 2) & 1, i0 = (cnt ^ group) & 1;
      uint8_t* raw = sRaw + group * C::RAW * C::RAW_BYTES;
      in.item(a, w, id);
      if (C::BITS == 4) {
        int pages[C::RAW];
#pragma unroll
        for (int k = 0; k < C::RAW; ++k) pages[k] = in.look(a, w.tile + i0 + 2 * k, in.tok);
#pragma unroll
        for (int k = 0; k < C::RAW; ++k) {
          in.page = pages[k];
          in.fetch(a, raw, k, w.tile + i0 + 2 * k, id);
          asm volatile("cp.async.commit_group;" ::: "memory");
        }
      } else {
        in.ask(a, w.tile + i0, id & 31);
      }
      int slot = 0;
      for (int i = i0; i < tiles; i += 2) {
        const int n = cnt + i, st = n % S;
        if (!tc_wait_warp(&aux->empty[st], ((uint32_t)(n / S) & 1u) ^ 1u, abort_flag)) break;
        uint8_t* mem = sT + st * STAGE;
        if (C::BITS == 16) {
          in.now[0] = in.next[0];
          in.now[1] = in.next[1];
          in.ask(a, w.tile + i + 2, id & 31);
          in.copy(a, mem, w.tile + i, id);
          asm volatile("cp.async.commit_group;" ::: "memory");
          if (id < 64) in.lost(a, aux, st, w.tile + i, (unsigned)(id < 32 ? in.now[0] : in.now[1]) < (unsigned)a.pages, id >> 5, id);
          // this tile's copies are issued, those of the group's tile before are there; at the end of the item all
          auto there = [&](int k) {
            const int at = (cnt + k) % S;
            in.finish(aux, sT + at * STAGE, w.tile + k, w.s.context, id);
            ptx::fence_proxy_async();
            ptx::mbar_arrive(&aux->full[at]);
          };
          if (i > i0) {
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            there(i - 2);
          }
          if (i + 2 >= tiles) {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            there(i);
          }
        } else {
          asm volatile("cp.async.wait_group %0;" ::"n"(C::RAW - 1) : "memory");
          in.put(a, aux, mem, raw, slot, st, id, (w.tile + i + 1) * ATTN_UNIT > w.s.context);
          if (id < 64) in.lost(a, aux, st, w.tile + i, (in.goods >> slot) & 1u, id >> 5, id);
          ptx::fence_proxy_async();
          ptx::mbar_arrive(&aux->full[st]);
          in.page = (in.ahead >> slot) & 1u ? *reinterpret_cast<const int*>(raw + slot * C::RAW_BYTES + 9216 + id * 4) : -1;
          in.fetch(a, raw, slot, w.tile + i + 2 * C::RAW, id);
          asm volatile("cp.async.commit_group;" ::: "memory");
          slot = slot + 1 == C::RAW ? 0 : slot + 1;
        }
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
    } else if constexpr (ROLE == TREE_PRODUCTS) {
      // ------------------------------------------------------------ products
      const uint32_t leader = ptx::elect_one();
      const uint32_t base = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 4) << 24);
      const uint32_t id_s = base | ((uint32_t)(64 >> 3) << 17), id_o = base | (1u << 16) | ((uint32_t)(D >> 3) << 17);
      const uint32_t t0 = ptx::smem_u32(sT);
      auto scores = [&](int n) {
        const int st = n % S;
        if (!tc_wait_warp(&aux->full[st], (uint32_t)(n / S) & 1u, abort_flag)) return false;
        ptx::tc_fence_after();
        const uint32_t k0 = t0 + st * STAGE;
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
          umma_from_tmem(leader, tmem + (n & 1) * 64, tQ + j * 8, tc_smem_desc(k0 + (j >> 2) * 8192 + (j & 3) * 32, 16, 1024), id_s, j > 0 ? 1u : 0u);
        ptx::umma_commit_by<false>(leader, ptx::smem_u32(&aux->scored[n & 1]));
        return true;
      };
      ok = scores(cnt) && (tiles < 2 || scores(cnt + 1));
      for (int i = 0; ok && i < tiles; ++i) {
        const int n = cnt + i, buf = n & 1;
        // the stream's next scores or this tile's P V, whichever can go first (a stage may have to be freed by this tile before the next keys come)
        bool next = i + 2 >= tiles;
        const long long since = clock64();
        while (!next && !arrived(&aux->ready[buf], (n >> 1) & 1)) {
          if (arrived(&aux->read[buf], (n >> 1) & 1) && arrived(&aux->full[(n + 2) % S], (uint32_t)((n + 2) / S) & 1u)) {
            ptx::tc_fence_after();
            if (!(ok = scores(n + 2))) break;
            next = true;
          } else if (__any_sync(0xffffffffu, *abort_flag || clock64() - since > TC_WAIT_LIMIT)) {
            *abort_flag = 1;
            ok = false;
            break;
          }
        }
        if (!(ok = ok && tc_wait_warp(&aux->ready[buf], (n >> 1) & 1, abort_flag))) break;
        ptx::tc_fence_after();
        const uint32_t v0 = t0 + (n % S) * STAGE + C::T_BYTES;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          umma_from_tmem(leader, tO + buf * 128, tP + buf * 32 + j * 8, tc_smem_desc(v0 + j * 2048, 8192, 1024), id_o, (i > 1 || j > 0) ? 1u : 0u);
        ptx::umma_commit_by<false>(leader, ptx::smem_u32(&aux->done[buf]));
        ptx::umma_commit_by<false>(leader, ptx::smem_u32(&aux->empty[n % S]));
        if (!next) ok = scores(n + 2);
      }
    } else {
      // ------------------------------------------------------------ a row a thread, every other tile
      const int buf = warp >> 2, r = tid & 127;
      const TreeRow row = tree_row<C>(a, w.s, w.item, r);
      const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
      float m = -INFINITY, l = 0.f;
      const int i0 = (cnt ^ buf) & 1;                          // the stream's first tile of this item
      for (int i = i0; i < tiles; i += 2) {
        const int n = cnt + i, st = n % S, first = (w.tile + i) * ATTN_UNIT;
        // (the steps come with the tile, the scores with its product)
        if (!(ok = tc_wait_warp(&aux->full[st], (uint32_t)(n / S) & 1u, abort_flag) && tc_wait_warp(&aux->scored[buf], (n >> 1) & 1, abort_flag))) break;
        ptx::tc_fence_after();
        const uint32_t tS = tmem + lanes + buf * 64;
        const unsigned long long bad = (unsigned long long)aux->bad[st][0] | ((unsigned long long)aux->bad[st][1] << 32);
        const bool edge = first + ATTN_UNIT > w.s.context || bad != 0ull;
        const unsigned long long see = edge ? seen64(row.mask, w.s.context, first) & ~bad : ~0ull;
        const uint64_t all = two(a.scale, a.scale);
        auto kstep = [&](int j) { return C::BITS == 4 ? *reinterpret_cast<const ulonglong2*>(&aux->kstep[st][j]) : make_ulonglong2(all, all); };
        auto blind = [&](float (&s)[64]) {                     // not seen: -inf
          const uint32_t lo = (uint32_t)see, hi = (uint32_t)(see >> 32);
#pragma unroll
          for (int j = 0; j < 64; ++j)
            if (!(((j < 32 ? lo : hi) >> (j & 31)) & 1u)) s[j] = -INFINITY;
        };
        float s[64];
        auto against = [&](float neg) {                        // scores minus the bound; their maximum
          const uint64_t neg2 = two(neg, neg);
          tmem_read64(tS, s);
#pragma unroll
          for (int j = 0; j < 64; j += 4) {
            const ulonglong2 k = kstep(j);
            const float2 x = apart(two_fma(two(s[j], s[j + 1]), k.x, neg2)), y = apart(two_fma(two(s[j + 2], s[j + 3]), k.y, neg2));
            s[j] = x.x; s[j + 1] = x.y; s[j + 2] = y.x; s[j + 3] = y.y;
          }
          if (edge) blind(s);
          float top = -INFINITY;
#pragma unroll
          for (int j = 0; j < 64; j += 2) top = fmaxf(top, fmaxf(s[j], s[j + 1]));
          return top;
        };
        // A score above the bound by 2^8 (there is none yet: any) raises it: the row's own scores decide, whatever its neighbours in the warp do.
        const bool up = against(m == -INFINITY ? 3e38f : -m) > 8.f;
        const bool raise = __any_sync(0xffffffffu, up);
        float f = 1.f;
        if (raise) {
          const float top = against(0.f);
          if (up) {
            f = ex2(m - top);
            m = top;
          }
          against(m == -INFINITY ? 3e38f : -m);
        }
        ptx::tc_fence_before();
        ptx::mbar_arrive(&aux->read[buf]);
        // P and O of the stream's tile before
        if (!(ok = tc_wait_warp(&aux->done[buf], ((n >> 1) & 1) ^ 1, abort_flag))) break;
        ptx::tc_fence_after();
        if (raise) {
          l *= f;
          if (i > i0) {                                        // (the item's first tile overwrites O)
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {
              uint32_t o[16];
              tmem_read16(tO + buf * 128 + lanes + c, o);
#pragma unroll
              for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
              tmem_write16(tO + buf * 128 + lanes + c, o);
            }
            tmem_write_wait();
          }
        }
        uint64_t sum = two(0.f, 0.f);                          // a tile's probabilities by themselves: fewer roundings of a long sum
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t p[16];
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            const int q = h * 32 + j;
            uint64_t x = two(ex2(s[q]), ex2(s[q + 1])), y = two(ex2(s[q + 2]), ex2(s[q + 3]));
            sum = two_add(two_add(sum, x), y);
            if (C::BITS == 4) {
              const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(&aux->vstep[st][q]);
              x = two_mul(x, v.x);
              y = two_mul(y, v.y);
            }
            const float2 e = apart(x), f = apart(y);
            p[j / 2] = bf16x2(e.x, e.y);
            p[j / 2 + 1] = bf16x2(f.x, f.y);
          }
          tmem_write16(tP + lanes + buf * 32 + h * 16, p);
        }
        const float2 sums = apart(sum);
        l += sums.x + sums.y;
        tmem_write_wait();
        ptx::tc_fence_before();
        ptx::mbar_arrive(&aux->ready[buf]);
      }
      const int mine = tiles > i0 ? (tiles - 1 - i0) / 2 : -1, last = cnt + i0 + 2 * mine;      // the stream's last tile of the item
      if (ok && mine >= 0) ok = tc_wait_warp(&aux->done[buf], (last >> 1) & 1, abort_flag);
      ptx::tc_fence_after();
      aux->bound[buf][r] = m;
      aux->sum[buf][r] = l;
      // the item is written only if every warp of both streams has seen its last product: each brings its own outcome to the barrier
      ok = !bar_any(BAR_ALL, 256, !ok);
      if (ok) {
        const bool whole = w.tile == 0 && w.end == w.s.tiles;
        // the two streams together; each group of warps takes half of the columns
        const float m0 = aux->bound[0][r], m1 = aux->bound[1][r];
        m = m1 > m0 ? m1 : m0;
        const bool two = tiles > 1;
        float f[2] = {m == -INFINITY ? 1.f : ex2(m0 - m), m == -INFINITY ? 1.f : ex2(m1 - m)};
        l = aux->sum[0][r] * f[0] + aux->sum[1][r] * f[1];
        const bool none = l == 0.f && m == -INFINITY;
        float* part = a.parts + (2 * (size_t)blockIdx.x + (head_of_run ? 0 : 1)) * C::SLOT + r;
        if (whole) {
          const float inv = none ? 0.f : 1.f / l;
          f[0] *= inv;
          f[1] *= inv;
        }
        const int only = (cnt & 1);                            // the stream of the item's first tile
        const int odd = *reinterpret_cast<volatile int*>(&aux->odd);
#pragma unroll 1
        for (int c = buf * (D / 2); c < (buf + 1) * (D / 2); c += 32) {
          float o[32];
          ptx::tmem_ld32(tO + only * 128 + lanes + c, o);
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] *= f[only];
          if (two) {
            float x[32];
            ptx::tmem_ld32(tO + (only ^ 1) * 128 + lanes + c, x);
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = fmaf(x[j], f[only ^ 1], o[j]);
          }
          if (odd && row.real) {
            // values that are not finite, of the tokens that the row sees (rare)
            for (int pos = max(w.tile * ATTN_UNIT, w.s.context & ~(ATTN_UNIT - 1)); pos < min(len, w.end * ATTN_UNIT); ++pos) {
              const int d = pos - w.s.context;
              if (d >= 0 && !((row.mask >> d) & 1ull)) continue;
              const int page = (pos >> a.log_page) < a.table_width ? a.table[(long long)w.b * a.table_stride + (pos >> a.log_page)] : -1;
              if ((unsigned)page >= (unsigned)a.pages) continue;
              const int at = pos & (a.page_size - 1);
              const uint8_t* v = a.cache + (long long)page * a.page_bytes + (long long)(w.item % a.kv_heads) * a.block_bytes;
              if (C::BITS == 4) {
                const float step = step_of(*reinterpret_cast<const uint32_t*>(v + 2 * a.codes_bytes + (a.page_size + at) * 4));
                if (!(fabsf(step) < INFINITY)) {
#pragma unroll
                  for (int j = 0; j < 32; ++j) o[j] = __uint_as_float(0x7FC00000u);
                }
                continue;
              }
              v += (PL + c / 64) * a.plane_bytes + at * 128;
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
          if (buf == 0 && row.real && a.lse) a.lse[row.row * a.lse_t + row.head] = none ? -INFINITY : (m == -INFINITY ? 0.f : m) * 0.6931471805599453f + logf(l);
        } else {
          if (buf == 0) {
            __stcg(part + D * 128, m);
            __stcg(part + (D + 1) * 128, l);
          }
          __threadfence();
          bar_sync(BAR_ALL, 256);
          const int c0 = w.owner(w.item_at), c1 = w.owner(w.item_at + w.s.tiles - 1);
          if (tid == 0) {
            const unsigned n = (unsigned)(c1 - c0);
            aux->last = atomicInc(a.counters + c0, n) == n;
            __threadfence();
          }
          bar_sync(BAR_ALL, 256);
          if (aux->last) {
            auto slot = [&](int k) { return a.parts + (2 * (size_t)k + (w.run_begin(k) < w.item_at ? 1 : 0)) * C::SLOT + r; };
            // the parts' loads go out several at a time: their latency is what this costs
            float tm = -INFINITY, tl = 0.f;
            for (int k = c0; k <= c1; k += 8) {
              float om[8], ol[8];
#pragma unroll
              for (int u = 0; u < 8; ++u) {
                const float* p = slot(min(k + u, c1));
                om[u] = k + u <= c1 ? __ldcg(p + D * 128) : -INFINITY;
                ol[u] = k + u <= c1 ? __ldcg(p + (D + 1) * 128) : 0.f;
              }
#pragma unroll
              for (int u = 0; u < 8; ++u) {
                const float to = om[u] > tm ? om[u] : tm;
                tl = tl * (to == -INFINITY ? 1.f : ex2(tm - to)) + ol[u] * (to == -INFINITY ? 1.f : ex2(om[u] - to));
                tm = to;
              }
            }
            const bool zero = tl == 0.f && tm == -INFINITY;
            const float ti = zero ? 0.f : 1.f / tl;
#pragma unroll 1
            for (int c = buf * (D / 2); c < (buf + 1) * (D / 2); c += 32) {
              float o[32] = {};
#pragma unroll 2
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
            if (buf == 0 && row.real && a.lse) a.lse[row.row * a.lse_t + row.head] = zero ? -INFINITY : (tm == -INFINITY ? 0.f : tm) * 0.6931471805599453f + logf(tl);
          }
        }
      }
      ptx::tc_fence_before();
    }
    if constexpr (ROLE != TREE_BRING) {
      if (bar_any(BAR_ITEM, 288, !ok)) break;                  // rows and accumulators may be replaced
    } else {
      if (__any_sync(0xffffffffu, *abort_flag)) break;
    }
    cnt += tiles;
    head_of_run = false;
    more = w.next(a);
  }
  if (ROLE == TREE_PRODUCTS && aux->w.left > 0) {
    // A wait that ran out leaves products under way: they end before TMEM, the tiles and the barriers they arrive on are given back.
    ptx::umma_commit_by<false>(ptx::elect_one(), ptx::smem_u32(&aux->drained));
    const long long since = clock64();
    while (!arrived(&aux->drained, 0u))
      if (__any_sync(0xffffffffu, clock64() - since > TC_WAIT_LIMIT)) break;
  }
}

template <typename C>
__global__ void __launch_bounds__(C::THREADS, 1) attn_tree_kernel(const AttnArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + (-ptx::smem_u32(smem_raw) & 1023u);         // (by an offset: the compiler goes on knowing that this is shared memory)
  uint8_t* sT = smem;                                          // stages of keys, values
  uint8_t* sRaw = sT + 2 * C::STAGES * C::T_BYTES;
  TreeAux<C>* aux = reinterpret_cast<TreeAux<C>*>(sRaw + (C::BITS == 4 ? 2 * C::RAW * C::RAW_BYTES : 0));
  static_assert(sizeof(TreeAux<C>) <= C::AUX_BYTES, "TreeCfg::AUX_BYTES");
  constexpr int S = C::STAGES;
  const int warp = warp_index(), lane = threadIdx.x & 31, tid = threadIdx.x;
  volatile int* abort_flag = &aux->abort_flag;
  if (tid == 0) {
    auto lost = [&](int site, int i) { return (int)blockIdx.x == a.lose_block && site == a.lose_site && i == a.lose_index ? 1 : 0; };
    for (int i = 0; i < S; ++i) {
      ptx::mbar_init(&aux->full[i], 128 + lost(CONQUR_TREE_WAIT_TILE, i));
      ptx::mbar_init(&aux->empty[i], 1 + lost(CONQUR_TREE_WAIT_STAGE, i));
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&aux->scored[i], 1 + lost(CONQUR_TREE_WAIT_SCORES, i));
      ptx::mbar_init(&aux->read[i], 128);
      ptx::mbar_init(&aux->ready[i], 128 + lost(CONQUR_TREE_WAIT_PROBABILITIES, i));
      ptx::mbar_init(&aux->done[i], 1 + lost(CONQUR_TREE_WAIT_OUTPUT, i));
    }
    ptx::mbar_init(&aux->drained, 1);
    aux->abort_flag = aux->ended = aux->odd = 0;
    ptx::fence_barrier_init();
    ptx::fence_proxy_async();
  }
  if (warp == 0) {
    Walk<C> b;
    b.begin(a);
    if (lane == 0) aux->w = b;
  }
  if (warp == 16) {
    ptx::tmem_alloc(&aux->tmem, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  // The block's registers are shared out again: 2 x 144 + 2 x 72 + 48 = 5 x 96, what it was launched with
  static_assert(C::THREADS == 640, "five groups of four warps at 96 registers");
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 144;");
    tree_role<C, TREE_ROWS>(a, aux, sT, sRaw, warp);
  } else if (warp < 16) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    tree_role<C, TREE_BRING>(a, aux, sT, sRaw, warp);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == 16) {
      tree_role<C, TREE_PRODUCTS>(a, aux, sT, sRaw, warp);
      aux->ended = 1;
    } else if (a.lose_site && (int)blockIdx.x == a.lose_block) {
      // test support: gives up in place of a wait of two seconds
      const long long since = clock64();
      while (!*reinterpret_cast<volatile int*>(&aux->ended) && !*abort_flag)
        if (clock64() - since > TREE_LOST_LIMIT) *abort_flag = 1;
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (tid == 0 && *abort_flag) atomicOr(a.flags, KV_FLAG_TIMEOUT);       // (behind the barrier: whichever warp gave up, and however late)
  if (warp == 16) ptx::tmem_dealloc(aux->tmem, 512);
}

}  // namespace kv
}  // namespace conqur
