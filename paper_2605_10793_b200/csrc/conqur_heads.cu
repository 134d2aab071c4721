// Query and key heads on their way into attention: position rotation (conqur_rope_heads), per-head RMS norm with the rotation
// (conqur_norm_rope_heads) and its backward pass, each with the online rotation R_3 of Appendix A in the same pass.
//
// All of them read every head row once and write it once; 2 (bf16) or 4 bytes each way an element against some 10 to 20
// instructions, so memory sets the pace and what has to be kept small is the work per element:
//   - A warp takes one token and walks its heads: the rotation's angles depend on the token and the pair alone, so each lane forms the eight
//     cosines and sines its elements need once and keeps them in registers over all heads.
//   - A head row of D elements lies in D/16 lanes, two 16-byte (bf16) pieces each, chosen so that both elements of every pair are in
//     one lane: no exchange for the rotation, log2(D/16) exchanges for the norm's sum and for R_3 (log2 16 of its levels are
//     inside a lane).
//   - Arithmetic goes two fp32 at a time (f32x2).  A lane's sixteen elements are kept as the eight first and the eight second ones of its pairs, whatever the
//     layout, so that a rotation is five packed operations for two pairs; a norm's factor comes last, where R_3's 1 / sqrt(d) is, and its weights lie in shared
//     memory (in registers they would cost a quarter of the warps).
//   - Angles: the table holds each frequency in turns per position as a 64-bit binary fraction.  position * fraction modulo 2^64 is the
//     turn modulo 1 (one 64-bit product, no range reduction; the fraction's own rounding leaves position * 2^-64), its top 32 bits go to sincospif.
//   - Lanes with the same place in their rows need the same angles: each computes its share of them and they hand them round.
// Measured in a graph of launches, heads of 128 in bf16: rotation of 16384 tokens of 32 + 8 heads 54 us (6.2 TB/s of 6.6), with R_3 65 us (5.1 TB/s: its
// exchanges, 2.5 of 4 instructions a cycle and the load/store pipe half busy); norm and rotation of 8192 tokens 35 us (4.8 TB/s: 24 warps an SM, 2.3 waves of
// blocks), its backward pass 54 us (4.6 TB/s: 16 warps an SM, a row of either input in flight each); some dozen tokens: 2.7 to 4 us, a launch.
// Every lane computing its own angles: 69 (R_3), 38 and 69 us.  Two warps a token, half of its heads each: 72, 36.6 and 77 us.
// Six blocks of four warps an SM leave 80 registers a thread (fp32: five blocks, 96): the normed kernels spill 92 to 172 bytes at that, the others up to 72.
// Rows that do not fit that scheme (head_dim not a multiple of 16 or without an instance below, half-layout pairs that do not lie in
// whole pieces, rows off 16-byte boundaries) take a kernel that keeps one row per warp in shared memory: 16384 tokens of 32 + 8 heads of 96, 24 of them
// rotated in halves, 182 us for 38 of bytes.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cfloat>
#include <cmath>

#include "../../include/conqur.h"

namespace {

using bf16 = __nv_bfloat16;

struct HeadsPtr {
  const void* in;
  void* out;
  const void* grad;
  int64_t in_b, in_t, in_h, out_b, out_t, out_h, grad_b, grad_t, grad_h;
  const void* weight;
  int heads;
};

struct HeadsArgs {
  HeadsPtr seg[2];                 // queries, keys
  int64_t n, tokens;               // rows per head in all, per sequence
  const int64_t* pos;
  int64_t pos_b;
  const unsigned long long* table;
  float* partial;                  // backward: one row of head_dim sums per block
  float eps, scale;                // scale: 1 / sqrt(head_dim), R_3
  int head_dim, rot, layout, hadamard, inverse, weight_bf16;
  int q_blocks;                    // backward: blocks [0, q_blocks) work on the queries, the others on the keys
};

enum { MODE_ROPE = 0, MODE_NORM = 1, MODE_GRAD = 2 };
constexpr int HEADS_THREADS = 128;
constexpr int HEADS_WARPS = HEADS_THREADS / 32;
constexpr float NORM_DOWN = 8.470329472543003e-22f;      // 2^-70
constexpr int GRAD_BLOCKS_MAX = 1184;      // 8 per SM: rows of partial weight gradients in the scratch

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// Eight consecutive elements, as 16-byte pieces.
template <typename T> struct Piece;
template <> struct Piece<bf16> {
  uint4 v;
  __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float* x) const {
    x[0] = lo_f(v.x); x[1] = hi_f(v.x); x[2] = lo_f(v.y); x[3] = hi_f(v.y);
    x[4] = lo_f(v.z); x[5] = hi_f(v.z); x[6] = lo_f(v.w); x[7] = hi_f(v.w);
  }
  static __device__ __forceinline__ void store(bf16* p, const float* x) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
  }
};
template <> struct Piece<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void get(float* x) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  static __device__ __forceinline__ void store(float* p, const float* x) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  }
};

__device__ __forceinline__ float load1(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ void store1(bf16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ float load_weight(const void* w, int bf, int i) {
  if (!w) return 1.f;
  return bf ? __bfloat162float(static_cast<const bf16*>(w)[i]) : static_cast<const float*>(w)[i];
}

// cos and sin of 2 pi * (position * turns mod 1).  The signed top half of the 64-bit product is the turn in [-1/2, 1/2) to 2^-32;
// rounded to fp32 it is off by at most 2^-26 of a turn.
__device__ __forceinline__ void angle(unsigned long long pos, unsigned long long turns, float amp, float& c, float& s) {
  const float x = (float)(int)(uint32_t)((pos * turns) >> 32) * 4.656612873077393e-10f;   // 2^-31: in half turns
  sincospif(x, &s, &c);
  c *= amp;
  s *= amp;
}

// Sum over a row's L consecutive lanes; every lane gets it.  `l`: the lane's place in its row.
template <int L>
__device__ __forceinline__ float row_sum(float v, int l, int lane) {
  if ((L & (L - 1)) == 0) {
#pragma unroll
    for (int m = 1; m < L; m <<= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    return v;
  }
  constexpr int P = L > 16 ? 16 : L > 8 ? 8 : L > 4 ? 4 : L > 2 ? 2 : 1;   // largest power of two below L
#pragma unroll
  for (int m = P; m >= 1; m >>= 1) {
    const float o = __shfl_down_sync(0xffffffffu, v, m);
    if (l < m && l + m < L) v += o;
  }
  return __shfl_sync(0xffffffffu, v, lane - l);
}

// A row is spread over D/16 lanes.
template <int D>
struct Row {
  static constexpr int L = D / 16;                 // lanes a row takes
  static constexpr int PER_WARP = 32 / L;          // rows a warp works on side by side
};

// ---- two fp32 at a time
using f2 = unsigned long long;
__device__ __forceinline__ f2 mk2(float lo, float hi) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ f2 mk2(float v) { return mk2(v, v); }
__device__ __forceinline__ void get2(f2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 sub2(f2 a, f2 b) {
  f2 r;
  asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float sum2(f2 v) {
  float a, b;
  get2(v, a, b);
  return a + b;
}

// A lane's sixteen elements: the first and the second elements of its eight pairs.  HALF: its two pieces; else the even and odd elements of both.
struct Pairs {
  f2 a[4], b[4];
};
template <bool HALF>
__device__ __forceinline__ Pairs pairs_of(const float (&x)[16]) {
  Pairs p;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    p.a[i] = HALF ? mk2(x[2 * i], x[2 * i + 1]) : mk2(x[4 * i], x[4 * i + 2]);
    p.b[i] = HALF ? mk2(x[8 + 2 * i], x[8 + 2 * i + 1]) : mk2(x[4 * i + 1], x[4 * i + 3]);
  }
  return p;
}
template <bool HALF>
__device__ __forceinline__ void pairs_to(const Pairs& p, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (HALF) {
      get2(p.a[i], x[2 * i], x[2 * i + 1]);
      get2(p.b[i], x[8 + 2 * i], x[8 + 2 * i + 1]);
    } else {
      get2(p.a[i], x[4 * i], x[4 * i + 2]);
      get2(p.b[i], x[4 * i + 1], x[4 * i + 3]);
    }
  }
}

// Without the 1 / sqrt(d).  (The levels may come in any order, and so may the elements of a lane.)
template <int L>
__device__ __forceinline__ void row_hadamard(Pairs& x, int l) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f2 s = add2(x.a[i], x.b[i]), d = sub2(x.a[i], x.b[i]);
    x.a[i] = s;
    x.b[i] = d;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    f2* v = k ? x.b : x.a;
#pragma unroll
    for (int m = 1; m < 4; m <<= 1)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!(i & m)) {
          const f2 s = add2(v[i], v[i | m]), d = sub2(v[i], v[i | m]);
          v[i] = s;
          v[i | m] = d;
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      get2(v[i], lo, hi);
      v[i] = mk2(lo + hi, lo - hi);
    }
#pragma unroll
    for (int m = 1; m < L; m <<= 1) {
      const f2 sgn = mk2((l & m) ? -1.f : 1.f);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float lo, hi;
        get2(v[i], lo, hi);
        lo = __shfl_xor_sync(0xffffffffu, lo, m);
        hi = __shfl_xor_sync(0xffffffffu, hi, m);
        v[i] = fma2(sgn, v[i], mk2(lo, hi));
      }
    }
  }
}

// Rows whose squares add up to more than an fp32 holds (rare; the whole warp comes here): scaled by 2^-70, beside which eps is nothing, they have a norm again.
// Returns the factor 1 / sqrt(mean x^2 + eps) that goes with what is left in x.
template <int L>
__device__ __forceinline__ float row_down(Pairs& x, float square, int l, int lane, float inv_d, float eps) {
  const bool big = !(square <= FLT_MAX);
  const f2 down = mk2(big ? NORM_DOWN : 1.f);
  f2 ss = 0ull;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x.a[i] = mul2(x.a[i], down);
    x.b[i] = mul2(x.b[i], down);
    ss = fma2(x.a[i], x.a[i], ss);
    ss = fma2(x.b[i], x.b[i], ss);
  }
  const float small = row_sum<L>(sum2(ss), l, lane);
  return rsqrtf(fmaf(big ? small : square, inv_d, big ? 0.f : eps));
}

// Pairs that do not turn keep to their own element (a sine of 0 would let what is not finite over); their cosine is the scale.
template <bool HALF>
__device__ __forceinline__ void row_spin(Pairs& x, const f2 (&c)[4], const f2 (&s)[4], uint32_t turned) {
  if (HALF && !turned) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x.a[i] = mul2(x.a[i], c[i]);
      x.b[i] = mul2(x.b[i], c[i]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f2 a = x.a[i], b = x.b[i];
    f2 u = sub2(mul2(a, c[i]), mul2(b, s[i])), v = fma2(a, s[i], mul2(b, c[i]));
    if (!HALF && turned != 0xFFu) {
      float u0, u1, v0, v1, a0, a1, b0, b1;
      get2(u, u0, u1);
      get2(v, v0, v1);
      get2(mul2(a, c[i]), a0, a1);
      get2(mul2(b, c[i]), b0, b1);
      const bool y = turned & (1u << (2 * i)), z = turned & (2u << (2 * i));
      u = mk2(y ? u0 : a0, z ? u1 : a1);
      v = mk2(y ? v0 : b0, z ? v1 : b1);
    }
    x.a[i] = u;
    x.b[i] = v;
  }
}

// A lane's two pieces of a row and the eight rotations they need.
struct LanePlan {
  int p0, p1;                       // first elements of the two pieces
  uint32_t turned;                  // which of its eight pairs rotate
  int f[2];                         // frequency of pair i < 4: f[0] + i, i >= 4: f[1] + i - 4
};
template <int D>
__device__ __forceinline__ LanePlan lane_plan(int l, int rot, int layout) {
  constexpr int L = D / 16;
  LanePlan q;
  if (layout == CONQUR_ROPE_HALF && rot > 0) {
    const int rp = rot >> 4;                                  // piece i of the first half pairs with piece i + rp
    int c0;
    if ((D & (D - 1)) == 0 && (rp & (rp - 1)) == 0) {         // a bit of the piece index becomes the register bit, for R_3
      const int b = 31 - __clz(rp);
      c0 = ((l >> b) << (b + 1)) | (l & (rp - 1));
      q.p1 = 8 * (c0 + rp);
    } else {
      c0 = l < rp ? l : 2 * rp + 2 * (l - rp);
      q.p1 = 8 * (l < rp ? l + rp : c0 + 1);
    }
    q.p0 = 8 * c0;
    q.turned = c0 < rp ? 0xFFu : 0u;
    q.f[0] = q.p0;
    q.f[1] = q.p0 + 4;
  } else {
    q.p0 = 8 * l;
    q.p1 = 8 * (l + L);
    q.f[0] = q.p0 >> 1;
    q.f[1] = q.p1 >> 1;
    q.turned = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (2 * (q.f[i >> 2] + (i & 3)) < rot) q.turned |= 1u << i;
  }
  return q;
}

__device__ __forceinline__ void token_of(const HeadsArgs& a, int64_t t, int64_t& b, int64_t& s) {
  b = 0;
  s = t;
  if (a.tokens != a.n) {
    b = t / a.tokens;
    s = t - b * a.tokens;
  }
}

// cos and sin of the lane's eight pairs (times the amplitude; the sine times `sign`); 1 and 0 where they do not turn.  Lanes with the same place in their
// rows need the same ones: each computes its share and they hand them round (the whole warp comes here).  `pos` counts only where something turns.
template <int D>
__device__ __forceinline__ void lane_angles(const HeadsArgs& a, unsigned long long pos, const LanePlan& q, int row, int l, float sign, f2 (&c)[4], f2 (&s)[4]) {
  constexpr int L = Row<D>::L, PW = Row<D>::PER_WARP, E = (8 + PW - 1) / PW;
  float cf[E], sf[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    cf[e] = 1.f;
    sf[e] = 0.f;
  }
  if (q.turned) {
    const float amp = (float)__longlong_as_double((long long)a.table[a.rot >> 1]);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = row * E + e;
      if (i < 8 && ((q.turned >> i) & 1u)) {
        angle(pos, a.table[(i < 4 ? q.f[0] : q.f[1]) + (i & 3)], amp, cf[e], sf[e]);
        sf[e] *= sign;
      }
    }
  }
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    cs[i] = __shfl_sync(0xffffffffu, cf[i % E], (i / E) * L + l);
    sn[i] = __shfl_sync(0xffffffffu, sf[i % E], (i / E) * L + l);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c[i] = mk2(cs[2 * i], cs[2 * i + 1]);
    s[i] = mk2(sn[2 * i], sn[2 * i + 1]);
  }
}

// Forward (and conqur_rope_heads' inverse).  Warp w of block x works on token HEADS_WARPS x + w; block row y of gridDim.y takes every gridDim.y-th group of
// Row<D>::PER_WARP heads (more than one only where the tokens alone would leave the GPU idle).  Two groups travel while one is worked on.
template <typename T, int D, bool NORM, bool HALF>
__global__ void __launch_bounds__(HEADS_THREADS, sizeof(T) == 2 ? 6 : 5) heads_kernel(const HeadsArgs a) {
  constexpr int L = Row<D>::L, PW = Row<D>::PER_WARP;
  __shared__ __align__(16) float weight[NORM ? 2 * D : 4];
  if (NORM) {
    for (int e = threadIdx.x; e < 2 * D; e += HEADS_THREADS) weight[e] = load_weight(a.seg[e >= D].weight, a.weight_bf16, e >= D ? e - D : e);
    __syncthreads();
  }
  const int lane = threadIdx.x & 31;
  const int row = lane / L, l = lane - row * L;
  const int64_t token = (int64_t)blockIdx.x * HEADS_WARPS + (threadIdx.x >> 5);
  if (token >= a.n) return;
  int64_t b, t;
  token_of(a, token, b, t);
  const LanePlan q = lane_plan<D>(l, a.rot, a.layout);
  const float scale = a.hadamard ? a.scale : 1.f;
  const bool before = !NORM && a.inverse && a.hadamard, after = a.hadamard && !before;
  const int nq = (a.seg[0].heads + PW - 1) / PW;
  int at = blockIdx.y;                                         // this block row's next group, queries first
  f2 c[4], s[4];
  bool have = false;
#pragma unroll 1
  for (int sg = 0; sg < 2; ++sg) {
    const HeadsPtr& g = a.seg[sg];
    const int groups = (g.heads + PW - 1) / PW;
    int it = sg ? at - nq : at;
    if (it >= groups) continue;
    const int64_t in_step = (int64_t)gridDim.y * PW * g.in_h, out_step = (int64_t)gridDim.y * PW * g.out_h;
    int h = it * PW + row;
    const int heads = row < PW ? g.heads : 0, h_step = gridDim.y * PW;
    const T* p = static_cast<const T*>(g.in) + b * g.in_b + t * g.in_t + h * g.in_h;
    T* o = static_cast<T*>(g.out) + b * g.out_b + t * g.out_t + h * g.out_h;
    Piece<T> r[2][2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (h + k * h_step < heads) {
        r[k][0].load(p + k * in_step + q.p0);
        r[k][1].load(p + k * in_step + q.p1);
      }
    if (!have) {
      lane_angles<D>(a, a.rot ? (unsigned long long)a.pos[b * a.pos_b + t] : 0ull, q, row, l, a.inverse ? -1.f : 1.f, c, s);
      have = true;
    }
    int k = 0;
#pragma unroll 2
    for (; it < groups; it += gridDim.y, k ^= 1) {
      float v[16];
      r[k][0].get(v);
      r[k][1].get(v + 8);
      Pairs x = pairs_of<HALF>(v);
      if (h + 2 * h_step < heads) {
        r[k][0].load(p + 2 * in_step + q.p0);
        r[k][1].load(p + 2 * in_step + q.p1);
      }
      float f = scale;
      if (NORM) {
        f2 ss = mul2(x.a[0], x.a[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) ss = fma2(x.a[i], x.a[i], ss);
#pragma unroll
        for (int i = 0; i < 4; ++i) ss = fma2(x.b[i], x.b[i], ss);
        const float square = row_sum<L>(sum2(ss), l, lane);
        if (__any_sync(0xffffffffu, h < heads && !(square <= FLT_MAX))) f *= row_down<L>(x, square, l, lane, 1.f / D, a.eps);
        else f *= rsqrtf(fmaf(square, 1.f / D, a.eps));
      }
      if (before) row_hadamard<L>(x, l);
      if (NORM) {
        Piece<float> w0, w1;
        w0.load(weight + sg * D + q.p0);
        w1.load(weight + sg * D + q.p1);
        w0.get(v); w1.get(v + 8);
        const Pairs w = pairs_of<HALF>(v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x.a[i] = mul2(x.a[i], w.a[i]);
          x.b[i] = mul2(x.b[i], w.b[i]);
        }
      }
      row_spin<HALF>(x, c, s, q.turned);
      if (after) row_hadamard<L>(x, l);
      if (NORM || a.hadamard) {
        const f2 f2v = mk2(f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x.a[i] = mul2(x.a[i], f2v);
          x.b[i] = mul2(x.b[i], f2v);
        }
      }
      if (h < heads) {
        pairs_to<HALF>(x, v);
        Piece<T>::store(o + q.p0, v);
        Piece<T>::store(o + q.p1, v + 8);
      }
      p += in_step;
      o += out_step;
      h += h_step;
    }
    at = sg ? at : it;                                         // the keys' groups go on in the same stride
  }
}

// Backward of the normed form.  With g = the gradient taken back through R_3 and the rotation, r = 1 / sqrt(mean x^2 + eps):
//   dw = sum over rows of g * x r        dx = r w g - x r (r^2 mean(w g x))
// A block works on the queries or on the keys; its warps walk tokens and keep their share of dw in registers.
template <typename T, int D, bool HALF>
__global__ void __launch_bounds__(HEADS_THREADS, sizeof(T) == 2 ? 4 : 3) heads_grad_kernel(const HeadsArgs a) {
  constexpr int L = Row<D>::L, PW = Row<D>::PER_WARP;
  __shared__ float sums[HEADS_WARPS][D];
  __shared__ __align__(16) float weight[D];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = lane / L, l = lane - row * L;
  const int sg = (int)blockIdx.x >= a.q_blocks;
  const int blk = sg ? blockIdx.x - a.q_blocks : blockIdx.x, blocks = sg ? gridDim.x - a.q_blocks : a.q_blocks;
  const HeadsPtr& g = a.seg[sg];
  const LanePlan q = lane_plan<D>(l, a.rot, a.layout);
  const int total = (g.heads + PW - 1) / PW;
  const float scale = a.hadamard ? a.scale : 1.f;
  Pairs dw;
#pragma unroll
  for (int i = 0; i < 4; ++i) dw.a[i] = dw.b[i] = 0ull;
  for (int e = threadIdx.x; e < D; e += HEADS_THREADS) weight[e] = load_weight(g.weight, a.weight_bf16, e);
  __syncthreads();
  // position and first rows of the next token travel while the present one is worked on
  const int64_t stride = (int64_t)blocks * HEADS_WARPS;
  int64_t token = (int64_t)blk * HEADS_WARPS + warp;
  const int heads = row < PW ? g.heads : 0;
  const T *xp = nullptr, *yp = nullptr;
  T* next_out = nullptr;
  unsigned long long pos = 0ull;
  Piece<T> x0, x1, y0, y1;
  int h = row;
  auto fetch = [&]() {
    x0.load(xp + q.p0);
    x1.load(xp + q.p1);
    y0.load(yp + q.p0);
    y1.load(yp + q.p1);
  };
  auto begin = [&](int64_t next) {
    int64_t b, t;
    token_of(a, next, b, t);
    xp = static_cast<const T*>(g.in) + b * g.in_b + t * g.in_t + row * g.in_h;
    yp = static_cast<const T*>(g.grad) + b * g.grad_b + t * g.grad_t + row * g.grad_h;
    next_out = static_cast<T*>(g.out) + b * g.out_b + t * g.out_t + row * g.out_h;
    if (a.rot) pos = (unsigned long long)a.pos[b * a.pos_b + t];
    h = row;
    if (h < heads) fetch();
  };
  if (token < a.n) begin(token);
  for (; token < a.n; token += stride) {
    T* op = next_out;
    f2 c[4], s[4];
    lane_angles<D>(a, pos, q, row, l, -1.f, c, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      c[i] = mul2(c[i], mk2(scale));
      s[i] = mul2(s[i], mk2(scale));
    }
#pragma unroll 1
    for (int it = 0; it < total; ++it) {
      float v[16];
      x0.get(v); x1.get(v + 8);
      Pairs x = pairs_of<HALF>(v);
      y0.get(v); y1.get(v + 8);
      Pairs y = pairs_of<HALF>(v);
      const bool now = h < heads;
      h += PW;
      xp += PW * g.in_h;
      yp += PW * g.grad_h;
      if (it + 1 < total) {
        if (h < heads) fetch();
      } else if (token + stride < a.n) {
        begin(token + stride);
      }
      f2 ss = mul2(x.a[0], x.a[0]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i) ss = fma2(x.a[i], x.a[i], ss);
        ss = fma2(x.b[i], x.b[i], ss);
      }
      const float square = row_sum<L>(sum2(ss), l, lane);
      float r = rsqrtf(fmaf(square, 1.f / D, a.eps));
      float down = 1.f;
      if (__any_sync(0xffffffffu, now && !(square <= FLT_MAX))) {
        r = row_down<L>(x, square, l, lane, 1.f / D, a.eps);
        down = square <= FLT_MAX ? 1.f : NORM_DOWN;
      }
      if (a.hadamard) row_hadamard<L>(y, l);
      row_spin<HALF>(y, c, s, q.turned);
      Piece<float> w0, w1;                                     // (shared memory: sixteen registers less)
      w0.load(weight + q.p0);
      w1.load(weight + q.p1);
      w0.get(v); w1.get(v + 8);
      const Pairs w = pairs_of<HALF>(v);
      f2 sx = 0ull;
      Pairs wy;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        wy.a[i] = mul2(w.a[i], y.a[i]);
        wy.b[i] = mul2(w.b[i], y.b[i]);
        sx = fma2(wy.a[i], x.a[i], sx);
        sx = fma2(wy.b[i], x.b[i], sx);
      }
      const float k = -row_sum<L>(sum2(sx), l, lane) * (1.f / D) * r * (r * down);
      if (now) {
        const f2 r2 = mk2(r), d2 = mk2(r * down), k2 = mk2(k);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x.a[i] = mul2(x.a[i], r2);
          x.b[i] = mul2(x.b[i], r2);
          dw.a[i] = fma2(y.a[i], x.a[i], dw.a[i]);
          dw.b[i] = fma2(y.b[i], x.b[i], dw.b[i]);
          y.a[i] = fma2(x.a[i], k2, mul2(wy.a[i], d2));
          y.b[i] = fma2(x.b[i], k2, mul2(wy.b[i], d2));
        }
        pairs_to<HALF>(y, v);
        Piece<T>::store(op + q.p0, v);
        Piece<T>::store(op + q.p1, v + 8);
      }
      op += PW * g.out_h;
    }
  }
  // rows of the warp, then warps of the block, in a fixed order
  float d[16];
  pairs_to<HALF>(dw, d);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float v = d[i];
#pragma unroll
    for (int j = 1; j < PW; ++j) {
      const float o = __shfl_sync(0xffffffffu, d[i], (j * L + l) & 31);
      v += o;
    }
    if (row == 0) sums[warp][(i < 8 ? q.p0 : q.p1) + (i & 7)] = v;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < D; e += HEADS_THREADS) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < HEADS_WARPS; ++k) v += sums[k][e];
    a.partial[(int64_t)blockIdx.x * D + e] = v;
  }
}

// Weight gradients from the blocks' rows: 32 columns and 32 shares of the rows a block, summed in a fixed order.
__global__ void __launch_bounds__(1024) heads_weight_kernel(const float* __restrict__ partial, int head_dim, int q_blocks, int k_blocks,
                                                            float* dq, float* dk) {
  __shared__ float part[32][33];
  float* out = blockIdx.y ? dk : dq;
  if (!out) return;
  const int first = blockIdx.y ? q_blocks : 0, count = blockIdx.y ? k_blocks : q_blocks;
  const int e = blockIdx.x * 32 + (threadIdx.x & 31), share = threadIdx.x >> 5;
  float v = 0.f;
  if (e < head_dim)
    for (int i = share; i < count; i += 32) v += partial[(int64_t)(first + i) * head_dim + e];
  part[share][threadIdx.x & 31] = v;
  __syncthreads();
  if (share == 0 && e < head_dim) {
    v = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v += part[i][threadIdx.x];
    out[e] = v;
  }
}

// Any head_dim up to 512, any even rotary_dim, any alignment: a warp takes one token and keeps one row at a time in shared memory.
// MODE_GRAD: as heads_grad_kernel.
template <typename T, int MODE>
__global__ void __launch_bounds__(HEADS_THREADS) heads_general_kernel(const HeadsArgs a) {
  extern __shared__ float sm[];
  const int D = a.head_dim, half = a.rot >> 1;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float* buf = sm + warp * (D + 2 * half);
  float* cs = buf + D;
  float* sn = cs + half;
  int first_seg = 0, last_seg = 1;
  int64_t blk = blockIdx.x, blocks = gridDim.x;
  if (MODE == MODE_GRAD) {
    first_seg = last_seg = (int)blockIdx.x >= a.q_blocks;
    blk = first_seg ? blockIdx.x - a.q_blocks : blockIdx.x;
    blocks = first_seg ? gridDim.x - a.q_blocks : a.q_blocks;
  }
  const float inv = 1.f / (float)D;
  float dw[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) dw[j] = 0.f;

  auto rotate = [&](float sign) {
    for (int i = lane; i < half; i += 32) {
      const int ia = a.layout == CONQUR_ROPE_HALF ? i : 2 * i, ib = a.layout == CONQUR_ROPE_HALF ? i + half : 2 * i + 1;
      const float u = buf[ia], v = buf[ib], c = cs[i], s = sign * sn[i];
      buf[ia] = fmaf(u, c, -v * s);
      buf[ib] = fmaf(u, s, v * c);
    }
    __syncwarp();
  };
  auto hadamard = [&]() {
    for (int m = 1; m < D; m <<= 1) {
      for (int i = lane; i < D / 2; i += 32) {
        const int ia = ((i & ~(m - 1)) << 1) | (i & (m - 1));
        const float u = buf[ia], v = buf[ia | m];
        buf[ia] = u + v;
        buf[ia | m] = u - v;
      }
      __syncwarp();
    }
    for (int i = lane; i < D; i += 32) buf[i] *= a.scale;
    __syncwarp();
  };
  auto warp_sum = [](float v) {
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    return v;
  };

  for (int64_t token = blk * HEADS_WARPS + warp; token < a.n; token += blocks * HEADS_WARPS) {
    int64_t b, t;
    token_of(a, token, b, t);
    if (half) {
      const unsigned long long pos = (unsigned long long)a.pos[b * a.pos_b + t];
      const float amp = (float)__longlong_as_double((long long)a.table[half]);
      for (int i = lane; i < half; i += 32) angle(pos, a.table[i], amp, cs[i], sn[i]);
      __syncwarp();
    }
    for (int sg = first_seg; sg <= last_seg; ++sg) {
      const HeadsPtr& g = a.seg[sg];
      for (int h = MODE == MODE_GRAD ? 0 : blockIdx.y; h < g.heads; h += MODE == MODE_GRAD ? 1 : gridDim.y) {
        const T* xp = static_cast<const T*>(g.in) + b * g.in_b + t * g.in_t + h * g.in_h;
        T* op = static_cast<T*>(g.out) + b * g.out_b + t * g.out_t + h * g.out_h;
        float x[16];
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int e = lane + 32 * j;
          x[j] = e < D ? load1(xp + e) : 0.f;
          ss = fmaf(x[j], x[j], ss);
        }
        float down = 1.f;                                      // as in row_down
        if (MODE != MODE_ROPE) {
          ss = warp_sum(ss);
          if (!(ss <= FLT_MAX)) {
            down = NORM_DOWN;
            ss = 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              x[j] *= down;
              ss = fmaf(x[j], x[j], ss);
            }
            ss = warp_sum(ss);
          }
        }
        const float r = MODE == MODE_ROPE ? 1.f : 1.f / sqrtf(ss * inv + a.eps * (down * down));
        if (MODE == MODE_GRAD) {
          const T* yp = static_cast<const T*>(g.grad) + b * g.grad_b + t * g.grad_t + h * g.grad_h;
          for (int e = lane; e < D; e += 32) buf[e] = load1(yp + e);
          __syncwarp();
          if (a.hadamard) hadamard();
          rotate(-1.f);
          float sx = 0.f;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int e = lane + 32 * j;
            if (e < D) sx = fmaf(load_weight(g.weight, a.weight_bf16, e) * buf[e], x[j], sx);
          }
          sx = warp_sum(sx);
          const float k = sx * inv * r * r;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int e = lane + 32 * j;
            if (e < D) {
              const float y = buf[e];
              dw[j] = fmaf(y, x[j] * r, dw[j]);
              store1(op + e, r * down * fmaf(load_weight(g.weight, a.weight_bf16, e), y, -x[j] * k));
            }
          }
          __syncwarp();
          continue;
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int e = lane + 32 * j;
          if (e < D) buf[e] = MODE == MODE_NORM ? x[j] * (r * load_weight(g.weight, a.weight_bf16, e)) : x[j];
        }
        __syncwarp();
        if (a.inverse) {
          if (a.hadamard) hadamard();
          rotate(-1.f);
        } else {
          rotate(1.f);
          if (a.hadamard) hadamard();
        }
        for (int e = lane; e < D; e += 32) store1(op + e, buf[e]);
        __syncwarp();
      }
    }
    __syncwarp();
  }
  if (MODE == MODE_GRAD) {
    // the warps' rows, in a fixed order
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int e = lane + 32 * j;
      if (e < D) buf[e] = dw[j];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < D; e += HEADS_THREADS) {
      float v = 0.f;
      for (int k = 0; k < HEADS_WARPS; ++k) v += sm[k * (D + 2 * half) + e];
      a.partial[(int64_t)blockIdx.x * D + e] = v;
    }
  }
}

struct RopeTable { unsigned long long word[257]; };
__global__ void rope_table_kernel(const RopeTable t, int words, unsigned long long* out) {
  for (int i = threadIdx.x; i < words; i += blockDim.x) out[i] = t.word[i];
}

// ---------------------------------------------------------------------------------------------------- host

bool rope_config_ok(const conqur_rope_config* c) {
  if (!c || c->struct_size != sizeof(conqur_rope_config) || c->reserved != 0) return false;
  if (c->rotary_dim < 2 || c->rotary_dim > 512 || (c->rotary_dim & 1)) return false;
  if (c->scaling < CONQUR_ROPE_SCALE_NONE || c->scaling > CONQUR_ROPE_SCALE_RAMP) return false;
  if (!(c->theta > 1.0) || !std::isfinite(c->theta)) return false;
  if (c->scaling != CONQUR_ROPE_SCALE_NONE && (!(c->factor >= 1.0) || !std::isfinite(c->factor))) return false;
  if (c->scaling == CONQUR_ROPE_SCALE_NTK && c->rotary_dim == 2 && c->factor != 1.0) return false;   // r / (r - 2)
  if (c->scaling >= CONQUR_ROPE_SCALE_BANDS &&
      (!(c->low > 0.0) || !(c->high > c->low) || !std::isfinite(c->high) || c->original < 1))
    return false;
  return true;
}

// Frequencies in extended precision: what is held of them, 64 bits of a turn, keeps its last bits at far positions.
void rope_frequencies(const conqur_rope_config* c, long double* f, double* amp) {
  const long double two_pi = 6.283185307179586476925286766559005768L;
  const int r = c->rotary_dim;
  long double log_theta = logl((long double)c->theta);
  const long double factor = (long double)c->factor;
  if (c->scaling == CONQUR_ROPE_SCALE_NTK && r > 2) log_theta += logl(factor) * r / (r - 2);
  long double a = 0, b = 0;
  *amp = 1.0;
  if (c->scaling == CONQUR_ROPE_SCALE_RAMP) {
    auto dim = [&](double turns) { return r * logl((long double)c->original / (two_pi * turns)) / (2 * log_theta); };
    a = fmaxl(floorl(dim(c->high)), 0);
    b = fminl(ceill(dim(c->low)), r - 1);
    *amp = 1.0 + 0.1 * std::log(c->factor);
  }
  for (int i = 0; i < r / 2; ++i) {
    long double v = expl(-log_theta * 2 * i / r);
    if (c->scaling == CONQUR_ROPE_SCALE_LINEAR) v /= factor;
    if (c->scaling == CONQUR_ROPE_SCALE_BANDS) {
      const long double turns = (long double)c->original * v / two_pi;
      const long double keep = fminl(fmaxl((turns - c->low) / ((long double)c->high - c->low), 0), 1);
      v *= keep + (1 - keep) / factor;
    }
    if (c->scaling == CONQUR_ROPE_SCALE_RAMP) {
      const long double g = fminl(fmaxl((i - a) / fmaxl(b - a, 0.001L), 0), 1);
      v = v * (1 - g) + v / factor * g;
    }
    f[i] = v;
  }
}

int device_sms() {
  static std::atomic<int> known[64];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  int n = known[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    known[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

int launched() { return cudaGetLastError() == cudaSuccess ? CONQUR_OK : CONQUR_ERR_CUDA; }

bool aligned16(const conqur_heads& h, int elem) {
  return ((reinterpret_cast<uintptr_t>(h.data_dev) | (uintptr_t)(h.batch_stride * elem) | (uintptr_t)(h.token_stride * elem) |
           (uintptr_t)(h.head_stride * elem)) & 15) == 0;
}

// Checks and translates a call; `grad`: the backward pass.
int heads_args(const conqur_heads_call* c, bool norm, bool grad, HeadsArgs& a, bool& vec) {
  if (!c || c->struct_size != sizeof(conqur_heads_call)) return CONQUR_ERR_INVALID_ARG;
  if (c->dtype != CONQUR_F32 && c->dtype != CONQUR_BF16) return CONQUR_ERR_INVALID_ARG;
  if (c->head_dim < 1 || c->head_dim > 512 || c->rotary_dim < 0 || (c->rotary_dim & 1) || c->rotary_dim > c->head_dim) return CONQUR_ERR_INVALID_ARG;
  if (c->layout != CONQUR_ROPE_HALF && c->layout != CONQUR_ROPE_INTERLEAVED) return CONQUR_ERR_INVALID_ARG;
  if (c->flags & ~(CONQUR_HEADS_HADAMARD | CONQUR_HEADS_INVERSE)) return CONQUR_ERR_INVALID_ARG;
  if ((c->flags & CONQUR_HEADS_HADAMARD) && (c->head_dim < 4 || (c->head_dim & (c->head_dim - 1)))) return CONQUR_ERR_INVALID_ARG;
  if (norm && ((c->flags & CONQUR_HEADS_INVERSE) || !(c->eps > 0.f) || !std::isfinite(c->eps))) return CONQUR_ERR_INVALID_ARG;
  if (norm && c->weight_dtype != CONQUR_F32 && c->weight_dtype != CONQUR_BF16) return CONQUR_ERR_INVALID_ARG;
  if (c->q_heads < 1 || c->k_heads < 0 || c->q_heads > 65536 || c->k_heads > 65536) return CONQUR_ERR_INVALID_ARG;
  if (c->batch < 0 || c->tokens < 0 || (c->tokens > 0 && c->batch > (int64_t)0x7fffffff / c->tokens)) return CONQUR_ERR_INVALID_ARG;
  const int64_t n = c->batch * c->tokens;
  if (n > 0) {
    if (c->rotary_dim > 0 && (!c->positions_dev || !c->table_dev || (reinterpret_cast<uintptr_t>(c->table_dev) & 7) ||
                              (reinterpret_cast<uintptr_t>(c->positions_dev) & 7)))
      return CONQUR_ERR_INVALID_ARG;
  }
  const int elem = c->dtype == CONQUR_F32 ? 4 : 2;
  vec = true;
  for (int i = 0; i < 2; ++i) {
    const conqur_heads &in = i ? c->k_in : c->q_in, &out = i ? c->k_out : c->q_out, &gr = i ? c->k_grad : c->q_grad;
    HeadsPtr& p = a.seg[i];
    p.heads = i ? c->k_heads : c->q_heads;
    if (p.heads == 0) { p = HeadsPtr{}; continue; }
    if (n > 0 && (!in.data_dev || !out.data_dev || (grad && !gr.data_dev))) return CONQUR_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(in.data_dev) | reinterpret_cast<uintptr_t>(out.data_dev) | (grad ? reinterpret_cast<uintptr_t>(gr.data_dev) : 0)) & (elem - 1))
      return CONQUR_ERR_INVALID_ARG;
    p.in = in.data_dev; p.out = out.data_dev; p.grad = grad ? gr.data_dev : nullptr;
    p.in_b = in.batch_stride; p.in_t = in.token_stride; p.in_h = in.head_stride;
    p.out_b = out.batch_stride; p.out_t = out.token_stride; p.out_h = out.head_stride;
    p.grad_b = gr.batch_stride; p.grad_t = gr.token_stride; p.grad_h = gr.head_stride;
    p.weight = norm ? (i ? c->k_weight_dev : c->q_weight_dev) : nullptr;
    if (p.weight && (reinterpret_cast<uintptr_t>(p.weight) & (c->weight_dtype == CONQUR_F32 ? 3 : 1))) return CONQUR_ERR_INVALID_ARG;
    // every element of an output has a place of its own
    if ((p.heads > 1 && out.head_stride == 0) || (c->tokens > 1 && out.token_stride == 0) || (c->batch > 1 && out.batch_stride == 0)) return CONQUR_ERR_INVALID_ARG;
    vec = vec && aligned16(in, elem) && aligned16(out, elem) && (!grad || aligned16(gr, elem));
  }
  a.n = n; a.tokens = c->tokens;
  a.pos = c->positions_dev; a.pos_b = c->positions_batch_stride;
  a.table = static_cast<const unsigned long long*>(c->table_dev);
  a.partial = nullptr;
  a.eps = c->eps; a.scale = (float)(1.0 / sqrt((double)c->head_dim));
  a.head_dim = c->head_dim; a.rot = c->rotary_dim; a.layout = c->layout;
  a.hadamard = (c->flags & CONQUR_HEADS_HADAMARD) != 0; a.inverse = (c->flags & CONQUR_HEADS_INVERSE) != 0;
  a.weight_bf16 = c->weight_dtype == CONQUR_BF16;
  a.q_blocks = 0;
  // half-layout pairs have to lie in whole pieces, and with R_3 in pieces that differ in one bit of their number
  if (c->layout == CONQUR_ROPE_HALF && (c->rotary_dim & 15)) vec = false;
  if (a.hadamard && c->layout == CONQUR_ROPE_HALF && (c->rotary_dim & (c->rotary_dim - 1))) vec = false;
  return CONQUR_OK;
}

// Calls f with the head_dim as a constant where it has an instance; false where not.
template <typename F>
bool with_dim(int d, F&& f) {
  switch (d) {
    case 64: f(std::integral_constant<int, 64>()); return true;
    case 80: f(std::integral_constant<int, 80>()); return true;
    case 96: f(std::integral_constant<int, 96>()); return true;
    case 112: f(std::integral_constant<int, 112>()); return true;
    case 128: f(std::integral_constant<int, 128>()); return true;
    case 192: f(std::integral_constant<int, 192>()); return true;
    case 256: f(std::integral_constant<int, 256>()); return true;
    default: return false;
  }
}

size_t general_smem(const HeadsArgs& a) { return sizeof(float) * HEADS_WARPS * (a.head_dim + 2 * (a.rot >> 1)); }

template <typename T, bool NORM>
int forward(const HeadsArgs& a, bool vec, cudaStream_t s) {
  const int sms = device_sms();
  if (!sms) return CONQUR_ERR_CUDA;
  const int64_t blocks = (a.n + HEADS_WARPS - 1) / HEADS_WARPS;
  // few tokens: their heads go to several warps, up to 24 warps an SM
  const int64_t want = (24ll * sms + a.n - 1) / a.n;
  bool done = false;
  if (vec)
    done = with_dim(a.head_dim, [&](auto d) {
      constexpr int D = decltype(d)::value, PW = Row<D>::PER_WARP;
      const int total = (a.seg[0].heads + PW - 1) / PW + (a.seg[1].heads + PW - 1) / PW;
      const int split = (int)(want < total ? want : total);
      if (a.layout == CONQUR_ROPE_HALF && a.rot) heads_kernel<T, D, NORM, true><<<dim3((unsigned)blocks, split), HEADS_THREADS, 0, s>>>(a);
      else heads_kernel<T, D, NORM, false><<<dim3((unsigned)blocks, split), HEADS_THREADS, 0, s>>>(a);
    });
  if (!done) {
    const int most = a.seg[0].heads > a.seg[1].heads ? a.seg[0].heads : a.seg[1].heads;
    const int split = (int)(want < most ? want : most);
    heads_general_kernel<T, NORM ? MODE_NORM : MODE_ROPE><<<dim3((unsigned)blocks, split), HEADS_THREADS, general_smem(a), s>>>(a);
  }
  return launched();
}

template <typename T>
int backward(HeadsArgs a, bool vec, float* dq, float* dk, cudaStream_t s) {
  const int sms = device_sms();
  if (!sms) return CONQUR_ERR_CUDA;
  int qb = 0, kb = 0;
  if (a.n > 0) {
    // as many blocks as stay resident, shared out in proportion to the heads; fewer where there are few tokens
    const int most = sms * (sizeof(T) == 2 ? 4 : 3) < GRAD_BLOCKS_MAX ? sms * (sizeof(T) == 2 ? 4 : 3) : GRAD_BLOCKS_MAX;
    const int64_t each = (a.n + HEADS_WARPS - 1) / HEADS_WARPS;
    const int hq = a.seg[0].heads, hk = a.seg[1].heads;
    kb = hk ? (int)((int64_t)most * hk / (hq + hk)) : 0;
    if (hk && kb < 1) kb = 1;
    qb = most - kb;
    if (qb < 1) qb = 1;
    if (qb > each) qb = (int)each;
    if (kb > each) kb = (int)each;
    a.q_blocks = qb;
    bool done = false;
    if (vec)
      done = with_dim(a.head_dim, [&](auto d) {
        if (a.layout == CONQUR_ROPE_HALF && a.rot) heads_grad_kernel<T, decltype(d)::value, true><<<qb + kb, HEADS_THREADS, 0, s>>>(a);
        else heads_grad_kernel<T, decltype(d)::value, false><<<qb + kb, HEADS_THREADS, 0, s>>>(a);
      });
    if (!done) heads_general_kernel<T, MODE_GRAD><<<qb + kb, HEADS_THREADS, general_smem(a), s>>>(a);
    const int rc = launched();
    if (rc != CONQUR_OK) return rc;
  }
  if (!dq && !dk) return CONQUR_OK;
  heads_weight_kernel<<<dim3((a.head_dim + 31) / 32, 2), 1024, 0, s>>>(a.partial, a.head_dim, qb, kb, dq, dk);
  return launched();
}

}  // namespace

extern "C" int conqur_rope_frequencies(const conqur_rope_config* cfg, double* freq_out, double* amplitude_out) {
  if (!rope_config_ok(cfg) || !freq_out || !amplitude_out) return CONQUR_ERR_INVALID_ARG;
  long double f[256];
  rope_frequencies(cfg, f, amplitude_out);
  for (int i = 0; i < cfg->rotary_dim / 2; ++i) freq_out[i] = (double)f[i];
  return CONQUR_OK;
}

extern "C" size_t conqur_rope_table_bytes(const conqur_rope_config* cfg) {
  return rope_config_ok(cfg) ? 8 * (size_t)(cfg->rotary_dim / 2 + 1) : 0;
}

extern "C" int conqur_rope_table(const conqur_rope_config* cfg, void* table_dev, void* cuda_stream) {
  if (!rope_config_ok(cfg) || !table_dev || (reinterpret_cast<uintptr_t>(table_dev) & 7)) return CONQUR_ERR_INVALID_ARG;
  long double f[256];
  double amp;
  rope_frequencies(cfg, f, &amp);
  const int half = cfg->rotary_dim / 2;
  RopeTable t = {};
  for (int i = 0; i < half; ++i) {
    // f < 2 pi, so the turn is a fraction; what rounds up to 2^64 is a whole turn
    const long double turn = f[i] / 6.283185307179586476925286766559005768L;
    const long double scaled = roundl(ldexpl(turn - floorl(turn), 64));
    t.word[i] = scaled >= 18446744073709551616.0L ? 0ull : (unsigned long long)scaled;
  }
  static_assert(sizeof(double) == sizeof(unsigned long long), "the amplitude's bits take one word");
  __builtin_memcpy(&t.word[half], &amp, sizeof(double));
  rope_table_kernel<<<1, 128, 0, static_cast<cudaStream_t>(cuda_stream)>>>(t, half + 1, static_cast<unsigned long long*>(table_dev));
  return launched();
}

extern "C" int conqur_rope_heads(const conqur_heads_call* call, void* cuda_stream) {
  HeadsArgs a;
  bool vec;
  const int rc = heads_args(call, false, false, a, vec);
  if (rc != CONQUR_OK || a.n == 0) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return call->dtype == CONQUR_F32 ? forward<float, false>(a, vec, s) : forward<bf16, false>(a, vec, s);
}

extern "C" int conqur_norm_rope_heads(const conqur_heads_call* call, void* cuda_stream) {
  HeadsArgs a;
  bool vec;
  const int rc = heads_args(call, true, false, a, vec);
  if (rc != CONQUR_OK || a.n == 0) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return call->dtype == CONQUR_F32 ? forward<float, true>(a, vec, s) : forward<bf16, true>(a, vec, s);
}

extern "C" size_t conqur_norm_rope_backward_scratch_bytes(int32_t head_dim) {
  return head_dim < 1 || head_dim > 512 ? 0 : sizeof(float) * GRAD_BLOCKS_MAX * (size_t)head_dim;
}

extern "C" int conqur_norm_rope_heads_backward(const conqur_heads_call* call, void* scratch_dev, size_t scratch_bytes, void* cuda_stream) {
  HeadsArgs a;
  bool vec;
  const int rc = heads_args(call, true, true, a, vec);
  if (rc != CONQUR_OK) return rc;
  if (!scratch_dev || (reinterpret_cast<uintptr_t>(scratch_dev) & 255)) return CONQUR_ERR_INVALID_ARG;
  if (scratch_bytes < conqur_norm_rope_backward_scratch_bytes(call->head_dim)) return CONQUR_ERR_WORKSPACE_TOO_SMALL;
  float *dq = call->dq_weight_dev, *dk = call->k_heads ? call->dk_weight_dev : nullptr;
  if ((reinterpret_cast<uintptr_t>(dq) | reinterpret_cast<uintptr_t>(dk)) & 3) return CONQUR_ERR_INVALID_ARG;
  a.partial = static_cast<float*>(scratch_dev);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return call->dtype == CONQUR_F32 ? backward<float>(a, vec, dq, dk, s) : backward<bf16>(a, vec, dq, dk, s);
}
