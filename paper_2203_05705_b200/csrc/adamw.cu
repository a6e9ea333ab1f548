// The optimiser's step over many tensors at once, and the norm of all gradients with the factor that clips them.
//
// Both are one pass over memory: per element the step reads p, g, m, v and writes p, m, v and the bf16 copy (28 to 30
// bytes with states in 32 bits, 16 to 18 in 8).  The table of tensors travels as a kernel parameter: nothing is copied
// or allocated per call.
#include <cuda_fp8.h>

#include "ard_internal.h"
#include "philox.h"
#include "sm100_ptx.h"

namespace {

constexpr int AW_THREADS = 256;
constexpr float E4M3_MAX = 448.f;
constexpr float AW_TINY = 7.70371977754894341e-34f;  // 2^-110

struct AwEntry {
  float* p;
  const void* g;
  __nv_bfloat16* w;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  long long n, cols, ldp, ldg, ldw;
  unsigned long long tile0;  // tiles of the tensors before this one
  float decay;
  unsigned number;           // 1 + place in the caller's table
  int g_is_bf16;
  int flat;                  // no gaps between rows, all pointers (but the scales') on 16 bytes: read and written in pieces of 4 elements
  int scales16;              // the scales too: they come with the bulk copies
};

template <int CAP>
struct AwTable {
  AwEntry e[CAP];
  int n;
  unsigned long long tiles;
};

// Tables travel in the launch: the small one keeps a launch over a handful of tensors as cheap as any other, the large
// one (26 KB of the 32 KB that parameters may have) takes a network's.
constexpr int AW_SMALL = 16, AW_LARGE = 216;

struct AwArgs {
  float lr, beta1, beta2, one_minus_beta1, one_minus_beta2, eps;
  float one;                // 1, as something that the compiler does not know
  float lift1, root_lift2;  // 1 / (1 - beta1^t) and the root of 1 / (1 - beta2^t), where the host knows t
  double ln_beta1, ln_beta2;
  uint32_t keys[20];  // the generator's, of its ten rounds: read where they are used, not carried in registers
  unsigned long long step;
  const unsigned long long* counter;
  const float* lr_factor;
  const float* grad_factor;
};

template <int CAP>
__device__ __forceinline__ int aw_find(const AwTable<CAP>& t, unsigned long long tile) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].tile0 <= tile) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Four elements i .. i+3 of a tensor's flat order; elements from n on are 0 and are not written.
__device__ __forceinline__ void aw_load4(const float* x, long long i, long long n, long long cols, long long ld, bool flat, float (&v)[4]) {
  if (flat && i + 4 <= n) {
    const float4 q = *reinterpret_cast<const float4*>(x + i);
    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    v[k] = i + k < n ? x[cols == ld ? i + k : (i + k) / cols * ld + (i + k) % cols] : 0.f;
}
__device__ __forceinline__ void aw_load4(const __nv_bfloat16* x, long long i, long long n, long long cols, long long ld, bool flat,
                                         float (&v)[4]) {
  if (flat && i + 4 <= n) {
    const uint2 q = *reinterpret_cast<const uint2*>(x + i);
    v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xFFFF0000u);
    v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xFFFF0000u);
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    v[k] = i + k < n ? __bfloat162float(x[cols == ld ? i + k : (i + k) / cols * ld + (i + k) % cols]) : 0.f;
}
__device__ __forceinline__ void aw_store4(float* x, long long i, long long n, long long cols, long long ld, bool flat, const float (&v)[4]) {
  if (flat && i + 4 <= n) {
    *reinterpret_cast<float4*>(x + i) = make_float4(v[0], v[1], v[2], v[3]);
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (i + k < n) x[cols == ld ? i + k : (i + k) / cols * ld + (i + k) % cols] = v[k];
}
__device__ __forceinline__ void aw_store4(__nv_bfloat16* x, long long i, long long n, long long cols, long long ld, bool flat,
                                          const float (&v)[4]) {
  if (flat && i + 4 <= n) {
    __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    uint2 q;
    q.x = *reinterpret_cast<uint32_t*>(&a);
    q.y = *reinterpret_cast<uint32_t*>(&b);
    *reinterpret_cast<uint2*>(x + i) = q;
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (i + k < n) x[cols == ld ? i + k : (i + k) / cols * ld + (i + k) % cols] = __float2bfloat16(v[k]);
}

// Four 8-bit floats.  Their blocks begin at the state's first byte, which need not lie on 4 bytes.
__device__ __forceinline__ uint32_t aw_load_codes(const uint8_t* x, long long i, long long n, bool wide) {
  if (wide && i + 4 <= n) return *reinterpret_cast<const uint32_t*>(x + i);
  uint32_t q = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (i + k < n) q |= (uint32_t)x[i + k] << (8 * k);
  return q;
}
__device__ __forceinline__ void aw_store_codes(uint8_t* x, long long i, long long n, bool wide, uint32_t q) {
  if (wide && i + 4 <= n) {
    *reinterpret_cast<uint32_t*>(x + i) = q;
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (i + k < n) x[i + k] = (uint8_t)(q >> (8 * k));
}
__device__ __forceinline__ void aw_decode(uint32_t q, float scale, float (&v)[4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(q >> (16 * h)), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r));
    v[2 * h] = f.x * scale;
    v[2 * h + 1] = f.y * scale;
  }
}

// sqrt(x) and 1 / x as the instructions approximate them, to a unit or two in the last place: rounded to the last bit
// they take 8 to 20 instructions each, with their special cases, and the kernel with states in 8 bits runs out of issue
// slots.
__device__ __forceinline__ float aw_root(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float aw_inverse(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Two elements in one instruction.
__device__ __forceinline__ float2 operator*(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 operator+(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 aw_fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 aw_both(float x) { return make_float2(x, x); }
// Roots to the last bit: one of Heron's steps with its residual in one rounding (Markstein, IBM J. Res. Dev. 34, 1990),
// from the instruction's estimate of 1 / sqrt(x), which takes subnormals (of those a unit or two in the last place).
// No branches: they keep a thread's quads from running beside one another. Of 0 and infinity the step gives NaN, which
// the maximum with 2^-66 x, less than the root of any other finite x, puts right; NaN stays what it is.
__device__ __forceinline__ float2 aw_roots(float2 x) {
  float2 y;
  asm("rsqrt.approx.f32 %0, %1;" : "=f"(y.x) : "f"(x.x));
  asm("rsqrt.approx.f32 %0, %1;" : "=f"(y.y) : "f"(x.y));
  const float2 q = x * y, r = aw_fma(aw_fma(q * aw_both(-1.f), q, x), y * aw_both(0.5f), q), less = x * aw_both(1.35525272e-20f);
  return make_float2(fmaxf(r.x, less.x), fmaxf(r.y, less.y));
}

// The 8-bit floats of a block of 128 values, four in each lane, and its scale (the same in all lanes).  ROOT: of values
// >= 0, from the words' high halves; else from their low halves. A value is rounded to the grid of the 8-bit floats (3
// bits of mantissa; steps of 2^-9 below 2^-6), up with the probability of what is cut off, which 16 random bits resolve
// to 2^-16 of a step: those bits are added below the mantissa's three, and all bits there cut off.  (Half a step less
// and the conversion's rounding to nearest in place of the cut would be wrong where a sum passes 2^-5.)  Below 2^-6 the
// grid is that of [2^-6, 2^-5): adding 2^-6 puts the value there.  Sums carry into the exponent where they should.
// What passes 448 the conversion cuts off.
template <bool ROOT>
__device__ __forceinline__ uint32_t aw_encode(const float2 (&v)[2], const uint32_t (&words)[4], float& scale) {
  float most = fmaxf(fmaxf(fabsf(v[0].x), fabsf(v[0].y)), fmaxf(fabsf(v[1].x), fabsf(v[1].y)));
  // a value that is not a number, which the maximum drops, spoils its block, as it spoils states in 32 bits; so does an
  // infinite m
  const float2 any = ROOT ? v[0] + v[1] : aw_fma(v[0], aw_both(0.f), v[1] * aw_both(0.f));
  if (!(any.x + any.y <= INFINITY)) most = __int_as_float(0x7FC00000);
  uint32_t bits = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most));  // of values >= 0, in their order
  // An infinite root (v beyond fp32) counts as 2^126, which no finite root reaches and whose square is infinite again:
  // with a scale of infinity the block's zeros would be lost.
  if (ROOT && bits == 0x7F800000u) bits = 0x7E800000u;
  const float big = __uint_as_float(bits);
  const bool none = big < AW_TINY;
  // (of m's largest value / 256: above 2^126 its own reciprocal is below the normal range, which the instruction takes
  // for zero)
  const float part = ROOT ? big : big * 0.00390625f, near = aw_inverse(part);
  const float inv = none ? 0.f : E4M3_MAX * (ROOT ? 1.f : 0.00390625f) * fmaf(near, fmaf(-part, near, 1.f), near), least = none ? 0.f : 0.001953125f;
  scale = none ? 0.f : big * (1.f / E4M3_MAX);
  uint32_t codes = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float2 a = make_float2(fabsf(v[h].x), fabsf(v[h].y)) * aw_both(inv);
    const float2 shift = make_float2(a.x < 0.015625f ? 0.015625f : 0.f, a.y < 0.015625f ? 0.015625f : 0.f);
    const float2 up = a + shift;
    auto cut = [](float x, uint32_t word) {
      return __uint_as_float((__float_as_uint(x) + ((ROOT ? word >> 12 : word << 4) & 0xFFFF0u) + 8u) & ~0xFFFFFu);
    };
    float2 q = aw_fma(shift, aw_both(-1.f), make_float2(cut(up.x, words[2 * h]), cut(up.y, words[2 * h + 1])));
    if (ROOT) q = make_float2(fmaxf(q.x, v[h].x > 0.f ? least : 0.f), fmaxf(q.y, v[h].y > 0.f ? least : 0.f));
    else q = make_float2(copysignf(q.x, v[h].x), copysignf(q.y, v[h].y));
    codes |= (uint32_t)__nv_cvt_float2_to_fp8x2(q, __NV_SATFINITE, __NV_E4M3) << (16 * h);
  }
  return codes;
}

// The piece of a tensor that a CTA takes at a time.
constexpr int AW_QUADS = 2;  // of each thread
constexpr int AW_TILE = AW_QUADS * AW_THREADS * 4;

// What is the same for all elements of a launch, and of a tensor.
struct AwStep {
  float gf, beta1, beta2, omb1, omb2, eps, root_lift2, step1, lr_decay, one;
  unsigned long long t;
};

template <int BITS>
struct AwState {
  float m[4], v[4];
  uint32_t mq, vq;
  float ms, vs;
};

// Four elements from i on (n, flat: see aw_load4).  WHOLE: all of them are there, flat.
template <int BITS, bool WHOLE>
__device__ __forceinline__ void aw_fetch(const AwEntry& e, long long i, bool flat, float (&p)[4], float (&g)[4], AwState<BITS>& st) {
  const long long n = WHOLE ? i + 4 : e.n;
  const bool f = WHOLE || flat;
  aw_load4(e.p, i, n, e.cols, e.ldp, f, p);
  if (e.g_is_bf16) aw_load4((const __nv_bfloat16*)e.g, i, n, e.cols, e.ldg, f, g);
  else aw_load4((const float*)e.g, i, n, e.cols, e.ldg, f, g);
  if constexpr (BITS == 32) {
    aw_load4((const float*)e.m, i, n, 1, 1, f, st.m);
    aw_load4((const float*)e.v, i, n, 1, 1, f, st.v);
  } else {
    st.mq = aw_load_codes((const uint8_t*)e.m, i, n, f);
    st.vq = aw_load_codes((const uint8_t*)e.v, i, n, f);
    st.ms = e.m_scale[i >> 7];
    st.vs = e.v_scale[i >> 7];
  }
}
template <int BITS, bool WHOLE>
__device__ __forceinline__ void aw_update(const AwEntry& e, const AwStep& a, const uint32_t (&keys)[20], long long i, bool flat, float (&p)[4],
                                          float (&g)[4], AwState<BITS>& st) {
  const long long n = WHOLE ? i + 4 : e.n;
  const bool f = WHOLE || flat;
  float (&m)[4] = st.m;
  float (&v)[4] = st.v;
  float2 gk[2], m2[2], v2[2], r2[2];
  if constexpr (BITS == 8) {
    aw_decode(st.mq, st.ms, m);
    aw_decode(st.vq, st.vs, v);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    gk[h] = make_float2(g[2 * h], g[2 * h + 1]) * aw_both(a.gf);
    m2[h] = make_float2(m[2 * h], m[2 * h + 1]);
    v2[h] = make_float2(v[2 * h], v[2 * h + 1]);
    if constexpr (BITS == 8) {
      // What decides how a state is rounded is computed operation by operation as the formulas stand, to the last bit:
      // one unit off moves a value in a million to its other neighbour.  (Sums as products with one and sums: of a sum
      // of two elements in one instruction the assembler makes one with the product before it, though both ask to be
      // rounded.)
      const float2 one = aw_both(a.one);
      m2[h] = aw_fma(aw_both(a.beta1) * m2[h], one, aw_both(a.omb1) * gk[h]);
      v2[h] = aw_fma(aw_both(a.beta2) * (v2[h] * v2[h]), one, (aw_both(a.omb2) * gk[h]) * gk[h]);
      r2[h] = aw_roots(v2[h]);
    } else {
      m2[h] = aw_fma(aw_both(a.beta1), m2[h], aw_both(a.omb1) * gk[h]);
      v2[h] = aw_fma(aw_both(a.beta2), v2[h], (aw_both(a.omb2) * gk[h]) * gk[h]);
      r2[h] = make_float2(aw_root(v2[h].x), aw_root(v2[h].y));
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float2 p2 = make_float2(p[2 * h], p[2 * h + 1]), den = aw_fma(r2[h], aw_both(a.root_lift2), aw_both(a.eps));
    const float2 move = (aw_both(a.step1) * m2[h]) * make_float2(aw_inverse(den.x), aw_inverse(den.y));
    const float2 to = aw_fma(aw_both(-1.f), aw_fma(aw_both(a.lr_decay), p2, move), p2);
    p[2 * h] = to.x;
    p[2 * h + 1] = to.y;
    m[2 * h] = m2[h].x;
    m[2 * h + 1] = m2[h].y;
    v[2 * h] = v2[h].x;
    v[2 * h + 1] = v2[h].y;
  }
  aw_store4(e.p, i, n, e.cols, e.ldp, f, p);
  if (e.w) aw_store4(e.w, i, n, e.cols, e.ldw, f, p);
  if constexpr (BITS == 32) {
    aw_store4((float*)e.m, i, n, 1, 1, f, m);
    aw_store4((float*)e.v, i, n, 1, 1, f, v);
  } else {
    uint32_t c[4] = {(uint32_t)a.t, (uint32_t)(a.t >> 32), (uint32_t)(i >> 2), e.number};
#pragma unroll
    for (int k = 0; k < 10; ++k) philox_round(c, keys[2 * k], keys[2 * k + 1]);
    if (!WHOLE)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (i + 2 * h >= n) m2[h].x = r2[h].x = 0.f;
        if (i + 2 * h + 1 >= n) m2[h].y = r2[h].y = 0.f;
      }
    float ms, vs;
    const uint32_t mq = aw_encode<false>(m2, c, ms), vq = aw_encode<true>(r2, c, vs);
    aw_store_codes((uint8_t*)e.m, i, n, f, mq);
    aw_store_codes((uint8_t*)e.v, i, n, f, vq);
    if ((threadIdx.x & 31) == 0) {
      e.m_scale[i >> 7] = ms;
      e.v_scale[i >> 7] = vs;
    }
  }
}

// 1 / (1 - beta^t), or its root.
__host__ __device__ inline float aw_lift(unsigned long long t, double ln_beta, bool root) {
  const double lift = -1.0 / expm1((double)t * ln_beta);
  return (float)(root ? sqrt(lift) : lift);
}

// What the kernels do first; false: nothing is to be done.
__device__ __forceinline__ bool aw_begin(const AwArgs& a, AwStep& st, float& lr, float (&s_lift)[2]) {
  st.t = a.step + (a.counter ? *a.counter : 0ull);
  st.gf = a.grad_factor ? *a.grad_factor : 1.f;
  if (st.t == 0 || !(fabsf(st.gf) < INFINITY)) return false;
  lr = a.lr_factor ? a.lr * *a.lr_factor : a.lr;
  float lift1 = a.lift1;
  st.root_lift2 = a.root_lift2;
  if (a.counter) {
    if (threadIdx.x < 2) s_lift[threadIdx.x] = aw_lift(st.t, threadIdx.x ? a.ln_beta2 : a.ln_beta1, threadIdx.x);
    __syncthreads();
    lift1 = s_lift[0];
    st.root_lift2 = s_lift[1];
  }
  st.step1 = lr * lift1;
  st.beta1 = a.beta1;
  st.beta2 = a.beta2;
  st.omb1 = a.one_minus_beta1;
  st.omb2 = a.one_minus_beta2;
  st.eps = a.eps;
  st.one = a.one;
  return true;
}
// A tile of QUADS x THREADS quads that ends inside, or whose elements do not lie one after the other on 16 bytes.
template <int BITS, int QUADS, int THREADS>
__device__ __forceinline__ void aw_ragged(const AwEntry& e, const AwStep& st, const uint32_t (&keys)[20], long long base, int thread) {
#pragma unroll 1
  for (int u = 0; u < QUADS; ++u) {
    const long long i = base + (u * THREADS + thread) * 4;
    if (BITS == 32 ? i >= e.n : (i & ~127ll) >= e.n) continue;  // (8 bits: a block's lanes stay together)
    float p[4], g[4];
    AwState<BITS> state;
    aw_fetch<BITS, false>(e, i, e.flat, p, g, state);
    aw_update<BITS, false>(e, st, keys, i, e.flat, p, g, state);
  }
}

// States in 32 bits: a CTA a tile, all of a thread's loads ahead of its stores.  (On a grid of the resident CTAs, each
// with many tiles, the step of 8192 x 8192 with a bf16 gradient took 310 us, so 274, 6.85 TB/s: the loads of a CTA that
// begins run beside the stores of one that ends.)
template <int CAP>
__global__ void __launch_bounds__(AW_THREADS, 4) adamw_kernel(const __grid_constant__ AwTable<CAP> table, const __grid_constant__ AwArgs a) {
  __shared__ float s_lift[2];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  AwStep st;
  float lr;
  if (!aw_begin(a, st, lr, s_lift)) return;
  for (unsigned long long tile = blockIdx.x; tile < table.tiles; tile += gridDim.x) {
    const AwEntry& e = table.e[aw_find(table, tile)];
    const long long base = (long long)(tile - e.tile0) * AW_TILE;
    st.lr_decay = lr * e.decay;
    if (e.flat && base + AW_TILE <= e.n) {
      float p[AW_QUADS][4], g[AW_QUADS][4];
      AwState<32> state[AW_QUADS];
#pragma unroll
      for (int u = 0; u < AW_QUADS; ++u) aw_fetch<32, true>(e, base + (u * AW_THREADS + threadIdx.x) * 4, true, p[u], g[u], state[u]);
#pragma unroll
      for (int u = 0; u < AW_QUADS; ++u)
        aw_update<32, true>(e, st, a.keys, base + (u * AW_THREADS + threadIdx.x) * 4, true, p[u], g[u], state[u]);
    } else {
      aw_ragged<32, AW_QUADS, AW_THREADS>(e, st, a.keys, base, (int)threadIdx.x);
    }
  }
}

// States in 8 bits: 8 to 10 bytes are read for an element whose arithmetic takes some 92 instructions, so registers
// cannot hold what has to be in flight (36 bytes for a thread's quad: 2.2 TB/s).  Every warp has its own tiles, which
// come through a ring in shared memory by bulk copies ahead of it: no barrier among warps, four quads of a lane to a
// search of the table.  36 M elements with a fp32 gradient 140 us, 150 where the scales come by lanes; with a bf16 one
// 141.  (Tiles of a CTA, two quads and four: 148 and 124 us with states rounded from values a unit or so off; to the
// last bit 133 in tiles of a warp; the rest is for moments at fp32's ends, infinity and subnormals.)
constexpr int AW8_QUADS = 4, AW8_TILE = AW8_QUADS * 128, AW8_SLOTS = 2, AW8_PER_SM = 2, AW8_WARPS = AW_THREADS / 32;
constexpr int AW8_UNROLL = 4;
static_assert(AW8_QUADS % 4 == 0, "bulk copies of the scales: multiples of 16 bytes");
constexpr int AW8_P = 0, AW8_G = AW8_TILE * 4, AW8_M = AW8_G + AW8_TILE * 4, AW8_V = AW8_M + AW8_TILE, AW8_MS = AW8_V + AW8_TILE,
              AW8_VS = AW8_MS + AW8_QUADS * 4, AW8_SLOT = AW8_VS + AW8_QUADS * 4;
template <int CAP>
__global__ void __launch_bounds__(AW_THREADS, AW8_PER_SM) adamw8_kernel(const __grid_constant__ AwTable<CAP> table, const __grid_constant__ AwArgs a,
                                                                       int* status) {
  extern __shared__ __align__(128) uint8_t slots[];  // [warps][AW8_SLOTS][AW8_SLOT]
  __shared__ __align__(8) uint64_t bars[AW8_WARPS][AW8_SLOTS];
  __shared__ float s_lift[2];
  __shared__ int s_gone;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint64_t* full = bars[warp];
  uint8_t* mine = slots + (size_t)warp * AW8_SLOTS * AW8_SLOT;
  if (lane == 0) {
    for (int k = 0; k < AW8_SLOTS; ++k) mbar_init(smem_u32(&full[k]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (threadIdx.x == 0) s_gone = 0;
  __syncthreads();
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  AwStep st;
  float lr;
  if (!aw_begin(a, st, lr, s_lift)) return;
  auto whole = [&](const AwEntry& e, long long base) { return e.flat && base + AW8_TILE <= e.n; };
  const unsigned long long stride = (unsigned long long)gridDim.x * AW8_WARPS;
  unsigned long long ahead = (unsigned long long)blockIdx.x * AW8_WARPS + warp;  // the next tile to ask for (lane 0)
  int asked = 0, slot = 0, phase = 0, taken = 0;
  bool gone = false;  // a copy did not come within two seconds: the rest is left, the status says so
  auto ask = [&] {
    if (ahead >= table.tiles || gone) return;
    const AwEntry& e = table.e[aw_find(table, ahead)];
    const long long base = (long long)(ahead - e.tile0) * AW8_TILE;
    const int to = asked++ % AW8_SLOTS;
    const uint32_t bar = smem_u32(&full[to]), dst = smem_u32(mine + to * AW8_SLOT);
    ahead += stride;
    if (!whole(e, base)) {
      mbar_arrive(bar);
      return;
    }
    const uint32_t gbytes = e.g_is_bf16 ? AW8_TILE * 2 : AW8_TILE * 4;
    mbar_arrive_expect_tx(bar, AW8_TILE * 6 + gbytes + (e.scales16 ? AW8_QUADS * 8 : 0));
    auto copy = [&](uint32_t at, const void* src, uint32_t bytes) {
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst + at), "l"(src),
                   "r"(bytes), "r"(bar)
                   : "memory");
    };
    copy(AW8_P, e.p + base, AW8_TILE * 4);
    copy(AW8_G, (const uint8_t*)e.g + base * (e.g_is_bf16 ? 2 : 4), gbytes);
    copy(AW8_M, (const uint8_t*)e.m + base, AW8_TILE);
    copy(AW8_V, (const uint8_t*)e.v + base, AW8_TILE);
    if (e.scales16) {
      copy(AW8_MS, e.m_scale + base / 128, AW8_QUADS * 4);
      copy(AW8_VS, e.v_scale + base / 128, AW8_QUADS * 4);
    }
  };
  if (lane == 0)
    for (int k = 0; k < AW8_SLOTS; ++k) ask();
  for (unsigned long long tile = (unsigned long long)blockIdx.x * AW8_WARPS + warp; tile < table.tiles; tile += stride) {
    const AwEntry& e = table.e[aw_find(table, tile)];
    const long long base = (long long)(tile - e.tile0) * AW8_TILE;
    st.lr_decay = lr * e.decay;
    // scales off the 16-byte grid (those of a tensor among others in one buffer): a lane each, behind the wait into the
    // copies' place
    const bool by_lanes = !e.scales16 && whole(e, base) && lane < 2 * AW8_QUADS;
    const float sc = by_lanes ? (lane < AW8_QUADS ? e.m_scale : e.v_scale - AW8_QUADS)[base / 128 + lane] : 0.f;
    if (!gone && !mbar_wait(smem_u32(&full[slot]), (uint32_t)phase, &s_gone, status)) gone = true;
    gone = __any_sync(0xFFFFFFFFu, gone);
    if (!gone) {
      ++taken;
      if (whole(e, base)) {
        uint8_t* from = mine + slot * AW8_SLOT;
        if (by_lanes) {
          reinterpret_cast<float*>(from + AW8_MS)[lane] = sc;  // (v's lie behind m's)
          fence_proxy_async_smem();                            // before a later tile's bulk copies into the same bytes
        }
        __syncwarp();
#pragma unroll AW8_UNROLL
        for (int u = 0; u < AW8_QUADS; ++u) {
          const int at = (u * 32 + lane) * 4;
          float p[4], g[4];
          AwState<8> state;
          aw_load4((const float*)(from + AW8_P), at, AW8_TILE, 0, 0, true, p);
          if (e.g_is_bf16) aw_load4((const __nv_bfloat16*)(from + AW8_G), at, AW8_TILE, 0, 0, true, g);
          else aw_load4((const float*)(from + AW8_G), at, AW8_TILE, 0, 0, true, g);
          state.mq = *reinterpret_cast<const uint32_t*>(from + AW8_M + at);
          state.vq = *reinterpret_cast<const uint32_t*>(from + AW8_V + at);
          state.ms = reinterpret_cast<const float*>(from + AW8_MS)[u];
          state.vs = reinterpret_cast<const float*>(from + AW8_VS)[u];
          aw_update<8, true>(e, st, a.keys, base + at, true, p, g, state);
        }
      } else {
        aw_ragged<8, AW8_QUADS, 32>(e, st, a.keys, base, lane);
      }
    }
    __syncwarp();  // the slot has been read
    if (lane == 0) ask();
    if (++slot == AW8_SLOTS) {
      slot = 0;
      phase ^= 1;
    }
  }
  if (lane == 0)  // copies that did not come get the same time again before the CTA ends: they write to its memory
    for (int k = taken; gone && k < asked; ++k) {
      bool ok = false;
      for (int poll = 0; poll < 2000 && !ok; ++poll) ok = mbar_try_wait_hint(smem_u32(&full[k % AW8_SLOTS]), (uint32_t)(k / AW8_SLOTS) & 1u, 1000000u);
    }
}

// ---- norm of all gradients ------------------------------------------------------------------------
constexpr int GN_EIGHTS = 4;
constexpr int GN_TILE = GN_EIGHTS * AW_THREADS * 8;

// The squares of eight values.  Added in fp32 where that is as good: a sum that neither overflowed nor lies where
// squares lose their bits (the additions' errors, of either sign, go under in millions of such sums).  Otherwise in
// fp64, which converts every value: 68 us in place of 24 for 64 Mi bf16 values.  (Zeros, as whole rows of dropped
// units, go that way too: every second row of 2048 zero 25.4 us, four of five 27.3.)
__device__ __forceinline__ double gn_squares(const float (&g)[8]) {
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) s = fmaf(g[k], g[k], s);
  if (s > 8.3e-25f && s < INFINITY) return (double)s;
  double x = 0.0;
#pragma unroll
  for (int k = 0; k < 8; ++k) x = fma((double)g[k], (double)g[k], x);
  return x;
}

// Every CTA leaves the sum of its squares; the last one of the last launch adds them in the order of the CTAs.
template <int CAP>
__global__ void __launch_bounds__(AW_THREADS) grad_norm_kernel(const __grid_constant__ AwTable<CAP> table, double* partial, int before,
                                                               int last_launch, unsigned int* count, double max_norm, float* out) {
  __shared__ double red[AW_THREADS / 32];
  __shared__ int s_last;
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  double sum = 0.0;
  for (unsigned long long tile = blockIdx.x; tile < table.tiles; tile += gridDim.x) {
    const AwEntry& e = table.e[aw_find(table, tile)];
    const long long base = (long long)(tile - e.tile0) * GN_TILE;
    const int t = (int)threadIdx.x;
    float g[GN_EIGHTS][8];
    if (e.flat && base + GN_TILE <= e.n) {
      if (e.g_is_bf16) {
        uint4 q[GN_EIGHTS];
#pragma unroll
        for (int u = 0; u < GN_EIGHTS; ++u) q[u] = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)e.g + base + (u * AW_THREADS + t) * 8);
#pragma unroll
        for (int u = 0; u < GN_EIGHTS; ++u) {
          const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            g[u][2 * k] = __uint_as_float(w[k] << 16);
            g[u][2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
          }
        }
      } else {
#pragma unroll
        for (int u = 0; u < GN_EIGHTS; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            // a warp's lanes read one after the other; which of a thread's eights a value belongs to does not matter
            const float4 q = *reinterpret_cast<const float4*>((const float*)e.g + base + ((2 * u + h) * AW_THREADS + t) * 4);
            g[u][4 * h] = q.x; g[u][4 * h + 1] = q.y; g[u][4 * h + 2] = q.z; g[u][4 * h + 3] = q.w;
          }
      }
    } else {
#pragma unroll
      for (int u = 0; u < GN_EIGHTS; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float q[4];
          const long long i = base + (u * AW_THREADS + t) * 8 + 4 * h;
          if (e.g_is_bf16) aw_load4((const __nv_bfloat16*)e.g, i, e.n, e.cols, e.ldg, e.flat, q);
          else aw_load4((const float*)e.g, i, e.n, e.cols, e.ldg, e.flat, q);
#pragma unroll
          for (int k = 0; k < 4; ++k) g[u][4 * h + k] = q[k];
        }
    }
#pragma unroll
    for (int u = 0; u < GN_EIGHTS; ++u) sum += gn_squares(g[u]);
  }
  auto block_sum = [&](double x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int k = 0; k < AW_THREADS / 32; ++k) x += red[k];
    return x;
  };
  sum = block_sum(sum);
  if (threadIdx.x == 0) {
    __stcg(partial + before + blockIdx.x, sum);
    s_last = 0;
    if (last_launch) {
      __threadfence();
      s_last = atomicAdd(count, 1u) == gridDim.x - 1;
    }
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  double x = 0.0;
  for (int k = threadIdx.x; k < before + (int)gridDim.x; k += AW_THREADS) x += __ldcg(partial + k);
  x = block_sum(x);
  if (threadIdx.x == 0) {
    *count = 0u;  // armed again for the next launch
    const double norm = sqrt(x);
    const bool fine = norm <= 3.4028234663852886e38;
    out[0] = (float)norm;
    out[1] = !fine ? __int_as_float(0x7FC00000) : max_norm > 0.0 ? (float)fmin(1.0, max_norm / (norm + 1e-6)) : 1.f;
  }
}

inline bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// One entry of the table; the caller has checked the tensor.
AwEntry aw_entry(const ard_adamw_tensor& t, int number, bool grads_only, unsigned long long tile0) {
  AwEntry e;
  e.p = grads_only ? nullptr : t.p;
  e.g = t.g;
  e.w = grads_only ? nullptr : (__nv_bfloat16*)t.w;
  e.m = grads_only ? nullptr : t.m;
  e.v = grads_only ? nullptr : t.v;
  e.m_scale = t.m_scale;
  e.v_scale = t.v_scale;
  e.n = (long long)t.rows * t.cols;
  e.cols = t.cols;
  const bool row = t.rows == 1;  // one row has no gaps, whatever its leading dimension
  e.ldp = row ? t.cols : t.ldp;
  e.ldg = row ? t.cols : t.ldg;
  e.ldw = row ? t.cols : t.ldw;
  e.tile0 = tile0;
  e.decay = (float)t.weight_decay;
  e.number = (unsigned)number + 1u;
  e.g_is_bf16 = t.g_dtype == ARD_BF16;
  e.flat = e.ldg == t.cols && on16(t.g);
  if (!grads_only)
    e.flat = e.flat && e.ldp == t.cols && on16(t.p) && on16(t.m) && on16(t.v) && (!t.w || (e.ldw == t.cols && on16(t.w)));
  e.scales16 = on16(t.m_scale) && on16(t.v_scale);
  return e;
}

// Cuts the table of tensors into launches: launch(table, number of tensors of the caller's table that are left).
template <typename Launch>
ard_status aw_launches(const ard_adamw_tensor* tensors, int n_tensors, bool grads_only, int tile, Launch launch) {
  int at = 0;
  do {
    int live = 0, k = at;
    for (; k < n_tensors && live < AW_LARGE; ++k) live += tensors[k].rows > 0 && tensors[k].cols > 0;
    auto fill = [&](auto& table) {
      table.n = 0;
      table.tiles = 0;
      for (int i = at; i < k; ++i) {
        if (tensors[i].rows == 0 || tensors[i].cols == 0) continue;
        table.e[table.n++] = aw_entry(tensors[i], i, grads_only, table.tiles);
        table.tiles += (unsigned long long)((tensors[i].rows * tensors[i].cols + tile - 1) / tile);
      }
    };
    ard_status st;
    if (live <= AW_SMALL) {
      AwTable<AW_SMALL> table;
      fill(table);
      st = launch(table, n_tensors - k);
    } else {
      AwTable<AW_LARGE> table;
      fill(table);
      st = launch(table, n_tensors - k);
    }
    if (st != ARD_OK) return st;
    at = k;
  } while (at < n_tensors);
  return ARD_OK;
}

}  // namespace

ard_status launch_adamw(ard_ctx* ctx, const ard_adamw_tensor* tensors, int n_tensors, double lr, double beta1, double beta2, double eps,
                        int bits, uint64_t seed, uint64_t step, const uint64_t* counter, const float* lr_factor, const float* grad_factor,
                        cudaStream_t s) {
  AwArgs a;
  a.lr = (float)lr;
  a.beta1 = (float)beta1;
  a.beta2 = (float)beta2;
  a.one = 1.f;
  a.one_minus_beta1 = (float)(1.0 - beta1);
  a.one_minus_beta2 = (float)(1.0 - beta2);
  a.eps = (float)eps;
  a.ln_beta1 = beta1 > 0.0 ? log(beta1) : -1e300;
  a.ln_beta2 = beta2 > 0.0 ? log(beta2) : -1e300;
  for (int k = 0; k < 10; ++k) {
    a.keys[2 * k] = (uint32_t)seed + (uint32_t)k * 0x9E3779B9u;
    a.keys[2 * k + 1] = (uint32_t)(seed >> 32) + (uint32_t)k * 0xBB67AE85u;
  }
  a.step = step;
  a.lift1 = aw_lift(step, a.ln_beta1, false);
  a.root_lift2 = aw_lift(step, a.ln_beta2, true);
  a.counter = reinterpret_cast<const unsigned long long*>(counter);
  a.lr_factor = lr_factor;
  a.grad_factor = grad_factor;
  return aw_launches(tensors, n_tensors, false, bits == 32 ? AW_TILE : AW8_TILE, [&](const auto& table, int) {
    if (table.n == 0) return ARD_OK;
    using T = std::remove_cv_t<std::remove_reference_t<decltype(table)>>;
    constexpr int CAP = sizeof(table.e) / sizeof(table.e[0]);
    if (bits == 32) {
      const unsigned long long most = 1ull << 30;
      const dim3 grid((unsigned)(table.tiles < most ? table.tiles : most));
      ARD_CUDA_OK(ard_launch(ctx, adamw_kernel<CAP>, grid, dim3(AW_THREADS), 0, s, (T)table, a));
    } else {
      constexpr int smem = AW8_WARPS * AW8_SLOTS * AW8_SLOT;
      const unsigned long long room = (unsigned long long)AW8_PER_SM * ctx->sm_count, want = (table.tiles + AW8_WARPS - 1) / AW8_WARPS;
      const dim3 grid((unsigned)(want < room ? want : room));
      ARD_CUDA_OK(cudaFuncSetAttribute(adamw8_kernel<CAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
      ARD_CUDA_OK(ard_launch(ctx, adamw8_kernel<CAP>, grid, dim3(AW_THREADS), smem, s, (T)table, a, ctx->d_status));
    }
    ctx->launches++;
    ARD_CUDA_OK(cudaGetLastError());
    return ARD_OK;
  });
}

ard_status launch_grad_norm(ard_ctx* ctx, const ard_adamw_tensor* tensors, int n_tensors, double max_norm, float* out, cudaStream_t s) {
  if (!ctx->d_sk_ws) return ARD_ERR_UNSUPPORTED;
  int before = 0;
  const int most = (int)(sk_ws_bytes(ctx->sm_count) / sizeof(double));
  return aw_launches(tensors, n_tensors, true, GN_TILE, [&](const auto& table, int left) {
    using T = std::remove_cv_t<std::remove_reference_t<decltype(table)>>;
    constexpr int CAP = sizeof(table.e) / sizeof(table.e[0]);
    const unsigned long long room = 4ull * ctx->sm_count;
    int grid = (int)(table.tiles < room ? table.tiles : room);
    if (grid < 1) grid = 1;  // no gradients at all: the norm is zero
    if (before + grid > most) return ARD_ERR_NOMEM;
    ARD_CUDA_OK(ard_launch(ctx, grad_norm_kernel<CAP>, dim3(grid), dim3(AW_THREADS), 0, s, (T)table, (double*)ctx->d_sk_ws, before,
                           left == 0 ? 1 : 0, (unsigned int*)ctx->d_sk_cnt, max_norm, out));
    before += grid;
    ctx->launches++;
    ARD_CUDA_OK(cudaGetLastError());
    return ARD_OK;
  });
}
