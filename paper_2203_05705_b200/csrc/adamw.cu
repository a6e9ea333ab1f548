// The optimiser's step over many tensors at once, and the norm of all gradients with the factor that clips them.
//
// Both are one pass over memory: per element the step reads p, g, m, v and writes p, m, v and the bf16 copy (28 to 30 bytes with
// states in 32 bits, 16 to 18 in 8).  The table of tensors travels as a kernel parameter: nothing is copied or allocated per call.
#include <cuda_fp8.h>

#include "ard_internal.h"
#include "philox.h"

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
  int flat;                  // no gaps between rows, all pointers on 16 bytes: read and written in pieces of 4 elements
};

template <int CAP>
struct AwTable {
  AwEntry e[CAP];
  int n;
  unsigned long long tiles;
};

// Tables travel in the launch: the small one keeps a launch over a handful of tensors as cheap as any other, the large one
// (26 KB of the 32 KB that parameters may have) takes a network's.
constexpr int AW_SMALL = 16, AW_LARGE = 216;

struct AwArgs {
  float lr, beta1, beta2, one_minus_beta1, one_minus_beta2, eps;
  double ln_beta1, ln_beta2;
  unsigned long long seed, step;
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

// 1 / x and sqrt(x) to the last bit or two in a few instructions: the instructions' approximations, improved once by Newton's step, in place of
// division and square root rounded to the last bit (8 to 20 instructions each with their special cases).  What is rounded to 8 bits is worth the
// step: an error of one unit more in the last place is a few values in a million more that fall on the other side of a border.
__device__ __forceinline__ float aw_inverse(float x) {  // x normal
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return fmaf(r, fmaf(-x, r, 1.f), r);
}
__device__ __forceinline__ float aw_root(float x) {  // subnormal: 0
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  const float s = x * r;
  const float better = fmaf(0.5f * r, fmaf(-s, s, x), s);
  return x < 1.17549435e-38f ? 0.f : better;
}
// The quotient of the step, and its root, which no rounding follows but the parameter's.
__device__ __forceinline__ float aw_quick_root(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float aw_quick_inverse(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// a >= 0 rounded to the grid of the 8-bit floats (3 bits of mantissa; steps of 2^-9 below 2^-6), up with the probability of what is
// cut off, which 16 random bits resolve to 2^-16 of a step.  Below 2^-6 the grid is that of [2^-6, 2^-5): adding 2^-6 puts the
// value there.  The sum of the bits carries into the exponent where it should.
__device__ __forceinline__ float aw_round(float a, uint32_t random16) {
  const bool low = a < 0.015625f;
  const float s = low ? a + 0.015625f : a;
  const float q = __uint_as_float((__float_as_uint(s) + (random16 << 4) + 8u) & ~0xFFFFFu);
  return fminf(low ? q - 0.015625f : q, E4M3_MAX);
}

// The 8-bit floats of a block of 128 values, four in each lane, and its scale (the same in all lanes).
template <bool POSITIVE>
__device__ __forceinline__ uint32_t aw_encode(const float (&v)[4], const uint32_t (&random16)[4], float& scale) {
  const float mine = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
  // fmaxf drops NaN: a value that is not a number has to spoil its block, as it spoils states in 32 bits
  const bool nan = v[0] != v[0] || v[1] != v[1] || v[2] != v[2] || v[3] != v[3];
  const uint32_t bits = __reduce_max_sync(0xFFFFFFFFu, nan ? 0x7FC00000u : __float_as_uint(mine));  // of values >= 0, in their order
  const float big = __uint_as_float(bits);
  const bool none = big < AW_TINY;
  const float inv = none ? 0.f : E4M3_MAX * aw_inverse(big);
  scale = none ? 0.f : big * (1.f / E4M3_MAX);
  float q[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    q[k] = aw_round(fabsf(v[k]) * inv, random16[k]);
    if (POSITIVE && v[k] > 0.f && !none) q[k] = fmaxf(q[k], 0.001953125f);
    if (!POSITIVE) q[k] = copysignf(q[k], v[k]);
  }
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(q[0], q[1]), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(q[2], q[3]), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}

// The piece of a tensor that a CTA takes at a time.
constexpr int AW_QUADS = 2;
constexpr int AW_TILE = AW_QUADS * AW_THREADS * 4;

// What is the same for all elements of a launch, and of a tensor.
struct AwStep {
  float gf, beta1, beta2, omb1, omb2, eps, root_lift2, step1, lr_decay;
  unsigned long long t, seed;
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
__device__ __forceinline__ void aw_update(const AwEntry& e, const AwStep& a, long long i, bool flat, float (&p)[4], float (&g)[4],
                                          AwState<BITS>& st) {
  const long long n = WHOLE ? i + 4 : e.n;
  const bool f = WHOLE || flat;
  float (&m)[4] = st.m;
  float (&v)[4] = st.v;
  float r[4];
  if constexpr (BITS == 8) {
    aw_decode(st.mq, st.ms, m);
    aw_decode(st.vq, st.vs, v);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float gk = g[k] * a.gf;
    m[k] = fmaf(a.beta1, m[k], a.omb1 * gk);
    v[k] = fmaf(a.beta2, BITS == 32 ? v[k] : v[k] * v[k], a.omb2 * gk * gk);
    r[k] = BITS == 32 ? aw_quick_root(v[k]) : aw_root(v[k]);
    const float move = a.step1 * m[k] * aw_quick_inverse(fmaf(r[k], a.root_lift2, a.eps));
    p[k] = p[k] - fmaf(a.lr_decay, p[k], move);
  }
  aw_store4(e.p, i, n, e.cols, e.ldp, f, p);
  if (e.w) aw_store4(e.w, i, n, e.cols, e.ldw, f, p);
  if constexpr (BITS == 32) {
    aw_store4((float*)e.m, i, n, 1, 1, f, m);
    aw_store4((float*)e.v, i, n, 1, 1, f, v);
  } else {
    uint32_t c[4] = {(uint32_t)a.t, (uint32_t)(a.t >> 32), (uint32_t)(i >> 2), e.number};
    philox4x32_10(c, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
    uint32_t low[4], high[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      low[k] = c[k] & 0xFFFFu;
      high[k] = c[k] >> 16;
      if (!WHOLE && i + k >= n) m[k] = r[k] = 0.f;
    }
    float ms, vs;
    const uint32_t mq = aw_encode<false>(m, low, ms), vq = aw_encode<true>(r, high, vs);
    aw_store_codes((uint8_t*)e.m, i, n, f, mq);
    aw_store_codes((uint8_t*)e.v, i, n, f, vq);
    if ((threadIdx.x & 31) == 0) {
      e.m_scale[i >> 7] = ms;
      e.v_scale[i >> 7] = vs;
    }
  }
}

template <int BITS, int CAP>
__global__ void __launch_bounds__(AW_THREADS, 4) adamw_kernel(const __grid_constant__ AwTable<CAP> table, const AwArgs a) {
  __shared__ float s_lift[2];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  AwStep st;
  st.t = a.step + (a.counter ? *a.counter : 0ull);
  if (st.t == 0) return;
  st.gf = a.grad_factor ? *a.grad_factor : 1.f;
  if (!(fabsf(st.gf) < INFINITY)) return;
  const float lr = a.lr_factor ? a.lr * *a.lr_factor : a.lr;
  if (threadIdx.x < 2) {
    const double lift = -1.0 / expm1((double)st.t * (threadIdx.x ? a.ln_beta2 : a.ln_beta1));
    s_lift[threadIdx.x] = (float)(threadIdx.x ? sqrt(lift) : lift);
  }
  __syncthreads();
  st.root_lift2 = s_lift[1];
  st.step1 = lr * s_lift[0];
  st.beta1 = a.beta1;
  st.beta2 = a.beta2;
  st.omb1 = a.one_minus_beta1;
  st.omb2 = a.one_minus_beta2;
  st.eps = a.eps;
  st.seed = a.seed;
  for (unsigned long long tile = blockIdx.x; tile < table.tiles; tile += gridDim.x) {
    const AwEntry& e = table.e[aw_find(table, tile)];
    const long long base = (long long)(tile - e.tile0) * AW_TILE;
    st.lr_decay = lr * e.decay;
    if (e.flat && base + AW_TILE <= e.n) {
      // all loads of the tile before its first store
      float p[AW_QUADS][4], g[AW_QUADS][4];
      AwState<BITS> state[AW_QUADS];
#pragma unroll
      for (int u = 0; u < AW_QUADS; ++u) aw_fetch<BITS, true>(e, base + (u * AW_THREADS + threadIdx.x) * 4, true, p[u], g[u], state[u]);
#pragma unroll
      for (int u = 0; u < AW_QUADS; ++u) aw_update<BITS, true>(e, st, base + (u * AW_THREADS + threadIdx.x) * 4, true, p[u], g[u], state[u]);
    } else {
#pragma unroll 1
      for (int u = 0; u < AW_QUADS; ++u) {
        const long long i = base + (u * AW_THREADS + threadIdx.x) * 4;
        if (BITS == 32 ? i >= e.n : (i & ~127ll) >= e.n) continue;  // (8 bits: a block's lanes stay together)
        float p[4], g[4];
        AwState<BITS> state;
        aw_fetch<BITS, false>(e, i, e.flat, p, g, state);
        aw_update<BITS, false>(e, st, i, e.flat, p, g, state);
      }
    }
  }
}

// ---- norm of all gradients ------------------------------------------------------------------------
constexpr int GN_EIGHTS = 4;
constexpr int GN_TILE = GN_EIGHTS * AW_THREADS * 8;

// The squares of eight values.  Added in fp32 where that is as good: a sum that neither overflowed nor lies where squares lose their bits
// (the additions' errors, of either sign, go under in millions of such sums).  Otherwise in fp64, which converts every value: 68 us in place of 24 for
// 64 Mi bf16 values.
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
                                                               int last_launch, unsigned int* count, float max_norm, float* out) {
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
    out[1] = !fine ? __int_as_float(0x7FC00000) : max_norm > 0.f ? (float)fmin(1.0, (double)max_norm / (norm + 1e-6)) : 1.f;
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
  a.one_minus_beta1 = (float)(1.0 - beta1);
  a.one_minus_beta2 = (float)(1.0 - beta2);
  a.eps = (float)eps;
  a.ln_beta1 = beta1 > 0.0 ? log(beta1) : -1e300;
  a.ln_beta2 = beta2 > 0.0 ? log(beta2) : -1e300;
  a.seed = seed;
  a.step = step;
  a.counter = reinterpret_cast<const unsigned long long*>(counter);
  a.lr_factor = lr_factor;
  a.grad_factor = grad_factor;
  return aw_launches(tensors, n_tensors, false, AW_TILE, [&](const auto& table, int) {
    if (table.n == 0) return ARD_OK;
    using T = std::remove_cv_t<std::remove_reference_t<decltype(table)>>;
    constexpr int CAP = sizeof(table.e) / sizeof(table.e[0]);
    const unsigned long long room = 4ull * ctx->sm_count;
    const dim3 grid((unsigned)(table.tiles < room ? table.tiles : room));
    if (bits == 32) ARD_CUDA_OK(ard_launch(ctx, adamw_kernel<32, CAP>, grid, dim3(AW_THREADS), 0, s, (T)table, a));
    else ARD_CUDA_OK(ard_launch(ctx, adamw_kernel<8, CAP>, grid, dim3(AW_THREADS), 0, s, (T)table, a));
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
                           left == 0 ? 1 : 0, (unsigned int*)ctx->d_sk_cnt, (float)max_norm, out));
    before += grid;
    ctx->launches++;
    ARD_CUDA_OK(cudaGetLastError());
    return ARD_OK;
  });
}
