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
  const float inv = none ? 0.f : E4M3_MAX / big;
  scale = none ? 0.f : big / E4M3_MAX;
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

template <int BITS, int CAP>
__global__ void __launch_bounds__(AW_THREADS) adamw_kernel(const __grid_constant__ AwTable<CAP> table, const AwArgs a) {
  __shared__ float s_lift[2];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const unsigned long long t = a.step + (a.counter ? *a.counter : 0ull);
  if (t == 0) return;
  const float gf = a.grad_factor ? *a.grad_factor : 1.f;
  if (!(fabsf(gf) < INFINITY)) return;
  const float lr = a.lr_factor ? a.lr * *a.lr_factor : a.lr;
  if (threadIdx.x < 2) s_lift[threadIdx.x] = (float)(-1.0 / expm1((double)t * (threadIdx.x ? a.ln_beta2 : a.ln_beta1)));
  __syncthreads();
  const float lift2 = s_lift[1], step1 = lr * s_lift[0];
  for (unsigned long long tile = blockIdx.x; tile < table.tiles; tile += gridDim.x) {
    const AwEntry& e = table.e[aw_find(table, tile)];
    const long long n = e.n, base = (long long)(tile - e.tile0) * AW_TILE;
    const bool flat = e.flat;
#pragma unroll
    for (int u = 0; u < AW_QUADS; ++u) {
      const long long i = base + (u * AW_THREADS + threadIdx.x) * 4;
      if (BITS == 32 ? i >= n : (i & ~127ll) >= n) continue;  // (8 bits: a block's lanes stay together)
      float p[4], g[4], m[4], v[4];
      aw_load4(e.p, i, n, e.cols, e.ldp, flat, p);
      if (e.g_is_bf16) aw_load4((const __nv_bfloat16*)e.g, i, n, e.cols, e.ldg, flat, g);
      else aw_load4((const float*)e.g, i, n, e.cols, e.ldg, flat, g);
      if (BITS == 32) {
        aw_load4((const float*)e.m, i, n, 1, 1, flat, m);
        aw_load4((const float*)e.v, i, n, 1, 1, flat, v);
      } else {
        const long long b = i >> 7;
        aw_decode(aw_load_codes((const uint8_t*)e.m, i, n, flat), e.m_scale[b], m);
        aw_decode(aw_load_codes((const uint8_t*)e.v, i, n, flat), e.v_scale[b], v);
      }
      float r[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float gk = g[k] * gf;
        m[k] = fmaf(a.beta1, m[k], a.one_minus_beta1 * gk);
        const float old = BITS == 32 ? v[k] : v[k] * v[k];
        v[k] = fmaf(a.beta2, old, a.one_minus_beta2 * gk * gk);
        r[k] = BITS == 32 ? 0.f : sqrtf(v[k]);
        const float move = step1 * m[k] / (sqrtf(v[k] * lift2) + a.eps);
        p[k] = p[k] - fmaf(lr * e.decay, p[k], move);
      }
      aw_store4(e.p, i, n, e.cols, e.ldp, flat, p);
      if (e.w) aw_store4(e.w, i, n, e.cols, e.ldw, flat, p);
      if (BITS == 32) {
        aw_store4((float*)e.m, i, n, 1, 1, flat, m);
        aw_store4((float*)e.v, i, n, 1, 1, flat, v);
      } else {
        uint32_t c[4] = {(uint32_t)t, (uint32_t)(t >> 32), (uint32_t)(i >> 2), e.number};
        philox4x32_10(c, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
        uint32_t low[4], high[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          low[k] = c[k] & 0xFFFFu;
          high[k] = c[k] >> 16;
          if (i + k >= n) m[k] = r[k] = 0.f;
        }
        float ms, vs;
        const uint32_t mq = aw_encode<false>(m, low, ms), vq = aw_encode<true>(r, high, vs);
        aw_store_codes((uint8_t*)e.m, i, n, flat, mq);
        aw_store_codes((uint8_t*)e.v, i, n, flat, vq);
        if ((threadIdx.x & 31) == 0) {
          e.m_scale[i >> 7] = ms;
          e.v_scale[i >> 7] = vs;
        }
      }
    }
  }
}

// ---- norm of all gradients ------------------------------------------------------------------------
constexpr int GN_QUADS = 4;
constexpr int GN_TILE = GN_QUADS * AW_THREADS * 4;

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
    float g[GN_QUADS][4];
#pragma unroll
    for (int u = 0; u < GN_QUADS; ++u) {
      const long long i = base + (u * AW_THREADS + threadIdx.x) * 4;
      if (e.g_is_bf16) aw_load4((const __nv_bfloat16*)e.g, i, e.n, e.cols, e.ldg, e.flat, g[u]);
      else aw_load4((const float*)e.g, i, e.n, e.cols, e.ldg, e.flat, g[u]);
    }
#pragma unroll
    for (int u = 0; u < GN_QUADS; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k) sum = fma((double)g[u][k], (double)g[u][k], sum);
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
    const unsigned long long room = 8ull * ctx->sm_count;
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
