// Layer norm over the rows of a matrix, and its adjoint with the reduction of the weight's and the bias's gradient; over all columns or
// over the compact columns that a row pattern keeps.
//
// One pass over memory bounds both: the forward call reads x and writes y, the backward call reads x and dy and writes dx.
#include "ard_internal.h"

namespace {

struct LnShape {
  const int32_t* hdr;  // nullptr: all N columns
  int rows, N;
};
struct LnCols {
  int n, dp, b0;  // compact columns, and the unit of column j: b0 + j * dp
};
__device__ __forceinline__ LnCols ln_cols(const LnShape& sh) {
  if (!sh.hdr) return {sh.N, 1, 0};
  return {sh.hdr[HDR_NKEEP], sh.hdr[HDR_DP], sh.hdr[HDR_B] - 1};
}

__device__ __forceinline__ float ln_get(const float* x, size_t i) { return x[i]; }
__device__ __forceinline__ float ln_get(const __nv_bfloat16* x, size_t i) { return __bfloat162float(x[i]); }
__device__ __forceinline__ void ln_put(float* x, size_t i, float v) { x[i] = v; }
__device__ __forceinline__ void ln_put(__nv_bfloat16* x, size_t i, float v) { x[i] = __float2bfloat16(v); }

constexpr int LN_ANY_THREADS = 256;

__device__ __forceinline__ float ln_block_sum(float x, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  x = 0.f;
#pragma unroll
  for (int k = 0; k < LN_ANY_THREADS / 32; ++k) x += red[k];
  return x;
}

// Rows of any alignment and any length: a CTA per row, element by element, the row read again for each sum.
template <typename T>
__global__ void __launch_bounds__(LN_ANY_THREADS) ln_fwd_any_kernel(LnShape sh, float eps, const T* X, int ldx, const float* weight,
                                                                   const float* bias, T* Y, int ldy, float* mean, float* rstd) {
  __shared__ float red[LN_ANY_THREADS / 32];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const LnCols c = ln_cols(sh);
  const float inv_n = 1.f / (float)c.n;
  for (int r = blockIdx.x; r < sh.rows; r += gridDim.x) {
    const T* x = X + (size_t)r * ldx;
    T* y = Y + (size_t)r * ldy;
    float s = 0.f;
    for (int j = threadIdx.x; j < c.n; j += LN_ANY_THREADS) s += ln_get(x, j);
    const float mu = ln_block_sum(s, red) * inv_n;
    s = 0.f;
    for (int j = threadIdx.x; j < c.n; j += LN_ANY_THREADS) {
      const float d = ln_get(x, j) - mu;
      s = fmaf(d, d, s);
    }
    const float rs = 1.f / sqrtf(fmaf(ln_block_sum(s, red), inv_n, eps));
    for (int j = threadIdx.x; j < c.n; j += LN_ANY_THREADS) {
      const int u = c.b0 + j * c.dp;
      ln_put(y, j, fmaf((ln_get(x, j) - mu) * rs, weight ? weight[u] : 1.f, bias ? bias[u] : 0.f));
    }
    if (threadIdx.x == 0) {
      if (mean) mean[r] = mu;
      if (rstd) rstd[r] = rs;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(LN_ANY_THREADS) ln_dx_any_kernel(LnShape sh, const T* dY, int lddy, const T* X, int ldx,
                                                                  const float* weight, const float* mean, const float* rstd, T* dX,
                                                                  int lddx) {
  __shared__ float red[LN_ANY_THREADS / 32];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const LnCols c = ln_cols(sh);
  const float inv_n = 1.f / (float)c.n;
  for (int r = blockIdx.x; r < sh.rows; r += gridDim.x) {
    const T* x = X + (size_t)r * ldx;
    const T* dy = dY + (size_t)r * lddy;
    T* dx = dX + (size_t)r * lddx;
    const float mu = mean[r], rs = rstd[r];
    float s1 = 0.f, s2 = 0.f;
    for (int j = threadIdx.x; j < c.n; j += LN_ANY_THREADS) {
      const float e = ln_get(dy, j) * (weight ? weight[c.b0 + j * c.dp] : 1.f);
      s1 += e;
      s2 = fmaf(e, (ln_get(x, j) - mu) * rs, s2);
    }
    s1 = ln_block_sum(s1, red) * inv_n;
    s2 = ln_block_sum(s2, red) * inv_n;
    for (int j = threadIdx.x; j < c.n; j += LN_ANY_THREADS) {
      const float e = ln_get(dy, j) * (weight ? weight[c.b0 + j * c.dp] : 1.f);
      ln_put(dx, j, rs * (e - s1 - (ln_get(x, j) - mu) * rs * s2));
    }
  }
}

// Sums of dy * xh and dy over a slice of the rows: partial [slice][2][N], column j at place j.
template <typename T>
__global__ void __launch_bounds__(LN_ANY_THREADS) ln_dw_any_kernel(LnShape sh, const T* dY, int lddy, const T* X, int ldx,
                                                                  const float* mean, const float* rstd, float* partial, int per_slice) {
  __shared__ float red[2][LN_ANY_THREADS / 32][32];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int n = ln_cols(sh).n, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slice = blockIdx.y, r1 = min((long long)sh.rows, (long long)(slice + 1) * per_slice);
  for (int c0 = blockIdx.x * 32; c0 < n; c0 += gridDim.x * 32) {
    const int j = c0 + lane;
    float w = 0.f, b = 0.f;
    if (j < n)
      for (int r = slice * per_slice + warp; r < r1; r += LN_ANY_THREADS / 32) {
        const float dy = ln_get(dY, (size_t)r * lddy + j);
        w = fmaf(dy, (ln_get(X, (size_t)r * ldx + j) - mean[r]) * rstd[r], w);
        b += dy;
      }
    red[0][warp][lane] = w;
    red[1][warp][lane] = b;
    __syncthreads();
    if (warp < 2 && j < n) {
      float t = 0.f;
#pragma unroll
      for (int k = 0; k < LN_ANY_THREADS / 32; ++k) t += red[warp][k][lane];
      partial[((size_t)slice * 2 + warp) * sh.N + j] = t;
    }
    __syncthreads();
  }
}

// The slices' sums added in their order, into the units' places: a warp's lanes take 32 columns, its CTA's 8 warps the slices.
__global__ void __launch_bounds__(LN_ANY_THREADS) ln_dw_sum_kernel(LnShape sh, const float* partial, int slices, float* dweight,
                                                                  float* dbias, int zero_fill) {
  __shared__ float red[LN_ANY_THREADS / 32][33];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const LnCols c = ln_cols(sh);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, which = blockIdx.y;
  float* out = which ? dbias : dweight;
  if (!out) return;
  const int j = blockIdx.x * 32 + lane;
  float t = 0.f;
  if (j < c.n)
    for (int k = warp; k < slices; k += LN_ANY_THREADS / 32) t += partial[((size_t)k * 2 + which) * sh.N + j];
  red[warp][lane] = t;
  __syncthreads();
  if (warp == 0) {
    t = 0.f;
#pragma unroll
    for (int k = 0; k < LN_ANY_THREADS / 32; ++k) t += red[k][lane];
    if (j < c.n) out[c.b0 + j * c.dp] = t;
    if (sh.hdr && zero_fill && j < sh.N) {  // this CTA's share of the dropped units
      const int rel = j - c.b0;
      if (rel < 0 || rel % c.dp != 0) out[j] = 0.f;
    }
  }
}

template <typename T>
ard_status ln_fwd(ard_ctx* ctx, const LnShape& sh, float eps, const T* X, int ldx, const float* weight, const float* bias, T* Y, int ldy,
                  float* mean, float* rstd, cudaStream_t s) {
  const int room = 8 * ctx->sm_count;
  ARD_CUDA_OK(ard_launch(ctx, ln_fwd_any_kernel<T>, dim3(sh.rows < room ? sh.rows : room), dim3(LN_ANY_THREADS), 0, s, sh, eps, X, ldx,
                         weight, bias, Y, ldy, mean, rstd));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}

template <typename T>
ard_status ln_bwd(ard_ctx* ctx, const LnShape& sh, const T* dY, int lddy, const T* X, int ldx, const float* weight, const float* mean,
                  const float* rstd, T* dX, int lddx, float* dweight, float* dbias, int zero_fill, cudaStream_t s) {
  if (dX && sh.rows > 0) {
    const int room = 8 * ctx->sm_count;
    ARD_CUDA_OK(ard_launch(ctx, ln_dx_any_kernel<T>, dim3(sh.rows < room ? sh.rows : room), dim3(LN_ANY_THREADS), 0, s, sh, dY, lddy, X,
                           ldx, weight, mean, rstd, dX, lddx));
    ctx->launches++;
  }
  if (dweight || dbias) {
    const long long fit = (long long)(sk_ws_bytes(ctx->sm_count) / sizeof(float) / 2) / sh.N;
    if (!ctx->d_sk_ws || fit < 1) return ARD_ERR_UNSUPPORTED;
    const int gx = (sh.N + 31) / 32;
    long long slices = (sh.rows + 63) / 64;
    if (slices > fit) slices = fit;
    if (slices > 1024) slices = 1024;
    int per = slices > 0 ? (int)((sh.rows + slices - 1) / slices) : 0;
    slices = per > 0 ? (sh.rows + per - 1) / per : 0;
    float* partial = (float*)ctx->d_sk_ws;
    if (slices > 0) {
      ARD_CUDA_OK(ard_launch(ctx, ln_dw_any_kernel<T>, dim3(gx < 4096 ? gx : 4096, (unsigned)slices), dim3(LN_ANY_THREADS), 0, s, sh, dY,
                             lddy, X, ldx, mean, rstd, partial, per));
      ctx->launches++;
    }
    ARD_CUDA_OK(ard_launch(ctx, ln_dw_sum_kernel, dim3(gx, 2), dim3(LN_ANY_THREADS), 0, s, sh, (const float*)partial, (int)slices, dweight,
                           dbias, zero_fill));
    ctx->launches++;
  }
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}

}  // namespace

ard_status launch_layer_norm_fwd(ard_ctx* ctx, const int32_t* hdr, ard_dtype dtype, int rows, int N, float eps, const void* X, int ldx,
                                 const float* weight, const float* bias, void* Y, int ldy, float* mean, float* rstd, cudaStream_t s) {
  if (rows == 0 || N == 0) return ARD_OK;
  const LnShape sh{hdr, rows, N};
  if (dtype == ARD_F32) return ln_fwd(ctx, sh, eps, (const float*)X, ldx, weight, bias, (float*)Y, ldy, mean, rstd, s);
  return ln_fwd(ctx, sh, eps, (const __nv_bfloat16*)X, ldx, weight, bias, (__nv_bfloat16*)Y, ldy, mean, rstd, s);
}

ard_status launch_layer_norm_bwd(ard_ctx* ctx, const int32_t* hdr, ard_dtype dtype, int rows, int N, const void* dY, int lddy,
                                 const void* X, int ldx, const float* weight, const float* mean, const float* rstd, void* dX, int lddx,
                                 float* dweight, float* dbias, int zero_fill, cudaStream_t s) {
  if (N == 0) return ARD_OK;
  const LnShape sh{hdr, rows, N};
  if (dtype == ARD_F32)
    return ln_bwd(ctx, sh, (const float*)dY, lddy, (const float*)X, ldx, weight, mean, rstd, (float*)dX, lddx, dweight, dbias, zero_fill, s);
  return ln_bwd(ctx, sh, (const __nv_bfloat16*)dY, lddy, (const __nv_bfloat16*)X, ldx, weight, mean, rstd, (__nv_bfloat16*)dX, lddx, dweight,
                dbias, zero_fill, s);
}
