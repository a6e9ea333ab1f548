// Layer norm over the rows of a matrix, and its adjoint with the reduction of the weight's and the bias's gradient;
// over all columns or over the compact columns that a row pattern keeps.
//
// One pass over memory bounds both: the forward call reads x and writes y, the backward call reads x and dy and writes
// dx.
#include <type_traits>

#include "ard_internal.h"
#include "sm100_ptx.h"

namespace {

struct LnShape {
  const int32_t* hdr;  // nullptr: all N columns
  int rows, N;
  __host__ __device__ __forceinline__ int pitch() const { return (N + 3) & ~3; }  // of a row of partial sums (N <= 4 million): written in pieces of 16 bytes
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

// The device's estimate and a Newton step: within an ulp or two, at a quarter of a root and a quotient's instructions,
// which every thread of a row spends.
__device__ __forceinline__ float ln_rsqrt(float x) {
  const float y = rsqrtf(x), h = y * fmaf(-x * y, y, 1.f);  // an infinite y (x = 0) or a NaN stays what it is
  return isfinite(h) ? fmaf(0.5f, h, y) : y;
}

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

// Rows of any length, and few short ones: a CTA per row, element by element, the row read again for each sum.  J counts
// the columns: int, or long long where the number behind the last trip's may pass 2^31 (for all rows: 700 x 1500
// forward 6.3 us in place of 4.4).
constexpr int LN_INT_N = 1 << 30;
template <typename T, typename J>
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
    for (J j = threadIdx.x; j < c.n; j += LN_ANY_THREADS) s += ln_get(x, j);
    const float mu = ln_block_sum(s, red) * inv_n;
    s = 0.f;
    for (J j = threadIdx.x; j < c.n; j += LN_ANY_THREADS) {
      const float d = ln_get(x, j) - mu;
      s = fmaf(d, d, s);
    }
    const float rs = ln_rsqrt(fmaf(ln_block_sum(s, red), inv_n, eps));
    for (J j = threadIdx.x; j < c.n; j += LN_ANY_THREADS) {
      const J u = c.b0 + j * c.dp;
      ln_put(y, j, fmaf((ln_get(x, j) - mu) * rs, weight ? weight[u] : 1.f, bias ? bias[u] : 0.f));
    }
    if (threadIdx.x == 0) {
      if (mean) mean[r] = mu;
      if (rstd) rstd[r] = rs;
    }
  }
}

template <typename T, typename J>
__device__ __forceinline__ void ln_dx_any(const LnShape& sh, const LnCols& c, const T* dY, int lddy, const T* X, int ldx, const float* weight,
                                          const float* mean, const float* rstd, T* dX, int lddx, int first, int blocks) {
  __shared__ float red[2][LN_ANY_THREADS / 32];
  const float inv_n = 1.f / (float)c.n;
  for (int r = first; r < sh.rows; r += blocks) {
    const T* x = X + (size_t)r * ldx;
    const T* dy = dY + (size_t)r * lddy;
    T* dx = dX + (size_t)r * lddx;
    const float mu = mean[r], rs = rstd[r];
    float s1 = 0.f, s2 = 0.f;
    for (J j = threadIdx.x; j < c.n; j += LN_ANY_THREADS) {
      const float e = ln_get(dy, j) * (weight ? weight[c.b0 + j * c.dp] : 1.f);
      s1 += e;
      s2 = fmaf(e, (ln_get(x, j) - mu) * rs, s2);
    }
    s1 = ln_block_sum(s1, red[0]) * inv_n;
    s2 = ln_block_sum(s2, red[1]) * inv_n;
    for (J j = threadIdx.x; j < c.n; j += LN_ANY_THREADS) {
      const float e = ln_get(dy, j) * (weight ? weight[c.b0 + j * c.dp] : 1.f);
      ln_put(dx, j, rs * (e - s1 - (ln_get(x, j) - mu) * rs * s2));
    }
  }
}
// Sums of dy * xh and dy over a slice of the rows: partial [slice][2][N], column j at place j.
template <typename T>
__device__ __forceinline__ void ln_dw_any(const LnShape& sh, int n, const T* dY, int lddy, const T* X, int ldx, const float* mean,
                                          const float* rstd, float* partial, int per_slice, int slice, int first, int blocks) {
  constexpr int WARPS = LN_ANY_THREADS / 32;
  __shared__ float red[2][WARPS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int r1 = (int)min((long long)sh.rows, (long long)(slice + 1) * per_slice);
  for (int c0 = first * 32; c0 < n; c0 += blocks * 32) {
    const int j = c0 + lane;
    float w = 0.f, b = 0.f;
    if (j < n)
      for (int r0 = slice * per_slice + warp; r0 < r1; r0 += 4 * WARPS) {  // four rows' loads at once
        float x[4], dy[4], m[4], q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int r = min(r0 + u * WARPS, r1 - 1);
          dy[u] = ln_get(dY, (size_t)r * lddy + j);
          x[u] = ln_get(X, (size_t)r * ldx + j);
          m[u] = mean[r];
          q[u] = rstd[r];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (r0 + u * WARPS < r1) {
            w = fmaf(dy[u], (x[u] - m[u]) * q[u], w);
            b += dy[u];
          }
      }
    red[0][warp][lane] = w;
    red[1][warp][lane] = b;
    __syncthreads();
    if (warp < 2 && j < n) {
      float t = 0.f;
#pragma unroll
      for (int k = 0; k < WARPS; ++k) t += red[warp][k][lane];
      partial[((size_t)slice * 2 + warp) * sh.pitch() + j] = t;
    }
    __syncthreads();
  }
}
// Both in one launch: the first dx_blocks CTAs take rows, the others columns, gx of them a slice.
template <typename T, typename J>
__global__ void __launch_bounds__(LN_ANY_THREADS) ln_bwd_any_kernel(LnShape sh, const T* dY, int lddy, const T* X, int ldx, const float* weight,
                                                                   const float* mean, const float* rstd, T* dX, int lddx, int dx_blocks,
                                                                   float* partial, int per_slice, int gx) {
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const LnCols c = ln_cols(sh);
  const int k = (int)blockIdx.x - dx_blocks;
  if (k < 0) ln_dx_any<T, J>(sh, c, dY, lddy, X, ldx, weight, mean, rstd, dX, lddx, (int)blockIdx.x, dx_blocks);
  else ln_dw_any(sh, c.n, dY, lddy, X, ldx, mean, rstd, partial, per_slice, k / gx, k % gx, gx);
}

// The slices' sums added in a fixed order, into the units' places: a warp's lanes take 32 columns, its CTA's warps the
// slices.
constexpr int LN_SUM_WARPS = 32;
__global__ void __launch_bounds__(LN_SUM_WARPS * 32) ln_dw_sum_kernel(LnShape sh, const float* partial, int slices, float* dweight,
                                                                     float* dbias, int zero_fill) {
  __shared__ float red[LN_SUM_WARPS][33];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const LnCols c = ln_cols(sh);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, which = blockIdx.y;
  float* out = which ? dbias : dweight;
  if (!out) return;
  const int j = blockIdx.x * 32 + lane;
  float t = 0.f;
  if (j < c.n) {
    // eight at once, asked one by one: left to itself the compiler takes the last seven of a loop after one another,
    // each a trip to the L2
    for (int k0 = warp; k0 < slices; k0 += 8 * LN_SUM_WARPS) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int k = k0 + u * LN_SUM_WARPS;
        x[u] = k < slices ? partial[((size_t)k * 2 + which) * sh.pitch() + j] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) t += x[u];
    }
  }
  red[warp][lane] = t;
  __syncthreads();
  if (warp == 0) {
    t = 0.f;
#pragma unroll
    for (int k = 0; k < LN_SUM_WARPS; ++k) t += red[k][lane];
    if (j < c.n) out[c.b0 + j * c.dp] = t;
    if (sh.hdr && zero_fill && j < sh.N) {  // this CTA's share of the dropped units
      const int rel = j - c.b0;
      if (rel < 0 || rel % c.dp != 0) out[j] = 0.f;
    }
  }
}

// ---- rows through rings of bulk copies ---------------------------------------------------------------
// TPR threads hold a row, V pieces of 16 bytes each: piece v of thread t is number v * TPR + t.  16384 x 2048 bf16, forward / backward: 27.6 / 46.7 us (a
// copy of the same bytes 20.6 / 30.8); the loads keep up, half of the issue slots are taken, warps wait for one another at the sums' barriers.  ON16: rows on
// a 16-byte grid; others are cut out of the copies in shared memory and stored in pieces as wide as their grid (on 8 bytes 39 / 72 us, on 2 bytes
// 53 / 77; a CTA a row element by element 75 / 141).
template <typename T>
constexpr int LN_PER = 16 / (int)sizeof(T);  // elements of a piece

// Two elements in one instruction (f32x2): with one each these kernels run out of issue slots before the memory is
// busy.
__device__ __forceinline__ float2 operator*(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 operator+(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 ln_fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 ln_both(float x) { return make_float2(x, x); }

template <typename T>
constexpr int LN_PAIRS = LN_PER<T> / 2;
template <typename T>
__device__ __forceinline__ void ln_unpack(const uint4& q, float2 (&v)[LN_PAIRS<T>]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = make_float2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xFFFF0000u));
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) v[k] = make_float2(__uint_as_float(w[2 * k]), __uint_as_float(w[2 * k + 1]));
  }
}
// The piece of column j from shared memory, elements from column n on as zero.  RAGGED: n may end inside a piece (asked
// once for all rows: the questions, predicated rather than branched around, were two thirds of the instructions).
// Without ON16 the row begins at byte `off` of its place: the piece is cut out of the 32 bytes that it lies in.
template <typename T, bool RAGGED, bool ON16>
__device__ __forceinline__ void ln_piece(const uint8_t* row, int off, int j, int n, float2 (&v)[LN_PAIRS<T>]) {
  uint4 q = make_uint4(0u, 0u, 0u, 0u);
  if (j < n) {
    q = *reinterpret_cast<const uint4*>(row + (size_t)j * sizeof(T));
    if constexpr (!ON16) {
      const uint4 r = *reinterpret_cast<const uint4*>(row + (size_t)j * sizeof(T) + 16);
      uint32_t w[8] = {q.x, q.y, q.z, q.w, r.x, r.y, r.z, r.w};
#pragma unroll
      for (int k = 0; k < 6; ++k) w[k] = off & 8 ? w[k + 2] : w[k];
#pragma unroll
      for (int k = 0; k < 5; ++k) w[k] = off & 4 ? w[k + 1] : w[k];
      const int bits = sizeof(T) == 2 ? (off & 2) * 8 : 0;
      q = make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                     __funnelshift_r(w[3], w[4], bits));
    }
  }
  ln_unpack<T>(q, v);
  if (RAGGED && j + LN_PER<T> > n)
#pragma unroll
    for (int k = 0; k < LN_PAIRS<T>; ++k) {
      if (j + 2 * k >= n) v[k].x = 0.f;
      if (j + 2 * k + 1 >= n) v[k].y = 0.f;
    }
}
// The first `valid` values of a piece.
template <typename T, bool RAGGED, bool ON16>
__device__ __forceinline__ void ln_store(T* p, int valid, const float2 (&v)[LN_PAIRS<T>]) {
  if (!RAGGED || valid >= LN_PER<T>) {
    uint32_t w[4];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        __nv_bfloat162 b = __floats2bfloat162_rn(v[k].x, v[k].y);
        w[k] = *reinterpret_cast<uint32_t*>(&b);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        w[2 * k] = __float_as_uint(v[k].x);
        w[2 * k + 1] = __float_as_uint(v[k].y);
      }
    }
    const uint32_t off = ON16 ? 0u : (uint32_t)reinterpret_cast<uintptr_t>(p);  // its low bits are those of all of a row's pieces
    if ((off & 15u) == 0) {
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else if ((off & 7u) == 0) {
#pragma unroll
      for (int k = 0; k < 2; ++k) reinterpret_cast<uint2*>(p)[k] = make_uint2(w[2 * k], w[2 * k + 1]);
    } else if ((off & 3u) == 0) {
#pragma unroll
      for (int k = 0; k < 4; ++k) reinterpret_cast<uint32_t*>(p)[k] = w[k];
    } else {  // 2-byte elements
      uint16_t* h = reinterpret_cast<uint16_t*>(p);
      h[0] = (uint16_t)w[0];
#pragma unroll
      for (int k = 0; k < 3; ++k) *reinterpret_cast<uint32_t*>(h + 1 + 2 * k) = __funnelshift_r(w[k], w[k + 1], 16);
      h[7] = (uint16_t)(w[3] >> 16);
    }
  } else {
#pragma unroll
    for (int k = 0; k < LN_PAIRS<T>; ++k) {
      if (2 * k < valid) ln_put(p, 2 * k, v[k].x);
      if (2 * k + 1 < valid) ln_put(p, 2 * k + 1, v[k].y);
    }
  }
}
// weight or bias at the units of a piece's columns; `other` where there is none.
template <int PAIRS>
__device__ __forceinline__ void ln_params(const float* w, float other, const LnCols& c, int j, float2 (&v)[PAIRS]) {
#pragma unroll
  for (int k = 0; k < PAIRS; ++k) {
    v[k].x = w && j + 2 * k < c.n ? w[c.b0 + (size_t)(j + 2 * k) * c.dp] : other;
    v[k].y = w && j + 2 * k + 1 < c.n ? w[c.b0 + (size_t)(j + 2 * k + 1) * c.dp] : other;
  }
}
// The same of whole pieces on 16 bytes, all columns kept; not to be kept in registers (CTAs of 1024 threads, 64
// registers each): they come from the L1 cache for every row.
template <int PAIRS>
__device__ __forceinline__ void ln_params_now(const float* w, float other, int j, float2 (&v)[PAIRS]) {
#pragma unroll
  for (int k = 0; k < PAIRS; k += 2) {
    float4 q = make_float4(other, other, other, other);
    if (w) asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w) : "l"(w + j + 2 * k));
    v[k] = make_float2(q.x, q.y);
    v[k + 1] = make_float2(q.z, q.w);
  }
}

// The sums of M values over the TPR threads of a row; with more than a warp through shared memory, of which a call and
// the next use different halves (one barrier of the group per call).
template <int TPR, int M>
__device__ __forceinline__ void ln_row_sums(float (&x)[M], float (*red)[M][32], int& half) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int m = 0; m < M; ++m) x[m] += __shfl_xor_sync(0xFFFFFFFFu, x[m], o);
  if constexpr (TPR > 32) {
    constexpr int W = TPR / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0)
#pragma unroll
      for (int m = 0; m < M; ++m) red[half][m][warp] = x[m];
    asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / TPR), "n"(TPR) : "memory");
#pragma unroll
    for (int m = 0; m < M; ++m) {
      float t = 0.f;
      const float* r = &red[half][m][warp / W * W];
#pragma unroll
      for (int k = 0; k < W; ++k) t += r[k];
      x[m] = t;
    }
    half ^= 1;
  }
}

// Rows reach the TPR threads that hold them through a ring of slots in shared memory, filled by bulk copies that the
// first of them asks for several rounds ahead: what is in flight costs no registers, and 100 to 200 KB an SM are in
// flight whatever the row's length.  A round is R consecutive rows: their sums share barriers and run beside one
// another.
constexpr int LN_SLOTS = 8;
struct LnRing {
  int slots;      // per group of threads
  int row_bytes;  // of an operand, rounded up to 16 bytes; 16 more where rows begin anywhere
};
template <typename T, int TPR, int G, int R, int M, bool ON16>
struct LnRows {
  const T* src[M];
  int ld[M];
  uint8_t* mine;
  uint64_t* full;
  LnRing ring;
  int g0, stride, rounds, rows, n;
  uint32_t bytes;
  int slot, phase;  // of the round that is being worked on
  bool gone;        // a copy did not come within two seconds: the rest is left, the status says so
  int gone_at;

  __device__ __forceinline__ LnRows(const LnShape& sh, const LnCols& c, LnRing rg, uint8_t* slots, uint64_t (*bars)[LN_SLOTS]) {
    const int g = threadIdx.x / TPR;
    ring = rg;
    mine = slots + (size_t)g * ring.slots * (M * R * ring.row_bytes);
    full = bars[g];
    bytes = ((uint32_t)c.n * (uint32_t)sizeof(T) + 15u) & ~15u;
    n = c.n;
    rows = sh.rows;
    stride = gridDim.x * G;
    rounds = ((rows + R - 1) / R + stride - 1) / stride;
    g0 = blockIdx.x * G + g;
    slot = phase = 0;
    gone = false;
    gone_at = 0;
  }
  __device__ __forceinline__ long long row(int it, int q) const { return (g0 + (long long)it * stride) * R + q; }
  __device__ __forceinline__ bool live(int it, int q) const { return row(it, q) < rows && !gone; }
  // Where operand m of row q of round `it` begins within 16 bytes: copies start at the 16-byte boundary before it.
  __device__ __forceinline__ int off(int it, int q, int m) const {
    return ON16 ? 0 : (int)(((uint32_t)reinterpret_cast<uintptr_t>(src[m]) + (uint32_t)row(it, q) * (uint32_t)ld[m] * (uint32_t)sizeof(T)) & 15u);
  }
  __device__ __forceinline__ uint32_t size(int it, int q, int m) const {
    return ON16 ? bytes : (uint32_t)(off(it, q, m) + n * (int)sizeof(T) + 15) & ~15u;
  }
  __device__ __forceinline__ const uint8_t* at(int q, int m) const { return mine + (size_t)((slot * R + q) * M + m) * ring.row_bytes; }
  // By the first thread of the group, for round `it`; whoever read the slot before has passed a barrier since.
  __device__ __forceinline__ void ask(int it) const {
    if (it >= rounds || row(it, 0) >= rows || gone) return;
    const int to = it % ring.slots, here = (int)min((long long)R, rows - row(it, 0));
    const uint32_t bar = smem_u32(&full[to]), dst = smem_u32(mine + (size_t)to * (M * R * ring.row_bytes));
    uint32_t all = (uint32_t)(M * here) * bytes;
    if constexpr (!ON16) {
      all = 0;
      for (int q = 0; q < here; ++q)
#pragma unroll
        for (int m = 0; m < M; ++m) all += size(it, q, m);
    }
    mbar_arrive_expect_tx(bar, all);
    for (int q = 0; q < here; ++q)
#pragma unroll
      for (int m = 0; m < M; ++m)
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                         dst + (uint32_t)((q * M + m) * ring.row_bytes)),
                     "l"(reinterpret_cast<const uint8_t*>(src[m] + (size_t)row(it, q) * ld[m]) - off(it, q, m)), "r"(size(it, q, m)), "r"(bar)
                     : "memory");
  }
  __device__ __forceinline__ void wait(int it, volatile int* s_gone, int* status) {
    if (!gone && row(it, 0) < rows && !mbar_wait(smem_u32(&full[slot]), (uint32_t)phase, s_gone, status)) {
      gone = true;
      gone_at = it;
    }
  }
  __device__ __forceinline__ void next() {
    if (++slot == ring.slots) {
      slot = 0;
      phase ^= 1;
    }
  }
  // Before the CTA ends without some of its copies (asked up to round `asked`): they get the same time, for they write
  // to its memory.
  __device__ __forceinline__ void drain(int asked) const {
    for (int it = gone_at; it <= asked && it < rounds && row(it, 0) < rows; ++it) {
      bool ok = false;
      for (int poll = 0; poll < 2000 && !ok; ++poll) ok = mbar_try_wait_hint(smem_u32(&full[it % ring.slots]), (uint32_t)(it / ring.slots) & 1u, 1000000u);
    }
  }
};
template <int G>
__device__ __forceinline__ void ln_setup(uint64_t (*full)[LN_SLOTS], int slots, int* s_gone) {
  if (threadIdx.x == 0) {
    *s_gone = 0;
    for (int g = 0; g < G; ++g)
      for (int k = 0; k < slots; ++k) mbar_init(smem_u32(&full[g][k]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  pdl_launch_dependents();
  pdl_wait_prior_grids();
}

// Forward: two sums over a row's registers, the second about the mean (a sum of squares alone loses the variance of a
// row with a large mean).  The barrier of the first one says that the round's slot has been read.
template <typename T, int TPR, int V, int NT, int R, bool ON16>
__global__ void __launch_bounds__(NT, NT >= 512 ? 1 : 512 / NT) ln_fwd_kernel(LnShape sh, float eps, const T* X, int ldx, const float* weight, const float* bias,
                                                       T* Y, int ldy, float* mean, float* rstd, LnRing ring, int* status) {
  constexpr int PER = LN_PER<T>, PAIRS = LN_PAIRS<T>, G = NT / TPR;
  constexpr bool KEEP = NT < 1024;
  constexpr int one = KEEP ? 1 : 0;
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ float red[2][R][32];
  __shared__ __align__(8) uint64_t full[G][LN_SLOTS];
  __shared__ int s_gone;
  ln_setup<G>(full, ring.slots, &s_gone);
  const int t = threadIdx.x % TPR;
  const LnCols c = ln_cols(sh);
  const float inv_n = 1.f / (float)c.n;
  LnRows<T, TPR, G, R, 1, ON16> in(sh, c, ring, slots, full);
  in.src[0] = X;
  in.ld[0] = ldx;
  if (t == 0)
    for (int k = 0; k < ring.slots; ++k) in.ask(k);
  float2 w[KEEP ? V : 1][PAIRS], b[KEEP ? V : 1][PAIRS];
  if constexpr (KEEP)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      ln_params<PAIRS>(weight, 1.f, c, (v * TPR + t) * PER, w[v]);
      ln_params<PAIRS>(bias, 0.f, c, (v * TPR + t) * PER, b[v]);
    }
  int half = 0;
  auto loop = [&](auto ragged) {
    constexpr bool RAGGED = decltype(ragged)::value;
    for (int it = 0; it < in.rounds; ++it) {
      in.wait(it, &s_gone, status);
      float2 x[R][V][PAIRS];
      float s[R], mu[R];
#pragma unroll
      for (int q = 0; q < R; ++q) {
        float2 sum = ln_both(0.f);
        const int n = in.live(it, q) ? c.n : 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          ln_piece<T, RAGGED, ON16>(in.at(q, 0), in.off(it, q, 0), (v * TPR + t) * PER, n, x[q][v]);
#pragma unroll
          for (int k = 0; k < PAIRS; ++k) sum = sum + x[q][v][k];
        }
        s[q] = sum.x + sum.y;
      }
      ln_row_sums<TPR, R>(s, red, half);
      if (TPR == 32) __syncwarp();
      if (t == 0) in.ask(it + ring.slots);
      in.next();
#pragma unroll
      for (int q = 0; q < R; ++q) {
        mu[q] = s[q] * inv_n;
        float2 sum = ln_both(0.f);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int j = (v * TPR + t) * PER;
#pragma unroll
          for (int k = 0; k < PAIRS; ++k) x[q][v][k] = x[q][v][k] + ln_both(-mu[q]);
          if (RAGGED ? j + PER > c.n : j >= c.n)
#pragma unroll
            for (int k = 0; k < PAIRS; ++k) {
              if (!RAGGED || j + 2 * k >= c.n) x[q][v][k].x = 0.f;
              if (!RAGGED || j + 2 * k + 1 >= c.n) x[q][v][k].y = 0.f;
            }
#pragma unroll
          for (int k = 0; k < PAIRS; ++k) sum = ln_fma(x[q][v][k], x[q][v][k], sum);
        }
        s[q] = sum.x + sum.y;
      }
      ln_row_sums<TPR, R>(s, red, half);
#pragma unroll
      for (int q = 0; q < R; ++q) {
        if (!in.live(it, q)) continue;
        const float rs = ln_rsqrt(fmaf(s[q], inv_n, eps));
        const long long r = in.row(it, q);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int j = (v * TPR + t) * PER;
          if (j < c.n) {
            if constexpr (!KEEP) {
              ln_params_now<PAIRS>(weight, 1.f, j, w[0]);
              ln_params_now<PAIRS>(bias, 0.f, j, b[0]);
            }
#pragma unroll
            for (int k = 0; k < PAIRS; ++k) x[q][v][k] = ln_fma(x[q][v][k] * ln_both(rs), w[one * v][k], b[one * v][k]);
            ln_store<T, RAGGED, ON16>(Y + (size_t)r * ldy + j, c.n - j, x[q][v]);
          }
        }
        if (t == 0) {
          if (mean) mean[r] = mu[q];
          if (rstd) rstd[r] = rs;
        }
      }
    }
  };
  if (c.n % PER) loop(std::true_type{});
  else loop(std::false_type{});
  if (in.gone && t == 0) in.drain(in.gone_at + ring.slots - 1);
}

// Backward: a thread keeps its columns' sums for the weight and the bias over all rows of the CTA and leaves them in
// `partial` [CTA][2][N].  A row is read from its slot twice, for its sums and for dx, which costs less than the
// registers that would hold it; its slot is asked for again one round later: the barrier of that round's sums says that
// nobody reads it any more.
template <typename T, int TPR, int V, int NT, int R, bool ON16>
__global__ void __launch_bounds__(NT, NT >= 512 ? 1 : 512 / NT) ln_bwd_kernel(LnShape sh, const T* dY, int lddy, const T* X, int ldx, const float* weight,
                                                       const float* mean, const float* rstd, T* dX, int lddx, float* partial,
                                                       LnRing ring, int* status) {
  constexpr int PER = LN_PER<T>, PAIRS = LN_PAIRS<T>, G = NT / TPR;
  constexpr bool KEEP = NT < 1024;
  constexpr int one = KEEP ? 1 : 0;
  extern __shared__ __align__(128) uint8_t slots[];  // at the end the sums of the CTA's groups
  __shared__ float red[2][2 * R][32];
  __shared__ __align__(8) uint64_t full[G][LN_SLOTS];
  __shared__ int s_gone;
  ln_setup<G>(full, ring.slots, &s_gone);
  const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
  const LnCols c = ln_cols(sh);
  const float inv_n = 1.f / (float)c.n;
  LnRows<T, TPR, G, R, 2, ON16> in(sh, c, ring, slots, full);
  in.src[0] = X;
  in.ld[0] = ldx;
  in.src[1] = dY;
  in.ld[1] = lddy;
  if (t == 0)
    for (int k = 0; k < ring.slots; ++k) in.ask(k);
  float2 dw[V][PAIRS], db[V][PAIRS], w[KEEP ? V : 1][PAIRS];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if constexpr (KEEP) ln_params<PAIRS>(weight, 1.f, c, (v * TPR + t) * PER, w[v]);
#pragma unroll
    for (int k = 0; k < PAIRS; ++k) dw[v][k] = db[v][k] = ln_both(0.f);
  }
  int half = 0;
  float mu[R], rs[R];  // of the round's rows; the next ones' are fetched behind this one's arithmetic
  auto stats = [&](int it, int q, float& m, float& r) {
    m = r = 0.f;
    if (it < in.rounds && in.row(it, q) < sh.rows) {
      m = mean[in.row(it, q)];
      r = rstd[in.row(it, q)];
    }
  };
#pragma unroll
  for (int q = 0; q < R; ++q) stats(0, q, mu[q], rs[q]);
  auto loop = [&](auto ragged) {
    constexpr bool RAGGED = decltype(ragged)::value;
    for (int it = 0; it < in.rounds; ++it) {
      in.wait(it, &s_gone, status);
      float mu2[R], rs2[R], s[2 * R];
#pragma unroll
      for (int q = 0; q < R; ++q) stats(it + 1, q, mu2[q], rs2[q]);
#pragma unroll
      for (int q = 0; q < R; ++q) {
        const float2 scale = ln_both(rs[q]), offset = ln_both(-mu[q]);
        float2 s1 = ln_both(0.f), s2 = ln_both(0.f);
        if (in.live(it, q)) {
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const int j = (v * TPR + t) * PER;
            if (j < c.n) {
              float2 x[PAIRS], dy[PAIRS];
              ln_piece<T, RAGGED, ON16>(in.at(q, 0), in.off(it, q, 0), j, c.n, x);
              ln_piece<T, RAGGED, ON16>(in.at(q, 1), in.off(it, q, 1), j, c.n, dy);
              if constexpr (!KEEP) ln_params_now<PAIRS>(weight, 1.f, j, w[0]);
#pragma unroll
              for (int k = 0; k < PAIRS; ++k) {
                const float2 xh = (x[k] + offset) * scale, e = dy[k] * w[one * v][k];
                s1 = s1 + e;
                s2 = ln_fma(e, xh, s2);
                dw[v][k] = ln_fma(dy[k], xh, dw[v][k]);
                db[v][k] = db[v][k] + dy[k];
              }
            }
          }
        }
        s[2 * q] = s1.x + s1.y;
        s[2 * q + 1] = s2.x + s2.y;
      }
      ln_row_sums<TPR, 2 * R>(s, red, half);
      if (TPR == 32) __syncwarp();
      if (t == 0 && it > 0) in.ask(it - 1 + ring.slots);
#pragma unroll
      for (int q = 0; q < R; ++q) {
        if (!dX || !in.live(it, q)) continue;
        const float2 scale = ln_both(rs[q]), offset = ln_both(-mu[q]);
        const float2 s1 = ln_both(-s[2 * q] * inv_n), s2 = ln_both(-s[2 * q + 1] * inv_n);
        T* dx = dX + (size_t)in.row(it, q) * lddx;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int j = (v * TPR + t) * PER;
          if (j < c.n) {
            float2 x[PAIRS], dy[PAIRS];
            ln_piece<T, RAGGED, ON16>(in.at(q, 0), in.off(it, q, 0), j, c.n, x);
            ln_piece<T, RAGGED, ON16>(in.at(q, 1), in.off(it, q, 1), j, c.n, dy);
            if constexpr (!KEEP) ln_params_now<PAIRS>(weight, 1.f, j, w[0]);
#pragma unroll
            for (int k = 0; k < PAIRS; ++k)
              x[k] = scale * ln_fma((x[k] + offset) * scale, s2, ln_fma(dy[k], w[one * v][k], s1));
            ln_store<T, RAGGED, ON16>(dx + j, c.n - j, x);
          }
        }
      }
      in.next();
#pragma unroll
      for (int q = 0; q < R; ++q) {
        mu[q] = mu2[q];
        rs[q] = rs2[q];
      }
    }
  };
  if (c.n % PER) loop(std::true_type{});
  else loop(std::false_type{});
  if (in.gone && t == 0) in.drain(in.gone_at + ring.slots - 1);
  if (!partial) return;
  // the groups' sums added in their order
  if constexpr (G > 1) {
    float2* sums = reinterpret_cast<float2*>(slots);  // [2][V * TPR * PAIRS]
    for (int k = 0; k < G; ++k) {
      __syncthreads();
      if (g == k)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int q = 0; q < PAIRS; ++q) {
            const int j = (v * PAIRS + q) * TPR + t;
            if (k > 0) {
              dw[v][q] = dw[v][q] + sums[j];
              db[v][q] = db[v][q] + sums[V * TPR * PAIRS + j];
            }
            sums[j] = dw[v][q];
            sums[V * TPR * PAIRS + j] = db[v][q];
          }
    }
    if (g != G - 1) return;
  }
  float* to = partial + (size_t)blockIdx.x * 2 * sh.pitch();
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int q = 0; q < PAIRS; q += 2) {
      const int j = (v * TPR + t) * PER + 2 * q;
      if (j < c.n) {  // (behind the last column zeros)
        *reinterpret_cast<float4*>(to + j) = make_float4(dw[v][q].x, dw[v][q].y, dw[v][q + 1].x, dw[v][q + 1].y);
        *reinterpret_cast<float4*>(to + sh.pitch() + j) = make_float4(db[v][q].x, db[v][q].y, db[v][q + 1].x, db[v][q + 1].y);
      }
    }
}

// ---- short rows ------------------------------------------------------------------------------------
// TPR lanes hold a row of up to 8 TPR elements, eight each, from global memory as it is: many rows and many warps (32 an SM) at once, and the next row's
// loads ahead of this one's arithmetic.  16384 x 64 bf16 3.5 / 6.2 us (rings, a warp a row: 8.4 / 12.5), 60000 x 65 8.5 / 17.2
// (29.5 / 46.6), 131072 x 256 forward 36.3 (39).
// WIDE: a lane's elements lie together on 16 bytes; otherwise lanes take neighbouring elements.
constexpr int LN_SHORT = 512, LN_SHORT_N = 256;
template <int TPR, bool WIDE>
__device__ __forceinline__ int ln_short_col(int t, int e) { return WIDE ? t * 8 + e : e * TPR + t; }
template <typename T, int TPR, bool WIDE>
__device__ __forceinline__ void ln_short_load(const T* row, int t, int n, float2 (&v)[4]) {
  if (WIDE && t * 8 + 8 <= n) {
    constexpr int PIECES = sizeof(T) / 2, PAIRS = LN_PAIRS<T>;
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
      const uint4 q = *reinterpret_cast<const uint4*>(row + t * 8 + k * LN_PER<T>);
      float2 x[PAIRS];
      ln_unpack<T>(q, x);
#pragma unroll
      for (int h = 0; h < PAIRS; ++h) v[k * PAIRS + h] = x[h];
    }
    return;
  }
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const int a = ln_short_col<TPR, WIDE>(t, 2 * h), b = ln_short_col<TPR, WIDE>(t, 2 * h + 1);
    v[h].x = a < n ? ln_get(row, a) : 0.f;
    v[h].y = b < n ? ln_get(row, b) : 0.f;
  }
}
template <typename T, int TPR, bool WIDE>
__device__ __forceinline__ void ln_short_store(T* row, int t, int n, const float2 (&v)[4]) {
  if (WIDE && t * 8 + 8 <= n) {
    constexpr int PIECES = sizeof(T) / 2, PAIRS = LN_PAIRS<T>;
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
      float2 x[PAIRS];
#pragma unroll
      for (int h = 0; h < PAIRS; ++h) x[h] = v[k * PAIRS + h];
      ln_store<T, false, true>(row + t * 8 + k * LN_PER<T>, LN_PER<T>, x);
    }
    return;
  }
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const int a = ln_short_col<TPR, WIDE>(t, 2 * h), b = ln_short_col<TPR, WIDE>(t, 2 * h + 1);
    if (a < n) ln_put(row, a, v[h].x);
    if (b < n) ln_put(row, b, v[h].y);
  }
}
template <int TPR, bool WIDE>
__device__ __forceinline__ void ln_short_params(const float* w, float other, const LnCols& c, int t, float2 (&v)[4]) {
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const int a = ln_short_col<TPR, WIDE>(t, 2 * h), b = ln_short_col<TPR, WIDE>(t, 2 * h + 1);
    v[h].x = w && a < c.n ? w[c.b0 + a * c.dp] : other;
    v[h].y = w && b < c.n ? w[c.b0 + b * c.dp] : other;
  }
}
template <int TPR, int M>
__device__ __forceinline__ void ln_lane_sums(float (&x)[M]) {
#pragma unroll
  for (int o = TPR / 2; o > 0; o >>= 1)
#pragma unroll
    for (int m = 0; m < M; ++m) x[m] += __shfl_xor_sync(0xFFFFFFFFu, x[m], o);
}

template <typename T, int TPR, bool WIDE>
__global__ void __launch_bounds__(LN_SHORT, 2) ln_fwd_short_kernel(LnShape sh, float eps, const T* X, int ldx, const float* weight, const float* bias,
                                                                  T* Y, int ldy, float* mean, float* rstd) {
  constexpr int G = LN_SHORT / TPR;
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const LnCols c = ln_cols(sh);
  const float inv_n = 1.f / (float)c.n;
  const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
  const long long stride = (long long)gridDim.x * G;
  float2 w[4], b[4], next[4];
  ln_short_params<TPR, WIDE>(weight, 1.f, c, t, w);
  ln_short_params<TPR, WIDE>(bias, 0.f, c, t, b);
  auto load = [&](long long r) { ln_short_load<T, TPR, WIDE>(X + (size_t)r * ldx, t, r < sh.rows ? c.n : 0, next); };
  long long r0 = (long long)blockIdx.x * G;
  load(r0 + g);
  for (; r0 < sh.rows; r0 += stride) {
    const long long r = r0 + g;
    float2 x[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) x[h] = next[h];
    load(r + stride);
    float2 sum = (x[0] + x[1]) + (x[2] + x[3]);
    float s[1] = {sum.x + sum.y};
    ln_lane_sums<TPR, 1>(s);
    const float mu = s[0] * inv_n;
    sum = ln_both(0.f);
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      x[h] = x[h] + ln_both(-mu);
      if (ln_short_col<TPR, WIDE>(t, 2 * h) >= c.n) x[h].x = 0.f;
      if (ln_short_col<TPR, WIDE>(t, 2 * h + 1) >= c.n) x[h].y = 0.f;
      sum = ln_fma(x[h], x[h], sum);
    }
    s[0] = sum.x + sum.y;
    ln_lane_sums<TPR, 1>(s);
    const float rs = ln_rsqrt(fmaf(s[0], inv_n, eps));
    if (r < sh.rows) {
#pragma unroll
      for (int h = 0; h < 4; ++h) x[h] = ln_fma(x[h] * ln_both(rs), w[h], b[h]);
      ln_short_store<T, TPR, WIDE>(Y + (size_t)r * ldy, t, c.n, x);
      if (t == 0) {
        if (mean) mean[r] = mu;
        if (rstd) rstd[r] = rs;
      }
    }
  }
}

template <typename T, int TPR, bool WIDE>
__global__ void __launch_bounds__(LN_SHORT, 2) ln_bwd_short_kernel(LnShape sh, const T* dY, int lddy, const T* X, int ldx, const float* weight,
                                                                  const float* mean, const float* rstd, T* dX, int lddx, float* partial) {
  constexpr int G = LN_SHORT / TPR, COLS = TPR * 8;
  __shared__ float2 sums[G][2][COLS / 2];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const LnCols c = ln_cols(sh);
  const float inv_n = 1.f / (float)c.n;
  const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
  const long long stride = (long long)gridDim.x * G;
  float2 w[4], dw[4], db[4];
  ln_short_params<TPR, WIDE>(weight, 1.f, c, t, w);
#pragma unroll
  for (int h = 0; h < 4; ++h) dw[h] = db[h] = ln_both(0.f);
  for (long long r0 = (long long)blockIdx.x * G; r0 < sh.rows; r0 += stride) {
    const long long r = r0 + g;
    const bool live = r < sh.rows;
    float2 x[4], dy[4];
    ln_short_load<T, TPR, WIDE>(X + (size_t)r * ldx, t, live ? c.n : 0, x);
    ln_short_load<T, TPR, WIDE>(dY + (size_t)r * lddy, t, live ? c.n : 0, dy);
    const float mu = live ? mean[r] : 0.f, rs = live ? rstd[r] : 0.f;
    float2 s1 = ln_both(0.f), s2 = ln_both(0.f);
#pragma unroll
    for (int h = 0; h < 4; ++h) {  // (behind the last column dy is zero)
      x[h] = (x[h] + ln_both(-mu)) * ln_both(rs);
      dw[h] = ln_fma(dy[h], x[h], dw[h]);
      db[h] = db[h] + dy[h];
      dy[h] = dy[h] * w[h];
      s1 = s1 + dy[h];
      s2 = ln_fma(dy[h], x[h], s2);
    }
    float s[2] = {s1.x + s1.y, s2.x + s2.y};
    ln_lane_sums<TPR, 2>(s);
    if (dX && live) {
      const float2 a = ln_both(-s[0] * inv_n), b = ln_both(-s[1] * inv_n);
#pragma unroll
      for (int h = 0; h < 4; ++h) x[h] = ln_both(rs) * ln_fma(x[h], b, dy[h] + a);
      ln_short_store<T, TPR, WIDE>(dX + (size_t)r * lddx, t, c.n, x);
    }
  }
  if (!partial) return;
  // [group][2][column, in the order of the lanes' elements], added in the groups' order
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    sums[g][0][h * TPR + t] = dw[h];
    sums[g][1][h * TPR + t] = db[h];
  }
  __syncthreads();
  for (int k = threadIdx.x; k < COLS; k += LN_SHORT) {  // pairs of columns of either sum
    const int which = k / (COLS / 2), at = k % (COLS / 2), h = at / TPR, lane = at % TPR;
    float2 sum = ln_both(0.f);
#pragma unroll 8
    for (int q = 0; q < G; ++q) sum = sum + sums[q][which][at];
    float* to = partial + ((size_t)blockIdx.x * 2 + which) * sh.pitch();
    const int ja = ln_short_col<TPR, WIDE>(lane, 2 * h), jb = ln_short_col<TPR, WIDE>(lane, 2 * h + 1);
    if (ja < c.n) to[ja] = sum.x;
    if (jb < c.n) to[jb] = sum.y;
  }
}

inline bool ln_on16(const void* p, long long ld_bytes) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld_bytes % 16 == 0; }

// A CTA for each of a few short rows, all of them at once, rather than rings, whose setup takes longer than their rows:
// backward up to this many rows (700 x 1500 7.5 us, with rings 8.9 and, off the 16-byte grid, 11.2; 148 x 2048 5.5 and
// 7.6; 2000 x 1024 11.6 and 9.5).
inline bool ln_few(int rows, int N, int sms) { return rows <= 8 * sms && N <= 2048; }

// Calls run(TPR, WIDE) for short rows.
template <typename T, typename Run>
void ln_short(const LnShape& sh, bool wide, Run run) {
  auto width = [&](auto w) {
    if (sh.N <= 64) run(std::integral_constant<int, 8>{}, w);
    else if (sh.N <= 128) run(std::integral_constant<int, 16>{}, w);
    else run(std::integral_constant<int, 32>{}, w);
  };
  if (wide) width(std::true_type{});
  else width(std::false_type{});
}

enum { LN_FORWARD, LN_BACKWARD, LN_FEW };
// Calls run(TPR, V, NT) (as integral constants) for rows of N elements: 16 elements a thread, 8 in short rows.  LN_FEW:
// in CTAs of 128 threads, which spread over the SMs (forward, 148 x 2048: 2.7 us, a CTA a row 3.6).  False: the row is
// too long.
template <typename T, int KIND, typename Run>
bool ln_groups(int N, Run run) {
  constexpr int PER = LN_PER<T>, V = 16 / PER;
#define LN_TRY(TPR, VV, NT)                                                                                        \
  if (N <= TPR * VV * PER) {                                                                                       \
    run(std::integral_constant<int, TPR>{}, std::integral_constant<int, VV>{}, std::integral_constant<int, NT>{}); \
    return true;                                                                                                   \
  }
  if constexpr (KIND == LN_FEW) {
    LN_TRY(32, V / 2, 128)
    LN_TRY(32, V, 128)
    LN_TRY(64, V, 128)
    LN_TRY(128, V, 128)
    return false;
  }
  // CTAs of 512 threads, one an SM: 148 rows of partial sums to add up, not 592 (those took 15 us)
  if constexpr (KIND == LN_BACKWARD) LN_TRY(32, V / 2, 512)
  LN_TRY(32, V, 512)
  LN_TRY(64, V, 512)
  LN_TRY(128, V, 512)
  LN_TRY(256, V, 512)
  LN_TRY(512, V, 512)
  LN_TRY(1024, V, 1024)
#undef LN_TRY
  return false;
}
// Two rows a round, or one where that leaves groups without rows, where the slots do not fit, and in CTAs of 1024
// threads.  M operands.  run(R, CTAs an SM, CTAs, slots); false: not even two rows fit.
constexpr int LN_SMEM = 200 << 10;  // of an SM, for the slots of its CTAs
template <int NT, int G, int M, typename Run>
bool ln_rounds(const ard_ctx* ctx, int rows, int row_bytes, Run run) {
  const int per_sm = NT >= 512 ? 1 : 512 / NT;
  const long long room = (long long)ctx->sm_count * per_sm;
  auto slots = [&](int R) {
    const int most = LN_SMEM / per_sm / (G * M * R * row_bytes);
    return most < LN_SLOTS ? most : LN_SLOTS;
  };
  auto blocks = [&](int R) {
    const long long want = (((long long)rows + R - 1) / R + G - 1) / G;
    return (int)(want < room ? want : room);
  };
  if constexpr (NT < 1024)
    if (slots(2) >= 2 && rows >= 2 * room * G) {
      run(std::integral_constant<int, 2>{}, blocks(2), slots(2));
      return true;
    }
  if (slots(1) < 2) return false;
  run(std::integral_constant<int, 1>{}, blocks(1), slots(1));
  return true;
}

template <typename T>
ard_status ln_fwd(ard_ctx* ctx, const LnShape& sh, float eps, const T* X, int ldx, const float* weight, const float* bias, T* Y, int ldy,
                  float* mean, float* rstd, cudaStream_t s) {
  cudaError_t err = cudaSuccess;
  bool done = false;
  const long long es = sizeof(T);
  auto run = [&](auto on16, auto small) {
    constexpr bool ON16 = decltype(on16)::value;
    const bool whole = ON16 && !sh.hdr && sh.N % LN_PER<T> == 0 && ln_on16(weight, 0) && ln_on16(bias, 0);
    LnRing ring;
    ring.row_bytes = (int)((sh.N * es + 15) / 16 * 16) + (ON16 ? 0 : 16);
    ln_groups<T, decltype(small)::value ? LN_FEW : LN_FORWARD>(sh.N, [&](auto tpr, auto v, auto nt) {
      constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value, NT = decltype(nt)::value, G = NT / TPR;
      if constexpr (ON16 || NT < 1024) {
        if (NT == 1024 && !whole) return;
        done = ln_rounds<NT, G, 1>(ctx, sh.rows, ring.row_bytes, [&](auto r, int blocks, int slots) {
          constexpr int R = decltype(r)::value;
          ring.slots = slots;
          auto kern = ln_fwd_kernel<T, TPR, V, NT, R, ON16>;
          err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, LN_SMEM);
          if (err == cudaSuccess)
            err = ard_launch(ctx, kern, dim3(blocks), dim3(NT), (size_t)G * slots * R * ring.row_bytes, s, sh, eps, X, ldx, weight, bias, Y, ldy,
                             mean, rstd, ring, ctx->d_status);
        });
      }
    });
  };
  const bool on16 = ln_on16(X, ldx * es) && ln_on16(Y, ldy * es), few = ln_few(sh.rows, sh.N, ctx->sm_count);
  if (few && on16 && sh.rows <= ctx->sm_count) run(std::true_type{}, std::true_type{});
  else if (!few && sh.N <= LN_SHORT_N)
    ln_short<T>(sh, on16, [&](auto tpr, auto wide) {
      constexpr int TPR = decltype(tpr)::value, G = LN_SHORT / TPR;
      const long long blocks = ((long long)sh.rows + G - 1) / G, room = 2 * ctx->sm_count;
      err = ard_launch(ctx, ln_fwd_short_kernel<T, TPR, decltype(wide)::value>, dim3((unsigned)(blocks < room ? blocks : room)), dim3(LN_SHORT), 0, s, sh,
                       eps, X, ldx, weight, bias, Y, ldy, mean, rstd);
      done = true;
    });
  else if (!few && on16) run(std::true_type{}, std::false_type{});
  else if (!few) run(std::false_type{}, std::false_type{});
  if (!done) {
    const int room = 8 * ctx->sm_count;
    auto kern = sh.N <= LN_INT_N ? ln_fwd_any_kernel<T, int> : ln_fwd_any_kernel<T, long long>;
    err = ard_launch(ctx, kern, dim3(sh.rows < room ? sh.rows : room), dim3(LN_ANY_THREADS), 0, s, sh, eps, X, ldx, weight, bias, Y, ldy, mean, rstd);
  }
  ARD_CUDA_OK(err);
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}

template <typename T>
ard_status ln_bwd(ard_ctx* ctx, const LnShape& sh, const T* dY, int lddy, const T* X, int ldx, const float* weight, const float* mean,
                  const float* rstd, T* dX, int lddx, float* dweight, float* dbias, int zero_fill, cudaStream_t s) {
  const bool sums = dweight || dbias;
  if (!dX && !sums) return ARD_OK;
  const long long fit = (long long)(sk_ws_bytes(ctx->sm_count) / sizeof(float) / 2) / (((long long)sh.N + 3) / 4 * 4);  // slices that the scratch holds
  if (sums && (!ctx->d_sk_ws || fit < 1)) return ARD_ERR_UNSUPPORTED;
  float* partial = sums ? (float*)ctx->d_sk_ws : nullptr;
  long long slices = 0;
  cudaError_t err = cudaSuccess;
  bool done = sh.rows == 0;
  const long long es = sizeof(T);
  auto run = [&](auto on16) {
    constexpr bool ON16 = decltype(on16)::value;
    const bool whole = ON16 && !sh.hdr && sh.N % LN_PER<T> == 0 && ln_on16(weight, 0);
    LnRing ring;
    ring.row_bytes = (int)((sh.N * es + 15) / 16 * 16) + (ON16 ? 0 : 16);
    ln_groups<T, LN_BACKWARD>(sh.N, [&](auto tpr, auto v, auto nt) {
      constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value, NT = decltype(nt)::value, G = NT / TPR;
      if constexpr (ON16 || (NT < 1024 && V * LN_PER<T> > 8)) {
        if (NT == 1024 && !whole) return;
        ln_rounds<NT, G, 2>(ctx, sh.rows, ring.row_bytes, [&](auto r, int blocks, int slots) {
          constexpr int R = decltype(r)::value;
          if (sums && blocks > fit) return;
          ring.slots = slots;
          size_t smem = (size_t)G * slots * 2 * R * ring.row_bytes;
          if constexpr (G > 1) {
            constexpr size_t exchange = 2 * sizeof(float) * V * TPR * LN_PER<T>;
            if (smem < exchange) smem = exchange;
          }
          auto kern = ln_bwd_kernel<T, TPR, V, NT, R, ON16>;
          err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, LN_SMEM);
          if (err == cudaSuccess)
            err = ard_launch(ctx, kern, dim3(blocks), dim3(NT), smem, s, sh, dY, lddy, X, ldx, weight, mean, rstd, dX, lddx, partial, ring,
                             ctx->d_status);
          slices = blocks;
          ctx->launches++;
          done = true;
        });
      }
    });
  };
  if (!done && !ln_few(sh.rows, sh.N, ctx->sm_count)) {
    const bool on16 = ln_on16(X, ldx * es) && ln_on16(dY, lddy * es) && ln_on16(dX, dX ? lddx * es : 0);
    // (rows of 129 to 256 on the grid through rings: 131072 x 256 56 us, by lanes 73)
    if (sh.N <= (on16 ? 128 : LN_SHORT_N)) {
      ln_short<T>(sh, on16, [&](auto tpr, auto wide) {
        constexpr int TPR = decltype(tpr)::value, G = LN_SHORT / TPR;
        constexpr bool WIDE = decltype(wide)::value;
        if constexpr (!WIDE || TPR < 32) {
          const long long most = ((long long)sh.rows + G - 1) / G, room = 2 * ctx->sm_count;
          const int blocks = (int)(most < room ? most : room);
          if (sums && blocks > fit) return;
          err = ard_launch(ctx, ln_bwd_short_kernel<T, TPR, WIDE>, dim3(blocks), dim3(LN_SHORT), 0, s, sh, dY, lddy, X, ldx, weight, mean, rstd, dX, lddx,
                           partial);
          slices = blocks;
          ctx->launches++;
          done = true;
        }
      });
    } else if (on16) {
      run(std::true_type{});
    } else {
      run(std::false_type{});
    }
    ARD_CUDA_OK(err);
  }
  if (!done) {
    const int room = 8 * ctx->sm_count, dx_blocks = !dX ? 0 : sh.rows < room ? sh.rows : room;
    int gx = 1, per = 0;
    if (sums) {
      gx = (sh.N + 31) / 32;
      if (gx > 4096) gx = 4096;
      slices = (sh.rows + 63) / 64;
      if (slices > fit) slices = fit;
      if (slices > 1024) slices = 1024;
      per = (int)((sh.rows + slices - 1) / slices);
      slices = (sh.rows + per - 1) / per;
    }
    auto kern = sh.N <= LN_INT_N ? ln_bwd_any_kernel<T, int> : ln_bwd_any_kernel<T, long long>;
    ARD_CUDA_OK(ard_launch(ctx, kern, dim3((unsigned)(dx_blocks + slices * gx)), dim3(LN_ANY_THREADS), 0, s, sh, dY, lddy, X, ldx, weight, mean, rstd,
                           dX, lddx, dx_blocks, partial, per, gx));
    ctx->launches++;
  }
  if (sums) {
    ARD_CUDA_OK(ard_launch(ctx, ln_dw_sum_kernel, dim3((sh.N + 31) / 32, 2), dim3(LN_SUM_WARPS * 32), 0, s, sh, (const float*)partial,
                           (int)slices, dweight, dbias, zero_fill));
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
