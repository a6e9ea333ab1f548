// Layer norm over the rows of a matrix, and its adjoint with the reduction of the weight's and the bias's gradient; over all columns or
// over the compact columns that a row pattern keeps.
//
// One pass over memory bounds both: the forward call reads x and writes y, the backward call reads x and dy and writes dx.
#include "ard_internal.h"
#include "sm100_ptx.h"

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

// The slices' sums added in a fixed order, into the units' places: a warp's lanes take 32 columns, its CTA's warps the slices.
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
#pragma unroll 8
    for (int k = warp; k < slices; k += LN_SUM_WARPS) t += partial[((size_t)k * 2 + which) * sh.N + j];
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

// ---- rows on a 16-byte grid -------------------------------------------------------------------------
// TPR threads hold a row, V pieces of 16 bytes each: piece v of thread t is number v * TPR + t.
template <typename T>
constexpr int LN_PER = 16 / (int)sizeof(T);  // elements of a piece

template <typename T>
__device__ __forceinline__ void ln_unpack(const uint4& q, float (&v)[LN_PER<T>]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(w[k] << 16);
      v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(w[k]);
  }
}
// The first `valid` values of a piece.
template <typename T>
__device__ __forceinline__ void ln_store(T* p, int valid, const float (&v)[LN_PER<T>]) {
  if (valid >= LN_PER<T>) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 2) {
        __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
        w[k] = *reinterpret_cast<uint32_t*>(&b);
      } else {
        w[k] = __float_as_uint(v[k]);
      }
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    return;
  }
#pragma unroll
  for (int k = 0; k < LN_PER<T>; ++k)
    if (k < valid) ln_put(p, k, v[k]);
}
// weight or bias at the units of a piece's columns; `other` where there is none.
template <int PER>
__device__ __forceinline__ void ln_params(const float* w, float other, const LnCols& c, int j, float (&v)[PER]) {
#pragma unroll
  for (int k = 0; k < PER; ++k) v[k] = w && j + k < c.n ? w[c.b0 + (size_t)(j + k) * c.dp] : other;
}
// The same of whole pieces on 16 bytes, all columns kept; not to be kept in registers (CTAs of 1024 threads, 64 registers each): they come from
// the L1 cache for every row.
template <int PER>
__device__ __forceinline__ void ln_params_now(const float* w, float other, int j, float (&v)[PER]) {
#pragma unroll
  for (int k = 0; k < PER; k += 4) {
    float4 q = make_float4(other, other, other, other);
    if (w) asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w) : "l"(w + j + k));
    v[k] = q.x; v[k + 1] = q.y; v[k + 2] = q.z; v[k + 3] = q.w;
  }
}

// The sums of M values over the TPR threads of a row; with more than a warp through shared memory, of which a call and the next use
// different halves (one barrier of the CTA per call, the same number of calls in all its threads).
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
    __syncthreads();
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

// Rows reach the TPR threads that hold them through a ring of slots in shared memory, filled by bulk copies that the first of them asks for
// several rows ahead: what is in flight costs no registers, and 100 to 200 KB an SM are in flight whatever the row's length.
constexpr int LN_SLOTS = 8;
struct LnRing {
  int slots;       // per row of threads
  int slot_bytes;  // M operands of a row, each rounded up to 16 bytes
};
template <typename T, int TPR, int G, int M>
struct LnRows {
  const T* src[M];
  int ld[M];
  uint8_t* mine;
  uint64_t* full;
  LnRing ring;
  int r0, stride, rounds, rows;
  uint32_t bytes;
  bool gone;  // a copy did not come within two seconds: the rest is left, the status says so
  int gone_at;

  __device__ __forceinline__ LnRows(const LnShape& sh, const LnCols& c, LnRing rg, uint8_t* slots, uint64_t (*bars)[LN_SLOTS]) {
    const int g = threadIdx.x / TPR;
    ring = rg;
    mine = slots + (size_t)g * ring.slots * ring.slot_bytes;
    full = bars[g];
    bytes = ((uint32_t)c.n * (uint32_t)sizeof(T) + 15u) & ~15u;
    rows = sh.rows;
    stride = gridDim.x * G;
    rounds = (rows + stride - 1) / stride;
    r0 = blockIdx.x * G + g;
    gone = false;
    gone_at = 0;
  }
  __device__ __forceinline__ long long row(int it) const { return r0 + (long long)it * stride; }
  __device__ __forceinline__ const uint8_t* slot(int it, int m) const {
    return mine + (size_t)(it % ring.slots) * ring.slot_bytes + m * (ring.slot_bytes / M);
  }
  // By the first thread of the row, for round `it`; whoever read the slot before has passed a barrier since.
  __device__ __forceinline__ void ask(int it) const {
    if (it >= rounds || row(it) >= rows) return;
    const uint32_t bar = smem_u32(&full[it % ring.slots]);
    mbar_arrive_expect_tx(bar, M * bytes);
#pragma unroll
    for (int m = 0; m < M; ++m)
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(slot(it, m))),
                   "l"(src[m] + (size_t)row(it) * ld[m]), "r"(bytes), "r"(bar)
                   : "memory");
  }
  __device__ __forceinline__ bool wait(int it, volatile int* s_gone, int* status) {
    if (!gone && !mbar_wait(smem_u32(&full[it % ring.slots]), (uint32_t)(it / ring.slots) & 1u, s_gone, status)) {
      gone = true;
      gone_at = it;
    }
    return !gone;
  }
  // Before the CTA ends without some of its copies (asked up to round `asked`): they get the same time, for they write to its memory.
  __device__ __forceinline__ void drain(int asked) const {
    for (int it = gone_at; it <= asked && it < rounds && row(it) < rows; ++it) {
      bool ok = false;
      for (int poll = 0; poll < 2000 && !ok; ++poll) ok = mbar_try_wait_hint(smem_u32(&full[it % ring.slots]), (uint32_t)(it / ring.slots) & 1u, 1000000u);
    }
  }
};

// Forward: two sums over a row's registers, the second about the mean (a sum of squares alone loses the variance of a row with a large
// mean).  The barrier of the first one says that the row's slot has been read.
template <typename T, int TPR, int V, int NT>
__global__ void __launch_bounds__(NT, 1) ln_fwd_kernel(LnShape sh, float eps, const T* X, int ldx, const float* weight, const float* bias,
                                                    T* Y, int ldy, float* mean, float* rstd, LnRing ring, int* status) {
  constexpr int PER = LN_PER<T>, G = NT / TPR;
  constexpr bool KEEP = NT < 1024;
  extern __shared__ __align__(128) uint8_t slots[];  // [G][slots][slot_bytes]
  __shared__ float red[2][1][32];
  __shared__ __align__(8) uint64_t full[G][LN_SLOTS];
  __shared__ int s_gone;
  const int t = threadIdx.x % TPR;
  if (t == 0)
    for (int k = 0; k < ring.slots; ++k) mbar_init(smem_u32(&full[threadIdx.x / TPR][k]), 1);
  if (threadIdx.x == 0) s_gone = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncthreads();
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const LnCols c = ln_cols(sh);
  const float inv_n = 1.f / (float)c.n;
  LnRows<T, TPR, G, 1> in(sh, c, ring, slots, full);
  in.src[0] = X;
  in.ld[0] = ldx;
  if (t == 0)
    for (int k = 0; k < ring.slots; ++k) in.ask(k);
  float w[KEEP ? V : 1][PER], b[KEEP ? V : 1][PER];
  if constexpr (KEEP)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      ln_params<PER>(weight, 1.f, c, (v * TPR + t) * PER, w[v]);
      ln_params<PER>(bias, 0.f, c, (v * TPR + t) * PER, b[v]);
    }
  int half = 0;
  for (int it = 0; it < in.rounds; ++it) {
    const long long r = in.row(it);
    const bool live = r < sh.rows && in.wait(it, &s_gone, status);
    float x[V][PER];
    float s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int j = (v * TPR + t) * PER;
      uint4 q = make_uint4(0u, 0u, 0u, 0u);
      if (live && j < c.n) q = *reinterpret_cast<const uint4*>(in.slot(it, 0) + (size_t)j * sizeof(T));
      ln_unpack<T>(q, x[v]);
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        if (j + k >= c.n) x[v][k] = 0.f;
        s[0] += x[v][k];
      }
    }
    ln_row_sums<TPR, 1>(s, red, half);
    if (TPR == 32) __syncwarp();
    if (t == 0 && !in.gone) in.ask(it + ring.slots);
    const float mu = s[0] * inv_n;
    s[0] = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        x[v][k] -= mu;
        if ((v * TPR + t) * PER + k < c.n) s[0] = fmaf(x[v][k], x[v][k], s[0]);
      }
    ln_row_sums<TPR, 1>(s, red, half);
    const float rs = 1.f / sqrtf(fmaf(s[0], inv_n, eps));
    if (!live) continue;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int j = (v * TPR + t) * PER;
      if (j < c.n) {
        constexpr int one = KEEP ? 1 : 0;
        if constexpr (!KEEP) {
          ln_params_now<PER>(weight, 1.f, j, w[0]);
          ln_params_now<PER>(bias, 0.f, j, b[0]);
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) x[v][k] = fmaf(x[v][k] * rs, w[one * v][k], b[one * v][k]);
        ln_store<T>(Y + (size_t)r * ldy + j, c.n - j, x[v]);
      }
    }
    if (t == 0) {
      if (mean) mean[r] = mu;
      if (rstd) rstd[r] = rs;
    }
  }
  if (in.gone && t == 0) in.drain(in.gone_at + ring.slots - 1);
}

// Backward: a thread keeps its columns' sums for the weight and the bias over all rows of the CTA and leaves them in `partial`
// [CTA][2][N].  A row is read from its slot twice, for its sums and for dx, which costs less than the registers that would hold it; its slot is
// asked for again one row later: the barrier of that row's sums says that nobody reads it any more.
template <typename T, int TPR, int V, int NT>
__global__ void __launch_bounds__(NT, 1) ln_bwd_kernel(LnShape sh, const T* dY, int lddy, const T* X, int ldx, const float* weight,
                                                    const float* mean, const float* rstd, T* dX, int lddx, float* partial,
                                                    LnRing ring, int* status) {
  constexpr int PER = LN_PER<T>, G = NT / TPR;
  constexpr bool KEEP = NT < 1024;
  extern __shared__ __align__(128) uint8_t slots[];  // [G][slots][slot_bytes]; at the end the sums of the G rows of threads
  __shared__ float red[2][2][32];
  __shared__ __align__(8) uint64_t full[G][LN_SLOTS];
  __shared__ int s_gone;
  const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
  if (t == 0)
    for (int k = 0; k < ring.slots; ++k) mbar_init(smem_u32(&full[g][k]), 1);
  if (threadIdx.x == 0) s_gone = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncthreads();
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const LnCols c = ln_cols(sh);
  const float inv_n = 1.f / (float)c.n;
  LnRows<T, TPR, G, 2> in(sh, c, ring, slots, full);
  in.src[0] = X;
  in.ld[0] = ldx;
  in.src[1] = dY;
  in.ld[1] = lddy;
  if (t == 0)
    for (int k = 0; k < ring.slots; ++k) in.ask(k);
  constexpr int one = KEEP ? 1 : 0;
  float dw[V][PER], db[V][PER], w[KEEP ? V : 1][PER];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if constexpr (KEEP) ln_params<PER>(weight, 1.f, c, (v * TPR + t) * PER, w[v]);
#pragma unroll
    for (int k = 0; k < PER; ++k) dw[v][k] = db[v][k] = 0.f;
  }
  int half = 0;
  float mu = 0.f, rs = 0.f;
  if (in.r0 < sh.rows) {
    mu = mean[in.r0];
    rs = rstd[in.r0];
  }
  for (int it = 0; it < in.rounds; ++it) {
    const long long row = in.row(it);
    const bool live = row < sh.rows && in.wait(it, &s_gone, status);
    float mu2 = 0.f, rs2 = 0.f;  // of the next row, fetched behind this one's arithmetic
    if (row + in.stride < sh.rows) {
      mu2 = mean[row + in.stride];
      rs2 = rstd[row + in.stride];
    }
    float s[2] = {0.f, 0.f};
    if (live) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int j = (v * TPR + t) * PER;
        if (j < c.n) {
          float x[PER], dy[PER];
          ln_unpack<T>(*reinterpret_cast<const uint4*>(in.slot(it, 0) + (size_t)j * sizeof(T)), x);
          ln_unpack<T>(*reinterpret_cast<const uint4*>(in.slot(it, 1) + (size_t)j * sizeof(T)), dy);
          if constexpr (!KEEP) ln_params_now<PER>(weight, 1.f, j, w[0]);
#pragma unroll
          for (int k = 0; k < PER; ++k) {
            const bool real = j + k < c.n;
            const float xh = real ? (x[k] - mu) * rs : 0.f, d = real ? dy[k] : 0.f, e = d * w[one * v][k];
            s[0] += e;
            s[1] = fmaf(e, xh, s[1]);
            dw[v][k] = fmaf(d, xh, dw[v][k]);
            db[v][k] += d;
          }
        }
      }
    }
    ln_row_sums<TPR, 2>(s, red, half);
    if (TPR == 32) __syncwarp();
    if (t == 0 && it > 0 && !in.gone) in.ask(it - 1 + ring.slots);
    if (live && dX) {
      const float s1 = s[0] * inv_n, s2 = s[1] * inv_n;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int j = (v * TPR + t) * PER;
        if (j < c.n) {
          float x[PER], dy[PER];
          ln_unpack<T>(*reinterpret_cast<const uint4*>(in.slot(it, 0) + (size_t)j * sizeof(T)), x);
          ln_unpack<T>(*reinterpret_cast<const uint4*>(in.slot(it, 1) + (size_t)j * sizeof(T)), dy);
          if constexpr (!KEEP) ln_params_now<PER>(weight, 1.f, j, w[0]);
#pragma unroll
          for (int k = 0; k < PER; ++k) x[k] = rs * (dy[k] * w[one * v][k] - s1 - (x[k] - mu) * rs * s2);
          ln_store<T>(dX + (size_t)row * lddx + j, c.n - j, x);
        }
      }
    }
    mu = mu2;
    rs = rs2;
  }
  if (in.gone && t == 0) in.drain(in.gone_at + ring.slots - 1);
  if (!partial) return;
  // the rows of threads added in their order
  if constexpr (G > 1) {
    float* sums = reinterpret_cast<float*>(slots);  // [2][V * TPR * PER]
    for (int k = 0; k < G; ++k) {
      __syncthreads();
      if (g == k)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int q = 0; q < PER; ++q) {
            const int j = (v * TPR + t) * PER + q;
            if (k > 0) {
              dw[v][q] += sums[j];
              db[v][q] += sums[V * TPR * PER + j];
            }
            sums[j] = dw[v][q];
            sums[V * TPR * PER + j] = db[v][q];
          }
    }
    if (g != G - 1) return;
  }
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const int j = (v * TPR + t) * PER + q;
      if (j < c.n) {
        partial[((size_t)blockIdx.x * 2 + 0) * sh.N + j] = dw[v][q];
        partial[((size_t)blockIdx.x * 2 + 1) * sh.N + j] = db[v][q];
      }
    }
}

inline bool ln_on16(const void* p, long long ld_bytes) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld_bytes % 16 == 0; }

// Calls run(TPR, V, NT) (as integral constants) for rows of N elements: 16 elements a thread, 8 in short rows.  False: the row is too long.
template <typename T, typename Run>
bool ln_rows_of_threads(int N, Run run) {
  constexpr int PER = LN_PER<T>, V = 16 / PER;
#define LN_TRY(TPR, VV, NT)                                                                                        \
  if (N <= TPR * VV * PER) {                                                                                       \
    run(std::integral_constant<int, TPR>{}, std::integral_constant<int, VV>{}, std::integral_constant<int, NT>{}); \
    return true;                                                                                                   \
  }
  LN_TRY(32, V / 2, 128)
  LN_TRY(32, V, 128)
  LN_TRY(64, V, 128)
  LN_TRY(128, V, 128)
  LN_TRY(256, V, 256)
  LN_TRY(512, V, 512)
  LN_TRY(1024, V, 1024)
#undef LN_TRY
  return false;
}
constexpr int LN_SMEM = 200 << 10;  // of an SM, for the slots of its CTAs
// Slots of a row of threads where per_sm CTAs of G such rows share an SM; below two: none.
inline int ln_slots(int per_sm, int G, int slot_bytes) {
  const int most = LN_SMEM / per_sm / (G * slot_bytes);
  return most < LN_SLOTS ? most : LN_SLOTS;
}

template <typename T>
ard_status ln_fwd(ard_ctx* ctx, const LnShape& sh, float eps, const T* X, int ldx, const float* weight, const float* bias, T* Y, int ldy,
                  float* mean, float* rstd, cudaStream_t s) {
  cudaError_t err = cudaSuccess;
  bool done = false;
  const long long es = sizeof(T);
  if (ln_on16(X, ldx * es) && ln_on16(Y, ldy * es)) {
    const bool whole = !sh.hdr && sh.N % LN_PER<T> == 0 && ln_on16(weight, 0) && ln_on16(bias, 0);
    LnRing ring;
    ring.slot_bytes = (int)((sh.N * es + 15) / 16 * 16);
    ln_rows_of_threads<T>(sh.N, [&](auto tpr, auto v, auto nt) {
      constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value, NT = decltype(nt)::value, G = NT / TPR;
      const int per_sm = NT >= 512 ? 1 : 512 / NT;
      ring.slots = ln_slots(per_sm, G, ring.slot_bytes);
      if (ring.slots < 2 || (NT == 1024 && !whole)) return;
      const int want = (sh.rows + G - 1) / G, room = ctx->sm_count * per_sm;
      auto kern = ln_fwd_kernel<T, TPR, V, NT>;
      err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, LN_SMEM);
      if (err == cudaSuccess)
        err = ard_launch(ctx, kern, dim3(want < room ? want : room), dim3(NT), (size_t)G * ring.slots * ring.slot_bytes, s, sh, eps, X, ldx,
                         weight, bias, Y, ldy, mean, rstd, ring, ctx->d_status);
      done = true;
    });
  }
  if (!done) {
    const int room = 8 * ctx->sm_count;
    err = ard_launch(ctx, ln_fwd_any_kernel<T>, dim3(sh.rows < room ? sh.rows : room), dim3(LN_ANY_THREADS), 0, s, sh, eps, X, ldx, weight,
                     bias, Y, ldy, mean, rstd);
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
  const long long fit = (long long)(sk_ws_bytes(ctx->sm_count) / sizeof(float) / 2) / sh.N;  // slices that the scratch holds
  if (sums && (!ctx->d_sk_ws || fit < 1)) return ARD_ERR_UNSUPPORTED;
  float* partial = sums ? (float*)ctx->d_sk_ws : nullptr;
  long long slices = 0;
  cudaError_t err = cudaSuccess;
  bool done = sh.rows == 0;
  const long long es = sizeof(T);
  if (!done && ln_on16(X, ldx * es) && ln_on16(dY, lddy * es) && ln_on16(dX, dX ? lddx * es : 0)) {
    const bool whole = !sh.hdr && sh.N % LN_PER<T> == 0 && ln_on16(weight, 0);
    LnRing ring;
    ring.slot_bytes = 2 * (int)((sh.N * es + 15) / 16 * 16);
    ln_rows_of_threads<T>(sh.N, [&](auto tpr, auto v, auto nt) {
      constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value, NT = decltype(nt)::value, G = NT / TPR;
      const int per_sm = NT >= 512 ? 1 : 512 / NT;
      ring.slots = ln_slots(per_sm, G, ring.slot_bytes);
      if (ring.slots < 2 || (NT == 1024 && !whole)) return;
      long long blocks = ((long long)sh.rows + G - 1) / G;
      if (blocks > (long long)ctx->sm_count * per_sm) blocks = (long long)ctx->sm_count * per_sm;
      if (sums && blocks > fit) return;
      size_t smem = (size_t)G * ring.slots * ring.slot_bytes;
      const size_t exchange = G > 1 ? 2 * sizeof(float) * V * TPR * LN_PER<T> : 0;
      if (smem < exchange) smem = exchange;
      auto kern = ln_bwd_kernel<T, TPR, V, NT>;
      err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, LN_SMEM);
      if (err == cudaSuccess)
        err = ard_launch(ctx, kern, dim3((unsigned)blocks), dim3(NT), smem, s, sh, dY, lddy, X, ldx, weight, mean, rstd, dX, lddx, partial,
                         ring, ctx->d_status);
      slices = blocks;
      ctx->launches++;
      done = true;
    });
    ARD_CUDA_OK(err);
  }
  if (!done) {
    if (dX) {
      const int room = 8 * ctx->sm_count;
      ARD_CUDA_OK(ard_launch(ctx, ln_dx_any_kernel<T>, dim3(sh.rows < room ? sh.rows : room), dim3(LN_ANY_THREADS), 0, s, sh, dY, lddy, X,
                             ldx, weight, mean, rstd, dX, lddx));
      ctx->launches++;
    }
    if (sums) {
      const int gx = (sh.N + 31) / 32;
      slices = (sh.rows + 63) / 64;
      if (slices > fit) slices = fit;
      if (slices > 1024) slices = 1024;
      const int per = (int)((sh.rows + slices - 1) / slices);
      slices = (sh.rows + per - 1) / per;
      ARD_CUDA_OK(ard_launch(ctx, ln_dw_any_kernel<T>, dim3(gx < 4096 ? gx : 4096, (unsigned)slices), dim3(LN_ANY_THREADS), 0, s, sh, dY,
                             lddy, X, ldx, mean, rstd, partial, per));
      ctx->launches++;
    }
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
