// Rows of a table by token, scaled, and the table's gradient:
//   Y[r][j] = alpha * table[ids[r]][col(j)],   dtable[v][col(j)] (+)= alpha * sum over r with ids[r] = v of dY[r][j],
// col(j) = j, or the j-th kept unit of a row pattern.
//
// Memory bounds both.  The gradient needs each token's rows side by side; sorting all of them through global memory would take
// several launches that hand one another the order.  Instead a CTA owns the tokens v = group (mod groups) and some columns: it
// looks through all ids (they come from the L2: 4 bytes a position where a row of dY has thousands), keeps those that are
// its own in shared memory, sorts them by token and position there, and adds their rows up in that order.  One launch, no scratch,
// and the same bits every time: each sum is cut at the same places.  Equal shares of the sorted list go to the warps, so a token that
// comes up in every other position costs no more than any other; tokens are dealt out in turn, so frequent ones, which
// lie side by side in a dictionary sorted by frequency, fall to different CTAs.
#include "ard_internal.h"
#include "sm100_ptx.h"

namespace {

constexpr int EM_THREADS = 256;

template <typename T>
__device__ __forceinline__ float em_f32(T x) {
  if constexpr (sizeof(T) == 2) return __bfloat162float(x);
  else return x;
}
template <typename T>
__device__ __forceinline__ T em_from(float x) {
  if constexpr (sizeof(T) == 2) return __float2bfloat16_rn(x);
  else return x;
}

template <int BYTES> struct EmRaw;
template <> struct EmRaw<16> { using type = uint4; };
template <> struct EmRaw<8> { using type = uint2; };
template <> struct EmRaw<4> { using type = uint32_t; };
template <> struct EmRaw<2> { using type = uint16_t; };

// BYTES a thread and access; `lanes` (a power of two, at most EM_THREADS) threads to a row, UNROLL accesses in flight.
template <typename T, int BYTES, int UNROLL>
__global__ void __launch_bounds__(EM_THREADS) embedding_fwd_kernel(const int32_t* hdr, int rows, int V, int N, float alpha, const int32_t* ids,
                                                                   const T* table, int ldt, T* Y, int ldy, int lanes, int* status) {
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  constexpr int VEC = BYTES / (int)sizeof(T);
  using Raw = typename EmRaw<BYTES>::type;
  const int lane = threadIdx.x & (lanes - 1);
  const long long r = (long long)blockIdx.x * (EM_THREADS / lanes) + threadIdx.x / lanes;
  if (r >= rows) return;
  const int id = ids[r];
  const bool there = id >= 0 && id < V;
  if (id >= V && lane == 0) atomicMax(status, (int)ARD_ERR_INVALID_ARG);
  int dp = 1, first = 0, n = N;
  if (hdr) dp = hdr[HDR_DP], first = hdr[HDR_B] - 1, n = hdr[HDR_NKEEP];
  const T* src = table + (size_t)(there ? id : 0) * ldt;
  T* dst = Y + (size_t)r * ldy;
  if (dp == 1) {
    const int vecs = n / VEC;  // the host has seen to it that nothing is left over
    for (int v0 = lane; v0 < vecs; v0 += lanes * UNROLL) {
      Raw q[UNROLL];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int v = v0 + u * lanes;
        if (v < vecs && there) q[u] = *reinterpret_cast<const Raw*>(src + (size_t)v * VEC);
      }
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int v = v0 + u * lanes;
        if (v >= vecs) break;
        T e[VEC];
        memcpy(e, &q[u], BYTES);
#pragma unroll
        for (int k = 0; k < VEC; ++k) e[k] = there ? em_from<T>(alpha * em_f32(e[k])) : em_from<T>(0.f);
        Raw o;
        memcpy(&o, e, BYTES);
        *reinterpret_cast<Raw*>(dst + (size_t)v * VEC) = o;
      }
    }
    return;
  }
  for (int j0 = lane; j0 < n; j0 += lanes * 4) {
    float x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int j = j0 + u * lanes;
      x[u] = j < n && there ? em_f32(src[first + (size_t)j * dp]) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int j = j0 + u * lanes;
      if (j < n) dst[j] = em_from<T>(there ? alpha * x[u] : 0.f);
    }
  }
}

// ---- gradient ---------------------------------------------------------------------------------------
constexpr int EB_THREADS = 1024, EB_WARPS = EB_THREADS / 32;
constexpr int EB_COLS = 128;            // columns of a CTA: 4 a lane
constexpr int EB_PLACE_BITS = 14;       // places of the list, which ends the key that is sorted
constexpr int EB_LIST = 1 << EB_PLACE_BITS;
constexpr int EB_STEP = 8 * EB_THREADS;  // ids looked at at a time
constexpr int EB_TOKENS = 1 << (32 - EB_PLACE_BITS);  // most tokens of a CTA (the last one's key would be the filler's: never used)
constexpr int EB_AHEAD = 8;             // rows of dY in flight a warp

struct EbShared {
  uint32_t key[EB_LIST];                       // token / groups, then the place in the list: by position
  int32_t row[EB_LIST];
  uint32_t seen[EB_TOKENS / 32];               // tokens whose row of the gradient has been written
  float part[2][EB_WARPS][EB_COLS];            // sums of tokens that several warps share: a share's first and its last
  int count[EB_WARPS];
};
static_assert(sizeof(EbShared) <= 227 * 1024, "shared memory of an SM");

template <typename T, bool VEC>
struct EbCols {  // a lane's columns: 4 * lane + k, or lane + 32 * k where those do not lie on a grid of four
  __device__ __forceinline__ static int col(int lane, int k) { return VEC ? 4 * lane + k : lane + 32 * k; }
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(EB_THREADS, 1) embedding_bwd_kernel(const int32_t* hdr, int rows, int V, int N, float alpha, const int32_t* ids,
                                                                      const T* dY, int lddy, float* dtable, int lddt, int accumulate,
                                                                      int wide, int* status) {
  extern __shared__ __align__(16) uint8_t eb_smem[];
  EbShared& sh = *reinterpret_cast<EbShared*>(eb_smem);
  pdl_launch_dependents();
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  pdl_wait_prior_grids();
  int dp = 1, first = 0, n = N;
  if (hdr) dp = hdr[HDR_DP], first = hdr[HDR_B] - 1, n = hdr[HDR_NKEEP];
  const int chunks = max(1, (n + EB_COLS - 1) / EB_COLS), groups = min((int)gridDim.x / chunks, V);
  if ((int)blockIdx.x >= groups * chunks) return;
  const int group = blockIdx.x % groups, c0 = (blockIdx.x / groups) * EB_COLS;
  const int tokens = (V - group - 1) / groups + 1;
  for (int i = t; i < (tokens + 31) / 32; i += EB_THREADS) sh.seen[i] = 0u;
  using Raw = typename EmRaw<4 * sizeof(T)>::type;
  const bool full = VEC && c0 + EB_COLS <= n;
  const bool tail = n - c0 <= EB_COLS;  // the columns behind the last kept unit's period are its own too

  // One token's sum to the gradient.
  auto flush = [&](int token, const float (&sum)[4]) {
    float* out = dtable + (size_t)(group + (long long)token * groups) * lddt;
    const bool old = (sh.seen[token >> 5] >> (token & 31)) & 1u;
    if (accumulate || old) {
      // one addition an element and pass over the list, so that its order is that of the passes; nothing waits for the old value
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int j = c0 + EbCols<T, VEC>::col(lane, k);
        if (j < n) atomicAdd(out + first + (size_t)j * dp, alpha * sum[k]);
      }
    } else if (dp == 1) {
      if (VEC && wide && c0 + 4 * lane + 3 < n) {
        *reinterpret_cast<float4*>(out + c0 + 4 * lane) = make_float4(alpha * sum[0], alpha * sum[1], alpha * sum[2], alpha * sum[3]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int j = c0 + EbCols<T, VEC>::col(lane, k);
          if (j < n) out[j] = alpha * sum[k];
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int j = c0 + EbCols<T, VEC>::col(lane, k);
        if (j >= n) continue;
        for (int d = 0; d < dp && (long long)j * dp + d < N; ++d) out[(size_t)j * dp + d] = d == first ? alpha * sum[k] : 0.f;
      }
    }
    __syncwarp();
    if (lane == 0 && !old) atomicOr(&sh.seen[token >> 5], 1u << (token & 31));
  };

  // Sorts the list and adds its rows up.
  auto work_off = [&](int m) {
    int size = 32;
    while (size < m) size *= 2;
    for (int i = m + t; i < size; i += EB_THREADS) sh.key[i] = 0xFFFFFFFFu;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
      for (int j = k / 2; j > 0; j /= 2) {
        for (int i = t; i < size / 2; i += EB_THREADS) {
          const int a = ((i & ~(j - 1)) << 1) | (i & (j - 1)), b = a | j;
          const uint32_t x = sh.key[a], y = sh.key[b];
          if ((x > y) == ((a & k) == 0)) sh.key[a] = y, sh.key[b] = x;
        }
        __syncthreads();
      }
    // a warp's share of the list; a token that a share begins or ends with may go on in the next one
    const int share = (m + EB_WARPS - 1) / EB_WARPS, from = min(m, warp * share), to = min(m, from + share);
    auto token_at = [&](int i) { return (int)(sh.key[i] >> EB_PLACE_BITS); };
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    bool open_front = false, open_back = false;
    if (from < to) {
      int cur = token_at(from);
      open_front = from > 0 && token_at(from - 1) == cur;
      open_back = to < m && token_at(to) == token_at(to - 1);
      bool front = open_front;
      for (int i0 = from; i0 < to; i0 += EB_AHEAD) {
        float x[EB_AHEAD][4];
        if (full) {  // all loads before the first use
          Raw q[EB_AHEAD];
#pragma unroll
          for (int u = 0; u < EB_AHEAD; ++u)
            q[u] = *reinterpret_cast<const Raw*>(dY + (size_t)sh.row[sh.key[min(i0 + u, to - 1)] & (EB_LIST - 1)] * lddy + c0 + 4 * lane);
#pragma unroll
          for (int u = 0; u < EB_AHEAD; ++u) {
            T e[4];
            memcpy(e, &q[u], sizeof(Raw));
#pragma unroll
            for (int k = 0; k < 4; ++k) x[u][k] = em_f32(e[k]);
          }
        } else {
          T e[EB_AHEAD][4];
#pragma unroll
          for (int u = 0; u < EB_AHEAD; ++u) {
            const T* src = dY + (size_t)sh.row[sh.key[min(i0 + u, to - 1)] & (EB_LIST - 1)] * lddy + c0;
#pragma unroll
            for (int k = 0; k < 4; ++k) e[u][k] = src[min(EbCols<T, VEC>::col(lane, k), n - 1 - c0)];  // (beyond them: nobody asks)
          }
#pragma unroll
          for (int u = 0; u < EB_AHEAD; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) x[u][k] = em_f32(e[u][k]);
        }
#pragma unroll
        for (int u = 0; u < EB_AHEAD; ++u) {
          if (i0 + u >= to) break;
          const int now = token_at(i0 + u);
          if (now != cur) {
            if (front) {
#pragma unroll
              for (int k = 0; k < 4; ++k) sh.part[0][warp][EbCols<T, VEC>::col(lane, k)] = sum[k];
              front = false;
            } else {
              flush(cur, sum);
            }
            cur = now;
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] = 0.f;
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) sum[k] += x[u][k];
        }
      }
      if (front || open_back) {  // a share of one token that is open on both sides counts as its first
#pragma unroll
        for (int k = 0; k < 4; ++k) sh.part[front ? 0 : 1][warp][EbCols<T, VEC>::col(lane, k)] = sum[k];
      } else {
        flush(cur, sum);
      }
      if (front) open_back = false;  // (its sum goes on from an earlier warp)
    }
    __syncthreads();
    // the warp with whose share a divided token begins adds up its pieces, in the list's order
    if (open_back) {
      const int token = token_at(to - 1);
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[k] = sh.part[1][warp][EbCols<T, VEC>::col(lane, k)];
      for (int w = warp + 1; w < EB_WARPS; ++w) {
        const int at = w * share;
        if (at >= m || token_at(at) != token) break;
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] += sh.part[0][w][EbCols<T, VEC>::col(lane, k)];
      }
      flush(token, sum);
    }
    __syncthreads();
  };

  int m = 0;
  for (long long p0 = 0; p0 < rows; p0 += EB_STEP) {
    if (m + EB_STEP > EB_LIST) {  // the next step might not fit
      work_off(m);
      m = 0;
    }
    // eight positions side by side a thread, so that the list is in their order
    const long long p = p0 + 8 * t;
    int id[8];
    unsigned mine = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      id[k] = p + k < rows ? ids[p + k] : -1;
      if (id[k] >= V && blockIdx.x == 0) atomicMax(status, (int)ARD_ERR_INVALID_ARG);
      if (id[k] >= 0 && id[k] < V && (unsigned)id[k] % (unsigned)groups == (unsigned)group) mine |= 1u << k;
    }
    int inc = __popc(mine);
    const int own = inc;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int x = __shfl_up_sync(0xFFFFFFFFu, inc, o);
      if (lane >= o) inc += x;
    }
    if (lane == 31) sh.count[warp] = inc;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < EB_WARPS; ++w) {
      const int c = sh.count[w];
      if (w < warp) before += c;
      all += c;
    }
    int at = m + before + inc - own;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if ((mine >> k) & 1u) {
        sh.key[at] = ((uint32_t)id[k] / (uint32_t)groups) << EB_PLACE_BITS | (uint32_t)at;
        sh.row[at] = (int32_t)(p + k);
        ++at;
      }
    m += all;
    __syncthreads();
  }
  if (m > 0) work_off(m);
  __syncthreads();
  if (accumulate) return;
  // tokens that no position holds; and what lies behind the last kept unit's period
  for (int token = warp; token < tokens; token += EB_WARPS) {
    float* out = dtable + (size_t)(group + (long long)token * groups) * lddt;
    if (!((sh.seen[token >> 5] >> (token & 31)) & 1u)) {
      if (dp == 1 && VEC && wide && c0 + EB_COLS <= n) {
        *reinterpret_cast<float4*>(out + c0 + 4 * lane) = make_float4(0.f, 0.f, 0.f, 0.f);
      } else {
        const long long end = min((long long)N, (long long)min(n, c0 + EB_COLS) * dp);
        for (long long j = (long long)c0 * dp + lane; j < end; j += 32) out[j] = 0.f;
      }
    }
    if (tail)
      for (long long j = (long long)n * dp + lane; j < N; j += 32) out[j] = 0.f;
  }
}

inline bool on(const void* p, long long ld, int bytes, int es) { return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * es % bytes == 0; }

template <typename T, int BYTES>
ard_status em_fwd(ard_ctx* ctx, const int32_t* hdr, int rows, int V, int N, float alpha, const int32_t* ids, const void* table, int ldt, void* Y,
                  int ldy, cudaStream_t s) {
  const int vecs = (N * (int)sizeof(T) + BYTES - 1) / BYTES;
  // four accesses a thread where that still leaves every SM its threads, else one
  const bool many = (double)rows * vecs >= 4.0 * 2048 * ctx->sm_count;
  int lanes = 1;
  while (lanes < EM_THREADS && lanes * (many ? 4 : 1) < vecs) lanes *= 2;
  const int per = EM_THREADS / lanes;
  const dim3 grid((unsigned)(((long long)rows + per - 1) / per));
  if (many)
    ARD_CUDA_OK(ard_launch(ctx, embedding_fwd_kernel<T, BYTES, 4>, grid, dim3(EM_THREADS), 0, s, hdr, rows, V, N, alpha, ids, (const T*)table, ldt,
                           (T*)Y, ldy, lanes, ctx->d_status));
  else
    ARD_CUDA_OK(ard_launch(ctx, embedding_fwd_kernel<T, BYTES, 1>, grid, dim3(EM_THREADS), 0, s, hdr, rows, V, N, alpha, ids, (const T*)table, ldt,
                           (T*)Y, ldy, lanes, ctx->d_status));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}

template <typename T>
ard_status em_bwd(ard_ctx* ctx, const int32_t* hdr, int rows, int V, int N, float alpha, const int32_t* ids, const void* dY, int lddy, float* dtable,
                  int lddt, int accumulate, cudaStream_t s) {
  const int chunks = (N + EB_COLS - 1) / EB_COLS;
  // one round of CTAs; more only where a CTA could not count its tokens.  The kernel divides them by the kept columns.
  const long long least = (long long)chunks * (((long long)V + EB_TOKENS - 2) / (EB_TOKENS - 1));
  const long long grid = least > ctx->sm_count ? least : ctx->sm_count;
  const bool vec = on(dY, lddy, 4 * (int)sizeof(T), (int)sizeof(T));
  const int wide = on(dtable, lddt, 16, 4);
  const int smem = (int)sizeof(EbShared);
  auto kern = vec ? embedding_bwd_kernel<T, true> : embedding_bwd_kernel<T, false>;
  ARD_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  if (grid > 0x7FFFFFFFll) return ARD_ERR_UNSUPPORTED;
  ARD_CUDA_OK(ard_launch(ctx, kern, dim3((unsigned)grid), dim3(EB_THREADS), smem, s, hdr, rows, V, N, alpha, ids, (const T*)dY, lddy, dtable, lddt,
                         accumulate, wide, ctx->d_status));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}

}  // namespace

ard_status launch_embedding_fwd(ard_ctx* ctx, const int32_t* hdr, ard_dtype dtype, int rows, int V, int N, float alpha, const int32_t* ids,
                                const void* table, int ldt, void* Y, int ldy, cudaStream_t s) {
  if (rows == 0 || N == 0) return ARD_OK;
  const int es = dtype == ARD_F32 ? 4 : 2;
  auto fits = [&](int bytes) { return on(table, ldt, bytes, es) && on(Y, ldy, bytes, es) && (long long)N * es % bytes == 0; };
  if (dtype == ARD_F32) {
    if (fits(16)) return em_fwd<float, 16>(ctx, hdr, rows, V, N, alpha, ids, table, ldt, Y, ldy, s);
    if (fits(8)) return em_fwd<float, 8>(ctx, hdr, rows, V, N, alpha, ids, table, ldt, Y, ldy, s);
    return em_fwd<float, 4>(ctx, hdr, rows, V, N, alpha, ids, table, ldt, Y, ldy, s);
  }
  if (fits(16)) return em_fwd<__nv_bfloat16, 16>(ctx, hdr, rows, V, N, alpha, ids, table, ldt, Y, ldy, s);
  if (fits(8)) return em_fwd<__nv_bfloat16, 8>(ctx, hdr, rows, V, N, alpha, ids, table, ldt, Y, ldy, s);
  if (fits(4)) return em_fwd<__nv_bfloat16, 4>(ctx, hdr, rows, V, N, alpha, ids, table, ldt, Y, ldy, s);
  return em_fwd<__nv_bfloat16, 2>(ctx, hdr, rows, V, N, alpha, ids, table, ldt, Y, ldy, s);
}

ard_status launch_embedding_bwd(ard_ctx* ctx, const int32_t* hdr, ard_dtype dtype, int rows, int V, int N, float alpha, const int32_t* ids,
                                const void* dY, int lddy, float* dtable, int lddt, int accumulate, cudaStream_t s) {
  if (V == 0 || N == 0 || (accumulate && rows == 0)) return ARD_OK;
  if (dtype == ARD_F32) return em_bwd<float>(ctx, hdr, rows, V, N, alpha, ids, dY, lddy, dtable, lddt, accumulate, s);
  return em_bwd<__nv_bfloat16>(ctx, hdr, rows, V, N, alpha, ids, dY, lddy, dtable, lddt, accumulate, s);
}
