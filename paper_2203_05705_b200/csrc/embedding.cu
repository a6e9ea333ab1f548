// Rows of a table by token, scaled, and the table's gradient:
//   Y[r][j] = alpha * table[ids[r]][col(j)],   dtable[v][col(j)] (+)= alpha * sum over r with ids[r] = v of dY[r][j],
// col(j) = j, or the j-th kept unit of a row pattern.
//
// Memory bounds both.  The gradient needs each token's rows side by side; sorting all of them through global memory would take several launches that
// hand one another the order.  Instead a CTA owns the tokens v = group (mod groups) and at most 128 columns: it looks through all ids (they come from the L2: 4
// bytes a position where a row of dY has thousands), keeps those that are its own in shared memory, sorts them there (by counting where they are few, else
// digit by digit, either way with a token's rows in their order), and adds their rows up.  One launch, no scratch, and the same bits every time: each
// sum is cut at the same places.  Equal shares of the sorted list go to the warps, so a frequent token has all warps of its CTA at work, but no other CTA's: with one
// token in half of 65536 positions, 128 columns take 342 us where tokens that are all alike often take 35.  Tokens are dealt out in turn, so frequent ones, which lie
// side by side in a dictionary sorted by frequency, fall to different CTAs.  Zeros for tokens that no position holds are written beside the sums, by warps that
// have nothing to add.
//
// 16384 positions, 32000 tokens, 2048 columns, bf16: lookup 20.6 us with tokens all alike often, 16.5 by falling frequency (5400 of them come up), gradient 81 (329 MB: 4.1
// TB/s) and 89: the list of a CTA, its sort and then its rows follow one another, and 64 registers a thread with 16 rows in flight spill 340 bytes; fp32 31 to 43, and 96
// and 109.  700 positions, 8800 tokens, 750 of 1500 columns kept: 4.2 and 18.5, of which 7.4 the 53 MB of the gradient and 4 the start (a CTA has
// looked at its ids 8000 cycles after it began).
#include <cooperative_groups.h>

#include "ard_internal.h"
#include "sm100_ptx.h"

namespace {

namespace cg = cooperative_groups;

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
constexpr int EB_THREADS = 1024, EB_WARPS = 24;  // all of them look for tokens; 24 warps add rows up, the others write zeros meanwhile
constexpr int EB_WORKERS = EB_WARPS * 32;
constexpr int EB_COLS = 128;             // columns of a CTA: 4 a lane
constexpr int EB_PLACE_BITS = 13;        // places of the list, which end the key that is sorted
constexpr int EB_LIST = 1 << EB_PLACE_BITS;
constexpr int EB_STEP = 4 * EB_THREADS;  // ids looked at at a time
constexpr int EB_TOKENS = 1 << 18;       // most tokens of a CTA
constexpr int EB_DIGIT = 6;              // bits of a token that a pass of the sort takes
constexpr int EB_FEW = 256;              // lists up to here are sorted by counting (58 keys: 2300 cycles, by two digits 7400)

// What of a token's row of the gradient a warp writes: some kept columns, at most 128, and the dropped ones of their periods; the last CTA of columns has the row's end too.
struct EbTable {
  float* p;
  int ld, dp, first, n, N, c0, c1;  // columns c0 .. c1 - 1 of the kept ones
  float alpha;
  int wide;  // rows on the grid of 16 bytes
  __device__ __forceinline__ long long end() const { return c1 == n ? N : (long long)c1 * dp; }
};

struct EbShared {
  uint32_t key[2][EB_LIST];                    // token / groups, then the place in the list
  int32_t row[EB_LIST];
  uint32_t here[EB_TOKENS / 32];               // tokens that come up
  uint32_t written[EB_TOKENS / 32];            // tokens whose row of the gradient holds a sum already
  float part[2][EB_WARPS][EB_COLS];            // sums of tokens that several warps share: a share's first and its last
  uint32_t digits[EB_WARPS][1 << EB_DIGIT];    // how often each comes up in a warp's share, then where the share's begin
  uint32_t total[2];
  int count[EB_THREADS / 32];
  int next;                                    // four tokens that nobody has written zeros for yet
  EbTable table;
};
static_assert(sizeof(EbShared) <= 227 * 1024, "shared memory of an SM");

template <bool VEC>
struct EbCols {  // a lane's columns: 4 * lane + k, or lane + 32 * k where those do not lie on a grid of four
  __device__ __forceinline__ static int col(int lane, int k) { return VEC ? 4 * lane + k : lane + 32 * k; }
};
__device__ __forceinline__ void eb_meet() {  // the warps that add up
  __syncwarp();
  asm volatile("bar.sync 1, %0;" ::"n"(EB_WORKERS) : "memory");
}
// x / d for x below 2^31, by a product: magic = ceil(2^(31 + bits) / d), bits = ceil(log2 d).
struct EbDivisor {
  uint32_t d, magic, shift;
  __device__ __forceinline__ explicit EbDivisor(uint32_t by) : d(by) {
    const int bits = 32 - __clz((int)(by - 1));
    shift = 31 + (by > 1 ? bits : 0);
    magic = (uint32_t)((double)(1ull << shift) / (double)by);  // (an integer division of 64 bits takes longer)
    while ((unsigned long long)magic * by < (1ull << shift)) ++magic;
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t x) const { return (uint32_t)(((unsigned long long)x * magic) >> shift); }
};

// (Out of line: it stands behind each of a round's rows, and sixteen copies of it do not fit the instruction cache.  `g` lies in shared memory: local memory
// would stand in line behind the stores of zeros.)
template <bool VEC>
__device__ __noinline__ void eb_write(const EbTable& g, long long token, float s0, float s1, float s2, float s3, bool add, int lane) {
  float* out = g.p + (size_t)token * g.ld;
  const float x[4] = {g.alpha * s0, g.alpha * s1, g.alpha * s2, g.alpha * s3};
  const int j0 = g.c0 + 4 * lane;
  if (VEC && g.wide && g.dp == 1 && (j0 + 3 < g.c1 || j0 >= g.c1)) {
    if (j0 >= g.c1) return;
    // one addition an element and pass over the list, so that its order is that of the passes; nothing waits for the old value
    if (add) asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(out + j0), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]) : "memory");
    else *reinterpret_cast<float4*>(out + j0) = make_float4(x[0], x[1], x[2], x[3]);
    return;
  }
  const bool whole = VEC && g.wide && !add && j0 + 3 < g.c1 && (j0 + 4ll) * g.dp <= g.N;
  if (whole) {  // four periods, which begin and end on 16 bytes
    float x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
    int d = 0;
    for (int q = 0; q < g.dp; ++q) {
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = d == g.first ? x0 : 0.f;
        if (++d == g.dp) d = 0, x0 = x1, x1 = x2, x2 = x3;
      }
      *reinterpret_cast<float4*>(out + (size_t)j0 * g.dp + 4 * q) = make_float4(v[0], v[1], v[2], v[3]);
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int j = g.c0 + EbCols<VEC>::col(lane, k);
    if (whole || j >= g.c1) continue;
    float* to = out + (size_t)j * g.dp;
    if (add) {
      atomicAdd(to + g.first, x[k]);
    } else {
      for (int d = 0; d < g.dp && (long long)j * g.dp + d < g.N; ++d) to[d] = d == g.first ? x[k] : 0.f;
    }
  }
  if (!add && g.c1 == g.n)
    for (long long j = (long long)g.n * g.dp + lane; j < g.N; j += 32) out[j] = 0.f;
}
// Zeros for a token that no position holds.
__device__ __forceinline__ void eb_zero(const EbTable& g, long long token, int lane) {
  float* out = g.p + (size_t)token * g.ld;
  const long long from = (long long)g.c0 * g.dp, end = g.end();
  if (g.wide) {
    long long j = from + 4 * lane;
    for (; j + 3 < end; j += 128) *reinterpret_cast<float4*>(out + j) = make_float4(0.f, 0.f, 0.f, 0.f);
    for (; j < end; ++j) out[j] = 0.f;  // (the lane that the row's end falls to)
  } else {
    for (long long j = from + lane; j < end; j += 32) out[j] = 0.f;
  }
}

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
  // columns in equal parts, so that no CTA has more to write than another
  const int width = ((n + chunks - 1) / chunks + 3) & ~3, group = blockIdx.x % groups, c0 = (blockIdx.x / groups) * width, c1 = min(n, c0 + width);
  if (c0 >= n && c0 > 0) return;
  const int tokens = (V - group - 1) / groups + 1;
  for (int i = t; i < (tokens + 31) / 32; i += EB_THREADS) sh.here[i] = sh.written[i] = 0u;
  using Raw = typename EmRaw<4 * sizeof(T)>::type;
  constexpr int EB_AHEAD = 32 / (int)sizeof(T);  // rows of dY in flight a warp: what 64 registers a thread hold
  const bool full = VEC && ((c1 - c0) & 3) == 0;  // a lane's columns are all there, or none is
  const bool on = c0 + 4 * lane < c1, fast = full && wide && dp == 1;
  const int mine = on ? 4 * lane : 0;
  const EbTable& g = sh.table;
  if (t == 0) sh.table = {dtable, lddt, dp, first, n, N, c0, c1, alpha, wide};
  const EbDivisor by(groups);
  float* const fast_p = dtable + (size_t)group * lddt + c0 + mine;  // the group's first token
  const size_t fast_step = (size_t)groups * lddt;
  const bool lists = rows > EB_LIST;  // perhaps more than one of them
  if (t == 0) sh.next = 0;
  auto token_of = [&](int at) { return group + (long long)at * groups; };

  auto flush = [&](int token, const float (&sum)[4]) {
    const bool old = lists && ((sh.written[token >> 5] >> (token & 31)) & 1u);
    if (fast) {
      if (on) {
        float* out = fast_p + (size_t)token * fast_step;
        if (accumulate || old) asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(out), "f"(alpha * sum[0]), "f"(alpha * sum[1]), "f"(alpha * sum[2]), "f"(alpha * sum[3]) : "memory");
        else *reinterpret_cast<float4*>(out) = make_float4(alpha * sum[0], alpha * sum[1], alpha * sum[2], alpha * sum[3]);
      }
    } else {
      eb_write<VEC>(g, token_of(token), sum[0], sum[1], sum[2], sum[3], accumulate || old, lane);
    }
    if (lists) {
      __syncwarp();
      if (lane == 0 && !old) atomicOr(&sh.written[token >> 5], 1u << (token & 31));
    }
  };

  // Sorts the list by token, each token's rows staying in order, and adds them up; by the first 24 warps.
  int bits = 0;
  while ((1 << bits) < tokens) ++bits;
  auto work_off = [&](int m) {
    const int share = (m + EB_WARPS - 1) / EB_WARPS, from = min(m, warp * share), to = min(m, from + share);
    const bool few = m <= EB_FEW;
    int src = 0;
    if (few) {  // a key's place is the number of smaller ones: no two are alike
      if (t < m) {
        const uint32_t k = sh.key[0][t];
        int place = 0;
#pragma unroll 4
        for (int i = 0; i < m; i += 4) {
          const uint4 q = *reinterpret_cast<const uint4*>(&sh.key[0][i]);
          place += (q.x < k) + (i + 1 < m && q.y < k) + (i + 2 < m && q.z < k) + (i + 3 < m && q.w < k);
        }
        sh.key[1][place] = k;
      }
      eb_meet();
      src = 1;
    }
    for (int at = EB_PLACE_BITS; !few && at < EB_PLACE_BITS + bits; at += EB_DIGIT) {
      // how often each digit comes up in a warp's share; the places follow from the counts of earlier digits and, for the same digit, earlier warps
      uint32_t* mine = sh.digits[warp];
      mine[lane] = mine[lane + 32] = 0u;
      __syncwarp();
      for (int i = from + lane; i < to; i += 32) atomicAdd(&mine[(sh.key[src][i] >> at) & ((1 << EB_DIGIT) - 1)], 1u);
      eb_meet();
      if (t < (1 << EB_DIGIT)) {
        uint32_t sum = 0;
#pragma unroll
        for (int w = 0; w < EB_WARPS; ++w) {
          const uint32_t c = sh.digits[w][t];
          sh.digits[w][t] = sum;
          sum += c;
        }
        uint32_t inc = sum;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
          const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, inc, o);
          if (lane >= o) inc += x;
        }
        if (lane == 31) sh.total[warp] = inc;
        asm volatile("bar.sync 2, 64;" ::: "memory");
        inc += (warp ? sh.total[0] : 0u) - sum;
#pragma unroll
        for (int w = 0; w < EB_WARPS; ++w) sh.digits[w][t] += inc;
      }
      eb_meet();
      for (int i0 = from; i0 < to; i0 += 32) {
        const int i = i0 + lane;
        const uint32_t k = i < to ? sh.key[src][i] : 0u, digit = i < to ? (k >> at) & ((1 << EB_DIGIT) - 1) : 64u + lane;
        const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit);
        if (i < to) sh.key[src ^ 1][mine[digit] + __popc(same & ((1u << lane) - 1u))] = k;
        __syncwarp();
        if (i < to && (same >> lane) == 1u) mine[digit] += __popc(same);  // the last of them
        __syncwarp();
      }
      eb_meet();
      src ^= 1;
    }
    const uint32_t* key = sh.key[src];
    uint32_t* order = sh.key[src ^ 1];  // rows in the list's order, with a mark at a token's last
    auto token_at = [&](int i) { return (int)(key[i] >> EB_PLACE_BITS); };
    for (int i = from + lane; i < to; i += 32)
      order[i] = (uint32_t)sh.row[key[i] & (EB_LIST - 1)] | (i + 1 < m && token_at(i + 1) == token_at(i) ? 0u : 0x80000000u);
    __syncwarp();
    // a warp's share of the list; a token that a share begins or ends with may go on in the next one
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    bool open_back = false;
    if (from < to) {
      bool front = from > 0 && token_at(from - 1) == token_at(from);
      open_back = !(order[to - 1] >> 31);
      auto next = [&](int i, uint32_t o, const float (&x)[4]) {
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] += x[k];
        if (!(o >> 31)) return;
        if (front) {
#pragma unroll
          for (int k = 0; k < 4; ++k) sh.part[0][warp][EbCols<VEC>::col(lane, k)] = sum[k];
          front = false;
        } else {
          flush(token_at(i), sum);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] = 0.f;
      };
      auto row_at = [&](uint32_t o) { return dY + (size_t)(o & 0x7FFFFFFFu) * lddy + c0; };
      if (full) {  // all loads before the first use
        for (int i0 = from; i0 < to; i0 += EB_AHEAD) {
          Raw q[EB_AHEAD];
#pragma unroll
          for (int u = 0; u < EB_AHEAD; ++u) q[u] = *reinterpret_cast<const Raw*>(row_at(order[min(i0 + u, to - 1)]) + mine);
#pragma unroll
          for (int u = 0; u < EB_AHEAD; ++u) {
            if (i0 + u >= to) break;
            T e[4];
            memcpy(e, &q[u], sizeof(Raw));
            const float x[4] = {em_f32(e[0]), em_f32(e[1]), em_f32(e[2]), em_f32(e[3])};
            next(i0 + u, order[i0 + u], x);
          }
        }
      } else {
        constexpr int AHEAD = 8;
        for (int i0 = from; i0 < to; i0 += AHEAD) {
          T e[AHEAD][4];
#pragma unroll
          for (int u = 0; u < AHEAD; ++u) {
            const T* src = row_at(order[min(i0 + u, to - 1)]);
#pragma unroll
            for (int k = 0; k < 4; ++k) e[u][k] = src[min(EbCols<VEC>::col(lane, k), c1 - 1 - c0)];  // (beyond them: nobody asks)
          }
#pragma unroll
          for (int u = 0; u < AHEAD; ++u) {
            if (i0 + u >= to) break;
            const float x[4] = {em_f32(e[u][0]), em_f32(e[u][1]), em_f32(e[u][2]), em_f32(e[u][3])};
            next(i0 + u, order[i0 + u], x);
          }
        }
      }
      if (open_back) {  // a share of one token that is open on both sides counts as its first
#pragma unroll
        for (int k = 0; k < 4; ++k) sh.part[front ? 0 : 1][warp][EbCols<VEC>::col(lane, k)] = sum[k];
      }
      if (front) open_back = false;  // (its sum goes on from an earlier warp)
    }
    eb_meet();
    // the warp with whose share a divided token begins adds up its pieces, in the list's order
    if (open_back) {
      const int token = token_at(to - 1);
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[k] = sh.part[1][warp][EbCols<VEC>::col(lane, k)];
      for (int w = warp + 1; w < EB_WARPS; ++w) {
        const int at = w * share;
        if (at >= m || token_at(at) != token) break;
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] += sh.part[0][w][EbCols<VEC>::col(lane, k)];
      }
      flush(token, sum);
    }
  };

  int m = 0;
  __syncthreads();
  for (long long p0 = 0; p0 < rows; p0 += EB_STEP) {
    if (m + EB_STEP > EB_LIST) {  // the next step might not fit
      if (warp < EB_WARPS) work_off(m);
      m = 0;
      __syncthreads();
    }
    // four positions side by side a thread, so that the list is in their order
    const long long p = p0 + 4 * t;
    int id[4];
    if (p + 3 < rows && (reinterpret_cast<uintptr_t>(ids + p) & 15u) == 0) {
      const int4 q = *reinterpret_cast<const int4*>(ids + p);
      id[0] = q.x, id[1] = q.y, id[2] = q.z, id[3] = q.w;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) id[k] = p + k < rows ? ids[p + k] : -1;
    }
    unsigned own = 0;
    uint32_t at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (id[k] >= V && blockIdx.x == 0) atomicMax(status, (int)ARD_ERR_INVALID_ARG);
      at[k] = by((uint32_t)max(id[k], 0));
      if (id[k] >= 0 && id[k] < V && (int)((uint32_t)id[k] - at[k] * by.d) == group) own |= 1u << k;
    }
    int inc = __popc(own);
    const int all_mine = inc;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int x = __shfl_up_sync(0xFFFFFFFFu, inc, o);
      if (lane >= o) inc += x;
    }
    if (lane == 31) sh.count[warp] = inc;
    __syncthreads();
    int before = 0, all = 0;
    {
      const int c = sh.count[lane];
      before = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? c : 0);
      all = __reduce_add_sync(0xFFFFFFFFu, c);
    }
    int place = m + before + inc - all_mine;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if ((own >> k) & 1u) {
        sh.key[0][place] = at[k] << EB_PLACE_BITS | (uint32_t)place;
        sh.row[place] = (int32_t)(p + k);
        atomicOr(&sh.here[at[k] >> 5], 1u << (at[k] & 31));
        ++place;
      }
    m += all;
    __syncthreads();
  }
  // the tokens that come up are known: the last of the list is added up beside the others' zeros, which all warps write that have nothing else to do
  if (warp < EB_WARPS && m > 0) work_off(m);
  if (accumulate) return;
  // (four tokens at a time, so that all warps of all CTAs write in one neighbourhood: 200000 rows of 300 in 32s 80 us)
  for (;;) {
    int q = 0;
    if (lane == 0) q = atomicAdd(&sh.next, 1);
    q = __shfl_sync(0xFFFFFFFFu, q, 0);
    if (4 * q >= tokens) return;
    const uint32_t here = sh.here[q >> 3] >> (4 * (q & 7));
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int token = 4 * q + b;
      if (token >= tokens || ((here >> b) & 1u)) continue;
      if (fast) {
        if (on) *reinterpret_cast<float4*>(fast_p + (size_t)token * fast_step) = make_float4(0.f, 0.f, 0.f, 0.f);
      } else {
        eb_zero(g, token_of(token), lane);
      }
    }
  }
}

// ---- gradient of few tokens -----------------------------------------------------------------------------
// Where V tokens of `chunks` times 128 columns leave SMs without work, a cluster of CTAs has one token: each looks through its part of the positions and adds up the rows that hold the
// token, 32 / lanes of them side by side; the cluster's sums meet in its first CTA, in order.
constexpr int EF_THREADS = 1024, EF_WARPS = EF_THREADS / 32, EF_CLUSTER = 8;

template <typename T, bool VEC>
__global__ void __launch_bounds__(EF_THREADS, 1) embedding_bwd_few_kernel(const int32_t* hdr, int rows, int V, int N, float alpha, const int32_t* ids,
                                                                          const T* dY, int lddy, float* dtable, int lddt, int accumulate,
                                                                          int wide, int parts, int* status) {
  __shared__ float sums[EF_WARPS][EB_COLS];
  __shared__ float all[EB_COLS];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const int rank = (int)(blockIdx.x % parts), unit = (int)(blockIdx.x / parts), token = unit % V, c0 = unit / V * EB_COLS;
  int dp = 1, first = 0, n = N;
  if (hdr) dp = hdr[HDR_DP], first = hdr[HDR_B] - 1, n = hdr[HDR_NKEEP];
  const bool any = c0 < n || (c0 == 0 && n == 0);  // (uniform over the cluster)
  const int cols = min(EB_COLS, n - c0);
  int lanes = VEC ? 1 : 32;
  while (lanes < 32 && lanes * 4 < cols) lanes *= 2;
  const int sub = lane / lanes, subs = 32 / lanes, sl = lane % lanes;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  if (any && cols > 0) {
    // a part's positions in rounds of 32 a warp
    const long long each = (((long long)rows + parts - 1) / parts + 31) / 32 * 32, from = rank * each, to = min((long long)rows, from + each);
    for (long long p0 = from + 32 * warp; p0 < to; p0 += 32 * EF_WARPS) {
      const int id = p0 + lane < to ? ids[p0 + lane] : -1;
      if (id >= V && unit == 0) atomicMax(status, (int)ARD_ERR_INVALID_ARG);
      unsigned left = __ballot_sync(0xFFFFFFFFu, id == token);
      constexpr int AHEAD = 8;
      while (left) {  // (uniform) rounds of AHEAD rows a group of lanes
        T e[AHEAD][4];
        bool there[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          unsigned mine = left;
          for (int i = 0; i < sub; ++i) mine &= mine - 1;  // the sub-th of those that are left
          there[u] = mine != 0;
          const long long r = p0 + (mine ? __ffs(mine) - 1 : 0);
          if (there[u]) {
            const T* src = dY + (size_t)r * lddy + c0;
            if (VEC && 4 * sl + 3 < cols) {
              using Raw = typename EmRaw<4 * sizeof(T)>::type;
              const Raw q = *reinterpret_cast<const Raw*>(src + 4 * sl);
              memcpy(e[u], &q, sizeof(q));
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k) e[u][k] = src[min(EbCols<VEC>::col(sl, k), cols - 1)];
            }
          }
          for (int i = 0; i < subs; ++i) left &= left - 1;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
          if (there[u])
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] += em_f32(e[u][k]);
      }
    }
  }
  for (int o = lanes; o < 32; o *= 2)
#pragma unroll
    for (int k = 0; k < 4; ++k) sum[k] += __shfl_xor_sync(0xFFFFFFFFu, sum[k], o);
  if (sub == 0)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (EbCols<VEC>::col(sl, k) < EB_COLS) sums[warp][EbCols<VEC>::col(sl, k)] = sum[k];
  __syncthreads();
  if (t < EB_COLS) {
    float x = 0.f;
    if (t < cols)
#pragma unroll 8
      for (int w = 0; w < EF_WARPS; ++w) x += sums[w][t];
    all[t] = x;
  }
  if (parts > 1) cg::this_cluster().sync();
  else __syncthreads();
  if (rank == 0 && warp == 0 && any) {
    __shared__ EbTable table;
    if (lane == 0) table = {dtable, lddt, dp, first, n, N, c0, c0 + max(cols, 0), alpha, wide};
    __syncwarp();
    float x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = EbCols<VEC>::col(lane, k);
      x[k] = all[c];
      for (int p = 1; p < parts; ++p) x[k] += *cg::this_cluster().map_shared_rank(&all[c], p);
    }
    eb_write<VEC>(table, token, x[0], x[1], x[2], x[3], accumulate, lane);
  }
  if (parts > 1) {
    __syncwarp();
    cg::this_cluster().sync();  // nobody leaves while its sums are read
  }
}

inline bool on(const void* p, long long ld, int bytes, int es) { return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * es % bytes == 0; }

template <typename T, int BYTES>
ard_status em_fwd(ard_ctx* ctx, const int32_t* hdr, int rows, int V, int N, float alpha, const int32_t* ids, const void* table, int ldt, void* Y,
                  int ldy, cudaStream_t s) {
  const int vecs = (int)(((long long)N * (int)sizeof(T) + BYTES - 1) / BYTES);
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
  const long long least = (long long)chunks * (((long long)V + EB_TOKENS - 1) / EB_TOKENS);
  const long long grid = least > ctx->sm_count ? least : ctx->sm_count;
  const bool vec = on(dY, lddy, 4 * (int)sizeof(T), (int)sizeof(T));
  const int wide = on(dtable, lddt, 16, 4);
  if ((long long)V * chunks * 2 <= ctx->sm_count) {
    int parts = 1;
    while (parts < EF_CLUSTER && (long long)V * chunks * parts * 2 <= ctx->sm_count) parts *= 2;
    auto few = vec ? embedding_bwd_few_kernel<T, true> : embedding_bwd_few_kernel<T, false>;
    ARD_CUDA_OK(ard_launch_cluster(ctx, few, parts, dim3((unsigned)(V * chunks * parts)), dim3(EF_THREADS), 0, s, hdr, rows, V, N, alpha, ids, (const T*)dY, lddy,
                                   dtable, lddt, accumulate, wide, parts, ctx->d_status));
    ctx->launches++;
    ARD_CUDA_OK(cudaGetLastError());
    return ARD_OK;
  }
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
