// The gated delta rule over whole sequences, forward and adjoint.  Per sequence and head, with a state S [Dk][Dv],
//   S_t = f_t S_{t-1} + k_t u_t^T,  u_t = b_t (v_t - f_t S_{t-1}^T k_t),  y_t = scale S_t^T q_t,
// f = s(zf), b = s(zb), q and k divided by their lengths.
//
// Step by step this is three products of a matrix with a vector, 3 Dk Dv multiply-adds that wait for the step before.  Over a chunk of 64
// steps the updates solve a triangular system whose matrix depends on keys and gates alone,
//   (I + A) U = b (V - g K S_0),   A_ij = b_i G_ij k_i.k_j (j < i),   G_ij = f_{j+1} .. f_i,   g_i = f_1 .. f_i,
//   Y = scale (g Q S_0 + (G o Q K^T) U),   S_C = g_C S_0 + (G_C K)^T U,
// so one kernel inverts I + A for all chunks at once (delta_prep_kernel), and what goes from chunk to chunk is products of
// matrices (delta_scan_kernel), with the columns of S, which do not see one another, on different SMs.  Decays are products of gates, never
// quotients or differences of logarithms: a gate of zero cuts the past off and nothing else.
//
// The adjoint has the same shape: with D the gradient of the state behind a chunk,
//   X = (I + A)^-T (scale P^T dY + (G_C K) D),  dV = b X,  D_0 = g_C D + scale (g Q)^T dY - (g K)^T b X
// goes from chunk to chunk (delta_back_kernel), and everything else of a chunk is its own (delta_grad_kernel).
//
// The state is fp32, and so are products that it goes through: an operand that is not bf16 to begin with is the sum of three bf16 matrices (24 bits), and
// the products of their parts that fp32 can hold are added up.  Where a product ends in a bf16 output two parts are enough (17 bits, an
// error of 2^-18 of a term where the output's rounding is 2^-9).  The products are small (64 x 32 x 128 a warp group, four in a row that wait for one another), which mma.sync takes from
// registers and leaves in registers; a tcgen05 product would bring each result from tensor memory to registers, split it, and put it back, and
// its 128 rows of an accumulator would leave half of the SMs without work at 64 heads.
#include "ard_internal.h"
#include "sm100_ptx.h"

namespace {

constexpr int DL_CHUNK = 64;
constexpr int DL_THREADS = 256;
constexpr int DL_LD64 = DL_CHUNK + 8;  // pitch of [64][64] matrices in shared memory: rows on different banks
constexpr int DL_CB = 32;              // columns of the state that a CTA of the scans holds
constexpr int DL_LDC = DL_CB + 8;

using bf = __nv_bfloat16;

struct DlArgs {
  int T, B, heads, Dk, Dv;
  float scale, eps;  // eps < 0: q and k as they are
  const bf *Q, *K, *V;
  long long ldq, ldk, ldv;
  const bf *Zf, *Zb;
  long long ldz;
  const int32_t* lens;
  const float* h0;
  bf* Y;
  long long ldy;
  float* hT;
  float* S;
  const bf* dY;
  long long lddy;
  const float* dhT;
  bf *dQ, *dK, *dV;
  long long lddq, lddk, lddv;
  bf *dZf, *dZb;
  long long lddz;
  float* dh0;
  int vec_q, vec_k, vec_dy;  // whether rows lie on a grid of 16 bytes
  // work, by unit = chunk * B * heads + sequence * heads + head
  bf* tri;       // [units][3][64][64] (I + A)^-1 in three parts
  bf* p;         // [units][3][64][64] scale * (G o Q K^T) in three parts
  float* row;    // [units][DL_ROWS][64] what each step has of its own
  float* x;      // [units][64][Dv]
  float* d;      // [units][Dk][Dv] the gradient of the state behind a chunk
};
enum { DL_RK, DL_RQ, DL_BETA, DL_F, DL_REST, DL_FIRST, DL_LAST, DL_ROWS };  // 1/|k|, 1/|q|, b, f, 1 - f, g_i, G_Ci

// ---- building blocks --------------------------------------------------------------------------------
__device__ __forceinline__ void dl_ldsm(uint32_t (&r)[4], const bf* p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(smem_u32(p))
               : "memory");
}
__device__ __forceinline__ void dl_ldsm_t(uint32_t (&r)[4], const bf* p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(smem_u32(p))
               : "memory");
}
// 16 x 16 of the left operand, rows m0, contraction k0: from [m][k], or from [k][m].
template <bool T>
__device__ __forceinline__ void dl_a(uint32_t (&r)[4], const bf* s, int ld, int m0, int k0, int lane) {
  if constexpr (!T) dl_ldsm(r, s + (m0 + (lane & 15)) * ld + k0 + (lane >> 4) * 8);
  else dl_ldsm_t(r, s + (k0 + (lane & 7) + ((lane >> 4) << 3)) * ld + m0 + ((lane >> 3) & 1) * 8);
}
// 16 (contraction k0) x 16 (columns n0) of the right operand: from [n][k], or from [k][n].  r[0], r[1]: columns n0 .. n0 + 7.
template <bool KN>
__device__ __forceinline__ void dl_b(uint32_t (&r)[4], const bf* s, int ld, int n0, int k0, int lane) {
  if constexpr (!KN) dl_ldsm(r, s + (n0 + (lane & 7) + ((lane >> 4) << 3)) * ld + k0 + ((lane >> 3) & 1) * 8);
  else dl_ldsm_t(r, s + (k0 + (lane & 7) + ((lane >> 3) & 1) * 8) * ld + n0 + (lane >> 4) * 8);
}
__device__ __forceinline__ void dl_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// c[NT][4] += A (16 rows m0) * B (8 NT columns n0) over the contraction [k0, k1), operands in PA and PB parts `sa`, `sb` elements apart.  Parts i
// and j are multiplied where i + j <= MOST: smaller products are below what is kept.
template <int NT, bool AT, bool BKN, int PA, int PB, int MOST>
__device__ __forceinline__ void dl_product(float (&c)[NT][4], const bf* a, int lda, int sa, const bf* b, int ldb, int sb, int m0, int n0, int k0, int k1,
                                           int lane) {
  static_assert(NT % 2 == 0, "columns by sixteens");
  for (int k = k0; k < k1; k += 16) {
    uint32_t ra[PA][4];
#pragma unroll
    for (int i = 0; i < PA; ++i) dl_a<AT>(ra[i], a + i * sa, lda, m0, k, lane);
#pragma unroll
    for (int n = 0; n < NT; n += 2) {
#pragma unroll
      for (int j = PB - 1; j >= 0; --j) {  // small parts first
        uint32_t rb[4];
        dl_b<BKN>(rb, b + j * sb, ldb, n0 + 8 * n, k, lane);
#pragma unroll
        for (int i = PA - 1; i >= 0; --i)
          if (i + j <= MOST) {
            dl_mma(c[n], ra[i], rb[0], rb[1]);
            dl_mma(c[n + 1], ra[i], rb[2], rb[3]);
          }
      }
    }
  }
}

// Two neighbours in PARTS bf16 parts, each pair in a word: x = sum of the parts.
template <int PARTS>
__device__ __forceinline__ void dl_split(float x, float y, uint32_t (&w)[PARTS]) {
#pragma unroll
  for (int i = 0; i < PARTS; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    memcpy(&w[i], &h, 4);
    if (i + 1 < PARTS) {
      x -= __low2float(h);
      y -= __high2float(h);
    }
  }
}
template <int PARTS>
__device__ __forceinline__ void dl_put(bf* s, int stride, float x, float y) {
  uint32_t w[PARTS];
  dl_split<PARTS>(x, y, w);
#pragma unroll
  for (int i = 0; i < PARTS; ++i) *reinterpret_cast<uint32_t*>(s + i * stride) = w[i];
}

// s(z) and 1 - s(z), each to a few units of its own size.
__device__ __forceinline__ void dl_gate(float z, float& f, float& rest) {
  const float e = __expf(-fabsf(z)), big = __frcp_rn(1.f + e), small = e * big;
  f = z >= 0.f ? big : small;
  rest = z >= 0.f ? small : big;
}

// [64][cols] of a matrix whose rows are `step` elements apart, to shared memory with pitch ld; rows from `live` on and columns up to
// `pad` are zeros.
__device__ __forceinline__ void dl_load(bf* s, int ld, const bf* g, long long step, int live, int cols, int pad, int vec) {
  const int pieces = pad / 8;
  for (int i = threadIdx.x; i < DL_CHUNK * pieces; i += blockDim.x) {
    const int r = i / pieces, c = (i - r * pieces) * 8;
    uint4 q = make_uint4(0, 0, 0, 0);
    if (r < live && c < cols) {
      const bf* p = g + r * step + c;
      if (vec) {
        q = *reinterpret_cast<const uint4*>(p);
      } else {
        bf e[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = c + k < cols ? p[k] : __float2bfloat16_rn(0.f);
        memcpy(&q, e, 16);
      }
    }
    *reinterpret_cast<uint4*>(s + r * ld + c) = q;
  }
}

struct DlUnit {
  int chunk, b, head, live;  // live: steps of the chunk that are inside the sequence
  long long n, unit, row0;   // sequence and head; its place in the work; row of the chunk's first step
};
__device__ __forceinline__ DlUnit dl_unit(const DlArgs& a, int chunk, long long n) {
  DlUnit u;
  u.chunk = chunk;
  u.n = n;
  u.b = (int)(n / a.heads);
  u.head = (int)(n - (long long)u.b * a.heads);
  const int len = a.lens ? min(max(a.lens[u.b], 0), a.T) : a.T;
  u.live = min(max(len - chunk * DL_CHUNK, 0), DL_CHUNK);
  u.unit = (long long)chunk * a.B * a.heads + n;
  u.row0 = (long long)chunk * DL_CHUNK * a.B + u.b;
  return u;
}

// ---- a chunk's triangular system ----------------------------------------------------------------------
template <int DK>
struct DlPrepShared {
  bf k[DL_CHUNK][DK + 8], q[DL_CHUNK][DK + 8];
  float g[DL_CHUNK][DL_CHUNK + 1];  // G_ij
  float a[DL_CHUNK][DL_CHUNK + 1];  // A, below the diagonal
  float t[DL_CHUNK][DL_CHUNK + 1];  // its inverse with ones on the diagonal
  float tmp[3][16][17];
  float row[DL_ROWS][DL_CHUNK];
};

template <int DK>
__global__ void __launch_bounds__(DL_THREADS) delta_prep_kernel(const DlArgs a) {
  extern __shared__ __align__(16) uint8_t dl_smem[];
  auto& sh = *reinterpret_cast<DlPrepShared<DK>*>(dl_smem);
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const long long units = (long long)a.B * a.heads;
  const DlUnit u = dl_unit(a, (int)(blockIdx.x / units), blockIdx.x % units);
  if (u.live == 0) return;  // nobody asks
  dl_load(&sh.k[0][0], DK + 8, a.K + u.row0 * a.ldk + (long long)u.head * a.Dk, a.B * a.ldk, u.live, a.Dk, DK, a.vec_k);
  dl_load(&sh.q[0][0], DK + 8, a.Q + u.row0 * a.ldq + (long long)u.head * a.Dk, a.B * a.ldq, u.live, a.Dk, DK, a.vec_q);
  if (t < DL_CHUNK) {
    float f = 1.f, rest = 0.f, beta = 0.f, no;
    if (t < u.live) {
      const long long r = (u.row0 + (long long)t * a.B) * a.ldz + u.head;
      dl_gate(__bfloat162float(a.Zf[r]), f, rest);
      dl_gate(__bfloat162float(a.Zb[r]), beta, no);
    }
    sh.row[DL_F][t] = f;
    sh.row[DL_REST][t] = rest;
    sh.row[DL_BETA][t] = beta;
  }
  __syncthreads();
  {  // lengths: four threads a row
    const int r = t >> 2, part = t & 3;
    float kk = 0.f, qq = 0.f;
    for (int c = part * 2; c < DK; c += 8) {
      const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&sh.k[r][c]));
      const float2 y = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&sh.q[r][c]));
      kk = fmaf(x.x, x.x, fmaf(x.y, x.y, kk));
      qq = fmaf(y.x, y.x, fmaf(y.y, y.y, qq));
    }
#pragma unroll
    for (int o = 1; o < 4; o *= 2) {
      kk += __shfl_xor_sync(0xFFFFFFFFu, kk, o);
      qq += __shfl_xor_sync(0xFFFFFFFFu, qq, o);
    }
    if (part == 0) {
      kk += a.eps, qq += a.eps;
      sh.row[DL_RK][r] = a.eps < 0.f ? 1.f : kk > 0.f ? 1.f / sqrtf(kk) : 0.f;
      sh.row[DL_RQ][r] = a.eps < 0.f ? 1.f : qq > 0.f ? 1.f / sqrtf(qq) : 0.f;
    }
  }
  if (t < DL_CHUNK) {  // a column of the decays
    float g = 1.f;
    sh.g[t][t] = 1.f;
    for (int i = t + 1; i < DL_CHUNK; ++i) sh.g[i][t] = g *= sh.row[DL_F][i];
    sh.row[DL_LAST][t] = g;
  } else if (t == DL_CHUNK) {
    float g = 1.f;
    for (int i = 0; i < DL_CHUNK; ++i) sh.row[DL_FIRST][i] = g *= sh.row[DL_F][i];
  }
  __syncthreads();
  // K K^T (warps 0..3) and Q K^T (4..7), sixteen rows a warp
  {
    float c[8][4] = {};
    const int m0 = (warp & 3) * 16;
    const bool keys = warp < 4;
    dl_product<8, false, false, 1, 1, 0>(c, keys ? &sh.k[0][0] : &sh.q[0][0], DK + 8, 0, &sh.k[0][0], DK + 8, 0, m0, 0, 0, DK, lane);
    bf* P = a.p + u.unit * 3 * DL_CHUNK * DL_CHUNK;
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = m0 + (lane >> 2) + 8 * h, j = 8 * n + 2 * (lane & 3);
        float x[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int jj = j + e;
          const bool on = keys ? jj < i : jj <= i;
          x[e] = on ? c[n][2 * h + e] * sh.row[DL_RK][jj] * sh.g[i][jj] * (keys ? sh.row[DL_RK][i] * sh.row[DL_BETA][i] : sh.row[DL_RQ][i] * a.scale) : 0.f;
          if (keys) sh.a[i][jj] = x[e];
        }
        if (!keys) dl_put<3>(P + i * DL_CHUNK + j, DL_CHUNK * DL_CHUNK, x[0], x[1]);
      }
  }
  __syncthreads();
  // the inverse: blocks of 16 on the diagonal by substitution, then those below it from block to block
  if (t < DL_CHUNK) {
    const int b0 = t & ~15, j = t & 15;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < i; ++k) s = fmaf(sh.a[b0 + i][b0 + k], x[k], s);
      x[i] = i == j ? 1.f : i > j ? -s : 0.f;
      sh.t[b0 + i][b0 + j] = x[i];
    }
  }
  __syncthreads();
  const int er = t >> 4, ec = t & 15;
  for (int d = 1; d < 4; ++d) {
    for (int j = 0; j + d < 4; ++j) {
      const int i = j + d;
      float s = 0.f;
      for (int k = 16 * j; k < 16 * i; ++k) s = fmaf(sh.a[16 * i + er][k], sh.t[k][16 * j + ec], s);
      sh.tmp[j][er][ec] = s;
    }
    __syncthreads();
    for (int j = 0; j + d < 4; ++j) {
      const int i = j + d;
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < 16; ++k) s = fmaf(sh.t[16 * i + er][16 * i + k], sh.tmp[j][k][ec], s);
      sh.t[16 * i + er][16 * j + ec] = -s;
    }
    __syncthreads();
  }
  bf* tri = a.tri + u.unit * 3 * DL_CHUNK * DL_CHUNK;
  for (int i = t; i < DL_CHUNK * DL_CHUNK / 2; i += DL_THREADS) {
    const int r = i / (DL_CHUNK / 2), c = 2 * (i % (DL_CHUNK / 2));
    const bool on = c / 16 <= r / 16;
    dl_put<3>(tri + r * DL_CHUNK + c, DL_CHUNK * DL_CHUNK, on ? sh.t[r][c] : 0.f, on ? sh.t[r][c + 1] : 0.f);
  }
  float* row = a.row + u.unit * DL_ROWS * DL_CHUNK;
  for (int i = t; i < DL_ROWS * DL_CHUNK; i += DL_THREADS) row[i] = (&sh.row[0][0])[i];
}

// PARTS matrices [64][64] from the work to shared memory.
__device__ __forceinline__ void dl_load64(bf* s, const bf* g, int parts) {
  for (int i = threadIdx.x; i < parts * DL_CHUNK * 8; i += blockDim.x) {
    const int r = i >> 3, c = (i & 7) * 8;  // rows of all parts, one after the other
    *reinterpret_cast<uint4*>(s + r * DL_LD64 + c) = *reinterpret_cast<const uint4*>(g + r * DL_CHUNK + c);
  }
}

// The warps' tiles of a state [DK][DL_CB]: 16 rows, NT times 8 columns.
template <int DK>
struct DlState {
  static constexpr int MT = DK / 16, WN = 8 / MT, NT = DL_CB / 8 / WN;
  __device__ __forceinline__ static int m0(int warp) { return (warp % MT) * 16; }
  __device__ __forceinline__ static int n0(int warp) { return (warp / MT) * NT * 8; }
};

// A state's tile from or to [Dk][Dv] in memory, or zeros.
template <int DK, typename F>
__device__ __forceinline__ void dl_each(int warp, int lane, F f) {
  using St = DlState<DK>;
#pragma unroll
  for (int n = 0; n < St::NT; ++n)
#pragma unroll
    for (int h = 0; h < 2; ++h) f(n, h, St::m0(warp) + (lane >> 2) + 8 * h, St::n0(warp) + 8 * n + 2 * (lane & 3));
}

// ---- forward from chunk to chunk --------------------------------------------------------------------
template <int DK>
struct DlScanShared {
  bf k[DL_CHUNK][DK + 8], q[DL_CHUNK][DK + 8];
  bf tri[3][DL_CHUNK][DL_LD64];
  bf p[2][DL_CHUNK][DL_LD64];
  bf s[3][DK][DL_LDC];
  bf r[3][DL_CHUNK][DL_LDC];   // b (V - g K S)
  bf u[2][DL_CHUNK][DL_LDC];
  bf us[3][DL_CHUNK][DL_LDC];  // U times G_Ci / |k_i|
  float row[DL_ROWS][DL_CHUNK];
};

template <int DK>
__global__ void __launch_bounds__(DL_THREADS) delta_scan_kernel(const DlArgs a) {
  using St = DlState<DK>;
  extern __shared__ __align__(16) uint8_t dl_smem[];
  auto& sh = *reinterpret_cast<DlScanShared<DK>*>(dl_smem);
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const int blocks = (a.Dv + DL_CB - 1) / DL_CB;
  const long long n = blockIdx.x / blocks;
  const int c0 = (int)(blockIdx.x % blocks) * DL_CB, cols = min(DL_CB, a.Dv - c0);
  const long long size = (long long)a.Dk * a.Dv;
  float s[St::NT][4];
  dl_each<DK>(warp, lane, [&](int i, int h, int d, int c) {
#pragma unroll
    for (int e = 0; e < 2; ++e) s[i][2 * h + e] = a.h0 && d < a.Dk && c + e < cols ? a.h0[n * size + (long long)d * a.Dv + c0 + c + e] : 0.f;
  });
  auto store = [&](float* out) {
    dl_each<DK>(warp, lane, [&](int i, int h, int d, int c) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (d < a.Dk && c + e < cols) out[(long long)d * a.Dv + c0 + c + e] = s[i][2 * h + e];
    });
  };
  const int chunks = (a.T + DL_CHUNK - 1) / DL_CHUNK;
  const int m0 = (warp & 3) * 16, n0 = (warp >> 2) * 16;  // this warp's tile of [64][DL_CB] matrices
  for (int chunk = 0; chunk < chunks; ++chunk) {
    const DlUnit u = dl_unit(a, chunk, n);
    if (a.S) store(a.S + ((long long)chunk * a.B * a.heads + n) * size);
    if (u.live < DL_CHUNK) {  // rows behind the sequence's end
      const int steps = min(DL_CHUNK, a.T - chunk * DL_CHUNK);
      for (int i = u.live * DL_CB + t; i < steps * DL_CB; i += DL_THREADS)
        if (i % DL_CB < cols) a.Y[(u.row0 + (long long)(i / DL_CB) * a.B) * a.ldy + (long long)u.head * a.Dv + c0 + i % DL_CB] = __float2bfloat16_rn(0.f);
      if (u.live == 0) continue;
    }
    dl_load(&sh.k[0][0], DK + 8, a.K + u.row0 * a.ldk + (long long)u.head * a.Dk, a.B * a.ldk, u.live, a.Dk, DK, a.vec_k);
    dl_load(&sh.q[0][0], DK + 8, a.Q + u.row0 * a.ldq + (long long)u.head * a.Dk, a.B * a.ldq, u.live, a.Dk, DK, a.vec_q);
    dl_load64(&sh.tri[0][0][0], a.tri + u.unit * 3 * DL_CHUNK * DL_CHUNK, 3);
    dl_load64(&sh.p[0][0][0], a.p + u.unit * 3 * DL_CHUNK * DL_CHUNK, 2);
    const float* row = a.row + u.unit * DL_ROWS * DL_CHUNK;
    for (int i = t; i < DL_ROWS * DL_CHUNK; i += DL_THREADS) (&sh.row[0][0])[i] = row[i];
    dl_each<DK>(warp, lane, [&](int i, int h, int d, int c) { dl_put<3>(&sh.s[0][d][c], DK * DL_LDC, s[i][2 * h], s[i][2 * h + 1]); });
    float v[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = m0 + (lane >> 2) + 8 * h, c = n0 + 8 * i + 2 * (lane & 3) + e;
          v[i][2 * h + e] = r < u.live && c < cols ? __bfloat162float(a.V[(u.row0 + (long long)r * a.B) * a.ldv + (long long)u.head * a.Dv + c0 + c]) : 0.f;
        }
    __syncthreads();
    float o[2][4] = {};
    {
      float e[2][4] = {};
      dl_product<2, false, true, 1, 3, 2>(e, &sh.k[0][0], DK + 8, 0, &sh.s[0][0][0], DL_LDC, DK * DL_LDC, m0, n0, 0, DK, lane);
      dl_product<2, false, true, 1, 2, 1>(o, &sh.q[0][0], DK + 8, 0, &sh.s[0][0][0], DL_LDC, DK * DL_LDC, m0, n0, 0, DK, lane);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = m0 + (lane >> 2) + 8 * h, c = n0 + 8 * i + 2 * (lane & 3);
          const float b = sh.row[DL_BETA][r], g = sh.row[DL_FIRST][r] * sh.row[DL_RK][r];
          dl_put<3>(&sh.r[0][r][c], DL_CHUNK * DL_LDC, b * fmaf(-g, e[i][2 * h], v[i][2 * h]), b * fmaf(-g, e[i][2 * h + 1], v[i][2 * h + 1]));
          const float go = a.scale * sh.row[DL_FIRST][r] * sh.row[DL_RQ][r];
          o[i][2 * h] *= go;
          o[i][2 * h + 1] *= go;
        }
    }
    __syncthreads();
    {
      float x[2][4] = {};
      dl_product<2, false, true, 3, 3, 2>(x, &sh.tri[0][0][0], DL_LD64, DL_CHUNK * DL_LD64, &sh.r[0][0][0], DL_LDC, DL_CHUNK * DL_LDC, m0, n0, 0, m0 + 16, lane);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = m0 + (lane >> 2) + 8 * h, c = n0 + 8 * i + 2 * (lane & 3);
          const float g = sh.row[DL_LAST][r] * sh.row[DL_RK][r];
          dl_put<2>(&sh.u[0][r][c], DL_CHUNK * DL_LDC, x[i][2 * h], x[i][2 * h + 1]);
          dl_put<3>(&sh.us[0][r][c], DL_CHUNK * DL_LDC, g * x[i][2 * h], g * x[i][2 * h + 1]);
        }
    }
    __syncthreads();
    const float whole = sh.row[DL_FIRST][DL_CHUNK - 1];
#pragma unroll
    for (int i = 0; i < St::NT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] *= whole;
    dl_product<St::NT, true, true, 1, 3, 2>(s, &sh.k[0][0], DK + 8, 0, &sh.us[0][0][0], DL_LDC, DL_CHUNK * DL_LDC, St::m0(warp), St::n0(warp), 0, DL_CHUNK, lane);
    dl_product<2, false, true, 2, 2, 1>(o, &sh.p[0][0][0], DL_LD64, DL_CHUNK * DL_LD64, &sh.u[0][0][0], DL_LDC, DL_CHUNK * DL_LDC, m0, n0, 0, m0 + 16, lane);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = m0 + (lane >> 2) + 8 * h, c = n0 + 8 * i + 2 * (lane & 3);
        if (r >= u.live) continue;
        bf* y = a.Y + (u.row0 + (long long)r * a.B) * a.ldy + (long long)u.head * a.Dv + c0 + c;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (c + e < cols) y[e] = __float2bfloat16_rn(o[i][2 * h + e]);
      }
    __syncthreads();
  }
  if (a.hT) store(a.hT + n * size);
}

// ---- step by step -----------------------------------------------------------------------------------
// The 8 warps of a CTA hold 128 rows of a state, 16 each, a lane the columns 4 lane + k (or lane + 32 k); a step needs one meeting of the warps, for what the old
// state gives with k and with q: y = scale (f S^T q + u (k.q)).
template <bool VEC>
__global__ void __launch_bounds__(DL_THREADS) delta_steps_kernel(const DlArgs a) {
  constexpr int ROWS = 16, WARPS = DL_THREADS / 32;
  __shared__ float kq[2][2][128];       // k and q of a step, of the next one
  __shared__ float part[2][2][WARPS][128];
  __shared__ float v_s[2][128], gates[2][2], dots[2][3][4];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const long long n = blockIdx.x;
  const int b = (int)(n / a.heads), head = (int)(n - (long long)b * a.heads);
  const int len = a.lens ? min(max(a.lens[b], 0), a.T) : a.T;
  const long long size = (long long)a.Dk * a.Dv;
  auto col = [&](int k) { return VEC ? 4 * lane + k : lane + 32 * k; };
  float s[ROWS][4];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int d = warp + WARPS * i;
    if (VEC) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (a.h0 && d < a.Dk && 4 * lane < a.Dv) x = *reinterpret_cast<const float4*>(a.h0 + n * size + (long long)d * a.Dv + 4 * lane);
      s[i][0] = x.x, s[i][1] = x.y, s[i][2] = x.z, s[i][3] = x.w;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) s[i][k] = a.h0 && d < a.Dk && col(k) < a.Dv ? a.h0[n * size + (long long)d * a.Dv + col(k)] : 0.f;
    }
  }
  auto store = [&](float* out) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int d = warp + WARPS * i;
      if (d >= a.Dk) continue;
      if (VEC) {
        if (4 * lane < a.Dv) *reinterpret_cast<float4*>(out + (long long)d * a.Dv + 4 * lane) = make_float4(s[i][0], s[i][1], s[i][2], s[i][3]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (col(k) < a.Dv) out[(long long)d * a.Dv + col(k)] = s[i][k];
      }
    }
  };
  // thread t < 128 fetches k[t], q[t] and v[t] of a step
  float nk = 0.f, nq = 0.f, nv = 0.f, nf = 0.f, nb = 0.f;
  auto fetch = [&](int step) {
    const long long r = (long long)step * a.B + b;
    if (t < 128) {
      nk = t < a.Dk ? __bfloat162float(a.K[r * a.ldk + (long long)head * a.Dk + t]) : 0.f;
      nq = t < a.Dk ? __bfloat162float(a.Q[r * a.ldq + (long long)head * a.Dk + t]) : 0.f;
      nv = t < a.Dv ? __bfloat162float(a.V[r * a.ldv + (long long)head * a.Dv + t]) : 0.f;
    } else if (t == 128) {
      nf = __bfloat162float(a.Zf[r * a.ldz + head]);
      nb = __bfloat162float(a.Zb[r * a.ldz + head]);
    }
  };
  if (len > 0) fetch(0);
  for (int step = 0; step < len; ++step) {
    const int at = step & 1;
    if (a.S && step % DL_CHUNK == 0) store(a.S + ((long long)(step / DL_CHUNK) * a.B * a.heads + n) * size);
    if (t < 128) {
      kq[at][0][t] = nk;
      kq[at][1][t] = nq;
      v_s[at][t] = nv;
      float kk = nk * nk, qq = nq * nq, kx = nk * nq;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        kk += __shfl_xor_sync(0xFFFFFFFFu, kk, o);
        qq += __shfl_xor_sync(0xFFFFFFFFu, qq, o);
        kx += __shfl_xor_sync(0xFFFFFFFFu, kx, o);
      }
      if (lane == 0) dots[at][0][warp] = kk, dots[at][1][warp] = qq, dots[at][2][warp] = kx;
    } else if (t == 128) {
      float f, beta, no;
      dl_gate(nf, f, no);
      dl_gate(nb, beta, no);
      gates[at][0] = f;
      gates[at][1] = beta;
    }
    __syncthreads();
    if (step + 1 < len) fetch(step + 1);
    float sk[4] = {}, sq[4] = {};
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const float k = kq[at][0][warp + WARPS * i], q = kq[at][1][warp + WARPS * i];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        sk[c] = fmaf(s[i][c], k, sk[c]);
        sq[c] = fmaf(s[i][c], q, sq[c]);
      }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      part[at][0][warp][col(c)] = sk[c];
      part[at][1][warp][col(c)] = sq[c];
    }
    __syncthreads();
    const float kk = dots[at][0][0] + dots[at][0][1] + dots[at][0][2] + dots[at][0][3] + a.eps;
    const float qq = dots[at][1][0] + dots[at][1][1] + dots[at][1][2] + dots[at][1][3] + a.eps;
    const float kx = dots[at][2][0] + dots[at][2][1] + dots[at][2][2] + dots[at][2][3];
    const float rk = a.eps < 0.f ? 1.f : kk > 0.f ? 1.f / sqrtf(kk) : 0.f, rq = a.eps < 0.f ? 1.f : qq > 0.f ? 1.f / sqrtf(qq) : 0.f;
    const float f = gates[at][0], beta = gates[at][1];
    float u[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) x += part[at][0][w][col(c)];
      u[c] = beta * fmaf(-f * rk, x, v_s[at][col(c)]);
    }
    if (warp == (step & 7)) {  // one warp has the outputs to write, another each time
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) x += part[at][1][w][col(c)];
        if (col(c) < a.Dv)
          a.Y[((long long)step * a.B + b) * a.ldy + (long long)head * a.Dv + col(c)] = __float2bfloat16_rn(a.scale * rq * fmaf(f, x, u[c] * rk * kx));
      }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const float k = kq[at][0][warp + WARPS * i] * rk;
#pragma unroll
      for (int c = 0; c < 4; ++c) s[i][c] = fmaf(k, u[c], f * s[i][c]);
    }
  }
  for (int step = len; step < a.T; ++step)
    if (t < a.Dv) a.Y[((long long)step * a.B + b) * a.ldy + (long long)head * a.Dv + t] = __float2bfloat16_rn(0.f);
  if (a.hT) store(a.hT + n * size);
}

// ---- adjoint from chunk to chunk --------------------------------------------------------------------
template <int DK>
struct DlBackShared {
  bf k[DL_CHUNK][DK + 8], q[DL_CHUNK][DK + 8];
  bf tri[3][DL_CHUNK][DL_LD64];
  bf p[3][DL_CHUNK][DL_LD64];
  bf d[3][DK][DL_LDC];
  bf dy[DL_CHUNK][DL_LDC];
  bf du[3][DL_CHUNK][DL_LDC];
  bf w[3][DL_CHUNK][DL_LDC];   // -g / |k| b X
  bf ys[3][DL_CHUNK][DL_LDC];  // scale g / |q| dY
  float row[DL_ROWS][DL_CHUNK];
};

template <int DK>
__global__ void __launch_bounds__(DL_THREADS) delta_back_kernel(const DlArgs a) {
  using St = DlState<DK>;
  extern __shared__ __align__(16) uint8_t dl_smem[];
  auto& sh = *reinterpret_cast<DlBackShared<DK>*>(dl_smem);
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const int blocks = (a.Dv + DL_CB - 1) / DL_CB;
  const long long n = blockIdx.x / blocks;
  const int c0 = (int)(blockIdx.x % blocks) * DL_CB, cols = min(DL_CB, a.Dv - c0);
  const long long size = (long long)a.Dk * a.Dv;
  float s[St::NT][4];
  dl_each<DK>(warp, lane, [&](int i, int h, int d, int c) {
#pragma unroll
    for (int e = 0; e < 2; ++e) s[i][2 * h + e] = a.dhT && d < a.Dk && c + e < cols ? a.dhT[n * size + (long long)d * a.Dv + c0 + c + e] : 0.f;
  });
  auto store = [&](float* out) {
    dl_each<DK>(warp, lane, [&](int i, int h, int d, int c) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (d < a.Dk && c + e < cols) out[(long long)d * a.Dv + c0 + c + e] = s[i][2 * h + e];
    });
  };
  const int m0 = (warp & 3) * 16, n0 = (warp >> 2) * 16;
  for (int chunk = (a.T + DL_CHUNK - 1) / DL_CHUNK - 1; chunk >= 0; --chunk) {
    const DlUnit u = dl_unit(a, chunk, n);
    if (u.live < DL_CHUNK) {
      const int steps = min(DL_CHUNK, a.T - chunk * DL_CHUNK);
      for (int i = u.live * DL_CB + t; i < steps * DL_CB; i += DL_THREADS)
        if (i % DL_CB < cols)
          a.dV[(u.row0 + (long long)(i / DL_CB) * a.B) * a.lddv + (long long)u.head * a.Dv + c0 + i % DL_CB] = __float2bfloat16_rn(0.f);
      if (u.live == 0) continue;
    }
    store(a.d + u.unit * size);
    dl_load(&sh.k[0][0], DK + 8, a.K + u.row0 * a.ldk + (long long)u.head * a.Dk, a.B * a.ldk, u.live, a.Dk, DK, a.vec_k);
    dl_load(&sh.q[0][0], DK + 8, a.Q + u.row0 * a.ldq + (long long)u.head * a.Dk, a.B * a.ldq, u.live, a.Dk, DK, a.vec_q);
    dl_load(&sh.dy[0][0], DL_LDC, a.dY + u.row0 * a.lddy + (long long)u.head * a.Dv + c0, a.B * a.lddy, u.live, cols, DL_CB, a.vec_dy);
    dl_load64(&sh.tri[0][0][0], a.tri + u.unit * 3 * DL_CHUNK * DL_CHUNK, 3);
    dl_load64(&sh.p[0][0][0], a.p + u.unit * 3 * DL_CHUNK * DL_CHUNK, 3);
    const float* row = a.row + u.unit * DL_ROWS * DL_CHUNK;
    for (int i = t; i < DL_ROWS * DL_CHUNK; i += DL_THREADS) (&sh.row[0][0])[i] = row[i];
    dl_each<DK>(warp, lane, [&](int i, int h, int d, int c) { dl_put<3>(&sh.d[0][d][c], DK * DL_LDC, s[i][2 * h], s[i][2 * h + 1]); });
    __syncthreads();
    {
      float f[2][4] = {}, g[2][4] = {};
      dl_product<2, false, true, 1, 3, 2>(f, &sh.k[0][0], DK + 8, 0, &sh.d[0][0][0], DL_LDC, DK * DL_LDC, m0, n0, 0, DK, lane);
      dl_product<2, true, true, 3, 1, 2>(g, &sh.p[0][0][0], DL_LD64, DL_CHUNK * DL_LD64, &sh.dy[0][0], DL_LDC, 0, m0, n0, m0, DL_CHUNK, lane);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = m0 + (lane >> 2) + 8 * h, c = n0 + 8 * i + 2 * (lane & 3);
          const float l = sh.row[DL_LAST][r] * sh.row[DL_RK][r];
          dl_put<3>(&sh.du[0][r][c], DL_CHUNK * DL_LDC, fmaf(l, f[i][2 * h], g[i][2 * h]), fmaf(l, f[i][2 * h + 1], g[i][2 * h + 1]));
          const float2 dy = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&sh.dy[r][c]));
          const float gq = a.scale * sh.row[DL_FIRST][r] * sh.row[DL_RQ][r];
          dl_put<3>(&sh.ys[0][r][c], DL_CHUNK * DL_LDC, gq * dy.x, gq * dy.y);
        }
    }
    __syncthreads();
    {
      float x[2][4] = {};
      dl_product<2, true, true, 3, 3, 2>(x, &sh.tri[0][0][0], DL_LD64, DL_CHUNK * DL_LD64, &sh.du[0][0][0], DL_LDC, DL_CHUNK * DL_LDC, m0, n0, m0, DL_CHUNK, lane);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = m0 + (lane >> 2) + 8 * h, c = n0 + 8 * i + 2 * (lane & 3);
          const float beta = sh.row[DL_BETA][r], g = -sh.row[DL_FIRST][r] * sh.row[DL_RK][r] * beta;
          dl_put<3>(&sh.w[0][r][c], DL_CHUNK * DL_LDC, g * x[i][2 * h], g * x[i][2 * h + 1]);
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (c + e < cols) {
              a.x[(u.unit * DL_CHUNK + r) * a.Dv + c0 + c + e] = x[i][2 * h + e];
              if (r < u.live)
                a.dV[(u.row0 + (long long)r * a.B) * a.lddv + (long long)u.head * a.Dv + c0 + c + e] = __float2bfloat16_rn(beta * x[i][2 * h + e]);
            }
        }
    }
    __syncthreads();
    const float whole = sh.row[DL_FIRST][DL_CHUNK - 1];
#pragma unroll
    for (int i = 0; i < St::NT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] *= whole;
    dl_product<St::NT, true, true, 1, 3, 2>(s, &sh.q[0][0], DK + 8, 0, &sh.ys[0][0][0], DL_LDC, DL_CHUNK * DL_LDC, St::m0(warp), St::n0(warp), 0, DL_CHUNK, lane);
    dl_product<St::NT, true, true, 1, 3, 2>(s, &sh.k[0][0], DK + 8, 0, &sh.w[0][0][0], DL_LDC, DL_CHUNK * DL_LDC, St::m0(warp), St::n0(warp), 0, DL_CHUNK, lane);
    __syncthreads();
  }
  if (a.dh0) store(a.dh0 + n * size);
}

// ---- a chunk's own gradients ------------------------------------------------------------------------
// With U again from the state that the forward call left, and o the products of entries,
//   N = scale G o (dY U^T) (j <= i),  M = -b G o (X U^T) (j < i),
//   dQ = scale g dY S_0^T + N K,  dK = N^T Q + (M + M^T) K - g b X S_0^T + G_C U D^T,  dZb = X.U (1 - b),
//   d log f_t = sum over the chunk's steps from t on of (q.dq - v.dv) + <D, S_C>,  S_C = g_C S_0 + (G_C K)^T U,
// for q and k divided by their lengths, then dq / |q| without its part along q.  (d log f: what scales the state by f scales what later queries read of it, less
// what the later values would have replaced; starting from <D, S_C> in every chunk keeps the sums short.)
constexpr int DL_GRAD_THREADS = 512;

template <int DK, int DV>
struct DlGradShared {
  bf k[DL_CHUNK][DK + 8], q[DL_CHUNK][DK + 8];
  bf dy[DL_CHUNK][DV + 8];
  bf x[2][DL_CHUNK][DV + 8];
  bf u[2][DL_CHUNK][DV + 8];   // b (V - g K S), then U
  union {
    bf s[2][DK][DV + 8];       // the state in front of the chunk, then the gradient D of that behind it
    bf m[3][2][DL_CHUNK][DL_LD64];  // N / |k_j|, N / |q_i|, (M + M^T) / |k_j|
  };
  bf tri[2][DL_CHUNK][DL_LD64];
  float g[DL_CHUNK][DL_CHUNK + 1];
  float row[DL_ROWS][DL_CHUNK];
  float red[3][4][DL_CHUNK];   // sums over a row, by groups of columns: q.dq, k.dk, k.(U D^T)
  float xu[DL_CHUNK], xv[DL_CHUNK];
  float ds[DL_GRAD_THREADS / 32];
};

// [rows][cols] fp32 without gaps to two bf16 parts in shared memory; the rest of [pad_rows][pad_cols] becomes zeros.
__device__ __forceinline__ void dl_load_f32(bf* s, int ld, int stride, const float* g, int rows, int cols, int pad_rows, int pad_cols, const float* with, float* dot) {
  const int pairs = pad_cols / 2;
  for (int i = threadIdx.x; i < pad_rows * pairs; i += blockDim.x) {
    const int r = i / pairs, c = 2 * (i - r * pairs);
    float x[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (r < rows && c + e < cols) {
        x[e] = g[(long long)r * cols + c + e];
        if (with) *dot = fmaf(x[e], with[(long long)r * cols + c + e], *dot);
      }
    dl_put<2>(s + r * ld + c, stride, x[0], x[1]);
  }
}
__device__ __forceinline__ void dl_store2(bf* p, float x, float y, bool two) {
  if (two && (reinterpret_cast<uintptr_t>(p) & 3u) == 0) {
    *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(x, y);
  } else {
    p[0] = __float2bfloat16_rn(x);
    if (two) p[1] = __float2bfloat16_rn(y);
  }
}

template <int DK, int DV>
__global__ void __launch_bounds__(DL_GRAD_THREADS) delta_grad_kernel(const DlArgs a) {
  constexpr int NK = DK / 32, NV = DV / 32;  // tiles of 8 columns a warp of [64][DK] and [64][DV] matrices
  constexpr int LDK = DK + 8, LDV = DV + 8, PV = DL_CHUNK * LDV, PM = DL_CHUNK * DL_LD64;
  extern __shared__ __align__(16) uint8_t dl_smem[];
  auto& sh = *reinterpret_cast<DlGradShared<DK, DV>*>(dl_smem);
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const long long units = (long long)a.B * a.heads;
  const DlUnit u = dl_unit(a, (int)(blockIdx.x / units), blockIdx.x % units);
  const int steps = min(DL_CHUNK, a.T - u.chunk * DL_CHUNK);
  bf* dq = a.dQ + u.row0 * a.lddq + (long long)u.head * a.Dk;
  bf* dk = a.dK + u.row0 * a.lddk + (long long)u.head * a.Dk;
  for (int i = u.live * DK + t; i < steps * DK; i += DL_GRAD_THREADS) {  // rows behind the sequence's end
    const int r = i / DK, c = i % DK;
    if (c >= a.Dk) continue;
    dq[(long long)r * a.B * a.lddq + c] = __float2bfloat16_rn(0.f);
    dk[(long long)r * a.B * a.lddk + c] = __float2bfloat16_rn(0.f);
  }
  if (t >= u.live && t < steps) {
    const long long z = (u.row0 + (long long)t * a.B) * a.lddz + u.head;
    a.dZf[z] = a.dZb[z] = __float2bfloat16_rn(0.f);
  }
  if (u.live == 0) return;
  const long long size = (long long)a.Dk * a.Dv;
  const float* S0 = a.S + u.unit * size;
  dl_load(&sh.k[0][0], LDK, a.K + u.row0 * a.ldk + (long long)u.head * a.Dk, a.B * a.ldk, u.live, a.Dk, DK, a.vec_k);
  dl_load(&sh.q[0][0], LDK, a.Q + u.row0 * a.ldq + (long long)u.head * a.Dk, a.B * a.ldq, u.live, a.Dk, DK, a.vec_q);
  dl_load(&sh.dy[0][0], LDV, a.dY + u.row0 * a.lddy + (long long)u.head * a.Dv, a.B * a.lddy, u.live, a.Dv, DV, a.vec_dy);
  dl_load64(&sh.tri[0][0][0], a.tri + u.unit * 3 * DL_CHUNK * DL_CHUNK, 2);
  for (int i = t; i < DL_ROWS * DL_CHUNK; i += DL_GRAD_THREADS) (&sh.row[0][0])[i] = a.row[u.unit * DL_ROWS * DL_CHUNK + i];
  dl_load_f32(&sh.s[0][0][0], LDV, DK * LDV, S0, a.Dk, a.Dv, DK, DV, nullptr, nullptr);
  dl_load_f32(&sh.x[0][0][0], LDV, PV, a.x + u.unit * DL_CHUNK * a.Dv, DL_CHUNK, a.Dv, DL_CHUNK, DV, nullptr, nullptr);
  __syncthreads();
  if (t < DL_CHUNK) {
    float g = 1.f;
    for (int i = 0; i < t; ++i) sh.g[i][t] = 0.f;
    sh.g[t][t] = 1.f;
    for (int i = t + 1; i < DL_CHUNK; ++i) sh.g[i][t] = g *= sh.row[DL_F][i];
  }
  const int m0 = (warp & 3) * 16, group = warp >> 2;
  const int nk0 = group * NK * 8, nv0 = group * NV * 8, nm0 = group * 16;  // this warp's columns
  const int r0 = m0 + (lane >> 2), cl = 2 * (lane & 3);
  auto v_at = [&](int r, int c) { return r < u.live && c < a.Dv ? __bfloat162float(a.V[(u.row0 + (long long)r * a.B) * a.ldv + (long long)u.head * a.Dv + c]) : 0.f; };
  float aq[NK][4] = {}, ak[NK][4] = {};
  {
    float e[NV][4] = {};
    dl_product<NV, false, true, 1, 2, 1>(e, &sh.k[0][0], LDK, 0, &sh.s[0][0][0], LDV, DK * LDV, m0, nv0, 0, DK, lane);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = r0 + 8 * h, c = nv0 + 8 * i + cl;
        const float b = sh.row[DL_BETA][r], g = sh.row[DL_FIRST][r] * sh.row[DL_RK][r];
        dl_put<2>(&sh.u[0][r][c], PV, b * fmaf(-g, e[i][2 * h], v_at(r, c)), b * fmaf(-g, e[i][2 * h + 1], v_at(r, c + 1)));
      }
  }
  dl_product<NK, false, false, 1, 2, 1>(aq, &sh.dy[0][0], LDV, 0, &sh.s[0][0][0], LDV, DK * LDV, m0, nk0, 0, DV, lane);
  dl_product<NK, false, false, 2, 2, 1>(ak, &sh.x[0][0][0], LDV, PV, &sh.s[0][0][0], LDV, DK * LDV, m0, nk0, 0, DV, lane);
#pragma unroll
  for (int i = 0; i < NK; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float g = sh.row[DL_FIRST][r0 + 8 * (e >> 1)];
      aq[i][e] *= a.scale * g;
      ak[i][e] *= -g * sh.row[DL_BETA][r0 + 8 * (e >> 1)];
    }
  __syncthreads();
  {
    float x[NV][4] = {};
    dl_product<NV, false, true, 2, 2, 1>(x, &sh.tri[0][0][0], DL_LD64, PM, &sh.u[0][0][0], LDV, PV, m0, nv0, 0, m0 + 16, lane);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) dl_put<2>(&sh.u[0][r0 + 8 * h][nv0 + 8 * i + cl], PV, x[i][2 * h], x[i][2 * h + 1]);
  }
  // the gradient of the state behind the chunk, where the state in front of it was
  float dot = 0.f;
  dl_load_f32(&sh.s[0][0][0], LDV, DK * LDV, a.d + u.unit * size, a.Dk, a.Dv, DK, DV, S0, &dot);
  dot = [&] {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, o);
    return dot;
  }();
  if (lane == 0) sh.ds[warp] = dot;
  __syncthreads();
  {  // X.U and X.V: eight threads a row
    const int r = t >> 3, part = t & 7;
    float xu = 0.f, xv = 0.f;
    for (int c = part * 2; c < DV; c += 16) {
      float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&sh.x[0][r][c])), xl = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&sh.x[1][r][c]));
      const float2 y = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&sh.u[0][r][c])), yl = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&sh.u[1][r][c]));
      x.x += xl.x, x.y += xl.y;
      xu = fmaf(x.x, y.x + yl.x, fmaf(x.y, y.y + yl.y, xu));
      xv = fmaf(x.x, v_at(r, c), fmaf(x.y, v_at(r, c + 1), xv));
    }
#pragma unroll
    for (int o = 1; o < 8; o *= 2) {
      xu += __shfl_xor_sync(0xFFFFFFFFu, xu, o);
      xv += __shfl_xor_sync(0xFFFFFFFFu, xv, o);
    }
    if (part == 0) sh.xu[r] = xu, sh.xv[r] = xv * sh.row[DL_BETA][r];
  }
  float nn[2][4] = {}, mm[2][4] = {};
  if (nm0 <= m0) {
    dl_product<2, false, false, 1, 2, 1>(nn, &sh.dy[0][0], LDV, 0, &sh.u[0][0][0], LDV, PV, m0, nm0, 0, DV, lane);
    dl_product<2, false, false, 2, 2, 1>(mm, &sh.x[0][0][0], LDV, PV, &sh.u[0][0][0], LDV, PV, m0, nm0, 0, DV, lane);
  }
  auto row_sums = [&](int which, const float (&x)[NK][4], const bf* with, int scaled) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const float2 w = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(with + (r0 + 8 * h) * LDK + nk0 + 8 * i + cl));
        s = fmaf(x[i][2 * h], w.x, fmaf(x[i][2 * h + 1], w.y, s));
      }
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 1);
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 2);
      if ((lane & 3) == 0) sh.red[which][group][r0 + 8 * h] = s * sh.row[scaled][r0 + 8 * h];
    }
  };
  {
    float x[NK][4] = {};
    dl_product<NK, false, false, 2, 2, 1>(x, &sh.u[0][0][0], LDV, PV, &sh.s[0][0][0], LDV, DK * LDV, m0, nk0, 0, DV, lane);
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[i][e] *= sh.row[DL_LAST][r0 + 8 * (e >> 1)];
        ak[i][e] += x[i][e];
      }
    row_sums(2, x, &sh.k[0][0], DL_RK);
  }
  __syncthreads();
  if (nm0 <= m0) {
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = r0 + 8 * h, j = nm0 + 8 * n + cl;
        const float g0 = sh.g[i][j], g1 = sh.g[i][j + 1];  // zero above the diagonal
        const float x = a.scale * g0 * nn[n][2 * h], y = a.scale * g1 * nn[n][2 * h + 1];
        dl_put<2>(&sh.m[0][0][i][j], PM, x * sh.row[DL_RK][j], y * sh.row[DL_RK][j + 1]);
        dl_put<2>(&sh.m[1][0][i][j], PM, x * sh.row[DL_RQ][i], y * sh.row[DL_RQ][i]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int jj = j + e;
          if (jj > i) continue;
          const float z = jj < i ? -sh.row[DL_BETA][i] * (e ? g1 : g0) * mm[n][2 * h + e] : 0.f;
          float lo = z * sh.row[DL_RK][jj], up = z * sh.row[DL_RK][i];
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            const bf bl = __float2bfloat16_rn(lo), bu = __float2bfloat16_rn(up);
            sh.m[2][part][i][jj] = bl;
            sh.m[2][part][jj][i] = bu;
            lo -= __bfloat162float(bl);
            up -= __bfloat162float(bu);
          }
        }
      }
  }
  __syncthreads();
  dl_product<NK, false, true, 2, 1, 1>(aq, &sh.m[0][0][0][0], DL_LD64, PM, &sh.k[0][0], LDK, 0, m0, nk0, 0, m0 + 16, lane);
  dl_product<NK, true, true, 2, 1, 1>(ak, &sh.m[1][0][0][0], DL_LD64, PM, &sh.q[0][0], LDK, 0, m0, nk0, m0, DL_CHUNK, lane);
  dl_product<NK, false, true, 2, 1, 1>(ak, &sh.m[2][0][0][0], DL_LD64, PM, &sh.k[0][0], LDK, 0, m0, nk0, 0, DL_CHUNK, lane);
  row_sums(0, aq, &sh.q[0][0], DL_RQ);
  row_sums(1, ak, &sh.k[0][0], DL_RK);
  __syncthreads();
  auto red = [&](int which, int r) { return (sh.red[which][0][r] + sh.red[which][1][r]) + (sh.red[which][2][r] + sh.red[which][3][r]); };
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = r0 + 8 * h;
    if (r >= u.live) continue;
    const float rq = sh.row[DL_RQ][r], rk = sh.row[DL_RK][r];
    // q of length one gives up what its gradient has along it
    const float along_q = a.eps < 0.f ? 0.f : red(0, r) * rq, along_k = a.eps < 0.f ? 0.f : red(1, r) * rk;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int c = nk0 + 8 * i + cl;
      if (c >= a.Dk) continue;
      const float2 q = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&sh.q[r][c])), k = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&sh.k[r][c]));
      dl_store2(dq + (long long)r * a.B * a.lddq + c, rq * fmaf(-along_q, q.x, aq[i][2 * h]), rq * fmaf(-along_q, q.y, aq[i][2 * h + 1]), c + 1 < a.Dk);
      dl_store2(dk + (long long)r * a.B * a.lddk + c, rk * fmaf(-along_k, k.x, ak[i][2 * h]), rk * fmaf(-along_k, k.y, ak[i][2 * h + 1]), c + 1 < a.Dk);
    }
  }
  if (warp == 0) {  // lane: steps lane and 32 + lane
    float ds = 0.f;
#pragma unroll
    for (int w = 0; w < DL_GRAD_THREADS / 32; ++w) ds += sh.ds[w];
    float x0 = red(0, lane) - sh.xv[lane], x1 = red(0, 32 + lane) - sh.xv[32 + lane], end = red(2, lane) + red(2, 32 + lane);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) end += __shfl_xor_sync(0xFFFFFFFFu, end, o);
    end = fmaf(sh.row[DL_FIRST][DL_CHUNK - 1], ds, end);
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const float y0 = __shfl_down_sync(0xFFFFFFFFu, x0, o), y1 = __shfl_down_sync(0xFFFFFFFFu, x1, o);
      if (lane + o < 32) x0 += y0, x1 += y1;
    }
    x0 += __shfl_sync(0xFFFFFFFFu, x1, 0);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = lane + 32 * h;
      if (r >= u.live) continue;
      const long long z = (u.row0 + (long long)r * a.B) * a.lddz + u.head;
      a.dZf[z] = __float2bfloat16_rn(((h ? x1 : x0) + end) * sh.row[DL_REST][r]);
      a.dZb[z] = __float2bfloat16_rn(sh.xu[r] * (1.f - sh.row[DL_BETA][r]));
    }
  }
}

constexpr int DL_STEPS = 16;  // up to so many steps go one by one

inline bool dl_on16(const void* p, long long ld, int head) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && head % 8 == 0; }
inline long long dl_units(int T, int B, int heads) { return (long long)((T + DL_CHUNK - 1) / DL_CHUNK) * B * heads; }

// Where a unit's parts lie in the work, in bytes from its start (all units of a kind side by side, each on 256 bytes).
struct DlPlan {
  size_t tri, p, row, x, d, bytes;
};
DlPlan dl_plan(int T, int B, int heads, int Dk, int Dv, bool backward) {
  const size_t units = (size_t)dl_units(T, B, heads);
  DlPlan w;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (units * bytes + 255) / 256 * 256;
    return here;
  };
  w.tri = take(3 * DL_CHUNK * DL_CHUNK * 2);
  w.p = take(3 * DL_CHUNK * DL_CHUNK * 2);
  w.row = take(DL_ROWS * DL_CHUNK * 4);
  w.x = take(backward ? (size_t)DL_CHUNK * Dv * 4 : 0);
  w.d = take(backward ? (size_t)Dk * Dv * 4 : 0);
  w.bytes = at + 256;  // the caller's memory may begin anywhere
  return w;
}
void dl_set_work(DlArgs& a, void* work, const DlPlan& w) {
  uint8_t* p = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(work) + 255) & ~(uintptr_t)255);
  a.tri = reinterpret_cast<bf*>(p + w.tri);
  a.p = reinterpret_cast<bf*>(p + w.p);
  a.row = reinterpret_cast<float*>(p + w.row);
  a.x = reinterpret_cast<float*>(p + w.x);
  a.d = reinterpret_cast<float*>(p + w.d);
}

template <int DK>
ard_status dl_prep(ard_ctx* ctx, const DlArgs& a, cudaStream_t s) {
  const int smem = (int)sizeof(DlPrepShared<DK>);
  ARD_CUDA_OK(cudaFuncSetAttribute(delta_prep_kernel<DK>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  ARD_CUDA_OK(ard_launch(ctx, delta_prep_kernel<DK>, dim3((unsigned)dl_units(a.T, a.B, a.heads)), dim3(DL_THREADS), smem, s, a));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}
template <int DK>
ard_status dl_forward(ard_ctx* ctx, const DlArgs& a, cudaStream_t s) {
  const ard_status st = dl_prep<DK>(ctx, a, s);
  if (st != ARD_OK) return st;
  const int smem = (int)sizeof(DlScanShared<DK>);
  const long long grid = (long long)a.B * a.heads * ((a.Dv + DL_CB - 1) / DL_CB);
  ARD_CUDA_OK(cudaFuncSetAttribute(delta_scan_kernel<DK>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  ARD_CUDA_OK(ard_launch(ctx, delta_scan_kernel<DK>, dim3((unsigned)grid), dim3(DL_THREADS), smem, s, a));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}

template <int DK>
ard_status dl_backward(ard_ctx* ctx, const DlArgs& a, cudaStream_t s) {
  const ard_status st = dl_prep<DK>(ctx, a, s);
  if (st != ARD_OK) return st;
  const int smem = (int)sizeof(DlBackShared<DK>);
  const long long grid = (long long)a.B * a.heads * ((a.Dv + DL_CB - 1) / DL_CB);
  ARD_CUDA_OK(cudaFuncSetAttribute(delta_back_kernel<DK>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  ARD_CUDA_OK(ard_launch(ctx, delta_back_kernel<DK>, dim3((unsigned)grid), dim3(DL_THREADS), smem, s, a));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  auto grad = [&](auto kern, int bytes) {
    ARD_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    ARD_CUDA_OK(ard_launch(ctx, kern, dim3((unsigned)dl_units(a.T, a.B, a.heads)), dim3(DL_GRAD_THREADS), bytes, s, a));
    ctx->launches++;
    ARD_CUDA_OK(cudaGetLastError());
    return ARD_OK;
  };
  if (a.Dv <= 64) return grad(delta_grad_kernel<DK, 64>, (int)sizeof(DlGradShared<DK, 64>));
  return grad(delta_grad_kernel<DK, 128>, (int)sizeof(DlGradShared<DK, 128>));
}

static_assert(sizeof(DlGradShared<128, 128>) <= 227 * 1024 && sizeof(DlBackShared<128>) <= 227 * 1024 && sizeof(DlScanShared<128>) <= 227 * 1024, "shared memory of an SM");

}  // namespace

size_t delta_work_bytes(int T, int B, int heads, int Dk, int Dv, bool backward) {
  if (T == 0 || B == 0 || heads == 0 || Dk == 0 || Dv == 0 || (!backward && T <= DL_STEPS)) return 0;
  return dl_plan(T, B, heads, Dk, Dv, backward).bytes;
}

ard_status launch_delta_forward(ard_ctx* ctx, int T, int B, int heads, int Dk, int Dv, float scale, float eps, const void* Q, int ldq, const void* K, int ldk,
                                const void* V, int ldv, const void* Zf, const void* Zb, int ldz, const int32_t* lens, const float* h0, void* Y, int ldy,
                                float* hT, float* S, void* work, cudaStream_t s) {
  if (B == 0 || heads == 0 || Dv == 0 || Dk == 0) return ARD_OK;
  DlArgs a = {};
  a.T = T, a.B = B, a.heads = heads, a.Dk = Dk, a.Dv = Dv, a.scale = scale, a.eps = eps;
  a.Q = (const bf*)Q, a.K = (const bf*)K, a.V = (const bf*)V, a.ldq = ldq, a.ldk = ldk, a.ldv = ldv;
  a.Zf = (const bf*)Zf, a.Zb = (const bf*)Zb, a.ldz = ldz;
  a.lens = lens, a.h0 = h0, a.Y = (bf*)Y, a.ldy = ldy, a.hT = hT, a.S = S;
  a.vec_q = dl_on16(Q, ldq, Dk), a.vec_k = dl_on16(K, ldk, Dk);
  if (T <= DL_STEPS) {
    auto on16 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
    const bool vec = Dv % 4 == 0 && on16(h0) && on16(hT) && on16(S);
    ARD_CUDA_OK(ard_launch(ctx, vec ? delta_steps_kernel<true> : delta_steps_kernel<false>, dim3((unsigned)((long long)B * heads)), dim3(DL_THREADS), 0, s, a));
    ctx->launches++;
    ARD_CUDA_OK(cudaGetLastError());
    return ARD_OK;
  }
  dl_set_work(a, work, dl_plan(T, B, heads, Dk, Dv, false));
  return Dk <= 64 ? dl_forward<64>(ctx, a, s) : dl_forward<128>(ctx, a, s);
}

ard_status launch_delta_backward(ard_ctx* ctx, int T, int B, int heads, int Dk, int Dv, float scale, float eps, const void* Q, int ldq, const void* K, int ldk,
                                 const void* V, int ldv, const void* Zf, const void* Zb, int ldz, const int32_t* lens, const float* S, const void* dY,
                                 int lddy, const float* dhT, void* dQ, int lddq, void* dK, int lddk, void* dV, int lddv, void* dZf, void* dZb, int lddz,
                                 float* dh0, void* work, cudaStream_t s) {
  if (B == 0 || heads == 0 || Dv == 0 || Dk == 0) return ARD_OK;
  if (T == 0) {
    const size_t bytes = (size_t)B * heads * Dk * Dv * 4;
    if (dh0 && dhT && dh0 != dhT) ARD_CUDA_OK(cudaMemcpyAsync(dh0, dhT, bytes, cudaMemcpyDeviceToDevice, s));
    if (dh0 && !dhT) ARD_CUDA_OK(cudaMemsetAsync(dh0, 0, bytes, s));
    return ARD_OK;
  }
  DlArgs a = {};
  a.T = T, a.B = B, a.heads = heads, a.Dk = Dk, a.Dv = Dv, a.scale = scale, a.eps = eps;
  a.Q = (const bf*)Q, a.K = (const bf*)K, a.V = (const bf*)V, a.ldq = ldq, a.ldk = ldk, a.ldv = ldv;
  a.Zf = (const bf*)Zf, a.Zb = (const bf*)Zb, a.ldz = ldz;
  a.lens = lens, a.S = const_cast<float*>(S);
  a.dY = (const bf*)dY, a.lddy = lddy, a.dhT = dhT;
  a.dQ = (bf*)dQ, a.dK = (bf*)dK, a.dV = (bf*)dV, a.lddq = lddq, a.lddk = lddk, a.lddv = lddv;
  a.dZf = (bf*)dZf, a.dZb = (bf*)dZb, a.lddz = lddz, a.dh0 = dh0;
  a.vec_q = dl_on16(Q, ldq, Dk), a.vec_k = dl_on16(K, ldk, Dk), a.vec_dy = dl_on16(dY, lddy, Dv);
  dl_set_work(a, work, dl_plan(T, B, heads, Dk, Dv, true));
  return Dk <= 64 ? dl_backward<64>(ctx, a, s) : dl_backward<128>(ctx, a, s);
}
