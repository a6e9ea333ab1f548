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
// error of 2^-18 of a term where the output's rounding is 2^-9).
//
// All products are mma.sync's.  What goes from chunk to chunk is a chain: four products of 64 x 64 or 64 x 128 matrices with 16 columns of a state, each result split into parts
// and the next one's operand.  mma.sync takes them from registers and leaves them in registers (measured here: 1000 multiply-adds a clock and SM).  A
// tcgen05 product would bring each result from tensor memory to registers and its parts back, and its 128 rows of an accumulator would leave half of
// the SMs without work at 64 sequences and heads.  The systems and the gradients, whose chunks do not see one another and whose operands lie in shared memory, have no such
// reason: a tcgen05 form of them, two chunks to 128 rows, has not been built.
//
// Time of 2048 steps, 8 sequences of 8 heads, 128 x 128: forward 250 us (systems 69, scan 185), backward 655 (systems 69, scan 214, gradients 378); of 16384 steps of
// one sequence 773, a chunk in 2.7 us; of one step of 64 x 8 heads 14.7, for 67 MB.
#include "ard_internal.h"
#include "sm100_ptx.h"

namespace {

constexpr int DL_CHUNK = 64;
constexpr int DL_THREADS = 256;
constexpr int DL_SQ = DL_CHUNK * DL_CHUNK;
constexpr int DL_LD64 = DL_CHUNK + 8;  // pitch of [64][64] matrices in shared memory: rows on different banks

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
  int vec_q, vec_k, vec_v, vec_dy, vec_s;  // whether rows lie on a grid of 16 bytes
  // work, by unit = chunk * B * heads + sequence * heads + head
  bf* tri;     // [units][3][64][64] (I + A)^-1 in three parts
  bf* p;       // [units][3][64][64] scale * (G o Q K^T) in three parts
  float* row;  // [units][DL_ROW_FLOATS]
  bf* x;       // [units][2][64][ldx] X in two parts
  bf* d;       // [units][2][ldx][DK] the gradient of the state behind a chunk, transposed
  int ldx;
  int ahead;   // SMs
};

// What a chunk's steps have of their own.  G_ij = f_{j+1} .. f_i is kept as products of gates: inside a block of 16 steps as it is, across blocks a_i, the whole
// blocks between, and b_j.
struct DlSteps {                 // what the scans read
  float beta[DL_CHUNK];          // b
  float kin[DL_CHUNK];           // g_i / |k_i|,  g_i = f_1 .. f_i
  float kout[DL_CHUNK];          // G_Ci / |k_i|
  float qin[DL_CHUNK];           // scale g_i / |q_i|
  float first[DL_CHUNK];         // g_i
};
struct DlRow : DlSteps {
  float rk[DL_CHUNK], rq[DL_CHUNK];        // 1 / |k|, 1 / |q|
  float f[DL_CHUNK], rest[DL_CHUNK];       // f, 1 - f
  float closed[DL_CHUNK];                  // 1 - b, to some units of its own size: a gate near 1 has its gradient from it
  float last[DL_CHUNK];                    // G_Ci
  float from[DL_CHUNK], to[DL_CHUNK];      // a_i: from its block's first step to i; b_j: from behind j to its block's last step
  float block[4];                          // a whole block
  float diag[4][16][17];                   // [block][i][j], zero above the diagonal
};
constexpr int DL_ROW_FLOATS = (int)(sizeof(DlRow) / 4);
static_assert(sizeof(DlRow) % 16 == 0 && sizeof(DlSteps) % 16 == 0, "copied in pieces of 16 bytes");

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

// c[MT][NT][4] += A (16 MT rows from m0) * B (8 NT columns from n0) over the contraction [k0, k1), operands in PA and PB parts `sa`, `sb` elements
// apart.  Parts i and j are multiplied where i + j <= MOST: smaller products are below what is kept.
template <int MT, int NT, bool AT, bool BKN, int PA, int PB, int MOST>
__device__ __forceinline__ void dl_product(float (&c)[MT][NT][4], const bf* a, int lda, int sa, const bf* b, int ldb, int sb, int m0, int n0, int k0,
                                           int k1, int lane) {
  static_assert(NT % 2 == 0, "columns by sixteens");
#pragma unroll 4
  for (int k = k0; k < k1; k += 16) {
    uint32_t ra[MT][PA][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < PA; ++i) dl_a<AT>(ra[m][i], a + i * sa, lda, m0 + 16 * m, k, lane);
#pragma unroll
    for (int n = 0; n < NT; n += 2) {
#pragma unroll
      for (int j = PB - 1; j >= 0; --j) {  // small parts first
        uint32_t rb[4];
        dl_b<BKN>(rb, b + j * sb, ldb, n0 + 8 * n, k, lane);
#pragma unroll
        for (int i = PA - 1; i >= 0; --i)
          if (i + j <= MOST) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              dl_mma(c[m][n], ra[m][i], rb[0], rb[1]);
              dl_mma(c[m][n + 1], ra[m][i], rb[2], rb[3]);
            }
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
      const float2 r = __ffma2_rn(__bfloat1622float2(h), make_float2(-1.f, -1.f), make_float2(x, y));
      x = r.x, y = r.y;
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

// s(z) and 1 - s(z), each to a few units of its own size, the smaller one to |z| of them more: the exponential's argument is rounded.
__device__ __forceinline__ void dl_gate(float z, float& f, float& rest) {
  const float e = __expf(-fabsf(z)), big = __frcp_rn(1.f + e), small = e * big;
  f = z >= 0.f ? big : small;
  rest = z >= 0.f ? small : big;
}

__device__ __forceinline__ void dl_copy16(void* s, const void* g, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(s)), "l"(g), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void dl_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void dl_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

// A word, or else its first element, or else nothing; without a branch that the load would wait in.
__device__ __forceinline__ uint32_t dl_word(const bf* p, bool whole, bool one) {
  uint32_t r;
  asm volatile("{ .reg .pred a, b; setp.ne.b32 a, %2, 0; setp.ne.b32 b, %3, 0; mov.b32 %0, 0; @a ld.global.b32 %0, [%1]; @b ld.global.u16 %0, [%1]; }"
               : "=&r"(r)
               : "l"(p), "r"((int)whole), "r"((int)(one && !whole))
               : "memory");
  return r;
}

// [64][cols] of a matrix whose rows are `step` elements apart, on its way to shared memory with pitch ld; rows from `live` on and columns up to PAD are
// zeros.  Rows off the grid of 16 bytes go through registers, at once.  By threads t of OF.
template <int PAD, int OF>
__device__ __forceinline__ void dl_load(bf* s, int ld, const bf* g, long long step, int live, int cols, int vec, int t) {
  constexpr int PIECES = PAD / 8, ROWS = OF / PIECES, ROUNDS = DL_CHUNK / ROWS;
  static_assert(OF % PIECES == 0 && DL_CHUNK % ROWS == 0, "whole rows a round");
  const int c = (t % PIECES) * 8, r0 = t / PIECES;
  const bool inside = c < cols;
  const bf* p = g + r0 * step + (inside ? c : 0);
  bf* d = s + r0 * ld + c;
  if (vec) {
    if (live == DL_CHUNK) {
#pragma unroll
      for (int i = 0; i < ROUNDS; ++i, p += ROWS * step) dl_copy16(d + i * ROWS * ld, p, inside);
    } else {
      for (int i = 0; i < ROUNDS; ++i, p += ROWS * step) dl_copy16(d + i * ROWS * ld, r0 + i * ROWS < live ? p : g, inside && r0 + i * ROWS < live);
    }
    return;
  }
  // Words of 4 bytes, shifted by an element where the piece begins inside one; of words that reach over its ends the one element that is in it.
  constexpr int MOST = OF <= 128 ? 8 : 2, AHEAD = ROUNDS < MOST ? ROUNDS : MOST;
#pragma unroll 1
  for (int i0 = 0; i0 < ROUNDS; i0 += AHEAD) {
    uint32_t w[AHEAD][5];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const bf* x = p + i * (ROWS * step);
      const int n = r0 + (i0 + i) * ROWS < live ? min(cols - c, 8) : 0, odd = (int)((reinterpret_cast<uintptr_t>(x) >> 1) & 1u);
      w[i][0] = dl_word(x, !odd && n > 1, n > 0);
#pragma unroll
      for (int k = 1; k < 5; ++k) w[i][k] = dl_word(x + 2 * k - odd, 2 * k - odd + 1 < n, 2 * k - odd < n);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int shift = (int)((reinterpret_cast<uintptr_t>(p + i * (ROWS * step)) >> 1) & 1u) * 16;
      w[i][0] <<= shift;
      *reinterpret_cast<uint4*>(d + (i0 + i) * ROWS * ld) = make_uint4(__funnelshift_r(w[i][0], w[i][1], shift), __funnelshift_r(w[i][1], w[i][2], shift),
                                                                       __funnelshift_r(w[i][2], w[i][3], shift), __funnelshift_r(w[i][3], w[i][4], shift));
    }
    p += AHEAD * (ROWS * step);
  }
}
// PARTS matrices [64][64] from the work.
template <int PARTS, int OF>
__device__ __forceinline__ void dl_load64(bf* s, const bf* g, int t) {
  bf* d = s + (t >> 3) * DL_LD64 + (t & 7) * 8;  // rows of all parts, one after the other
  g += t * 8;
#pragma unroll
  for (int i = 0; i < PARTS * DL_CHUNK * 8 / OF; ++i) dl_copy16(d + i * (OF / 8) * DL_LD64, g + i * OF * 8, true);
}
template <typename Row>  // all of a row's numbers, or those that come first
__device__ __forceinline__ void dl_load_row(Row& s, const float* g, int t, int of) {
  for (int i = t; i < (int)(sizeof(Row) / 16); i += of) dl_copy16(reinterpret_cast<float*>(&s) + 4 * i, g + 4 * i, true);
}

struct DlUnit {
  int chunk, b, head, len, live;  // len: the sequence's steps; live: those of the chunk that are inside it
  uint32_t n;                     // sequence and head
  long long unit, row0;           // its place in the work; row of the chunk's first step
};
// (Sequences times heads, and chunks times those, are below 2^31.)
__device__ __forceinline__ void dl_move(const DlArgs& a, DlUnit& u, int chunk) {
  u.chunk = chunk;
  u.live = min(max(u.len - chunk * DL_CHUNK, 0), DL_CHUNK);
  u.unit = (long long)chunk * (a.B * a.heads) + u.n;
  u.row0 = (long long)chunk * DL_CHUNK * a.B + u.b;
}
__device__ __forceinline__ DlUnit dl_unit(const DlArgs& a, int chunk, uint32_t n) {
  DlUnit u;
  u.n = n;
  u.b = (int)(n / (uint32_t)a.heads);
  u.head = (int)(n - (uint32_t)u.b * (uint32_t)a.heads);
  u.len = a.lens ? min(max(a.lens[u.b], 0), a.T) : a.T;
  dl_move(a, u, chunk);
  return u;
}

// ---- a chunk's triangular system ----------------------------------------------------------------------
constexpr int DL_LDA = DL_CHUNK + 4;  // four neighbours at once, eight rows on different banks
template <int DK>
struct DlPrepShared {
  union {
    struct {
      bf k[DL_CHUNK][DK + 8], q[DL_CHUNK][DK + 8];
    };
    struct {
      float a[DL_CHUNK][DL_LDA];  // A, below the diagonal
      union {
        bf p[3][DL_CHUNK][DL_LD64];
        struct {
          float t[DL_CHUNK][DL_LDA];  // the inverse, with ones on the diagonal
          float tmp[6][16][8];
        };
      };
    };
  };
  DlRow row;
};

// s += A T, two rows of A (from a) by two columns of T (from b), over `count` entries.
__device__ __forceinline__ void dl_two_by_two(float (&s)[2][2], const float* a, const float* b, int ldb, int count) {
#pragma unroll 4
  for (int k = 0; k < count; k += 4, a += 4, b += 4 * ldb) {
    const float4 a0 = *reinterpret_cast<const float4*>(a), a1 = *reinterpret_cast<const float4*>(a + DL_LDA);
    const float2 b0 = *reinterpret_cast<const float2*>(b), b1 = *reinterpret_cast<const float2*>(b + ldb),
                 b2 = *reinterpret_cast<const float2*>(b + 2 * ldb), b3 = *reinterpret_cast<const float2*>(b + 3 * ldb);
    s[0][0] = fmaf(a0.w, b3.x, fmaf(a0.z, b2.x, fmaf(a0.y, b1.x, fmaf(a0.x, b0.x, s[0][0]))));
    s[0][1] = fmaf(a0.w, b3.y, fmaf(a0.z, b2.y, fmaf(a0.y, b1.y, fmaf(a0.x, b0.y, s[0][1]))));
    s[1][0] = fmaf(a1.w, b3.x, fmaf(a1.z, b2.x, fmaf(a1.y, b1.x, fmaf(a1.x, b0.x, s[1][0]))));
    s[1][1] = fmaf(a1.w, b3.y, fmaf(a1.z, b2.y, fmaf(a1.y, b1.y, fmaf(a1.x, b0.y, s[1][1]))));
  }
}
// The blocks below the diagonal of 16 x 16 blocks, T_ij = -T_ii sum_{j <= k < i} A_ik T_kj.  Columns do not see one another: a warp takes eight of them from top to
// bottom, two rows by two columns a lane, which reads shared memory a third as often as an entry a thread does (the kernel spends most of its time there).
template <typename Sh>
__device__ __forceinline__ void dl_inverse_columns(Sh& sh, int warp, int lane) {
  const int j = warp >> 1, r = 2 * (lane >> 2), c = 2 * (lane & 3), at = 8 * warp + c;
  for (int i = j + 1; i < 4; ++i) {
    float s[2][2] = {};
    dl_two_by_two(s, &sh.a[16 * i + r][16 * j], &sh.t[16 * j][at], DL_LDA, 16 * (i - j));
#pragma unroll
    for (int e = 0; e < 2; ++e) *reinterpret_cast<float2*>(&sh.tmp[warp][r + e][c]) = make_float2(s[e][0], s[e][1]);
    __syncwarp();
    s[0][0] = s[0][1] = s[1][0] = s[1][1] = 0.f;
    dl_two_by_two(s, &sh.t[16 * i + r][16 * i], &sh.tmp[warp][0][c], 8, 16);
#pragma unroll
    for (int e = 0; e < 2; ++e) *reinterpret_cast<float2*>(&sh.t[16 * i + r + e][at]) = make_float2(-s[e][0], -s[e][1]);
    __syncwarp();
  }
}

// A CTA to a chunk of a head, four of them an SM, so that one's loads and barriers pass while others compute; K and Q come once, and what is made of them takes their
// place in shared memory, which is busy for 60 % of the time: 2048 chunks of 128 columns 69 us.
template <int DK>
__global__ void __launch_bounds__(DL_THREADS, 4) delta_prep_kernel(const DlArgs a) {
  extern __shared__ __align__(16) uint8_t dl_smem[];
  auto& sh = *reinterpret_cast<DlPrepShared<DK>*>(dl_smem);
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const uint32_t units = (uint32_t)a.B * (uint32_t)a.heads;
  const DlUnit u = dl_unit(a, (int)(blockIdx.x / units), blockIdx.x % units);
  if (u.live == 0) return;  // nobody asks
  dl_load<DK, DL_THREADS>(&sh.k[0][0], DK + 8, a.K + u.row0 * a.ldk + (long long)u.head * a.Dk, a.B * a.ldk, u.live, a.Dk, a.vec_k, t);
  dl_load<DK, DL_THREADS>(&sh.q[0][0], DK + 8, a.Q + u.row0 * a.ldq + (long long)u.head * a.Dk, a.B * a.ldq, u.live, a.Dk, a.vec_q, t);
  dl_commit();
  if (t < DL_CHUNK) {
    float f = 1.f, rest = 0.f, beta = 0.f, closed = 1.f;
    if (t < u.live) {
      const long long r = (u.row0 + (long long)t * a.B) * a.ldz + u.head;
      dl_gate(__bfloat162float(a.Zf[r]), f, rest);
      dl_gate(__bfloat162float(a.Zb[r]), beta, closed);
    }
    sh.row.closed[t] = closed;
    sh.row.f[t] = f;
    sh.row.rest[t] = rest;
    sh.row.beta[t] = beta;
  }
  dl_wait<0>();
  __syncthreads();
  {  // lengths: four threads a row
    const int r = t >> 2, part = t & 3;
    float kk = 0.f, qq = 0.f;
#pragma unroll 8
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
      sh.row.rk[r] = a.eps < 0.f ? 1.f : kk > 0.f ? 1.f / sqrtf(kk) : 0.f;
      sh.row.rq[r] = a.eps < 0.f ? 1.f : qq > 0.f ? 1.f / sqrtf(qq) : 0.f;
    }
  }
  if (t < DL_CHUNK) {  // a column of the decays inside its block
    const int b = t >> 4, j = t & 15;
    float f[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = sh.row.f[16 * b + i];
    float g = 1.f, all = 1.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i > j) g *= f[i];
      sh.row.diag[b][i][j] = i < j ? 0.f : g;
      all *= f[i];
      if (i == j) sh.row.from[t] = all;
    }
    sh.row.to[t] = g;
    if (j == 15) sh.row.block[b] = all;
  }
  __syncthreads();
  if (t < DL_CHUNK) {
    const int b = t >> 4;
    float first = sh.row.from[t], last = sh.row.to[t];
    for (int i = 0; i < b; ++i) first *= sh.row.block[i];
    for (int i = b + 1; i < 4; ++i) last *= sh.row.block[i];
    sh.row.first[t] = first;
    sh.row.last[t] = last;
    sh.row.kin[t] = first * sh.row.rk[t];
    sh.row.kout[t] = last * sh.row.rk[t];
    sh.row.qin[t] = a.scale * first * sh.row.rq[t];
  }
  // K K^T (warps 0..3) and Q K^T (4..7), sixteen rows a warp
  {
    float c[1][8][4] = {};
    const int m0 = (warp < 4 ? warp : 7 - warp) * 16;
    const bool keys = warp < 4;
    dl_product<1, 8, false, false, 1, 1, 0>(c, keys ? &sh.k[0][0] : &sh.q[0][0], DK + 8, 0, &sh.k[0][0], DK + 8, 0, m0, 0, 0, DK, lane);
    __syncthreads();  // q and k have been read: A and P lie where they were
    const int bi = m0 >> 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = (lane >> 2) + 8 * h, i = m0 + r;
      const float by = keys ? sh.row.rk[i] * sh.row.beta[i] : sh.row.rq[i] * a.scale;
#pragma unroll
      for (int bj = 0; bj < 4; ++bj) {
        float across = by * sh.row.from[i];  // of what lies in earlier blocks
        for (int b = bj + 1; b < bi; ++b) across *= sh.row.block[b];
#pragma unroll
        for (int n = 2 * bj; n < 2 * bj + 2; ++n) {
          const int j = 8 * n + 2 * (lane & 3);
          float x[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int jj = j + e;
            const float g = bj < bi ? across * sh.row.to[jj] : bj == bi ? by * sh.row.diag[bj][r][jj & 15] : 0.f;
            x[e] = keys && jj >= i ? 0.f : c[0][n][2 * h + e] * sh.row.rk[jj] * g;
            if (bj > bi || jj > i) x[e] = 0.f;
            if (keys) sh.a[i][jj] = x[e];
          }
          if (!keys) dl_put<3>(&sh.p[0][i][j], DL_CHUNK * DL_LD64, x[0], x[1]);
        }
      }
    }
  }
  __syncthreads();
  {
    bf* P = a.p + u.unit * 3 * DL_SQ;
#pragma unroll
    for (int i = t; i < 3 * DL_CHUNK * 8; i += DL_THREADS)
      *reinterpret_cast<uint4*>(P + i * 8) = *reinterpret_cast<const uint4*>(&sh.p[0][0][0] + (i >> 3) * DL_LD64 + (i & 7) * 8);
  }
  __syncthreads();
  // the inverse, where P was: blocks of 16 on the diagonal by substitution, then those below it
  if (t < DL_CHUNK) {
    const int b0 = t & ~15, j = t & 15;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s = 0.f, s1 = 0.f;
#pragma unroll
      for (int k = 0; k < i; ++k) (k & 1 ? s1 : s) = fmaf(sh.a[b0 + i][b0 + k], x[k], k & 1 ? s1 : s);
      x[i] = i == j ? 1.f : i > j ? -(s + s1) : 0.f;
      sh.t[b0 + i][b0 + j] = x[i];
    }
  }
  __syncthreads();
  if (warp < 6) dl_inverse_columns(sh, warp, lane);
  __syncthreads();
  bf* tri = a.tri + u.unit * 3 * DL_SQ;
#pragma unroll
  for (int i = t; i < DL_SQ / 2; i += DL_THREADS) {
    const int r = i / (DL_CHUNK / 2), c = 2 * (i % (DL_CHUNK / 2));
    const bool on = c / 16 <= r / 16;
    const float2 x = on ? *reinterpret_cast<const float2*>(&sh.t[r][c]) : make_float2(0.f, 0.f);
    dl_put<3>(tri + r * DL_CHUNK + c, DL_SQ, x.x, x.y);
  }
  float* row = a.row + u.unit * DL_ROW_FLOATS;
  for (int i = t; i < DL_ROW_FLOATS; i += DL_THREADS) row[i] = reinterpret_cast<const float*>(&sh.row)[i];
}

// ---- from chunk to chunk ----------------------------------------------------------------------------
// Two warps hold 16 columns of the state, transposed, as accumulators [16 columns][DK / 2]: one the first half of its rows, one the second.  As rows of a left
// operand they lie in registers the way a product wants them, and so do the results that follow from them: E' = S' K', R' = b (V' - g E'), U' = R' T', S' += U' K.
// Of a chunk's 64 steps each of the two finishes 32; they meet three times a chunk, for the sums E, for what the earlier steps' R says to the later ones, and for U.
// What all columns share (K, Q, T, P) lies in shared memory.
// Beside each two stands a warp that fetches the next chunk and does what nobody waits for: forward the outputs, which take the state's and U's parts over shared
// memory, backward what comes from dY alone.  With 64 columns a CTA (2048 x 8 x 8: 128 CTAs) main warps and helpers have alike to do, 11 thousand cycles a chunk, of
// which the tensor pipe is busy for 45 %.  With one or two times 16 columns the helper's copies and products were the longer chain, and registers are left: there a warp
// beside each helper does nothing but fetch (16384 x 1 x 8 forward 842 -> 773 us, 2.7 a chunk).  (A warp to 16 columns, with all of the state: 217 / 260 us for the two
// scans of 2048 x 8 x 8 in place of 185 / 214, since its chain is twice as long and a scheduler has one of them; the state's parts in shared memory, eight warps to a
// product: the forward call 599 us.)
template <int NP>
struct DlTeams {
  static constexpr int HELP = 32 * NP, FETCH = NP <= 2 ? HELP : 0, FIRST = 3 * HELP, ALL = FIRST + FETCH;  // threads; FIRST: mains, and who brings the keys
  // barriers: 0 the keys are there; three for each pair of mains; among helpers, or between helpers and who fetches for them
  static constexpr int LATE = 1 + 3 * NP, EARLY = LATE + 1, PAST = LATE + 2, READ = LATE + 3;
};
// Some of a CTA's warps, in branches of their own (0: all of them).
__device__ __forceinline__ void dl_meet(int id, int threads) {
  __syncwarp();
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ void dl_tell(int id, int threads) {  // who need not wait
  __syncwarp();
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ void dl_take(const uint4& q, uint32_t (&a)[4]) { a[0] = q.x, a[1] = q.y, a[2] = q.z, a[3] = q.w; }
__device__ __forceinline__ uint32_t dl_transposed(uint32_t x) {  // of 8 x 8 bf16, a pair a lane
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t dl_pack(float x, float y) {
  uint32_t w[1];
  dl_split<1>(x, y, w);
  return w[0];
}
__device__ __forceinline__ float2 dl_unpack(uint32_t w) {
  __nv_bfloat162 h;
  memcpy(&h, &w, 4);
  return __bfloat1622float2(h);
}
// Sixteen of an accumulator's columns (tiles c0, c1 of 8) as a left operand in PARTS parts.
template <int PARTS>
__device__ __forceinline__ void dl_left(const float (&c0)[4], const float (&c1)[4], uint32_t (&a)[PARTS][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t w[PARTS];
    const float(&c)[4] = i < 2 ? c0 : c1;
    dl_split<PARTS>(c[2 * (i & 1)], c[2 * (i & 1) + 1], w);
#pragma unroll
    for (int p = 0; p < PARTS; ++p) a[p][i] = w[p];
  }
}
// c += A * B for the blocks FROM .. TO - 1 of 16 columns of the right operand, whose contraction begins at k0, in PB parts, products of parts i + j <= MOST.  An accumulator is not asked for
// again before all others have had their turn.
template <int FROM, int TO, int PA, int PB, int MOST, bool KN, int TILES>
__device__ __forceinline__ void dl_step(float (&c)[TILES][4], const uint32_t (&a)[PA][4], const bf* b, int ld, int stride, int k0, int lane) {
#pragma unroll
  for (int j = PB - 1; j >= 0; --j) {  // small parts first
    uint32_t rb[TO - FROM][4];
#pragma unroll
    for (int n = FROM; n < TO; ++n) dl_b<KN>(rb[n - FROM], b + j * stride, ld, 16 * n, k0, lane);
#pragma unroll
    for (int i = PA - 1; i >= 0; --i)
      if (i + j <= MOST) {
#pragma unroll
        for (int n = FROM; n < TO; ++n) {
          dl_mma(c[2 * n], a[i], rb[n - FROM][0], rb[n - FROM][1]);
          dl_mma(c[2 * n + 1], a[i], rb[n - FROM][2], rb[n - FROM][3]);
        }
      }
  }
}
// The blocks k .. 3, and 0 .. k, of [64] columns: what a triangular matrix leaves of the contraction's block k.
template <int PA, int PB, int MOST, bool KN>
__device__ __forceinline__ void dl_later(int k, float (&c)[8][4], const uint32_t (&a)[PA][4], const bf* b, int ld, int stride, int lane) {
  if (k == 0) dl_step<0, 4, PA, PB, MOST, KN>(c, a, b, ld, stride, 0, lane);
  if (k == 1) dl_step<1, 4, PA, PB, MOST, KN>(c, a, b, ld, stride, 16, lane);
  if (k == 2) dl_step<2, 4, PA, PB, MOST, KN>(c, a, b, ld, stride, 32, lane);
  if (k == 3) dl_step<3, 4, PA, PB, MOST, KN>(c, a, b, ld, stride, 48, lane);
}
template <int PA, int PB, int MOST, bool KN>
__device__ __forceinline__ void dl_earlier(int k, float (&c)[8][4], const uint32_t (&a)[PA][4], const bf* b, int ld, int stride, int lane) {
  if (k == 0) dl_step<0, 1, PA, PB, MOST, KN>(c, a, b, ld, stride, 0, lane);
  if (k == 1) dl_step<0, 2, PA, PB, MOST, KN>(c, a, b, ld, stride, 16, lane);
  if (k == 2) dl_step<0, 3, PA, PB, MOST, KN>(c, a, b, ld, stride, 32, lane);
  if (k == 3) dl_step<0, 4, PA, PB, MOST, KN>(c, a, b, ld, stride, 48, lane);
}
// A warp's state S' [16][DK], from and to [Dk][Dv] in memory: f(tile, element, row d, column c).
template <int DK, typename F>
__device__ __forceinline__ void dl_state(int lane, F f) {
#pragma unroll
  for (int n = 0; n < DK / 8; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) f(n, e, 8 * n + 2 * (lane & 3) + (e & 1), (lane >> 2) + 8 * (e >> 1));
}
__device__ __forceinline__ void dl_store2(bf* p, float x, float y, bool two) {
  if (two && (reinterpret_cast<uintptr_t>(p) & 3u) == 0) {
    *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(x, y);
  } else {
    p[0] = __float2bfloat16_rn(x);
    if (two) p[1] = __float2bfloat16_rn(y);
  }
}
// Sixteen columns of a chunk's steps r0 .. r0 + 8 N - 1, in accumulators [16][8 N], to rows of bf16; x times by[step] where by is given.
template <int N>
__device__ __forceinline__ void dl_rows_out(const float (&x)[N][4], const float* by, bf* g, long long step, int r0, int live, int cols, int lane) {
  const int r = r0 + (lane >> 2), c = 2 * (lane & 3);
  bf* p = g + r * step + c;
  const bool pairs = ((reinterpret_cast<uintptr_t>(g) | (uintptr_t)(step * 2)) & 3u) == 0 && (cols & 1) == 0;  // both of two columns are there, on a grid of 4 bytes
#pragma unroll
  for (int n = 0; n < N; ++n, p += 8 * step) {
    float2 m = make_float2(1.f, 1.f);
    if (by) m = *reinterpret_cast<const float2*>(by + r0 + 8 * n + 2 * (lane & 3));
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) w[h] = dl_transposed(dl_pack(x[n][2 * h] * m.x, x[n][2 * h + 1] * m.y));
    if (r + 8 * n >= live) continue;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (c + 8 * h >= cols) continue;
      if (pairs) {
        *reinterpret_cast<uint32_t*>(p + 8 * h) = w[h];
      } else {
        bf e[2];
        memcpy(e, &w[h], 4);
        p[8 * h] = e[0];
        if (c + 8 * h + 1 < cols) p[8 * h + 1] = e[1];
      }
    }
  }
}
// Rows of a chunk behind the sequence's end.
__device__ __forceinline__ void dl_zero_rows(bf* g, long long step, int from, int to, int cols, int t, int of) {
  for (int i = from * cols + t; i < to * cols; i += of) g[(i / cols) * step + i % cols] = __float2bfloat16_rn(0.f);
}

template <int DK, int NP>
struct DlScanShared {
  bf k[2][DL_CHUNK][DK + 8], q[DL_CHUNK][DK + 8];
  bf tri[3][DL_CHUNK][DL_LD64];
  bf p[2][DL_CHUNK][DL_LD64];
  bf v[DL_CHUNK][NP * 16 + 8];
  uint4 s[NP][DK / 16][2][32];  // the state's parts as left operands
  uint4 u[NP][4][2][32];        // U's
  uint4 us[NP][4][3][32];       // those of U G_C / |k|
  uint4 r[NP][2][3][32];        // the earlier steps' R
  float4 e[NP][2][4][32];       // what a half of the state gives to the other half's steps
  DlSteps row[2];
};

template <int DK, int NP>
__global__ void __launch_bounds__(DlTeams<NP>::ALL, 1) delta_scan_kernel(const DlArgs a) {
  constexpr int LDK = DK + 8, LDV = NP * 16 + 8, PT = DL_CHUNK * DL_LD64, HALF = DK / 2;
  using Teams = DlTeams<NP>;
  constexpr int HELP = Teams::HELP, FIRST = Teams::FIRST, ALL = Teams::ALL;
  constexpr bool FETCH = Teams::FETCH != 0;
  extern __shared__ __align__(16) uint8_t dl_smem[];
  auto& sh = *reinterpret_cast<DlScanShared<DK, NP>*>(dl_smem);
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pair = warp % NP, half = warp / NP;  // half 2: the helper; 3: who fetches
  const int states = 1 + pair, updates = 1 + NP + pair, early = 1 + 2 * NP + pair;  // barriers
  const int blocks = (a.Dv + NP * 16 - 1) / (NP * 16);
  const uint32_t n = blockIdx.x / (uint32_t)blocks;
  const long long size = (long long)a.Dk * a.Dv;
  const int c0 = (int)(blockIdx.x - n * (uint32_t)blocks) * NP * 16, cols = min(NP * 16, a.Dv - c0);  // the CTA's columns
  const int mine = min(max(cols - 16 * pair, 0), 16);                                    // the three warps'
  DlUnit u = dl_unit(a, 0, n);
  const int chunks = (u.len + DL_CHUNK - 1) / DL_CHUNK;
  const bf *Q = a.Q + (long long)u.head * a.Dk, *K = a.K + (long long)u.head * a.Dk, *V = a.V + (long long)u.head * a.Dv + c0;
  bf* Y = a.Y + (long long)u.head * a.Dv + c0;
  if (half >= 2) {
    const int t = threadIdx.x - (FETCH ? 3 : 2) * HELP;
    auto fetch_k = [&](int chunk) {
      if (chunk >= chunks) return;
      dl_move(a, u, chunk);
      dl_load<DK, HELP>(&sh.k[chunk & 1][0][0], LDK, K + u.row0 * a.ldk, a.B * a.ldk, u.live, a.Dk, a.vec_k, t);
      dl_load_row(sh.row[chunk & 1], a.row + u.unit * DL_ROW_FLOATS, t, HELP);
    };
    auto fetch_others = [&](int chunk) {
      if (chunk >= chunks) return;
      dl_move(a, u, chunk);
      dl_load<DK, HELP>(&sh.q[0][0], LDK, Q + u.row0 * a.ldq, a.B * a.ldq, u.live, a.Dk, a.vec_q, t);
      dl_load<NP * 16, HELP>(&sh.v[0][0], LDV, V + u.row0 * a.ldv, a.B * a.ldv, u.live, cols, a.vec_v, t);
      dl_load64<3, HELP>(&sh.tri[0][0][0], a.tri + u.unit * 3 * DL_SQ, t);
    };
    auto fetch_p = [&](int chunk) { dl_load64<2, HELP>(&sh.p[0][0][0], a.p + ((long long)chunk * (a.B * a.heads) + n) * 3 * DL_SQ, t); };
    if (half == (FETCH ? 3 : 2)) {
      fetch_k(0);
      dl_commit();
      fetch_others(0);
      dl_commit();
      dl_wait<1>();
      if (chunks > 0) dl_tell(0, FIRST);  // K is there: nobody else waits for a helper, whose outputs may lag behind
    }
    if (half == 3) {
      dl_wait<0>();
      if (chunks > 0) dl_tell(Teams::LATE, 2 * HELP);  // Q, V and T are there
      for (int chunk = 0; chunk < chunks; ++chunk) {
        const bool more = chunk + 1 < chunks;
        dl_meet(Teams::PAST, 2 * HELP);  // all have gone on to this chunk: nobody reads P any more, nor the keys before it
        fetch_k(chunk + 1);
        fetch_p(chunk);
        dl_commit();
        dl_wait<0>();
        if (more) dl_tell(0, FIRST);
        dl_tell(Teams::EARLY, 2 * HELP);
        if (!more) break;
        dl_meet(Teams::READ, 2 * HELP);  // nobody reads Q, V and T any more
        fetch_others(chunk + 1);
        dl_commit();
        dl_wait<0>();
        dl_tell(Teams::LATE, 2 * HELP);
      }
    }
    for (int chunk = 0; half == 2 && chunk < chunks; ++chunk) {
      const int at = chunk & 1;
      if constexpr (FETCH) {
        dl_meet(Teams::LATE, 2 * HELP);
        dl_meet(states, 96);
        dl_tell(Teams::PAST, 2 * HELP);
      } else {
        dl_wait<0>();
        dl_meet(Teams::LATE, HELP);  // Q, V and T are there, and nobody reads P any more
        dl_meet(states, 96);         // nor, since all have gone on to this chunk, the keys before it
        fetch_k(chunk + 1);
        fetch_p(chunk);
        dl_commit();
      }
      float o[8][4] = {};
#pragma unroll
      for (int kd = 0; kd < DK / 16; ++kd) {
        uint32_t s[2][4];
#pragma unroll
        for (int p = 0; p < 2; ++p) dl_take(sh.s[pair][kd][p][lane], s[p]);
        dl_step<0, 4, 2, 1, 1, false>(o, s, &sh.q[0][0], LDK, 0, 16 * kd, lane);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 g = *reinterpret_cast<const float2*>(&sh.row[at].qin[8 * i + 2 * (lane & 3)]);
        o[i][0] *= g.x, o[i][1] *= g.y, o[i][2] *= g.x, o[i][3] *= g.y;
      }
      dl_meet(updates, 96);
      if constexpr (FETCH) {
        if (chunk + 1 < chunks) dl_tell(Teams::READ, 2 * HELP);
        dl_meet(Teams::EARLY, 2 * HELP);  // P is there
      } else {
        dl_wait<0>();
        dl_meet(Teams::LATE, HELP);  // P and the next keys are there, and nobody reads Q, V and T any more
        if (chunk + 1 < chunks) dl_tell(0, FIRST);
        fetch_others(chunk + 1);
        dl_commit();
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t x[2][4];
#pragma unroll
        for (int p = 0; p < 2; ++p) dl_take(sh.u[pair][k][p][lane], x[p]);
        dl_later<2, 2, 1, false>(k, o, x, &sh.p[0][0][0], DL_LD64, PT, lane);
      }
      dl_move(a, u, chunk);
      dl_rows_out<8>(o, nullptr, Y + u.row0 * a.ldy + 16 * pair, a.B * a.ldy, 0, u.live, mine, lane);
    }
  } else {
    float s[DK / 16][4];
    const int d0 = half * HALF;  // this warp's rows of the state, and steps 32 half .. 32 half + 31 of a chunk
    const float* h0 = a.h0 ? a.h0 + n * size + c0 + 16 * pair : nullptr;
    dl_state<HALF>(lane, [&](int i, int e, int d, int c) { s[i][e] = h0 && d0 + d < a.Dk && c < mine ? h0[(long long)(d0 + d) * a.Dv + c] : 0.f; });
    const bool even = a.Dk % 2 == 0 && (reinterpret_cast<uintptr_t>(a.S) & 7u) == 0;
    auto keep = [&](float* g) {  // for the backward call: transposed, as it lies here
#pragma unroll
      for (int i = 0; i < DK / 16; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int d = d0 + 8 * i + 2 * (lane & 3), c = (lane >> 2) + 8 * h;
          if (d >= a.Dk || c >= mine) continue;
          float* p = g + c * a.Dk + d;
          if (even) {
            *reinterpret_cast<float2*>(p) = make_float2(s[i][2 * h], s[i][2 * h + 1]);
          } else {
            p[0] = s[i][2 * h];
            if (d + 1 < a.Dk) p[1] = s[i][2 * h + 1];
          }
        }
    };
    for (int chunk = 0; chunk < chunks; ++chunk) {
      const DlSteps& row = sh.row[chunk & 1];
      const bf* k0 = &sh.k[chunk & 1][0][0];
      const bf* tri = &sh.tri[0][0][0] + half * 32 * DL_LD64;  // this warp's steps
      dl_meet(0, FIRST);
      float r[4][4];
      {
        float e[8][4] = {};
#pragma unroll
        for (int kd = 0; kd < DK / 32; ++kd) {
          uint32_t x[3][4];
          dl_left<3>(s[2 * kd], s[2 * kd + 1], x);
          sh.s[pair][half * (DK / 32) + kd][0][lane] = make_uint4(x[0][0], x[0][1], x[0][2], x[0][3]);
          sh.s[pair][half * (DK / 32) + kd][1][lane] = make_uint4(x[1][0], x[1][1], x[1][2], x[1][3]);
          dl_step<0, 4, 3, 1, 2, false>(e, x, k0, LDK, 0, d0 + 16 * kd, lane);
        }
        // each half of the state adds to all steps; a warp has the sums of its own
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float(&give)[4] = e[i + 4], (&give0)[4] = e[i];
          sh.e[pair][half][i][lane] = half ? make_float4(give0[0], give0[1], give0[2], give0[3]) : make_float4(give[0], give[1], give[2], give[3]);
#pragma unroll
          for (int j = 0; j < 4; ++j) r[i][j] = half ? e[i + 4][j] : e[i][j];
        }
      }
      if (a.S) keep(a.S + ((long long)chunk * (a.B * a.heads) + n) * size + (long long)(c0 + 16 * pair) * a.Dk);
      dl_meet(states, 96);
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        uint32_t v[4];
        dl_ldsm_t(v, &sh.v[32 * half + 8 * i + (lane & 7) + ((lane >> 4) << 3)][16 * pair + ((lane >> 3) & 1) * 8]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float4 o = sh.e[pair][half ^ 1][i + j][lane];
          const int at = 32 * half + 8 * (i + j) + 2 * (lane & 3);
          const float2 b = *reinterpret_cast<const float2*>(&row.beta[at]), g = *reinterpret_cast<const float2*>(&row.kin[at]), x0 = dl_unpack(v[2 * j]), x1 = dl_unpack(v[2 * j + 1]);
          r[i + j][0] = b.x * fmaf(-g.x, r[i + j][0] + o.x, x0.x);
          r[i + j][1] = b.y * fmaf(-g.y, r[i + j][1] + o.y, x0.y);
          r[i + j][2] = b.x * fmaf(-g.x, r[i + j][2] + o.z, x1.x);
          r[i + j][3] = b.y * fmaf(-g.y, r[i + j][3] + o.w, x1.y);
        }
      }
      float x[4][4] = {};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t w[3][4];
        dl_left<3>(r[2 * k], r[2 * k + 1], w);
        if (half == 0)
#pragma unroll
          for (int p = 0; p < 3; ++p) sh.r[pair][k][p][lane] = make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]);
        if (k == 0) dl_step<0, 2, 3, 3, 2, false>(x, w, tri, DL_LD64, PT, 32 * half, lane);
        else dl_step<1, 2, 3, 3, 2, false>(x, w, tri, DL_LD64, PT, 32 * half + 16, lane);
      }
      if (half == 0) {
        dl_tell(early, 64);
      } else {
        dl_meet(early, 64);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t w[3][4];
#pragma unroll
          for (int p = 0; p < 3; ++p) dl_take(sh.r[pair][k][p][lane], w[p]);
          dl_step<0, 2, 3, 3, 2, false>(x, w, tri, DL_LD64, PT, 16 * k, lane);
        }
      }
      uint32_t own[2][3][4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t w[2][4];
        dl_left<2>(x[2 * k], x[2 * k + 1], w);
#pragma unroll
        for (int p = 0; p < 2; ++p) sh.u[pair][2 * half + k][p][lane] = make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]);
#pragma unroll
        for (int i = 2 * k; i < 2 * k + 2; ++i) {
          const float2 g = *reinterpret_cast<const float2*>(&row.kout[32 * half + 8 * i + 2 * (lane & 3)]);
          x[i][0] *= g.x, x[i][1] *= g.y, x[i][2] *= g.x, x[i][3] *= g.y;
        }
        dl_left<3>(x[2 * k], x[2 * k + 1], own[k]);
#pragma unroll
        for (int p = 0; p < 3; ++p) sh.us[pair][2 * half + k][p][lane] = make_uint4(own[k][p][0], own[k][p][1], own[k][p][2], own[k][p][3]);
      }
      dl_meet(updates, 96);
      const float whole = row.first[DL_CHUNK - 1];
#pragma unroll
      for (int i = 0; i < DK / 16; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] *= whole;
#pragma unroll
      for (int k = 0; k < 2; ++k) dl_step<0, DK / 32, 3, 1, 2, true>(s, own[k], k0 + d0, LDK, 0, 32 * half + 16 * k, lane);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t w[3][4];
#pragma unroll
        for (int p = 0; p < 3; ++p) dl_take(sh.us[pair][2 * (half ^ 1) + k][p][lane], w[p]);
        dl_step<0, DK / 32, 3, 1, 2, true>(s, w, k0 + d0, LDK, 0, 32 * (half ^ 1) + 16 * k, lane);
      }
    }
    if (a.hT) dl_state<HALF>(lane, [&](int i, int e, int d, int c) { if (d0 + d < a.Dk && c < mine) a.hT[n * size + (long long)(d0 + d) * a.Dv + c0 + 16 * pair + c] = s[i][e]; });
  }
  for (int chunk = u.len / DL_CHUNK; chunk * DL_CHUNK < a.T; ++chunk) {
    dl_move(a, u, chunk);
    dl_zero_rows(Y + u.row0 * a.ldy, a.B * a.ldy, u.live, min(DL_CHUNK, a.T - chunk * DL_CHUNK), cols, threadIdx.x, ALL);
  }
}

// The adjoint: F' = D' K', dU' = G' + G_C F', X' = dU' T, D' = g_C D' + Y' + W' K with W = -g b X; the helpers bring G = scale P^T dY and Y = Q^T (scale g dY), which come
// from the chunk alone.
template <int DK, int NP>
struct DlBackShared {
  bf k[2][DL_CHUNK][DK + 8], q[DL_CHUNK][DK + 8];
  bf tri[3][DL_CHUNK][DL_LD64];
  bf p[3][DL_CHUNK][DL_LD64];
  bf dy[DL_CHUNK][NP * 16 + 8];
  float4 g[NP][8][32];
  float4 y[NP][DK / 8][32];
  uint4 w[NP][4][3][32];   // W's parts as left operands
  uint4 r[NP][2][3][32];   // the later steps' dU
  float4 e[NP][2][4][32];
  DlSteps row[2];
};

template <int DK, int NP>
__global__ void __launch_bounds__(DlTeams<NP>::ALL, 1) delta_back_kernel(const DlArgs a) {
  constexpr int LDK = DK + 8, LDV = NP * 16 + 8, PT = DL_CHUNK * DL_LD64, HALF = DK / 2;
  using Teams = DlTeams<NP>;
  constexpr int HELP = Teams::HELP, FIRST = Teams::FIRST, ALL = Teams::ALL;
  constexpr bool FETCH = Teams::FETCH != 0;
  extern __shared__ __align__(16) uint8_t dl_smem[];
  auto& sh = *reinterpret_cast<DlBackShared<DK, NP>*>(dl_smem);
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pair = warp % NP, half = warp / NP;
  const int states = 1 + pair, updates = 1 + NP + pair, late = 1 + 2 * NP + pair;
  const int blocks = (a.Dv + NP * 16 - 1) / (NP * 16);
  const uint32_t n = blockIdx.x / (uint32_t)blocks;
  const long long size = (long long)a.Dk * a.Dv;
  const int c0 = (int)(blockIdx.x - n * (uint32_t)blocks) * NP * 16, cols = min(NP * 16, a.Dv - c0);
  const int mine = min(max(cols - 16 * pair, 0), 16);
  DlUnit u = dl_unit(a, 0, n);
  const int chunks = (u.len + DL_CHUNK - 1) / DL_CHUNK;
  const bf *Q = a.Q + (long long)u.head * a.Dk, *K = a.K + (long long)u.head * a.Dk, *dY = a.dY + (long long)u.head * a.Dv + c0;
  bf* dV = a.dV + (long long)u.head * a.Dv + c0;
  if (half >= 2) {
    const int t = threadIdx.x - (FETCH ? 3 : 2) * HELP;
    auto fetch_k = [&](int chunk) {
      if (chunk < 0) return;
      dl_move(a, u, chunk);
      dl_load<DK, HELP>(&sh.k[chunk & 1][0][0], LDK, K + u.row0 * a.ldk, a.B * a.ldk, u.live, a.Dk, a.vec_k, t);
      dl_load_row(sh.row[chunk & 1], a.row + u.unit * DL_ROW_FLOATS, t, HELP);
    };
    auto fetch_mine = [&](int chunk) {  // what the helpers read
      if (chunk < 0) return;
      dl_move(a, u, chunk);
      dl_load<NP * 16, HELP>(&sh.dy[0][0], LDV, dY + u.row0 * a.lddy, a.B * a.lddy, u.live, cols, a.vec_dy, t);
      dl_load64<3, HELP>(&sh.p[0][0][0], a.p + u.unit * 3 * DL_SQ, t);
      dl_load<DK, HELP>(&sh.q[0][0], LDK, Q + u.row0 * a.ldq, a.B * a.ldq, u.live, a.Dk, a.vec_q, t);
    };
    auto fetch_tri = [&](int chunk) {
      if (chunk >= 0) dl_load64<3, HELP>(&sh.tri[0][0][0], a.tri + ((long long)chunk * (a.B * a.heads) + n) * 3 * DL_SQ, t);
    };
    // G to shared memory and Y to registers: a chunk ahead of the state
    float y[DK / 8][4];
    auto ahead = [&](int chunk) {
      uint32_t dy[4][1][4];  // dY' as a left operand
#pragma unroll
      for (int k = 0; k < 4; ++k) dl_a<true>(dy[k][0], &sh.dy[0][0], LDV, 16 * pair, 16 * k, lane);
      {
        float g[8][4] = {};
#pragma unroll
        for (int k = 0; k < 4; ++k) dl_earlier<1, 3, 2, true>(k, g, dy[k], &sh.p[0][0][0], DL_LD64, PT, lane);
#pragma unroll
        for (int i = 0; i < 8; ++i) sh.g[pair][i][lane] = make_float4(g[i][0], g[i][1], g[i][2], g[i][3]);
      }
#pragma unroll
      for (int i = 0; i < DK / 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) y[i][j] = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float* by = &sh.row[chunk & 1].qin[16 * k + 2 * (lane & 3)];
        const float2 m0 = *reinterpret_cast<const float2*>(by), m1 = *reinterpret_cast<const float2*>(by + 8);
        uint32_t x[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 v = dl_unpack(dy[k][0][i]);
          const float2 m = i < 2 ? m0 : m1;
          uint32_t w[3];
          dl_split<3>(v.x * m.x, v.y * m.y, w);
#pragma unroll
          for (int p = 0; p < 3; ++p) x[p][i] = w[p];
        }
        dl_step<0, 4, 3, 1, 2, true>(y, x, &sh.q[0][0], LDK, 0, 16 * k, lane);
        if constexpr (DK > 64) dl_step<4, 8, 3, 1, 2, true>(y, x, &sh.q[0][0], LDK, 0, 16 * k, lane);
      }
    };
    if (half == (FETCH ? 3 : 2) && chunks > 0) {
      fetch_k(chunks - 1);
      fetch_mine(chunks - 1);
      dl_commit();
      fetch_tri(chunks - 1);
      dl_commit();
      dl_wait<1>();
      if (!FETCH) dl_meet(Teams::LATE, HELP);
      dl_tell(0, FIRST);  // K is there
    }
    if (half == 3 && chunks > 0) {
      dl_tell(Teams::EARLY, 2 * HELP);  // P, Q and dY are there
      dl_wait<0>();
      dl_tell(Teams::LATE, 2 * HELP);   // T is there
      for (int chunk = chunks - 1; chunk > 0; --chunk) {
        dl_meet(Teams::PAST, 2 * HELP);  // all have gone on to this chunk: nobody reads P, Q and dY any more, nor the keys behind it
        fetch_k(chunk - 1);
        fetch_mine(chunk - 1);
        dl_commit();
        dl_wait<0>();
        dl_tell(0, FIRST);
        dl_tell(Teams::EARLY, 2 * HELP);
        dl_meet(Teams::READ, 2 * HELP);  // nobody reads T any more
        fetch_tri(chunk - 1);
        dl_commit();
        dl_wait<0>();
        dl_tell(Teams::LATE, 2 * HELP);
      }
    }
    if (half == 2 && chunks > 0) {
      if (FETCH) dl_meet(Teams::EARLY, 2 * HELP);
      ahead(chunks - 1);
    }
    for (int chunk = chunks - 1; half == 2 && chunk >= 0; --chunk) {
      if constexpr (FETCH) {
        dl_meet(Teams::LATE, 2 * HELP);
      } else {
        dl_wait<0>();
        dl_meet(Teams::LATE, HELP);  // T is there, and nobody reads P, Q and dY any more
      }
      dl_meet(states, 96);  // nor, since all have gone on to this chunk, the keys behind it and the last Y
      if (FETCH && chunk > 0) dl_tell(Teams::PAST, 2 * HELP);
#pragma unroll
      for (int i = 0; i < DK / 8; ++i) sh.y[pair][i][lane] = make_float4(y[i][0], y[i][1], y[i][2], y[i][3]);
      if constexpr (!FETCH) {
        fetch_k(chunk - 1);
        fetch_mine(chunk - 1);
        dl_commit();
      }
      dl_meet(updates, 96);
      if constexpr (FETCH) {
        if (chunk == 0) break;
        dl_tell(Teams::READ, 2 * HELP);
        dl_meet(Teams::EARLY, 2 * HELP);
      } else {
        dl_wait<0>();
        dl_meet(Teams::LATE, HELP);  // the next keys, P, Q and dY are there, and nobody reads T any more
        if (chunk == 0) break;
        dl_tell(0, FIRST);
        fetch_tri(chunk - 1);
        dl_commit();
      }
      ahead(chunk - 1);
    }
  } else {
    float s[DK / 16][4];
    const int d0 = half * HALF;
    const float* last = a.dhT ? a.dhT + n * size + c0 + 16 * pair : nullptr;
    dl_state<HALF>(lane, [&](int i, int e, int d, int c) { s[i][e] = last && d0 + d < a.Dk && c < mine ? last[(long long)(d0 + d) * a.Dv + c] : 0.f; });
    const bool here = c0 + 16 * pair < a.ldx;  // the work's rows end with 64 or 128 columns
    for (int chunk = chunks - 1; chunk >= 0; --chunk) {
      const DlSteps& row = sh.row[chunk & 1];
      const bf* k0 = &sh.k[chunk & 1][0][0];
      const bf* tri = &sh.tri[0][0][0] + half * 32;  // this warp's steps
      dl_move(a, u, chunk);
      dl_meet(0, FIRST);
      float r[4][4];
      {
        float f[8][4] = {};
        bf* D = a.d + u.unit * 2 * DK * a.ldx + (long long)(c0 + 16 * pair) * DK + d0;
#pragma unroll
        for (int kd = 0; kd < DK / 32; ++kd) {
          uint32_t x[3][4];
          dl_left<3>(s[2 * kd], s[2 * kd + 1], x);
          if (here)
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
              for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(D + (p * a.ldx + 8 * (i & 1) + (lane >> 2)) * DK + 16 * kd + 8 * (i >> 1) + 2 * (lane & 3)) = x[p][i];
          dl_step<0, 4, 3, 1, 2, false>(f, x, k0, LDK, 0, d0 + 16 * kd, lane);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float(&give)[4] = f[i + 4], (&give0)[4] = f[i];
          sh.e[pair][half][i][lane] = half ? make_float4(give0[0], give0[1], give0[2], give0[3]) : make_float4(give[0], give[1], give[2], give[3]);
#pragma unroll
          for (int j = 0; j < 4; ++j) r[i][j] = half ? f[i + 4][j] : f[i][j];
        }
      }
      dl_meet(states, 96);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 o = sh.e[pair][half ^ 1][i][lane], g = sh.g[pair][4 * half + i][lane];
        const float2 l = *reinterpret_cast<const float2*>(&row.kout[32 * half + 8 * i + 2 * (lane & 3)]);
        r[i][0] = fmaf(l.x, r[i][0] + o.x, g.x), r[i][1] = fmaf(l.y, r[i][1] + o.y, g.y), r[i][2] = fmaf(l.x, r[i][2] + o.z, g.z), r[i][3] = fmaf(l.y, r[i][3] + o.w, g.w);
      }
      float x[4][4] = {};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t w[3][4];
        dl_left<3>(r[2 * k], r[2 * k + 1], w);
        if (half == 1)
#pragma unroll
          for (int p = 0; p < 3; ++p) sh.r[pair][k][p][lane] = make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]);
        if (k == 0) dl_step<0, 1, 3, 3, 2, true>(x, w, tri, DL_LD64, PT, 32 * half, lane);
        else dl_step<0, 2, 3, 3, 2, true>(x, w, tri, DL_LD64, PT, 32 * half + 16, lane);
      }
      if (half == 1) {
        dl_tell(late, 64);
      } else {
        dl_meet(late, 64);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t w[3][4];
#pragma unroll
          for (int p = 0; p < 3; ++p) dl_take(sh.r[pair][k][p][lane], w[p]);
          dl_step<0, 2, 3, 3, 2, true>(x, w, tri, DL_LD64, PT, 32 + 16 * k, lane);
        }
      }
      uint32_t own[2][3][4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float m[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int at = 32 * half + 8 * (2 * k + i) + 2 * (lane & 3);
          const float2 b = *reinterpret_cast<const float2*>(&row.beta[at]), g = *reinterpret_cast<const float2*>(&row.kin[at]);
          const float(&v)[4] = x[2 * k + i];
          m[i][0] = v[0] * -b.x * g.x, m[i][1] = v[1] * -b.y * g.y, m[i][2] = v[2] * -b.x * g.x, m[i][3] = v[3] * -b.y * g.y;
        }
        dl_left<3>(m[0], m[1], own[k]);
#pragma unroll
        for (int p = 0; p < 3; ++p) sh.w[pair][2 * half + k][p][lane] = make_uint4(own[k][p][0], own[k][p][1], own[k][p][2], own[k][p][3]);
      }
      const float whole = row.first[DL_CHUNK - 1];
#pragma unroll
      for (int i = 0; i < DK / 16; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] *= whole;
#pragma unroll
      for (int k = 0; k < 2; ++k) dl_step<0, DK / 32, 3, 1, 2, true>(s, own[k], k0 + d0, LDK, 0, 32 * half + 16 * k, lane);
      dl_meet(updates, 96);
#pragma unroll
      for (int i = 0; i < DK / 16; ++i) {
        const float4 y = sh.y[pair][half * (DK / 16) + i][lane];
        s[i][0] += y.x, s[i][1] += y.y, s[i][2] += y.z, s[i][3] += y.w;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t w[3][4];
#pragma unroll
        for (int p = 0; p < 3; ++p) dl_take(sh.w[pair][2 * (half ^ 1) + k][p][lane], w[p]);
        dl_step<0, DK / 32, 3, 1, 2, true>(s, w, k0 + d0, LDK, 0, 32 * (half ^ 1) + 16 * k, lane);
      }
      // nobody waits for these
      dl_rows_out<4>(x, row.beta, dV + u.row0 * a.lddv + 16 * pair, a.B * a.lddv, 32 * half, u.live, mine, lane);
      bf* X = a.x + u.unit * 2 * DL_CHUNK * a.ldx + c0 + 16 * pair;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t w[2];
          dl_split<2>(x[i][2 * h], x[i][2 * h + 1], w);
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const uint32_t y = dl_transposed(w[p]);
            if (here) *reinterpret_cast<uint32_t*>(X + (p * DL_CHUNK + 32 * half + 8 * i + (lane >> 2)) * a.ldx + 8 * h + 2 * (lane & 3)) = y;
          }
        }
    }
    if (a.dh0) dl_state<HALF>(lane, [&](int i, int e, int d, int c) { if (d0 + d < a.Dk && c < mine) a.dh0[n * size + (long long)(d0 + d) * a.Dv + c0 + 16 * pair + c] = s[i][e]; });
  }
  for (int chunk = u.len / DL_CHUNK; chunk * DL_CHUNK < a.T; ++chunk) {
    dl_move(a, u, chunk);
    dl_zero_rows(dV + u.row0 * a.lddv, a.B * a.lddv, u.live, min(DL_CHUNK, a.T - chunk * DL_CHUNK), cols, threadIdx.x, ALL);
  }
}

// ---- step by step -----------------------------------------------------------------------------------
// The 8 warps of a CTA hold 128 rows of a state, 16 each, a lane the columns 4 lane + k (or lane + 32 k); a step needs one meeting of the warps, for what the old
// state gives with k and with q: y = scale (f S^T q + u (k.q)).  Memory bounds it: a state is read and written once, 512 of them in 14.7 us (4.6 TB/s).
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
    if (a.S && step == 0) {  // (there is one chunk) transposed, as the backward call reads it
#pragma unroll
      for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (warp + WARPS * i < a.Dk && col(k) < a.Dv) a.S[n * size + (long long)col(k) * a.Dk + warp + WARPS * i] = s[i][k];
    }
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

// ---- a chunk's own gradients ------------------------------------------------------------------------
// With U again from the state S_0 that the forward call left, and o the products of entries,
//   N = scale G o (dY U^T) (j <= i),  M = -b G o (X U^T) (j < i),
//   dQ = scale g dY S_0^T + N K,  dK = N^T Q + (M + M^T) K - g b X S_0^T + G_C U D^T,  dZb = X.U (1 - b),
// for q and k divided by their lengths, then dq / |q| without its part along q.  What gate t sees is all that passes it:
//   d log f_t = sum_{i >= t > j} W_ij + sum_{i >= t} a_i + sum_{j < t} c_j + g_C <D, S_0>,   W = N o Q K^T + M o K K^T,
// a_i the parts of q_i.dq_i and k_i.dk_i that come from S_0, c_j that of k_j.dk_j that comes from D.  Each of them has f_t for a factor, so small
// gates have small gradients to the last bit; (q.dq - v.dv) summed up backwards is the same in exact arithmetic and leaves a difference of large sums.
// One CTA of 16 warps an SM, which holds everything of a chunk (222 KB).  2048 chunks of 128 x 128: 378 us; of a chunk's 46 thousand cycles 13 are its
// loads (64 KB of S_0 and twice 64 KB of D; without the prefetch to L2 20), 17 what the products take at the tensor pipe's rate, the rest barriers between them and sums.
constexpr int DL_GRAD_THREADS = 512, DL_GRAD_WARPS = DL_GRAD_THREADS / 32;

template <int DK, int DV>
struct DlGradShared {
  bf k[DL_CHUNK][DK + 8], q[DL_CHUNK][DK + 8];
  bf dy[DL_CHUNK][DV + 8];
  bf x[2][DL_CHUNK][DV + 8];
  bf u[2][DL_CHUNK][DV + 8];   // b (V - g K S), then U
  union {
    bf s[2][DV][DK + 8];       // S_0 transposed, then D
    bf m[3][2][DL_CHUNK][DL_LD64];  // N / |k_j|, N / |q_i|, (M + M^T) / |k_j|
  };
  union {
    bf tri[2][DL_CHUNK][DL_LD64];
    float w[DL_CHUNK][DL_CHUNK + 1];  // W, then its sums over i >= t inside blocks of 8
  };
  float over[8][DL_CHUNK];     // a block's whole sum
  DlRow row;
  float red[4][4][DL_CHUNK];   // sums over a row, by groups of columns: a_i, c_j, q.dq, k.dk
  float xu[DL_CHUNK], seen[DL_CHUNK];
  float ds[DL_GRAD_WARPS];
};

// A state [Dv][Dk] in fp32 to two bf16 parts in shared memory, zeros around it.  Returns this thread's share of its product, entry by entry, with what `with` [2][rows][DK] holds in
// two parts in memory.
template <int DK, int DV>
__device__ __forceinline__ float dl_load_state(bf* s, const float* g, int Dk, int Dv, int vec, const bf* with, int rows) {
  constexpr int LD = DK + 8, QUADS = DK / 4, AHEAD = DV * QUADS / DL_GRAD_THREADS;  // all of them at once: nothing else is held yet
  float dot = 0.f;
  {
    float4 x[AHEAD];
    uint2 hi[AHEAD], lo[AHEAD];
    const int d = threadIdx.x % QUADS * 4, c0 = threadIdx.x / QUADS;
    constexpr int STEP = DL_GRAD_THREADS / QUADS;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      hi[i] = lo[i] = make_uint2(0u, 0u);
    }
    if (vec) {
      if (d < Dk) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
          if (c0 + i * STEP < Dv) x[i] = *reinterpret_cast<const float4*>(g + (c0 + i * STEP) * Dk + d);
      }
    } else {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const float* p = g + (c0 + i * STEP) * Dk + d;
        const int n = c0 + i * STEP < Dv ? Dk - d : 0;
        if (n > 0) x[i].x = p[0];
        if (n > 1) x[i].y = p[1];
        if (n > 2) x[i].z = p[2];
        if (n > 3) x[i].w = p[3];
      }
    }
    if (d < Dk) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (c0 + i * STEP < Dv) {
          hi[i] = *reinterpret_cast<const uint2*>(with + (c0 + i * STEP) * DK + d);
          lo[i] = *reinterpret_cast<const uint2*>(with + (rows + c0 + i * STEP) * DK + d);
        }
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int c = c0 + i * STEP;
      auto pair = [](uint32_t w) {
        __nv_bfloat162 h;
        memcpy(&h, &w, 4);
        return __bfloat1622float2(h);
      };
      const float2 h0 = pair(hi[i].x), h1 = pair(hi[i].y), l0 = pair(lo[i].x), l1 = pair(lo[i].y);
      dot = fmaf(x[i].x, h0.x + l0.x, fmaf(x[i].y, h0.y + l0.y, fmaf(x[i].z, h1.x + l1.x, fmaf(x[i].w, h1.y + l1.y, dot))));
      uint32_t a[2], b[2];
      dl_split<2>(x[i].x, x[i].y, a);
      dl_split<2>(x[i].z, x[i].w, b);
#pragma unroll
      for (int e = 0; e < 2; ++e) *reinterpret_cast<uint2*>(s + (e * DV + c) * LD + d) = make_uint2(a[e], b[e]);
    }
  }
  return dot;
}
// PARTS matrices [from][pitch] from the work, their first ROWS rows of up to PAD columns, on their way to shared memory; what is not in `rows` and `cols` becomes zeros.
template <int ROWS, int PAD, int PARTS>
__device__ __forceinline__ void dl_load_parts(bf* s, const bf* g, int from, int pitch, int rows, int cols) {
  constexpr int PIECES = PAD / 8, ROUNDS = PARTS * ROWS * PIECES / DL_GRAD_THREADS, STEP = DL_GRAD_THREADS / PIECES;
  const int c = threadIdx.x % PIECES * 8, r0 = threadIdx.x / PIECES;
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const int all = r0 + i * STEP, part = all / ROWS, r = all % ROWS;
    const bool there = c < cols && r < rows;
    dl_copy16(s + all * (PAD + 8) + c, g + (there ? (part * from + r) * pitch + c : 0), there);
  }
}

// The k-th line of 128 bytes of those that hold `bytes` from p on, on its way to L2.
__device__ __forceinline__ bool dl_ahead_line(const void* p, long long bytes, long long k) {
  const uintptr_t from = reinterpret_cast<uintptr_t>(p), at = k == 0 ? from : (from & ~(uintptr_t)127) + 128 * k;
  if (at >= from + bytes) return false;
  asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
  return true;
}
__device__ __forceinline__ void dl_ahead(const void* p, long long bytes) {
  for (long long k = threadIdx.x; dl_ahead_line(p, bytes, k); k += DL_GRAD_THREADS) {}
}
__device__ __forceinline__ void dl_ahead_rows(const bf* p, long long step, int live, int cols) {  // rows of a chunk, of up to 128 columns
  const int r = threadIdx.x >> 3;
  if (r < live) dl_ahead_line(p + r * step, 2ll * cols, threadIdx.x & 7);
}
// All that the unit of the CTA after this one on the SM reads, while this one computes: the loads of all SMs together are as fast as memory is, and nothing overlaps
// them where one CTA fills an SM.
__device__ __forceinline__ void dl_ahead(const DlArgs& a, long long at) {
  const uint32_t units = (uint32_t)a.B * (uint32_t)a.heads;
  const DlUnit u = dl_unit(a, (int)(at / units), (uint32_t)(at % units));
  if (u.live == 0) return;
  dl_ahead(a.S + u.unit * a.Dk * a.Dv, 4ll * a.Dk * a.Dv);
  dl_ahead_rows(a.K + u.row0 * a.ldk + (long long)u.head * a.Dk, a.B * a.ldk, u.live, a.Dk);
  dl_ahead_rows(a.Q + u.row0 * a.ldq + (long long)u.head * a.Dk, a.B * a.ldq, u.live, a.Dk);
  dl_ahead_rows(a.V + u.row0 * a.ldv + (long long)u.head * a.Dv, a.B * a.ldv, u.live, a.Dv);
  dl_ahead_rows(a.dY + u.row0 * a.lddy + (long long)u.head * a.Dv, a.B * a.lddy, u.live, a.Dv);
  dl_ahead(a.x + u.unit * 2 * DL_CHUNK * a.ldx, 4ll * DL_CHUNK * a.ldx);
  const long long dk = a.Dk <= 64 ? 64 : 128;
  for (int p = 0; p < 2; ++p) dl_ahead(a.d + (u.unit * 2 + p) * dk * a.ldx, 2ll * a.Dv * dk);  // of each part the rows that are read
  dl_ahead(a.tri + u.unit * 3 * DL_SQ, 4ll * DL_SQ);
  dl_ahead(a.row + u.unit * DL_ROW_FLOATS, 4ll * DL_ROW_FLOATS);
}

template <int DK, int DV>
__global__ void __launch_bounds__(DL_GRAD_THREADS) delta_grad_kernel(const DlArgs a) {
  constexpr int NK = DK / 32, NV = DV / 32;  // tiles of 8 columns a warp of [64][DK] and [64][DV] matrices
  constexpr int LDK = DK + 8, LDV = DV + 8, PV = DL_CHUNK * LDV, PM = DL_CHUNK * DL_LD64, PS = DV * LDK;
  extern __shared__ __align__(16) uint8_t dl_smem[];
  auto& sh = *reinterpret_cast<DlGradShared<DK, DV>*>(dl_smem);
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const uint32_t units = (uint32_t)a.B * (uint32_t)a.heads;
  const DlUnit u = dl_unit(a, (int)(blockIdx.x / units), blockIdx.x % units);
  const int steps = min(DL_CHUNK, a.T - u.chunk * DL_CHUNK);
  bf* dq = a.dQ + u.row0 * a.lddq + (long long)u.head * a.Dk;
  bf* dk = a.dK + u.row0 * a.lddk + (long long)u.head * a.Dk;
  dl_zero_rows(dq, a.B * a.lddq, u.live, steps, a.Dk, t, DL_GRAD_THREADS);
  dl_zero_rows(dk, a.B * a.lddk, u.live, steps, a.Dk, t, DL_GRAD_THREADS);
  if (t >= u.live && t < steps) {
    const long long z = (u.row0 + (long long)t * a.B) * a.lddz + u.head;
    a.dZf[z] = a.dZb[z] = __float2bfloat16_rn(0.f);
  }
  if (u.live == 0) return;
  dl_load<DK, DL_GRAD_THREADS>(&sh.k[0][0], LDK, a.K + u.row0 * a.ldk + (long long)u.head * a.Dk, a.B * a.ldk, u.live, a.Dk, a.vec_k, t);
  dl_load<DK, DL_GRAD_THREADS>(&sh.q[0][0], LDK, a.Q + u.row0 * a.ldq + (long long)u.head * a.Dk, a.B * a.ldq, u.live, a.Dk, a.vec_q, t);
  dl_load<DV, DL_GRAD_THREADS>(&sh.dy[0][0], LDV, a.dY + u.row0 * a.lddy + (long long)u.head * a.Dv, a.B * a.lddy, u.live, a.Dv, a.vec_dy, t);
  dl_load64<2, DL_GRAD_THREADS>(&sh.tri[0][0][0], a.tri + u.unit * 3 * DL_SQ, t);
  dl_load_row(sh.row, a.row + u.unit * DL_ROW_FLOATS, t, DL_GRAD_THREADS);
  dl_load_parts<DL_CHUNK, DV, 2>(&sh.x[0][0][0], a.x + u.unit * 2 * DL_CHUNK * a.ldx, DL_CHUNK, a.ldx, DL_CHUNK, a.Dv);
  dl_commit();
  // this warp's tile; where work grows or falls with the row, the warps of a scheduler have the same between them
  const int group = warp >> 2, m0 = (group < 2 ? warp & 3 : 3 - (warp & 3)) * 16;
  const int nk0 = group * NK * 8, nv0 = group * NV * 8, nm0 = group * 16;
  const int r0 = m0 + (lane >> 2), cl = 2 * (lane & 3);
  uint32_t v[NV][2];  // pairs of V
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = r0 + 8 * h;
    const bf* p = a.V + (u.row0 + (long long)r * a.B) * a.ldv + (long long)u.head * a.Dv + nv0 + cl;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = nv0 + 8 * i + cl;
      v[i][h] = 0u;
      if (r >= u.live || c >= a.Dv) continue;
      if (a.vec_v) {
        v[i][h] = *reinterpret_cast<const uint32_t*>(p + 8 * i);
      } else {
        bf e[2] = {p[8 * i], c + 1 < a.Dv ? p[8 * i + 1] : __float2bfloat16_rn(0.f)};
        memcpy(&v[i][h], e, 4);
      }
    }
  }
  const bf* D = a.d + u.unit * 2 * DK * a.ldx;
  float dot = dl_load_state<DK, DV>(&sh.s[0][0][0], a.S + u.unit * a.Dk * a.Dv, a.Dk, a.Dv, a.vec_s, D, a.ldx);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, o);
  if (lane == 0) sh.ds[warp] = dot;
  dl_wait<0>();
  if (blockIdx.x + (long long)a.ahead < gridDim.x) dl_ahead(a, blockIdx.x + (long long)a.ahead);
  __syncthreads();
  auto row_sums = [&](int which, const float (&x)[1][NK][4], const bf* with, const float* by, bool more) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const float2 w = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(with + (r0 + 8 * h) * LDK + nk0 + 8 * i + cl));
        s = fmaf(x[0][i][2 * h], w.x, fmaf(x[0][i][2 * h + 1], w.y, s));
      }
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 1);
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 2);
      s *= by[r0 + 8 * h];
      if ((lane & 3) == 0) sh.red[which][group][r0 + 8 * h] = more ? sh.red[which][group][r0 + 8 * h] + s : s;
    }
  };
  {
    float e[1][NV][4] = {};
    dl_product<1, NV, false, false, 1, 2, 1>(e, &sh.k[0][0], LDK, 0, &sh.s[0][0][0], LDK, PS, m0, nv0, 0, DK, lane);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = r0 + 8 * h;
        const float b = sh.row.beta[r], g = -sh.row.kin[r];
        const float2 x = dl_unpack(v[i][h]);
        dl_put<2>(&sh.u[0][r][nv0 + 8 * i + cl], PV, b * fmaf(g, e[0][i][2 * h], x.x), b * fmaf(g, e[0][i][2 * h + 1], x.y));
      }
  }
  float aq[1][NK][4] = {}, ak[1][NK][4] = {};
#pragma unroll 2
  for (int k = 0; k < DV; k += 16) {
    uint32_t dy[4], x[2][4];
    dl_a<false>(dy, &sh.dy[0][0], LDV, m0, k, lane);
#pragma unroll
    for (int p = 0; p < 2; ++p) dl_a<false>(x[p], &sh.x[p][0][0], LDV, m0, k, lane);
#pragma unroll
    for (int n = 0; n < NK; n += 2) {
      uint32_t w[2][4];
#pragma unroll
      for (int p = 0; p < 2; ++p) dl_b<true>(w[p], &sh.s[p][0][0], LDK, nk0 + 8 * n, k, lane);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        dl_mma(aq[0][n + e], dy, w[1][2 * e], w[1][2 * e + 1]);
        dl_mma(ak[0][n + e], x[0], w[1][2 * e], w[1][2 * e + 1]);
        dl_mma(aq[0][n + e], dy, w[0][2 * e], w[0][2 * e + 1]);
        dl_mma(ak[0][n + e], x[1], w[0][2 * e], w[0][2 * e + 1]);
        dl_mma(ak[0][n + e], x[0], w[0][2 * e], w[0][2 * e + 1]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NK; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float g = sh.row.first[r0 + 8 * (e >> 1)];
      aq[0][i][e] *= a.scale * g;
      ak[0][i][e] *= -g * sh.row.beta[r0 + 8 * (e >> 1)];
    }
  row_sums(0, aq, &sh.q[0][0], sh.row.rq, false);
  row_sums(0, ak, &sh.k[0][0], sh.row.rk, true);
  __syncthreads();
  dl_load_parts<DV, DK, 2>(&sh.s[0][0][0], D, a.ldx, DK, a.Dv, DK);  // D, where S_0 was
  dl_commit();
  {
    float x[1][NV][4] = {};
    dl_product<1, NV, false, true, 2, 2, 1>(x, &sh.tri[0][0][0], DL_LD64, PM, &sh.u[0][0][0], LDV, PV, m0, nv0, 0, m0 + 16, lane);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) dl_put<2>(&sh.u[0][r0 + 8 * h][nv0 + 8 * i + cl], PV, x[0][i][2 * h], x[0][i][2 * h + 1]);
  }
  __syncthreads();
  {  // X.U: eight threads a row
    const int r = t >> 3, part = t & 7;
    float xu = 0.f;
#pragma unroll
    for (int c = part * 2; c < DV; c += 16) {
      auto both = [&](bf (&m)[2][DL_CHUNK][DV + 8]) {
        const float2 h = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&m[0][r][c])), l = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&m[1][r][c]));
        return make_float2(h.x + l.x, h.y + l.y);
      };
      const float2 x = both(sh.x), y = both(sh.u);
      xu = fmaf(x.x, y.x, fmaf(x.y, y.y, xu));
    }
#pragma unroll
    for (int o = 1; o < 8; o *= 2) xu += __shfl_xor_sync(0xFFFFFFFFu, xu, o);
    if (part == 0) sh.xu[r] = xu;
  }
  float nn[1][2][4] = {}, mm[1][2][4] = {};
  if (nm0 <= m0) {
    float qk[1][2][4] = {}, kk[1][2][4] = {};
    // two products at a time share their right operand, and are more sums for the tensor pipe to go on with
#pragma unroll 4
    for (int k = 0; k < DV; k += 16) {
      uint32_t dy[4], x[2][4], w[2][4];
      dl_a<false>(dy, &sh.dy[0][0], LDV, m0, k, lane);
#pragma unroll
      for (int p = 0; p < 2; ++p) dl_a<false>(x[p], &sh.x[p][0][0], LDV, m0, k, lane), dl_b<false>(w[p], &sh.u[p][0][0], LDV, nm0, k, lane);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        dl_mma(nn[0][n], dy, w[1][2 * n], w[1][2 * n + 1]);
        dl_mma(mm[0][n], x[0], w[1][2 * n], w[1][2 * n + 1]);
        dl_mma(nn[0][n], dy, w[0][2 * n], w[0][2 * n + 1]);
        dl_mma(mm[0][n], x[1], w[0][2 * n], w[0][2 * n + 1]);
        dl_mma(mm[0][n], x[0], w[0][2 * n], w[0][2 * n + 1]);
      }
    }
#pragma unroll 4
    for (int k = 0; k < DK; k += 16) {
      uint32_t q[4], key[4], w[4];
      dl_a<false>(q, &sh.q[0][0], LDK, m0, k, lane);
      dl_a<false>(key, &sh.k[0][0], LDK, m0, k, lane);
      dl_b<false>(w, &sh.k[0][0], LDK, nm0, k, lane);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        dl_mma(qk[0][n], q, w[2 * n], w[2 * n + 1]);
        dl_mma(kk[0][n], key, w[2 * n], w[2 * n + 1]);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = r0 + 8 * h, bi = m0 >> 4;
      const float rqi = sh.row.rq[i], rki = sh.row.rk[i], beta = sh.row.beta[i];
      float across = sh.row.from[i];
      for (int b = group + 1; b < bi; ++b) across *= sh.row.block[b];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int j = nm0 + 8 * n + cl + e;
          const float g = group < bi ? across * sh.row.to[j] : sh.row.diag[bi][i & 15][j & 15];
          float &x = nn[0][n][2 * h + e], &y = mm[0][n][2 * h + e];
          x = j <= i ? x * a.scale * g : 0.f;
          y = j < i ? y * -beta * g : 0.f;
          sh.w[i][j] = j < i ? sh.row.rk[j] * fmaf(x * rqi, qk[0][n][2 * h + e], y * rki * kk[0][n][2 * h + e]) : 0.f;
        }
    }
  } else {
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) sh.w[r0 + 8 * (e >> 1)][nm0 + 8 * n + cl + (e & 1)] = 0.f;
  }
  dl_wait<0>();
  __syncthreads();
  {
    float x[1][NK][4] = {};
    dl_product<1, NK, false, true, 2, 2, 1>(x, &sh.u[0][0][0], LDV, PV, &sh.s[0][0][0], LDK, PS, m0, nk0, 0, DV, lane);
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[0][i][e] *= sh.row.last[r0 + 8 * (e >> 1)];
        ak[0][i][e] += x[0][i][e];
      }
    row_sums(1, x, &sh.k[0][0], sh.row.rk, false);
  }
  {  // W summed over later rows, in blocks of eight
    const int j = t & 63, b = t >> 6;
    float s = 0.f;
#pragma unroll
    for (int i = 7; i >= 0; --i) sh.w[8 * b + i][j] = s += sh.w[8 * b + i][j];
    sh.over[b][j] = s;
  }
  __syncthreads();
  if (nm0 <= m0) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = r0 + 8 * h;
      const float rq = sh.row.rq[i], rk = sh.row.rk[i];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int j = nm0 + 8 * n + cl;
        const float x = nn[0][n][2 * h], y = nn[0][n][2 * h + 1], z0 = mm[0][n][2 * h], z1 = mm[0][n][2 * h + 1], rk0 = sh.row.rk[j], rk1 = sh.row.rk[j + 1];
        dl_put<2>(&sh.m[0][0][i][j], PM, x * rk0, y * rk1);
        dl_put<2>(&sh.m[1][0][i][j], PM, x * rq, y * rq);
        uint32_t lo[2], up[2];
        dl_split<2>(z0 * rk0, z1 * rk1, lo);
        dl_split<2>(z0 * rk, z1 * rk, up);
        const int r = nm0 + 8 * n + (lane >> 2), c = m0 + 8 * h + cl;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          const uint32_t w = dl_transposed(up[part]);
          // on the diagonal of 8 x 8 blocks both halves meet in one word, each zero where the other is not
          if (nm0 == m0 && h == n) {
            *reinterpret_cast<uint32_t*>(&sh.m[2][part][i][j]) = lo[part] | w;
          } else if (nm0 < m0 || h > n) {
            *reinterpret_cast<uint32_t*>(&sh.m[2][part][i][j]) = lo[part];
            *reinterpret_cast<uint32_t*>(&sh.m[2][part][r][c]) = w;
          }
        }
      }
    }
  }
  {  // what passes gate r: eight threads
    const int r = t >> 3, part = t & 7;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = part + 8 * e;
      if (j >= r) continue;
      s += sh.w[r][j];
      for (int b = (r >> 3) + 1; b < 8; ++b) s += sh.over[b][j];
    }
#pragma unroll
    for (int o = 1; o < 8; o *= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (part == 0) sh.seen[r] = s;
  }
  __syncthreads();
  dl_product<1, NK, false, true, 2, 1, 1>(aq, &sh.m[0][0][0][0], DL_LD64, PM, &sh.k[0][0], LDK, 0, m0, nk0, 0, m0 + 16, lane);
  dl_product<1, NK, true, true, 2, 1, 1>(ak, &sh.m[1][0][0][0], DL_LD64, PM, &sh.q[0][0], LDK, 0, m0, nk0, m0, DL_CHUNK, lane);
  dl_product<1, NK, false, true, 2, 1, 1>(ak, &sh.m[2][0][0][0], DL_LD64, PM, &sh.k[0][0], LDK, 0, m0, nk0, 0, DL_CHUNK, lane);
  row_sums(2, aq, &sh.q[0][0], sh.row.rq, false);
  row_sums(3, ak, &sh.k[0][0], sh.row.rk, false);
  __syncthreads();
  auto red = [&](int which, int r) { return (sh.red[which][0][r] + sh.red[which][1][r]) + (sh.red[which][2][r] + sh.red[which][3][r]); };
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = r0 + 8 * h;
    if (r >= u.live) continue;
    const float rq = sh.row.rq[r], rk = sh.row.rk[r];
    // q of length one gives up what its gradient has along it
    const float along_q = a.eps < 0.f ? 0.f : red(2, r) * rq, along_k = a.eps < 0.f ? 0.f : red(3, r) * rk;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int c = nk0 + 8 * i + cl;
      if (c >= a.Dk) continue;
      const float2 q = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&sh.q[r][c])), k = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&sh.k[r][c]));
      dl_store2(dq + (long long)r * a.B * a.lddq + c, rq * fmaf(-along_q, q.x, aq[0][i][2 * h]), rq * fmaf(-along_q, q.y, aq[0][i][2 * h + 1]), c + 1 < a.Dk);
      dl_store2(dk + (long long)r * a.B * a.lddk + c, rk * fmaf(-along_k, k.x, ak[0][i][2 * h]), rk * fmaf(-along_k, k.y, ak[0][i][2 * h + 1]), c + 1 < a.Dk);
    }
  }
  if (warp == 0) {  // lane: steps lane and 32 + lane
    float ds = 0.f;
#pragma unroll
    for (int w = 0; w < DL_GRAD_WARPS; ++w) ds += sh.ds[w];
    ds *= sh.row.first[DL_CHUNK - 1];
    float x0 = red(0, lane), x1 = red(0, 32 + lane);           // a: sums from here on
    const float c0 = red(1, lane), c1 = red(1, 32 + lane);
    float y0 = c0, y1 = c1;                                    // c: sums up to here
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const float dx0 = __shfl_down_sync(0xFFFFFFFFu, x0, o), dx1 = __shfl_down_sync(0xFFFFFFFFu, x1, o);
      const float dy0 = __shfl_up_sync(0xFFFFFFFFu, y0, o), dy1 = __shfl_up_sync(0xFFFFFFFFu, y1, o);
      if (lane + o < 32) x0 += dx0, x1 += dx1;
      if (lane >= o) y0 += dy0, y1 += dy1;
    }
    x0 += __shfl_sync(0xFFFFFFFFu, x1, 0);
    y1 += __shfl_sync(0xFFFFFFFFu, y0, 31);
    // c of the step itself does not pass its own gate; taken off by the neighbour's sum, not by a difference
    const float before0 = __shfl_up_sync(0xFFFFFFFFu, y0, 1), before1 = __shfl_up_sync(0xFFFFFFFFu, y1, 1), half = __shfl_sync(0xFFFFFFFFu, y0, 31);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = lane + 32 * h;
      const float c = lane > 0 ? (h ? before1 : before0) : h ? half : 0.f;
      if (r >= u.live) continue;
      const long long z = (u.row0 + (long long)r * a.B) * a.lddz + u.head;
      a.dZf[z] = __float2bfloat16_rn((sh.seen[r] + (h ? x1 : x0) + c + ds) * sh.row.rest[r]);
      a.dZb[z] = __float2bfloat16_rn(sh.xu[r] * sh.row.closed[r]);
    }
  }
}

// Heads without keys' or without values' columns: sums over nothing, and gates that nothing depends on.
struct DlZeros {
  bf* p[5];
  long long step[5];
  int cols[5];
};
__global__ void __launch_bounds__(DL_THREADS) delta_zeros_kernel(const DlZeros z, long long rows) {
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  for (int m = 0; m < 5; ++m)
    for (long long i = (long long)blockIdx.x * DL_THREADS + threadIdx.x; i < rows * z.cols[m]; i += (long long)gridDim.x * DL_THREADS)
      z.p[m][i / z.cols[m] * z.step[m] + i % z.cols[m]] = __float2bfloat16_rn(0.f);
}

// Up to so many steps go one by one, which needs no workspace: 17 steps of 64 x 8 states of 128 x 128 take 83 us so and 86 as a chunk, of 4 x 8 states 33 and 21 (there 9
// steps would be the edge).
constexpr int DL_STEPS = 16;

inline bool dl_on16(const void* p, long long ld, int head) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && head % 8 == 0; }
inline long long dl_units(int T, int B, int heads) { return (long long)((T + DL_CHUNK - 1) / DL_CHUNK) * B * heads; }

// Where a unit's parts lie in the work, in bytes from its start (all units of a kind side by side, each on 256 bytes).
struct DlPlan {
  size_t tri, p, row, x, d, bytes;
};
inline int dl_ldx(int Dv) { return Dv <= 64 ? 64 : 128; }
DlPlan dl_plan(int T, int B, int heads, int Dk, int Dv, bool backward) {
  const size_t units = (size_t)dl_units(T, B, heads), pitch = (size_t)dl_ldx(Dv) * 2;
  DlPlan w;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (units * bytes + 255) / 256 * 256;
    return here;
  };
  w.tri = take(3 * DL_SQ * 2);
  w.p = take(3 * DL_SQ * 2);
  w.row = take(sizeof(DlRow));
  w.x = take(backward ? 2 * DL_CHUNK * pitch : 0);
  w.d = take(backward ? 2 * (Dk <= 64 ? 64 : 128) * pitch : 0);
  w.bytes = at + 256;  // the caller's memory may begin anywhere
  return w;
}
void dl_set_work(DlArgs& a, void* work, const DlPlan& w) {
  uint8_t* p = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(work) + 255) & ~(uintptr_t)255);
  a.tri = reinterpret_cast<bf*>(p + w.tri);
  a.p = reinterpret_cast<bf*>(p + w.p);
  a.row = reinterpret_cast<float*>(p + w.row);
  a.x = reinterpret_cast<bf*>(p + w.x);
  a.d = reinterpret_cast<bf*>(p + w.d);
  a.ldx = dl_ldx(a.Dv);
}

template <typename K>
ard_status dl_run(ard_ctx* ctx, K kern, long long grid, int threads, size_t smem, const DlArgs& a, cudaStream_t s) {
  ARD_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  ARD_CUDA_OK(ard_launch(ctx, kern, dim3((unsigned)grid), dim3(threads), smem, s, a));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}
ard_status dl_zeros(ard_ctx* ctx, const DlZeros& z, long long rows, cudaStream_t s) {
  int most = 0;
  for (int cols : z.cols) most = cols > most ? cols : most;
  if (rows == 0 || most == 0) return ARD_OK;
  const long long want = (rows * most + DL_THREADS - 1) / DL_THREADS, room = 8ll * ctx->sm_count;
  ARD_CUDA_OK(ard_launch(ctx, delta_zeros_kernel, dim3((unsigned)(want < room ? want : room)), dim3(DL_THREADS), 0, s, z, rows));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}
template <int DK, int NP>
ard_status dl_scan(ard_ctx* ctx, const DlArgs& a, bool backward, cudaStream_t s) {
  const long long grid = (long long)a.B * a.heads * ((a.Dv + NP * 16 - 1) / (NP * 16));
  return backward ? dl_run(ctx, delta_back_kernel<DK, NP>, grid, DlTeams<NP>::ALL, sizeof(DlBackShared<DK, NP>), a, s)
                  : dl_run(ctx, delta_scan_kernel<DK, NP>, grid, DlTeams<NP>::ALL, sizeof(DlScanShared<DK, NP>), a, s);
}
template <int DK>
ard_status dl_chunks(ard_ctx* ctx, const DlArgs& a, bool backward, cudaStream_t s) {
  const long long units = dl_units(a.T, a.B, a.heads), groups = (a.Dv + 15) / 16, pairs = (long long)a.B * a.heads * groups;
  ard_status st = dl_run(ctx, delta_prep_kernel<DK>, units, DL_THREADS, sizeof(DlPrepShared<DK>), a, s);
  if (st != ARD_OK) return st;
  // columns go to as many SMs as there are, at most 64 to one
  if (groups == 1 || pairs <= ctx->sm_count) st = dl_scan<DK, 1>(ctx, a, backward, s);
  else if (groups == 2 || pairs <= 2ll * ctx->sm_count) st = dl_scan<DK, 2>(ctx, a, backward, s);
  else st = dl_scan<DK, 4>(ctx, a, backward, s);
  if (st != ARD_OK || !backward) return st;
  if (a.Dv <= 64) return dl_run(ctx, delta_grad_kernel<DK, 64>, units, DL_GRAD_THREADS, sizeof(DlGradShared<DK, 64>), a, s);
  return dl_run(ctx, delta_grad_kernel<DK, 128>, units, DL_GRAD_THREADS, sizeof(DlGradShared<DK, 128>), a, s);
}
ard_status dl_chunks(ard_ctx* ctx, const DlArgs& a, bool backward, cudaStream_t s) {
  return a.Dk <= 64 ? dl_chunks<64>(ctx, a, backward, s) : dl_chunks<128>(ctx, a, backward, s);
}

static_assert(sizeof(DlGradShared<128, 128>) <= 227 * 1024 && sizeof(DlBackShared<128, 4>) <= 227 * 1024 && sizeof(DlScanShared<128, 4>) <= 227 * 1024,
              "shared memory of an SM");

}  // namespace

size_t delta_work_bytes(int T, int B, int heads, int Dk, int Dv, bool backward) {
  if (T == 0 || B == 0 || heads == 0 || Dk == 0 || Dv == 0 || (!backward && T <= DL_STEPS)) return 0;
  return dl_plan(T, B, heads, Dk, Dv, backward).bytes;
}

ard_status launch_delta_forward(ard_ctx* ctx, int T, int B, int heads, int Dk, int Dv, float scale, float eps, const void* Q, int ldq, const void* K, int ldk,
                                const void* V, int ldv, const void* Zf, const void* Zb, int ldz, const int32_t* lens, const float* h0, void* Y, int ldy,
                                float* hT, float* S, void* work, cudaStream_t s) {
  if (B == 0 || heads == 0 || Dv == 0) return ARD_OK;
  if (Dk == 0) return dl_zeros(ctx, {{(bf*)Y}, {ldy}, {heads * Dv}}, (long long)T * B, s);
  DlArgs a = {};
  a.T = T, a.B = B, a.heads = heads, a.Dk = Dk, a.Dv = Dv, a.scale = scale, a.eps = eps;
  a.Q = (const bf*)Q, a.K = (const bf*)K, a.V = (const bf*)V, a.ldq = ldq, a.ldk = ldk, a.ldv = ldv;
  a.Zf = (const bf*)Zf, a.Zb = (const bf*)Zb, a.ldz = ldz;
  a.lens = lens, a.h0 = h0, a.Y = (bf*)Y, a.ldy = ldy, a.hT = hT, a.S = S;
  a.vec_q = dl_on16(Q, ldq, Dk), a.vec_k = dl_on16(K, ldk, Dk), a.vec_v = dl_on16(V, ldv, Dv);
  if (T <= DL_STEPS) {
    auto on16 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
    const bool vec = Dv % 4 == 0 && on16(h0) && on16(hT) && on16(S);
    ARD_CUDA_OK(ard_launch(ctx, vec ? delta_steps_kernel<true> : delta_steps_kernel<false>, dim3((unsigned)((long long)B * heads)), dim3(DL_THREADS), 0, s, a));
    ctx->launches++;
    ARD_CUDA_OK(cudaGetLastError());
    return ARD_OK;
  }
  dl_set_work(a, work, dl_plan(T, B, heads, Dk, Dv, false));
  return dl_chunks(ctx, a, false, s);
}

ard_status launch_delta_backward(ard_ctx* ctx, int T, int B, int heads, int Dk, int Dv, float scale, float eps, const void* Q, int ldq, const void* K, int ldk,
                                 const void* V, int ldv, const void* Zf, const void* Zb, int ldz, const int32_t* lens, const float* S, const void* dY,
                                 int lddy, const float* dhT, void* dQ, int lddq, void* dK, int lddk, void* dV, int lddv, void* dZf, void* dZb, int lddz,
                                 float* dh0, void* work, cudaStream_t s) {
  if (B == 0 || heads == 0) return ARD_OK;
  if (Dk == 0 || Dv == 0)
    return dl_zeros(ctx, {{(bf*)dQ, (bf*)dK, (bf*)dV, (bf*)dZf, (bf*)dZb}, {lddq, lddk, lddv, lddz, lddz}, {heads * Dk, heads * Dk, heads * Dv, heads, heads}},
                    (long long)T * B, s);
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
  a.vec_v = dl_on16(V, ldv, Dv);
  a.vec_s = Dk % 4 == 0 && (reinterpret_cast<uintptr_t>(S) & 15u) == 0;
  dl_set_work(a, work, dl_plan(T, B, heads, Dk, Dv, true));
  a.ahead = ctx->sm_count;
  return dl_chunks(ctx, a, true, s);
}
