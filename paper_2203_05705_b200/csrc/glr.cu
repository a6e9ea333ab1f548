// The gated linear recurrence over whole sequences, forward and adjoint:
//   f_t = s(zf_t),  c_t = f_t c_{t-1} + (1 - f_t) g_t,  y_t = alpha s(zo_t) c_t
//   d_t = alpha s(zo_t) dy_t + q_t,  q_{t-1} = f_t d_t,
//   dzo_t = alpha dy_t c_t s(zo_t) (1 - s(zo_t)),  dzf_t = d_t (c_{t-1} - g_t) f_t (1 - f_t),  dzg_t = d_t (1 - f_t).
//
// Both recurrences are compositions of maps x -> A x + B, so the time axis can be cut: a thread holds SPT steps of its
// channels in registers, composes their map, and applies the steps once it knows the state that enters them.  The maps of a slab's
// warps meet in shared memory, those of consecutive slabs in the shared memory of a cluster of CTAs (few channels, long
// sequences), so gates are read once and outputs written once.  The adjoint starts its states from those that the forward call left
// every ARD_GLR_CHUNK steps and computes the ones between again: 4 bytes in 64 steps in place of 4 in each.
#include <cooperative_groups.h>

#include <initializer_list>
#include <utility>

#include "ard_internal.h"
#include "sm100_ptx.h"

namespace {

namespace cg = cooperative_groups;

constexpr int GLR_CLUSTER = 8;  // most CTAs that share a sequence

struct GlrArgs {
  const int32_t* hdr;  // nullptr: all H units
  int T, B, H;
  float alpha;
  const void *Zf, *Zg, *Zo;
  int ldz;
  const int32_t* lens;
  const float* h0;  // backward: dhT
  const void* dY;
  void* Y;
  int ldy;
  float* hT;  // backward: dh0
  float* S;
  void *dZf, *dZg, *dZo;
  int lddz;
  int* status;
};

// exp(x) and 1 / x to about two units in the last place, results below the normal range zero (x in range otherwise): the forms that keep
// subnormals cost five instructions each, of which a gate has two.
__device__ __forceinline__ float glr_exp(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.44269504f));
  return r;
}
__device__ __forceinline__ float glr_inverse(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// s(z), and 1 - s(z), each to the last bits of its own: where s(z) is above a half the other one is exp(-z) times it, not a difference.  exp(-z) of
// infinity gives 0 and 1.
__device__ __forceinline__ float glr_gate(float z) { return glr_inverse(1.f + glr_exp(-z)); }
__device__ __forceinline__ float glr_gate(float z, float& rest) {
  const float u = glr_exp(-z), f = glr_inverse(1.f + u);
  rest = z >= 0.f ? u * f : 1.f - f;
  return f;
}

// VEC channels of one step as they lie in memory, in one register.
template <typename T, int VEC>
__device__ __forceinline__ uint32_t glr_fetch(const T* p) {
  uint32_t q;
  if constexpr (sizeof(T) * VEC == 4) {
    asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(q) : "l"(p));
  } else {
    uint16_t h;
    asm volatile("ld.global.L1::no_allocate.u16 %0, [%1];" : "=h"(h) : "l"(p));
    q = h;
  }
  return q;
}
template <typename T, int VEC>
__device__ __forceinline__ void glr_unpack(uint32_t q, float (&v)[VEC]) {
  if constexpr (sizeof(T) == 4) {
    v[0] = __uint_as_float(q);
  } else {
    v[0] = __uint_as_float(q << 16);
    if constexpr (VEC == 2) v[1] = __uint_as_float(q & 0xFFFF0000u);
  }
}
// The first `valid` of the values.
template <typename T, int VEC>
__device__ __forceinline__ void glr_store(T* p, int valid, const float (&v)[VEC]) {
  if constexpr (VEC == 2) {
    if (valid >= 2) {
      *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(v[0], v[1]);
      return;
    }
  }
  if (valid >= 1) {
    if constexpr (sizeof(T) == 4) *p = v[0];
    else *p = __float2bfloat16(v[0]);
  }
}

// Maps x -> A x + B of a lane's channels: [A, B][channel].
template <int VEC>
struct GlrMap {
  float a[VEC], b[VEC];
  __device__ __forceinline__ static GlrMap none() {
    GlrMap m;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      m.a[v] = 1.f;
      m.b[v] = 0.f;
    }
    return m;
  }
  // this one, then `next`
  __device__ __forceinline__ void then(const GlrMap& next) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      a[v] *= next.a[v];
      b[v] = fmaf(next.a[v], b[v], next.b[v]);
    }
  }
  __device__ __forceinline__ float of(float x, int v) const { return fmaf(a[v], x, b[v]); }
};

// What the kernels run over: units of CW * 32 * VEC channels of one sequence, `rounds` times CL slabs of WT * SPT steps each.
struct GlrSpan {
  int n, dp, b0, groups, units, rounds;
  __device__ __forceinline__ GlrSpan(const GlrArgs& a, int channels, int steps) {
    n = a.H;
    dp = 1;
    b0 = 0;
    if (a.hdr) {
      n = a.hdr[HDR_NKEEP];
      dp = a.hdr[HDR_DP];
      b0 = a.hdr[HDR_B] - 1;
    }
    groups = (n + channels - 1) / channels;
    units = groups * a.B;
    rounds = (a.T + steps - 1) / steps;
  }
  __device__ __forceinline__ int len(const GlrArgs& a, int b) const { return a.lens ? min(max(a.lens[b], 0), a.T) : a.T; }
};
// A thread's place in a unit: VEC channels of one sequence, SPT consecutive steps of every slab.
template <int VEC, int CW, int WT>
struct GlrPlace {
  int wt, ch, b, j, valid, col, len;
  __device__ __forceinline__ GlrPlace(const GlrArgs& a, const GlrSpan& sp, int unit) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    wt = warp % WT;
    ch = warp / WT * 32 + lane;
    b = unit / sp.groups;
    j = ((unit - b * sp.groups) * CW * 32 + ch) * VEC;
    valid = max(0, min(VEC, sp.n - j));
    col = min(j, (sp.n - 1) / VEC * VEC);  // where a lane without channels reads
    len = sp.len(a, b);
  }
  __device__ __forceinline__ size_t of(const GlrArgs& a, const GlrSpan& sp, int v) const {
    return (size_t)b * a.H + sp.b0 + (size_t)(j + v) * sp.dp;
  }
};

// Where M operands of a slab come from.  BULK: tiles [WT * SPT steps][32 * VEC channels] that the copy engine brings into a ring of
// slots, several slabs ahead and over the ends of units (rows of 16-byte aligned pieces).  Otherwise registers, into which a
// thread fetches its own values of the unit's next slab as soon as this one's are used.
struct GlrTiles {
  CUtensorMap map[4];
};
template <typename T, int VEC, int M, int WT, int SPT, bool BULK>
struct GlrFeed;

template <typename T, int VEC, int M, int WT, int SPT>
struct GlrFeed<T, VEC, M, WT, SPT, true> {
  static constexpr int ROW = 32 * VEC * (int)sizeof(T), TILE = WT * SPT * ROW, SLOT = M * TILE;
  static constexpr int SLOTS = M == 4 ? 2 : 3;  // two CTAs an SM with 64 to 72 KB each
  uint8_t* slots;
  uint64_t* full;
  int taken, slot, phase;       // slabs so far, and where the one that is being worked on lies
  int asked, unit, round, len;  // of the next one to ask for (thread 0)
  bool gone;                    // a copy did not come within two seconds: the outputs are unspecified, the status says so
  volatile int* s_gone;

  __device__ __forceinline__ GlrFeed(uint8_t* smem, uint64_t* bars, volatile int* g, int first)
      : slots(smem), full(bars), taken(0), slot(0), phase(0), asked(0), unit(first), round(0), len(0), gone(false), s_gone(g) {}

  __device__ __forceinline__ void ask(const GlrArgs& a, const GlrSpan& sp, const GlrTiles& tiles, int CL, int rank, int clusters, bool backward) {
    if (unit >= sp.units || gone) return;
    if (round == 0) len = sp.len(a, unit / sp.groups);
    const int ts = (backward ? sp.rounds * CL - 1 - (round * CL + rank) : round * CL + rank) * (WT * SPT);
    const int to = asked++ % SLOTS;
    const uint32_t bar = smem_u32(&full[to]), dst = smem_u32(slots + to * SLOT);
    if (ts < len) {
      const int b = unit / sp.groups, x = (unit - b * sp.groups) * 32 * VEC;
      mbar_arrive_expect_tx(bar, SLOT);
#pragma unroll
      for (int m = 0; m < M; ++m)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst + m * TILE),
            "l"(&tiles.map[m]), "r"(bar), "r"(x), "r"(b), "r"(ts)
            : "memory");
    } else {
      mbar_arrive(bar);  // nothing of the slab is used
    }
    if (++round == sp.rounds) {
      round = 0;
      unit += clusters;
    }
  }
  __device__ __forceinline__ void wait(int* status) {
    if (!gone && !mbar_wait(smem_u32(&full[slot]), (uint32_t)phase, s_gone, status)) gone = true;
  }
  __device__ __forceinline__ void next() {
    if (!gone) ++taken;
    if (++slot == SLOTS) {
      slot = 0;
      phase ^= 1;
    }
  }
  // Before a CTA ends whose copies did not come: they get the same time again, for they write to its memory.
  __device__ __forceinline__ void drain() const {
    for (int k = taken; gone && k < asked; ++k) {
      bool ok = false;
      for (int poll = 0; poll < 2000 && !ok; ++poll) ok = mbar_try_wait_hint(smem_u32(&full[k % SLOTS]), (uint32_t)(k / SLOTS) & 1u, 1000000u);
    }
  }
  __device__ __forceinline__ uint32_t raw(int wt, int m, int k) const {  // CW = 1
    const uint8_t* p = slots + slot * SLOT + m * TILE + (wt * SPT + k) * ROW + (threadIdx.x & 31) * (VEC * (int)sizeof(T));
    return *reinterpret_cast<const uint32_t*>(p);
  }
};
template <typename T, int VEC, int M, int WT, int SPT>
struct GlrFeed<T, VEC, M, WT, SPT, false> {
  uint32_t q[M][SPT];
  const T* src[M];
  size_t step[M];
  __device__ __forceinline__ GlrFeed(uint8_t*, uint64_t*, volatile int*, int) {}
  __device__ __forceinline__ void fetch(int t0, int len) {
    if (t0 >= len) return;
#pragma unroll
    for (int k = 0; k < SPT; ++k)
#pragma unroll
      for (int m = 0; m < M; ++m)  // behind the end: the last row, whose values are not used
        q[m][k] = glr_fetch<T, VEC>(src[m] + (size_t)min(t0 + k, len - 1) * step[m]);
  }
  __device__ __forceinline__ uint32_t raw(int, int m, int k) const { return q[m][k]; }
};

// The exchange of a slab: from this thread's map and the state x that enters the round, the state that enters this thread's steps and, in x, the
// one behind the round.  The warps' maps are in s_warp, and a barrier has been passed.  The cluster's CTAs send each other their slabs' maps
// by asynchronous stores that count on the receiver's barrier: a barrier of the cluster would wait for the outputs' stores, 2 us a round.
// Every CTA hears from all of them in every round, so none is more than a round ahead and two sets of places are enough.
template <int VEC, int CW>
struct GlrMail {
  GlrMap<VEC> box[2][GLR_CLUSTER][CW * 32];
  uint64_t bar[2];
};
template <int VEC>
__device__ __forceinline__ void glr_send(GlrMap<VEC>* box, uint64_t* bar, int r, const GlrMap<VEC>& m) {
  uint32_t dst, rbar;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst) : "r"(smem_u32(box)), "r"(r));
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(rbar) : "r"(smem_u32(bar)), "r"(r));
  if constexpr (VEC == 2)
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(dst), "f"(m.a[0]),
                 "f"(m.a[1]), "f"(m.b[0]), "f"(m.b[1]), "r"(rbar)
                 : "memory");
  else
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(dst), "f"(m.a[0]), "f"(m.b[0]),
                 "r"(rbar)
                 : "memory");
}
// `mail`: rounds of the cluster so far.
template <int VEC, int CW, int WT>
__device__ __forceinline__ void glr_exchange(int wt, int ch, int mail, int set, int CL, int rank, bool forward, const GlrMap<VEC>& mine,
                                             const GlrMap<VEC> (*s_warp)[WT][CW * 32], GlrMail<VEC, CW>* post, float (&x)[VEC], float (&enters)[VEC],
                                             volatile int* s_gone, int* status) {
  GlrMap<VEC> before = GlrMap<VEC>::none(), all = mine;
  if constexpr (WT > 1) {
    all = before;
#pragma unroll
    for (int k = 0; k < WT; ++k) {
      const int w = forward ? k : WT - 1 - k;
      if (w == wt) before = all;
      all.then(s_warp[set][w][ch]);
    }
  }
  if (CL > 1) {
    const int p = mail & 1;
    if (wt == 0)
      for (int r = 0; r < CL; ++r) glr_send<VEC>(&post->box[p][rank][ch], &post->bar[p], r, all);
    if (threadIdx.x == 0) mbar_arrive_expect_tx(smem_u32(&post->bar[p]), (uint32_t)(CL * CW * 32 * sizeof(GlrMap<VEC>)));
    mbar_wait(smem_u32(&post->bar[p]), (uint32_t)(mail >> 1) & 1u, s_gone, status);
    for (int r = 0; r < CL; ++r) {
      const GlrMap<VEC> m = post->box[p][r][ch];
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        if (r == rank) enters[v] = x[v];
        x[v] = m.of(x[v], v);
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      enters[v] = x[v];
      x[v] = all.of(x[v], v);
    }
  }
#pragma unroll
  for (int v = 0; v < VEC; ++v) enters[v] = before.of(enters[v], v);
}

// Shared memory and barriers of either kernel, before it touches global memory.
template <int VEC, int CW>
__device__ __forceinline__ void glr_setup(int CL, GlrMail<VEC, CW>* post, uint64_t* full, int* s_gone, bool bulk) {
  if (threadIdx.x == 0) {
    *s_gone = 0;
    if (CL > 1) {
      mbar_init(smem_u32(&post->bar[0]), 1);
      mbar_init(smem_u32(&post->bar[1]), 1);
    }
    if (bulk)
      for (int k = 0; k < 3; ++k) mbar_init(smem_u32(&full[k]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (CL > 1) cg::this_cluster().sync();  // the others' memory is written only once they run
  else __syncthreads();
  pdl_launch_dependents();
  pdl_wait_prior_grids();
}

template <typename T, int VEC, bool GATE, int CW, int WT, int SPT, bool BULK>
__global__ void __launch_bounds__(CW* WT * 32, CW* WT == 8 ? 2 : 1)
    glr_fwd_kernel(const GlrArgs a, int CL, const __grid_constant__ GlrTiles tiles) {
  constexpr int M = GATE ? 3 : 2, SLAB = WT * SPT;
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ __align__(16) GlrMap<VEC> s_warp[2][WT][CW * 32];
  __shared__ __align__(16) GlrMail<VEC, CW> post;
  __shared__ uint64_t full[3];
  __shared__ int s_gone;
  glr_setup<VEC, CW>(CL, &post, full, &s_gone, BULK);
  const int cluster = blockIdx.x / CL, rank = blockIdx.x % CL, clusters = gridDim.x / CL;
  const GlrSpan sp(a, CW * 32 * VEC, SLAB * CL);
  GlrFeed<T, VEC, M, WT, SPT, BULK> in(slots, full, &s_gone, cluster);
  if constexpr (BULK)
    if (threadIdx.x == 0)
      for (int k = 0; k < in.SLOTS; ++k) in.ask(a, sp, tiles, CL, rank, clusters, false);
  int mail = 0;
  for (int unit = cluster; unit < sp.units; unit += clusters) {
    const GlrPlace<VEC, CW, WT> at(a, sp, unit);
    const size_t step_y = (size_t)a.B * a.ldy;
    T* y = (T*)a.Y + (size_t)at.b * a.ldy + at.j;
    if constexpr (!BULK) {
      const size_t off = (size_t)at.b * a.ldz + at.col;
      in.src[0] = (const T*)a.Zf + off;
      in.src[1] = (const T*)a.Zg + off;
      if constexpr (GATE) in.src[2] = (const T*)a.Zo + off;
#pragma unroll
      for (int m = 0; m < M; ++m) in.step[m] = (size_t)a.B * a.ldz;
      in.fetch(rank * SLAB + at.wt * SPT, at.len);
    }
    float cs[VEC];  // the state that enters the round
#pragma unroll
    for (int v = 0; v < VEC; ++v) cs[v] = a.h0 && v < at.valid ? a.h0[at.of(a, sp, v)] : 0.f;
    for (int it = 0; it < sp.rounds; ++it, ++mail) {
      const int t0 = (it * CL + rank) * SLAB + at.wt * SPT;
      if constexpr (BULK) in.wait(a.status);
      float f[SPT][VEC], x[SPT][VEC], o[GATE ? SPT : 1][VEC];
      GlrMap<VEC> map = GlrMap<VEC>::none();
#pragma unroll
      for (int k = 0; k < SPT; ++k) {
        glr_unpack<T, VEC>(in.raw(at.wt, 0, k), f[k]);
        glr_unpack<T, VEC>(in.raw(at.wt, 1, k), x[k]);
        if constexpr (GATE) glr_unpack<T, VEC>(in.raw(at.wt, 2, k), o[k]);
        const bool live = t0 + k < at.len;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          float rest;
          f[k][v] = glr_gate(f[k][v], rest);
          x[k][v] *= rest;
          if (!live) {
            f[k][v] = 1.f;
            x[k][v] = 0.f;
          }
          map.a[v] *= f[k][v];
          map.b[v] = fmaf(f[k][v], map.b[v], x[k][v]);
          if constexpr (GATE) o[k][v] = a.alpha * glr_gate(o[k][v]);
        }
      }
      if constexpr (!BULK)
        if (it + 1 < sp.rounds) in.fetch(t0 + SLAB * CL, at.len);
      if constexpr (WT > 1) {
        s_warp[mail & 1][at.wt][at.ch] = map;
        __syncthreads();
      }
      if constexpr (BULK) {  // everybody has read the slot
        if (threadIdx.x == 0) in.ask(a, sp, tiles, CL, rank, clusters, false);
        in.next();
      }
      float c[VEC];
      glr_exchange<VEC, CW, WT>(at.wt, at.ch, mail, mail & 1, CL, rank, true, map, s_warp, &post, cs, c, &s_gone, a.status);
      if (a.S && t0 % ARD_GLR_CHUNK == 0 && t0 < a.T)
#pragma unroll
        for (int v = 0; v < VEC; ++v)
          if (v < at.valid) a.S[((size_t)(t0 / ARD_GLR_CHUNK) * a.B + at.b) * a.H + at.j + v] = c[v];
      T* out = y + (size_t)t0 * step_y;
#pragma unroll
      for (int k = 0; k < SPT; ++k) {
        float w[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          c[v] = fmaf(f[k][v], c[v], x[k][v]);
          w[v] = t0 + k < at.len ? (GATE ? o[k][v] : a.alpha) * c[v] : 0.f;
        }
        if (t0 + k < a.T) glr_store<T, VEC>(out, at.valid, w);
        out += step_y;
      }
    }
    if (a.hT && rank == 0 && at.wt == 0)
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        if (v < at.valid) a.hT[at.of(a, sp, v)] = cs[v];
  }
  if constexpr (BULK)
    if (threadIdx.x == 0) in.drain();
  if (CL > 1) cg::this_cluster().sync();  // nobody leaves while mail may still come
}

template <typename T, int VEC, bool GATE, int CW, int WT, int SPT, bool BULK>
__global__ void __launch_bounds__(CW* WT * 32, CW* WT == 8 ? 2 : 1)
    glr_bwd_kernel(const GlrArgs a, int CL, const __grid_constant__ GlrTiles tiles) {
  constexpr int M = GATE ? 4 : 3, SLAB = WT * SPT;
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ __align__(16) GlrMap<VEC> s_warp[2][WT][CW * 32], s_back[2][WT][CW * 32];
  __shared__ __align__(16) GlrMail<VEC, CW> post;
  __shared__ uint64_t full[3];
  __shared__ int s_gone;
  glr_setup<VEC, CW>(CL, &post, full, &s_gone, BULK);
  const int cluster = blockIdx.x / CL, rank = blockIdx.x % CL, clusters = gridDim.x / CL;
  const GlrSpan sp(a, CW * 32 * VEC, SLAB * CL);
  GlrFeed<T, VEC, M, WT, SPT, BULK> in(slots, full, &s_gone, cluster);
  if constexpr (BULK)
    if (threadIdx.x == 0)
      for (int k = 0; k < in.SLOTS; ++k) in.ask(a, sp, tiles, CL, rank, clusters, true);
  int mail = 0;
  for (int unit = cluster; unit < sp.units; unit += clusters) {
    const GlrPlace<VEC, CW, WT> at(a, sp, unit);
    const size_t step_d = (size_t)a.B * a.lddz, off_d = (size_t)at.b * a.lddz + at.j;
    T* dzf = (T*)a.dZf + off_d;
    T* dzg = (T*)a.dZg + off_d;
    T* dzo = GATE ? (T*)a.dZo + off_d : nullptr;
    // rounds and ranks run from the end; the first slabs may lie behind T
    auto start = [&](int it) { return (sp.rounds * CL - 1 - (it * CL + rank)) * SLAB; };
    if constexpr (!BULK) {
      const size_t off = (size_t)at.b * a.ldz + at.col;
      in.src[0] = (const T*)a.Zf + off;
      in.src[1] = (const T*)a.Zg + off;
      in.src[2] = (const T*)a.dY + (size_t)at.b * a.ldy + at.col;
      if constexpr (GATE) in.src[3] = (const T*)a.Zo + off;
#pragma unroll
      for (int m = 0; m < M; ++m) in.step[m] = (size_t)a.B * (m == 2 ? a.ldy : a.ldz);
      if (sp.rounds > 0) in.fetch(start(0) + at.wt * SPT, at.len);
    }
    float qs[VEC];  // what arrives behind the round's last step
#pragma unroll
    for (int v = 0; v < VEC; ++v) qs[v] = a.h0 && v < at.valid ? a.h0[at.of(a, sp, v)] : 0.f;
    for (int it = 0; it < sp.rounds; ++it, ++mail) {
      const int ts = start(it), t0 = ts + at.wt * SPT;
      float c0[VEC];  // the state that enters the slab
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        c0[v] = ts < a.T && v < at.valid ? a.S[((size_t)(ts / ARD_GLR_CHUNK) * a.B + at.b) * a.H + at.j + v] : 0.f;
      if constexpr (BULK) in.wait(a.status);
      // e: alpha s(zo) dy, what arrives at c from y; no: 1 - s(zo)
      float f[SPT][VEC], i[SPT][VEC], g[SPT][VEC], e[SPT][VEC], no[GATE ? SPT : 1][VEC];
      GlrMap<VEC> map = GlrMap<VEC>::none(), back;
#pragma unroll
      for (int k = 0; k < SPT; ++k) {
        glr_unpack<T, VEC>(in.raw(at.wt, 0, k), f[k]);
        glr_unpack<T, VEC>(in.raw(at.wt, 1, k), g[k]);
        glr_unpack<T, VEC>(in.raw(at.wt, 2, k), e[k]);
        if constexpr (GATE) glr_unpack<T, VEC>(in.raw(at.wt, 3, k), no[k]);
        const bool live = t0 + k < at.len;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          f[k][v] = glr_gate(f[k][v], i[k][v]);
          e[k][v] *= a.alpha;
          if constexpr (GATE) e[k][v] *= glr_gate(no[k][v], no[k][v]);
          if (!live) {
            f[k][v] = 1.f;
            i[k][v] = g[k][v] = e[k][v] = 0.f;
            if constexpr (GATE) no[k][v] = 0.f;
          }
          map.a[v] *= f[k][v];
          map.b[v] = fmaf(f[k][v], map.b[v], i[k][v] * g[k][v]);
        }
      }
      if constexpr (!BULK)
        if (it + 1 < sp.rounds) in.fetch(start(it + 1) + at.wt * SPT, at.len);
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        back.a[v] = map.a[v];
        back.b[v] = 0.f;
#pragma unroll
        for (int k = SPT - 1; k >= 0; --k) back.b[v] = f[k][v] * (e[k][v] + back.b[v]);
      }
      GlrMap<VEC> before = GlrMap<VEC>::none();
      if constexpr (WT > 1) {
        s_warp[mail & 1][at.wt][at.ch] = map;
        s_back[mail & 1][at.wt][at.ch] = back;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WT - 1; ++w)
          if (w < at.wt) before.then(s_warp[mail & 1][w][at.ch]);
      }
      if constexpr (BULK) {
        if (threadIdx.x == 0) in.ask(a, sp, tiles, CL, rank, clusters, true);
        in.next();
      }
      float q[VEC];
      glr_exchange<VEC, CW, WT>(at.wt, at.ch, mail, mail & 1, CL, rank, false, back, s_back, &post, qs, q, &s_gone, a.status);
      float c[SPT + 1][VEC];
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        c[0][v] = before.of(c0[v], v);
#pragma unroll
        for (int k = 0; k < SPT; ++k) c[k + 1][v] = fmaf(f[k][v], c[k][v], i[k][v] * g[k][v]);
      }
      size_t row = (size_t)(t0 + SPT - 1) * step_d;
#pragma unroll
      for (int k = SPT - 1; k >= 0; --k) {
        float of[VEC], og[VEC], oo[VEC];
        const bool live = t0 + k < at.len;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const float d = e[k][v] + q[v], di = d * i[k][v];
          q[v] = f[k][v] * d;
          of[v] = live ? di * f[k][v] * (c[k][v] - g[k][v]) : 0.f;
          og[v] = live ? di : 0.f;
          if constexpr (GATE) oo[v] = live ? e[k][v] * c[k + 1][v] * no[k][v] : 0.f;
        }
        if (t0 + k < a.T) {
          glr_store<T, VEC>(dzf + row, at.valid, of);
          glr_store<T, VEC>(dzg + row, at.valid, og);
          if constexpr (GATE) glr_store<T, VEC>(dzo + row, at.valid, oo);
        }
        row -= step_d;
      }
    }
    if (a.hT && rank == 0 && at.wt == 0)
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        if (v < at.valid) a.hT[at.of(a, sp, v)] = qs[v];
  }
  if constexpr (BULK)
    if (threadIdx.x == 0) in.drain();
  if (CL > 1) cg::this_cluster().sync();
}

// bf16 columns on a grid of two: read and written in pairs.
inline bool glr_pairs(std::initializer_list<const void*> ps, std::initializer_list<int> lds) {
  for (const void* p : ps)
    if (reinterpret_cast<uintptr_t>(p) % 4) return false;
  for (int ld : lds)
    if (ld % 2) return false;
  return true;
}

// A cluster's CTAs take consecutive slabs of the time axis where the channels alone leave SMs idle.  With bulk copies the grid is what
// the device holds at once (two CTAs an SM) and a CTA goes from unit to unit, its copies ahead of it; without, a CTA per unit.
template <typename K>
ard_status glr_launch(ard_ctx* ctx, K kern, const GlrArgs& a, const GlrTiles& tiles, int channels, int slab, int threads, int smem,
                      cudaStream_t s) {
  const long long slabs = ((long long)a.T + slab - 1) / slab, units = (long long)((a.H + channels - 1) / channels) * a.B;
  const int resident = 2 * ctx->sm_count;
  int CL = 1;
  while (CL < GLR_CLUSTER && 2 * CL <= slabs && units * 2 * CL <= resident) CL *= 2;
  long long blocks = units * CL;
  if (smem > 0) {
    ARD_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    if (blocks > resident) blocks = resident;
  }
  if (units > 0x7FFFFFFFll || blocks > 0x7FFFFFFFll) return ARD_ERR_UNSUPPORTED;
  if (CL > 1) ARD_CUDA_OK(ard_launch_cluster(ctx, kern, CL, dim3((unsigned)blocks), dim3(threads), smem, s, a, CL, tiles));
  else ARD_CUDA_OK(ard_launch(ctx, kern, dim3((unsigned)blocks), dim3(threads), smem, s, a, CL, tiles));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}

template <typename F>
constexpr int glr_ring() { return F::SLOTS * F::SLOT; }

// Descriptors [T][B][H] of the M operands; false: not on a 16-byte grid.
template <typename T, int VEC>
bool glr_tiles(ard_ctx* ctx, const GlrArgs& a, std::initializer_list<std::pair<const void*, int>> operands, int steps, GlrTiles* out) {
  int m = 0;
  for (const auto& op : operands) {
    if ((reinterpret_cast<uintptr_t>(op.first) & 15u) || (op.second * sizeof(T)) % 16) return false;
    if (!ard_encode_steps(ctx, &out->map[m++], sizeof(T) == 4, op.first, a.H, a.B, a.T, op.second, 32 * VEC, steps)) return false;
  }
  return true;
}

template <typename T, int VEC, bool GATE>
struct GlrFwd {
  static ard_status run(ard_ctx* ctx, const GlrArgs& a, cudaStream_t s) {
    GlrTiles tiles;
    if (a.T <= 1) return glr_launch(ctx, glr_fwd_kernel<T, VEC, GATE, 4, 1, 1, false>, a, tiles, 4 * 32 * VEC, 1, 128, 0, s);
    if constexpr (VEC * sizeof(T) == 4) {
      bool ok;
      if constexpr (GATE) ok = glr_tiles<T, VEC>(ctx, a, {{a.Zf, a.ldz}, {a.Zg, a.ldz}, {a.Zo, a.ldz}}, 64, &tiles);
      else ok = glr_tiles<T, VEC>(ctx, a, {{a.Zf, a.ldz}, {a.Zg, a.ldz}}, 64, &tiles);
      if (ok)
        return glr_launch(ctx, glr_fwd_kernel<T, VEC, GATE, 1, 8, 8, true>, a, tiles, 32 * VEC, 64, 256,
                          glr_ring<GlrFeed<T, VEC, GATE ? 3 : 2, 8, 8, true>>(), s);
    }
    return glr_launch(ctx, glr_fwd_kernel<T, VEC, GATE, 1, 8, 8, false>, a, tiles, 32 * VEC, 64, 256, 0, s);
  }
};
template <typename T, int VEC, bool GATE>
struct GlrBwd {
  static ard_status run(ard_ctx* ctx, const GlrArgs& a, cudaStream_t s) {
    GlrTiles tiles;
    if (a.T <= 1) return glr_launch(ctx, glr_bwd_kernel<T, VEC, GATE, 4, 1, 1, false>, a, tiles, 4 * 32 * VEC, 1, 128, 0, s);
    if constexpr (VEC * sizeof(T) == 4) {
      bool ok;
      if constexpr (GATE) ok = glr_tiles<T, VEC>(ctx, a, {{a.Zf, a.ldz}, {a.Zg, a.ldz}, {a.dY, a.ldy}, {a.Zo, a.ldz}}, 64, &tiles);
      else ok = glr_tiles<T, VEC>(ctx, a, {{a.Zf, a.ldz}, {a.Zg, a.ldz}, {a.dY, a.ldy}}, 64, &tiles);
      if (ok)
        return glr_launch(ctx, glr_bwd_kernel<T, VEC, GATE, 1, 8, 8, true>, a, tiles, 32 * VEC, 64, 256,
                          glr_ring<GlrFeed<T, VEC, GATE ? 4 : 3, 8, 8, true>>(), s);
    }
    return glr_launch(ctx, glr_bwd_kernel<T, VEC, GATE, 1, 8, 8, false>, a, tiles, 32 * VEC, 64, 256, 0, s);
  }
};

template <template <typename, int, bool> class Op>
ard_status glr_dispatch(ard_ctx* ctx, bool f32, bool pairs, const GlrArgs& a, cudaStream_t s) {
  const bool gate = a.Zo != nullptr;
  if (f32) return gate ? Op<float, 1, true>::run(ctx, a, s) : Op<float, 1, false>::run(ctx, a, s);
  if (pairs) return gate ? Op<__nv_bfloat16, 2, true>::run(ctx, a, s) : Op<__nv_bfloat16, 2, false>::run(ctx, a, s);
  return gate ? Op<__nv_bfloat16, 1, true>::run(ctx, a, s) : Op<__nv_bfloat16, 1, false>::run(ctx, a, s);
}

}  // namespace

ard_status launch_glr_forward(ard_ctx* ctx, const int32_t* hdr, ard_dtype dtype, int T, int B, int H, float alpha, const void* Zf,
                              const void* Zg, const void* Zo, int ldz, const int32_t* lens, const float* h0, void* Y, int ldy, float* hT,
                              float* S, cudaStream_t s) {
  if (B == 0 || H == 0) return ARD_OK;
  GlrArgs a = {};
  a.hdr = hdr;
  a.T = T; a.B = B; a.H = H;
  a.alpha = alpha;
  a.Zf = Zf; a.Zg = Zg; a.Zo = Zo;
  a.ldz = ldz;
  a.lens = lens;
  a.h0 = h0;
  a.Y = Y;
  a.ldy = ldy;
  a.hT = hT;
  a.S = S;
  a.status = ctx->d_status;
  return glr_dispatch<GlrFwd>(ctx, dtype == ARD_F32, glr_pairs({Zf, Zg, Zo, Y}, {ldz, ldy}), a, s);
}

ard_status launch_glr_backward(ard_ctx* ctx, const int32_t* hdr, ard_dtype dtype, int T, int B, int H, float alpha, const void* Zf,
                               const void* Zg, const void* Zo, int ldz, const int32_t* lens, const float* S, const void* dY, int lddy,
                               const float* dhT, void* dZf, void* dZg, void* dZo, int lddz, float* dh0, cudaStream_t s) {
  if (B == 0 || H == 0) return ARD_OK;
  GlrArgs a = {};
  a.hdr = hdr;
  a.T = T; a.B = B; a.H = H;
  a.alpha = alpha;
  a.Zf = Zf; a.Zg = Zg; a.Zo = Zo;
  a.ldz = ldz;
  a.lens = lens;
  a.S = const_cast<float*>(S);
  a.dY = dY;
  a.ldy = lddy;
  a.h0 = dhT;
  a.dZf = dZf; a.dZg = dZg; a.dZo = dZo;
  a.lddz = lddz;
  a.hT = dh0;
  a.status = ctx->d_status;
  return glr_dispatch<GlrBwd>(ctx, dtype == ARD_F32, glr_pairs({Zf, Zg, Zo, dY, dZf, dZg, dZo}, {ldz, lddy, lddz}), a, s);
}
