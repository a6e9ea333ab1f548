// The gated linear recurrence over whole sequences, forward and adjoint:
//   f_t = s(zf_t),  c_t = f_t c_{t-1} + (1 - f_t) g_t,  y_t = alpha s(zo_t) c_t
//   d_t = alpha s(zo_t) dy_t + q_t,  q_{t-1} = f_t d_t,
//   dzo_t = alpha dy_t c_t s(zo_t) (1 - s(zo_t)),  dzf_t = d_t (c_{t-1} - g_t) f_t (1 - f_t),  dzg_t = d_t (1 - f_t).
//
// Both recurrences are compositions of maps x -> A x + B, so the time axis can be cut: a thread holds SPT steps of its
// channels in registers, composes their map, and applies the steps once it knows the state that enters them.  The maps
// of a slab's warps meet in shared memory, those of consecutive slabs in the shared memory of a cluster of CTAs (few
// channels, long sequences), so gates are read once and outputs written once.  The adjoint starts its states from those
// that the forward call left every ARD_GLR_CHUNK steps and computes the ones between again: 4 bytes in 64 steps in
// place of 4 in each.
//
// Memory would bound both (gates in, outputs out); what does is instruction issue and the way of the maps: 2048 x 8 x
// 2048 bf16 56 / 87 us forward / backward (its bytes at a copy's rate 41.1 / 71.9; half to 60 % of the issue slots
// taken, 256 units on 296 places), 16384 x 1 x 1024 40.5 / 69 us (20.6 / 36; sixteen rounds, each with the maps' way
// round a cluster), 35 x 64 x 1024 8.8 / 14.4 us (2.8 / 4.9), a single step of 64 x 1024 2.2 us. A slab behind a
// sequence's end costs as much as one inside it: gates of what the slot holds, maps, the barrier, and the zeros by
// stores that ask. With three fifths of the cells of 2048 x 8 x 2048 inside 62 / 99 us.
#include <cooperative_groups.h>

#include <initializer_list>
#include <type_traits>
#include <utility>

#include "ard_internal.h"
#include "sm100_ptx.h"

namespace {

namespace cg = cooperative_groups;

constexpr int GLR_CLUSTER = 16;  // most CTAs that share a sequence

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

// A lane's channels.  Two of them go through one instruction (f32x2): these kernels run out of issue slots before
// anything else.
template <int VEC>
struct GlrV {
  float v[VEC];
  __device__ __forceinline__ static GlrV all(float x) {
    GlrV r;
#pragma unroll
    for (int k = 0; k < VEC; ++k) r.v[k] = x;
    return r;
  }
};
template <int VEC>
__device__ __forceinline__ GlrV<VEC> operator*(const GlrV<VEC>& a, const GlrV<VEC>& b) {
  if constexpr (VEC == 2) {
    const float2 r = __fmul2_rn(make_float2(a.v[0], a.v[1]), make_float2(b.v[0], b.v[1]));
    return {{r.x, r.y}};
  } else {
    return {{a.v[0] * b.v[0]}};
  }
}
template <int VEC>
__device__ __forceinline__ GlrV<VEC> operator+(const GlrV<VEC>& a, const GlrV<VEC>& b) {
  if constexpr (VEC == 2) {
    const float2 r = __fadd2_rn(make_float2(a.v[0], a.v[1]), make_float2(b.v[0], b.v[1]));
    return {{r.x, r.y}};
  } else {
    return {{a.v[0] + b.v[0]}};
  }
}
template <int VEC>
__device__ __forceinline__ GlrV<VEC> glr_fma(const GlrV<VEC>& a, const GlrV<VEC>& b, const GlrV<VEC>& c) {
  if constexpr (VEC == 2) {
    const float2 r = __ffma2_rn(make_float2(a.v[0], a.v[1]), make_float2(b.v[0], b.v[1]), make_float2(c.v[0], c.v[1]));
    return {{r.x, r.y}};
  } else {
    return {{fmaf(a.v[0], b.v[0], c.v[0])}};
  }
}
// 2^x and 1 / x to about two units in the last place, results below the normal range zero: the forms that keep
// subnormals cost five instructions each, of which a gate has two.
__device__ __forceinline__ float glr_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float glr_inverse(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// s(z), and 1 - s(z), each relative to its own size: where s(z) is above a half the other one is exp(-z) times it, not
// a difference.  The exponential's argument is a rounded product, so the smaller of the two is off by some |z| units in
// the last place beside the instructions' own two or three.  exp(-z) of infinity gives 0 and 1.
template <int VEC>
__device__ __forceinline__ GlrV<VEC> glr_gate(const GlrV<VEC>& z, GlrV<VEC>& rest) {
  GlrV<VEC> u = z * GlrV<VEC>::all(-1.44269504f);
#pragma unroll
  for (int k = 0; k < VEC; ++k) u.v[k] = glr_exp2(u.v[k]);
  GlrV<VEC> f = u + GlrV<VEC>::all(1.f);
#pragma unroll
  for (int k = 0; k < VEC; ++k) f.v[k] = glr_inverse(f.v[k]);
  const GlrV<VEC> small = u * f, large = glr_fma(f, GlrV<VEC>::all(-1.f), GlrV<VEC>::all(1.f));
#pragma unroll
  for (int k = 0; k < VEC; ++k) rest.v[k] = z.v[k] >= 0.f ? small.v[k] : large.v[k];
  return f;
}
template <int VEC>
__device__ __forceinline__ GlrV<VEC> glr_gate(const GlrV<VEC>& z) {
  GlrV<VEC> rest;
  return glr_gate(z, rest);  // (what is not used is not computed)
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
__device__ __forceinline__ GlrV<VEC> glr_unpack(uint32_t q) {
  GlrV<VEC> r;
  if constexpr (sizeof(T) == 4) {
    r.v[0] = __uint_as_float(q);
  } else {
    r.v[0] = __uint_as_float(q << 16);
    if constexpr (VEC == 2) r.v[1] = __uint_as_float(q & 0xFFFF0000u);
  }
  return r;
}
// The first `valid` of the values.
template <typename T, int VEC>
__device__ __forceinline__ void glr_store(T* p, int valid, const GlrV<VEC>& x) {
  const float* v = x.v;
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

// Maps x -> a x + b of a lane's channels.
template <int VEC>
struct GlrMap {
  GlrV<VEC> a, b;
  // this one, then `next`
  __device__ __forceinline__ void then(const GlrMap& next) {
    b = glr_fma(next.a, b, next.b);
    a = a * next.a;
  }
  __device__ __forceinline__ GlrV<VEC> of(const GlrV<VEC>& x) const { return glr_fma(a, x, b); }
};

// What the kernels run over: units of W * VEC channels of one sequence, `rounds` times CL slabs of WT * SPT steps each.
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
    groups = (int)(((long long)n + channels - 1) / channels);
    units = groups * a.B;  // (at most 2^31 - 1: the host asks)
    rounds = (a.T + steps - 1) / steps;
  }
  // The unit of a CTA (a cluster) after this one: so many further, or behind the last, whose number the sum may not
  // pass.
  __device__ __forceinline__ int after(int unit, int clusters) const { return units - unit > clusters ? unit + clusters : units; }
  __device__ __forceinline__ bool inside(int unit, int channels) const { return n - unit % groups * channels >= channels; }
  __device__ __forceinline__ int len(const GlrArgs& a, int b) const { return a.lens ? min(max(a.lens[b], 0), a.T) : a.T; }
};
// A thread's place in a unit: VEC channels of one sequence, SPT consecutive steps of every slab.  W threads stand side
// by side over the unit's channels (warps, or half a warp), WT groups of them over a slab's steps.
template <int VEC, int W, int WT>
struct GlrPlace {
  int wt, ch, b, j, valid, col, len;
  __device__ __forceinline__ GlrPlace(const GlrArgs& a, const GlrSpan& sp, int unit) {
    wt = threadIdx.x / W;
    ch = threadIdx.x % W;
    b = unit / sp.groups;
    j = ((unit - b * sp.groups) * W + ch) * VEC;
    valid = max(0, min(VEC, sp.n - j));
    col = min(j, (sp.n - 1) / VEC * VEC);  // where a lane without channels reads
    len = sp.len(a, b);
  }
  __device__ __forceinline__ size_t of(const GlrArgs& a, const GlrSpan& sp, int v) const {
    return (size_t)b * a.H + sp.b0 + (size_t)(j + v) * sp.dp;
  }
};

// Where M operands of a slab come from.  BULK: tiles [WT * SPT steps][W * VEC channels] that the copy engine brings
// into a ring of slots, several slabs ahead and over the ends of units (rows of 16-byte aligned pieces).  Otherwise
// registers, into which a thread fetches its own values of the unit's next slab as soon as this one's are used.
struct GlrTiles {
  CUtensorMap map[4];
};
template <typename T, int VEC, int M, int W, int WT, int SPT, bool BULK>
struct GlrFeed;

template <typename T, int VEC, int M, int W, int WT, int SPT>
struct GlrFeed<T, VEC, M, W, WT, SPT, true> {
  static constexpr int ROW = W * VEC * (int)sizeof(T), TILE = WT * SPT * ROW, SLOT = M * TILE;
  static constexpr int SLOTS = M == 4 ? 2 : 3;  // two CTAs an SM with 48 to 72 KB each
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
      const int b = unit / sp.groups, x = (unit - b * sp.groups) * W * VEC;
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
      unit = sp.after(unit, clusters);
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
  __device__ __forceinline__ uint32_t raw(int wt, int m, int k) const {
    const uint8_t* p = slots + slot * SLOT + m * TILE + (wt * SPT + k) * ROW + (threadIdx.x % W) * (VEC * (int)sizeof(T));
    return *reinterpret_cast<const uint32_t*>(p);
  }
};
template <typename T, int VEC, int M, int W, int WT, int SPT>
struct GlrFeed<T, VEC, M, W, WT, SPT, false> {
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

// The maps of a slab's warps meet in `warp`; its last warp (in the order of the recurrence) leaves the state behind the
// round in `state`, where the next round finds it.  The cluster's CTAs send each other their slabs' maps by
// asynchronous stores that count on the receiver's barrier: a barrier of the cluster would wait for the outputs'
// stores, 2 us a round (bulk copies between their memories: forward the same, backward 30 % slower).  Every CTA hears
// from all of them in every round, so none is more than a round ahead and two sets of places are enough.
template <int VEC, int W, int FROM>
struct GlrMail {
  GlrMap<VEC> box[2][FROM][W];
  uint64_t bar[2];
};
template <int VEC>
__device__ __forceinline__ void glr_send(GlrMap<VEC>* box, uint64_t* bar, int r, const GlrMap<VEC>& m) {
  uint32_t dst, rbar;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst) : "r"(smem_u32(box)), "r"(r));
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(rbar) : "r"(smem_u32(bar)), "r"(r));
  if constexpr (VEC == 2)
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(dst), "f"(m.a.v[0]),
                 "f"(m.a.v[1]), "f"(m.b.v[0]), "f"(m.b.v[1]), "r"(rbar)
                 : "memory");
  else
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(dst), "f"(m.a.v[0]), "f"(m.b.v[0]),
                 "r"(rbar)
                 : "memory");
}
template <int VEC, int W, int WT>
struct GlrShared {
  GlrMap<VEC> warp[2][WT][W];
  GlrV<VEC> state[2][W];
  GlrMail<VEC, W, (WT > 1 ? GLR_CLUSTER : 1)> post;
  uint64_t full[3];
  int gone;
};

// Behind the barrier that follows the warps' maps: the state that enters this warp's steps.  x: what enters the unit's
// first round.  FORWARD: warps count in the order of the steps, else against it.  `mail`: rounds of the cluster so far.
template <bool FORWARD, int VEC, int W, int WT>
__device__ __forceinline__ GlrV<VEC> glr_enter(GlrShared<VEC, W, WT>& sh, int wt, int ch, bool first, int mail, int CL, int rank,
                                              const GlrV<VEC>& x, int* status) {
  GlrV<VEC> c = x;
  if constexpr (WT > 1) {
    constexpr int LAST = FORWARD ? WT - 1 : 0;
    const int set = mail & 1;
    if (!first) c = sh.state[set][ch];
    if (CL > 1) {
      if (wt == LAST) {
        GlrMap<VEC> all = sh.warp[set][WT - 1 - LAST][ch];
#pragma unroll
        for (int k = 1; k < WT; ++k) all.then(sh.warp[set][FORWARD ? k : WT - 1 - k][ch]);
        for (int r = 0; r < CL; ++r) glr_send<VEC>(&sh.post.box[set][rank][ch], &sh.post.bar[set], r, all);
      }
      if (threadIdx.x == 0) mbar_arrive_expect_tx(smem_u32(&sh.post.bar[set]), (uint32_t)(CL * W * sizeof(GlrMap<VEC>)));
      // an acquire of the cluster's scope: other CTAs wrote what is read behind it
      mbar_wait_cluster(smem_u32(&sh.post.bar[set]), (uint32_t)(mail >> 1) & 1u, &sh.gone, status);
      for (int r = 0; r < rank; ++r) c = sh.post.box[set][r][ch].of(c);
      if (wt == LAST) {
        GlrV<VEC> behind = c;
        for (int r = rank; r < CL; ++r) behind = sh.post.box[set][r][ch].of(behind);
        sh.state[set ^ 1][ch] = behind;
      }
    }
    if constexpr (FORWARD) {
      for (int w = 0; w < wt; ++w) c = sh.warp[set][w][ch].of(c);
    } else {
      for (int w = WT - 1; w > wt; --w) c = sh.warp[set][w][ch].of(c);
    }
  }
  return c;
}

// Shared memory and barriers of either kernel, before it touches global memory.
template <typename Shared>
__device__ __forceinline__ void glr_setup(int CL, Shared& sh) {
  if (threadIdx.x == 0) {
    sh.gone = 0;
    mbar_init(smem_u32(&sh.post.bar[0]), 1);
    mbar_init(smem_u32(&sh.post.bar[1]), 1);
    for (int k = 0; k < 3; ++k) mbar_init(smem_u32(&sh.full[k]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (CL > 1) cg::this_cluster().sync();  // the others' memory is written only once they run
  else __syncthreads();
  pdl_launch_dependents();
  pdl_wait_prior_grids();
}

template <typename T, int VEC, bool GATE, int W, int WT, int SPT, bool BULK>
__global__ void __launch_bounds__(W* WT, W* WT < 256 ? 1 : SPT < 8 && SPT != 4 ? 3 : 2)
    glr_fwd_kernel(const GlrArgs a, int CL, const __grid_constant__ GlrTiles tiles) {
  using V = GlrV<VEC>;
  constexpr int M = GATE ? 3 : 2, SLAB = WT * SPT;
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ __align__(16) GlrShared<VEC, W, WT> sh;
  glr_setup(CL, sh);
  const int cluster = blockIdx.x / CL, rank = blockIdx.x % CL, clusters = gridDim.x / CL;
  const GlrSpan sp(a, W * VEC, SLAB * CL);
  GlrFeed<T, VEC, M, W, WT, SPT, BULK> in(slots, sh.full, &sh.gone, cluster);
  if constexpr (BULK)
    if (threadIdx.x == 0)
      for (int k = 0; k < in.SLOTS; ++k) in.ask(a, sp, tiles, CL, rank, clusters, false);
  const V alpha = V::all(a.alpha);
  int mail = 0;
  for (int unit = cluster; unit < sp.units; unit = sp.after(unit, clusters)) {
    const GlrPlace<VEC, W, WT> at(a, sp, unit);
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
    V first;  // the state that enters the unit
#pragma unroll
    for (int v = 0; v < VEC; ++v) first.v[v] = a.h0 && v < at.valid ? a.h0[at.of(a, sp, v)] : 0.f;
    const bool inside = sp.inside(unit, W * VEC);
    V c = first;
    // FULL: all steps of the slab are a sequence's, all channels of the unit exist; nothing is asked per step
    auto slab = [&](auto full, int it) {
      constexpr bool FULL = decltype(full)::value;
      const int t0 = (it * CL + rank) * SLAB + at.wt * SPT;
      V f[SPT], x[SPT], o[GATE ? SPT : 1];
      GlrMap<VEC> map;
#pragma unroll
      for (int k = 0; k < SPT; ++k) {
        V rest;
        f[k] = glr_gate(glr_unpack<T, VEC>(in.raw(at.wt, 0, k)), rest);
        x[k] = rest * glr_unpack<T, VEC>(in.raw(at.wt, 1, k));
        if constexpr (GATE) o[k] = alpha * glr_gate(glr_unpack<T, VEC>(in.raw(at.wt, 2, k)));
        if constexpr (!FULL)
          if (t0 + k >= at.len) {
            f[k] = V::all(1.f);
            x[k] = V::all(0.f);
          }
        if (k == 0) map = {f[0], x[0]};
        else map.then({f[k], x[k]});
      }
      if constexpr (!BULK)
        if (it + 1 < sp.rounds) in.fetch(t0 + SLAB * CL, at.len);
      if constexpr (WT > 1) {
        sh.warp[mail & 1][at.wt][at.ch] = map;
        __syncthreads();
      }
      if constexpr (BULK) {  // everybody has read the slot
        if (threadIdx.x == 0) in.ask(a, sp, tiles, CL, rank, clusters, false);
        in.next();
      }
      c = glr_enter<true>(sh, at.wt, at.ch, it == 0, mail, CL, rank, first, a.status);
      if (a.S && t0 % ARD_GLR_CHUNK == 0 && t0 < a.T)
#pragma unroll
        for (int v = 0; v < VEC; ++v)
          if (v < at.valid) a.S[((size_t)(t0 / ARD_GLR_CHUNK) * a.B + at.b) * a.H + at.j + v] = c.v[v];
      T* out = y + (size_t)t0 * step_y;
#pragma unroll
      for (int k = 0; k < SPT; ++k) {
        c = glr_fma(f[k], c, x[k]);
        V w = (GATE ? o[k] : alpha) * c;
        if constexpr (FULL) {
          glr_store<T, VEC>(out, VEC, w);
        } else {
          if (t0 + k >= at.len) w = V::all(0.f);
          if (t0 + k < a.T) glr_store<T, VEC>(out, at.valid, w);
        }
        out += step_y;
      }
      if (WT > 1 && CL == 1 && at.wt == WT - 1) sh.state[(mail & 1) ^ 1][at.ch] = c;
    };
    for (int it = 0; it < sp.rounds; ++it, ++mail) {
      if constexpr (BULK) in.wait(a.status);
      if (inside && ((it + 1) * CL) * SLAB <= at.len) slab(std::true_type{}, it);
      else slab(std::false_type{}, it);
    }
    if (CL > 1 && a.hT && a.hT == a.h0) cg::this_cluster().sync();  // the others have read what is about to be overwritten
    if (a.hT && rank == 0 && at.wt == WT - 1) {  // (the last warp's own words)
      const V behind = WT > 1 && sp.rounds > 0 ? sh.state[mail & 1][at.ch] : c;
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        if (v < at.valid) a.hT[at.of(a, sp, v)] = behind.v[v];
    }
  }
  if constexpr (BULK)
    if (threadIdx.x == 0) in.drain();
  if (CL > 1) cg::this_cluster().sync();  // nobody leaves while mail may still come
}

template <typename T, int VEC, bool GATE, int W, int WT, int SPT, bool BULK>
__global__ void __launch_bounds__(W* WT, W* WT < 256 ? 1 : SPT < 8 && SPT != 4 ? 3 : 2)
    glr_bwd_kernel(const GlrArgs a, int CL, const __grid_constant__ GlrTiles tiles) {
  using V = GlrV<VEC>;
  constexpr int M = GATE ? 4 : 3, SLAB = WT * SPT;
  extern __shared__ __align__(128) uint8_t slots[];
  __shared__ __align__(16) GlrShared<VEC, W, WT> sh;  // of the adjoint's maps
  __shared__ __align__(16) GlrMap<VEC> s_states[2][WT][W];
  glr_setup(CL, sh);
  const int cluster = blockIdx.x / CL, rank = blockIdx.x % CL, clusters = gridDim.x / CL;
  const GlrSpan sp(a, W * VEC, SLAB * CL);
  GlrFeed<T, VEC, M, W, WT, SPT, BULK> in(slots, sh.full, &sh.gone, cluster);
  if constexpr (BULK)
    if (threadIdx.x == 0)
      for (int k = 0; k < in.SLOTS; ++k) in.ask(a, sp, tiles, CL, rank, clusters, true);
  const V alpha = V::all(a.alpha), minus = V::all(-1.f);
  int mail = 0;
  for (int unit = cluster; unit < sp.units; unit = sp.after(unit, clusters)) {
    const GlrPlace<VEC, W, WT> at(a, sp, unit);
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
    V first;  // what arrives behind the unit's last step
#pragma unroll
    for (int v = 0; v < VEC; ++v) first.v[v] = a.h0 && v < at.valid ? a.h0[at.of(a, sp, v)] : 0.f;
    const bool inside = sp.inside(unit, W * VEC);
    V q = first;
    auto slab = [&](auto full, int it) {
      constexpr bool FULL = decltype(full)::value;
      const int ts = start(it), t0 = ts + at.wt * SPT;
      V c0;  // the state that enters the slab
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        c0.v[v] = ts < a.T && v < at.valid ? a.S[((size_t)(ts / ARD_GLR_CHUNK) * a.B + at.b) * a.H + at.j + v] : 0.f;
      // e: alpha s(zo) dy, what arrives at c from y; no: 1 - s(zo)
      V f[SPT], i[SPT], g[SPT], e[SPT];
      [[maybe_unused]] V no[GATE ? SPT : 1];
      GlrMap<VEC> map, back;
#pragma unroll
      for (int k = 0; k < SPT; ++k) {
        f[k] = glr_gate(glr_unpack<T, VEC>(in.raw(at.wt, 0, k)), i[k]);
        g[k] = glr_unpack<T, VEC>(in.raw(at.wt, 1, k));
        e[k] = alpha * glr_unpack<T, VEC>(in.raw(at.wt, 2, k));
        if constexpr (GATE) e[k] = e[k] * glr_gate(glr_unpack<T, VEC>(in.raw(at.wt, 3, k)), no[k]);
        if constexpr (!FULL)
          if (t0 + k >= at.len) {
            f[k] = V::all(1.f);
            i[k] = g[k] = e[k] = V::all(0.f);
            if constexpr (GATE) no[k] = V::all(0.f);
          }
        const V b = i[k] * g[k];
        if (k == 0) map = {f[0], b};
        else map.then({f[k], b});
      }
      if constexpr (!BULK)
        if (it + 1 < sp.rounds) in.fetch(start(it + 1) + at.wt * SPT, at.len);
      back.a = map.a;
      back.b = f[SPT - 1] * e[SPT - 1];
#pragma unroll
      for (int k = SPT - 2; k >= 0; --k) back.b = f[k] * (e[k] + back.b);
      if constexpr (WT > 1) {
        s_states[mail & 1][at.wt][at.ch] = map;
        sh.warp[mail & 1][at.wt][at.ch] = back;
        __syncthreads();
      }
      if constexpr (BULK) {
        if (threadIdx.x == 0) in.ask(a, sp, tiles, CL, rank, clusters, true);
        in.next();
      }
      q = glr_enter<false>(sh, at.wt, at.ch, it == 0, mail, CL, rank, first, a.status);
      V c[SPT + 1];
      c[0] = c0;
      if constexpr (WT > 1)
        for (int w = 0; w < at.wt; ++w) c[0] = s_states[mail & 1][w][at.ch].of(c[0]);
#pragma unroll
      for (int k = 0; k < SPT; ++k) c[k + 1] = glr_fma(f[k], c[k], i[k] * g[k]);
      size_t row = (size_t)(t0 + SPT - 1) * step_d;
#pragma unroll
      for (int k = SPT - 1; k >= 0; --k) {
        const V d = e[k] + q, di = d * i[k];
        q = f[k] * d;
        V of = (di * f[k]) * glr_fma(g[k], minus, c[k]), og = di;
        [[maybe_unused]] V oo;
        if constexpr (GATE) oo = (e[k] * no[k]) * c[k + 1];
        if constexpr (FULL) {
          glr_store<T, VEC>(dzf + row, VEC, of);
          glr_store<T, VEC>(dzg + row, VEC, og);
          if constexpr (GATE) glr_store<T, VEC>(dzo + row, VEC, oo);
        } else {
          if (t0 + k >= at.len) {
            of = og = V::all(0.f);
            if constexpr (GATE) oo = of;
          }
          if (t0 + k < a.T) {
            glr_store<T, VEC>(dzf + row, at.valid, of);
            glr_store<T, VEC>(dzg + row, at.valid, og);
            if constexpr (GATE) glr_store<T, VEC>(dzo + row, at.valid, oo);
          }
        }
        row -= step_d;
      }
      if (WT > 1 && CL == 1 && at.wt == 0) sh.state[(mail & 1) ^ 1][at.ch] = q;
    };
    for (int it = 0; it < sp.rounds; ++it, ++mail) {
      if constexpr (BULK) in.wait(a.status);
      // (the round's last slab is rank 0's)
      if (inside && (sp.rounds - it) * CL * SLAB <= at.len) slab(std::true_type{}, it);
      else slab(std::false_type{}, it);
    }
    if (CL > 1 && a.hT && a.hT == a.h0) cg::this_cluster().sync();
    if (a.hT && rank == 0 && at.wt == 0) {
      const V behind = WT > 1 && sp.rounds > 0 ? sh.state[mail & 1][at.ch] : q;
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        if (v < at.valid) a.hT[at.of(a, sp, v)] = behind.v[v];
    }
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

template <typename F>
constexpr int glr_ring() { return F::SLOTS * F::SLOT; }

inline long long glr_units(const GlrArgs& a, int channels) { return ((long long)a.H + channels - 1) / channels * a.B; }

// With bulk copies the grid is what the device holds at once (per_sm CTAs an SM) and a CTA goes from unit to unit, its
// copies ahead of it; without, a CTA (a cluster) per unit.
template <typename K>
ard_status glr_launch(ard_ctx* ctx, K kern, const GlrArgs& a, const GlrTiles& tiles, int channels, int CL, int threads, int smem, int per_sm,
                      cudaStream_t s) {
  const long long units = glr_units(a, channels);
  long long blocks = units * CL;
  if (units > 0x7FFFFFFFll || blocks > 0x7FFFFFFFll) return ARD_ERR_UNSUPPORTED;
  if (CL > 8) ARD_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  if (smem > 0) {
    ARD_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    const int resident = per_sm * ctx->sm_count;
    if (blocks > resident) blocks = resident / CL * CL;
  }
  if (CL > 1) ARD_CUDA_OK(ard_launch_cluster(ctx, kern, CL, dim3((unsigned)blocks), dim3(threads), smem, s, a, CL, tiles));
  else ARD_CUDA_OK(ard_launch(ctx, kern, dim3((unsigned)blocks), dim3(threads), smem, s, a, CL, tiles));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}

// CTAs of a cluster that share a sequence's slabs, where the units alone leave more than half of the SMs idle: as many
// as let all units run at once.  How many clusters of a size the device holds goes by how its SMs are grouped, and is
// asked once.
inline int glr_cluster(ard_ctx* ctx, long long units, long long slabs) {
  if (slabs < 2) return 1;
  if (ctx->glr_room[2] == 0) {
    auto kern = glr_fwd_kernel<__nv_bfloat16, 2, true, 16, 16, 8, true>;
    constexpr int smem = glr_ring<GlrFeed<__nv_bfloat16, 2, 3, 16, 16, 8, true>>();
    cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    for (int cl = 2; cl <= GLR_CLUSTER; ++cl) ctx->glr_room[cl] = ard_cluster_room(ctx, kern, cl, 256, smem) / cl;
    (void)cudaGetLastError();
  }
  int CL = GLR_CLUSTER;
  while (CL > 1 && (CL > slabs || ctx->glr_room[CL] < units)) --CL;
  const long long rounds = (slabs + CL - 1) / CL;
  return (int)((slabs + rounds - 1) / rounds);
}

// Descriptors [T][B][H] of the M operands; false: not on a 16-byte grid.
template <typename T, int VEC>
bool glr_tiles(ard_ctx* ctx, const GlrArgs& a, std::initializer_list<std::pair<const void*, int>> operands, int channels, int steps, GlrTiles* out) {
  int m = 0;
  for (const auto& op : operands) {
    if ((reinterpret_cast<uintptr_t>(op.first) & 15u) || (op.second * sizeof(T)) % 16) return false;
    if (!ard_encode_steps(ctx, &out->map[m++], sizeof(T) == 4, op.first, a.H, a.B, a.T, op.second, channels, steps)) return false;
  }
  return true;
}

// Steps of a thread.  A slab either holds the whole sequence or begins where the forward call left a state, every 64
// steps: 2 or 5 steps a thread where 8 warps of them reach the end, three CTAs an SM, otherwise 8, two CTAs an SM.  T x
// 64 x 1024 bf16, forward / backward:
//   T = 16         2 steps 6.3 / 7.8 us    5 steps 8.5 / 11.8     8 steps 10.8 / 15.9
//   T = 17, 24     5 steps 8.4 / 11.9, 8.5 / 12.6                 8 steps 10.8 / 16.0, 10.8 / 16.6
//   T = 35, 40     5 steps 8.8 / 14.5, 8.3 / 13.6                 8 steps 11.2 / 17.6, 11.5 / 18.1
//   T = 48, 64     8 steps 12.4 / 18.9, 12.6 / 17.9
// (16 in clusters, one CTA an SM: what a round costs besides its steps is paid half as often, but nothing runs beside
// it: 16384 x 1 x 1024 50.9 / 81.2 us.) Clusters where the units leave more than half of the SMs idle.  T = 4096, units
// a warp wide: 60 of them 36 / 58 us, 74 48 / 76, in clusters; 75, 100, 147, 148 a CTA each 76 / 116, 88 / 137, 89 /
// 139, 72 / 112, where clusters of two or three (two CTAs fit an SM) would take 48 / 76, 65 / 105, 66 / 107, 66 / 107:
// the edge stands too low. Units as wide as a warp, or as half of one, twice as many steps long, where clusters of all
// that may share a sequence would leave SMs idle: 16384 x 1 x 1024 49.5 / 76.5 us in whole warps, 40.3 / 69.2 in
// halves; 16384 x 1 x 2048, which fills them either way, 71 / 117 and 71 / 128. run(SPT, W, CTAs an SM, cluster).
template <typename Run>
ard_status glr_steps(ard_ctx* ctx, const GlrArgs& a, int vec, Run run) {
  constexpr std::integral_constant<int, 32> warp{};
  constexpr std::integral_constant<int, 16> half{};
  constexpr std::integral_constant<int, 8> eight{};
  if (a.T <= 16) return run(std::integral_constant<int, 2>{}, warp, 3, 1);
  if (a.T <= 40) return run(std::integral_constant<int, 5>{}, warp, 3, 1);
  const long long units = glr_units(a, 32 * vec);
  if (2 * units > ctx->sm_count) return run(eight, warp, 2, 1);
  if (units * GLR_CLUSTER > 2 * ctx->sm_count) return run(eight, warp, 2, glr_cluster(ctx, units, ((long long)a.T + 63) / 64));
  return run(eight, half, 2, glr_cluster(ctx, glr_units(a, 16 * vec), ((long long)a.T + 127) / 128));
}

template <typename T, int VEC, bool GATE>
struct GlrFwd {
  static ard_status run(ard_ctx* ctx, const GlrArgs& a, cudaStream_t s) {
    GlrTiles tiles;
    if (a.T <= 1) return glr_launch(ctx, glr_fwd_kernel<T, VEC, GATE, 128, 1, 1, false>, a, tiles, 128 * VEC, 1, 128, 0, 8, s);
    return glr_steps(ctx, a, VEC, [&](auto steps, auto width, int per_sm, int CL) {
      constexpr int SPT = decltype(steps)::value, W = decltype(width)::value, WT = 256 / W;
      if constexpr (VEC * sizeof(T) == 4) {
        bool ok;
        if constexpr (GATE) ok = glr_tiles<T, VEC>(ctx, a, {{a.Zf, a.ldz}, {a.Zg, a.ldz}, {a.Zo, a.ldz}}, W * VEC, WT * SPT, &tiles);
        else ok = glr_tiles<T, VEC>(ctx, a, {{a.Zf, a.ldz}, {a.Zg, a.ldz}}, W * VEC, WT * SPT, &tiles);
        if (ok)
          return glr_launch(ctx, glr_fwd_kernel<T, VEC, GATE, W, WT, SPT, true>, a, tiles, W * VEC, CL, 256,
                            glr_ring<GlrFeed<T, VEC, GATE ? 3 : 2, W, WT, SPT, true>>(), per_sm, s);
      }
      return glr_launch(ctx, glr_fwd_kernel<T, VEC, GATE, W, WT, SPT, false>, a, tiles, W * VEC, CL, 256, 0, per_sm, s);
    });
  }
};
template <typename T, int VEC, bool GATE>
struct GlrBwd {
  static ard_status run(ard_ctx* ctx, const GlrArgs& a, cudaStream_t s) {
    GlrTiles tiles;
    if (a.T <= 1) return glr_launch(ctx, glr_bwd_kernel<T, VEC, GATE, 128, 1, 1, false>, a, tiles, 128 * VEC, 1, 128, 0, 8, s);
    return glr_steps(ctx, a, VEC, [&](auto steps, auto width, int per_sm, int CL) {
      constexpr int SPT = decltype(steps)::value, W = decltype(width)::value, WT = 256 / W;
      if constexpr (VEC * sizeof(T) == 4) {
        bool ok;
        if constexpr (GATE) ok = glr_tiles<T, VEC>(ctx, a, {{a.Zf, a.ldz}, {a.Zg, a.ldz}, {a.dY, a.ldy}, {a.Zo, a.ldz}}, W * VEC, WT * SPT, &tiles);
        else ok = glr_tiles<T, VEC>(ctx, a, {{a.Zf, a.ldz}, {a.Zg, a.ldz}, {a.dY, a.ldy}}, W * VEC, WT * SPT, &tiles);
        if (ok)
          return glr_launch(ctx, glr_bwd_kernel<T, VEC, GATE, W, WT, SPT, true>, a, tiles, W * VEC, CL, 256,
                            glr_ring<GlrFeed<T, VEC, GATE ? 4 : 3, W, WT, SPT, true>>(), per_sm, s);
      }
      // 2-byte values fetched into registers: half the steps a thread, in units of half a warp (a slab is 64 steps, as
      // the states lie), rather than registers spilt: 2048 x 8 x 2044 192 -> 152 us (4-byte values 118 -> 128, forward
      // 75 -> 82: those stay)
      if constexpr (SPT == 8 && sizeof(T) == 2)
        return glr_launch(ctx, glr_bwd_kernel<T, VEC, GATE, 16, 16, 4, false>, a, tiles, 16 * VEC, CL, 256, 0, per_sm, s);
      else return glr_launch(ctx, glr_bwd_kernel<T, VEC, GATE, W, WT, SPT, false>, a, tiles, W * VEC, CL, 256, 0, per_sm, s);
    });
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
