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

#include "ard_internal.h"

namespace {

namespace cg = cooperative_groups;

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
  int groups;  // groups of channels of a sequence
};

// s(z) and 1 - s(z), each to the last bits of its own: where s(z) is above a half the other one is exp(-z) times it, not a difference.  exp(-z) of
// infinity gives 0 and 1.
__device__ __forceinline__ float glr_gate(float z, float& rest) {
  const float u = __expf(-z), f = __fdividef(1.f, 1.f + u);
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

// What a thread works on: VEC channels of one sequence, SPT consecutive steps of every slab.
template <int VEC, int CW, int WT>
struct GlrPlace {
  int lane, cw, wt, b, j, n, valid, col, len, dp, b0;
  __device__ __forceinline__ GlrPlace(const GlrArgs& a, int group) {
    const int warp = threadIdx.x >> 5;
    lane = threadIdx.x & 31;
    cw = warp / WT;
    wt = warp % WT;
    n = a.H;
    dp = 1;
    b0 = 0;
    if (a.hdr) {
      n = a.hdr[HDR_NKEEP];
      dp = a.hdr[HDR_DP];
      b0 = a.hdr[HDR_B] - 1;
    }
    b = group / a.groups;
    j = ((group % a.groups) * CW + cw) * 32 * VEC + lane * VEC;
    valid = max(0, min(VEC, n - j));
    col = min(j, (n - 1) / VEC * VEC);  // where a lane without channels reads
    len = a.T;
    if (a.lens) len = min(max(a.lens[b], 0), a.T);
  }
  __device__ __forceinline__ size_t unit(const GlrArgs& a, int v) const { return (size_t)b * a.H + b0 + (size_t)(j + v) * dp; }
};

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

// The exchange of a slab: from this thread's map and the state x that enters the round, the state that enters this thread's steps and, in x, the
// one behind the round.  s_warp: [2][WT][CW * 32]; s_slab: [2][8][CW * 32], where the cluster's CTAs leave their slabs' maps.  Warps count in the order
// of the steps (first = 0, +1) or against it.
template <int VEC, int CW, int WT>
__device__ __forceinline__ void glr_exchange(const GlrPlace<VEC, CW, WT>& at, int it, int CL, int rank, bool forward, const GlrMap<VEC>& mine,
                                             GlrMap<VEC> (*s_warp)[WT][CW * 32], GlrMap<VEC> (*s_slab)[8][CW * 32], float (&x)[VEC],
                                             float (&enters)[VEC]) {
  GlrMap<VEC> before = GlrMap<VEC>::none(), all = mine;
  const int ch = at.cw * 32 + at.lane;
  if constexpr (WT > 1) {  // (the caller has stored the maps and passed a barrier)
    all = before;
#pragma unroll
    for (int k = 0; k < WT; ++k) {
      const int w = forward ? k : WT - 1 - k;
      if (w == at.wt) before = all;
      all.then(s_warp[it & 1][w][ch]);
    }
  }
  if (CL > 1) {
    cg::cluster_group cl = cg::this_cluster();
    if (at.wt == 0)
      for (int r = 0; r < CL; ++r) *cl.map_shared_rank(&s_slab[it & 1][rank][ch], r) = all;
    cl.sync();
    for (int r = 0; r < CL; ++r) {
      const GlrMap<VEC> m = s_slab[it & 1][r][ch];
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

// The values of the next slab are fetched as soon as this one's are out of their registers, so that they are on their way while the
// maps are exchanged and the outputs written.
template <typename T, int VEC, bool GATE, int CW, int WT, int SPT>
__global__ void __launch_bounds__(CW* WT * 32) glr_fwd_kernel(const GlrArgs a, int CL) {
  __shared__ GlrMap<VEC> s_warp[2][WT][CW * 32];
  __shared__ GlrMap<VEC> s_slab[2][8][CW * 32];
  if (CL > 1) cg::this_cluster().sync();  // the others' memory is written only once they run
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int group = blockIdx.x / CL, rank = blockIdx.x % CL;
  const GlrPlace<VEC, CW, WT> at(a, group);
  if ((group % a.groups) * CW * 32 * VEC >= at.n) return;  // all CTAs of a cluster alike
  constexpr int SLAB = WT * SPT;
  const size_t step_z = (size_t)a.B * a.ldz, step_y = (size_t)a.B * a.ldy;
  const T* zf = (const T*)a.Zf + (size_t)at.b * a.ldz + at.col;
  const T* zg = (const T*)a.Zg + (size_t)at.b * a.ldz + at.col;
  const T* zo = GATE ? (const T*)a.Zo + (size_t)at.b * a.ldz + at.col : nullptr;
  T* y = (T*)a.Y + (size_t)at.b * a.ldy + at.j;
  uint32_t qf[SPT], qg[SPT], qo[GATE ? SPT : 1];
  auto fetch = [&](int t0) {
    if (t0 >= at.len) return;
#pragma unroll
    for (int k = 0; k < SPT; ++k) {
      const size_t row = (size_t)min(t0 + k, at.len - 1) * step_z;  // behind the end: the last row, whose values are not used
      qf[k] = glr_fetch<T, VEC>(zf + row);
      qg[k] = glr_fetch<T, VEC>(zg + row);
      if constexpr (GATE) qo[k] = glr_fetch<T, VEC>(zo + row);
    }
  };
  const int rounds = (a.T + SLAB * CL - 1) / (SLAB * CL);
  fetch(rank * SLAB + at.wt * SPT);
  float cs[VEC];  // the state that enters the round
#pragma unroll
  for (int v = 0; v < VEC; ++v) cs[v] = a.h0 && v < at.valid ? a.h0[at.unit(a, v)] : 0.f;
  for (int it = 0; it < rounds; ++it) {
    const int t0 = (it * CL + rank) * SLAB + at.wt * SPT;
    float f[SPT][VEC], x[SPT][VEC], o[GATE ? SPT : 1][VEC];
    GlrMap<VEC> map = GlrMap<VEC>::none();
#pragma unroll
    for (int k = 0; k < SPT; ++k) {
      glr_unpack<T, VEC>(qf[k], f[k]);
      glr_unpack<T, VEC>(qg[k], x[k]);
      if constexpr (GATE) glr_unpack<T, VEC>(qo[k], o[k]);
      const bool in = t0 + k < at.len;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        float rest;
        f[k][v] = glr_gate(f[k][v], rest);
        x[k][v] *= rest;
        if (!in) {
          f[k][v] = 1.f;
          x[k][v] = 0.f;
        }
        map.a[v] *= f[k][v];
        map.b[v] = fmaf(f[k][v], map.b[v], x[k][v]);
        if constexpr (GATE) o[k][v] = a.alpha * __fdividef(1.f, 1.f + __expf(-o[k][v]));
      }
    }
    if (it + 1 < rounds) fetch(t0 + SLAB * CL);
    if constexpr (WT > 1) {
      s_warp[it & 1][at.wt][at.cw * 32 + at.lane] = map;
      __syncthreads();
    }
    float c[VEC];
    glr_exchange<VEC, CW, WT>(at, it, CL, rank, true, map, s_warp, s_slab, cs, c);
    if (a.S && t0 % ARD_GLR_CHUNK == 0 && t0 < a.T)
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        if (v < at.valid) a.S[((size_t)(t0 / ARD_GLR_CHUNK) * a.B + at.b) * a.H + at.j + v] = c[v];
#pragma unroll
    for (int k = 0; k < SPT; ++k) {
      float out[VEC];
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        c[v] = fmaf(f[k][v], c[v], x[k][v]);
        out[v] = t0 + k < at.len ? (GATE ? o[k][v] : a.alpha) * c[v] : 0.f;
      }
      if (t0 + k < a.T) glr_store<T, VEC>(y + (size_t)(t0 + k) * step_y, at.valid, out);
    }
  }
  if (a.hT && rank == 0 && at.wt == 0)
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      if (v < at.valid) a.hT[at.unit(a, v)] = cs[v];
}

template <typename T, int VEC, bool GATE, int CW, int WT, int SPT>
__global__ void __launch_bounds__(CW* WT * 32) glr_bwd_kernel(const GlrArgs a, int CL) {
  __shared__ GlrMap<VEC> s_warp[2][WT][CW * 32], s_back[2][WT][CW * 32];
  __shared__ GlrMap<VEC> s_slab[2][8][CW * 32];
  if (CL > 1) cg::this_cluster().sync();
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int group = blockIdx.x / CL, rank = blockIdx.x % CL;
  const GlrPlace<VEC, CW, WT> at(a, group);
  if ((group % a.groups) * CW * 32 * VEC >= at.n) return;
  constexpr int SLAB = WT * SPT;
  const int ch = at.cw * 32 + at.lane;
  const size_t step_z = (size_t)a.B * a.ldz, step_y = (size_t)a.B * a.ldy, step_d = (size_t)a.B * a.lddz;
  const T* zf = (const T*)a.Zf + (size_t)at.b * a.ldz + at.col;
  const T* zg = (const T*)a.Zg + (size_t)at.b * a.ldz + at.col;
  const T* zo = GATE ? (const T*)a.Zo + (size_t)at.b * a.ldz + at.col : nullptr;
  const T* dy = (const T*)a.dY + (size_t)at.b * a.ldy + at.col;
  const size_t off_d = (size_t)at.b * a.lddz + at.j;
  T* dzf = (T*)a.dZf + off_d;
  T* dzg = (T*)a.dZg + off_d;
  T* dzo = GATE ? (T*)a.dZo + off_d : nullptr;
  const int rounds = (a.T + SLAB * CL - 1) / (SLAB * CL);
  // rounds and ranks run from the end; the first slabs may lie behind T
  auto start = [&](int it) { return (rounds * CL - 1 - (it * CL + rank)) * SLAB; };
  uint32_t qf[SPT], qg[SPT], qy[SPT], qo[GATE ? SPT : 1];
  auto fetch = [&](int t0) {
    if (t0 >= at.len) return;
#pragma unroll
    for (int k = 0; k < SPT; ++k) {
      const size_t t = (size_t)min(t0 + k, at.len - 1);
      qf[k] = glr_fetch<T, VEC>(zf + t * step_z);
      qg[k] = glr_fetch<T, VEC>(zg + t * step_z);
      if constexpr (GATE) qo[k] = glr_fetch<T, VEC>(zo + t * step_z);
      qy[k] = glr_fetch<T, VEC>(dy + t * step_y);
    }
  };
  if (rounds > 0) fetch(start(0) + at.wt * SPT);
  float qs[VEC];  // what arrives behind the round's last step
#pragma unroll
  for (int v = 0; v < VEC; ++v) qs[v] = a.h0 && v < at.valid ? a.h0[at.unit(a, v)] : 0.f;
  for (int it = 0; it < rounds; ++it) {
    const int ts = start(it), t0 = ts + at.wt * SPT;
    float c0[VEC];  // the state that enters the slab
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      c0[v] = ts < a.T && v < at.valid ? a.S[((size_t)(ts / ARD_GLR_CHUNK) * a.B + at.b) * a.H + at.j + v] : 0.f;
    // e: alpha s(zo) dy, what arrives at c from y; no: 1 - s(zo)
    float f[SPT][VEC], i[SPT][VEC], g[SPT][VEC], e[SPT][VEC], no[GATE ? SPT : 1][VEC];
    GlrMap<VEC> map = GlrMap<VEC>::none(), back;
#pragma unroll
    for (int k = 0; k < SPT; ++k) {
      glr_unpack<T, VEC>(qf[k], f[k]);
      glr_unpack<T, VEC>(qg[k], g[k]);
      glr_unpack<T, VEC>(qy[k], e[k]);
      if constexpr (GATE) glr_unpack<T, VEC>(qo[k], no[k]);
      const bool in = t0 + k < at.len;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        f[k][v] = glr_gate(f[k][v], i[k][v]);
        e[k][v] *= a.alpha;
        if constexpr (GATE) e[k][v] *= glr_gate(no[k][v], no[k][v]);
        if (!in) {
          f[k][v] = 1.f;
          i[k][v] = g[k][v] = e[k][v] = 0.f;
          if constexpr (GATE) no[k][v] = 0.f;
        }
        map.a[v] *= f[k][v];
        map.b[v] = fmaf(f[k][v], map.b[v], i[k][v] * g[k][v]);
      }
    }
    if (it + 1 < rounds) fetch(start(it + 1) + at.wt * SPT);
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      back.a[v] = map.a[v];
      back.b[v] = 0.f;
#pragma unroll
      for (int k = SPT - 1; k >= 0; --k) back.b[v] = f[k][v] * (e[k][v] + back.b[v]);
    }
    GlrMap<VEC> before = GlrMap<VEC>::none();
    if constexpr (WT > 1) {
      s_warp[it & 1][at.wt][ch] = map;
      s_back[it & 1][at.wt][ch] = back;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < WT - 1; ++w)
        if (w < at.wt) before.then(s_warp[it & 1][w][ch]);
    }
    float q[VEC];
    glr_exchange<VEC, CW, WT>(at, it, CL, rank, false, back, s_back, s_slab, qs, q);
    float c[SPT + 1][VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      c[0][v] = before.of(c0[v], v);
#pragma unroll
      for (int k = 0; k < SPT; ++k) c[k + 1][v] = fmaf(f[k][v], c[k][v], i[k][v] * g[k][v]);
    }
#pragma unroll
    for (int k = SPT - 1; k >= 0; --k) {
      float of[VEC], og[VEC], oo[VEC];
      const bool in = t0 + k < at.len;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float d = e[k][v] + q[v], di = d * i[k][v];
        q[v] = f[k][v] * d;
        of[v] = in ? di * f[k][v] * (c[k][v] - g[k][v]) : 0.f;
        og[v] = in ? di : 0.f;
        if constexpr (GATE) oo[v] = in ? e[k][v] * c[k + 1][v] * no[k][v] : 0.f;
      }
      if (t0 + k < a.T) {
        const size_t row = (size_t)(t0 + k) * step_d;
        glr_store<T, VEC>(dzf + row, at.valid, of);
        glr_store<T, VEC>(dzg + row, at.valid, og);
        if constexpr (GATE) glr_store<T, VEC>(dzo + row, at.valid, oo);
      }
    }
  }
  if (a.hT && rank == 0 && at.wt == 0)
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      if (v < at.valid) a.hT[at.unit(a, v)] = qs[v];
}

// bf16 columns on a grid of two: read and written in pairs.
inline bool glr_pairs(std::initializer_list<const void*> ps, std::initializer_list<int> lds) {
  for (const void* p : ps)
    if (reinterpret_cast<uintptr_t>(p) % 4) return false;
  for (int ld : lds)
    if (ld % 2) return false;
  return true;
}

// A cluster's CTAs take consecutive slabs of the time axis where the channels alone leave SMs idle.
template <typename K>
ard_status glr_launch(ard_ctx* ctx, K kern, GlrArgs a, int channels, int slab, int threads, cudaStream_t s) {
  a.groups = (a.H + channels - 1) / channels;
  const long long slabs = ((long long)a.T + slab - 1) / slab, units = (long long)a.groups * a.B;
  int CL = 1;
  while (CL < 8 && 2 * CL <= slabs && units * CL < 2 * ctx->sm_count) CL *= 2;
  const long long blocks = units * CL;
  if (blocks > 0x7FFFFFFFll) return ARD_ERR_UNSUPPORTED;
  if (CL > 1) ARD_CUDA_OK(ard_launch_cluster(ctx, kern, CL, dim3((unsigned)blocks), dim3(threads), 0, s, a, CL));
  else ARD_CUDA_OK(ard_launch(ctx, kern, dim3((unsigned)blocks), dim3(threads), 0, s, a, CL));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}

template <typename T, int VEC, bool GATE>
struct GlrFwd {
  static ard_status run(ard_ctx* ctx, const GlrArgs& a, cudaStream_t s) {
    if (a.T <= 1) return glr_launch(ctx, glr_fwd_kernel<T, VEC, GATE, 4, 1, 1>, a, 4 * 32 * VEC, 1, 128, s);
    return glr_launch(ctx, glr_fwd_kernel<T, VEC, GATE, 1, 8, 8>, a, 32 * VEC, 64, 256, s);
  }
};
template <typename T, int VEC, bool GATE>
struct GlrBwd {
  static ard_status run(ard_ctx* ctx, const GlrArgs& a, cudaStream_t s) {
    if (a.T <= 1) return glr_launch(ctx, glr_bwd_kernel<T, VEC, GATE, 4, 1, 1>, a, 4 * 32 * VEC, 1, 128, s);
    return glr_launch(ctx, glr_bwd_kernel<T, VEC, GATE, 1, 8, 8>, a, 32 * VEC, 64, 256, s);
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
  return glr_dispatch<GlrBwd>(ctx, dtype == ARD_F32, glr_pairs({Zf, Zg, Zo, dY, dZf, dZg, dZo}, {ldz, lddy, lddz}), a, s);
}
