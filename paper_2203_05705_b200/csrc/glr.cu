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

// s(z) and 1 - s(z), each to the last bits of its own: u = exp(-|z|) never overflows, and neither is a difference.
__device__ __forceinline__ void glr_gate(float z, float& f, float& i) {
  const float u = __expf(-fabsf(z)), r = __fdividef(1.f, 1.f + u), ur = u * r;
  f = z >= 0.f ? r : ur;
  i = z >= 0.f ? ur : r;
}

template <int VEC>
__device__ __forceinline__ void glr_load(const float* p, float (&v)[VEC]) {
  if constexpr (VEC == 2) {
    const float2 q = *reinterpret_cast<const float2*>(p);
    v[0] = q.x;
    v[1] = q.y;
  } else {
    v[0] = *p;
  }
}
template <int VEC>
__device__ __forceinline__ void glr_load(const __nv_bfloat16* p, float (&v)[VEC]) {
  if constexpr (VEC == 2) {
    const uint32_t q = *reinterpret_cast<const uint32_t*>(p);
    v[0] = __uint_as_float(q << 16);
    v[1] = __uint_as_float(q & 0xFFFF0000u);
  } else {
    v[0] = __bfloat162float(*p);
  }
}
// The first `valid` of the values.
template <int VEC>
__device__ __forceinline__ void glr_store(float* p, int valid, const float (&v)[VEC]) {
  if constexpr (VEC == 2) {
    if (valid >= 2) {
      *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
      return;
    }
  }
  if (valid >= 1) *p = v[0];
}
template <int VEC>
__device__ __forceinline__ void glr_store(__nv_bfloat16* p, int valid, const float (&v)[VEC]) {
  if constexpr (VEC == 2) {
    if (valid >= 2) {
      *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(v[0], v[1]);
      return;
    }
  }
  if (valid >= 1) *p = __float2bfloat16(v[0]);
}

// What a thread works on: VEC channels of one sequence, SPT consecutive steps of every slab.
template <int VEC, int CW, int WT>
struct GlrPlace {
  int lane, cw, wt, b, j, n, valid, len, dp, b0;
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
    len = a.T;
    if (a.lens) len = min(max(a.lens[b], 0), a.T);
  }
  __device__ __forceinline__ size_t unit(const GlrArgs& a, int v) const { return (size_t)b * a.H + b0 + (size_t)(j + v) * dp; }
};

// The maps of a slab's warps, or of the cluster's slabs: [A, B][channel].
template <int VEC, int CW>
struct GlrMaps {
  float a[CW * 32 * VEC], b[CW * 32 * VEC];
};

template <typename T, int VEC, bool GATE, int CW, int WT, int SPT>
__global__ void __launch_bounds__(CW* WT * 32) glr_fwd_kernel(const GlrArgs a, int CL) {
  __shared__ GlrMaps<VEC, CW> s_warp[2][WT];
  __shared__ GlrMaps<VEC, CW> s_slab[2];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int group = blockIdx.x / CL, rank = blockIdx.x % CL;
  const GlrPlace<VEC, CW, WT> at(a, group);
  if ((group % a.groups) * CW * 32 * VEC >= at.n) return;  // all CTAs of a cluster alike
  constexpr int SLAB = WT * SPT;
  const int ch = at.cw * 32 * VEC + at.lane * VEC;
  const size_t step_z = (size_t)a.B * a.ldz, step_y = (size_t)a.B * a.ldy;
  const T* zf = (const T*)a.Zf + (size_t)at.b * a.ldz + at.j;
  const T* zg = (const T*)a.Zg + (size_t)at.b * a.ldz + at.j;
  const T* zo = GATE ? (const T*)a.Zo + (size_t)at.b * a.ldz + at.j : nullptr;
  T* y = (T*)a.Y + (size_t)at.b * a.ldy + at.j;
  float cs[VEC];  // the state that enters the cluster's slabs
#pragma unroll
  for (int v = 0; v < VEC; ++v) cs[v] = a.h0 && v < at.valid ? a.h0[at.unit(a, v)] : 0.f;
  const int rounds = (a.T + SLAB * CL - 1) / (SLAB * CL);
  for (int it = 0; it < rounds; ++it) {
    const int t0 = (it * CL + rank) * SLAB + at.wt * SPT;
    float f[SPT][VEC], x[SPT][VEC], o[GATE ? SPT : 1][VEC];
#pragma unroll
    for (int k = 0; k < SPT; ++k) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) f[k][v] = x[k][v] = 0.f;
      if (t0 + k < at.len && at.valid > 0) {
        glr_load<VEC>(zf + (size_t)(t0 + k) * step_z, f[k]);
        glr_load<VEC>(zg + (size_t)(t0 + k) * step_z, x[k]);
        if constexpr (GATE) glr_load<VEC>(zo + (size_t)(t0 + k) * step_z, o[k]);
      }
    }
    float A[VEC], Bv[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      A[v] = 1.f;
      Bv[v] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < SPT; ++k)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        float ff, ii;
        glr_gate(f[k][v], ff, ii);
        const bool in = t0 + k < at.len;
        f[k][v] = in ? ff : 1.f;
        x[k][v] = in ? ii * x[k][v] : 0.f;
        A[v] *= f[k][v];
        Bv[v] = fmaf(f[k][v], Bv[v], x[k][v]);
      }
    // the state that enters this thread's steps, and the one behind the cluster's slabs
    float c[VEC];
    float pa[VEC], pb[VEC];  // of the warps before this one
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      pa[v] = 1.f;
      pb[v] = 0.f;
    }
    if constexpr (WT > 1) {
      GlrMaps<VEC, CW>* maps = s_warp[it & 1];
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        maps[at.wt].a[ch + v] = A[v];
        maps[at.wt].b[ch + v] = Bv[v];
      }
      __syncthreads();
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        A[v] = 1.f;
        Bv[v] = 0.f;
      }
#pragma unroll
      for (int w = 0; w < WT; ++w)
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          if (w == at.wt) {
            pa[v] = A[v];
            pb[v] = Bv[v];
          }
          const float ma = maps[w].a[ch + v], mb = maps[w].b[ch + v];
          A[v] *= ma;
          Bv[v] = fmaf(ma, Bv[v], mb);
        }
    }
    if (CL > 1) {
      GlrMaps<VEC, CW>* mine = &s_slab[it & 1];
      if (at.wt == 0)
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          mine->a[ch + v] = A[v];
          mine->b[ch + v] = Bv[v];
        }
      cg::cluster_group cl = cg::this_cluster();
      cl.sync();
      for (int r = 0; r < CL; ++r) {
        const GlrMaps<VEC, CW>* m = cl.map_shared_rank(mine, r);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          if (r == rank) c[v] = cs[v];
          cs[v] = fmaf(m->a[ch + v], cs[v], m->b[ch + v]);
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        c[v] = cs[v];
        cs[v] = fmaf(A[v], cs[v], Bv[v]);
      }
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) c[v] = fmaf(pa[v], c[v], pb[v]);
    if (a.S && t0 % ARD_GLR_CHUNK == 0 && t0 < a.T)
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        if (v < at.valid) a.S[((size_t)(t0 / ARD_GLR_CHUNK) * a.B + at.b) * a.H + at.j + v] = c[v];
#pragma unroll
    for (int k = 0; k < SPT; ++k) {
      if (t0 + k >= a.T) break;
      float out[VEC];
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        c[v] = fmaf(f[k][v], c[v], x[k][v]);
        float gate = a.alpha, rest;
        if constexpr (GATE) {
          glr_gate(o[k][v], gate, rest);
          gate *= a.alpha;
        }
        out[v] = t0 + k < at.len ? gate * c[v] : 0.f;
      }
      glr_store<VEC>(y + (size_t)(t0 + k) * step_y, at.valid, out);
    }
  }
  if (a.hT && rank == 0 && at.wt == 0)
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      if (v < at.valid) a.hT[at.unit(a, v)] = cs[v];
  if (CL > 1) cg::this_cluster().sync();  // nobody leaves while its maps may still be read
}

template <typename T, int VEC, bool GATE, int CW, int WT, int SPT>
__global__ void __launch_bounds__(CW* WT * 32) glr_bwd_kernel(const GlrArgs a, int CL) {
  struct Maps {
    GlrMaps<VEC, CW> fwd;
    float b[CW * 32 * VEC];  // of the adjoint's map, whose A is the same
  };
  __shared__ Maps s_warp[2][WT];
  __shared__ GlrMaps<VEC, CW> s_slab[2];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int group = blockIdx.x / CL, rank = blockIdx.x % CL;
  const GlrPlace<VEC, CW, WT> at(a, group);
  if ((group % a.groups) * CW * 32 * VEC >= at.n) return;
  constexpr int SLAB = WT * SPT;
  const int ch = at.cw * 32 * VEC + at.lane * VEC;
  const size_t step_z = (size_t)a.B * a.ldz, step_y = (size_t)a.B * a.ldy, step_d = (size_t)a.B * a.lddz;
  const size_t off_z = (size_t)at.b * a.ldz + at.j, off_d = (size_t)at.b * a.lddz + at.j;
  const T* zf = (const T*)a.Zf + off_z;
  const T* zg = (const T*)a.Zg + off_z;
  const T* zo = GATE ? (const T*)a.Zo + off_z : nullptr;
  const T* dy = (const T*)a.dY + (size_t)at.b * a.ldy + at.j;
  T* dzf = (T*)a.dZf + off_d;
  T* dzg = (T*)a.dZg + off_d;
  T* dzo = GATE ? (T*)a.dZo + off_d : nullptr;
  float qs[VEC];  // what arrives behind the cluster's slabs
#pragma unroll
  for (int v = 0; v < VEC; ++v) qs[v] = a.h0 && v < at.valid ? a.h0[at.unit(a, v)] : 0.f;
  const int rounds = (a.T + SLAB * CL - 1) / (SLAB * CL);
  for (int it = 0; it < rounds; ++it) {
    const int slab = rounds * CL - 1 - (it * CL + rank);  // from the end; the first ones may lie behind T
    const int ts = slab * SLAB, t0 = ts + at.wt * SPT;
    float f[SPT][VEC], i[SPT][VEC], g[SPT][VEC], e[SPT][VEC], o[GATE ? SPT : 1][VEC];
#pragma unroll
    for (int k = 0; k < SPT; ++k) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        f[k][v] = g[k][v] = e[k][v] = 0.f;
        if constexpr (GATE) o[k][v] = 0.f;
      }
      if (t0 + k < at.len && at.valid > 0) {
        glr_load<VEC>(zf + (size_t)(t0 + k) * step_z, f[k]);
        glr_load<VEC>(zg + (size_t)(t0 + k) * step_z, g[k]);
        glr_load<VEC>(dy + (size_t)(t0 + k) * step_y, e[k]);
        if constexpr (GATE) glr_load<VEC>(zo + (size_t)(t0 + k) * step_z, o[k]);
      }
    }
    float A[VEC], Bv[VEC], Q[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      A[v] = 1.f;
      Bv[v] = Q[v] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < SPT; ++k)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const bool in = t0 + k < at.len;
        glr_gate(f[k][v], f[k][v], i[k][v]);
        if (!in) {
          f[k][v] = 1.f;
          i[k][v] = 0.f;
        }
        A[v] *= f[k][v];
        Bv[v] = fmaf(f[k][v], Bv[v], i[k][v] * g[k][v]);
        e[k][v] *= a.alpha;  // e: alpha dy
      }
    float go[GATE ? SPT : 1][VEC];
#pragma unroll
    for (int k = SPT - 1; k >= 0; --k)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        float arrives = e[k][v];
        if constexpr (GATE) {
          glr_gate(o[k][v], go[k][v], o[k][v]);  // s(zo), 1 - s(zo)
          arrives *= go[k][v];
        }
        Q[v] = f[k][v] * (arrives + Q[v]);
      }
    float c[VEC], q[VEC], ca[VEC], cb[VEC], qa[VEC], qb[VEC];  // maps of the warps before and behind this one
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      c[v] = ts < a.T && v < at.valid ? a.S[((size_t)(ts / ARD_GLR_CHUNK) * a.B + at.b) * a.H + at.j + v] : 0.f;
      ca[v] = qa[v] = 1.f;
      cb[v] = qb[v] = 0.f;
    }
    if constexpr (WT > 1) {
      Maps* maps = s_warp[it & 1];
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        maps[at.wt].fwd.a[ch + v] = A[v];
        maps[at.wt].fwd.b[ch + v] = Bv[v];
        maps[at.wt].b[ch + v] = Q[v];
      }
      __syncthreads();
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        A[v] = 1.f;
        Q[v] = 0.f;
      }
#pragma unroll
      for (int w = 0; w < WT; ++w)
        if (w < at.wt)
#pragma unroll
          for (int v = 0; v < VEC; ++v) {
            const float ma = maps[w].fwd.a[ch + v];
            ca[v] *= ma;
            cb[v] = fmaf(ma, cb[v], maps[w].fwd.b[ch + v]);
          }
#pragma unroll
      for (int w = WT - 1; w >= 0; --w)
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          if (w == at.wt) {
            qa[v] = A[v];
            qb[v] = Q[v];
          }
          const float ma = maps[w].fwd.a[ch + v];
          A[v] *= ma;
          Q[v] = fmaf(ma, Q[v], maps[w].b[ch + v]);
        }
    }
    if (CL > 1) {
      GlrMaps<VEC, CW>* mine = &s_slab[it & 1];
      if (at.wt == 0)
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          mine->a[ch + v] = A[v];
          mine->b[ch + v] = Q[v];
        }
      cg::cluster_group cl = cg::this_cluster();
      cl.sync();
      for (int r = 0; r < CL; ++r) {
        const GlrMaps<VEC, CW>* m = cl.map_shared_rank(mine, r);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          if (r == rank) q[v] = qs[v];
          qs[v] = fmaf(m->a[ch + v], qs[v], m->b[ch + v]);
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        q[v] = qs[v];
        qs[v] = fmaf(A[v], qs[v], Q[v]);
      }
    }
    float before[SPT][VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      c[v] = fmaf(ca[v], c[v], cb[v]);
      q[v] = fmaf(qa[v], q[v], qb[v]);
#pragma unroll
      for (int k = 0; k < SPT; ++k) {
        before[k][v] = c[v];
        c[v] = fmaf(f[k][v], c[v], i[k][v] * g[k][v]);
      }
    }
#pragma unroll
    for (int k = SPT - 1; k >= 0; --k) {
      float of[VEC], og[VEC], oo[VEC];
      const bool in = t0 + k < at.len;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        float arrives = e[k][v];
        oo[v] = 0.f;
        if constexpr (GATE) {
          const float now = fmaf(f[k][v], before[k][v], i[k][v] * g[k][v]);
          arrives *= go[k][v];
          oo[v] = in ? arrives * now * o[k][v] : 0.f;
        }
        const float d = arrives + q[v], di = d * i[k][v];
        q[v] = f[k][v] * d;
        of[v] = in ? di * f[k][v] * (before[k][v] - g[k][v]) : 0.f;
        og[v] = in ? di : 0.f;
      }
      if (t0 + k < a.T) {
        glr_store<VEC>(dzf + (size_t)(t0 + k) * step_d, at.valid, of);
        glr_store<VEC>(dzg + (size_t)(t0 + k) * step_d, at.valid, og);
        if constexpr (GATE) glr_store<VEC>(dzo + (size_t)(t0 + k) * step_d, at.valid, oo);
      }
    }
  }
  if (a.hT && rank == 0 && at.wt == 0)
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      if (v < at.valid) a.hT[at.unit(a, v)] = qs[v];
  if (CL > 1) cg::this_cluster().sync();
}

inline bool glr_pairs(size_t es, std::initializer_list<const void*> ps, std::initializer_list<int> lds) {
  for (const void* p : ps)
    if (reinterpret_cast<uintptr_t>(p) % (2 * es)) return false;
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
    return glr_launch(ctx, glr_bwd_kernel<T, VEC, GATE, 1, 16, 4>, a, 32 * VEC, 64, 512, s);
  }
};

template <template <typename, int, bool> class Op>
ard_status glr_dispatch(ard_ctx* ctx, bool f32, bool pairs, const GlrArgs& a, cudaStream_t s) {
  const bool gate = a.Zo != nullptr;
  if (f32) {
    if (pairs) return gate ? Op<float, 2, true>::run(ctx, a, s) : Op<float, 2, false>::run(ctx, a, s);
    return gate ? Op<float, 1, true>::run(ctx, a, s) : Op<float, 1, false>::run(ctx, a, s);
  }
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
  const size_t es = dtype == ARD_F32 ? 4 : 2;
  return glr_dispatch<GlrFwd>(ctx, dtype == ARD_F32, glr_pairs(es, {Zf, Zg, Zo, Y}, {ldz, ldy}), a, s);
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
  const size_t es = dtype == ARD_F32 ? 4 : 2;
  return glr_dispatch<GlrBwd>(ctx, dtype == ARD_F32, glr_pairs(es, {Zf, Zg, Zo, dY, dZf, dZg, dZo}, {ldz, lddy, lddz}), a, s);
}
