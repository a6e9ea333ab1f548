// Loss of a row of logits z against its label and a teacher's top logits t over the tokens id, with its gradient:
//   p = softmax(t / tau),  L = hard (lse(z) - z[label]) + soft tau^2 sum_i p_i (log p_i - log softmax(z / tau)[id_i])
//   dL/dz = hard (softmax(z) - [label]) + soft tau (softmax(z / tau) - sum_i p_i [id_i])
//
// Memory bounds it: a row is read once and its gradient written once, 4 bytes an element in bf16.  So a row stays where
// it was read: in the registers of a CTA's threads (up to 32768 logits in bf16), or, longer than that, in the L2, which
// holds the rows of all SMs twice over; the second look does not reach memory.  Each thread keeps the maximum of what
// it holds and sums of exponentials relative to it, and these pairs meet once a row.  The gradient's few entries at the label and the
// teacher's tokens are written again behind the others, by the threads that know all that falls on the same token.
// A row of up to 128 logits is held by 8 or 32 lanes.
#include "ard_internal.h"
#include "sm100_ptx.h"

namespace {

constexpr int DS_MOST_TEACHER = 1024;
constexpr float DS_LOG2E = 1.4426950408889634f;

struct DsArgs {
  int rows, V, k, ldk;
  long long ldz, lddz;
  const void* Z;
  const int32_t* labels;
  const int32_t* t_ids;
  const float* t;
  float c, c_tau;  // log2(e), log2(e) / tau
  float inv_tau, tau, hard, soft;
  const float* weight;
  float* loss;
  float* total;
  double* partial;      // one a CTA
  unsigned int* count;  // zero between launches
  void* dZ;
  int* status;
};

__device__ __forceinline__ float ds_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
template <typename T>
__device__ __forceinline__ float ds_f32(T x) {
  if constexpr (sizeof(T) == 2) return __bfloat162float(x);
  else return x;
}
template <typename T>
__device__ __forceinline__ T ds_from(float x) {
  if constexpr (sizeof(T) == 2) return __float2bfloat16_rn(x);
  else return x;
}
// A thread's maximum where it has seen nothing but -infinity (or nothing): differences from it stay numbers.
__device__ __forceinline__ float ds_floor(float m) { return fmaxf(m, -3.402823466e38f); }

// exp of all but a maximum's share: the sums of another maximum in this one's terms.
__device__ __forceinline__ float ds_shift(float from, float to, float c) { return ds_exp2((from - to) * c); }

// The teacher's entries of a row as smem holds them, and the label as one more.
struct DsEntries {
  int id[DS_MOST_TEACHER + 1];
  float p[DS_MOST_TEACHER + 1];     // share of the teacher's distribution (the label's: not used)
  float lp[DS_MOST_TEACHER];        // its logarithm
  float z[DS_MOST_TEACHER + 1];     // the student's logit
};

__device__ __forceinline__ int ds_teacher_id(const DsArgs& a, long long r, int i) {
  const int id = a.t_ids[r * a.ldk + i];
  if (id >= a.V) atomicMax(a.status, (int)ARD_ERR_INVALID_ARG);
  return id < a.V ? id : -1;
}

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  return x;
}

// One warp: a row's entries to shared memory.  Returns how many of the teacher's count (the softmax over them is complete).
template <typename T>
__device__ int ds_entries(const DsArgs& a, long long r, const T* z, int label, DsEntries& e) {
  const int lane = threadIdx.x & 31;
  float m = -INFINITY;
  int live = 0;
  for (int i = lane; i < a.k; i += 32) {
    const int id = ds_teacher_id(a, r, i);
    const float t = a.t[r * a.ldk + i];
    const bool on = id >= 0 && t != -INFINITY;
    e.id[i] = on ? id : -1;
    e.lp[i] = t;
    e.z[i] = on ? ds_f32(z[id]) : 0.f;
    if (on) m = fmaxf(m, t), ++live;
    if (on && t != t) m = t;
  }
  if (lane == 0) {
    e.id[a.k] = label;
    e.z[a.k] = label >= 0 ? ds_f32(z[label]) : 0.f;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) live += __shfl_xor_sync(0xFFFFFFFFu, live, o);
  if (live == 0) return 0;
  m = warp_max(m);
  float s = 0.f;
  for (int i = lane; i < a.k; i += 32)
    if (e.id[i] >= 0) s += expf((e.lp[i] - m) * a.inv_tau);
  s = warp_sum(s);
  const float log_s = logf(s);
  for (int i = lane; i < a.k; i += 32)
    if (e.id[i] >= 0) {
      const float d = (e.lp[i] - m) * a.inv_tau;
      e.p[i] = expf(d) / s;
      e.lp[i] = d - log_s;
    }
  return live;
}

// Sum of a CTA's rows' losses, weighted, to its place; the last CTA adds all of them in a fixed order.  All threads call it.
template <int THREADS>
__device__ void ds_total(const DsArgs& a, double mine, double* red, int* s_last) {
  const int t = threadIdx.x;
  auto block_sum = [&](double x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    __syncthreads();
    if ((t & 31) == 0) red[t >> 5] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int k = 0; k < THREADS / 32; ++k) x += red[k];
    return x;
  };
  mine = block_sum(mine);
  if (t == 0) {
    __stcg(a.partial + blockIdx.x, mine);
    __threadfence();
    *s_last = atomicAdd(a.count, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!*s_last) return;
  __threadfence();
  double x = 0.0;
  for (int k = t; k < (int)gridDim.x; k += THREADS) x += __ldcg(a.partial + k);
  x = block_sum(x);
  if (t == 0) {
    *a.count = 0u;
    *a.total = (float)x;
  }
}

// ---- a CTA a row ------------------------------------------------------------------------------------
// Elements of a row as its threads take them: `head` ones in front of the first 16-byte boundary, vectors, and the rest; head and rest are less than a
// vector each and go to the first threads, one element each.
template <typename T>
struct DsRow {
  static constexpr int VEC = 16 / (int)sizeof(T);
  int head, vecs, loose;  // loose: head and rest
  __device__ __forceinline__ DsRow(const T* z, int V) {
    const int off = (int)((reinterpret_cast<uintptr_t>(z) & 15u) / sizeof(T));
    head = min(V, (VEC - off) & (VEC - 1));
    vecs = (V - head) / VEC;
    loose = V - vecs * VEC;
  }
  __device__ __forceinline__ int loose_at(int i) const { return i < head ? i : i + vecs * VEC; }
};

// NV vectors a thread in registers; NV = 0: looked at twice in memory.  TWO: the softmax at temperature 1 and the one at tau.
template <typename T, int THREADS, int NV, bool TWO>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) distill_row_kernel(const DsArgs a) {
  constexpr int VEC = 16 / (int)sizeof(T), WARPS = THREADS / 32;
  __shared__ DsEntries ent;
  __shared__ float red_m[WARPS], red_s[WARPS], red_u[WARPS];
  __shared__ double red_d[WARPS];
  __shared__ int s_live, s_last;
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const float c1 = TWO || a.soft == 0.f ? a.c : a.c_tau;  // of the only softmax, or of temperature 1's
  double sum_loss = 0.0;
  for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* z = (const T*)a.Z + r * a.ldz;
    T* dz = a.dZ ? (T*)a.dZ + r * a.lddz : nullptr;
    const DsRow<T> row(z, a.V);
    const float w = a.weight ? a.weight[r] : 1.f;
    int label = a.labels ? a.labels[r] : -1;
    if (label >= a.V && t == 0) atomicMax(a.status, (int)ARD_ERR_INVALID_ARG);
    if (label >= a.V || a.hard == 0.f) label = -1;
    auto nothing = [&]() {  // there is nothing to learn from
      if (dz) {
        const DsRow<T> out(dz, a.V);
        for (int i = t; i < out.vecs; i += THREADS) reinterpret_cast<uint4*>(dz + out.head)[i] = make_uint4(0, 0, 0, 0);
        if (t < out.loose) dz[out.loose_at(t)] = ds_from<T>(0.f);
      }
      if (t == 0) a.loss[r] = 0.f;
    };
    if (w == 0.f || (label < 0 && a.k == 0)) {
      nothing();
      continue;
    }
    // what this thread holds: its maximum, then the exponentials' sums relative to it
    uint4 q[NV > 0 ? NV : 1];
    const uint4* zv = reinterpret_cast<const uint4*>(z + row.head);
    const float edge = t < row.loose ? ds_f32(z[row.loose_at(t)]) : -INFINITY;
    float m = edge, s = 0.f, u = 0.f;
    auto unpack = [&](const uint4& v, float (&x)[VEC]) {
      T e[VEC];
      memcpy(e, &v, 16);
#pragma unroll
      for (int k = 0; k < VEC; ++k) x[k] = ds_f32(e[k]);
    };
    auto vector_max = [&](const float (&x)[VEC]) {
      float y = x[0];
#pragma unroll
      for (int k = 1; k < VEC; ++k) y = fmaxf(y, x[k]);
      return y;
    };
    auto add = [&](const float (&x)[VEC], float top) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float d = x[k] - top;
        s += ds_exp2(d * c1);
        if (TWO) u += ds_exp2(d * a.c_tau);
      }
    };
    if constexpr (NV > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (t + i * THREADS < row.vecs) q[i] = zv[t + i * THREADS];
    }
    if (warp == 0) {
      const int live = ds_entries<T>(a, r, z, label, ent);
      if (lane == 0) s_live = live;
    }
    if constexpr (NV > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (t + i * THREADS < row.vecs) {
          float x[VEC];
          unpack(q[i], x);
          m = fmaxf(m, vector_max(x));
        }
      m = ds_floor(m);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (t + i * THREADS < row.vecs) {
          float x[VEC];
          unpack(q[i], x);
          add(x, m);
        }
    } else {
      m = ds_floor(m);
      constexpr int AHEAD = 4;
      for (int i0 = t; i0 < row.vecs; i0 += AHEAD * THREADS) {
        uint4 v[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
          if (i0 + j * THREADS < row.vecs) v[j] = zv[i0 + j * THREADS];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
          if (i0 + j * THREADS >= row.vecs) break;
          float x[VEC];
          unpack(v[j], x);
          const float top = vector_max(x);
          if (top > m) {
            s *= ds_shift(m, top, c1);
            if (TWO) u *= ds_shift(m, top, a.c_tau);
            m = top;
          }
          add(x, m);
        }
      }
    }
    if (t < row.loose) {
      s += ds_exp2((edge - m) * c1);  // fmaxf passes NaN over; the sums do not
      if (TWO) u += ds_exp2((edge - m) * a.c_tau);
    }
    // the pairs of all threads
    {
      const float top = warp_max(m), by = ds_shift(m, top, c1);
      s = warp_sum(s * by);
      if (TWO) u = warp_sum(u * ds_shift(m, top, a.c_tau));
      if (lane == 0) {
        red_m[warp] = top;
        red_s[warp] = s;
        if (TWO) red_u[warp] = u;
      }
      __syncthreads();
      m = red_m[0];
#pragma unroll
      for (int i = 1; i < WARPS; ++i) m = fmaxf(m, red_m[i]);
      s = 0.f, u = 0.f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) {
        s += red_s[i] * ds_shift(red_m[i], m, c1);
        if (TWO) u += red_u[i] * ds_shift(red_m[i], m, a.c_tau);
      }
    }
    const float hard = label >= 0 ? a.hard : 0.f, soft = s_live > 0 ? a.soft : 0.f;
    if (hard == 0.f && soft == 0.f) {  // none of the teacher's entries counts
      nothing();
      __syncthreads();
      continue;
    }
    const float by1 = w * (TWO ? hard : hard + soft * a.tau) / s, by_tau = TWO ? w * soft * a.tau / u : 0.f;
    auto slope = [&](float x) {
      const float d = x - m;
      float g = by1 * ds_exp2(d * c1);
      if (TWO) g = fmaf(by_tau, ds_exp2(d * a.c_tau), g);
      return g;
    };
    if (dz) {
      const bool same = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15u) == 0;
      auto put = [&](int i, const uint4& v) {
        float x[VEC];
        unpack(v, x);
        T e[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) e[k] = ds_from<T>(slope(x[k]));
        if (same) {
          uint4 o;
          memcpy(&o, e, 16);
          reinterpret_cast<uint4*>(dz + row.head)[i] = o;
        } else {
#pragma unroll
          for (int k = 0; k < VEC; ++k) dz[row.head + i * VEC + k] = e[k];
        }
      };
      if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (t + i * THREADS < row.vecs) put(t + i * THREADS, q[i]);
      } else {
        constexpr int AHEAD = 4;
        for (int i0 = t; i0 < row.vecs; i0 += AHEAD * THREADS) {
          uint4 v[AHEAD];
#pragma unroll
          for (int j = 0; j < AHEAD; ++j)
            if (i0 + j * THREADS < row.vecs) v[j] = zv[i0 + j * THREADS];
#pragma unroll
          for (int j = 0; j < AHEAD; ++j)
            if (i0 + j * THREADS < row.vecs) put(i0 + j * THREADS, v[j]);
        }
      }
      if (t < row.loose) dz[row.loose_at(t)] = ds_from<T>(slope(edge));
      __syncthreads();
      for (int i = t; i <= a.k; i += THREADS) {
        const int id = ent.id[i];
        if (id < 0) continue;
        float p = 0.f;  // all that falls on this token, in the entries' order
        if (soft != 0.f)
          for (int j = 0; j < a.k; ++j)
            if (ent.id[j] == id) p += ent.p[j];
        const float less = (id == label ? hard : 0.f) + soft * a.tau * p;
        dz[id] = ds_from<T>(fmaf(-w, less, slope(ent.z[i])));
      }
    }
    if (warp == 0) {
      float kl = 0.f;
      const float log_u = logf(TWO ? u : s);
      if (soft != 0.f)
        for (int i = lane; i < a.k; i += 32)
          if (ent.id[i] >= 0 && ent.p[i] > 0.f) kl += ent.p[i] * (ent.lp[i] - ((ent.z[i] - m) * a.inv_tau - log_u));
      kl = warp_sum(kl);
      if (lane == 0) {
        float L = soft * a.tau * a.tau * kl;
        if (label >= 0) L = fmaf(hard, logf(s) - (ent.z[a.k] - m), L);
        a.loss[r] = L;
        sum_loss += (double)w * L;
      }
    }
    __syncthreads();
  }
  if (a.total) ds_total<THREADS>(a, sum_loss, red_d, &s_last);
}

// ---- short rows -------------------------------------------------------------------------------------
constexpr int DS_SHORT_THREADS = 256;

template <int LANES>
__device__ __forceinline__ float lanes_max(float x) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  return x;
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  return x;
}

// LANES lanes a row of up to 4 * LANES logits.  The teacher's entries are looked at one after the other, and the lane that holds an entry's logit
// takes it.
template <typename T, int LANES>
__global__ void __launch_bounds__(DS_SHORT_THREADS) distill_short_kernel(const DsArgs a) {
  constexpr int EPT = 4, PER = DS_SHORT_THREADS / LANES;
  __shared__ double red_d[DS_SHORT_THREADS / 32];
  __shared__ int s_last;
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int t = threadIdx.x, lane = t & (LANES - 1);
  double sum_loss = 0.0;
  for (long long r0 = (long long)blockIdx.x * PER; r0 < a.rows; r0 += (long long)gridDim.x * PER) {
    const long long r = r0 + t / LANES;
    const bool in = r < a.rows;
    const T* z = (const T*)a.Z + (in ? r : 0) * a.ldz;
    const float w = !in ? 0.f : a.weight ? a.weight[r] : 1.f;
    int label = in && a.labels ? a.labels[r] : -1;
    if (label >= a.V) atomicMax(a.status, (int)ARD_ERR_INVALID_ARG);
    if (label >= a.V || a.hard == 0.f) label = -1;
    const int k = in ? a.k : 0;
    const bool look = w != 0.f && (label >= 0 || k > 0);
    float x[EPT], less[EPT];
    float m = -INFINITY;
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      x[e] = look && lane + e * LANES < a.V ? ds_f32(z[lane + e * LANES]) : -INFINITY;
      m = fmaxf(m, x[e]);
      less[e] = 0.f;
    }
    m = ds_floor(lanes_max<LANES>(m));
    float s = 0.f, u = 0.f;
#pragma unroll
    for (int e = 0; e < EPT; ++e)
      if (lane + e * LANES < a.V) {
        s += ds_exp2((x[e] - m) * a.c);
        u += ds_exp2((x[e] - m) * a.c_tau);
      }
    s = lanes_sum<LANES>(s);
    u = lanes_sum<LANES>(u);
    // the teacher's softmax
    float tm = -INFINITY, ts = 0.f;
    int live = 0;
    if (look)
      for (int i = lane; i < k; i += LANES) {
        const int id = ds_teacher_id(a, r, i);
        const float tv = a.t[r * a.ldk + i];
        if (id >= 0 && tv != -INFINITY) tm = tv != tv ? tv : fmaxf(tm, tv), live = 1;
      }
    tm = lanes_max<LANES>(tm);
    if (look && tm != -INFINITY)
      for (int i = lane; i < k; i += LANES) {
        const int id = a.t_ids[r * a.ldk + i];
        const float tv = a.t[r * a.ldk + i];
        if (id >= 0 && id < a.V && tv != -INFINITY) ts += expf((tv - tm) * a.inv_tau);
      }
    ts = lanes_sum<LANES>(ts);
    live = lanes_sum<LANES>((float)live) > 0.f;
    const float hard = label >= 0 ? a.hard : 0.f, soft = live ? a.soft : 0.f;
    float L = 0.f;
    if (look && live) {
      const float log_ts = logf(ts), log_u = logf(u);
      for (int i = 0; i < k; ++i) {
        const int id = a.t_ids[r * a.ldk + i];
        const float tv = a.t[r * a.ldk + i];
        if (id < 0 || id >= a.V || tv == -INFINITY || (id & (LANES - 1)) != lane) continue;
        const float d = (tv - tm) * a.inv_tau, p = expf(d) / ts;
#pragma unroll
        for (int e = 0; e < EPT; ++e)
          if (id == lane + e * LANES) {
            less[e] += soft * a.tau * p;
            if (p > 0.f) L += p * (d - log_ts - ((x[e] - m) * a.inv_tau - log_u));
          }
      }
      L *= soft * a.tau * a.tau;
    }
    const float by1 = hard / s, by_tau = soft * a.tau / u;
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      const int j = lane + e * LANES;
      if (j >= a.V) continue;
      if (j == label) {
        less[e] += hard;
        L = fmaf(hard, logf(s) - (x[e] - m), L);
      }
      if (in && a.dZ) {
        const float d = x[e] - m;
        float g = 0.f;
        if (hard != 0.f) g = by1 * ds_exp2(d * a.c);
        if (soft != 0.f) g = fmaf(by_tau, ds_exp2(d * a.c_tau), g);
        ((T*)a.dZ)[r * a.lddz + j] = ds_from<T>(look ? w * (g - less[e]) : 0.f);
      }
    }
    L = lanes_sum<LANES>(L);
    if (in && lane == 0) {
      a.loss[r] = look ? L : 0.f;
      if (look) sum_loss += (double)w * L;
    }
  }
  if (a.total) ds_total<DS_SHORT_THREADS>(a, sum_loss, red_d, &s_last);
}

template <typename T, int THREADS, int NV>
ard_status ds_rows(ard_ctx* ctx, const DsArgs& a, bool two, cudaStream_t s) {
  const long long room = (long long)(1024 / THREADS) * ctx->sm_count;
  const dim3 grid((unsigned)(a.rows < room ? a.rows : room));
  ARD_CUDA_OK(ard_launch(ctx, two ? distill_row_kernel<T, THREADS, NV, true> : distill_row_kernel<T, THREADS, NV, false>, grid, dim3(THREADS), 0, s, a));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}

template <typename T>
ard_status ds_launch(ard_ctx* ctx, const DsArgs& a, bool two, cudaStream_t s) {
  constexpr int VEC = 16 / (int)sizeof(T);
  if (a.V <= 128) {
    const int lanes = a.V <= 32 ? 8 : 32, per = DS_SHORT_THREADS / lanes;
    const long long want = ((long long)a.rows + per - 1) / per, room = 8ll * ctx->sm_count;
    const dim3 grid((unsigned)(want < room ? want : room));
    ARD_CUDA_OK(ard_launch(ctx, lanes == 8 ? distill_short_kernel<T, 8> : distill_short_kernel<T, 32>, grid, dim3(DS_SHORT_THREADS), 0, s, a));
    ctx->launches++;
    ARD_CUDA_OK(cudaGetLastError());
    return ARD_OK;
  }
  if (a.V <= 128 * 4 * VEC) return ds_rows<T, 128, 4>(ctx, a, two, s);
  if (a.V <= 256 * 8 * VEC) return ds_rows<T, 256, 8>(ctx, a, two, s);
  if (a.V <= 512 * 8 * VEC) return ds_rows<T, 512, 8>(ctx, a, two, s);
  return ds_rows<T, 512, 0>(ctx, a, two, s);
}

}  // namespace

ard_status launch_distill_loss(ard_ctx* ctx, ard_dtype dtype, int rows, int V, const void* Z, long long ldz, const int32_t* labels, int k,
                               const int32_t* t_ids, const float* t, int ldk, float tau, float hard, float soft, const float* weight, float* loss,
                               float* total, void* dZ, long long lddz, cudaStream_t s) {
  if (rows == 0) {
    if (total) ARD_CUDA_OK(cudaMemsetAsync(total, 0, sizeof(float), s));
    return ARD_OK;
  }
  if (!ctx->d_sk_ws) return ARD_ERR_UNSUPPORTED;
  DsArgs a;
  a.rows = rows, a.V = V, a.k = soft != 0.f ? k : 0, a.ldk = ldk, a.ldz = ldz, a.lddz = lddz;
  a.Z = Z, a.labels = labels, a.t_ids = t_ids, a.t = t;
  a.c = DS_LOG2E;
  a.c_tau = (float)(1.4426950408889634 / (double)tau);
  a.inv_tau = (float)(1.0 / (double)tau);
  a.tau = tau;
  a.hard = labels ? hard : 0.f;
  a.soft = k > 0 ? soft : 0.f;
  a.weight = weight, a.loss = loss, a.total = total, a.dZ = dZ, a.status = ctx->d_status;
  a.partial = (double*)ctx->d_sk_ws;
  a.count = (unsigned int*)ctx->d_sk_cnt;
  const bool two = a.hard != 0.f && a.soft != 0.f && tau != 1.f;
  return dtype == ARD_F32 ? ds_launch<float>(ctx, a, two, s) : ds_launch<__nv_bfloat16>(ctx, a, two, s);
}
