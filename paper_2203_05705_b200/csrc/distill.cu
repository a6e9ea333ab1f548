// Loss of a row of logits z against its label and a teacher's top logits t over the tokens id, with its gradient:
//   p = softmax(t / tau),  L = hard (lse(z) - z[label]) + soft tau^2 sum_i p_i (log p_i - log softmax(z / tau)[id_i])
//   dL/dz = hard (softmax(z) - [label]) + soft tau (softmax(z / tau) - sum_i p_i [id_i])
//
// Memory bounds it: a row is read once and its gradient written once, 4 bytes an element in bf16; its exponentials, two an element (four where both temperatures
// are wanted), take seven tenths of that time on the special function units.  So rows stream through a ring in shared memory, filled by bulk copies that one warp
// asks for, while the others work on what is there, and a row too long for a ring of three is cut over a cluster of CTAs, which exchange a maximum and
// sums once a row.  A third kind of warp does what depends on a few scattered logits: the teacher's softmax for the next row, and for this one the loss and the
// gradient's entries at the label and the teacher's tokens, which are written once more behind the others.  Each thread keeps the maximum of what it looks at and
// sums of exponentials relative to it; these pairs meet once a row.  Rows of up to 4096 logits (fp32: 2048) are held by a warp or 8 lanes, in registers.
//
// bf16, 64 entries of a teacher, one temperature: 8192 x 32000 190 us (5.5 TB/s, 85 % of a copy; without a teacher 182); 1023 x 100003, labels alone, rows over
// clusters of two or more 100 us (4.1 TB/s: 132 SMs' worth of clusters, each of which waits for its sums once a row); 65536 x 1000 by warps 82 us cold (issue slots 73 %).
#include <cooperative_groups.h>

#include "ard_internal.h"
#include "sm100_ptx.h"

namespace {

namespace cg = cooperative_groups;

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
  double* partial;      // one a CTA or cluster
  unsigned int* count;  // zero between launches
  void* dZ;
  int* status;
  int slots, slot_bytes, slice;  // the ring; a CTA's vectors of a row
};

__device__ __forceinline__ float ds_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float2 ds_exps(float2 d, float c) {
  const float2 y = __fmul2_rn(d, make_float2(c, c));
  return make_float2(ds_exp2(y.x), ds_exp2(y.y));
}
// MODE: 0 one softmax; 1 that at temperature 1 and that at tau; 2, 3 both with tau = 2, 4, where exp(d) is exp(d / tau) squared once or twice: half of the
// exponentials, which bound the two (8192 x 32000 bf16 283 us with them all, 206 so), for an error of one or two more units in the last place.
template <int MODE>
__device__ __forceinline__ float ds_power(float e) {
  e *= e;
  return MODE == 3 ? e * e : e;
}
template <int MODE>
__device__ __forceinline__ float2 ds_power(float2 e) {
  e = __fmul2_rn(e, e);
  return MODE == 3 ? __fmul2_rn(e, e) : e;
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

// Sums relative to the maximum `from` in terms of a larger one.
__device__ __forceinline__ float ds_shift(float from, float to, float c) { return ds_exp2((from - to) * c); }

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

// Sixteen bytes of logits as pairs.
template <typename T>
struct DsVec {
  static constexpr int N = 16 / (int)sizeof(T);
  float2 v[N / 2];
  __device__ __forceinline__ explicit DsVec(const uint4& q) {
    if constexpr (sizeof(T) == 2) {
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
    } else {
      v[0] = make_float2(__uint_as_float(q.x), __uint_as_float(q.y));
      v[1] = make_float2(__uint_as_float(q.z), __uint_as_float(q.w));
    }
  }
  __device__ __forceinline__ float max() const {
    float m = fmaxf(v[0].x, v[0].y);
#pragma unroll
    for (int i = 1; i < N / 2; ++i) m = fmaxf(m, fmaxf(v[i].x, v[i].y));
    return m;
  }
  // Exponentials of (x - m) c1, and of (x - m) c_tau, added up in pairs.
  template <int MODE>
  __device__ __forceinline__ void add(float2& s, float2& u, float m, float c1, float c_tau) const {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float2 d = __fadd2_rn(v[i], make_float2(-m, -m));
      if (MODE == 0) {
        s = __fadd2_rn(s, ds_exps(d, c1));
      } else {
        const float2 e = ds_exps(d, c_tau);
        u = __fadd2_rn(u, e);
        s = __fadd2_rn(s, MODE == 1 ? ds_exps(d, c1) : ds_power<MODE>(e));
      }
    }
  }
};

// Elements of a row as vectors of 16 bytes: `head` ones in front of the first boundary, vectors, and the rest; head and rest are less than a vector each.
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
  // which vector an element is in, -1: loose
  __device__ __forceinline__ int vec_of(int j) const { return j < head || j >= head + vecs * VEC ? -1 : (j - head) / VEC; }
};

// The gradient's factors of a row: g = by1 exp((x - m) c1) + by_tau exp((x - m) c_tau).
struct DsSlope {
  float m, by1, by_tau, c1, c_tau;
  template <int MODE>
  __device__ __forceinline__ float at(float x) const {
    const float d = x - m;
    if (MODE == 0) return by1 * ds_exp2(d * c1);
    const float e = ds_exp2(d * c_tau);
    return fmaf(by1, MODE == 1 ? ds_exp2(d * c1) : ds_power<MODE>(e), by_tau * e);
  }
  template <int MODE>
  __device__ __forceinline__ float2 at(float2 x) const {
    const float2 d = __fadd2_rn(x, make_float2(-m, -m)), f1 = make_float2(by1, by1);
    if (MODE == 0) return __fmul2_rn(f1, ds_exps(d, c1));
    const float2 e = ds_exps(d, c_tau);
    return __ffma2_rn(f1, MODE == 1 ? ds_exps(d, c1) : ds_power<MODE>(e), __fmul2_rn(make_float2(by_tau, by_tau), e));
  }
};
// A vector's gradient to memory; same: dz lies on the 16-byte grid where z does.
template <typename T, int MODE>
__device__ __forceinline__ void ds_put(const DsSlope& f, const uint4& q, T* dz, bool same) {
  constexpr int VEC = 16 / (int)sizeof(T);
  const DsVec<T> x(q);
  T e[VEC];
#pragma unroll
  for (int k = 0; k < VEC; k += 2) {
    const float2 g = f.at<MODE>(x.v[k / 2]);
    if constexpr (sizeof(T) == 2) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(g.x, g.y);
      memcpy(e + k, &h, 4);
    } else {
      e[k] = g.x, e[k + 1] = g.y;
    }
  }
  if (same) {
    uint4 o;
    memcpy(&o, e, 16);
    *reinterpret_cast<uint4*>(dz) = o;
  } else {
#pragma unroll
    for (int k = 0; k < VEC; ++k) dz[k] = e[k];
  }
}
// A row's zeros, by `shares` groups of `of` threads each.
template <typename T>
__device__ __forceinline__ void ds_zero(T* dz, int V, int share, int shares, int t, int of) {
  if (!dz) return;
  const DsRow<T> out(dz, V);
  for (int i = share * of + t; i < out.vecs; i += shares * of) reinterpret_cast<uint4*>(dz + out.head)[i] = make_uint4(0, 0, 0, 0);
  if (share == 0)
    for (int i = t; i < out.loose; i += of) dz[out.loose_at(i)] = ds_from<T>(0.f);
}

// The sum of a warp's rows' losses to its place; the last warp of the grid to come adds all of them in a fixed order.
__device__ void ds_total(const DsArgs& a, double mine, int place, int places, int lane) {
  unsigned last = 0;
  if (lane == 0) {
    __stcg(a.partial + place, mine);
    __threadfence();
    last = atomicAdd(a.count, 1u) == (unsigned)places - 1u;
  }
  if (!__shfl_sync(0xFFFFFFFFu, last, 0)) return;
  __threadfence();
  double x = 0.0;
  for (int k = lane; k < places; k += 32) x += __ldcg(a.partial + k);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  if (lane == 0) {
    *a.count = 0u;
    *a.total = (float)x;
  }
}

__device__ __forceinline__ int ds_label(const DsArgs& a, long long r) {
  const int label = a.labels ? a.labels[r] : -1;
  if (label >= a.V) atomicMax(a.status, (int)ARD_ERR_INVALID_ARG);
  return label >= a.V || a.hard == 0.f ? -1 : label;
}
// An entry of the teacher's that counts, or -1.
__device__ __forceinline__ int ds_entry(const DsArgs& a, long long r, int i, float& t) {
  const int id = a.t_ids[r * a.ldk + i];
  t = a.t[r * a.ldk + i];
  if (id >= a.V) atomicMax(a.status, (int)ARD_ERR_INVALID_ARG);
  return id >= 0 && id < a.V && t != -INFINITY ? id : -1;
}

// ---- short rows -------------------------------------------------------------------------------------
constexpr int DS_SHORT_THREADS = 256;

// LANES lanes a row, NV vectors of 16 bytes a lane (WIDE) or NV single logits, E of the teacher's entries a lane.
template <typename T, int LANES, bool WIDE, int NV, int E, int MODE>
__global__ void __launch_bounds__(DS_SHORT_THREADS) distill_lanes_kernel(const DsArgs a) {
  constexpr int VEC = WIDE ? 16 / (int)sizeof(T) : 1, PER = DS_SHORT_THREADS / LANES;
  constexpr int EDGES = WIDE ? (2 * VEC - 2 + LANES - 1) / LANES : 1;  // a lane's loose logits
  __shared__ double s_sum[DS_SHORT_THREADS / 32];
  pdl_launch_dependents();
  pdl_wait_prior_grids();
  const int t = threadIdx.x, lane = t & (LANES - 1);
  constexpr bool TWO = MODE != 0;
  const float c1 = TWO || a.soft == 0.f ? a.c : a.c_tau;  // of the only softmax, or of temperature 1's
  double sum_loss = 0.0;
  for (long long r0 = (long long)blockIdx.x * PER; r0 < a.rows; r0 += (long long)gridDim.x * PER) {
    const bool in = r0 + t / LANES < a.rows;
    const long long r = in ? r0 + t / LANES : 0;
    const T* z = (const T*)a.Z + r * a.ldz;
    T* dz = a.dZ && in ? (T*)a.dZ + r * a.lddz : nullptr;
    const DsRow<T> row(z, a.V);
    // everything that has to come from memory is asked for at once; what a row without use holds is not looked at
    const float w = !in ? 0.f : a.weight ? a.weight[r] : 1.f;
    const int label = in ? ds_label(a, r) : -1;
    int id[E];
    float p[E], lp[E], ze[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      lp[e] = 0.f;
      id[e] = in && lane + e * LANES < a.k ? ds_entry(a, r, lane + e * LANES, lp[e]) : -1;
    }
    const bool look = w != 0.f && (label >= 0 || a.k > 0);
    uint4 q[WIDE ? NV : 1];
    float x[WIDE ? 1 : NV];
    float edge[EDGES], m = -INFINITY;
    if constexpr (WIDE) {
      const uint4* zv = reinterpret_cast<const uint4*>(z + row.head);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (look && lane + i * LANES < row.vecs) q[i] = zv[lane + i * LANES];
#pragma unroll
      for (int i = 0; i < EDGES; ++i) {
        edge[i] = look && lane + i * LANES < row.loose ? ds_f32(z[row.loose_at(lane + i * LANES)]) : -INFINITY;
        m = fmaxf(m, edge[i]);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (look && lane + i * LANES < row.vecs) m = fmaxf(m, DsVec<T>(q[i]).max());
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        x[i] = look && lane + i * LANES < a.V ? ds_f32(z[lane + i * LANES]) : -INFINITY;
        m = fmaxf(m, x[i]);
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) ze[e] = look && id[e] >= 0 ? ds_f32(z[id[e]]) : 0.f;
    const float zl = look && label >= 0 ? ds_f32(z[label]) : 0.f;
    m = ds_floor(lanes_max<LANES>(m));
    float2 s2 = make_float2(0.f, 0.f), u2 = make_float2(0.f, 0.f);
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (look && lane + i * LANES < row.vecs) {
          DsVec<T>(q[i]).template add<MODE>(s2, u2, m, c1, a.c_tau);
        }
#pragma unroll
      for (int i = 0; i < EDGES; ++i) {
        s2.x += ds_exp2((edge[i] - m) * c1);
        if (TWO) u2.x += ds_exp2((edge[i] - m) * a.c_tau);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        s2.x += ds_exp2((x[i] - m) * c1);
        if (TWO) u2.x += ds_exp2((x[i] - m) * a.c_tau);
      }
    }
    const float s = lanes_sum<LANES>(s2.x + s2.y), u = TWO ? lanes_sum<LANES>(u2.x + u2.y) : s;
    // the teacher's softmax
    float tm = -INFINITY, ts = 0.f, live = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (id[e] >= 0) {
        live = 1.f;
        tm = lp[e] != lp[e] ? lp[e] : fmaxf(tm, lp[e]);
      }
    live = lanes_sum<LANES>(live);
    tm = lanes_max<LANES>(tm);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      lp[e] = (lp[e] - tm) * a.inv_tau;
      p[e] = id[e] >= 0 ? expf(lp[e]) : 0.f;
      ts += p[e];
    }
    ts = lanes_sum<LANES>(ts);
    const float hard = label >= 0 ? a.hard : 0.f, soft = live > 0.f ? a.soft : 0.f;
    const bool some = look && (hard != 0.f || soft != 0.f);
    const float log_s = logf(s), log_u = TWO ? logf(u) : log_s, log_ts = logf(ts);
    float kl = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      p[e] = id[e] >= 0 ? p[e] / ts : 0.f;
      if (id[e] >= 0 && p[e] != 0.f) kl += p[e] * (lp[e] - log_ts - ((ze[e] - m) * a.inv_tau - log_u));
    }
    kl = lanes_sum<LANES>(kl);
    if (in && lane == 0) {
      float L = 0.f;
      if (some && soft != 0.f) L = soft * a.tau * a.tau * kl;
      if (some && hard != 0.f) L = fmaf(hard, log_s - (zl - m), L);
      a.loss[r] = L;
      if (some) sum_loss += (double)w * L;
    }
    if (a.dZ) {
      const DsSlope f = {m, w * (TWO ? hard : hard + soft * a.tau) / s, TWO ? w * soft * a.tau / u : 0.f, c1, a.c_tau};
      if (dz && !some) ds_zero(dz, a.V, 0, 1, lane, LANES);
      if (dz && some) {
        if constexpr (WIDE) {
          const bool same = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15u) == 0;
#pragma unroll
          for (int i = 0; i < NV; ++i)
            if (lane + i * LANES < row.vecs) ds_put<T, MODE>(f, q[i], dz + row.head + (lane + i * LANES) * VEC, same);
#pragma unroll
          for (int i = 0; i < EDGES; ++i)
            if (lane + i * LANES < row.loose) dz[row.loose_at(lane + i * LANES)] = ds_from<T>(f.at<MODE>(edge[i]));
        } else {
#pragma unroll
          for (int i = 0; i < NV; ++i)
            if (lane + i * LANES < a.V) dz[lane + i * LANES] = ds_from<T>(f.at<MODE>(x[i]));
        }
      }
      __syncwarp();
      // the label's entry and the teacher's once more, with all that falls on the same token, in the entries' order
      float on[E], on_label = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) on[e] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e)
        for (int j = 0; j < LANES && j + e * LANES < a.k; ++j) {
          const int other = __shfl_sync(0xFFFFFFFFu, id[e], j, LANES);
          const float share = __shfl_sync(0xFFFFFFFFu, p[e], j, LANES);
          if (other == label && label >= 0) on_label += share;
#pragma unroll
          for (int d = 0; d < E; ++d)
            if (id[d] == other) on[d] += share;
        }
      if (dz && some) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (id[e] >= 0) dz[id[e]] = ds_from<T>(fmaf(-w, (id[e] == label ? hard : 0.f) + soft * a.tau * on[e], f.at<MODE>(ze[e])));
        if (lane == 0 && label >= 0) dz[label] = ds_from<T>(fmaf(-w, hard + soft * a.tau * on_label, f.at<MODE>(zl)));
      }
      __syncwarp();
    }
  }
  if (!a.total) return;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum_loss += __shfl_xor_sync(0xFFFFFFFFu, sum_loss, o);
  if ((t & 31) == 0) s_sum[t >> 5] = sum_loss;
  __syncthreads();
  if (t >= 32) return;
  double x = 0.0;
  for (int k = 0; k < DS_SHORT_THREADS / 32; ++k) x += s_sum[k];
  ds_total(a, x, blockIdx.x, gridDim.x, t);
}

// ---- rows through a ring ------------------------------------------------------------------------------
// A CTA's rows go to its TEAMS in turn, so that one team's barriers and sums pass while another's exponentials are at work.  A team is WORKERS threads, a warp that gets the next row's
// entries ready and one that writes the last one's, with the loss; one more warp fills the ring for all of them.  `parts` CTAs, a cluster, share a row.
constexpr int DS_SLOTS = 8, DS_PARTS = 8;

struct DsInfo {
  float w;
  int label;  // -1: none
  int skip;
};
struct DsTeam {
  float red_m[2][8], red_s[2][8], red_u[2][8];  // of its warps
  float4 mail[2][DS_PARTS];                      // of the cluster's CTAs
  unsigned long long post[2];                    // complete when all of them have come
  float4 sums[2];                                // a row's maximum and sums, for the entries
  float soft[2];                                 // whether a row has a teacher
  float label_z[2], w[2];
  int label[2];
};
template <int TEAMS>
struct DsShared {
  // A slot serves any team's rows, a parity tells a wait one phase from the next alone: so a row's barrier `full` goes by the row's number and is one team's, which
  // meets every phase of it.  By slots, a team could ask for a phase while the one before, another team's, was yet to complete, and take that for its own.
  static_assert(DS_SLOTS % TEAMS == 0, "a barrier to a team");
  unsigned long long full[DS_SLOTS], empty[DS_SLOTS];
  DsInfo info[DS_SLOTS];
  float edge[DS_SLOTS][32];  // a row's loose logits
  DsTeam team[TEAMS];
  int abort;
};
// Some of a CTA's warps, in branches of their own: those that wait, and those that only have to have come so far.
__device__ __forceinline__ void ds_meet(int id, int threads) {
  __syncwarp();
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ void ds_tell(int id, int threads) {
  __syncwarp();
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// Bytes of the teacher's entries of one row: token, share, its logarithm, logit; in fours, so that they are looked through four at a time.
__host__ __device__ inline int ds_padded(int k) { return (k + 3) & ~3; }

template <typename T, int WORKERS, int TEAMS, int MODE>
__global__ void __launch_bounds__(TEAMS * (WORKERS + 64) + 32, 1) distill_ring_kernel(const DsArgs a, int parts) {
  constexpr int VEC = 16 / (int)sizeof(T), WARPS = WORKERS / 32;
  extern __shared__ __align__(128) uint8_t ds_smem[];
  __shared__ DsShared<TEAMS> sh;
  pdl_launch_dependents();
  const int t = threadIdx.x, lane = t & 31;
  const int rank = (int)(blockIdx.x % parts), first = (int)(blockIdx.x / parts), stride = (int)(gridDim.x / parts);
  if (t == 0) {
    for (int i = 0; i < DS_SLOTS; ++i) {
      mbar_init(smem_u32(&sh.full[i]), 1);
      mbar_init(smem_u32(&sh.empty[i]), WARPS);
    }
    for (int i = 0; i < TEAMS; ++i)
      for (int p = 0; p < 2; ++p) mbar_init(smem_u32(&sh.team[i].post[p]), 1);
    sh.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (parts > 1) cg::this_cluster().sync();  // every CTA of it is there
  pdl_wait_prior_grids();
  constexpr bool TWO = MODE != 0;
  const float c1 = TWO || a.soft == 0.f ? a.c : a.c_tau;
  const int v0 = rank * a.slice;  // this CTA's vectors of a row: v0 .. v0 + slice - 1
  if (t >= TEAMS * (WORKERS + 64)) {
    // fills the ring; a row's weight, label and loose logits are asked for a row ahead
    float w, edge;
    int label;
    auto ask = [&](long long r) {
      const T* z = (const T*)a.Z + r * a.ldz;
      const DsRow<T> row(z, a.V);
      w = a.weight ? a.weight[r] : 1.f;
      label = ds_label(a, r);
      edge = rank == 0 && lane < row.loose ? ds_f32(z[row.loose_at(lane)]) : 0.f;
    };
    int n = 0;
    ask(first);
    for (long long r = first; r < a.rows; r += stride, ++n) {
      const int slot = n % a.slots;
      const T* z = (const T*)a.Z + r * a.ldz;
      const DsRow<T> row(z, a.V);
      if (n >= a.slots) mbar_wait(smem_u32(&sh.empty[slot]), (uint32_t)(n / a.slots - 1) & 1u, &sh.abort, a.status);
      const bool skip = w == 0.f || (label < 0 && a.k == 0);
      sh.edge[slot][lane] = edge;
      __syncwarp();
      if (lane == 0) {
        sh.info[slot] = {w, label, skip ? 1 : 0};
        const uint32_t bytes = skip ? 0u : (uint32_t)max(0, min(row.vecs - v0, a.slice)) * 16u, bar = smem_u32(&sh.full[n % DS_SLOTS]);
        if (bytes == 0u) {
          mbar_arrive(bar);
        } else {
          mbar_arrive_expect_tx(bar, bytes);
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(ds_smem + (size_t)slot * a.slot_bytes)),
                       "l"(z + row.head + (long long)v0 * VEC), "r"(bytes), "r"(bar)
                       : "memory");
        }
      }
      if (r + stride < a.rows) ask(r + stride);
    }
  } else {
    const int team = t / (WORKERS + 64), tw = t % (WORKERS + 64), warp = tw >> 5;
    DsTeam& tm = sh.team[team];
    const int come = 1 + 2 * team, gone = 2 + 2 * team;  // barriers: a row's sums are there; its gradient has been written
    const long long r1 = first + (long long)team * stride, step = (long long)TEAMS * stride;
    const int kp = ds_padded(a.k);
    int* e_id = reinterpret_cast<int*>(ds_smem + (size_t)a.slots * a.slot_bytes) + team * 8 * kp;
    float *e_p = reinterpret_cast<float*>(e_id + 2 * kp), *e_lp = e_p + 2 * kp, *e_z = e_lp + 2 * kp;
    if (warp == WARPS) {  // gets entries ready
      // A row's entries come in two steps of memory, tokens and then their logits; the first is taken a row ahead of the second.
      constexpr int AHEAD = 2;  // entries a lane that are held meanwhile
      int next_id[AHEAD], next_label = -1;
      float next_t[AHEAD], next_w = 0.f;
      auto ask = [&](long long r) {
        if (r >= a.rows) return;
        next_label = ds_label(a, r);
        next_w = a.weight ? a.weight[r] : 1.f;
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) next_id[e] = lane + 32 * e < a.k ? ds_entry(a, r, lane + 32 * e, next_t[e]) : -1;
      };
      auto prepare = [&](long long r, int at) {
        int* id = e_id + at * kp;
        float *p = e_p + at * kp, *lp = e_lp + at * kp, *ze = e_z + at * kp;
        const T* z = (const T*)a.Z + r * a.ldz;
        const bool use = next_w != 0.f;
        const float zl = use && next_label >= 0 ? ds_f32(z[next_label]) : 0.f;
        float m = -INFINITY;
        int live = 0;
        auto entry = [&](int i, int j, float tv, float zj) {
          id[i] = j;
          lp[i] = tv;
          p[i] = 0.f;
          ze[i] = zj;
          if (j >= 0) live = 1, m = tv != tv ? tv : fmaxf(m, tv);
        };
        float zj[AHEAD];
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) zj[e] = use && next_id[e] >= 0 ? ds_f32(z[next_id[e]]) : 0.f;
#pragma unroll
        for (int e = 0; e < AHEAD; ++e)
          if (lane + 32 * e < kp) entry(lane + 32 * e, next_id[e], next_t[e], zj[e]);
        for (int i = lane + 32 * AHEAD; i < kp; i += 32) {
          float tv = 0.f;
          const int j = i < a.k ? ds_entry(a, r, i, tv) : -1;
          entry(i, j, tv, use && j >= 0 ? ds_f32(z[j]) : 0.f);
        }
        live = __any_sync(0xFFFFFFFFu, live);
        m = lanes_max<32>(m);
        float s = 0.f;
        for (int i = lane; i < a.k; i += 32)
          if (id[i] >= 0) s += p[i] = expf(lp[i] = (lp[i] - m) * a.inv_tau);
        s = lanes_sum<32>(s);
        const float log_s = logf(s);
        for (int i = lane; i < a.k; i += 32)
          if (id[i] >= 0) p[i] /= s, lp[i] -= log_s;
        if (lane == 0) {
          tm.soft[at] = live ? a.soft : 0.f;
          tm.label_z[at] = zl;
          tm.w[at] = next_w;
          tm.label[at] = next_label;
        }
        __syncwarp();
      };
      int n = 0;
      ask(r1);
      if (r1 < a.rows) prepare(r1, 0);
      for (long long r = r1; r < a.rows; r += step, ++n) {
        ask(r + step);
        ds_meet(come, WORKERS + 64);
        if (r + step < a.rows) prepare(r + step, ~n & 1);
      }
    } else if (warp == WARPS + 1) {  // writes them
      double sum_loss = 0.0;
      int n = 0;
      for (long long r = r1; r < a.rows; r += step, ++n) {
        const int at = n & 1;
        const int* id = e_id + at * kp;
        const float *p = e_p + at * kp, *lp = e_lp + at * kp, *ze = e_z + at * kp;
        ds_tell(come, WORKERS + 64);  // the row before is done with: its entries' place may be taken
        ds_meet(gone, WORKERS + 32);
        const float w = tm.w[at];
        const int label = tm.label[at];
        const float hard = label >= 0 ? a.hard : 0.f, soft = tm.soft[at];
        if (w == 0.f || (hard == 0.f && soft == 0.f)) {
          if (rank == 0 && lane == 0) a.loss[r] = 0.f;
          continue;
        }
        const float4 q = tm.sums[at];
        const float zl = tm.label_z[at];
        const DsSlope f = {q.x, w * (TWO ? hard : hard + soft * a.tau) / q.y, TWO ? w * soft * a.tau / q.z : 0.f, c1, a.c_tau};
        if (a.dZ) {
          const DsRow<T> row((const T*)a.Z + r * a.ldz, a.V);
          T* dz = (T*)a.dZ + r * a.lddz;
          for (int i = lane; i <= a.k; i += 32) {  // the label is the last one
            const int j = i < a.k ? id[i] : label;
            if (j < 0) continue;
            const int v = row.vec_of(j);
            if (v < 0 ? rank != 0 : v < v0 || v >= v0 + a.slice) continue;  // another CTA's
            float share = 0.f;  // all that falls on this token, in the entries' order
            if (soft != 0.f)
              for (int o = 0; o < kp; o += 4) {
                const int4 oi = *reinterpret_cast<const int4*>(id + o);
                const float4 op = *reinterpret_cast<const float4*>(p + o);
                share += oi.x == j ? op.x : 0.f;
                share += oi.y == j ? op.y : 0.f;
                share += oi.z == j ? op.z : 0.f;
                share += oi.w == j ? op.w : 0.f;
              }
            dz[j] = ds_from<T>(fmaf(-w, (j == label ? hard : 0.f) + soft * a.tau * share, f.at<MODE>(i < a.k ? ze[i] : zl)));
          }
        }
        if (rank == 0) {
          float kl = 0.f;
          const float log_u = logf(TWO ? q.z : q.y);
          if (soft != 0.f)
            for (int i = lane; i < a.k; i += 32)
              if (id[i] >= 0 && p[i] != 0.f) kl += p[i] * (lp[i] - ((ze[i] - q.x) * a.inv_tau - log_u));
          kl = lanes_sum<32>(kl);
          float L = soft != 0.f ? soft * a.tau * a.tau * kl : 0.f;
          if (label >= 0) L = fmaf(hard, logf(q.y) - (zl - q.x), L);
          if (lane == 0) {
            a.loss[r] = L;
            sum_loss += (double)w * L;
          }
        }
        __syncwarp();
      }
      if (a.total && rank == 0) ds_total(a, sum_loss, first * TEAMS + team, stride * TEAMS, lane);
    } else {
      int n = 0;
      for (long long r = r1; r < a.rows; r += step, ++n) {
        const int all = n * TEAMS + team, slot = all % a.slots, at = n & 1;  // (rows of all teams lie in the ring in turn)
        const T* z = (const T*)a.Z + r * a.ldz;
        T* dz = a.dZ ? (T*)a.dZ + r * a.lddz : nullptr;
        const DsRow<T> row(z, a.V);
        const int mine = max(0, min(row.vecs - v0, a.slice));
        mbar_wait(smem_u32(&sh.full[all % DS_SLOTS]), (uint32_t)(all / DS_SLOTS) & 1u, &sh.abort, a.status);
        const DsInfo info = sh.info[slot];
        const uint4* zs = reinterpret_cast<const uint4*>(ds_smem + (size_t)slot * a.slot_bytes);
        const bool edged = rank == 0 && tw < row.loose && !info.skip;
        const float edge = edged ? sh.edge[slot][tw] : -INFINITY;
        float m = edge;
        float2 s2 = make_float2(0.f, 0.f), u2 = make_float2(0.f, 0.f);
        if (!info.skip) {
#pragma unroll 4
          for (int i = tw; i < mine; i += WORKERS) m = fmaxf(m, DsVec<T>(zs[i]).max());
        }
        m = ds_floor(m);
        if (!info.skip) {
#pragma unroll 4
          for (int i = tw; i < mine; i += WORKERS) {
            DsVec<T>(zs[i]).template add<MODE>(s2, u2, m, c1, a.c_tau);
          }
          s2.x += ds_exp2((edge - m) * c1);  // fmaxf passes NaN over; the sums do not
          if (TWO) u2.x += ds_exp2((edge - m) * a.c_tau);
        }
        float s = s2.x + s2.y, u = u2.x + u2.y;
        {
          const float top = lanes_max<32>(m);
          s = lanes_sum<32>(s * ds_shift(m, top, c1));
          if (TWO) u = lanes_sum<32>(u * ds_shift(m, top, a.c_tau));
          if (lane == 0) {
            tm.red_m[at][warp] = top;
            tm.red_s[at][warp] = s;
            if (TWO) tm.red_u[at][warp] = u;
          }
        }
        ds_meet(come, WORKERS + 64);
        m = tm.red_m[at][0];
#pragma unroll
        for (int i = 1; i < WARPS; ++i) m = fmaxf(m, tm.red_m[at][i]);
        s = 0.f, u = 0.f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) {
          s += tm.red_s[at][i] * ds_shift(tm.red_m[at][i], m, c1);
          if (TWO) u += tm.red_u[at][i] * ds_shift(tm.red_m[at][i], m, a.c_tau);
        }
        if (parts > 1) {
          // to every CTA's mail; a place is written again two rows on, when its reader has sent the row between
          const uint32_t post = smem_u32(&tm.post[at]);
          if (tw == 0) mbar_arrive_expect_tx(post, (uint32_t)parts * 16u);
          if (tw < parts) {
            uint32_t place, bar;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(place) : "r"(smem_u32(&tm.mail[at][rank])), "r"(tw));
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar) : "r"(post), "r"(tw));
            st_async_f4(place, bar, m, s, u, 0.f);
          }
          mbar_wait_cluster(post, (uint32_t)(n >> 1) & 1u, &sh.abort, a.status);
          m = tm.mail[at][0].x;
          for (int i = 1; i < parts; ++i) m = fmaxf(m, tm.mail[at][i].x);
          s = 0.f, u = 0.f;
          for (int i = 0; i < parts; ++i) {
            const float4 q = tm.mail[at][i];
            s += q.y * ds_shift(q.x, m, c1);
            if (TWO) u += q.z * ds_shift(q.x, m, a.c_tau);
          }
        }
        if (tw == 0) tm.sums[at] = make_float4(m, s, u, 0.f);
        const float hard = info.label >= 0 ? a.hard : 0.f, soft = tm.soft[at];
        if (info.skip || (hard == 0.f && soft == 0.f)) {
          ds_zero(dz, a.V, rank, parts, tw, WORKERS);
        } else if (dz) {
          const DsSlope f = {m, info.w * (TWO ? hard : hard + soft * a.tau) / s, TWO ? info.w * soft * a.tau / u : 0.f, c1, a.c_tau};
          const bool same = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15u) == 0;
          T* out = dz + row.head + (long long)v0 * VEC;
#pragma unroll 4
          for (int i = tw; i < mine; i += WORKERS) ds_put<T, MODE>(f, zs[i], out + i * VEC, same);
          if (edged) dz[row.loose_at(tw)] = ds_from<T>(f.at<MODE>(edge));
        }
        fence_proxy_async_smem();  // what was read from the slot, before the next copy into it
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh.empty[slot]));
        ds_tell(gone, WORKERS + 32);
      }
    }
  }
  if (parts > 1) {
    __syncwarp();
    cg::this_cluster().sync();  // nobody leaves while mail may still come
  }
}

template <typename T, int LANES, bool WIDE, int NV, int E = 2>
ard_status ds_lanes(ard_ctx* ctx, const DsArgs& a, int mode, cudaStream_t s) {
  const int per = DS_SHORT_THREADS / LANES;
  const long long want = ((long long)a.rows + per - 1) / per, room = 8ll * ctx->sm_count;
  const dim3 grid((unsigned)(want < room ? want : room));
  ARD_CUDA_OK(ard_launch(ctx, mode ? distill_lanes_kernel<T, LANES, WIDE, NV, E, 1> : distill_lanes_kernel<T, LANES, WIDE, NV, E, 0>, grid,
                         dim3(DS_SHORT_THREADS), 0, s, a));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}

constexpr int DS_ROOM = 227 * 1024 - 4096;  // a CTA's ring and entries (beside the kernel's own variables)

// Slots of a ring for rows of `vecs` vectors cut into `parts`.
template <int TEAMS>
int ds_slots(long long vecs, int k, int parts) {
  const long long slot = ((vecs + parts - 1) / parts * 16 + 127) / 128 * 128;
  return slot > 0 ? (int)((DS_ROOM - TEAMS * 32ll * ds_padded(k)) / slot) : DS_SLOTS;
}
template <typename T, int WORKERS, int TEAMS>
ard_status ds_ring(ard_ctx* ctx, DsArgs a, int mode, int parts, cudaStream_t s) {
  constexpr int THREADS = TEAMS * (WORKERS + 64) + 32;
  auto kern = mode == 0   ? distill_ring_kernel<T, WORKERS, TEAMS, 0>
              : mode == 1 ? distill_ring_kernel<T, WORKERS, TEAMS, 1>
              : mode == 2 ? distill_ring_kernel<T, WORKERS, TEAMS, 2>
                          : distill_ring_kernel<T, WORKERS, TEAMS, 3>;
  const long long vecs = (long long)a.V * (int)sizeof(T) / 16;
  a.slice = (int)((vecs + parts - 1) / parts);
  a.slot_bytes = a.slice > 0 ? (a.slice * 16 + 127) / 128 * 128 : 128;
  const int slots = ds_slots<TEAMS>(vecs, a.k, parts);
  if (slots < 1) return ARD_ERR_UNSUPPORTED;
  a.slots = slots < DS_SLOTS ? slots : DS_SLOTS;
  const size_t smem = (size_t)a.slots * a.slot_bytes + TEAMS * 32ull * ds_padded(a.k);
  ARD_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  long long clusters = ctx->sm_count;
  if (parts > 1) clusters = ard_cluster_room(ctx, kern, parts, THREADS, (int)smem) / parts;
  if (clusters > a.rows) clusters = a.rows;
  ARD_CUDA_OK(ard_launch_cluster(ctx, kern, parts, dim3((unsigned)(clusters * parts)), dim3(THREADS), smem, s, a, parts));
  ctx->launches++;
  ARD_CUDA_OK(cudaGetLastError());
  return ARD_OK;
}

template <typename T>
ard_status ds_launch(ard_ctx* ctx, const DsArgs& a, int mode, cudaStream_t s) {
  constexpr int VEC = 16 / (int)sizeof(T);
  // as few lanes a row as hold it and the teacher's entries: what a row needs once costs a warp the same for one row as for four
  if (a.k <= 16) {
    if (a.V <= 32) return ds_lanes<T, 8, false, 4>(ctx, a, mode, s);
    if (a.V <= 128) return ds_lanes<T, 8, false, 16>(ctx, a, mode, s);
    if (a.V <= 8 * 8 * VEC) return ds_lanes<T, 8, true, 8>(ctx, a, mode, s);
  }
  if (a.k <= 64) {
    if (a.V <= 128) return ds_lanes<T, 32, false, 4>(ctx, a, mode, s);
    if (a.V <= 32 * 4 * VEC) return ds_lanes<T, 32, true, 4>(ctx, a, mode, s);
    if (a.V <= 32 * 8 * VEC) return ds_lanes<T, 32, true, 8>(ctx, a, mode, s);
    if (a.V <= 32 * 16 * VEC) return ds_lanes<T, 32, true, 16>(ctx, a, mode, s);
  }
  if (a.k <= 128) {  // 20000 bf16 rows with 100 entries: of 300 71 us (in the ring 178), of 2000 116 (206); of 4000 219 either way, few of them 15.5 (11.8)
    if (a.V <= 128) return ds_lanes<T, 32, false, 4, 4>(ctx, a, mode, s);
    if (a.V <= 32 * 4 * VEC) return ds_lanes<T, 32, true, 4, 4>(ctx, a, mode, s);
    if (a.V <= 32 * 8 * VEC) return ds_lanes<T, 32, true, 8, 4>(ctx, a, mode, s);
  }
  // four teams where the ring holds a row for each and one on its way, else two, with rows cut over as few CTAs as that takes
  const long long vecs = (long long)a.V / VEC;
  if (ds_slots<4>(vecs, a.k, 1) >= 5) return ds_ring<T, 160, 4>(ctx, a, mode, 1, s);
  int parts = 1;
  while (parts < DS_PARTS && ds_slots<2>(vecs, a.k, parts) < 3) parts *= 2;
  return ds_ring<T, 256, 2>(ctx, a, mode, parts, s);
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
  const int mode = a.hard == 0.f || a.soft == 0.f || tau == 1.f ? 0 : tau == 2.f ? 2 : tau == 4.f ? 3 : 1;
  return dtype == ARD_F32 ? ds_launch<float>(ctx, a, mode, s) : ds_launch<__nv_bfloat16>(ctx, a, mode, s);
}
