// Group norm with an activation on channels-last maps: y = act(gamma[c] * (x - mean_g) / sqrt(var_g + eps) + beta[c] (+ residual)),
// mean and (biased) variance over the pixels of a sample and the channels of its group g.
//
// What bounds it is memory: x read once, y written once.  So a sample's slice of whole groups (about 128 bytes of channels) is
// fetched into the shared memory of a cluster of up to eight CTAs, each with a range of the pixels, and stays there between the
// statistics and the normalisation.  The statistics take two passes over what is in shared memory, the sum and then the squares
// about the CTA's own mean, so that they do not cancel where a mean is large against its deviation; the CTAs exchange
// (mean, sum of squares) through distributed shared memory and every CTA joins them in the same order:
//   mean = sum n_i mean_i / n,   S = sum (S_i + n_i (mean_i - mean)^2).
// All sums are fp32.  Slice, cluster and order of the sums follow from the map's shape alone, never from the batch: a sample's bits
// do not depend on whom it rides with.
//
// A thread keeps one column of 16 bytes of channels and walks down the pixels, so gamma and beta live in registers and a vector may
// hold several groups or parts of them.  Rows that are not whole 16-byte vectors, or pointers off a 16-byte boundary, take one element at a time.
#pragma once
#include <algorithm>

#include "common.cuh"

namespace ee {

constexpr int kNormThreads = 256;
constexpr int kNormMaxCluster = 8;
constexpr int kNormChunk = 56 << 10;        // bytes of a CTA's part of a slice that a cluster is cut for: three CTAs share an SM
constexpr int kNormMaxChunk = 192 << 10;    // beyond this, and at eight CTAs, the map is read again from global memory instead

struct NormPlan {
  int v;             // elements per access
  int sv, slices;    // accesses per pixel of a slice, slices of a sample
  int groups;        // groups of a slice
  int cluster, rows; // CTAs of a slice, pixels of each
  bool wide;         // a pixel of the slice is more than the CTA's threads take at once; the slice is then one group
  bool merged;       // an access lies in one group: its elements are summed together
  bool resident;
  int smem, off_red, off_stat;
};

struct NormArgs {
  const void* x;
  const void* residual;
  void* y;
  const float* gamma;
  const float* beta;
  float eps;
  int hw, c, cpg, act;
  int sv, slices, groups, rows, off_red, off_stat;
  int rev;           // 1: from the last sample down (the newest samples of the input are the ones still in L2)
};

inline int norm_gcd(int a, int b) {
  while (b) {
    const int t = a % b;
    a = b, b = t;
  }
  return a;
}

inline NormPlan norm_plan(int hw, int c, int groups, int es, bool aligned) {
  NormPlan p = {};
  const int cpg = c / groups;
  p.v = aligned && (size_t)c * es % 16 == 0 ? 16 / es : 1;
  int unit = cpg / norm_gcd(cpg, p.v) * p.v;               // channels that are whole groups and whole accesses
  if (unit / p.v > kNormThreads && cpg % p.v) p.v = 1, unit = cpg;
  p.wide = unit / p.v > kNormThreads;
  // Wide enough for whole 128-byte lines, and on maps of few pixels for every thread to have something.
  const long most = std::max<long>(128, (long)kNormThreads * 16 / std::max(hw, 1));
  const int units = c / unit;
  int m = 1;
  if (!p.wide)
    for (int d = 1; d <= units; ++d)
      if (units % d == 0 && (long)unit * d * es <= most && unit * d / p.v <= kNormThreads) m = d;
  const int s = unit * m;
  p.sv = s / p.v, p.slices = c / s, p.groups = s / cpg, p.merged = cpg % p.v == 0;
  p.cluster = 1;
  const long row = (long)s * es;
  while (p.cluster < kNormMaxCluster && p.cluster * 2 <= hw && ((long)hw + p.cluster - 1) / p.cluster * row > kNormChunk) p.cluster *= 2;
  p.rows = (hw + p.cluster - 1) / p.cluster;
  p.resident = p.rows * row <= kNormMaxChunk;
  p.off_red = p.resident ? (int)align_up((size_t)(p.rows * row), 16) : 0;
  p.off_stat = p.off_red + kNormThreads * (p.merged ? 1 : p.v) * 4;
  p.smem = p.off_stat + p.groups * 4 * 4;                   // mean and squares of this CTA, of all
  return p;
}

template <typename T, int V> struct NormVec {   // V elements as they are stored
  T e[V];
};
template <> struct __align__(16) NormVec<bf16, 8> { bf16 e[8]; };
template <> struct __align__(16) NormVec<float, 4> { float e[4]; };

template <typename T, int V>
__device__ __forceinline__ void norm_unpack(const NormVec<T, V>& r, float* f) {
  if constexpr (V == 1) {
    f[0] = Elem<T>::ld(r.e);
  } else {
    Vec16<T> t;
    t.unpack(*reinterpret_cast<const uint4*>(&r));
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = t.v[i];
  }
}

// SiLU: the fast exponential is off by 2 + 1.2 |v| units in the last place, which weigh with exp(-v) / (1 + exp(-v)) where v > 0 and
// relative to a vanishing result where v < 0; the fast quotient is 0 where exp(-v) passes 2^126, v < -87.
__device__ __forceinline__ float norm_act(float v, int act) {
  if (act == EE_ACT_SILU) return __fdividef(v, 1.f + __expf(-v));
  return apply_act(v, act);
}
// Pairwise sum of an access.
template <int V>
__device__ __forceinline__ float norm_tree(const float* f) {
  if constexpr (V == 1) return f[0];
  else return norm_tree<V / 2>(f) + norm_tree<V / 2>(f + V / 2);
}

// V elements per access, MERGED and WIDE as in NormPlan; RESIDENT: the CTA's pixels stay in shared memory.
template <typename T, int V, bool MERGED, bool WIDE, bool RESIDENT>
__global__ void __launch_bounds__(kNormThreads)
group_norm_kernel(NormArgs p) {
  static_assert(!WIDE || MERGED, "a wide slice is one group");
  typedef NormVec<T, V> Vec;
  constexpr int K = MERGED ? 1 : V;      // sums per thread
  extern __shared__ __align__(16) uint8_t norm_smem[];
  float* red = reinterpret_cast<float*>(norm_smem + p.off_red);
  float* stat = reinterpret_cast<float*>(norm_smem + p.off_stat);   // [mean, squares] of this CTA, then [mean, 1 / deviation] of the slice
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t rank, cluster;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
  const long unit = (p.rev ? gridDim.x - 1 - blockIdx.x : blockIdx.x) / cluster;
  const int slice = (int)(unit % p.slices);
  const long sample = unit / p.slices;
  const int row0 = min((int)rank * p.rows, p.hw), rows = min(p.rows, p.hw - row0);
  const size_t first = ((size_t)sample * p.hw + row0) * p.c + (size_t)slice * p.sv * V;
  const T* x = reinterpret_cast<const T*>(p.x) + first;
  // this thread's accesses: column, pixel, and the step to the next one
  const int ty_n = WIDE ? 1 : kNormThreads / p.sv;
  const int col0 = WIDE ? tid : tid % p.sv, ty = WIDE ? 0 : tid / p.sv;
  const bool active = WIDE || ty < ty_n;
  auto each = [&](auto&& body) {
    if constexpr (WIDE) {
      for (int col = tid, row = 0; row < rows;) {
        while (col >= p.sv) {
          col -= p.sv;
          if (++row >= rows) return;
        }
        body(row, col);
        col += kNormThreads;
      }
    } else if (active) {
#pragma unroll 4
      for (int row = ty; row < rows; row += ty_n) body(row, col0);
    }
  };
  auto held = [&](int row, int col) {
    if constexpr (RESIDENT)
      return *reinterpret_cast<const Vec*>(norm_smem + ((size_t)row * p.sv + col) * sizeof(Vec));
    else
      return *reinterpret_cast<const Vec*>(x + (size_t)row * p.c + col * V);
  };
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if constexpr (RESIDENT) {   // a thread reads back what it fetched itself
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(norm_smem);
    each([&](int row, int col) {
      const T* src = x + (size_t)row * p.c + col * V;
      const uint32_t dst = at + (uint32_t)((row * p.sv + col) * (int)sizeof(Vec));
      if constexpr (sizeof(Vec) == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
      else if constexpr (sizeof(Vec) == 4)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
      else
        *reinterpret_cast<Vec*>(norm_smem + ((size_t)row * p.sv + col) * sizeof(Vec)) = *reinterpret_cast<const Vec*>(src);
    });
    cp_async_commit();
    cp_async_wait<0>();
  }
  // sums of the groups: each thread leaves its K sums in red, a warp adds up a group
  const int bins = WIDE ? 1 : p.sv * K, per_group = bins / p.groups;   // bins of a pixel, of a group of it
  const int reducers = WIDE ? kNormThreads : ty_n;                     // rows of red
  float sum[K];
  auto group_sums = [&](auto&& done) {
    if (active) {
#pragma unroll
      for (int k = 0; k < K; ++k) red[WIDE ? tid : ty * bins + col0 * K + k] = sum[k];
    }
    __syncthreads();
    const int n = reducers * per_group;
    for (int g = warp; g < p.groups; g += kNormThreads / 32) {
      float s = 0.f;
      for (int i = lane; i < n; i += 32) {
        const int r = i / per_group;
        s += red[r * bins + g * per_group + (i - r * per_group)];
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
      if (lane == 0) done(g, s);
    }
    __syncthreads();
  };
  const float n_here = (float)rows * (float)p.cpg;
#pragma unroll
  for (int k = 0; k < K; ++k) sum[k] = 0.f;
  each([&](int row, int col) {
    float f[V];
    norm_unpack<T, V>(held(row, col), f);
    if constexpr (MERGED) {
      sum[0] += norm_tree<V>(f);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += f[i];
    }
  });
  group_sums([&](int g, float s) { stat[2 * g] = rows > 0 ? s / n_here : 0.f; });
  int group_of[K];     // the groups of this thread's columns; threads without a column take any
  float mean[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    group_of[k] = WIDE ? 0 : min((col0 * V + k) / p.cpg, p.groups - 1);
    mean[k] = stat[2 * group_of[k]], sum[k] = 0.f;
  }
  each([&](int row, int col) {
    float f[V];
    norm_unpack<T, V>(held(row, col), f);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = f[i] - mean[MERGED ? 0 : i];
      if constexpr (MERGED) f[i] = d * d;
      else sum[i] = fmaf(d, d, sum[i]);
    }
    if constexpr (MERGED) sum[0] += norm_tree<V>(f);
  });
  group_sums([&](int g, float s) { stat[2 * g + 1] = s; });
  // the cluster's statistics
  float* all = stat + 2 * p.groups;
  if (cluster > 1) {
    asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
    const uint32_t stat_s = (uint32_t)__cvta_generic_to_shared(stat);
    for (int g = tid; g < p.groups; g += kNormThreads) {
      float m[kNormMaxCluster], q[kNormMaxCluster], s = 0.f;
#pragma unroll
      for (int r = 0; r < kNormMaxCluster; ++r)
        if (r < (int)cluster) {
          uint32_t from;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(stat_s + 8u * g), "r"(r));
          asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(m[r]), "=f"(q[r]) : "r"(from) : "memory");
        }
      const float n = (float)p.hw * (float)p.cpg;
#pragma unroll
      for (int r = 0; r < kNormMaxCluster; ++r)
        if (r < (int)cluster) s = fmaf((float)max(0, min(p.rows, p.hw - r * p.rows)) * (float)p.cpg, m[r], s);
      const float mu = s / n;
      s = 0.f;
#pragma unroll
      for (int r = 0; r < kNormMaxCluster; ++r)
        if (r < (int)cluster) {
          const float d = m[r] - mu;
          s += fmaf((float)max(0, min(p.rows, p.hw - r * p.rows)) * (float)p.cpg, d * d, q[r]);
        }
      all[2 * g] = mu, all[2 * g + 1] = 1.f / sqrtf(s / n + p.eps);
    }
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");   // this CTA reads no other one's memory any more
    __syncthreads();
  } else {
    for (int g = tid; g < p.groups; g += kNormThreads) all[2 * g] = stat[2 * g], all[2 * g + 1] = 1.f / sqrtf(stat[2 * g + 1] / n_here + p.eps);
    __syncthreads();
  }
  // y = (x - mean) * (gamma / deviation) + beta
  const T* res = p.residual ? reinterpret_cast<const T*>(p.residual) + first : nullptr;
  T* y = reinterpret_cast<T*>(p.y) + first;
  float a[V], b[V];
  auto affine = [&](int col) {
    const int c = slice * p.sv * V + col * V;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float rstd = all[2 * group_of[MERGED ? 0 : i] + 1];
      a[i] = p.gamma ? p.gamma[c + i] * rstd : rstd, b[i] = p.beta ? p.beta[c + i] : 0.f;
    }
  };
#pragma unroll
  for (int k = 0; k < K; ++k) mean[k] = all[2 * group_of[k]];
  if (!WIDE && active) affine(col0);
  each([&](int row, int col) {
    if (WIDE) affine(col);
    const size_t at = (size_t)row * p.c + col * V;
    Vec r;
    if (res) r = *reinterpret_cast<const Vec*>(res + at);
    float f[V], q[V];
    norm_unpack<T, V>(held(row, col), f);
    if (res) norm_unpack<T, V>(r, q);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float t = fmaf(f[i] - mean[MERGED ? 0 : i], a[i], b[i]);
      if (res) t += q[i];
      f[i] = norm_act(t, p.act);
    }
    if constexpr (V == 1) {
      Elem<T>::st(y + at, f[0]);
    } else {
      Vec16<T> o;
#pragma unroll
      for (int i = 0; i < V; ++i) o.v[i] = f[i];
      o.store(y + at);
    }
  });
  if (cluster > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");   // nobody reads this CTA's shared memory any more
}

template <typename T, int V, bool MERGED, bool WIDE, bool RESIDENT>
inline cudaError_t norm_launch_k(const NormPlan& pl, const NormArgs& a, long batch, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  if (pl.smem > 48 << 10) e = cudaFuncSetAttribute(group_norm_kernel<T, V, MERGED, WIDE, RESIDENT>, cudaFuncAttributeMaxDynamicSharedMemorySize, pl.smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(batch * pl.slices * pl.cluster));
  cfg.blockDim = dim3(kNormThreads);
  cfg.dynamicSmemBytes = pl.smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = pl.cluster, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pl.cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, group_norm_kernel<T, V, MERGED, WIDE, RESIDENT>, a);
}

template <typename T, int V>
inline cudaError_t norm_launch_v(const NormPlan& pl, const NormArgs& a, long batch, cudaStream_t st) {
  if (pl.wide) return pl.resident ? norm_launch_k<T, V, true, true, true>(pl, a, batch, st) : norm_launch_k<T, V, true, true, false>(pl, a, batch, st);
  if (pl.merged) return pl.resident ? norm_launch_k<T, V, true, false, true>(pl, a, batch, st) : norm_launch_k<T, V, true, false, false>(pl, a, batch, st);
  if constexpr (V > 1)
    return pl.resident ? norm_launch_k<T, V, false, false, true>(pl, a, batch, st) : norm_launch_k<T, V, false, false, false>(pl, a, batch, st);
  return cudaErrorInvalidValue;
}

// Whether a grid holds a call's blocks: its limit is 2^31 - 1.
inline bool norm_fits(const NormPlan& pl, long batch) { return batch * pl.slices * pl.cluster <= 0x7fffffffL; }

template <typename T>
inline cudaError_t norm_launch(const void* x, const void* residual, void* y, const float* gamma, const float* beta, float eps, long batch, int hw, int c,
                               int groups, int act, bool rev, cudaStream_t st) {
  const bool aligned = (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)y) & 15) == 0;
  const NormPlan pl = norm_plan(hw, c, groups, (int)sizeof(T), aligned);
  if (!norm_fits(pl, batch)) return cudaErrorInvalidValue;
  const NormArgs a = {x, residual, y, gamma, beta, eps, hw, c, c / groups, act, pl.sv, pl.slices, pl.groups, pl.rows, pl.off_red, pl.off_stat, rev ? 1 : 0};
  return pl.v > 1 ? norm_launch_v<T, Elem<T>::kVec>(pl, a, batch, st) : norm_launch_v<T, 1>(pl, a, batch, st);
}

}  // namespace ee
