// Group norm with an activation on channels-last maps: y = act(gamma[c] * (x - mean_g) / sqrt(var_g + eps) + beta[c] (+ residual)),
// mean and (biased) variance over the pixels of a sample and the channels of its group g.
//
// What bounds it is memory: x read once, y written once.  So a unit, a sample's slice of whole groups (about 128 bytes of channels), is
// fetched into the shared memory of a cluster of CTAs, each with a range of the pixels, and stays there between the
// statistics and the normalisation.  Four small CTAs share an SM, so that one's loads and stores run beside another's barriers.  (Clusters that take one unit
// after the other, the next one on its way into a second buffer, were slower: 91 against 63 us on 64 x 56 x 56 x 256 with a residual.)
// Sums of squares would cancel where a mean is large against its deviation, so every part (a thread's
// values, a warp's, a CTA's, the cluster's) is (mean, squares about it), and parts are joined, in a fixed order, as
//   mean = sum n_i mean_i / n,   S = sum (S_i + n_i (mean_i - mean)^2);
// the CTAs send each other theirs as asynchronous stores, which the receiver's barrier counts: nothing but the data is waited for.
// All sums are fp32.  Slice, cluster and order of the sums follow from the map's shape and from whether rows lie on 16-byte boundaries, never from the batch: a sample's
// bits do not depend on whom it rides with.  64 x 56 x 56 x 256 bf16 with a residual 62.7 us (4.9 TB/s), 32 x 112 x 112 x 96 53.0, 1 x 7 x 7 x 2048 3.3.
//
// A thread keeps one column of 16 bytes of channels and walks down the pixels, so gamma and beta live in registers and a vector may
// hold several groups or parts of them.  Rows that are not whole 16-byte vectors, or pointers off a 16-byte boundary, take one element at a time.
#pragma once
#include <algorithm>

#include "common.cuh"
#include "conv_tc.cuh"

namespace ee {

constexpr int kNormMaxCluster = 8;
// Bytes of a CTA's part of a unit that a cluster is cut for, and up to which it stays in shared memory where eight CTAs are not enough for that: four CTAs then
// share an SM.  Larger parts are read a second time, from L2.  us, 28 / 56 KB parts: 13 x 33 x 29 x 96 fp32 6.4 / 7.9; the second read in place of two CTAs an SM:
// 32 x 112 x 112 x 96 84 -> 65 (parts of 150 KB), of four: 64 x 56 x 56 x 256 62 -> 68 (50 KB).  Parts of up to 104 KB kept by CTAs of 512 threads won and lost:
// 64 x 80 x 80 x 128 63 -> 56, 16 of them 18.6 -> 19.8, 32 x 72 x 72 x 96 28.8 -> 30.
constexpr int kNormChunk = 28 << 10;
constexpr int kNormMaxChunk = 56 << 10;
// What a CTA asks for at most: its part, 16 KB of partial statistics of 256 threads (8 bytes for each of up to eight runs of an access), and 8 bytes for each group and
// CTA, of which there are 1024 where one CTA has the whole slice (of 2 KB) and 64 where eight have.
constexpr int kNormMaxSmem = 80 << 10;

struct NormPlan {
  int v;             // elements per access
  int sv, slices;    // accesses per pixel of a slice, slices of a sample
  int groups;        // groups of a slice
  int cluster, rows; // CTAs of a slice, pixels of each
  int threads;
  bool wide;         // a pixel of the slice is more than the CTA's threads take at once; the slice is then one group
  int parts;         // an access falls into so many runs that lie in one group each and are summed together
  bool resident;
  int chunk, red_rows, bins;   // bytes of a CTA's part; partial statistics: rows and columns
  int smem() const { return chunk + red_rows * bins * 8 + groups * 8 * (cluster + 1) + 8; }
};

struct NormArgs {
  const void* x;
  const void* residual;
  void* y;
  const float* gamma;
  const float* beta;
  float eps;
  int hw, c, cpg, act;
  int sv, slices, groups, rows, chunk, red_rows, bins;
  int* err_flag;
  long long wait_cycles;   // limit of the wait for the cluster's statistics
  int rev;           // 1: from the last sample down (the newest samples of the input are the ones still in L2)
};

inline int norm_gcd(int a, int b) {
  while (b) {
    const int t = a % b;
    a = b, b = t;
  }
  return a;
}

// Threads of a CTA: many where the part does not stay in shared memory and is read twice, for the loads in flight of few samples.  us, 256 / 512 threads there:
// 4 x 128 x 128 x 128 30 / 22.5, 1 x 224 x 224 x 32 33 / 24, 16 x 112 x 112 x 64 28.5 / 23.4, 32 x 112 x 112 x 96 51 / 54 (1024: 76).
constexpr int kNormThreads = 256, kNormFew = 128, kNormMany = 512;

inline NormPlan norm_plan(int hw, int c, int groups, int es, bool aligned) {
  NormPlan p = {};
  const int cpg = c / groups;
  p.v = aligned && (size_t)c * es % 16 == 0 ? 16 / es : 1;
  int unit = cpg / norm_gcd(cpg, p.v) * p.v;               // channels that are whole groups and whole accesses
  if (unit / p.v > kNormThreads && cpg % p.v) p.v = 1, unit = cpg;
  p.wide = unit / p.v > kNormThreads;
  // Wide enough for whole 128-byte lines, and on maps of few pixels for 128 threads to have something.
  const long most = std::max<long>(128, (long)kNormFew * 16 / std::max(hw, 1));
  const int units = c / unit;
  int m = 1;
  if (!p.wide)
    for (int d = 1; d <= units; ++d)
      if (units % d == 0 && (long)unit * d * es <= most && unit * d / p.v <= kNormThreads) m = d;
  const int s = unit * m;
  p.sv = s / p.v, p.slices = c / s, p.groups = s / cpg, p.parts = p.v / norm_gcd(p.v, cpg);
  p.cluster = 1;
  const long row = (long)s * es;
  while (p.cluster < kNormMaxCluster && p.cluster * 2 <= hw && ((long)hw + p.cluster - 1) / p.cluster * row > kNormChunk) p.cluster *= 2;
  p.rows = (int)(((long)hw + p.cluster - 1) / p.cluster);
  p.resident = p.rows * row <= kNormMaxChunk;
  p.chunk = p.resident ? (int)align_up((size_t)(p.rows * row), 16) : 0;
  // few accesses: few threads, so that each still has some
  p.threads = !p.resident ? kNormMany : p.sv <= kNormFew && (long)p.rows * p.sv <= 4 * kNormFew ? kNormFew : kNormThreads;
  p.bins = p.wide ? 1 : p.sv * p.parts;
  p.red_rows = p.wide || p.sv <= 32 ? p.threads / 32 : p.threads / p.sv;
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

// SiLU, v / (1 + exp(-v)): 2^x is off by 2 units in the last place and x = -v log2(e) by 1.2 |v| of them in the power, which weigh with exp(-v) / (1 + exp(-v))
// where v > 0 and relative to a vanishing result where v < 0; the reciprocal adds one.
// The other activations are clamps: to [lo, hi], NaN staying NaN.
struct NormClamp {
  float lo, hi;
  __device__ __forceinline__ explicit NormClamp(int act) : lo(act == EE_ACT_NONE ? -INFINITY : 0.f), hi(act == EE_ACT_RELU6 ? 6.f : INFINITY) {}
};
template <bool SILU>
__device__ __forceinline__ float norm_act(float v, const NormClamp& c) {
  if constexpr (SILU) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return v * r;
  }
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(c.lo));
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(c.hi));
  return v;
}
template <bool B> struct Flag { static constexpr bool value = B; };
// Two floats in one register pair: the packed instructions round each half like the scalar ones.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair_of(float lo, float hi) {
  f32x2 d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void pair_split(f32x2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 pair_add(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ f32x2 pair_fma(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}

// V elements per access in K parts, WIDE as in NormPlan; RESIDENT: the CTA's pixels stay in shared memory; NT threads.  With up to two
// sums, or four of pairs, a thread's state leaves room for 1024 threads an SM (64 registers): 64 x 56 x 56 x 192 in groups of 6 60 -> 51 us; four single ones, 13 x 33 x 29 x 96 fp32
// in groups of 3, take 6.4 us with 80 registers and 8.1 with 64.
template <typename T, int V, int K, bool WIDE, bool RESIDENT, int NT>
__global__ void __launch_bounds__(NT, !RESIDENT || K <= 2 || (K == 4 && V == 8) ? 1024 / NT : 768 / NT)
group_norm_kernel(const __grid_constant__ NormArgs p) {
  static_assert(!WIDE || K == 1, "a wide slice is one group");
  typedef NormVec<T, V> Vec;
  constexpr int G = V / K;                             // elements of a part
  constexpr int P = V > 1 ? V / 2 : 1;                 // pairs of an access
  constexpr int NW = NT / 32;
  extern __shared__ __align__(16) uint8_t norm_smem[];
  float2* red = reinterpret_cast<float2*>(norm_smem + p.chunk);
  float2* stat = red + p.red_rows * p.bins;            // [groups][cluster]: (mean, squares) of every CTA
  uint32_t rank, cluster;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
  float2* all = stat + p.groups * (int)cluster;    // [groups]: (mean, 1 / deviation) of the unit
  const uint32_t arrived = (uint32_t)__cvta_generic_to_shared(all + p.groups);      // counts what the CTAs send
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (cluster > 1) {
    if (tid == 0) {
      mbar_init(arrived, 1);
      mbar_expect_tx(arrived, (uint32_t)p.groups * cluster * 8u);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");    // waited for before anything is sent
  }
  const int rows = min(p.rows, p.hw - min((int)rank * p.rows, p.hw));
  // This thread's accesses: its column, its first pixel, and the step to the next one.  Slices of up to 32 accesses: a warp has whole pixels.
  const bool by_warp = !WIDE && p.sv <= 32;
  const int warp_rows = by_warp ? 32 / p.sv : 1;
  const int ty_n = WIDE ? 1 : by_warp ? NW * warp_rows : NT / p.sv;
  const int lane_row = by_warp ? lane / p.sv : 0;
  const int col0 = WIDE ? tid : by_warp ? lane - lane_row * p.sv : tid % p.sv;
  const int ty = WIDE ? 0 : by_warp ? warp * warp_rows + lane_row : tid / p.sv;
  const bool active = WIDE || (by_warp ? lane_row < warp_rows : ty < ty_n);
  auto each = [&](auto&& body) {
    if constexpr (WIDE) {
      for (int col = tid, row = 0; row < rows;) {
        while (col >= p.sv) {
          col -= p.sv;
          if (++row >= rows) return;
        }
        body(row, col);
        col += NT;
      }
    } else if (active) {
#pragma unroll 4
      for (int row = ty; row < rows; row += ty_n) body(row, col0);
    }
  };
  const long unit = (p.rev ? gridDim.x - 1 - blockIdx.x : blockIdx.x) / cluster, sample = unit / p.slices;
  const int channel = (int)(unit - sample * p.slices) * p.sv * V;            // of the slice
  const size_t first = ((size_t)sample * p.hw + min((int)rank * p.rows, p.hw)) * p.c + (size_t)channel;
  const T* x = reinterpret_cast<const T*>(p.x) + first;
  auto held = [&](int row, int col) {
    if constexpr (RESIDENT)
      return *reinterpret_cast<const Vec*>(norm_smem + (size_t)(row * p.sv + col) * sizeof(Vec));
    else
      return *reinterpret_cast<const Vec*>(x + (size_t)row * p.c + col * V);
  };
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if constexpr (RESIDENT) {            // a thread reads back what it fetched itself: no barrier
    const uint32_t smem_s = (uint32_t)__cvta_generic_to_shared(norm_smem);
    each([&](int row, int col) {
      const T* src = x + (size_t)row * p.c + col * V;
      const uint32_t dst = smem_s + (uint32_t)((row * p.sv + col) * (int)sizeof(Vec));
      if constexpr (sizeof(Vec) == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
      else if constexpr (sizeof(Vec) == 4)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
      else
        *reinterpret_cast<Vec*>(norm_smem + (size_t)(row * p.sv + col) * sizeof(Vec)) = *reinterpret_cast<const Vec*>(src);
    });
    cp_async_commit();
    if (p.residual) {                  // on its way to L2 while the statistics are taken
      const char* res = reinterpret_cast<const char*>(p.residual) + first * sizeof(T);
      for (int row = tid; row < rows; row += NT)
        for (int i = 0; i < p.sv * (int)sizeof(Vec); i += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(res + (size_t)row * p.c * sizeof(T) + i));
    }
    cp_async_wait<0>();
  }
  const float n_here = (float)rows * (float)p.cpg, inv_here = rows > 0 ? 1.f / n_here : 0.f, inv_all = 1.f / ((float)p.hw * (float)p.cpg);
  const int lin = WIDE ? rows * p.sv : rows, step = WIDE ? NT : ty_n;    // thread r takes r, r + step, ... of lin
  const int full = lin / step, more = lin - full * step;
  auto count_of = [&](int r) { return (float)((full + (r < more ? 1 : 0)) * G); };
  // A row of red is a warp (its pixels together), or, where a pixel is more than a warp, the threads of one ty.
  const int red_row = WIDE || by_warp ? warp : ty;
  auto count_of_row = [&](int r) {
    if (WIDE) {
      float n = 0.f;
      for (int i = 0; i < 32; ++i) n += count_of(r * 32 + i);
      return n;
    }
    return by_warp ? (float)((full * warp_rows + min(max(more - r * warp_rows, 0), warp_rows)) * G) : count_of(r);
  };
  const int per_group = p.bins / p.groups;             // bins of a group
  const int r_first = lane / per_group, r_step = 32 / per_group, b_first = lane - r_first * per_group, b_step = 32 - r_step * per_group;

  // One pass, in runs of kRun accesses: a thread sums d = x - mean and d^2, about its own first value of the group (or channel) in the first run and its mean so far in
  // the later ones.  With s and q the run's sums and N the thread's values with it, the mean moves by s / N and the squares grow by q - s^2 / N.  In short runs, because
  // where the first value is an extreme one, n values in chains of m lose n m / 2 roundings (u = 2^-24) of what they say of it: 512 u with 16 fp32 accesses (32 of one
  // value), 8192 u with 32 of bf16, an eighth of the result's own rounding; without runs 2 % of the deviation of a map of 1024 x 1024.
  float mean[K], m2[K];                                // mean: what the differences are from
#pragma unroll
  for (int k = 0; k < K; ++k) mean[k] = m2[k] = 0.f;
  {
    const int r0 = WIDE ? tid / p.sv : ty, c0 = WIDE ? tid % p.sv : col0;
    if (active && r0 < rows) {
      float f[V];
      norm_unpack<T, V>(held(r0, c0), f);
#pragma unroll
      for (int k = 0; k < K; ++k) mean[k] = f[k * G];
    }
  }
  // Pairs of accumulators: of one part, two elements of it (and two chains where an access is summed together); else of two neighbouring parts.
  constexpr int A = K == 1 ? 2 : G > 1 ? K : P;
  constexpr int kRun = V == 4 ? 16 : 32;
  f32x2 s[A], q[A], less[P];
  float s1 = 0.f, q1 = 0.f;              // V = 1
  auto begin = [&]() {
    if constexpr (V == 1) {
      s1 = q1 = 0.f;
    } else {
#pragma unroll
      for (int i = 0; i < A; ++i) s[i] = q[i] = 0ull;
#pragma unroll
      for (int i = 0; i < P; ++i) less[i] = pair_of(-mean[2 * i / G], -mean[(2 * i + 1) / G]);
    }
  };
  auto add = [&](int row, int col) {
    float f[V];
    norm_unpack<T, V>(held(row, col), f);
    if constexpr (V == 1) {
      const float d = f[0] - mean[0];
      s1 += d, q1 = fmaf(d, d, q1);
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int at = K == 1 ? i & 1 : G > 1 ? 2 * i / G : i;
        const f32x2 d = pair_add(pair_of(f[2 * i], f[2 * i + 1]), less[i]);
        s[at] = pair_add(s[at], d);
        q[at] = pair_fma(d, d, q[at]);
      }
    }
  };
  auto end = [&](float inv) {            // 1 / N
    auto join = [&](int k, float u, float v) {
      m2[k] += fmaxf(fmaf(-u * inv, u, v), 0.f);
      mean[k] = fmaf(u, inv, mean[k]);
    };
    if constexpr (V == 1) {
      join(0, s1, q1);
    } else if constexpr (K == 1) {
      float u[4], v[4];
      pair_split(s[0], u[0], u[1]), pair_split(s[1], u[2], u[3]), pair_split(q[0], v[0], v[1]), pair_split(q[1], v[2], v[3]);
      join(0, (u[0] + u[1]) + (u[2] + u[3]), (v[0] + v[1]) + (v[2] + v[3]));
    } else {
#pragma unroll
      for (int i = 0; i < A; ++i) {
        float u[2], v[2];
        pair_split(s[i], u[0], u[1]), pair_split(q[i], v[0], v[1]);
        if constexpr (G > 1) join(i, u[0] + u[1], v[0] + v[1]);
        else join(2 * i, u[0], v[0]), join(2 * i + 1, u[1], v[1]);
      }
    }
  };
  const int mine = active ? full + ((WIDE ? tid : ty) < more ? 1 : 0) : 0;     // accesses of this thread
  if constexpr (WIDE) {
    for (int done = 0, col = tid, row = 0; done < mine;) {
      const int last = mine - done > kRun ? done + kRun : mine;
      begin();
      for (; done < last; ++done, col += NT) {
        while (col >= p.sv) col -= p.sv, ++row;
        add(row, col);
      }
      end(1.f / ((float)done * (float)G));
    }
  } else {
    for (int done = 0, row = ty; done < mine;) {
      const int last = mine - done > kRun ? done + kRun : mine;
      begin();
#pragma unroll 4
      for (; done < last; ++done, row += ty_n) add(row, col0);
      end(1.f / ((float)done * (float)G));
    }
  }
  // (mean, squares) of the thread's K columns; of a warp's, about the mean of its first pixel's thread; of a group, by one warp over the rows of red
  {
    const float n = (float)mine * (float)G;
    const float n_row = WIDE || by_warp ? count_of_row(warp) : n, inv_row = n_row > 0.f ? 1.f / n_row : 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float mu = mean[k], m = m2[k];
      if (WIDE || by_warp) {
        const int stride = WIDE ? 1 : p.sv, others = WIDE ? 32 : warp_rows;
        const float ref = __shfl_sync(0xffffffffu, mu, col0 & 31), d = n > 0.f ? mu - (WIDE ? __shfl_sync(0xffffffffu, mu, 0) : ref) : 0.f;
        const float base = WIDE ? __shfl_sync(0xffffffffu, mu, 0) : ref;
        float td = n * d, tq = fmaf(n * d, d, n > 0.f ? m : 0.f);
        for (int left = others; left > 1;) {         // the pixels behind the half are added to those before it
          const int half = (left + 1) >> 1;
          const float od = __shfl_down_sync(0xffffffffu, td, half * stride), oq = __shfl_down_sync(0xffffffffu, tq, half * stride);
          if ((WIDE ? lane : lane_row) + half < left) td += od, tq += oq;
          left = half;
        }
        mu = fmaf(td, inv_row, base), m = fmaxf(fmaf(-td * inv_row, td, tq), 0.f);
        if (n_row == 0.f) mu = m = 0.f;
      } else if (n == 0.f) {
        mu = m = 0.f;
      }
      if (WIDE ? lane == 0 : by_warp ? lane < p.sv : active) red[red_row * p.bins + (WIDE ? 0 : col0 * K + k)] = make_float2(mu, m);
    }
  }
  __syncthreads();
  bool lost = false;
  if (cluster > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");    // every CTA's barrier is set up
  for (int g = warp; g < p.groups; g += NW) {
    auto over = [&](auto&& term) {       // the group's bins of every row, 32 at a time
      float s = 0.f;
      const float2* at = red + r_first * p.bins + g * per_group + b_first;
      for (int r = r_first, c = b_first; r < p.red_rows;) {
        s += term(count_of_row(r), *at);
        r += r_step, c += b_step, at += r_step * p.bins + b_step;
        if (c >= per_group) c -= per_group, ++r, at += p.bins - per_group;
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
      return s;
    };
    const float ref = red[g * per_group].x;          // a mean among them: what all are equal to comes out as that
    const float mu = fmaf(over([&](float w, float2 v) { return w * (v.x - ref); }), inv_here, ref);
    const float squares = over([&](float w, float2 v) {
      const float d = v.x - mu;
      return fmaf(w * d, d, v.y);
    });
    if (cluster == 1) {
      if (lane == 0) all[g] = make_float2(mu, rsqrtf(fmaf(squares, inv_here, p.eps)));
    } else if (lane < (int)cluster) {
      asm volatile(
          "{\n .reg .b32 a, b;\n mapa.shared::cluster.u32 a, %0, %2;\n mapa.shared::cluster.u32 b, %1, %2;\n"
          " st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [a], {%3, %4}, [b];\n}"
          ::"r"((uint32_t)__cvta_generic_to_shared(stat + g * (int)cluster + (int)rank)), "r"(arrived), "r"(lane), "f"(mu), "f"(squares)
          : "memory");
    }
  }
  // The cluster's statistics.
  if (cluster > 1) {
    for (int g0 = warp * 2; g0 < p.groups; g0 += NW * 2) {      // sixteen lanes a group
      if (g0 == warp * 2 && !__all_sync(0xffffffffu, mbar_wait_cluster(arrived, 0, p.err_flag, p.wait_cycles))) lost = true;
      const int r = lane & 15, g = g0 + (lane >> 4);
      const float w = r < (int)cluster ? (float)max(0, min(p.rows, p.hw - r * p.rows)) * (float)p.cpg : 0.f;
      const float2 v = w > 0.f && g < p.groups ? stat[g * (int)cluster + r] : make_float2(0.f, 0.f);
      const float ref = __shfl_sync(0xffffffffu, v.x, lane & 16);      // of the first CTA, which is never empty
      float s = w > 0.f ? w * (v.x - ref) : 0.f;
#pragma unroll
      for (int d = 8; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
      const float mu = fmaf(s, inv_all, ref);
      s = w > 0.f ? fmaf(w * (v.x - mu), v.x - mu, v.y) : 0.f;
#pragma unroll
      for (int d = 8; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
      if (r == 0 && g < p.groups) all[g] = make_float2(mu, rsqrtf(fmaf(s, inv_all, p.eps)));
    }
  }
  if (__syncthreads_or(lost)) {            // a wait that ran out: the status says so, and y stays as it is
    cluster_drain(arrived, 0, p.err_flag);
    return;
  }
  // y = (x - mean) * (gamma / deviation) + beta
  const T* res = p.residual ? reinterpret_cast<const T*>(p.residual) + first : nullptr;
  T* y = reinterpret_cast<T*>(p.y) + first;
  // The mean is taken off first, for bf16 too: in the offset beta - mean * a it would leave 2^-24 of mean * gamma / deviation, which in a group that hardly varies is
  // more than the result's own rounding (0.018 for a constant 3008 at eps 1e-5, where the result is beta).
  float a[V], b[V];
  auto affine = [&](int col) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = channel + col * V + i;
      const float2 st = all[WIDE ? 0 : min((col * V + i) / p.cpg, p.groups - 1)];
      a[i] = p.gamma ? p.gamma[c] * st.y : st.y, b[i] = p.beta ? p.beta[c] : 0.f;
      if (i % G == 0) mean[i / G] = st.x;
    }
  };
  if (!WIDE && active) affine(col0);
  const NormClamp clamp(p.act);
  auto store = [&](auto act, auto with_residual) {
    constexpr bool SILU = decltype(act)::value;
    constexpr bool RES = decltype(with_residual)::value;
    auto finish = [&](size_t at, const Vec& held_x, const Vec& r) {
      float f[V], q[V];
      norm_unpack<T, V>(held_x, f);
      if (RES) norm_unpack<T, V>(r, q);
      if constexpr (V == 1) {
        float t = fmaf(f[0] - mean[0], a[0], b[0]);
        if (RES) t += q[0];
        Elem<T>::st(y + at, norm_act<SILU>(t, clamp));
      } else {
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const f32x2 d = pair_add(pair_of(f[2 * i], f[2 * i + 1]), pair_of(-mean[2 * i / G], -mean[(2 * i + 1) / G]));
          f32x2 t = pair_fma(d, pair_of(a[2 * i], a[2 * i + 1]), pair_of(b[2 * i], b[2 * i + 1]));
          if (RES) t = pair_add(t, pair_of(q[2 * i], q[2 * i + 1]));
          pair_split(t, f[2 * i], f[2 * i + 1]);
        }
        Vec16<T> o;
#pragma unroll
        for (int i = 0; i < V; ++i) o.v[i] = norm_act<SILU>(f[i], clamp);
        o.store(y + at);
      }
    };
    if constexpr (WIDE) {
      each([&](int row, int col) {
        affine(col);
        const size_t at = (size_t)row * p.c + col * V;
        Vec r;
        if (RES) r = *reinterpret_cast<const Vec*>(res + at);
        finish(at, held(row, col), r);
      });
    } else if (active) {
      // Four pixels' loads before the first one's store: y may be the residual or x, so the compiler keeps loads behind stores.
      constexpr int U = RES && !RESIDENT ? 2 : RES || !RESIDENT ? 4 : 1;
      for (int row = ty; row < rows; row += U * ty_n) {
        Vec h[U], r[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (row + u * ty_n < rows) {
            if (!RESIDENT) h[u] = held(row + u * ty_n, col0);
            if (RES) r[u] = *reinterpret_cast<const Vec*>(res + (size_t)(row + u * ty_n) * p.c + col0 * V);
          }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (row + u * ty_n < rows) finish((size_t)(row + u * ty_n) * p.c + col0 * V, RESIDENT ? held(row + u * ty_n, col0) : h[u], r[u]);
      }
    }
  };
  if (p.act == EE_ACT_SILU) {
    if (res) store(Flag<true>(), Flag<true>());
    else store(Flag<true>(), Flag<false>());
  } else {
    if (res) store(Flag<false>(), Flag<true>());
    else store(Flag<false>(), Flag<false>());
  }
}

template <typename T, int V, int K, bool WIDE, bool RESIDENT, int NT>
inline cudaError_t norm_launch_k(const NormPlan& pl, const NormArgs& a, long units, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * pl.cluster));
  cfg.blockDim = dim3(NT);
  cfg.dynamicSmemBytes = pl.smem();
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = pl.cluster, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pl.cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, group_norm_kernel<T, V, K, WIDE, RESIDENT, NT>, a);
}

template <typename T, int V, int K>
inline cudaError_t norm_launch_p(const NormPlan& pl, const NormArgs& a, long units, cudaStream_t st) {
  if (pl.threads == kNormMany) return norm_launch_k<T, V, K, false, false, kNormMany>(pl, a, units, st);
  return pl.threads == kNormFew ? norm_launch_k<T, V, K, false, true, kNormFew>(pl, a, units, st) : norm_launch_k<T, V, K, false, true, kNormThreads>(pl, a, units, st);
}

template <typename T, int V>
inline cudaError_t norm_launch_v(const NormPlan& pl, const NormArgs& a, long units, cudaStream_t st) {
  if (pl.wide) return pl.resident ? norm_launch_k<T, V, 1, true, true, kNormThreads>(pl, a, units, st) : norm_launch_k<T, V, 1, true, false, kNormMany>(pl, a, units, st);
  if (pl.parts == 1) return norm_launch_p<T, V, 1>(pl, a, units, st);
  if constexpr (V > 1)
    if (pl.parts == 2) return norm_launch_p<T, V, 2>(pl, a, units, st);
  if constexpr (V > 2)
    if (pl.parts == 4) return norm_launch_p<T, V, 4>(pl, a, units, st);
  if constexpr (V > 4) return norm_launch_p<T, V, 8>(pl, a, units, st);
  return cudaErrorInvalidValue;
}

// Whether a grid holds a call's blocks, and an int a CTA's accesses: the limit is 2^31 - 1.
inline bool norm_fits(const NormPlan& pl, long batch) {
  return batch * pl.slices * pl.cluster <= 0x7fffffffL && (long)pl.rows * pl.sv <= 0x7fffffffL - 4096 && pl.smem() <= kNormMaxSmem;
}

// Once per device, before the first launch.  What a kernel may ask for is the kernel's, not the launch's: a call that set it to its own need would lower it under
// the launch of another host thread.  Parts that are read again need no more than the 48 KB that every kernel has.
template <typename T, int V, int K, bool WIDE>
inline cudaError_t norm_allow() {
  cudaError_t e = cudaFuncSetAttribute(group_norm_kernel<T, V, K, WIDE, true, kNormThreads>, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormMaxSmem);
  if constexpr (!WIDE)
    if (e == cudaSuccess) e = cudaFuncSetAttribute(group_norm_kernel<T, V, K, false, true, kNormFew>, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormMaxSmem);
  return e;
}
inline cudaError_t norm_context_init() {
  cudaError_t e = norm_allow<bf16, 8, 1, false>();
  if (e == cudaSuccess) e = norm_allow<bf16, 8, 2, false>();
  if (e == cudaSuccess) e = norm_allow<bf16, 8, 4, false>();
  if (e == cudaSuccess) e = norm_allow<bf16, 8, 8, false>();
  if (e == cudaSuccess) e = norm_allow<bf16, 8, 1, true>();
  if (e == cudaSuccess) e = norm_allow<bf16, 1, 1, false>();
  if (e == cudaSuccess) e = norm_allow<bf16, 1, 1, true>();
  if (e == cudaSuccess) e = norm_allow<float, 4, 1, false>();
  if (e == cudaSuccess) e = norm_allow<float, 4, 2, false>();
  if (e == cudaSuccess) e = norm_allow<float, 4, 4, false>();
  if (e == cudaSuccess) e = norm_allow<float, 4, 1, true>();
  if (e == cudaSuccess) e = norm_allow<float, 1, 1, false>();
  if (e == cudaSuccess) e = norm_allow<float, 1, 1, true>();
  return e;
}

template <typename T>
inline cudaError_t norm_launch(const void* x, const void* residual, void* y, const float* gamma, const float* beta, float eps, long batch, int hw, int c,
                               int groups, int act, bool rev, int* err_flag, long long wait_cycles, cudaStream_t st) {
  const bool aligned = (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)y) & 15) == 0;
  const NormPlan pl = norm_plan(hw, c, groups, (int)sizeof(T), aligned);
  if (!norm_fits(pl, batch)) return cudaErrorInvalidValue;
  const NormArgs a = {x, residual, y, gamma, beta, eps, hw, c, c / groups, act, pl.sv, pl.slices, pl.groups, pl.rows, pl.chunk, pl.red_rows, pl.bins,
                      err_flag, wait_cycles, rev ? 1 : 0};
  const long units = batch * pl.slices;
  constexpr int V = Elem<T>::kVec;
  return pl.v > 1 ? norm_launch_v<T, V>(pl, a, units, st) : norm_launch_v<T, 1>(pl, a, units, st);
}

}  // namespace ee
