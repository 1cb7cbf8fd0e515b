// Class probabilities, and the verification of classes (tokens) that an early exit drafted against the probabilities of a later one.
//
// softmax: p[v] = exp((l[v] - max) / t) / sum, a row at a time.  Bound by memory: a logit read once, a probability written once, and not far behind by
// instructions, so the joins are kept off the threads' path.  A short row is one warp's, in registers.  A long one is cut over a cluster of
// CTAs, up to six of which share an SM so that one's loads run beside another's barriers.  A CTA fetches its part into shared memory, takes its maximum and the sum of the
// exponentials against that, sends both to the other CTAs, and writes exp((l - max) / t) / sum once it has theirs.  Rows of any length and any alignment: whole 16-byte
// words are fetched, the odd elements in front of and behind them one by one (one element a lane takes 4 us for 32 of them: 2-byte loads); exponentials are taken and
// probabilities leave one element a lane, 128 bytes a warp, so that the order of the sum does not follow the row's alignment.  How a row is cut follows from its length
// alone, so its bits do not depend on the other rows.  320 x 128001 bf16: 50.8 us, 4.8 TB/s; fp32 73.7, 4.4; 64 x 1000 fp32: 1.8 us.  An SM issues 60 % of the
// time; of the 17 cycles from one issue of a warp to its next 3.9 are barriers, 4.2 shared memory, 2.1 loads: fetch, maximum, sum and stores of a part
// follow one another, and six CTAs cover them in part.
//
// verify: draft i of a sequence is accepted while u_i q_i(x_i) < p_i(x_i); at the first rejection a token is drawn from max(p_i - q_i, 0), where
// all hold from the row behind the last draft, as the first v whose running sum exceeds r times the total.  What is compared is exact: u q in fp64 is the
// exact product of two floats, and the sums are fp64, because a draw must not depend on how a sum over a hundred thousand floats was grouped
// (2^-53 against steps of about 1e-5).  It reads one row of p and one of q per sequence: which row it is (two dependent loads), then the sums of blocks of
// 512 values, all CTAs of 64 sequences side by side; the CTAs send each other their totals, and the one in whose part the sum crosses scans its block sums
// and then that one block.  64 sequences of 5 drafts, 128001 tokens: 21.8 us, 3.0 TB/s of the two rows that are read, of which the dependent loads, the exchange and the scan are
// about half (an SM issues 42 % of the time; loads and barriers are 4.4 and 3.7 of a warp's 14.6 cycles an issue); certain drafts 20.2; one sequence of 1000: 5.7 us.
#pragma once
#include <float.h>

#include "common.cuh"
#include "conv_tc.cuh"

namespace ee {

// ----------------------------------------------------------------------------- softmax

constexpr int kSmWarpMost = 1024;        // longest row of the one-warp form: 32 values a lane
constexpr int kSmThreads = 256;
constexpr int kSmPart = 16384;           // elements of a CTA's part that a cluster is cut for: six CTAs an SM (fp32: three)
constexpr int kSmMaxCluster = 16;        // above eight, the portable size, the kernel asks
constexpr int kSmMaxPart = 38400;        // elements that a CTA has room for

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
  return v;
}
template <typename F>
__device__ __forceinline__ F warp_total(F v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// A row's temperature: heat > 0 divides; anything else puts the whole mass on the first of the largest logits.
// weight = exp((l - top) / t) as 2^((l / 2 - top / 2) c), c = 2 log2(e) / t.  The difference is taken first: the largest logit weighs exactly 1 however cold the row; and
// of halves, in one multiply-add, which is exact where l - top is and does not overflow where that does (logits of -3e38 and 3e38 in a hot row).
// c is kept finite, so that 0 * c is 0, and above 0, so that a masked logit (-inf) weighs nothing however hot: at t = inf, where it is 2^-149, a weight is off by
// 3.4e38 * 2^-149 * ln 2 = 3.3e-7 (5.6 u) at most, and where c is below 2^-126 by the rounding of c, half of that.  NaN and +inf make NaN.  Off by 2 u |l - top| / t of the
// product's two roundings and 2 units of the power; what is below 2^-126 is 0.
struct SmScale {
  float c;
  bool greedy;
  __device__ __forceinline__ SmScale(const float* heat, long row) : c(2.f * 1.4426950408889634f), greedy(false) {
    if (heat) {
      const float t = heat[row];
      greedy = !(t > 0.f);
      c = fmaxf(fminf(2.f * 1.4426950408889634f / t, FLT_MAX), __int_as_float(1));
    }
  }
  __device__ __forceinline__ float weight(float l, float top) const {
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fmaf(l, 0.5f, -0.5f * top) * c));
    return e;
  }
  // What the weights of a part are taken from: its maximum, or any number where everything is masked.
  __device__ __forceinline__ static float base(float top) { return top == -INFINITY ? 0.f : top; }
};

// Nothing that is read here is __restrict__: the kernel starts while the one in front, which may write it, still runs.
template <typename T, int N>   // N values a lane
__global__ void __launch_bounds__(128)
softmax_warp_kernel(const T* x, const float* heat, float* y, long rows, int n) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const long row = (long)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (row >= rows) return;
  const T* src = x + (size_t)row * n;
  float v[N], top = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lane + 32 * i < n ? Elem<T>::ld(src + lane + 32 * i) : -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) top = fmaxf(top, v[i]);
  top = warp_max(top);
  const SmScale sc(heat, row);
  float* dst = y + (size_t)row * n;
  float s = 0.f;
  if (sc.greedy) {
    int at = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (v[i] == top && lane + 32 * i < at) at = lane + 32 * i;
      s += v[i] != v[i] ? v[i] : 0.f;                      // NaN wherever the row has one
    }
    at = __reduce_min_sync(0xffffffffu, at);
    s = warp_total(s) + (top == INFINITY ? NAN : 0.f);
    const float hit = top == -INFINITY ? s : 1.f + s;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (lane + 32 * i < n) dst[lane + 32 * i] = lane + 32 * i == at ? hit : s;
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = sc.weight(v[i], SmScale::base(top));
    s += v[i];
  }
  s = warp_total(s);
  const float scale = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (lane + 32 * i < n) dst[lane + 32 * i] = v[i] * scale;
}

// (maximum, sum, first place of it) of a warp, of a CTA, of the row.
struct SmJoin {
  float top, sum, at;
};
__device__ __forceinline__ SmJoin sm_join(const SmScale& sc, SmJoin v) {   // over the warp; lanes without a part pass (-inf, 0, far)
  float top = v.top;
#pragma unroll
  for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  if (!sc.greedy) v.sum *= v.top == -INFINITY ? (v.sum == 0.f ? 0.f : 1.f) : sc.weight(v.top, top);   // a part that is masked throughout adds 0, or its NaN
  if (v.top != top) v.at = 1e9f;
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    v.sum += __shfl_xor_sync(0xffffffffu, v.sum, d);
    v.at = fminf(v.at, __shfl_xor_sync(0xffffffffu, v.at, d));
  }
  v.top = top;
  return v;
}

// Largest of the 16-byte words of a part; bf16 two at a time.
template <typename T>
__device__ __forceinline__ float sm_word_max(uint4 w, float top) {
  if constexpr (sizeof(T) == 2) {
    __nv_bfloat162 a, b;
    *reinterpret_cast<uint32_t*>(&a) = w.x, *reinterpret_cast<uint32_t*>(&b) = w.y;
    __nv_bfloat162 m = __hmax2(a, b);
    *reinterpret_cast<uint32_t*>(&a) = w.z, *reinterpret_cast<uint32_t*>(&b) = w.w;
    m = __hmax2(m, __hmax2(a, b));
    return fmaxf(top, fmaxf(__low2float(m), __high2float(m)));
  } else {
    return fmaxf(fmaxf(top, fmaxf(__uint_as_float(w.x), __uint_as_float(w.y))), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
  }
}

// per: elements of a CTA's part (the last one's is shorter, or empty).
template <typename T>
__global__ void __launch_bounds__(kSmThreads, 7)
softmax_cluster_kernel(const T* x, const float* heat, float* y, int n, int per, int* err_flag, long long wait_cycles) {
  constexpr int NW = kSmThreads / 32;
  extern __shared__ __align__(16) uint8_t sm_smem[];
  __shared__ float tops[NW];
  __shared__ SmJoin warps[NW], row_join;
  __shared__ __align__(16) float4 parts[kSmMaxCluster];     // of every CTA
  __shared__ uint64_t bar;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t rank, cluster;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
  const uint32_t arrived = smem_u32(&bar);
  if (cluster > 1) {
    if (tid == 0) {
      mbar_init(arrived, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      mbar_expect_tx(arrived, cluster * 16u);
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  }
  const long row = blockIdx.x / cluster;
  const int i0 = min((int)rank * per, n), cnt = min(per, n - i0);
  const T* src = x + (size_t)row * n + i0;
  float* dst = y + (size_t)row * n + i0;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // Shared memory keeps the logits at their own offset within a 16-byte word: whole words arrive by cp.async, what is in front and behind alone.
  constexpr int W = 16 / (int)sizeof(T);
  const int skew = (int)(((uintptr_t)src & 15) / sizeof(T));
  T* part = reinterpret_cast<T*>(sm_smem) + skew;
  const int head = min(cnt, skew ? W - skew : 0), words = (cnt - head) / W, tail = head + words * W;
#pragma unroll 4
  for (int i = tid; i < words; i += kSmThreads)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(part + head + i * W)), "l"(src + head + (size_t)i * W) : "memory");
  cp_async_commit();
  float top = -INFINITY;
  if (tid < head) part[tid] = src[tid], top = Elem<T>::ld(part + tid);
  if (tid < cnt - tail) part[tail + tid] = src[tail + tid], top = fmaxf(top, Elem<T>::ld(part + tail + tid));
  const SmScale sc(heat, row);
  cp_async_wait<0>();
  // the words that this thread fetched are here
#pragma unroll 4
  for (int i = tid; i < words; i += kSmThreads) top = sm_word_max<T>(*reinterpret_cast<const uint4*>(part + head + i * W), top);
  top = warp_max(top);
  if (lane == 0) tops[warp] = top;
  if (cluster > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");      // every CTA's barrier is set up
  __syncthreads();                                                                  // and everybody's words are here
  top = tops[lane & (NW - 1)];
#pragma unroll
  for (int d = NW / 2; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  SmJoin mine = {top, 0.f, 1e9f};         // places up to 2^24 are exact in a float: rows are shorter
  if (sc.greedy) {
    for (int i = tid; i < cnt; i += kSmThreads) {
      const float v = Elem<T>::ld(part + i);
      if (v == top) mine.at = fminf(mine.at, (float)(i0 + i));
      mine.sum += v != v || v == INFINITY ? NAN : 0.f;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) mine.at = fminf(mine.at, __shfl_xor_sync(0xffffffffu, mine.at, d));
  } else {
    const float base = SmScale::base(top);
#pragma unroll 8
    for (int i = tid; i < cnt; i += kSmThreads) mine.sum += sc.weight(Elem<T>::ld(part + i), base);
  }
  mine.sum = warp_total(mine.sum);
  if (lane == 0) warps[warp] = mine;
  __syncthreads();
  bool lost = false;
  if (warp == 0) {
    SmJoin all = sm_join(sc, lane < NW ? warps[lane] : SmJoin{-INFINITY, 0.f, 1e9f});
    if (cluster > 1) {
      if (lane < (int)cluster)
        asm volatile(
            "{\n .reg .b32 a, b;\n mapa.shared::cluster.u32 a, %0, %2;\n mapa.shared::cluster.u32 b, %1, %2;\n"
            " st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [a], {%3, %4, %5, %4}, [b];\n}"
            ::"r"(smem_u32(&parts[rank])), "r"(arrived), "r"(lane), "f"(all.top), "f"(all.sum), "f"(all.at)
            : "memory");
      lost = !__all_sync(0xffffffffu, mbar_wait_cluster(arrived, 0, err_flag, wait_cycles));
      const float4 o = lane < (int)cluster ? parts[lane] : make_float4(-INFINITY, 0.f, 1e9f, 0.f);
      all = sm_join(sc, SmJoin{o.x, o.y, o.z});
    }
    if (!sc.greedy && lane == 0) all.sum = all.sum == 0.f ? 0.f : 1.f / all.sum;
    if (lane == 0) row_join = all;
  }
  if (__syncthreads_or(lost)) {            // the status says so, and y stays as it is
    cluster_drain(arrived, 0, err_flag);
    return;
  }
  const SmJoin all = row_join;
  if (sc.greedy) {
    const float hit = all.top == -INFINITY ? all.sum : 1.f + all.sum;      // the sum is 0, or NaN
    for (int i = tid; i < cnt; i += kSmThreads) dst[i] = (float)(i0 + i) == all.at ? hit : all.sum;
  } else {
    const float base = SmScale::base(all.top);
#pragma unroll 8
    for (int i = tid; i < cnt; i += kSmThreads) dst[i] = sc.weight(Elem<T>::ld(part + i), base) * all.sum;
  }
}

constexpr int kSmMost = kSmMaxCluster * kSmMaxPart;     // longest row that softmax takes

template <typename T>
inline size_t softmax_smem(int per) { return align_up((size_t)per * sizeof(T) + 16, 16); }

// Once per device, before the first launch: set by a launch to its own need, it would be lowered under the launch of another host thread.
inline cudaError_t softmax_context_init() {
  cudaError_t e = cudaSuccess;
  auto set = [&](auto kernel, size_t bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  };
  set(softmax_cluster_kernel<bf16>, softmax_smem<bf16>(kSmMaxPart));
  set(softmax_cluster_kernel<float>, softmax_smem<float>(kSmMaxPart));
  return e;
}

template <typename T>
inline cudaError_t softmax_launch(const T* x, const float* heat, float* y, long rows, int n, int* err_flag, long long wait_cycles, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (n <= kSmWarpMost) {
    cfg.gridDim = dim3((unsigned)((rows + 3) / 4));
    cfg.blockDim = dim3(128);
    if (n <= 128) return cudaLaunchKernelEx(&cfg, softmax_warp_kernel<T, 4>, x, heat, y, rows, n);
    return cudaLaunchKernelEx(&cfg, softmax_warp_kernel<T, 32>, x, heat, y, rows, n);
  }
  int cluster = 1;
  while (cluster < 8 && cdiv(n, cluster) > kSmPart) cluster *= 2;
  if (cdiv(n, cluster) > kSmMaxPart) cluster *= 2;
  const int per = cdiv(n, cluster);
  cfg.gridDim = dim3((unsigned)(rows * cluster));
  cfg.blockDim = dim3(kSmThreads);
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  cfg.dynamicSmemBytes = softmax_smem<T>(per);
  return cudaLaunchKernelEx(&cfg, softmax_cluster_kernel<T>, x, heat, y, n, per, err_flag, wait_cycles);
}

// ----------------------------------------------------------------------------- verification of drafts

constexpr int kVfThreads = 256, kVfWarps = kVfThreads / 32;
constexpr int kVfMaxCluster = 8;
constexpr int kVfPart = 8192;             // values of a CTA's part of a row that a cluster is cut for
constexpr int kVfBlocks = 1024;           // blocks of a part, at most

struct VerifyArgs {
  const float* p;          // [batch][k + 1][n]
  const float* q;          // [batch][k][n], or null: a draft was certain
  const int32_t* drafts;   // [batch][k]
  const float* u;          // [batch][k]
  const float* r;          // [batch]
  const int32_t* n_draft;  // [batch], or null: k
  int32_t* tokens;         // [batch][k + 1]
  int32_t* accepted;       // [batch]
  int k, n, per, block;    // values of a CTA's part, of a block (a multiple of 512)
  int* err_flag;
  long long wait_cycles;   // limit of the waits for the cluster's totals
};

// The weight of one value: what the draw goes by.  Values that are not positive and finite weigh nothing.
__device__ __forceinline__ double verify_weight(float p, float q) {
  return p > q && p < INFINITY && q > -INFINITY ? (double)p - (double)q : 0.0;     // compared as floats: fp64 comparisons took 33 us in place of 20 for 64 rows of 128001
}

__device__ __forceinline__ double warp_scan(double v, int lane) {   // inclusive
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const double o = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += o;
  }
  return v;
}

__global__ void __launch_bounds__(kVfThreads, 4)
verify_drafts_kernel(VerifyArgs a) {
  __shared__ int s_got, s_count, s_next;
  __shared__ double s_block[kVfBlocks], s_total[2][kVfMaxCluster];
  __shared__ uint64_t bars[2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t rank, cluster;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
  const uint32_t arrived = smem_u32(bars);
  if (cluster > 1) {
    if (tid == 0) {
      mbar_init(arrived, 1), mbar_init(arrived + 8, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      mbar_expect_tx(arrived, cluster * 8u), mbar_expect_tx(arrived + 8, cluster * 8u);
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  }
  const long b = blockIdx.x / cluster;
  const size_t n = (size_t)a.n;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // every CTA of the cluster decides for itself how many drafts hold
  if (warp == 0) {
    const int count = a.n_draft ? min(a.n_draft[b], a.k) : a.k;
    int got = max(count, 0);
    for (int i0 = 0; i0 < a.k; i0 += 32) {
      bool no = false;
      const int at = i0 + lane;
      if (at < a.k) {
        const size_t i = (size_t)b * a.k + at;
        const int t = a.drafts[i];                                 // not behind the count's load
        const float u = a.u[i];
        no = t < 0 || t >= a.n;            // not a class: nothing is read for it, and it is rejected
        if (at < count && !no) no = !((double)u * (a.q ? (double)a.q[i * n + t] : 1.0) < (double)a.p[((size_t)b * (a.k + 1) + at) * n + t]);
        no = no && at < count;
      }
      const unsigned m = __ballot_sync(0xffffffffu, no);
      if (m) {
        got = i0 + __ffs(m) - 1;
        break;
      }
    }
    if (lane == 0) s_got = got, s_count = count;
  }
  if (cluster > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");      // every CTA's barriers are set up
  __syncthreads();
  const int got = s_got, count = s_count;
  if (count < 0) return;                   // an empty place of a padded batch (all CTAs of its cluster): left as it is
  const int i0 = (int)min((long)rank * a.per, (long)a.n), cnt = min(a.per, a.n - i0);
  const float* p = a.p + ((size_t)b * (a.k + 1) + got) * n + i0;
  const float* q = got < count && a.q ? a.q + ((size_t)b * a.k + got) * n + i0 : nullptr;
  const int struck = got < count && !a.q ? a.drafts[(size_t)b * a.k + got] - i0 : -1;   // a certain draft that did not hold: everything but it is left
  const int blocks = (cnt + a.block - 1) / a.block;
  // The second round, where p - q leaves nothing, draws from p itself.
  for (int round = 0; round < 2; ++round) {
    auto weight = [&](int i) {
      const float v = p[i], less = q && round == 0 ? q[i] : 0.f;
      return i == struck && round == 0 ? 0.0 : verify_weight(v, less);
    };
    for (int k = warp; k < blocks; k += kVfWarps) {
      const int end = min((k + 1) * a.block, cnt);
      double s = 0.0;
      for (int i = k * a.block + lane; i < end; i += 512) {
        float v[16], less[16];             // all on their way before the first is needed
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const bool in = i + 32 * j < end;
          v[j] = in ? p[i + 32 * j] : 0.f;
          less[j] = in && q && round == 0 ? q[i + 32 * j] : 0.f;
          if (round == 0 && i + 32 * j == struck) v[j] = 0.f;
        }
        double w[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j & 3] += verify_weight(v[j], less[j]);
        s += (w[0] + w[1]) + (w[2] + w[3]);
      }
      s = warp_total(s);
      if (lane == 0) s_block[k] = s;
    }
    __syncthreads();
    if (warp == 0) {
      double mine = 0.0;
      for (int k = 0; k < blocks; k += 32) mine += warp_total(k + lane < blocks ? s_block[k + lane] : 0.0);
      bool ok = true;
      double before = 0.0, total = mine;
      int last = (int)rank;                // the last CTA whose part weighs anything
      if (cluster > 1) {
        const uint32_t here = arrived + 8u * round;
        if (lane < (int)cluster)
          asm volatile(
              "{\n .reg .b32 a, b;\n mapa.shared::cluster.u32 a, %0, %2;\n mapa.shared::cluster.u32 b, %1, %2;\n"
              " st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [a], %3, [b];\n}"
              ::"r"(smem_u32(&s_total[round][rank])), "r"(here), "r"(lane), "l"(__double_as_longlong(mine))
              : "memory");
        ok = __all_sync(0xffffffffu, mbar_wait_cluster(here, 0, a.err_flag, a.wait_cycles));
        total = 0.0;
        for (int c = 0; c < (int)cluster; ++c) {
          const double o = s_total[round][c];
          if (c == (int)rank) before = total;
          if (o > 0.0) last = c;
          total += o;
        }
      }
      const bool again = ok && !(total > 0.0) && round == 0 && got < count;
      const double goal = fmax((double)a.r[b] * total, 0.0);
      // The CTA in whose part the running sum passes the goal; where rounding leaves it unpassed, the last one that weighs anything.
      const bool here = total > 0.0 ? mine > 0.0 && before <= goal && (before + mine > goal || last == (int)rank) : rank == 0;
      if (ok && !again && here) {
        int token = -1;                    // nothing weighs anything: no token
        if (total > 0.0) {
          // the block, then the 32 values in which the sum crosses; or the last that weigh anything
          int at = -1;
          double run = before, start = before;
          for (int k = 0; k < blocks; k += 32) {
            const double w = k + lane < blocks ? s_block[k + lane] : 0.0, cum = run + warp_scan(w, lane);
            const unsigned over = __ballot_sync(0xffffffffu, w > 0.0 && cum > goal), some = __ballot_sync(0xffffffffu, w > 0.0);
            const int j = over ? __ffs(over) - 1 : 31 - __clz(some);
            if (some) at = k + j, start = __shfl_sync(0xffffffffu, cum - w, j);
            if (over) break;
            run = __shfl_sync(0xffffffffu, cum, 31);
          }
          const int end = min((at + 1) * a.block, cnt);
          bool found = false;
          for (int i = at * a.block + lane; i - lane < end && !found; i += 256) {
            double w[8], cum[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = i + 32 * j < end ? weight(i + 32 * j) : 0.0;
#pragma unroll
            for (int j = 0; j < 8; ++j) cum[j] = warp_scan(w[j], lane);      // side by side; the running sum goes on top
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const double passed = start + cum[j];
              const unsigned over = __ballot_sync(0xffffffffu, w[j] > 0.0 && passed > goal), some = __ballot_sync(0xffffffffu, w[j] > 0.0);
              if (!found && some) token = i0 + i - lane + 32 * j + (over ? __ffs(over) - 1 : 31 - __clz(some));
              found = found || over != 0;
              start += __shfl_sync(0xffffffffu, cum[j], 31);
            }
          }
        }
        int32_t* out = a.tokens + (size_t)b * (a.k + 1);
        for (int i = lane; i <= a.k; i += 32) out[i] = i < got ? a.drafts[(size_t)b * a.k + i] : i == got ? token : -1;
        if (lane == 0) a.accepted[b] = got;
      }
      if (lane == 0) s_next = ok ? again : 2;
    }
    __syncthreads();
    if (s_next != 1) {
      if (s_next == 2) cluster_drain(arrived + 8u * round, 0, a.err_flag);      // the status says so, and where the token would have been of this part, the outputs stay as they are
      break;
    }
  }
}

inline cudaError_t verify_launch(VerifyArgs a, long batch, cudaStream_t st) {
  int cluster = 1;
  while (cluster < kVfMaxCluster && cdiv(a.n, cluster) > kVfPart) cluster *= 2;
  a.per = cdiv(a.n, cluster);
  a.block = 512 * cdiv(a.per, 512L * kVfBlocks);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(batch * cluster));
  cfg.blockDim = dim3(kVfThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, verify_drafts_kernel, a);
}

}  // namespace ee
