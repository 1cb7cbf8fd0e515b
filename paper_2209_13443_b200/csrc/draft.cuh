// Class probabilities, and the verification of classes (tokens) that an early exit drafted against the probabilities of a later one.
//
// softmax: p[v] = exp((l[v] - max) / t) / sum, a row at a time.  Bound by memory: a logit read once, a probability written once.  A short row is one
// warp's, in registers; a long one is cut over a cluster of up to eight CTAs, each of which holds its part in shared memory between the maximum,
// the sum and the quotient, and the CTAs exchange maximum and sum through distributed shared memory.  Rows of any length and any alignment: the
// part is fetched in whole 16-byte words, the odd elements in front of and behind them one by one, and probabilities leave one per lane, 128 bytes a warp.
// How a row is cut follows from its length alone, so its bits do not depend on the other rows.
//
// verify: draft i of a sequence is accepted while u_i q_i(x_i) < p_i(x_i); at the first rejection a token is drawn from max(p_i - q_i, 0), where
// all hold from the row behind the last draft, as the first v whose running sum exceeds r times the total.  What is compared is exact: u q in fp64 is the
// exact product of two floats, and the sums are fp64, because a draw must not depend on how a sum over a hundred thousand floats was grouped
// (2^-53 against steps of about 1e-5).  It reads one row of p and one of q per sequence, so it is latency: which row it is (two dependent
// loads), the row's part sums, the exchange of the CTAs' totals, and the search inside the one stretch of 32 x 32 where the sum crosses.
#pragma once
#include <float.h>

#include "common.cuh"
#include "conv_tc.cuh"

namespace ee {

// ----------------------------------------------------------------------------- softmax

constexpr int kSmWarpMost = 1024;        // longest row of the one-warp form: 32 values a lane
constexpr int kSmThreads = 512;
constexpr int kSmChunk = 64 << 10;       // bytes of a CTA's part of a row that a cluster is cut for
constexpr int kSmMaxCluster = 8;
constexpr int kSmMaxChunk = 200 << 10;

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

// A row's temperature: heat > 0 scales by 1 / heat; anything else puts the whole mass on the first of the largest logits.
struct SmScale {
  float inv;
  bool greedy;
  __device__ __forceinline__ SmScale(const float* heat, long row) : inv(1.f), greedy(false) {
    if (heat) {
      const float t = heat[row];
      greedy = !(t > 0.f);
      inv = fminf(1.f / t, FLT_MAX);   // a denormal temperature must leave 0 * inv = 0 for the largest logit
    }
  }
  // exp((l - top) / t); a masked logit (-inf) weighs nothing, also where the whole row is masked.  NaN and +inf make NaN.
  __device__ __forceinline__ float weight(float l, float top) const { return l == -INFINITY ? 0.f : expf((l - top) * inv); }
};

template <typename T, int N>   // N values a lane
__global__ void __launch_bounds__(128)
softmax_warp_kernel(const T* x, const float* __restrict__ heat, float* y, long rows, int n) {
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
    v[i] = sc.weight(v[i], top);
    s += v[i];
  }
  s = warp_total(s);
  const float scale = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (lane + 32 * i < n) dst[lane + 32 * i] = v[i] * scale;
}

struct SmMax { __device__ float operator()(float a, float b) const { return fmaxf(a, b); } };
struct SmSum { __device__ float operator()(float a, float b) const { return a + b; } };

// Joins a value over the threads of the CTA; buf: one float per warp.  Every thread gets the result.
template <typename Op>
__device__ __forceinline__ float block_join(float v, float* buf, Op op) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
  __syncthreads();                        // buf may still be read from the call before
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = buf[threadIdx.x & (kSmThreads / 32 - 1)];
#pragma unroll
  for (int d = kSmThreads / 64; d; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
  return v;
}
// The same over the cluster; word: this CTA's slot, which the others read.  Every call has a slot of its own, so one barrier a call is enough.
template <typename Op>
__device__ __forceinline__ float cluster_join(float v, float* word, uint32_t cluster, Op op) {
  if (cluster == 1) return v;
  if (threadIdx.x == 0) *word = v;
  asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
  const uint32_t at = smem_u32(word);
  for (uint32_t r = 0; r < cluster; ++r) {
    uint32_t from;
    float o;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(at), "r"(r));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o) : "r"(from) : "memory");
    v = r == 0 ? o : op(v, o);
  }
  return v;
}

// per: elements of a CTA's part (the last one's is shorter, or empty).
template <typename T>
__global__ void __launch_bounds__(kSmThreads)
softmax_cluster_kernel(const T* x, const float* __restrict__ heat, float* y, int n, int per) {
  extern __shared__ __align__(16) uint8_t sm_smem[];
  __shared__ float buf[kSmThreads / 32], word[3];
  const int tid = threadIdx.x;
  uint32_t rank, cluster;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
  const long row = blockIdx.x / cluster;
  const int i0 = min((int)rank * per, n), cnt = min(per, n - i0);
  const T* src = x + (size_t)row * n + i0;
  float* dst = y + (size_t)row * n + i0;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // Shared memory keeps the part at its own offset within a 16-byte word: whole words arrive by cp.async, what is in front and behind alone.
  constexpr int W = 16 / (int)sizeof(T);
  const int skew = (int)(((uintptr_t)src & 15) / sizeof(T));
  T* part = reinterpret_cast<T*>(sm_smem) + skew;
  const int head = min(cnt, skew ? W - skew : 0), words = (cnt - head) / W, tail = head + words * W;
  for (int i = tid; i < words; i += kSmThreads)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(part + head + i * W)), "l"(src + head + (size_t)i * W) : "memory");
  cp_async_commit();
  if (tid < head) part[tid] = src[tid];
  if (tid < cnt - tail) part[tail + tid] = src[tail + tid];
  cp_async_wait<0>();
  __syncthreads();
  const SmScale sc(heat, row);
  float top = -INFINITY;
  for (int i = tid; i < words; i += kSmThreads) {
    Vec16<T> v;
    v.load(part + head + i * W);
#pragma unroll
    for (int k = 0; k < W; ++k) top = fmaxf(top, v.v[k]);
  }
  if (tid < head) top = fmaxf(top, Elem<T>::ld(part + tid));
  if (tid < cnt - tail) top = fmaxf(top, Elem<T>::ld(part + tail + tid));
  top = cluster_join(block_join(top, buf, SmMax()), &word[0], cluster, SmMax());
  float s = 0.f;
  if (sc.greedy) {
    float at = 1e9f;      // positions up to 2^24 are exact in a float: rows are shorter (kSmMaxChunk)
    for (int i = tid; i < cnt; i += kSmThreads) {
      const float v = Elem<T>::ld(part + i);
      if (v == top) at = fminf(at, (float)(i0 + i));
      s += v != v ? v : 0.f;
    }
    s = cluster_join(block_join(s, buf, SmSum()), &word[1], cluster, SmSum()) + (top == INFINITY ? NAN : 0.f);
    at = -cluster_join(block_join(-at, buf, SmMax()), &word[2], cluster, SmMax());
    const float hit = top == -INFINITY ? s : 1.f + s;
    for (int i = tid; i < cnt; i += kSmThreads) dst[i] = (float)(i0 + i) == at ? hit : s;
  } else {
    // one element after the other, not in 16-byte words: the order of the sum must not follow the row's alignment
#pragma unroll 4
    for (int i = tid; i < cnt; i += kSmThreads) s += sc.weight(Elem<T>::ld(part + i), top);
    s = cluster_join(block_join(s, buf, SmSum()), &word[1], cluster, SmSum());
    const float scale = s == 0.f ? 0.f : 1.f / s;
#pragma unroll 4
    for (int i = tid; i < cnt; i += kSmThreads) dst[i] = sc.weight(Elem<T>::ld(part + i), top) * scale;
  }
  // a CTA may leave once the others have read its words
  if (cluster > 1) asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}

// Longest row that softmax takes.
template <typename T> inline long softmax_most() { return (long)kSmMaxCluster * (kSmMaxChunk / (int)sizeof(T)); }

template <typename T>
inline cudaError_t softmax_launch(const T* x, const float* heat, float* y, long rows, int n, cudaStream_t st) {
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
  while (cluster < kSmMaxCluster && (long)cdiv(n, cluster) * (long)sizeof(T) > kSmChunk) cluster *= 2;
  const int per = cdiv(n, cluster);
  const int smem = (int)align_up((size_t)per * sizeof(T) + 16, 16);
  if (smem > 48 << 10) {
    const cudaError_t e = cudaFuncSetAttribute(softmax_cluster_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
  }
  cfg.gridDim = dim3((unsigned)(rows * cluster));
  cfg.blockDim = dim3(kSmThreads);
  cfg.dynamicSmemBytes = smem;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, softmax_cluster_kernel<T>, x, heat, y, n, per);
}

// ----------------------------------------------------------------------------- verification of drafts

constexpr int kVfThreads = 512, kVfWarps = kVfThreads / 32;
constexpr int kVfMaxCluster = 8;
constexpr int kVfPart = 8192;             // values of a CTA's part of a row that a cluster is cut for

struct VerifyArgs {
  const float* p;          // [batch][k + 1][n]
  const float* q;          // [batch][k][n], or null: a draft was certain
  const int32_t* drafts;   // [batch][k]
  const float* u;          // [batch][k]
  const float* r;          // [batch]
  const int32_t* n_draft;  // [batch], or null: k
  int32_t* tokens;         // [batch][k + 1]
  int32_t* accepted;       // [batch]
  int k, n, per;           // per: values of a CTA's part
};

// The weight of one value: what the draw goes by.  Values that are not positive and finite weigh nothing.
__device__ __forceinline__ double verify_weight(float p, float q) {
  const double w = (double)p - (double)q;
  return w > 0.0 && p < INFINITY ? w : 0.0;
}

__global__ void __launch_bounds__(kVfThreads)
verify_drafts_kernel(VerifyArgs a) {
  __shared__ int s_got, s_count;
  __shared__ double s_warp[kVfWarps], s_total[2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t rank, cluster;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
  const long b = blockIdx.x / cluster;
  const size_t n = (size_t)a.n;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // every CTA of the cluster decides for itself how many drafts hold
  if (warp == 0) {
    const int count = a.n_draft ? min(a.n_draft[b], a.k) : a.k;
    int got = max(count, 0);
    for (int i0 = 0; i0 < count; i0 += 32) {
      bool no = false;
      if (i0 + lane < count) {
        const size_t i = (size_t)b * a.k + i0 + lane;
        const int t = a.drafts[i];
        no = t < 0 || t >= a.n;            // not a class: nothing is read for it, and it is rejected
        if (!no) no = !((double)a.u[i] * (a.q ? (double)a.q[i * n + t] : 1.0) < (double)a.p[((size_t)b * (a.k + 1) + i0 + lane) * n + t]);
      }
      const unsigned m = __ballot_sync(0xffffffffu, no);
      if (m) {
        got = i0 + __ffs(m) - 1;
        break;
      }
    }
    if (lane == 0) s_got = got, s_count = count;
  }
  __syncthreads();
  const int got = s_got, count = s_count;
  if (count < 0) return;                   // an empty place of a padded batch (all CTAs of its cluster): left as it is
  const float* p = a.p + ((size_t)b * (a.k + 1) + got) * n;
  const float* q = got < count && a.q ? a.q + ((size_t)b * a.k + got) * n : nullptr;
  const int struck = got < count && !a.q ? a.drafts[(size_t)b * a.k + got] : -1;   // a certain draft that did not hold: everything but it is left
  const int i0 = (int)min((long)rank * a.per, (long)a.n), cnt = min(a.per, a.n - i0);
  const int sub = ((a.per + kVfWarps - 1) / kVfWarps + 31) / 32 * 32;             // a warp's stretch of the part
  const int w0 = min(warp * sub, cnt), w1 = min(w0 + sub, cnt);
  // The second round, where p - q leaves nothing, draws from p itself.
  for (int round = 0; round < 2; ++round) {
    auto weight = [&](int i) { return i == struck && round == 0 ? 0.0 : verify_weight(p[i], q && round == 0 ? q[i] : 0.f); };
    double s = 0.0;
#pragma unroll 4
    for (int i = w0 + lane; i < w1; i += 32) s += weight(i0 + i);
    s = warp_total(s);
    if (lane == 0) s_warp[warp] = s;
    __syncthreads();
    double mine = 0.0;
#pragma unroll
    for (int w = 0; w < kVfWarps; ++w) mine += s_warp[w];
    double before = 0.0, total = mine;
    int last = (int)rank;                  // the last CTA whose part weighs anything
    if (cluster > 1) {
      if (tid == 0) s_total[round] = mine;
      asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
      total = 0.0;
      for (uint32_t c = 0; c < cluster; ++c) {
        uint32_t from;
        double o;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(smem_u32(&s_total[round])), "r"(c));
        asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(o) : "r"(from) : "memory");
        if (c == rank) before = total;
        if (o > 0.0) last = (int)c;
        total += o;
      }
    }
    if (!(total > 0.0) && round == 0 && got < count) {
      __syncthreads();                     // s_warp is written again
      continue;
    }
    const double goal = fmax((double)a.r[b] * total, 0.0);
    // The CTA in whose part the running sum passes the goal; where rounding leaves it unpassed, the last one that weighs anything.
    const bool here = total > 0.0 ? mine > 0.0 && before <= goal && (before + mine > goal || last == (int)rank) : rank == 0;
    if (here && warp == 0) {
      int token = -1;                      // nothing weighs anything: no token
      if (total > 0.0) {
        double run = before, start = before;
        int w_at = -1;
        for (int w = 0; w < kVfWarps; ++w) {
          const double o = s_warp[w];
          if (o > 0.0 && (w_at < 0 || run <= goal)) w_at = w, start = run;
          run += o;
        }
        // inside the warp's stretch: 32 runs, then the 32-blocks of the run that passes
        const int b0 = min(w_at * sub, cnt), b1 = min(b0 + sub, cnt), len = sub / 32;
        const int r0 = min(b0 + lane * len, b1), r1 = min(r0 + len, b1);
        double t = 0.0;
#pragma unroll 8
        for (int i = r0; i < r1; ++i) t += weight(i0 + i);
        auto scan = [&](double v) {
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) {
            const double o = __shfl_up_sync(0xffffffffu, v, d);
            if (lane >= d) v += o;
          }
          return v;
        };
        double cum = start + scan(t);
        unsigned over = __ballot_sync(0xffffffffu, t > 0.0 && cum > goal), some = __ballot_sync(0xffffffffu, t > 0.0);
        const int run_at = over ? __ffs(over) - 1 : 31 - __clz(some);
        double base = __shfl_sync(0xffffffffu, cum - t, run_at);
        const int f0 = __shfl_sync(0xffffffffu, r0, run_at), f1 = __shfl_sync(0xffffffffu, r1, run_at);
        for (int i = f0; i < f1; i += 32) {
          const double w = i + lane < f1 ? weight(i0 + i + lane) : 0.0;
          cum = base + scan(w);
          over = __ballot_sync(0xffffffffu, w > 0.0 && cum > goal), some = __ballot_sync(0xffffffffu, w > 0.0);
          if (over) {
            token = i0 + i + __ffs(over) - 1;
            break;
          }
          if (some) token = i0 + i + 31 - __clz(some);
          base = __shfl_sync(0xffffffffu, cum, 31);
        }
      }
      int32_t* out = a.tokens + (size_t)b * (a.k + 1);
      for (int i = lane; i <= a.k; i += 32) out[i] = i < got ? a.drafts[(size_t)b * a.k + i] : i == got ? token : -1;
      if (lane == 0) a.accepted[b] = got;
    }
    break;
  }
  if (cluster > 1) asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");   // the totals have been read
}

inline cudaError_t verify_launch(VerifyArgs a, long batch, cudaStream_t st) {
  int cluster = 1;
  while (cluster < kVfMaxCluster && cdiv(a.n, cluster) > kVfPart) cluster *= 2;
  a.per = cdiv(a.n, cluster);
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
