// The draw of a class (token) from a row of logits: temperature, the k largest, the nucleus, the share of the best, a given random number.
//
// w[v] = exp((l[v] - max) / t).  Classes are ordered by their logits, the lower index first where those are equal.  What is kept is a beginning of that order: of the
// first k, those before which less than p of the k's weight lies, of these the ones that weigh at least m.  So it is told by its last member (a logit and
// an index).  The token is the first kept class, by index, at which the running sum of weights exceeds u times their total.
//
// Weights and sums are fp64: a row of 10^5 classes has as many borders that u may fall next to, and sums that are off by 10^-7 would take another class on one draw in
// a hundred.  2^z by the power series of exp on |z - integer| <= 1/2, to 2^-50 of itself.
//
// A row is kept in the shared memory of a CTA, or of a cluster of them.  Its last member is found digit by digit of the logit's bits: the CTAs count (and weigh) what
// has the digits found so far by its next one, read each other's counts, and each takes the digit in which the k-th member, or the p-th part of the weight, lies.
#pragma once
#include "common.cuh"
#include "conv_pair.cuh"
#include "conv_tc.cuh"
#include "draft.cuh"

namespace ee {

constexpr int kSpThreads = 256, kSpWarps = kSpThreads / 32;
constexpr int kSpPart = 16384;           // elements of a CTA's part that a cluster is cut for
constexpr int kSpMaxCluster = 16, kSpMaxPart = 38400;
constexpr int kSpBlock = 512;            // elements of a block whose sum is kept
constexpr int kSpMost = kSpMaxCluster * kSpMaxPart;

struct SampleArgs {
  const void* x;           // [rows][n]
  const float* heat;       // [rows], or null: 1
  const int32_t* top_k;    // [rows], or null
  const float* top_p;
  const float* min_p;
  const float* u;          // [rows]; null without tokens
  int32_t* tokens;         // [rows], or null
  float* probs;            // [rows][n], or null
  int n, per;
};

// 2^z, z <= 0.  With g = (z - k) ln 2, |g| <= 0.35: the series up to g^12 / 12! leaves 2^-52.
__device__ __forceinline__ double sp_pow2(double z) {
  if (!(z > -1080.0)) return 0.0;
  const double r = z + 6755399441055744.0;            // 1.5 * 2^52: the sum's last place is 1
  const int k = __double2loint(r);
  const double g = (z - (r - 6755399441055744.0)) * 0.69314718055994531;
  double p = 1.0 / 479001600;
  p = fma(p, g, 1.0 / 39916800);
  p = fma(p, g, 1.0 / 3628800);
  p = fma(p, g, 1.0 / 362880);
  p = fma(p, g, 1.0 / 40320);
  p = fma(p, g, 1.0 / 5040);
  p = fma(p, g, 1.0 / 720);
  p = fma(p, g, 1.0 / 120);
  p = fma(p, g, 1.0 / 24);
  p = fma(p, g, 1.0 / 6);
  p = fma(p, g, 0.5);
  p = fma(p, g, 1.0);
  p = fma(p, g, 1.0);
  if (k < -1000) return __hiloint2double(__double2hiint(p) + ((k + 200) << 20), __double2loint(p)) * 6.223015277861142e-61;   // 2^-200: down to the smallest double
  return __hiloint2double(__double2hiint(p) + (k << 20), __double2loint(p));
}

// An integer that orders like the float; both zeros are one.
__device__ __forceinline__ uint32_t sp_key(float l) {
  const uint32_t b = __float_as_uint(l + 0.f);
  return b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float sp_logit(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

struct SpWeight {
  double c, top;
  __device__ __forceinline__ SpWeight(float heat, float top_) : c(1.4426950408889634 / (double)heat), top((double)top_) {}
  __device__ __forceinline__ double operator()(float l) const { return l == -INFINITY ? 0.0 : sp_pow2(((double)l - top) * c); }
};

__device__ __forceinline__ float sp_max(float a, float b) {      // NaN where either is
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
template <typename T>
__device__ __forceinline__ float sp_word_max(uint4 w, float top) {
  if constexpr (sizeof(T) == 2) {
    __nv_bfloat162 a, b;
    *reinterpret_cast<uint32_t*>(&a) = w.x, *reinterpret_cast<uint32_t*>(&b) = w.y;
    __nv_bfloat162 m = __hmax2_nan(a, b);
    *reinterpret_cast<uint32_t*>(&a) = w.z, *reinterpret_cast<uint32_t*>(&b) = w.w;
    m = __hmax2_nan(m, __hmax2_nan(a, b));
    return sp_max(top, sp_max(__low2float(m), __high2float(m)));
  } else {
    return sp_max(sp_max(top, sp_max(__uint_as_float(w.x), __uint_as_float(w.y))), sp_max(__uint_as_float(w.z), __uint_as_float(w.w)));
  }
}

struct SpSlot {            // what a CTA tells the others
  double d;
  int i;
  float f;
};
struct SpHist {            // by digit: members, and their weight in units of 2^-43 (at most 614400 of them, each at most 1)
  uint32_t count[256];
  unsigned long long mass[256];
};
struct SpFound {           // the digit, and what lies above it
  int digit;
  int above, in;
};

template <typename T>
__global__ void __launch_bounds__(kSpThreads)
sample_kernel(SampleArgs a) {
  extern __shared__ __align__(16) uint8_t sp_smem[];
  __shared__ SpSlot s_slot[2];
  __shared__ SpHist s_hist[2];
  __shared__ SpFound s_found;
  __shared__ double s_warp[kSpWarps], s_block[(kSpMaxPart + kSpBlock - 1) / kSpBlock];
  __shared__ unsigned long long s_scan_m[kSpWarps];
  __shared__ uint32_t s_scan_c[kSpWarps];
  __shared__ int s_int;
  __shared__ float s_tops[kSpWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t rank, cluster;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
  const long row = blockIdx.x / cluster;
  const int i0 = min((int)rank * a.per, a.n), cnt = min(a.per, a.n - i0);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const T* src = (const T*)a.x + (size_t)row * a.n + i0;

  // ---- the CTAs of a cluster speak in turns: each leaves something in its shared memory, all meet, each reads the others'.  Two places are enough: what is left in
  // one is overwritten after the meeting behind the one in which it was read.
  int turn = 0;
  auto meet = [&]() {
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
    else __syncthreads();
  };
  auto tell = [&](double d, int i, float f) {            // by thread 0; all threads meet
    if (tid == 0) s_slot[turn & 1] = SpSlot{d, i, f};
    meet();
    ++turn;
  };
  auto told = [&](int c) {                               // what CTA c told last
    SpSlot s;
    const uint32_t at = map_to_rank(smem_u32(&s_slot[(turn - 1) & 1]), (uint32_t)c);
    asm volatile("ld.shared::cluster.v2.b32 {%0, %1}, [%2];" : "=r"(s.i), "=r"(*reinterpret_cast<int*>(&s.f)) : "r"(at + 8u) : "memory");
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(s.d) : "r"(at) : "memory");
    return s;
  };
  auto cta_sum = [&](double v) {                         // of the CTA's threads, in fixed order
    v = warp_total(v);
    __syncthreads();
    if (lane == 0) s_warp[warp] = v;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < kSpWarps; ++k) sum += s_warp[k];
    return sum;
  };

  // ---- the row, at its own offset within a 16-byte word, and its maximum
  constexpr int W = 16 / (int)sizeof(T);
  const int skew = (int)(((uintptr_t)src & 15) / sizeof(T));
  T* part = reinterpret_cast<T*>(sp_smem) + skew;
  const int head = min(cnt, skew ? W - skew : 0), words = (cnt - head) / W, tail = head + words * W;
#pragma unroll 4
  for (int i = tid; i < words; i += kSpThreads)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(part + head + i * W)), "l"(src + head + (size_t)i * W) : "memory");
  cp_async_commit();
  float top = -INFINITY;
  if (tid < head) part[tid] = src[tid], top = Elem<T>::ld(part + tid);
  if (tid < cnt - tail) part[tail + tid] = src[tail + tid], top = sp_max(top, Elem<T>::ld(part + tail + tid));
  float heat = a.heat ? a.heat[row] : 1.f;
  int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f, m = a.min_p ? a.min_p[row] : 0.f;
  cp_async_wait<0>();
#pragma unroll 4
  for (int i = tid; i < words; i += kSpThreads) top = sp_word_max<T>(*reinterpret_cast<const uint4*>(part + head + i * W), top);
#pragma unroll
  for (int d = 16; d; d >>= 1) top = sp_max(top, __shfl_xor_sync(0xffffffffu, top, d));
  if (lane == 0) s_tops[warp] = top;
  __syncthreads();
  top = s_tops[lane & (kSpWarps - 1)];
#pragma unroll
  for (int d = kSpWarps / 2; d; d >>= 1) top = sp_max(top, __shfl_xor_sync(0xffffffffu, top, d));
  tell(0.0, 0, top);
  top = told(lane < (int)cluster ? lane : 0).f;
#pragma unroll
  for (int d = 16; d; d >>= 1) top = sp_max(top, __shfl_xor_sync(0xffffffffu, top, d));

  auto logit = [&](int i) { return Elem<T>::ld(part + i); };
  float* probs = a.probs ? a.probs + (size_t)row * a.n + i0 : nullptr;
  const bool nothing = !(top < INFINITY) || top == -INFINITY;       // no class, or NaN or +inf among the logits
  const bool first = !(heat > 0.f) || k == 1 || p <= 0.f || m > 1.f;   // only the first stays
  if (k < 0 || k >= a.n) k = 0;
  const bool by_p = p < 1.f, by_m = m > 0.f;
  int token = -1;                          // of this CTA: the one that has it stores it
  bool mine = rank == 0;
  if (nothing) {
    const float v = top == -INFINITY ? 0.f : NAN;
    if (probs)
      for (int i = tid; i < cnt; i += kSpThreads) probs[i] = v;
  } else if (first) {
    int at = 0x7fffffff;
    for (int i = tid; i < cnt; i += kSpThreads)
      if (at == 0x7fffffff && logit(i) == top) at = i0 + i;
    at = __reduce_min_sync(0xffffffffu, at);
    if (tid == 0) s_int = 0x7fffffff;
    __syncthreads();
    if (lane == 0) atomicMin(&s_int, at);
    __syncthreads();
    tell(0.0, s_int, 0.f);
    token = __reduce_min_sync(0xffffffffu, told(lane < (int)cluster ? lane : 0).i);
    if (probs)
      for (int i = tid; i < cnt; i += kSpThreads) probs[i] = i0 + i == token ? 1.f : 0.f;
  } else {
    const SpWeight weight(heat, top);
    // The last member: what is above it by logit, or beside it and not behind it by index, is kept.
    uint32_t last = 0u;
    int last_at = 0x7fffffff;
    auto kept = [&](uint32_t key, int i) { return key > last || (key == last && i0 + i <= last_at); };

    // Of what is kept, the new last member: by count (the goal-th), or by weight (the last before which there is less than goal).
    auto select = [&](bool by_weight, double goal) {
      constexpr int kRounds = sizeof(T) == 2 ? 2 : 4;      // a bf16's bits end after two digits
      uint32_t prefix = 0u;
      uint32_t above = 0u;
      unsigned long long above_m = 0ull;
      const double unit = 8796093022208.0;                 // 2^43
      const unsigned long long goal_m = (unsigned long long)fmin(ceil(goal * (by_weight ? unit : 1.0)), 1.8e19);
      int in = 0;
      for (int r = 0; r < kRounds; ++r) {
        const int shift = 24 - 8 * r;
        SpHist& h = s_hist[r & 1];
        h.count[tid] = 0u, h.mass[tid] = 0ull;
        __syncthreads();
        for (int i = tid; i < cnt; i += kSpThreads) {
          const float l = logit(i);
          const uint32_t key = sp_key(l);
          if ((r == 0 || key >> (shift + 8) == prefix) && kept(key, i)) {
            const int d = key >> shift & 255;
            atomicAdd(&h.count[d], 1u);
            if (by_weight) atomicAdd(&h.mass[d], (unsigned long long)__double2ull_rn(weight(l) * unit));
          }
        }
        meet();
        // digit 255 - tid, over the cluster; then what lies above it
        const int d = 255 - tid;
        uint32_t c = 0u;
        unsigned long long ms = 0ull;
        for (int o = 0; o < (int)cluster; ++o) {
          uint32_t v;
          unsigned long long w;
          asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(map_to_rank(smem_u32(&h.count[d]), (uint32_t)o)) : "memory");
          asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(w) : "r"(map_to_rank(smem_u32(&h.mass[d]), (uint32_t)o)) : "memory");
          c += v, ms += w;
        }
        uint32_t cc = c;
        unsigned long long cm = ms;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t v = __shfl_up_sync(0xffffffffu, cc, o);
          const unsigned long long w = __shfl_up_sync(0xffffffffu, cm, o);
          if (lane >= o) cc += v, cm += w;
        }
        if (lane == 31) s_scan_c[warp] = cc, s_scan_m[warp] = cm;
        if (tid == 0) s_int = -1;
        __syncthreads();
        for (int o = 0; o < warp; ++o) cc += s_scan_c[o], cm += s_scan_m[o];
        const uint32_t before = above + cc - c;
        const unsigned long long before_m = above_m + cm - ms;
        // The digit in which the goal lies: the last one with members before which less lies.
        if (c > 0 && (by_weight ? before_m < goal_m : (unsigned long long)before < goal_m)) atomicMax(&s_int, tid);
        __syncthreads();
        if (tid == s_int) s_found = SpFound{d, (int)before, (int)c}, s_scan_m[0] = before_m;
        __syncthreads();
        prefix = prefix << 8 | (uint32_t)s_found.digit;
        above = (uint32_t)s_found.above, in = s_found.in, above_m = s_scan_m[0];
      }
      // Every one that is left has the same logit: as many of them as the goal asks for, the lower indices first.
      uint32_t key = kRounds == 4 ? prefix : prefix << 16;
      if (kRounds == 2 && !(key & 0x80000000u)) key |= 0xffffu;       // a negative float's bits are turned round
      int take;
      if (by_weight) {
        double v = 0.0;                                    // what lies above, exactly
        for (int i = tid; i < cnt; i += kSpThreads) {
          const float l = logit(i);
          const uint32_t o = sp_key(l);
          if (o > key && kept(o, i)) v += weight(l);
        }
        tell(cta_sum(v), 0, 0.f);
        v = 0.0;
        for (int c = 0; c < (int)cluster; ++c) v += told(c).d;
        const double w = weight(sp_logit(key));
        take = w > 0.0 ? (int)fmin(fmax(ceil((goal - v) / w), 1.0), (double)in) : in;
      } else {
        take = (int)goal - (int)above;
      }
      int at = 0x7fffffff;
      if (take < in) {
        int c = 0;
        for (int i = tid; i < cnt; i += kSpThreads) c += sp_key(logit(i)) == key && kept(key, i);
        c = __reduce_add_sync(0xffffffffu, c);
        if (tid == 0) s_int = 0;
        __syncthreads();
        if (lane == 0) atomicAdd(&s_int, c);
        __syncthreads();
        const int have = s_int;
        tell(0.0, have, 0.f);
        int before = 0;
        for (int c2 = 0; c2 < (int)rank; ++c2) before += told(c2).i;
        // the CTA that has the take-th looks for its index
        if (tid == 0) s_int = 0;
        __syncthreads();
        if (before < take && take <= before + have && warp == 0) {
          int left = take - before;
          for (int i = lane; i - lane < cnt; i += 32) {
            const unsigned b = __ballot_sync(0xffffffffu, i < cnt && sp_key(logit(min(i, cnt - 1))) == key && kept(key, i));
            if (__popc(b) >= left) {
              const int j = __fns(b, 0, left);
              if (lane == 0) s_int = i0 + i + j;
              break;
            }
            left -= __popc(b);
          }
        }
        __syncthreads();
        tell(0.0, s_int, 0.f);
        at = 0;
        for (int c2 = 0; c2 < (int)cluster; ++c2) at = max(at, told(c2).i);      // the others say 0
      }
      if (key == last && take >= in) at = last_at;         // of the same logit, what was kept before
      last = key, last_at = at;
    };
    if (k) select(false, (double)k);
    if (by_p) {
      double v = 0.0;
      for (int i = tid; i < cnt; i += kSpThreads) {
        const float l = logit(i);
        if (kept(sp_key(l), i)) v += weight(l);
      }
      tell(cta_sum(v), 0, 0.f);
      v = 0.0;
      for (int c = 0; c < (int)cluster; ++c) v += told(c).d;
      select(true, (double)p * v);
    }
    const bool all = !k && !by_p;
    auto mass = [&](int i) {               // what class i adds to the sum
      const float l = logit(i);
      if (!all && !kept(sp_key(l), i)) return 0.0;
      const double w = weight(l);
      return by_m && w < (double)m ? 0.0 : w;
    };
    // ---- sums of blocks, the total, and the block in which the running sum passes its goal
    const int blocks = (cnt + kSpBlock - 1) / kSpBlock;
    for (int b = warp; b < blocks; b += kSpWarps) {
      const int end = min((b + 1) * kSpBlock, cnt);
      double s = 0.0;
#pragma unroll 4
      for (int i = b * kSpBlock + lane; i < end; i += 32) s += mass(i);
      s = warp_total(s);
      if (lane == 0) s_block[b] = s;
    }
    __syncthreads();
    double sum = 0.0;
    for (int b = 0; b < blocks; b += 32) sum += warp_total(b + lane < blocks ? s_block[b + lane] : 0.0);
    tell(sum, 0, 0.f);
    double before = 0.0, total = 0.0;
    int last_one = 0;                      // the last CTA that has any weight
    for (int c = 0; c < (int)cluster; ++c) {
      const double o = told(c).d;
      if (c == (int)rank) before = total;
      if (o > 0.0) last_one = c;
      total += o;
    }
    if (a.tokens) {
      const double goal = fmax((double)a.u[row] * total, 0.0);
      mine = sum > 0.0 && before <= goal && (before + sum > goal || last_one == (int)rank);
      if (mine && warp == 0) {
        int at = -1;
        double run = before, start = before;
        for (int b = 0; b < blocks; b += 32) {
          const double w = b + lane < blocks ? s_block[b + lane] : 0.0, cum = run + warp_scan(w, lane);
          const unsigned over = __ballot_sync(0xffffffffu, w > 0.0 && cum > goal), some = __ballot_sync(0xffffffffu, w > 0.0);
          const int j = over ? __ffs(over) - 1 : 31 - __clz(some);
          if (some) at = b + j, start = __shfl_sync(0xffffffffu, cum - w, j);
          if (over) break;
          run = __shfl_sync(0xffffffffu, cum, 31);
        }
        const int end = min((at + 1) * kSpBlock, cnt);
        bool found = false;
        for (int i = at * kSpBlock + lane; i - lane < end && !found; i += 32) {
          const double w = i < end ? mass(i) : 0.0, cum = start + warp_scan(w, lane);
          const unsigned over = __ballot_sync(0xffffffffu, w > 0.0 && cum > goal), some = __ballot_sync(0xffffffffu, w > 0.0);
          if (some) token = i0 + i - lane + (over ? __ffs(over) - 1 : 31 - __clz(some));
          found = over != 0;
          start = __shfl_sync(0xffffffffu, cum, 31);
        }
      }
    }
    if (probs) {
      const double scale = 1.0 / total;
      for (int i = tid; i < cnt; i += kSpThreads) probs[i] = (float)(mass(i) * scale);
    }
  }
  if (a.tokens && mine && tid == 0) a.tokens[row] = token;
  if (cluster > 1) asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");   // nobody reads this CTA's shared memory any more
}

template <typename T>
inline size_t sample_smem(int per) { return align_up((size_t)per * sizeof(T) + 16, 16); }

inline cudaError_t sample_context_init() {     // once per device
  cudaError_t e = cudaSuccess;
  auto set = [&](auto kernel, size_t bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  };
  set(sample_kernel<bf16>, sample_smem<bf16>(kSpMaxPart));
  set(sample_kernel<float>, sample_smem<float>(kSpMaxPart));
  return e;
}

template <typename T>
inline cudaError_t sample_launch(SampleArgs a, long rows, cudaStream_t st) {
  int cluster = 1;
  while (cluster < 8 && cdiv(a.n, cluster) > kSpPart) cluster *= 2;
  if (cdiv(a.n, cluster) > kSpMaxPart) cluster *= 2;
  a.per = cdiv(a.n, cluster);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * cluster));
  cfg.blockDim = dim3(kSpThreads);
  cfg.dynamicSmemBytes = sample_smem<T>(a.per);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, sample_kernel<T>, a);
}

}  // namespace ee
