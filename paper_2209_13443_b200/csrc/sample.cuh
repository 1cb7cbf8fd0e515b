// The draw of a class (token) from a row of logits: temperature, the k largest, the nucleus, the share of the best, a given random number.
//
// w[v] = exp((l[v] - max) / t).  Classes are ordered by their logits, the lower index first where those are equal.  What is kept is a beginning of that order: of the
// first k, those before which less than p of the k's weight lies, of these the ones that weigh at least m.  So it is told by its last member (a logit and
// an index).  The token is the first kept class, by index, at which the running sum of weights exceeds u times their total.
//
// Weights and sums are fp64: a row of 10^5 classes has as many borders that u may fall next to, and sums that are off by 10^-7 would take another class on one draw in
// a hundred.  2^z = 2^(k / 256) 2^g with the first factor from a table and |g| <= 1 / 512: the power series of exp up to its fourth term leaves 2^-54 and takes ten fp64 operations
// with the sum, half of what it takes without a table.
//
// A row is kept in the shared memory of a CTA, or of a cluster of them, which speak in turns (meet).  The last member is looked for among few:
//   k: as many groups of lanes as k have a maximum at or above the smallest of those maxima, so the k-th largest lies there too.  Groups are as large as k allows (a warp, four
//   lanes, a lane): 64 warps of 2000 logits each leave about 250 candidates.  Where they are too many, they are counted in 1024 bins, equally wide in the logit.
//   p: a class weighs at least (1 - p) / n of the total if it is kept (those behind it would otherwise weigh less than 1 - p), which bounds its logit.  Candidates are weighed in 1024
//   bins, in the pass that sums the total: a bin is 0.04 octaves wide at most, so a member's share of its bin's largest weight, 17 bits, goes into a 32-bit sum.
// What lies in the bin of the goal, or everything down to it if that is little, is gathered in a list, ordered by counting, and weighed exactly.
// Otherwise (thousands of equal logits, k above the list's length, no finite bound) it is found digit by digit of the logit's bits: the CTAs count (and weigh) what
// has the digits found so far by its next one, read each other's counts, and each takes the digit in which the goal lies.
#pragma once
#include <float.h>

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
constexpr int kSpBins = 1024, kSpList = 512;
constexpr int kSpTable = 256;

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

// 2^(j / 256) by the series of exp up to its 12th term.
__device__ __forceinline__ double sp_root(int j) {
  const double g = j * (0.69314718055994531 / kSpTable);
  double p = 1.0;
#pragma unroll
  for (int n = 16; n >= 1; --n) p = fma(p, g * (1.0 / n), 1.0);
  return p;
}

// An integer that orders like the float; both zeros are one.
__device__ __forceinline__ uint32_t sp_key(float l) {
  const uint32_t b = __float_as_uint(l + 0.f);
  return b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float sp_logit(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

struct SpWeight {
  const double* roots;
  double c, top;
  uint32_t far;            // upper half of the difference behind which nothing is left; as bits, that of a negative number grows with its size
  __device__ __forceinline__ SpWeight(const double* table, float heat, float top_)
      : roots(table), c(1.4426950408889634 / (double)heat), top((double)top_) {
    far = (uint32_t)__double2hiint(fmax(-1080.0 / c, -DBL_MAX));
  }
  __device__ __forceinline__ double operator()(float l) const {
    constexpr double kMagic = 26388279066624.0;        // 1.5 * 2^44: the sum's last place is 1 / 256
    const double d = (double)l - top;
    if ((uint32_t)__double2hiint(d) > far) return 0.0; // also -inf at any temperature (0 * inf)
    const double r = fma(d, c, kMagic);
    const int k = __double2loint(r);
    const double g = fma(d, c, -(r - kMagic));         // octaves
    double q = fma(g, 9.6181291076284772e-3, 5.5504108664821580e-2);      // ln(2)^n / n!
    q = fma(q, g, 0.24022650695910071);
    q = fma(q, g, 0.69314718055994531);
    q *= g;
    const double root = roots[k & (kSpTable - 1)];
    const int e = k >> 8;
    const double w = __hiloint2double(__double2hiint(root) + ((e < -1000 ? e + 200 : e) << 20), __double2loint(root));
    return e < -1000 ? fma(w, q, w) * 6.223015277861142e-61 : fma(w, q, w);     // 2^-200: down to the smallest double
  }
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
struct SpTop {             // of a CTA: its maximum; the smallest maximum of a lane, of four, of a warp, and how many of them have one
  float top, low[3];
  int have[3];
};
struct SpWork {
  union {
    uint32_t bins[kSpBins];              // members of a bin, or their weight; read by the others
    unsigned long long all[kSpList];     // the lists of all CTAs; after that
  };
  unsigned long long list[kSpList];      // logit << 32 | ~index; read by the others
  union {
    struct {
      unsigned long long sorted[kSpList];
      double weight[kSpList];
    };
    SpHist hist[2];
  };
};

template <typename T>
__global__ void __launch_bounds__(kSpThreads, 4)
sample_kernel(SampleArgs a) {
  extern __shared__ __align__(16) uint8_t sp_smem[];
  __shared__ SpSlot s_slot[2];
  __shared__ SpTop s_top, s_tops[kSpWarps];
  __shared__ SpWork s_work;
  __shared__ double s_roots[kSpTable];
  __shared__ double s_warp[kSpWarps], s_block[(kSpMaxPart + kSpBlock - 1) / kSpBlock], s_double;
  __shared__ unsigned long long s_scan_m[kSpWarps];
  __shared__ uint32_t s_scan_c[kSpWarps];
  __shared__ SpFound s_found;
  __shared__ int s_int, s_int2;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t rank, cluster;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
  const long row = blockIdx.x / cluster;
  const int i0 = min((int)rank * a.per, a.n), cnt = min(a.per, a.n - i0);
  s_roots[tid] = sp_root(tid);
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
  // The maximum; and of the groups of lanes that have one, the smallest, by the size of the group.
  float low[3] = {INFINITY, INFINITY, INFINITY};
  int have[3];
  {
    float mine = top;
#pragma unroll
    for (int g = 0; g < 3; ++g) {          // of a lane, of four, of a warp
      const bool some = mine > -INFINITY;
      low[g] = some ? mine : INFINITY;
      have[g] = __popc(__ballot_sync(0xffffffffu, some)) >> (g == 0 ? 0 : g == 1 ? 2 : 5);
#pragma unroll
      for (int d = 16; d; d >>= 1) low[g] = fminf(low[g], __shfl_xor_sync(0xffffffffu, low[g], d));
      if (g == 0) mine = sp_max(mine, __shfl_xor_sync(0xffffffffu, mine, 1)), mine = sp_max(mine, __shfl_xor_sync(0xffffffffu, mine, 2));
      if (g == 1) mine = sp_max(mine, __shfl_xor_sync(0xffffffffu, mine, 4)), mine = sp_max(mine, __shfl_xor_sync(0xffffffffu, mine, 8)), mine = sp_max(mine, __shfl_xor_sync(0xffffffffu, mine, 16));
    }
    top = mine;
  }
  auto join = [&](SpTop& t, int n) {       // over lanes 0 to n - 1
    if (lane >= n) t = SpTop{-INFINITY, {INFINITY, INFINITY, INFINITY}, {0, 0, 0}};
#pragma unroll
    for (int d = 8; d; d >>= 1) {
      t.top = sp_max(t.top, __shfl_xor_sync(0xffffffffu, t.top, d));
#pragma unroll
      for (int g = 0; g < 3; ++g) {
        t.low[g] = fminf(t.low[g], __shfl_xor_sync(0xffffffffu, t.low[g], d));
        t.have[g] += __shfl_xor_sync(0xffffffffu, t.have[g], d);
      }
    }
  };
  if (lane == 0) s_tops[warp] = SpTop{top, {low[0], low[1], low[2]}, {have[0], have[1], have[2]}};
  __syncthreads();
  SpTop best = s_tops[lane & (kSpWarps - 1)];
  join(best, kSpWarps);
  if (cluster > 1) {
    if (tid == 0) s_top = best;
    meet();
    const uint32_t at = map_to_rank(smem_u32(&s_top), (uint32_t)(lane < (int)cluster ? lane : 0));
    float v[4];
    int w[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[i]) : "r"(at + 4u * i) : "memory");
#pragma unroll
    for (int i = 0; i < 3; ++i) asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(w[i]) : "r"(at + 16u + 4u * i) : "memory");
    best = SpTop{v[0], {v[1], v[2], v[3]}, {w[0], w[1], w[2]}};
    join(best, (int)cluster);
  }
  // lanes 16 to 31 have joined nothing
  top = __shfl_sync(0xffffffffu, best.top, 0);
#pragma unroll
  for (int g = 0; g < 3; ++g) best.low[g] = __shfl_sync(0xffffffffu, best.low[g], 0), best.have[g] = __shfl_sync(0xffffffffu, best.have[g], 0);

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
    const SpWeight weight(s_roots, heat, top);
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
        SpHist& h = s_work.hist[r & 1];
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

    // ---- the list: members whose bin lies in [from, to] (bins of width 1 / scale below the maximum; nothing beyond `reach`); with_sums: the sums of blocks of what lies above them.
    // Returns how many there are, kSpList at most, or -1.
    const float ftop = top;
    auto gather = [&](float scale, float reach, int from, int to, bool with_sums) {
      if (tid == 0) s_int = 0;
      __syncthreads();
      for (int b = warp; b < (cnt + kSpBlock - 1) / kSpBlock; b += kSpWarps) {
        const int end = min((b + 1) * kSpBlock, cnt);
        double sum = 0.0;
#pragma unroll 4
        for (int i = b * kSpBlock + lane; i < end; i += 32) {
          const float l = logit(i), x = ftop - l, f = x * scale;
          if (!(x <= reach && f < (float)kSpBins)) continue;
          const int bin = (int)f;
          if (bin > to) continue;
          if (bin >= from) {
            const int at = atomicAdd(&s_int, 1);
            if (at < kSpList) s_work.list[at] = (unsigned long long)sp_key(l) << 32 | (uint32_t)~(i0 + i);
          } else if (with_sums) {
            sum += weight(l);
          }
        }
        if (with_sums) {
          sum = warp_total(sum);
          if (lane == 0) s_block[b] = sum;
        }
      }
      __syncthreads();
      double above = 0.0;
      if (with_sums)
        for (int b = 0; b < (cnt + kSpBlock - 1) / kSpBlock; b += 32) above += warp_total(b + lane < (cnt + kSpBlock - 1) / kSpBlock ? s_block[b + lane] : 0.0);
      tell(above, s_int, 0.f);
      // everybody copies all lists, in the order of the CTAs
      const SpSlot o = told(lane < (int)cluster ? lane : 0);
      const int count = lane < (int)cluster ? min(o.i, kSpList + 1) : 0;
      int upto = count;
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += v;
      }
      const int members = __shfl_sync(0xffffffffu, upto, (int)cluster - 1);
      if (with_sums) {
        above = 0.0;
        for (int c = 0; c < (int)cluster; ++c) above += __shfl_sync(0xffffffffu, o.d, c);
        if (tid == 0) s_double = above;
      }
      if (members > kSpList) return -1;
      for (int i = tid; i - lane < members; i += kSpThreads) {
        int c = 0, start = 0;
        for (int r = 0; r < (int)cluster - 1; ++r) {
          const int v = __shfl_sync(0xffffffffu, upto, r);
          if (i >= v) c = r + 1, start = v;
        }
        if (i < members) {
          unsigned long long e;
          asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(e) : "r"(map_to_rank(smem_u32(&s_work.list[i - start]), (uint32_t)c)) : "memory");
          s_work.all[i] = e;
        }
      }
      __syncthreads();
      // in order: a member's place is the number of those in front of it
      for (int i = tid; i < members; i += kSpThreads) {
        const unsigned long long e = s_work.all[i];
        int place = 0;
#pragma unroll 4
        for (int j = 0; j < members; ++j) place += s_work.all[j] > e;
        s_work.sorted[place] = e;
        s_work.weight[place] = weight(sp_logit((uint32_t)(e >> 32)));
      }
      __syncthreads();
      return members;
    };
    // Counts or weighs candidates in bins, sums the row (by_weight), and finds the bins in which the goal lies: `goal` in members, or in parts of the sum.
    // Returns what lies above them, in members (by_weight: at most as many), or -1.
    double sum_all = 0.0;
    int from = 0, to = 0, inside = 0;
    auto look = [&](float scale, float reach, bool by_weight, double goal, double octaves) {
      for (int i = tid; i < kSpBins; i += kSpThreads) s_work.bins[i] = 0u;
      if (tid == 0) s_int = kSpBins, s_int2 = -1;
      __syncthreads();
      double sum = 0.0;
      const float fall = -(float)octaves;          // of a bin
#pragma unroll 4
      for (int i = tid; i < cnt; i += kSpThreads) {
        const float l = logit(i), x = ftop - l, f = x * scale;
        if (by_weight) sum += weight(l);
        if (!(x <= reach && f < (float)kSpBins)) continue;
        const int bin = (int)f;
        uint32_t v = 1u;
        if (by_weight) {
          float share;
          asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(share) : "f"((f - (float)bin) * fall));
          v = (uint32_t)(share * 131072.f + 0.5f);       // 17 bits: 38400 members of a part stay below 2^33, so parts that long are found digit by digit
        }
        atomicAdd(&s_work.bins[bin], v);
      }
      if (by_weight) {
        tell(cta_sum(sum), 0, 0.f);
        for (int c = 0; c < (int)cluster; ++c) sum_all += told(c).d;
        goal *= sum_all;
      } else {
        meet();
      }
      // four bins a thread, over the cluster
      uint32_t v[4] = {0u, 0u, 0u, 0u};
      double m[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 4
      for (int c = 0; c < (int)cluster; ++c) {
        uint32_t w[4];
        asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(map_to_rank(smem_u32(&s_work.bins[4 * tid]), (uint32_t)c)) : "memory");
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (by_weight) m[j] += (double)w[j];
          else v[j] += w[j];
        }
      }
      if (by_weight) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[j] = (uint32_t)(m[j] * (1.0 / 131072) * 1.04) + (m[j] > 0.0);          // a bin is 0.04 octaves wide at most: never fewer than there are
          m[j] *= exp2(-octaves * (4 * tid + j)) * (1.0 / 131072);
        }
      }
      const uint32_t c4 = v[0] + v[1] + v[2] + v[3];
      const double m4 = m[0] + m[1] + m[2] + m[3];
      uint32_t cc = c4;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, cc, d);
        if (lane >= d) cc += o;
      }
      double cm = by_weight ? warp_scan(m4, lane) : 0.0;
      __syncthreads();
      if (lane == 31) s_scan_c[warp] = cc, s_warp[warp] = cm;
      __syncthreads();
      for (int w = 0; w < warp; ++w) cc += s_scan_c[w], cm += s_warp[w];
      uint32_t before = cc - c4;
      double before_m = cm - m4;
      const double slack = by_weight ? 4e-6 * sum_all : 0.0;          // 17 bits a member, and the difference of the two forms of its weight
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int bin = 4 * tid + j;
        if (v[j] > 0u) {
          if (by_weight) {
            if (before_m + m[j] >= goal - slack) atomicMin(&s_int, bin);
            if (before_m < goal + slack) atomicMax(&s_int2, bin);
          } else if ((double)before < goal && (double)(before + v[j]) >= goal) {
            s_int = s_int2 = bin;
          }
        }
        before += v[j], before_m += m[j];
      }
      __syncthreads();
      from = s_int, to = s_int2;
      __syncthreads();
      if (to < 0) return -1;
      from = min(from, to);
      before = cc - c4;
      if (tid == 0) s_int2 = 0;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int bin = 4 * tid + j;
        if (bin == from) s_int = (int)before;
        if (bin >= from && bin <= to && v[j]) atomicAdd(&s_int2, (int)v[j]);
        before += v[j];
      }
      __syncthreads();
      const int above = s_int;
      inside = s_int2;
      __syncthreads();
      return above;
    };

    bool whole = false;                    // the list holds all that is kept
    bool summed = false;                   // s_block holds the sums of what is kept
    int members = -1, cut = 0;
    bool found_k = !k, found_p = !by_p;
    double total = 0.0;
    if (k && k <= kSpList) {
      const int g = k <= best.have[2] ? 2 : k <= best.have[1] ? 1 : 0;
      const float reach = ftop - best.low[g], scale = reach > 0.f ? 1023.9f / reach : 0.f;
      if (k <= best.have[g] && scale < FLT_MAX && reach < FLT_MAX) {
        if (g == 2 || a.n <= kSpList) members = gather(scale, reach, 0, kSpBins - 1, false);
        whole = members > 0;
        if (!whole) {
          const int above = look(scale, reach, false, (double)k, 0.0);
          if (above >= 0 && above + inside <= kSpList) {
            members = gather(scale, reach, 0, to, false);
            whole = members > 0;
          } else if (above >= 0 && inside <= kSpList) {
            members = gather(scale, reach, from, to, false);
            if (members >= k - above && k > above) {
              const unsigned long long e = s_work.sorted[k - above - 1];
              last = (uint32_t)(e >> 32), last_at = (int)~(uint32_t)e;
              found_k = true;
            }
          }
        }
      }
      if (whole) members = min(members, k);
    } else if (!k && by_p) {
      // 1 - p is exact; the total is 1 at least
      const double octaves = (log2((double)a.n) - log2(1.0 - (double)p)) * 1.0001;
      const float reach = (float)(octaves / weight.c), scale = (float)(kSpBins * weight.c / octaves);
      if (a.per <= 32767 && reach < FLT_MAX && scale < FLT_MAX && scale > 0.f) {
        const int above = look(scale, reach, true, (double)p, octaves / kSpBins);
        const double goal = (double)p * sum_all;
        if (above >= 0 && above + inside <= kSpList) {
          members = gather(scale, reach, 0, to, false);
          whole = members > 0;
        } else if (above >= 0) {
          members = gather(scale, reach, from, to, true);
          if (members > 0) {
            if (warp == 0) {
              double before = s_double;
              int j = 0;
              for (int i = 0; i < members; i += 32) {
                const double w = i + lane < members ? s_work.weight[i + lane] : 0.0, cum = before + warp_scan(w, lane);
                const unsigned in = __ballot_sync(0xffffffffu, i + lane < members && cum - w < goal);
                j += __popc(in);
                before = __shfl_sync(0xffffffffu, cum, 31);
              }
              if (lane == 0) s_int = max(j, 1);
            }
            __syncthreads();
            cut = s_int;
            const unsigned long long e = s_work.sorted[cut - 1];
            last = (uint32_t)(e >> 32), last_at = (int)~(uint32_t)e;
            found_p = true;
            summed = !by_m;
          }
        }
      }
    }
    if (whole) {
      // all from the list: what is kept of it, and their total, in order
      if (warp == 0) {
        double want = INFINITY;
        if (by_p) {
          double sum = 0.0;
          if (k)
            for (int i = 0; i < members; i += 32) sum += warp_total(i + lane < members ? s_work.weight[i + lane] : 0.0);
          else sum = sum_all;
          want = (double)p * sum;
        }
        double before = 0.0;
        int j = 0;
        for (int i = 0; i < members; i += 32) {
          const double w = i + lane < members ? s_work.weight[i + lane] : 0.0, cum = before + warp_scan(w, lane);
          const bool in = i + lane < members && cum - w < want && !(by_m && w < (double)m);
          const unsigned b = __ballot_sync(0xffffffffu, in || (i == 0 && lane == 0));
          const int n = b == 0xffffffffu ? 32 : __ffs(~b) - 1;
          j += n;
          before = n > 0 ? __shfl_sync(0xffffffffu, cum, n - 1) : before;
          if (n < 32) break;
        }
        if (lane == 0) s_int = j, s_double = before;
      }
      __syncthreads();
      cut = s_int, total = s_double;
      const unsigned long long e = s_work.sorted[cut - 1];
      last = (uint32_t)(e >> 32), last_at = (int)~(uint32_t)e;
      __syncthreads();
      if (a.tokens) {
        // by index: a class that the running sum passes the goal with, the first of them; or the last that weighs anything
        const double goal = fmax((double)a.u[row] * total, 0.0);
        if (tid == 0) s_int = 0x7fffffff, s_int2 = -1;
        __syncthreads();
        for (int i = tid; i < cut; i += kSpThreads) {
          const uint32_t at = (uint32_t)s_work.sorted[i];          // the larger, the lower the index
          const double w = s_work.weight[i];
          double before = 0.0;
#pragma unroll 4
          for (int j = 0; j < cut; ++j)
            if ((uint32_t)s_work.sorted[j] > at) before += s_work.weight[j];
          if (w > 0.0) {
            if (before + w > goal) atomicMin(&s_int, (int)~at);
            atomicMax(&s_int2, (int)~at);
          }
        }
        __syncthreads();
        token = s_int != 0x7fffffff ? s_int : s_int2;
      }
    } else {
      if (!found_k) select(false, (double)k);
      if (!found_p) {
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
    }
    const bool all = !k && !by_p;
    auto mass = [&](int i) {               // what class i adds to the sum
      const float l = logit(i);
      if (!all && !kept(sp_key(l), i)) return 0.0;
      const double w = weight(l);
      return by_m && w < (double)m ? 0.0 : w;
    };
    // ---- sums of blocks, the total, and the block in which the running sum passes its goal
    if (!whole) {
    const int blocks = (cnt + kSpBlock - 1) / kSpBlock;
    if (summed) {
      // those of the list that are kept join their blocks, in order
      for (int b = tid; b < blocks; b += kSpThreads) {
        double s = s_block[b];
        for (int j = 0; j < cut; ++j) {
          const int at = (int)~(uint32_t)s_work.sorted[j] - i0;
          if (at >= 0 && at < cnt && at / kSpBlock == b) s += s_work.weight[j];
        }
        s_block[b] = s;
      }
    } else {
      for (int b = warp; b < blocks; b += kSpWarps) {
        const int end = min((b + 1) * kSpBlock, cnt);
        double s = 0.0;
#pragma unroll 4
        for (int i = b * kSpBlock + lane; i < end; i += 32) s += mass(i);
        s = warp_total(s);
        if (lane == 0) s_block[b] = s;
      }
    }
    __syncthreads();
    double sum = 0.0;
    for (int b = 0; b < blocks; b += 32) sum += warp_total(b + lane < blocks ? s_block[b + lane] : 0.0);
    tell(sum, 0, 0.f);
    double before = 0.0;
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
