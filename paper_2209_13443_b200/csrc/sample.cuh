// The draw of a class (token) from a row of logits: temperature, the k largest, the nucleus, the share of the best, a given random number.
//
// w[v] = exp((l[v] - max) / t).  Classes are ordered by their logits, the lower index first where those are equal.  What is kept is a beginning of that order: of the
// first k, those before which less than p of the k's weight lies, of these the ones that weigh at least m.  So it is told by its last member (a logit and
// an index).  The token is the first kept class, by index, at which the running sum of weights exceeds u times their total.
//
// Weights and sums that decide are fp64: a row of 10^5 classes has as many borders that u may fall next to, and sums that are off by 10^-7 would take another class on one draw in
// a hundred.  2^z = 2^(k / 16) 2^g with the first factor from a table and |g| <= 1 / 32: the power series of exp up to its sixth term leaves 2^-51.
//
// A row is kept in the shared memory of a CTA, or of a cluster of them, which speak in turns (meet).  The last member is looked for among few:
//   k: a logit that k of 512 groups of lanes reach with their largest: k-th and better lie at or above it, and little else does (60 of 128001 for k = 50; the smallest maximum of 64
//   warps left 270).  Where equal logits make too many of them, candidates are counted in 2048 bins (one CTA: 1024), equally wide in the logit.
//   p: a class weighs at least (1 - p) / n of the total if it is kept (those behind it would otherwise weigh less than 1 - p), which bounds its logit.  Candidates are weighed in such
//   bins, in fp32: a bin is 0.043 octaves wide at most, so a member's share of its bin's largest weight, 17 bits, goes into a 32-bit sum.
// What lies in the bins in which the goal may lie, or everything down to them if that is little, is gathered in a list, which the first CTA orders by counting; the pass that gathers it also
// sums the row, and what lies above, in fp64.  Bins with more members than the list has room for are looked at again, 2048 times closer.
// Otherwise the last member is found digit by digit of the logit's bits: the CTAs count (and weigh) what has the digits found so far by its next one, read each other's counts, and each takes the
// digit in which the goal lies.  That is so for k above 256, for p behind such a k or with no finite bound, for CTAs' parts above 32767 (p and 262137 to 307200 classes, or more than 524272; 17-bit
// shares would pass 32 bits), where more than the list's 512 places hold have the logit at the border, where p leaves out less than some 10^-5 and the goal may lie in too many bins, and where a CTA has more members than its share of the list's room (128 of eight, when few rows
// of a vocabulary ordered by frequency have most of the weight).  Equal logits happen to ordinary bf16 rows: the further they lie from 0 the more of them there are.
//
// us alone, 64 x 128001 bf16: no filter 25, k = 1 to 100 19, p = 0.8 to 0.99 62; 320 rows 94, 78 and 235, with probabilities 139, 109 and 275; one row 12, 12 and 31; one of 1000 classes 7, 10 and 16;
// the best alone (t = 0) 11, one of 1000 classes 3.  These are N(0, 3).  p on 64 rows by digits: N(4, 2) 850, N(8, 2) and N(-8, 1) 630, logits that fall with the index 990, 262144 classes 1060, 614400 2860; 128001
// in fp32, where few are equal, 78 to 96, 262144 1950; k = 1000 102, with p behind it 229 (k = 5000); k = 200 39, 84 where the logits fall with the index.
// Bound by instructions, then by what a row waits for: a warp's 32 logits take 47 instructions without a filter (13 of them fp64, at two clocks), 28 for k, 124 for p (a look of about 50, the
// exact pass of 45), and an SM issues 60 % of the time; joins, exchanges (400 clocks a meeting, 300 a remote load) and the list are serial, 3.5 CTAs an SM cover them in part.
// 64 registers let four CTAs share an SM, and put some 110 bytes of a thread in local memory.
// Steps for p, 64 rows: digits only 351 (mixed settings), bins and a list 134, without calls and branches in the loops 120, fp32 bins 69, one CTA for the list 62.
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
constexpr int kSpBins = 2048, kSpList = 512;
constexpr int kSpTable = 16;

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

// 2^(j / 16) by the series of exp.
struct SpRoots {
  double v[kSpTable];
};
constexpr SpRoots sp_roots() {
  SpRoots r{};
  for (int j = 0; j < kSpTable; ++j) {
    const double g = j * (0.69314718055994531 / kSpTable);
    double p = 1.0;
    for (int n = 20; n >= 1; --n) p = 1.0 + p * g / n;
    r.v[j] = p;
  }
  return r;
}
static __device__ const SpRoots g_sp_roots = sp_roots();

// An integer that orders like the float; both zeros are one.
__device__ __forceinline__ uint32_t sp_key(float l) {
  const uint32_t b = __float_as_uint(l + 0.f);
  return b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float sp_logit(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// v, or 0: without a branch round what v is made of.
__device__ __forceinline__ double sp_pick(bool keep, double v) {
  double r;
  asm("{\n .reg .pred p;\n setp.ne.u32 p, %2, 0;\n selp.f64 %0, %1, 0d0000000000000000, p;\n}" : "=d"(r) : "d"(v), "r"((int)keep));
  return r;
}

// A float as a double, by its bits: the conversion instruction takes 8 clocks a warp of a scheduler, fp64 arithmetic 2.  What is below 2^-126 comes out between 2^-127 and
// that, in order.
__device__ __forceinline__ double sp_wide(float l) {
  const int b = __float_as_int(l);
  return __hiloint2double(((b >> 3) & (int)0x8fffffff) + 0x38000000, b << 29);
}

// The weight of a logit.  Below 2^-1000, which no sum of 2^20 of them brings near any u that is not 0, it is 0; whether it would be more is asked for where u is 0 (live).
// There is neither a branch nor a call in it: with a call for the rare case a row of 128001 took 138 clocks a warp and 32 logits, its elements one after the other.
// The table has as many entries as 16 lanes read without a conflict: one of 256 took 15 clocks a lookup, and saved two fp64 operations of 2.
struct SpWeight {
  const double* roots;
  double c, top;
  uint32_t near;           // upper half of the difference from which on the weight is 0; as bits, that of a negative number grows with its size
  __device__ __forceinline__ SpWeight(const double* table, float heat, float top_) : roots(table), c(1.4426950408889634 / (double)heat), top(sp_wide(top_)) {
    near = (uint32_t)__double2hiint(fmax(-1000.0 / c, -DBL_MAX));
  }
  __device__ __forceinline__ double operator()(float l) const {
    constexpr double kMagic = 6755399441055744.0 / kSpTable;        // 1.5 * 2^52 / 16: the sum's last place is 1 / 16
    const double d = sp_wide(l) - top, r = fma(d, c, kMagic);
    const int k = __double2loint(r);
    const double g = fma(d, c, -(r - kMagic));         // octaves, up to 1 / 32
    double q = fma(g, 1.5403530393381609e-4, 1.3333558146428443e-3);      // ln(2)^n / n!: what is left out is 2^-51
    q = fma(q, g, 9.6181291076284772e-3);
    q = fma(q, g, 5.5504108664821580e-2);
    q = fma(q, g, 0.24022650695910071);
    q = fma(q, g, 0.69314718055994531);
    q *= g;
    const double root = roots[k & (kSpTable - 1)];
    const double w = __hiloint2double(__double2hiint(root) + ((k & ~(kSpTable - 1)) << (20 - 4)), __double2loint(root));
    return sp_pick((uint32_t)__double2hiint(d) <= near && l > -INFINITY, fma(w, q, w));
  }
  __device__ __forceinline__ bool live(float l) const { return l > -INFINITY && (sp_wide(l) - top) * c > -1075.0; }      // half of the smallest double
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
  double d, e;
  int i;
};
struct SpHist {            // by digit: members, and their weight in whole units
  uint32_t count[256];
  unsigned long long mass[256];
};
struct SpFound {           // the digit, and what lies above it
  int digit;
  int above, in;
};
struct SpKept {            // the last member, what is kept of the list, and its weight
  float last;
  int last_at;
  double total;
};
struct SpBorder {          // of a CTA's bins: the first in which the goal may lie and what lies before it (and its weight), the last and what lies up to its end
  int from, before, to, end;
  double weight;
};
struct SpWork {
  union {
    uint32_t bins[kSpBins];              // members of a bin, or their weight; read by the others
    unsigned long long all[2 * kSpList]; // the lists of all CTAs, as many places each, written by them into the first CTA's; after that
  };
  union {
    unsigned long long list[kSpList];    // logit << 32 | ~index
    uint32_t groups[kSpThreads];         // maxima of groups of lanes; read by the others, before that
  };
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
  constexpr int W = 16 / (int)sizeof(T), kBlockWords = kSpBlock / W;
  extern __shared__ __align__(16) uint8_t sp_smem[];
  __shared__ SpSlot s_slot[2];
  __shared__ uint32_t s_top, s_tops[kSpWarps];
  __shared__ SpWork s_work;
  __shared__ double s_roots[kSpTable];
  __shared__ double s_chunk[kSpList / 32], s_warp[kSpWarps], s_block[kSpMaxPart / kSpBlock + 2], s_double;
  __shared__ unsigned long long s_scan_m[kSpWarps];
  __shared__ uint32_t s_scan_c[kSpWarps];
  __shared__ SpFound s_found;
  __shared__ __align__(16) SpBorder s_border;
  __shared__ int s_counts[kSpMaxCluster];
  __shared__ __align__(16) SpKept s_kept;
  __shared__ int s_int, s_int2;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t rank, cluster;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(cluster));
  const long row = blockIdx.x / cluster;
  const int i0 = min((int)rank * a.per, a.n), cnt = min(a.per, a.n - i0);
  const double root = g_sp_roots.v[tid & (kSpTable - 1)];
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
  auto tell = [&](double d, int i, double e = 0.0) {     // by thread 0; all threads meet
    if (tid == 0) s_slot[turn & 1] = SpSlot{d, e, i};
    meet();
    ++turn;
  };
  auto told = [&](int c) {                               // what CTA c told last
    SpSlot s;
    const uint32_t at = map_to_rank(smem_u32(&s_slot[(turn - 1) & 1]), (uint32_t)c);
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(s.i) : "r"(at + 16u) : "memory");
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(s.d) : "r"(at) : "memory");
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(s.e) : "r"(at + 8u) : "memory");
    return s;
  };
  auto in_order = [&](double d) {                        // the sum over the CTAs, of which each lane has one's
    double sum = 0.0;
    for (int c = 0; c < (int)cluster; ++c) sum += __shfl_sync(0xffffffffu, d, c);
    return sum;
  };
  auto told_sum = [&]() { return in_order(told(lane < (int)cluster ? lane : 0).d); };
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

  // ---- the row, at its own offset within a 16-byte word (what else is in its first and its last word is masked), and its maximum
  const int skew = (int)(((uintptr_t)src & 15) / sizeof(T)), all_words = cnt > 0 ? (skew + cnt + W - 1) / W : 0;
  const uint4* words = reinterpret_cast<const uint4*>(sp_smem);
  T* part = reinterpret_cast<T*>(sp_smem) + skew;
  const int head = min(cnt, skew ? W - skew : 0), whole_words = (cnt - head) / W, tail = head + whole_words * W;
#pragma unroll 4
  for (int i = tid; i < whole_words; i += kSpThreads)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(part + head + i * W)), "l"(src + head + (size_t)i * W) : "memory");
  cp_async_commit();
  float top = -INFINITY;
  if (tid < head) part[tid] = src[tid], top = Elem<T>::ld(part + tid);
  if (tid < cnt - tail) part[tail + tid] = src[tail + tid], top = sp_max(top, Elem<T>::ld(part + tail + tid));
  if (tid < skew && cnt > 0) Elem<T>::st(part - 1 - tid, -INFINITY);
  if (tid < all_words * W - skew - cnt) Elem<T>::st(part + cnt + tid, -INFINITY);
  float heat = a.heat ? a.heat[row] : 1.f;
  int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f, m = a.min_p ? a.min_p[row] : 0.f;
  const float u = a.tokens ? a.u[row] : 0.f;
  if (tid < kSpTable) s_roots[tid] = root;
  cp_async_wait<0>();
#pragma unroll 4
  for (int i = tid; i < whole_words; i += kSpThreads) top = sp_word_max<T>(*reinterpret_cast<const uint4*>(part + head + i * W), top);
  // The maximum, as its key (NaN above everything), and the maxima of groups of lanes (where a row may ask for its k largest): up to 512 over the cluster.
  uint32_t peak = sp_key(top);
  const int log_group = cluster <= 2 ? 0 : 30 - __clz(cluster), groups = kSpThreads >> log_group;
  if (a.top_k) {
    uint32_t g = peak;
    for (int d = 1; d < 1 << log_group; d *= 2) g = max(g, __shfl_xor_sync(0xffffffffu, g, d));
    if ((tid & ((1 << log_group) - 1)) == 0) s_work.groups[tid >> log_group] = g;
  }
  peak = __reduce_max_sync(0xffffffffu, peak);
  if (lane == 0) s_tops[warp] = peak;
  __syncthreads();
  peak = __reduce_max_sync(0xffffffffu, s_tops[lane & (kSpWarps - 1)]);
  if (cluster > 1) {
    if (tid == 0) s_top = peak;
    meet();
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(peak) : "r"(map_to_rank(smem_u32(&s_top), (uint32_t)(lane < (int)cluster ? lane : 0))) : "memory");
    peak = __reduce_max_sync(0xffffffffu, peak);
  }
  top = sp_logit(peak);

  auto logit = [&](int i) { return Elem<T>::ld(part + i); };
  float* probs = a.probs ? a.probs + (size_t)row * a.n + i0 : nullptr;
  const bool nothing = !(top < INFINITY) || top == -INFINITY;       // no class, or NaN or +inf among the logits
  const bool first = !(heat > 0.f) || k == 1 || p <= 0.f || m > 1.f;   // only the first stays
  if (k < 0 || k >= a.n) k = 0;
  const bool by_p = p < 1.f, by_m = m > 0.f;
  auto fill = [&](float v) {               // this CTA's part of the probabilities
    const int skip = min(cnt, (int)(-((uintptr_t)probs >> 2) & 3));
    float4* mid = reinterpret_cast<float4*>(probs + skip);
    const int quads = (cnt - skip) / 4;
    if (tid < skip) probs[tid] = v;
    for (int i = tid; i < quads; i += kSpThreads) mid[i] = make_float4(v, v, v, v);
    if (tid < cnt - skip - 4 * quads) probs[skip + 4 * quads + tid] = v;
  };
  int token = -1;                          // of this CTA: the one that has it stores it
  bool mine = rank == 0;
  if (nothing) {
    if (probs) fill(top == -INFINITY ? 0.f : NAN);
  } else if (first) {
    int at = 0x7fffffff;
    for (int i = tid; i < cnt; i += kSpThreads)
      if (at == 0x7fffffff && logit(i) == top) at = i0 + i;
    at = __reduce_min_sync(0xffffffffu, at);
    if (tid == 0) s_int = 0x7fffffff;
    __syncthreads();
    if (lane == 0) atomicMin(&s_int, at);
    __syncthreads();
    tell(0.0, s_int);
    token = __reduce_min_sync(0xffffffffu, told(lane < (int)cluster ? lane : 0).i);
    if (probs) {
      fill(0.f);
      __syncthreads();
      if (tid == 0 && token >= i0 && token - i0 < cnt) probs[token - i0] = 1.f;
    }
  } else {
    const float lift = heat < 1e-20f && fabsf(top) < 1e-10f ? 0x1p64f : 1.f;
    if (lift > 1.f) {
      // So cold that logits below 2^-126 matter, which sp_wide does not tell apart: all of them times 2^64, and the temperature.  What overflows weighs nothing either way.
      for (int i = tid; i < cnt; i += kSpThreads) Elem<T>::st(part + i, logit(i) * lift);
      heat *= lift, top *= lift;
      __syncthreads();
    }
    const SpWeight weight(s_roots, heat, top);
    const int blocks = (all_words + kBlockWords - 1) / kBlockWords;
    // The last member: what is above it by logit, or beside it and not behind it by index, is kept.
    float last = -INFINITY;
    int last_at = 0x7fffffff;
    auto kept = [&](float l, int i) { return l > last || (l == last && i0 + i <= last_at); };

    // Of what is kept, the new last member: by count (the goal-th), or by weight (the last before which there is less than goal; all of it weighs `sum`).
    // Weights are added as whole numbers, in any order.  Their unit is the power of 2 between 2^-62 and 2^-63 of the sum: n of them are off by n 2^-63 of it at most, 2^-43.7, where chains of fp64
    // additions could be by n 2^-53.  (In units of 2^-43 a top_p of 1 - 2^-24 over 262144 classes ended in another class in one row of four.)
    auto select = [&](bool by_weight, double goal, double sum) {
      constexpr int kRounds = sizeof(T) == 2 ? 2 : 4;      // a bf16's bits end after two digits
      uint32_t prefix = 0u;
      uint32_t above = 0u;
      unsigned long long above_m = 0ull;
      const double units = __hiloint2double((int)((2u * 1023u + 62u << 20) - ((unsigned)__double2hiint(sum) & 0x7ff00000u)), 0);      // of 1: 2^62 over the power of 2 in the sum, which is 1 at least
      const unsigned long long goal_m = (unsigned long long)ceil(goal * (by_weight ? units : 1.0));       // below 2^63
      int in = 0;
#pragma unroll 1
      for (int r = 0; r < kRounds; ++r) {
        const int shift = 24 - 8 * r;
        SpHist& h = s_work.hist[r & 1];
        h.count[tid] = 0u, h.mass[tid] = 0ull;
        __syncthreads();
        for (int i = tid; i < cnt; i += kSpThreads) {
          const float l = logit(i);
          const uint32_t key = sp_key(l);
          if ((r == 0 || key >> (shift + 8) == prefix) && kept(l, i)) {
            const int d = key >> shift & 255;
            atomicAdd(&h.count[d], 1u);
            if (by_weight) atomicAdd(&h.mass[d], (unsigned long long)__double2ull_rn(weight(l) * units));
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
      const float border = sp_logit(key);
      int take;
      if (by_weight) {
        double v = 0.0;                                    // what lies above, exactly
        for (int i = tid; i < cnt; i += kSpThreads) {
          const float l = logit(i);
          if (l > border && kept(l, i)) v += weight(l);
        }
        tell(cta_sum(v), 0);
        v = told_sum();
        const double w = weight(border);
        take = w > 0.0 ? (int)fmin(fmax(ceil((goal - v) / w), 1.0), (double)in) : in;
      } else {
        take = (int)goal - (int)above;
      }
      int at = 0x7fffffff;
      if (take < in) {
        int c = 0;
        for (int i = tid; i < cnt; i += kSpThreads) c += logit(i) == border && kept(border, i);
        c = __reduce_add_sync(0xffffffffu, c);
        if (tid == 0) s_int = 0;
        __syncthreads();
        if (lane == 0) atomicAdd(&s_int, c);
        __syncthreads();
        const int have = s_int;
        tell(0.0, have);
        int before = 0;
        for (int c2 = 0; c2 < (int)rank; ++c2) before += told(c2).i;
        // the CTA that has the take-th looks for its index
        if (tid == 0) s_int = 0;
        __syncthreads();
        if (before < take && take <= before + have && warp == 0) {
          int left = take - before;
          for (int i = lane; i - lane < cnt; i += 32) {
            const unsigned b = __ballot_sync(0xffffffffu, i < cnt && logit(min(i, cnt - 1)) == border && kept(border, i));
            if (__popc(b) >= left) {
              const int j = __fns(b, 0, left);
              if (lane == 0) s_int = i0 + i + j;
              break;
            }
            left -= __popc(b);
          }
        }
        __syncthreads();
        tell(0.0, s_int);
        at = 0;
        for (int c2 = 0; c2 < (int)cluster; ++c2) at = max(at, told(c2).i);      // the others say 0
      }
      if (border == last && take >= in) at = last_at;      // of the same logit, what was kept before
      last = border, last_at = at;
    };

    // ---- few candidates.  Bins of width 1 / scale in the logit, below the maximum; what lies beyond the last of them is no candidate.
    const int n_bins = cluster == 1 ? kSpBins / 2 : kSpBins;          // four a thread at most
    float scale = 0.f, base = 0.f, zoom = 1.f;        // looked at closer, the bins divide what lies from `base` on
    double octaves = 0.0;                  // of all bins, for weights
    // In bins below `base`.  Rounded step by step wherever it is asked: a logit lies in one bin only.
    auto far_of = [&](float l) { return __fmul_rn(__fsub_rn(top, l), scale); };
    auto place = [&](float l) { return __fmul_rn(__fsub_rn(far_of(l), base), zoom); };
    // The list: members whose place lies in [f0, f1); in the first CTA that of all CTAs, in order, with their weights, in another its own.  by_weight: and the exact sum of the row in sum_all, of blocks of what lies above them in s_block, and of
    // the row of those in s_double.  Returns how many members there are, or -1: more than the list has room for.
    double sum_all = 0.0;
    int own = 0;                           // members of this CTA's part
    auto gather = [&](float f0, float f1, bool by_weight) {
      const int list_room = min(2 * kSpList / (int)cluster, kSpList);
      if (tid == 0) s_int = 0;
      __syncthreads();
      double row_sum = 0.0;
      constexpr int kWords = kBlockWords / 32;         // of a lane and block
#pragma unroll 1
      for (int b0 = warp; b0 < blocks; b0 += 4 * kSpWarps) {
        // Four blocks' members as 64 bits of a lane, put away together: put away one by one, with an atomic each, they took twice the time of everything else here.
        unsigned long long hits = 0ull;
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          const int b = b0 + q * kSpWarps;
          if (b >= blocks) break;
          double sum = 0.0;
#pragma unroll 1
          for (int j = 0; j < kWords; ++j) {
            const int w = b * kBlockWords + j * 32 + lane;
            if (w >= all_words) break;
            const uint4 word = words[w];
            Vec16<T> v;
            v.unpack(word);
            unsigned in = 0u;
            if (by_weight) {
#pragma unroll
              for (int e = 0; e < W; ++e) {
                const double g = weight(v.v[e]);
                const float f = place(v.v[e]);
                row_sum += g, sum += sp_pick(f < f0, g);
                if (f >= f0 && f < f1) in |= 1u << e;
              }
            } else if (place(sm_word_max<T>(word, -INFINITY)) < f1) {
#pragma unroll
              for (int e = 0; e < W; ++e) {
                const float f = place(v.v[e]);
                if (f >= f0 && f < f1) in |= 1u << e;
              }
            }
            hits |= (unsigned long long)in << ((q * kWords + j) * W);
          }
          if (by_weight) {
            sum = warp_total(sum);
            if (lane == 0) s_block[b] = sum;
          }
        }
        if (__any_sync(0xffffffffu, hits != 0ull)) {
          const int count = __popcll(hits);
          int at = count;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, at, d);
            if (lane >= d) at += o;
          }
          int first = 0;
          if (lane == 31) first = atomicAdd(&s_int, at);
          at += __shfl_sync(0xffffffffu, first, 31) - count;
          for (; hits; hits &= hits - 1ull, ++at) {
            const int bit = __ffsll((long long)hits) - 1, seq = bit / W;
            const int i = ((b0 + seq / kWords * kSpWarps) * kBlockWords + seq % kWords * 32 + lane) * W + bit % W - skew;
            if (at < list_room) s_work.list[at] = (unsigned long long)sp_key(logit(i)) << 32 | (uint32_t)~(i0 + i);
          }
        }
      }
      if (by_weight) row_sum = cta_sum(row_sum);
      __syncthreads();
      double above = 0.0;
      if (by_weight)
        for (int b = 0; b < blocks; b += 32) above += warp_total(b + lane < blocks ? s_block[b + lane] : 0.0);
      // to the first CTA, in places of this CTA's own
      const int room = 2 * kSpList / (int)cluster;
      own = s_int;
      for (int i = tid; i < min(own, list_room); i += kSpThreads)
        asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(map_to_rank(smem_u32(&s_work.all[rank * room + i]), 0u)), "l"(s_work.list[i]) : "memory");
      if (tid < (int)cluster) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_rank(smem_u32(&s_counts[rank]), (uint32_t)tid)), "r"(own) : "memory");
      tell(above, 0, row_sum);
      if (by_weight) {
        const SpSlot o = told(lane < (int)cluster ? lane : 0);
        above = in_order(o.d), sum_all = in_order(o.e);
        if (tid == 0) s_double = above;
      }
      int upto = lane < (int)cluster ? min(s_counts[lane], room + 1) : 0;
      const bool spilt = __any_sync(0xffffffffu, upto > room);
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += v;
      }
      const int members = __shfl_sync(0xffffffffu, upto, (int)cluster - 1);
      if (spilt || members > kSpList) return -1;
      if (rank != 0) return members;
      // side by side, then in order: a member's place is the number of those in front of it (four lanes a member)
      for (int i = tid; i - lane < members; i += kSpThreads) {
        int from_cta = 0, start = 0;
        for (int c = 0; c < (int)cluster - 1; ++c) {
          const int end = __shfl_sync(0xffffffffu, upto, c);
          if (i >= end) from_cta = c + 1, start = end;
        }
        if (i < members) s_work.list[i] = s_work.all[from_cta * room + i - start];
      }
      __syncthreads();
      for (int i = tid >> 2; i - (lane >> 2) < members; i += kSpThreads / 4) {
        const unsigned long long e = s_work.list[min(i, members - 1)];
        int place = 0;
#pragma unroll 8
        for (int j = lane & 3; j < members; j += 4) place += s_work.list[j] > e;
        place += __shfl_xor_sync(0xffffffffu, place, 1);
        place += __shfl_xor_sync(0xffffffffu, place, 2);
        if (i < members && (lane & 3) == 0) {
          s_work.sorted[place] = e;
          s_work.weight[place] = weight(sp_logit((uint32_t)(e >> 32)));
        }
      }
      __syncthreads();
      return members;
    };
    // Counts or weighs candidates in bins and finds those, [from, to], in which the goal lies: `goal` in members, or in parts of the sum (both in fp32, and so known to some 10^-5: where
    // the goal lies nearer than that to a border of bins, both of its sides are taken).  Returns what lies above them, in members (by_weight: at most as many), or -1.
    int from = 0, to = n_bins - 1, inside = 0;
    int count0 = 0;                        // what lies above `base`
    double weight0 = 0.0, border_weight = 0.0, sum_row = 0.0;
    auto look = [&](bool by_weight, double goal) {
      for (int i = tid; i < n_bins; i += kSpThreads) s_work.bins[i] = 0u;
      __syncthreads();
      float sum = 0.f;
      const float drop = -(float)octaves / n_bins, fall = 0.69314718f * drop / zoom;   // of a bin, as powers of 2 and of e
#pragma unroll 1
      for (int w = tid; w < all_words; w += kSpThreads) {
        Vec16<T> v;
        v.unpack(words[w]);
#pragma unroll
        for (int e = 0; e < W; ++e) {
          // Conversions by sums with 2^23: the instructions take 8 clocks a warp.
          const float far = far_of(v.v[e]), f = place(v.v[e]), down = __fadd_rd(f, 8388608.f);
          uint32_t member = 1u;
          if (by_weight) {
            float g;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(g) : "f"(far * drop));
            sum += g;
            const float y = (f - (down - 8388608.f)) * fall;       // exp(y) to y^4 / 24, 3e-8
            member = __float_as_uint(fmaf(fmaf(fmaf(131072.f / 6.f, y, 0.5f * 131072.f), y, 131072.f), y, 131072.f + 8388608.f)) - 0x4b000000u;       // 17 bits; a part has fewer than 2^15 members
          }
          const uint32_t bin = __float_as_uint(down) - 0x4b000000u;       // beyond all bins where f is below 0, or no number
          if (bin < (uint32_t)n_bins) atomicAdd(&s_work.bins[bin], member);
        }
      }
      if (by_weight) {
        tell(cta_sum((double)sum), 0);
        sum_row = told_sum();                // the same when looked at closer
        goal *= sum_row;
      } else {
        meet();
      }
      // This CTA adds up its part of the bins over the cluster (all of them would be 32 KB from other SMs, at 16 bytes a clock).
      const int share = n_bins / (int)cluster, each = max(1, share / kSpThreads), bin0 = (int)rank * share + tid * each;
      const bool has = tid * each < share;
      uint32_t v[4] = {0u, 0u, 0u, 0u};
      double m[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (has && j < each) {
          double sum_m = 0.0;
#pragma unroll 8
          for (int c = 0; c < (int)cluster; ++c) {
            uint32_t w;
            asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(w) : "r"(map_to_rank(smem_u32(&s_work.bins[bin0 + j]), (uint32_t)c)) : "memory");
            if (by_weight) sum_m += __hiloint2double(0x43300000, (int)w) - 4503599627370496.0;       // as a double
            else v[j] += w;
          }
          if (by_weight) {
            v[j] = (uint32_t)(sum_m * (1.0 / 131072) * 1.04) + (sum_m > 0.0);        // a bin is 0.043 octaves wide at most: never fewer than there are
            float g;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(g) : "f"(drop * (base + (float)(bin0 + j) / zoom)));
            m[j] = sum_m * (double)g * (1.0 / 131072);
          }
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
      uint32_t sum_c = 0u;
      double sum_w = 0.0;
#pragma unroll
      for (int w = 0; w < kSpWarps; ++w) {
        if (w == warp) cc += sum_c, cm += sum_w;
        sum_c += s_scan_c[w], sum_w += s_warp[w];
      }
      if (tid == 0) s_border = SpBorder{kSpBins, 0, -1, 0, 0.0};
      if (cluster > 1) {                   // what the CTAs in front have
        tell(sum_w, (int)sum_c);
        const SpSlot o = told(lane < (int)cluster ? lane : 0);
        for (int c = 0; c < (int)rank; ++c) cc += (uint32_t)__shfl_sync(0xffffffffu, o.i, c), cm += __shfl_sync(0xffffffffu, o.d, c);
      } else {
        __syncthreads();
      }
      uint32_t before = (uint32_t)count0 + cc - c4;
      double before_m = weight0 + cm - m4;
      // What lies before a bin, against the goal, is off by 1.8e-5 of the sum at most.  A rounding of an exponent of z octaves is z 2^-24 ln 2 of a weight; weighed, the mean z is at most the
      // entropy of the row, log2 n < 19, so that each counts 7.9e-7.  Four in a logit's place (difference, product, the two constants), in the row's sum and the bins alike: 3.2e-6.  In the sum the
      // exponent's product 0.8e-6, the power 0.3e-6, up to 136 additions a thread 8.1e-6.  In the bins half a unit of a share of 127000 or more 3.9e-6, the exponent of a bin's largest weight (its
      // place, looked at closer, and the product) 1.6e-6, the power 0.3e-6.
      const double slack = by_weight ? 2e-5 * sum_row : 0.0;
      int first_bin = kSpBins, last_bin = -1, first_before = 0, last_end = 0;
      double first_weight = 0.0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (v[j] > 0u) {
          const bool starts = by_weight ? before_m + m[j] >= goal - slack : (double)(before + v[j]) >= goal, ends = by_weight ? before_m < goal + slack : (double)before < goal;
          if (starts && first_bin == kSpBins) first_bin = bin0 + j, first_before = (int)before, first_weight = before_m;
          if (ends) last_bin = bin0 + j, last_end = (int)(before + v[j]);
        }
        before += v[j], before_m += m[j];
      }
      const int wf = __reduce_min_sync(0xffffffffu, first_bin), wl = __reduce_max_sync(0xffffffffu, last_bin);
      if (lane == 0 && wf < kSpBins) atomicMin(&s_border.from, wf);
      if (lane == 0 && wl >= 0) atomicMax(&s_border.to, wl);
      __syncthreads();
      if (first_bin < kSpBins && first_bin == s_border.from) s_border.before = first_before, s_border.weight = first_weight;
      if (last_bin >= 0 && last_bin == s_border.to) s_border.end = last_end;
      SpBorder o;
      meet();
      {
        const uint32_t at = map_to_rank(smem_u32(&s_border), (uint32_t)(lane < (int)cluster ? lane : 0));
        asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(o.from), "=r"(o.before), "=r"(o.to), "=r"(o.end) : "r"(at) : "memory");
        asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(o.weight) : "r"(at + 16u) : "memory");
      }
      from = __reduce_min_sync(0xffffffffu, o.from), to = __reduce_max_sync(0xffffffffu, o.to);
      if (to < 0) return -1;
      const int has_from = __ffs(__ballot_sync(0xffffffffu, o.from == from)) - 1, has_to = __ffs(__ballot_sync(0xffffffffu, o.to == to)) - 1;
      const int end = __shfl_sync(0xffffffffu, o.end, has_to);
      int above = __shfl_sync(0xffffffffu, o.before, has_from);
      border_weight = __shfl_sync(0xffffffffu, o.weight, has_from);
      if (from > to) return -1;              // the sum of all bins falls short of the goal
      inside = end - above;
      return above;
    };

    bool listed = false, direct = false;   // worth a list; without a look at the bins
    double goal = 0.0;
    if (k && k <= kSpThreads) {
      // A logit that k of the groups' maxima reach, by halving what lies between the smallest and the largest, until no more than a quarter more do.
      if (warp == 0) {
        uint32_t v[16], low = 0xffffffffu;      // 16 maxima a lane
        int some = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int at = j * 32 + lane;
          v[j] = 0u;
          if (at < groups * (int)cluster)
            asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v[j]) : "r"(map_to_rank(smem_u32(&s_work.groups[at & (groups - 1)]), (uint32_t)at / (uint32_t)groups)) : "memory");
        }
        const bool fold = k <= 64;              // 128 groups are enough
        if (fold)
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = max(max(v[j], v[j + 4]), max(v[j + 8], v[j + 12]));
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (v[j] <= sp_key(-INFINITY) || (fold && j >= 4)) v[j] = 0u;          // has none
          else low = min(low, v[j]), ++some;
        }
        low = __reduce_min_sync(0xffffffffu, low), some = __reduce_add_sync(0xffffffffu, some);
        uint32_t high = peak;
        for (int t = 0; t < 20 && some > max(k + k / 4, 32) && high - low > 1; ++t) {
          const uint32_t mid = low + (high - low) / 2;
          int c = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) c += v[j] >= mid;
          if (!fold)
#pragma unroll
            for (int j = 4; j < 16; ++j) c += v[j] >= mid;
          c = __reduce_add_sync(0xffffffffu, c);
          if (c >= k) low = mid, some = c;
          else high = mid;
        }
        if (lane == 0) s_int = some >= k ? (int)low : 0;
      }
      __syncthreads();
      const uint32_t low = (uint32_t)s_int;
      scale = fminf(0.9995f * (float)n_bins / (top - sp_logit(low) * lift), FLT_MAX);
      listed = low != 0u && scale > 0.f;
      direct = true;
      goal = (double)k;
      meet();                              // the maxima have been read: the lists come in their place
    } else if (!k && by_p) {
      octaves = (log2((double)a.n) - log2(1.0 - (double)p)) * 1.0001;     // 1 - p is exact; the total is 1 at least
      scale = (float)(n_bins * weight.c / octaves);
      listed = scale > 0.f && scale < FLT_MAX && a.per <= 32767;
      goal = (double)p;
    }
    bool whole = false;                    // the list holds all that is kept
    bool summed = false;                   // s_block holds the sums of what is kept
    int members = -1, above = 0, cut = 0;
    double total = 0.0;
    if (listed) {
#pragma unroll 1
      for (;;) {
        bool complete = direct;
        if (!direct) {
          above = look(!k, goal);
          complete = above >= 0 && above + inside <= kSpList;
          if (above < 0) break;
          if (!complete && inside > kSpList) {
            const float closer = 0.9995f * (float)n_bins / (float)(to - from + 1);
            if (zoom > 1.f || !(closer > 1.f)) break;           // equal logits, then; or the goal may lie in any bin (a class with all but some 10^-5 of the weight, and p beyond it): no closer look to take
            base = (float)from, zoom = closer;        // `far` - base is exact: what lay in these bins lies in the new ones, and nothing else
            count0 = above, weight0 = border_weight;
            continue;
          }
        }
        members = gather(complete ? -FLT_MAX : (float)from, (float)(to + 1), !k);
        whole = complete && members > 0;
        if (!direct || members >= 0) break;
        direct = false;
      }
    }
    if (whole && rank == 0) {
      // all from the list: what is kept of it, and their total.  Running sums by warps of 32, then over those in front.
      if (k) members = min(members, k);
      double w[2], cum[2];
      static_assert(kSpList == 2 * kSpThreads, "a thread has two members");
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int i = r * kSpThreads + tid;
        w[r] = i < members ? s_work.weight[i] : 0.0, cum[r] = 0.0;
        if (i - lane < members) {
          cum[r] = warp_scan(w[r], lane);
          if (lane == 31) s_chunk[i >> 5] = cum[r];
        }
      }
      __syncthreads();
      double want = INFINITY, sum = 0.0;
#pragma unroll
      for (int c = 0; c < kSpList / 32; ++c) {
        if (c * 32 < members) {
          if (c == warp) cum[0] += sum;
          if (c == warp + kSpWarps) cum[1] += sum;
          sum += s_chunk[c];
        }
      }
      if (by_p) want = (double)p * (k ? sum : sum_all);
      cut = 0;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int i = r * kSpThreads + tid;
        if (r * kSpThreads < members) cut += __syncthreads_count(i < members && ((cum[r] - w[r] < want && !(by_m && w[r] < (double)m)) || i == 0));
      }
#pragma unroll
      for (int r = 0; r < 2; ++r)
        if (r * kSpThreads + tid == cut - 1) s_double = cum[r];
      if (tid == 0) s_int = 0x7fffffff, s_int2 = -1;
      __syncthreads();
      total = s_double;
      const unsigned long long e = s_work.sorted[cut - 1];
      if (tid == 0) s_kept = SpKept{sp_logit((uint32_t)(e >> 32)), (int)~(uint32_t)e, total};
      if (a.tokens) {
        // by index: the first class with which the running sum passes the goal; or the last that weighs anything (four lanes a member)
        goal = fmax((double)u * total, 0.0);
        for (int i = tid >> 2; i - (lane >> 2) < cut; i += kSpThreads / 4) {
          const uint32_t at = (uint32_t)s_work.sorted[min(i, cut - 1)];          // the larger, the lower the index
          const double g = s_work.weight[min(i, cut - 1)];
          double before = 0.0;
#pragma unroll 8
          for (int j = lane & 3; j < cut; j += 4) before += sp_pick((uint32_t)s_work.sorted[j] > at, s_work.weight[j]);
          before += __shfl_xor_sync(0xffffffffu, before, 1);
          before += __shfl_xor_sync(0xffffffffu, before, 2);
          if (g > 0.0 && i < cut && (lane & 3) == 0) {
            if (before + g > goal) atomicMin(&s_int, (int)~at);
            atomicMax(&s_int2, (int)~at);
          }
        }
        __syncthreads();
        token = s_int != 0x7fffffff ? s_int : s_int2;
      }
    }
    bool need_k = k != 0, need_p = by_p;
    if (!whole && members > 0) {
      if (rank == 0) {
        if (k) {                             // the bin in which the k-th lies
          cut = k - above;
        } else {                             // the bins in which the p-th part ends
          if (warp == 0) {
            double before = s_double;
            int j = 0;
            for (int i = 0; i < members; i += 32) {
              const double w = i + lane < members ? s_work.weight[i + lane] : 0.0, cum = before + warp_scan(w, lane);
              j += __popc(__ballot_sync(0xffffffffu, i + lane < members && cum - w < goal * sum_all));
              before = __shfl_sync(0xffffffffu, cum, 31);
            }
            if (lane == 0) s_int = max(j, 1);
          }
          __syncthreads();
          cut = s_int;
        }
        const unsigned long long e = s_work.sorted[cut - 1];
        if (tid == 0) s_kept = SpKept{sp_logit((uint32_t)(e >> 32)), (int)~(uint32_t)e, 0.0};
      } else if (!k && !by_m) {
        // This CTA's members, in order, for the sums of its blocks.
        cut = own;
        for (int i = tid >> 2; i - (lane >> 2) < own; i += kSpThreads / 4) {
          const unsigned long long e = s_work.list[min(i, own - 1)];
          int place = 0;
#pragma unroll 4
          for (int j = lane & 3; j < own; j += 4) place += s_work.list[j] > e;
          place += __shfl_xor_sync(0xffffffffu, place, 1);
          place += __shfl_xor_sync(0xffffffffu, place, 2);
          if (i < own && (lane & 3) == 0) {
            s_work.sorted[place] = e;
            s_work.weight[place] = weight(sp_logit((uint32_t)(e >> 32)));
          }
        }
      }
      need_k = need_k && !k, need_p = need_p && k;
      summed = !k && !by_m;
    }
    if (members > 0 && !(whole && !probs && u > 0.f)) {      // everybody needs to know
      meet();
      const uint32_t at = map_to_rank(smem_u32(&s_kept), 0u);
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(last) : "r"(at) : "memory");
      asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(last_at) : "r"(at + 4u) : "memory");
      if (whole) asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(total) : "r"(at + 8u) : "memory");
    }
    if (!whole) {
#pragma unroll 1
      for (int by_weight = 0; by_weight < 2; ++by_weight) {
        if (!(by_weight ? need_p : need_k)) continue;
        double v = 0.0;
        if (by_weight) {
          for (int i = tid; i < cnt; i += kSpThreads) {
            const float l = logit(i);
            if (kept(l, i)) v += weight(l);
          }
          tell(cta_sum(v), 0);
          v = told_sum();
        }
        select(by_weight != 0, by_weight ? (double)p * v : (double)k, v);
      }
    }
    const double least = by_m ? (double)m : 0.0;
    const bool all = last == -INFINITY;
    auto mass = [&](float l, int i) {      // what class i adds to the sum
      if (!kept(l, i)) return 0.0;
      const double w = weight(l);
      return sp_pick(w >= least, w);
    };
    if (!whole) {
      // ---- sums of blocks, the total, and the block in which the running sum passes its goal
      if (summed) {
        // those of the list that are kept join their blocks, in order
        for (int b = warp; b < blocks; b += kSpWarps) {
          double s = 0.0;
          for (int j = lane; j < cut; j += 32) {
            const int at = (int)~(uint32_t)s_work.sorted[j] - i0;
            s += sp_pick(at >= 0 && at < cnt && (at + skew) / kSpBlock == b && kept(sp_logit((uint32_t)(s_work.sorted[j] >> 32)), at), s_work.weight[j]);
          }
          s = warp_total(s);
          if (lane == 0) s_block[b] += s;
        }
      } else {
#pragma unroll 1
        for (int b = warp; b < blocks; b += kSpWarps) {
          double s = 0.0;
#pragma unroll 1
          for (int w = b * kBlockWords + lane; w < min((b + 1) * kBlockWords, all_words); w += 32) {
            Vec16<T> v;
            v.unpack(words[w]);
            if (all && !by_m) {
#pragma unroll
              for (int e = 0; e < W; ++e) s += weight(v.v[e]);
            } else {
#pragma unroll
              for (int e = 0; e < W; ++e) {
                const double g = weight(v.v[e]);
                s += sp_pick(g >= least && kept(v.v[e], w * W + e - skew), g);
              }
            }
          }
          s = warp_total(s);
          if (lane == 0) s_block[b] = s;
        }
      }
      __syncthreads();
      double sum = 0.0;
      for (int b = 0; b < blocks; b += 32) sum += warp_total(b + lane < blocks ? s_block[b + lane] : 0.0);
      tell(sum, 0);
      const double o = told(lane < (int)cluster ? lane : 0).d;
      double before = 0.0;
      int last_one = 0;                    // the last CTA that has any weight
      for (int c = 0; c < (int)cluster; ++c) {
        const double v = __shfl_sync(0xffffffffu, o, c);
        if (c == (int)rank) before = total;
        if (v > 0.0) last_one = c;
        total += v;
      }
      if (a.tokens) {
        goal = fmax((double)u * total, 0.0);
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
          const int end = min((at + 1) * kSpBlock - skew, cnt);
          bool found = false;
          for (int i = max(at * kSpBlock - skew, 0) + lane; i - lane < end && !found; i += 32) {
            const double w = i < end ? mass(logit(i), i) : 0.0, cum = start + warp_scan(w, lane);
            const unsigned over = __ballot_sync(0xffffffffu, w > 0.0 && cum > goal), some = __ballot_sync(0xffffffffu, w > 0.0);
            if (some) token = i0 + i - lane + (over ? __ffs(over) - 1 : 31 - __clz(some));
            found = over != 0;
            start = __shfl_sync(0xffffffffu, cum, 31);
          }
        }
      }
    }
    if (a.tokens && !(u > 0.f)) {          // u is 0: the first that weighs anything, however little
      int at = 0x7fffffff;
      for (int i = tid; i < cnt; i += kSpThreads) {
        const float l = logit(i);
        if (at == 0x7fffffff && kept(l, i) && weight.live(l) && !(by_m && weight(l) < (double)m)) at = i0 + i;
      }
      at = __reduce_min_sync(0xffffffffu, at);
      __syncthreads();
      if (tid == 0) s_int = 0x7fffffff;
      __syncthreads();
      if (lane == 0) atomicMin(&s_int, at);
      __syncthreads();
      tell(0.0, s_int);
      token = __reduce_min_sync(0xffffffffu, told(lane < (int)cluster ? lane : 0).i);
      mine = rank == 0;
    }
    if (probs) {
      // w / total in fp32: the exponent's fraction to 2^-23, the power to two units.  Who weighs at least m is asked in fp64, where the last member does not say it.
      const float ch = fminf((float)weight.c, FLT_MAX), cl = ch < FLT_MAX ? (float)(weight.c - (double)ch) : 0.f, part_of = (float)(1.0 / total);
      auto prob = [&](float l) {
        const float d = l - top, r = fmaf(d, ch, 12582912.f), z = r - 12582912.f;
        float g;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(g) : "f"(fmaf(d, cl, fmaf(d, ch, -z))));
        g *= part_of * __int_as_float(max(__float_as_int(r) - 0x4b400000 + 127, 0) << 23);
        return z >= -126.f ? g : 0.f;
      };
      if (whole) {                         // few: zeros, and over them what the list has
        fill(0.f);
        __syncthreads();
        for (int j = tid; j < (rank == 0 ? cut : own); j += kSpThreads) {
          const unsigned long long e = rank == 0 ? s_work.sorted[j] : s_work.list[j];
          const float l = sp_logit((uint32_t)(e >> 32));
          const int i = (int)~(uint32_t)e - i0;
          if (i >= 0 && i < cnt && kept(l, i)) probs[i] = prob(l);
        }
      } else {
#pragma unroll 4
        for (int i = tid; i < cnt; i += kSpThreads) {
          const float l = logit(i);
          probs[i] = kept(l, i) && (!by_m || weight(l) >= least) ? prob(l) : 0.f;
        }
      }
    }
  }
  if (a.tokens && mine && tid == 0) a.tokens[row] = token;
  if (cluster > 1) asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");   // nobody reads this CTA's shared memory any more
}

template <typename T>
inline size_t sample_smem(int per) { return align_up((size_t)per * sizeof(T), 16) + 32; }

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
