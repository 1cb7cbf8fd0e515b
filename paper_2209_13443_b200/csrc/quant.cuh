// Rows in 8 bits, and the projection of such rows.
//
// quantise: s = max |x| (1 / 127) of a row, both rounded to fp32, and q = the integer nearest to x / s, of two the even one.  The quotient is meant, not its rounding to
// fp32: n, x times 1 / s rounded, is that integer or, within 3e-5 of the middle of two, its neighbour.  e = x - n s is one multiply-add and exact (a multiple of the last place of s, or of x where
// |x| < s, and not much above s / 2), so |e| against s / 2 says which, and where the middle is hit.  A row is read once and kept in the registers of 8 lanes to 16 warps, up to four
// 16-byte words a lane; longer rows are read twice, from L2 the second time.
// 50176 x 512 bf16: 15 us of 11.8 that its bytes take, 4096 x 4096 11.5 of 7.7; fp32 20.6 of 19.6 and 25 of 12.8 (rows above 2048 take a CTA of 512 threads, two an SM: a warp waits 6.6 of the 16
// clocks between two issues for its loads); 89 instructions for eight values of a warp's lanes.  With the neighbours of a middle told by their distance to it,
// 3e-5 either way, 117 and 18 us: of values with 8 bits a great many lie that near, and most warps went the rare way.  Tried and taken
// back: rows copied ahead into shared memory (20 us), persistent CTAs with the next row in registers (19), two multiply-adds an instruction (nothing; the moves to pairs).
//
// dequantise: y = q s, rounded once.  Rows in any order.  12544 x 1024 bf16 10 us of 5.9, 50176 x 512 16.5 of 11.8, fp32 14.4 of 9.8 and 27 of 19.6, gathered 0.4 to 4 more.  Bound by its loads' latency: a
// warp waits for them 26 of the 35 clocks between two issues (index, then scale and bytes; nothing of the next row is on its way).
//
// projection: y[t][f] = xs[t] ws[f] sum_k q[t][k] w[f][k] + bias[f], the sum on tcgen05 (kind::i8, 32-bit integers).  A sum of integers is exact, so however
// K is cut and whatever else is in the batch, a row has the same bits.  The tile is turned, as in lowrank.cuh: filters are the rows of the accumulator, whose scale
// and bias a thread keeps in registers, rows of the batch its columns; W, which bounds small batches, is read once.
// Two forms.  Few tiles: a CTA of its own for each, K cut over a cluster whose CTAs send each other their parts as asynchronous stores.  More: CTA pairs
// (cta_group::2), persistent, 256 filters by 256 rows with two accumulators: each SM of a pair fetches half of either operand, 32 KB for 512 clocks of products, which is
// what L2 gives (64 bytes a clock); 128 x 256 tiles of a single SM would need 96.  4096 x 4096 x 4096: 45.5 us (3.0 POP/s, 0.90 of twice the bf16 rate); from bf16 rows 55.  To fp32
// 60 to 65: the epilogue, 7 us a tile (K = 128: 25 us, bf16 16), waits for the fp64 units and the way back from fp64 (4.4 of 13 clocks between two issues), and the last one lies under no product; from
// fp32 rows 90 to 96.
// 64 x 4096 x 4096: 6.7 us, of which its 17 MB take 2.7: the set-up and the first bytes 2, the exchange 1.5, the epilogue 1.
#pragma once
#include "common.cuh"
#include "conv_pair.cuh"
#include "conv_tc.cuh"

namespace ee {

// Longest row of the projection: 128 * 128 * 131071 < 2^31.
constexpr int kQMaxRow = 131071;
__host__ __device__ constexpr int q_pitch(int c) { return (c + 15) / 16 * 16; }   // bytes of a quantised row: TMA wants rows on 16-byte boundaries

// ----------------------------------------------------------------------------- quantise

// The larger magnitude, NaN where either is.
__device__ __forceinline__ float q_max(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// 16 bytes of T.
template <typename T> struct QWord {
  static constexpr int N = 16 / (int)sizeof(T);
  uint32_t w[4];
  __device__ __forceinline__ void set(uint4 t) { w[0] = t.x, w[1] = t.y, w[2] = t.z, w[3] = t.w; }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    return i & 1 ? __uint_as_float(w[i / 2] & 0xffff0000u) : __uint_as_float(w[i / 2] << 16);
  }
  __device__ __forceinline__ float top(float t) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) t = q_max(t, fabsf(at(i)));
      return t;
    } else {                                            // two at a time
      __nv_bfloat162 m[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(&m[i]) = w[i] & 0x7fff7fffu;
      m[0] = __hmax2_nan(__hmax2_nan(m[0], m[1]), __hmax2_nan(m[2], m[3]));
      return q_max(t, q_max(__low2float(m[0]), __high2float(m[0])));
    }
  }
};

struct QScale {
  float s, inv;      // inv 0: everything is 0; s NaN: a row that is not finite
  bool tiny;         // 1 / s is no finite float
  __device__ __forceinline__ explicit QScale(float top) {
    s = top < INFINITY ? top * (1.f / 127.f) : __uint_as_float(0x7fffffffu);
    tiny = s < 1e-37f && s > 0.f;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));       // to 2^-23
    inv = s > 0.f && !tiny ? inv : 0.f;
    // Values of few bits are often (n + 1/2) max / 127: an inverse on the side of 1 / s on which 127 / max is not puts them where s does.
    const float below = fmaf(127.f, s, -top), off = fmaf(inv, s, -1.f);
    if (inv > 0.f && below * off > 0.f) inv = __uint_as_float(__float_as_uint(inv) + (off < 0.f ? 1u : ~0u));
  }
  static __device__ __noinline__ int slow(float x, float s) {
    const double q = rint((double)x / (double)s);
    return (int)fmin(fmax(q, -127.0), 127.0);        // s below 2^-126 has fewer bits: x / s may pass 127
  }
  // A word as bytes, four a register.  By all lanes of a warp.
  template <typename T>
  __device__ __forceinline__ void bytes(const QWord<T>& v, uint32_t* out) const {
    constexpr int N = QWord<T>::N;
    constexpr float kMagic = 12582912.f;             // 1.5 * 2^23: the sum's last place is 1, its low byte the integer
    const float half = 0.5f * s;
    float worst = 0.f, e[N];
    uint32_t b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float x = v.at(i), r = fmaf(x, inv, kMagic);
      b[i] = __float_as_uint(r);
      e[i] = fmaf(kMagic - r, s, x);                 // what is left of x
      worst = fmaxf(worst, fabsf(e[i]));
    }
    // Rare, and so asked for by whole warps: predicated, these were half of all instructions.
    if (__any_sync(0xffffffffu, worst >= half || !(inv > 0.f))) {
      const bool none = !(s > 0.f);
#pragma unroll
      for (int i = 0; i < N; ++i) {                  // more than half is left, or half of an odd integer's
        const uint32_t left = (__float_as_uint(e[i]) & 0x7fffffffu) + (b[i] & 1u);
        if (left > __float_as_uint(half)) b[i] += 1 | (int)__float_as_uint(e[i]) >> 31;
        if (none) b[i] = 0u;
      }
      if (__any_sync(0xffffffffu, tiny)) {
#pragma unroll 1
        for (int i = 0; i < N; ++i) {
          float x = 0.f;
#pragma unroll
          for (int j = 0; j < N; ++j) x = i == j ? v.at(j) : x;
          const uint32_t q = (uint32_t)slow(x, s);
#pragma unroll
          for (int j = 0; j < N; ++j) b[j] = i == j && tiny ? q : b[j];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      out[i] = __byte_perm(__byte_perm(b[4 * i], b[4 * i + 1], 0x0040), __byte_perm(b[4 * i + 2], b[4 * i + 3], 0x0040), 0x5410);
  }
};

constexpr int kQThreads = 256, kQKeep = 4;      // threads of a CTA, words of a lane

// L lanes a row (8, 16, or a warp) and WARPS such groups of it; KEEP words of a lane stay in its registers (0: the row is read again).
// SHIFT: rows that do not all start on 16-byte boundaries.  L lanes then take the aligned words that hold the next L - 1 groups of N values, quantise them (what is not of
// the row counts as 0), and each lane puts its group together from its word's bytes and the next lane's: wide accesses on both sides.
// Nothing that is read here is __restrict__: the kernel starts while the one in front, which may write it, still runs.
// CTAs an SM: as many as their words in registers allow (1000 x 20000 fp32, read twice: 26 us with three, 31 with two; 4096 x 4096 bf16 11.5 with four, 12.1 with no number given).
template <typename T, bool SHIFT, int L, int WARPS, int KEEP>
__global__ void __launch_bounds__(WARPS > 8 ? 32 * WARPS : kQThreads, KEEP == 0 ? 3 : WARPS > 8 ? 2 : sizeof(T) == 4 ? 5 : 4)
quantize_rows_kernel(const T* x, int8_t* q, float* scale, long rows, int c, int pitch) {
  constexpr int N = QWord<T>::N, kRows = (WARPS > 8 ? 32 * WARPS : kQThreads) / (L * WARPS), kWords = SHIFT ? L - 1 : L, kSteps = WARPS * kWords;
  typedef typename std::conditional<N == 8, uint2, uint32_t>::type Group;
  __shared__ uint32_t s_top[WARPS * kRows];
  const int tid = threadIdx.x, lane = tid % L, warp = tid / L % WARPS;      // of the row
  const long row = (long)blockIdx.x * kRows + tid / (L * WARPS);
  // The next launch may start once the past of the stream is over for this one: it may then read what no launch but this one writes.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const bool live = row < rows;
  const T* src = x + (size_t)(live ? row : 0) * c;
  const int skew = SHIFT ? (int)(((uintptr_t)src & 15) / sizeof(T)) : 0;    // what the first aligned word has in front of the row
  const int w0 = warp * kWords + lane, groups = live ? pitch / N : 0;
  const int words = live ? (skew + c + N - 1) / N - w0 : 0;                 // from this lane's first on
  const uint4* from = reinterpret_cast<const uint4*>(src - skew) + w0;
  Group* to = reinterpret_cast<Group*>(q + (size_t)row * pitch) + w0;
  auto load = [&](int k) {                              // word k of this lane's, with zeros in place of what is not of the row
    QWord<T> v;
    if (!SHIFT) {
      v.set(k * kSteps < words ? from[k * kSteps] : make_uint4(0u, 0u, 0u, 0u));
      return v;
    }
    const int lo = skew - (w0 + k * kSteps) * N, hi = lo + c;               // its values in [lo, hi) are the row's
    if (lo <= 0 && hi >= N) {
      v.set(from[k * kSteps]);
    } else {
      v.set(make_uint4(0u, 0u, 0u, 0u));
      const T* p = reinterpret_cast<const T*>(from + k * kSteps);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i >= lo && i < hi && live) {
          if constexpr (sizeof(T) == 4) v.w[i] = *reinterpret_cast<const uint32_t*>(p + i);
          else v.w[i / 2] |= (uint32_t)*reinterpret_cast<const unsigned short*>(p + i) << 16 * (i & 1);
        }
    }
    return v;
  };
  const int chunks = (pitch / N + kWords - 1) / kWords;                     // of L lanes
  QWord<T> v[KEEP > 0 ? KEEP : 1];
  float top = 0.f;
  if constexpr (KEEP > 0) {
#pragma unroll
    for (int i = 0; i < KEEP; ++i) v[i] = load(i);
#pragma unroll
    for (int i = 0; i < KEEP; ++i) top = v[i].top(top);
  } else {
#pragma unroll 4
    for (int k = 0; warp + k * WARPS < chunks; ++k) top = load(k).top(top);
  }
  // of the lanes, as bits (magnitudes, infinity and NaN order like them)
  uint32_t bits = __float_as_uint(top);
  if constexpr (L < 32) {
#pragma unroll
    for (int d = L / 2; d; d >>= 1) bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, d));
  } else {
    bits = __reduce_max_sync(0xffffffffu, bits);
  }
  if constexpr (WARPS > 1) {
    if (lane == 0) s_top[tid / L] = bits;
    __syncthreads();
    bits = __reduce_max_sync(0xffffffffu, s_top[tid / (L * WARPS) * WARPS + (lane & (WARPS - 1))]);
  }
  const QScale sc(__uint_as_float(bits));
  if (warp == 0 && lane == 0 && live) scale[row] = sc.s;
  auto put = [&](const QWord<T>& w, int k) {
    uint32_t out[N / 4];
    sc.bytes(w, out);
    if (SHIFT) {
      uint32_t next[N / 4];
#pragma unroll
      for (int i = 0; i < N / 4; ++i) next[i] = __shfl_down_sync(0xffffffffu, out[i], 1, L);
      if constexpr (N == 8) {
        const uint32_t a = skew & 4 ? out[1] : out[0], b = skew & 4 ? next[0] : out[1], d = skew & 4 ? next[1] : next[0];
        out[0] = __funnelshift_r(a, b, 8 * (skew & 3)), out[1] = __funnelshift_r(b, d, 8 * (skew & 3));
      } else {
        out[0] = __funnelshift_r(out[0], next[0], 8 * skew);
      }
    }
    if (w0 + k * kSteps < groups && (!SHIFT || lane < L - 1)) {
      if constexpr (N == 8) to[k * kSteps] = make_uint2(out[0], out[1]);
      else to[k * kSteps] = out[0];
    }
  };
  if constexpr (KEEP > 0) {
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
      if (i == 0 || warp + i * WARPS < chunks) put(v[i], i);
  } else {
#pragma unroll 2
    for (int k = 0; warp + k * WARPS < chunks; ++k) put(load(k), k);
  }
}

template <typename T, bool SHIFT, int L, int WARPS, int KEEP>
inline cudaError_t quantize_go(const T* x, int8_t* q, float* scale, long rows, int c, cudaStream_t st) {
  constexpr int kThreads = WARPS > 8 ? 32 * WARPS : kQThreads, kRows = kThreads / (L * WARPS);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((rows + kRows - 1) / kRows));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, quantize_rows_kernel<T, SHIFT, L, WARPS, KEEP>, x, q, scale, rows, c, q_pitch(c));
}
// Four words a lane where a row has them: what a row costs besides its words (its maximum, its scale) is shared by as many rows as a warp has.
template <typename T, bool SHIFT>
inline cudaError_t quantize_size(const T* x, int8_t* q, float* scale, long rows, int c, cudaStream_t st) {
  const int groups = q_pitch(c) / QWord<T>::N, less = SHIFT ? 1 : 0;
  if (groups <= kQKeep * (8 - less)) return quantize_go<T, SHIFT, 8, 1, kQKeep>(x, q, scale, rows, c, st);
  if (groups <= kQKeep * (16 - less)) return quantize_go<T, SHIFT, 16, 1, kQKeep>(x, q, scale, rows, c, st);
  const int chunks = cdiv(groups, 32 - less);
  if (chunks <= kQKeep) return quantize_go<T, SHIFT, 32, 1, kQKeep>(x, q, scale, rows, c, st);
  if (chunks <= 2 * kQKeep) return quantize_go<T, SHIFT, 32, 2, kQKeep>(x, q, scale, rows, c, st);
  if (chunks <= 4 * kQKeep) return quantize_go<T, SHIFT, 32, 4, kQKeep>(x, q, scale, rows, c, st);
  if (chunks <= 16 * kQKeep) return quantize_go<T, SHIFT, 32, 16, kQKeep>(x, q, scale, rows, c, st);
  return quantize_go<T, SHIFT, 32, 16, 0>(x, q, scale, rows, c, st);
}
template <typename T>
inline cudaError_t quantize_launch(const T* x, int8_t* q, float* scale, long rows, int c, cudaStream_t st) {
  const bool aligned = (((uintptr_t)x | (uintptr_t)((size_t)c * sizeof(T))) & 15) == 0;
  return aligned ? quantize_size<T, false>(x, q, scale, rows, c, st) : quantize_size<T, true>(x, q, scale, rows, c, st);
}

// ----------------------------------------------------------------------------- dequantise

// N values, the bytes in w, times s: 16 bytes of T.
template <typename T>
__device__ __forceinline__ Vec16<T> q_values(const uint32_t* w, float s) {
  Vec16<T> o;
#pragma unroll
  for (int i = 0; i < 16 / (int)sizeof(T); ++i) o.v[i] = (float)(int8_t)(w[i / 4] >> (8 * (i & 3))) * s;
  return o;
}

// 2^lanes threads a row.  SHIFT: rows of y that do not all start on 16-byte boundaries; L lanes (8, or a warp) then take as many groups of bytes for L - 1 aligned words of y, each
// put together from a lane's group and the one in front.
template <typename T, bool SHIFT, int L>
__global__ void __launch_bounds__(256)
dequantize_rows_kernel(const int8_t* q, const float* scale, const int32_t* index, T* y, long rows, int pool, int c, int pitch, int lanes) {
  constexpr int N = 16 / (int)sizeof(T);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const long row = (long)blockIdx.x * (256 >> lanes) + (threadIdx.x >> lanes);
  const long from = row < rows ? index ? (long)index[row] : row : -1;
  const bool live = from >= 0 && from < pool;           // else: left as it is
  if (SHIFT && L < 32 ? __all_sync(0xffffffffu, !live) : !live) return;
  const float s = live ? scale[from] : 0.f;
  const int8_t* src = q + (size_t)(live ? from : 0) * pitch;
  T* dst = y + (size_t)row * c;
  auto group = [&](int g, uint32_t* w) {
    if constexpr (N == 8) {
      const uint2 t = *reinterpret_cast<const uint2*>(src + (size_t)g * 8);
      w[0] = t.x, w[1] = t.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(src + (size_t)g * 4);
    }
  };
  const int lane = threadIdx.x % L, tid = threadIdx.x & ((1 << lanes) - 1);
  if constexpr (!SHIFT) {
#pragma unroll 4
    for (int g = tid; g < c / N; g += 1 << lanes) {
      uint32_t w[N / 4];
      group(g, w);
      q_values<T>(w, s).store(dst + (size_t)g * N);
    }
  } else {
    const int skew = (int)(((uintptr_t)dst & 15) / sizeof(T)), groups = pitch / N, words = (skew + c + N - 1) / N;
    T* first = dst - skew;
#pragma unroll 2
    for (int k = tid / L; k * (L - 1) < (L < 32 ? L - 1 : words); k += (1 << lanes) / L) {      // eight lanes have a row of one round, so that the warp stays together
      const int g = k * (L - 1) + lane - 1;                  // word g of y: the group in front, then this one
      uint32_t w[N / 4] = {}, last[N / 4];
      if (g >= 0 && g < groups) group(g, w);
#pragma unroll
      for (int i = 0; i < N / 4; ++i) last[i] = __shfl_up_sync(0xffffffffu, w[i], 1, L);
      if (lane == 0 || g >= words || !live) continue;
      // the word's first value is number g * N - skew: byte N - skew of the group in front
      if constexpr (N == 8) {
        const int b = 8 - skew;                         // 1 to 8
        uint32_t d[4] = {last[0], last[1], w[0], w[1]};
        const uint32_t a0 = b >= 8 ? d[2] : b >= 4 ? d[1] : d[0], a1 = b >= 8 ? d[3] : b >= 4 ? d[2] : d[1], a2 = b >= 8 ? 0u : b >= 4 ? d[3] : d[2];
        w[0] = __funnelshift_r(a0, a1, 8 * (b & 3)), w[1] = __funnelshift_r(a1, a2, 8 * (b & 3));
      } else if (skew) {
        w[0] = __funnelshift_r(last[0], w[0], 8 * (4 - skew));
      }
      const Vec16<T> o = q_values<T>(w, s);
      const int lo = max(skew - g * N, 0), hi = min(skew + c - g * N, N);
      if (lo == 0 && hi == N) {
        o.store(first + (size_t)g * N);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (i >= lo && i < hi) Elem<T>::st(first + (size_t)g * N + i, o.v[i]);
      }
    }
  }
}

template <typename T, bool SHIFT, int L>
inline cudaError_t dequantize_go(const int8_t* q, const float* scale, const int32_t* index, T* y, long rows, int pool, int c, cudaStream_t st) {
  int lanes = L == 32 ? 5 : 3;                          // threads of a row: enough for four accesses each, up to a CTA
  while ((!SHIFT || L == 32) && lanes < 8 && c * (int)sizeof(T) / 16 > 4 << lanes) ++lanes;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((rows + (256 >> lanes) - 1) / (256 >> lanes)));
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, dequantize_rows_kernel<T, SHIFT, L>, q, scale, index, y, rows, pool, c, q_pitch(c), lanes);
}
template <typename T>
inline cudaError_t dequantize_launch(const int8_t* q, const float* scale, const int32_t* index, T* y, long rows, int pool, int c, cudaStream_t st) {
  constexpr int E = 16 / (int)sizeof(T);                // a row of c values lies in (c + 2 E - 2) / E aligned words at most
  const bool aligned = (((uintptr_t)y | (uintptr_t)((size_t)c * sizeof(T))) & 15) == 0;
  if (aligned) return dequantize_go<T, false, 8>(q, scale, index, y, rows, pool, c, st);
  return (c + 2 * E - 2) / E <= 7 ? dequantize_go<T, true, 8>(q, scale, index, y, rows, pool, c, st) : dequantize_go<T, true, 32>(q, scale, index, y, rows, pool, c, st);
}

// ----------------------------------------------------------------------------- projection

constexpr int kI8None = (int)0x80000000;   // no sum of products: those end at 128 * 128 * 131071
constexpr int kI8FewRows = 4;   // up to this many rows every CTA quantises for itself

struct I8Args {
  const float* xs;     // [rows]
  const void* raw;     // [rows][c], few rows that are quantised here
  const float* ws;     // [n] or null
  const float* bias;   // [n] or null
  void* y;             // [rows][n]
  int rows, c, n;
  int early;           // the launch in front writes x and xs, and nothing else that is read here
  int full;            // pairs: tiles in front of those that are halved
  int* err_flag;
  long long wait_cycles;
};

// s8 x s8 -> s32, both operands K-major, M = m, N = n.
__host__ __device__ constexpr uint32_t i8_idesc(int n, int m) { return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

// The four MMAs of a K block of 128 bytes: K = 32 each.
__device__ __forceinline__ void i8_block(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, bool accumulate) {
#pragma unroll
  for (int k = 0; k < 4; ++k)
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(da + 2 * k), "l"(db + 2 * k), "r"(idesc), "r"((uint32_t)(accumulate || k != 0))
                 : "memory");
}
__device__ __forceinline__ void i8_block2(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, bool accumulate) {   // over a CTA pair
#pragma unroll
  for (int k = 0; k < 4; ++k)
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(da + 2 * k), "l"(db + 2 * k), "r"(idesc), "r"((uint32_t)(accumulate || k != 0))
                 : "memory");
}

// Behind a wait that ran out: K blocks `from` and on that may be on their way land before their CTA goes, or another limit passes.
__device__ __noinline__ void i8_drain(uint32_t full0, int stages, int from, int blocks, int* err_flag) {
  for (int j = from; j < min(from + stages, blocks); ++j)
    if (!mbar_wait(full0 + 8u * (j % stages), (uint32_t)(j / stages) & 1u, err_flag)) return;
}

// A value of y, rounded once: in fp32 for bf16 (three roundings of 2^-24 before one of 2^-8), in fp64 for fp32, where integers and scales become doubles by their bits: the
// instruction for that takes 8 clocks a warp.
template <typename T> struct I8Value;
template <> struct I8Value<bf16> {
  float ws, bias;
  __device__ __forceinline__ I8Value(float ws_, float bias_) : ws(ws_), bias(bias_) {}
  __device__ __forceinline__ float operator()(int acc, float xs) const { return fmaf((float)acc * ws, xs, bias); }
};
template <> struct I8Value<float> {
  double ws, bias;
  __device__ __forceinline__ I8Value(float ws_, float bias_) : ws(ws_), bias(bias_) {}
  __device__ __forceinline__ float operator()(int acc, double xs) const {
    const double a = __hiloint2double(0x43300000, (int)((unsigned)acc ^ 0x80000000u)) - 4503601774854144.0;      // 2^52 + 2^31
    return (float)fma(a * ws, xs, bias);
  }
};
template <typename T> using I8Xs = typename std::conditional<sizeof(T) == 4, double, float>::type;    // scales of rows as the epilogue keeps them

// Stores of a warp that holds 32 filters of two rows: of bf16, two neighbouring lanes trade, and the even one stores both filters of the even row, the odd one those of the odd.
template <typename T> struct I8Store {
  T* y;
  int rows, n, f, lane;
  bool pairs, ok;
  __device__ __forceinline__ I8Store(const I8Args& p, int f_, int lane_)
      : y((T*)p.y), rows(p.rows), n(p.n), f(f_), lane(lane_), pairs(sizeof(T) == 2 && p.n % 2 == 0 && ((uintptr_t)p.y & 3) == 0), ok(true) {}
  __device__ __forceinline__ void put2(int t, float v0, float v1) const {       // rows t and t + 1
    if (sizeof(T) == 2 && pairs) {
      const float give = lane & 1 ? v0 : v1, keep = lane & 1 ? v1 : v0, got = __shfl_xor_sync(0xffffffffu, give, 1);
      t += lane & 1;
      if (ok && f < n && t < rows) *reinterpret_cast<uint32_t*>(y + (size_t)t * n + (f & ~1)) = lane & 1 ? pack_bf16x2(got, keep) : pack_bf16x2(keep, got);
    } else if (ok && f < n) {
      if (t < rows) Elem<T>::st(y + (size_t)t * n + f, v0);
      if (t + 1 < rows) Elem<T>::st(y + (size_t)(t + 1) * n + f, v1);
    }
  }
};

__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, int* v, std::integral_constant<int, 32>) { tmem_ld32(taddr, reinterpret_cast<float*>(v)); }
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, int* v, std::integral_constant<int, 16>) { tmem_ld16(taddr, reinterpret_cast<float*>(v)); }

constexpr int kI8Epi = 8, kI8Threads = 32 * (3 + kI8Epi), kI8XWarp = 2 + kI8Epi;   // producer of W, MMA, epilogue warps (two a quarter of the lanes), producer of x

template <int TN>
struct I8Smem {
  static constexpr int kABytes = 128 * 128, kBBytes = TN * 128, kStage = kABytes + kBBytes;
  static constexpr int kStages = TN == 128 ? 4 : TN == 64 ? 6 : 8;
  static constexpr int kPart = TN * 128 * 4;                 // what the cluster's CTAs send
  static constexpr int kOffPart = kStages * kStage, kOffXs = kOffPart + kPart, kOffBars = kOffXs + TN * 8;
  static constexpr int kBars = 2 * kStages + 2;
  static constexpr int kBytes = kOffBars + 8 * kBars + 16 + 1024;
  static_assert(kBytes <= 227 * 1024, "exceeds the shared memory of an SM");
};

// tmW: rows of W in boxes of 128, tmX: rows of x in boxes of TN; 128 bytes of K each.  blockIdx: x of filters, y of rows, z: range of K.
// FEW: up to four rows come as they are.  Every CTA finds their scales, for which it reads them whole (8 KB a row of 4096 bf16), and quantises its range of K into the slots, of which
// there is one for every block: a launch less (1 x 2048 x 1000: 4.0 us in place of 4.7).
template <typename T, int TN, bool FEW>
__global__ void __launch_bounds__(kI8Threads)
int8_linear_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, I8Args p) {
  using S = I8Smem<TN>;
  constexpr int kStages = S::kStages;
  extern __shared__ uint8_t i8_smem[];
  const uint32_t raw = smem_u32(i8_smem), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = i8_smem + (base - raw);
  I8Xs<T>* s_xs = reinterpret_cast<I8Xs<T>*>(gen + S::kOffXs);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + S::kOffBars + 8 * S::kBars);
  const uint32_t bar0 = base + S::kOffBars;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kStages + s); };
  const uint32_t accum_bar = bar0 + 8u * (2 * kStages), part_bar = accum_bar + 8u;
  __shared__ uint32_t s_top[kI8FewRows][kI8Epi];
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int z = (int)blockIdx.z, Z = (int)gridDim.z;
  const int n0 = (int)blockIdx.x * 128, t0 = (int)blockIdx.y * TN;
  const int kb_all = (p.c + 127) / 128;
  const int kb0 = (int)((long)kb_all * z / Z), num_kb = (int)((long)kb_all * (z + 1) / Z) - kb0;   // Z <= kb_all: never empty

  if ((warp == 0 || (warp == kI8XWarp && !FEW)) && lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(warp == 0 ? &tmW : &tmX) : "memory");
  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) mbar_init(full_bar(s), 2), mbar_init(empty_bar(s), 1);
    mbar_init(accum_bar, 1), mbar_init(part_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (Z > 1) mbar_expect_tx(part_bar, (uint32_t)S::kPart);     // TN / Z columns from each of Z CTAs
  }
  constexpr uint32_t kCols = TN < 32 ? 32 : TN;
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // The producer of W needs nothing but its barriers, which its own warp set up.
  if (warp == 0) {
    __syncwarp();
    asm volatile("bar.arrive 2, %0;" ::"n"(kI8Threads) : "memory");
  } else {
    tc_fence_before();
    asm volatile("bar.sync 2, %0;" ::"n"(kI8Threads) : "memory");
    tc_fence_after();
  }
  const uint32_t tmem = warp == 0 ? 0u : *tmem_slot;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (Z > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");       // waited for before anything is sent
  if (!(warp == 0 && p.early)) asm volatile("griddepcontrol.wait;" ::: "memory");
  bool lost = false;                             // the cluster's parts have not come

  if (warp == 0 || (warp == kI8XWarp && !FEW)) {
    if (elect_one()) {
      const CUtensorMap* tm = warp == 0 ? &tmW : &tmX;
      const uint32_t off = warp == 0 ? 0u : (uint32_t)S::kABytes, bytes = warp == 0 ? S::kABytes : S::kBBytes;
      const int row = warp == 0 ? n0 : t0;
      int s = 0;
      uint32_t ph = 1u;
      for (int i = 0; i < num_kb; ++i) {
        if (i >= kStages && !mbar_wait(empty_bar(s), ph, p.err_flag)) break;
        mbar_expect_tx(full_bar(s), bytes);
        tma_load_2d(base + (uint32_t)s * S::kStage + off, tm, full_bar(s), (kb0 + i) * 128, row);
        if (++s == kStages) s = 0, ph ^= 1u;
      }
    }
    __syncwarp();
  } else if (warp == kI8XWarp) {
  } else if (warp == 1) {
    if (elect_one()) {
      constexpr uint32_t idesc = i8_idesc(TN, 128);
      const uint64_t da0 = umma_desc(base), db0 = umma_desc(base + S::kABytes);
      int s = 0, done = 0;
      uint32_t ph = 0u;
      bool ok = true;
      for (; done < num_kb; ++done) {
        const int i = done;
        ok = mbar_wait(full_bar(s), ph, p.err_flag);
        if (!ok) break;
        tc_fence_after();
        const uint64_t off = (uint64_t)(s * (S::kStage >> 4));
        i8_block(tmem, da0 + off, db0 + off, idesc, i != 0);
        umma_commit(empty_bar(s));
        if (++s == kStages) s = 0, ph ^= 1u;
      }
      if (ok) umma_commit(accum_bar);
      else i8_drain(full_bar(0), kStages, done, num_kb, p.err_flag);
    }
    __syncwarp();
  } else {
    const int et = tid - 64, q = warp & 3, h = (warp - 2) >> 2, row = q * 32 + lane, f = n0 + row;
    constexpr int kEpi = 32 * kI8Epi, CH = TN < 64 ? 16 : 32;              // threads; columns read at a time
    const std::integral_constant<int, CH> ch;
    const float ws = f < p.n ? (p.ws ? p.ws[f] : 1.f) : 0.f, bias = p.bias && f < p.n ? p.bias[f] : 0.f;
    if constexpr (FEW) {
      constexpr int N = QWord<T>::N;
      const T* x = (const T*)p.raw;
      const bool wide = (((uintptr_t)x | (uintptr_t)((size_t)p.c * sizeof(T))) & 15) == 0;
      auto load = [&](int t, int i) {                    // N values of row t from number i on, 0 behind the last
        QWord<T> v;
        const T* src = x + (size_t)t * p.c + i;
        if (wide) {
          v.set(i < p.c ? *reinterpret_cast<const uint4*>(src) : make_uint4(0u, 0u, 0u, 0u));
        } else {
          v.set(make_uint4(0u, 0u, 0u, 0u));
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (i + e < p.c) {
              if constexpr (sizeof(T) == 4) v.w[e] = *reinterpret_cast<const uint32_t*>(src + e);
              else v.w[e / 2] |= (uint32_t)*reinterpret_cast<const unsigned short*>(src + e) << 16 * (e & 1);
            }
        }
        return v;
      };
      for (int t = 0; t < p.rows; ++t) {
        float top = 0.f;
#pragma unroll 4
        for (int i = et * N; i < p.c; i += kEpi * N) top = load(t, i).top(top);
        const uint32_t bits = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
        if (lane == 0) s_top[t][warp - 2] = bits;
      }
      asm volatile("bar.sync 1, %0;" ::"n"(kEpi) : "memory");
      for (int t = 0; t < p.rows; ++t) {
        const QScale sc(__uint_as_float(__reduce_max_sync(0xffffffffu, s_top[t][lane & (kI8Epi - 1)])));
        if (et == 0) s_xs[t] = sc.s;
        // behind the last channel W is 0, whatever stands here
        for (int k = et * N; k - lane * N < num_kb * 128; k += kEpi * N) {
          uint32_t out[N / 4];
          sc.bytes(load(t, kb0 * 128 + k), out);
          if (k < num_kb * 128) {
            uint8_t* dst = gen + (size_t)(k >> 7) * S::kStage + S::kABytes + t * 128 + (((k & 127) >> 4 ^ t & 7) << 4) + (k & 15);
            if constexpr (N == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(out[0], out[1]);
            else *reinterpret_cast<uint32_t*>(dst) = out[0];
          }
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      asm volatile("bar.sync 1, %0;" ::"n"(kEpi) : "memory");
      if (et < num_kb) mbar_arrive_n(full_bar(et), 1);   // a slot a block
    } else {
      if (et < TN) s_xs[et] = t0 + et < p.rows ? p.xs[t0 + et] : 0.f;
      asm volatile("bar.sync 1, %0;" ::"n"(kEpi) : "memory");
    }
    I8Store<T> out(p, f, lane);
    const bool own = __all_sync(0xffffffffu, mbar_wait_within(accum_bar, 0, p.err_flag, Z > 1 ? p.wait_cycles : kTcWaitCycles));
    out.ok = own;
    tc_fence_after();
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
    const I8Value<T> of(ws, bias);
    auto value = [&](int acc, int col) { return of(acc, s_xs[col]); };
    if (Z == 1) {
#pragma unroll 1
      for (int c = h * CH; c < TN && t0 + c < p.rows; c += 2 * CH) {
        int v[CH];
        tmem_ld_cols(lane_base + c, v, ch);
#pragma unroll
        for (int i = 0; i < CH; i += 2) out.put2(t0 + c + i, value(v[i], c + i), value(v[i + 1], c + i + 1));
      }
    } else {
      // CTA o of the cluster finishes columns [o * share, + share): everybody sends it its part of them, in runs of four columns (two where a share has no more)
      const int share = TN / Z, log_share = 31 - __clz(share);
      asm volatile("barrier.cluster.wait.acquire;" ::: "memory");      // every CTA's barriers are set up
      const uint32_t recv = base + S::kOffPart;
#pragma unroll 1
      for (int c = h * CH; c < TN; c += 2 * CH) {
        int v[CH];
        if (own) {
          tmem_ld_cols(lane_base + c, v, ch);
        } else {                  // nobody waits for bytes that are never sent, nor takes these for a part
#pragma unroll
          for (int i = 0; i < CH; ++i) v[i] = kI8None;
        }
        if (share >= 4) {
#pragma unroll
          for (int i = 0; i < CH; i += 4) {
            const int o = (c + i) >> log_share, at = ((z * share + (c + i) - (o << log_share)) * 128 + row * 4) * 4;
            asm volatile(
                "{\n .reg .b32 a, b;\n mapa.shared::cluster.u32 a, %0, %2;\n mapa.shared::cluster.u32 b, %1, %2;\n"
                " st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [a], {%3, %4, %5, %6}, [b];\n}"
                ::"r"(recv + (uint32_t)at), "r"(part_bar), "r"(o), "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3])
                : "memory");
          }
        } else {
#pragma unroll
          for (int i = 0; i < CH; i += 2) {
            const int o = (c + i) >> 1, at = (z * 256 + row * 2) * 4;
            asm volatile(
                "{\n .reg .b32 a, b;\n mapa.shared::cluster.u32 a, %0, %2;\n mapa.shared::cluster.u32 b, %1, %2;\n"
                " st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [a], {%3, %4}, [b];\n}"
                ::"r"(recv + (uint32_t)at), "r"(part_bar), "r"(o), "r"(v[i]), "r"(v[i + 1])
                : "memory");
          }
        }
      }
      lost = !__all_sync(0xffffffffu, mbar_wait_cluster(part_bar, 0, p.err_flag, p.wait_cycles));
      out.ok = own && !lost;
      const int* in = reinterpret_cast<const int*>(gen + S::kOffPart);
#pragma unroll 1
      for (int i = 4 * h; i < share; i += 8) {
        uint32_t sum[4] = {0u, 0u, 0u, 0u};
        int least = 0;
        if (share >= 4) {
#pragma unroll 2
          for (int k = 0; k < Z; ++k) {
            const int4 o = *reinterpret_cast<const int4*>(in + (k * share + i) * 128 + row * 4);
            sum[0] += o.x, sum[1] += o.y, sum[2] += o.z, sum[3] += o.w, least = min(least, o.x);      // a warp sends a run of columns whole
          }
        } else {
#pragma unroll 2
          for (int k = 0; k < Z; ++k) {
            const int2 o = *reinterpret_cast<const int2*>(in + k * 256 + row * 2);
            sum[0] += o.x, sum[1] += o.y, least = min(least, o.x);
          }
        }
        out.ok = __all_sync(0xffffffffu, out.ok && least != kI8None);
        const int c = z * share + i;
        out.put2(t0 + c, value((int)sum[0], c), value((int)sum[1], c + 1));
        if (share >= 4) out.put2(t0 + c + 2, value((int)sum[2], c + 2), value((int)sum[3], c + 3));
      }
      if (!own) mbar_wait(accum_bar, 0, p.err_flag);      // the tensor memory is not given back under a product
    }
    tc_fence_before();
  }
  if (Z > 1 && !(warp >= 2 && warp < kI8XWarp)) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");   // the other warps' part in the barrier at the start
  if (__syncthreads_or(lost)) cluster_drain(part_bar, 0, p.err_flag);      // the status says so, and y stays as it is
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
}

// ---- CTA pairs

constexpr int kI8PairEpi = 8, kI8PairThreads = 64 + 32 * kI8PairEpi;

template <int TN>
struct I8PairSmem {
  static constexpr int kABytes = 128 * 128, kBBytes = TN / 2 * 128, kStage = kABytes + kBBytes;   // this CTA's filters, its half of the rows of x
  static constexpr int kStages = TN == 256 ? 6 : 8;
  static constexpr int kOffXs = kStages * kStage, kOffBars = kOffXs + 2 * TN * 8;
  static constexpr int kBars = 2 * kStages + 5;
  static constexpr int kBytes = kOffBars + 8 * kBars + 16 + 1024;
  static_assert(kBytes <= 227 * 1024, "exceeds the shared memory of an SM");
};

template <typename T, int TN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kI8PairThreads, 1)
int8_linear_pair_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmH, I8Args p) {
  using S = I8PairSmem<TN>;
  constexpr int kStages = S::kStages, HALF = TN / 2;
  extern __shared__ uint8_t i8_smem[];
  const uint32_t raw = smem_u32(i8_smem), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = i8_smem + (base - raw);
  I8Xs<T>* s_xs = reinterpret_cast<I8Xs<T>*>(gen + S::kOffXs);     // [2][TN]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + S::kOffBars + 8 * S::kBars);
  const uint32_t bar0 = base + S::kOffBars;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };            // the leader's counts both CTAs' loads
  auto empty_bar = [&](int s) { return bar0 + 8u * (kStages + s); };
  auto acc_full = [&](int b) { return bar0 + 8u * (2 * kStages + b); };
  auto acc_empty = [&](int b) { return bar0 + 8u * (2 * kStages + 2 + b); };
  const uint32_t stop_bar = bar0 + 8u * (2 * kStages + 4);         // behind a wait that ran out: what was issued has ended
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t rank = cluster_rank();                            // 0: leader
  const int pair = (int)(blockIdx.x >> 1), n_pairs = (int)(gridDim.x >> 1);
  const int tiles_n = (p.n + 255) / 256, num_kb = (p.c + 127) / 128;
  // Whole tiles, then halves (of the rows) of those that are left: 4096 x 4096 are 3.46 tiles a pair, which take 3.5 rounds so in place of four.
  const int tiles = 2 * tiles_n * ((p.rows + TN - 1) / TN) - p.full;
  auto place = [&](int i, int& nt, int& t0) {            // returns whether it is a whole one
    const bool whole = i < p.full;
    const int tile = whole ? i : p.full + (i - p.full) / 2;
    nt = tile % tiles_n, t0 = tile / tiles_n * TN + (whole ? 0 : (i - p.full) % 2 * HALF);
    return whole;
  };

  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmW) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(p.full ? &tmX : &tmH) : "memory");
    for (int s = 0; s < kStages; ++s) mbar_init(full_bar(s), 1), mbar_init(empty_bar(s), 1);
    for (int b = 0; b < 2; ++b) mbar_init(acc_full(b), 1), mbar_init(acc_empty(b), 2 * kI8PairEpi);
    mbar_init(stop_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(2 * TN) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  cluster_sync_all();     // barriers and tensor memory of both CTAs are there
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  if (warp == 0) {
    if (elect_one()) {
      int s = 0, g = 0;
      uint32_t ph = 1u;
      bool ok = true;
      for (int tile = pair; tile < tiles && ok; tile += n_pairs) {
        int nt, t0;
        const bool whole = place(tile, nt, t0);
        const int n0 = nt * 256 + (int)rank * 128;
        t0 += (int)rank * (whole ? HALF : HALF / 2);
        for (int i = 0; i < num_kb; ++i, ++g) {
          ok = g < kStages || mbar_wait(empty_bar(s), ph, p.err_flag);
          if (!ok) break;
          if (rank == 0) mbar_expect_tx(full_bar(s), (uint32_t)(2 * S::kABytes + (whole ? 2 : 1) * S::kBBytes));
          const uint32_t dst = base + (uint32_t)s * S::kStage, bar = map_to_rank(full_bar(s), 0);
          tma2_load_2d(dst, &tmW, bar, i * 128, n0);
          tma2_load_2d(dst + S::kABytes, whole ? &tmX : &tmH, bar, i * 128, t0);
          if (++s == kStages) s = 0, ph ^= 1u;
        }
      }
      // The other CTA's loads count here too, and it waits for this CTA below.
      if (!ok && rank == 0) i8_drain(full_bar(0), kStages, max(0, g - kStages), g, p.err_flag);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && elect_one()) {
      const uint64_t da0 = umma_desc(base), db0 = umma_desc(base + S::kABytes);
      int s = 0, it = 0;
      uint32_t ph = 0u;
      bool ok = true;
      for (int tile = pair; tile < tiles && ok; tile += n_pairs, ++it) {
        const int b = it & 1;
        if (it >= 2) ok = mbar_wait(acc_empty(b), (uint32_t)(it / 2 - 1) & 1u, p.err_flag);
        if (!ok) break;
        tc_fence_after();
        int nt, t0;
        const uint32_t idesc = place(tile, nt, t0) ? i8_idesc(TN, 256) : i8_idesc(HALF, 256);
        for (int i = 0; i < num_kb; ++i) {
          ok = mbar_wait(full_bar(s), ph, p.err_flag);
          if (!ok) break;
          tc_fence_after();
          const uint64_t off = (uint64_t)(s * (S::kStage >> 4));
          i8_block2(tmem + (uint32_t)(b * TN), da0 + off, db0 + off, idesc, i != 0);
          umma2_commit_both(empty_bar(s));
          if (++s == kStages) s = 0, ph ^= 1u;
        }
        if (ok) umma2_commit_both(acc_full(b));
      }
      if (!ok) {
        umma2_commit_both(stop_bar);
        mbar_wait(stop_bar, 0, p.err_flag);
      }
    }
    __syncwarp();
  } else {
    const int ew = warp - 2, q = warp & 3, h = ew >> 2, et = tid - 64;
    const uint32_t drained[2] = {map_to_rank(acc_empty(0), 0), map_to_rank(acc_empty(1), 0)};
    // A tile's scales and bias are on their way while the tile before it is stored.
    float ws = 0.f, bias = 0.f, row_scale = 0.f;
    auto fetch = [&](int tile) {
      int nt, t0;
      if (tile >= tiles) return;
      place(tile, nt, t0);
      const int f = nt * 256 + (int)rank * 128 + q * 32 + lane;
      ws = f < p.n ? (p.ws ? p.ws[f] : 1.f) : 0.f, bias = p.bias && f < p.n ? p.bias[f] : 0.f;
      row_scale = et < TN && t0 + et < p.rows ? p.xs[t0 + et] : 0.f;
    };
    fetch(pair);
    int it = 0;
    bool ok = true;
    for (int tile = pair; tile < tiles; tile += n_pairs, ++it) {    // a warp whose wait ran out stores nothing but meets the others
      int nt, t0;
      const int cols = place(tile, nt, t0) ? HALF : HALF / 2;        // of this warp
      const int b = it & 1, f = nt * 256 + (int)rank * 128 + q * 32 + lane;
      const I8Store<T> out(p, f, lane);
      const I8Value<T> of(ws, bias);
      // The scales of this tile's rows, in the half of the array that the tile before the last one left.
      I8Xs<T>* xs = s_xs + b * TN;
      if (et < TN) xs[et] = row_scale;
      asm volatile("bar.sync 1, %0;" ::"n"(32 * kI8PairEpi) : "memory");
      fetch(tile + n_pairs);
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait(acc_full(b), (uint32_t)(it / 2) & 1u, p.err_flag));
      if (!ok) continue;
      tc_fence_after();
      const uint32_t acc = tmem + (uint32_t)(b * TN + h * cols) + ((uint32_t)(q * 32) << 16);
      auto store = [&](const float* v, int col) {
        if (t0 + col >= p.rows) return;
#pragma unroll
        for (int i = 0; i < 32; i += 2)
          out.put2(t0 + col + i, of(__float_as_int(v[i]), xs[col + i]), of(__float_as_int(v[i + 1]), xs[col + i + 1]));
      };
#pragma unroll 1
      for (int c = 0; c < cols; c += 64) {
        const int col = h * cols + c;
        float v[32], w[32];
        if (c + 32 < cols) {
          tmem_ld32_issue(acc + c, v);
          tmem_ld32_issue(acc + c + 32, w);
          tmem_ld_wait(v, w);
        } else {
          tmem_ld32(acc + c, v);
        }
        if (c + 64 >= cols) {          // this warp's share is in registers
          tc_fence_before();
          __syncwarp();
          // relaxed: nothing but the loads above, which have ended, goes before it; a release waited for the stores too
          if (lane == 0) asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(drained[b]) : "memory");
        }
        store(v, col);
        if (c + 32 < cols) store(w, col + 32);
      }
    }
  }
  // Both CTAs stay until the other is done with their barriers and tensor memory.
  tc_fence_before();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * TN) : "memory");
  }
}

// ---- host side

struct I8Context {
  PFN_encodeTiled encode_tiled = nullptr;
  int sm_count = 148;
  int fit[4] = {};   // clusters of 1, 2, 4 and 8 CTAs, one an SM, that run side by side
};

inline cudaError_t i8_map(const I8Context& c, CUtensorMap* tm, const void* base, long rows, int cols, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};      // what lies behind a row's values is not read
  const cuuint64_t strides[1] = {(cuuint64_t)q_pitch(cols)};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
  const cuuint32_t es[2] = {1, 1};
  return c.encode_tiled(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess
             : cudaErrorInvalidValue;
}

template <typename T>
inline cudaError_t i8_context_init(I8Context& ctx) {   // once per device and type
  cudaError_t e = cudaSuccess;
  auto set = [&](auto kernel, int bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  set(int8_linear_kernel<T, 16, true>, I8Smem<16>::kBytes);
  set(int8_linear_kernel<T, 16, false>, I8Smem<16>::kBytes);
  set(int8_linear_kernel<T, 32, false>, I8Smem<32>::kBytes);
  set(int8_linear_kernel<T, 64, false>, I8Smem<64>::kBytes);
  set(int8_linear_kernel<T, 128, false>, I8Smem<128>::kBytes);
  set(int8_linear_pair_kernel<T, 128>, I8PairSmem<128>::kBytes);
  set(int8_linear_pair_kernel<T, 256>, I8PairSmem<256>::kBytes);
  for (int i = 0; i < 4 && e == cudaSuccess; ++i) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1u << i;
    cfg.gridDim = dim3(1, 1, 1u << i);
    cfg.blockDim = dim3(kI8Threads);
    cfg.dynamicSmemBytes = I8Smem<64>::kBytes;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&ctx.fit[i], int8_linear_kernel<T, 64, false>, &cfg);
  }
  return e;
}

struct I8Plan {
  int tn, splits;    // rows of a tile; CTAs that share its K
  bool pair;
};

// Measured, us (rows of a tile / CTAs of a cluster, p: pairs): 64 x 4096 x 4096 16/1 7.7, 32/2 6.7, 64/4 7.2, 64/1 7.7; 128 x 4096 x 4096 32/1 8.2, 64/2 9.3, 128/4 11.0, 128/1p 9.8;
// 256 64/1 10.3, 128/2 14.4, 128/1p 10.3; 512 128/1 14.9, 128/1p 11.8, 256/1p 16.5; 1024 128/1p 17.0, 256/1p 17.5; 4096 49.7 and 47.7; 128 x 1024 x 1024 16/1 3.6, 16/2 4.2, 32/1 4.2, 128/1 6.2.
// So: tiles of few rows while they fit side by side, since what a tile's epilogue and exchange take grows with its rows, and pairs when tiles of 64 do not fit.
inline I8Plan i8_plan(int rows, int c, int n, const I8Context& ctx) {
  const int kb = cdiv(c, 128), pairs = ctx.sm_count / 2;
  auto tiles = [&](int tn) { return (long)cdiv(n, 128) * cdiv(rows, tn); };
  if (rows > 64 && n > 128 && tiles(64) > ctx.sm_count) {
    auto rounds = [&](int tn) { return ((long)cdiv(n, 256) * cdiv(rows, tn) + pairs - 1) / pairs; };
    return {rounds(256) * 5 <= rounds(128) * 3 ? 256 : 128, 1, true};
  }
  // us of a K block, of the epilogue, of the exchange, by the rows of a tile
  constexpr float kBlock[4] = {0.155f, 0.155f, 0.16f, 0.25f}, kEpilogue[4] = {0.55f, 0.8f, 1.1f, 1.9f}, kExchange[4] = {0.9f, 1.2f, 3.f, 6.f};
  I8Plan best = {16, 1, false};
  float least = 1e30f;
  for (int i = 0; i < 4; ++i) {
    const int tn = 16 << i;
    if (i > 0 && rows <= tn / 2) break;
    for (int s = 0; s < 4 && kb >= 1 << s; ++s) {
      if (s > 0 && tiles(tn) > ctx.fit[s]) break;
      const long waves = s > 0 ? 1 : (tiles(tn) + ctx.sm_count - 1) / ctx.sm_count;
      const float t = (float)waves * ((float)cdiv(kb, 1 << s) * kBlock[i] + kEpilogue[i] + (s > 0 ? kExchange[i] : 0.f) + 1.f);
      if (t < least) least = t, best = {tn, 1 << s, false};
    }
  }
  return best;
}

template <typename T, int TN, bool FEW>
inline cudaError_t i8_one(const I8Plan& pl, const CUtensorMap& tmW, const CUtensorMap& tmX, const I8Args& a, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cdiv(a.n, 128), cdiv(a.rows, TN), pl.splits);
  cfg.blockDim = dim3(kI8Threads);
  cfg.dynamicSmemBytes = I8Smem<TN>::kBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = pl.splits;
  cfg.attrs = attr;
  cfg.numAttrs = pl.splits > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, int8_linear_kernel<T, TN, FEW>, tmW, tmX, a);
}
template <typename T, int TN>
inline cudaError_t i8_pair(const I8Context& ctx, const CUtensorMap& tmW, const CUtensorMap& tmX, const CUtensorMap& tmH, I8Args a, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  const long pairs = ctx.sm_count / 2, tiles = (long)cdiv(a.n, 256) * cdiv(a.rows, TN), over = tiles % pairs;
  a.full = (int)(2 * over <= pairs ? tiles - over : tiles);
  cfg.gridDim = dim3(2 * (unsigned)std::min(pairs, 2 * tiles - a.full));
  cfg.blockDim = dim3(kI8PairThreads);
  cfg.dynamicSmemBytes = I8PairSmem<TN>::kBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, int8_linear_pair_kernel<T, TN>, tmW, tmX, tmH, a);
}

// x8: quantised rows; raw: rows that are quantised into them first, or null.
template <typename T>
inline cudaError_t i8_run(const I8Context& ctx, const T* raw, const int8_t* x8, const int8_t* w, I8Args a, cudaStream_t st) {
  const I8Plan pl = i8_plan(a.rows, a.c, a.n, ctx);
  CUtensorMap tmW = {}, tmX = {};
  cudaError_t e = i8_map(ctx, &tmW, w, a.n, a.c, 128);
  if (e != cudaSuccess) return e;
  if (raw && a.rows <= kI8FewRows && !pl.pair && cdiv(cdiv(a.c, 128), pl.splits) <= I8Smem<16>::kStages) {
    a.raw = raw;
    return i8_one<T, 16, true>(pl, tmW, tmX, a, st);
  }
  e = i8_map(ctx, &tmX, x8, a.rows, a.c, pl.pair ? pl.tn / 2 : pl.tn);
  if (e != cudaSuccess) return e;
  a.early = raw != nullptr;
  if (raw) {
    e = quantize_launch<T>(raw, const_cast<int8_t*>(x8), const_cast<float*>(a.xs), a.rows, a.c, st);
    if (e != cudaSuccess) return e;
  }
  if (pl.pair) {
    CUtensorMap tmH;                     // halves of tiles
    e = i8_map(ctx, &tmH, x8, a.rows, a.c, pl.tn / 4);
    if (e != cudaSuccess) return e;
    return pl.tn == 256 ? i8_pair<T, 256>(ctx, tmW, tmX, tmH, a, st) : i8_pair<T, 128>(ctx, tmW, tmX, tmH, a, st);
  }
  switch (pl.tn) {
    case 16: return i8_one<T, 16, false>(pl, tmW, tmX, a, st);
    case 32: return i8_one<T, 32, false>(pl, tmW, tmX, a, st);
    case 64: return i8_one<T, 64, false>(pl, tmW, tmX, a, st);
    default: return i8_one<T, 128, false>(pl, tmW, tmX, a, st);
  }
}

}  // namespace ee
