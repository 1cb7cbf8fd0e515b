// A projection shared by all rows of a batch, with a low-rank adapter of each row's own beside it:
//   y[t] = W x[t] + bias + s_a B_a (A_a x[t]),  a = which[t]  (no adapter where which[t] is not one).
//
// Two launches.  The first forms h[t] = s_a A_a x[t], rank numbers a row, in the caller's workspace; the second is the product with W on
// tcgen05, whose K loop goes on behind the last channel: for the adapters that occur in its tile of rows it appends columns, of
// B_a on one side and of h[t] on the other, zero in the rows of other adapters.  So the adapters of a tile, in any order and mix, cost
// their rank in additional K, and the sum is rounded once.  Where in the sum a row's columns come, and in which CTA of a cluster, follows from the place of its adapter in
// the tile's list: its fp32 sum is grouped by what the other rows of the tile name.  Columns of zeros change no sum: a row without an adapter is not touched by them.  h is kept and multiplied as two bf16 parts, h and what its rounding left (2^-17
// of h together, 2 rank columns): rounded to one part the adapter's share would carry a second rounding of the size of the result's.
//
// The tile is turned: 128 filters are the rows of the accumulator (lanes) and 16 to 128 rows of the batch its columns, so that few
// rows cost few columns, and W, which bounds small batches, is read once.  There K is cut over a cluster of up to eight CTAs, which
// send each other their parts as asynchronous stores and add them in fixed order.  The first launch is a product of the same shape, 128 rows of
// stacked A_a over 64 rows of the batch; up to kLrSimtWork products CUDA cores do it, a warp a row of A_a.
// The second launch starts while the first runs and waits for it only before it fills in h.  The adapters' columns have slots of their own beside the ring of the
// channels: eight warps list the adapters of a tile and fill the slots, a tile ahead of the four that store; the blocks are multiplied at fixed places, spread over the later
// channels, or behind the last one where h is not there before (a persistent CTA's first tile, short K).  Four warps that filled and stored in turn took 139 us
// in place of 131 for 4096 x 4096 x 4096 with nine adapters of rank 64, 90 in place of 68 for 2048 x 1024 x 4096 with eight of 32 in mixed order, and 6.9 in place of 7.3 for
// one row of 2048 x 1000.
// Two forms.  At most one tile an SM: a deep ring, for the bytes in flight.  More: persistent CTAs with two accumulators, so that one tile's list of adapters, columns
// and stores lie under the next one's products.  128 x 256 tiles where that takes less time: 128 x 128 ones ask 128 bytes a clock of L2 for every SM, and get 97.
// What bounds it: few rows the latency of the two launches, 64 x 4096 x 4096 the bytes of W (9.3 of 19.8 us, at 3.6 TB/s), thousands of rows the tensor cores; rows in mixed
// order the columns of all their adapters, most of them zero: a block of 64 takes the filling warps about 2600 clocks (addresses 500, h 900, the look for infinities and the hand-over
// 700, the slot 400; plain stores in place of copies of zeros change nothing), its products 470.
//
// Channels that are not whole 16-byte vectors, or operands off a 16-byte boundary, cannot be fetched by TMA: eight warps then copy the
// tiles (COPY), 8 or 4 bytes at a time without waiting for them, or 2 where a row may start between two words.  Ranks, too, need not be whole vectors: columns are
// fetched in the widest units (8, 4, 2 or 1 values) that divide the rank.
#pragma once
#include "common.cuh"
#include "conv_f32.cuh"
#include "conv_tc.cuh"

namespace ee {

constexpr int kLrParts = 2;            // bf16 parts of h
constexpr int kLrMaxRank = 128;
constexpr float kLrBf16Max = 3.3895313892515355e38f;   // the largest bf16
constexpr int kLrShrinkTN = 64;        // rows of a tile of the first launch
constexpr long kLrSimtWork = 24L << 20;  // products of the first launch up to which CUDA cores take it: every row of x reads its adapter from L2
constexpr int kLrCopyWarps = 8, kLrFillWarps = 8;
template <bool COPY, bool SHRINK> constexpr int kLrThreads = 192 + 32 * (COPY ? kLrCopyWarps : 1) + (SHRINK ? 0 : 32 * kLrFillWarps);

struct LrArgs {
  const bf16* x;       // [rows][c]
  const bf16* w;       // [n][c]
  const float* bias;   // [n] or null
  const bf16* a;       // [adapters][rank][c]
  const bf16* b;       // [adapters][n][rank]
  const float* scale;  // [adapters] or null
  const int32_t* which;
  bf16* h;             // [rows][2][rank]: the two parts
  bf16* y;             // [rows][n]
  int rows, c, n, rank, r8, adapters;
  int unit;            // COPY: bytes of a copy, 8, 4 or 2: rows are whole units and start on their boundaries
  int* err_flag;
  long long wait_cycles;   // limit of the wait for the cluster's partial sums
};

template <int TN, bool PERSIST, bool SHRINK = false>
struct LrSmem {
  static constexpr int kABytes = 128 * 128, kBBytes = TN * 128, kStage = kABytes + kBBytes;
  static constexpr int kStages = SHRINK ? 3 : PERSIST ? (TN == 256 ? 3 : 4) : TN == 128 ? 3 : 5, kExt = SHRINK ? 0 : TN == 256 ? 1 : 2;   // slots of the ring, of adapter columns
  static constexpr int kAcc = PERSIST ? 2 : 1;                      // accumulators
  static constexpr int kPart = TN * 128 * 4;                        // partial sums: a shrink's h of its rows (up to 128 numbers each); else what the cluster's CTAs send
  static constexpr int kOffExt = kStages * kStage, kOffPart = kOffExt + kExt * kStage;
  static constexpr int kOffInts = kOffPart + (PERSIST ? 0 : kPart); // persistent CTAs do not cut K
  static constexpr int kInts = (2 * kAcc + 1) * TN + 16;            // adapter and slot of each row of a tile (and the next), adapters of the tile, masks and counts
  static constexpr int kOffBars = kOffInts + kInts * 4;
  static constexpr int kBytes = kOffBars + 8 * (2 * kStages + 2 * kExt + 9) + 1024;
  static_assert(kBytes <= 227 * 1024, "exceeds the shared memory of an SM");
  static_assert(!SHRINK || 2 * (kBytes + 1024) <= 228 * 1024, "two CTAs of a shrink share an SM");
};

__device__ __forceinline__ void mbar_arrive_n(uint32_t bar, uint32_t n) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}

// Number j of row t's h: for the bf16 product as two parts, for the fp32 one as it is.
__device__ __forceinline__ void lr_store(bf16* h, int t, int j, int rank, float v) {
  const bf16 hi = isfinite(v) && fabsf(v) > kLrBf16Max ? __float2bfloat16_rz(v) : __float2bfloat16_rn(v);   // what would round to an infinity is cut: the rest has the remainder
  h[((size_t)t * 2) * rank + j] = hi;
  const float rest = v - __bfloat162float(hi);
  h[((size_t)t * 2 + 1) * rank + j] = __float2bfloat16_rn(isfinite(rest) ? rest : 0.f);   // of an infinity nothing is left
}
__device__ __forceinline__ void lr_store(float* h, int t, int j, int rank, float v) { h[(size_t)t * rank + j] = v; }

// Whether one of two bf16 values is an infinity or NaN: its exponent's carry.  Nonzero bits where so.
__device__ __forceinline__ uint32_t lr_odd(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
// Zeros in their place.
__device__ __forceinline__ uint32_t lr_drop(uint32_t w) { return w & ~__vcmpeq2(w & 0x7f807f80u, 0x7f807f80u); }
// What the values dropped from B_a give row t and filter f, of the columns in the blocks of this CTA (z of Z); the second part of h would only make
// inf - inf of an infinity.
__device__ __noinline__ float lr_not_finite(const LrArgs& p, int t, int f, int ad, int slot, int z, int Z) {
  float sum = 0.f;
  if (slot < 0) return sum;
  const bf16* b = p.b + ((size_t)ad * p.n + f) * p.rank;
  for (int j = 0; j < p.rank; ++j) {
    const float v = __bfloat162float(b[j]);
    if (!isfinite(v) && (int)(((long)slot * kLrParts * p.rank + j) / 64 % Z) == z) sum += __bfloat162float(p.h[(size_t)t * kLrParts * p.rank + j]) * v;
  }
  return sum;
}

// tmA: rows of operand A (W in boxes of 128 filters; SHRINK: all adapters' A in boxes of r8 rows), tmX: rows of x in boxes of TN.
// Tile: blockIdx.x of filters, y of rows, z: range of K.  Persistent: every gridDim.x-th tile, filters first.  SHRINK: blockIdx.x of rows; their adapters in groups
// that fill the 128 rows of operand A, every gridDim.y-th from blockIdx.y on; a row of x has one adapter, so all groups of a CTA leave their numbers in the same array.
template <int TN, bool PERSIST, bool SHRINK, bool COPY>
__global__ void __launch_bounds__(kLrThreads<COPY, SHRINK>)
lowrank_tcgen05_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmX, LrArgs p) {
  using S = LrSmem<TN, PERSIST, SHRINK>;
  constexpr int kStages = S::kStages, kExt = S::kExt, kAcc = S::kAcc;
  constexpr bool kPersist = PERSIST;
  constexpr uint32_t kFull = COPY ? 32 * kLrCopyWarps : 2;   // arrivals that fill a slot
  extern __shared__ uint8_t lr_smem[];
  const uint32_t raw = smem_u32(lr_smem), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = lr_smem + (base - raw);
  int* s_ad0 = reinterpret_cast<int*>(gen + S::kOffInts);    // [kAcc][TN] adapter of a row, -1: none
  int* s_slot0 = s_ad0 + kAcc * TN;                          // [kAcc][TN] its place among the tile's adapters
  int* s_list = s_slot0 + kAcc * TN;                         // [TN] the tile's adapters, in order of first occurrence
  unsigned* s_mask = reinterpret_cast<unsigned*>(s_list + TN);   // [8]
  int* s_count = reinterpret_cast<int*>(s_mask) + 8;         // [2] adapters of the tile, by its parity
  int* s_bad = s_count + 2;                                  // [2] set where a B_a of the tile holds infinities or NaN
  uint32_t* tmem_slot = s_mask + 12;
  const uint32_t bar0 = base + S::kOffBars;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kStages + s); };
  auto accum_bar = [&](int a) { return bar0 + 8u * (2 * kStages + a); };     // the accumulator is complete
  auto drain_bar = [&](int a) { return bar0 + 8u * (2 * kStages + 2 + a); }; // and has been read
  auto list_bar = [&](int i) { return bar0 + 8u * (2 * kStages + 4 + i); };  // the tile's adapters are known
  const uint32_t part_bar = bar0 + 8u * (2 * kStages + 6);
  auto ext_full = [&](int x) { return part_bar + 8u + 8u * x; };             // slots of adapter columns
  auto ext_empty = [&](int x) { return part_bar + 8u + 8u * (kExt + x); };
  auto filled_bar = [&](int i) { return part_bar + 8u + 8u * (2 * kExt + i); };   // all that the tile's epilogue reads of its adapters is there
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int z = (int)blockIdx.z, Z = (int)gridDim.z;
  const int tiles_n = (p.n + 127) / 128;
  int tiles = kPersist ? tiles_n * ((p.rows + TN - 1) / TN) : 1;
  const int tile0 = kPersist ? (int)blockIdx.x : SHRINK ? (int)blockIdx.y : 0, tile_step = kPersist ? (int)gridDim.x : SHRINK ? (int)gridDim.y : 1;
  auto place_of = [&](int tile, int& n0, int& t0) {
    if (SHRINK) {
      n0 = 0, t0 = (int)blockIdx.x * TN;
      return;
    }
    n0 = (kPersist ? tile % tiles_n : (int)blockIdx.x) * 128, t0 = (kPersist ? tile / tiles_n : (int)blockIdx.y) * TN;
  };
  const int kb_all = (p.c + 63) / 64;
  const int kb0 = (int)((long)kb_all * z / Z), num_kb = (int)((long)kb_all * (z + 1) / Z) - kb0;   // Z <= kb_all: never empty
  int n_first, t_first;
  place_of(tile0, n_first, t_first);

  if (!COPY && (warp == 0 || warp == 6) && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmA) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmX) : "memory");
  }
  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) mbar_init(full_bar(s), kFull), mbar_init(empty_bar(s), 1);
    for (int x = 0; x < kExt; ++x) mbar_init(ext_full(x), 1), mbar_init(ext_empty(x), 1);
    for (int a = 0; a < 2; ++a) mbar_init(accum_bar(a), 1), mbar_init(drain_bar(a), 1), mbar_init(list_bar(a), 1), mbar_init(filled_bar(a), 1);
    mbar_init(part_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (!SHRINK && Z > 1) mbar_expect_tx(part_bar, (uint32_t)S::kPart);     // TN / Z columns from each of Z CTAs
  }
  constexpr uint32_t kCols = TN < 32 ? 32 : TN * kAcc;
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // The producer of W needs nothing but its barriers: it goes ahead while the others wait for the accumulator's address, about 1600 clocks.
  constexpr int kThreads = kLrThreads<COPY, SHRINK>, kFill0 = COPY ? 6 + kLrCopyWarps : 7;
  if (warp == 0) {
    __syncwarp();
    asm volatile("bar.arrive 2, %0;" ::"n"(kThreads) : "memory");
  } else {
    tc_fence_before();
    asm volatile("bar.sync 2, %0;" ::"n"(kThreads) : "memory");
    tc_fence_after();
  }
  const uint32_t tmem = warp == 0 ? 0u : *tmem_slot;
  if (SHRINK) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (Z > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");       // waited for before anything is sent

  const int ext_cols = kLrParts * p.rank;        // columns of an adapter
  // blocks of adapter columns that this CTA takes: z, z + Z, ...
  auto ext_blocks = [&](int count) {
    const int all = (int)(((long)count * ext_cols + 63) / 64);
    return all > z ? (all - z + Z - 1) / Z : 0;
  };
  // The tile's adapters: a row is the first of its adapter, or refers to it.  By the kList threads from `et` = 0 on.
  constexpr int kList = SHRINK ? 128 : 32 * kLrFillWarps;
  auto list_adapters = [&](int et, int t0, int par) {
    static_assert(TN <= kList, "a thread has a row");
    int *s_ad = s_ad0 + (par & (kAcc - 1)) * TN, *s_slot = s_slot0 + (par & (kAcc - 1)) * TN;
    asm volatile("bar.sync 1, %0;" ::"n"(kList) : "memory");       // the list of the tile before is not needed any more
    if (et < TN) {
      const int t = t0 + et, a = t < p.rows && p.adapters > 0 ? p.which[t] : -1;
      s_ad[et] = a >= 0 && a < p.adapters ? a : -1;
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kList) : "memory");
    const int w0 = et & ~31, a = et < TN ? s_ad[et] : -1;
    int f = w0 + __ffs(__match_any_sync(0xffffffffu, a)) - 1;       // the first of its warp
    if (a >= 0 && f == et)
      for (int u = 0; u < w0; u += 4) {
        const int4 o = *reinterpret_cast<const int4*>(s_ad + u);
        if (o.w == a) f = min(f, u + 3);
        if (o.z == a) f = min(f, u + 2);
        if (o.y == a) f = min(f, u + 1);
        if (o.x == a) f = min(f, u);
      }
    f = __shfl_sync(0xffffffffu, f, f >= w0 ? f & 31 : lane);       // the others of the warp take what their first found
    const unsigned lead = __ballot_sync(0xffffffffu, a >= 0 && f == et);
    if (lane == 0 && et < TN) s_mask[et >> 5] = lead;
    asm volatile("bar.sync 1, %0;" ::"n"(kList) : "memory");
    int count = 0;
#pragma unroll
    for (int k = 0; k < (TN + 31) / 32; ++k) count += __popc(s_mask[k]);
    if (et < TN) {
      int slot = -1;
      if (a >= 0) {
        slot = __popc(s_mask[f >> 5] & ((1u << (f & 31)) - 1u));
        for (int k = 0; k < f >> 5; ++k) slot += __popc(s_mask[k]);
        if (f == et) s_list[slot] = a;
      }
      s_slot[et] = slot;
    }
    if (et == 0) s_count[par] = count, s_bad[par] = 0;
    asm volatile("bar.sync 1, %0;" ::"n"(kList) : "memory");
    if (et == 0) mbar_arrive_n(list_bar(par), 1);
    return count;
  };
  const int per_tile = 128 / p.r8;               // SHRINK: adapters of a tile
  if (SHRINK) {
    if (warp >= 2 && warp < 6) list_adapters(tid - 64, t_first, 0);
    __syncthreads();
    tiles = (s_count[0] + per_tile - 1) / per_tile;
  }
  const bool idle = SHRINK && tiles <= tile0;    // no adapters here
  bool lost = false;                             // the cluster's parts have not come
  auto here = [&](int group) { return min(per_tile, s_count[0] - group * per_tile); };      // adapters of a group

  struct Walk {      // over the ring
    int s;
    uint32_t ph;
    __device__ __forceinline__ void next() {
      if (++s == kStages) s = 0, ph ^= 1u;
    }
  };
  auto produce = [&](auto&& load) {
    Walk w{0, 1u};
    int used = 0;                                // slots start out free
    for (int tile = tile0; tile < tiles; tile += tile_step) {
      int n0, t0;
      place_of(tile, n0, t0);
      for (int i = 0; i < num_kb; ++i) {
        if (used == kStages && !mbar_wait(empty_bar(w.s), w.ph, p.err_flag)) return;
        load(w.s, kb0 + i, SHRINK ? tile : n0, t0);
        used = min(used + 1, kStages), w.next();
      }
    }
  };

  if (idle) {
  } else if (warp == 0) {
    if (!COPY && elect_one())
      produce(
              [&](int s, int kb, int n0, int) {
                const uint32_t dst = base + (uint32_t)s * S::kStage;
                if (SHRINK) {
                  const int group = n0, n = here(group);
                  mbar_expect_tx(full_bar(s), (uint32_t)(n * p.r8 * 128));
                  for (int k = 0; k < n; ++k)
                    tma_load_2d(dst + (uint32_t)(k * p.r8 * 128), &tmA, full_bar(s), kb * 64, s_list[group * per_tile + k] * p.rank);
                } else {
                  mbar_expect_tx(full_bar(s), S::kABytes);
                  tma_load_2d(dst, &tmA, full_bar(s), kb * 64, n0);
                }
              });
    __syncwarp();
  } else if (!COPY && warp == 6) {
    if (elect_one())
      produce(
              [&](int s, int kb, int, int t0) {
                mbar_expect_tx(full_bar(s), S::kBBytes);
                tma_load_2d(base + (uint32_t)s * S::kStage + S::kABytes, &tmX, full_bar(s), kb * 64, t0);
              });
    __syncwarp();
  } else if (COPY && warp >= 6 && warp < 6 + kLrCopyWarps) {
    const int ct = tid - 192;
    int late = -1;                       // slot whose copies are on their way
    auto landed = [&]() {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive_n(full_bar(late), 1);
    };
    produce([&](int s, int kb, int n0, int t0) {
      uint8_t* dst = gen + (size_t)s * S::kStage;
      const uint32_t dst_s = base + (uint32_t)s * S::kStage;
      const int shift = p.unit == 8 ? 4 : 5, col = ct & ((1 << shift) - 1);      // copies of a row: 16 of 8 bytes, 32 of 4 (or of 2 x 2)
      const int k0 = kb * 64 + col * (64 >> shift);
      const uint32_t chunk = (uint32_t)(col >> (shift - 3)), within = (uint32_t)(col & ((1 << (shift - 3)) - 1)) * (uint32_t)(128 >> shift);
      auto row_of = [&](int r) -> const bf16* {
        if (r >= 128) return t0 + r - 128 < p.rows ? p.x + (size_t)(t0 + r - 128) * p.c : nullptr;
        if (SHRINK) {                    // n0: the group
          const int k = r / p.r8, j = r - k * p.r8;
          return k < here(n0) && j < p.rank ? p.a + ((size_t)s_list[n0 * per_tile + k] * p.rank + j) * p.c : nullptr;
        }
        return n0 + r < p.n ? p.w + (size_t)(n0 + r) * p.c : nullptr;
      };
      auto place = [&](int r) { return (uint32_t)r * 128 + ((chunk ^ (uint32_t)(r & 7)) << 4) + within; };
      if (p.unit > 2) {
#pragma unroll 4
        for (int r = ct >> shift; r < 128 + TN; r += 32 * kLrCopyWarps >> shift) {
          const bf16* src = row_of(r);
          const bool in = src && k0 < p.c;               // rows are whole units: one lies inside its row or outside it
          if (p.unit == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst_s + place(r)), "l"(in ? src + k0 : p.x), "r"(in ? 8 : 0) : "memory");
          else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst_s + place(r)), "l"(in ? src + k0 : p.x), "r"(in ? 4 : 0) : "memory");
        }
      } else {
#pragma unroll 1
        for (int r0 = ct >> 5; r0 < 128 + TN; r0 += 8 * kLrCopyWarps) {      // eight rows' values on their way before the first is stored
          unsigned short lo[8], hi[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = r0 + i * kLrCopyWarps;
            const unsigned short* src = r < 128 + TN ? reinterpret_cast<const unsigned short*>(row_of(r)) : nullptr;
            lo[i] = src && k0 < p.c ? src[k0] : (unsigned short)0;
            hi[i] = src && k0 + 1 < p.c ? src[k0 + 1] : (unsigned short)0;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = r0 + i * kLrCopyWarps;
            if (r < 128 + TN) *reinterpret_cast<uint32_t*>(dst + place(r)) = (uint32_t)lo[i] | (uint32_t)hi[i] << 16;
          }
        }
      }
      cp_async_commit();
      if (late >= 0) {                   // one block behind
        cp_async_wait<1>();
        landed();
      }
      late = s;
    });
    if (late >= 0) {
      cp_async_wait<0>();
      landed();
    }
  } else if (warp == 1) {
    if (elect_one()) {
      constexpr uint32_t idesc = umma_idesc(TN);
      const uint64_t da0 = umma_desc(base), db0 = umma_desc(base + S::kABytes);
      Walk w{0, 0u};
      bool ok = true;
      uint32_t xs = 0;                                 // blocks of adapter columns so far
      for (int tile = tile0, it = 0; tile < tiles && ok; tile += tile_step, ++it) {
        const int a = it & (kAcc - 1);
        const uint32_t acc = tmem + (uint32_t)(a * TN);
        if (it >= kAcc) ok = mbar_wait(drain_bar(a), (uint32_t)(it / kAcc - 1) & 1u, p.err_flag);
        // Where the adapters' columns go, in K blocks: spread from where the list is asked for, or behind the last block, if h is not there before.
        const int ask = kPersist ? (it > 0 ? (num_kb + 3) / 4 : num_kb) : num_kb >= 8 ? num_kb * 5 / 8 : num_kb;
        int ext = 0, e = 0;
        for (int i = 0; i < num_kb && ok; ++i) {
          ok = mbar_wait(full_bar(w.s), w.ph, p.err_flag);
          if (!ok) break;
          tc_fence_after();
          const uint64_t off = (uint64_t)(w.s * (S::kStage >> 4));
          umma_block(acc, da0 + off, db0 + off, idesc, i != 0);
          umma_commit(empty_bar(w.s));
          w.next();
          if constexpr (!SHRINK) {
            if (i + 1 == ask) {
              ok = mbar_wait(list_bar(it & 1), (uint32_t)(it >> 1) & 1u, p.err_flag);
              ext = ok ? ext_blocks(s_count[it & 1]) : 0;
            }
            for (; ok && e < ext && (i + 1 == num_kb || (long)(i + 1 - ask) * (ext + 1) >= (long)(e + 1) * (num_kb - ask)); ++e, ++xs) {
              const int x = (int)(xs % kExt);
              ok = mbar_wait(ext_full(x), xs / kExt & 1u, p.err_flag);
              if (!ok) break;
              tc_fence_after();
              const uint64_t at = (uint64_t)((S::kOffExt + x * S::kStage) >> 4);
              umma_block(acc, da0 + at, db0 + at, idesc, true);
              umma_commit(ext_empty(x));
            }
          }
        }
        if (ok) umma_commit(accum_bar(a));
      }
    }
    __syncwarp();
  } else if (!SHRINK && warp >= kFill0) {
    if constexpr (!SHRINK) {
      const int et = tid - 32 * kFill0;
      bool ok = true;
      uint32_t xs = 0;                                 // blocks of adapter columns so far
      bool waited = false;                             // for h
      for (int tile = tile0, it = 0; tile < tiles; tile += tile_step, ++it) {
        int n0, t0;
        place_of(tile, n0, t0);
        if (it >= kAcc) ok = ok && mbar_wait(drain_bar(it & (kAcc - 1)), (uint32_t)(it / kAcc - 1) & 1u, p.err_flag);    // the list of that tile is not needed any more
        const int count = list_adapters(et, t0, it & 1);
        const int* s_slot = s_slot0 + (it & (kAcc - 1)) * TN;
        // A thread has the 16-byte chunk et % 8 of a block's 64 columns, in every 32nd row of either operand.
        const int ext = ext_blocks(count), all = count * ext_cols, c8 = et & 7, r0 = et >> 3;
        // values of a unit of B_a, of h: they lie in one part of one adapter
        const int unit_h = p.rank % 8 == 0 ? 8 : p.rank % 4 == 0 ? 4 : p.rank % 2 == 0 ? 2 : 1;
        int unit_b = unit_h;
        while ((uintptr_t)p.b & (unit_b * 2 - 1)) unit_b >>= 1;
        // The code of this part is kept short (loops, not copies): it runs a few times a tile, and what it costs is its way into the instruction cache.
        const uint32_t place0 = (uint32_t)(r0 * 128 + ((c8 ^ (r0 & 7)) << 4));      // of row r0; every 32nd row is 4096 bytes on
        const float per_col = 1.f / (float)ext_cols;
        auto column = [&](int e, int k, int& slot, int& rem) {       // adapter and place in its 2 * rank columns; slot -1: behind the last
          const int c = (z + e * Z) * 64 + c8 * 8 + k;
          slot = (int)(((float)c + 0.5f) * per_col), rem = c - slot * ext_cols;      // c < 2^16: the quotient is off by less than half a column
          if (c >= all) slot = -1;
        };
        auto fetch = [&](uint32_t dst, const void* src, bool in, int bytes) {
          if (bytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
          else if (bytes == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(in ? 8 : 0) : "memory");
          else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
        };
        auto slot_of_block = [&](int e) { return (int)((xs + (uint32_t)e) % kExt); };
        auto at_block = [&](int e) { return (uint32_t)(S::kOffExt + slot_of_block(e) * S::kStage); };
        auto fill_b = [&](int e) {
          const uint32_t use = xs + (uint32_t)e;
          if (use >= kExt) ok = ok && mbar_wait(ext_empty(slot_of_block(e)), (use / kExt - 1) & 1u, p.err_flag);
#pragma unroll 1
          for (int k = 0; k < 8; k += unit_b) {
            int slot, rem;
            column(e, k, slot, rem);
            const bf16* src = p.b + ((size_t)(slot >= 0 ? s_list[slot] : 0) * p.n + n0 + r0) * p.rank + (rem < p.rank ? rem : rem - p.rank);
            if (unit_b > 1) {
              const uint32_t dst = base + at_block(e) + place0 + 2 * k;
#pragma unroll
              for (int m = 0; m < 4; ++m) {
                const bool in = slot >= 0 && n0 + r0 + 32 * m < p.n;
                fetch(dst + 4096 * m, in ? src + (size_t)32 * m * p.rank : p.b, in, unit_b * 2);
              }
            } else {
              unsigned short* dst = reinterpret_cast<unsigned short*>(gen + at_block(e) + place0) + k;
              unsigned short v[4];
#pragma unroll
              for (int m = 0; m < 4; ++m) v[m] = slot >= 0 && n0 + r0 + 32 * m < p.n ? reinterpret_cast<const unsigned short*>(src)[(size_t)32 * m * p.rank] : (unsigned short)0;
#pragma unroll
              for (int m = 0; m < 4; ++m) dst[m * 2048] = v[m];
            }
          }
        };
        auto fill_h = [&](int e) {         // the workspace is aligned
#pragma unroll 1
          for (int k = 0; k < 8; k += unit_h) {
            int slot, rem;
            column(e, k, slot, rem);
            const bf16* src = p.h + (size_t)(t0 + r0) * ext_cols + rem;
            if (unit_h > 1) {
              uint32_t dst = base + at_block(e) + S::kABytes + place0 + 2 * k;
#pragma unroll 4
              for (int t = r0; t < TN; t += 32, dst += 4096, src += 32 * ext_cols) {
                const bool in = slot >= 0 && s_slot[t] == slot;
                fetch(dst, in ? src : p.h, in, unit_h * 2);
              }
            } else {
              unsigned short* dst = reinterpret_cast<unsigned short*>(gen + at_block(e) + S::kABytes + place0) + k;
#pragma unroll 4
              for (int t = r0; t < TN; t += 32, dst += 2048, src += 32 * ext_cols) *dst = slot >= 0 && s_slot[t] == slot ? *reinterpret_cast<const unsigned short*>(src) : (unsigned short)0;
            }
          }
        };
        // What there is no slot for yet is on its way to L2.
#pragma unroll 1
        for (int e = kExt; e < ext; ++e) {
          const int first = (z + e * Z) * 64 / ext_cols, last = min(((z + e * Z) * 64 + 63) / ext_cols, count - 1);
          const int bytes = min(128, p.n - n0) * p.rank * 2, lines = (bytes + 127) / 128;
          for (int k = first; k <= last; ++k)
#pragma unroll 1
            for (int i = et; i < lines; i += kList)
              asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const char*>(p.b + ((size_t)s_list[k] * p.n + n0) * p.rank) + min(i * 128, bytes - 2)));
        }
        // A block is fetched while the one before it arrives.  B_a, which no kernel in front writes, is fetched before the wait for h.
        auto finish = [&](int e) {
          // what this thread fetched is here: an infinity would turn the zeros of other adapters' rows into NaN, so lr_not_finite adds it to its own rows
          uint4* at = reinterpret_cast<uint4*>(gen + at_block(e) + place0);
#pragma unroll 2
          for (int m = 0; m < 4; ++m) {
            const uint4 v = at[m * 256];
            if (lr_odd(v.x) | lr_odd(v.y) | lr_odd(v.z) | lr_odd(v.w)) at[m * 256] = make_uint4(lr_drop(v.x), lr_drop(v.y), lr_drop(v.z), lr_drop(v.w)), s_bad[it & 1] = 1;
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          asm volatile("bar.sync 1, %0;" ::"n"(kList) : "memory");
          if (et == 0) mbar_arrive_n(ext_full(slot_of_block(e)), 1);
        };
        constexpr int kBehind = kExt - 1;      // blocks on their way behind the one that is finished
        int have = 0;                          // blocks whose B_a is on its way
#pragma unroll 1
        for (int e = 0; e < ext + kBehind; ++e) {
          if (e < ext) {
            const int to = waited ? e + 1 : min(kExt, ext);
#pragma unroll 1
            for (; have < to; ++have) fill_b(have);
            if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
            waited = true;
            fill_h(e);
          }
          cp_async_commit();
          if (e >= kBehind) {
            cp_async_wait<kBehind>();
            finish(e - kBehind);
          }
        }
        xs += (uint32_t)ext;
        if (et == 0) mbar_arrive_n(filled_bar(it & 1), 1);
      }
    }
  } else {
    const int et = tid - 64, q = warp & 3;
    const int row = q * 32 + lane;                     // accumulator lane of this thread
    constexpr int CH = TN < 32 ? TN : 32;              // columns read at a time
    bool ok = true;
    if constexpr (SHRINK) {
      // this CTA's part of h: [TN][r8] floats
      const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
      const int k = row / p.r8, j = row - k * p.r8;
      float* part = reinterpret_cast<float*>(gen + S::kOffPart);
      for (int group = tile0, it = 0; group < tiles; group += tile_step, ++it) {
        ok = __all_sync(0xffffffffu, mbar_wait(accum_bar(0), (uint32_t)it & 1u, p.err_flag)) && ok;
        tc_fence_after();
        const int slot = k < per_tile ? group * per_tile + k : -2;
#pragma unroll 1
        for (int c = 0; c < TN; c += CH) {
          float v[CH];
          if constexpr (CH == 32) tmem_ld32(lane_base + c, v);
          else tmem_ld16(lane_base + c, v);
#pragma unroll
          for (int i = 0; i < CH; ++i)
            if (s_slot0[c + i] == slot) part[(c + i) * p.r8 + j] = v[i];
        }
        tc_fence_before();
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (et == 0) mbar_arrive_n(drain_bar(0), 1);
      }
    } else {
      asm volatile("griddepcontrol.wait;" ::: "memory");      // nothing is stored before, nor h read
      for (int tile = tile0, it = 0; tile < tiles; tile += tile_step, ++it) {
        int n0, t0;
        place_of(tile, n0, t0);
        const int* s_ad = s_ad0 + (it & (kAcc - 1)) * TN;
        const int* s_slot = s_slot0 + (it & (kAcc - 1)) * TN;
        const int acc = it & (kAcc - 1);
        ok = __all_sync(0xffffffffu, mbar_wait(accum_bar(acc), (uint32_t)(it / kAcc) & 1u, p.err_flag) && mbar_wait(filled_bar(it & 1), (uint32_t)(it >> 1) & 1u, p.err_flag)) && ok;
        tc_fence_after();
        const uint32_t lane_base = tmem + (uint32_t)(acc * TN) + ((uint32_t)(q * 32) << 16);
        const int f = n0 + row;
        const float bias = p.bias && f < p.n ? p.bias[f] : 0.f;
        const bool bad = s_bad[it & 1] != 0 && f < p.n;
        auto columns_of = [&](int c, float* v) {
          if constexpr (CH == 32) tmem_ld32(lane_base + c, v);
          else tmem_ld16(lane_base + c, v);
          if (bad)
#pragma unroll
            for (int i = 0; i < CH; ++i) v[i] += lr_not_finite(p, t0 + c + i, f, s_ad[c + i], s_slot[c + i], z, Z);
        };
        // Two neighbouring lanes trade: the even one stores both filters of the even rows, the odd one those of the odd rows, 4 bytes each.
        const bool pairs = p.n % 2 == 0 && ((uintptr_t)p.y & 3) == 0;
        auto store2 = [&](int t, float v0, float v1) {       // of rows t and t + 1; n is even: both filters of a pair are there, or neither
          const float give = lane & 1 ? v0 : v1, keep = lane & 1 ? v1 : v0, got = __shfl_xor_sync(0xffffffffu, give, 1);
          t += lane & 1;
          if (ok && f < p.n && t < p.rows) *reinterpret_cast<uint32_t*>(p.y + (size_t)t * p.n + (f & ~1)) = lane & 1 ? pack_bf16x2(got, keep) : pack_bf16x2(keep, got);
        };
        if (Z == 1) {
#pragma unroll 1
          for (int c = 0; c < TN; c += CH) {
            float v[CH];
            columns_of(c, v);
            if (pairs) {
#pragma unroll
              for (int i = 0; i < CH; i += 2) store2(t0 + c + i, v[i] + bias, v[i + 1] + bias);
            } else if (ok && f < p.n) {
#pragma unroll
              for (int i = 0; i < CH; ++i)
                if (t0 + c + i < p.rows) p.y[(size_t)(t0 + c + i) * p.n + f] = __float2bfloat16_rn(v[i] + bias);
            }
          }
          if (kPersist) {          // the accumulator is free for the tile after the next
            tc_fence_before();
            asm volatile("bar.sync 3, 128;" ::: "memory");
            if (et == 0) mbar_arrive_n(drain_bar(acc), 1);
          }
        } else if constexpr (!kPersist) {
          // CTA o of the cluster finishes columns [o * share, + share): everybody sends it its part of them, in runs of four columns (two where a share has no more)
          const int share = TN / Z, log_share = 31 - __clz(share);
          asm volatile("barrier.cluster.wait.acquire;" ::: "memory");      // every CTA's barriers are set up
          const uint32_t recv = base + S::kOffPart;
#pragma unroll 1
          for (int c = 0; c < TN; c += CH) {
            float v[CH];
            columns_of(c, v);
            if (share >= 4) {
#pragma unroll
              for (int i = 0; i < CH; i += 4) {
                const int o = (c + i) >> log_share, at = ((z * share + (c + i) - (o << log_share)) * 128 + row * 4) * 4;
                asm volatile(
                    "{\n .reg .b32 a, b;\n mapa.shared::cluster.u32 a, %0, %2;\n mapa.shared::cluster.u32 b, %1, %2;\n"
                    " st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [a], {%3, %4, %5, %6}, [b];\n}"
                    ::"r"(recv + (uint32_t)at), "r"(part_bar), "r"(o), "f"(v[i]), "f"(v[i + 1]), "f"(v[i + 2]), "f"(v[i + 3])
                    : "memory");
              }
            } else {
#pragma unroll
              for (int i = 0; i < CH; i += 2) {
                const int o = (c + i) >> 1, at = (z * 256 + row * 2) * 4;
                asm volatile(
                    "{\n .reg .b32 a, b;\n mapa.shared::cluster.u32 a, %0, %2;\n mapa.shared::cluster.u32 b, %1, %2;\n"
                    " st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [a], {%3, %4}, [b];\n}"
                    ::"r"(recv + (uint32_t)at), "r"(part_bar), "r"(o), "f"(v[i]), "f"(v[i + 1])
                    : "memory");
              }
            }
          }
          lost = !__all_sync(0xffffffffu, mbar_wait_cluster(part_bar, 0, p.err_flag, p.wait_cycles));
          ok = ok && !lost;
          const float* in = reinterpret_cast<const float*>(gen + S::kOffPart);
          const int run = min(share, 4);
#pragma unroll 1
          for (int i = 0; i < share; i += run) {
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
            if (run == 4) {
#pragma unroll 2
              for (int k = 0; k < Z; ++k) {
                const float4 o = *reinterpret_cast<const float4*>(in + (k * share + i) * 128 + row * 4);
                sum[0] += o.x, sum[1] += o.y, sum[2] += o.z, sum[3] += o.w;
              }
            } else {
#pragma unroll 2
              for (int k = 0; k < Z; ++k) {
                const float2 o = *reinterpret_cast<const float2*>(in + k * 256 + row * 2);
                sum[0] += o.x, sum[1] += o.y;
              }
            }
            const int t = t0 + z * share + i;
            if (pairs) {
              store2(t, sum[0] + bias, sum[1] + bias);
              if (run == 4) store2(t + 2, sum[2] + bias, sum[3] + bias);
            } else {
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (j < run && ok && f < p.n && t + j < p.rows) p.y[(size_t)(t + j) * p.n + f] = __float2bfloat16_rn(sum[j] + bias);
            }
          }
        }
      }
    }
    tc_fence_before();
  }
  // The warps that send wait for what is sent to them; the others' part in the barrier at the start.
  if (Z > 1 && (SHRINK || !(warp >= 2 && warp < 6))) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  if constexpr (SHRINK) {
    if (!idle) {
      // The parts are complete in every CTA of the cluster; this one finishes every Z-th row.
      if (Z > 1) asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
      else __syncthreads();
      const uint32_t part = base + S::kOffPart;
      for (int i = tid; i < TN / Z * p.rank; i += (int)blockDim.x) {
        const int t = i / p.rank * Z + z, j = i - i / p.rank * p.rank;
        if (s_slot0[t] < 0 || s_slot0[t] / per_tile % tile_step != tile0) continue;
        float sum = 0.f;
        for (int r = 0; r < Z; ++r) {
          uint32_t from;
          float v;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(part + 4u * (t * p.r8 + j)), "r"(r));
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(from) : "memory");
          sum += v;
        }
        lr_store(p.h, t_first + t, j, p.rank, p.scale ? sum * p.scale[s_ad0[t]] : sum);
      }
      if (Z > 1) asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");   // nobody reads this CTA's part any more
    }
  }
  if (!SHRINK && !kPersist) {
    if (__syncthreads_or(lost)) cluster_drain(part_bar, 0, p.err_flag);      // the status says so, and y stays as it is
  } else {
    __syncthreads();
  }
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
}

// h[t] = s_a A_a x[t] on CUDA cores.  A CTA has a row of x and `jn` (1, 2, 4 or 8) rows of its adapter, each of which 8 / jn warps share: few rows of the batch
// are many short CTAs.  V elements per load.
template <typename T, int V>
__global__ void __launch_bounds__(256)
lowrank_shrink_kernel(const T* __restrict__ x, const T* __restrict__ a, const float* __restrict__ scale, const int32_t* __restrict__ which, T* __restrict__ h, int c,
                      int rank, int adapters, int jn) {
  typedef typename Accum<T>::type acc_t;
  __shared__ acc_t s_sum[8];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int t = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int ad = which[t];
  if (ad < 0 || ad >= adapters) return;
  const int j = (int)blockIdx.y * jn + warp % jn, part = warp / jn, parts = 8 / jn;
  const int steps = (c + 32 * V - 1) / (32 * V), s0 = (int)((long)steps * part / parts), s1 = (int)((long)steps * (part + 1) / parts);
  const T* xr = x + (size_t)t * c;
  acc_t sum = 0;
  if (j < rank) {
    const T* ar = a + ((size_t)ad * rank + j) * c;
#pragma unroll 8
    for (int s = s0; s < s1; ++s) {
      const int k = (s * 32 + lane) * V;
      if (k < c) {                              // V divides c
        if constexpr (V == 1) {
          sum = acc_fma(Elem<T>::ld(xr + k), Elem<T>::ld(ar + k), sum);
        } else if constexpr (V * sizeof(T) == 8) {       // four bf16, or two floats
          const uint2 u = *reinterpret_cast<const uint2*>(xr + k), v = *reinterpret_cast<const uint2*>(ar + k);
          if constexpr (sizeof(T) == 2) {
            sum = acc_fma(__uint_as_float(u.x << 16), __uint_as_float(v.x << 16), sum);
            sum = acc_fma(__uint_as_float(u.x & 0xffff0000u), __uint_as_float(v.x & 0xffff0000u), sum);
            sum = acc_fma(__uint_as_float(u.y << 16), __uint_as_float(v.y << 16), sum);
            sum = acc_fma(__uint_as_float(u.y & 0xffff0000u), __uint_as_float(v.y & 0xffff0000u), sum);
          } else {
            sum = acc_fma(__uint_as_float(u.x), __uint_as_float(v.x), sum);
            sum = acc_fma(__uint_as_float(u.y), __uint_as_float(v.y), sum);
          }
        } else {
          Vec16<T> u, v;
          u.load(xr + k);
          v.load(ar + k);
#pragma unroll
          for (int i = 0; i < V; ++i) sum = acc_fma(u.v[i], v.v[i], sum);
        }
      }
    }
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) s_sum[warp] = sum;
  __syncthreads();
  if (lane != 0 || part != 0 || j >= rank) return;
  for (int k = 1; k < parts; ++k) sum += s_sum[warp + k * jn];
  lr_store(h, t, j, rank, (float)(scale ? sum * (acc_t)scale[ad] : sum));
}

// fp32: y[t] = s_a B_a h[t], 0 without an adapter; the projection's launch adds it as its residual operand.  Starts while the launch that writes h runs: h must not be
// __restrict__, which would promise that nobody writes it for as long as this kernel lives.
__global__ void __launch_bounds__(256)
lowrank_delta_kernel(const float* __restrict__ b, const int32_t* __restrict__ which, const float* h, float* y, int n, int rank, int adapters) {
  __shared__ float s_h[kLrMaxRank];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int t = blockIdx.x, f = (int)blockIdx.y * 256 + threadIdx.x;
  const int ad = which[t];
  const bool has = ad >= 0 && ad < adapters;
  if (has)
    for (int j = threadIdx.x; j < rank; j += 256) s_h[j] = h[(size_t)t * rank + j];
  __syncthreads();
  if (f >= n) return;
  double sum = 0.0;
  if (has) {
    const float* br = b + ((size_t)ad * n + f) * rank;
    for (int j = 0; j < rank; ++j) sum = acc_fma(s_h[j], br[j], sum);
  }
  y[(size_t)t * n + f] = (float)sum;
}

// ----------------------------------------------------------------------------- host side

struct LrContext {
  PFN_encodeTiled encode_tiled = nullptr;
  int sm_count = 148;
  int fit[4] = {};   // clusters of 1, 2, 4 and 8 CTAs, one an SM, that run side by side: what a group of SMs has left over is too few for another
};

inline cudaError_t lr_map(const LrContext& c, CUtensorMap* tm, const void* base, long rows, int cols, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)cols * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  const cuuint32_t es[2] = {1, 1};
  return c.encode_tiled(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess
             : cudaErrorInvalidValue;
}

inline cudaError_t lr_context_init(LrContext& ctx) {   // once per device
  cudaError_t e = cudaSuccess;
  auto set = [&](auto kernel, int bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  set(lowrank_tcgen05_kernel<16, false, false, false>, LrSmem<16, false>::kBytes);
  set(lowrank_tcgen05_kernel<16, false, false, true>, LrSmem<16, false>::kBytes);
  set(lowrank_tcgen05_kernel<32, false, false, false>, LrSmem<32, false>::kBytes);
  set(lowrank_tcgen05_kernel<32, false, false, true>, LrSmem<32, false>::kBytes);
  set(lowrank_tcgen05_kernel<64, false, false, false>, LrSmem<64, false>::kBytes);
  set(lowrank_tcgen05_kernel<64, false, false, true>, LrSmem<64, false>::kBytes);
  set(lowrank_tcgen05_kernel<128, false, false, false>, LrSmem<128, false>::kBytes);
  set(lowrank_tcgen05_kernel<128, false, false, true>, LrSmem<128, false>::kBytes);
  set(lowrank_tcgen05_kernel<128, true, false, false>, LrSmem<128, true>::kBytes);
  set(lowrank_tcgen05_kernel<128, true, false, true>, LrSmem<128, true>::kBytes);
  set(lowrank_tcgen05_kernel<256, true, false, false>, LrSmem<256, true>::kBytes);
  set(lowrank_tcgen05_kernel<256, true, false, true>, LrSmem<256, true>::kBytes);
  set(lowrank_tcgen05_kernel<kLrShrinkTN, false, true, false>, LrSmem<kLrShrinkTN, false, true>::kBytes);
  set(lowrank_tcgen05_kernel<kLrShrinkTN, false, true, true>, LrSmem<kLrShrinkTN, false, true>::kBytes);
  for (int i = 0; i < 4 && e == cudaSuccess; ++i) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1u << i;
    cfg.gridDim = dim3(1, 1, 1u << i);
    cfg.blockDim = dim3(kLrThreads<false, false>);
    cfg.dynamicSmemBytes = LrSmem<64, false>::kBytes;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&ctx.fit[i], lowrank_tcgen05_kernel<64, false, false, false>, &cfg);
  }
  return e;
}

template <int TN, bool PERSIST, bool SHRINK, bool COPY>
inline cudaError_t lr_launch_k(const CUtensorMap& tmA, const CUtensorMap& tmX, const LrArgs& a, dim3 grid, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kLrThreads<COPY, SHRINK>);
  cfg.dynamicSmemBytes = LrSmem<TN, PERSIST, SHRINK>::kBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (!SHRINK && a.adapters > 0) {   // the first launch follows the stream plainly, so what both read and what this one overwrites is the stream's past
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (grid.z > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = grid.z;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, lowrank_tcgen05_kernel<TN, PERSIST, SHRINK, COPY>, tmA, tmX, a);
}

struct LrPlan {
  int tn, splits;          // rows of a tile; CTAs that share its K
  bool persist;            // more tiles than SMs
  bool simt;               // h on CUDA cores
  int jn;                  // rows of A_a of a CTA there
  int h_groups, h_splits;  // on the tensor cores: CTAs that share a tile's groups of adapters, and the K of one
};

inline LrPlan lr_plan(int rows, int c, int n, int rank, int adapters, const LrContext& ctx) {
  const int sms = ctx.sm_count;
  LrPlan p;
  // Clocks a K block of a tile takes in a full grid, 470 of 128 rows and 750 of 256, times the tiles an SM gets.
  auto rounds = [&](int tn) { return ((long)cdiv(n, 128) * cdiv(rows, tn) + sms - 1) / sms; };
  p.tn = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : rounds(256) * 750 <= rounds(128) * 470 ? 256 : 128;
  const int kb = cdiv(c, 64);
  // Twice as many CTAs while their clusters fit side by side (16 of eight CTAs do not: 16 x 2048 x 2048 13.6 us, with clusters of four 8.5) and each has a block of K: an exchange costs less than what further CTAs take off the adapters' columns and the copies.
  // us, one / two / four blocks at least: 160x360x1756 with 23 adapters of rank 32 19 / 27 / 37, 1166x444x184 16 / 20 / 24, 7x304x300 12 / 16 / 21, 196x312x35
  // 14 / 16 / 13.  The adapters have no say: rows without one come out the same whatever the others have.
  auto share = [&](long tiles, int per_sm) {
    int i = 0;
    while (i < 3 && tiles <= ctx.fit[i + 1] * per_sm && kb >= 2 << i) ++i;
    return 1 << i;
  };
  const long tiles = (long)cdiv(n, 128) * cdiv(rows, p.tn);
  p.persist = p.tn == 256 || (p.tn == 128 && tiles > sms);
  p.splits = p.persist ? 1 : share(tiles, 1);
  p.simt = (long)rows * rank * c <= kLrSimtWork;
  p.jn = 8;
  while (p.jn > 1 && (long)rows * cdiv(rank, p.jn) < 2L * sms) p.jn /= 2;
  // A tile whose rows are sorted has a group or two, one of mixed rows up to all: K is cut for two groups a tile, or for four CTAs, and further ones take what groups there
  // are side by side.  us of a call, sorted / mixed rows, all for the cut and one group after the other / so: 256 x 4096 x 4096 with eight adapters of rank 64 40 / 54, 35 / 40,
  // 1402 x 2288 x 1802 with ten 52 / 94, 50 / 85; 4096 x 4096 x 4096 with nine, never more than half for the cut / so: 141 / 257, 134 / 262.
  const int h_tiles = cdiv(rows, kLrShrinkTN), groups = cdiv(std::min(adapters, kLrShrinkTN), 128 / (int)align_up(rank, 8));
  p.h_splits = std::max(share((long)h_tiles * std::min(std::max(groups, 1), 2), 2), std::min(share(h_tiles, 2), 4));
  p.h_groups = std::max(1, std::min(groups, 2 * sms / (h_tiles * p.h_splits)));
  return p;
}

template <int TN, bool PERSIST>
inline cudaError_t lr_expand(bool copy, const CUtensorMap& tmW, const CUtensorMap& tmX, const LrArgs& a, int splits, int sms, cudaStream_t st) {
  const dim3 grid = PERSIST ? dim3(std::min(sms, cdiv(a.n, 128) * cdiv(a.rows, TN))) : dim3(cdiv(a.n, 128), cdiv(a.rows, TN), splits);
  return copy ? lr_launch_k<TN, PERSIST, false, true>(tmW, tmX, a, grid, st) : lr_launch_k<TN, PERSIST, false, false>(tmW, tmX, a, grid, st);
}

template <typename T>
inline cudaError_t lr_shrink_simt(const T* x, const T* a, const float* scale, const int32_t* which, T* h, int rows, int c, int rank, int adapters, int jn, cudaStream_t st) {
  constexpr int V = Elem<T>::kVec;
  const uintptr_t bits = (uintptr_t)x | (uintptr_t)a;
  const dim3 grid(rows, cdiv(rank, jn));
  if (c % V == 0 && (bits & 15) == 0) lowrank_shrink_kernel<T, V><<<grid, 256, 0, st>>>(x, a, scale, which, h, c, rank, adapters, jn);
  else if (c % (V / 2) == 0 && (bits & 7) == 0) lowrank_shrink_kernel<T, V / 2><<<grid, 256, 0, st>>>(x, a, scale, which, h, c, rank, adapters, jn);
  else lowrank_shrink_kernel<T, 1><<<grid, 256, 0, st>>>(x, a, scale, which, h, c, rank, adapters, jn);
  return cudaGetLastError();
}

inline cudaError_t lr_run_bf16(const LrContext& ctx, LrArgs a, cudaStream_t st) {
  const LrPlan p = lr_plan(a.rows, a.c, a.n, a.rank, a.adapters, ctx);
  const uintptr_t bits = (uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.a;
  const bool copy = a.c % 8 != 0 || (bits & 15) != 0;
  a.unit = a.c % 4 == 0 && (bits & 7) == 0 ? 8 : a.c % 2 == 0 && (bits & 3) == 0 ? 4 : 2;
  a.r8 = (int)align_up(a.rank, 8);
  const bool wide = a.adapters > 0 && !p.simt;         // h on the tensor cores
  CUtensorMap tmW = {}, tmX = {}, tmA = {}, tmH = {};
  cudaError_t e = cudaSuccess;
  if (!copy) {
    e = lr_map(ctx, &tmW, a.w, a.n, a.c, 128);
    if (e == cudaSuccess) e = lr_map(ctx, &tmX, a.x, a.rows, a.c, p.tn);
    if (e == cudaSuccess && wide) e = lr_map(ctx, &tmA, a.a, (long)a.adapters * a.rank, a.c, a.r8);
    if (e == cudaSuccess && wide) e = lr_map(ctx, &tmH, a.x, a.rows, a.c, kLrShrinkTN);
    if (e != cudaSuccess) return e;
  }
  if (wide) {
    const dim3 grid(cdiv(a.rows, kLrShrinkTN), p.h_groups, p.h_splits);
    e = copy ? lr_launch_k<kLrShrinkTN, false, true, true>(tmA, tmH, a, grid, st) : lr_launch_k<kLrShrinkTN, false, true, false>(tmA, tmH, a, grid, st);
  } else if (a.adapters > 0) {
    e = lr_shrink_simt<bf16>(a.x, a.a, a.scale, a.which, a.h, a.rows, a.c, a.rank, a.adapters, p.jn, st);
  }
  if (e != cudaSuccess) return e;
  switch (p.tn) {
    case 16: return lr_expand<16, false>(copy, tmW, tmX, a, p.splits, ctx.sm_count, st);
    case 32: return lr_expand<32, false>(copy, tmW, tmX, a, p.splits, ctx.sm_count, st);
    case 64: return lr_expand<64, false>(copy, tmW, tmX, a, p.splits, ctx.sm_count, st);
    case 128: return p.persist ? lr_expand<128, true>(copy, tmW, tmX, a, p.splits, ctx.sm_count, st) : lr_expand<128, false>(copy, tmW, tmX, a, p.splits, ctx.sm_count, st);
    default: return lr_expand<256, true>(copy, tmW, tmX, a, p.splits, ctx.sm_count, st);
  }
}

// fp32: h and the adapters' share on CUDA cores (summed in fp64, like everything of the fp32 model), then the projection on the convolution kernel of
// the fp32 model as a 1x1 layer of one pixel a row, which adds that share.
inline cudaError_t lr_run_f32(const LrContext& ctx, const float* x, const float* w, const float* bias, const float* a, const float* b, const float* scale,
                              const int32_t* which, float* h, float* y, int rows, int c, int n, int rank, int adapters, int* err_flag, long long wait_cycles,
                              cudaStream_t st) {
  const LrPlan p = lr_plan(rows, c, n, std::max(rank, 1), adapters, ctx);
  if (adapters > 0) {
    cudaError_t e = lr_shrink_simt<float>(x, a, scale, which, h, rows, c, rank, adapters, p.jn, st);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(rows, cdiv(n, 256));
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, lowrank_delta_kernel, b, which, (const float*)h, y, n, rank, adapters);
    if (e != cudaSuccess) return e;
  }
  const bool vec = c % 4 == 0 && (((uintptr_t)x | (uintptr_t)w) & 15) == 0;
  const ConvGeom g{rows, 1, 1, c, 1, 1, n, 1, 1, 1, 0, 0, EE_ACT_NONE};
  // Behind the adapters' launches, which the stream's past is over for, W and the bias may be fetched early; behind anything else they may be its output.
  return f32_launch(f32_plan(rows, n, c, ctx.sm_count, vec), x, w, nullptr, bias, adapters > 0 ? y : nullptr, y, g, err_flag, wait_cycles, st, adapters > 0);
}

}  // namespace ee
