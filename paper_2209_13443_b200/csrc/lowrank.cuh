// A projection shared by all rows of a batch, with a low-rank adapter of each row's own beside it:
//   y[t] = W x[t] + bias + s_a B_a (A_a x[t]),  a = which[t]  (no adapter where which[t] is not one).
//
// Two launches.  The first forms h[t] = s_a A_a x[t], rank numbers a row, in the caller's workspace; the second is the product with W on
// tcgen05, whose K loop goes on behind the last channel: for the adapters that occur in its tile of rows it appends columns, of
// B_a on one side and of h[t] on the other, zero in the rows of other adapters.  So the adapters of a tile, in any order and mix, cost
// their rank in additional K, and the sum is rounded once.  h is kept and multiplied as two bf16 parts, h and what its rounding left (2^-17
// of h together, 2 rank columns): rounded to one part the adapter's share would carry a second rounding of the size of the result's.
//
// The tile is turned: 128 filters are the rows of the accumulator (lanes) and 16 to 128 rows of the batch its columns, so that few
// rows cost few columns, and W, which bounds small batches, is read once.  There K is cut over a cluster of up to eight CTAs, which
// send each other their parts as asynchronous stores and add them in fixed order.  The first launch is a product of the same shape, 128 rows of
// stacked A_a over 64 rows of the batch; up to kLrSimtRows rows CUDA cores do it, a warp a row of A_a.
// The second launch starts while the first runs and waits for it only before it fills in h.  The adapters' columns take ring slots behind the last channel's: the
// producer of W, which walks the ring anyway, hands them to the four warps that gather the columns, while the products before them still run.  Grids of more than one
// tile an SM use a ring of three slots, so that two CTAs share an SM and one's columns and stores lie under the other's products; smaller ones a
// deep ring, for the bytes in flight.
//
// Channels that are not whole 16-byte vectors, or operands off a 16-byte boundary, cannot be fetched by TMA: eight warps then copy the
// tiles (COPY), 2 or 4 bytes at a time.
#pragma once
#include "common.cuh"
#include "conv_f32.cuh"
#include "conv_tc.cuh"

namespace ee {

constexpr int kLrParts = 2;            // bf16 parts of h
constexpr int kLrMaxRank = 128;
constexpr int kLrMaxSplits = 8;        // CTAs of a cluster
constexpr int kLrShrinkTN = 64;        // rows of a tile of the first launch
constexpr int kLrSimtRows = 96;
constexpr int kLrCopyWarps = 8;

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
  bool pairs;          // COPY: rows start on 4-byte boundaries
  int* err_flag;
};

template <int TN, bool DEEP>
struct LrSmem {
  static constexpr int kABytes = 128 * 128, kBBytes = TN * 128, kStage = kABytes + kBBytes;
  static constexpr int kStages = !DEEP ? 3 : TN == 128 ? 4 : 7;
  static constexpr int kPart = TN * 128 * 4;                        // partial sums: a shrink's h of its rows (up to 128 numbers each); else what the cluster's CTAs send
  static constexpr int kOffPart = kStages * kStage;
  static constexpr int kOffInts = kOffPart + (DEEP ? kPart : 0);    // grids of a shallow ring do not cut K
  static constexpr int kInts = 3 * TN + 16;                         // adapter and slot of each row, adapters of the tile, masks and counts
  static constexpr int kOffBars = kOffInts + kInts * 4;
  static constexpr int kBytes = kOffBars + 8 * (3 * kStages + 3) + 1024;
  static_assert(kBytes <= 227 * 1024, "exceeds the shared memory of an SM");
  static_assert(DEEP || 2 * (kBytes + 1024) <= 228 * 1024, "two CTAs of a shallow ring share an SM");
};

__device__ __forceinline__ void mbar_arrive_n(uint32_t bar, uint32_t n) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}

// Number j of row t's h: for the bf16 product as two parts, for the fp32 one as it is.
__device__ __forceinline__ void lr_store(bf16* h, int t, int j, int rank, float v) {
  const bf16 hi = __float2bfloat16_rn(v);
  h[((size_t)t * 2) * rank + j] = hi;
  h[((size_t)t * 2 + 1) * rank + j] = __float2bfloat16_rn(v - __bfloat162float(hi));
}
__device__ __forceinline__ void lr_store(float* h, int t, int j, int rank, float v) { h[(size_t)t * rank + j] = v; }

// Zeros in the place of infinities and NaN among two bf16 values; whether there were any.
__device__ __forceinline__ uint32_t lr_drop(uint32_t& w) {
  const uint32_t m = __vcmpeq2(w & 0x7f807f80u, 0x7f807f80u);
  w &= ~m;
  return m;
}
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
// blockIdx.x: tile of filters (SHRINK: of stacked adapters), y: tile of rows, z: range of K.
template <int TN, bool DEEP, bool SHRINK, bool COPY>
__global__ void __launch_bounds__(COPY ? 192 + 32 * kLrCopyWarps : 224)
lowrank_tcgen05_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmX, LrArgs p) {
  static_assert(DEEP || !SHRINK, "a shrink keeps its partial sums beside the ring");
  using S = LrSmem<TN, DEEP>;
  constexpr int kStages = S::kStages;
  constexpr uint32_t kFull = COPY ? 32 * kLrCopyWarps : 2;   // arrivals that fill a slot
  extern __shared__ uint8_t lr_smem[];
  const uint32_t raw = smem_u32(lr_smem), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = lr_smem + (base - raw);
  int* s_ad = reinterpret_cast<int*>(gen + S::kOffInts);     // [TN] adapter of a row, -1: none
  int* s_slot = s_ad + TN;                                   // [TN] its place among the tile's adapters
  int* s_list = s_slot + TN;                                 // [TN] the tile's adapters, in order of first occurrence
  unsigned* s_mask = reinterpret_cast<unsigned*>(s_list + TN);   // [4]
  int* s_count = reinterpret_cast<int*>(s_mask) + 8;
  uint32_t* tmem_slot = s_mask + 9;
  int* s_bad = s_count + 2;                                  // set where a B_a of the tile holds infinities or NaN
  const uint32_t bar0 = base + S::kOffBars;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kStages + s); };
  auto grant_bar = [&](int s) { return bar0 + 8u * (2 * kStages + s); };     // the slot is free for adapter columns
  const uint32_t accum_bar = bar0 + 8u * (3 * kStages), list_bar = accum_bar + 8u, part_bar = list_bar + 8u;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int t0 = (int)blockIdx.y * TN, n0 = (int)blockIdx.x * 128;
  const int z = (int)blockIdx.z, Z = (int)gridDim.z;
  const int kb_all = (p.c + 63) / 64;
  const int kb0 = (int)((long)kb_all * z / Z), num_kb = (int)((long)kb_all * (z + 1) / Z) - kb0;   // Z <= kb_all: never empty

  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) mbar_init(full_bar(s), kFull), mbar_init(empty_bar(s), 1), mbar_init(grant_bar(s), 1);
    mbar_init(accum_bar, 1);
    mbar_init(list_bar, 1);
    mbar_init(part_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (!SHRINK && Z > 1) mbar_expect_tx(part_bar, (uint32_t)S::kPart);     // TN / Z columns from each of Z CTAs
  }
  constexpr uint32_t kCols = TN < 32 ? 32 : TN;
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  if (SHRINK) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (Z > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");       // waited for before anything is sent

  // The tile's adapters: a row is the first of its adapter, or refers to it.
  if (warp >= 2 && warp < 6) {
    const int et = tid - 64;
    for (int i = et; i < TN; i += 128) {
      const int t = t0 + i, a = t < p.rows && p.adapters > 0 ? p.which[t] : -1;
      s_ad[i] = a >= 0 && a < p.adapters ? a : -1;
    }
    asm volatile("bar.sync 1, 128;" ::: "memory");
    const int a = et < TN ? s_ad[et] : -1;
    int f = (et & ~31) + __ffs(__match_any_sync(0xffffffffu, a)) - 1;       // the first of its warp
    if (a >= 0 && f == et)
      for (int u = 0; u < (et & ~31); u += 4) {
        const int4 o = *reinterpret_cast<const int4*>(s_ad + u);
        if (o.w == a) f = min(f, u + 3);
        if (o.z == a) f = min(f, u + 2);
        if (o.y == a) f = min(f, u + 1);
        if (o.x == a) f = min(f, u);
      }
    f = __shfl_sync(0xffffffffu, f, f >= (et & ~31) ? f & 31 : lane);       // the others of the warp take what their first found
    const unsigned lead = __ballot_sync(0xffffffffu, a >= 0 && f == et);
    if (lane == 0 && et < TN) s_mask[et >> 5] = lead;
    asm volatile("bar.sync 1, 128;" ::: "memory");
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
    if (et == 0) *s_count = count, *s_bad = 0;
    asm volatile("bar.sync 1, 128;" ::: "memory");
    if (et == 0) mbar_arrive_n(list_bar, 1);
  }
  const int per_tile = 128 / p.r8;               // SHRINK: adapters of a tile
  int here = 0;
  if (SHRINK) {
    __syncthreads();
    here = min(per_tile, *s_count - (int)blockIdx.x * per_tile);
  }
  const bool idle = SHRINK && here <= 0;         // this CTA's adapters do not occur
  const int ext_cols = kLrParts * p.rank;        // columns of an adapter
  // blocks of adapter columns that this CTA takes: z, z + Z, ...
  auto ext_blocks = [&](int count) {
    const int all = (int)(((long)count * ext_cols + 63) / 64);
    return all > z ? (all - z + Z - 1) / Z : 0;
  };

  if (idle) {
  } else if (warp == 0) {
    if (elect_one()) {
      int s = 0;
      uint32_t ph = 1;
      bool ok = true;
      for (int i = 0; !COPY && i < num_kb; ++i) {
        if (i >= kStages && !(ok = mbar_wait(empty_bar(s), ph, p.err_flag))) break;
        const uint32_t dst = base + (uint32_t)s * S::kStage;
        if (SHRINK) {
          mbar_expect_tx(full_bar(s), (uint32_t)(here * p.r8 * 128));
          for (int k = 0; k < here; ++k)
            tma_load_2d(dst + (uint32_t)(k * p.r8 * 128), &tmA, full_bar(s), (kb0 + i) * 64, s_list[(int)blockIdx.x * per_tile + k] * p.rank);
        } else {
          mbar_expect_tx(full_bar(s), S::kABytes);
          tma_load_2d(dst, &tmA, full_bar(s), (kb0 + i) * 64, n0);
        }
        if (++s == kStages) s = 0, ph ^= 1u;
      }
      if (!SHRINK && !COPY && ok && mbar_wait(list_bar, 0, p.err_flag)) {     // COPY: the first of its warps does this
        const int ext = ext_blocks(*s_count);
        for (int i = num_kb; i < num_kb + ext; ++i) {
          if (i >= kStages && !mbar_wait(empty_bar(s), ph, p.err_flag)) break;
          mbar_arrive_n(grant_bar(s), 1);
          if (++s == kStages) s = 0, ph ^= 1u;
        }
      }
    }
    __syncwarp();
  } else if (!COPY && warp == 6) {
    if (elect_one()) {
      int s = 0;
      uint32_t ph = 1;
      for (int i = 0; i < num_kb; ++i) {
        if (i >= kStages && !mbar_wait(empty_bar(s), ph, p.err_flag)) break;
        mbar_expect_tx(full_bar(s), S::kBBytes);
        tma_load_2d(base + (uint32_t)s * S::kStage + S::kABytes, &tmX, full_bar(s), (kb0 + i) * 64, t0);
        if (++s == kStages) s = 0, ph ^= 1u;
      }
    }
    __syncwarp();
  } else if (COPY && warp >= 6) {
    const int cw = warp - 6;
    int s = 0;
    uint32_t ph = 1;
    for (int i = 0; i < num_kb; ++i) {
      if (i >= kStages && !mbar_wait(empty_bar(s), ph, p.err_flag)) break;
      uint8_t* dst = gen + (size_t)s * S::kStage;
      const int k0 = (kb0 + i) * 64 + 2 * lane;
#pragma unroll 8
      for (int r = cw; r < 128 + TN; r += kLrCopyWarps) {
        const bf16* src = nullptr;
        if (r >= 128) {
          if (t0 + r - 128 < p.rows) src = p.x + (size_t)(t0 + r - 128) * p.c;
        } else if (SHRINK) {
          const int k = r / p.r8, j = r - k * p.r8;
          if (k < here && j < p.rank) src = p.a + ((size_t)s_list[(int)blockIdx.x * per_tile + k] * p.rank + j) * p.c;
        } else if (n0 + r < p.n) {
          src = p.w + (size_t)(n0 + r) * p.c;
        }
        uint32_t v = 0;
        if (src) {
          if (p.pairs) {                               // c is even: a pair lies inside the row or outside it
            if (k0 < p.c) v = *reinterpret_cast<const uint32_t*>(src + k0);
          } else {
            const unsigned short* e = reinterpret_cast<const unsigned short*>(src);
            if (k0 < p.c) v = e[k0];
            if (k0 + 1 < p.c) v |= (uint32_t)e[k0 + 1] << 16;
          }
        }
        *reinterpret_cast<uint32_t*>(dst + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4) = v;
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive_n(full_bar(s), 1);
      if (++s == kStages) s = 0, ph ^= 1u;
    }
    if (!SHRINK && cw == 0 && elect_one() && mbar_wait(list_bar, 0, p.err_flag)) {
      const int ext = ext_blocks(*s_count);
      for (int i = num_kb; i < num_kb + ext; ++i) {
        if (i >= kStages && !mbar_wait(empty_bar(s), ph, p.err_flag)) break;
        mbar_arrive_n(grant_bar(s), 1);
        if (++s == kStages) s = 0, ph ^= 1u;
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (elect_one()) {
      constexpr uint32_t idesc = umma_idesc(TN);
      const uint64_t da0 = umma_desc(base), db0 = umma_desc(base + S::kABytes);
      int s = 0, blocks = num_kb;
      uint32_t ph = 0;
      bool ok = true;
      for (int i = 0;; ++i) {
        if (!SHRINK && i == num_kb) {                  // by now the list is long there
          ok = mbar_wait(list_bar, 0, p.err_flag);
          if (!ok) break;
          blocks += ext_blocks(*s_count);
        }
        if (i >= blocks) break;
        ok = mbar_wait(full_bar(s), ph, p.err_flag);
        if (!ok) break;
        tc_fence_after();
        const uint64_t off = (uint64_t)(s * (S::kStage >> 4));
        umma_block(tmem, da0 + off, db0 + off, idesc, i != 0);
        umma_commit(empty_bar(s));
        if (++s == kStages) s = 0, ph ^= 1u;
      }
      if (ok) umma_commit(accum_bar);
    }
    __syncwarp();
  } else {
    const int et = tid - 64, q = warp & 3;
    const int row = q * 32 + lane;                     // accumulator lane of this thread
    bool ok = true;
    if constexpr (!SHRINK) {
      // Block e of adapter columns goes into the ring as K block num_kb + e.  A thread has the 16-byte chunk et % 8 of 64 columns, in every sixteenth row of either operand.
      const int ext = ext_blocks(*s_count), all = *s_count * ext_cols, c8 = et & 7, r0 = et >> 3;
      const bool whole = p.rank % 8 == 0, vec = whole && ((uintptr_t)p.b & 15) == 0;   // eight columns are one part of one adapter; of B_a one load
      auto place = [&](int r) { return (uint32_t)(r * 128 + ((c8 ^ (r & 7)) << 4)); };
      auto column = [&](int e, int k, int& slot, int& rem) {       // adapter and place in its 2 * rank columns; slot -1: behind the last
        const int c = (z + e * Z) * 64 + c8 * 8 + k;
        slot = c / ext_cols, rem = c - slot * ext_cols;
        if (c >= all) slot = -1;
      };
      auto fetch = [&](uint32_t dst, const void* src, bool in) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
      };
      auto slot_of_block = [&](int e) { return (num_kb + e) % kStages; };
      auto fill_b = [&](int e) {
        const int s = slot_of_block(e);
        // use u of this slot: the u-th grant of it follows those of the blocks of adapter columns before this one
        ok = ok && mbar_wait(grant_bar(s), (uint32_t)(e / kStages) & 1u, p.err_flag);
        uint8_t* tile = gen + (size_t)s * S::kStage;
        int slot, rem;
        if (vec) {
          column(e, 0, slot, rem);
          const bf16* src = slot >= 0 ? p.b + ((size_t)s_list[slot] * p.n + n0) * p.rank + (rem < p.rank ? rem : rem - p.rank) : p.b;
#pragma unroll
          for (int m = 0; m < 8; ++m) {
            const int r = r0 + 16 * m;
            const bool in = slot >= 0 && n0 + r < p.n;
            fetch(base + (uint32_t)s * S::kStage + place(r), in ? src + (size_t)r * p.rank : p.b, in);
          }
        } else {
          int ad[8], j[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            column(e, k, slot, rem);
            ad[k] = slot >= 0 ? s_list[slot] : -1, j[k] = rem < p.rank ? rem : rem - p.rank;
          }
#pragma unroll 2
          for (int m = 0; m < 8; ++m) {
            const int r = r0 + 16 * m, f = n0 + r;
            uint32_t v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = ad[k] >= 0 && f < p.n ? reinterpret_cast<const unsigned short*>(p.b)[((size_t)ad[k] * p.n + f) * p.rank + j[k]] : 0u;
            *reinterpret_cast<uint4*>(tile + place(r)) = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
          }
        }
      };
      auto fill_h = [&](int e) {
        const int s = slot_of_block(e);
        const uint32_t at = base + (uint32_t)s * S::kStage + S::kABytes;
        int slot, rem;
        if (whole) {                       // the workspace is aligned, and so are eight columns of a row
          column(e, 0, slot, rem);
#pragma unroll
          for (int m = 0; m < TN / 16; ++m) {
            const int t = r0 + 16 * m;
            const bool in = slot >= 0 && s_slot[t] == slot;
            fetch(at + place(t), in ? p.h + (size_t)(t0 + t) * ext_cols + rem : p.h, in);
          }
        } else {
          int slots[8], rems[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) column(e, k, slots[k], rems[k]);
#pragma unroll 2
          for (int m = 0; m < TN / 16; ++m) {
            const int t = r0 + 16 * m, mine = s_slot[t];
            const unsigned short* h = reinterpret_cast<const unsigned short*>(p.h) + (size_t)(t0 + t) * ext_cols;
            uint32_t v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = mine >= 0 && slots[k] == mine ? h[rems[k]] : 0u;
            *reinterpret_cast<uint4*>(gen + (size_t)s * S::kStage + S::kABytes + place(t)) = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
          }
        }
        cp_async_commit();
      };
      auto finish = [&](int e) {           // what this thread fetched is here: an infinity would turn the zeros of other adapters' rows into NaN, so
        const int s = slot_of_block(e);    // lr_not_finite adds it to its own rows
        uint8_t* tile = gen + (size_t)s * S::kStage;
#pragma unroll
        for (int m = 0; m < 8; ++m) {
          uint4* o = reinterpret_cast<uint4*>(tile + place(r0 + 16 * m));
          uint4 v = *o;
          if (lr_drop(v.x) | lr_drop(v.y) | lr_drop(v.z) | lr_drop(v.w)) *s_bad = 1, *o = v;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (et == 0) mbar_arrive_n(full_bar(s), kFull);
      };
      // B_a of the first blocks before the wait for h (no kernel writes it); then one block is fetched while the one before it is finished
      constexpr int kAhead = 2;
      for (int e = 0; e < ext && e < kAhead; ++e) fill_b(e);
      asm volatile("griddepcontrol.wait;" ::: "memory");
      if (ext > 0) fill_h(0);
      if (ext > 1) fill_h(1);
      for (int e = 0; e < ext; ++e) {
        if (e + 1 < ext) cp_async_wait<1>();
        else cp_async_wait<0>();
        finish(e);
        if (e + kAhead < ext) fill_b(e + kAhead), fill_h(e + kAhead);
      }
    }
    ok = __all_sync(0xffffffffu, mbar_wait(accum_bar, 0, p.err_flag));
    tc_fence_after();
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
    constexpr int CH = TN < 32 ? TN : 32;              // columns read at a time
    if constexpr (SHRINK) {
      // this CTA's part of h: [TN][r8] floats, of the rows whose adapter is in its tile
      const int k = row / p.r8, j = row - k * p.r8, slot = (int)blockIdx.x * per_tile + k;
      float* part = reinterpret_cast<float*>(gen + S::kOffPart);
#pragma unroll 1
      for (int c = 0; c < TN; c += CH) {
        float v[CH];
        if constexpr (CH == 32) tmem_ld32(lane_base + c, v);
        else tmem_ld16(lane_base + c, v);
        if (k < here)
#pragma unroll
          for (int i = 0; i < CH; ++i)
            if (s_slot[c + i] == slot) part[(c + i) * p.r8 + j] = v[i];
      }
    } else {
      const int f = n0 + row;
      const float bias = p.bias && f < p.n ? p.bias[f] : 0.f;
      const bool bad = *s_bad != 0 && f < p.n;
      auto columns_of = [&](int c, float* v) {
        if constexpr (CH == 32) tmem_ld32(lane_base + c, v);
        else tmem_ld16(lane_base + c, v);
        if (bad)
#pragma unroll
          for (int i = 0; i < CH; ++i) v[i] += lr_not_finite(p, t0 + c + i, f, s_ad[c + i], s_slot[c + i], z, Z);
      };
      if (Z == 1) {
        // Two neighbouring lanes trade: the even one stores both filters of the even rows, the odd one those of the odd rows, 4 bytes each.
        const bool pairs = p.n % 2 == 0 && ((uintptr_t)p.y & 3) == 0;
#pragma unroll 1
        for (int c = 0; c < TN; c += CH) {
          float v[CH];
          columns_of(c, v);
          if (pairs) {
#pragma unroll
            for (int i = 0; i < CH; i += 2) {
              const float give = (lane & 1 ? v[i] : v[i + 1]) + bias, keep = (lane & 1 ? v[i + 1] : v[i]) + bias, got = __shfl_xor_sync(0xffffffffu, give, 1);
              const int t = t0 + c + i + (lane & 1);
              if (ok && f < p.n && t < p.rows)         // n is even: both filters of a pair are there, or neither
                *reinterpret_cast<uint32_t*>(p.y + (size_t)t * p.n + (f & ~1)) = lane & 1 ? pack_bf16x2(got, keep) : pack_bf16x2(keep, got);
            }
          } else if (ok && f < p.n) {
#pragma unroll
            for (int i = 0; i < CH; ++i)
              if (t0 + c + i < p.rows) p.y[(size_t)(t0 + c + i) * p.n + f] = __float2bfloat16_rn(v[i] + bias);
          }
        }
      } else if constexpr (DEEP) {
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
        const bool sent = mbar_wait_cluster(part_bar, 0, p.err_flag, kTcWaitCycles) || mbar_wait_cluster(part_bar, 0, p.err_flag, kTcWaitCycles);
        const float* in = reinterpret_cast<const float*>(gen + S::kOffPart);
        const int run = min(share, 4);
        for (int i = 0; i < share; i += run) {
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
          for (int k = 0; k < Z; ++k) {
            if (run == 4) {
              const float4 o = *reinterpret_cast<const float4*>(in + (k * share + i) * 128 + row * 4);
              sum[0] += o.x, sum[1] += o.y, sum[2] += o.z, sum[3] += o.w;
            } else {
              const float2 o = *reinterpret_cast<const float2*>(in + k * 256 + row * 2);
              sum[0] += o.x, sum[1] += o.y;
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int t = t0 + z * share + i + j;
            if (j < run && ok && sent && f < p.n && t < p.rows) p.y[(size_t)t * p.n + f] = __float2bfloat16_rn(sum[j] + bias);
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
        const int t = i / p.rank * Z + z, j = i - i / p.rank * p.rank, slot = s_slot[t] - (int)blockIdx.x * per_tile;
        if (slot < 0 || slot >= here) continue;
        float sum = 0.f;
        for (int r = 0; r < Z; ++r) {
          uint32_t from;
          float v;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(part + 4u * (t * p.r8 + j)), "r"(r));
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(from) : "memory");
          sum += v;
        }
        lr_store(p.h, t0 + t, j, p.rank, p.scale ? sum * p.scale[s_ad[t]] : sum);
      }
      if (Z > 1) asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");   // nobody reads this CTA's part any more
    }
  }
  __syncthreads();
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
  const float f = (float)sum;
  lr_store(h, t, j, rank, scale ? f * scale[ad] : f);
}

// fp32: y[t] = s_a B_a h[t], 0 without an adapter; the projection's launch adds it as its residual operand.
__global__ void __launch_bounds__(256)
lowrank_delta_kernel(const float* __restrict__ b, const int32_t* __restrict__ which, const float* __restrict__ h, float* __restrict__ y, int n, int rank, int adapters) {
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

inline cudaError_t lr_context_init() {   // once per device
  cudaError_t e = cudaSuccess;
  auto set = [&](auto kernel, int bytes) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  set(lowrank_tcgen05_kernel<16, true, false, false>, LrSmem<16, true>::kBytes);
  set(lowrank_tcgen05_kernel<16, true, false, true>, LrSmem<16, true>::kBytes);
  set(lowrank_tcgen05_kernel<32, true, false, false>, LrSmem<32, true>::kBytes);
  set(lowrank_tcgen05_kernel<32, true, false, true>, LrSmem<32, true>::kBytes);
  set(lowrank_tcgen05_kernel<64, true, false, false>, LrSmem<64, true>::kBytes);
  set(lowrank_tcgen05_kernel<64, true, false, true>, LrSmem<64, true>::kBytes);
  set(lowrank_tcgen05_kernel<128, true, false, false>, LrSmem<128, true>::kBytes);
  set(lowrank_tcgen05_kernel<128, true, false, true>, LrSmem<128, true>::kBytes);
  set(lowrank_tcgen05_kernel<128, false, false, false>, LrSmem<128, false>::kBytes);
  set(lowrank_tcgen05_kernel<128, false, false, true>, LrSmem<128, false>::kBytes);
  set(lowrank_tcgen05_kernel<kLrShrinkTN, true, true, false>, LrSmem<kLrShrinkTN, true>::kBytes);
  set(lowrank_tcgen05_kernel<kLrShrinkTN, true, true, true>, LrSmem<kLrShrinkTN, true>::kBytes);
  return e;
}

template <int TN, bool DEEP, bool SHRINK, bool COPY>
inline cudaError_t lr_launch_k(const CUtensorMap& tmA, const CUtensorMap& tmX, const LrArgs& a, dim3 grid, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(COPY ? 192 + 32 * kLrCopyWarps : 224);
  cfg.dynamicSmemBytes = LrSmem<TN, DEEP>::kBytes;
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
  return cudaLaunchKernelEx(&cfg, lowrank_tcgen05_kernel<TN, DEEP, SHRINK, COPY>, tmA, tmX, a);
}

struct LrPlan {
  int tn, splits;          // rows of a tile; CTAs that share its K
  bool deep;               // ring: one tile an SM at most
  bool simt;               // h on CUDA cores
  int jn, h_splits;        // rows of A_a of a CTA there; CTAs that share the K of a tile on the tensor cores
};

inline LrPlan lr_plan(int rows, int c, int n, int rank, int adapters, int sms) {
  LrPlan p;
  p.tn = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  const int kb = cdiv(c, 64);
  auto share = [&](long tiles) {           // twice as many CTAs while they fit side by side and each has four blocks of K
    int z = 1;
    while (z < kLrMaxSplits && tiles * z * 2 <= sms && kb >= z * 2 * 4) z *= 2;
    return z;
  };
  const long tiles = (long)cdiv(n, 128) * cdiv(rows, p.tn);
  p.splits = share(tiles);
  p.deep = p.tn < 128 || tiles <= sms;
  p.simt = rows <= kLrSimtRows;
  p.jn = 8;
  while (p.jn > 1 && (long)rows * cdiv(rank, p.jn) < 2L * sms) p.jn /= 2;
  p.h_splits = share((long)cdiv(rows, kLrShrinkTN) * cdiv(std::min(adapters, kLrShrinkTN), 128 / (int)align_up(rank, 8)));
  return p;
}

template <int TN, bool DEEP>
inline cudaError_t lr_expand(bool copy, const CUtensorMap& tmW, const CUtensorMap& tmX, const LrArgs& a, int splits, cudaStream_t st) {
  const dim3 grid(cdiv(a.n, 128), cdiv(a.rows, TN), splits);
  return copy ? lr_launch_k<TN, DEEP, false, true>(tmW, tmX, a, grid, st) : lr_launch_k<TN, DEEP, false, false>(tmW, tmX, a, grid, st);
}

template <typename T>
inline cudaError_t lr_shrink_simt(const T* x, const T* a, const float* scale, const int32_t* which, T* h, int rows, int c, int rank, int adapters, int jn, cudaStream_t st) {
  constexpr int V = Elem<T>::kVec;
  const bool vec = c % V == 0 && (((uintptr_t)x | (uintptr_t)a) & 15) == 0;
  const dim3 grid(rows, cdiv(rank, jn));
  if (vec) lowrank_shrink_kernel<T, V><<<grid, 256, 0, st>>>(x, a, scale, which, h, c, rank, adapters, jn);
  else lowrank_shrink_kernel<T, 1><<<grid, 256, 0, st>>>(x, a, scale, which, h, c, rank, adapters, jn);
  return cudaGetLastError();
}

inline cudaError_t lr_run_bf16(const LrContext& ctx, LrArgs a, cudaStream_t st) {
  const LrPlan p = lr_plan(a.rows, a.c, a.n, a.rank, a.adapters, ctx.sm_count);
  const uintptr_t bits = (uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.a;
  const bool copy = a.c % 8 != 0 || (bits & 15) != 0;
  a.pairs = a.c % 2 == 0 && (bits & 3) == 0;
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
    const int per_tile = 128 / a.r8;
    const dim3 grid(cdiv(std::min(a.adapters, kLrShrinkTN), per_tile), cdiv(a.rows, kLrShrinkTN), p.h_splits);
    e = copy ? lr_launch_k<kLrShrinkTN, true, true, true>(tmA, tmH, a, grid, st) : lr_launch_k<kLrShrinkTN, true, true, false>(tmA, tmH, a, grid, st);
  } else if (a.adapters > 0) {
    e = lr_shrink_simt<bf16>(a.x, a.a, a.scale, a.which, a.h, a.rows, a.c, a.rank, a.adapters, p.jn, st);
  }
  if (e != cudaSuccess) return e;
  switch (p.tn) {
    case 16: return lr_expand<16, true>(copy, tmW, tmX, a, p.splits, st);
    case 32: return lr_expand<32, true>(copy, tmW, tmX, a, p.splits, st);
    case 64: return lr_expand<64, true>(copy, tmW, tmX, a, p.splits, st);
    default: return p.deep ? lr_expand<128, true>(copy, tmW, tmX, a, p.splits, st) : lr_expand<128, false>(copy, tmW, tmX, a, p.splits, st);
  }
}

// fp32: h and the adapters' share on CUDA cores (summed in fp64, like everything of the fp32 model), then the projection on the convolution kernel of
// the fp32 model as a 1x1 layer of one pixel a row, which adds that share.
inline cudaError_t lr_run_f32(const LrContext& ctx, const float* x, const float* w, const float* bias, const float* a, const float* b, const float* scale,
                              const int32_t* which, float* h, float* y, int rows, int c, int n, int rank, int adapters, int* err_flag, cudaStream_t st) {
  const LrPlan p = lr_plan(rows, c, n, std::max(rank, 1), adapters, ctx.sm_count);
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
  return f32_launch(f32_plan(rows, n, c, ctx.sm_count, vec), x, w, nullptr, bias, adapters > 0 ? y : nullptr, y, g, err_flag, kTcWaitCycles, st);
}

}  // namespace ee
