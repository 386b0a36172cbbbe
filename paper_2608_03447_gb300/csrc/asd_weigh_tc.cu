// libasd: the attention weight that each cached slot receives, on the tensor cores
// (asd_kv_weigh for 16-bit types).
//
// Per tile of 128 slots: S = K Q^T, the slots as the 128 rows of tensor memory and
// the query rows as columns, at most 128 at a time. One thread owns a slot: it reads
// its lane's columns and adds up exp2(scale S - lse) over them, so a slot's weight
// never leaves a register until it is written, and no threads exchange anything.
//
// Four groups of 128 threads take the tiles in turn, each with an accumulator, so
// that products and exponentials of several tiles are under way. With more than 128
// rows some tiles, one a group, meet every slab of queries; the slabs stay where
// they all fit.
//
// A CTA per SM: warps 0 to 15 are the groups, warp 16 walks the units and loads keys,
// warp 17 issues the MMAs, warps 18 and 19 copy queries and the rows' scales.
// Keys are TMA boxes of as many slots as the page size and the tile have as a common
// divisor, or 16-byte copies by four warps, 32 rows each, where that is less than the
// swizzle's eight rows (the chains below in pages of five slots 117 us; one warp 389, and
// 464 if it looks up a tile's pages when it needs them).
//
// What bounds it: few rows, memory: 32 paths of up to 9 on 8000 slots, 40 heads on 8 of
// 128 in bf16, 79 to 81 us (471 MB read, 6.0 TB/s). Many rows, the exponentials (32 a
// clock and SM), what goes with them, and the products behind them: 64 rows of 16
// prompts of 9000 to 12000 slots, 32 heads on 4 of 64 in f16, 73 us, of which the 345
// million exponentials need 37; without any sums the same takes 49, with sums but no
// exponentials 67, and a group waits 15 % of its time for a product. One token on 4200
// slots takes 7.2 us, a chain of latencies. A prompt of 4093 on itself (40 heads on 8 of
// 128) takes 321 us: the CTAs that have the first slots meet all 160 slabs of rows one
// after the other, 2 us each. 775 us with every row's place compared with every slot,
// 697 where only a slab that crosses a tile's causal edge does that, 321 since slabs
// that see nothing of a step are neither copied nor multiplied and a row's sum is read
// while its slab is waited for. Heads beyond 128 have room for one slab and two tiles of
// 64 KB: four rows of 8 requests on 4000 slots, 16 heads on 4 of 256, 15.4 us (floor
// 8.6; on the CUDA cores 171). What else was measured for the 64 rows: two groups with
// two accumulators each 113 us; halves of 64 rows, one multiplied while the other is
// added up, 97 us; the next columns read while some are added up 77 us; row scales read
// as pairs, both numbers for every column, 132 us; one part of the scale only 75 us (its
// rounding was then in every weight); two warps that issue MMAs 79 us against 75, by
// their registers. Truncation in the tensor cores' sums makes products smaller by about
// 2^-22: weights are 2 to 5e-7 too small, the largest error against 64 bits.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "asd.h"
#include "asd_launch.cuh"
#include "asd_tcgen05.cuh"
#include "asd_weigh.cuh"

namespace {

using namespace asd_detail;

constexpr int kTile = kSlabRows;  // slots
constexpr int kCols = 128;        // query rows of a slab
constexpr int kChunk = 32;        // that are added up at once
// log2: how far apart the sums of a chunk's rows may be for one offset to serve them all: exp2(scale S - offset) is
// then above the smallest 32-bit numbers wherever a weight is above 2^-86.
constexpr float kSpread = 40.0f;
constexpr int kGroups = 4;        // of 128 threads
constexpr int kSumThreads = kGroups * 128;
constexpr int kKeyWarp = 16, kMmaWarp = 17, kQueryWarp = 18;
constexpr int kQueryThreads = 64;
// Twenty warps, five a scheduler: 96 registers each. Where keys are copied by threads, three more share that.
constexpr int kCopyWarp = 20;
constexpr int threads_for(bool tma) { return (tma ? kCopyWarp : kCopyWarp + 3) * 32; }
constexpr int kTmemCols = 512;
constexpr int kMaxStages = 12;
constexpr int kMaxQueries = 4;
constexpr unsigned long long kLandNs = 10000000;  // longer than any load takes
constexpr size_t kSmemMax = 232448;

constexpr int slab_bytes(int dim) { return kTile * dim * 2; }  // 128 rows of a padded head
// Slabs of queries: 64 KB. A unit that needs no more keeps them for all its tiles.
constexpr int query_slabs(int dim) { return dim <= 64 ? kMaxQueries : dim <= 128 ? kMaxQueries / 2 : 1; }
// Tiles that meet a slab of queries one after the other where a unit has several slabs: their keys stay meanwhile, and
// at heads of 128 there are four stages, at 256 two.
constexpr int tiles_at_once(int dim) { return dim <= 64 ? kGroups : dim <= 128 ? kGroups - 1 : 1; }

// What the roles know of a unit; the keys' warp walks the CTA's range and publishes its units through a ring.
struct alignas(16) WeighUnit {
  int b, h, rows, valid;   // request, key/value head, query rows; 0: there are no more units
  int span, ctx, j0, j1;   // slots that the last row sees, that all do; this CTA's tiles
  int tiles, cols, pad[2]; // slabs of queries, and the columns of each (a multiple of 16)
};
constexpr int kUnits = 4;
constexpr int kUnitReaders = kSumThreads / 32 + 3;  // warps, without those that copy keys

struct WeighShared {
  unsigned long long k_full[kMaxStages], k_empty[kMaxStages];  // loads have landed; the MMAs have read them
  unsigned long long unit_full[kUnits], unit_empty[kUnits];
  unsigned long long q_full[kMaxQueries], q_empty[kMaxQueries];
  unsigned long long s_full[kGroups], s_empty[kGroups];  // a group's accumulator is complete; has been read
  unsigned long long drain;
  uint32_t tmem_base;
  int abort;
  WeighUnit unit[kUnits];
  AttnDeal deal;
  RowScale scale[kMaxQueries][kCols];
  alignas(16) float factor[kMaxQueries][kCols];   // 2^offset / (sum of exponentials) of each row,
  float offset[kMaxQueries][kCols / kChunk];      // with one whole offset a chunk of rows, or NaN: too far apart
};
constexpr int stages_for(int dim) {
  const size_t fit = (kSmemMax - 1024 - sizeof(WeighShared) - query_slabs(dim) * slab_bytes(dim)) / slab_bytes(dim);
  return fit < static_cast<size_t>(kMaxStages) ? static_cast<int>(fit) : kMaxStages;
}
constexpr size_t smem_for(int dim) {
  return 1024 + static_cast<size_t>(query_slabs(dim) + stages_for(dim)) * slab_bytes(dim) + sizeof(WeighShared);
}
static_assert(stages_for(128) >= 4 && stages_for(256) >= 2, "ring depth: more than the tiles of a step");

// Set by any call that gives up a wait, until asd_weigh_error reads it: there is no workspace to keep it in, and a call
// without a status array would lose it.
__device__ unsigned g_gave_up;

__device__ __forceinline__ bool warp_wait(unsigned long long* bar, uint32_t parity, WeighShared& sh) {
  if (__all_sync(kFull, mbar_try_wait(bar, parity))) return true;
  return __all_sync(kFull, warp_wait_on(bar, parity, &sh.abort, &g_gave_up));
}

// A place in the ring of units.
struct UnitFeed {
  int slot = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next() {
    if (++slot == kUnits) {
      slot = 0;
      phase ^= 1u;
    }
  }
  // the next unit, or null after the last one (or a wait that gave up); done() when it has been read
  __device__ __forceinline__ const WeighUnit* wait(WeighShared& sh) {
    if (!warp_wait(&sh.unit_full[slot], phase, sh) || !sh.unit[slot].valid) return nullptr;
    return &sh.unit[slot];
  }
  __device__ __forceinline__ void done(WeighShared& sh) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(&sh.unit_empty[slot]);
    next();
  }
};
// A place in a ring of stages or slabs.
template <int kStages>
struct Ring {
  int at = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next() {
    if (++at == kStages) {
      at = 0;
      phase ^= 1u;
    }
  }
};

// Where slabs come again for every step of tiles: the first that has a row which sees tile j.
__device__ __forceinline__ int first_slab(int ctx, int cols, int j, int group) {
  const int after = j * kTile - ctx;  // the tokens before this one see nothing of it
  return after <= 0 ? 0 : after * group / cols;
}
__device__ __forceinline__ int first_slab(const WeighUnit& u, int j, int group) {
  return first_slab(u.ctx, u.cols, j, group);
}

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor_sync(kFull, x, off));
  return x;
}

// 32 or 16 consecutive columns of this thread's lane, there when it returns.
__device__ __forceinline__ void tmem_take(uint32_t taddr, float (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
        "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]),
        "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]),
        "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_take(uint32_t taddr, float (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
        "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
      : "r"(taddr));
}

// exp2(scale z - offset) factor summed over kN columns of this thread's lane.
template <int kN>
__device__ __forceinline__ float sum_columns(uint32_t from, const float* factor, float2 scale, float offset) {
  const float2 by = {scale.x, scale.x}, rest = {scale.y, scale.y}, less = {-offset, -offset};
  float z[kN];
  tmem_take(from, z);
  float2 sum[2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
#pragma unroll
  for (int k = 0; k < kN; k += 4) {
    const float4 f = *reinterpret_cast<const float4*>(factor + k);
    const float2 z0 = {z[k], z[k + 1]}, z1 = {z[k + 2], z[k + 3]};
    // the rest comes last: added to the whole of the offset it would be rounded away
    const float2 t0 = fma2(z0, rest, fma2(z0, by, less)), t1 = fma2(z1, rest, fma2(z1, by, less));
    sum[0] = fma2(make_float2(exp2_fast(t0.x), exp2_fast(t0.y)), make_float2(f.x, f.y), sum[0]);
    sum[1] = fma2(make_float2(exp2_fast(t1.x), exp2_fast(t1.y)), make_float2(f.z, f.w), sum[1]);
  }
  const float2 both = add2(sum[0], sum[1]);
  return both.x + both.y;
}
// The same row by row, for any sums and any products: neither a row that adds nothing
// nor one before `first` counts, whatever its product is.
__device__ __noinline__ float sum_carefully(uint32_t from, int cols, const RowScale* rows, float2 scale, int first) {
  float sum = 0.0f;
#pragma unroll 1
  for (int c = 0; c < cols; c += 16) {
    float z[16];
    tmem_take(from + c, z);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const RowScale s = rows[c + k];
      const float e = exp2_fast(fmaf(z[k], scale.y, fmaf(z[k], scale.x, -s.x)));
      if (s.y != 0.0f && c + k >= first) sum = fmaf(e, s.y, sum);
    }
  }
  return sum;
}

// kDim: the head, padded. kTma: keys are loaded as TMA boxes.
template <typename T, int kDim, bool kTma>
__global__ void __launch_bounds__(threads_for(kTma), 1)
    weigh_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ WeighParams p, int box) {
  constexpr int kSlab = slab_bytes(kDim), kStages = stages_for(kDim), kQueries = query_slabs(kDim);
  constexpr int kStep = tiles_at_once(kDim), kThreads = threads_for(kTma);
  constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
  constexpr int kChunks = kDim / 8;          // 16-byte chunks of a row
  constexpr int kRowsAtOnce = 32 / kChunks;  // rows that a warp copies per instruction
  extern __shared__ __align__(1024) unsigned char weigh_smem_raw[];
  const uint32_t raw = smem_u32(weigh_smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  const uint32_t sq = base, sk = base + kQueries * kSlab;
  WeighShared& sh = *reinterpret_cast<WeighShared*>(weigh_smem_raw + (base - raw) + (kQueries + kStages) * kSlab);

  const int warp = __shfl_sync(kFull, static_cast<int>(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  pdl_signal_dependents();
  if (warp == kQueryWarp) {  // a barrier or two a lane
    if (lane < kMaxStages) {
      mbar_init(&sh.k_full[lane], kTma ? 1 : kTile);  // a thread a row
      mbar_init(&sh.k_empty[lane], 1);
    }
    if (lane < kUnits) {
      mbar_init(&sh.unit_full[lane], 1);
      mbar_init(&sh.unit_empty[lane], kUnitReaders + kThreads / 32 - kCopyWarp);
    }
    if (lane >= 16 && lane < 16 + kQueries) {
      mbar_init(&sh.q_full[lane - 16], 2 * kQueryThreads);  // each thread's copies, and its scales
      mbar_init(&sh.q_empty[lane - 16], 1 + kSumThreads / 32);
    }
    if (lane >= 20 && lane < 20 + kGroups) {
      mbar_init(&sh.s_full[lane - 20], 1);
      mbar_init(&sh.s_empty[lane - 20], 4);
    }
    if (lane == 31) {
      mbar_init(&sh.drain, 1);
      sh.abort = 0;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_for_mma();
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (kTma && warp == kKeyWarp && lane == 0)
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_k)) : "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __reduce_max_sync(kFull, sh.tmem_base);

  pdl_wait_prerequisites();
  const int chunk = lane % kChunks, sub = lane / kChunks;
  // where chunk `chunk` of row r lies in a slab
  auto place = [&](int r) {
    return static_cast<uint32_t>((chunk >> 3) * kHalfSlab + r * 128 + (((chunk & 7) ^ (r & 7)) << 4));
  };
  const bool has_chunk = chunk * 8 < p.a.D;
  // A unit's keys by 16-byte copies: rows 32 n to 32 n + 31 of every tile, whose pages are looked up a tile ahead.
  auto copy_keys = [&](const WeighUnit& u, int n, Ring<kStages>& ring, bool& ok) {
    const CacheView& c = p.a.cache;
    int page = 0;
    auto look_up = [&](int j) {
      if (j >= u.j1 || 32 * n + lane >= min(kTile, u.span - j * kTile)) return;
      page = __ldcg(c.table + static_cast<long long>(u.b) * c.table_width + c.div.quot(j * kTile + 32 * n + lane));
    };
    look_up(u.j0);
    for (int j = u.j0; ok && j < u.j1; ++j) {
      const int rows = min(32, u.span - j * kTile - 32 * n);  // below 1: none
      long long off = -1;  // of this lane's row
      if (lane < rows) {
        const int slot = j * kTile + 32 * n + lane;
        if (static_cast<unsigned>(page) < static_cast<unsigned>(c.pages))
          off = page * c.page_stride + static_cast<long long>(slot - c.div.quot(slot) * c.div.size) * c.token_stride +
                u.h * c.head_stride;
        else if (p.a.status)
          atomicOr(p.a.status + u.b, static_cast<int>(ASD_STATUS_PAGE));
      }
      look_up(j + 1);
      ok = warp_wait(&sh.k_empty[ring.at], ring.phase ^ 1u, sh);
      if (!ok) break;
      const uint32_t dst = sk + ring.at * kSlab;
#pragma unroll 4
      for (int i = 0; i < 32 / kRowsAtOnce; ++i) {
        const int r = i * kRowsAtOnce + sub;
        const long long o = __shfl_sync(kFull, off, r);
        const bool has = o >= 0 && has_chunk;
        if (r < rows) copy16(dst + place(32 * n + r), has ? c.k + 2 * (o + chunk * 8) : p.a.q, has);
      }
      copies_arrive(&sh.k_full[ring.at]);
      ring.next();
    }
  };

  if (warp == kKeyWarp) {
    // ---------------- units and keys
    const AttnParams a = weigh_deal_params(p);
    const bool elected = elect_lane();
    attn_deal<kTile>(a, sh.deal);
    bool ok = true;
    UnitFeed feed;  // the next free slot
    Ring<kStages> ring;
    auto publish = [&](const WeighUnit& u) {
      ok = ok && warp_wait(&sh.unit_empty[feed.slot], feed.phase ^ 1u, sh);
      if (lane == 0) {
        sh.unit[feed.slot] = u;
        mbar_arrive(&sh.unit_full[feed.slot]);
      }
      __syncwarp();
      feed.next();
    };
    AttnWalk<kTile> w(a, sh.deal);
    for (w.start(); ok && w.more(); w.next()) {
      WeighUnit u = {};
      u.b = w.b, u.h = w.h, u.rows = w.rows(), u.valid = 1;
      u.span = w.span(), u.ctx = w.r.ctx, u.j0 = w.j0, u.j1 = w.j1();
      u.tiles = (u.rows + kCols - 1) / kCols;
      u.cols = ((u.rows + u.tiles - 1) / u.tiles + 15) & ~15;
      publish(u);
      if constexpr (kTma) {
        // where this lane's box of the next tile begins; the page table is read a tile ahead
        int page = 0, at = 0;
        auto look_up = [&](int j) {
          if (j >= u.j1 || lane * box >= min(kTile, u.span - j * kTile)) return;
          const int slot = j * kTile + lane * box, n = a.cache.div.quot(slot);
          page = __ldcg(a.cache.table + static_cast<long long>(u.b) * a.cache.table_width + n);
          at = slot - n * a.cache.div.size;
        };
        look_up(u.j0);
        for (int j = u.j0; ok && j < u.j1; ++j) {
          const int rows = min(kTile, u.span - j * kTile), page_of = page, at_of = at;
          const uint32_t dst = sk + ring.at * kSlab;
          unsigned long long* const bar = &sh.k_full[ring.at];
          look_up(j + 1);
          ok = warp_wait(&sh.k_empty[ring.at], ring.phase ^ 1u, sh);
          if (!ok) break;
          const int n = uniform((rows + box - 1) / box), head = uniform(u.h);
          if (elected) mbar_expect_tx(bar, static_cast<uint32_t>(n * box) * (kDim * 2));
          __syncwarp();
          // a page out of range lies outside the tensor: the box is filled with zeros
#pragma unroll 4
          for (int i = 0; i < n; ++i) {
            const int pg = __shfl_sync(kFull, page_of, i), first = __shfl_sync(kFull, at_of, i);
            if (elected) {
#pragma unroll
              for (int half = 0; half < kDim / 64; ++half)
                load_box(dst + half * kHalfSlab + i * box * 128, &map_k, bar, half * 64, first, head, pg);
            }
          }
          if (lane < n && static_cast<unsigned>(page_of) >= static_cast<unsigned>(a.cache.pages) && a.status)
            atomicOr(a.status + u.b, static_cast<int>(ASD_STATUS_PAGE));
          __syncwarp();
          ring.next();
        }
      } else {
        copy_keys(u, 0, ring, ok);
      }
    }
    publish(WeighUnit{});
    if (!kTma) asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp >= kCopyWarp) {
    // ---------------- keys that threads copy: the other rows of each tile
    UnitFeed feed;
    Ring<kStages> ring;
    bool ok = true;
    while (ok) {
      const WeighUnit* next = feed.wait(sh);
      if (!next) break;
      const WeighUnit u = *next;
      feed.done(sh);
      copy_keys(u, warp - kCopyWarp + 1, ring, ok);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp >= kQueryWarp) {
    // ---------------- queries; those that need more slabs than there are come again for every step
    const int part = warp - kQueryWarp;
    UnitFeed feed;
    Ring<kQueries> ring;
    bool ok = true;
    while (ok) {
      const WeighUnit* next = feed.wait(sh);
      if (!next) break;
      const WeighUnit u = *next;
      feed.done(sh);
      const bool stays = u.tiles <= kQueries;
      for (int j = u.j0; ok && j < u.j1; j = stays ? u.j1 : j + kStep) {
        for (int tile = stays ? 0 : first_slab(u, j, p.a.group); ok && tile < u.tiles; ++tile) {
          // 32 rows at a time, a lane a row: where it lies and its sum are read while the slab is waited for
          constexpr int kParts = kCols / kQueryThreads;
          long long offs[kParts];
          float lse[kParts];
#pragma unroll
          for (int n = 0; n < kParts; ++n) {
            const int at = part * 32 + n * kQueryThreads + lane, row = tile * u.cols + at, t = p.a.by_group.quot(row);
            const int token = at < u.cols && row < u.rows ? weigh_token(p, u.b, t) : -1;
            const int head = u.h * p.a.group + row - t * p.a.group;
            offs[n] = token < 0 ? -1 : u.b * p.a.q_batch + token * p.a.q_token + head * p.a.q_head;
            lse[n] = row_lse(p, u.b, token, head);
          }
          ok = warp_wait(&sh.q_empty[ring.at], ring.phase ^ 1u, sh);
          if (!ok) break;
#pragma unroll
          for (int n = 0; n < kParts; ++n) {
            const int r0 = part * 32 + n * kQueryThreads, r = r0 + lane;
            if (r0 >= u.cols) break;
            const long long off = offs[n];
            // exp2(z - x) y as exp2(z - m) f with one whole m for the chunk: no number but f that differs from row to row
            const RowScale scale = row_scale(lse[n]);
            const float most = warp_max(scale.y == 0.0f ? -INFINITY : scale.x);
            const float least = -warp_max(scale.y == 0.0f ? -INFINITY : -scale.x);
            const float m = most == -INFINITY ? 0.0f : ceilf(most);
            if (r < u.cols) {
              sh.scale[ring.at][r] = scale;
              sh.factor[ring.at][r] = scale.y == 0.0f ? 0.0f : exp2f(m - scale.x) * scale.y;
            }
            if (lane == 0)
              sh.offset[ring.at][r0 / kChunk] = most - least > kSpread || !(m - m == 0.0f) ? NAN : m;
#pragma unroll 4
            for (int k = 0; k < 32 / kRowsAtOnce; ++k) {
              const int to = k * kRowsAtOnce + sub;
              const long long o = __shfl_sync(kFull, off, to);
              const bool has = o >= 0 && has_chunk;
              if (r0 + to < u.cols)
                copy16(sq + ring.at * kSlab + place(r0 + to), has ? p.a.q + 2 * (o + chunk * 8) : p.a.q, has);
            }
          }
          copies_arrive(&sh.q_full[ring.at]);
          mbar_arrive(&sh.q_full[ring.at]);
          ring.next();
        }
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == kMmaWarp) {
    // ---------------- S = K Q^T
    const bool elected = elect_lane();
    UnitFeed feed;
    Ring<kStages> keys;
    Ring<kQueries> queries;
    uint32_t empty = (1u << kGroups) - 1u;  // per accumulator the parity to wait for
    int turn = 0;                           // of the groups: the next tile's
    bool ok = true;
    while (ok) {
      const WeighUnit* u = feed.wait(sh);
      if (!u) break;
      const int tiles = uniform(u->tiles), cols = uniform(u->cols), ctx = uniform(u->ctx);
      const uint32_t desc = instr_desc(kBf16, cols, false);
      int j = uniform(u->j0), left = uniform(u->j1) - j;
      feed.done(sh);
      const bool stays = tiles <= kQueries;
      bool first = true;  // of the unit's steps
      while (ok && left > 0) {
        const int count = tiles == 1 ? 1 : min(left, kStep);
        const bool ends = left == count;
        const int stage0 = keys.at;
        const int begin = stays ? 0 : first_slab(ctx, cols, j, p.a.group);
        Ring<kQueries> slab = queries;
#pragma unroll 1
        for (int tile = begin; ok && tile < tiles; ++tile) {
          if (first || !stays) {
            ok = warp_wait(&sh.q_full[slab.at], slab.phase, sh);
            fence_for_mma();  // threads copied them
          }
#pragma unroll 1
          for (int i = 0; ok && i < count; ++i) {
            if (tile == begin) {
              ok = warp_wait(&sh.k_full[keys.at], keys.phase, sh);
              if (!kTma) fence_for_mma();
              keys.next();
            }
            const int s = stage0 + i < kStages ? stage0 + i : stage0 + i - kStages;
            const int g = (turn + i) & (kGroups - 1);
            ok = ok && warp_wait(&sh.s_empty[g], (empty >> g) & 1u, sh);
            empty ^= 1u << g;
            if (!ok) break;
            tc_fence_after();
            const uint32_t ka = (sk + s * kSlab) >> 4, qb = (sq + slab.at * kSlab) >> 4;
            const uint32_t d = tmem + static_cast<uint32_t>(g * kCols);
            if (elected) {
#pragma unroll
              for (int k = 0; k < kDim / 16; ++k) {
                const uint32_t at = ((k >> 2) * kHalfSlab + (k & 3) * 32) >> 4;
                mma_smem(d, tile_desc(ka + at, false), tile_desc(qb + at, false), desc, k > 0 ? 1u : 0u);
              }
              mma_commit(&sh.s_full[g]);
              if (tile == tiles - 1) mma_commit(&sh.k_empty[s]);
            }
            __syncwarp();
          }
          if (ends || !stays) {
            if (elected) mma_commit(&sh.q_empty[slab.at]);
            __syncwarp();
          }
          slab.next();
        }
        if (ends || !stays) queries = slab;
        turn = (turn + count) & (kGroups - 1);
        first = false;
        left -= count;
        j += count;
      }
    }
    drain(&sh.drain, elected);
  } else {
    // ---------------- sums: thread `slot` of group g
    const int g = warp >> 2;
    const int slot_of = threadIdx.x & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    UnitFeed feed;
    Ring<kQueries> queries;
    const float2 scale = {p.a.scale_log2, p.scale_rest};
    uint32_t full = 0;  // the parity to wait for
    int turn = 0;
    bool ok = true;
    while (ok) {
      const WeighUnit* next = feed.wait(sh);
      if (!next) break;
      const WeighUnit u = *next;
      feed.done(sh);
      const bool stays = u.tiles <= kQueries;
      for (int j = u.j0; ok && j < u.j1;) {
        const int count = u.tiles == 1 ? 1 : min(u.j1 - j, kStep);
        const int i = (g - turn) & (kGroups - 1), mine = j + i;
        const bool has = i < count;  // whether this group has one of the tiles
        turn = (turn + count) & (kGroups - 1);
        const int begin = stays ? 0 : first_slab(u, j, p.a.group);
        j += count;
        const bool ends = j == u.j1;
        if (!has && !ends && stays) continue;
        const int slot = mine * kTile + slot_of;
        const bool exists = has && slot < u.span;
        const long long at = (static_cast<long long>(u.b) * p.a.heads + u.h) * p.width + slot;
        float before = 0.0f;
        if (exists && slot < u.ctx && p.decay != 0.0f) before = __ldcg(p.weight + at);
        const int slot0 = mine * kTile, last_slot = min(slot0 + (kTile - 1), u.span - 1);
        float sum = 0.0f;
        Ring<kQueries> slab = queries;
        for (int tile = begin; ok && tile < u.tiles; ++tile) {
          // the rows' scales; and no slab is given back before it is there, by a group without a tile either
          if (has || ends || !stays) ok = warp_wait(&sh.q_full[slab.at], slab.phase, sh);
          if (has) {
            ok = ok && warp_wait(&sh.s_full[g], full, sh);
            full ^= 1u;
            if (ok) {
              tc_fence_after();
              const uint32_t from = tmem + static_cast<uint32_t>(g * kCols) + lanes;
              // whether all of the slab's rows see all of the tile, or none sees any of it
              const int first_row = tile * u.cols, last_row = min(first_row + u.cols, u.rows) - 1;
              const bool none = u.ctx + p.a.by_group.quot(last_row) < slot0;
              float add = 0.0f;
              bool careful = !none && u.ctx + p.a.by_group.quot(first_row) < last_slot;
              const float* factor = sh.factor[slab.at];
              const float* offset = sh.offset[slab.at];
              if (careful || none) {
              } else if (u.cols == kCols) {  // unrolled: the 64 rows of 16 prompts 73 us, in a loop 78
#pragma unroll
                for (int c = 0; c < kCols; c += kChunk)
                  add += sum_columns<kChunk>(from + c, factor + c, scale, offset[c / kChunk]);
              } else {
                for (int c = 0; c < u.cols; c += kChunk)
                  add += u.cols - c >= kChunk ? sum_columns<kChunk>(from + c, factor + c, scale, offset[c / kChunk])
                                              : sum_columns<16>(from + c, factor + c, scale, offset[c / kChunk]);
              }
              // a key that is not finite makes the product with a row that adds nothing NaN too
              careful = __any_sync(kFull, careful || add != add);
              if (careful) {
                // the slab's first row that sees the slot
                const long long sees = static_cast<long long>(slot - u.ctx) * p.a.group - first_row;
                const int first = slot > u.ctx ? static_cast<int>(min(sees, static_cast<long long>(kCols))) : 0;
                add = sum_carefully(from, u.cols, sh.scale[slab.at], scale, first);
              }
              sum += add;
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&sh.s_empty[g]);
            }
          }
          if (ends || !stays) {
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.q_empty[slab.at]);
          }
          slab.next();
        }
        if (ends || !stays) queries = slab;
        if (ok && exists) p.weight_out[at] = fmaf(before, p.decay, sum);
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (sh.abort) {
    attn_incomplete(p.a.status, p.a.B, threadIdx.x, kThreads);
    // loads that nobody waited for: give them time to land before the CTA's memory is another's
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < kLandNs) {
    }
  }
  if (warp == kMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// ---------------------------------------------------------------- host side

constexpr int kMaxDevices = 64;

template <typename T, int kDim, bool kTma>
int launch(const CUtensorMap& map, const WeighParams& p, int box, cudaStream_t stream) {
  auto kernel = weigh_tc_kernel<T, kDim, kTma>;
  static std::atomic<int> grid_of[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return ASD_ERR_CUDA;
  if (dev < 0 || dev >= kMaxDevices) return ASD_ERR_DEVICE;
  int grid = grid_of[dev].load(std::memory_order_acquire);
  if (grid == 0) {
    int sms = 0, major = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return ASD_ERR_CUDA;
    if (major != 10) return ASD_ERR_DEVICE;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(smem_for(kDim))) != cudaSuccess)
      return ASD_ERR_CUDA;
    grid = sms;
    grid_of[dev].store(grid, std::memory_order_release);
  }
  cudaLaunchAttribute attr;
  cudaLaunchConfig_t cfg =
      pdl_config(dim3(static_cast<unsigned>(grid)), dim3(threads_for(kTma)), stream, &attr);
  cfg.dynamicSmemBytes = smem_for(kDim);
  if (cudaLaunchKernelEx(&cfg, kernel, map, p, box) != cudaSuccess) return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

template <typename T, int kDim>
int launch_dim(const asd_kv_cache* cache, const WeighParams& p, cudaStream_t stream) {
  CUtensorMap map;
  const int box = box_slots(cache);
  if (box && make_map(&map, cache->dtype == ASD_BF16, p.a.cache.k, cache, box))
    return launch<T, kDim, true>(map, p, box, stream);
  return launch<T, kDim, false>(map, p, 0, stream);
}

}  // namespace

namespace asd_detail {

// 16-bit types, heads whose rows are whole 16-byte words on 16-byte boundaries.
bool weigh_tc_takes(const asd_kv_cache* cache, const WeighParams& p) {
  return cache->dtype != ASD_F32 && p.a.D % 8 == 0 &&
         rows_aligned(p.a.cache.k, 2, 16, p.a.cache.page_stride, p.a.cache.token_stride, p.a.cache.head_stride) &&
         rows_aligned(p.a.q, 2, 16, p.a.q_batch, p.a.q_token, p.a.q_head);
}

int launch_weigh_tc(const asd_kv_cache* cache, const WeighParams& p, cudaStream_t stream) {
  const bool bf16 = cache->dtype == ASD_BF16;
  if (p.a.D <= 64)
    return bf16 ? launch_dim<__nv_bfloat16, 64>(cache, p, stream) : launch_dim<__half, 64>(cache, p, stream);
  if (p.a.D <= 128)
    return bf16 ? launch_dim<__nv_bfloat16, 128>(cache, p, stream) : launch_dim<__half, 128>(cache, p, stream);
  return bf16 ? launch_dim<__nv_bfloat16, 256>(cache, p, stream) : launch_dim<__half, 256>(cache, p, stream);
}

}  // namespace asd_detail

extern "C" int asd_weigh_error(int* error, asd_stream_t stream) {
  if (!error) return ASD_ERR_NULL;
  void* word = nullptr;
  unsigned value = 0;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (cudaGetSymbolAddress(&word, g_gave_up) != cudaSuccess ||
      cudaMemcpyAsync(&value, word, sizeof value, cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess ||
      (value != 0 && cudaMemsetAsync(word, 0, sizeof value, s) != cudaSuccess))
    return ASD_ERR_CUDA;
  *error = static_cast<int>(value);
  return ASD_OK;
}
