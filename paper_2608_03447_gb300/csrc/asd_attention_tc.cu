// libasd: attention over a paged cache on the tensor cores (asd_tree_attention
// for 16-bit types).
//
// Per tile of 128 slots: S = Q K^T (128 query rows by 128 slots, fp32 in tensor
// memory), P = exp2(scale S - m) by one thread per row, O += P V with P read from
// tensor memory where S was. m is the row's running maximum, but follows it only
// when it has grown by more than 2^8 in weight: O is then rescaled in tensor
// memory, else left as it is (the quotient O / l does not depend on m).
//
// What bounds it: up to about 250 rows per key/value head the keys and values
// stream from memory faster than they are used, beyond that the tensor cores set
// the pace. Two softmax groups of 128 threads, each with its own S and O, keep
// both busy: with at most 128 rows they take turns at the tiles and their results
// are added at the end; with more, a unit is 256 rows, each group has 128 of them
// and every tile of keys and values serves both.
//
// A CTA per SM: warps 0-3 and 4-7 are the softmax groups (a warp reads the TMEM
// lanes of its quarter), warp 8 loads keys and values into a ring of stages in
// the order in which they are used, warp 9 issues the MMAs, warp 10 loads
// queries, warp 11 goes over the tiles that hold new tokens or a request's end
// before their values are used. Loads are TMA boxes of as many slots as the page
// size and the tile have as a common divisor (a page of 48 is three boxes of 16);
// where that is less than the swizzle's eight rows, 16-byte copies.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>
#include <mutex>

#include "asd.h"
#include "asd_attention.cuh"
#include "asd_attention_tc.h"
#include "asd_launch.cuh"

namespace {

using namespace asd_detail;

constexpr int kTile = 128;      // slots
constexpr int kGroupRows = 128;
constexpr int kSoftmaxThreads = 256;
constexpr int kLoadWarp = 8, kMmaWarp = 9, kQueryWarp = 10, kTailWarp = 11;
constexpr int kThreads = 12 * 32;  // three warps a scheduler: 168 registers each
constexpr int kTmemCols = 512;
constexpr int kMaxStages = 12;
constexpr float kGrowth = 8.0f; // log2: how far the maximum may outgrow the reference

constexpr int slab_bytes(int dim) { return kTile * dim * 2; }  // 128 rows of a padded head
constexpr int kHalfSlab = kTile * 128;                         // 64 elements of all of them
constexpr size_t kSmemMax = 232448;

struct TcShared {
  unsigned long long full[kMaxStages];   // a stage's loads have landed
  unsigned long long empty[kMaxStages];  // the MMAs have read it, and the tail warp has seen it
  unsigned long long clean[kMaxStages];  // values of a tile with new tokens or a request's end: gone over
  unsigned long long q_full[2], q_empty[2];  // a query slab is there; is no longer needed
  unsigned long long s_full[2];          // per group: its scores are in tensor memory
  unsigned long long p_ready[2];         // per group: its weights are, and the sum so far is rescaled
  unsigned long long o_done[2];          // per group: the unit's last product is complete
  unsigned long long drain;
  uint32_t tmem_base;
  int abort;
  int last;         // this CTA arrived last at a unit in pieces
  int poison[4];    // of unit u, at u % 4: u + 1 if a new token's values hold NaN or infinities
  AttnDeal deal;
};
constexpr int stages_for(int dim) {
  const size_t fit = (kSmemMax - 1024 - sizeof(TcShared) - 2 * slab_bytes(dim)) / slab_bytes(dim);
  return fit < static_cast<size_t>(kMaxStages) ? static_cast<int>(fit) : kMaxStages;
}
constexpr size_t smem_for(int dim) {
  return 1024 + static_cast<size_t>(2 + stages_for(dim)) * slab_bytes(dim) + sizeof(TcShared);
}
// With 16-byte copies: fills in flight before the warp waits for the oldest. A
// shared tile's values are released after the next tile's keys have landed, so at
// least two stages of the ring are not in flight.
constexpr int lag_for(int dim) { return stages_for(dim) - 2 < 8 ? stages_for(dim) - 2 : 8; }
static_assert(stages_for(128) == 5, "ring depth at the widest head");

// ---------------------------------------------------------------- tcgen05

// Operand tiles of rows of 128 bytes (64 elements) with the 128-byte swizzle,
// eight rows 1024 bytes apart, the next 64 elements of all 128 rows a half slab
// on. Along the rows (keys, queries: K-major) the leading offset is not used; the
// values are read across them (MN-major), where it steps over the half slab.
__device__ __forceinline__ uint64_t tile_desc(uint32_t saddr, bool across) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr >> 4) & 0x3FFFu);
  d |= static_cast<uint64_t>(across ? kHalfSlab >> 4 : 1) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;  // descriptor version
  d |= static_cast<uint64_t>(2) << 61;  // 128-byte swizzle
  return d;
}
// kind::f16, fp32 accumulators, A and B both bf16 or both f16, M = 128.
__device__ __forceinline__ constexpr uint32_t instr_desc(bool bf16, int n, bool b_across) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (b_across ? 1u << 16 : 0u) |
         (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(kGroupRows >> 4) << 24);
}
__device__ __forceinline__ void mma_smem(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// The barrier arrives once every tcgen05 operation this thread issued so far has completed.
__device__ __forceinline__ void mma_commit(unsigned long long* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void tc_fence_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_fence_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
// 32 consecutive fp32 columns of this thread's TMEM lane.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
        "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]),
        "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]),
        "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
        "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---------------------------------------------------------------- copies, waits, small arithmetic

// 16 bytes, or zeros, straight into shared memory.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool has) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(has ? 16 : 0) : "memory");
}
// A TMA box of a paged cache: 64 elements of consecutive slots of one page and head.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, unsigned long long* bar, int d, int at,
                                         int head, int page) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(d), "r"(at), "r"(head), "r"(page)
      : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}
// Shared memory that this thread wrote, or whose copies it saw land, is the tensor cores' to read.
__device__ __forceinline__ void fence_for_mma() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A bounded wait by a whole warp, one answer for all of it. After one wait has
// given up the others return at once, so that every role still runs through its
// loops and meets the others at the barriers.
__device__ __forceinline__ bool warp_wait(unsigned long long* bar, uint32_t parity, TcShared& sh, const AttnParams& p) {
  const bool got = __all_sync(kFull, mbar_wait(bar, parity, &sh.abort));
  if (!got) {
    *const_cast<volatile int*>(&sh.abort) = 1;
    atomicExch(p.error, static_cast<unsigned>(ASD_ERR_TIMEOUT));
  }
  return got;
}
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxThreads) : "memory"); }

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <typename T> constexpr uint32_t kExponent = 0x7f807f80u;  // of a pair of elements: all ones is NaN or infinite
template <> constexpr uint32_t kExponent<__half> = 0x7c007c00u;

// Zeros the NaN and infinities of a pair.
template <typename T>
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
  constexpr uint32_t lo = kExponent<T> & 0xffffu, hi = kExponent<T> & 0xffff0000u;
  if ((w & lo) == lo) w &= 0xffff0000u;
  if ((w & hi) == hi) w &= 0xffffu;
  return w;
}

// ---------------------------------------------------------------- kernel

// What the roles know of a tile, in one word.
enum : int {
  kValid = 1,
  kFirst = 2,    // of the CTA's tiles of the unit
  kEarly = 4,    // one of the first two
  kLast = 8,     // the last
  kLate = 16,    // one of the last two
  kPair = 32,    // the unit has rows for both groups, which share its tiles
  kTail = 64,    // new tokens, or the request's end
  kUnit = 128,   // the unit's number among the CTA's units with work starts here
};

// The CTA's tiles one after the other, over the units that see anything. The
// fields tell of the tile that `flags` describes; advance() goes to the next.
struct TileWalk {
  AttnWalk<kTile> w;
  int j, unit, span;
  __device__ __forceinline__ TileWalk(const AttnParams& p, const AttnDeal& d) : w(p, d), unit(-1) { enter(); }
  __device__ __forceinline__ void enter() {
    span = 0;
    while (w.more() && (span = w.span()) == 0) w.next();
    j = w.j0;
    ++unit;
  }
  __device__ __forceinline__ int slot0() const { return j * kTile; }
  __device__ __forceinline__ int flags() const {
    if (!w.more()) return 0;
    const int from = j - w.j0, to = w.j1() - 1 - j;
    return kValid | (from == 0 ? kFirst : 0) | (from < 2 ? kEarly : 0) | (to == 0 ? kLast : 0) | (to < 2 ? kLate : 0) |
           (w.live_rows() > kGroupRows ? kPair : 0) | (slot0() + kTile > w.r.ctx ? kTail : 0) | unit * kUnit;
  }
  __device__ __forceinline__ void advance() {
    if (++j == w.j1()) {
      w.next();
      enter();
    }
  }
};

// Whether a unit's first scores wait for the last product of the unit before:
// where one of the two is shared, its queries need the slab of the other.
__device__ __forceinline__ bool starts_after(int next, int cur) { return (next & kFirst) && ((next | cur) & kPair); }

// The order in which a CTA's tiles of keys and values go through the ring. The
// MMAs run S(0), then S(i + 1) P V(i), where i counts a tile that the groups take
// in turn once and a tile that they share twice; a tile is loaded when it is
// first needed. Whether the values of `cur` go before the keys of `next`:
__device__ __forceinline__ bool values_first(int next, int cur) {
  return (cur & kPair) || !(next & kValid) || starts_after(next, cur);
}

// A position in the ring.
template <int kStages>
struct Ring {
  int stage = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next() {
    if (++stage == kStages) {
      stage = 0;
      phase ^= 1u;
    }
  }
};

// kDim: the head, padded. kTma: loads are TMA boxes.
template <typename T, int kDim, bool kTma>
__global__ void __launch_bounds__(kThreads, 1)
    attention_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                        const __grid_constant__ AttnParams p, int box) {
  constexpr int kStages = stages_for(kDim);
  constexpr int kSlab = slab_bytes(kDim);
  constexpr bool kBf16 = kExponent<T> == 0x7f807f80u;
  constexpr int kChunks = kDim / 8;          // 16-byte chunks of a row
  constexpr int kRowsAtOnce = 32 / kChunks;  // rows that a warp copies per instruction
  extern __shared__ __align__(1024) unsigned char tc_smem_raw[];
  const uint32_t raw = smem_u32(tc_smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  unsigned char* gbase = tc_smem_raw + (base - raw);
  const uint32_t sq = base, skv = base + 2 * kSlab;
  TcShared& sh = *reinterpret_cast<TcShared*>(gbase + (2 + kStages) * kSlab);

  const int warp = __shfl_sync(kFull, static_cast<int>(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  pdl_signal_dependents();
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sh.full[s], kTma ? 1 : 32);
      mbar_init(&sh.empty[s], 1 + 32);
      mbar_init(&sh.clean[s], 32);
    }
    for (int g = 0; g < 2; ++g) {
      mbar_init(&sh.q_full[g], 32);
      mbar_init(&sh.q_empty[g], kSoftmaxThreads);
      mbar_init(&sh.s_full[g], 1);
      mbar_init(&sh.p_ready[g], 128);
      mbar_init(&sh.o_done[g], 1);
    }
    mbar_init(&sh.drain, 1);
    sh.abort = 0;
    for (int i = 0; i < 4; ++i) sh.poison[i] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_for_mma();
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (kTma && warp == kLoadWarp && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_k)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_v)) : "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __reduce_max_sync(kFull, sh.tmem_base);
  auto tmem_s = [&](int g) { return tmem + static_cast<uint32_t>(g * kTile); };
  auto tmem_o = [&](int g) { return tmem + static_cast<uint32_t>(2 * kTile + g * kDim); };

  pdl_wait_prerequisites();
  const bool work = attn_deal<kTile>(p, sh.deal);  // the same for all threads
  const int chunk = lane % kChunks, sub = lane / kChunks;
  // where chunk `chunk` of row r lies in a slab
  auto place = [&](int r) {
    return static_cast<uint32_t>((chunk >> 3) * kHalfSlab + r * 128 + (((chunk & 7) ^ (r & 7)) << 4));
  };
  const bool has_chunk = chunk * 8 < p.D;
  // 32 rows of a slab from row0 on; off: of row row0 + lane, elements of `src`
  auto copy_rows = [&](uint32_t dst, int row0, const char* src, long long off, int rows) {
#pragma unroll
    for (int i = 0; i < 32 / kRowsAtOnce; ++i) {
      const int r = i * kRowsAtOnce + sub;
      const long long o = __shfl_sync(kFull, off, r);
      const bool has = o >= 0 && has_chunk;
      if (r < rows) copy16(dst + place(row0 + r), has ? src + 2 * (o + chunk * 8) : p.q, has);
    }
  };

  if (work && warp == kLoadWarp) {
    // ---------------- keys and values
    Ring<kStages> ring;
    bool ok = true;
    if constexpr (kTma) {
      const int boxes = kTile / box;  // of a tile, each in kDim / 64 halves: one a lane
      const int part = lane % boxes, half = lane / boxes;
      const uint32_t dst0 = static_cast<uint32_t>(half * kHalfSlab + part * box * 128);
      // this lane's box of a tile
      struct Box {
        int flags, b, h;
        int page, at;  // and the place in it; page is read ahead
        bool has;
      };
      TileWalk walk(p, sh.deal);
      auto look_up = [&] {
        Box x = {walk.flags(), walk.w.b, walk.w.h, 0, 0, false};
        if (x.flags & kValid) {
          const int slot = walk.slot0() + part * box;
          if (slot < walk.span && half < kDim / 64) {
            const int n = p.cache.div.quot(slot);
            x.page = __ldcg(p.cache.table + static_cast<long long>(x.b) * p.cache.table_width + n);
            x.at = slot - n * p.cache.div.size;
            x.has = true;
          }
          walk.advance();
        }
        return x;
      };
      auto fill = [&](const CUtensorMap* map, const Box& x) {
        if (ok) ok = warp_wait(&sh.empty[ring.stage], ring.phase ^ 1u, sh, p);
        if (ok) {
          const uint32_t bytes = __popc(__ballot_sync(kFull, x.has)) * box * 128u;
          if (lane == 0) mbar_expect_tx(&sh.full[ring.stage], bytes);
          __syncwarp();
          // a page out of range lies outside the tensor: the box is filled with zeros
          if (x.has) load_box(skv + ring.stage * kSlab + dst0, map, &sh.full[ring.stage], half * 64, x.at, x.h, x.page);
          __syncwarp();
        }
        ring.next();
      };
      Box cur = look_up(), next = cur;
      if (cur.flags) {
        next = look_up();
        fill(&map_k, cur);
      }
      while (cur.flags) {
        if (cur.has && static_cast<unsigned>(cur.page) >= static_cast<unsigned>(p.cache.pages) && p.status)
          atomicOr(p.status + cur.b, static_cast<int>(ASD_STATUS_PAGE));
        const bool before = values_first(next.flags, cur.flags);
        if (before) fill(&map_v, cur);
        Box after = next;
        if (next.flags) {
          after = look_up();
          fill(&map_k, next);
        }
        if (!before) fill(&map_v, cur);
        cur = next;
        next = after;
      }
    } else {
      constexpr int kLag = lag_for(kDim);
      int issued = 0, arrived = 0, stage_out = 0;
      auto arrive = [&] {  // this thread's copies of the stage have landed
        fence_for_mma();
        mbar_arrive(&sh.full[stage_out]);
        if (++stage_out == kStages) stage_out = 0;
        ++arrived;
      };
      struct Rows {
        int flags, b, h, slot0, rows;
      };
      TileWalk walk(p, sh.deal);
      auto take = [&] {
        const Rows x = {walk.flags(), walk.w.b, walk.w.h, walk.slot0(), min(kTile, walk.span - walk.slot0())};
        if (x.flags) walk.advance();
        return x;
      };
      auto fill = [&](const char* src, const Rows& x, bool report) {
        if (ok) ok = warp_wait(&sh.empty[ring.stage], ring.phase ^ 1u, sh, p);
#pragma unroll 1
        for (int q = 0; ok && q < x.rows; q += 32) {
          long long off = -1;
          if (q + lane < x.rows) {
            off = slot_offset(p.cache, x.b, x.slot0 + q + lane);
            if (off < 0 && report && p.status) atomicOr(p.status + x.b, static_cast<int>(ASD_STATUS_PAGE));
            if (off >= 0) off += x.h * p.cache.head_stride;
          }
          copy_rows(skv + ring.stage * kSlab, q, src, off, x.rows - q);
        }
        copies_commit();
        ring.next();
        ++issued;
        if (issued - arrived > kLag) {
          copies_wait<kLag>();
          arrive();
        }
      };
      Rows cur = take();
      if (cur.flags) fill(p.cache.k, cur, true);
      while (cur.flags) {
        const Rows next = take();
        const bool before = values_first(next.flags, cur.flags);
        if (before) fill(p.cache.v, cur, false);
        if (next.flags) fill(p.cache.k, next, true);
        if (!before) fill(p.cache.v, cur, false);
        cur = next;
      }
      copies_wait<0>();
      while (arrived < issued) arrive();
    }
  } else if (work && warp == kQueryWarp) {
    // ---------------- queries: a unit's slab, or both slabs of a unit that the groups share
    bool ok = true;
    uint32_t uses = 0;  // a bit a slab: whether an odd number of fills
    int slab = 0;
    for (AttnWalk<kTile> w(p, sh.deal); w.more(); w.next()) {
      if (w.span() == 0) continue;
      const int live = w.live_rows();
      const bool pair = live > kGroupRows;
      for (int tile = 0; tile * kGroupRows < live; ++tile) {
        const int to = pair ? tile : slab;
        if (ok) ok = warp_wait(&sh.q_empty[to], ((uses >> to) & 1u) ^ 1u, sh, p);
        uses ^= 1u << to;
        for (int r0 = 0; ok && r0 < kGroupRows && tile * kGroupRows + r0 < live; r0 += 32) {
          const int r = tile * kGroupRows + r0 + lane;
          long long off = -1;
          if (r < live) {
            const int row = w.row0() + r, t = row / p.group;
            off = w.b * p.q_batch + t * p.q_token + (w.h * p.group + (row - t * p.group)) * p.q_head;
          }
          copy_rows(sq + to * kSlab, r0, p.q, off, 32);
        }
        copies_commit();
        copies_wait<0>();
        fence_for_mma();
        mbar_arrive(&sh.q_full[to]);
      }
      if (!pair) slab ^= 1;
    }
  } else if (work && warp == kTailWarp) {
    // ---------------- tiles with new tokens or a request's end
    // Rows past the end become zeros (what lies there may be anything, and 0 times NaN is NaN). Of a new token some
    // rows may see nothing, so its values' NaN and infinities become zeros too and the unit is marked: its rows look
    // at the end for those that they do see.
    // This warp follows every fill, one by one, and a stage is filled again only when it has: a wait by parity must
    // never be a round of the ring away from the barrier.
    Ring<kStages> ring;
    bool ok = true;
    auto seen = [&] {
      if (ok) ok = warp_wait(&sh.full[ring.stage], ring.phase, sh, p);
    };
    auto done = [&] {
      mbar_arrive(&sh.empty[ring.stage]);
      ring.next();
    };
    struct Range {
      int flags, lo, end;  // rows of the tile: new tokens from lo on, nothing from end on
    };
    TileWalk walk(p, sh.deal);
    auto take = [&] {
      const Range x = {walk.flags(), max(0, walk.w.r.ctx - walk.slot0()), walk.span - walk.slot0()};
      if (x.flags) walk.advance();
      return x;
    };
    auto keys = [&] {
      seen();
      done();
    };
    auto values = [&](const Range& x) {
      seen();
      if (x.flags & kTail) {
        if (ok) {
          bool found = false;
          for (int r = x.lo + sub; r < kTile; r += kRowsAtOnce) {
            uint4* at = reinterpret_cast<uint4*>(gbase + (2 + ring.stage) * kSlab + place(r));
            if (r >= x.end) {
              *at = make_uint4(0u, 0u, 0u, 0u);
              continue;
            }
            const uint4 was = *at;
            const uint4 now = {finite_pair<T>(was.x), finite_pair<T>(was.y), finite_pair<T>(was.z),
                               finite_pair<T>(was.w)};
            if (now.x != was.x || now.y != was.y || now.z != was.z || now.w != was.w) {
              *at = now;
              found = true;
            }
          }
          const int unit = x.flags / kUnit;
          if (found) sh.poison[unit & 3] = unit + 1;
          fence_for_mma();
        }
        __syncwarp();
        mbar_arrive(&sh.clean[ring.stage]);
      }
      done();
    };
    Range cur = take();
    if (cur.flags) keys();
    while (cur.flags) {
      const Range next = take();
      const bool before = values_first(next.flags, cur.flags);
      if (before) values(cur);
      if (next.flags) keys();
      if (!before) values(cur);
      cur = next;
    }
  } else if (work && warp == kMmaWarp) {
    // ---------------- MMAs
    constexpr uint32_t kDescS = instr_desc(kBf16, kTile, false);
    constexpr uint32_t kDescO = instr_desc(kBf16, kDim, true);
    bool elected;
    {
      uint32_t one;
      asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
      elected = one != 0;
    }
    bool ok = true;
    Ring<kStages> ring;
    int k_stage = 0, v_stage = 0;       // of the tiles whose scores and whose product are being issued
    uint32_t p_phase = 0, q_phase = 0, clean_phase = 0;  // a bit a group, slab, stage
    int slab = 1;                       // of the unit that the groups take in turn
    TileWalk walk(p, sh.deal);
    auto take = [&] {
      const int flags = walk.flags();
      if (flags) walk.advance();
      return flags;
    };

    // the scores of one group's rows against a tile; `second`: the other group has done so with the same tile
    auto scores = [&](int tile, bool second, int g) {
      const bool pair = tile & kPair;
      if ((tile & kFirst) && !second) {
        if (!pair) slab ^= 1;
        for (int s = pair ? 0 : slab; s <= (pair ? 1 : slab); ++s) {
          if (ok) ok = warp_wait(&sh.q_full[s], (q_phase >> s) & 1u, sh, p);
          q_phase ^= 1u << s;
        }
      }
      if (!second) {
        k_stage = ring.stage;
        if (ok) ok = warp_wait(&sh.full[k_stage], ring.phase, sh, p);
        ring.next();
      }
      tc_fence_after();
      if (ok && elected) {
        const uint64_t a = tile_desc(sq + (pair ? g : slab) * kSlab, false);
        const uint64_t b = tile_desc(skv + k_stage * kSlab, false);
#pragma unroll
        for (int k = 0; k < kDim / 16; ++k) {
          const uint32_t at = ((k >> 2) * kHalfSlab + (k & 3) * 32) >> 4;
          mma_smem(tmem_s(g), a + at, b + at, kDescS, k > 0 ? 1u : 0u);
        }
        mma_commit(&sh.s_full[g]);
        if (!pair || second) mma_commit(&sh.empty[k_stage]);
      }
    };
    auto product = [&](int tile, bool second, int g) {
      const bool pair = tile & kPair;
      if (!second) {
        v_stage = ring.stage;
        if (ok) ok = warp_wait(&sh.full[v_stage], ring.phase, sh, p);
        ring.next();
        if (tile & kTail) {
          if (ok) ok = warp_wait(&sh.clean[v_stage], (clean_phase >> v_stage) & 1u, sh, p);
          clean_phase ^= 1u << v_stage;
        }
      }
      if (ok) ok = warp_wait(&sh.p_ready[g], (p_phase >> g) & 1u, sh, p);
      p_phase ^= 1u << g;
      tc_fence_after();
      if (ok && elected) {
        const bool first = tile & (pair ? kFirst : kEarly);  // of this group: the unit's first may be the other's
        const uint64_t b = tile_desc(skv + v_stage * kSlab, true);
#pragma unroll
        for (int k = 0; k < kTile / 16; ++k)
          mma_tmem(tmem_o(g), tmem_s(g) + kTile / 2 + 8 * k, b + ((k * 16 * 128) >> 4), kDescO,
                   !first || k > 0 ? 1u : 0u);
        if (tile & (pair ? kLast : kLate)) mma_commit(&sh.o_done[g]);
        if (!pair || second) mma_commit(&sh.empty[v_stage]);
      }
    };
    int a = take();
    bool a_second = false;
    int g = 0;
    if (a) scores(a, false, 0);
    while (a) {
      const bool b_second = (a & kPair) && !a_second;
      const int b = b_second ? a : take();
      const bool later = !b_second && starts_after(b, a);
      if (b && !later) scores(b, b_second, g ^ 1);
      product(a, a_second, g);
      if (later) scores(b, false, g ^ 1);
      a = b;
      a_second = b_second;
      g ^= 1;
    }
    if (elected) {
      mma_commit(&sh.drain);
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait(&sh.drain, 0) && global_ns() - t0 < kWaitLimitNs) {
      }
    }
    __syncwarp();
  } else if (work) {
    // ---------------- softmax: thread `row` of group g
    const int g = warp >> 2;
    const int row = threadIdx.x & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = tmem_s(g) + lanes, tw = ts + kTile / 2, to = tmem_o(g) + lanes;  // scores, weights, sum
    bool ok = true;
    uint32_t s_phase = 0, o_phase = 0;
    int turn = 0, unit = 0, slab = 0;
    for (AttnWalk<kTile> w(p, sh.deal); w.more(); w.next()) {
      const int span = w.span(), rows = w.rows(), live = w.live_rows();
      const bool pair = live > kGroupRows;
      const bool shares = rows > kGroupRows;                       // rows for both groups to write
      const int group_row0 = shares ? g * kGroupRows : 0;
      const int r = group_row0 + row;                              // of the unit
      const int rl = (pair ? g * kGroupRows : 0) + row;            // whose scores this thread has
      const bool warp_live = (pair ? g * kGroupRows : 0) + (warp & 3) * 32 < live;  // the same for the warp
      const int t = (w.row0() + min(rl, max(live - 1, 0))) / p.group;
      float m = -INFINITY, l = 0.0f;
      bool had = false;
      const int j1 = w.j1();
      for (int j = w.j0; span > 0 && j < j1; ++j) {
        const int whose = turn & 1;
        turn += pair ? 2 : 1;
        if (!pair && whose != g) continue;
        const int slot0 = j * kTile;
        const bool masked = slot0 + kTile > w.r.ctx;
        uint32_t sees[4];
        if (masked && warp_live) {
#pragma unroll
          for (int c = 0; c < 4; ++c) sees[c] = attn_sees(p, w.r, w.b, t, slot0 + 32 * c);
        }
        if (ok) ok = warp_wait(&sh.s_full[g], s_phase, sh, p);
        s_phase ^= 1u;
        tc_fence_after();
        if (ok && warp_live) {
          float x[2][32];
          auto read_half = [&](int half) {
            tmem_ld32(ts + 64 * half, x[0]);
            tmem_ld32(ts + 64 * half + 32, x[1]);
            tmem_ld_wait();
          };
          auto hide = [&](int half) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!((sees[2 * half + c] >> i) & 1u)) x[c][i] = -INFINITY;
          };
          // four chains: one warp a scheduler has little else to cover an operation's latency with
          float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          auto top_half = [&] {
#pragma unroll
            for (int i = 0; i < 32; i += 4)
#pragma unroll
              for (int k = 0; k < 4; ++k) tops[k] = fmaxf(tops[k], fmaxf(x[0][i + k], x[1][i + k]));
          };
          // weights of 64 slots, over scores that are in registers or have been read
          float sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          auto weigh_half = [&](int half, float ref) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              uint32_t w2[16];
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const float e0 = exp2_fast(fmaf(x[c][i], p.scale_log2, -ref));
                const float e1 = exp2_fast(fmaf(x[c][i + 1], p.scale_log2, -ref));
                sums[i & 2] += e0;
                sums[(i & 2) + 1] += e1;
                w2[i >> 1] = pack2<T>(e0, e1);
              }
              tmem_st16(tw + 32 * half + 16 * c, w2);
            }
          };
          read_half(0);
          if (masked) hide(0);
          top_half();
          read_half(1);
          if (masked) hide(1);
          top_half();
          const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * p.scale_log2;
          if (__any_sync(kFull, rl < live && top > m + kGrowth)) {
            const float m_new = fmaxf(m, top);
            const float fade = exp2_fast(m - (m_new == -INFINITY ? 0.0f : m_new));
            l *= fade;
            m = m_new;
            if (had) {
              // every product of this group so far has completed: it came before these scores
#pragma unroll 1
              for (int c = 0; c < kDim; c += 16) {
                float o[16];
                tmem_ld16(to + c, o);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] *= fade;
                uint32_t bits[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) bits[i] = __float_as_uint(o[i]);
                tmem_st16(to + c, bits);
              }
            }
          }
          const float ref = m == -INFINITY ? 0.0f : m;
          weigh_half(1, ref);  // still in registers; the weights lie over the second half's scores
          read_half(0);
          if (masked) hide(0);
          weigh_half(0, ref);
          l += (sums[0] + sums[1]) + (sums[2] + sums[3]);
          tmem_st_wait();
        }
        had = true;
        tc_fence_before();
        mbar_arrive(&sh.p_ready[g]);
      }

      // the unit's rows, or this CTA's piece of them
      const bool whole = w.whole();
      float f_self = 1.0f, f_other = 1.0f;  // what the groups' sums are multiplied with
      bool other_had = false;
      if (span > 0) {
        if (had) {
          if (ok) ok = warp_wait(&sh.o_done[g], o_phase, sh, p);
          o_phase ^= 1u;
          tc_fence_after();
        }
        if (!pair) {
          // both groups' statistics, in the slab of the unit's queries, which no MMA reads any more
          other_had = !had || j1 - w.j0 > 1;
          float2* stat = reinterpret_cast<float2*>(gbase + slab * kSlab);
          tc_fence_before();
          softmax_sync();  // both groups' products are complete, the queries have been read
          stat[g * kGroupRows + row] = make_float2(m, l);
          softmax_sync();
          tc_fence_after();
          const float2 other = stat[(g ^ 1) * kGroupRows + row];
          const float top = fmaxf(m, other.x);
          const float ref = top == -INFINITY ? 0.0f : top;
          f_self = exp2_fast(m - ref);
          f_other = exp2_fast(other.x - ref);
          l = l * f_self + other.y * f_other;
          m = top;
        }
      }
      const bool poisoned = span > 0 && *const_cast<volatile int*>(&sh.poison[unit & 3]) == unit + 1;
      // Who writes what: of shared rows each group its own; else row `row`'s halves of the head, one each. In a unit
      // that has rows for both groups but tokens for one, the second group's rows are zeros.
      const bool split = !shares;
      const bool lives = r < live;
      const bool mine = ok && r < rows;
      const int row_t = (w.row0() + r) / p.group;
      const long long at = (static_cast<long long>(w.b) * p.T + row_t) * p.q_heads + w.h * p.group + w.row0() + r -
                           row_t * p.group;
      const float inv = lives && l > 0.0f ? 1.0f / l : lives ? l : 0.0f;
      const int cols = split ? kDim / 2 : kDim;
      const int col0 = split ? g * cols : 0;
#pragma unroll 1
      for (int c = 0; c < cols; c += 32) {
        const int col = col0 + c;
        __syncwarp();
        float v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = 0.0f;
        if (ok && span > 0 && group_row0 + (warp & 3) * 32 < live) {
          float x[32];
          if (had) {
            tmem_ld32(to + col, x);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = f_self * x[i];
          }
          if (other_had) {
            tmem_ld32(tmem_o(g ^ 1) + lanes + col, x);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = fmaf(f_other, x[i], v[i]);
          }
          if (poisoned && lives) {
            const int end = min(span, j1 * kTile);
            for (int slot = max(w.r.ctx, w.j0 * kTile); slot < end; ++slot) {
              if (!(attn_sees(p, w.r, w.b, t, slot) & 1u)) continue;
              const long long off = slot_offset(p.cache, w.b, slot);
              if (off < 0) continue;
              const T* src = reinterpret_cast<const T*>(p.cache.v) + off + w.h * p.cache.head_stride + col;
              for (int i = 0; i < 32 && col + i < p.D; ++i) {
                const float e = Store<T>::widen(src[i]);
                if (!(e - e == 0.0f)) {
#pragma unroll
                  for (int k = 0; k < 32; ++k)
                    if (k == i) v[k] += e;
                }
              }
            }
          }
        }
        if (mine && whole) {
          T* dst = reinterpret_cast<T*>(p.out) + at * p.D + col;
          const bool zero = !lives || l == 0.0f;
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            if (col + i >= p.D) break;
            uint4 o;
            o.x = zero ? 0u : pack2<T>(v[i] * inv, v[i + 1] * inv);
            o.y = zero ? 0u : pack2<T>(v[i + 2] * inv, v[i + 3] * inv);
            o.z = zero ? 0u : pack2<T>(v[i + 4] * inv, v[i + 5] * inv);
            o.w = zero ? 0u : pack2<T>(v[i + 6] * inv, v[i + 7] * inv);
            *reinterpret_cast<uint4*>(dst + i) = o;
          }
        } else if (mine && lives) {
          // [piece][column / 4][row]: a warp's rows lie side by side
          float* dst =
              p.part_o + (static_cast<long long>(w.piece()) * (kDim / 4) + col / 4) * (p.unit_rows * 4) + r * 4;
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            *reinterpret_cast<float4*>(dst + i * p.unit_rows) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        }
      }
      if (mine && (!split || g == 0)) {
        if (whole) {
          if (p.lse) p.lse[at] = !lives || l == 0.0f ? -INFINITY : 0.6931471805599453f * (m + log2f(l));
        } else if (lives) {
          *reinterpret_cast<float2*>(p.part_ml + 2 * (static_cast<long long>(w.piece()) * p.unit_rows + r)) =
              make_float2(m, l);
        }
      }
      if (span > 0) {
        tc_fence_before();
        if (pair) {
          mbar_arrive(&sh.q_empty[0]);
          mbar_arrive(&sh.q_empty[1]);
        } else {
          softmax_sync();  // both sums and the statistics have been read
          mbar_arrive(&sh.q_empty[slab]);
          slab ^= 1;
        }
        tc_fence_after();
        ++unit;
      }
      if (whole) continue;

      // a unit in pieces
      __threadfence();
      softmax_sync();
      const int c0 = w.first_cta(), c1 = w.last_cta();
      if (threadIdx.x == 0) {
        bool last = false;
        if (ok) {
          last = atomicAdd(p.counters + c0, 1u) == static_cast<unsigned>(c1 - c0);
          if (last) p.counters[c0] = 0u;  // zero again for the next call
        }
        sh.last = last;
      }
      softmax_sync();
      if (!*const_cast<volatile int*>(&sh.last)) continue;
      __threadfence();
      const int quads = p.D / 4;
      for (int i = threadIdx.x; i < rows * quads; i += kSoftmaxThreads) {
        const int rr = i % rows, d4 = i / rows;
        const int tt = (w.row0() + rr) / p.group;
        const long long dst = (static_cast<long long>(w.b) * p.T + tt) * p.q_heads + w.h * p.group + w.row0() + rr -
                              tt * p.group;
        float top = -INFINITY, sum = 0.0f;
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (rr < live) {
#pragma unroll 4
          for (int c = c0; c <= c1; ++c) {
            const long long piece = c == c0 ? 2 * c + 1 : 2 * c;
            top = fmaxf(top, __ldcg(p.part_ml + 2 * (piece * p.unit_rows + rr)));
          }
          const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
          for (int c = c0; c <= c1; ++c) {
            const long long piece = c == c0 ? 2 * c + 1 : 2 * c;
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(p.part_ml + 2 * (piece * p.unit_rows + rr)));
            const float4 v = __ldcg(reinterpret_cast<const float4*>(
                p.part_o + (piece * (kDim / 4) + d4) * (p.unit_rows * 4) + rr * 4));
            const float e = exp2_fast(ml.x - ref);
            sum += e * ml.y;
            acc.x += e * v.x, acc.y += e * v.y, acc.z += e * v.z, acc.w += e * v.w;
          }
        }
        const float k = sum > 0.0f ? 1.0f / sum : sum;
        const uint2 o = sum == 0.0f ? make_uint2(0u, 0u)
                                    : make_uint2(pack2<T>(acc.x * k, acc.y * k), pack2<T>(acc.z * k, acc.w * k));
        *reinterpret_cast<uint2*>(reinterpret_cast<T*>(p.out) + dst * p.D + 4 * d4) = o;
        if (d4 == 0 && p.lse) p.lse[dst] = sum == 0.0f ? -INFINITY : 0.6931471805599453f * (top + log2f(sum));
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// ---------------------------------------------------------------- host side

constexpr int kMaxDevices = 64;

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_tiled() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult res;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault, &res) ==
            cudaSuccess &&
        res == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(ptr);
  });
  return fn;
}

// One layer of keys or values as [page][head][slot of the page][element], boxes
// of `box` slots of one page and head by 64 elements; elements past the head and
// pages out of range read as zero.
bool make_map(CUtensorMap* map, bool bf16, const void* ptr, const asd_kv_cache* c, int box) {
  EncodeTiledFn fn = encode_tiled();
  if (!fn) return false;
  auto stride = [&](long long elements, int size) -> cuuint64_t {  // of a dimension of one entry: any
    return size == 1 ? 256u * 2u : static_cast<cuuint64_t>(elements) * 2;
  };
  const cuuint64_t dims[4] = {static_cast<cuuint64_t>(c->head_dim), static_cast<cuuint64_t>(c->page_size),
                              static_cast<cuuint64_t>(c->heads), static_cast<cuuint64_t>(c->pages)};
  const cuuint64_t strides[3] = {stride(c->token_stride, c->page_size), stride(c->head_stride, c->heads),
                                 stride(c->page_stride, c->pages)};
  const cuuint32_t boxes[4] = {64, static_cast<cuuint32_t>(box), 1, 1};
  const cuuint32_t steps[4] = {1, 1, 1, 1};
  return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(ptr),
            dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int kDim, bool kTma>
int launch(const CUtensorMap& map_k, const CUtensorMap& map_v, AttnParams p, int box, char* workspace,
           cudaStream_t stream) {
  auto kernel = attention_tc_kernel<T, kDim, kTma>;
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
    grid = sms < kAttnMaxCtas ? sms : kAttnMaxCtas;
    grid_of[dev].store(grid, std::memory_order_release);
  }
  const AttnLayout l = attn_layout(kAttnMaxCtas, p.unit_rows, kDim);
  p.counters = reinterpret_cast<unsigned*>(workspace + l.counters);
  p.part_ml = reinterpret_cast<float*>(workspace + l.ml);
  p.part_o = reinterpret_cast<float*>(workspace + l.o);
  cudaLaunchAttribute attr;
  cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(grid)), dim3(kThreads), stream, &attr);
  cfg.dynamicSmemBytes = smem_for(kDim);
  if (cudaLaunchKernelEx(&cfg, kernel, map_k, map_v, p, box) != cudaSuccess) return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

// Rows of a unit: what one softmax group holds, or both where there are more.
int unit_rows(long long rows) { return rows > kGroupRows ? 2 * kGroupRows : kGroupRows; }

// Slots of a TMA box: what the page size and the tile have in common, and at
// least the swizzle's eight rows; 0: none.
int box_slots(const asd_kv_cache* c) {
  int box = kTile;
  while (c->page_size % box != 0) box /= 2;
  return box >= 8 && c->pages > 0 ? box : 0;
}

template <typename T, int kDim>
int launch_dim(const asd_kv_cache* cache, const AttnParams& p, char* workspace, cudaStream_t stream) {
  CUtensorMap map_k, map_v;
  const int box = box_slots(cache);
  const bool bf16 = cache->dtype == ASD_BF16;
  if (box && make_map(&map_k, bf16, p.cache.k, cache, box) && make_map(&map_v, bf16, p.cache.v, cache, box))
    return launch<T, kDim, true>(map_k, map_v, p, box, workspace, stream);
  return launch<T, kDim, false>(map_k, map_v, p, 0, workspace, stream);
}

}  // namespace

namespace asd_detail {

// 16-bit types, heads of at most 128 whose rows are whole 16-byte words on
// 16-byte boundaries, and scores that grow with q . k (the row's maximum is taken
// before it is scaled).
bool attention_tc_takes(const asd_kv_cache* cache, const AttnParams& p) {
  return cache->dtype != ASD_F32 && p.D <= 128 && p.D % 8 == 0 && p.scale > 0.0f &&
         rows_aligned(p.cache.k, 2, 16, p.cache.page_stride, p.cache.token_stride, p.cache.head_stride) &&
         reinterpret_cast<uintptr_t>(p.cache.v) % 16 == 0 &&
         rows_aligned(p.q, 2, 16, p.q_batch, p.q_token, p.q_head) && reinterpret_cast<uintptr_t>(p.out) % 16 == 0;
}

size_t attention_tc_bytes(const asd_kv_cache* cache, int T, int q_heads) {
  if (cache->dtype == ASD_F32 || cache->head_dim > 128) return 0;
  return attn_layout(kAttnMaxCtas, unit_rows(static_cast<long long>(T) * (q_heads / cache->heads)),
                     cache->head_dim <= 64 ? 64 : 128)
      .total;
}

int launch_attention_tc(const asd_kv_cache* cache, AttnParams p, char* workspace, cudaStream_t stream) {
  p.unit_rows = unit_rows(static_cast<long long>(p.T) * p.group);
  p.row_tiles = (p.T * p.group + p.unit_rows - 1) / p.unit_rows;
  if (cache->dtype == ASD_BF16)
    return p.D <= 64 ? launch_dim<__nv_bfloat16, 64>(cache, p, workspace, stream)
                     : launch_dim<__nv_bfloat16, 128>(cache, p, workspace, stream);
  return p.D <= 64 ? launch_dim<__half, 64>(cache, p, workspace, stream)
                   : launch_dim<__half, 128>(cache, p, workspace, stream);
}

}  // namespace asd_detail
