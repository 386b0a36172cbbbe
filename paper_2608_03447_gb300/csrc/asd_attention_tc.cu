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
// lanes of its quarter), warps 8-11 copy, warp 12 issues the MMAs. Keys and
// values go through one ring of stages in the order in which they are used.
// Copies are 16 bytes per thread and instruction, since a page may hold any
// number of slots and a tile many pages: four warps look 128 slots up at once,
// one a lane, and each row goes to its place in the 128-byte swizzle; slots that
// do not exist are filled with zeros.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>

#include "asd.h"
#include "asd_attention.cuh"
#include "asd_attention_tc.h"
#include "asd_launch.cuh"

namespace {

using namespace asd_detail;

constexpr int kTile = 128;      // slots
constexpr int kGroupRows = 128;
constexpr int kSoftmaxThreads = 256;
constexpr int kCopyThreads = 128;
constexpr int kThreads = kSoftmaxThreads + kCopyThreads + 32;
constexpr int kMmaWarp = (kSoftmaxThreads + kCopyThreads) / 32;
constexpr int kTmemCols = 512;
constexpr int kMaxStages = 12;
constexpr float kGrowth = 8.0f; // log2: how far the maximum may outgrow the reference

constexpr int slab_bytes(int dim) { return kTile * dim * 2; }  // 128 rows of a padded head
constexpr size_t kSmemMax = 232448;

struct TcShared {
  unsigned long long full[kMaxStages];   // a stage's 128 copying threads have seen their copies land
  unsigned long long empty[kMaxStages];  // the MMAs have read it
  unsigned long long q_empty[2];         // a query slab is no longer needed
  unsigned long long s_full[2];          // per group: its scores are in tensor memory
  unsigned long long p_ready[2];         // per group: its weights are, and the sum so far is rescaled
  unsigned long long o_done[2];          // per group: the unit's last product is complete
  unsigned long long drain;
  uint32_t tmem_base;
  int abort;
  int last;         // this CTA arrived last at a unit in pieces
  int poison[4];    // of unit u, at u % 4: u + 1 if a new token's values hold NaN or infinities
  int4 scan[kMaxStages][kCopyThreads / 32];  // per copying warp: rows [x, y) of a stage to look over for unit z
  AttnDeal deal;
};
constexpr int stages_for(int dim) {
  const size_t fit = (kSmemMax - 1024 - sizeof(TcShared) - 2 * slab_bytes(dim)) / slab_bytes(dim);
  return fit < static_cast<size_t>(kMaxStages) ? static_cast<int>(fit) : kMaxStages;
}
constexpr size_t smem_for(int dim) {
  return 1024 + static_cast<size_t>(2 + stages_for(dim)) * slab_bytes(dim) + sizeof(TcShared);
}
// Fills in flight per copying thread before it waits for the oldest. A stage is
// released when the fill after it has landed (the pairs' order of MMAs), so at
// least two of the ring are not in flight.
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
  d |= static_cast<uint64_t>(across ? ((kTile * 128) >> 4) : 1) << 16;
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
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]),
        "f"(r[8]), "f"(r[9]), "f"(r[10]), "f"(r[11]), "f"(r[12]), "f"(r[13]), "f"(r[14]), "f"(r[15]),
        "f"(r[16]), "f"(r[17]), "f"(r[18]), "f"(r[19]), "f"(r[20]), "f"(r[21]), "f"(r[22]), "f"(r[23]),
        "f"(r[24]), "f"(r[25]), "f"(r[26]), "f"(r[27]), "f"(r[28]), "f"(r[29]), "f"(r[30]), "f"(r[31])
      : "memory");
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

// One tile of a unit, as the copying warps and the MMA warp walk them.
struct Item {
  int b, h, slot0, span, ctx, row0, live;
  int unit;    // number of the unit among this CTA's units with work
  int left;    // tiles of the unit after this one
  bool first, valid;
};

// The CTA's tiles one after the other, over the units that see anything.
struct ItemWalk {
  AttnWalk<kTile> w;
  int j, unit;
  __device__ __forceinline__ ItemWalk(const AttnParams& p, const AttnDeal& d) : w(p, d), unit(-1) { enter(); }
  __device__ __forceinline__ void enter() {
    while (w.more() && w.span() == 0) w.next();
    j = w.j0;
    ++unit;
  }
  __device__ __forceinline__ Item get() {
    Item it;
    it.valid = w.more();
    it.first = false;
    if (!it.valid) return it;
    it.b = w.b;
    it.h = w.h;
    it.slot0 = j * kTile;
    it.span = w.span();
    it.ctx = w.r.ctx;
    it.row0 = w.row0();
    it.live = w.live_rows();
    it.unit = unit;
    it.first = j == w.j0;
    it.left = w.j1 - 1 - j;
    if (++j == w.j1) {
      w.next();
      enter();
    }
    return it;
  }
};

// kDim: the head, padded. kPair: units of 256 rows, 128 for each softmax group,
// on shared tiles; else units of 128 rows whose tiles the groups take in turn.
template <typename T, int kDim, bool kPair>
__global__ void __launch_bounds__(kThreads, 1) attention_tc_kernel(const __grid_constant__ AttnParams p) {
  constexpr int kStages = stages_for(kDim), kLag = lag_for(kDim);
  constexpr int kSlab = slab_bytes(kDim);
  constexpr bool kBf16 = sizeof(T) == 2 && kExponent<T> == 0x7f807f80u;
  constexpr int kUnitRows = kPair ? 2 * kGroupRows : kGroupRows;
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
      mbar_init(&sh.full[s], kCopyThreads);
      mbar_init(&sh.empty[s], 1);
    }
    for (int g = 0; g < 2; ++g) {
      mbar_init(&sh.q_empty[g], kPair ? 128 : kSoftmaxThreads);
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
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __reduce_max_sync(kFull, sh.tmem_base);
  const uint32_t tmem_s[2] = {tmem, tmem + kTile};
  const uint32_t tmem_o[2] = {tmem + 2 * kTile, tmem + 2 * kTile + kDim};

  pdl_wait_prerequisites();
  const bool failed = __syncthreads_or(threadIdx.x == 0 && __ldcg(p.error) != 0);
  if (failed && blockIdx.x == 0 && p.status)
    for (int b = threadIdx.x; b < p.B; b += kThreads) atomicOr(p.status + b, static_cast<int>(ASD_STATUS_INCOMPLETE));
  const bool work = !failed && attn_deal<kTile>(p, sh.deal);  // the same for all threads

  if (work && warp >= kSoftmaxThreads / 32 && warp < kMmaWarp) {
    // ---------------- copies
    constexpr int kChunks = kDim / 8;           // 16-byte chunks of a row
    constexpr int kRowsAtOnce = 32 / kChunks;   // rows that a warp copies per instruction
    const int cw = warp - kSoftmaxThreads / 32; // rows cw * 32 .. of every slab
    const int chunk = lane % kChunks, sub = lane / kChunks;
    const bool has_chunk = chunk * 8 < p.D;
    // where chunk `chunk` of row r lies in a slab
    auto place = [&](int r) {
      return static_cast<uint32_t>((chunk >> 3) * (kTile * 128) + r * 128 + (((chunk & 7) ^ (r & 7)) << 4));
    };
    int issued = 0, arrived = 0, stage_in = 0, stage_out = 0;
    uint32_t phase_in = 0;
    bool ok = true;
    uint32_t q_uses[2] = {0, 0};
    // New tokens' values: some row may not see them, and its weight of 0 times a NaN or an infinity would reach it.
    // Such elements become 0 and the unit is marked; its rows look for what they do see at the end.
    auto look_over = [&](int4 rows) {
      bool found = false;
      for (int r = cw * 32 + sub; r < cw * 32 + 32; r += kRowsAtOnce) {
        if (r < rows.x || r >= rows.y) continue;
        uint4* at = reinterpret_cast<uint4*>(gbase + (2 + stage_out) * kSlab + place(r));
        const uint4 was = *at;
        const uint4 now = {finite_pair<T>(was.x), finite_pair<T>(was.y), finite_pair<T>(was.z), finite_pair<T>(was.w)};
        if (now.x != was.x || now.y != was.y || now.z != was.z || now.w != was.w) {
          *at = now;
          found = true;
        }
      }
      if (found) sh.poison[rows.z & 3] = rows.z + 1;
    };
    auto arrive = [&] {  // this thread's copies of the stage have landed
      const int4 rows = sh.scan[stage_out][cw];
      if (rows.x < rows.y) look_over(rows);
      fence_for_mma();
      mbar_arrive(&sh.full[stage_out]);
      if (++stage_out == kStages) stage_out = 0;
      ++arrived;
    };
    // A fill is announced kLag fills later, or before a wait for the rest of the kernel.
    auto flush = [&] {
      copies_wait<0>();
      while (arrived < issued) arrive();
    };
    auto announce = [&](int lo, int hi, int unit) {
      copies_commit();
      if (lane == 0) sh.scan[stage_in][cw] = make_int4(lo, hi, unit, 0);
      __syncwarp();
      ++issued;
      if (++stage_in == kStages) {
        stage_in = 0;
        phase_in ^= 1u;
      }
      if (issued - arrived > kLag) {
        copies_wait<kLag>();
        arrive();
      }
    };
    auto wait_stage = [&] {
      if (ok) ok = warp_wait(&sh.empty[stage_in], phase_in ^ 1u, sh, p);
      return skv + stage_in * kSlab;
    };
    auto copy_rows = [&](uint32_t dst, const char* src, long long off) {  // off: of row cw * 32 + lane, elements; < 0: zeros
#pragma unroll
      for (int i = 0; i < 32 / kRowsAtOnce; ++i) {
        const int r = i * kRowsAtOnce + sub;
        const long long o = __shfl_sync(kFull, off, r);
        const bool has = o >= 0 && has_chunk;
        copy16(dst + place(cw * 32 + r), has ? src + 2 * (o + chunk * 8) : p.q, has);
      }
    };
    auto slot_of = [&](const Item& it) -> long long {
      const int slot = it.slot0 + cw * 32 + lane;
      if (slot >= it.span) return -1;
      const long long off = slot_offset(p.cache, it.b, slot);
      if (off < 0) {
        if (p.status) atomicOr(p.status + it.b, static_cast<int>(ASD_STATUS_PAGE));
        return -1;
      }
      return off + it.h * p.cache.head_stride;
    };
    auto load_q = [&](const Item& it, int tile, int slab) {  // query rows tile * 128 .. of the unit
      const uint32_t parity = (q_uses[slab] & 1u) ^ 1u;
      if (ok && !__all_sync(kFull, mbar_try_wait(&sh.q_empty[slab], parity))) {
        flush();
        ok = warp_wait(&sh.q_empty[slab], parity, sh, p);
      }
      ++q_uses[slab];
      const int r = tile * kGroupRows + cw * 32 + lane;
      long long off = -1;
      if (r < it.live) {
        const int row = it.row0 + r, t = row / p.group;
        off = it.b * p.q_batch + t * p.q_token + (it.h * p.group + (row - t * p.group)) * p.q_head;
      }
      if (ok) copy_rows(sq + slab * kSlab, p.q, off);
    };
    auto load_k = [&](const Item& it, long long off) {
      const uint32_t dst = wait_stage();
      if (it.first) {
        if (kPair) {
          load_q(it, 0, 0);
          if (it.live > kGroupRows) load_q(it, 1, 1);
        } else {
          load_q(it, 0, it.unit & 1);
        }
      }
      if (ok) copy_rows(dst, p.cache.k, off);
      announce(0, 0, 0);
    };
    auto load_v = [&](const Item& it, long long off) {
      const uint32_t dst = wait_stage();
      if (ok) copy_rows(dst, p.cache.v, off);
      announce(max(0, it.ctx - it.slot0), ok ? min(kTile, it.span - it.slot0) : 0, it.unit);
    };

    ItemWalk walk(p, sh.deal);
    Item a = walk.get();
    if (a.valid) {
      long long off_a = slot_of(a);
      load_k(a, off_a);
      while (a.valid) {
        if (kPair) {
          load_v(a, off_a);
          a = walk.get();
          if (!a.valid) break;
          off_a = slot_of(a);
          load_k(a, off_a);
        } else {
          const Item next = walk.get();
          long long off_next = -1;
          if (next.valid) {
            off_next = slot_of(next);
            load_k(next, off_next);
          }
          load_v(a, off_a);
          a = next;
          off_a = off_next;
        }
      }
    }
    flush();
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
    int stage = 0;
    uint32_t phase = 0;
    uint32_t p_phase[2] = {0, 0};
    auto next_stage = [&] {
      if (++stage == kStages) {
        stage = 0;
        phase ^= 1u;
      }
    };
    auto wait_full = [&] {
      if (ok) ok = warp_wait(&sh.full[stage], phase, sh, p);
      tc_fence_after();
    };
    auto scores = [&](int g, int slab) {
      if (ok && elected) {
        const uint64_t a = tile_desc(sq + slab * kSlab, false), b = tile_desc(skv + stage * kSlab, false);
#pragma unroll
        for (int k = 0; k < kDim / 16; ++k) {
          const uint32_t at = ((k >> 2) * (kTile * 128) + (k & 3) * 32) >> 4;
          mma_smem(tmem_s[g], a + at, b + at, kDescS, k > 0 ? 1u : 0u);
        }
        mma_commit(&sh.s_full[g]);
      }
    };
    auto product = [&](int g, bool first, bool last) {
      if (ok) ok = warp_wait(&sh.p_ready[g], p_phase[g], sh, p);
      p_phase[g] ^= 1u;
      tc_fence_after();
      if (ok && elected) {
        const uint64_t b = tile_desc(skv + stage * kSlab, true);
#pragma unroll
        for (int k = 0; k < kTile / 16; ++k)
          mma_tmem(tmem_o[g], tmem_s[g] + 8 * k, b + ((k * 16 * 128) >> 4), kDescO, !first || k > 0 ? 1u : 0u);
        if (last) mma_commit(&sh.o_done[g]);
      }
    };
    auto release = [&] {
      if (ok && elected) mma_commit(&sh.empty[stage]);
      next_stage();
    };
    if (kPair) {
      // S0(0) S1(0), then per tile j: PV0(j) S0(j + 1) PV1(j) S1(j + 1); a unit ends without a next tile
      for (AttnWalk<kTile> w(p, sh.deal); w.more(); w.next()) {
        if (w.span() == 0) continue;
        const bool two = w.live_rows() > kGroupRows;
        wait_full();
        scores(0, 0);
        if (two) scores(1, 1);
        release();
        for (int j = w.j0; j < w.j1; ++j) {
          const bool more = j + 1 < w.j1;
          wait_full();  // V(j)
          const int v_stage = stage;
          int k_stage = stage + 1;
          uint32_t k_phase = phase;
          if (k_stage == kStages) {
            k_stage = 0;
            k_phase ^= 1u;
          }
          product(0, j == w.j0, !more);
          if (more) {
            if (ok) ok = warp_wait(&sh.full[k_stage], k_phase, sh, p);
            tc_fence_after();
            stage = k_stage;
            scores(0, 0);
            stage = v_stage;
          }
          if (two) product(1, j == w.j0, !more);
          release();  // V(j)
          if (more) {
            if (two) scores(1, 1);
            release();  // K(j + 1)
          }
        }
      }
    } else {
      // tile i of the CTA goes to group i % 2: S(0), then S(i + 1) PV(i)
      ItemWalk walk(p, sh.deal);
      Item a = walk.get();
      int i = 0;
      if (a.valid) {
        wait_full();
        scores(0, a.unit & 1);
        release();
      }
      int seen[2] = {-1, -1};  // the unit whose sum a group's accumulator holds
      while (a.valid) {
        const Item next = walk.get();
        if (next.valid) {
          wait_full();
          scores((i + 1) & 1, next.unit & 1);
          release();
        }
        const int g = i & 1;
        wait_full();
        product(g, seen[g] != a.unit, a.left < 2);  // the last for the group: the unit's next tile is the other's
        seen[g] = a.unit;
        release();
        a = next;
        ++i;
      }
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
    bool ok = true;
    uint32_t s_phase = 0, o_phase = 0;
    int tile_count = 0, unit = 0;
    for (AttnWalk<kTile> w(p, sh.deal); w.more(); w.next()) {
      const int span = w.span(), rows = w.rows(), live = w.live_rows();
      const int group_row0 = kPair ? g * kGroupRows : 0;
      const int r = group_row0 + row;                                    // of the unit
      const bool warp_live = group_row0 + (warp & 3) * 32 < live;        // the same for the warp
      const bool works = span > 0 && (!kPair || live > group_row0);      // the same for the group
      const int t = (w.row0() + min(r, max(live - 1, 0))) / p.group;
      float m = -INFINITY, l = 0.0f;
      bool had = false;
      for (int j = w.j0; works && j < w.j1; ++j) {
        if (!kPair && ((tile_count++) & 1) != g) continue;
        const int slot0 = j * kTile;
        const bool masked = slot0 + kTile > w.r.ctx;
        uint32_t sees[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
        if (masked && warp_live) {
#pragma unroll
          for (int c = 0; c < 4; ++c) sees[c] = attn_sees(p, w.r, w.b, t, slot0 + 32 * c);
        }
        if (ok) ok = warp_wait(&sh.s_full[g], s_phase, sh, p);
        s_phase ^= 1u;
        tc_fence_after();
        if (ok && warp_live) {
          const uint32_t ts = tmem_s[g] + lanes, to = tmem_o[g] + lanes;
          float x[32];
          float top = -INFINITY;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            tmem_ld32(ts + 32 * c, x);
            tmem_ld_wait();
            if (masked) {
#pragma unroll
              for (int i = 0; i < 32; ++i) x[i] = (sees[c] >> i) & 1u ? x[i] : -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) top = fmaxf(top, x[i]);
          }
          top *= p.scale_log2;
          if (__any_sync(kFull, r < live && top > m + kGrowth)) {
            const float m_new = fmaxf(m, top);
            const float fade = exp2_fast(m - (m_new == -INFINITY ? 0.0f : m_new));
            l *= fade;
            m = m_new;
            if (had) {
              // every product of this group so far has completed: it came before these scores
#pragma unroll
              for (int c = 0; c < kDim / 32; ++c) {
                tmem_ld32(to + 32 * c, x);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] *= fade;
                tmem_st32(to + 32 * c, x);
              }
            }
          }
          const float ref = m == -INFINITY ? 0.0f : m;
          float sum = 0.0f;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            tmem_ld32(ts + 32 * c, x);
            tmem_ld_wait();
            uint32_t w2[16];
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              float e0 = exp2_fast(fmaf(x[i], p.scale_log2, -ref));
              float e1 = exp2_fast(fmaf(x[i + 1], p.scale_log2, -ref));
              if (masked) {
                e0 = (sees[c] >> i) & 1u ? e0 : 0.0f;
                e1 = (sees[c] >> (i + 1)) & 1u ? e1 : 0.0f;
              }
              sum += e0 + e1;
              w2[i >> 1] = pack2<T>(e0, e1);
            }
            tmem_st16(ts + 16 * c, w2);  // over scores that have been read
          }
          l += sum;
          tmem_st_wait();
        }
        had = true;
        tc_fence_before();
        mbar_arrive(&sh.p_ready[g]);
      }

      // the unit's rows, or this CTA's piece of them
      const bool whole = w.whole();
      float scale_self = 1.0f, scale_other = 0.0f;
      bool has[2] = {kPair && g == 0 && had, kPair && g == 1 && had};
      if (works) {
        if (had) {
          if (ok) ok = warp_wait(&sh.o_done[g], o_phase, sh, p);
          o_phase ^= 1u;
          tc_fence_after();
        }
        if (kPair) {
          mbar_arrive(&sh.q_empty[g]);
        } else {
          // both groups' statistics, in the slab of the unit's queries, which no MMA reads any more
          const int n = w.j1 - w.j0, first = (tile_count - n) & 1;
          has[first] = true;
          has[first ^ 1] = n > 1;
          float2* stat = reinterpret_cast<float2*>(gbase + (unit & 1) * kSlab);
          tc_fence_before();
          softmax_sync();  // both groups' products are complete, the queries have been read
          stat[g * kGroupRows + row] = make_float2(m, l);
          softmax_sync();
          tc_fence_after();
          const float2 other = stat[(g ^ 1) * kGroupRows + row];
          const float m2 = fmaxf(m, other.x);
          const float ref = m2 == -INFINITY ? 0.0f : m2;
          scale_self = exp2_fast(m - ref);
          scale_other = exp2_fast(other.x - ref);
          l = l * scale_self + other.y * scale_other;
          m = m2;
        }
      }
      const bool poisoned = works && *const_cast<volatile int*>(&sh.poison[unit & 3]) == unit + 1;
      const bool mine = ok && r < rows;
      const long long at =
          (static_cast<long long>(w.b) * p.T + (w.row0() + r) / p.group) * p.q_heads + w.h * p.group +
          (w.row0() + r) % p.group;
      const float inv = r < live && l > 0.0f ? 1.0f / l : r < live ? l : 0.0f;
      constexpr int kCols = kPair ? kDim : kDim / 2;  // that this thread writes
      const int col0 = kPair ? 0 : g * kCols;
#pragma unroll 1
      for (int c = 0; c < kCols; c += 32) {
        const int col = col0 + c;
        __syncwarp();
        float v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = 0.0f;
        if (ok && works && warp_live) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (!has[k]) continue;
            const float f = kPair ? 1.0f : (k == g ? scale_self : scale_other);
            float x[32];
            tmem_ld32(tmem_o[k] + lanes + col, x);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = fmaf(f, x[i], v[i]);
          }
          if (poisoned && r < live) {
            const int end = min(span, w.j1 * kTile);
            for (int slot = max(w.r.ctx, w.j0 * kTile); slot < end; ++slot) {
              if (!(attn_sees(p, w.r, w.b, t, slot) & 1u)) continue;
              const long long off = slot_offset(p.cache, w.b, slot);
              if (off < 0) continue;
              const T* src = reinterpret_cast<const T*>(p.cache.v) + off + w.h * p.cache.head_stride + col;
              for (int i = 0; i < 32; ++i) {
                if (col + i >= p.D) break;
                const float f = Store<T>::widen(src[i]);
                if (!(f - f == 0.0f)) {
#pragma unroll
                  for (int k = 0; k < 32; ++k)
                    if (k == i) v[k] += f;
                }
              }
            }
          }
        }
        if (mine && whole) {
          T* dst = reinterpret_cast<T*>(p.out) + at * p.D + col;
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            if (col + i >= p.D) break;
            const bool zero = r >= live || l == 0.0f;
            uint4 o;
            o.x = zero ? 0u : pack2<T>(v[i] * inv, v[i + 1] * inv);
            o.y = zero ? 0u : pack2<T>(v[i + 2] * inv, v[i + 3] * inv);
            o.z = zero ? 0u : pack2<T>(v[i + 4] * inv, v[i + 5] * inv);
            o.w = zero ? 0u : pack2<T>(v[i + 6] * inv, v[i + 7] * inv);
            *reinterpret_cast<uint4*>(dst + i) = o;
          }
        } else if (mine && r < live) {
          // [piece][column / 4][row]: a warp's rows lie side by side
          float* dst = p.part_o + (static_cast<long long>(w.piece()) * (kDim / 4) + col / 4) * (kUnitRows * 4) + r * 4;
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            *reinterpret_cast<float4*>(dst + i * kUnitRows) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        }
      }
      if (mine && (kPair || g == 0)) {
        if (whole) {
          if (p.lse) p.lse[at] = r >= live || l == 0.0f ? -INFINITY : 0.6931471805599453f * (m + log2f(l));
        } else if (r < live) {
          *reinterpret_cast<float2*>(p.part_ml + 2 * (static_cast<long long>(w.piece()) * kUnitRows + r)) =
              make_float2(m, l);
        }
      }
      if (!kPair && works) {
        tc_fence_before();
        softmax_sync();  // both sums and the statistics have been read
        tc_fence_after();
        mbar_arrive(&sh.q_empty[unit & 1]);
      }
      if (span > 0) ++unit;
      if (whole) continue;

      // a unit in pieces (it sees more than one tile, so every row group has work or writes zeros below)
      __threadfence();
      softmax_sync();
      const int c0 = w.first_cta(), c1 = w.last_cta();
      if (threadIdx.x == 0) {
        bool last = false;
        if (ok) {
          last = atomicAdd(p.counters + c0, 1u) == static_cast<unsigned>(c1 - c0);
          if (last) p.counters[c0] = 0u;
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
        const long long to = (static_cast<long long>(w.b) * p.T + tt) * p.q_heads + w.h * p.group + w.row0() + rr -
                             tt * p.group;
        float top = -INFINITY, sum = 0.0f;
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (rr < live) {
#pragma unroll 4
          for (int c = c0; c <= c1; ++c) {
            const long long piece = c == c0 ? 2 * c + 1 : 2 * c;
            top = fmaxf(top, __ldcg(p.part_ml + 2 * (piece * kUnitRows + rr)));
          }
          const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
          for (int c = c0; c <= c1; ++c) {
            const long long piece = c == c0 ? 2 * c + 1 : 2 * c;
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(p.part_ml + 2 * (piece * kUnitRows + rr)));
            const float4 v = __ldcg(reinterpret_cast<const float4*>(
                p.part_o + (piece * (kDim / 4) + d4) * (kUnitRows * 4) + rr * 4));
            const float f = exp2_fast(ml.x - ref);
            sum += f * ml.y;
            acc.x += f * v.x, acc.y += f * v.y, acc.z += f * v.z, acc.w += f * v.w;
          }
        }
        const float k = sum > 0.0f ? 1.0f / sum : sum;
        const uint2 o = sum == 0.0f ? make_uint2(0u, 0u)
                                    : make_uint2(pack2<T>(acc.x * k, acc.y * k), pack2<T>(acc.z * k, acc.w * k));
        *reinterpret_cast<uint2*>(reinterpret_cast<T*>(p.out) + to * p.D + 4 * d4) = o;
        if (d4 == 0 && p.lse) p.lse[to] = sum == 0.0f ? -INFINITY : 0.6931471805599453f * (top + log2f(sum));
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

template <typename T, int kDim, bool kPair>
int launch(AttnParams p, char* workspace, cudaStream_t stream) {
  auto kernel = attention_tc_kernel<T, kDim, kPair>;
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
  p.unit_rows = kPair ? 2 * kGroupRows : kGroupRows;
  p.row_tiles = (p.T * p.group + p.unit_rows - 1) / p.unit_rows;
  const AttnLayout l = attn_layout(kAttnMaxCtas, p.unit_rows, kDim);
  p.counters = reinterpret_cast<unsigned*>(workspace + l.counters);
  p.part_ml = reinterpret_cast<float*>(workspace + l.ml);
  p.part_o = reinterpret_cast<float*>(workspace + l.o);
  cudaLaunchAttribute attr;
  cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(grid)), dim3(kThreads), stream, &attr);
  cfg.dynamicSmemBytes = smem_for(kDim);
  if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

bool paired(const AttnParams& p) { return p.T * p.group > kGroupRows; }

template <typename T>
int launch_typed(const AttnParams& p, char* workspace, cudaStream_t stream) {
  if (p.D <= 64)
    return paired(p) ? launch<T, 64, true>(p, workspace, stream) : launch<T, 64, false>(p, workspace, stream);
  return paired(p) ? launch<T, 128, true>(p, workspace, stream) : launch<T, 128, false>(p, workspace, stream);
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
  const int rows = T * (q_heads / cache->heads) > kGroupRows ? 2 * kGroupRows : kGroupRows;
  return attn_layout(kAttnMaxCtas, rows, cache->head_dim <= 64 ? 64 : 128).total;
}

int launch_attention_tc(const asd_kv_cache* cache, AttnParams p, char* workspace, cudaStream_t stream) {
  return cache->dtype == ASD_BF16 ? launch_typed<__nv_bfloat16>(p, workspace, stream)
                                  : launch_typed<__half>(p, workspace, stream);
}

}  // namespace asd_detail
