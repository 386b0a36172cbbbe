// libasd: attention over a paged cache on the tensor cores (asd_tree_attention
// for 16-bit types).
//
// Per tile of 128 slots: S = Q K^T (128 query rows by 128 slots, fp32 in tensor
// memory), P = exp2(scale S - m) by one thread per row, O += P V with P read from
// tensor memory where S was. m is the row's running maximum (in f16 7 less, so that
// small weights keep their bits), but follows it only when it has grown by more
// than 2^8 in weight: O is then rescaled in tensor memory, else left as it is (the
// quotient O / l does not depend on m).
//
// What bounds it: up to 128 rows per key/value head memory, which the keys and
// values leave once; with more the two MMAs and the softmax between them, and above
// 256 rows memory again, since tensor memory holds two sums of 128 rows and the
// next row tile reads the keys and values anew. Eight key/value heads of 128 in
// bf16, five query heads on each: 32 requests of 9 tokens and 8000 cached ones 115
// to 120 us (5.6 TB/s, 1 % more read than there is), a single token on 250000 158
// to 163 us (6.4 TB/s); four trees on 90000, 50 tokens 244 to 252 us (930
// TFLOP/s), 61 tokens 344 to 358 us (1.76 GB read, 5.1 TB/s); a prompt of 4093 513 us
// (335 TFLOP/s). Short requests are bound by what a
// unit costs at its ends (4 to 5 thousand cycles): 160 of five tokens and up to 577
// cached ones, heads of 64 in f16, 41 to 44 us.
//
// Two softmax groups of 128 threads, each with its own S and O, keep both pipes
// busy: with at most 128 rows they take turns at the tiles and their results are
// added at the end; with more, a unit is 256 rows, each group has 128 of them and
// every tile of keys and values serves both.
//
// A CTA per SM: warps 0-3 and 4-7 are the softmax groups (a warp reads the TMEM
// lanes of its quarter), warp 8 walks the units and loads keys, warp 9 issues the
// MMAs of the scores, warp 10 those of the products, warp 11 loads queries and
// values. Loads are TMA boxes of as many slots as the page size and the tile have
// as a common divisor (a page of 48 is three boxes of 16); where that is less than
// the swizzle's eight rows, 16-byte copies, whose own rate then bounds a call (the
// 32 requests above: pages of 8 121 to 123 us, of 12 286 to 293, of 5 322 to 329, of
// one 380).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>
#include <mutex>
#include <type_traits>

#include "asd.h"
#include "asd_attention.cuh"
#include "asd_attention_tc.h"
#include "asd_launch.cuh"

namespace {

using namespace asd_detail;

constexpr int kTile = 128;      // slots
constexpr int kGroupRows = 128;  // that a softmax group has threads for; a call may use fewer (AttnParams::group_rows)
constexpr int kSoftmaxThreads = 256;
constexpr int kKeyWarp = 8, kScoreWarp = 9, kProductWarp = 10, kValueWarp = 11;
constexpr int kThreads = 12 * 32;  // three warps a scheduler: 168 registers each
constexpr int kTmemCols = 512;
constexpr int kMaxStages = 12;
constexpr unsigned long long kLandNs = 10000000;  // longer than any load takes
constexpr float kGrowth = 8.0f; // log2: how far the maximum may outgrow the reference
// log2: how far below the maximum the reference is set. f16 weights begin to lose bits at 2^-14 and vanish at 2^-25,
// which the many small ones of a long context are, against a largest of 1 (one key ahead of 250000 at 2^-20.6 each: the
// result off by 5.7e-3 of the values' size, with a reference 7 lower by 2e-5); the largest may be 2^15 all the same.
template <typename T> constexpr float kLead = 0.0f;
template <> constexpr float kLead<__half> = 7.0f;

constexpr int slab_bytes(int dim) { return kTile * dim * 2; }  // 128 rows of a padded head
constexpr int kHalfSlab = kTile * 128;                         // 64 elements of all of them
constexpr size_t kSmemMax = 232448;

// What the roles know of a unit: the keys' warp walks the CTA's range and
// publishes its units through a small ring, so that the walk's code exists once
// (the roles' code has to fit the instruction cache beside one another).
struct alignas(16) TcUnit {
  int b, h, row0, rows;      // request, key/value head, first row and rows
  int span, ctx, n, valid;   // slots that the rows see; the request's lengths; 0: there are no more units
  int j0, j1, whole, piece;  // this CTA's tiles, whether they are all of the unit's, the piece's place in the workspace
  int c0, c1, pad[2];        // the CTAs that have a piece each
};
constexpr int kUnits = 8;
constexpr int kUnitReaders = 11;  // warps

struct TcShared {
  unsigned long long k_full[kMaxStages], k_empty[kMaxStages];  // loads have landed; the MMAs have read them
  unsigned long long v_full[kMaxStages], v_empty[kMaxStages];
  unsigned long long unit_full[kUnits], unit_empty[kUnits];
  unsigned long long q_full[2], q_empty[2];  // a query slab is there; is no longer needed
  unsigned long long s_full[2];          // per group: its scores are in tensor memory
  unsigned long long p_ready[2];         // per group: its weights are, and the sum so far is rescaled
  unsigned long long pv_done[2];         // per group: their product is complete
  unsigned long long meet;               // the softmax warps
  unsigned long long drain[2];
  uint32_t tmem_base;
  int abort;
  int last;         // this CTA arrived last at a unit in pieces
  int poison[4];    // of unit u, at u % 4: u + 1 if a new token's values hold NaN or infinities
  TcUnit unit[kUnits];
  AttnDeal deal;
};
// Slabs of a CTA: two of queries, then a ring of keys and one of values, which
// are held longer (their product waits for the softmax).
constexpr int stages_for(int dim) {
  const size_t fit = (kSmemMax - 1024 - sizeof(TcShared) - 2 * slab_bytes(dim)) / slab_bytes(dim);
  return fit < static_cast<size_t>(kMaxStages) ? static_cast<int>(fit) : kMaxStages;
}
constexpr int key_stages(int dim) { return stages_for(dim) / 2; }
constexpr int value_stages(int dim) { return stages_for(dim) - key_stages(dim); }
constexpr size_t smem_for(int dim) {
  return 1024 + static_cast<size_t>(2 + stages_for(dim)) * slab_bytes(dim) + sizeof(TcShared);
}
static_assert(stages_for(128) == 5, "ring depth at the widest head");

// ---------------------------------------------------------------- tcgen05

// Operand tiles of rows of 128 bytes (64 elements) with the 128-byte swizzle,
// eight rows 1024 bytes apart, the next 64 elements of all 128 rows a half slab
// on. Along the rows (keys, queries: K-major) the leading offset is not used; the
// values are read across them (MN-major), where it steps over the half slab.
__device__ __forceinline__ uint64_t tile_desc(uint32_t saddr16, bool across) {  // saddr16: in 16-byte words
  uint64_t d = 0;
  d |= static_cast<uint64_t>(saddr16);  // shared memory ends below 2^18: the field's 14 bits hold it
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
// A TMA box of queries: 64 elements of a group's heads of consecutive tokens.
__device__ __forceinline__ void load_queries(uint32_t dst, const CUtensorMap* map, unsigned long long* bar, int d,
                                             int head, int token, int request) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}],"
      " [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(d), "r"(0), "r"(head), "r"(token),
        "r"(request)
      : "memory");
}
// This thread's arrival at the barrier once all copies that it has issued so far have landed.
__device__ __forceinline__ void copies_arrive(unsigned long long* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Shared memory that this thread wrote, or knows to be written, is the tensor cores' to read.
__device__ __forceinline__ void fence_for_mma() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A bounded wait by a whole warp, one answer for all of it. What follows the
// first look is out of line: the roles' code has to stay small. Where a wait
// gives up, the others do too, and every role leaves its loop; all waits between
// roles are of this kind.
__device__ __noinline__ bool warp_wait_on(unsigned long long* bar, uint32_t parity, int* abort, unsigned* error) {
  const unsigned long long t0 = global_ns();
  for (unsigned it = 1;; ++it) {
    if (__all_sync(kFull, mbar_try_wait(bar, parity))) return true;
    if ((it & 255u) == 0 &&
        __any_sync(kFull, *const_cast<volatile int*>(abort) != 0 || global_ns() - t0 > kWaitLimitNs))
      break;
  }
  *const_cast<volatile int*>(abort) = 1;
  atomicExch(error, static_cast<unsigned>(ASD_ERR_TIMEOUT));
  return false;
}
__device__ __forceinline__ bool warp_wait(unsigned long long* bar, uint32_t parity, TcShared& sh, const AttnParams& p) {
  if (__all_sync(kFull, mbar_try_wait(bar, parity))) return true;
  return __all_sync(kFull, warp_wait_on(bar, parity, &sh.abort, p.error));
}
// Waits (bounded) for all MMAs of this warp.
__device__ __forceinline__ void drain(unsigned long long* bar, bool elected) {
  if (elected) {
    mma_commit(bar);
    const unsigned long long t0 = global_ns();
    while (!mbar_try_wait(bar, 0) && global_ns() - t0 < kWaitLimitNs) {
    }
  }
  __syncwarp();
}
// The same value in every lane, to the compiler too: MMAs and TMA loads take their operands from uniform registers.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __reduce_or_sync(kFull, x); }
__device__ __forceinline__ int uniform(int x) {
  return static_cast<int>(__reduce_or_sync(kFull, static_cast<unsigned>(x)));
}
__device__ __forceinline__ bool elect_lane() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two fp32 operations an instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(r)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)),
        "l"(*reinterpret_cast<unsigned long long*>(&c)));
  return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(r)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
  return *reinterpret_cast<float2*>(&r);
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

// A warp's place in the ring of units.
struct UnitFeed {
  int slot = 0;
  uint32_t phase = 0;
  // the next unit, or null after the last one (or a wait that gave up); done() when it has been read
  __device__ __forceinline__ const TcUnit* wait(TcShared& sh, const AttnParams& p) {
    if (!warp_wait(&sh.unit_full[slot], phase, sh, p) || !sh.unit[slot].valid) return nullptr;
    return &sh.unit[slot];
  }
  __device__ __forceinline__ void done(TcShared& sh) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(&sh.unit_empty[slot]);
    if (++slot == kUnits) {
      slot = 0;
      phase ^= 1u;
    }
  }
};

// A position in a ring of stages.
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
                        const __grid_constant__ CUtensorMap map_q, const __grid_constant__ AttnParams p, int box) {
  constexpr int kSlab = slab_bytes(kDim);
  constexpr bool kBf16 = kExponent<T> == 0x7f807f80u;
  constexpr int kChunks = kDim / 8;          // 16-byte chunks of a row
  constexpr int kRowsAtOnce = 32 / kChunks;  // rows that a warp copies per instruction
  extern __shared__ __align__(1024) unsigned char tc_smem_raw[];
  const uint32_t raw = smem_u32(tc_smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  unsigned char* gbase = tc_smem_raw + (base - raw);
  constexpr int kKeys = key_stages(kDim), kValues = value_stages(kDim);
  const uint32_t sq = base, sk = base + 2 * kSlab, sv = sk + kKeys * kSlab;
  TcShared& sh = *reinterpret_cast<TcShared*>(gbase + (2 + kKeys + kValues) * kSlab);

  const int warp = __shfl_sync(kFull, static_cast<int>(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  pdl_signal_dependents();
  if (warp == kValueWarp) {  // a barrier or two a lane
    if (lane < kMaxStages) {
      mbar_init(&sh.k_full[lane], kTma ? 1 : 32);
      mbar_init(&sh.k_empty[lane], 1);
      mbar_init(&sh.v_full[lane], kTma ? 1 : 32);
      mbar_init(&sh.v_empty[lane], 1);
    }
    if (lane < kUnits) {
      mbar_init(&sh.unit_full[lane], 1);
      mbar_init(&sh.unit_empty[lane], kUnitReaders);
    }
    if (lane >= 16 && lane < 18) {
      const int g = lane - 16;
      mbar_init(&sh.q_full[g], kTma ? 1 : 32);
      mbar_init(&sh.q_empty[g], kSoftmaxThreads / 32);
      mbar_init(&sh.s_full[g], 1);
      mbar_init(&sh.p_ready[g], 4);
      mbar_init(&sh.pv_done[g], 1);
      mbar_init(&sh.drain[g], 1);
    }
    if (lane == 18) {
      mbar_init(&sh.meet, kSoftmaxThreads / 32);
      sh.abort = 0;
    }
    if (lane < 4) sh.poison[lane] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_for_mma();
  }
  if (warp == kScoreWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (kTma && warp == kKeyWarp && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_k)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_v)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_q)) : "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __reduce_max_sync(kFull, sh.tmem_base);
  auto tmem_s = [&](int g) { return tmem + static_cast<uint32_t>(g * kTile); };
  auto tmem_o = [&](int g) { return tmem + static_cast<uint32_t>(2 * kTile + g * kDim); };

  pdl_wait_prerequisites();
  const int chunk = lane % kChunks, sub = lane / kChunks;
  // where chunk `chunk` of row r lies in a slab
  auto place = [&](int r) {
    return static_cast<uint32_t>((chunk >> 3) * kHalfSlab + r * 128 + (((chunk & 7) ^ (r & 7)) << 4));
  };
  const bool has_chunk = chunk * 8 < p.D;
  // 32 rows of a slab from row0 on; off: of row row0 + lane, elements of `src`
  auto copy_rows = [&](uint32_t dst, int row0, const char* src, long long off, int rows) {
#pragma unroll 4
    for (int i = 0; i < 32 / kRowsAtOnce; ++i) {
      const int r = i * kRowsAtOnce + sub;
      const long long o = __shfl_sync(kFull, off, r);
      const bool has = o >= 0 && has_chunk;
      if (r < rows) copy16(dst + place(row0 + r), has ? src + 2 * (o + chunk * 8) : p.q, has);
    }
  };

  if (warp == kKeyWarp || warp == kValueWarp) {
    // ---------------- units and keys; queries and values
    const bool of_v = warp == kValueWarp;
    const bool elected = elect_lane();
    if (!of_v) attn_deal<kTile>(p, sh.deal);
    bool ok = true;
    UnitFeed feed;  // keys: the next free slot
    auto publish = [&](const TcUnit& u) {
      if (ok) ok = warp_wait(&sh.unit_empty[feed.slot], feed.phase ^ 1u, sh, p);
      if (lane == 0) {
        sh.unit[feed.slot] = u;
        mbar_arrive(&sh.unit_full[feed.slot]);
      }
      __syncwarp();
      if (++feed.slot == kUnits) {
        feed.slot = 0;
        feed.phase ^= 1u;
      }
    };
    // the ring
    unsigned long long* const full = of_v ? sh.v_full : sh.k_full;
    unsigned long long* const empty = of_v ? sh.v_empty : sh.k_empty;
    const int stages = of_v ? kValues : kKeys;
    int stage = 0;
    uint32_t phase = 0;
    uint32_t uses = 0;  // of the query slabs, a bit each: whether an odd number of fills
    int slab = 0;       // of a unit that the groups take in turn
    auto load_unit_queries = [&](int b, int h, int row0, int rows) {
      const bool pair = rows > p.group_rows;
#pragma unroll 1
      for (int tile = 0; ok && tile * p.group_rows < rows; ++tile) {
        const int to = pair ? tile : slab, first = row0 + tile * p.group_rows;
        ok = warp_wait(&sh.q_empty[to], ((uses >> to) & 1u) ^ 1u, sh, p);
        uses ^= 1u << to;
        if (!ok) break;
        if constexpr (kTma) {
          // whole tokens: [element][head of the group][key/value head][token][request]
          if (elected) {
            mbar_expect_tx(&sh.q_full[to], static_cast<uint32_t>(p.group_rows) * (kDim * 2));
#pragma unroll
            for (int half = 0; half < kDim / 64; ++half)
              load_queries(sq + to * kSlab + half * kHalfSlab, &map_q, &sh.q_full[to], half * 64, h,
                           p.by_group.quot(first), b);
          }
          __syncwarp();
        } else {
          const int end = min(p.group_rows, rows - tile * p.group_rows);
#pragma unroll 1
          for (int r0 = 0; r0 < end; r0 += 32) {
            const int row = first + r0 + lane, t = p.by_group.quot(row);
            const long long off =
                r0 + lane < end ? b * p.q_batch + t * p.q_token + (h * p.group + (row - t * p.group)) * p.q_head : -1;
            copy_rows(sq + to * kSlab, r0, p.q, off, 32);
          }
          copies_arrive(&sh.q_full[to]);
        }
      }
      if (!pair) slab ^= 1;
    };
    struct Share {
      int b, h;
      int slot0, rows;  // of the tile: rows exist; 0: there is no tile
      // the page table is read a tile ahead
      int page, at;                   // TMA: where this lane's box begins
      long long off[kTile / 32];      // copies: where rows `lane`, 32 + lane .. lie, in elements; -1: none
    };
    const Share none = {};
    AttnWalk<kTile> w(p, sh.deal);       // keys
    bool started = false;
    int b = 0, h = 0, j = 0, j1 = 0, span = 0;  // the unit's next tile
    auto take = [&] {
      Share x = none;
      int row0 = 0, rows = 0;  // of a new unit
      if (ok && j == j1) {
        if (of_v) {
          const TcUnit* u = feed.wait(sh, p);
          if (!u) return x;
          b = u->b, h = u->h, j = u->j0, j1 = u->j1, span = u->span;
          row0 = u->row0, rows = u->rows;
          feed.done(sh);
        } else {
          if (started)
            w.next();
          else
            w.start();
          started = true;
          if (!w.more()) {
            publish(TcUnit{});
            return x;
          }
          b = w.b, h = w.h, j = w.j0, j1 = w.j1(), span = w.span();
          row0 = w.row0(), rows = w.rows();
        }
      }
      if (!ok) return x;
      x.b = b, x.h = h;
      x.slot0 = j * kTile;
      x.rows = min(kTile, span - x.slot0);
      if (kTma && lane * box < x.rows) {
        const int slot = x.slot0 + lane * box, n = p.cache.div.quot(slot);
        x.page = __ldcg(p.cache.table + static_cast<long long>(x.b) * p.cache.table_width + n);
        x.at = slot - n * p.cache.div.size;
      }
      if constexpr (!kTma) {
#pragma unroll
        for (int q = 0; q < kTile / 32; ++q)
          x.off[q] = 32 * q + lane < x.rows ? slot_offset(p.cache, x.b, x.slot0 + 32 * q + lane) : -1;
      }
      ++j;
      if (rows && of_v) load_unit_queries(b, h, row0, rows);
      if (rows && !of_v) {  // while the table is read
        TcUnit u = {};
        u.b = b, u.h = h, u.row0 = row0, u.rows = rows;
        u.span = span, u.ctx = w.r.ctx, u.n = w.r.n, u.valid = 1;
        u.j0 = w.j0, u.j1 = j1, u.whole = w.whole(), u.piece = w.piece();
        if (!u.whole) {
          u.c0 = w.first_cta();
          u.c1 = w.last_cta();
        }
        publish(u);
      }
      return x;
    };
    auto fill = [&](const Share& x) {
      if (ok) ok = warp_wait(&empty[stage], phase ^ 1u, sh, p);
      if (!ok) return;
      const uint32_t dst = (of_v ? sv : sk) + stage * kSlab;
      if constexpr (kTma) {
        unsigned long long* bar = &full[stage];
        const int n = uniform((x.rows + box - 1) / box), head = uniform(x.h);
        if (elected) mbar_expect_tx(bar, static_cast<uint32_t>(n * box) * (kDim * 2));
        __syncwarp();
        // a page out of range lies outside the tensor: the box is filled with zeros
        const CUtensorMap* map = of_v ? &map_v : &map_k;
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
          const int page = __shfl_sync(kFull, x.page, i), at = __shfl_sync(kFull, x.at, i);
          if (elected) {
#pragma unroll
            for (int half = 0; half < kDim / 64; ++half)
              load_box(dst + half * kHalfSlab + i * box * 128, map, bar, half * 64, at, head, page);
          }
        }
        if (!of_v && lane < n && static_cast<unsigned>(x.page) >= static_cast<unsigned>(p.cache.pages) && p.status)
          atomicOr(p.status + x.b, static_cast<int>(ASD_STATUS_PAGE));
        __syncwarp();
      } else {
#pragma unroll
        for (int q = 0; q < kTile / 32; ++q) {
          if (32 * q >= x.rows) break;
          long long off = x.off[q];
          if (off >= 0)
            off += x.h * p.cache.head_stride;
          else if (!of_v && 32 * q + lane < x.rows && p.status)
            atomicOr(p.status + x.b, static_cast<int>(ASD_STATUS_PAGE));
          copy_rows(dst, 32 * q, of_v ? p.cache.v : p.cache.k, off, x.rows - 32 * q);
        }
        copies_arrive(&full[stage]);
      }
      if (++stage == stages) {
        stage = 0;
        phase ^= 1u;
      }
    };
    Share cur = take();
    bool late = true;
    while (ok && cur.rows) {
      // The next tile is looked up first, but not over a unit's end by the values' warp: the unit's queries may have
      // to wait for the one before, and that for this tile. Nothing holds up the CTA's first tile.
      late = j == j1 && (late || of_v);
      Share next = none;
#pragma unroll 1
      for (int i = 0; i < 2; ++i) {
        if ((i == 1) == late)
          next = take();
        else
          fill(cur);
      }
      cur = next;
      late = false;
    }
    if (!kTma) asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == kScoreWarp) {
    // ---------------- S = Q K^T
    constexpr uint32_t kDesc = instr_desc(kBf16, kTile, false);
    const bool elected = elect_lane();
    UnitFeed feed;
    Ring<kKeys> ring;
    bool ok = true;
    uint32_t q_phase = 0, pv_phase = 3;  // a bit a slab; a group
    int turn = 0;                        // the group whose turn it is
    int slab = 0;                        // of a unit that the groups take in turn
    while (ok) {
      const TcUnit* u = feed.wait(sh, p);
      if (!u) break;
      const bool pair = uniform(u->rows) > p.group_rows;
      int left = uniform(u->j1 - u->j0);
      feed.done(sh);
#pragma unroll 1
      for (int s = pair ? 0 : slab; s <= (pair ? 1 : slab); ++s) {
        if (ok) ok = warp_wait(&sh.q_full[s], (q_phase >> s) & 1u, sh, p);
        q_phase ^= 1u << s;
      }
#pragma unroll 1
      for (bool second = false; ok && left > 0;) {
        // the group's scores and weights so far lie where these go
        ok = warp_wait(&sh.pv_done[turn], (pv_phase >> turn) & 1u, sh, p);
        pv_phase ^= 1u << turn;
        if (ok && !second) ok = warp_wait(&sh.k_full[ring.stage], ring.phase, sh, p);
        if (!ok) break;
        if (!kTma) fence_for_mma();  // queries and keys were copied by threads
        tc_fence_after();
        const uint32_t a = uniform((sq + (pair ? turn : slab) * kSlab) >> 4);
        const uint32_t b = uniform((sk + ring.stage * kSlab) >> 4);
        const uint32_t d = uniform(tmem_s(turn));
        const bool ends = !pair || second;  // no group needs the tile's keys any more
        if (elected) {
#pragma unroll
          for (int k = 0; k < kDim / 16; ++k) {
            const uint32_t at = ((k >> 2) * kHalfSlab + (k & 3) * 32) >> 4;
            mma_smem(d, tile_desc(a + at, false), tile_desc(b + at, false), kDesc, k > 0 ? 1u : 0u);
          }
          mma_commit(&sh.s_full[turn]);
          if (ends) mma_commit(&sh.k_empty[ring.stage]);
        }
        __syncwarp();
        turn ^= 1;
        second = !ends;
        if (ends) {
          ring.next();
          --left;
        }
      }
      if (!pair) slab ^= 1;
    }
    drain(&sh.drain[0], elected);
  } else if (warp == kProductWarp) {
    // ---------------- O += P V
    constexpr uint32_t kDesc = instr_desc(kBf16, kDim, true);
    const bool elected = elect_lane();
    UnitFeed feed;
    Ring<kValues> ring;
    bool ok = true;
    uint32_t p_phase = 0;  // a bit a group
    int turn = 0;
    for (int number = 0; ok; ++number) {
      const TcUnit* u = feed.wait(sh, p);
      if (!u) break;
      const bool pair = uniform(u->rows) > p.group_rows;
      const int j0 = uniform(u->j0), j1 = uniform(u->j1), span = uniform(u->span), ctx = uniform(u->ctx);
      feed.done(sh);
#pragma unroll 1
      for (int j = j0; ok && j < j1; ++j) {
        ok = warp_wait(&sh.v_full[ring.stage], ring.phase, sh, p);
        if (!ok) break;
        if (!kTma) fence_for_mma();
        const int end = min(kTile, span - j * kTile);  // rows of the tile that exist
        if (j * kTile > ctx - kTile) {  // (j + 1) * kTile may be 2^31
          // New tokens, or the request's end. Rows past the end become zeros (what lies there may be anything, and 0
          // times NaN is NaN); of a new token some rows may see nothing, so its values' NaN and infinities become
          // zeros too and the unit is marked: its rows look at the end for those that they do see.
          unsigned char* tile = gbase + (sv - base) + ring.stage * kSlab;
          // of the rows past the end the product reads only the rest of the last 16
          for (int r = end + sub; r < min(kTile, (end + 15) & ~15); r += kRowsAtOnce)
            *reinterpret_cast<uint4*>(tile + place(r)) = make_uint4(0u, 0u, 0u, 0u);
          bool found = false;
#pragma unroll 4
          for (int r = max(0, ctx - j * kTile) + sub; r < end; r += kRowsAtOnce) {
            uint4* at = reinterpret_cast<uint4*>(tile + place(r));
            const uint4 was = *at;
            const uint4 now = {finite_pair<T>(was.x), finite_pair<T>(was.y), finite_pair<T>(was.z),
                               finite_pair<T>(was.w)};
            if (now.x != was.x || now.y != was.y || now.z != was.z || now.w != was.w) {
              *at = now;
              found = true;
            }
          }
          if (found) sh.poison[number & 3] = number + 1;
          fence_for_mma();
          __syncwarp();
        }
#pragma unroll 1
        for (bool second = false;;) {
          ok = warp_wait(&sh.p_ready[turn], (p_phase >> turn) & 1u, sh, p);
          p_phase ^= 1u << turn;
          if (!ok) break;
          tc_fence_after();
          const uint32_t a = uniform(tmem_s(turn) + kTile / 2), d = uniform(tmem_o(turn));
          const uint32_t b = uniform((sv + ring.stage * kSlab) >> 4);
          const uint32_t fresh = j - j0 < (pair ? 1 : 2);  // the group's first tile of the unit
          const int steps = uniform((end + 15) >> 4);
          const bool ends = !pair || second;
          if (elected) {
#pragma unroll
            for (int k = 0; k < kTile / 16; ++k)
              if (k < steps)
                mma_tmem(d, a + 8 * k, tile_desc(b + ((k * 16 * 128) >> 4), true), kDesc, k > 0 ? 1u : 1u - fresh);
            mma_commit(&sh.pv_done[turn]);
            if (ends) mma_commit(&sh.v_empty[ring.stage]);
          }
          __syncwarp();
          turn ^= 1;
          if (ends) break;
          second = true;
        }
        ring.next();
      }
    }
    drain(&sh.drain[1], elected);
  } else {
    // ---------------- softmax: thread `row` of group g
    const int g = warp >> 2;
    const int row = threadIdx.x & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = tmem_s(g) + lanes, tw = ts + kTile / 2, to = tmem_o(g) + lanes;  // scores, weights, sum
    bool ok = true;
    uint32_t s_phase = 0, meet_phase = 0;
    int turn = 0, number = 0, slab = 0;
    auto meet = [&] {  // the two groups
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.meet);
      if (ok) ok = warp_wait(&sh.meet, meet_phase, sh, p);
      meet_phase ^= 1u;
    };
    attn_zero_rows<T>(p, threadIdx.x, kSoftmaxThreads);
    UnitFeed feed;
    while (ok) {
      const TcUnit* u = feed.wait(sh, p);
      if (!u) break;
      const AttnRequest req = {u->ctx, u->n};
      const int rows = u->rows, row0 = u->row0, j0 = u->j0, j1 = u->j1;
      const bool pair = rows > p.group_rows;               // each group has rows of its own; else both have the same
      const int r = (pair ? g * p.group_rows : 0) + row;   // of the unit
      const bool lives = row < p.group_rows && r < rows;
      const bool warp_lives = row - lane < p.group_rows && r - lane < rows;  // the same for the warp
      const int t = p.by_group.quot(row0 + min(r, rows - 1));
      float m = -INFINITY, l = 0.0f;
      bool had = false;
#pragma unroll 1
      for (int j = j0; j < j1; ++j) {
        const int whose = turn & 1;
        turn += pair ? 2 : 1;
        if (!pair && whose != g) continue;
        const bool masked = j * kTile > req.ctx - kTile;
        uint32_t sees0 = 0, sees1 = 0, sees2 = 0, sees3 = 0;
        if (masked && warp_lives) {
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            sees0 = sees1, sees1 = sees2, sees2 = sees3;
            sees3 = attn_sees(p, req, u->b, t, j * kTile + 32 * c);
          }
        }
        if (ok) ok = warp_wait(&sh.s_full[g], s_phase, sh, p);
        s_phase ^= 1u;
        tc_fence_after();
        if (ok && warp_lives) {
          float x[2][32];
          float ref = 0.0f;
          // four chains each: one warp a scheduler has little else to cover an operation's latency with
          float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          float2 sums[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
          // The maximum over the first and the second half of the slots; then the weights of the second, which is
          // still in registers, and of the first. The weights lie over the second half's scores. A loop, not four
          // stretches of code: see TcUnit.
#pragma unroll 1
          for (int step = 0; step < 3; ++step) {
            const int half = step & 1;
            tmem_ld32(ts + 64 * half, x[0]);
            tmem_ld32(ts + 64 * half + 32, x[1]);
            tmem_ld_wait();
            if (masked) {
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                const uint32_t sees = half ? (c ? sees3 : sees2) : (c ? sees1 : sees0);
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (!((sees >> i) & 1u)) x[c][i] = -INFINITY;
              }
            }
            if (step < 2) {
#pragma unroll
              for (int i = 0; i < 32; i += 4)
#pragma unroll
                for (int k = 0; k < 4; ++k) tops[k] = fmaxf(tops[k], fmaxf(x[0][i + k], x[1][i + k]));
            }
            if (step == 0) continue;
            if (step == 1) {
              const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * p.scale_log2;
              if (__any_sync(kFull, lives && top > m + (kGrowth + kLead<T>))) {
                const float m_new = fmaxf(m, top - kLead<T>);
                const float fade = exp2_fast(m - (m_new == -INFINITY ? 0.0f : m_new));
                l *= fade;
                m = m_new;
                if (had) {
                  // every product of this group so far is complete: these scores were computed after it
#pragma unroll 1
                  for (int c = 0; c < kDim; c += 16) {
                    float o[16];
                    tmem_ld16(to + c, o);
                    tmem_ld_wait();
                    uint32_t bits[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) bits[i] = __float_as_uint(o[i] * fade);
                    tmem_st16(to + c, bits);
                  }
                }
              }
              ref = m == -INFINITY ? 0.0f : m;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              uint32_t w2[16];
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                float2 e = fma2(make_float2(x[c][i], x[c][i + 1]), make_float2(p.scale_log2, p.scale_log2),
                                make_float2(-ref, -ref));
                e = make_float2(exp2_fast(e.x), exp2_fast(e.y));
                sums[(i >> 1) & 1] = add2(sums[(i >> 1) & 1], e);
                w2[i >> 1] = pack2<T>(e.x, e.y);
              }
              tmem_st16(tw + 32 * half + 16 * c, w2);
            }
          }
          l += (sums[0].x + sums[0].y) + (sums[1].x + sums[1].y);
          tmem_st_wait();
        }
        had = true;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_ready[g]);
      }

      // the unit's rows, or this CTA's piece of them
      const bool whole = u->whole;
      float f_self = 1.0f, f_other = 1.0f;  // what the groups' sums are multiplied with
      bool other_had = false;
      if (had) {
        if (ok) ok = warp_wait(&sh.pv_done[g], s_phase ^ 1u, sh, p);  // of the group's last tile
        tc_fence_after();
      }
      if (!pair) {
        // both groups' statistics, in the slab of the unit's queries, which no MMA reads any more
        other_had = !had || j1 - j0 > 1;
        float2* stat = reinterpret_cast<float2*>(gbase + slab * kSlab);
        tc_fence_before();
        meet();  // both groups' products are complete, the queries have been read
        stat[g * kGroupRows + row] = make_float2(m, l);
        fence_for_mma();  // the slab's next queries come by TMA
        meet();
        tc_fence_after();
        const float2 other = stat[(g ^ 1) * kGroupRows + row];
        const float top = fmaxf(m, other.x);
        const float ref = top == -INFINITY ? 0.0f : top;
        f_self = exp2_fast(m - ref);
        f_other = exp2_fast(other.x - ref);
        l = l * f_self + other.y * f_other;
        m = top;
      }
      // Who writes what: each group its own rows, or of the rows that both have each group a half of the head.
      const bool mine = ok && lives;
      const long long at = (static_cast<long long>(u->b) * p.T + t) * p.q_heads + u->h * p.group + row0 + r -
                           t * p.group;
      const int cols = pair ? kDim : kDim / 2;
      const int col0 = pair ? 0 : g * cols;
      const bool zero = l == 0.0f;  // sees nothing
      if (whole) {
        const float inv = l > 0.0f ? 1.0f / l : l;  // a NaN stays one
        f_self *= inv;
        f_other *= inv;
      }
      T* const dst = reinterpret_cast<T*>(p.out) + at * p.D;
      // [piece][column / 4][row]: a warp's rows lie side by side
      float* const part = p.part_o + static_cast<long long>(u->piece) * kDim * p.unit_rows + r * 4;
#pragma unroll 1
      for (int col = col0; col < col0 + cols; col += 32) {
        __syncwarp();
        float v[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = 0.0f;
        if (ok && warp_lives) {
          float x[32], y[32];
          tmem_ld32(to + col, x);
          tmem_ld32(tmem_o(g ^ 1) + lanes + col, y);
          tmem_ld_wait();
          if (had) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = f_self * x[i];
          }
          if (other_had) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = fmaf(f_other, y[i], v[i]);
          }
        }
        if (mine && whole) {
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            if (col + i >= p.D) break;
            uint4 o;
            o.x = zero ? 0u : pack2<T>(v[i], v[i + 1]);
            o.y = zero ? 0u : pack2<T>(v[i + 2], v[i + 3]);
            o.z = zero ? 0u : pack2<T>(v[i + 4], v[i + 5]);
            o.w = zero ? 0u : pack2<T>(v[i + 6], v[i + 7]);
            *reinterpret_cast<uint4*>(dst + col + i) = o;
          }
        } else if (mine) {
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            *reinterpret_cast<float4*>(part + (col + i) * p.unit_rows) =
                make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        }
      }
      if (mine && (pair || g == 0)) {
        if (whole) {
          if (p.lse) p.lse[at] = zero ? -INFINITY : 0.6931471805599453f * (m + log2f(l));
        } else {
          *reinterpret_cast<float2*>(p.part_ml + 2 * (static_cast<long long>(u->piece) * p.unit_rows + r)) =
              make_float2(m, l);
        }
      }
      if (mine && *const_cast<volatile int*>(&sh.poison[number & 3]) == number + 1) {
        // NaN and infinities that the row does see, onto what this thread has just written
#pragma unroll 1
        const int last = (j1 - 1) * kTile + (kTile - 1);  // j1 * kTile may be 2^31
        for (int slot = max(req.ctx, j0 * kTile); slot < u->span && slot <= last; ++slot) {
          if (!(attn_sees(p, req, u->b, t, slot) & 1u)) continue;
          const long long off = slot_offset(p.cache, u->b, slot);
          if (off < 0) continue;
          const T* src = reinterpret_cast<const T*>(p.cache.v) + off + u->h * p.cache.head_stride;
#pragma unroll 1
          for (int c = col0; c < min(col0 + cols, p.D); ++c) {
            const float e = Store<T>::widen(src[c]);
            if (e - e == 0.0f) continue;
            if (whole)
              dst[c] = Store<T>::narrow(Store<T>::widen(dst[c]) + e);
            else
              part[(c & ~3) * p.unit_rows + (c & 3)] += e;
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (pair) {
        if (lane < 2) mbar_arrive(&sh.q_empty[lane]);
      } else {
        meet();  // both sums and the statistics have been read
        if (lane == 0) mbar_arrive(&sh.q_empty[slab]);
        slab ^= 1;
      }
      tc_fence_after();
      ++number;
      if (!whole && ok) {
        // a unit in pieces
        const int c0 = u->c0, c1 = u->c1;
        __threadfence();
        meet();
        if (threadIdx.x == 0) {
          bool last = false;
          if (ok) {
            last = atomicAdd(p.counters + c0, 1u) == static_cast<unsigned>(c1 - c0);
            if (last) p.counters[c0] = 0u;  // zero again for the next call
          }
          sh.last = last;
        }
        meet();
        if (ok && *const_cast<volatile int*>(&sh.last)) {
          __threadfence();
          // Four columns of a row an item: 16 pieces of one at once, or four of four. On five pieces and more the former,
          // whose loads are in flight together (152 pieces of 5 rows 27 us for the call, with the latter 42); below it
          // the latter (45 rows in 1.7 pieces on average, the 32 chains, 117.8, with the former 119.2). Each alone is
          // smaller code than the choice: with the former alone other calls were 0 to 4 % faster (5 to 125 rows in 2 to
          // 152 pieces), with the latter up to 8 % at 125 rows in few pieces and slower by half at 152.
          auto merge = [&](auto many_items, auto many_pieces) {
            constexpr int kItems = decltype(many_items)::value, kPieces = decltype(many_pieces)::value;
            const int items = rows * (p.D / 4);
#pragma unroll 1
            for (int i0 = threadIdx.x; i0 < items; i0 += kItems * kSoftmaxThreads) {
              float top[kItems], sum[kItems];
              float4 acc[kItems];
#pragma unroll
              for (int i = 0; i < kItems; ++i) {
                top[i] = -INFINITY;
                sum[i] = 0.0f;
                acc[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
              }
#pragma unroll 1
              for (int c = c0; c <= c1; c += kPieces) {
                float2 s[kItems][kPieces];
                float4 v[kItems][kPieces];
#pragma unroll
                for (int i = 0; i < kItems; ++i) {
                  const int item = i0 + i * kSoftmaxThreads, d4 = item / rows, rr = item - d4 * rows;
#pragma unroll
                  for (int k = 0; k < kPieces; ++k) {
                    s[i][k] = make_float2(-INFINITY, 0.0f);
                    v[i][k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    if (item < items && c + k <= c1) {
                      const long long piece = c + k == c0 ? 2 * (c + k) + 1 : 2 * (c + k);
                      s[i][k] = __ldcg(reinterpret_cast<const float2*>(p.part_ml + 2 * (piece * p.unit_rows + rr)));
                      v[i][k] = __ldcg(reinterpret_cast<const float4*>(p.part_o + piece * kDim * p.unit_rows +
                                                                       d4 * (p.unit_rows * 4) + rr * 4));
                    }
                  }
                }
#pragma unroll
                for (int i = 0; i < kItems; ++i) {
                  float most = top[i];
#pragma unroll
                  for (int k = 0; k < kPieces; ++k) most = fmaxf(most, s[i][k].x);
                  const float ref = most == -INFINITY ? 0.0f : most;
                  const float fade = exp2_fast(top[i] - ref);
                  sum[i] *= fade, acc[i].x *= fade, acc[i].y *= fade, acc[i].z *= fade, acc[i].w *= fade;
#pragma unroll
                  for (int k = 0; k < kPieces; ++k) {
                    const float e = exp2_fast(s[i][k].x - ref);
                    sum[i] += e * s[i][k].y;
                    acc[i].x += e * v[i][k].x, acc[i].y += e * v[i][k].y;
                    acc[i].z += e * v[i][k].z, acc[i].w += e * v[i][k].w;
                  }
                  top[i] = most;
                }
              }
#pragma unroll
              for (int i = 0; i < kItems; ++i) {
                const int item = i0 + i * kSoftmaxThreads, d4 = item / rows, rr = item - d4 * rows;
                if (item >= items) break;
                const int tt = p.by_group.quot(row0 + rr);
                const long long to_row = (static_cast<long long>(u->b) * p.T + tt) * p.q_heads + u->h * p.group + row0 +
                                         rr - tt * p.group;
                const float k = sum[i] > 0.0f ? 1.0f / sum[i] : sum[i];
                const uint2 o = sum[i] == 0.0f ? make_uint2(0u, 0u)
                                               : make_uint2(pack2<T>(acc[i].x * k, acc[i].y * k),
                                                            pack2<T>(acc[i].z * k, acc[i].w * k));
                *reinterpret_cast<uint2*>(reinterpret_cast<T*>(p.out) + to_row * p.D + 4 * d4) = o;
                if (d4 == 0 && p.lse)
                  p.lse[to_row] = sum[i] == 0.0f ? -INFINITY : 0.6931471805599453f * (top[i] + log2f(sum[i]));
              }
            }
          };
          if (c1 - c0 < 4)
            merge(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{});
          else
            merge(std::integral_constant<int, 1>{}, std::integral_constant<int, 16>{});
        }
      }
      feed.done(sh);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (sh.abort) {
    attn_incomplete(p.status, p.B, threadIdx.x, kThreads);
    // loads that nobody waited for: give them time to land before the CTA's memory is another's
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < kLandNs) {
    }
  }
  if (warp == kScoreWarp) {
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

// Queries as [request][token][key/value head][head of its group][element], boxes
// of one key/value head's heads of as many tokens as a softmax group has rows
// for; tokens past the last read as zero.
bool make_query_map(CUtensorMap* map, bool bf16, const AttnParams& p) {
  EncodeTiledFn fn = encode_tiled();
  if (!fn) return false;
  auto stride = [&](long long elements, int size) -> cuuint64_t {  // of a dimension of one entry: any
    return size == 1 ? 256u * 2u : static_cast<cuuint64_t>(elements) * 2;
  };
  const cuuint64_t dims[5] = {static_cast<cuuint64_t>(p.D), static_cast<cuuint64_t>(p.group),
                              static_cast<cuuint64_t>(p.heads), static_cast<cuuint64_t>(p.T),
                              static_cast<cuuint64_t>(p.B)};
  const cuuint64_t strides[4] = {stride(p.q_head, p.group), stride(p.q_head * p.group, p.heads), stride(p.q_token, p.T),
                                 stride(p.q_batch, p.B)};
  for (const cuuint64_t s : strides)
    if (s == 0) return false;  // one row for several: copied
  const cuuint32_t boxes[5] = {64, static_cast<cuuint32_t>(p.group), 1,
                               static_cast<cuuint32_t>(p.group_rows / p.group), 1};
  const cuuint32_t steps[5] = {1, 1, 1, 1, 1};
  return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5,
            const_cast<char*>(p.q), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int kDim, bool kTma>
int launch(const CUtensorMap (&maps)[3], AttnParams p, int box, char* workspace, cudaStream_t stream) {
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
  if (cudaLaunchKernelEx(&cfg, kernel, maps[0], maps[1], maps[2], p, box) != cudaSuccess) return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

// Rows of a softmax group: whole tokens, so that a TMA box holds them (a group of
// more than 128 heads has its rows copied).
int group_rows(int group) { return group <= kGroupRows ? kGroupRows / group * group : kGroupRows; }
// Rows of a unit: what one softmax group holds, or both where there are more.
int unit_rows(long long rows, int group) {
  return rows > group_rows(group) ? 2 * group_rows(group) : group_rows(group);
}

// Slots of a TMA box: what the page size and the tile have in common, and at
// least the swizzle's eight rows; 0: none.
int box_slots(const asd_kv_cache* c) {
  int box = kTile;
  while (c->page_size % box != 0) box /= 2;
  return box >= 8 && c->pages > 0 ? box : 0;
}

template <typename T, int kDim>
int launch_dim(const asd_kv_cache* cache, const AttnParams& p, char* workspace, cudaStream_t stream) {
  CUtensorMap maps[3];
  const int box = box_slots(cache);
  const bool bf16 = cache->dtype == ASD_BF16;
  if (box && p.group <= kGroupRows && make_map(&maps[0], bf16, p.cache.k, cache, box) &&
      make_map(&maps[1], bf16, p.cache.v, cache, box) && make_query_map(&maps[2], bf16, p))
    return launch<T, kDim, true>(maps, p, box, workspace, stream);
  return launch<T, kDim, false>(maps, p, 0, workspace, stream);
}

}  // namespace

namespace asd_detail {

// 16-bit types, heads of at most 128 whose rows are whole 16-byte words on
// 16-byte boundaries, and scores that grow with q . k (the row's maximum is taken
// before it is scaled).
bool attention_tc_takes(const asd_kv_cache* cache, const AttnParams& p) {
  return cache->dtype != ASD_F32 && p.D <= 128 && p.D % 8 == 0 && p.scale_log2 > 0.0f &&
         rows_aligned(p.cache.k, 2, 16, p.cache.page_stride, p.cache.token_stride, p.cache.head_stride) &&
         reinterpret_cast<uintptr_t>(p.cache.v) % 16 == 0 &&
         rows_aligned(p.q, 2, 16, p.q_batch, p.q_token, p.q_head) && reinterpret_cast<uintptr_t>(p.out) % 16 == 0;
}

size_t attention_tc_bytes(const asd_kv_cache* cache, int T, int q_heads) {
  if (cache->dtype == ASD_F32 || cache->head_dim > 128) return 0;
  const int group = q_heads / cache->heads;
  const bool shared = static_cast<long long>(T) * group > group_rows(group);
  return attn_layout(kAttnMaxCtas, shared ? 2 * kGroupRows : kGroupRows, cache->head_dim <= 64 ? 64 : 128).total;
}

int launch_attention_tc(const asd_kv_cache* cache, AttnParams p, char* workspace, cudaStream_t stream) {
  p.group_rows = group_rows(p.group);
  p.unit_rows = unit_rows(static_cast<long long>(p.T) * p.group, p.group);
  p.row_tiles = (p.T * p.group + p.unit_rows - 1) / p.unit_rows;
  p.weighted = p.unit_rows > p.group_rows;
  if (cache->dtype == ASD_BF16)
    return p.D <= 64 ? launch_dim<__nv_bfloat16, 64>(cache, p, workspace, stream)
                     : launch_dim<__nv_bfloat16, 128>(cache, p, workspace, stream);
  return p.D <= 64 ? launch_dim<__half, 64>(cache, p, workspace, stream)
                   : launch_dim<__half, 128>(cache, p, workspace, stream);
}

}  // namespace asd_detail
