// libasd: what the tensor-core kernels over a paged cache (asd_attention_tc.cu,
// asd_weigh_tc.cu) share: tcgen05 operands and instructions, copies and TMA boxes of
// pages, bounded waits of a warp, tensor maps.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <mutex>

#include "asd.h"
#include "asd_device.cuh"

namespace asd_detail {

constexpr int kSlabRows = 128;              // rows of an operand slab: slots, or query rows
constexpr int kHalfSlab = kSlabRows * 128;  // bytes of 64 elements of all of them

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
         (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(kSlabRows >> 4) << 24);
}
__device__ __forceinline__ void mma_smem(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
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
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

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
// This thread's arrival at the barrier once all copies that it has issued so far have landed.
__device__ __forceinline__ void copies_arrive(unsigned long long* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Shared memory that this thread wrote, or knows to be written, is the tensor cores' to read.
__device__ __forceinline__ void fence_for_mma() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A bounded wait by a whole warp, one answer for all of it. What follows the
// first look is out of line: the roles' code has to stay small. Where a wait
// gives up, the others do too, and every role leaves its loop; all waits between
// roles are of this kind. error: the workspace's error word, or null.
static __device__ __noinline__ bool warp_wait_on(unsigned long long* bar, uint32_t parity, int* abort, unsigned* error) {
  const unsigned long long t0 = global_ns();
  for (unsigned it = 1;; ++it) {
    if (__all_sync(kFull, mbar_try_wait(bar, parity))) return true;
    if ((it & 255u) == 0 &&
        __any_sync(kFull, *const_cast<volatile int*>(abort) != 0 || global_ns() - t0 > kWaitLimitNs))
      break;
  }
  *const_cast<volatile int*>(abort) = 1;
  if (error) atomicExch(error, static_cast<unsigned>(ASD_ERR_TIMEOUT));
  return false;
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

// ---------------------------------------------------------------- tensor maps (host)

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_tiled() {
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
inline bool make_map(CUtensorMap* map, bool bf16, const void* ptr, const asd_kv_cache* c, int box) {
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

// Slots of a TMA box: what the page size and the tile have in common, and at
// least the swizzle's eight rows; 0: none.
inline int box_slots(const asd_kv_cache* c) {
  int box = kSlabRows;
  while (c->page_size % box != 0) box /= 2;
  return box >= 8 && c->pages > 0 ? box : 0;
}

}  // namespace asd_detail
