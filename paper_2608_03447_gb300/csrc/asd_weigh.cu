// libasd: the attention weight that each cached slot receives (asd_kv_weigh): the
// entry point, and the kernel on the CUDA cores, for 32-bit caches and layouts that the
// tensor-core kernel does not take.
//
// w[s] = sum over rows of exp(scale q k_s - lse): the rows' softmax is known by its
// log-sum-exp, so one pass over the keys does, and every slot's sum stands alone.
//
// A CTA of 256 threads has 16 kI query rows that share a key/value head against
// tiles of 64 slots. Thread (y, x) of 16 x 16 computes the scores of rows y + 16 i
// and slots x + 16 j, four elements of the head at a time from shared memory, adds up
// its rows' weights, and the sixteen threads of a slot are added up at the end of the
// tile, always in the same order.
//
// What bounds it: fp32 multiply-adds, and the end of a range, which is four or five
// tiles long: 17 rows of 8 trees on up to 2900 slots, 16 heads on 4 of 96, take 43 to 44
// us (FMA pipe 49 % busy; 68 rows of a group's heads are computed as 80). Queries and
// the next tile's keys are copied in the background: with loads by way of registers,
// one row after the other, 103 us.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "asd.h"
#include "asd_launch.cuh"
#include "asd_weigh.cuh"

namespace {

using namespace asd_detail;

constexpr int kSimtThreads = 256;
constexpr int kSimtTile = 64;
constexpr int kMaxDevices = 64;

// Shared memory, in floats: rows of the head padded to a multiple of four and
// one more vector, so that a warp's sixteen rows start in different banks.
__host__ __device__ constexpr int simt_pitch(int dim) { return (dim + 3) / 4 * 4 + 4; }
// queries, two tiles of keys, where the rows lie, their scales, the warps' sums
constexpr size_t simt_smem(int rows, int dim) {
  return sizeof(float) * static_cast<size_t>(rows + 2 * kSimtTile) * simt_pitch(dim) +
         sizeof(long long) * (rows + 2 * kSimtTile) + sizeof(RowScale) * rows +
         sizeof(float) * (kSimtThreads / 32) * kSimtTile;
}

template <typename T>
__device__ __forceinline__ void load4(const T* p, bool vec, int valid, float (&x)[4]) {
  if (vec) {
    if constexpr (sizeof(T) == 4) {
      const float4 w = __ldcg(reinterpret_cast<const float4*>(p));
      x[0] = w.x, x[1] = w.y, x[2] = w.z, x[3] = w.w;
    } else {
      const uint2 w = __ldcg(reinterpret_cast<const uint2*>(p));
      T e[4];
      memcpy(e, &w, 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = Store<T>::widen(e[i]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = i < valid ? Store<T>::widen(p[i]) : 0.0f;
}

__device__ __forceinline__ void copy16(float* dst, const float* src, bool has) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(has ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(r)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)),
        "l"(*reinterpret_cast<unsigned long long*>(&c)));
  return *reinterpret_cast<float2*>(&r);
}

// kI: query rows of a thread.
template <typename T, int kI>
__global__ void __launch_bounds__(kSimtThreads, 2)
    weigh_kernel(const __grid_constant__ WeighParams p, bool vec_q, bool vec_k) {
  constexpr int kRows = 16 * kI, kWarps = kSimtThreads / 32;
  extern __shared__ __align__(16) float smem[];
  __shared__ AttnDeal deal;
  const AttnParams a = weigh_deal_params(p);
  const int D = a.D, pitch = simt_pitch(D), quads = (D + 3) / 4;
  float* sq = smem;                // [kRows][pitch]
  float* sk = sq + kRows * pitch;  // [2][kSimtTile][pitch]
  long long* s_at = reinterpret_cast<long long*>(sk + 2 * kSimtTile * pitch);  // [2][kSimtTile] of a tile's keys
  long long* s_row = s_at + 2 * kSimtTile;                                     // [kRows] of the queries
  RowScale* s_scale = reinterpret_cast<RowScale*>(s_row + kRows);              // [kRows]
  float* s_sum = reinterpret_cast<float*>(s_scale + kRows);                    // [kWarps][kSimtTile]
  const int tid = threadIdx.x, x = tid & 15, y = tid >> 4, lane = tid & 31, warp = tid >> 5;
  pdl_signal_dependents();
  pdl_wait_prerequisites();
  if (tid < 32) attn_deal<kSimtTile>(a, deal);
  __syncthreads();
  if (deal.begin == deal.end) return;

  AttnWalk<kSimtTile> w(a, deal);
  for (w.start(); w.more(); w.next()) {
    const int rows = w.rows(), span = w.span(), ctx = w.r.ctx, j0 = w.j0, j1 = w.j1();
    const int tiles = (rows + kRows - 1) / kRows;
    // a thread a row says where it lies; then a warp a row copies it
    auto find_rows = [&](int row0) {
      for (int r = tid; r < kRows; r += kSimtThreads) {
        const int row = row0 + r, t = row < rows ? a.by_group.quot(row) : 0;
        const int head = w.h * a.group + row - t * a.group;
        const int token = row < rows ? weigh_token(p, w.b, t) : -1;
        s_row[r] = token < 0 ? -1 : w.b * a.q_batch + token * a.q_token + head * a.q_head;
        s_scale[r] = row_scale(row_lse(p, w.b, token, head));
      }
    };
    // in the background, or (types to widen, odd rows) by way of registers
    auto load_tile = [&](float* dst, const long long* offsets, const char* from, int n, bool vec) {
      const T* base = reinterpret_cast<const T*>(from);
#pragma unroll 4
      for (int r = warp; r < n; r += kWarps) {
        const long long o = offsets[r];
        for (int d4 = lane; d4 < quads; d4 += 32) {
          if constexpr (sizeof(T) == 4) {
            if (vec) {
              copy16(dst + r * pitch + 4 * d4, o >= 0 ? base + o + 4 * d4 : base, o >= 0);
              continue;
            }
          }
          float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          if (o >= 0) load4(base + o + 4 * d4, vec, D - 4 * d4, f);
          *reinterpret_cast<float4*>(dst + r * pitch + 4 * d4) = make_float4(f[0], f[1], f[2], f[3]);
        }
      }
    };
    auto find_keys = [&](int j) {
      const int slot = j * kSimtTile + tid;
      if (tid >= kSimtTile || j >= j1) return;
      long long at = -1;
      if (slot < span) {
        at = slot_offset(a.cache, w.b, slot);
        if (at >= 0)
          at += w.h * a.cache.head_stride;
        else if (a.status)
          atomicOr(a.status + w.b, static_cast<int>(ASD_STATUS_PAGE));
      }
      s_at[(j & 1) * kSimtTile + tid] = at;
    };
    auto load_keys = [&](int j) {
      if (j < j1) load_tile(sk + (j & 1) * kSimtTile * pitch, s_at + (j & 1) * kSimtTile, a.cache.k, kSimtTile, vec_k);
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    __syncthreads();  // the unit before is done with shared memory
    find_rows(0);
    find_keys(j0);
    find_keys(j0 + 1);
    __syncthreads();
    load_tile(sq, s_row, a.q, kRows, vec_q);
    load_keys(j0);
    for (int j = j0; j < j1; ++j) {
      const int slot0 = j * kSimtTile;
      const float* keys = sk + (j & 1) * kSimtTile * pitch;
      load_keys(j + 1);  // the other buffer, which the tile before is done with
      asm volatile("cp.async.wait_group 1;" ::: "memory");
      const bool masked = slot0 > ctx - kSimtTile;  // slot0 + kSimtTile may be 2^31
      float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      for (int tile = 0; tile < tiles; ++tile) {
        if (tiles > 1 && (tile > 0 || j > j0)) {
          __syncthreads();
          find_rows(tile * kRows);
          __syncthreads();
          load_tile(sq, s_row, a.q, kRows, vec_q);
          asm volatile("cp.async.wait_all;" ::: "memory");
        }
        __syncthreads();
        float2 s[kI][4];
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c) s[i][c] = make_float2(0.0f, 0.0f);
#pragma unroll 2
        for (int d4 = 0; d4 < quads; ++d4) {
          float4 q[kI], kk[4];
#pragma unroll
          for (int i = 0; i < kI; ++i) q[i] = *reinterpret_cast<const float4*>(sq + (y + 16 * i) * pitch + 4 * d4);
#pragma unroll
          for (int c = 0; c < 4; ++c) kk[c] = *reinterpret_cast<const float4*>(keys + (x + 16 * c) * pitch + 4 * d4);
#pragma unroll
          for (int i = 0; i < kI; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              s[i][c] = fma2(make_float2(q[i].x, q[i].y), make_float2(kk[c].x, kk[c].y), s[i][c]);
              s[i][c] = fma2(make_float2(q[i].z, q[i].w), make_float2(kk[c].z, kk[c].w), s[i][c]);
            }
        }
#pragma unroll
        for (int i = 0; i < kI; ++i) {
          const RowScale scale = s_scale[y + 16 * i];
          if (scale.y == 0.0f) continue;
          // the last slot that the row sees
          const int see = masked ? ctx - slot0 + a.by_group.quot(tile * kRows + y + 16 * i) : kSimtTile;
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (x + 16 * c <= see) {
              const float z = s[i][c].x + s[i][c].y;
              // the rest comes last: added to the whole of the lse it would be rounded away
              sum[c] = fmaf(exp2_fast(fmaf(z, p.scale_rest, fmaf(z, a.scale_log2, -scale.x))), scale.y, sum[c]);
            }
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        sum[c] += __shfl_xor_sync(kFull, sum[c], 16);
        if (lane < 16) s_sum[warp * kSimtTile + x + 16 * c] = sum[c];
      }
      __syncthreads();
      find_keys(j + 2);
      const int slot = slot0 + tid;
      if (tid < kSimtTile && tid < span - slot0) {
        float total = s_sum[tid];
#pragma unroll
        for (int i = 1; i < kWarps; ++i) total += s_sum[i * kSimtTile + tid];
        const long long at = (static_cast<long long>(w.b) * a.heads + w.h) * p.width + slot;
        if (slot < ctx && p.decay != 0.0f) total = fmaf(__ldcg(p.weight + at), p.decay, total);
        p.weight_out[at] = total;
      }
      __syncthreads();
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  }
}

template <typename T, int kI>
int launch_simt(const WeighParams& p, cudaStream_t stream) {
  auto kernel = weigh_kernel<T, kI>;
  const size_t smem = simt_smem(16 * kI, p.a.D);
  static std::atomic<int> sm_count[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return ASD_ERR_CUDA;
  if (dev < 0 || dev >= kMaxDevices) return ASD_ERR_DEVICE;
  int sms = sm_count[dev].load(std::memory_order_acquire);
  if (sms == 0) {
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(simt_smem(16 * kI, ASD_MAX_HEAD_DIM))) != cudaSuccess)
      return ASD_ERR_CUDA;
    sm_count[dev].store(sms, std::memory_order_release);
  }
  const size_t es = sizeof(T), four = 4 * es;
  const bool vec_q = p.a.D % 4 == 0 && rows_aligned(p.a.q, es, four, p.a.q_batch, p.a.q_token, p.a.q_head);
  const bool vec_k = p.a.D % 4 == 0 && rows_aligned(p.a.cache.k, es, four, p.a.cache.page_stride,
                                                    p.a.cache.token_stride, p.a.cache.head_stride);
  cudaLaunchAttribute attr;
  cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(2 * sms)), dim3(kSimtThreads), stream, &attr);
  cfg.dynamicSmemBytes = smem;
  if (cudaLaunchKernelEx(&cfg, kernel, p, vec_q, vec_k) != cudaSuccess) return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

template <typename T>
int launch_rows(const WeighParams& p, cudaStream_t stream) {
  const int tiles = (p.a.unit_rows + 79) / 80;
  const int i = p.a.unit_rows <= 16 ? 1 : ((p.a.unit_rows + tiles - 1) / tiles + 15) / 16;
  if constexpr (sizeof(T) == 4) {
    if (i == 2) return launch_simt<T, 2>(p, stream);
    if (i == 3) return launch_simt<T, 3>(p, stream);
    if (i == 5) return launch_simt<T, 5>(p, stream);
  }
  return i == 1 ? launch_simt<T, 1>(p, stream) : launch_simt<T, 4>(p, stream);
}

int check_weigh(const asd_kv_cache* cache, const asd_weigh& a) {
  const int rc = check_cache(cache);
  if (rc != ASD_OK) return rc;
  if (a.layer < 0 || a.layer >= cache->layers || a.T < 0 || a.rows < 0 || a.q_heads < 1 ||
      a.q_heads % cache->heads != 0 || a.width < 0 || (!a.path && a.rows != a.T))
    return ASD_ERR_SHAPE;
  // rows and tiles are counted in 32 bits
  const long long group = a.q_heads / cache->heads;
  if (a.rows * group > (1 << 28) || a.T * group > (1 << 28)) return ASD_ERR_SHAPE;
  const long long slots = static_cast<long long>(cache->table_width) * cache->page_size;
  const double tiles = static_cast<double>(slots < 0x7fffffffll ? slots : 0x7fffffffll) / kSimtTile + 1;
  if (tiles * static_cast<double>(a.rows * group / 16 + 1) * cache->heads * cache->B > 2147483647.0)
    return ASD_ERR_SHAPE;
  return ASD_OK;
}

}  // namespace

extern "C" int asd_kv_weigh(const asd_kv_cache* cache, const asd_weigh* args, asd_stream_t stream) {
  if (!args) return cache ? ASD_ERR_NULL : check_cache(cache);
  const asd_weigh& a = *args;
  const int rc = check_weigh(cache, a);
  if (rc != ASD_OK) return rc;
  const double scale = a.scale * 1.4426950408889634;
  const float scale_log2 = static_cast<float>(scale);
  if (!(scale_log2 - scale_log2 == 0.0f) || !(a.decay - a.decay == 0.0f) || a.decay < 0.0f) return ASD_ERR_CONTROL;
  if (cache->B == 0 || a.rows == 0) return ASD_OK;
  if (!a.q || !a.lse || !a.kv_len || !a.weight_out || (!a.weight && a.decay != 0.0f)) return ASD_ERR_NULL;
  const size_t es = store_bytes(cache->dtype);
  if (reinterpret_cast<uintptr_t>(a.q) % es != 0) return ASD_ERR_ALIGN;
  const void* const words[] = {a.lse, a.weight, a.weight_out, a.kv_len, a.new_len, a.path, a.status};
  for (const void* x : words)
    if (reinterpret_cast<uintptr_t>(x) % 4 != 0) return ASD_ERR_ALIGN;
  WeighParams p = {};
  p.a.cache = cache_view(cache, a.layer);
  if (p.a.cache.slots > a.width) p.a.cache.slots = a.width;
  p.a.q = static_cast<const char*>(a.q);
  p.a.q_batch = a.q_strides.batch;
  p.a.q_token = a.q_strides.token;
  p.a.q_head = a.q_strides.head;
  p.a.kv_len = a.kv_len;
  p.a.new_len = a.new_len;
  p.a.status = a.status;
  p.a.B = cache->B;
  p.a.T = a.rows;
  p.a.q_heads = a.q_heads;
  p.a.heads = cache->heads;
  p.a.group = a.q_heads / cache->heads;
  p.a.by_group = page_div(p.a.group);
  p.a.D = cache->head_dim;
  p.a.scale_log2 = scale_log2;
  p.a.unit_rows = p.a.group_rows = a.rows * p.a.group;
  p.a.row_tiles = 1;
  p.a.weighted = false;
  p.lse = a.lse;
  p.weight = a.weight;
  p.weight_out = a.weight_out;
  p.path = a.path;
  p.tokens = a.T;
  p.width = a.width;
  p.decay = a.decay;
  p.scale_rest = static_cast<float>(scale - scale_log2);
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (weigh_tc_takes(cache, p)) return launch_weigh_tc(cache, p, s);
  if (cache->dtype == ASD_F32) return launch_rows<float>(p, s);
  if (cache->dtype == ASD_BF16) return launch_rows<__nv_bfloat16>(p, s);
  return launch_rows<__half>(p, s);
}
