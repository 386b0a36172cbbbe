// libasd: the attention weight that each cached slot receives (asd_kv_weigh): the
// entry point, and the kernel on the CUDA cores, for 32-bit caches, wide heads and
// layouts that the tensor-core kernel does not take.
//
// w[s] = sum over rows of exp(scale q k_s - lse): the rows' softmax is known by its
// log-sum-exp, so one pass over the keys does, and every slot's sum stands alone.
//
// A CTA of 256 threads has 16 kI query rows that share a key/value head against
// tiles of 64 slots. Thread (y, x) of 16 x 16 computes the scores of rows y + 16 i
// and slots x + 16 j, four elements of the head at a time from shared memory, adds up
// its rows' weights, and the sixteen threads of a slot are added up at the end of the
// tile, always in the same order.
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
// queries, keys twice where that fits, row scales, sums of the warps
constexpr size_t simt_smem(int rows, int dim) {
  return sizeof(float) * static_cast<size_t>(rows + kSimtTile) * simt_pitch(dim) + sizeof(RowScale) * rows +
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

// kI: query rows of a thread.
template <typename T, int kI>
__global__ void __launch_bounds__(kSimtThreads)
    weigh_kernel(const __grid_constant__ WeighParams p, bool vec_q, bool vec_k) {
  constexpr int kRows = 16 * kI;
  extern __shared__ __align__(16) float smem[];
  __shared__ AttnDeal deal;
  const AttnParams a = weigh_deal_params(p);
  const int D = a.D, pitch = simt_pitch(D), quads = (D + 3) / 4;
  float* sq = smem;                                                       // [kRows][pitch]
  float* sk = sq + kRows * pitch;                                         // [kSimtTile][pitch]
  RowScale* s_scale = reinterpret_cast<RowScale*>(sk + kSimtTile * pitch);  // [kRows]
  float* s_sum = reinterpret_cast<float*>(s_scale + kRows);               // [warps][kSimtTile]

  const int tid = threadIdx.x, x = tid & 15, y = tid >> 4, lane = tid & 31, warp = tid >> 5;
  pdl_signal_dependents();
  pdl_wait_prerequisites();
  if (tid < 32) attn_deal<kSimtTile>(a, deal);
  __syncthreads();
  if (deal.begin == deal.end) return;

  AttnWalk<kSimtTile> w(a, deal);
  for (w.start(); w.more(); w.next()) {
    const int rows = w.rows(), span = w.span(), ctx = w.r.ctx;
    const int tiles = (rows + kRows - 1) / kRows;
    auto load_rows = [&](int row0) {
      for (int r = warp; r < kRows; r += kSimtThreads / 32) {
        const int row = row0 + r, t = row < rows ? a.by_group.quot(row) : 0;
        const int head = w.h * a.group + row - t * a.group;
        const int token = row < rows ? weigh_token(p, w.b, t) : -1;
        const T* src = reinterpret_cast<const T*>(a.q) + w.b * a.q_batch + token * a.q_token + head * a.q_head;
        for (int d4 = lane; d4 < quads; d4 += 32) {
          float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          if (token >= 0) load4(src + 4 * d4, vec_q, D - 4 * d4, f);
          *reinterpret_cast<float4*>(sq + r * pitch + 4 * d4) =
              make_float4(f[0] * a.scale_log2, f[1] * a.scale_log2, f[2] * a.scale_log2, f[3] * a.scale_log2);
        }
        if (lane == 0) s_scale[r] = row_scale(p, w.b, token, head);
      }
    };
    bool loaded = false;
    const int j1 = w.j1();
    for (int j = w.j0; j < j1; ++j) {
      const int slot0 = j * kSimtTile;
      __syncthreads();  // the tile before is done with shared memory
      for (int s = warp; s < kSimtTile; s += kSimtThreads / 32) {
        long long at = -1;
        if (s < span - slot0) {
          at = slot_offset(a.cache, w.b, slot0 + s);
          if (at < 0 && lane == 0 && a.status) atomicOr(a.status + w.b, static_cast<int>(ASD_STATUS_PAGE));
        }
        const T* src = reinterpret_cast<const T*>(a.cache.k) + w.h * a.cache.head_stride + at;
        for (int d4 = lane; d4 < quads; d4 += 32) {
          float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          if (at >= 0) load4(src + 4 * d4, vec_k, D - 4 * d4, f);
          *reinterpret_cast<float4*>(sk + s * pitch + 4 * d4) = make_float4(f[0], f[1], f[2], f[3]);
        }
      }
      const bool masked = slot0 > ctx - kSimtTile;  // slot0 + kSimtTile may be 2^31
      float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      for (int tile = 0; tile < tiles; ++tile) {
        if (!loaded || tiles > 1) {
          if (tile > 0) __syncthreads();
          load_rows(tile * kRows);
          loaded = true;
        }
        __syncthreads();
        float s[kI][4];
#pragma unroll
        for (int i = 0; i < kI; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.0f;
        for (int d4 = 0; d4 < quads; ++d4) {
          float4 q[kI], kk[4];
#pragma unroll
          for (int i = 0; i < kI; ++i) q[i] = *reinterpret_cast<const float4*>(sq + (y + 16 * i) * pitch + 4 * d4);
#pragma unroll
          for (int c = 0; c < 4; ++c) kk[c] = *reinterpret_cast<const float4*>(sk + (x + 16 * c) * pitch + 4 * d4);
#pragma unroll
          for (int i = 0; i < kI; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              s[i][c] = fmaf(q[i].x, kk[c].x, s[i][c]);
              s[i][c] = fmaf(q[i].y, kk[c].y, s[i][c]);
              s[i][c] = fmaf(q[i].z, kk[c].z, s[i][c]);
              s[i][c] = fmaf(q[i].w, kk[c].w, s[i][c]);
            }
        }
#pragma unroll
        for (int i = 0; i < kI; ++i) {
          const RowScale scale = s_scale[y + 16 * i];
          const int row = tile * kRows + y + 16 * i;
          if (scale.y == 0.0f) continue;
          // the row's last slot
          const int see = masked ? ctx - slot0 + a.by_group.quot(row) : kSimtTile;
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (x + 16 * c <= see) sum[c] = fmaf(exp2f(s[i][c] - scale.x), scale.y, sum[c]);
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        sum[c] += __shfl_xor_sync(kFull, sum[c], 16);
        if (lane < 16) s_sum[warp * kSimtTile + x + 16 * c] = sum[c];
      }
      __syncthreads();
      const int slot = slot0 + tid;
      if (tid < kSimtTile && tid < span - slot0) {
        float total = s_sum[tid];
#pragma unroll
        for (int i = 1; i < kSimtThreads / 32; ++i) total += s_sum[i * kSimtTile + tid];
        const long long at = (static_cast<long long>(w.b) * a.heads + w.h) * p.width + slot;
        if (slot < ctx && p.decay != 0.0f) total = fmaf(__ldcg(p.weight + at), p.decay, total);
        p.weight_out[at] = total;
      }
    }
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
  return p.a.unit_rows <= 16 ? launch_simt<T, 1>(p, stream) : launch_simt<T, 4>(p, stream);
}

int check_weigh(const asd_kv_cache* cache, const asd_weigh& a) {
  const int rc = check_cache(cache);
  if (rc != ASD_OK) return rc;
  if (a.layer < 0 || a.layer >= cache->layers || a.T < 0 || a.rows < 0 || a.q_heads < 1 ||
      a.q_heads % cache->heads != 0 || a.width < 0 || a.reserved != 0 || (!a.path && a.rows != a.T))
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
  const float scale_log2 = a.scale * 1.4426950408889634f;
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
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (weigh_tc_takes(cache, p)) return launch_weigh_tc(cache, p, s);
  if (cache->dtype == ASD_F32) return launch_rows<float>(p, s);
  if (cache->dtype == ASD_BF16) return launch_rows<__nv_bfloat16>(p, s);
  return launch_rows<__half>(p, s);
}
