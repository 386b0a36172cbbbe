// libasd: attention of a draft chain's or tree's tokens over a paged cache
// (asd_tree_attention): the entry point, and the kernel on the CUDA cores, for
// 32-bit caches, wide heads and layouts that the tensor-core kernel does not
// take.
//
// out = softmax(scale q k^T) v over the slots that each row sees, in one pass
// over the keys and values: per row the running maximum m and sum l of
// exp2(s - m), and the output's sum rescaled when m grows.
//
// A CTA of 256 threads has 16 kI query rows that share a key/value head against
// tiles of 64 slots. Thread (y, x) of 16 x 16 computes the scores of rows y + 16 i
// and slots x + 16 j, four elements of the head at a time from shared memory, and
// holds the output's columns 4 x + 64 c .. + 3 of its rows.
//
// What bounds it: fp32 multiply-adds from about 12 rows on (two for each element
// that crosses from memory), so rows are cut into as few and as equal tiles of at
// most 80 as hold them, and a tile's instance has no more than 15 to spare. Keys
// and values have a buffer each: 32-bit rows are copied straight into shared
// memory, values while the scores are computed and the next keys while the values
// are used. Two CTAs an SM hide each other's barriers (heads up to 128; registers
// are held to 128 for that). A warp copies a tile's rows whole, so that no copy
// divides, and the pieces of a split unit are merged with several in flight: eight
// trees of up to 17 tokens, 16 query heads on 4 of 96, up to 2900 cached tokens in
// fp32 take 72 to 76 us, FMA pipe 46 % and issue slots 42 % busy; with one thread
// index over the tile and one piece at a time, 6 us more. 16-bit heads of 256 have no
// background copies and one CTA an SM: 32 requests of 9 tokens and 8000 cached ones,
// 40 heads on 8, take 4.7 ms (floor 0.2).
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

constexpr int kSimtThreads = 256;
constexpr int kSimtTile = 64;

// Shared memory, in floats: rows of the head padded to a multiple of four and
// one more vector, so that a warp's sixteen rows start in different banks.
__host__ __device__ constexpr int simt_pitch(int dim) { return (dim + 3) / 4 * 4 + 4; }
constexpr int kScorePitch = kSimtTile + 4;
constexpr size_t simt_smem(int rows, int dim) {
  return sizeof(float) * (static_cast<size_t>(rows + 2 * kSimtTile) * simt_pitch(dim) + rows * kScorePitch) +
         2 * sizeof(long long) * kSimtTile;
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

// kI: query rows of a thread. kCols: the output's groups of 64 columns.
template <typename T, int kI, int kCols>
__global__ void __launch_bounds__(kSimtThreads, kCols <= 2 ? 2 : 1)
    attention_kernel(const __grid_constant__ AttnParams p, bool vec_q, bool vec_kv) {
  constexpr int kRows = 16 * kI;
  extern __shared__ __align__(16) float smem[];
  __shared__ AttnDeal deal;
  __shared__ int s_last;
  const int D = p.D, pitch = simt_pitch(D), quads = (D + 3) / 4;
  float* sq = smem;                        // [kRows][pitch]
  float* sk = sq + kRows * pitch;          // [kSimtTile][pitch]
  float* sv = sk + kSimtTile * pitch;      // [kSimtTile][pitch]
  float* sp = sv + kSimtTile * pitch;      // [kRows][kScorePitch]
  // [2][kSimtTile] the slots' offsets, of this tile and the next
  long long* s_off = reinterpret_cast<long long*>(sp + kRows * kScorePitch);
  const bool async = sizeof(T) == 4 && vec_kv;

  const int tid = threadIdx.x, x = tid & 15, y = tid >> 4, lane = tid & 31, warp = tid >> 5;
  pdl_signal_dependents();
  pdl_wait_prerequisites();
  attn_zero_rows<T>(p, tid, kSimtThreads);
  if (tid < 32) attn_deal<kSimtTile>(p, deal);
  __syncthreads();
  if (deal.begin == deal.end) return;

  AttnWalk<kSimtTile> w(p, deal);
  for (w.start(); w.more(); w.next()) {
    const int row0 = w.row0(), rows = w.rows();
    const int span = w.span();
    // With up to 16 rows a warp has two: where neither exists it only copies (a token of four heads 29 us, not 44).
    const bool idle = kI == 1 && 2 * warp >= rows;
    __syncthreads();  // the unit before is done with shared memory
    for (int r = warp; r < kRows; r += kSimtThreads / 32) {
      const int t = p.by_group.quot(row0 + r), g = row0 + r - t * p.group;
      const T* src = reinterpret_cast<const T*>(p.q) + w.b * p.q_batch + t * p.q_token + (w.h * p.group + g) * p.q_head;
      for (int d4 = lane; d4 < quads; d4 += 32) {
        float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (r < rows) load4(src + 4 * d4, vec_q, D - 4 * d4, f);
        *reinterpret_cast<float4*>(sq + r * pitch + 4 * d4) =
            make_float4(f[0] * p.scale_log2, f[1] * p.scale_log2, f[2] * p.scale_log2, f[3] * p.scale_log2);
      }
    }
    float m[kI], l[kI], o[kI][kCols][4];
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.0f;
#pragma unroll
      for (int c = 0; c < kCols; ++c) o[i][c][0] = o[i][c][1] = o[i][c][2] = o[i][c][3] = 0.0f;
    }

    // One tile's keys or values: copied in the background, or (types to widen, odd rows) by way of registers.
    auto load_tile = [&](float* dst, const char* base, const long long* off, int slots) {
      const T* src = reinterpret_cast<const T*>(base) + w.h * p.cache.head_stride;
      // a row a warp: no division, and a row's offset is one load for all lanes
#pragma unroll 4
      for (int s = warp; s < kSimtTile; s += kSimtThreads / 32) {
        const long long at = s < slots ? off[s] : -1;
        const bool has = at >= 0;
#pragma unroll
        for (int d0 = 0; d0 < kCols * 16; d0 += 32) {
          const int d4 = d0 + lane;
          if (d4 >= quads) break;
          if constexpr (sizeof(T) == 4) {
            if (async) {
              copy16(dst + s * pitch + 4 * d4, has ? src + at + 4 * d4 : src, has);
              continue;
            }
          }
          float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          if (has) load4(src + at + 4 * d4, vec_kv, D - 4 * d4, f);
          *reinterpret_cast<float4*>(dst + s * pitch + 4 * d4) = make_float4(f[0], f[1], f[2], f[3]);
        }
      }
      if (async) asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto look_up = [&](int j) {  // the slots' offsets of tile j
      if (tid >= kSimtTile) return;
      const int slot = j * kSimtTile + tid;
      if (slot >= span) return;
      const long long off = slot_offset(p.cache, w.b, slot);
      if (off < 0 && p.status) atomicOr(p.status + w.b, static_cast<int>(ASD_STATUS_PAGE));
      s_off[(j & 1) * kSimtTile + tid] = off;
    };
    const int j1 = w.j1();
    look_up(w.j0);
    __syncthreads();
    load_tile(sk, p.cache.k, s_off + (w.j0 & 1) * kSimtTile, span - w.j0 * kSimtTile);
    for (int j = w.j0; j < j1; ++j) {
      const int slot0 = j * kSimtTile;
      const long long* off = s_off + (j & 1) * kSimtTile;
      if (j + 1 < j1) look_up(j + 1);
      load_tile(sv, p.cache.v, off, span - slot0);
      if (async) asm volatile("cp.async.wait_group 1;" ::: "memory");  // the keys
      __syncthreads();
      float s[kI][4];
#pragma unroll
      for (int i = 0; i < kI; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.0f;
      for (int d4 = idle ? quads : 0; d4 < quads; ++d4) {
        float4 a[kI], kk[4];
#pragma unroll
        for (int i = 0; i < kI; ++i) a[i] = *reinterpret_cast<const float4*>(sq + (y + 16 * i) * pitch + 4 * d4);
#pragma unroll
        for (int c = 0; c < 4; ++c) kk[c] = *reinterpret_cast<const float4*>(sk + (x + 16 * c) * pitch + 4 * d4);
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            s[i][c] = fmaf(a[i].x, kk[c].x, s[i][c]);
            s[i][c] = fmaf(a[i].y, kk[c].y, s[i][c]);
            s[i][c] = fmaf(a[i].z, kk[c].z, s[i][c]);
            s[i][c] = fmaf(a[i].w, kk[c].w, s[i][c]);
          }
      }
      // the tile's mask where it reaches past the context (or the span)
      const bool masked = slot0 > w.r.ctx - kSimtTile;  // slot0 + kSimtTile may be 2^31
#pragma unroll
      for (int i = 0; i < kI; ++i) {
        if (idle) break;
        const int r = y + 16 * i;
        uint32_t lo = ~0u, hi = ~0u;
        if (masked) {
          lo = hi = 0;
          if (r < rows) {
            const int t = p.by_group.quot(row0 + r);
            lo = attn_sees(p, w.r, w.b, t, slot0);
            hi = attn_sees(p, w.r, w.b, t, slot0 + 32);
          }
          if (!((lo >> x) & 1u)) s[i][0] = -INFINITY;
          if (!((lo >> (x + 16)) & 1u)) s[i][1] = -INFINITY;
          if (!((hi >> x) & 1u)) s[i][2] = -INFINITY;
          if (!((hi >> (x + 16)) & 1u)) s[i][3] = -INFINITY;
        }
        float top = fmax_nan(fmax_nan(s[i][0], s[i][1]), fmax_nan(s[i][2], s[i][3]));
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) top = fmax_nan(top, __shfl_xor_sync(kFull, top, off));
        const float m_new = fmax_nan(m[i], top);
        const float ref = m_new == -INFINITY ? 0.0f : m_new;  // nothing seen yet: every weight is exp2(-inf) = 0
        const float fade = exp2f(m[i] - ref);
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float e = exp2f(s[i][c] - ref);
          sum += e;
          // -0 stands for a slot that the row does not see; the weight of one that it sees may be too small and +0
          sp[r * kScorePitch + x + 16 * c] = (((c & 2 ? hi : lo) >> (x + 16 * (c & 1))) & 1u) ? e : -0.0f;
        }
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor_sync(kFull, sum, off);
        l[i] = l[i] * fade + sum;
        m[i] = m_new;
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][c][e] *= fade;
      }
      __syncthreads();  // the scores are written, the keys read
      if (j + 1 < j1) {
        load_tile(sk, p.cache.k, s_off + ((j + 1) & 1) * kSimtTile, span - slot0 - kSimtTile);
        if (async) asm volatile("cp.async.wait_group 1;" ::: "memory");  // the values
      } else if (async) {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      __syncthreads();
      for (int s4 = idle ? kSimtTile : 0; s4 < kSimtTile; s4 += 4) {
        float4 a[kI];
#pragma unroll
        for (int i = 0; i < kI; ++i) a[i] = *reinterpret_cast<const float4*>(sp + (y + 16 * i) * kScorePitch + s4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float4 v[kCols];
#pragma unroll
          for (int c = 0; c < kCols; ++c)
            if (4 * x + 64 * c < D) v[c] = *reinterpret_cast<const float4*>(sv + (s4 + e) * pitch + 4 * x + 64 * c);
#pragma unroll
          for (int i = 0; i < kI; ++i) {
            const float f = e == 0 ? a[i].x : e == 1 ? a[i].y : e == 2 ? a[i].z : a[i].w;
            // what a row does not see does not reach it: 0 * NaN would
            if (masked && __float_as_uint(f) == 0x80000000u) continue;
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
              o[i][c][0] = fmaf(f, v[c].x, o[i][c][0]);
              o[i][c][1] = fmaf(f, v[c].y, o[i][c][1]);
              o[i][c][2] = fmaf(f, v[c].z, o[i][c][2]);
              o[i][c][3] = fmaf(f, v[c].w, o[i][c][3]);
            }
          }
        }
      }
      __syncthreads();  // the values have been read
    }

    // the rows' results, or this CTA's piece of them
    auto write_row = [&](int r, const float (&acc)[kCols][4], float ml, float sum) {
      const int t = p.by_group.quot(row0 + r), g = row0 + r - t * p.group;
      const long long at = (static_cast<long long>(w.b) * p.T + t) * p.q_heads + w.h * p.group + g;
      const float inv = sum > 0.0f ? 1.0f / sum : sum;  // a row that sees nothing: 0; a NaN stays one
      T* dst = reinterpret_cast<T*>(p.out) + at * D;
#pragma unroll
      for (int c = 0; c < kCols; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (4 * x + 64 * c + e < D) dst[4 * x + 64 * c + e] = Store<T>::narrow(sum == 0.0f ? 0.0f : acc[c][e] * inv);
      if (x == 0 && p.lse) p.lse[at] = sum == 0.0f ? -INFINITY : 0.6931471805599453f * (ml + log2f(sum));
    };
    if (w.whole()) {
#pragma unroll
      for (int i = 0; i < kI; ++i)
        if (y + 16 * i < rows) write_row(y + 16 * i, o[i], m[i], l[i]);
      continue;
    }
    const int slot = w.piece();
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      const int r = y + 16 * i;
      if (r >= rows) continue;
      const long long at = static_cast<long long>(slot) * kRows + r;
      if (x == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at) = make_float2(m[i], l[i]);
#pragma unroll
      for (int c = 0; c < kCols; ++c)
        if (4 * x + 64 * c < D)
          *reinterpret_cast<float4*>(p.part_o + at * (quads * 4) + 4 * x + 64 * c) =
              make_float4(o[i][c][0], o[i][c][1], o[i][c][2], o[i][c][3]);
    }
    __threadfence();
    __syncthreads();
    const int c0 = w.first_cta(), c1 = w.last_cta();
    if (tid == 0) {
      const unsigned pieces = static_cast<unsigned>(c1 - c0 + 1);
      const bool last = atomicAdd(p.counters + c0, 1u) == pieces - 1;
      if (last) p.counters[c0] = 0u;  // zero again for the next call
      s_last = last;
    }
    __syncthreads();
    if (!s_last) continue;
    __threadfence();
    // the pieces one after the other, all rows' loads of a few of them in flight
    auto piece_row = [&](int c, int i) {
      return static_cast<long long>(c == c0 ? 2 * c + 1 : 2 * c) * kRows + min(y + 16 * i, rows - 1);
    };
#pragma unroll
    for (int i = 0; i < kI; ++i) m[i] = -INFINITY;
#pragma unroll 4
    for (int c = c0; c <= c1; ++c)
#pragma unroll
      for (int i = 0; i < kI; ++i) m[i] = fmax_nan(m[i], __ldcg(p.part_ml + 2 * piece_row(c, i)));
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      l[i] = 0.0f;
#pragma unroll
      for (int k = 0; k < kCols; ++k) o[i][k][0] = o[i][k][1] = o[i][k][2] = o[i][k][3] = 0.0f;
    }
#pragma unroll 2
    for (int c = c0; c <= c1; ++c)
#pragma unroll
      for (int i = 0; i < kI; ++i) {
        const long long at = piece_row(c, i);
        const float2 ml = __ldcg(reinterpret_cast<const float2*>(p.part_ml + 2 * at));
        const float f = exp2f(ml.x - (m[i] == -INFINITY ? 0.0f : m[i]));
        l[i] += f * ml.y;
#pragma unroll
        for (int k = 0; k < kCols; ++k) {
          const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * (quads * 4) +
                                                                  min(4 * x + 64 * k, 4 * quads - 4)));
          o[i][k][0] += f * v.x, o[i][k][1] += f * v.y, o[i][k][2] += f * v.z, o[i][k][3] += f * v.w;
        }
      }
#pragma unroll
    for (int i = 0; i < kI; ++i)
      if (y + 16 * i < rows) write_row(y + 16 * i, o[i], m[i], l[i]);
  }
}

// ---------------------------------------------------------------- host side

constexpr int kMaxDevices = 64;
constexpr size_t kSmemPerSm = 233472;

template <typename T, int kI, int kCols>
int launch_simt(AttnParams p, char* workspace, cudaStream_t stream) {
  constexpr int kRows = 16 * kI;
  auto kernel = attention_kernel<T, kI, kCols>;
  // CTAs that an SM's registers hold, and SMs (0: not asked yet)
  static std::atomic<int> by_registers[kMaxDevices], sm_count[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return ASD_ERR_CUDA;
  if (dev < 0 || dev >= kMaxDevices) return ASD_ERR_DEVICE;
  int per = by_registers[dev].load(std::memory_order_acquire);
  if (per == 0) {
    int sms = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(simt_smem(kRows, kCols * 64))) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, kSimtThreads, 0) != cudaSuccess || per < 1)
      return ASD_ERR_CUDA;
    sm_count[dev].store(sms, std::memory_order_relaxed);
    by_registers[dev].store(per, std::memory_order_release);
  }
  const size_t smem = simt_smem(kRows, p.D);
  const int by_smem = static_cast<int>(kSmemPerSm / (smem + 2048));  // the CTA's static part and the system's KB
  per = by_smem < per ? by_smem : per;
  int ctas = sm_count[dev].load(std::memory_order_relaxed) * (per < 1 ? 1 : per);
  ctas = ctas < kAttnMaxCtas ? ctas : kAttnMaxCtas;
  const AttnLayout l = attn_layout(kAttnMaxCtas, kRows, simt_pitch(p.D) - 4);
  p.counters = reinterpret_cast<unsigned*>(workspace + l.counters);
  p.part_ml = reinterpret_cast<float*>(workspace + l.ml);
  p.part_o = reinterpret_cast<float*>(workspace + l.o);
  const int rows = p.T * p.group;
  p.row_tiles = (rows + kRows - 1) / kRows;
  p.unit_rows = p.group_rows = kRows;
  p.weighted = false;
  const size_t es = sizeof(T), four = 4 * es;
  const bool vec_q = p.D % 4 == 0 && rows_aligned(p.q, es, four, p.q_batch, p.q_token, p.q_head);
  const bool vec_kv = p.D % 4 == 0 &&
                      rows_aligned(p.cache.k, es, four, p.cache.page_stride, p.cache.token_stride,
                                   p.cache.head_stride) &&
                      reinterpret_cast<uintptr_t>(p.cache.v) % four == 0;
  cudaLaunchAttribute attr;
  cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(ctas)), dim3(kSimtThreads), stream, &attr);
  cfg.dynamicSmemBytes = smem;
  if (cudaLaunchKernelEx(&cfg, kernel, p, vec_q, vec_kv) != cudaSuccess) return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

// Rows of a thread: the fewest tiles of at most 80 rows, as equal as they go.
// 16-bit types (what the tensor cores do not take) have two instances. Heads wider
// than 128 leave shared memory for 64 rows.
int simt_i(long long rows, int dtype, int dim) {
  const int most = dim > 128 ? 4 : 5;
  if (dtype != ASD_F32 || dim > 128) return rows > 16 ? 4 : 1;
  const long long tiles = (rows + 16 * most - 1) / (16 * most);
  const long long i = (rows + 16 * tiles - 1) / (16 * tiles);
  return i < 1 ? 1 : static_cast<int>(i);
}

template <typename T, int kI>
int launch_cols(const AttnParams& p, char* workspace, cudaStream_t stream) {
  if (p.D <= 64) return launch_simt<T, kI, 1>(p, workspace, stream);
  if (p.D <= 128) return launch_simt<T, kI, 2>(p, workspace, stream);
  if constexpr (kI == 1 || kI == 4) return launch_simt<T, kI, 4>(p, workspace, stream);
  return ASD_ERR_SHAPE;
}

template <typename T>
int launch_rows(const AttnParams& p, int dtype, char* workspace, cudaStream_t stream) {
  const int i = simt_i(static_cast<long long>(p.T) * p.group, dtype, p.D);
  if constexpr (sizeof(T) == 4) {
    if (i == 2) return launch_cols<T, 2>(p, workspace, stream);
    if (i == 3) return launch_cols<T, 3>(p, workspace, stream);
    if (i == 5) return launch_cols<T, 5>(p, workspace, stream);
  }
  return i == 4 ? launch_cols<T, 4>(p, workspace, stream) : launch_cols<T, 1>(p, workspace, stream);
}

int check_attention(const asd_kv_cache* cache, int T, int q_heads) {
  const int rc = check_cache(cache);
  if (rc != ASD_OK) return rc;
  if (T < 0 || q_heads < 1 || q_heads % cache->heads != 0) return ASD_ERR_SHAPE;
  // rows and tiles are counted in 32 bits
  const long long rows = static_cast<long long>(T) * (q_heads / cache->heads);
  if (rows > (1 << 28)) return ASD_ERR_SHAPE;
  const long long slots = static_cast<long long>(cache->table_width) * cache->page_size;
  const double tiles = static_cast<double>(slots < 0x7fffffffll ? slots : 0x7fffffffll) / kSimtTile + 1;
  if (tiles * static_cast<double>(rows / 16 + 1) * cache->heads * cache->B > 2147483647.0)
    return ASD_ERR_SHAPE;
  return ASD_OK;
}

size_t attention_bytes(const asd_kv_cache* cache, int T, int q_heads) {
  const long long rows = static_cast<long long>(T) * (q_heads / cache->heads);
  // the tile of a smaller T may have more rows
  const int tile = rows <= 16 ? 16 : rows <= 64 ? 64 : 80;
  const size_t simt = attn_layout(kAttnMaxCtas, tile, simt_pitch(cache->head_dim) - 4).total;
  const size_t tc = attention_tc_bytes(cache, T, q_heads);
  return simt > tc ? simt : tc;
}

}  // namespace

extern "C" {

int asd_attention_workspace_size(const asd_kv_cache* cache, int T, int q_heads, size_t* bytes) {
  if (!bytes) return ASD_ERR_NULL;
  const int rc = check_attention(cache, T, q_heads);
  if (rc != ASD_OK) return rc;
  *bytes = attention_bytes(cache, T, q_heads);
  return ASD_OK;
}

int asd_tree_attention(const asd_kv_cache* cache, const asd_attention* args, asd_stream_t stream) {
  if (!args) return cache ? ASD_ERR_NULL : check_cache(cache);
  const asd_attention& a = *args;
  const int rc = check_attention(cache, a.T, a.q_heads);
  if (rc != ASD_OK) return rc;
  if (a.layer < 0 || a.layer >= cache->layers) return ASD_ERR_SHAPE;
  const float scale_log2 = a.scale * 1.4426950408889634f;
  if (!(scale_log2 - scale_log2 == 0.0f)) return ASD_ERR_CONTROL;  // infinite or NaN
  if (cache->B == 0 || a.T == 0) return ASD_OK;
  if (!a.q || !a.kv_len || !a.out || !a.workspace) return ASD_ERR_NULL;
  const size_t es = store_bytes(cache->dtype);
  if (reinterpret_cast<uintptr_t>(a.q) % es != 0 || reinterpret_cast<uintptr_t>(a.out) % es != 0) return ASD_ERR_ALIGN;
  const void* const words[] = {a.kv_len, a.new_len, a.tree_mask, a.lse, a.status};
  for (const void* x : words)
    if (reinterpret_cast<uintptr_t>(x) % 4 != 0) return ASD_ERR_ALIGN;
  if (a.workspace_bytes < attention_bytes(cache, a.T, a.q_heads)) return ASD_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(a.workspace) % 16 != 0) return ASD_ERR_ALIGN;
  AttnParams p = {};
  p.cache = cache_view(cache, a.layer);
  p.q = static_cast<const char*>(a.q);
  p.q_batch = a.q_strides.batch;
  p.q_token = a.q_strides.token;
  p.q_head = a.q_strides.head;
  p.out = static_cast<char*>(a.out);
  p.lse = a.lse;
  p.kv_len = a.kv_len;
  p.new_len = a.new_len;
  p.mask = a.tree_mask;
  p.mask_words = (a.T + 31) / 32;
  p.status = a.status;
  p.error = static_cast<unsigned*>(a.workspace);
  p.B = cache->B;
  p.T = a.T;
  p.q_heads = a.q_heads;
  p.heads = cache->heads;
  p.group = a.q_heads / cache->heads;
  p.by_group = page_div(p.group);
  p.D = cache->head_dim;
  p.scale_log2 = scale_log2;
  char* ws = static_cast<char*>(a.workspace);
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (attention_tc_takes(cache, p)) return launch_attention_tc(cache, p, ws, s);
  if (cache->dtype == ASD_F32) return launch_rows<float>(p, cache->dtype, ws, s);
  if (cache->dtype == ASD_BF16) return launch_rows<__nv_bfloat16>(p, cache->dtype, ws, s);
  return launch_rows<__half>(p, cache->dtype, ws, s);
}

}  // extern "C"
