// libasd: appending to a paged cache, and moving a verified path next to the
// context (asd_kv_append, asd_kv_compact).
//
// Append. Every element of the new rows is read once and written once, so memory
// bounds it, or the launch where there are few tokens. A head's row is handled
// by a group of lanes that holds it in registers: the norm needs its sum of
// squares (shuffles within the group) and the rotation pairs elements half a
// rotation apart, so a lane takes a chunk and the chunk that turns with it.
#include <cuda_runtime.h>
#include <stdint.h>

#include "asd.h"
#include "asd_cache.cuh"
#include "asd_device.cuh"
#include "asd_launch.cuh"

namespace {

using namespace asd_detail;

constexpr int kAppendThreads = 256;

struct Rows {
  const char* data;
  long long batch, token, head;  // elements
};

struct AppendParams {
  CacheView cache;
  Rows k, v, q;
  char* q_out;
  const int32_t* kv_len;
  const int32_t* new_len;
  const int32_t* positions;
  const float* cos;
  const float* sin;
  const char* q_norm;
  const char* k_norm;
  int32_t* status;
  float eps;
  int B, T, q_heads, kv_heads, D;
  int rot, rot_positions, interleaved;
  int q_slices, kv_slices;  // groups of kHeads heads
  bool vec_tables;          // rows of cosines and sines start on 16 bytes and are read from multiples of 4
  long long items;          // B * T * (q_slices + 2 kv_slices)
};

// kVec consecutive elements, as they are stored.
template <typename T, int kVec> struct alignas(sizeof(T) * kVec) Chunk {
  T e[kVec];
};

// A chunk is read once by the kernel, past L1 and coherently.
template <typename T, int kVec>
__device__ __forceinline__ Chunk<T, kVec> load_chunk(const T* p) {
  Chunk<T, kVec> c;
  if constexpr (sizeof(c) == 16) {
    const uint4 w = __ldcg(reinterpret_cast<const uint4*>(p));
    memcpy(&c, &w, 16);
  } else if constexpr (sizeof(c) == 8) {
    const uint2 w = __ldcg(reinterpret_cast<const uint2*>(p));
    memcpy(&c, &w, 8);
  } else if constexpr (sizeof(c) == 4) {
    const unsigned w = __ldcg(reinterpret_cast<const unsigned*>(p));
    memcpy(&c, &w, 4);
  } else {
    const unsigned short w = __ldcg(reinterpret_cast<const unsigned short*>(p));
    memcpy(&c, &w, 2);
  }
  return c;
}

// Cosines or sines, by ordinary loads: the heads of a token share them.
template <int kCount>
__device__ __forceinline__ void load_table(const float* p, float* x, bool vec) {
  if (kCount % 4 == 0 && vec) {
#pragma unroll
    for (int e = 0; e < kCount; e += 4) {
      const float4 w = *reinterpret_cast<const float4*>(p + e);
      x[e] = w.x, x[e + 1] = w.y, x[e + 2] = w.z, x[e + 3] = w.w;
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < kCount; ++e) x[e] = p[e];
}

// kVec: elements per chunk. kPairs: chunk pairs per lane. kHeads: heads of one
// token that a group of lanes handles, their loads in flight together and their
// cosines and sines loaded once.
template <typename T, int kVec, int kPairs, int kHeads>
__global__ void __launch_bounds__(kAppendThreads)
    append_kernel(const __grid_constant__ AppendParams p, int lanes_log) {
  pdl_signal_dependents();
  const int lanes = 1 << lanes_log;
  const int lane = threadIdx.x & (lanes - 1);
  const long long item = static_cast<long long>(blockIdx.x) * (kAppendThreads >> lanes_log) + (threadIdx.x >> lanes_log);
  bool live = item < p.items;
  const int slices = p.q_slices + 2 * p.kv_slices;
  const long long token = live ? item / slices : 0;
  int slice = live ? static_cast<int>(item - token * slices) : 0;
  const int b = static_cast<int>(token / p.T), t = static_cast<int>(token - static_cast<long long>(b) * p.T);
  const int which = slice < p.q_slices ? 0 : slice < p.q_slices + p.kv_slices ? 1 : 2;  // q, k, v
  slice -= which == 0 ? 0 : which == 1 ? p.q_slices : p.q_slices + p.kv_slices;
  const Rows& rows = which == 0 ? p.q : which == 1 ? p.k : p.v;
  const int head0 = slice * kHeads;
  const int heads = (which == 0 ? p.q_heads : p.kv_heads) - head0;  // the slice's, at most kHeads
  const int chunks = p.D / kVec;
  // chunk pairs: those that turn together first, then the rest two by two
  const int turning = p.rot / (2 * kVec);
  const bool across = !p.interleaved || kVec == 1;  // the two chunks of a pair turn with one another
  const bool turns = which != 2 && p.rot > 0;

  pdl_wait_prerequisites();

  const int start = live ? __ldcg(p.kv_len + b) : 0;
  const int n = live && p.new_len ? __ldcg(p.new_len + b) : p.T;
  int pos = 0;
  if (live && p.positions && p.rot > 0) pos = __ldcg(p.positions + token);

  // the rows themselves do not wait for lengths and positions
  Chunk<T, kVec> x[kHeads][kPairs][2];
  int at[kPairs][2];
#pragma unroll
  for (int j = 0; j < kPairs; ++j) {
    const int q = lane + (j << lanes_log);
    if (across && !p.interleaved && q < turning) {
      at[j][0] = q;
      at[j][1] = q + turning;
    } else {
      at[j][0] = 2 * q;
      at[j][1] = 2 * q + 1;
    }
    if (at[j][0] >= chunks) at[j][0] = -1;
    if (at[j][1] >= chunks) at[j][1] = -1;
  }
  const T* src = reinterpret_cast<const T*>(rows.data) + b * rows.batch + t * rows.token;
#pragma unroll
  for (int h = 0; h < kHeads; ++h)
#pragma unroll
    for (int j = 0; j < kPairs; ++j)
#pragma unroll
      for (int s = 0; s < 2; ++s)
        if (live && h < heads && at[j][s] >= 0)
          x[h][j][s] = load_chunk<T, kVec>(src + (head0 + h) * rows.head + at[j][s] * kVec);
        else
          for (int e = 0; e < kVec; ++e) x[h][j][s].e[e] = Store<T>::narrow(0.0f);

  const bool bad_length = start < 0 || n < 0 || n > p.T || static_cast<long long>(start) + n > p.cache.slots;
  const bool reports = live && which == 1 && slice == 0 && lane == 0 && p.status;
  if (reports && t == 0 && bad_length) atomicOr(p.status + b, static_cast<int>(ASD_STATUS_LENGTH));
  live = live && !bad_length && t < n;
  if (!p.positions) pos = start + t;
  if (p.rot > 0 && live && static_cast<unsigned>(pos) >= static_cast<unsigned>(p.rot_positions)) {
    if (reports) atomicOr(p.status + b, static_cast<int>(ASD_STATUS_POSITION));
    live = false;
  }
  T* dst = nullptr;
  long long dst_head = p.D;
  if (live) {
    if (which == 0) {
      dst = reinterpret_cast<T*>(p.q_out) + (token * p.q_heads + head0) * p.D;
    } else {
      const long long off = slot_offset(p.cache, b, start + t);
      if (off < 0) {
        if (reports) atomicOr(p.status + b, static_cast<int>(ASD_STATUS_PAGE));
        live = false;
      } else {
        dst_head = p.cache.head_stride;
        dst = reinterpret_cast<T*>(which == 1 ? p.cache.k : p.cache.v) + off + head0 * dst_head;
      }
    }
  }

  const T* weight = reinterpret_cast<const T*>(which == 0 ? p.q_norm : which == 1 ? p.k_norm : nullptr);
  if (which == 2 || (!weight && !turns)) {  // moved as they are (the groups of a warp may differ: no shuffle below)
    if (live)
#pragma unroll
      for (int h = 0; h < kHeads; ++h)
#pragma unroll
        for (int j = 0; j < kPairs; ++j)
#pragma unroll
          for (int s = 0; s < 2; ++s)
            if (h < heads && at[j][s] >= 0)
              *reinterpret_cast<Chunk<T, kVec>*>(dst + h * dst_head + at[j][s] * kVec) = x[h][j][s];
  }
  const bool norm = weight != nullptr;
  const unsigned members = __ballot_sync(kFull, norm);  // whole groups
  float r[kHeads];
#pragma unroll
  for (int h = 0; h < kHeads; ++h) r[h] = 1.0f;
  if (norm) {
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < kPairs; ++j)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            const float f = Store<T>::widen(x[h][j][s].e[e]);
            sum = fmaf(f, f, sum);
          }
      for (int off = lanes >> 1; off > 0; off >>= 1) sum += __shfl_xor_sync(members, sum, off);
      r[h] = 1.0f / sqrtf(sum / static_cast<float>(p.D) + p.eps);
    }
  }
  if (!live || which == 2 || (!weight && !turns)) return;

  const float* cos = p.cos + static_cast<long long>(pos) * (p.rot / 2);
  const float* sin = p.sin + static_cast<long long>(pos) * (p.rot / 2);
#pragma unroll
  for (int j = 0; j < kPairs; ++j) {
    const int a = at[j][0], c = at[j][1];
    if (a < 0) continue;
    Chunk<T, kVec> wa = {}, wc = {};
    if (norm) {
      wa = *reinterpret_cast<const Chunk<T, kVec>*>(weight + a * kVec);
      if (c >= 0) wc = *reinterpret_cast<const Chunk<T, kVec>*>(weight + c * kVec);
    }
    // the chunk pair's cosines and sines: one for each element of the first chunk, or one for every two of both
    const bool whole = turns && across && lane + (j << lanes_log) < turning;
    float cs[kVec], sn[kVec];
    bool turn_a = false, turn_c = false;
    if (whole) {
      const int i0 = (lane + (j << lanes_log)) * kVec;
      load_table<kVec>(cos + i0, cs, p.vec_tables);
      load_table<kVec>(sin + i0, sn, p.vec_tables);
    } else if (turns && !across) {
      turn_a = a * kVec < p.rot;
      turn_c = c >= 0 && c * kVec < p.rot;
      constexpr int kHalf = kVec / 2 > 0 ? kVec / 2 : 1;
      // the second chunk's elements follow the first's; what lies past the rotation's end is not used
      if (turn_c) {
        load_table<kVec>(cos + a * kHalf, cs, p.vec_tables);
        load_table<kVec>(sin + a * kHalf, sn, p.vec_tables);
      } else if (turn_a) {
        load_table<kHalf>(cos + a * kHalf, cs, false);
        load_table<kHalf>(sin + a * kHalf, sn, false);
      }
    }
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      if (h >= heads) break;
      float u[kVec], w[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        u[e] = Store<T>::widen(x[h][j][0].e[e]);
        w[e] = Store<T>::widen(x[h][j][1].e[e]);
        if (norm) {
          u[e] = u[e] * r[h] * Store<T>::widen(wa.e[e]);
          w[e] = w[e] * r[h] * Store<T>::widen(wc.e[e]);
        }
      }
      if (whole) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const float f = u[e], g = w[e];
          u[e] = f * cs[e] - g * sn[e];
          w[e] = g * cs[e] + f * sn[e];
        }
      } else if (turn_a || turn_c) {
#pragma unroll
        for (int e = 0; e + 1 < kVec; e += 2) {
          const float f = u[e], g = u[e + 1];
          if (turn_a) {
            u[e] = f * cs[e / 2] - g * sn[e / 2];
            u[e + 1] = g * cs[e / 2] + f * sn[e / 2];
          }
          const float f2 = w[e], g2 = w[e + 1];
          if (turn_c) {
            w[e] = f2 * cs[kVec / 2 + e / 2] - g2 * sn[kVec / 2 + e / 2];
            w[e + 1] = g2 * cs[kVec / 2 + e / 2] + f2 * sn[kVec / 2 + e / 2];
          }
        }
      }
      Chunk<T, kVec> o;
#pragma unroll
      for (int e = 0; e < kVec; ++e) o.e[e] = Store<T>::narrow(u[e]);
      *reinterpret_cast<Chunk<T, kVec>*>(dst + h * dst_head + a * kVec) = o;
      if (c >= 0) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) o.e[e] = Store<T>::narrow(w[e]);
        *reinterpret_cast<Chunk<T, kVec>*>(dst + h * dst_head + c * kVec) = o;
      }
    }
  }
}

int div_up(int a, int b) { return (a + b - 1) / b; }

template <typename T, int kVec, int kPairs, int kHeads>
int launch_append(AppendParams p, cudaStream_t stream) {
  p.q_slices = div_up(p.q_heads, kHeads);
  p.kv_slices = div_up(p.kv_heads, kHeads);
  p.items = static_cast<long long>(p.B) * p.T * (p.q_slices + 2 * p.kv_slices);
  int lanes_log = 0;
  while (lanes_log < 5 && (kPairs << lanes_log) * 2 * kVec < p.D) ++lanes_log;
  const long long groups = kAppendThreads >> lanes_log;
  const long long grid = (p.items + groups - 1) / groups;
  if (grid > 0x7fffffffll) return ASD_ERR_SHAPE;
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(grid)), dim3(kAppendThreads), stream, &attr);
  if (cudaLaunchKernelEx(&cfg, append_kernel<T, kVec, kPairs, kHeads>, p, lanes_log) != cudaSuccess)
    return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

// Heads per group of lanes: four where that still gives every SM 1024 threads
// (loads of four heads in flight, their cosines and sines loaded once: 32744
// tokens of 56 heads of 128 in 357 us with one head, 196 with four), else one (a
// batch of 288 tokens is bound by latency).
template <typename T, int kVec>
int launch_vec(const AppendParams& p, cudaStream_t stream) {
  const long long threads = static_cast<long long>(p.B) * p.T * ((p.q_heads + 3) / 4 + 2 * ((p.kv_heads + 3) / 4)) *
                            ((p.D + 2 * kVec - 1) / (2 * kVec));
  if (threads >= 1024ll * 152) return launch_append<T, kVec, 1, 4>(p, stream);
  return launch_append<T, kVec, 1, 1>(p, stream);
}

// Elements per chunk: as many as 16 bytes hold, where rows start on such a
// boundary and the rotation's halves and ends fall between chunks; half as many
// for the 16-bit types (heads of 80 of which 40 turn); else one.
template <typename T>
int append_typed(AppendParams p, cudaStream_t stream) {
  // a row of the tables is rot / 2 floats, and chunks start at multiples of half a chunk or of one
  p.vec_tables = (p.rot / 2) % 4 == 0 && reinterpret_cast<uintptr_t>(p.cos) % 16 == 0 &&
                 reinterpret_cast<uintptr_t>(p.sin) % 16 == 0;
  auto fits = [&](int vec) {
    const size_t bytes = vec * sizeof(T);
    if (p.D % vec != 0 || (p.interleaved ? p.rot % vec : (p.rot / 2) % vec) != 0) return false;
    if (!rows_aligned(p.k.data, sizeof(T), bytes, p.k.batch, p.k.token, p.k.head) ||
        !rows_aligned(p.v.data, sizeof(T), bytes, p.v.batch, p.v.token, p.v.head) ||
        !rows_aligned(p.cache.k, sizeof(T), bytes, p.cache.page_stride, p.cache.token_stride, p.cache.head_stride) ||
        !rows_aligned(p.cache.v, sizeof(T), bytes, 0, 0, 0))
      return false;
    if (p.q_heads > 0 && (!rows_aligned(p.q.data, sizeof(T), bytes, p.q.batch, p.q.token, p.q.head) ||
                          !rows_aligned(p.q_out, sizeof(T), bytes, 0, 0, 0)))
      return false;
    return reinterpret_cast<uintptr_t>(p.q_norm) % bytes == 0 && reinterpret_cast<uintptr_t>(p.k_norm) % bytes == 0;
  };
  constexpr int kFullVec = 16 / static_cast<int>(sizeof(T));
  if (fits(kFullVec)) return launch_vec<T, kFullVec>(p, stream);
  if constexpr (sizeof(T) == 2) {
    if (fits(4)) return launch_vec<T, 4>(p, stream);
  }
  return launch_append<T, 1, 4, 1>(p, stream);
}

// ---------------------------------------------------------------- compaction
//
// A CTA moves one request's path in one layer, keys or values: its offsets
// first, checked and left in shared memory, then every thread walks the path
// with its own chunk of the token. Sources lie at or past their destinations and
// ascend, so what a thread stores for node i is never what it loads for a later
// node, and a batch of loads can be in flight at once.

constexpr int kCompactThreads = 128;
constexpr int kCompactBatch = 8;

struct CompactParams {
  CacheView cache;
  long long layer_stride;
  const int32_t* kv_len;
  const int32_t* path;
  const int32_t* path_len;
  int32_t* status;
  int B, P, heads, D;
};

template <typename W>
__global__ void __launch_bounds__(kCompactThreads) compact_kernel(const __grid_constant__ CompactParams p, int words) {
  __shared__ long long s_src[ASD_MAX_PATH], s_dst[ASD_MAX_PATH];
  pdl_signal_dependents();
  pdl_wait_prerequisites();
  const int b = blockIdx.x;
  const int start = __ldcg(p.kv_len + b);
  const int n = __ldcg(p.path_len + b);
  int bad = 0;
  if (start < 0 || n < 0 || n > p.P) bad = ASD_STATUS_LENGTH;
  for (int i = threadIdx.x; !bad && i < n; i += kCompactThreads) {
    const int32_t* path = p.path + static_cast<long long>(b) * p.P;
    const int node = __ldcg(path + i);
    if (node < i || (i > 0 && node <= __ldcg(path + i - 1))) {
      bad |= ASD_STATUS_PATH;
    } else if (static_cast<long long>(start) + node >= p.cache.slots) {
      bad |= ASD_STATUS_LENGTH;
    } else {
      const long long src = slot_offset(p.cache, b, start + node), dst = slot_offset(p.cache, b, start + i);
      if (src < 0 || dst < 0) bad |= ASD_STATUS_PAGE;
      s_src[i] = src;
      s_dst[i] = dst;
    }
  }
  const int why = __syncthreads_or(bad);
  if (why) {
    if (bad && p.status && blockIdx.y == 0 && blockIdx.z == 0) atomicOr(p.status + b, bad);
    return;
  }
  // elements of W: offsets and strides count elements of the cache's type
  const int per = p.D / words;  // of those in a word
  W* base = reinterpret_cast<W*>(blockIdx.z ? p.cache.v : p.cache.k);
  const long long layer = blockIdx.y * (p.layer_stride / per);
  const int all = p.heads * words;
  for (int c = threadIdx.x; c < all; c += kCompactThreads) {
    const int head = c / words;
    W* col = base + layer + head * (p.cache.head_stride / per) + (c - head * words);
    for (int i0 = 0; i0 < n; i0 += kCompactBatch) {
      W x[kCompactBatch];
#pragma unroll
      for (int i = 0; i < kCompactBatch; ++i)
        if (i0 + i < n && s_src[i0 + i] != s_dst[i0 + i]) x[i] = __ldcg(col + s_src[i0 + i] / per);
#pragma unroll
      for (int i = 0; i < kCompactBatch; ++i)
        if (i0 + i < n && s_src[i0 + i] != s_dst[i0 + i]) col[s_dst[i0 + i] / per] = x[i];
    }
  }
}

template <typename W>
int launch_compact(const CompactParams& p, int layers, int words, cudaStream_t stream) {
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg =
      pdl_config(dim3(static_cast<unsigned>(p.B), static_cast<unsigned>(layers), 2), dim3(kCompactThreads), stream,
                 &attr);
  if (cudaLaunchKernelEx(&cfg, compact_kernel<W>, p, words) != cudaSuccess) return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

}  // namespace

extern "C" {

int asd_kv_append(const asd_kv_cache* cache, const asd_append* args, asd_stream_t stream) {
  const int rc = check_cache(cache);
  if (rc != ASD_OK) return rc;
  if (!args) return ASD_ERR_NULL;
  const asd_append& a = *args;
  if (a.layer < 0 || a.layer >= cache->layers || a.T < 0 || a.q_heads < 0) return ASD_ERR_SHAPE;
  if ((a.cos == nullptr) != (a.sin == nullptr)) return ASD_ERR_NULL;
  if (a.cos ? (a.rot_dim < 2 || a.rot_dim % 2 != 0 || a.rot_dim > cache->head_dim || a.rot_positions < 0)
            : a.rot_dim != 0)
    return ASD_ERR_SHAPE;
  if (a.interleaved != 0 && a.interleaved != 1) return ASD_ERR_SHAPE;
  if (a.eps != a.eps || a.eps < 0.0f) return ASD_ERR_CONTROL;
  if (cache->B == 0 || a.T == 0) return ASD_OK;
  if (!a.k || !a.v || !a.kv_len || (a.q_heads > 0 && (!a.q || !a.q_out))) return ASD_ERR_NULL;
  const size_t es = store_bytes(cache->dtype);
  const void* const typed[] = {a.k, a.v, a.q, a.q_out, a.q_norm, a.k_norm};
  for (const void* x : typed)
    if (reinterpret_cast<uintptr_t>(x) % es != 0) return ASD_ERR_ALIGN;
  const void* const words[] = {a.kv_len, a.new_len, a.positions, a.cos, a.sin, a.status};
  for (const void* x : words)
    if (reinterpret_cast<uintptr_t>(x) % 4 != 0) return ASD_ERR_ALIGN;
  AppendParams p = {};
  p.cache = cache_view(cache, a.layer);
  p.k = {static_cast<const char*>(a.k), a.k_strides.batch, a.k_strides.token, a.k_strides.head};
  p.v = {static_cast<const char*>(a.v), a.v_strides.batch, a.v_strides.token, a.v_strides.head};
  p.q = {static_cast<const char*>(a.q), a.q_strides.batch, a.q_strides.token, a.q_strides.head};
  p.q_out = static_cast<char*>(a.q_out);
  p.kv_len = a.kv_len;
  p.new_len = a.new_len;
  p.positions = a.positions;
  p.cos = a.cos;
  p.sin = a.sin;
  p.q_norm = static_cast<const char*>(a.q_norm);
  p.k_norm = static_cast<const char*>(a.k_norm);
  p.status = a.status;
  p.eps = a.eps;
  p.B = cache->B;
  p.T = a.T;
  p.q_heads = a.q_heads;
  p.kv_heads = cache->heads;
  p.D = cache->head_dim;
  p.rot = a.rot_dim;
  p.rot_positions = a.rot_positions;
  p.interleaved = a.interleaved;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (cache->dtype == ASD_F32) return append_typed<float>(p, s);
  if (cache->dtype == ASD_BF16) return append_typed<__nv_bfloat16>(p, s);
  return append_typed<__half>(p, s);
}

int asd_kv_compact(const asd_kv_cache* cache, int P, const int32_t* kv_len, const int32_t* path,
                   const int32_t* path_len, int32_t* status, asd_stream_t stream) {
  const int rc = check_cache(cache);
  if (rc != ASD_OK) return rc;
  if (P < 0 || P > ASD_MAX_PATH || cache->layers > 65535) return ASD_ERR_SHAPE;
  if (cache->B == 0 || P == 0) return ASD_OK;
  if (!kv_len || !path || !path_len) return ASD_ERR_NULL;
  const void* const words[] = {kv_len, path, path_len, status};
  for (const void* x : words)
    if (reinterpret_cast<uintptr_t>(x) % 4 != 0) return ASD_ERR_ALIGN;
  CompactParams p = {};
  p.cache = cache_view(cache, 0);
  p.layer_stride = cache->layer_stride;
  p.kv_len = kv_len;
  p.path = path;
  p.path_len = path_len;
  p.status = status;
  p.B = cache->B;
  p.P = P;
  p.heads = cache->heads;
  p.D = cache->head_dim;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  // whole 16-byte words where every row starts on one, else elements
  const size_t es = store_bytes(cache->dtype);
  const int per = static_cast<int>(16 / es);
  if (p.D % per == 0 && cache->layer_stride % per == 0 &&
      rows_aligned(p.cache.k, es, 16, cache->page_stride, cache->token_stride, cache->head_stride) &&
      reinterpret_cast<uintptr_t>(p.cache.v) % 16 == 0)
    return launch_compact<uint4>(p, cache->layers, p.D / per, s);
  if (es == 4) return launch_compact<unsigned>(p, cache->layers, p.D, s);
  return launch_compact<unsigned short>(p, cache->layers, p.D, s);
}

}  // extern "C"
