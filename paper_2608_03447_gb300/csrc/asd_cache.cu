// libasd: appending to a paged cache, and moving a verified path next to the
// context (asd_kv_append, asd_kv_compact).
//
// Append. Every element of the new rows is read once and written once, so memory
// bounds it, or the launch where there are few tokens. A head's row is handled
// by a group of lanes that holds it in registers: the norm needs its sum of
// squares (shuffles within the group) and the rotation pairs elements half a
// rotation apart, so a lane takes a chunk and the chunk that turns with it. Norm
// weight, cosine and sine of an element make two factors, the same for every head
// of the token: an output is r (x p + z q), z the element that x turns with, r
// the head's 1 / sqrt(mean + eps).
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

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
  float eps, inv_dim;
  int B, T, q_heads, kv_heads, D;
  int rot, rot_positions, interleaved;
  int q_slices, kv_slices;  // groups of kHeads heads
  bool vec_tables;          // rows of cosines and sines start on 16 bytes and are read from multiples of 4
  int items;                // B * T * (q_slices + 2 kv_slices)
  PageDiv by_slices, by_tokens;
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

// A chunk's elements in fp32, two to a register pair.
template <int kVec> struct Wide {
  static constexpr int kPairs = (kVec + 1) / 2;
  float2 e[kPairs];  // a single element: the second is 0
};
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(r)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
  return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(r)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)),
        "l"(*reinterpret_cast<unsigned long long*>(&c)));
  return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 widen2(const float* x) { return make_float2(x[0], x[1]); }
__device__ __forceinline__ float2 widen2(const __nv_bfloat16* x) {
  return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(x));
}
__device__ __forceinline__ float2 widen2(const __half* x) {
  return __half22float2(*reinterpret_cast<const __half2*>(x));
}
__device__ __forceinline__ void narrow2(float* x, float2 v) { x[0] = v.x, x[1] = v.y; }
__device__ __forceinline__ void narrow2(__nv_bfloat16* x, float2 v) {
  *reinterpret_cast<__nv_bfloat162*>(x) = __float22bfloat162_rn(v);
}
__device__ __forceinline__ void narrow2(__half* x, float2 v) { *reinterpret_cast<__half2*>(x) = __float22half2_rn(v); }

template <typename T, int kVec>
__device__ __forceinline__ Wide<kVec> widen(const Chunk<T, kVec>& c) {
  Wide<kVec> w;
  if constexpr (kVec == 1) {
    w.e[0] = make_float2(Store<T>::widen(c.e[0]), 0.0f);
  } else {
#pragma unroll
    for (int i = 0; i < kVec / 2; ++i) w.e[i] = widen2(c.e + 2 * i);
  }
  return w;
}

// Which heads of which token an item is: head0 .. of the queries (which = 0), keys
// or values.
struct AppendItem {
  int b, t, token, which, slice, head0, heads;
  const char* src;  // of head0
};
template <typename T, int kHeads>
__device__ __forceinline__ AppendItem append_item(const AppendParams& p, int item) {
  AppendItem i;
  i.token = p.by_slices.quot(item);
  i.slice = item - i.token * p.by_slices.size;
  i.b = p.by_tokens.quot(i.token);
  i.t = i.token - i.b * p.T;
  i.which = i.slice < p.q_slices ? 0 : i.slice < p.q_slices + p.kv_slices ? 1 : 2;
  i.slice -= i.which == 0 ? 0 : i.which == 1 ? p.q_slices : p.q_slices + p.kv_slices;
  const Rows& rows = i.which == 0 ? p.q : i.which == 1 ? p.k : p.v;
  i.head0 = i.slice * kHeads;
  i.heads = (i.which == 0 ? p.q_heads : p.kv_heads) - i.head0;  // the slice's, at most kHeads
  i.src = rows.data + (i.b * rows.batch + i.t * rows.token + i.head0 * rows.head) * static_cast<long long>(sizeof(T));
  return i;
}

// kVec: elements per chunk. kPairs: chunk pairs per lane. kHeads: heads of one
// token that a group of lanes handles, their factors made once. kStages: 0: an
// item per group of lanes, loaded into registers. Else a group works through items
// one after the other, the next kStages - 1 on their way into shared memory: each
// thread copies and reads its own chunks, so nothing has to meet.
template <typename T, int kVec, int kPairs, int kHeads, int kStages>
__global__ void __launch_bounds__(kAppendThreads, kStages > 0 ? 3 : 2)
    append_kernel(const __grid_constant__ AppendParams p, int lanes_log) {
  static_assert(kStages == 0 || kPairs == 1, "a stage holds one chunk pair a lane and head");
  constexpr int kWide = Wide<kVec>::kPairs;
  constexpr int kChunk = static_cast<int>(sizeof(Chunk<T, kVec>));
  extern __shared__ __align__(16) unsigned char append_smem[];
  pdl_signal_dependents();
  const int lanes = 1 << lanes_log;
  const int lane = threadIdx.x & (lanes - 1);
  const int groups = kAppendThreads >> lanes_log, group = threadIdx.x >> lanes_log;
  const int stride = static_cast<int>(gridDim.x) * groups;
  const int chunks = p.D / kVec;
  // chunk pairs: those that turn together first, then the rest two by two
  const int turning = p.rot / (2 * kVec);
  const bool across = !p.interleaved || kVec == 1;  // the two chunks of a pair turn with one another
  int at[kPairs][2];
#pragma unroll
  for (int j = 0; j < kPairs; ++j) {
    const int q = lane + (j << lanes_log);
    const bool apart = !p.interleaved && q < turning;
    at[j][0] = apart ? q : 2 * q;
    at[j][1] = apart ? q + turning : 2 * q + 1;
    if (at[j][0] >= chunks) at[j][0] = -1;
    if (at[j][1] >= chunks) at[j][1] = -1;
  }
  auto stage_chunk = [&](int stage, int h, int s) {
    return append_smem + (((stage * kHeads + h) * 2 + s) * kAppendThreads + threadIdx.x) * kChunk;
  };
  auto fetch = [&](int item, int stage) {
    if (item < p.items) {
      const AppendItem i = append_item<T, kHeads>(p, item);
      const Rows& rows = i.which == 0 ? p.q : i.which == 1 ? p.k : p.v;
      const T* src = reinterpret_cast<const T*>(i.src);
#pragma unroll
      for (int h = 0; h < kHeads; ++h)
#pragma unroll
        for (int s = 0; s < 2; ++s)
          if (h < i.heads && at[0][s] >= 0)
            asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(stage_chunk(stage, h, s))),
                         "l"(src + h * rows.head + at[0][s] * kVec), "n"(kChunk >= 4 ? kChunk : 4)
                         : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  pdl_wait_prerequisites();
  int item = static_cast<int>(blockIdx.x) * groups + group, stage = 0;
  if constexpr (kStages > 0) {
#pragma unroll
    for (int k = 0; k < kStages - 1; ++k) fetch(item + k * stride, k);
  }
  // every lane of a warp goes as often round as its first group: the norm's shuffles need the whole group
  for (int first = item - group; first < p.items; first += stride, item += stride) {
    bool live = item < p.items;
    const AppendItem it = append_item<T, kHeads>(p, live ? item : 0);
    const int b = it.b, t = it.t, token = it.token, which = it.which, slice = it.slice, head0 = it.head0,
              heads = it.heads;
    const bool turns = which != 2 && p.rot > 0;

    // lengths, positions, pages and tables serve many rows: ordinary loads, which find them in L1
    const int start = live ? p.kv_len[b] : 0;
    const int n = live && p.new_len ? p.new_len[b] : p.T;
    int pos = 0;
    if (live && p.positions && p.rot > 0) pos = p.positions[token];

    // the rows themselves do not wait for lengths and positions
    Chunk<T, kVec> x[kHeads][kPairs][2];
    if constexpr (kStages > 0) {
      const int next = stage == 0 ? kStages - 1 : stage - 1;
      fetch(item + (kStages - 1) * stride, next);
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages > 0 ? kStages - 1 : 0) : "memory");
    } else {
      const Rows& rows = which == 0 ? p.q : which == 1 ? p.k : p.v;
      const T* src = reinterpret_cast<const T*>(it.src);
#pragma unroll
      for (int h = 0; h < kHeads; ++h)
#pragma unroll
        for (int j = 0; j < kPairs; ++j)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            x[h][j][s] = Chunk<T, kVec>{};
            if (live && h < heads && at[j][s] >= 0)
              x[h][j][s] = load_chunk<T, kVec>(src + h * rows.head + at[j][s] * kVec);
          }
    }
    auto own_chunk = [&](int h, int j, int s) -> Chunk<T, kVec> {
      if constexpr (kStages > 0) {
        if (item >= p.items || h >= heads || at[j][s] < 0) return Chunk<T, kVec>{};
        return *reinterpret_cast<const Chunk<T, kVec>*>(stage_chunk(stage, h, s));
      } else {
        return x[h][j][s];
      }
    };

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
        dst = reinterpret_cast<T*>(p.q_out) + (static_cast<long long>(token) * p.q_heads + head0) * p.D;
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
    const bool norm = weight != nullptr;
    const unsigned members = __ballot_sync(kFull, norm);  // whole groups; the others of the warp may not be
    if (!norm && !turns) {  // moved as they are
      if (live)
#pragma unroll
        for (int h = 0; h < kHeads; ++h)
#pragma unroll
          for (int j = 0; j < kPairs; ++j)
#pragma unroll
            for (int s = 0; s < 2; ++s)
              if (h < heads && at[j][s] >= 0)
                *reinterpret_cast<Chunk<T, kVec>*>(dst + h * dst_head + at[j][s] * kVec) = own_chunk(h, j, s);
    } else {
      // The factors. Of chunk s of pair j: fp multiplies its own elements, fq those that they turn with (the other
      // chunk's, or each element's neighbour).
      Wide<kVec> fp[kPairs][2], fq[kPairs][2];
      bool turned[kPairs][2];
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        const int a = at[j][0], c = at[j][1];
        Wide<kVec> wa, wc;
#pragma unroll
        for (int i = 0; i < kWide; ++i) wa.e[i] = wc.e[i] = make_float2(1.0f, 1.0f);
        if (norm && a >= 0) wa = widen<T, kVec>(*reinterpret_cast<const Chunk<T, kVec>*>(weight + a * kVec));
        if (norm && c >= 0) wc = widen<T, kVec>(*reinterpret_cast<const Chunk<T, kVec>*>(weight + c * kVec));
#pragma unroll
        for (int i = 0; i < kWide; ++i) {
          fp[j][0].e[i] = wa.e[i];
          fp[j][1].e[i] = wc.e[i];
        }
        turned[j][0] = turned[j][1] = false;
        if (!turns || !live) continue;
        const float* cos = p.cos + static_cast<long long>(pos) * (p.rot / 2);
        const float* sin = p.sin + static_cast<long long>(pos) * (p.rot / 2);
        const int q = lane + (j << lanes_log);
        if (across) {
          if (q >= turning) continue;
          turned[j][0] = turned[j][1] = true;
          float cs[kVec + 1], sn[kVec + 1];
          cs[kVec] = sn[kVec] = 0.0f;
          load_table<kVec>(cos + q * kVec, cs, p.vec_tables);
          load_table<kVec>(sin + q * kVec, sn, p.vec_tables);
#pragma unroll
          for (int i = 0; i < kWide; ++i) {
            const float2 co = make_float2(cs[2 * i], cs[2 * i + 1]), si = make_float2(sn[2 * i], sn[2 * i + 1]);
            fp[j][0].e[i] = mul2(wa.e[i], co);
            fq[j][0].e[i] = mul2(wc.e[i], make_float2(-si.x, -si.y));
            fp[j][1].e[i] = mul2(wc.e[i], co);
            fq[j][1].e[i] = mul2(wa.e[i], si);
          }
        } else if constexpr (kVec > 1) {
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if (at[j][s] < 0 || at[j][s] * kVec >= p.rot) continue;
            turned[j][s] = true;
            const Wide<kVec>& w = s ? wc : wa;
            float cs[kVec / 2], sn[kVec / 2];
            load_table<kVec / 2>(cos + at[j][s] * (kVec / 2), cs, p.vec_tables);
            load_table<kVec / 2>(sin + at[j][s] * (kVec / 2), sn, p.vec_tables);
#pragma unroll
            for (int i = 0; i < kWide; ++i) {
              fp[j][s].e[i] = mul2(w.e[i], make_float2(cs[i], cs[i]));
              fq[j][s].e[i] = make_float2(-w.e[i].y * sn[i], w.e[i].x * sn[i]);
            }
          }
        }
      }

#pragma unroll
      for (int h = 0; h < kHeads; ++h) {
        Wide<kVec> y[kPairs][2];
        float2 sum2 = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < kPairs; ++j)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            y[j][s] = widen<T, kVec>(own_chunk(h, j, s));
#pragma unroll
            for (int i = 0; i < kWide; ++i) sum2 = fma2(y[j][s].e[i], y[j][s].e[i], sum2);
          }
        float r = 1.0f;
        if (norm) {
          float sum = sum2.x + sum2.y;
          for (int off = lanes >> 1; off > 0; off >>= 1) sum += __shfl_xor_sync(members, sum, off);
          r = rsqrtf(fmaf(sum, p.inv_dim, p.eps));
        }
        if (!live || h >= heads) continue;
#pragma unroll
        for (int j = 0; j < kPairs; ++j)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if (at[j][s] < 0) continue;
            Chunk<T, kVec> o;
#pragma unroll
            for (int i = 0; i < kWide; ++i) {
              const float2 own = y[j][s].e[i];
              const float2 with = across ? y[j][s ^ 1].e[i] : make_float2(own.y, own.x);
              // an element that does not turn must not see another's NaN or infinity
              const float2 made = turned[j][s] ? fma2(own, fp[j][s].e[i], mul2(with, fq[j][s].e[i]))
                                               : mul2(own, fp[j][s].e[i]);
              const float2 v = mul2(made, make_float2(r, r));
              if constexpr (kVec == 1)
                o.e[0] = Store<T>::narrow(v.x);
              else
                narrow2(o.e + 2 * i, v);
            }
            *reinterpret_cast<Chunk<T, kVec>*>(dst + h * dst_head + at[j][s] * kVec) = o;
          }
      }
    }
    if constexpr (kStages > 0) stage = stage == kStages - 1 ? 0 : stage + 1;
  }
}

constexpr int kSms = 152;

int div_up(int a, int b) { return a / b + (a % b != 0); }

template <typename T, int kVec, int kPairs, int kHeads, int kStages>
int launch_append(AppendParams p, cudaStream_t stream) {
  auto kernel = append_kernel<T, kVec, kPairs, kHeads, kStages>;
  p.q_slices = div_up(p.q_heads, kHeads);
  p.kv_slices = div_up(p.kv_heads, kHeads);
  const int slices = p.q_slices + 2 * p.kv_slices;
  p.items = p.B * p.T * slices;  // the entry point has seen that it fits
  p.by_slices = page_div(slices);
  p.by_tokens = page_div(p.T);
  int lanes_log = 0;
  while (lanes_log < 5 && (kPairs << lanes_log) * 2 * kVec < p.D) ++lanes_log;
  int grid = div_up(p.items, kAppendThreads >> lanes_log);
  const size_t smem = static_cast<size_t>(kStages) * kHeads * 2 * kAppendThreads * sizeof(Chunk<T, kVec>);
  if constexpr (kStages > 0) {
    constexpr int kMaxDevices = 64;
    static std::atomic<int> resident[kMaxDevices];  // CTAs at once; 0: not asked yet
    int dev = 0, per = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return ASD_ERR_CUDA;
    if (dev < 0 || dev >= kMaxDevices) return ASD_ERR_DEVICE;
    int ctas = resident[dev].load(std::memory_order_acquire);
    if (ctas == 0) {
      if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) !=
              cudaSuccess ||
          cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
          cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, kAppendThreads, smem) != cudaSuccess || per < 1)
        return ASD_ERR_CUDA;
      ctas = sms * per;
      resident[dev].store(ctas, std::memory_order_release);
    }
    grid = grid < ctas ? grid : ctas;
  }
  cudaLaunchAttribute attr;
  cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(grid)), dim3(kAppendThreads), stream, &attr);
  cfg.dynamicSmemBytes = smem;
  if (cudaLaunchKernelEx(&cfg, kernel, p, lanes_log) != cudaSuccess) return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

// Large 16-bit calls go through shared memory, four heads per group of lanes: what
// a row needs in registers beside its factors would leave too few threads to cover
// memory's latency (32744 tokens of 56 heads of 128: 179 us, 5.3 TB/s, against 319
// with two heads in registers; 1024 tokens 7.5 against 9.1, 512 5.8 against 6.3).
// Small ones are bound by latency and take two heads in registers (256 tokens 3.8
// us against 6.0), 32-bit ones too, whose chunks hold half the elements (some 2000
// tokens of 24 heads of 96 in 13.9 us against 15.0, their 49 MB in L2; from memory
// 18.6, latency: DRAM 26 % and issue slots 40 % busy). The line lies at 352 threads
// of the former kind per SM. Where four heads a group would be two or fewer on
// average it is two (51212 tokens of 5 + 1 + 1 heads of 128: 68 us against 83; of
// 8 + 2 + 2, three on average, 87 both ways).
template <typename T, int kVec>
int launch_vec(const AppendParams& p, cudaStream_t stream) {
  if constexpr (sizeof(T) == 2) {
    const int slices = div_up(p.q_heads, 4) + 2 * div_up(p.kv_heads, 4);
    const long long threads = static_cast<long long>(p.B) * p.T * slices * div_up(p.D, 2 * kVec);
    if (threads >= 352ll * kSms)
      return p.q_heads + 2 * p.kv_heads <= 2 * slices ? launch_append<T, kVec, 1, 2, 2>(p, stream)
                                                      : launch_append<T, kVec, 1, 4, 2>(p, stream);
  }
  return launch_append<T, kVec, 1, 2, 0>(p, stream);
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
  return launch_append<T, 1, 4, 1, 0>(p, stream);
}

// ---------------------------------------------------------------- compaction
//
// A CTA moves one request's path in one layer, keys or values: its offsets
// first, checked and left in shared memory, then every thread walks the path
// with its own chunk of the token. Sources lie at or past their destinations and
// ascend, so what a thread stores for node i is never what it loads for a later
// node, and a batch of loads can be in flight at once. A few rows are bound by the
// launch: one request's path of 6 in 40 layers of 8 heads of 128 in bf16 takes 3.8
// us. 32 requests' paths of 9 take 17.9 us from memory and 14.7 where the 71 MB are
// in L2 from the call before; what bounds them is instructions (7.4 million, the
// 64-bit divisions by a word's elements among them; issue slots 31 % busy) and two
// rounds of loads, not memory (DRAM 24 % busy).

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
  if (static_cast<double>(cache->B) * a.T * (a.q_heads + 2.0 * cache->heads) > 1073741824.0) return ASD_ERR_SHAPE;
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
  p.inv_dim = 1.0f / static_cast<float>(cache->head_dim);
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
