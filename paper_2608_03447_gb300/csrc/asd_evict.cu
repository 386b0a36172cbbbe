// libasd: eviction from a paged cache (asd_kv_evict).
//
// Per layer, request and key/value head: n of len slots stay, the first and the
// last ones and the heaviest between them. Kept slots at or past n fill the free
// places below n in ascending order, so sources and places never overlap, no two
// moves depend on one another, and what already lies below n is not touched.
//
// A CTA, or for few long heads a cluster, has a head: it keeps the weights in shared
// memory, as integers that grow with them, and finds the lightest weight that stays
// digit by digit from histograms. Digits are of the distance to the smallest key and
// as fine as 2048 bins allow: floats of like size share their upper bits, and
// additions to the same few bins wait for one another. Two words of bits per 32 slots
// say which stay and which are free; their counts, added up over the CTA and the
// cluster, give every move its number, and the moves are dealt in equal shares to the
// cluster's CTAs, into the memory the weights were in.
//
// What is newest: the last slots, as long as tokens lie in their order. Moves fill places
// anywhere, so a token that one eviction kept as new may lie anywhere at the next. With
// numbers (asd_kv_evict_numbered) every slot's token is known and the newest tokens stay
// wherever they are; a number moves with its weight. Without them (kNumbered = false)
// nothing of this is compiled in.
//
// What bounds it: moves, rows of 256 bytes anywhere: 8 prompts of up to 16000 slots cut
// to 4000, four layers of 8 heads of 128, 145 us for 765 MB (5.3 TB/s; 736 of them in the
// DRAM counters, with numbers 147 us). A conversation of
// 4224 slots cut by 128 in 40 layers of 8 heads: 21.5 us (with numbers 23), a third of it the moves, the
// rest a chain of latencies (lengths, weights, three histograms, two sums over the CTA,
// the list). What else was measured for the two: four rows in flight a lane instead of
// two 24 and 152 us (spills), one 23.6 and 150; clusters of two and four where there are
// heads for every SM 30 to 55 and 220 to 270 us; digits of the raw bits, whose few bins
// take turns, 29 and 161 us.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>

#include "asd.h"
#include "asd_cache.cuh"
#include "asd_device.cuh"
#include "asd_launch.cuh"

namespace {

using namespace asd_detail;

constexpr int kBinBits = 11, kBins = 1 << kBinBits;
constexpr int kDigits = 3;  // that 32 bits have
constexpr int kMaxCluster = 8;
constexpr int kMaxPart = ASD_MAX_EVICT_SLOTS / kMaxCluster;  // slots of a CTA
constexpr int kAtOnce = 2;  // rows of keys and of values that a lane has in flight
static_assert(kMaxPart % 32 == 0, "parts are whole words of bits");

// Dynamic shared memory: histograms; weights (then moves); per 32 slots two words of bits and the counts before them.
constexpr size_t evict_smem(int part) {
  return 4 * static_cast<size_t>(part) + 12 * static_cast<size_t>(part / 32) + sizeof(unsigned) * kDigits * kBins;
}
static_assert(evict_smem(kMaxPart) <= 232448 - 1024, "shared memory of the longest part");

struct EvictParams {
  CacheView cache;  // of layer 0
  long long layer_bytes;
  const float* weight;
  float* weight_out;
  const int32_t* kv_len;
  int32_t* kv_len_out;
  const int32_t* keep;
  int32_t* status;
  int32_t* number;       // kNumbered: [layers, B, heads, width]
  const int32_t* tokens;  // kNumbered: [B] appended in all
  int B, H;
  int width, first, last;
  int ctas;       // of a cluster
  int part;       // slots that a CTA has room for
  int element;    // bytes
  int words;      // copy words of a row
  int lane_bits;  // log2 of the lanes that copy a row
};

__device__ __forceinline__ void cluster_sync(int ctas) {
  if (ctas == 1) {
    __syncthreads();
  } else {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
}
__device__ __forceinline__ uint32_t at_rank(const void* smem, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(smem)), "r"(rank));
  return r;
}
__device__ __forceinline__ unsigned load_cluster(uint32_t addr) {
  unsigned v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void store_cluster(uint32_t addr, unsigned v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// The sum of x over the threads before this one; *total over all. A barrier on either side.
template <int kWarps>
__device__ __forceinline__ unsigned block_scan(unsigned x, unsigned* warp_sums, unsigned* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned sum = x;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const unsigned o = __shfl_up_sync(kFull, sum, off);
    if (lane >= off) sum += o;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = sum;
  __syncthreads();
  unsigned before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const unsigned s = warp_sums[w];
    if (w < warp) before += s;
    all += s;
  }
  *total = all;
  return before + sum - x;
}

// Word: what a row is copied in. Up to four CTAs an SM of 256 threads, two of 512: the
// larger ones where no more than two heads come on an SM (8 prompts 145 us, with 256
// threads 165; the conversation, two to three heads an SM, 21.5 us against 24.4).
template <typename Word, int kThreads, bool kNumbered>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) evict_kernel(const __grid_constant__ EvictParams p) {
  constexpr int kWarps = kThreads / 32;
  extern __shared__ __align__(16) unsigned s_mem[];
  __shared__ unsigned s_warp[kWarps];
  __shared__ unsigned s_found[3];  // the digit, how many of its slots stay, how many there are
  // this CTA's counts, its smallest and largest key, how many slots stay in any case, for the cluster
  __shared__ unsigned s_total[5];
  unsigned* s_hist = s_mem;                   // [kDigits][kBins], cleared by 16-byte words
  unsigned* s_key = s_hist + kDigits * kBins; // [part]
  unsigned* s_above = s_key + p.part;         // [part / 32] bits: heavier than the lightest that stays; then moves
  unsigned* s_equal = s_above + p.part / 32;  // as heavy; then free places
  unsigned* s_base = s_equal + p.part / 32;   // [part / 32] how many come before: free places above, moves below

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, C = p.ctas;
  const int head_id = blockIdx.x / C, rank = blockIdx.x - head_id * C;
  const int h = head_id % p.H, lb = head_id / p.H, b = lb % p.B, layer = lb / p.B;
  pdl_signal_dependents();
  for (int i = tid; i < kDigits * kBins / 4; i += kThreads)
    reinterpret_cast<uint4*>(s_hist)[i] = make_uint4(0u, 0u, 0u, 0u);
  pdl_wait_prerequisites();

  const int len = __ldcg(p.kv_len + b), keep = __ldcg(p.keep + b);
  const int tokens = kNumbered ? __ldcg(p.tokens + b) : 0;
  const bool bad = len < 0 || len > p.cache.slots || len > p.width || keep < 0 || (kNumbered && tokens < len);
  const int n = bad ? 0 : min(keep, len);
  if (layer == 0 && h == 0 && rank == 0 && tid == 0) {
    if (bad && p.status) atomicOr(p.status + b, static_cast<int>(ASD_STATUS_LENGTH));
    p.kv_len_out[b] = bad ? len : n;
  }
  if (bad || (n == 0 && !kNumbered)) return;
  const float* weight = p.weight + static_cast<long long>(head_id) * p.width;
  float* weight_out = p.weight_out + static_cast<long long>(head_id) * p.width;
  int32_t* number = kNumbered ? p.number + static_cast<long long>(head_id) * p.width : nullptr;
  const bool copies = p.weight != p.weight_out;
  const int per = ((len + C - 1) / C + 31) & ~31;
  const int s0 = min(rank * per, len), count = min(per, len - s0);
  if (kNumbered && n == 0) {
    for (int i = tid; i < count; i += kThreads) number[s0 + i] = -1;
    return;
  }
  if (n == len) {
    if (copies)
      for (int i = tid; i < count; i += kThreads) weight_out[s0 + i] = __ldcg(weight + s0 + i);
    return;
  }
  const int first = min(p.first, n), last = min(p.last, n - first);
  // a slot without a number has been appended since the last eviction, in order
  auto token_of = [&](int given, int s) { return given >= 0 ? given : tokens - len + s; };

  // keys; those that stay in any case are above every weight and in no histogram
  constexpr unsigned kStays = 0xffffffffu;
  unsigned smallest = kStays, largest = 0u, always = 0u;
  constexpr int kLoads = kNumbered ? 8 : 16;  // in flight at once: no store between them, which a load might not pass
  for (int i0 = tid; i0 < count; i0 += kLoads * kThreads) {
    float w[kLoads];
    int given[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      w[k] = i0 + k * kThreads < count ? __ldcg(weight + s0 + i0 + k * kThreads) : 0.0f;
      if (kNumbered) given[k] = i0 + k * kThreads < count ? __ldcg(number + s0 + i0 + k * kThreads) : 0;
    }
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int i = i0 + k * kThreads, s = s0 + i;
      if (i >= count) break;
      if (copies && s < n) weight_out[s] = w[k];
      unsigned key = w[k] == w[k] ? ordered_bits(w[k]) : ordered_bits(-INFINITY);
      bool newest = s >= len - last;
      if (kNumbered) {
        const int token = token_of(given[k], s);
        if (given[k] < 0 && s < n) number[s] = token;
        newest = token >= tokens - last;
      }
      if (s < first || newest) {
        key = kStays;
        ++always;
      } else {
        smallest = min(smallest, key);
        largest = max(largest, key);
      }
      s_key[i] = key;
    }
  }
  smallest = __reduce_min_sync(kFull, smallest);
  largest = __reduce_max_sync(kFull, largest);
  if (kNumbered) always = __reduce_add_sync(kFull, always);
  if (tid == 0) s_total[2] = kStays, s_total[3] = 0u, s_total[4] = 0u;
  __syncthreads();
  if (lane == 0) {
    atomicMin(&s_total[2], smallest);
    atomicMax(&s_total[3], largest);
    if (kNumbered) atomicAdd(&s_total[4], always);
  }
  cluster_sync(C);
  smallest = s_total[2], largest = s_total[3];
  always = kNumbered ? s_total[4] : static_cast<unsigned>(first + last);
  for (int r = 0; C > 1 && r < C; ++r) {
    smallest = min(smallest, load_cluster(at_rank(&s_total[2], r)));
    largest = max(largest, load_cluster(at_rank(&s_total[3], r)));
    if (kNumbered && r != rank) always += load_cluster(at_rank(&s_total[4], r));
  }
  if (kNumbered && always > static_cast<unsigned>(n)) {  // numbers that no call wrote: twice the same, or too large
    if (rank == 0 && tid == 0 && p.status) atomicOr(p.status + b, static_cast<int>(ASD_STATUS_POSITION));
    for (int i = max(n - s0, 0) + tid; i < count; i += kThreads) number[s0 + i] = -1;
    if (C > 1) cluster_sync(C);  // this CTA's counts have been read
    return;
  }

  // The lightest weight that stays: of the keys' distances to the smallest, digit by digit from the top. All whose upper
  // bits are above `prefix` stay, of the `equal` ones that share it `need`.
  const int range = 32 - __clz(largest - smallest);  // bits; n < len, so some keys are no kStays (always <= n)
  unsigned prefix = 0, need = static_cast<unsigned>(n) - always, equal = static_cast<unsigned>(len) - always;
  int shift = range;
  for (int digit = 0; need > 0 && need < equal && shift > 0; ++digit) {
    unsigned* hist = s_hist + digit * kBins;
    const int next = max(0, shift - kBinBits);
    const unsigned mask = (1u << (shift - next)) - 1u;
#pragma unroll 4
    for (int i = tid; i < count; i += kThreads) {
      const unsigned key = s_key[i], d = key - smallest;
      if (key != kStays && (shift == 32 || d >> shift == prefix)) atomicAdd(&hist[(d >> next) & mask], 1u);
    }
    cluster_sync(C);
    if (C > 1) {  // a CTA adds up its share of the bins for all
      const int from = kBins / C * rank;
      for (int i = tid; i < kBins / C; i += kThreads) {
        unsigned some[kMaxCluster], total = 0;
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r) some[r] = r < C ? load_cluster(at_rank(hist + from + i, r)) : 0u;
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r) total += some[r];
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r)
          if (r < C) store_cluster(at_rank(hist + from + i, r), total);
      }
      cluster_sync(C);
    }
    constexpr int kEach = kBins / kThreads;
    unsigned mine[kEach], sum = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      mine[k] = hist[kBins - 1 - (tid * kEach + k)];
      sum += mine[k];
    }
    unsigned all;
    unsigned before = block_scan<kWarps>(sum, s_warp, &all);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      if (before < need && before + mine[k] >= need) {
        s_found[0] = static_cast<unsigned>(kBins - 1 - (tid * kEach + k));
        s_found[1] = need - before;
        s_found[2] = mine[k];
      }
      before += mine[k];
    }
    __syncthreads();
    prefix = (prefix << (shift - next)) | s_found[0];
    need = s_found[1];
    equal = s_found[2];
    shift = next;
  }
  const bool some = need > 0 && need < equal;  // of equal ones the lowest slots stay

  const int words = (count + 31) / 32;
#pragma unroll 4
  for (int i = warp; i < words; i += kWarps) {
    const int at = 32 * i + lane;
    const unsigned key = at < count ? s_key[at] : 0u, d = key - smallest;
    const unsigned top = shift == 32 ? 0u : d >> shift;
    const unsigned above = __ballot_sync(kFull, at < count && (key == kStays || top > prefix));
    const unsigned same = __ballot_sync(kFull, at < count && key != kStays && top == prefix);
    if (lane == 0) s_above[i] = above, s_equal[i] = same;
  }
  __syncthreads();
  const int each = (words + kThreads - 1) / kThreads;  // consecutive words of a thread
  const int w0 = min(tid * each, words), w1 = min(w0 + each, words);
  unsigned all = 0;
  if (some) {
    unsigned sum = 0;
    for (int i = w0; i < w1; ++i) sum += __popc(s_equal[i]);
    unsigned before = block_scan<kWarps>(sum, s_warp, &all);
    if (C > 1) {
      if (tid == 0) s_total[0] = all;
      cluster_sync(C);
      for (int r = 0; r < rank; ++r) before += load_cluster(at_rank(&s_total[0], r));
      cluster_sync(C);  // read by all before it is written again
    }
    for (int i = w0; i < w1; ++i) {
      s_base[i] = before;
      before += __popc(s_equal[i]);
    }
    __syncthreads();
    for (int i = warp; i < words; i += kWarps) {
      const unsigned same = s_equal[i];
      const bool stays = ((same >> lane) & 1u) && s_base[i] + __popc(same & ((1u << lane) - 1u)) < need;
      const unsigned keeps = __ballot_sync(kFull, stays);
      if (lane == 0) s_equal[i] = keeps;
    }
    __syncthreads();
  }
  unsigned counts = 0;  // of this thread's words: free places above, moves below
  for (int i = w0; i < w1; ++i) {
    const unsigned stays = s_above[i] | (need > 0 ? s_equal[i] : 0u);
    const int low_bits = n - (s0 + 32 * i);
    const unsigned low = low_bits >= 32 ? kFull : low_bits <= 0 ? 0u : (1u << low_bits) - 1u;
    const unsigned free = ~stays & low, moves = stays & ~low;
    s_above[i] = moves, s_equal[i] = free;
    s_base[i] = counts;
    counts += (static_cast<unsigned>(__popc(free)) << 16) + static_cast<unsigned>(__popc(moves));
  }
  static_assert(kMaxPart < 65536, "a CTA's counts have 16 bits");
  const unsigned before = block_scan<kWarps>(counts, s_warp, &all);
  for (int i = w0; i < w1; ++i) s_base[i] += before;
  unsigned place = 0, source = 0, total = all & 0xffffu;  // in the CTAs before; in all
  if (C > 1) {
    if (tid == 0) s_total[0] = all;
    cluster_sync(C);
    total = 0;
    for (int r = 0; r < C; ++r) {
      const unsigned other = load_cluster(at_rank(&s_total[0], r));
      total += other & 0xffffu;
      if (r < rank) place += other >> 16, source += other & 0xffffu;
    }
  } else {
    __syncthreads();
  }
  // The moves' list, a share a CTA, where the weights were: every CTA of the cluster is done with its own.
  const unsigned share = (total + C - 1) / C;
  auto put = [&](unsigned number, unsigned offset, unsigned slot) {
    if (C == 1) {
      s_key[offset + number] = slot;
    } else {
      const unsigned to = number / share;
      store_cluster(at_rank(s_key + offset + (number - to * share), static_cast<int>(to)), slot);
    }
  };
  const unsigned below = (1u << lane) - 1u;
#pragma unroll 4
  for (int i = warp; i < words; i += kWarps) {
    const unsigned moves = s_above[i], free = s_equal[i], base = s_base[i];
    const unsigned slot = static_cast<unsigned>(s0 + 32 * i + lane);
    if ((moves >> lane) & 1u) put(source + (base & 0xffffu) + __popc(moves & below), 0u, slot);
    if (kNumbered && !((moves >> lane) & 1u) && slot >= static_cast<unsigned>(n) && slot < static_cast<unsigned>(len))
      number[slot] = -1;
    if ((free >> lane) & 1u) put(place + (base >> 16) + __popc(free & below), share, slot);
  }
  cluster_sync(C);

  const unsigned begin = min(share * rank, total);
  const int moves = static_cast<int>(min(share, total - begin));
  char* const k = p.cache.k + layer * p.layer_bytes;
  char* const v = p.cache.v + layer * p.layer_bytes;
  const int per_row = 1 << p.lane_bits, rows = 32 >> p.lane_bits;
  const int sub = lane >> p.lane_bits, word0 = lane & (per_row - 1);
  // A warp's moves: as many as a lane each are looked up at once, the next ones while these are copied. Few moves are
  // spread over the warps.
  const int batch = min(32, max(kAtOnce * rows, (moves + kWarps - 1) / kWarps));
  long long from = -1, to = -1;
  auto look_up = [&](int m) {
    from = to = -1;
    if (lane >= batch || m + lane >= moves) return;
    const int src = static_cast<int>(s_key[m + lane]), dst = static_cast<int>(s_key[share + m + lane]);
    const long long f = slot_offset(p.cache, b, src), t = slot_offset(p.cache, b, dst);
    weight_out[dst] = __ldcg(weight + src);
    if (kNumbered) {
      number[dst] = token_of(__ldcg(number + src), src);
      number[src] = -1;
    }
    if (f >= 0 && t >= 0) {
      from = (f + h * p.cache.head_stride) * p.element;
      to = (t + h * p.cache.head_stride) * p.element;
    } else if (p.status) {
      atomicOr(p.status + b, static_cast<int>(ASD_STATUS_PAGE));
    }
  };
  look_up(warp * batch);
  for (int m0 = warp * batch; m0 < moves; m0 += kWarps * batch) {
    const int many = min(batch, moves - m0);
    const long long f = from, t = to;
    bool next = true;
    for (int r0 = 0; r0 < many; r0 += kAtOnce * rows) {
      long long src[kAtOnce], dst[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int r = r0 + i * rows + sub;
        src[i] = __shfl_sync(kFull, f, r & 31);
        dst[i] = __shfl_sync(kFull, t, r & 31);
        if (r >= many) src[i] = -1;
      }
      for (int w = word0; w < p.words; w += per_row) {
        Word kw[kAtOnce], vw[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          if (src[i] >= 0) {
            kw[i] = __ldcg(reinterpret_cast<const Word*>(k + src[i]) + w);
            vw[i] = __ldcg(reinterpret_cast<const Word*>(v + src[i]) + w);
          }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          if (src[i] >= 0) {
            reinterpret_cast<Word*>(k + dst[i])[w] = kw[i];
            reinterpret_cast<Word*>(v + dst[i])[w] = vw[i];
          }
      }
      if (next) look_up(m0 + kWarps * batch);
      next = false;
      __syncwarp();
    }
  }
}

// ---------------------------------------------------------------- host side

constexpr int kMaxDevices = 64;

template <typename Word, int kThreads, bool kNumbered>
int launch_evict(EvictParams p, long long heads, int sms, cudaStream_t stream) {
  auto kernel = evict_kernel<Word, kThreads, kNumbered>;
  int ctas = 1;
  while (ctas < kMaxCluster && (p.width > ctas * kMaxPart || (heads * ctas < sms && p.width > 1024 * ctas))) ctas *= 2;
  if (heads * ctas > INT32_MAX) return ASD_ERR_SHAPE;
  p.ctas = ctas;
  p.part = ((p.width + ctas - 1) / ctas + 31) / 32 * 32;
  p.lane_bits = 0;
  while (p.lane_bits < 5 && (1 << p.lane_bits) < p.words) ++p.lane_bits;
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(heads * ctas)), dim3(kThreads), stream, attr);
  cfg.dynamicSmemBytes = evict_smem(p.part);
  if (ctas > 1) {
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(ctas);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
  }
  if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

template <typename Word, bool kNumbered>
int launch_word(const EvictParams& p, int layers, cudaStream_t stream) {
  static std::atomic<int> sms_of[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return ASD_ERR_CUDA;
  if (dev < 0 || dev >= kMaxDevices) return ASD_ERR_DEVICE;
  int sms = sms_of[dev].load(std::memory_order_acquire);
  if (sms == 0) {
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaFuncSetAttribute(evict_kernel<Word, 256, kNumbered>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(evict_smem(kMaxPart))) != cudaSuccess ||
        cudaFuncSetAttribute(evict_kernel<Word, 512, kNumbered>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(evict_smem(kMaxPart))) != cudaSuccess)
      return ASD_ERR_CUDA;
    sms_of[dev].store(sms, std::memory_order_release);
  }
  const long long heads = static_cast<long long>(layers) * p.B * p.H;
  return heads <= 2 * sms ? launch_evict<Word, 512, kNumbered>(p, heads, sms, stream)
                          : launch_evict<Word, 256, kNumbered>(p, heads, sms, stream);
}

template <bool kNumbered>
int evict(const asd_kv_cache* cache, const asd_evict* args, int32_t* number, const int32_t* tokens,
          asd_stream_t stream) {
  const int rc = check_cache(cache);
  if (rc != ASD_OK) return rc;
  if (!args) return ASD_ERR_NULL;
  const asd_evict& a = *args;
  if (a.first < 0 || a.last < 0 || a.width < 0 || a.width > ASD_MAX_EVICT_SLOTS || a.reserved != 0) return ASD_ERR_SHAPE;
  if (cache->B == 0) return ASD_OK;
  if (!a.kv_len || !a.kv_len_out || !a.keep || (a.width > 0 && (!a.weight || !a.weight_out))) return ASD_ERR_NULL;
  if (kNumbered && (!tokens || (a.width > 0 && !number))) return ASD_ERR_NULL;
  if (a.kv_len_out == a.kv_len || a.kv_len_out == a.keep || (kNumbered && a.kv_len_out == tokens)) return ASD_ERR_SHAPE;
  const void* const words[] = {a.weight, a.weight_out, a.kv_len, a.kv_len_out, a.keep, a.status, number, tokens};
  for (const void* x : words)
    if (reinterpret_cast<uintptr_t>(x) % 4 != 0) return ASD_ERR_ALIGN;
  const size_t es = store_bytes(cache->dtype);
  EvictParams p = {};
  p.cache = cache_view(cache, 0);
  p.layer_bytes = cache->layer_stride * static_cast<long long>(es);
  p.weight = a.weight;
  p.weight_out = a.weight_out;
  p.kv_len = a.kv_len;
  p.kv_len_out = a.kv_len_out;
  p.keep = a.keep;
  p.status = a.status;
  p.number = number;
  p.tokens = tokens;
  p.B = cache->B;
  p.H = cache->heads;
  p.element = static_cast<int>(es);
  p.width = a.width;
  p.first = a.first;
  p.last = a.last;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  // whole 16-byte words where every row starts on one, else elements
  const int per = static_cast<int>(16 / es);
  if (cache->head_dim % per == 0 && cache->layer_stride % per == 0 &&
      rows_aligned(p.cache.k, es, 16, cache->page_stride, cache->token_stride, cache->head_stride) &&
      reinterpret_cast<uintptr_t>(p.cache.v) % 16 == 0) {
    p.words = cache->head_dim / per;
    return launch_word<uint4, kNumbered>(p, cache->layers, s);
  }
  p.words = cache->head_dim;
  if (es == 4) return launch_word<unsigned, kNumbered>(p, cache->layers, s);
  return launch_word<unsigned short, kNumbered>(p, cache->layers, s);
}

}  // namespace

extern "C" {

int asd_kv_evict(const asd_kv_cache* cache, const asd_evict* args, asd_stream_t stream) {
  return evict<false>(cache, args, nullptr, nullptr, stream);
}

int asd_kv_evict_numbered(const asd_kv_cache* cache, const asd_evict* args, int32_t* number, const int32_t* tokens,
                          asd_stream_t stream) {
  return evict<true>(cache, args, number, tokens, stream);
}

}  // extern "C"
