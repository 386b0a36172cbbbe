// libasd: logits under a request's rules (penalties, biases, grammar):
// asd_rules_verify, asd_rules_logits, asd_tokens_record, asd_tokens_bias.
//
//   z <- z > 0 ? z / rho : z rho   tokens said or in the prompt
//   z <- z - c f - p               tokens said c > 0 times, the drafts before the row among them
//   z <- z + bias                  tokens that have a record
//   z <- -inf                      tokens that the grammar does not allow
//
// Few tokens have a record, so a row is read as the verifier reads it, by 128-bit
// loads with a running maximum, in which the elements that a bit of the grammar
// rules out or a mark sets aside count as -infinity; the marked ones, and the
// block's drafts, are taken one by one from a list: their logit, their record, the
// operations above in fp32, each rounded. One CTA takes a range of the vocabulary
// for all rows of a request, one warp a row, so that a range's marks are looked
// through once.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "asd.h"
#include "asd_device.cuh"
#include "asd_launch.cuh"
#include "asd_select.cuh"

namespace {

using namespace asd_detail;

constexpr int kMaxWarps = 10;  // rows at once; more take turns
constexpr uint32_t kTimes = 0x7fffffffu;
constexpr int kMarked = 0x8000;  // of a list entry: the token has a record (else it is only a draft)

struct RulesParams {
  const void* logits;
  void* out;              // asd_rules_logits
  const int32_t* draft;   // [B, K]
  const uint32_t* marks;
  const asd_token_record* records;
  const float* repetition;
  const float* frequency;
  const float* presence;
  const uint32_t* allow;
  long long allow_batch, allow_row;
  int B, R, K, V;
  int words;              // of a row of marks
  int chunks;             // ranges of the vocabulary
  unsigned long long* row_key;  // asd_rules_verify: as in VerifyParams
  float* draft_logit;
  unsigned* flags;
};

__device__ __forceinline__ uint4 load_row(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

__device__ __forceinline__ uint32_t max_of(uint32_t a, uint32_t b, float) {
  return __float_as_uint(fmax_nan(__uint_as_float(a), __uint_as_float(b)));
}
__device__ __forceinline__ uint32_t max_of(uint32_t a, uint32_t b, __nv_bfloat16) {
  uint32_t m;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
  return m;
}
template <typename T>
__device__ __forceinline__ uint32_t max_of(const uint4& v) {
  return max_of(max_of(v.x, v.y, T()), max_of(v.z, v.w, T()), T());
}
__device__ __forceinline__ float widest(uint32_t m, float) { return __uint_as_float(m); }
__device__ __forceinline__ float widest(uint32_t m, __nv_bfloat16) {
  return fmax_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
}

// Elements whose bit of `keep` is 0 become -infinity.
__device__ __forceinline__ uint32_t only(uint32_t w, uint32_t keep, float) { return keep & 1u ? w : 0xff800000u; }
__device__ __forceinline__ uint32_t only(uint32_t w, uint32_t keep, __nv_bfloat16) {
  if (!(keep & 1u)) w = (w & 0xffff0000u) | 0xff80u;
  if (!(keep & 2u)) w = (w & 0xffffu) | 0xff800000u;
  return w;
}
template <typename T>
__device__ __forceinline__ uint4 only(const uint4& v, uint32_t keep) {
  constexpr int n = Elem<T>::kVec / 4;  // elements of a word
  return make_uint4(only(v.x, keep, T()), only(v.y, keep >> n, T()), only(v.z, keep >> 2 * n, T()),
                    only(v.w, keep >> 3 * n, T()));
}

// The first element of the unit's vectors that equals best; one of them does.
template <typename T, int kU>
__device__ __forceinline__ int first_of(const uint4 (&v)[kU], float best) {
  int at = 0;
#pragma unroll
  for (int u = kU - 1; u >= 0; --u)
    if (widest(max_of<T>(v[u]), T()) == best) {
#pragma unroll
      for (int t = Elem<T>::kVec - 1; t >= 0; --t)
        if (Elem<T>::lane(v[u], t) == best) at = u * Elem<T>::kVec + t;
    }
  return at;
}

__device__ __forceinline__ float narrow(float v, float) { return v; }
__device__ __forceinline__ __nv_bfloat16 narrow(float v, __nv_bfloat16) { return __float2bfloat16_rn(v); }

// kU: vectors a lane has of a row's range. kWrite: writes the changed logits,
// else reduces them to the row's (value, index) key and its draft's logit.
template <typename T, int kU, bool kWrite>
__global__ void __launch_bounds__(kMaxWarps * 32, 3) rules_kernel(const __grid_constant__ RulesParams p) {
  constexpr int VN = Elem<T>::kVec;
  constexpr int kChunk = 32 * kU * VN, kWords = kChunk / 32, kWordsLane = (kWords + 31) / 32;
  __shared__ uint32_t s_special[kWords + 1];  // tokens with a record, and drafts
  __shared__ uint32_t s_allow[kMaxWarps][kWords + 1];
  __shared__ uint16_t s_list[kChunk];
  __shared__ int s_count;

  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int b = blockIdx.x / p.chunks;
  const int t0 = (blockIdx.x - b * p.chunks) * kChunk;
  const int len = min(kChunk, p.V - t0);
  const bool grammar = p.allow != nullptr;
  pdl_signal_dependents();
  pdl_wait_prerequisites();

  uint4 v[kU];
  uint32_t allowed[kWordsLane];
  const T* z;
  int lead, nvec;
  // a row's range: loose elements up to a 16-byte boundary, whole vectors, loose ones; all loads in flight at once
  auto load = [&](int j) {
    z = static_cast<const T*>(p.logits) + (static_cast<long long>(b) * p.R + j) * p.V + t0;
    lead = min(static_cast<int>((16u - static_cast<unsigned>(reinterpret_cast<uintptr_t>(z) & 15u)) & 15u) /
                   static_cast<int>(sizeof(T)),
               len);
    nvec = (len - lead) / VN;
    const uint4* vp = reinterpret_cast<const uint4*>(z + lead);
    if (nvec > 0) {
#pragma unroll
      for (int u = 0; u < kU; ++u) v[u] = load_row(vp + min(lane + 32 * u, nvec - 1));
    }
    if (grammar) {
      const uint32_t* row = p.allow + b * p.allow_batch + j * p.allow_row + t0 / 32;
#pragma unroll
      for (int i = 0; i < kWordsLane; ++i) {
        const int w = lane + 32 * i;
        allowed[i] = w < kWords && t0 / 32 + w < p.words ? __ldcg(row + w) : 0u;
      }
    }
  };
  load(warp);

  const int mine = lane < p.K ? __ldcg(p.draft + static_cast<long long>(b) * p.K + lane) - t0 : -1;
  const unsigned near = __ballot_sync(kFull, mine >= 0 && mine < len);  // drafts in the range
  if (warp == 0) {
    uint32_t mark[kWordsLane], all[kWordsLane];
#pragma unroll
    for (int i = 0; i < kWordsLane; ++i) {
      const int w = lane + 32 * i;
      mark[i] = 0u;
      if (w < kWords && t0 / 32 + w < p.words)
        mark[i] = __ldcg(p.marks + static_cast<long long>(b) * p.words + t0 / 32 + w);
      const int left = p.V - t0 - 32 * w;  // bits past the vocabulary may be anything
      if (left < 32) mark[i] &= left <= 0 ? 0u : (1u << left) - 1u;
      all[i] = mark[i];
    }
    for (unsigned left = near; left; left &= left - 1) {
      const int x = __shfl_sync(kFull, mine, __ffs(left) - 1);
#pragma unroll
      for (int i = 0; i < kWordsLane; ++i)
        if (x >> 5 == lane + 32 * i) all[i] |= 1u << (x & 31);
    }
    int n = 0;
#pragma unroll
    for (int i = 0; i < kWordsLane; ++i) n += __popc(all[i]);
    int before = n;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(kFull, before, off);
      if (lane >= off) before += o;
    }
    if (lane == 31) s_count = before;
    before -= n;
#pragma unroll
    for (int i = 0; i < kWordsLane; ++i) {
      const int w = lane + 32 * i;
      if (w <= kWords) s_special[w] = all[i];
      for (uint32_t left = all[i]; left; left &= left - 1) {
        const int bit = __ffs(left) - 1;
        s_list[before++] = static_cast<uint16_t>(32 * w + bit + ((mark[i] >> bit) & 1u) * kMarked);
      }
    }
    if (kWords % 32 == 0 && lane == 0) s_special[kWords] = 0u;
  }
  float rho = 1.0f, f = 0.0f, pr = 0.0f;
  if (p.repetition) rho = __ldcg(p.repetition + b);
  if (p.frequency) f = __ldcg(p.frequency + b);
  if (p.presence) pr = __ldcg(p.presence + b);
  __syncthreads();
  const int count = s_count;

  for (int j = warp; j < p.R; j += warps) {
    if (j != warp) load(j);
    const long long row = static_cast<long long>(b) * p.R + j;
    // what the list's entries need is asked for before the vectors are waited for
    struct Entry {
      int tok;  // of the range; -1: none
      bool marked;
      float z;
      uint2 record;
    };
    auto fetch = [&](int i) {
      Entry e = {-1, false, 0.0f, make_uint2(0u, 0u)};
      if (i < count) {
        const int x = s_list[i];
        e.tok = x & (kMarked - 1);
        e.marked = (x & kMarked) != 0;
        e.z = Elem<T>::load_cg(z, e.tok);
        if (e.marked)
          e.record = *reinterpret_cast<const uint2*>(p.records + static_cast<long long>(b) * p.V + t0 + e.tok);
      }
      return e;
    };
    Entry e0 = fetch(lane), e1 = fetch(lane + 32);
    if (grammar) {
      __syncwarp();  // the row before is done with the words
#pragma unroll
      for (int i = 0; i < kWordsLane; ++i)
        if (lane + 32 * i <= kWords) s_allow[warp][lane + 32 * i] = allowed[i];
      if (kWords % 32 == 0 && lane == 0) s_allow[warp][kWords] = 0u;
      __syncwarp();
    }
    auto may = [&](int at) { return !grammar || ((s_allow[warp][at >> 5] >> (at & 31)) & 1u); };
    auto bits = [&](const uint32_t* words, int at) {  // of the VN elements from `at` on
      return __funnelshift_r(words[at >> 5], words[(at >> 5) + 1], at & 31);
    };

    unsigned long long key = 0ull;
    bool nan = false;
    uint32_t order = 0u;
    float best = 0.0f;
    T* out = kWrite ? static_cast<T*>(p.out) + row * p.V + t0 : nullptr;
    if (nvec > 0) {
      if (kWrite ? grammar : grammar || count > 0) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const int at = lead + min(lane + 32 * u, nvec - 1) * VN;
          uint32_t keep = grammar ? bits(s_allow[warp], at) : 0xffffffffu;
          if (!kWrite) keep &= ~bits(s_special, at);
          v[u] = only<T>(v[u], keep);
        }
      }
      if (kWrite) {
        if ((reinterpret_cast<uintptr_t>(out + lead) & 15u) == 0) {
#pragma unroll
          for (int u = 0; u < kU; ++u)
            if (lane + 32 * u < nvec) reinterpret_cast<uint4*>(out + lead)[lane + 32 * u] = v[u];
        } else {
#pragma unroll
          for (int u = 0; u < kU; ++u)
            if (lane + 32 * u < nvec)
#pragma unroll
              for (int t = 0; t < VN; ++t)
                out[lead + (lane + 32 * u) * VN + t] = narrow(Elem<T>::lane(v[u], t), T());
        }
      } else {
        uint32_t m = max_of<T>(v[0]);
#pragma unroll
        for (int u = 1; u < kU; ++u) m = max_of(m, max_of<T>(v[u]), T());
        best = widest(m, T());
        nan = __any_sync(kFull, best != best);
        order = nan ? 0u : ordered_bits(best);
      }
    }
    if (lead > 0 || lead + nvec * VN < len) {  // loose elements, one a lane
      const int at = lane < VN ? lane : lead + nvec * VN + lane - VN;
      if ((lane < VN ? at < lead : lane < 2 * VN && at < len)) {
        const bool special = (s_special[at >> 5] >> (at & 31)) & 1u;
        float x = Elem<T>::load_cg(z, at);
        if (!may(at)) x = -INFINITY;
        if (kWrite) {
          out[at] = narrow(x, T());
        } else if (!special) {
          if (x == x)
            key = make_key(x, static_cast<uint32_t>(t0 + at));
          else
            nan = true;
        }
      }
    }
    if (kWrite) __syncwarp();  // entries are written over what the vectors had
    const int here = j < p.K ? __shfl_sync(kFull, mine, j) : -1;  // the row's draft
    const unsigned said = near & ((1u << j) - 1u);                // drafts before the row, in the range
    auto finish = [&](const Entry& e) {
      uint32_t times = e.record.x & kTimes;
      for (unsigned left = said; left; left &= left - 1) times += __shfl_sync(kFull, mine, __ffs(left) - 1) == e.tok;
      if (e.tok < 0) return;
      float x = e.z;
      if (times > 0u || (e.record.x & ASD_TOKEN_PROMPT))
        if (p.repetition) x = x > 0.0f ? __fdiv_rn(x, rho) : __fmul_rn(x, rho);
      if (times > 0u) {
        x = __fsub_rn(x, __fmul_rn(static_cast<float>(times), f));
        x = __fsub_rn(x, pr);
      }
      if (e.marked) x = __fadd_rn(x, __uint_as_float(e.record.y));
      if (!may(e.tok)) x = -INFINITY;
      if (kWrite) {
        out[e.tok] = narrow(x, T());
        return;
      }
      if (e.tok == here) p.draft_logit[row] = x;
      if (x == x) {
        const unsigned long long k = make_key(x, static_cast<uint32_t>(t0 + e.tok));
        key = k > key ? k : key;
      } else {
        nan = true;
      }
    };
    if (count > 0) finish(e0);
    if (count > 32) finish(e1);
    for (int i = 64; i < count; i += 64) {
      const Entry a = fetch(i + lane), c = fetch(i + 32 + lane);
      finish(a);
      finish(c);
    }
    if (kWrite) continue;
    const uint32_t high = static_cast<uint32_t>(key >> 32);
    const uint32_t top = __reduce_max_sync(kFull, order > high ? order : high);
    uint32_t low = 0u;
    if (order == top && top != 0u) {
      const int at = first_of<T, kU>(v, best);
      low = 0xffffffffu - static_cast<uint32_t>(t0 + lead + min(lane + 32 * (at / VN), nvec - 1) * VN + at % VN);
    }
    if (high == top && static_cast<uint32_t>(key) > low) low = static_cast<uint32_t>(key);
    low = __reduce_max_sync(kFull, low);
    nan = __any_sync(kFull, nan);
    if (lane == 0) {
      if (top != 0u) atomicMax(p.row_key + row, (static_cast<unsigned long long>(top) << 32) | low);
      if (nan) atomicOr(p.flags + b, ASD_STATUS_NAN_LOGIT);
    }
  }
}

// A token a thread. Marks and records are only added to, by atomics whose order does not matter.
__global__ void __launch_bounds__(256)
    record_kernel(const __grid_constant__ RulesParams p, const int32_t* tokens, int n, const int32_t* token_len,
                  int prompt, int32_t* status) {
  pdl_signal_dependents();
  pdl_wait_prerequisites();
  const long long at = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (at >= static_cast<long long>(p.B) * n) return;
  const int b = static_cast<int>(at / n), i = static_cast<int>(at - static_cast<long long>(b) * n);
  const int length = token_len ? __ldcg(token_len + b) : n;
  if (length < 0 || length > n) {
    if (i == 0 && status) atomicOr(status + b, static_cast<int>(ASD_STATUS_LENGTH));
    return;
  }
  if (i >= length) return;
  const int x = __ldcg(tokens + at);
  if (x < 0) return;
  if (x >= p.V) {
    if (status) atomicOr(status + b, static_cast<int>(ASD_STATUS_TOKEN));
    return;
  }
  uint32_t* seen = const_cast<uint32_t*>(&p.records[static_cast<long long>(b) * p.V + x].seen);
  if (prompt)
    atomicOr(seen, ASD_TOKEN_PROMPT);
  else
    atomicAdd(seen, 1u);
  atomicOr(const_cast<uint32_t*>(p.marks) + static_cast<long long>(b) * p.words + (x >> 5), 1u << (x & 31));
}

// A request a CTA, an entry a thread: it counts unless the same id comes again behind it.
__global__ void __launch_bounds__(ASD_MAX_BIAS)
    bias_kernel(const __grid_constant__ RulesParams p, const int32_t* ids, const float* bias, int n,
                const int32_t* lengths, int32_t* status) {
  __shared__ int s_id[ASD_MAX_BIAS];
  pdl_signal_dependents();
  pdl_wait_prerequisites();
  const int i = threadIdx.x;
  for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
    const int length = lengths ? __ldcg(lengths + b) : n;
    const bool bad = length < 0 || length > n;
    if (bad && i == 0 && status) atomicOr(status + b, static_cast<int>(ASD_STATUS_LENGTH));
    int x = -1;
    if (!bad && i < length) x = __ldcg(ids + static_cast<long long>(b) * n + i);
    __syncthreads();
    s_id[i] = x;
    __syncthreads();
    if (x < 0) continue;
    if (x >= p.V) {
      if (status) atomicOr(status + b, static_cast<int>(ASD_STATUS_TOKEN));
      continue;
    }
    bool last = true;
    for (int k = i + 1; k < length; ++k) last = last && s_id[k] != x;
    if (!last) continue;
    const_cast<asd_token_record*>(p.records)[static_cast<long long>(b) * p.V + x].bias =
        __ldcg(bias + static_cast<long long>(b) * n + i);
    atomicOr(const_cast<uint32_t*>(p.marks) + static_cast<long long>(b) * p.words + (x >> 5), 1u << (x & 31));
  }
}

// ---------------------------------------------------------------- host side

int check_rules(const asd_token_rules* r) {
  if (!r) return ASD_ERR_NULL;
  if (r->B < 0 || r->V < 1 || r->allow_batch < 0 || r->allow_row < 0) return ASD_ERR_SHAPE;
  if (r->B > 0 && (!r->marks || !r->records)) return ASD_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(r->marks) % 4 != 0 || reinterpret_cast<uintptr_t>(r->records) % 8 != 0 ||
      reinterpret_cast<uintptr_t>(r->allow) % 4 != 0 || reinterpret_cast<uintptr_t>(r->repetition) % 4 != 0 ||
      reinterpret_cast<uintptr_t>(r->frequency) % 4 != 0 || reinterpret_cast<uintptr_t>(r->presence) % 4 != 0)
    return ASD_ERR_ALIGN;
  return ASD_OK;
}

RulesParams rules_params(const asd_token_rules* r) {
  RulesParams p = {};
  p.marks = r->marks;
  p.records = r->records;
  p.repetition = r->repetition;
  p.frequency = r->frequency;
  p.presence = r->presence;
  p.allow = r->allow;
  p.allow_batch = r->allow_batch;
  p.allow_row = r->allow_row;
  p.B = r->B;
  p.V = r->V;
  p.words = static_cast<int>((static_cast<long long>(r->V) + 31) / 32);
  return p;
}

template <typename T, int kU, bool kWrite>
int launch_rows(RulesParams p, long long chunks, cudaStream_t stream) {
  p.chunks = static_cast<int>(chunks);
  const int turns = (p.R + kMaxWarps - 1) / kMaxWarps;
  const int warps = (p.R + turns - 1) / turns;
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(p.B * chunks)),
                                            dim3(static_cast<unsigned>(32 * warps)), stream, &attr);
  if (cudaLaunchKernelEx(&cfg, rules_kernel<T, kU, kWrite>, p) != cudaSuccess) return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

template <typename T, bool kWrite>
int launch_rules(const RulesParams& p, cudaStream_t stream) {
  constexpr int kWide = 8, kNarrow = 2;
  auto chunks = [&](int u) { return (static_cast<long long>(p.V) + 32 * u * Elem<T>::kVec - 1) / (32 * u * Elem<T>::kVec); };
  if (p.B * chunks(kWide) > INT32_MAX) return ASD_ERR_SHAPE;
  if (p.B * chunks(kWide) * p.R >= 1200) return launch_rows<T, kWide, kWrite>(p, chunks(kWide), stream);
  return launch_rows<T, kNarrow, kWrite>(p, chunks(kNarrow), stream);
}

}  // namespace

extern "C" {

int asd_rules_verify(const asd_token_rules* rules, const void* logits, int dtype, int K, const int32_t* draft,
                     asd_ledger* ledger, float gate, int cap, int32_t* accepted_len, int32_t* committed,
                     int32_t* recovery, int32_t* row_argmax, float* row_regret, int32_t* status, void* workspace,
                     size_t workspace_bytes, asd_stream_t stream) {
  int rc = check_rules(rules);
  if (rc != ASD_OK) return rc;
  if (dtype != ASD_F32 && dtype != ASD_BF16) return ASD_ERR_DTYPE;
  rc = check_shape(rules->B, K, rules->V, dtype);
  if (rc != ASD_OK) return rc;
  if (rules->B == 0) return ASD_OK;
  if (!logits || !workspace || !accepted_len || !committed || !recovery || (K > 0 && !draft)) return ASD_ERR_NULL;
  if (ledger && (gate != gate || gate < 0.0f || cap < 0)) return ASD_ERR_CONTROL;
  const WorkspaceLayout l = layout_for(rules->B, K);
  if (workspace_bytes < l.total) return ASD_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0 ||
      reinterpret_cast<uintptr_t>(logits) % (dtype == ASD_F32 ? 4 : 2) != 0)
    return ASD_ERR_ALIGN;
  char* ws = static_cast<char*>(workspace);
  RulesParams p = rules_params(rules);
  p.logits = logits;
  p.draft = draft;
  p.R = K + 1;
  p.K = K;
  p.row_key = reinterpret_cast<unsigned long long*>(ws + l.row_key);
  p.draft_logit = reinterpret_cast<float*>(ws + l.draft_logit);
  p.flags = reinterpret_cast<unsigned*>(ws + l.flags);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  rc = dtype == ASD_F32 ? launch_rules<float, false>(p, s) : launch_rules<__nv_bfloat16, false>(p, s);
  if (rc != ASD_OK) return rc;

  VerifyParams q = {};  // without logits: the selection takes a zero maximum as it is
  q.B = rules->B;
  q.K = K;
  q.V = q.v_total = rules->V;
  q.nblk = 1;
  q.draft = draft;
  q.ledger = ledger;
  q.gate = gate;
  q.cap = cap;
  q.accepted_len = accepted_len;
  q.committed = committed;
  q.recovery = recovery;
  q.row_argmax = row_argmax;
  q.row_regret = row_regret;
  q.status = status;
  q.row_key = p.row_key;
  q.draft_logit = p.draft_logit;
  q.done = reinterpret_cast<unsigned long long*>(ws + l.done);
  q.flags = p.flags;
  q.error = reinterpret_cast<unsigned*>(ws + l.error);
  return ledger ? launch_select<float, false>(q, true, s) : launch_select<float, true>(q, true, s);
}

int asd_rules_logits(const asd_token_rules* rules, const void* logits, int dtype, int rows, const int32_t* draft,
                     void* out, asd_stream_t stream) {
  int rc = check_rules(rules);
  if (rc != ASD_OK) return rc;
  if (dtype != ASD_F32 && dtype != ASD_BF16) return ASD_ERR_DTYPE;
  rc = check_shape(rules->B, rows - 1, rules->V, dtype);
  if (rc != ASD_OK) return rc;
  if (rules->B == 0) return ASD_OK;
  if (!logits || !out) return ASD_ERR_NULL;
  const uintptr_t es = dtype == ASD_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(logits) % es != 0 || reinterpret_cast<uintptr_t>(out) % es != 0) return ASD_ERR_ALIGN;
  RulesParams p = rules_params(rules);
  p.logits = logits;
  p.out = out;
  p.draft = draft;
  p.R = rows;
  p.K = draft ? rows - 1 : 0;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return dtype == ASD_F32 ? launch_rules<float, true>(p, s) : launch_rules<__nv_bfloat16, true>(p, s);
}

int asd_tokens_record(const asd_token_rules* rules, const int32_t* tokens, int n, const int32_t* token_len, int prompt,
                      int32_t* status, asd_stream_t stream) {
  const int rc = check_rules(rules);
  if (rc != ASD_OK) return rc;
  constexpr int kThreads = 256;
  const long long total = static_cast<long long>(rules->B) * n;
  if (n < 0 || total / kThreads >= INT32_MAX) return ASD_ERR_SHAPE;
  if (total == 0) return ASD_OK;
  if (!tokens) return ASD_ERR_NULL;
  const void* const words[] = {tokens, token_len, status};
  for (const void* x : words)
    if (reinterpret_cast<uintptr_t>(x) % 4 != 0) return ASD_ERR_ALIGN;
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg =
      pdl_config(dim3(static_cast<unsigned>((total + kThreads - 1) / kThreads)), dim3(kThreads),
                 reinterpret_cast<cudaStream_t>(stream), &attr);
  if (cudaLaunchKernelEx(&cfg, record_kernel, rules_params(rules), tokens, n, token_len, prompt ? 1 : 0, status) !=
      cudaSuccess)
    return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

int asd_tokens_bias(const asd_token_rules* rules, const int32_t* ids, const float* bias, int n, const int32_t* length,
                    int32_t* status, asd_stream_t stream) {
  const int rc = check_rules(rules);
  if (rc != ASD_OK) return rc;
  if (n < 0 || n > ASD_MAX_BIAS) return ASD_ERR_SHAPE;
  if (rules->B == 0 || n == 0) return ASD_OK;
  if (!ids || !bias) return ASD_ERR_NULL;
  const void* const words[] = {ids, bias, length, status};
  for (const void* x : words)
    if (reinterpret_cast<uintptr_t>(x) % 4 != 0) return ASD_ERR_ALIGN;
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(rules->B)), dim3(ASD_MAX_BIAS),
                                            reinterpret_cast<cudaStream_t>(stream), &attr);
  if (cudaLaunchKernelEx(&cfg, bias_kernel, rules_params(rules), ids, bias, n, length, status) != cudaSuccess)
    return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

}  // extern "C"
