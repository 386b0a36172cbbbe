// libasd: logits under a request's rules (penalties, biases, grammar):
// asd_rules_verify, asd_rules_logits, asd_tokens_record, asd_tokens_bias.
//
//   z <- z > 0 ? z / rho : z rho   tokens said or in the prompt
//   z <- z - c f - p               tokens said c > 0 times, the drafts before the row among them
//   z <- z + bias                  tokens that have a record
//   z <- -inf                      tokens that the grammar does not allow
//
// Few tokens have a record, and hardly any of them matter to a maximum: penalties and
// biases that lower a logit leave it at most what it was. asd_rules_verify streams
// the rows as asd_verify does, a warp a unit of one row with a running maximum of the
// logits as they are (only the grammar's bits turn elements into -infinity), and looks
// at the marks of the unit's best token alone: if it has a record, it is worked out,
// taken out of the unit, and the next best one is looked for. What may be larger than
// its logit (a bias above 0, a penalty that rewards) is other warps' work: each looks
// through the marks of a part of the vocabulary for such tokens and takes their
// logits in every row. Both kinds merge (value, index) keys into the rows' slots,
// from which the selection runs as after any other row stage.
// asd_rules_logits writes what it reads, so there a warp lists its own unit's tokens.
//
// What bounds it: 32 requests of 9 rows of 151936 (bf16, 4000 tokens said, 300 biases,
// grammars) take 24 to 25 us, selection included, for 95 MB (3.9 TB/s): instructions,
// 660 a unit of 4 KB where asd_verify has 244 (the grammar's masks 127, the marks and
// what is worked out 118, the tokens that may grow 76, the search for the index 63).
// Without grammars and biases the same rows take 20.6 us, with biases 21.5, with
// grammars 23.1; 256 requests of 5 rows of 129280 in fp32 119 us (5.6 TB/s). 64 x 5
// rows of 129280 written in fp32 take 59 us for 331 MB (5.6 TB/s): memory. What else
// was measured for the 32 requests: all rows of a part by one CTA, its marked tokens
// excluded from the maximum and taken one by one in every row, 50 us; the same by CTAs
// of their own 33 to 48 us (1.3 million gathers of a logit); only those that may grow, a
// lane's token in one row after the other, 33 us. The selection by a request's last CTA
// instead of a kernel of its own saves the host 2.5 us of a call (9.8 to 7.2 us) and costs
// the GPU 2.2 (one request, consecutive calls in a graph 5.1 to 7.3 us; 64 requests of 2
// rows of 32000 6.5 to 9.7).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>

#include "asd.h"
#include "asd_device.cuh"
#include "asd_launch.cuh"
#include "asd_select.cuh"

namespace {

using namespace asd_detail;

constexpr uint32_t kTimes = 0x7fffffffu;
constexpr uint32_t kLowest = 0x007fffffu;  // ordered_bits(-infinity)
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
  int chunks;             // asd_rules_logits: units of a row
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

// Elements whose bit of `keep` is 0 become -infinity. Four bits at a time are
// spread over the signs of a word's bytes by a multiplication, and a byte
// permutation that repeats signs makes masks of them: 13 instructions for 8 elements.
__device__ __forceinline__ uint32_t sign_masks(uint32_t spread, uint32_t which) {
  uint32_t m;
  asm("prmt.b32 %0, %1, 0, %2;" : "=r"(m) : "r"(spread), "r"(which));
  return m;
}
__device__ __forceinline__ uint32_t choose(uint32_t mask, uint32_t w, uint32_t other) { return (w & mask) | (other & ~mask); }
__device__ __forceinline__ uint4 only(const uint4& v, uint32_t keep, float) {
  constexpr uint32_t kNone = 0xff800000u;
  const uint32_t a = (keep & 15u) * 0x10204080u;
  return make_uint4(choose(sign_masks(a, 0x8888u), v.x, kNone), choose(sign_masks(a, 0x9999u), v.y, kNone),
                    choose(sign_masks(a, 0xaaaau), v.z, kNone), choose(sign_masks(a, 0xbbbbu), v.w, kNone));
}
__device__ __forceinline__ uint4 only(const uint4& v, uint32_t keep, __nv_bfloat16) {
  constexpr uint32_t kNone = 0xff80ff80u;
  const uint32_t a = (keep & 15u) * 0x10204080u, b = ((keep >> 4) & 15u) * 0x10204080u;
  return make_uint4(choose(sign_masks(a, 0x9988u), v.x, kNone), choose(sign_masks(a, 0xbbaau), v.y, kNone),
                    choose(sign_masks(b, 0x9988u), v.z, kNone), choose(sign_masks(b, 0xbbaau), v.w, kNone));
}

// VN u + t: element t of v[u] is the first that equals best, one of them does. One lane looks, so it stops at its vector.
template <typename T, int u, int kU>
__device__ __forceinline__ int first_of(const uint4 (&v)[kU], float best) {
  if constexpr (u + 1 < kU) {
    if (widest(max_of<T>(v[u]), T()) != best) return first_of<T, u + 1>(v, best);
  }
  int at = 0;
#pragma unroll
  for (int t = Elem<T>::kVec - 1; t >= 0; --t)
    if (Elem<T>::lane(v[u], t) == best) at = t;
  return Elem<T>::kVec * u + at;
}

__device__ __forceinline__ float narrow(float v, float) { return v; }
__device__ __forceinline__ __nv_bfloat16 narrow(float v, __nv_bfloat16) { return __float2bfloat16_rn(v); }

// A request's penalties.
struct Penalties {
  float rho, f, pr;
  __device__ __forceinline__ Penalties(const RulesParams& p, int b) {
    rho = p.repetition ? __ldcg(p.repetition + b) : 1.0f;
    f = p.frequency ? __ldcg(p.frequency + b) : 0.0f;
    pr = p.presence ? __ldcg(p.presence + b) : 0.0f;
  }
  // Whether no logit grows, and none turns NaN (infinities less infinities; the products of counts below 2^31 are finite).
  __device__ __forceinline__ bool lower() const {
    return rho >= 1.0f && rho <= 1e30f && f >= 0.0f && f <= 1e20f && pr >= 0.0f && pr <= 1e30f;
  }
};

// The logit z of a token that has been said `times` times before the row.
__device__ __forceinline__ float changed_logit(const RulesParams& p, const Penalties& q, float z, uint32_t times,
                                               bool marked, uint2 record) {
  if (p.repetition && (times > 0u || (record.x & ASD_TOKEN_PROMPT)))
    z = z > 0.0f ? __fdiv_rn(z, q.rho) : __fmul_rn(z, q.rho);
  if (times > 0u) {
    z = __fsub_rn(z, __fmul_rn(static_cast<float>(times), q.f));
    z = __fsub_rn(z, q.pr);
  }
  return marked ? __fadd_rn(z, __uint_as_float(record.y)) : z;
}

// Bit i: whether draft i is this lane's token. `mine`: the lane's draft, `near` the lanes that may match.
__device__ __forceinline__ unsigned drafts_equal(int tok, int mine, unsigned near) {
  unsigned equal = 0;
  for (unsigned left = near; left; left &= left - 1) {
    const int i = __ffs(left) - 1;
    if (__shfl_sync(kFull, mine, i) == tok) equal |= 1u << i;
  }
  return equal;
}

// A word of a request's marks; its bits past the vocabulary may be anything and are dropped.
__device__ __forceinline__ uint32_t load_marks(const RulesParams& p, int b, int w) {
  if (w >= p.words) return 0u;
  const uint32_t x = __ldcg(p.marks + static_cast<long long>(b) * p.words + w);
  const int left = p.V - 32 * w;
  return left >= 32 ? x : x & ((1u << left) - 1u);
}

// Appends the tokens of this lane's words to the list, in order of the lanes. Returns how many a warp has.
template <int kN>
__device__ __forceinline__ int append_list(uint16_t* list, int at, const int (&word)[kN], const uint32_t (&all)[kN],
                                           const uint32_t (&mark)[kN]) {
  const int lane = threadIdx.x & 31;
  int n = 0;
#pragma unroll
  for (int i = 0; i < kN; ++i) n += __popc(all[i]);
  int before = n;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int o = __shfl_up_sync(kFull, before, off);
    if (lane >= off) before += o;
  }
  const int total = __shfl_sync(kFull, before, 31);
  before += at - n;
#pragma unroll
  for (int i = 0; i < kN; ++i)
    for (uint32_t left = all[i]; left; left &= left - 1) {
      const int bit = __ffs(left) - 1;
      list[before++] = static_cast<uint16_t>(32 * word[i] + bit + ((mark[i] >> bit) & 1u) * kMarked);
    }
  return total;
}

// A row's share of a CTA or warp: len elements from z on, as loose ones up to a 16-byte boundary, whole vectors, loose.
template <typename T>
struct Range {
  static constexpr int VN = Elem<T>::kVec;
  const T* z;
  int len, lead, nvec;
  __device__ __forceinline__ Range() {}
  __device__ __forceinline__ Range(const T* from, int n) : z(from), len(n) {
    lead = static_cast<int>((16u - static_cast<unsigned>(reinterpret_cast<uintptr_t>(z) & 15u)) & 15u) /
           static_cast<int>(sizeof(T));
    lead = lead < len ? lead : len;
    nvec = (len - lead) / VN;
  }
  __device__ __forceinline__ const uint4* vectors() const { return reinterpret_cast<const uint4*>(z + lead); }
  __device__ __forceinline__ bool has_loose() const { return lead > 0 || lead + nvec * VN < len; }
  // the loose element of this lane, or -1
  __device__ __forceinline__ int loose(int lane) const {
    const int at = lane < VN ? lane : lead + nvec * VN + lane - VN;
    return (lane < VN ? at < lead : lane < 2 * VN && at < len) ? at : -1;
  }
};

// ---------------------------------------------------------------- asd_rules_verify's row stage

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kMinBlocks = 8;
constexpr int kPart = 2048;  // tokens that a warp looks through for those that may grow

// n / d for n < 2^31 by a product.
struct Divide {
  unsigned mul, shift, by;
  void set(unsigned d) {
    unsigned l = 0;
    while ((1ull << l) < d) ++l;
    mul = static_cast<unsigned>((1ull << (31 + l)) / d + 1);
    shift = 31 + l;
    by = d;
  }
  __device__ __forceinline__ int quot(int n) const {
    return static_cast<int>((static_cast<unsigned long long>(static_cast<unsigned>(n)) * mul) >> shift);
  }
};

struct StreamPlan {
  Divide by_parts, by_ctas;
  int parts;     // units of a row
  int unit_ctas; // CTAs of a request that have kWarps units each,
  int part_ctas; // and those that have kWarps parts of the vocabulary each
};

__device__ __forceinline__ void merge_key(const RulesParams& p, long long row, unsigned long long key) {
  if (key != 0ull) atomicMax(p.row_key + row, key);
}

// By a warp: the tokens of a part that may grow, in all rows of the request; and the logits of the drafts that lie in
// it. A lane has two words of marks, and reads the biases of several tokens at once.
template <typename T>
__device__ __forceinline__ void growing_rows(const RulesParams& p, int b, int part, uint16_t* list) {
  constexpr int kN = kPart / 32 / 32;
  const int lane = threadIdx.x & 31;
  if (part > (p.V - 1) / kPart) return;
  const int t0 = part * kPart, len = min(kPart, p.V - t0);
  const int mine = lane < p.K ? __ldcg(p.draft + static_cast<long long>(b) * p.K + lane) - t0 : -1;
  unsigned long long mark = 0ull;  // bit 32 i + k: token 32 (32 i + lane) + k
#pragma unroll
  for (int i = 0; i < kN; ++i)
    mark |= static_cast<unsigned long long>(load_marks(p, b, t0 / 32 + 32 * i + lane)) << (32 * i);
  const Penalties penalties(p, b);
  const bool lower = penalties.lower();
  const unsigned near = __ballot_sync(kFull, mine >= 0 && mine < len);
  const T* z = static_cast<const T*>(p.logits) + static_cast<long long>(b) * p.R * p.V + t0;
  const uint32_t* allow = p.allow ? p.allow + b * p.allow_batch + t0 / 32 : nullptr;
  const asd_token_record* records = p.records + static_cast<long long>(b) * p.V + t0;
  auto token = [&](int bit) { return 32 * (bit & ~31) + 32 * lane + (bit & 31); };
  auto bit_of = [&](int tok) { return (tok >> 10) * 32 + (tok & 31); };  // of lane tok / 32 % 32

  unsigned long long grows = 0ull;
  if (lower) {  // a bias above 0; one that makes -infinity, or NaN of an infinite logit
    constexpr int kAtOnce = 4;
    for (unsigned long long left = mark; __any_sync(kFull, left != 0ull);) {
      float bias[kAtOnce];
      int bit[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        bit[k] = __ffsll(static_cast<long long>(left)) - 1;
        bias[k] = 0.0f;
        if (bit[k] >= 0) bias[k] = records[token(bit[k])].bias;
        left &= left - 1;
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k)
        if (!(bias[k] <= 0.0f && bias[k] > -INFINITY)) grows |= 1ull << bit[k];
    }
  } else {  // any; and drafts in the rows behind them
    grows = mark;
    for (unsigned left = near; left; left &= left - 1) {
      const int x = __shfl_sync(kFull, mine, __ffs(left) - 1);
      if ((x >> 5 & 31) == lane) grows |= 1ull << bit_of(x);
    }
  }

  bool nan = false;
  if (near) {  // a draft's logit in its own row
    const unsigned equal = drafts_equal(mine, mine, near);
    const unsigned long long marks = __shfl_sync(kFull, mark, mine >> 5 & 31);
    if ((near >> lane) & 1u) {
      const bool marked = (marks >> bit_of(mine)) & 1ull;
      const bool may = !allow || ((__ldcg(allow + lane * p.allow_row + mine / 32) >> (mine & 31)) & 1u);
      const float x = Elem<T>::load_cg(z, static_cast<long long>(lane) * p.V + mine);
      const uint2 record = marked ? *reinterpret_cast<const uint2*>(records + mine) : make_uint2(0u, 0u);
      const uint32_t times = (record.x & kTimes) + __popc(equal & ((1u << lane) - 1u));
      p.draft_logit[static_cast<long long>(b) * p.R + lane] =
          may ? changed_logit(p, penalties, x, times, marked, record) : -INFINITY;
    }
  }

  // A token in a row is a lane's: few tokens in all rows are one round of loads. Few of them lead their row, whose units
  // have mostly been merged by now: a slot is only touched where that shows.
  int n = __popcll(grows), before = n;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int o = __shfl_up_sync(kFull, before, off);
    if (lane >= off) before += o;
  }
  const int count = __shfl_sync(kFull, before, 31);
  before -= n;
  for (unsigned long long left = grows; left; left &= left - 1) {
    const int bit = __ffsll(static_cast<long long>(left)) - 1;
    list[before++] = static_cast<uint16_t>(token(bit) + ((mark >> bit) & 1ull) * kMarked);
  }
  __syncwarp();
  const int items = count * p.R;  // at most kPart * (ASD_MAX_K + 1)
  for (int i0 = 0; i0 < items; i0 += 32) {
    const int i = i0 + lane;
    const bool has = i < items;
    const int e = i / p.R, j = i - e * p.R, x = has ? list[e] : 0, tok = x & (kMarked - 1);
    const bool marked = (x & kMarked) != 0;
    const long long row = static_cast<long long>(b) * p.R + j;
    float value = 0.0f;
    uint32_t may = kFull;
    uint2 record = make_uint2(0u, 0u);
    unsigned long long most = 0ull;
    if (has) {
      value = Elem<T>::load_cg(z, static_cast<long long>(j) * p.V + tok);
      if (allow) may = __ldcg(allow + j * p.allow_row + (tok >> 5));
      if (marked) record = *reinterpret_cast<const uint2*>(records + tok);
      most = __ldcg(p.row_key + row);
    }
    const unsigned equal = drafts_equal(tok, mine, near);
    if (has) {
      const uint32_t times = (record.x & kTimes) + __popc(equal & ((1u << j) - 1u));
      value = changed_logit(p, penalties, value, times, marked, record);
      if (!((may >> (tok & 31)) & 1u)) value = -INFINITY;
      nan = nan || value != value;
      const unsigned long long key = make_key(value, static_cast<uint32_t>(t0 + tok));
      if (value == value && key > most) merge_key(p, row, key);
    }
  }
  nan = __any_sync(kFull, nan);
  if (nan && lane == 0) atomicOr(p.flags + b, ASD_STATUS_NAN_LOGIT);
}

// Element t of a vector becomes -infinity.
__device__ __forceinline__ void take_out(uint4& v, int t, float) {
  constexpr uint32_t kNone = 0xff800000u;
  if (t == 0) v.x = kNone;
  if (t == 1) v.y = kNone;
  if (t == 2) v.z = kNone;
  if (t == 3) v.w = kNone;
}
__device__ __forceinline__ void take_out(uint4& v, int t, __nv_bfloat16) {
  const uint32_t mask = t & 1 ? 0xffffu : 0xffff0000u, none = 0xff80ff80u & ~mask;
  if (t >> 1 == 0) v.x = (v.x & mask) | none;
  if (t >> 1 == 1) v.y = (v.y & mask) | none;
  if (t >> 1 == 2) v.z = (v.z & mask) | none;
  if (t >> 1 == 3) v.w = (v.w & mask) | none;
}

// The key of len tokens from t0 on of request b's row j, every one by the rules. By a warp; out of line: a unit comes
// here when several of its best tokens have turned out to be lowered (most of the vocabulary is banned, say).
template <typename T>
__device__ __noinline__ unsigned long long work_out_all(const RulesParams& p, int b, int j, int t0, int len, bool& nan) {
  const int lane = threadIdx.x & 31;
  const T* z = static_cast<const T*>(p.logits) + (static_cast<long long>(b) * p.R + j) * p.V + t0;
  const uint32_t* marks = p.marks + static_cast<long long>(b) * p.words + t0 / 32;
  const uint32_t* allow = p.allow ? p.allow + b * p.allow_batch + j * p.allow_row + t0 / 32 : nullptr;
  const asd_token_record* records = p.records + static_cast<long long>(b) * p.V + t0;
  const Penalties penalties(p, b);
  const int mine = lane < j ? __ldcg(p.draft + static_cast<long long>(b) * p.K + lane) - t0 : -1;
  const unsigned said = __ballot_sync(kFull, mine >= 0 && mine < len);
  unsigned long long key = 0ull;
  bool bad = false;
  constexpr int kAtOnce = 4;
#pragma unroll 1
  for (int w0 = 0; 32 * w0 < len; w0 += kAtOnce) {  // a word of bits, a token a lane
    float x[kAtOnce];
    uint32_t mark[kAtOnce], may[kAtOnce];
    uint2 record[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int at = 32 * (w0 + k) + lane;
      x[k] = -INFINITY, mark[k] = 0u, may[k] = 0u, record[k] = make_uint2(0u, 0u);
      if (at >= len) continue;
      x[k] = Elem<T>::load_cg(z, at);
      mark[k] = __ldcg(marks + w0 + k);
      may[k] = allow ? __ldcg(allow + w0 + k) : kFull;
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      if ((mark[k] >> lane) & 1u) record[k] = *reinterpret_cast<const uint2*>(records + 32 * (w0 + k) + lane);
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int at = 32 * (w0 + k) + lane;
      const uint32_t times = (record[k].x & kTimes) + __popc(drafts_equal(at, mine, said));
      if (at >= len) continue;
      float value = changed_logit(p, penalties, x[k], times, (mark[k] >> lane) & 1u, record[k]);
      if (!((may[k] >> lane) & 1u)) value = -INFINITY;
      bad = bad || value != value;
      const unsigned long long other = make_key(value, static_cast<uint32_t>(t0 + at));
      if (value == value && other > key) key = other;
    }
  }
  nan = __any_sync(kFull, bad);
  return warp_max_key(key);
}

// kU: vectors a lane has of a unit, all in flight at once.
template <typename T, int kU>
__global__ void __launch_bounds__(kThreads, kMinBlocks)
    rules_stream_kernel(const __grid_constant__ RulesParams p, const __grid_constant__ StreamPlan q) {
  constexpr int VN = Elem<T>::kVec;
  constexpr int kUnit = 32 * kU * VN, kWords = kUnit / 32, kN = (kWords + 31) / 32;
  __shared__ uint32_t s_may[kWarps][kWords + 1];
  __shared__ uint16_t s_list[kWarps][kPart];
  __shared__ unsigned long long s_key[kWarps];
  __shared__ unsigned s_row[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_signal_dependents();
  // what may grow comes behind the request's units
  const int b = q.by_ctas.quot(static_cast<int>(blockIdx.x));
  const int at_cta = static_cast<int>(blockIdx.x) - b * static_cast<int>(q.by_ctas.by);
  if (at_cta >= q.unit_ctas) {
    pdl_wait_prerequisites();
    growing_rows<T>(p, b, (at_cta - q.unit_ctas) * kWarps + warp, s_list[warp]);
    return;
  }
  const int unit = at_cta * kWarps + warp, units = p.R * q.parts;
  const bool exists = unit < units;
  const int j = exists ? q.by_parts.quot(unit) : 0;
  const int t0 = exists ? (unit - j * q.parts) * kUnit : 0;
  const unsigned row = static_cast<unsigned>(b) * static_cast<unsigned>(p.R) + static_cast<unsigned>(j);
  const Range<T> r(static_cast<const T*>(p.logits) + static_cast<long long>(row) * p.V + t0, min(kUnit, p.V - t0));
  pdl_wait_prerequisites();

  // one round of loads: the elements, their marks and the grammar's bits, the block's drafts
  const bool whole = r.lead == 0 && r.nvec == 32 * kU;  // no index to bound, no bits across words
  uint4 v[kU];
  if (whole) {
#pragma unroll
    for (int u = 0; u < kU; ++u) v[u] = load_row(reinterpret_cast<const uint4*>(r.z) + lane + 32 * u);
  } else if (r.nvec > 0) {
    // past its end a unit repeats its last vector, which changes no maximum and no index
#pragma unroll
    for (int u = 0; u < kU; ++u) v[u] = load_row(r.vectors() + min(lane + 32 * u, r.nvec - 1));
  }
  const int at_loose = r.has_loose() ? r.loose(lane) : -1;
  float loose = -INFINITY;
  if (at_loose >= 0) loose = Elem<T>::load_cg(r.z, at_loose);
  uint32_t special[kN], may[kN];  // a bit an element: whether it is marked or a draft before the row; may come
  const uint32_t* marks = p.marks + static_cast<long long>(b) * p.words + t0 / 32;
  const uint32_t* allow = p.allow + b * p.allow_batch + j * p.allow_row + t0 / 32;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const int w = 32 * i + lane;
    special[i] = t0 / 32 + w < p.words ? __ldcg(marks + w) : 0u;
    if (p.allow) may[i] = t0 / 32 + w < p.words ? __ldcg(allow + w) : 0u;
  }
  const int mine = lane < p.K ? __ldcg(p.draft + static_cast<long long>(b) * p.K + lane) - t0 : -1;
  const unsigned said = __ballot_sync(kFull, lane < j && mine >= 0 && mine < r.len);
  uint32_t* words = s_may[warp];
  if (p.allow) {
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (32 * i + lane <= kWords) words[32 * i + lane] = may[i];
    if (kWords % 32 == 0 && lane == 0) words[kWords] = 0u;
    __syncwarp();
    if (whole) {
      const unsigned char* bits = reinterpret_cast<const unsigned char*>(words) + lane * VN / 8;
#pragma unroll
      for (int u = 0; u < kU; ++u) v[u] = only(v[u], static_cast<uint32_t>(bits[32 * u * VN / 8]) >> (lane * VN % 8), T());
    } else if (r.nvec > 0) {
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int at = r.lead + min(lane + 32 * u, r.nvec - 1) * VN;
        v[u] = only(v[u], __funnelshift_r(words[at >> 5], words[(at >> 5) + 1], at & 31), T());
      }
    }
    if (at_loose >= 0 && !((words[at_loose >> 5] >> (at_loose & 31)) & 1u)) loose = -INFINITY;
  }

  // The unit's best token, until it is one without rules or not better than those worked out; all together where several
  // have to be.
  constexpr int kOneByOne = 3;
  int worked = 0;
  unsigned long long key = 0ull;
  bool nan = false;
  for (bool again = false;; again = true) {
    const uint32_t loose_order = at_loose >= 0 ? ordered_bits(loose) : 0u;
    uint32_t order = 0u;
    float best = 0.0f;
    if (r.nvec > 0) {
      uint32_t m = max_of<T>(v[0]);
#pragma unroll
      for (int u = 1; u < kU; ++u) m = max_of(m, max_of<T>(v[u]), T());
      best = widest(m, T());
      order = ordered_bits(best);
    }
    if (!again) {
      nan = __any_sync(kFull, best != best || loose != loose);
      if (nan) break;
    }
    const uint32_t top = __reduce_max_sync(kFull, max(order, loose_order));
    uint32_t low = 0u;
    if (r.nvec > 0 && order == top) {
      const int at = first_of<T, 0>(v, best);
      low = 0xffffffffu - static_cast<uint32_t>(t0 + r.lead + min(lane + 32 * (at / VN), r.nvec - 1) * VN + at % VN);
    }
    if (at_loose >= 0 && loose_order == top) low = max(low, 0xffffffffu - static_cast<uint32_t>(t0 + at_loose));
    low = __reduce_max_sync(kFull, low);
    const unsigned long long found = (static_cast<unsigned long long>(top) << 32) | low;
    if (found <= key) break;
    const int at = static_cast<int>(0xffffffffu - low) - t0, w = at >> 5;
    uint32_t bits = 0u;
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (w / 32 == i) bits = __shfl_sync(kFull, special[i], w & 31);
    const bool marked = (bits >> (at & 31)) & 1u;
    unsigned equal = 0u;
    for (unsigned left = said; left; left &= left - 1) equal += __shfl_sync(kFull, mine, __ffs(left) - 1) == at;
    // nothing is left but -infinity: that rules leave as it is, or is one that may grow
    if ((!marked && equal == 0u) || top == kLowest) {
      key = found;
      break;
    }
    const Penalties penalties(p, b);
    const asd_token_record* records = p.records + static_cast<long long>(b) * p.V + t0;
    if (worked++ == kOneByOne) {
      key = work_out_all<T>(p, b, j, t0, r.len, nan);
      break;
    }
    const uint2 record = marked ? *reinterpret_cast<const uint2*>(records + at) : make_uint2(0u, 0u);
    const float value = changed_logit(p, penalties, ordered_value(top), (record.x & kTimes) + equal, marked, record);
    if (value == value) {
      const unsigned long long changed = make_key(value, static_cast<uint32_t>(t0 + at));
      key = changed > key ? changed : key;
    } else {
      nan = true;
    }
    // out of the unit, wherever it is (a repeated last vector has it too)
    const int e = at - r.lead;
    if (e >= 0 && e < r.nvec * VN) {
#pragma unroll
      for (int u = 0; u < kU; ++u)
        if (min(lane + 32 * u, r.nvec - 1) == e / VN) take_out(v[u], e % VN, T());
    } else if (at_loose == at) {
      loose = -INFINITY;
    }
  }
  if (nan && exists && lane == 0) atomicOr(p.flags + b, ASD_STATUS_NAN_LOGIT);

  // one reduction per row and CTA
  if (lane == 0) {
    s_key[warp] = exists ? key : 0ull;
    s_row[warp] = exists ? row : 0xffffffffu;
  }
  __syncthreads();
  if (warp != 0) return;
  const unsigned of = lane < kWarps ? s_row[lane] : 0xffffffffu;
  unsigned long long k = lane < kWarps ? s_key[lane] : 0ull;
#pragma unroll
  for (int d = 1; d < kWarps; d *= 2) {
    const unsigned long long o = __shfl_down_sync(kFull, k, d);
    if (__shfl_down_sync(kFull, of, d) == of && o > k) k = o;
  }
  const unsigned before = __shfl_up_sync(kFull, of, 1);
  if (of != 0xffffffffu && (lane == 0 || before != of)) merge_key(p, of, k);
}

// ---------------------------------------------------------------- asd_rules_logits

// A warp a unit of one row: the elements pass through shared memory, where the listed ones are changed in between, so
// that they are written with the rest. kU: vectors a lane has of a unit, all in flight at once.
template <typename T, int kU>
__global__ void __launch_bounds__(kThreads, kMinBlocks) rules_write_kernel(const __grid_constant__ RulesParams p) {
  constexpr int VN = Elem<T>::kVec;
  constexpr int kUnit = 32 * kU * VN, kWords = kUnit / 32, kN = (kWords + 31) / 32;
  constexpr int kList = kUnit < 512 ? kUnit : 512;  // tokens changed at once
  __shared__ __align__(16) T s_z[kWarps][kUnit + VN];
  __shared__ uint32_t s_allow[kWarps][kWords + 1];
  __shared__ uint16_t s_list[kWarps][kList];

  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long unit = static_cast<long long>(blockIdx.x) * kWarps + warp;
  pdl_signal_dependents();
  const long long row = unit / p.chunks;
  if (row >= static_cast<long long>(p.B) * p.R) return;
  const int t0 = static_cast<int>(unit - row * p.chunks) * kUnit;
  const int b = static_cast<int>(row / p.R), j = static_cast<int>(row - static_cast<long long>(b) * p.R);
  const Range<T> r(static_cast<const T*>(p.logits) + row * p.V + t0, min(kUnit, p.V - t0));
  T* const out = static_cast<T*>(p.out) + row * p.V + t0;
  const bool grammar = p.allow != nullptr;
  pdl_wait_prerequisites();

  uint4 v[kU];
#pragma unroll
  for (int u = 0; u < kU; ++u)
    if (lane + 32 * u < r.nvec) v[u] = load_row(r.vectors() + lane + 32 * u);
  const int at_loose = r.has_loose() ? r.loose(lane) : -1;
  T loose = {};
  if (at_loose >= 0) loose = r.z[at_loose];
  uint32_t mark[kN], all[kN];
  int word[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    word[i] = 32 * i + lane;
    mark[i] = all[i] = word[i] < kWords ? load_marks(p, b, t0 / 32 + word[i]) : 0u;
    if (grammar && word[i] <= kWords)
      s_allow[warp][word[i]] = word[i] < kWords && t0 / 32 + word[i] < p.words
                                   ? __ldcg(p.allow + b * p.allow_batch + j * p.allow_row + t0 / 32 + word[i])
                                   : 0u;
  }
  if (kWords % 32 == 0 && lane == 0) s_allow[warp][kWords] = 0u;
  const int mine = lane < p.K ? __ldcg(p.draft + static_cast<long long>(b) * p.K + lane) - t0 : -1;
  const unsigned said = __ballot_sync(kFull, lane < j && mine >= 0 && mine < r.len);  // drafts before the row, in the unit
  for (unsigned left = said; left; left &= left - 1) {
    const int x = __shfl_sync(kFull, mine, __ffs(left) - 1);
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (x >> 5 == word[i]) all[i] |= 1u << (x & 31);
  }
  const Penalties penalties(p, b);
  T* const z = s_z[warp] + (r.lead > 0 ? VN - r.lead : 0);  // so that vectors lie on 16-byte boundaries here too
  uint4* const vectors = reinterpret_cast<uint4*>(z + r.lead);
#pragma unroll
  for (int u = 0; u < kU; ++u)
    if (lane + 32 * u < r.nvec) vectors[lane + 32 * u] = v[u];
  if (at_loose >= 0) z[at_loose] = loose;

  // the listed tokens; all at once unless the list is too short for them
  int n = 0;
#pragma unroll
  for (int i = 0; i < kN; ++i) n += __popc(all[i]);
  n = __reduce_add_sync(kFull, n);
  const int each = n <= kList ? kWords : kList / 32;  // words at once
  for (int w0 = 0; w0 < kWords && n > 0; w0 += each) {
    uint32_t now[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) now[i] = word[i] >= w0 && word[i] < w0 + each ? all[i] : 0u;
    __syncwarp();
    const int count = append_list(s_list[warp], 0, word, now, mark);
    __syncwarp();
    for (int i0 = 0; i0 < count; i0 += 64) {
      int tok[2];
      bool marked[2];
      uint2 record[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int i = i0 + 32 * k + lane, x = i < count ? s_list[warp][i] : -1;
        tok[k] = x < 0 ? -1 : x & (kMarked - 1);
        marked[k] = x >= 0 && (x & kMarked);
        record[k] = make_uint2(0u, 0u);
        if (marked[k])
          record[k] = *reinterpret_cast<const uint2*>(p.records + static_cast<long long>(b) * p.V + t0 + tok[k]);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (i0 + 32 * k >= count) break;
        const uint32_t times = (record[k].x & kTimes) + __popc(drafts_equal(tok[k], mine, said));
        if (tok[k] >= 0)
          z[tok[k]] = narrow(changed_logit(p, penalties, Elem<T>::load(z, tok[k]), times, marked[k], record[k]), T());
      }
    }
  }
  __syncwarp();

  // what may not come is -infinity on the way out
  if (((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(r.z)) & 15u) == 0) {
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (lane + 32 * u < r.nvec) {
        uint4 x = vectors[lane + 32 * u];
        if (grammar) {
          const int at = r.lead + (lane + 32 * u) * VN;
          x = only(x, __funnelshift_r(s_allow[warp][at >> 5], s_allow[warp][(at >> 5) + 1], at & 31), T());
        }
        reinterpret_cast<uint4*>(out + r.lead)[lane + 32 * u] = x;
      }
    if (at_loose >= 0)
      out[at_loose] = !grammar || ((s_allow[warp][at_loose >> 5] >> (at_loose & 31)) & 1u) ? z[at_loose]
                                                                                           : narrow(-INFINITY, T());
  } else {
    for (int at = lane; at < r.len; at += 32)
      out[at] = !grammar || ((s_allow[warp][at >> 5] >> (at & 31)) & 1u) ? z[at] : narrow(-INFINITY, T());
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

// Many tokens of a request: a CTA has some thousand of them and sees by a bitmap of its own which it has met before.
// A mark is then one addition a word, and of a prompt's tokens the record is touched once each: 64 prompts of up to
// 8000 tokens, half of them repeated, 8.0 to 8.5 us, by a thread a token 9.8. At 2048 tokens, where it takes over,
// it gains only for many prompts: 64 of them 2.6 us against 2.8 (by 2047 tokens of a thread each), 8 of them 2.3
// against 1.6, and what was said (every record is touched) 3.1 and 2.7 against 2.8 and 1.6. Bound by what each record costs, 64 bytes
// of memory for four (25 MB read).
constexpr int kBulkThreads = 512, kBulkTokens = 4096;
constexpr int kBulkWords = 50000;  // of a bitmap that fits shared memory
__global__ void __launch_bounds__(kBulkThreads)
    record_many_kernel(const __grid_constant__ RulesParams p, const int32_t* tokens, int n, int parts,
                       const int32_t* token_len, int prompt, int32_t* status) {
  extern __shared__ uint32_t s_seen[];  // [words]
  pdl_signal_dependents();
  for (int w = threadIdx.x; w < p.words; w += kBulkThreads) s_seen[w] = 0u;
  __syncthreads();
  pdl_wait_prerequisites();
  const int b = static_cast<int>(blockIdx.x) / parts, from = (static_cast<int>(blockIdx.x) - b * parts) * kBulkTokens;
  const int length = token_len ? __ldcg(token_len + b) : n;
  if (length < 0 || length > n) {
    if (from == 0 && threadIdx.x == 0 && status) atomicOr(status + b, static_cast<int>(ASD_STATUS_LENGTH));
    return;
  }
  constexpr int kEach = kBulkTokens / kBulkThreads;
  int x[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int i = from + k * kBulkThreads + static_cast<int>(threadIdx.x);
    x[k] = i < length ? __ldcg(tokens + static_cast<long long>(b) * n + i) : -1;
  }
  asd_token_record* records = const_cast<asd_token_record*>(p.records) + static_cast<long long>(b) * p.V;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    if (x[k] < 0) continue;
    if (x[k] >= p.V) {
      if (status) atomicOr(status + b, static_cast<int>(ASD_STATUS_TOKEN));
      continue;
    }
    const uint32_t bit = 1u << (x[k] & 31), before = atomicOr(&s_seen[x[k] >> 5], bit);
    if (!prompt)
      atomicAdd(&records[x[k]].seen, 1u);
    else if (!(before & bit))
      atomicOr(&records[x[k]].seen, ASD_TOKEN_PROMPT);
  }
  __syncthreads();
  uint32_t* marks = const_cast<uint32_t*>(p.marks) + static_cast<long long>(b) * p.words;
  for (int w = threadIdx.x; w < p.words; w += kBulkThreads)
    if (s_seen[w]) atomicOr(marks + w, s_seen[w]);
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

constexpr int kMaxDevices = 64;

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

int launch_many(const RulesParams& p, const int32_t* tokens, int n, const int32_t* token_len, int prompt,
                int32_t* status, asd_stream_t stream) {
  static std::atomic<bool> ready[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return ASD_ERR_CUDA;
  if (dev < 0 || dev >= kMaxDevices) return ASD_ERR_DEVICE;
  if (!ready[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(record_many_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 4 * kBulkWords) !=
        cudaSuccess)
      return ASD_ERR_CUDA;
    ready[dev].store(true, std::memory_order_release);
  }
  const int parts = (n - 1) / kBulkTokens + 1;
  cudaLaunchAttribute attr;
  cudaLaunchConfig_t cfg = pdl_config(dim3(static_cast<unsigned>(p.B) * static_cast<unsigned>(parts)),
                                      dim3(kBulkThreads), reinterpret_cast<cudaStream_t>(stream), &attr);
  cfg.dynamicSmemBytes = 4 * static_cast<size_t>(p.words);
  if (cudaLaunchKernelEx(&cfg, record_many_kernel, p, tokens, n, parts, token_len, prompt ? 1 : 0, status) !=
      cudaSuccess)
    return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

template <typename T>
long long parts_of(int V, int vectors) {
  const long long n = 32ll * vectors * Elem<T>::kVec;
  return (V + n - 1) / n;
}

template <typename T, int kU>
int launch_write(RulesParams p, cudaStream_t stream) {
  p.chunks = static_cast<int>(parts_of<T>(p.V, kU));
  const unsigned units = static_cast<unsigned>(p.B) * static_cast<unsigned>(p.R) * static_cast<unsigned>(p.chunks);
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg = pdl_config(dim3((units + kWarps - 1) / kWarps), dim3(kThreads), stream, &attr);
  if (cudaLaunchKernelEx(&cfg, rules_write_kernel<T, kU>, p) != cudaSuccess) return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

template <typename T, int kU>
int launch_stream(const RulesParams& p, cudaStream_t stream) {
  StreamPlan q = {};
  q.parts = static_cast<int>(parts_of<T>(p.V, kU));
  q.unit_ctas = (p.R * q.parts + kWarps - 1) / kWarps;
  q.part_ctas = ((p.V - 1) / kPart + kWarps) / kWarps;
  q.by_parts.set(static_cast<unsigned>(q.parts));
  q.by_ctas.set(static_cast<unsigned>(q.unit_ctas + q.part_ctas));
  const unsigned ctas = static_cast<unsigned>(p.B) * static_cast<unsigned>(q.part_ctas + q.unit_ctas);
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg = pdl_config(dim3(ctas), dim3(kThreads), stream, &attr);
  if (cudaLaunchKernelEx(&cfg, rules_stream_kernel<T, kU>, p, q) != cudaSuccess) return ASD_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? ASD_OK : ASD_ERR_CUDA;
}

// Units of eight vectors a lane, or of four where those would be fewer than fill the GPU several times over: 1350 of the
// wide ones (two requests of 9 rows of 151936, bf16) 6.3 us against 5.7 of twice as many, 2700 7.0 against 6.2, 5400
// the same 9.9, 10800 13.9 against 15.2, 21600 24.2 against 28.7; written in fp32, 1200 5.2 against 4.8 us, 10200 16.9
// against 18.4. Units of two vectors are never the fastest (675 wide ones' rows: 5.3 us, as wide; of four 5.0).
constexpr int kWide = 8, kNarrow = 4;
constexpr long long kWideUnits = 5000;
template <typename T, bool kWrite>
int launch_rules(const RulesParams& p, cudaStream_t stream) {
  const long long wide = parts_of<T>(p.V, kWide) * p.B;
  if (wide * p.R > INT32_MAX / 8) return ASD_ERR_SHAPE;  // units and CTAs are counted in 32 bits
  const bool few = wide * p.R < kWideUnits;
  if (kWrite) return few ? launch_write<T, kNarrow>(p, stream) : launch_write<T, kWide>(p, stream);
  return few ? launch_stream<T, kNarrow>(p, stream) : launch_stream<T, kWide>(p, stream);
}

}  // namespace

extern "C" {

int asd_rules_verify(const asd_token_rules* rules, const asd_rules_block* block, asd_stream_t stream) {
  int rc = check_rules(rules);
  if (rc != ASD_OK) return rc;
  if (!block) return ASD_ERR_NULL;
  const asd_rules_block& a = *block;
  const int K = a.K;
  const int dtype = a.dtype & ~ASD_FLAG_EMPTY_ROWS;
  if (dtype != ASD_F32 && dtype != ASD_BF16) return ASD_ERR_DTYPE;
  rc = check_shape(rules->B, K, rules->V, dtype);
  if (rc != ASD_OK) return rc;
  if (rules->B == 0) return ASD_OK;
  if (!a.logits || !a.workspace || !a.accepted_len || !a.committed || !a.recovery || (K > 0 && !a.draft))
    return ASD_ERR_NULL;
  if (a.ledger && (a.gate != a.gate || a.gate < 0.0f || a.cap < 0)) return ASD_ERR_CONTROL;
  const WorkspaceLayout l = layout_for(rules->B, K);
  if (a.workspace_bytes < l.total) return ASD_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(a.workspace) % 16 != 0 ||
      reinterpret_cast<uintptr_t>(a.logits) % (dtype == ASD_F32 ? 4 : 2) != 0)
    return ASD_ERR_ALIGN;
  const void* const words[] = {a.draft, a.ledger, a.accepted_len, a.committed, a.recovery, a.row_argmax, a.row_regret,
                               a.status};
  for (const void* x : words)
    if (reinterpret_cast<uintptr_t>(x) % 4 != 0) return ASD_ERR_ALIGN;
  char* ws = static_cast<char*>(a.workspace);
  RulesParams p = rules_params(rules);
  p.logits = a.logits;
  p.draft = a.draft;
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
  q.draft = a.draft;
  q.ledger = a.ledger;
  q.gate = a.gate;
  q.cap = a.cap;
  q.accepted_len = a.accepted_len;
  q.committed = a.committed;
  q.recovery = a.recovery;
  q.row_argmax = a.row_argmax;
  q.row_regret = a.row_regret;
  q.status = a.status;
  q.row_key = p.row_key;
  q.draft_logit = p.draft_logit;
  q.done = reinterpret_cast<unsigned long long*>(ws + l.done);
  q.flags = p.flags;
  q.error = reinterpret_cast<unsigned*>(ws + l.error);
  q.flag_empty = dtype != a.dtype;
  return a.ledger ? launch_select<float, false, true>(q, true, s) : launch_select<float, true, true>(q, true, s);
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
  if (reinterpret_cast<uintptr_t>(logits) % es != 0 || reinterpret_cast<uintptr_t>(out) % es != 0 ||
      reinterpret_cast<uintptr_t>(draft) % 4 != 0)
    return ASD_ERR_ALIGN;
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
  const RulesParams p = rules_params(rules);
  if (n >= kBulkTokens / 2 && p.words <= kBulkWords) return launch_many(p, tokens, n, token_len, prompt, status, stream);
  const cudaLaunchConfig_t cfg =
      pdl_config(dim3(static_cast<unsigned>((total + kThreads - 1) / kThreads)), dim3(kThreads),
                 reinterpret_cast<cudaStream_t>(stream), &attr);
  if (cudaLaunchKernelEx(&cfg, record_kernel, p, tokens, n, token_len, prompt ? 1 : 0, status) !=
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
