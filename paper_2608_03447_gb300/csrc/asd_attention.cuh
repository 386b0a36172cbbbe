// libasd: what the two attention kernels (asd_attention.cu on the CUDA cores,
// asd_attention_tc.cu on the tensor cores) share: parameters and the deal of the
// work to CTAs.
//
// Work. A unit is one row tile (some of a request's T * group query rows that
// share a key/value head, row t * group + g; those of tokens that exist) against
// all the tiles of key/value slots that it sees. All units' tiles, one request
// after the other, form one sequence that is cut into contiguous ranges of equal
// work, one a CTA, whatever the requests' lengths. A tile is one work item, but
// three of a unit whose rows are too many for one softmax group and two of one
// whose rows are not, where a call has both (61 tokens, 5 query heads on one, four
// contexts of 90000: 348 us, with equal tiles 394; four of 40000: heads of 64, 40
// tokens, groups of 8, 89 against 97; heads of 128, 70 tokens, groups of 4, 192
// against 217; 300 tokens, groups of one, 200 against 218; 32 requests of up to 30
// tokens on up to 8000, groups of 8, 83.1 against 83.2). A tile belongs to the range
// that its first item is in, and ranges have at least as many items as a tile, so
// that none is without tiles. Lengths are device data, so every CTA adds them up
// itself. A unit that a range's end cuts is in pieces: each CTA leaves its piece's
// softmax statistics and unnormalised sums in the workspace, and the one that
// arrives last adds them up in the order of the slots, so results do not depend on
// who that is.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "asd.h"
#include "asd_cache.cuh"
#include "asd_device.cuh"

namespace asd_detail {

constexpr int kAttnMaxCtas = 320;  // of one launch: a counter and two pieces each
constexpr int kAttnScan = 32;      // requests of a CTA's range whose lengths it keeps: one a lane
constexpr int kAttnWorkMost = 3, kAttnWorkLeast = 2;  // of a tile, where a call has both kinds

struct AttnParams {
  CacheView cache;
  const char* q;
  long long q_batch, q_token, q_head;
  char* out;
  float* lse;
  const int32_t* kv_len;
  const int32_t* new_len;
  const uint32_t* mask;
  int mask_words;
  int32_t* status;
  unsigned* error;
  unsigned* counters;  // [kAttnMaxCtas] arrivals at the unit that starts in a CTA's range and ends beyond it
  float* part_ml;      // [2 * grid][rows of a unit][2] running maximum (log2 units) and sum
  float* part_o;       // [2 * grid][rows of a unit][D], in the kernel's own order
  int B, T, q_heads, heads, group, D;
  PageDiv by_group;
  int unit_rows, row_tiles;
  int group_rows;  // tensor cores: rows of a softmax group
  bool weighted;   // whether a tile's work depends on that
  float scale_log2;
};

struct AttnRequest {
  int ctx;  // slots that every row sees
  int n;    // new tokens
};

// A request's lengths, clamped to what its row of the page table covers.
__device__ __forceinline__ AttnRequest attn_request(const AttnParams& p, int b, bool* bad) {
  AttnRequest r;
  r.ctx = __ldcg(p.kv_len + b);
  r.n = p.new_len ? __ldcg(p.new_len + b) : p.T;
  *bad = r.ctx < 0 || r.n < 0 || r.n > p.T || static_cast<long long>(r.ctx) + r.n > p.cache.slots;
  if (*bad) r.ctx = r.n = 0;
  return r;
}

// Slots that a row tile of a request sees: none where it has no rows of tokens
// that exist; a chain's rows see nothing past their own token.
__device__ __forceinline__ int attn_span(const AttnParams& p, const AttnRequest& r, int row_tile) {
  const int row0 = row_tile * p.unit_rows;
  if (row0 >= r.n * p.group) return 0;
  if (p.mask) return r.ctx + r.n;
  const int last = p.by_group.quot(row0 + p.unit_rows - 1);
  return r.ctx + (last < r.n ? last + 1 : r.n);
}

template <int kTile>
__device__ __forceinline__ int attn_tiles(const AttnParams& p, const AttnRequest& r, int row_tile) {
  const int span = attn_span(p, r, row_tile);
  return span > 0 ? (span - 1) / kTile + 1 : 0;
}

__device__ __forceinline__ int attn_tile_work(const AttnParams& p, const AttnRequest& r, int row_tile) {
  if (!p.weighted) return 1;
  return r.n * p.group - row_tile * p.unit_rows > p.group_rows ? kAttnWorkMost : kAttnWorkLeast;
}
// Tiles that begin among a unit's first `items` items.
__device__ __forceinline__ int attn_tiles_of(int items, int work) {
  const unsigned n = static_cast<unsigned>(items);
  return static_cast<int>(work == 1 ? n : work == kAttnWorkLeast ? (n + kAttnWorkLeast - 1) / kAttnWorkLeast
                                                                 : (n + kAttnWorkMost - 1) / kAttnWorkMost);
}

template <int kTile>
__device__ __forceinline__ int attn_head_work(const AttnParams& p, const AttnRequest& r) {  // of each of its heads
  int w = 0;
#pragma unroll 1
  for (int i = 0; i < p.row_tiles; ++i) w += attn_tiles<kTile>(p, r, i) * attn_tile_work(p, r, i);
  return w;
}

// The output rows of tokens that do not exist, which no unit has: zeros and
// -infinity. Threads `tid` of `threads` of every CTA.
template <typename T>
__device__ __forceinline__ void attn_zero_rows(const AttnParams& p, int tid, int threads) {
  for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
    bool bad;
    const AttnRequest r = attn_request(p, b, &bad);
    if (r.n == p.T || __ldcg(p.error)) continue;
    const long long row = (static_cast<long long>(b) * p.T + r.n) * p.q_heads;
    const long long rows = static_cast<long long>(p.T - r.n) * p.q_heads, bytes = rows * p.D * sizeof(T);
    char* dst = p.out + row * p.D * sizeof(T);
    if (((reinterpret_cast<uintptr_t>(dst) | static_cast<uintptr_t>(bytes)) & 15) == 0) {
      for (long long i = tid; i < bytes / 16; i += threads) reinterpret_cast<uint4*>(dst)[i] = make_uint4(0, 0, 0, 0);
    } else {
      for (long long i = tid; i < rows * p.D; i += threads) reinterpret_cast<T*>(dst)[i] = Store<T>::narrow(0.0f);
    }
    if (p.lse)
      for (long long i = tid; i < rows; i += threads) p.lse[row + i] = -INFINITY;
  }
}

// Flags every request: a CTA has given up a wait, or the workspace says that one
// has. What a CTA leaves out may be any request's (units in pieces have no last
// CTA then), so it does not say which. Threads `tid` of `threads`.
__device__ __forceinline__ void attn_incomplete(int32_t* status, int B, int tid, int threads) {
  if (!status) return;
  for (int b = tid; b < B; b += threads) atomicOr(status + b, static_cast<int>(ASD_STATUS_INCOMPLETE));
}

// What a CTA works out before it starts. Work is counted in 32 bits (the entry
// point refuses what would not fit).
struct AttnDeal {
  int begin, end;  // this CTA's work items; none where begin == end
  int each, more;  // items of a CTA; that have one more
  int b;           // request of the first item
  int b_first;     // that request's first item
  int cached;      // requests b .. b + cached - 1 are in `request`
  AttnRequest request[kAttnScan];
};

// By one warp: adds up the requests' work, a block of consecutive requests a
// lane, finds the lane where this CTA's range begins, and again in that block until
// it is one request: two rounds of loads for up to 128 requests, three for 256.
// Every CTA starts with this, so it is short, one loop for all rounds (code that
// runs once comes from beyond the instruction cache), and the walk that follows
// divides as little as it can. 160 requests took 4.5 us of 43 when a warp went
// through them 32 at a time, twice.
// Flags requests whose lengths are out of range; where the workspace's error word
// is set, all requests, and the range is empty.
template <int kTile>
__device__ __forceinline__ void attn_deal(const AttnParams& p, AttnDeal& d) {
  const int lane = threadIdx.x & 31, c = blockIdx.x;
  const unsigned error = __ldcg(p.error);  // in one round trip with the first lengths
  if (lane == 0) d.begin = d.end = 0;
  int b = 0, count = p.B, b_first = 0;  // the block, and the work before it
  int total = 0, each = 0, more = 0, begin = 0, at = 0;
  AttnRequest r = {0, 0};
#pragma unroll 1
  for (bool first = true;; first = false) {
    const int per = (count - 1) / 32 + 1;
    const int from = b + lane * per, to = min(from + per, b + count);
    int mine = 0;
    constexpr int kBatch = 4;
#pragma unroll 1
    for (int i0 = 0; i0 < per; i0 += kBatch) {
      AttnRequest some[kBatch];
      bool bad[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) some[i] = attn_request(p, min(from + i0 + i, p.B - 1), &bad[i]);
      if (i0 == 0) r = some[0];
#pragma unroll 1
      for (int i = 0; from + i0 + i < to && i < kBatch; ++i) {
        const AttnRequest x = i == 0 ? some[0] : i == 1 ? some[1] : i == 2 ? some[2] : some[3];
        mine += attn_head_work<kTile>(p, x) * p.heads;
      }
      if (first && !error && c == 0 && p.status)
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (bad[i] && from + i0 + i < to) atomicOr(p.status + from + i0 + i, static_cast<int>(ASD_STATUS_LENGTH));
    }
    int before = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(kFull, before, off);
      if (lane >= off) before += o;
    }
    before += b_first - mine;
    if (first) {
      total = __shfl_sync(kFull, before + mine, 31);
      const int ctas = total == 0 ? 0 : max(1, min(p.weighted ? total / kAttnWorkMost : total,
                                                   static_cast<int>(gridDim.x)));
      if (error || c >= ctas) {
        if (error && c == 0) attn_incomplete(p.status, p.B, lane, 32);
        __syncwarp();
        return;
      }
      each = total / ctas;
      more = total - each * ctas;
      begin = c * each + min(c, more);
    }
    const unsigned holds = __ballot_sync(kFull, mine > 0 && before <= begin && begin < before + mine);
    if (!holds) {  // the lengths have changed meanwhile
      __syncwarp();
      return;
    }
    at = __ffs(holds) - 1;
    b_first = __shfl_sync(kFull, before, at);
    if (per == 1) break;
    const int end = b + count;
    b += at * per;
    count = min(per, end - b);
  }
  // the lengths of the request and of those after it that the last round has read
  const int who = min(lane + at, 31);
  const AttnRequest next = {__shfl_sync(kFull, r.ctx, who), __shfl_sync(kFull, r.n, who)};
  b += at;
  d.request[lane] = next;
  if (lane == 0) {
    d.begin = begin;
    d.end = begin + each + (c < more ? 1 : 0);
    d.each = each;
    d.more = more;
    d.b = b;
    d.b_first = b_first;
    d.cached = min(p.B - b, kAttnScan - at);
  }
  __syncwarp();
}

// A walk over the CTA's range, unit by unit.
template <int kTile>
struct AttnWalk {
  const AttnParams& p;
  const AttnDeal& d;
  int b, h, row_tile;
  AttnRequest r;
  int tiles;  // the unit's
  int work;   // of each of them
  int at;     // the unit's first item
  int j0;     // the first tile that is this CTA's

  __device__ __forceinline__ AttnWalk(const AttnParams& p_, const AttnDeal& d_) : p(p_), d(d_) {}
  // to the first unit, if the range has any
  __device__ __forceinline__ void start() {
    at = d.end;
    if (d.begin == d.end) return;
    b = d.b;
    load();
    // find the unit that holds the first item
    const int per_head = attn_head_work<kTile>(p, r);
    int in = d.begin - d.b_first;
    h = in / per_head;
    in -= h * per_head;
    row_tile = 0;
    for (;;) {
      measure();
      if (in < tiles * work) break;
      in -= tiles * work;
      ++row_tile;
    }
    at = d.begin - in;
    j0 = attn_tiles_of(in, work);
    if (j0 == tiles) next();  // inside its last tile, which is the range's before
  }
  __device__ __forceinline__ void measure() {
    tiles = attn_tiles<kTile>(p, r, row_tile);
    work = attn_tile_work(p, r, row_tile);
  }
  __device__ __forceinline__ void load() {
    const int i = b - d.b;
    bool bad;
    r = i < d.cached ? d.request[i] : attn_request(p, b, &bad);
  }
  __device__ __forceinline__ bool more() const { return at < d.end; }
  __device__ __forceinline__ int j1() const {  // this CTA has tiles j0 .. j1 - 1
    const int in = d.end - at;
    return in >= tiles * work ? tiles : attn_tiles_of(in, work);
  }
  __device__ __forceinline__ void next() {
    at += tiles * work;
    if (at >= d.end) return;
    j0 = 0;
    do {
      if (++row_tile == p.row_tiles) {
        row_tile = 0;
        if (++h == p.heads) {
          h = 0;
          if (++b >= p.B) {  // the lengths have changed meanwhile
            at = d.end;
            return;
          }
          load();
        }
      }
      measure();
    } while (tiles == 0);  // no rows of tokens that exist
  }
  __device__ __forceinline__ bool whole() const { return j0 == 0 && d.end - at >= (tiles - 1) * work + 1; }
  __device__ __forceinline__ int span() const { return attn_span(p, r, row_tile); }
  __device__ __forceinline__ int row0() const { return row_tile * p.unit_rows; }
  // rows of the unit, of tokens that exist
  __device__ __forceinline__ int rows() const { return min(p.unit_rows, r.n * p.group - row0()); }
  // the workspace slot of this CTA's piece, and the unit's CTAs
  __device__ __forceinline__ int piece() const { return 2 * static_cast<int>(blockIdx.x) + (j0 == 0 ? 1 : 0); }
  __device__ __forceinline__ int first_cta() const { return j0 == 0 ? static_cast<int>(blockIdx.x) : cta_of(at); }
  __device__ __forceinline__ int last_cta() const {
    return j1() == tiles ? static_cast<int>(blockIdx.x) : cta_of(at + (tiles - 1) * work);
  }
  __device__ __forceinline__ int cta_of(int item) const {
    const int cut = d.more * (d.each + 1);
    return item < cut ? item / (d.each + 1) : d.more + (item - cut) / d.each;
  }
};

// Bit i: whether a row of token t sees slot j0 + i (i < 32; r.n > t). Slots past the span are not seen.
__device__ __forceinline__ uint32_t attn_sees(const AttnParams& p, const AttnRequest& r, int b, int t, int j0) {
  const int u0 = j0 - r.ctx;  // the first bit's new token; negative: context
  if (u0 <= -32) return 0xffffffffu;
  uint32_t bits = 0;
  if (!p.mask) {
    const int see = min(t + 1, r.n) - u0;  // the first `see` bits
    return see >= 32 ? 0xffffffffu : see <= 0 ? 0u : (1u << see) - 1u;
  }
  const uint32_t* row = p.mask + (static_cast<long long>(b) * p.T + t) * p.mask_words;
  // word w of the row, without bits at or past n
  auto word = [&](int w) -> uint32_t {
    if (w < 0 || 32 * w >= r.n) return 0u;
    const uint32_t x = __ldcg(row + w);
    return r.n - 32 * w >= 32 ? x : x & ((1u << (r.n - 32 * w)) - 1u);
  };
  if (u0 < 0) {
    bits = (word(0) << -u0) | ((1u << -u0) - 1u);
  } else {
    bits = __funnelshift_r(word(u0 >> 5), word((u0 >> 5) + 1), u0 & 31);
  }
  return bits;
}

// Workspace: the error word first (where asd_workspace_error reads it), the
// counters at a place of their own for every shape (they are zero between calls;
// the pieces are not), then the pieces.
struct AttnLayout {
  size_t error, counters, ml, o, total;
};
inline AttnLayout attn_layout(int ctas, int unit_rows, int dim) {
  AttnLayout l;
  l.error = 0;
  l.counters = 256;
  l.ml = align_up(l.counters + 4 * kAttnMaxCtas, 256);
  l.o = align_up(l.ml + 2 * static_cast<size_t>(ctas) * unit_rows * 8, 256);
  l.total = align_up(l.o + 2 * static_cast<size_t>(ctas) * unit_rows * dim * 4, 256);
  return l;
}

}  // namespace asd_detail
