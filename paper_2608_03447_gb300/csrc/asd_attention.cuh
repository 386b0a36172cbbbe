// libasd: what the two attention kernels (asd_attention.cu on the CUDA cores,
// asd_attention_tc.cu on the tensor cores) share: parameters and the deal of the
// work to CTAs.
//
// Work. A unit is one row tile (some of a request's T * group query rows that
// share a key/value head, row t * group + g) against all the tiles of key/value
// slots that it sees. All units' tiles, one request after the other, form one
// sequence that is cut into equal contiguous ranges, one a CTA, whatever the
// requests' lengths: no CTA has more than one tile more than another. Lengths
// are device data, so every CTA adds them up itself. A unit that a range's end
// cuts is in pieces: each CTA leaves its piece's softmax statistics and
// unnormalised sums in the workspace, and the one that arrives last adds them up
// in the order of the slots, so results do not depend on who that is.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "asd.h"
#include "asd_cache.cuh"
#include "asd_device.cuh"

namespace asd_detail {

constexpr int kAttnMaxCtas = 320;  // of one launch: a counter and two pieces each
constexpr int kAttnScan = 32;      // requests of a CTA's range whose lengths it keeps

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
  int unit_rows, row_tiles;
  float scale;
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

// Slots that a row tile of a request sees: none where it has no rows; a chain's
// rows see nothing past their own token.
__device__ __forceinline__ int attn_span(const AttnParams& p, const AttnRequest& r, int row_tile) {
  const int row0 = row_tile * p.unit_rows;
  if (row0 >= r.n * p.group) return 0;
  if (p.mask) return r.ctx + r.n;
  const int last = (row0 + p.unit_rows - 1) / p.group;
  return r.ctx + (last < r.n ? last + 1 : r.n);
}

template <int kTile>
__device__ __forceinline__ int attn_tiles(const AttnParams& p, const AttnRequest& r, int row_tile) {
  const int span = attn_span(p, r, row_tile);
  return span > kTile ? (span - 1) / kTile + 1 : 1;  // a unit that sees nothing still has its rows to write
}

template <int kTile>
__device__ __forceinline__ long long attn_request_tiles(const AttnParams& p, const AttnRequest& r) {
  long long w = 0;
  for (int i = 0; i < p.row_tiles; ++i) w += attn_tiles<kTile>(p, r, i);
  return w * p.heads;
}

// What a CTA works out before it starts.
struct AttnDeal {
  long long total;    // tiles of all units
  long long begin, end;  // this CTA's
  int ctas;           // that have any
  int b;              // request of the first tile
  long long b_first;  // that request's first tile
  int cached;         // requests b .. b + cached - 1 are in `request`
  unsigned error;     // the workspace's error word
  AttnRequest request[kAttnScan];
  long long sums[33];  // scratch of the scan
};

// The CTA that holds tile x of `total` dealt to `ctas`: cta c has tiles from floor(c * total / ctas) on.
__device__ __forceinline__ int attn_cta_of(long long x, long long total, int ctas) {
  return static_cast<int>(((x + 1) * ctas - 1) / total);
}

// By the whole CTA: adds up the requests' tiles, a chunk of blockDim.x requests
// at a time, and finds where this CTA's range begins. Returns false where it has
// none, or where the workspace's error word is set, with the requests flagged.
// Flags requests whose lengths are out of range.
template <int kTile>
__device__ bool attn_deal(const AttnParams& p, AttnDeal& d) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nwarps = blockDim.x >> 5;
  // total, and what comes before this thread's request of the last chunk
  long long total = 0, before = 0, mine = 0;
  AttnRequest r = {0, 0};
  if (tid == 0) d.error = __ldcg(p.error);  // in one round trip with the lengths
  const int chunks = (p.B + blockDim.x - 1) / blockDim.x;
  auto scan = [&](int chunk) {
    const int b = chunk * static_cast<int>(blockDim.x) + tid;
    mine = 0;
    if (b < p.B) {
      bool bad;
      r = attn_request(p, b, &bad);
      mine = attn_request_tiles<kTile>(p, r);
      if (bad && blockIdx.x == 0 && p.status) atomicOr(p.status + b, static_cast<int>(ASD_STATUS_LENGTH));
    }
    long long inc = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const long long o = __shfl_up_sync(kFull, inc, off);
      if (lane >= off) inc += o;
    }
    __syncthreads();
    if (lane == 31) d.sums[warp] = inc;
    __syncthreads();
    long long base = total, all = 0;
    for (int w = 0; w < nwarps; ++w) {
      if (w < warp) base += d.sums[w];
      all += d.sums[w];
    }
    before = base + inc - mine;
    total += all;
  };
  for (int c = 0; c < chunks; ++c) scan(c);
  if (d.error) {
    if (blockIdx.x == 0 && p.status)
      for (int b = tid; b < p.B; b += blockDim.x) atomicOr(p.status + b, static_cast<int>(ASD_STATUS_INCOMPLETE));
    return false;
  }
  const long long w = total;
  const int ctas = w < static_cast<long long>(gridDim.x) ? static_cast<int>(w) : static_cast<int>(gridDim.x);
  const long long c = blockIdx.x;
  if (c >= ctas) return false;
  const long long begin = c * w / ctas, end = (c + 1) * w / ctas;
  auto place = [&](int chunk) {
    const int b = chunk * static_cast<int>(blockDim.x) + tid;
    if (b < p.B && mine > 0 && before <= begin && begin < before + mine) {
      d.b = b;
      d.b_first = before;
    }
  };
  if (chunks == 1) {
    place(0);
  } else {
    total = 0;
    for (int k = 0; k < chunks; ++k) {
      scan(k);
      place(k);
    }
  }
  __syncthreads();
  if (chunks == 1) {
    if (tid < p.B && tid >= d.b && tid < d.b + kAttnScan) d.request[tid - d.b] = r;
  } else if (tid < kAttnScan && d.b + tid < p.B) {
    bool bad;
    d.request[tid] = attn_request(p, d.b + tid, &bad);
  }
  if (tid == 0) {
    d.total = w;
    d.begin = begin;
    d.end = end;
    d.ctas = ctas;
    d.cached = p.B - d.b < kAttnScan ? p.B - d.b : kAttnScan;
  }
  __syncthreads();
  return true;
}

// One role's walk over the CTA's range, unit by unit. Few words of state: the
// roles of the tensor-core kernel keep it in registers beside their tiles.
template <int kTile>
struct AttnWalk {
  const AttnParams& p;
  const AttnDeal& d;
  int b, h, row_tile;
  AttnRequest r;
  int tiles;  // the unit's
  int j0;     // the first of them that is this CTA's
  int left;   // tiles of the CTA's range from there on

  __device__ __forceinline__ AttnWalk(const AttnParams& p_, const AttnDeal& d_) : p(p_), d(d_) {
    b = d.b;
    load();
    // find the unit that holds the first tile
    long long at = d.begin - d.b_first;
    long long per_head = 0;
    for (int i = 0; i < p.row_tiles; ++i) per_head += attn_tiles<kTile>(p, r, i);
    h = static_cast<int>(at / per_head);
    at -= h * per_head;
    row_tile = 0;
    for (;;) {
      tiles = attn_tiles<kTile>(p, r, row_tile);
      if (at < tiles) break;
      at -= tiles;
      ++row_tile;
    }
    j0 = static_cast<int>(at);
    left = static_cast<int>(d.end - d.begin);
  }
  __device__ __forceinline__ void load() {
    const int i = b - d.b;
    bool bad;
    r = i < d.cached ? d.request[i] : attn_request(p, b, &bad);
  }
  __device__ __forceinline__ bool more() const { return left > 0; }
  __device__ __forceinline__ int j1() const { return min(tiles, j0 + left); }  // this CTA has tiles j0 .. j1 - 1
  __device__ __forceinline__ void next() {
    left -= j1() - j0;
    if (left <= 0) return;
    j0 = 0;
    if (++row_tile == p.row_tiles) {
      row_tile = 0;
      if (++h == p.heads) {
        h = 0;
        ++b;
        load();
      }
    }
    tiles = attn_tiles<kTile>(p, r, row_tile);
  }
  __device__ __forceinline__ bool whole() const { return j0 == 0 && left >= tiles; }
  __device__ __forceinline__ int span() const { return attn_span(p, r, row_tile); }
  __device__ __forceinline__ int row0() const { return row_tile * p.unit_rows; }
  // rows of the unit that exist in the output, and those of tokens that exist
  __device__ __forceinline__ int rows() const { return min(p.unit_rows, p.T * p.group - row0()); }
  __device__ __forceinline__ int live_rows() const { return min(rows(), max(0, r.n * p.group - row0())); }
  // the workspace slot of this CTA's piece, and the unit's CTAs
  __device__ __forceinline__ int piece() const { return 2 * static_cast<int>(blockIdx.x) + (j0 == 0 ? 1 : 0); }
  __device__ __forceinline__ long long unit_first() const { return d.end - left - j0; }
  __device__ __forceinline__ int first_cta() const { return attn_cta_of(unit_first(), d.total, d.ctas); }
  __device__ __forceinline__ int last_cta() const { return attn_cta_of(unit_first() + tiles - 1, d.total, d.ctas); }
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
