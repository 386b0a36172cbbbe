// libasd: what the two kernels of asd_kv_weigh (asd_weigh.cu on the CUDA cores,
// asd_weigh_tc.cu on the tensor cores) share.
//
// A unit of the deal (asd_attention.cuh) is a request's key/value head, one row
// tile of all its rows, so the sequence that is cut into the CTAs' ranges is that
// of the slots' tiles. Every slot's weight is a sum of its own: nothing is merged,
// and results do not depend on the cut.
#pragma once

#include "asd_attention.cuh"

namespace asd_detail {

struct WeighParams {
  AttnParams a;  // T: rows; unit_rows: T * group; cache.slots: not past the weights' width
  const float* lse;
  const float* weight;
  float* weight_out;
  const int32_t* path;
  int tokens;  // of q and lse
  int width;
  float decay;
  float scale_rest;  // what a.scale_log2 is short of scale * log2(e)
};

// No kernel of this entry point has a workspace: its error word for the deal, always 0.
static __device__ unsigned g_weigh_no_error;

__device__ __forceinline__ AttnParams weigh_deal_params(const WeighParams& p) {
  AttnParams a = p.a;
  a.error = &g_weigh_no_error;
  return a;
}

// Row r (token row r / group) of request b: its token in q and lse; -1 where its path leads nowhere.
__device__ __forceinline__ int weigh_token(const WeighParams& p, int b, int row) {
  if (!p.path) return row;
  const int t = __ldcg(p.path + static_cast<long long>(b) * p.a.T + row);
  if (static_cast<unsigned>(t) < static_cast<unsigned>(p.tokens)) return t;
  if (p.a.status) atomicOr(p.a.status + b, static_cast<int>(ASD_STATUS_PATH));
  return -1;
}

// What a row's exponentials are taken with: exp(z - lse) = exp2(z' - x) * y with z' in
// log2 units, x the rounded lse and y what that rounding lost (near 1; 0: the row adds
// nothing). Without y it would be in every weight of the row alike, up to 2^-20 where
// the lse is 16; likewise the scale has two parts.
struct RowScale {
  float x, y;
};
__device__ __forceinline__ float row_lse(const WeighParams& p, int b, int token, int head) {
  if (token < 0) return INFINITY;
  return __ldcg(p.lse + (static_cast<long long>(b) * p.tokens + token) * p.a.q_heads + head);
}
__device__ __forceinline__ RowScale row_scale(float lse) {
  RowScale r = {0.0f, 0.0f};
  if (fabsf(lse) == INFINITY) return r;
  r.x = lse * 1.4426950408889634f;
  const float lost = fmaf(lse, 1.4426950408889634f, -r.x) + lse * 1.9259629911266175e-8f;
  r.y = fabsf(r.x) == INFINITY ? 1.0f : exp2f(-lost);  // from 2.4e38 on nothing says what was lost
  return r;
}

bool weigh_tc_takes(const asd_kv_cache* cache, const WeighParams& p);
int launch_weigh_tc(const asd_kv_cache* cache, const WeighParams& p, cudaStream_t stream);

}  // namespace asd_detail
