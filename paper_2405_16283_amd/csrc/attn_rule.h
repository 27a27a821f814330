// The score rule of attention vertices (score_cap, slopes, spans; see turnip.h) as the kernels see it.
#pragma once

#include "device.h"
#include "kernels.h"

#include <climits>

namespace tn {
namespace {

typedef __attribute__((ext_vector_type(2))) int int2_t;
constexpr float kLog2e = 1.44269504088896340736f;

// tanh to a few units in the last place: for small arguments its series up to x^13 (the next term is below 2^-23 of the sum at
// 0.45), for others 1 - 2 / (exp(2 x) + 1), which loses half a bit of what it keeps there.
__device__ __forceinline__ float tanh_f32(float x) {
  const float a = fabsf(x), e = __builtin_amdgcn_exp2f(a * (2.f * kLog2e));
  const float large = __builtin_copysignf(1.f - 2.f / (e + 1.f), x), y = x * x;
  float p = fmaf(y, 21844.f / 6081075.f, -1382.f / 155925.f);
  p = fmaf(y, p, 62.f / 2835.f);
  p = fmaf(y, p, -17.f / 315.f);
  p = fmaf(y, p, 2.f / 15.f);
  p = fmaf(y, p, -1.f / 3.f);
  return a < 0.45f ? fmaf(x * y, p, x) : large;  // (a NaN takes the second form and stays one)
}

struct Rule {
  float cap, inv_cap;
  const float* slopes;    // of the heads of the column group, or null
  void* const* spans;     // one tensor per Q row tile, or null
  int tq, q_pos0, k_pos0, kv_rows, causal;
  bool one_tile;          // of queries
  __device__ Rule() : cap(0.f), inv_cap(0.f), slopes(nullptr), spans(nullptr), tq(1), q_pos0(0), k_pos0(0), kv_rows(0), causal(0), one_tile(true) {}
  __device__ Rule(const DeviceTables& t, const OpDesc& d) {
    const int* ax = t.aux + d.aux0;
    cap = __int_as_float(ax[kRuleCap]);
    inv_cap = cap > 0.f ? 1.f / cap : 0.f;
    slopes = ax[kRuleSlopes] >= 0 ? (const float*)t.ptrs[d.ptr0 + ax[kRuleSlopes]] : nullptr;
    spans = ax[kRuleSpans] >= 0 ? t.ptrs + d.ptr0 + ax[kRuleSpans] : nullptr;
    tq = ax[0];
    kv_rows = ax[4];
    q_pos0 = d.p.q_pos0;
    k_pos0 = d.p.k_pos0;
    causal = d.p.causal;
    one_tile = d.p.n_q_tiles == 1;
  }
  __device__ float slope(int h) const { return slopes ? get_global(slopes + h) : 0.f; }
  // The keys of the block that query row `row` (a row that exists) sees: [lo, hi), counted from the block's first; lo == hi == 0 for none.
  __device__ void visible(int row, int& lo, int& hi) const {
    int2_t span = {INT_MIN, INT_MAX};
    if (spans) {
      const int rt = one_tile ? 0 : row / tq;
      span = get_global((const int2_t*)spans[rt] + (row - rt * tq));
    }
    clip(row, span, lo, hi);
  }
  // The same of its span.  (Positions are any integers: clipped to the block before its start is taken off.)
  __device__ void clip(int row, int2_t span, int& lo, int& hi) const {
    lo = min(max(span.x, k_pos0), k_pos0 + kv_rows) - k_pos0;
    hi = min(max(span.y, k_pos0), k_pos0 + kv_rows) - k_pos0;
    if (causal) hi = min(hi, q_pos0 + row - k_pos0 + 1);
    if (lo >= hi) lo = hi = 0;
  }
  // The query behind the last whose position lies in the span of query `row`.
  __device__ int span_end(int row, int q_rows) const {
    const int rt = one_tile ? 0 : row / tq;
    return min(max(get_global((const int*)spans[rt] + (size_t)(row - rt * tq) * 2 + 1), q_pos0), q_pos0 + q_rows) - q_pos0;
  }
  // The score by the rule, of z = scale * q.k; th: tanh(z / cap), whose square the gradient needs
  __device__ float score(float z, float slope, int distance, float& th) const {
    if (cap > 0.f) {
      th = tanh_f32(z * inv_cap);
      z = cap * th;
    }
    return slopes ? z - slope * fabsf((float)distance) : z;
  }
};

}  // namespace
}  // namespace tn
