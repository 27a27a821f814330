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

// minimum over the wavefront, as a scalar: exchanges inside the vector unit for each sixteen lanes, the four by scalars
template <int CTRL>
__device__ __forceinline__ int exchanged(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, false); }
__device__ __forceinline__ int wave_min(int v) {
  v = min(v, exchanged<0xB1>(v));   // neighbours
  v = min(v, exchanged<0x4E>(v));   // pairs
  v = min(v, exchanged<0x141>(v));  // the mirrored half of eight
  v = min(v, exchanged<0x140>(v));  // of sixteen
  return min(min(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)), min(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}

// Head and row block of a workgroup: the blocks that see most go first, of all heads, so that none of them is started when the others
// are nearly done.  Two workgroups share a compute unit from the start, the n-th and the one a chipful later: the first chipful goes
// from its smallest to its largest, so that the largest share theirs with the smallest of the second.  Where the heads
// are a multiple of 8, every XCD gets heads of its own, whose keys and values its L2 then serves to all their row blocks.
constexpr int kComputeUnits = 256;
__device__ __forceinline__ void head_and_rank(int bx, int total, int hpg, int& h, int& rank) {
  if ((hpg & 7) == 0) {
    const int per = hpg >> 3, one_each = min(kComputeUnits, total) >> 3;
    int n = bx >> 3;
    if (n < one_each) n = one_each - 1 - n;
    h = (bx & 7) * per + n % per;
    rank = n / per;
  } else {
    if (bx < kComputeUnits) bx = min(kComputeUnits, total) - 1 - bx;
    h = bx % hpg;
    rank = bx / hpg;
  }
}

// Whose turn is `rank`-th of `blocks` blocks of ROWS rows (queries, or keys)?  Without spans late queries and early keys see most under a
// causal mask.  With spans it goes by what a block's first and last row see: an estimate, which decides the order and nothing
// else.  Every workgroup finds the same order, each thread the place of one block (of at most 256; beyond, the order without spans).
// Three packed documents in 4096 rows of 32 heads: forward 123 us in the order without spans, 98 so, dQ 151 and 117, dK 247 and 178, dV 208 and
// 156.  (All heads' largest blocks before any smaller one costs nothing over one head after the other where launches are long.)
template <int ROWS, bool OWN_Q>
__device__ __forceinline__ int block_of_rank(const Rule& rule, int rank, int blocks, int my_rows, int q_rows, int* shared) {
  const int plain = OWN_Q ? blocks - 1 - rank : rank;
  if (!rule.spans || blocks > 256) return plain;
  const int tid = threadIdx.x;
  int mine = -1;
  if (tid < blocks) {
    mine = 0;
    int first = INT_MAX, behind = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = e ? min(my_rows, (tid + 1) * ROWS) - 1 : tid * ROWS;
      if (OWN_Q) {
        int lo, hi;
        rule.visible(row, lo, hi);
        if (lo < hi) {
          first = min(first, lo);
          behind = max(behind, hi);
        }
      } else {  // queries from the one at the key's own position to the end of that one's span
        const int q = min(max(row + rule.k_pos0 - rule.q_pos0, 0), q_rows - 1);
        first = min(first, q);
        behind = max(behind, rule.span_end(q, q_rows));
      }
    }
    if (first < behind) mine = behind - first;
  }
  shared[tid] = mine;
  __syncthreads();
  int place = 0;
  for (int j = 0; j < blocks; j += 4) {
    const int4 v = *(const int4*)(shared + j);
    const int e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) place += e[k] > mine || (e[k] == mine && j + k < tid);
  }
  if (tid < blocks && place == rank) shared[256] = tid;
  __syncthreads();
  const int block = __builtin_amdgcn_readfirstlane(shared[256]);
  __syncthreads();
  return block;
}

}  // namespace
}  // namespace tn
