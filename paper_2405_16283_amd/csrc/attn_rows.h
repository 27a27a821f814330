// Attention rows summed one by one over what they see, sixteen lanes to a row: where something that a row does not see is
// infinite or NaN, which the matrix cores would multiply by a weight of zero.  Many times slower than the kernels that
// fall back on it.
#pragma once

#include "attn_rule.h"

namespace tn {
namespace {

// One side's tile grid, seen from one head.
template <typename T, int HD>
struct Side {
  void* const* t;
  int nc, trows, tc, rows;
  int c0;       // first column of the head
  bool whole;   // the head lies inside one column tile: ct, cin name it
  int ct, cin;
  __device__ Side(void* const* tiles, int nc_, int trows_, int tc_, int rows_, int h)
      : t(tiles), nc(nc_), trows(trows_), tc(tc_), rows(rows_), c0(h * HD), whole(tc_ % HD == 0), ct(c0 / tc_), cin(c0 - ct * tc_) {}
  // columns c..c+3 of the head in row `row`
  __device__ f32x4 at(int row, int c) const {
    if (whole) {
      const int rt = row / trows;
      return ld4_global((const T*)t[rt * nc + ct] + (size_t)(row - rt * trows) * tc + cin + c);
    }
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = ld_global(tile_elem<T>(t, nc, trows, tc, row, c0 + c + i));
    return v;
  }
  // the same where the tiles hold the transpose
  __device__ f32x4 at_t(int row, int c) const {
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = ld_global(tile_elem_t<T>(t, nc, trows, tc, rows, row, c0 + c + i));
    return v;
  }
};

__device__ __forceinline__ float dot4(f32x4 a, f32x4 b) { return fmaf(a[0], b[0], fmaf(a[1], b[1], fmaf(a[2], b[2], a[3] * b[3]))); }
__device__ __forceinline__ float row_sum(float v) {  // over the sixteen lanes of a row
#pragma unroll
  for (int off = 1; off < 16; off <<= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// A finished row of attention: sums over the sum of weights, zeros where nothing was seen.
template <typename T>
__device__ __forceinline__ void st4_finished(T* o, f32x4 v, float l) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
  st4(o, l == 0.f ? (f32x4){0.f, 0.f, 0.f, 0.f} : v * inv);
}

// Rows first + id, first + id + stride, .. below `behind`; a lane's place among the sixteen of its row is threadIdx.x & 15.
template <typename T, int HD, bool RULE>
__device__ __forceinline__ void attn_by_rows(DeviceTables t, const OpDesc& d, int h, int first, int behind, int id, int stride) {
  const int* ax = t.aux + d.aux0;
  const int tq = ax[0], tk = ax[1], tc = ax[2], q_rows = ax[3], kv_rows = ax[4], nc = d.p.n_col_tiles, gw = nc * tc;
  void* const* Qt = t.ptrs + d.ptr0;
  void* const* Kt = Qt + d.p.n_q_tiles * nc;
  const Side<T, HD> Q(Qt, nc, tq, tc, q_rows, h), K(Kt, nc, tk, tc, kv_rows, h), V(Kt + d.p.n_kv_tiles * nc, nc, tk, tc, kv_rows, h);
  constexpr int C = HD / 64;  // pieces of four columns per lane: c0, c0 + 64
  const int c0 = (threadIdx.x & 15) * 4;
#pragma unroll 1
  for (int row = first + id; row < min(Q.rows, behind); row += stride) {
    f32x4 q[C], o[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      q[i] = Q.at(row, c0 + 64 * i) * d.p.scale;
      o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    float m = -INFINITY, l = 0.f;
    int from = 0, seen = min(K.rows, d.p.q_pos0 + row - d.p.k_pos0 + 1);
    float slope = 0.f;
    const Rule rule = RULE ? Rule(t, d) : Rule();
    if constexpr (RULE) {
      rule.visible(row, from, seen);
      slope = rule.slope(h);
    }
#pragma unroll 1
    for (int k = from; k < seen; ++k) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < C; ++i) s += dot4(q[i], K.at(k, c0 + 64 * i));
      s = row_sum(s);
      if constexpr (RULE) {
        float th;
        s = rule.score(s, slope, d.p.q_pos0 + row - d.p.k_pos0 - k, th);
      }
      const float mn = fmaxf(m, s), ms = mn == -INFINITY ? 0.f : mn;
      const float alpha = __expf(m - ms), p = __expf(s - ms);
      m = mn;
      l = l * alpha + p;
#pragma unroll
      for (int i = 0; i < C; ++i) o[i] = o[i] * alpha + (d.p.v_trans ? V.at_t(k, c0 + 64 * i) : V.at(k, c0 + 64 * i)) * p;
    }
    if constexpr (RULE)
      if (ax[kRuleFinish]) {
#pragma unroll
        for (int i = 0; i < C; ++i) st4_finished((T*)d.out + (size_t)row * gw + h * HD + c0 + 64 * i, o[i], l);
        continue;
      }
    float* out = (float*)d.out + (size_t)row * d.cols;
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) out[h * HD + c0 + 64 * i + e] = o[i][e];
    if (c0 == 0) {
      out[gw + h] = m;
      out[gw + gw / HD + h] = l;
    }
  }
}

// The same for the gradients: own rows are queries (MODE 1) or keys (2, 3).
template <typename T, int HD, int MODE, bool RULE, typename Stat>
__device__ __forceinline__ void attn_bwd_by_rows(const DeviceTables& t, const OpDesc& d, const Side<T, HD>& Q, const Side<T, HD>& K, const Side<T, HD>& V,
                                                 const Side<T, HD>& D, int h, int gw, int first, int behind, int id, int stride, Stat stat) {
  constexpr int C = HD / 64;
  const Side<T, HD>&own = MODE == 1 ? Q : K, &other = MODE == 1 ? K : Q;
  const int c0 = (threadIdx.x & 15) * 4;
  auto v_at = [&](int r, int c) { return d.p.v_trans ? V.at_t(r, c) : V.at(r, c); };
#pragma unroll 1
  for (int row = first + id; row < min(own.rows, behind); row += stride) {
    f32x4 m1[C], m2[C], acc[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      m1[i] = own.at(row, c0 + 64 * i);
      m2[i] = MODE == 1 ? D.at(row, c0 + 64 * i) : v_at(row, c0 + 64 * i);
      acc[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    int begin = MODE == 1 ? 0 : max(0, d.p.k_pos0 + row - d.p.q_pos0);
    int end = MODE == 1 ? min(K.rows, d.p.q_pos0 + row - d.p.k_pos0 + 1) : Q.rows;
    float slope = 0.f;
    const Rule rule = RULE ? Rule(t, d) : Rule();
    if constexpr (RULE) {
      if (MODE == 1) rule.visible(row, begin, end);
      else begin = 0;
      slope = rule.slope(h);
    }
#pragma unroll 1
    for (int o = begin; o < end; ++o) {
      if constexpr (RULE && MODE >= 2) {
        int lo, hi;
        rule.visible(o, lo, hi);
        if (row < lo || row >= hi) continue;
      }
      float s = 0.f, dp = 0.f;
#pragma unroll
      for (int i = 0; i < C; ++i) {
        s += dot4(m1[i], other.at(o, c0 + 64 * i));
        if (MODE != 3) dp += dot4(m2[i], MODE == 1 ? v_at(o, c0 + 64 * i) : D.at(o, c0 + 64 * i));
      }
      const int q = MODE == 1 ? row : o;
      float z = row_sum(s) * d.p.scale, th = 0.f;
      if constexpr (RULE) z = rule.score(z, slope, d.p.q_pos0 + q - d.p.k_pos0 - (MODE == 1 ? o : row), th);
      float p = __expf(z - stat(q, 0));
      if (MODE != 3) p *= (row_sum(dp) - stat(q, 1)) * d.p.scale;
      if (RULE && MODE != 3) p *= 1.f - th * th;
#pragma unroll
      for (int i = 0; i < C; ++i) acc[i] += (MODE == 3 ? D.at(o, c0 + 64 * i) : other.at(o, c0 + 64 * i)) * p;
    }
    T* out = (T*)d.out + (size_t)row * gw + h * HD + c0;
#pragma unroll
    for (int i = 0; i < C; ++i) st4(out + 64 * i, acc[i]);
  }
}

}  // namespace
}  // namespace tn
