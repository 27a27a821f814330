// Norm and rotation of the heads of queries and keys, forward and reverse: every head x of a row becomes
// n = x * rsqrt(mean x^2 + eps) * gain (where a norm is asked for), then its pairs (a, b) turn by the angle of
// the row's position, (a cos - b sin, a sin + b cos).  Reverse, with u the inverse rotation of dY and n = x * rsqrt(..):
// dX = rsqrt(..) * (u * gain - n * mean(u * gain * n)), and the gain's gradient is the sum of u * n over rows and heads.
//
// Angles are turns: position * turns per position in 64 bits (a position of 10^5 turns thousands of times, and 32
// bits would keep 1e-3 of the angle), of which the whole ones are dropped before sine and cosine are taken in 32.
// Statistics, products and sums are fp32 and every output is rounded once.
#include "device.h"
#include "kernels.h"

namespace tn {
namespace {

// A head's pairs in the order i = 0 .. head_dim / 2 - 1, those that turn first; the others stay.
struct Pairs {
  int half_rotary, head_dim;
  bool half;
  __device__ void elements(int i, int& a, int& b) const {
    if (i < half_rotary && half) {
      a = i;
      b = i + half_rotary;
    } else {
      a = 2 * i;
      b = 2 * i + 1;
    }
  }
  __device__ bool turns(int i) const { return i < half_rotary; }
};

// sine and cosine of what a position turns a pair by
__device__ __forceinline__ void turn(double position, double turns, float& sn, float& cs) {
  double a = position * turns;
  a -= rint(a);
  sincospif(2.f * (float)a, &sn, &cs);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// What a row's workgroup needs of its vertex.
struct Head {
  const int* ax;
  int rows, cols, head_dim, heads;
  Pairs pairs;
  bool norm;
  const double* turns;
  const int* positions;
  int pos0;
  float eps;
  __device__ Head(const DeviceTables& t, const OpDesc& d) {
    ax = t.aux + d.aux0;
    rows = ax[kHeadRows];
    cols = ax[kHeadCols];
    head_dim = d.p.head_dim;
    heads = cols / head_dim;
    pairs = {ax[kHeadRotary] / 2, head_dim, ax[kHeadHalf] != 0};
    norm = ax[kHeadNorm] != 0;
    turns = t.rope_theta + ax[kHeadTheta];
    positions = ax[kHeadPositions] ? (const int*)t.ptrs[d.ptr0 + d.n_in - 1] : nullptr;
    pos0 = d.p.pos0;
    eps = d.p.eps;
  }
  __device__ double position(int row) const { return (double)pos0 + (positions ? (double)positions[row] : (double)row); }
  __device__ float rstd(float sum) const { return 1.f / sqrtf(sum / (float)head_dim + eps); }
};

constexpr int kPer = 8;  // pairs per lane: heads of up to 1024 elements

// Any head size: a wavefront per row and head, lane by lane through its pairs.
template <typename T>
__global__ void __launch_bounds__(256) head_rope_kernel(DeviceTables t, Batch b) {
  const OpDesc& d = t.descs[b.at(blockIdx.y)];
  if ((int)blockIdx.x >= d.nblocks) return;
  const Head s(t, d);
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= (int64_t)s.rows * s.heads) return;
  const int row = (int)(id / s.heads), h = (int)(id % s.heads);
  const size_t at = (size_t)row * s.cols + (size_t)h * s.head_dim;
  const T* x = (const T*)t.ptrs[d.ptr0] + at;
  const T* gain = s.norm ? (const T*)t.ptrs[d.ptr0 + 1] : nullptr;
  T* o = (T*)d.out + at;
  float va[kPer], vb[kPer], ss = 0.f;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = lane + 64 * k;
    va[k] = vb[k] = 0.f;
    if (i >= s.head_dim / 2) continue;
    int ea, eb;
    s.pairs.elements(i, ea, eb);
    va[k] = ld(x + ea);
    vb[k] = ld(x + eb);
    ss += va[k] * va[k] + vb[k] * vb[k];
  }
  const float r = s.norm ? s.rstd(wave_sum(ss)) : 1.f;
  const double pos = s.position(row);
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = lane + 64 * k;
    if (i >= s.head_dim / 2) continue;
    int ea, eb;
    s.pairs.elements(i, ea, eb);
    float a = va[k], c = vb[k];
    if (s.norm) {
      a *= r * ld(gain + ea);
      c *= r * ld(gain + eb);
    }
    float sn = 0.f, cs = 1.f;
    if (s.pairs.turns(i)) turn(pos, s.turns[i], sn, cs);
    if (d.p.mode) sn = -sn;
    st(o + ea, a * cs - c * sn);
    st(o + eb, a * sn + c * cs);
  }
}

// The reverse of a head in registers: u (the inverse rotation of dY) and x of this lane's pairs, and 1 / rms.
template <typename T>
__device__ __forceinline__ float load_reverse(const Head& s, const T* dy, const T* x, double pos, int lane, float (&ua)[kPer], float (&ub)[kPer],
                                              float (&xa)[kPer], float (&xb)[kPer]) {
  float ss = 0.f;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = lane + 64 * k;
    ua[k] = ub[k] = xa[k] = xb[k] = 0.f;
    if (i >= s.head_dim / 2) continue;
    int ea, eb;
    s.pairs.elements(i, ea, eb);
    xa[k] = ld(x + ea);
    xb[k] = ld(x + eb);
    ss += xa[k] * xa[k] + xb[k] * xb[k];
    const float a = ld(dy + ea), c = ld(dy + eb);
    float sn = 0.f, cs = 1.f;
    if (s.pairs.turns(i)) turn(pos, s.turns[i], sn, cs);
    ua[k] = a * cs + c * sn;
    ub[k] = c * cs - a * sn;
  }
  return s.rstd(wave_sum(ss));
}

template <typename T>
__global__ void __launch_bounds__(256) head_rope_bwd_kernel(DeviceTables t, Batch b) {
  const OpDesc& d = t.descs[b.at(blockIdx.y)];
  if ((int)blockIdx.x >= d.nblocks) return;
  const Head s(t, d);
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= (int64_t)s.rows * s.heads) return;
  const int row = (int)(id / s.heads), h = (int)(id % s.heads);
  const size_t at = (size_t)row * s.cols + (size_t)h * s.head_dim;
  const T* gain = (const T*)t.ptrs[d.ptr0 + 2];
  float ua[kPer], ub[kPer], xa[kPer], xb[kPer], dot = 0.f;
  const float r = load_reverse(s, (const T*)t.ptrs[d.ptr0] + at, (const T*)t.ptrs[d.ptr0 + 1] + at, s.position(row), lane, ua, ub, xa, xb);
  T* o = (T*)d.out + at;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = lane + 64 * k;
    if (i >= s.head_dim / 2) continue;
    int ea, eb;
    s.pairs.elements(i, ea, eb);
    ua[k] *= ld(gain + ea);
    ub[k] *= ld(gain + eb);
    dot += ua[k] * xa[k] + ub[k] * xb[k];
  }
  const float m = wave_sum(dot) * r * r / (float)s.head_dim;  // mean(u gain n) * rsqrt(..): the second rsqrt(..) is n's below
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = lane + 64 * k;
    if (i >= s.head_dim / 2) continue;
    int ea, eb;
    s.pairs.elements(i, ea, eb);
    st(o + ea, r * (ua[k] - xa[k] * m));
    st(o + eb, r * (ub[k] - xb[k] * m));
  }
}

// Sums of the gain's gradient: a workgroup per kGainRows rows, a wavefront takes every fourth (row, head) of them and keeps its
// sums in registers; the four are added in order.
template <typename T>
__global__ void __launch_bounds__(256) head_gain_kernel(DeviceTables t, Batch b) {
  const OpDesc& d = t.descs[b.at(blockIdx.y)];
  if ((int)blockIdx.x >= d.nblocks) return;
  const Head s(t, d);
  __shared__ float part[4][1024];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int row0 = blockIdx.x * kGainRows, n = min(kGainRows, s.rows - row0);
  float ga[kPer], gb[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) ga[k] = gb[k] = 0.f;
  for (int64_t id = w; id < (int64_t)n * s.heads; id += 4) {
    const int row = row0 + (int)(id / s.heads), h = (int)(id % s.heads);
    const size_t at = (size_t)row * s.cols + (size_t)h * s.head_dim;
    float ua[kPer], ub[kPer], xa[kPer], xb[kPer];
    const float r = load_reverse(s, (const T*)t.ptrs[d.ptr0] + at, (const T*)t.ptrs[d.ptr0 + 1] + at, s.position(row), lane, ua, ub, xa, xb);
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      ga[k] += ua[k] * (xa[k] * r);
      gb[k] += ub[k] * (xb[k] * r);
    }
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = lane + 64 * k;
    if (i >= s.head_dim / 2) continue;
    int ea, eb;
    s.pairs.elements(i, ea, eb);
    part[w][ea] = ga[k];
    part[w][eb] = gb[k];
  }
  __syncthreads();
  float* o = (float*)d.out + (size_t)blockIdx.x * s.head_dim;
  for (int c = threadIdx.x; c < s.head_dim; c += 256) o[c] = (part[0][c] + part[1][c]) + (part[2][c] + part[3][c]);
}

// Sum of all rows of the operands: a workgroup per 32 columns, eight threads to a column, each every eighth row; their sums are
// added in order.
__global__ void __launch_bounds__(256) col_sum_kernel(DeviceTables t, Batch b) {
  const OpDesc& d = t.descs[b.at(blockIdx.y)];
  if ((int)blockIdx.x >= d.nblocks) return;
  __shared__ float part[8][32];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), g = threadIdx.x >> 5;
  float sum = 0.f;
  if (c < d.cols)
    for (int i = 0; i < d.n_in; ++i) {
      const float* p = (const float*)t.ptrs[d.ptr0 + i] + c;
      const int rows = t.aux[d.aux0 + i];
#pragma unroll 8
      for (int r = g; r < rows; r += 8) sum += p[(size_t)r * d.cols];
    }
  part[g][threadIdx.x & 31] = sum;
  __syncthreads();
  if (g == 0 && c < d.cols) {
    float total = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) total += part[k][threadIdx.x];
    ((float*)d.out)[c] = total;
  }
}

}  // namespace

int32_t head_blocks(int cls, const OpDesc& d, const int32_t* aux) {
  const int32_t* ax = aux + d.aux0;
  switch (cls) {
    case LC_HEAD_ROPE:
    case LC_HEAD_ROPE_BWD: return (int32_t)(((int64_t)ax[kHeadRows] * (ax[kHeadCols] / d.p.head_dim) + 3) / 4);
    case LC_HEAD_GAIN: return d.rows;
    default: return (d.cols + 31) / 32;
  }
}

hipError_t launch_heads(int cls, int dtype, const DeviceTables& t, const Batch& b, int32_t max_blocks, hipStream_t s) {
  const dim3 grid((unsigned)max_blocks, (unsigned)b.n), wg(256);
  const bool bf = dtype == TN_BF16;
  switch (cls) {
    case LC_HEAD_ROPE:
      if (bf) hipLaunchKernelGGL(head_rope_kernel<bf16_t>, grid, wg, 0, s, t, b);
      else hipLaunchKernelGGL(head_rope_kernel<float>, grid, wg, 0, s, t, b);
      break;
    case LC_HEAD_ROPE_BWD:
      if (bf) hipLaunchKernelGGL(head_rope_bwd_kernel<bf16_t>, grid, wg, 0, s, t, b);
      else hipLaunchKernelGGL(head_rope_bwd_kernel<float>, grid, wg, 0, s, t, b);
      break;
    case LC_HEAD_GAIN:
      if (bf) hipLaunchKernelGGL(head_gain_kernel<bf16_t>, grid, wg, 0, s, t, b);
      else hipLaunchKernelGGL(head_gain_kernel<float>, grid, wg, 0, s, t, b);
      break;
    case LC_COL_SUM: hipLaunchKernelGGL(col_sum_kernel, grid, wg, 0, s, t, b); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace tn
