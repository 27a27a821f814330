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

#include <algorithm>

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

template <int CTRL>
__device__ __forceinline__ float exchanged(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}
// over the wavefront: in each sixteen lanes by exchanges inside the vector unit (neighbours, pairs, the mirrored half of eight, of sixteen)
__device__ __forceinline__ float wave_sum(float v) {
  v += exchanged<0xB1>(v);
  v += exchanged<0x4E>(v);
  v += exchanged<0x141>(v);
  v += exchanged<0x140>(v);
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
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
constexpr int64_t kGenericBlocks = 1 << 16;  // far more wavefronts than the chip holds, and far from what a launch may have

// sines and cosines of this lane's pairs in a row at `pos`
template <int PER>
__device__ __forceinline__ void angles(const Head& s, double pos, int lane, float (&sn)[PER], float (&cs)[PER]) {
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    sn[k] = 0.f;
    cs[k] = 1.f;
    if (s.pairs.turns(lane + 64 * k)) turn(pos, s.turns[lane + 64 * k], sn[k], cs[k]);
  }
}

// Heads of any size: a wavefront to a row and a run of its heads at a time (kHeadWalk), a lane to every 64th pair, whose angles serve the whole
// run.  Elements of a head of up to 128 are fetched while the head before it is worked on; larger ones have a kernel of their own, whose
// eight pairs to a lane leave registers for one head (in one kernel with them, small heads had a fifth of the wavefronts).  2000 rows of 32 heads
// of 80 of which 20 turn, bf16: 18 us (20 MB); a head to a wavefront, each with its angles, 35.  Both gradients 76 us; four wavefronts to 32 rows of
// the gain's and angles for every head 332.
struct Run {
  int row, h0, h1;
  __device__ Run(const Head& s, int64_t id) {
    const int walk = s.ax[kHeadWalk], runs = (s.heads + walk - 1) / walk;
    row = (int)(id / runs);
    h0 = (int)(id % runs) * walk;
    h1 = min(s.heads, h0 + walk);
  }
  __device__ static int64_t count(const Head& s) { return (int64_t)s.rows * ((s.heads + s.ax[kHeadWalk] - 1) / s.ax[kHeadWalk]); }
};
// (of large heads every head's addresses are formed anew: kept, they would take the registers)
template <int PER>
__device__ __forceinline__ int own_lane() {
  int lane = threadIdx.x & 63;
  if (PER > 1) asm volatile("" : "+v"(lane));
  return lane;
}
template <typename T, int PER>
struct Pieces {  // of a head, as loaded
  T a[PER], b[PER];
  __device__ void fetch(const Head& s, const T* p, int lane) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = lane + 64 * k;
      a[k] = b[k] = T(0);
      if (i >= s.head_dim / 2) continue;
      int ea, eb;
      s.pairs.elements(i, ea, eb);
      a[k] = get_global(p + ea);
      b[k] = get_global(p + eb);
    }
  }
};
__device__ __forceinline__ float wide(float v) { return v; }
__device__ __forceinline__ float wide(bf16_t v) { return bf2f(v); }

template <typename T, int PER>
__global__ void __launch_bounds__(256) head_rope_kernel(DeviceTables t, Batch b) {
  const OpDesc& d = t.descs[b.at(blockIdx.y)];
  if ((int)blockIdx.x >= d.nblocks) return;
  const Head s(t, d);
  const int lane = threadIdx.x & 63;
  const T* gain = s.norm ? (const T*)t.ptrs[d.ptr0 + 1] : nullptr;
  const int64_t count = Run::count(s);
  for (int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); id < count; id += (int64_t)d.nblocks * 4) {
    const Run at(s, id);
    const T* x = (const T*)t.ptrs[d.ptr0] + (size_t)at.row * s.cols;
    T* o = (T*)d.out + (size_t)at.row * s.cols;
    Pieces<T, PER> next;
    next.fetch(s, x + (size_t)at.h0 * s.head_dim, lane);
    float sn[PER], cs[PER];
    angles(s, s.position(at.row), lane, sn, cs);
#pragma unroll 1
    for (int h = at.h0; h < at.h1; ++h) {
      const int lane = own_lane<PER>();
      if (PER > 1 && h > at.h0) next.fetch(s, x + (size_t)h * s.head_dim, lane);
      const Pieces<T, PER> v = next;
      if (PER == 1 && h + 1 < at.h1) next.fetch(s, x + (size_t)(h + 1) * s.head_dim, lane);
      float ss = 0.f;
#pragma unroll
      for (int k = 0; k < PER; ++k) ss += wide(v.a[k]) * wide(v.a[k]) + wide(v.b[k]) * wide(v.b[k]);
      const float r = s.norm ? s.rstd(wave_sum(ss)) : 1.f;
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int i = lane + 64 * k;
        if (i >= s.head_dim / 2) continue;
        int ea, eb;
        s.pairs.elements(i, ea, eb);
        float a = wide(v.a[k]), c = wide(v.b[k]);
        if (s.norm) {
          a *= r * ld_global(gain + ea);
          c *= r * ld_global(gain + eb);
        }
        const float n = d.p.mode ? -sn[k] : sn[k];
        st(o + (size_t)h * s.head_dim + ea, a * cs[k] - c * n);
        st(o + (size_t)h * s.head_dim + eb, a * n + c * cs[k]);
      }
    }
  }
}

// The reverse of a head in registers: u (the inverse rotation of dY) and x of this lane's pairs, and 1 / rms.
template <typename T, int PER>
__device__ __forceinline__ float load_reverse(const Head& s, const T* dy, const T* x, const float (&sn)[PER], const float (&cs)[PER], int lane, float (&ua)[PER],
                                              float (&ub)[PER], float (&xa)[PER], float (&xb)[PER]) {
  float ss = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = lane + 64 * k;
    ua[k] = ub[k] = xa[k] = xb[k] = 0.f;
    if (i >= s.head_dim / 2) continue;
    int ea, eb;
    s.pairs.elements(i, ea, eb);
    xa[k] = ld_global(x + ea);
    xb[k] = ld_global(x + eb);
    ss += xa[k] * xa[k] + xb[k] * xb[k];
    const float a = ld_global(dy + ea), c = ld_global(dy + eb);
    ua[k] = a * cs[k] + c * sn[k];
    ub[k] = c * cs[k] - a * sn[k];
  }
  return s.rstd(wave_sum(ss));
}

constexpr int any_threads(int per) { return per == 1 ? 1024 : 512; }  // (of large heads 1024 threads have not the registers)
constexpr int any_columns(int per) { return 128 * per; }
template <typename T, int PER>
__device__ __forceinline__ void head_input(const DeviceTables& t, const OpDesc& d) {
  const Head s(t, d);
  const int lane = threadIdx.x & 63;
  constexpr int W = any_threads(PER) / 64;
  for (int64_t id = (int64_t)blockIdx.x * W + (threadIdx.x >> 6); id < (int64_t)s.rows * s.heads; id += (int64_t)d.nblocks * W) {
    const int row = (int)(id / s.heads), h = (int)(id % s.heads);
    const size_t at = (size_t)row * s.cols + (size_t)h * s.head_dim;
    const T* gain = (const T*)t.ptrs[d.ptr0 + 2];
    float ua[PER], ub[PER], xa[PER], xb[PER], sn[PER], cs[PER], dot = 0.f;
    angles(s, s.position(row), lane, sn, cs);
    const float r = load_reverse(s, (const T*)t.ptrs[d.ptr0] + at, (const T*)t.ptrs[d.ptr0 + 1] + at, sn, cs, lane, ua, ub, xa, xb);
    T* o = (T*)d.out + at;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
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
    for (int k = 0; k < PER; ++k) {
      const int i = lane + 64 * k;
      if (i >= s.head_dim / 2) continue;
      int ea, eb;
      s.pairs.elements(i, ea, eb);
      st(o + ea, r * (ua[k] - xa[k] * m));
      st(o + eb, r * (ub[k] - xb[k] * m));
    }
  }
}

// How many of `all` (a power of two) that work on n rows share one.
__device__ __forceinline__ int share(int all, int n) {
  int rows = 1;
  while (rows < n) rows *= 2;
  return max(1, all / rows);
}

// Sums of the gain's gradient: a workgroup per kGainRows rows, a wavefront takes every W-th of them (where they are few, several share a row), forms its angles once and keeps its
// sums in registers; the W are added in order.
template <typename T, int PER>
__device__ __forceinline__ void head_gain(const DeviceTables& t, const OpDesc& d, float (*part)[any_columns(PER)]) {
  constexpr int W = any_threads(PER) / 64;
  const Head s(t, d);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int block = d.nblocks - 1 - (int)blockIdx.x, row0 = block * kGainRows, n = min(kGainRows, s.rows - row0);
  float ga[PER], gb[PER], sn[PER], cs[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) ga[k] = gb[k] = 0.f;
  const int per_row = share(W, n);  // wavefronts that share a row
  for (int r = w / per_row; r < n; r += W / per_row) {
    const size_t at = (size_t)(row0 + r) * s.cols;
    const T* dy = (const T*)t.ptrs[d.ptr0] + at;
    const T* x = (const T*)t.ptrs[d.ptr0 + 1] + at;
    angles(s, s.position(row0 + r), lane, sn, cs);
#pragma unroll(PER == 1 ? 4 : 1)
    for (int h = w % per_row; h < s.heads; h += per_row) {
      float ua[PER], ub[PER], xa[PER], xb[PER];
      const float rstd = load_reverse(s, dy + (size_t)h * s.head_dim, x + (size_t)h * s.head_dim, sn, cs, lane, ua, ub, xa, xb);
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        ga[k] += ua[k] * (xa[k] * rstd);
        gb[k] += ub[k] * (xb[k] * rstd);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = lane + 64 * k;
    if (i >= s.head_dim / 2) continue;
    int ea, eb;
    s.pairs.elements(i, ea, eb);
    part[w][ea] = ga[k];
    part[w][eb] = gb[k];
  }
  __syncthreads();
  float* o = (float*)d.out + (size_t)block * s.head_dim;
  for (int c = threadIdx.x; c < s.head_dim; c += any_threads(PER)) {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) sum += part[k][c];
    o[c] = sum;
  }
}

// Both gradients go in one launch.
template <typename T, int PER>
__global__ void __launch_bounds__(any_threads(PER)) head_rope_bwd_kernel(DeviceTables t, Batch b) {
  const OpDesc& d = t.descs[b.at(blockIdx.y)];
  if ((int)blockIdx.x >= d.nblocks) return;
  __shared__ float part[any_threads(PER) / 64][any_columns(PER)];
  if (d.p.mode) head_gain<T, PER>(t, d, part);
  else head_input<T, PER>(t, d);
}

// ---- heads of a multiple of 16 elements, pairs that come in eights ---------------------------------
// Eight pairs to a lane -- two runs of eight elements, 16-byte accesses -- and a head to 4, 8, 16 .. lanes, of which those past its end
// are idle.  What bounds these is memory; a lane's angles, 8 of them with 64-bit products, are formed once for the heads it walks
// over, as many as leave enough wavefronts to fill the chip (kHeadWalk).  16384 rows of 32 heads of 128, bf16, with norm: 52 us (268 MB,
// 5.1 TB/s), both gradients 117 (671 MB, 5.7 TB/s); by wavefronts of a pair to a lane, a head each, 218 and 704.  One row: 5.2 us, a
// launch and three dependent loads.

// eight elements as loaded, which may be on their way while the head before them is worked on
template <typename T>
struct Raw8 {
  f32x4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Raw8<T> fetch8(const T* p) {
  Raw8<T> r;
#pragma unroll
  for (int k = 0; k < (int)sizeof(T) / 2; ++k) r.w[k] = get_global((const f32x4*)p + k);
  return r;
}
template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T>& r, float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if constexpr (sizeof(T) == 4) {
      v[k] = r.w[k / 4][k % 4];
    } else {
      const uint32_t w = __float_as_uint(r.w[0][k / 2]);
      v[k] = __uint_as_float(k & 1 ? w & 0xFFFF0000u : w << 16);
    }
  }
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) { unpack8(fetch8(p), v); }
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *(f32x4*)p = (f32x4){v[0], v[1], v[2], v[3]};
  *(f32x4*)(p + 4) = (f32x4){v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
  *(uint4*)p = make_uint4(f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7]));
}

// A lane's place in its head: where its two runs begin, and whether its pairs are (run 0, run 1) or neighbours.
struct Eights {
  int lanes, j;
  bool there, apart;  // the lane has pairs; they lie half a rotation apart
  int first, second;  // elements
  bool turns;
  __device__ Eights(const Head& s) {
    lanes = head_lanes(s.head_dim);
    j = threadIdx.x & (lanes - 1);
    there = 16 * j < s.head_dim;
    turns = 8 * j < s.pairs.half_rotary;
    apart = s.pairs.half && turns;
    first = apart ? 8 * j : 16 * j;
    second = apart ? s.pairs.half_rotary + 8 * j : 16 * j + 8;
  }
  __device__ void angles(const Head& s, int row, float (&sn)[8], float (&cs)[8]) const {
    const double pos = s.position(row);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      sn[k] = 0.f;
      cs[k] = 1.f;
      if (there && 8 * j + k < s.pairs.half_rotary) turn(pos, s.turns[8 * j + k], sn[k], cs[k]);
    }
  }
  // over the lanes of a head.  Within 16 lanes by exchanges inside the vector unit: neighbours, pairs, then the mirrored half
  __device__ float sum(float v) const {
    if (lanes > 1) v += exchanged<0xB1>(v);
    if (lanes > 2) v += exchanged<0x4E>(v);
    if (lanes > 4) v += exchanged<0x141>(v);
    if (lanes > 8) v += exchanged<0x140>(v);
    for (int off = 16; off < lanes; off <<= 1) v += __shfl_xor(v, off, 64);
    return v;
  }
};

// (u, v) turned in place
template <bool APART>
__device__ __forceinline__ void rotate8(float (&u)[8], float (&v)[8], const float (&sn)[8], const float (&cs)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    float& a = APART ? u[k] : k < 4 ? u[2 * k] : v[2 * k - 8];
    float& b = APART ? v[k] : k < 4 ? u[2 * k + 1] : v[2 * k - 7];
    const float x = a, y = b;
    a = x * cs[k] - y * sn[k];
    b = x * sn[k] + y * cs[k];
  }
}

// Where a lane of the grid starts: its row, and the first of the kHeadWalk heads that it walks over.
struct Walk {
  int row, h0, h1;
  bool any;
  __device__ Walk(const Head& s, int lanes, int threads) {
    const int walk = s.ax[kHeadWalk], runs = (s.heads + walk - 1) / walk;
    const int64_t id = ((int64_t)blockIdx.x * threads + threadIdx.x) / lanes;
    any = id < (int64_t)s.rows * runs;
    row = any ? (int)(id % s.rows) : 0;
    h0 = any ? (int)(id / s.rows) * walk : 0;
    h1 = any ? min(s.heads, h0 + walk) : 0;
  }
};

template <typename T>
__global__ void __launch_bounds__(256) head_rope_eights_kernel(DeviceTables t, Batch b) {
  const OpDesc& d = t.descs[b.at(blockIdx.y)];
  if ((int)blockIdx.x >= d.nblocks) return;
  const Head s(t, d);
  const Eights e(s);
  const Walk at(s, e.lanes, 256);
  const bool on = e.there && at.any;
  const T* x = (const T*)t.ptrs[d.ptr0] + (size_t)at.row * s.cols;
  T* o = (T*)d.out + (size_t)at.row * s.cols;
  float ga[8], gb[8], sn[8], cs[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) ga[k] = gb[k] = 1.f;
  if (s.norm && on) {
    load8((const T*)t.ptrs[d.ptr0 + 1] + e.first, ga);
    load8((const T*)t.ptrs[d.ptr0 + 1] + e.second, gb);
  }
  e.angles(s, at.row, sn, cs);
  if (d.p.mode) {
#pragma unroll
    for (int k = 0; k < 8; ++k) sn[k] = -sn[k];
  }
  Raw8<T> nu{}, nv{};
  auto fetch = [&](int h) {
    if (!on) return;
    nu = fetch8(x + (size_t)h * s.head_dim + e.first);
    nv = fetch8(x + (size_t)h * s.head_dim + e.second);
  };
  if (at.h0 < at.h1) fetch(at.h0);
  for (int h = at.h0; h < at.h1; ++h) {
    const Raw8<T> ru = nu, rv = nv;
    if (h + 1 < at.h1) fetch(h + 1);
    float u[8], v[8];
    unpack8(ru, u);
    unpack8(rv, v);
    if (s.norm) {
      float ss = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) ss += u[k] * u[k] + v[k] * v[k];
      const float r = s.rstd(e.sum(ss));
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        u[k] *= r * ga[k];
        v[k] *= r * gb[k];
      }
    }
    if (e.apart) rotate8<true>(u, v, sn, cs);
    else rotate8<false>(u, v, sn, cs);
    if (on) {
      store8(o + (size_t)h * s.head_dim + e.first, u);
      store8(o + (size_t)h * s.head_dim + e.second, v);
    }
  }
}

constexpr int kBwdThreads = 512;
template <typename T>
__device__ __forceinline__ void head_input_eights(const DeviceTables& t, const OpDesc& d) {
  const Head s(t, d);
  const Eights e(s);
  const Walk at(s, e.lanes, kBwdThreads);
  const bool on = e.there && at.any;
  const T* dy = (const T*)t.ptrs[d.ptr0] + (size_t)at.row * s.cols;
  const T* x = (const T*)t.ptrs[d.ptr0 + 1] + (size_t)at.row * s.cols;
  T* o = (T*)d.out + (size_t)at.row * s.cols;
  float ga[8] = {}, gb[8] = {}, sn[8], cs[8];
  if (on) {
    load8((const T*)t.ptrs[d.ptr0 + 2] + e.first, ga);
    load8((const T*)t.ptrs[d.ptr0 + 2] + e.second, gb);
  }
  e.angles(s, at.row, sn, cs);
#pragma unroll
  for (int k = 0; k < 8; ++k) sn[k] = -sn[k];
  Raw8<T> nu{}, nv{}, np{}, nq{};
  auto fetch = [&](int h) {
    if (!on) return;
    const size_t c = (size_t)h * s.head_dim;
    nu = fetch8(dy + c + e.first);
    nv = fetch8(dy + c + e.second);
    np = fetch8(x + c + e.first);
    nq = fetch8(x + c + e.second);
  };
  if (at.h0 < at.h1) fetch(at.h0);
  for (int h = at.h0; h < at.h1; ++h) {
    const Raw8<T> ru = nu, rv = nv, rp = np, rq = nq;
    if (h + 1 < at.h1) fetch(h + 1);
    float u[8], v[8], p[8], q[8];
    unpack8(ru, u);
    unpack8(rv, v);
    unpack8(rp, p);
    unpack8(rq, q);
    if (e.apart) rotate8<true>(u, v, sn, cs);
    else rotate8<false>(u, v, sn, cs);
    float ss = 0.f, dot = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      u[k] *= ga[k];
      v[k] *= gb[k];
      ss += p[k] * p[k] + q[k] * q[k];
      dot += u[k] * p[k] + v[k] * q[k];
    }
    const float r = s.rstd(e.sum(ss)), m = e.sum(dot) * r * r / (float)s.head_dim;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      u[k] = r * (u[k] - p[k] * m);
      v[k] = r * (v[k] - q[k] * m);
    }
    if (on) {
      store8(o + (size_t)h * s.head_dim + e.first, u);
      store8(o + (size_t)h * s.head_dim + e.second, v);
    }
  }
}

// Sums of the gain's gradient: the lanes of a head keep to one row at a time and walk over its heads; what the groups of a wavefront
// and the wavefronts of the workgroup have summed is added in a fixed order.  Blocks of rows go from the last to the first: the gradient
// of the input, formed from the same operands, leaves its last ones in the caches.  Alone, 16384 rows of 32 heads of 128, bf16: 55 us (268
// MB, 4.9 TB/s), from the first row on 63.  64 rows: 18 us, sixteen heads one behind the other; with 256 threads, which take 32,
// 23; with 1024 17, but three heads of 64 in fp32 14 instead of 9, since registers spill.
template <typename T>
__device__ __forceinline__ void head_gain_eights(const DeviceTables& t, const OpDesc& d, float (*part)[1024]) {
  const Head s(t, d);
  const Eights e(s);
  const int block = d.nblocks - 1 - (int)blockIdx.x, row0 = block * kGainRows, n = min(kGainRows, s.rows - row0);
  const int groups = kBwdThreads / e.lanes, group = threadIdx.x / e.lanes;
  const int per_row = share(groups, n);  // groups that share a row
  float ga[8] = {}, gb[8] = {};
  for (int r = group / per_row; r < n; r += groups / per_row) {
    const T* dy = (const T*)t.ptrs[d.ptr0] + (size_t)(row0 + r) * s.cols;
    const T* x = (const T*)t.ptrs[d.ptr0 + 1] + (size_t)(row0 + r) * s.cols;
    float sn[8], cs[8];
    e.angles(s, row0 + r, sn, cs);
#pragma unroll
    for (int k = 0; k < 8; ++k) sn[k] = -sn[k];
    Raw8<T> nu{}, nv{}, np{}, nq{};
    auto fetch = [&](int h) {
      if (!e.there) return;
      const size_t c = (size_t)h * s.head_dim;
      nu = fetch8(dy + c + e.first);
      nv = fetch8(dy + c + e.second);
      np = fetch8(x + c + e.first);
      nq = fetch8(x + c + e.second);
    };
    if (group % per_row < s.heads) fetch(group % per_row);
    for (int h = group % per_row; h < s.heads; h += per_row) {
      const Raw8<T> ru = nu, rv = nv, rp = np, rq = nq;
      if (h + per_row < s.heads) fetch(h + per_row);
      float u[8], v[8], p[8], q[8];
      unpack8(ru, u);
      unpack8(rv, v);
      unpack8(rp, p);
      unpack8(rq, q);
      if (e.apart) rotate8<true>(u, v, sn, cs);
      else rotate8<false>(u, v, sn, cs);
      float ss = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) ss += p[k] * p[k] + q[k] * q[k];
      const float rstd = s.rstd(e.sum(ss));
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        ga[k] = fmaf(u[k], p[k] * rstd, ga[k]);
        gb[k] = fmaf(v[k], q[k] * rstd, gb[k]);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k)
    for (int off = e.lanes; off < 64; off <<= 1) {
      ga[k] += __shfl_xor(ga[k], off, 64);
      gb[k] += __shfl_xor(gb[k], off, 64);
    }
  if ((int)(threadIdx.x & 63) < e.lanes && e.there) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      part[threadIdx.x >> 6][e.first + k] = ga[k];
      part[threadIdx.x >> 6][e.second + k] = gb[k];
    }
  }
  __syncthreads();
  float* o = (float*)d.out + (size_t)block * s.head_dim;
  for (int c = threadIdx.x; c < s.head_dim; c += kBwdThreads) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kBwdThreads / 64; ++w) sum += part[w][c];
    o[c] = sum;
  }
}

// Both gradients go in one launch.
template <typename T>
__global__ void __launch_bounds__(kBwdThreads) head_rope_bwd_eights_kernel(DeviceTables t, Batch b) {
  const OpDesc& d = t.descs[b.at(blockIdx.y)];
  if ((int)blockIdx.x >= d.nblocks) return;
  __shared__ float part[kBwdThreads / 64][1024];
  if (d.p.mode) head_gain_eights<T>(t, d, part);
  else head_input_eights<T>(t, d);
}

// Sum of all rows of the operands: a workgroup per 32 columns, eight threads to a column, each every eighth row; their sums are
// added in order.  (512 rows of 128 columns 5 us: 64 loads one behind the other in four workgroups.)
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
  if (cls == LC_COL_SUM) return (d.cols + 31) / 32;
  if (ax[kHeadBack] && d.p.mode) return d.rows;  // sums of the gain's gradient
  const int64_t runs = (int64_t)ax[kHeadRows] * ((ax[kHeadCols] / d.p.head_dim + ax[kHeadWalk] - 1) / ax[kHeadWalk]);
  auto blocks = [&](int64_t lanes, int64_t threads) { return (runs * lanes + threads - 1) / threads; };
  switch (cls) {
    case LC_HEAD_ROPE: return (int32_t)std::min(blocks(64, 256), kGenericBlocks);
    case LC_HEAD_ROPE_BWD: {
      const int64_t waves = any_threads(d.p.head_dim > kHeadSmall ? kPer : 1) / 64;
      return (int32_t)std::min(((int64_t)ax[kHeadRows] * (ax[kHeadCols] / d.p.head_dim) + waves - 1) / waves, kGenericBlocks);
    }
    case LC_HEAD_ROPE_EIGHTS: return (int32_t)blocks(head_lanes(d.p.head_dim), 256);
    default: return (int32_t)blocks(head_lanes(d.p.head_dim), kBwdThreads);
  }
}

namespace {
template <typename T>
hipError_t launch(int cls, bool large, const DeviceTables& t, const Batch& b, int32_t max_blocks, hipStream_t s) {
  const dim3 grid((unsigned)max_blocks, (unsigned)b.n);
  void (*kernel)(DeviceTables, Batch);
  int threads = 256;
  switch (cls) {
    case LC_HEAD_ROPE: kernel = large ? head_rope_kernel<T, kPer> : head_rope_kernel<T, 1>; break;
    case LC_HEAD_ROPE_BWD:
      kernel = large ? head_rope_bwd_kernel<T, kPer> : head_rope_bwd_kernel<T, 1>;
      threads = any_threads(large ? kPer : 1);
      break;
    case LC_HEAD_ROPE_EIGHTS: kernel = head_rope_eights_kernel<T>; break;
    case LC_HEAD_ROPE_BWD_EIGHTS:
      kernel = head_rope_bwd_eights_kernel<T>;
      threads = kBwdThreads;
      break;
    case LC_COL_SUM: kernel = col_sum_kernel; break;
    default: return hipErrorInvalidValue;
  }
  hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, t, b);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_heads(int cls, int dtype, int head_dim, const DeviceTables& t, const Batch& b, int32_t max_blocks, hipStream_t s) {
  const bool large = head_dim > kHeadSmall;
  return dtype == TN_BF16 ? launch<bf16_t>(cls, large, t, b, max_blocks, s) : launch<float>(cls, large, t, b, max_blocks, s);
}

}  // namespace tn
