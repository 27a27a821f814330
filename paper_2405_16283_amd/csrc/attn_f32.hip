// Attention forward and reverse with fp32 products on the matrix cores (MFMA 16x16x4): fp32 graphs, and
// bf16 graphs whose tiling the bf16 kernels in kernels.hip do not take (key tiles that are no multiple of
// 64 rows, heads that straddle column tiles).  Any tile grid the executor admits is served.
//
// One workgroup = one head x 64 rows of its own side (queries; keys in the dK and dV forms); a wavefront
// owns 16 of them and a lane (n = lane & 15, g = lane >> 4) row n of those 16.  The other side comes
// through LDS as fp32, 64 rows at a time.  Scores are formed transposed, S^T = K Q^T, so that a lane holds
// the scores of its own row against rows 4g + i of a 16-row tile -- which is the B operand of the second
// product if step c of its four MFMAs takes the rows 4g + c: probabilities never leave their registers.
//
// Bound: the matrix cores (256 flop per clock and CU in fp32, 157 TFLOP/s); 64 keys cost a wavefront 256
// MFMAs of 32 cycles at head size 128 against 64 KiB of LDS reads, a quarter of what LDS delivers in that time.
// The kernels these replace ran one query row per thread on the vector ALUs with every operand read from
// memory.  Per launch, before -> after: fp32, 16 heads of 64, 1024 positions in blocks of 512, 5.6 ms -> 58 us;
// fp32 reverse, 3 heads of 64, 160 positions, 2.8 ms -> 17 us (latency: a handful of workgroups); bf16, 32 heads
// of 128, 347 queries against 1371 keys, 6.6 ms -> 0.10 ms.  (Reverse pass with the own rows by
// way of LDS and all loads up to the first chunk issued before any is waited for: 18.1 -> 17.8 us, not kept.)
#include "attn_rows.h"

#include <climits>
#include <type_traits>

namespace tn {
namespace {

constexpr int fwd_lds(int hd) { return 4 * (64 * (hd + 4) + hd * (64 + 4)); }
constexpr int kRows = 64;  // rows of a workgroup's own side, and rows of the other side per round

constexpr int kPieces(int hd) { return kRows * hd / 4 / 256; }  // pieces of four elements per thread and chunk

// Rows row0 .. row0 + 63 into registers: piece p = i * 256 + tid is columns 4 (p % (HD / 4)) .. of row p / (HD / 4).
// Rows past the end are zero.
// (pieces I0 .. I0 + N - 1 only.)
template <typename T, int HD, int I0 = 0, int N = kPieces(HD)>
__device__ __forceinline__ void load_chunk(const Side<T, HD>& s, bool transposed, int row0, f32x4 (&v)[N]) {
  const int rt0 = row0 / s.trows, rin0 = row0 - rt0 * s.trows, n = min(kRows, s.rows - row0);
  const bool plain = s.whole && !transposed && rin0 + n <= s.trows;  // one tile: the address is linear in the row
  const T* base = plain ? (const T*)s.t[rt0 * s.nc + s.ct] + (size_t)rin0 * s.tc + s.cin : nullptr;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = (I0 + i) * 256 + (threadIdx.x & 255), r = p / (HD / 4), c = (p % (HD / 4)) * 4;
    v[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    if (r < n) v[i] = plain ? ld4_global(base + (size_t)r * s.tc + c) : transposed ? s.at_t(row0 + r, c) : s.at(row0 + r, c);
  }
}
template <int HD, int I0 = 0, int N = kPieces(HD)>
__device__ __forceinline__ void store_chunk(float (*buf)[HD + 4], const f32x4 (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = (I0 + i) * 256 + (threadIdx.x & 255);
    *(f32x4*)&buf[p / (HD / 4)][(p % (HD / 4)) * 4] = v[i];
  }
}

// The 64-row chunk of V as V^T[HD][64]: piece p is keys 4 (p % 16) .. of head column p / 16.
template <typename T, int HD, int I0 = 0, int N = kPieces(HD)>
__device__ __forceinline__ void load_chunk_vt(const Side<T, HD>& s, bool transposed, int row0, f32x4 (&v)[N]) {
  const int rt0 = row0 / s.trows, rin0 = row0 - rt0 * s.trows, n = min(kRows, s.rows - row0);
  const int pitch = min(s.trows, s.rows - rt0 * s.trows);
  const bool linear = s.whole && transposed && rin0 + n <= s.trows;  // one tile: the address is linear in the key and the column
  const bool plain = linear && pitch % 4 == 0 && rin0 % 4 == 0;
  const T* base = linear ? (const T*)s.t[rt0 * s.nc + s.ct] + (size_t)s.cin * pitch + rin0 : nullptr;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = (I0 + i) * 256 + (threadIdx.x & 255), c = p / 16, k = (p % 16) * 4;
    v[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    if (plain) {  // n is a multiple of 4 here: the tile's rows are
      if (k < n) v[i] = ld4_global(base + (size_t)c * pitch + k);
    } else if (linear) {  // (347 keys: with the tile looked up for every element 132 us a launch, so 103)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (k + e < n) v[i][e] = ld_global(base + (size_t)c * pitch + k + e);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (k + e < n)
          v[i][e] = ld_global(transposed ? tile_elem_t<T>(s.t, s.nc, s.trows, s.tc, s.rows, row0 + k + e, s.c0 + c)
                                  : tile_elem<T>(s.t, s.nc, s.trows, s.tc, row0 + k + e, s.c0 + c));
    }
  }
}

template <int HD, int I0 = 0, int N = kPieces(HD)>
__device__ __forceinline__ void store_chunk_vt(float (*buf)[kRows + 4], const f32x4 (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = (I0 + i) * 256 + (threadIdx.x & 255);
    *(f32x4*)&buf[p / 16][(p % 16) * 4] = v[i];
  }
}

// V by rows as stored (pieces as load_chunk has them), turned round on its way into LDS.  (Fetched by columns, element by element, 1024
// positions of 16 heads of 64 took 150 us; so 100.)
template <int HD, int I0 = 0, int N = kPieces(HD)>
__device__ __forceinline__ void store_chunk_turned(float (*buf)[kRows + 4], const f32x4 (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = (I0 + i) * 256 + (threadIdx.x & 255);
#pragma unroll
    for (int e = 0; e < 4; ++e) buf[p % (HD / 4) * 4 + e][p / (HD / 4)] = v[i][e];
  }
}

// A row's sum leaves out what the causal mask hides from it.  The matrix cores multiply that by a weight of zero, which
// is the same as long as it is finite.  Chunks the diagonal crosses are looked through for infinities and NaN in LDS;
// a workgroup that finds some forms its rows again, each summed over what it sees, sixteen lanes to a row (`*_by_rows`: many
// times slower, and outside the loops on the matrix cores, whose registers and order of instructions it must not cost
// anything: inside them, and with the look between loads and stores, it took 2 % of a decode program).
template <int ROWS, int COLS, int PITCH>
__device__ __forceinline__ bool not_finite(const float (*buf)[PITCH]) {
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < ROWS * COLS / 4 / 256; ++i) {
    const int p = i * 256 + (threadIdx.x & 255);
    const f32x4 v = *(const f32x4*)&buf[p / (COLS / 4)][p % (COLS / 4) * 4];
#pragma unroll
    for (int e = 0; e < 4; ++e) z = fmaf(v[e], 0.f, z);
  }
  return !(z == 0.f);
}

// whether any lane of the workgroup says so, once its chunks in LDS are done with
__device__ __forceinline__ bool any_wave(bool mine, char* lds) {
  const int wave = __ballot(mine) != 0;
  int* const said = (int*)lds;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) said[threadIdx.x >> 6] = wave;
  __syncthreads();
  int any = 0;
  for (int w = 0; w < (int)blockDim.x >> 6; ++w) any |= said[w];
  return __builtin_expect(any != 0, 0);
}

// What the rows of a workgroup see together, of per-lane ranges (all lanes of the workgroup, lo == hi for nothing): keys before `begin` and from
// `end` on nobody sees, those in [all_lo, all_hi) everybody does.  lds: 16 integers.
struct Seen {
  int begin, end, all_lo, all_hi;
};
__device__ __forceinline__ Seen seen_by_all(int lo, int hi, bool exists, int* lds) {
  int v[4] = {exists && lo < hi ? lo : INT_MAX, exists ? -hi : 0, exists ? -lo : INT_MAX, exists ? hi : INT_MAX};  // minima all
#pragma unroll
  for (int off = 32; off > 0; off >>= 1)
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = min(v[k], __shfl_xor(v[k], off, 64));
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < 4; ++k) lds[((threadIdx.x & 255) >> 6) * 4 + k] = v[k];  // (both halves find the same)
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w)
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = min(v[k], lds[w * 4 + k]);
  __syncthreads();
  return {v[0], -v[1], -v[2], v[3]};
}

// aux: [rows per Q tile, rows per K/V tile, columns per tile, q rows, kv rows]
// RULE: scores go by a rule or rows are finished (attn_rule.h); the rest of aux is read.  Then two halves of four wavefronts take
// alternate chunks and are joined at the end: a launch of few workgroups waits for its longest walk over the keys, and one of many
// has the same eight wavefronts to a compute unit (1024 positions of 16 heads of 64, 256 workgroups: 100 us without, 70 with;
// attn_rule_f32.hip, which takes grids whose chunks lie inside one tile, 37).
template <typename T, int HD, bool RULE>
__global__ void __launch_bounds__(RULE ? 512 : 256, 2) attn_f32_kernel(DeviceTables t, Batch b) {
  const OpDesc& d = t.descs[b.at(blockIdx.y)];
  if ((int)blockIdx.x >= d.nblocks) return;
  const int* ax = t.aux + d.aux0;
  const int tq = ax[0], tk = ax[1], tc = ax[2], q_rows = ax[3], kv_rows = ax[4];
  const int nc = d.p.n_col_tiles, gw = nc * tc, hpg = gw / HD;
  const int qblocks = (q_rows + kRows - 1) / kRows;
  const int h = blockIdx.x / qblocks, qb = blockIdx.x % qblocks;
  const int lane = threadIdx.x & 63, w = (threadIdx.x & 255) >> 6, n = lane & 15, g = lane >> 4;
  const int half = RULE ? threadIdx.x >> 8 : 0;
  void* const* Qt = t.ptrs + d.ptr0;
  void* const* Kt = Qt + d.p.n_q_tiles * nc;
  void* const* Vt = Kt + d.p.n_kv_tiles * nc;
  const Side<T, HD> Q(Qt, nc, tq, tc, q_rows, h), K(Kt, nc, tk, tc, kv_rows, h), V(Vt, nc, tk, tc, kv_rows, h);
  const bool v_trans = d.p.v_trans != 0;
  const int causal = d.p.causal, k_pos0 = d.p.k_pos0;

  extern __shared__ __attribute__((aligned(16))) char lds[];
  char* const mine = lds + half * fwd_lds(HD);
  float(*const ks)[HD + 4] = (float(*)[HD + 4])mine;                                   // K chunk [64][HD], padded
  float(*const vs)[kRows + 4] = (float(*)[kRows + 4])(mine + sizeof(float) * kRows * (HD + 4));  // V^T chunk [HD][64], padded
  bool odd = false;  // a chunk on the diagonal whose V is not finite

  const int row = qb * kRows + w * 16 + n, qpos = d.p.q_pos0 + row;
  const int wpos0 = d.p.q_pos0 + qb * kRows + w * 16;  // first position of the wavefront
  f32x4 q[HD / 16];
#pragma unroll
  for (int j = 0; j < HD / 16; ++j) q[j] = Q.at(min(row, q_rows - 1), 16 * j + 4 * g) * d.p.scale;
  f32x4 o[HD / 16];
#pragma unroll
  for (int j = 0; j < HD / 16; ++j) o[j] = (f32x4){0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  int begin = 0, end = kv_rows;  // keys above the diagonal of this workgroup's rows contribute nothing
  if (causal) end = min(kv_rows, d.p.q_pos0 + qb * kRows + kRows - k_pos0);
  int lo = 0, hi = 0;  // RULE: what this lane's query sees
  Seen seen{};
  float slope = 0.f;
  const Rule rule = RULE ? Rule(t, d) : Rule();
  if constexpr (RULE) {
    if (row < q_rows) rule.visible(row, lo, hi);
    seen = seen_by_all(lo, hi, row < q_rows, (int*)lds);
    begin = seen.begin < seen.end ? seen.begin & ~(kRows - 1) : 0;
    end = seen.end;
    slope = rule.slope(h);
  }
  // head size 64 has the registers to fetch the next chunk while one is multiplied; at 128 the second
  // workgroup of the compute unit covers the wait instead
  constexpr bool kAhead = HD == 64;
  constexpr int P = kAhead ? kPieces(HD) : kPieces(HD) / 2;
  f32x4 kn[P], vn[P];
  auto load_v = [&](int kv0, auto from) {
    constexpr int I0 = decltype(from)::value;
    if (v_trans) load_chunk_vt<T, HD, I0, P>(V, true, kv0, vn);
    else load_chunk<T, HD, I0, P>(V, false, kv0, vn);
  };
  auto store_v = [&](auto from) {
    constexpr int I0 = decltype(from)::value;
    if (v_trans) store_chunk_vt<HD, I0, P>(vs, vn);
    else store_chunk_turned<HD, I0, P>(vs, vn);
  };
  constexpr std::integral_constant<int, 0> kFirst{};
  constexpr std::integral_constant<int, P> kRest{};
  constexpr int kStep = RULE ? 2 * kRows : kRows;
  const int from = begin + half * kRows;
  if (kAhead && end > from) {
    load_chunk<T, HD, 0, P>(K, false, from, kn);
    load_v(from, kFirst);
  }
  for (int kv0 = from; kv0 - half * kRows < end; kv0 += kStep) {
    const bool there = !RULE || kv0 < end;  // the second half may have no last chunk
    __syncthreads();  // everybody is done with the chunk before
    if (there) {
      if constexpr (!kAhead) {
        load_chunk<T, HD, 0, P>(K, false, kv0, kn);
        load_v(kv0, kFirst);
      }
      store_chunk<HD, 0, P>(ks, kn);
      store_v(kFirst);
      if constexpr (!kAhead) {
        load_chunk<T, HD, P, P>(K, false, kv0, kn);
        load_v(kv0, kRest);
        store_chunk<HD, P, P>(ks, kn);
        store_v(kRest);
      }
    }
    __syncthreads();
    if (!there) continue;
    if (kAhead && kv0 + kStep < end) {
      load_chunk<T, HD, 0, P>(K, false, kv0 + kStep, kn);
      load_v(kv0 + kStep, kFirst);
    }
    if constexpr (RULE) {
      if ((kv0 < seen.all_lo || min(kv0 + kRows, kv_rows) > seen.all_hi) && not_finite<HD, kRows>(vs)) odd = true;
    } else {
      if (causal && k_pos0 + kv0 + kRows - 1 > d.p.q_pos0 + qb * kRows && not_finite<HD, kRows>(vs)) odd = true;
    }
    f32x4 s[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < HD / 16; ++j) {
      f32x4 a[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) a[k] = *(const f32x4*)&ks[16 * k + n][16 * j + 4 * g];
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] = mfma_f32(a[k][c], q[j][c], s[k]);
      if (j & 1) __builtin_amdgcn_sched_barrier(0);  // no more than two steps' fragments at a time: registers
    }
    // element i of s[k]: key kv0 + 16 k + 4 g + i
    float mx = -INFINITY;
    const bool mask = kv0 + kRows > kv_rows || (causal && k_pos0 + kv0 + kRows - 1 > wpos0);
    if constexpr (RULE) {
      if (rule.cap > 0.f) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[k][i] = rule.cap * tanh_f32(s[k][i] * rule.inv_cap);
      }
      if (rule.slopes) {
        const float base = (float)(qpos - k_pos0 - kv0 - 4 * g);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[k][i] = fmaf(-slope, fabsf(base - (float)(16 * k + i)), s[k][i]);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int kv = kv0 + 16 * k + 4 * g + i;
        if constexpr (RULE) {
          if (kv < lo || kv >= hi) s[k][i] = -INFINITY;
        } else {
          if (mask && (kv >= kv_rows || (causal && k_pos0 + kv > qpos))) s[k][i] = -INFINITY;
        }
        mx = fmaxf(mx, s[k][i]);
      }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float mn = fmaxf(m, mx), ms = mn == -INFINITY ? 0.f : mn;  // nothing visible yet: every weight is exp(-inf)
    const float alpha = __expf(m - ms);
    m = mn;
    l *= alpha;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[k][i] = __expf(s[k][i] - ms);
        l += s[k][i];
      }
#pragma unroll
    for (int j = 0; j < HD / 16; ++j) o[j] *= alpha;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < HD / 16; j += 4) {
        f32x4 a[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = *(const f32x4*)&vs[16 * (j + e) + n][16 * k + 4 * g];
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[j + e] = mfma_f32(a[e][c], s[k][c], o[j + e]);
        if (j & 4) __builtin_amdgcn_sched_barrier(0);
      }
  }
  if ((causal || RULE) && any_wave(odd, lds)) return attn_by_rows<T, HD, RULE>(t, d, h, qb * kRows, (qb + 1) * kRows, threadIdx.x >> 4, blockDim.x >> 4);
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if constexpr (RULE) {  // the second half's state by way of LDS (any_wave has seen to it that the chunks are done with)
    f32x4* const theirs = (f32x4*)lds;
    float* const stats = (float*)(lds + 4 * 64 * (HD / 16) * 16);
    __syncthreads();
    if (half) {
#pragma unroll
      for (int j = 0; j < HD / 16; ++j) theirs[(w * (HD / 16) + j) * 64 + lane] = o[j];
      stats[w * 64 + lane] = m;
      stats[256 + w * 64 + lane] = l;
    }
    __syncthreads();
    if (half) return;
    const float m2 = stats[w * 64 + lane], l2 = stats[256 + w * 64 + lane];
    const float mn = fmaxf(m, m2), ms = mn == -INFINITY ? 0.f : mn, w1 = __expf(m - ms), w2 = __expf(m2 - ms);
    m = mn;
    l = l * w1 + l2 * w2;
#pragma unroll
    for (int j = 0; j < HD / 16; ++j) o[j] = o[j] * w1 + theirs[(w * (HD / 16) + j) * 64 + lane] * w2;
  }
  if (row >= q_rows) return;
  if constexpr (RULE)
    if (ax[kRuleFinish]) {
#pragma unroll
      for (int j = 0; j < HD / 16; ++j) st4_finished((T*)d.out + (size_t)row * gw + h * HD + 16 * j + 4 * g, o[j], l);
      return;
    }
  float* out = (float*)d.out + (size_t)row * d.cols;
#pragma unroll
  for (int j = 0; j < HD / 16; ++j) {
    float* o4 = out + h * HD + 16 * j + 4 * g;
    if ((d.cols & 3) == 0) {  // rows of the partial are 16-byte aligned
      st4(o4, o[j]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) o4[i] = o[j][i];
    }
  }
  if (g == 0) {
    out[gw + h] = m;
    out[gw + hpg + h] = l;
  }
}

// Reverse pass.  Modes 0 (statistics) and 1 (dQ): the workgroup's own rows are queries, keys come in
// chunks.  Modes 2 (dK) and 3 (dV): its own rows are keys, queries and their statistics come in chunks.
// Scores are formed again from Q and K; p = exp(scale q.k - lse).
template <typename T, int HD, int MODE, bool RULE>
__device__ __forceinline__ void attn_bwd_f32_body(const DeviceTables& t, const OpDesc& d, char* lds) {
  const int* ax = t.aux + d.aux0;
  const int tq = ax[0], tk = ax[1], tc = ax[2], q_rows = ax[3], kv_rows = ax[4];
  const int nc = d.p.n_col_tiles, gw = nc * tc, hpg = gw / HD, nq = d.p.n_q_tiles, nkv = d.p.n_kv_tiles;
  void* const* Qt = t.ptrs + d.ptr0;
  void* const* Kt = Qt + nq * nc;
  void* const* Vt = Kt + nkv * nc;
  void* const* Dt = Vt + nkv * nc;  // dO tiles
  void* const* St = Dt + nq * nc;   // statistics, one tensor per Q row tile (modes 1..3)
  const int my_rows = MODE <= 1 ? q_rows : kv_rows, o_rows = MODE <= 1 ? kv_rows : q_rows;
  const int rblocks = (my_rows + kRows - 1) / kRows;
  const int h = blockIdx.x / rblocks, rb = blockIdx.x % rblocks;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  const Side<T, HD> Q(Qt, nc, tq, tc, q_rows, h), K(Kt, nc, tk, tc, kv_rows, h), V(Vt, nc, tk, tc, kv_rows, h),
      D(Dt, nc, tq, tc, q_rows, h);
  const bool v_trans = d.p.v_trans != 0;
  const int causal = d.p.causal;
  const float scale = d.p.scale;
  auto stat = [&](int r, int which) -> float {  // which 0: lse, 1: D
    const int rt = r / tq;
    return get_global((const float*)St[rt] + (size_t)(r - rt * tq) * (2 * hpg) + which * hpg + h);
  };
  float(*const x1)[HD + 4] = (float(*)[HD + 4])lds;                                             // K, or Q
  float(*const x2)[HD + 4] = (float(*)[HD + 4])(lds + sizeof(float) * kRows * (HD + 4));        // V, or dO
  float(*const xs)[2] = (float(*)[2])(lds + 2 * sizeof(float) * kRows * (HD + 4));              // statistics of the queries
  int(*const sees)[2] = (int(*)[2])(xs + kRows);  // RULE, modes 2 and 3: what they see
  bool odd = false;  // a chunk on the diagonal that is not finite

  const int row = rb * kRows + w * 16 + n, rc = min(row, my_rows - 1);
  const int pos = (MODE <= 1 ? d.p.q_pos0 : d.p.k_pos0) + row;
  f32x4 m1[HD / 16], m2[HD / 16], acc[HD / 16];  // this lane's own row: Q and dO, or K and V
#pragma unroll
  for (int j = 0; j < HD / 16; ++j) {
    m1[j] = MODE <= 1 ? Q.at(rc, 16 * j + 4 * g) : K.at(rc, 16 * j + 4 * g);
    if (MODE <= 1) m2[j] = D.at(rc, 16 * j + 4 * g);
    if (MODE == 2) m2[j] = v_trans ? V.at_t(rc, 16 * j + 4 * g) : V.at(rc, 16 * j + 4 * g);
    acc[j] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }
  const float lse = MODE == 1 ? stat(rc, 0) : 0.f, Dr = MODE == 1 ? stat(rc, 1) : 0.f;
  float mrun = -INFINITY, l = 0.f, dsum = 0.f;  // mode 0: this lane's share of the keys
  int begin = 0, end = o_rows;
  if (causal && MODE <= 1) end = min(kv_rows, d.p.q_pos0 + rb * kRows + kRows - d.p.k_pos0);
  if (causal && MODE >= 2) begin = max(0, d.p.k_pos0 + rb * kRows - d.p.q_pos0);
  int lo = 0, hi = 0;  // RULE, mode 1: what this lane's query sees
  Seen seen{};
  float slope = 0.f;
  const Rule rule = RULE ? Rule(t, d) : Rule();
  if constexpr (RULE) {
    slope = rule.slope(h);
    if (MODE == 1) {
      if (row < my_rows) rule.visible(row, lo, hi);
      seen = seen_by_all(lo, hi, row < my_rows, (int*)lds);
      begin = seen.begin < seen.end ? seen.begin & ~(kRows - 1) : 0;
      end = seen.end;
    }
  }

  for (int r0 = begin; r0 < end; r0 += kRows) {
    bool all_see = true;  // RULE, modes 2 and 3: every query of the chunk sees every key of the workgroup
    if constexpr (RULE && MODE >= 2) {
      int ql = 0, qh = 0;  // lane by lane the chunk's queries; every wavefront finds the same
      if (r0 + lane < q_rows) rule.visible(r0 + lane, ql, qh);
      const int k0 = rb * kRows, k1 = min(k0 + kRows, kv_rows);
      if (!__any(max(ql, k0) < min(qh, k1))) continue;
      all_see = __all(ql <= k0 && qh >= k1);
      lo = ql;
      hi = qh;
    }
    f32x4 v1[kPieces(HD)], v2[kPieces(HD)];
    load_chunk<T, HD>(MODE <= 1 ? K : Q, false, r0, v1);
    load_chunk<T, HD>(MODE <= 1 ? V : D, MODE <= 1 && v_trans, r0, v2);
    float sv = 0.f;
    if (MODE >= 2 && threadIdx.x < 2 * kRows) sv = stat(min(r0 + (int)threadIdx.x / 2, q_rows - 1), threadIdx.x & 1);
    __syncthreads();  // everybody is done with the chunk before
    store_chunk<HD>(x1, v1);
    store_chunk<HD>(x2, v2);
    if (MODE >= 2 && threadIdx.x < 2 * kRows) xs[threadIdx.x / 2][threadIdx.x & 1] = sv;
    if (RULE && MODE >= 2 && threadIdx.x < kRows) {
      sees[threadIdx.x][0] = lo;
      sees[threadIdx.x][1] = hi;
    }
    __syncthreads();
    // some row of the workgroup and some row of the chunk do not see each other
    if (RULE && (MODE == 1 ? r0 < seen.all_lo || min(r0 + kRows, kv_rows) > seen.all_hi : !all_see) && not_finite<kRows, HD>(MODE == 3 ? x2 : x1))
      odd = true;
    if (!RULE && MODE != 0 && causal && (MODE == 1 ? d.p.k_pos0 + r0 + kRows - 1 > d.p.q_pos0 + rb * kRows
                                          : d.p.k_pos0 + rb * kRows + kRows - 1 > d.p.q_pos0 + r0) &&
        not_finite<kRows, HD>(MODE == 3 ? x2 : x1))
      odd = true;
#pragma unroll 1
    for (int k = 0; k < 4; k += 2) {  // two 16-row tiles of the other side at a time
      f32x4 s[2], dp[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) s[e] = dp[e] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < HD / 16; ++j) {
        f32x4 a[2], a2[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          a[e] = *(const f32x4*)&x1[16 * (k + e) + n][16 * j + 4 * g];
          if (MODE != 3) a2[e] = *(const f32x4*)&x2[16 * (k + e) + n][16 * j + 4 * g];
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            s[e] = mfma_f32(a[e][c], m1[j][c], s[e]);
            if (MODE != 3) dp[e] = mfma_f32(a2[e][c], m2[j][c], dp[e]);
          }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        // element i: row r0 + 16 (k + e) + 4 g + i of the other side
        f32x4 wgt;
        float mx = mrun;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int lr = 16 * (k + e) + 4 * g + i, o = r0 + lr;
          bool ok = o < o_rows;
          float z = s[e][i] * scale, th = 0.f;
          if constexpr (RULE) {
            ok = MODE == 1 ? o >= lo && o < hi : row >= sees[lr][0] && row < sees[lr][1];
            z = rule.score(z, slope, MODE == 1 ? pos - d.p.k_pos0 - o : d.p.q_pos0 + o - pos, th);
          } else {
            if (causal) ok = ok && (MODE <= 1 ? d.p.k_pos0 + o <= pos : pos <= d.p.q_pos0 + o);
          }
          if (MODE == 0) {
            s[e][i] = ok ? z : -INFINITY;
            if (!ok) dp[e][i] = 0.f;
            mx = fmaxf(mx, s[e][i]);
          } else {
            float p = __expf(z - (MODE == 1 ? lse : xs[lr][0]));
            if (MODE == 1) p *= (dp[e][i] - Dr) * scale;
            if (MODE == 2) p *= (dp[e][i] - xs[lr][1]) * scale;
            if (RULE && MODE != 3) p *= 1.f - th * th;
            wgt[i] = ok ? p : 0.f;
          }
        }
        if (MODE == 0) {
          const float ms = mx == -INFINITY ? 0.f : mx, alpha = __expf(mrun - ms);
          l *= alpha;
          dsum *= alpha;
          mrun = mx;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = __expf(s[e][i] - ms);
            l += p;
            dsum = fmaf(p, dp[e][i], dsum);
          }
          continue;
        }
        // acc^T[column, own row] += X^T[column, other row] wgt[other row, own row]; X: K, Q or dO
        float(*const xt)[HD + 4] = MODE == 3 ? x2 : x1;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int j = 0; j < HD / 16; ++j) acc[j] = mfma_f32(xt[16 * (k + e) + 4 * g + c][16 * j + n], wgt[c], acc[j]);
      }
    }
  }
  if (MODE == 0) {
    // the four lanes of a query saw different keys: merge their states
#pragma unroll
    for (int off = 16; off <= 32; off <<= 1) {
      const float m2_ = __shfl_xor(mrun, off, 64), l2 = __shfl_xor(l, off, 64), d2 = __shfl_xor(dsum, off, 64);
      const float mn = fmaxf(mrun, m2_), ms = mn == -INFINITY ? 0.f : mn;
      const float w1 = __expf(mrun - ms), w2 = __expf(m2_ - ms);
      l = l * w1 + l2 * w2;
      dsum = dsum * w1 + d2 * w2;
      mrun = mn;
    }
    if (row < my_rows && g == 0) {
      float* out = (float*)d.out + (size_t)row * (2 * hpg);
      out[h] = mrun + __logf(l);
      out[hpg + h] = dsum / l;
    }
    return;
  }
  if ((causal || RULE) && any_wave(odd, lds)) return attn_bwd_by_rows<T, HD, MODE, RULE>(t, d, Q, K, V, D, h, gw, rb * kRows, (rb + 1) * kRows, threadIdx.x >> 4, 16, stat);
  if (row >= my_rows) return;
  T* out = (T*)d.out + (size_t)row * gw + h * HD;
#pragma unroll
  for (int j = 0; j < HD / 16; ++j) st4(out + 16 * j + 4 * g, acc[j]);
}

template <typename T, int HD, bool RULE>
__global__ void __launch_bounds__(256, 2) attn_bwd_f32_kernel(DeviceTables t, Batch b) {
  const OpDesc& d = t.descs[b.at(blockIdx.y)];
  if ((int)blockIdx.x >= d.nblocks) return;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  switch (d.p.mode) {
    case 0:
      if constexpr (!RULE) attn_bwd_f32_body<T, HD, 0, RULE>(t, d, lds);
      break;
    case 1: attn_bwd_f32_body<T, HD, 1, RULE>(t, d, lds); break;
    case 2: attn_bwd_f32_body<T, HD, 2, RULE>(t, d, lds); break;
    default: attn_bwd_f32_body<T, HD, 3, RULE>(t, d, lds); break;
  }
}

constexpr int fwd_rule_lds(int hd) { return 2 * fwd_lds(hd); }
constexpr int bwd_lds(int hd) { return 4 * (2 * kRows * (hd + 4) + 2 * kRows); }
constexpr int bwd_rule_lds(int hd) { return bwd_lds(hd) + 4 * 2 * kRows; }

template <auto kernel, int THREADS>
hipError_t launch(int lds, const DeviceTables& t, const Batch& b, int32_t max_blocks, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  if (const hipError_t e = allow_lds(allowed, (const void*)kernel, lds); e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)max_blocks, (unsigned)b.n), dim3(THREADS), lds, s, t, b);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_f32(bool reverse, bool rule, int dtype, int head_dim, const DeviceTables& t, const Batch& b, int32_t max_blocks,
                           hipStream_t s) {
  const bool bf = dtype == TN_BF16;
  if (head_dim != 64 && head_dim != 128) return hipErrorInvalidValue;
#define TN_PICK(kernel, R, threads, lds)                                                                                  \
  (head_dim == 64 ? (bf ? launch<kernel<bf16_t, 64, R>, threads>(lds(64), t, b, max_blocks, s)                            \
                        : launch<kernel<float, 64, R>, threads>(lds(64), t, b, max_blocks, s))                            \
                  : (bf ? launch<kernel<bf16_t, 128, R>, threads>(lds(128), t, b, max_blocks, s)                          \
                        : launch<kernel<float, 128, R>, threads>(lds(128), t, b, max_blocks, s)))
  if (rule) return reverse ? TN_PICK(attn_bwd_f32_kernel, true, 256, bwd_rule_lds) : TN_PICK(attn_f32_kernel, true, 512, fwd_rule_lds);
  return reverse ? TN_PICK(attn_bwd_f32_kernel, false, 256, bwd_lds) : TN_PICK(attn_f32_kernel, false, 256, fwd_lds);
#undef TN_PICK
}

}  // namespace tn
