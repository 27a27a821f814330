// Attention by a score rule (turnip.h: score_cap, slopes, spans) with bf16 products on the matrix cores: forward.
//
// One workgroup = one head x 128 query rows; each of its 4 wavefronts owns 32 of them, two workgroups share a compute unit.  Per
// 32 keys a wavefront forms the transposed scores S^T = K Q^T (MFMA 32x32x16), so that a lane owns one query -- its span, position and
// statistics are the lane's own scalars -- with the key rows fed in the permuted order pi(i) = 16 (a >> 1) + 8 g + 4 (a & 1) + b, i =
// 8 a + 4 g + b, which leaves a lane with 8 consecutive keys per 16-key slab: P^T is the B operand of O^T += V^T P^T.  The A
// operand, V^T, is read out of plain V rows by LDS reads that transpose (ds_read_b64_tr_b16: 16 lanes exchange 4 rows x 16
// columns), so V needs no transposed copy.
//
// Keys and values come 64 rows at a time through two LDS stages filled by direct global-to-LDS loads.  The 16-byte pieces of a
// row are stored in an order that depends on the row (`swizzle`), chosen so that neither the 16-byte reads of K (16 rows at one
// column) nor the transposing reads of V (4 rows at 4 columns per 32 lanes) meet in a bank.
//
// What a row sees is one interval of keys: spans, the causal bound and the block's end intersect to [lo, hi) per lane.  Chunks
// no row of the workgroup sees are skipped, 32-key slabs no row of the wavefront sees too, and only slabs that some row sees in
// part pay for masking.
//
// Weights enter the second product as single bf16 (half a step, 2^-8 relative, of each weight; the sum they are divided by is
// of the unrounded ones): the output is bf16 as well, and a second rounding of the same size under a sum that averages it
// costs less than the product with their remainders, which would be half as much again on the matrix cores.
#include "attn_rows.h"

#include <climits>

namespace tn {
namespace {

constexpr int kRuleRows = 128;  // query rows of a workgroup
constexpr int kRuleKeys = 64;   // keys per stage
constexpr float kLazyMax = 8.f; // see the rescaling step
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

// Where piece `piece` (16 bytes) of a row of 2 HD bytes is stored: reads of one piece of 16 rows, and of 4 pieces of 4 rows, fall on
// different banks.
template <int HD>
__device__ __forceinline__ int swizzle(int row) {
  return HD == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : ((row & 2) << 1) | ((row >> 2) & 3);
}

// tanh where an absolute error of 2^-23 is small beside the rounding of the weights: 1 - 2 / (exp(2 x) + 1)
__device__ __forceinline__ float tanh_of_scaled(float two_log2e_x) {
  return __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(two_log2e_x) + 1.f), 1.f);
}

__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = min(v, __shfl_xor(v, off, 64));
  return __builtin_amdgcn_readfirstlane(v);
}

// Head and row block of a workgroup.  Where the heads are a multiple of 8, every XCD gets heads of its own, whose keys and values
// its L2 then serves to all their row blocks; late rows, which under a causal mask see most, go first.
__device__ __forceinline__ void head_and_block(int bx, int hpg, int blocks, int& h, int& rb) {
  if ((hpg & 7) == 0) {
    h = (bx & 7) * (hpg >> 3) + (bx >> 3) / blocks;
    rb = (bx >> 3) % blocks;
  } else {
    h = bx / blocks;
    rb = bx % blocks;
  }
}

template <int HD, bool CAP, bool SLOPES>
__global__ void __launch_bounds__(256, 2) attn_rule_kernel(DeviceTables t, Batch b) {
  const OpDesc& d = t.descs[b.at(blockIdx.y)];
  if ((int)blockIdx.x >= d.nblocks) return;
  constexpr int CPR = HD / 8;                                   // pieces per row
  constexpr int KBYTES = kRuleKeys * HD * 2, STAGE = 2 * KBYTES;  // K chunk, then V chunk
  constexpr int NLD = kRuleKeys * CPR / 256;                    // loads per thread and operand
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int* ax = t.aux + d.aux0;
  const int tq = ax[0], tk = ax[1], tc = ax[2], q_rows = ax[3], kv_rows = ax[4];
  const int nc = d.p.n_col_tiles, gw = nc * tc, hpg = gw / HD;
  int h, rb;
  {
    const int blocks = (q_rows + kRuleRows - 1) / kRuleRows;
    head_and_block(blockIdx.x, hpg, blocks, h, rb);
    rb = blocks - 1 - rb;
  }
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l32 = lane & 31, g = lane >> 5;
  void* const* Qp = t.ptrs + d.ptr0;
  void* const* Kp = Qp + d.p.n_q_tiles * nc;
  void* const* Vp = Kp + d.p.n_kv_tiles * nc;
  const int row = rb * kRuleRows + w * 32 + l32;
  const bool exists = row < q_rows;
  const Rule rule(t, d);
  int lo = 0, hi = 0;
  if (exists) rule.visible(row, lo, hi);
  // of the wavefront: what some row sees, and what all rows that exist see
  const int w_begin = wave_min(lo < hi ? lo : INT_MAX), w_end = -wave_min(-hi);
  const int all_lo = -wave_min(exists ? -lo : INT_MAX), all_hi = wave_min(exists ? hi : INT_MAX);
  int begin, end;  // of the workgroup
  {
    int* const shared = (int*)lds;
    if (lane == 0) {
      shared[2 * w] = w_begin;
      shared[2 * w + 1] = w_end;
    }
    __syncthreads();
    begin = min(min(shared[0], shared[2]), min(shared[4], shared[6]));
    end = max(max(shared[1], shared[3]), max(shared[5], shared[7]));
    begin = begin < end ? begin & ~(kRuleKeys - 1) : end;
    begin = __builtin_amdgcn_readfirstlane(begin);
    end = __builtin_amdgcn_readfirstlane(end);
    __syncthreads();
  }

  bf16x8 qf[HD / 16];
#pragma unroll
  for (int s = 0; s < HD / 16; ++s)
    qf[s] = *(const bf16x8*)tile_elem<bf16_t>(Qp, nc, tq, tc, min(row, q_rows - 1), h * HD + s * 16 + g * 8);
  f32x16 ot[HD / 32];
#pragma unroll
  for (int i = 0; i < HD / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) ot[i][r] = 0.f;
  float m = -INFINITY, l = 0.f;

  // loader: piece p = i * 256 + tid of a chunk is stored at byte 16 p: row p / CPR, and there piece (p % CPR) ^ swizzle(row).  A head's
  // columns lie inside one column tile and a chunk inside one row tile (the executor checks both).
  const uint32_t lds0 = (uint32_t)(size_t)(lptr_t)lds;
  const int ct = (h * HD) / tc, cin0 = (h * HD) % tc;
  int rt = -1, trows = 0;
  const bf16_t* Kt = nullptr;
  const bf16_t* Vt = nullptr;
  auto issue = [&](int kv0, int stg) {
    const int nrt = kv0 / tk;
    if (nrt != rt) {
      rt = nrt;
      Kt = (const bf16_t*)sload_ptr((const void* const*)(Kp + rt * nc + ct));
      Vt = (const bf16_t*)sload_ptr((const void* const*)(Vp + rt * nc + ct));
      trows = min(tk, kv_rows - rt * tk);
    }
    const int kin = kv0 - rt * tk;
    const uint32_t dst = __builtin_amdgcn_readfirstlane(lds0 + stg * STAGE + w * 1024);
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      const int p = i * 256 + threadIdx.x, r = p / CPR;
      const size_t at = (size_t)min(kin + r, trows - 1) * tc + (cin0 + ((p % CPR) ^ swizzle<HD>(r)) * 8);  // rows past the end: one that exists, hidden below
      load_lds(Kt + at, dst + i * 4096);
      load_lds(Vt + at, dst + KBYTES + i * 4096);
    }
  };

  const float scale2 = d.p.scale * kLog2e;  // scores in units of log2: exp(x) = exp2(x log2 e)
  const float cap2 = rule.cap * kLog2e, into_tanh = 2.f * kLog2e * d.p.scale * rule.inv_cap;
  const float slope2 = SLOPES ? rule.slope(h) * kLog2e : 0.f;
  const float from_me = (float)(rule.q_pos0 + row - rule.k_pos0);  // distance of the block's first key
  const int a_ = l32 >> 3, b_ = l32 & 3, g_ = (l32 >> 2) & 1;
  const int kperm = 16 * (a_ >> 1) + 8 * g_ + 4 * (a_ & 1) + b_;
  // fragment addresses inside a stage.  K: row sub * 32 + kperm (whose swizzle sub leaves alone), piece 2 s + g.  V: rows 8 g + 4 i +
  // (lane & 15) / 4 of a slab of 16 keys, 16 columns from 16 * (lane >> 4 & 1), 4 of them from 4 * (lane & 3).
  const int k_at = kperm * (HD * 2), k_sw = swizzle<HD>(kperm);
  const int v_row = 8 * g + ((lane & 15) >> 2), v_piece = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), v_in = (lane & 1) * 8;

  if (begin < end) issue(begin, 0);
  int stg = 0;
  for (int kv0 = begin; kv0 < end; kv0 += kRuleKeys, stg ^= 1) {
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this chunk has arrived
    __syncthreads();                     // ... for everybody, and everybody is done with the other stage
    if (kv0 + kRuleKeys < end) issue(kv0 + kRuleKeys, stg ^ 1);
    const char* kb = lds + stg * STAGE;
    const char* vb = kb + KBYTES;
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      const int kvs = kv0 + sub * 32;
      if (kvs + 32 <= w_begin || kvs >= w_end) continue;
      f32x16 s;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
      for (int j = 0; j < HD / 16; ++j)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(kb + sub * 32 * (HD * 2) + k_at + ((2 * j + g) ^ k_sw) * 16), qf[j], s, 0, 0, 0);
      // register r of this lane: key kvs + 16 (r >> 3) + 8 g + (r & 7)
      const float base = from_me - (float)(kvs + 8 * g);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (CAP) s[r] = cap2 * tanh_of_scaled(s[r] * into_tanh);
        else s[r] *= scale2;
        if (SLOPES) s[r] = __builtin_fmaf(-slope2, fabsf(base - (float)(16 * (r >> 3) + (r & 7))), s[r]);
      }
      float mx = -INFINITY;
      if (kvs < all_lo || kvs + 32 > all_hi) {
        const int first = lo - kvs - 8 * g;
        const uint32_t len = hi - lo;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = (uint32_t)(16 * (r >> 3) + (r & 7) - first) < len ? s[r] : -INFINITY;
          mx = fmaxf(mx, s[r]);
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
      }
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mn = fmaxf(m, mx);
      // What is summed so far is rescaled only when the maximum of some query of the wavefront has grown by more than kLazyMax (in
      // units of log2): until then weights are relative to the older maximum and stay below 2^kLazyMax.
      if (__any(mn > m + kLazyMax)) {
        const float alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
        l *= alpha;
#pragma unroll
        for (int i = 0; i < HD / 32; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) ot[i][r] *= alpha;
        m = mn;
      }
      const float msub = m == -INFINITY ? 0.f : m;  // nothing seen yet: every weight is exp2(-inf) = 0
      union { uint32_t u[4]; bf16x8 v; } p[2];
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const float pa = __builtin_amdgcn_exp2f(s[r] - msub), pb = __builtin_amdgcn_exp2f(s[r + 1] - msub);
        l += pa + pb;
        p[r >> 3].u[(r & 7) >> 1] = f2bf2(pa, pb);
      }
      // O^T[d, q] += sum over 16 keys of V^T[d, key] P^T[key, q]
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) {
          union { s16x4 h[2]; bf16x8 v; } a;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = sub * 32 + ks * 16 + 4 * e + v_row;
            a.h[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(vb + r * (HD * 2) + ((i * 4 + v_piece) ^ swizzle<HD>(r)) * 16 + v_in));
          }
          ot[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, p[ks].v, ot[i], 0, 0, 0);
        }
    }
  }
  // a weight of zero times an infinity or NaN of a key the row does not see: such rows are formed again
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < HD / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) z = fmaf(ot[i][r], 0.f, z);
  if (__builtin_expect(__any(exists && !(z == 0.f)), 0)) {
    const int first = rb * kRuleRows + w * 32;
    return attn_by_rows<bf16_t, HD, true>(t, d, h, first, first + 32, lane >> 4, 4);
  }
  l += __shfl_xor(l, 32, 64);
  if (!exists) return;
  if (ax[kRuleFinish]) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bf16_t* out = (bf16_t*)d.out + (size_t)row * gw + h * HD + 4 * g;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i)
#pragma unroll
      for (int a = 0; a < 4; ++a)
        *(uint2*)(out + i * 32 + 8 * a) = make_uint2(f2bf2(ot[i][4 * a] * inv, ot[i][4 * a + 1] * inv), f2bf2(ot[i][4 * a + 2] * inv, ot[i][4 * a + 3] * inv));
    return;
  }
  float* out = (float*)d.out + (size_t)row * d.cols;
#pragma unroll
  for (int i = 0; i < HD / 32; ++i)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      float* o4 = out + h * HD + i * 32 + 8 * a + 4 * g;
      if ((d.cols & 3) == 0) {  // rows of the partial are 16-byte aligned
        *(float4*)o4 = make_float4(ot[i][4 * a], ot[i][4 * a + 1], ot[i][4 * a + 2], ot[i][4 * a + 3]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) o4[k] = ot[i][4 * a + k];
      }
    }
  if (g == 0) {
    out[gw + h] = m * 0.69314718055994530942f;  // back to natural-log units for the combine step
    out[gw + hpg + h] = l;
  }
}

template <auto kernel>
hipError_t launch(int threads, int lds, const DeviceTables& t, const Batch& b, int32_t max_blocks, hipStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  if (lds > 65536)
    if (const hipError_t e = allow_lds(allowed, (const void*)kernel, lds); e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)max_blocks, (unsigned)b.n), dim3(threads), lds, s, t, b);
  return hipGetLastError();
}

template <int HD>
hipError_t launch_forward(int rule, const DeviceTables& t, const Batch& b, int32_t n, hipStream_t s) {
  constexpr int lds = 4 * kRuleKeys * HD * 2;
  switch (rule) {
    case 0: return launch<attn_rule_kernel<HD, false, false>>(256, lds, t, b, n, s);
    case kRuleHasCap: return launch<attn_rule_kernel<HD, true, false>>(256, lds, t, b, n, s);
    case kRuleHasSlopes: return launch<attn_rule_kernel<HD, false, true>>(256, lds, t, b, n, s);
    default: return launch<attn_rule_kernel<HD, true, true>>(256, lds, t, b, n, s);
  }
}

}  // namespace

int32_t attn_rule_blocks(int cls, const OpDesc& d, const int32_t* aux) {
  const int32_t* ax = aux + d.aux0;
  return d.p.n_col_tiles * ax[2] / d.p.head_dim * ((ax[3] + kRuleRows - 1) / kRuleRows);
}

hipError_t launch_attn_rule(int cls, int head_dim, const DeviceTables& t, const Batch& b, int32_t max_blocks, hipStream_t s) {
  if (head_dim == 64) return launch_forward<64>(cls - LC_ATTN_RULE_BF16, t, b, max_blocks, s);
  if (head_dim == 128) return launch_forward<128>(cls - LC_ATTN_RULE_BF16, t, b, max_blocks, s);
  return hipErrorInvalidValue;
}

}  // namespace tn
