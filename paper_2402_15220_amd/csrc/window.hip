// gfx950 (MI355X) decode attention over a plan (plan.hpp): rows that see a
// sliding window and sinks of their paths, over fp16, fp32 and 4-bit pools,
// and every decode call over a 4-bit pool.
//
// A row of length L, its query at position L - 1, sees the positions j < L
// with j < sinks or j >= L - window:
//   o = sum_j softmax_j(scale q.k_j) v_j.
// One block per (item, head): up to 16 query rows over up to 64 chunks that
// they share, or one row over its own. The four wavefronts take steps of 32
// tokens (fp32: 16) in turn, each with its own softmax state (m, n, O^T),
// and are folded (Eqn 2 of the paper) at the end; a row with several items
// leaves partials, and the last of its blocks to arrive folds them.
//
// S^T = K Q^T and O^T += V^T P^T run on the matrix cores with tokens, then
// channels, as M and query rows as N (a lane holds column n = lane % 16 in
// its group g = lane / 16), so P stays in the registers S^T came out in:
// tokens 4g .. 4g + 3 of each 16. A lone row fills one of the 16 columns; its
// matrix ops still take less of the chip than the memory it waits for.
//   fp16   K rows are the A operand as loaded; V rows are turned over through
//          the wavefront's own LDS tile (ds_read_b64_tr_b16).
//   fp32   16x16x4 ops; element j of a lane's 16-byte load belongs to op j,
//          for K along d, for V along the channels, so nothing is turned over.
//   4-bit  the codes as stored are the operands: masking a word leaves codes in
//          the low (or second) four bits of fp16 halves, that is code * 2^-24
//          (or * 2^-20, undone in q and in P), which fp16 matrix ops take
//          exactly. With k = low_k + s_k code, v = low_v + s_v code:
//            q.k = s_k (q.code) + low_k sum(q),
//            sum p v = sum (p s_v) (code - 8) + sum p (low_v + 8 s_v);
//          p s_v is rounded to fp16 for the matrix op, relative to a running
//          reference of the scales so that it neither overflows nor leaves
//          the normal range, and the -8 takes the same rounded weights, so
//          that rounding acts on codes of -8..7 instead of 0..15.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cstdint>

#include "device_common.hpp"
#include "kernels.hpp"
#include "kv4.hpp"

namespace ca {
namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// slack of the softmax reference maximum, in log2 units: P <= 2^kLazy, so
// that most steps leave the accumulators alone
constexpr float kLazy = 4.f;
// 4-bit: the largest scale in use stands for 2^kScaleTop, so P s_v <= 2^15
constexpr float kScaleTop = 2048.f;

template <int S>
struct Traits;
template <>
struct Traits<kStoreF16> {
  using T = _Float16;
  static constexpr int kTiles = 2;  // 16-token tiles of a step
};
template <>
struct Traits<kStoreF32> {
  using T = float;
  static constexpr int kTiles = 1;
};
template <>
struct Traits<kStoreKv4> {
  using T = _Float16;
  static constexpr int kTiles = 2;
};

// What one step loads, per lane.
template <int S, int D>
struct Stage;
template <int D>
struct Stage<kStoreF16, D> {
  half8 k[2][D / 32];
  u32x4 v[D / 16];  // granules of the 32 x D block, row-major
};
template <int D>
struct Stage<kStoreF32, D> {
  floatx4 k[D / 16];
  floatx4 v[4][D / 64];
};
template <int D>
struct Stage<kStoreKv4, D> {
  uint32_t k[2][D / 32];
  uint32_t v[2][D / 32];
  u32x4 kp[2], vp[2];  // (scale, low) of tokens 4g .. 4g + 3
};

// Where a step's tokens lie: wave-uniform.
struct Place {
  int slot[2];
  int row[2];  // first row of the tile in its chunk
  int pos[2];  // its position
  int end[2];  // position after the chunk's last token; <= pos: no token
};

// A (scale, low) pair. (__builtin_bit_cast of a vector's element itself reads
// element 0 whatever the index: the element is copied out first.)
__device__ __forceinline__ half2v param(const u32x4& v, int i) {
  const uint32_t w = v[i];
  return __builtin_bit_cast(half2v, w);
}

__device__ __forceinline__ half8 unpack8(uint32_t w) {
  const uint32_t x = w >> 8;
  const u32x4 r = {w & 0x000f000fu, w & 0x00f000f0u, x & 0x000f000fu, x & 0x00f000f0u};
  return __builtin_bit_cast(half8, r);
}

__device__ __forceinline__ bool any_nonfinite(half8 x) {
  const u32x4 r = __builtin_bit_cast(u32x4, x);
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad |= ((r[i] & 0x7c00u) == 0x7c00u) || ((r[i] & 0x7c000000u) == 0x7c000000u);
  return bad;
}

template <int S, int D>
__global__ __launch_bounds__(256) void kwd_kernel(PlanArgs A) {
  using T = typename Traits<S>::T;
  constexpr int TP = Traits<S>::kTiles;
  constexpr int KS = D / 32, DT = D / 16;
  constexpr int VS = D + 16;                   // V tile row stride in LDS (halves)
  constexpr int OS = D + 4;                    // merge buffer row stride (floats)
  constexpr int VB = S == kStoreF16 ? 4 * 32 * VS * 2 : 0;
  constexpr int MB = 4 * kPlanRows * OS * 4;
  constexpr int BIG = VB > MB ? VB : MB;
  __shared__ __align__(16) char lds[BIG];
  __shared__ float s_m[4][kPlanRows], s_n[4][kPlanRows];
  __shared__ int s_last[kPlanRows];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int H = A.H, C = A.C;
  const int h = static_cast<int>(blockIdx.x % static_cast<unsigned>(H));
  const int ib = static_cast<int>(blockIdx.x / static_cast<unsigned>(H));
  const PlanItem item = A.items[ib];
  // the chunks, one a lane (chunk_stride <= 64)
  const PlanChunk my = A.chunks[static_cast<size_t>(ib) * A.chunk_stride + min(lane, A.chunk_stride - 1)];
  const int nr = item.n_rows, nch = item.n_chunks;
  const PlanRow prow = A.rows[item.row_begin + min(n16, nr - 1)];
  const int io = A.row_map ? A.row_map[item.row_begin + min(n16, nr - 1)] : item.row_begin + min(n16, nr - 1);
  const int len = prow.last_start + A.slot_len[prow.last_slot];
  const int lo = max(0, len - A.window);
  const int sinks = A.sinks;

  // q as the B operand of S^T; a lane past the rows repeats the last one.
  // 4-bit: q times 2^-e with |q| 2^-e in [2^10, 2^11], so that neither the
  // 2^-4 of the second code of a pair nor a small q leaves the normal range.
  const T* qrow = static_cast<const T*>(A.q) + (static_cast<size_t>(io) * H + h) * D;
  half8 qf[S == kStoreF32 ? 1 : KS];
  floatx4 qx[S == kStoreF32 ? D / 16 : 1];
  float qk = 0.f, ql = 0.f;  // 4-bit: factors of s_k and low_k
  if constexpr (S == kStoreF32) {
#pragma unroll
    for (int u = 0; u < D / 16; ++u) qx[u] = *reinterpret_cast<const floatx4*>(qrow + 16 * u + 4 * g);
  } else if constexpr (S == kStoreF16) {
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const half8*>(qrow + 32 * s + 8 * g);
  } else {
    float amax = 0.f, sum = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qf[s] = *reinterpret_cast<const half8*>(qrow + KS * 8 * g + 8 * s);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = static_cast<float>(qf[s][i]);
        amax = fmaxf(amax, fabsf(x));
        sum += x;
      }
    }
    amax = rows4_max(amax);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const int e = amax > 0.f && amax < INFINITY ? 11 - __builtin_amdgcn_frexp_expf(amax) : 0;
    const float up = __builtin_amdgcn_ldexpf(1.f, e);
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        qf[s][i] = static_cast<_Float16>(static_cast<float>(qf[s][i]) * ((i & 2) ? up * 0.0625f : up));
    qk = __builtin_amdgcn_ldexpf(A.qscale, 24 - e);
    ql = A.qscale * sum;
  }

  const char* kbase = static_cast<const char*>(A.kpool);
  const char* vbase = static_cast<const char*>(A.vpool);
  constexpr int ES = S == kStoreF16 ? 2 : S == kStoreF32 ? 4 : 1;
  const int64_t ssb = A.ss * ES, hsb = A.hs * ES;

  // tiles per chunk; a step is TP tiles of one chunk, or, over chunks of at
  // most 16 tokens, one tile each of TP chunks
  const int tpc = (C + 15) >> 4;
  const bool small = tpc == 1;
  const int spc = small ? 1 : (tpc + TP - 1) / TP;  // steps of a chunk (or of TP small ones)
  const int ngrp = small ? (nch + TP - 1) / TP : nch;
  const int steps = ngrp * spc;
  auto place = [&](int st) {
    Place p;
    const int c = st / spc, sub = st - c * spc;
#pragma unroll
    for (int t = 0; t < TP; ++t) {
      const int cj = small ? min(c * TP + t, nch - 1) : c;
      const int tile = small ? 0 : sub * TP + t;
      p.slot[t] = __builtin_amdgcn_readlane(my.slot, cj);
      const int start = __builtin_amdgcn_readlane(my.start, cj);
      const int end = __builtin_amdgcn_readlane(my.end, cj);
      const bool there = small ? c * TP + t < nch : tile < tpc;
      p.row[t] = there ? tile * 16 : 0;
      p.pos[t] = start + p.row[t];
      p.end[t] = there ? end : 0;
    }
    return p;
  };
  // nothing of the step is seen, whatever the rows' present lengths
  auto hidden = [&](const Place& p) {
    bool hid = true;
#pragma unroll
    for (int t = 0; t < TP; ++t) {
      const int last = min(p.end[t], p.pos[t] + 16) - 1;
      hid &= last < p.pos[t] || (p.pos[t] >= sinks && last < item.lo);
    }
    return hid;
  };
  auto next = [&](int st, Place& p) {  // first step at or after st of this wavefront that is seen
    for (; st < steps; st += 4) {
      p = place(st);
      if (!hidden(p)) break;
    }
    return st;
  };

  // Rows past a chunk's last token are loaded all the same (a tile's rows
  // exist in the pool up to the chunk size; beyond it the last row is read
  // again) and masked.
  auto load = [&](Stage<S, D>& x, const Place& p) {
    if constexpr (S == kStoreF16) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char* kt = kbase + p.slot[t] * ssb + h * hsb;
        const int r = min(p.row[t] + n16, C - 1);
#pragma unroll
        for (int s = 0; s < KS; ++s)
          x.k[t][s] = *reinterpret_cast<const half8*>(kt + static_cast<size_t>(r) * (D * 2) + 64 * s + 16 * g);
      }
      constexpr int GPR = D / 8, RPL = 64 / GPR;  // granules a row, rows a load
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const int t = i / (D / 32);
        const int r = min(p.row[t] + (i % (D / 32)) * RPL + lane / GPR, C - 1);
        x.v[i] = *reinterpret_cast<const u32x4*>(vbase + p.slot[t] * ssb + h * hsb +
                                                 static_cast<size_t>(r) * (D * 2) + 16 * (lane % GPR));
      }
    } else if constexpr (S == kStoreF32) {
      const char* kt = kbase + p.slot[0] * ssb + h * hsb;
      const char* vt = vbase + p.slot[0] * ssb + h * hsb;
      const int r = min(p.row[0] + n16, C - 1);
#pragma unroll
      for (int u = 0; u < D / 16; ++u)
        x.k[u] = *reinterpret_cast<const floatx4*>(kt + static_cast<size_t>(r) * (D * 4) + 64 * u + 16 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int rv = min(p.row[0] + 4 * g + i, C - 1);
#pragma unroll
        for (int u = 0; u < D / 64; ++u)
          x.v[i][u] = *reinterpret_cast<const floatx4*>(vt + static_cast<size_t>(rv) * (D * 4) + 256 * u + 16 * n16);
      }
    } else {
      const int pb = kv4_rows(C) * (D / 2);  // the parameters' place in the tile
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char* kt = kbase + p.slot[t] * ssb + h * hsb;
        const char* vt = vbase + p.slot[t] * ssb + h * hsb;
        const char* kc = kt + (p.row[t] + n16) * (D / 2) + g * (D / 8);
        const char* vc = vt + p.row[t] * (D / 2) + lane * (D / 8);
        if constexpr (D == 128) {
          const u32x4 a = *reinterpret_cast<const u32x4*>(kc), b = *reinterpret_cast<const u32x4*>(vc);
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            x.k[t][s] = a[s];
            x.v[t][s] = b[s];
          }
        } else {
          const u32x2 a = *reinterpret_cast<const u32x2*>(kc), b = *reinterpret_cast<const u32x2*>(vc);
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            x.k[t][s] = a[s];
            x.v[t][s] = b[s];
          }
        }
        x.kp[t] = *reinterpret_cast<const u32x4*>(kt + pb + (p.row[t] + 4 * g) * 4);
        x.vp[t] = *reinterpret_cast<const u32x4*>(vt + pb + (p.row[t] + 4 * g) * 4);
      }
    }
  };

  float m_run = kNegBig, n_run = 0.f;
  float base = 0.f, corr = 0.f;  // 4-bit: sum p (low_v + 8 s_v); sum of rounded weights
  float s_ref = 0.f;             // 4-bit: scale that stands for kScaleTop (uniform)
  floatx4 acc[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  _Float16* vl = reinterpret_cast<_Float16*>(lds) + wv * (32 * VS);

  // bounds over the item's rows: a tile inside them needs no mask
  int lo_max = lo, lo_min = lo, len_min = len, len_max = len;
#pragma unroll
  for (int x = 1; x < 16; x <<= 1) {
    lo_max = max(lo_max, __shfl_xor(lo_max, x));
    lo_min = min(lo_min, __shfl_xor(lo_min, x));
    len_min = min(len_min, __shfl_xor(len_min, x));
    len_max = max(len_max, __shfl_xor(len_max, x));
  }
  lo_max = __builtin_amdgcn_readfirstlane(lo_max);
  lo_min = __builtin_amdgcn_readfirstlane(lo_min);
  len_min = __builtin_amdgcn_readfirstlane(len_min);
  len_max = __builtin_amdgcn_readfirstlane(len_max);

  auto compute = [&](Stage<S, D>& x, const Place& p) {
    bool whole[TP], all = true;
#pragma unroll
    for (int t = 0; t < TP; ++t) {
      const int last = p.pos[t] + 16;
      whole[t] = last <= p.end[t] && last <= len_min && (p.pos[t] >= lo_max || last <= sinks);
      all &= whole[t];
    }
    // token i of this lane's four in tile t, seen by row (l, b): by any row
    // with the extreme bounds
    auto seen = [&](int t, int i, int l, int b) {
      const int j = p.pos[t] + i;
      return j < p.end[t] && j < l && (j >= b || j < sinks);
    };
    float sc[TP][4];
#pragma unroll
    for (int t = 0; t < TP; ++t) {
      floatx4 a = {0.f, 0.f, 0.f, 0.f};
      if constexpr (S == kStoreF32) {
#pragma unroll
        for (int u = 0; u < D / 16; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            a = __builtin_amdgcn_mfma_f32_16x16x4f32(x.k[u][j], qx[u][j], a, 0, 0, 0);
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          half8 kk;
          if constexpr (S == kStoreF16) kk = x.k[t][s];
          else kk = unpack8(x.k[t][s]);
          a = __builtin_amdgcn_mfma_f32_16x16x32_f16(kk, qf[s], a, 0, 0, 0);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (S == kStoreKv4) {
          const half2v kp = param(x.kp[t], i);
          sc[t][i] = __builtin_fmaf(a[i], static_cast<float>(kp[0]) * qk, static_cast<float>(kp[1]) * ql);
        } else {
          sc[t][i] = a[i] * A.qscale;
        }
      }
      if (!whole[t]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!seen(t, 4 * g + i, len, lo)) sc[t][i] = -INFINITY;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < TP; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[t][i]);
    mx = rows4_max(mx);
    const float mn = mx > m_run + kLazy ? mx : m_run;
    if (__any(mn != m_run)) {
      const float al = fast_exp2(m_run - mn);
      n_run *= al;
      base *= al;
      corr *= al;
#pragma unroll
      for (int t = 0; t < DT; ++t) acc[t] *= al;
      m_run = mn;
    }
    float pr[TP][4];
#pragma unroll
    for (int t = 0; t < TP; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) pr[t][i] = fast_exp2(sc[t][i] - m_run);

    if constexpr (S == kStoreF32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) n_run += pr[0][i];
      if (!all) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!seen(0, 4 * g + i, len_max, lo_min))
#pragma unroll
            for (int u = 0; u < D / 64; ++u) x.v[i][u] = floatx4{0.f, 0.f, 0.f, 0.f};
        // a token that some rows see and others do not: where its V is not
        // finite, 0 * V would reach the others, so each column gets its own
        // operand (never in ordinary data)
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int u = 0; u < D / 64; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) bad |= !(fabsf(x.v[i][u][j]) < INFINITY);
        if (nr > 1 && __any(bad)) {
          for (int c = 0; c < nr; ++c) {
            const int lc = __builtin_amdgcn_readlane(len, c), bc = __builtin_amdgcn_readlane(lo, c);
#pragma unroll
            for (int u = 0; u < D / 64; ++u)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                floatx4 tmp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  tmp = __builtin_amdgcn_mfma_f32_16x16x4f32(
                      seen(0, 4 * g + i, lc, bc) ? x.v[i][u][j] : 0.f, pr[0][i], tmp, 0, 0, 0);
                if (n16 == c) acc[4 * u + j] += tmp;
              }
          }
          return;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int u = 0; u < D / 64; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[4 * u + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[i][u][j], pr[0][i], acc[4 * u + j], 0, 0, 0);
    } else if constexpr (S == kStoreF16) {
      half8 pb;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pb[4 * t + i] = static_cast<_Float16>(pr[t][i]);
          n_run += static_cast<float>(pb[4 * t + i]);
        }
      constexpr int GPR = D / 8, RPL = 64 / GPR;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const int t = i / (D / 32), r = (i % (D / 32)) * RPL + lane / GPR;
        u32x4 y = x.v[i];
        if (!all && !seen(t, r, len_max, lo_min)) y = u32x4{0, 0, 0, 0};
        *reinterpret_cast<u32x4*>(vl + (16 * t + r) * VS + 8 * (lane % GPR)) = y;
      }
      // the wavefront's own tile: its LDS ops complete in order
      compiler_fence();
      half8 va[DT];
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const _Float16* at = vl + (4 * g + (n16 >> 2)) * VS + 16 * d + 4 * (n16 & 3);
        const half4 a = lds_read_tr16(at), b = lds_read_tr16(at + 16 * VS);
        va[d] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
      }
      compiler_fence();
      if (!all && nr > 1) {
        bool bad = false;
#pragma unroll
        for (int d = 0; d < DT; ++d) bad |= any_nonfinite(va[d]);
        if (__any(bad)) {  // as for fp32 above
          for (int c = 0; c < nr; ++c) {
            const int lc = __builtin_amdgcn_readlane(len, c), bc = __builtin_amdgcn_readlane(lo, c);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
              half8 vc = va[d];
#pragma unroll
              for (int k = 0; k < 8; ++k)
                if (!seen(k / 4, 4 * g + k % 4, lc, bc)) vc[k] = static_cast<_Float16>(0.f);
              const floatx4 tmp =
                  __builtin_amdgcn_mfma_f32_16x16x32_f16(vc, pb, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
              if (n16 == c) acc[d] += tmp;
            }
          }
          return;
        }
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va[d], pb, acc[d], 0, 0, 0);
    } else {
      float sv[2][4], lv[2][4];
      float smax = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const half2v vp = param(x.vp[t], i);
          sv[t][i] = static_cast<float>(vp[0]);
          lv[t][i] = static_cast<float>(vp[1]);
          if (!whole[t]) {
            // a place without a token, or one this row does not see: whatever
            // is stored there adds nothing
            const bool on = seen(t, 4 * g + i, len, lo);
            sv[t][i] = on ? sv[t][i] : 0.f;
            lv[t][i] = on ? lv[t][i] : 0.f;
          }
          smax = fmaxf(smax, sv[t][i]);
        }
      if (__any(smax > s_ref)) {
        const float s_new = wave_max(smax) * 2.f;
        const float al = s_ref / s_new;  // s_new > s_ref >= 0
        corr *= al;
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] *= al;
        s_ref = s_new;
      }
      const float f = s_ref > 0.f ? kScaleTop / s_ref : 0.f;
      half8 pb;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          n_run += pr[t][i] + pr[t][i + 1];
          base = __builtin_fmaf(pr[t][i], __builtin_fmaf(8.f, sv[t][i], lv[t][i]), base);
          base = __builtin_fmaf(pr[t][i + 1], __builtin_fmaf(8.f, sv[t][i + 1], lv[t][i + 1]), base);
          const float u = i ? f * 0.0625f : f;  // the second pair's codes stand 2^4 higher
          const half2v w = {static_cast<_Float16>(pr[t][i] * sv[t][i] * u),
                            static_cast<_Float16>(pr[t][i + 1] * sv[t][i + 1] * u)};
          const _Float16 one = static_cast<_Float16>(i ? 16.f : 1.f);
          corr = __builtin_amdgcn_fdot2(w, half2v{one, one}, corr, false);
          pb[4 * t + i] = w[0];
          pb[4 * t + i + 1] = w[1];
        }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const half8 a = unpack8(x.v[0][s]), b = unpack8(x.v[1][s]);
        const half8 even = __builtin_shufflevector(a, b, 0, 1, 2, 3, 8, 9, 10, 11);
        const half8 odd = __builtin_shufflevector(a, b, 4, 5, 6, 7, 12, 13, 14, 15);
        acc[2 * s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(even, pb, acc[2 * s], 0, 0, 0);
        acc[2 * s + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(odd, pb, acc[2 * s + 1], 0, 0, 0);
      }
    }
  };

  {
    Stage<S, D> xa, xb;
    Place pa, pb;
    int sa = next(wv, pa);
    if (sa < steps) load(xa, pa);
    while (sa < steps) {
      const int sb = next(sa + 4, pb);
      if (sb < steps) load(xb, pb);
      compute(xa, pa);
      if (sb >= steps) break;
      sa = next(sb + 4, pa);
      if (sa < steps) load(xa, pa);
      compute(xb, pb);
    }
  }

  // Fold the four wavefronts (Eqn 2) through LDS: [wave][row][channel].
  float n_col = n_run;
  n_col += __shfl_xor(n_col, 16);
  n_col += __shfl_xor(n_col, 32);
  if constexpr (S == kStoreKv4) {
    base += __shfl_xor(base, 16);
    base += __shfl_xor(base, 32);
    corr += __shfl_xor(corr, 16);
    corr += __shfl_xor(corr, 32);
    const float back = s_ref * (1.f / kScaleTop);
    const float off = base - 8.f * corr * back;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[d][i] = __builtin_fmaf(acc[d][i], 16777216.f * back, off);
  }
  if constexpr (S == kStoreF16) __syncthreads();  // the V tiles' place is used again
  float* mb = reinterpret_cast<float*>(lds);
  if (n16 < nr) {
    float* at = mb + (wv * kPlanRows + n16) * OS;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      if constexpr (S == kStoreF32) {
        // op tile 4u + j, element i: channel 64u + 16g + 4i + j
#pragma unroll
        for (int i = 0; i < 4; ++i) at[64 * (d / 4) + 16 * g + 4 * i + d % 4] = acc[d][i];
      } else {
        *reinterpret_cast<floatx4*>(at + 16 * d + 4 * g) = acc[d];
      }
    }
    if (g == 0) {
      s_m[wv][n16] = m_run;
      s_n[wv][n16] = n_col;
    }
  }
  __syncthreads();
  constexpr int TPR = D / 4, NG = 256 / TPR;  // threads a row, rows at once
  const int gi = tid / TPR, ch = 4 * (tid % TPR);
  const __amdgpu_buffer_rsrc_t rs = part_rsrc(A.ws_o, A.ws_o_bytes);
  T* out = static_cast<T*>(A.o);
  auto write_row = [&](int row, const floatx4& v, float n) {
    const int r = A.row_map ? A.row_map[row] : row;
    T* at = out + (static_cast<size_t>(r) * H + h) * D + ch;
    const float inv = 1.f / n;
    if constexpr (S == kStoreF32) {
      *reinterpret_cast<floatx4*>(at) = v * inv;
    } else {
      half4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = static_cast<_Float16>(v[i] * inv);
      *reinterpret_cast<half4*>(at) = y;
    }
  };
  for (int r = gi; r < nr; r += NG) {
    float m = fmaxf(fmaxf(s_m[0][r], s_m[1][r]), fmaxf(s_m[2][r], s_m[3][r]));
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    float n = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = fast_exp2(s_m[w][r] - m);
      n += s_n[w][r] * f;
      v += *reinterpret_cast<const floatx4*>(mb + (w * kPlanRows + r) * OS + ch) * f;
    }
    const PlanRow pr = A.rows[item.row_begin + r];
    if (pr.np == 1) {
      write_row(item.row_begin + r, v, n);
    } else {
      const int p = pr.pbase + item.ord;
      st_dev4(rs, ((static_cast<uint32_t>(p) * H + h) * D + ch) * 4u, v[0], v[1], v[2], v[3]);
      if (ch == 0) {
        float* ml = A.ws_ml + (static_cast<size_t>(p) * H + h) * 2;
        st_dev(ml, m);
        st_dev(ml + 1, n);
      }
    }
  }
  // Partials: the last block to arrive on a row folds them (the exchange
  // protocol of device_common.hpp).
  wait_stores();
  __syncthreads();
  if (tid < nr) {
    const PlanRow pr = A.rows[item.row_begin + tid];
    bool last = false;
    if (pr.np > 1) {
      const int row = item.row_begin + tid;
      int32_t* c = A.cnt_layout < 0 ? A.cnt + (static_cast<size_t>(row) * H + h)
                                    : A.cnt + (static_cast<size_t>(row >> A.cnt_layout) * H + h) * 32 +
                                          (row & ((1 << A.cnt_layout) - 1));
      last = arrive_last(c, pr.np);
    }
    s_last[tid] = last;
  }
  __syncthreads();
  auto fold_from = [&](int p0, int step, int p1, float& m, float& n, floatx4& v) {
    for (int p = p0; p < p1; p += step) {
      const float* ml = A.ws_ml + (static_cast<size_t>(p) * H + h) * 2;
      const float pm = ld_dev(ml), pn = ld_dev(ml + 1);
      const float4 x = ld_dev4(rs, ((static_cast<uint32_t>(p) * H + h) * D + ch) * 4u);
      const float M = fmaxf(m, pm);
      const float a = fast_exp2(m - M), b = fast_exp2(pm - M);
      n = n * a + pn * b;
      v = v * a + floatx4{x.x, x.y, x.z, x.w} * b;
      m = M;
    }
  };
  if (nr > 1) {  // a row to each group of threads
    for (int r = gi; r < nr; r += NG) {
      if (!s_last[r]) continue;
      const PlanRow pr = A.rows[item.row_begin + r];
      float m = kNegBig, n = 0.f;
      floatx4 v = {0.f, 0.f, 0.f, 0.f};
      fold_from(pr.pbase, 1, pr.pbase + pr.np, m, n, v);
      write_row(item.row_begin + r, v, n);
    }
  } else if (s_last[0]) {  // one row: its partials dealt out to the groups
    const PlanRow pr = A.rows[item.row_begin];
    float m = kNegBig, n = 0.f;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    fold_from(pr.pbase + gi, NG, pr.pbase + pr.np, m, n, v);
    *reinterpret_cast<floatx4*>(mb + gi * OS + ch) = v;
    float* gm = mb + NG * OS;
    if (ch == 0) {
      gm[2 * gi] = m;
      gm[2 * gi + 1] = n;
    }
    __syncthreads();
    if (gi == 0) {
      float M = kNegBig;
      for (int k = 0; k < NG; ++k) M = fmaxf(M, gm[2 * k]);
      floatx4 o = {0.f, 0.f, 0.f, 0.f};
      float nn = 0.f;
      for (int k = 0; k < NG; ++k) {
        const float f = fast_exp2(gm[2 * k] - M);
        nn += gm[2 * k + 1] * f;
        o += *reinterpret_cast<const floatx4*>(mb + k * OS + ch) * f;
      }
      write_row(item.row_begin, o, nn);
    }
  }
}

}  // namespace

hipError_t launch_plan_attention(const PlanArgs& a, hipStream_t stream) {
  if (a.n_items <= 0) return hipSuccess;
  if (a.chunk_stride < 1 || a.chunk_stride > kPlanChunks) return hipErrorInvalidValue;
  const unsigned grid = static_cast<unsigned>(a.n_items) * static_cast<unsigned>(a.H);
  auto go = [&](auto kernel) { kernel<<<grid, 256, 0, stream>>>(a); };
  if (a.D == 128) {
    if (a.store == kStoreF16) go(kwd_kernel<kStoreF16, 128>);
    else if (a.store == kStoreF32) go(kwd_kernel<kStoreF32, 128>);
    else go(kwd_kernel<kStoreKv4, 128>);
  } else if (a.D == 64) {
    if (a.store == kStoreF16) go(kwd_kernel<kStoreF16, 64>);
    else if (a.store == kStoreF32) go(kwd_kernel<kStoreF32, 64>);
    else go(kwd_kernel<kStoreKv4, 64>);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace ca
