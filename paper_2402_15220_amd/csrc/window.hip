// gfx950 (MI355X) decode attention over a plan (plan.hpp): rows that see a
// sliding window and sinks of their paths, over fp16, fp32 and 4-bit pools,
// and every decode call over a 4-bit pool.
//
// A row of length L, its query at position L - 1, sees the positions j < L
// with j < sinks or j >= L - window:
//   o = sum_j softmax_j(scale q.k_j) v_j.
// One block per (item, head): up to 16 query rows over up to 64 chunks that
// they share, or one row over its own. The four wavefronts take steps of
// tokens in turn, each with its own softmax state (m, n, O), and are folded
// (Eqn 2 of the paper) at the end; a row with several items leaves partials,
// and the last of its blocks to arrive folds them. Items of single rows that are
// long and many go a head to a wavefront, four heads to a block (plan.cpp).
//
// Rows that share (rows_shared): S^T = K Q^T and O^T += V^T P^T run on the
// matrix cores with tokens, then channels, as M and query rows as N (a lane
// holds column n = lane % 16 in its group g = lane / 16), so P stays in the
// registers S^T came out in: tokens 4g .. 4g + 3 of each 16. A single row has
// loops of its own (row_kv4, row_plain).
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
//          the normal range, and what that rounds off goes in as an operand of
//          its own, so that P keeps 22 bits; the -8 takes the same weights.
//
// What bounds it, and what it takes (32 heads of 128, chunks of 64; the rate is
// of the bytes that the call has to read): the memory, where rows are many.
//   fp16, 32 rows, 512 of their 1,024 visible tokens shared     50.1 us  5.5 TB/s
//   fp16, 16 rows, 2,048 visible tokens of their own            87.0 us  6.2 TB/s
//   4-bit, 64 rows, 1,024 visible tokens, most of their own     51.2 us  5.5 TB/s
//   4-bit, 128 rows, 64 to 1,024 tokens behind 2,048 shared     59.0 us  5.3 TB/s
//   4-bit, 1 row of 32,765 tokens                               26.9 us  5.3 TB/s
//   4-bit, 32 rows, 512 behind 1,024 shared                     19.5 us  3.9 TB/s
// (a copy of 2 GiB moves 4.96 TB/s). The last is a round of blocks whose chain of
// dependent loads (item, length, rows, partials, fold) is most of it, as are
// calls of a few rows: 8.6 us. In a first version that ran single rows through
// rows_shared and cut all rows alike the six took 74, 110, 98, 137, 44 and 32 us.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cstdint>
#include <type_traits>

#include "device_common.hpp"
#include "divide.hpp"
#include "kernels.hpp"
#include "kv4.hpp"

namespace ca {
namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// slack of the softmax reference maximum, in log2 units: P <= 2^kLazy, so
// that most steps leave the accumulators alone
constexpr float kLazy = 4.f;
// 4-bit: the reference of the scales stands for 2^kScaleTop, so that
// P s_v <= 2^(kScaleTop + kLazy) stays in fp16's range
constexpr int kScaleTop = 11;

template <int S>
struct Traits {
  using T = _Float16;
};
template <>
struct Traits<kStoreF32> {
  using T = float;
};

// A (scale, low) pair. (__builtin_bit_cast of a vector's element itself reads
// element 0 whatever the index: the element is copied out first.)
__device__ __forceinline__ half2v param(const u32x4& v, int i) {
  const uint32_t w = v[i];
  return __builtin_bit_cast(half2v, w);
}

// The eight codes of a word as fp16 halves: code * 2^-24 for elements 0, 1, 4
// and 5, code * 2^-20 for 2, 3, 6 and 7.
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

// w to the nearest fp16 below in size, as a float: the rest, w - rtz(w), takes
// the next 11 bits
__device__ __forceinline__ float top11(float w) {
  return __uint_as_float(__float_as_uint(w) & 0xffffe000u);
}

// Keeps a rarely taken branch a branch.
__device__ __forceinline__ void rare() { asm volatile(""); }

// What a block works on, wave-uniform except where said.
struct Work {
  const char* kbase;  // the head's tiles
  const char* vbase;
  int64_t ssb;        // bytes of a slot
  PlanChunk my;       // per lane: chunk `lane` of the item
  int nch;            // chunks
  int C, tpc;         // rows and 16-row tiles of a chunk
  uint32_t magic;     // inverse32(tpc)
  int n_tiles;
  int sinks, lo_item;
  int len, lo;        // per lane: length and window start of the lane's row
};
struct Tile {
  int slot, row, pos, end;  // end <= pos: no token
};
__device__ __forceinline__ Tile tile_at(const Work& W, int i) {  // uniform i
  const bool in = i < W.n_tiles;
  i = in ? i : 0;
  const int c = divide32(i, W.tpc, W.magic);
  const int r = (i - c * W.tpc) * 16;
  Tile t;
  t.slot = __builtin_amdgcn_readlane(W.my.slot, c);
  t.row = r;
  t.pos = __builtin_amdgcn_readlane(W.my.start, c) + r;
  t.end = in ? __builtin_amdgcn_readlane(W.my.end, c) : 0;
  return t;
}
// Nothing of the tile is seen, whatever the rows' present lengths.
__device__ __forceinline__ bool tile_hidden(const Work& W, const Tile& t) {
  const int last = min(t.end, t.pos + 16) - 1;
  return last < t.pos || (t.pos >= W.sinks && last < W.lo_item);
}

// The state a wavefront leaves for the fold: m_run, the sum n and, written to
// `out` [row][OS], the unnormalised O of each row.

// One row over a 4-bit pool, a wavefront's share: steps of 64 tokens, four
// 16-token tiles. Here q is the A operand (16 equal rows) and the K rows are
// columns, so the score of tile t's token n is in every lane of column n and
// lane (g, n) takes tile g's: each lane has one token's softmax, its
// parameters come in one 4-byte load, and P goes through 256 bytes of LDS to
// the lanes that need it as B operand, its rounded part in even columns, the
// rest in odd ones, so P loses nothing to fp16.
template <int D>
__device__ __forceinline__ void row_kv4(const PlanArgs& A, const Work& W, const _Float16* qrow, int wv, int nw, int lane,
                                        char* plds, float* out, float* om, float* on) {
  constexpr int KS = D / 32, DT = D / 16;
  const int n16 = lane & 15, g = lane >> 4;
  half8 qf[KS];  // asked for first, used after the first step's loads are out
#pragma unroll
  for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const half8*>(qrow + KS * 8 * g + 8 * s);

  const int pb = kv4_rows(W.C) * (D / 2);
  uint32_t kx[4][KS], vx[4][KS];
  uint32_t kp = 0, vp = 0;
  Tile tn[4];  // the step being loaded
  auto fetch = [&](int st) {
#pragma unroll
    for (int t = 0; t < 4; ++t) tn[t] = tile_at(W, 4 * st + t);
  };
  auto mine = [&](int Tile::*f) {  // the lane's tile's value
    const int a = g & 1 ? tn[1].*f : tn[0].*f, b = g & 1 ? tn[3].*f : tn[2].*f;
    return g & 2 ? b : a;
  };
  auto load_words = [&](const char* at, uint32_t (&x)[KS], auto nt) {
    if constexpr (D == 128) {
      const u32x4 a = decltype(nt)::value ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at)) : *reinterpret_cast<const u32x4*>(at);
#pragma unroll
      for (int s = 0; s < KS; ++s) x[s] = a[s];
    } else {
      const u32x2 a = *reinterpret_cast<const u32x2*>(at);
#pragma unroll
      for (int s = 0; s < KS; ++s) x[s] = a[s];
    }
  };
  int pos_n = 0, end_n = 0;
  int64_t par_n = 0;
  int lane_off = lane * (D / 8);
  auto load_k = [&]() {
#pragma unroll
    for (int t = 0; t < 4; ++t) load_words(W.kbase + tn[t].slot * W.ssb + tn[t].row * (D / 2) + lane_off, kx[t], std::true_type{});
    par_n = mine(&Tile::slot) * W.ssb + pb + (mine(&Tile::row) + n16) * 4;
    kp = *reinterpret_cast<const uint32_t*>(W.kbase + par_n);
    pos_n = mine(&Tile::pos) + n16;
    end_n = mine(&Tile::end);
  };
  Tile tv[4];
  auto load_v = [&](int64_t par) {
    vp = *reinterpret_cast<const uint32_t*>(W.vbase + par);  // needed before the codes
#pragma unroll
    for (int t = 0; t < 4; ++t) load_words(W.vbase + tv[t].slot * W.ssb + tv[t].row * (D / 2) + lane_off, vx[t], std::true_type{});
  };
  auto next = [&](int st) {
    const int steps = (W.n_tiles + 3) / 4;
    for (; st < steps; st += nw) {
      fetch(st);
      if (!(tile_hidden(W, tn[0]) && tile_hidden(W, tn[1]) && tile_hidden(W, tn[2]) && tile_hidden(W, tn[3]))) break;
    }
    return st < steps ? st : -1;
  };

  // m: reference of the scores plus log2 of the scales' reference
  float m_run = kNegBig, m_sc = kNegBig, n_run = 0.f, base = 0.f, s_ref = 0.f;
  floatx4 acc[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  _Float16* pl = reinterpret_cast<_Float16*>(plds);  // [hi, lo][pair][group][8]
  int st = next(wv);
  if (st >= 0) {
    load_k();
#pragma unroll
    for (int t = 0; t < 4; ++t) tv[t] = tn[t];
    load_v(par_n);
  }
  float amax = 0.f, sum = 0.f;
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = static_cast<float>(qf[s][i]);
      amax = fmaxf(amax, fabsf(x));
      sum += x;
    }
  amax = rows4_max(amax);
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  // q times 2^e with |q| 2^e in [2^10, 2^11): the 2^-4 of every second pair
  // and a small q stay in the normal range
  const int e = amax > 0.f && amax < INFINITY ? 11 - __builtin_amdgcn_frexp_expf(amax) : 0;
  const float up = __builtin_amdgcn_ldexpf(1.f, e);
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      qf[s][i] = static_cast<_Float16>(static_cast<float>(qf[s][i]) * ((i & 2) ? up * 0.0625f : up));
  const float qk = __builtin_amdgcn_ldexpf(A.qscale, 24 - e);  // score = qk (s_k a + low_k ql)
  const float ql = __builtin_amdgcn_ldexpf(sum, e - 24);

  // Every step issues the same loads, so that a wait covers only the rows it
  // needs (loads under a condition would make each wait one for all of them);
  // past the last step they are one line of the last tiles each, not used.
  while (st >= 0) {
    floatx4 a[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      a[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s)
        a[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(qf[s], unpack8(kx[t][s]), a[t], 0, 0, 0);
    }
    const float raw = g & 2 ? (g & 1 ? a[3][0] : a[2][0]) : (g & 1 ? a[1][0] : a[0][0]);
    const half2v kq = __builtin_bit_cast(half2v, kp);
    const int pos = pos_n, end = end_n;
    st = next(st + nw);
    lane_off = st >= 0 ? lane_off : 0;
    load_k();
    const bool on = pos < end && pos < W.len && (pos >= W.lo || pos < W.sinks);
    float sc = qk * __builtin_fmaf(raw, static_cast<float>(kq[0]), static_cast<float>(kq[1]) * ql);
    sc = on ? sc : -INFINITY;
    const half2v vq = __builtin_bit_cast(half2v, vp);
    const float sv = on ? static_cast<float>(vq[0]) : 0.f, lv = on ? static_cast<float>(vq[1]) : 0.f;
    if (__any(sc > m_sc + kLazy || sv > s_ref)) {
      rare();
      const float mx = wave_max(sc), sx = wave_max(sv);
      if (mx > m_sc + kLazy) m_sc = mx;
      if (sx > s_ref) s_ref = 2.f * sx;
      const float m_new = s_ref > 0.f ? m_sc + __builtin_amdgcn_logf(s_ref) - kScaleTop : m_sc;
      const float al = fast_exp2(m_run - m_new);
      n_run *= al;
      base *= al;
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[d] *= al;
      m_run = m_new;
    }
    const float p = fast_exp2(sc - m_run);
    n_run += p;
    base = __builtin_fmaf(p, lv, base);
    const float w = p * sv * ((n16 & 2) ? 0.0625f : 1.f);
    const float hi = top11(w);
    const int at = (((g >> 1) * 4 + (n16 >> 2)) * 8) + (g & 1) * 4 + (n16 & 3);
    pl[at] = static_cast<_Float16>(hi);
    pl[64 + at] = static_cast<_Float16>(w - hi);
    compiler_fence();
    half8 pf[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) pf[r] = *reinterpret_cast<const half8*>(pl + 64 * (n16 & 1) + (r * 4 + g) * 8);
    compiler_fence();
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const half8 x = unpack8(vx[2 * r][s]), y = unpack8(vx[2 * r + 1][s]);
        const half8 even = __builtin_shufflevector(x, y, 0, 1, 2, 3, 8, 9, 10, 11);
        const half8 odd = __builtin_shufflevector(x, y, 4, 5, 6, 7, 12, 13, 14, 15);
        acc[2 * s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(even, pf[r], acc[2 * s], 0, 0, 0);
        acc[2 * s + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(odd, pf[r], acc[2 * s + 1], 0, 0, 0);
      }
#pragma unroll
    for (int t = 0; t < 4; ++t) tv[t] = tn[t];
    load_v(par_n);
  }
  n_run = wave_sum(n_run);
  base = wave_sum(base);
#pragma unroll
  for (int d = 0; d < DT; ++d) {
    floatx4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __builtin_fmaf(acc[d][i] + dpp<0xB1>(acc[d][i]), 16777216.f, base);
    if (n16 == 0) *reinterpret_cast<floatx4*>(out + 16 * d + 4 * g) = o;
  }
  if (lane == 0) {
    *om = m_run;
    *on = n_run;
  }
}

// One row over an fp16 or fp32 pool, a wavefront's share: a row of the pool is
// read by LPR lanes, 16 bytes each, a load covers RPL rows (1 KB), a step NL
// loads of K and of V. Each group of LPR lanes keeps the softmax state of the
// rows it saw, with P in 32 bits; the groups are folded at the end.
template <int S, int D>
__device__ __forceinline__ void row_plain(const PlanArgs& A, const Work& W, const typename Traits<S>::T* qrow, int wv,
                                          int nw, int lane, float* out, float* om, float* on) {
  using T = typename Traits<S>::T;
  constexpr int E = 16 / sizeof(T);                 // elements of a lane
  constexpr int LPR = D / E, RPL = 64 / LPR;
  constexpr int NL = 8;                             // loads of a step
  constexpr int TP = NL * RPL / 16;                 // its tiles
  constexpr int LT = NL / TP;                       // loads of a tile
  constexpr int RB = D * static_cast<int>(sizeof(T));
  const int gi = lane / LPR, li = lane % LPR;
  const uint4 q_raw = *reinterpret_cast<const uint4*>(qrow + E * li);
  uint4 kx[NL], vx[NL];
  Tile tn[TP], tv[TP];
  auto fetch = [&](int st) {
#pragma unroll
    for (int t = 0; t < TP; ++t) tn[t] = tile_at(W, TP * st + t);
  };
  int li_off = 16 * li, gi_off = gi;
  auto load = [&](const char* base, const Tile (&t)[TP], uint4 (&x)[NL], auto nt) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const Tile& y = t[i / LT];
      // a scalar base and a small offset of the lane; rows past the chunk's
      // size read its last one again
      const char* at = base + y.slot * W.ssb + static_cast<int64_t>(y.row) * RB;
      const unsigned off = min((i % LT) * RPL + gi_off, W.C - 1 - y.row) * RB + li_off;
      if constexpr (decltype(nt)::value)
        x[i] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at + off)));
      else x[i] = *reinterpret_cast<const uint4*>(at + off);
    }
  };
  auto next = [&](int st) {
    const int steps = (W.n_tiles + TP - 1) / TP;
    for (; st < steps; st += nw) {
      fetch(st);
      bool hid = true;
#pragma unroll
      for (int t = 0; t < TP; ++t) hid &= tile_hidden(W, tn[t]);
      if (!hid) break;
    }
    return st < steps ? st : -1;
  };
  float m = kNegBig, n = 0.f;
  float acc[E];
#pragma unroll
  for (int j = 0; j < E; ++j) acc[j] = 0.f;
  int st = next(wv);
  if (st >= 0) {
    load(W.kbase, tn, kx, std::true_type{});
    load(W.vbase, tn, vx, std::true_type{});
  }
  float qv[E];
  Elem<T>::unpack(q_raw, qv);
  while (st >= 0) {
#pragma unroll
    for (int t = 0; t < TP; ++t) tv[t] = tn[t];
    float sc[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      float x[E], d = 0.f;
      Elem<T>::unpack(kx[i], x);
#pragma unroll
      for (int j = 0; j < E; ++j) d = __builtin_fmaf(x[j], qv[j], d);
      sc[i] = group_sum<LPR>(d) * A.qscale;
    }
    st = next(st + nw);
    li_off = st >= 0 ? li_off : 0;  // as over 4-bit pools
    gi_off = st >= 0 ? gi_off : 0;
    load(W.kbase, tn, kx, std::true_type{});
    bool all = true;
#pragma unroll
    for (int t = 0; t < TP; ++t) {
      const int last = tv[t].pos + 16;
      all &= last <= tv[t].end && last <= W.len && (tv[t].pos >= W.lo || last <= W.sinks);
    }
    if (!__builtin_amdgcn_readfirstlane(all)) {
      rare();
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int j = tv[i / LT].pos + (i % LT) * RPL + gi;
        const bool on = j < tv[i / LT].end && j < W.len && (j >= W.lo || j < W.sinks);
        sc[i] = on ? sc[i] : -INFINITY;
        if (!on) vx[i] = make_uint4(0, 0, 0, 0);
      }
    }
    float mx = sc[0];
#pragma unroll
    for (int i = 1; i < NL; ++i) mx = fmaxf(mx, sc[i]);
    const float mn = mx > m + kLazy ? mx : m;
    if (__any(mn != m)) {
      rare();
      const float al = fast_exp2(m - mn);
      n *= al;
#pragma unroll
      for (int j = 0; j < E; ++j) acc[j] *= al;
      m = mn;
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const float p = fast_exp2(sc[i] - m);
      n += p;
      float x[E];
      Elem<T>::unpack(vx[i], x);
#pragma unroll
      for (int j = 0; j < E; ++j) acc[j] = __builtin_fmaf(p, x[j], acc[j]);
    }
    load(W.vbase, tn, vx, std::true_type{});
  }
#pragma unroll
  for (int off = LPR; off < 64; off <<= 1) {
    const float mo = __shfl_xor(m, off), no = __shfl_xor(n, off);
    float x[E];
#pragma unroll
    for (int j = 0; j < E; ++j) x[j] = __shfl_xor(acc[j], off);
    fold<E>(m, n, acc, mo, no, x);
  }
  if (lane < LPR) {
#pragma unroll
    for (int j = 0; j < E; ++j) out[E * li + j] = acc[j];
  }
  if (lane == 0) {
    *om = m;
    *on = n;
  }
}

// 2 to 16 rows that share the item's chunks: S^T = K Q^T and O^T += V^T P^T,
// tokens, then channels, as rows and query rows as columns, so P stays in the
// registers S^T came out in: tokens 4g .. 4g + 3 of each 16.
template <int S, int D>
__device__ __forceinline__ void rows_shared(const PlanArgs& A, const Work& W, int nr, const typename Traits<S>::T* qrow,
                                            int wv, int lane, char* vlds, float* out, float* om, float* on) {
  using T = typename Traits<S>::T;
  constexpr bool kF16 = S == kStoreF16, kF32 = S == kStoreF32, kQ4 = S == kStoreKv4;
  constexpr int TP = kF32 ? 1 : 2;  // tiles of a step
  constexpr int KS = D / 32, DT = D / 16;
  constexpr int VS = D + 16, OS = D + 4;
  constexpr int ES = static_cast<int>(sizeof(T));
  const int n16 = lane & 15, g = lane >> 4;
  // 4-bit, up to 8 rows: columns 8 .. 15 repeat them and take the part of P
  // that fp16 rounds off; with more rows it takes matrix ops of its own
  const bool half = kQ4 && nr <= 8;
  const bool low_part = half && n16 >= 8;

  half8 qf[kF32 ? 1 : KS];
  floatx4 qx[kF32 ? D / 16 : 1];
  float qk = A.qscale, ql = 0.f;
  if constexpr (kF32) {
#pragma unroll
    for (int u = 0; u < D / 16; ++u) qx[u] = *reinterpret_cast<const floatx4*>(qrow + 16 * u + 4 * g);
  } else if constexpr (kF16) {
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const half8*>(qrow + 32 * s + 8 * g);
  } else {  // as for one row
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
    ql = __builtin_amdgcn_ldexpf(sum, e - 24);
  }

  // bounds over the item's rows: a tile inside them needs no mask
  int lo_max = W.lo, lo_min = W.lo, len_min = W.len, len_max = W.len;
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

  half8 kh[kF16 ? 2 : 1][kF16 ? KS : 1];
  u32x4 vh[kF16 ? D / 16 : 1];
  floatx4 kf[kF32 ? D / 16 : 1], vf[kF32 ? 4 : 1][kF32 ? D / 64 : 1];
  uint32_t kc[kQ4 ? 2 : 1][kQ4 ? KS : 1], vc[kQ4 ? 2 : 1][kQ4 ? KS : 1];
  u32x4 kp[kQ4 ? 2 : 1], vp[kQ4 ? 2 : 1];
  Tile tn[TP], tc[TP];
  const int pb = kv4_rows(W.C) * (D / 2);
  auto words = [&](const char* at, uint32_t* x) {
    if constexpr (D == 128) {
      const u32x4 a = *reinterpret_cast<const u32x4*>(at);
#pragma unroll
      for (int s = 0; s < KS; ++s) x[s] = a[s];
    } else {
      const u32x2 a = *reinterpret_cast<const u32x2*>(at);
#pragma unroll
      for (int s = 0; s < KS; ++s) x[s] = a[s];
    }
  };
  auto load_k = [&]() {
#pragma unroll
    for (int t = 0; t < TP; ++t) {
      const char* kt = W.kbase + tn[t].slot * W.ssb;
      if constexpr (kQ4) {
        words(kt + tn[t].row * (D / 2) + lane * (D / 8), kc[t]);
        kp[t] = *reinterpret_cast<const u32x4*>(kt + pb + (tn[t].row + 4 * g) * 4);
      } else {
        const char* at = kt + static_cast<int64_t>(tn[t].row) * (D * ES);
        const unsigned off = min(n16, W.C - 1 - tn[t].row) * (D * ES) + 16 * g;
        if constexpr (kF16) {
#pragma unroll
          for (int s = 0; s < KS; ++s) kh[t][s] = *reinterpret_cast<const half8*>(at + (off + 64 * s));
        } else {
#pragma unroll
          for (int u = 0; u < D / 16; ++u) kf[u] = *reinterpret_cast<const floatx4*>(at + (off + 64 * u));
        }
      }
    }
  };
  auto load_v = [&]() {
    if constexpr (kQ4) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char* vt = W.vbase + tn[t].slot * W.ssb;
        vp[t] = *reinterpret_cast<const u32x4*>(vt + pb + (tn[t].row + 4 * g) * 4);  // needed first
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
        words(W.vbase + tn[t].slot * W.ssb + tn[t].row * (D / 2) + lane * (D / 8), vc[t]);
    } else if constexpr (kF16) {
      constexpr int GPR = D / 8, RPL = 64 / GPR;  // granules a row, rows a load
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const Tile& t = tn[i / (D / 32)];
        const char* at = W.vbase + t.slot * W.ssb + static_cast<int64_t>(t.row) * (D * 2);
        const unsigned off = min((i % (D / 32)) * RPL + lane / GPR, W.C - 1 - t.row) * (D * 2) + 16 * (lane % GPR);
        vh[i] = *reinterpret_cast<const u32x4*>(at + off);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const char* at = W.vbase + tn[0].slot * W.ssb + static_cast<int64_t>(tn[0].row) * (D * 4);
        const unsigned off = min(4 * g + i, W.C - 1 - tn[0].row) * (D * 4) + 16 * n16;
#pragma unroll
        for (int u = 0; u < D / 64; ++u) vf[i][u] = *reinterpret_cast<const floatx4*>(at + (off + 256 * u));
      }
    }
  };
  auto next = [&](int st) {
    const int steps = (W.n_tiles + TP - 1) / TP;
    for (; st < steps; st += 4) {
      bool hid = true;
#pragma unroll
      for (int t = 0; t < TP; ++t) {
        tn[t] = tile_at(W, TP * st + t);
        hid &= tile_hidden(W, tn[t]);
      }
      if (!hid) break;
    }
    return st < steps ? st : -1;
  };
  // token k of tile t, seen by a row of length l whose window starts at b
  auto seen = [&](int t, int k, int l, int b) {
    const int j = tc[t].pos + k;
    return j < tc[t].end && j < l && (j >= b || j < W.sinks);
  };

  float m_run = kNegBig, n_run = 0.f;
  float m_sc = kNegBig, base = 0.f, s_ref = 0.f;  // 4-bit: as for one row
  floatx4 acc[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  _Float16* vl = reinterpret_cast<_Float16*>(vlds);

  int st = next(wv);
  if (st >= 0) {
    load_k();
    load_v();
  }
  while (st >= 0) {
#pragma unroll
    for (int t = 0; t < TP; ++t) tc[t] = tn[t];
    bool all = true;
#pragma unroll
    for (int t = 0; t < TP; ++t) {
      const int last = tc[t].pos + 16;
      all &= last <= tc[t].end && last <= len_min && (tc[t].pos >= lo_max || last <= W.sinks);
    }
    float sc[TP][4];
#pragma unroll
    for (int t = 0; t < TP; ++t) {
      floatx4 a = {0.f, 0.f, 0.f, 0.f};
      if constexpr (kF32) {
#pragma unroll
        for (int u = 0; u < D / 16; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) a = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[u][j], qx[u][j], a, 0, 0, 0);
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          half8 x;
          if constexpr (kF16) x = kh[t][s];
          else x = unpack8(kc[t][s]);
          a = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, qf[s], a, 0, 0, 0);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (kQ4) {
          const half2v y = param(kp[t], i);
          sc[t][i] = qk * __builtin_fmaf(a[i], static_cast<float>(y[0]), static_cast<float>(y[1]) * ql);
        } else {
          sc[t][i] = a[i] * qk;
        }
      }
    }
    const int st_next = next(st + 4);
    load_k();  // unconditional, as for one row; past the last step, its last tiles again
    float sv[kQ4 ? 2 : 1][4], lv[kQ4 ? 2 : 1][4];
    float smax = 0.f;
    if constexpr (kQ4) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const half2v y = param(vp[t], i);
          sv[t][i] = static_cast<float>(y[0]);
          lv[t][i] = static_cast<float>(y[1]);
        }
    }
    if (!all) {
      rare();
#pragma unroll
      for (int t = 0; t < TP; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool vis = seen(t, 4 * g + i, W.len, W.lo);
          sc[t][i] = vis ? sc[t][i] : -INFINITY;
          if constexpr (kQ4) {  // whatever is stored where nothing is seen
            sv[t][i] = vis ? sv[t][i] : 0.f;
            lv[t][i] = vis ? lv[t][i] : 0.f;
          }
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < TP; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mx = fmaxf(mx, sc[t][i]);
        if constexpr (kQ4) smax = fmaxf(smax, sv[t][i]);
      }
    const float ref = kQ4 ? m_sc : m_run;
    if (__any(mx > ref + kLazy || (kQ4 && smax > s_ref))) {
      rare();
      mx = rows4_max(mx);
      float m_new = mx > ref + kLazy ? mx : ref;
      if constexpr (kQ4) {
        m_sc = m_new;
        const float sx = wave_max(smax);
        if (sx > s_ref) s_ref = 2.f * sx;
        if (s_ref > 0.f) m_new += __builtin_amdgcn_logf(s_ref) - kScaleTop;
      }
      const float al = fast_exp2(m_run - m_new);
      n_run *= al;
      base *= al;
#pragma unroll
      for (int t = 0; t < DT; ++t) acc[t] *= al;
      m_run = m_new;
    }
    float pr[TP][4];
#pragma unroll
    for (int t = 0; t < TP; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pr[t][i] = fast_exp2(sc[t][i] - m_run);
        if constexpr (!kF16) n_run += pr[t][i];
      }

    // A token that some rows see and others do not: where its V is not finite
    // (never in ordinary data), 0 * V would reach the others. It counts as 0
    // then, and o is NaN for the rows that see it: where the product of "not
    // finite" and "seen" is not zero.
    if constexpr (kF32) {
      if (!all) {
        rare();
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool any_row = seen(0, 4 * g + i, len_max, lo_min);
#pragma unroll
          for (int u = 0; u < D / 64; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              vf[i][u][j] = any_row ? vf[i][u][j] : 0.f;
              bad |= !(fabsf(vf[i][u][j]) < INFINITY);
            }
        }
        if (__any(bad)) {
#pragma unroll
          for (int u = 0; u < D / 64; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              floatx4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const bool x = !(fabsf(vf[i][u][j]) < INFINITY);
                z = __builtin_amdgcn_mfma_f32_16x16x4f32(x ? 1.f : 0.f, seen(0, 4 * g + i, W.len, W.lo) ? 1.f : 0.f,
                                                         z, 0, 0, 0);
                vf[i][u][j] = x ? 0.f : vf[i][u][j];
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[4 * u + j][i] = z[i] > 0.f ? __builtin_nanf("") : acc[4 * u + j][i];
            }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int u = 0; u < D / 64; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[4 * u + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[i][u][j], pr[0][i], acc[4 * u + j], 0, 0, 0);
    } else if constexpr (kF16) {
      half8 pf;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pf[4 * t + i] = static_cast<_Float16>(pr[t][i]);
          n_run += static_cast<float>(pf[4 * t + i]);
        }
      constexpr int GPR = D / 8, RPL = 64 / GPR;
      bool bad = false;
      if (!all) {
        rare();
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          if (!seen(i / (D / 32), (i % (D / 32)) * RPL + lane / GPR, len_max, lo_min)) vh[i] = u32x4{0, 0, 0, 0};
          bad |= any_nonfinite(__builtin_bit_cast(half8, vh[i]));
        }
        bad = __any(bad);
      }
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const int r = 16 * (i / (D / 32)) + (i % (D / 32)) * RPL + lane / GPR;
        *reinterpret_cast<u32x4*>(vl + r * VS + 8 * (lane % GPR)) = vh[i];
      }
      // the wavefront's own tile: its LDS ops complete in order
      compiler_fence();
      auto read_v = [&](int d) {
        const _Float16* at = vl + (4 * g + (n16 >> 2)) * VS + 16 * d + 4 * (n16 & 3);
        const half4 x = lds_read_tr16(at), y = lds_read_tr16(at + 16 * VS);
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
      };
      if (bad) {
        rare();
        half8 vis;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          vis[k] = static_cast<_Float16>(seen(k / 4, 4 * g + k % 4, W.len, W.lo) ? 1.f : 0.f);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          half8 va = read_v(d), x;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const bool f = fabsf(static_cast<float>(va[k])) < INFINITY;
            x[k] = static_cast<_Float16>(f ? 0.f : 1.f);
            va[k] = f ? va[k] : static_cast<_Float16>(0.f);
          }
          const floatx4 z = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, vis, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
          acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, pf, acc[d], 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[d][i] = z[i] > 0.f ? __builtin_nanf("") : acc[d][i];
        }
      } else {
        constexpr int HD = 4;  // operands in registers at once
#pragma unroll
        for (int d0 = 0; d0 < DT; d0 += HD) {
          half8 va[HD];
#pragma unroll
          for (int d = 0; d < HD; ++d) va[d] = read_v(d0 + d);
#pragma unroll
          for (int d = 0; d < HD; ++d)
            acc[d0 + d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va[d], pf, acc[d0 + d], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      compiler_fence();
    } else {
      half8 pf, pl;  // P s_v: rounded; what is left, where it has ops of its own
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          base = __builtin_fmaf(pr[t][i], lv[t][i], base);
          const float w = pr[t][i] * sv[t][i] * (i & 2 ? 0.0625f : 1.f);  // these codes stand 2^4 higher
          const float hi = top11(w);
          pf[4 * t + i] = static_cast<_Float16>(low_part ? w - hi : hi);
          pl[4 * t + i] = static_cast<_Float16>(w - hi);
        }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const half8 x = unpack8(vc[0][s]), y = unpack8(vc[1][s]);
        const half8 even = __builtin_shufflevector(x, y, 0, 1, 2, 3, 8, 9, 10, 11);
        const half8 odd = __builtin_shufflevector(x, y, 4, 5, 6, 7, 12, 13, 14, 15);
        acc[2 * s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(even, pf, acc[2 * s], 0, 0, 0);
        acc[2 * s + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(odd, pf, acc[2 * s + 1], 0, 0, 0);
        if (!half) {
          acc[2 * s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(even, pl, acc[2 * s], 0, 0, 0);
          acc[2 * s + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(odd, pl, acc[2 * s + 1], 0, 0, 0);
        }
      }
    }
    st = st_next;
    load_v();
  }

  n_run += __shfl_xor(n_run, 16);
  n_run += __shfl_xor(n_run, 32);
  if constexpr (kQ4) {
    base += __shfl_xor(base, 16);
    base += __shfl_xor(base, 32);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float o = half ? acc[d][i] + __shfl_xor(acc[d][i], 8) : acc[d][i];
        acc[d][i] = __builtin_fmaf(o, 16777216.f, base);
      }
  }
  if (kF16) __syncthreads();  // the V tiles' place is used again
  if (n16 < nr) {
    float* at = out + n16 * OS;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      if constexpr (kF32) {
        // op tile 4u + j, element i: channel 64u + 16g + 4i + j
#pragma unroll
        for (int i = 0; i < 4; ++i) at[64 * (d / 4) + 16 * g + 4 * i + d % 4] = acc[d][i];
      } else {
        *reinterpret_cast<floatx4*>(at + 16 * d + 4 * g) = acc[d];
      }
    }
    if (g == 0) {
      om[n16] = m_run;
      on[n16] = n_run;
    }
  }
}

template <int S, int D>
__global__ __launch_bounds__(256, S == kStoreKv4 ? 3 : 2) void kwd_kernel(PlanArgs A) {
  using T = typename Traits<S>::T;
  constexpr int OS = D + 4;                    // merge buffer row stride (floats)
  constexpr int VB = S == kStoreF16 ? 4 * 32 * (D + 16) * 2 : S == kStoreKv4 ? 4 * 256 : 0;
  constexpr int MB = 4 * kPlanRows * OS * 4;
  constexpr int LDS = S == kStoreKv4 ? VB + MB : VB > MB ? VB : MB;
  __shared__ __align__(16) char lds[LDS];
  __shared__ float s_m[4][kPlanRows], s_n[4][kPlanRows];
  __shared__ int s_last[kPlanRows], s_pbase[kPlanRows], s_np[kPlanRows], s_io[kPlanRows];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int H = A.H;
  // An item of a block: one head of it, the wavefronts share its tokens. An
  // item of wavefronts: four heads of it, one a wavefront.
  const int b = static_cast<int>(blockIdx.x), n_blk = A.n_block_items * H;
  const bool solo = b >= n_blk;
  int ib, h0;
  if (solo) {
    const int hb = (H + 3) >> 2;
    ib = (b - n_blk) / hb;
    h0 = 4 * (b - n_blk - ib * hb);
    ib += A.n_block_items;
  } else {
    ib = b / H;
    h0 = b - ib * H;
  }
  const int h = solo ? min(h0 + wv, H - 1) : h0;  // a wavefront past the heads repeats the last one
  const PlanItem item = A.items[ib];
  const int nr = item.n_rows;
  constexpr int ES = S == kStoreF16 ? 2 : S == kStoreF32 ? 4 : 1;
  Work W;
  // the chunks, one a lane (chunk_stride <= 64)
  W.my = A.chunks[static_cast<size_t>(ib) * A.chunk_stride + min(lane, A.chunk_stride - 1)];
  W.kbase = static_cast<const char*>(A.kpool) + h * (A.hs * ES);
  W.vbase = static_cast<const char*>(A.vpool) + h * (A.hs * ES);
  W.ssb = A.ss * ES;
  W.nch = item.n_chunks;
  W.C = A.C;
  W.tpc = (A.C + 15) >> 4;
  W.magic = inverse32(W.tpc);
  W.n_tiles = item.n_chunks * W.tpc;
  W.sinks = A.sinks;
  W.lo_item = item.lo;
  float* mb = reinterpret_cast<float*>(lds + (S == kStoreKv4 ? VB : 0));  // [wave][row][OS]
  if (nr == 1) {
    // the row's length is asked for here and waited for where the first
    // scores are
    const int io = A.row_map ? A.row_map[item.row_begin] : item.row_begin;
    W.len = item.last_start + A.slot_len[item.last_slot];
    W.lo = max(0, W.len - A.window);
    const T* qrow = static_cast<const T*>(A.q) + (static_cast<size_t>(io) * H + h) * D;
    float* out = mb + wv * kPlanRows * OS;
    const int w0 = solo ? 0 : wv, nw = solo ? 1 : 4;
    if constexpr (S == kStoreKv4) row_kv4<D>(A, W, qrow, w0, nw, lane, lds + wv * 256, out, &s_m[wv][0], &s_n[wv][0]);
    else row_plain<S, D>(A, W, qrow, w0, nw, lane, out, &s_m[wv][0], &s_n[wv][0]);
    if (tid == 0) {
      s_pbase[0] = item.pbase;
      s_np[0] = item.np;
      s_io[0] = io;
    }
  } else {
    // 4-bit, up to 8 rows: columns 8 .. 15 repeat them
    const int col = S == kStoreKv4 && nr <= 8 ? lane & 7 : lane & 15;
    const int row = item.row_begin + min(col, nr - 1);
    const PlanRow prow = A.rows[row];
    const int io = A.row_map ? A.row_map[row] : row;
    const T* qrow = static_cast<const T*>(A.q) + (static_cast<size_t>(io) * H + h) * D;
    W.len = prow.last_start + A.slot_len[prow.last_slot];
    W.lo = max(0, W.len - A.window);
    rows_shared<S, D>(A, W, nr, qrow, wv, lane, lds + (S == kStoreF16 ? wv * (32 * (D + 16) * 2) : 0),
                      mb + wv * kPlanRows * OS, s_m[wv], s_n[wv]);
    if (tid < kPlanRows) {
      s_pbase[tid] = prow.pbase;
      s_np[tid] = prow.np;
      s_io[tid] = io;
    }
  }
  // Result r of the block: row r of the item, folded from the four wavefronts
  // (Eqn 2) through LDS, [wave][row][channel]; or, of an item of wavefronts,
  // head h0 + r as wavefront r left it.
  __syncthreads();
  constexpr int TPR = D / 4, NG = 256 / TPR;  // threads a result, results at once
  const int gi = tid / TPR, ch = 4 * (tid % TPR);
  const int n_res = solo ? min(4, H - h0) : nr;
  const __amdgpu_buffer_rsrc_t rs = part_rsrc(A.ws_o, A.ws_o_bytes);
  T* out = static_cast<T*>(A.o);
  auto row_of = [&](int r) { return solo ? 0 : r; };
  auto head_of = [&](int r) { return solo ? h0 + r : h0; };
  auto write_row = [&](int r, const floatx4& v, float n) {
    T* at = out + (static_cast<size_t>(s_io[row_of(r)]) * H + head_of(r)) * D + ch;
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
  bool parts = false;
  for (int r = gi; r < n_res; r += NG) {
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    float n = 0.f, m;
    if (solo) {
      m = s_m[r][0];
      n = s_n[r][0];
      v = *reinterpret_cast<const floatx4*>(mb + r * kPlanRows * OS + ch);
    } else {
      m = fmaxf(fmaxf(s_m[0][r], s_m[1][r]), fmaxf(s_m[2][r], s_m[3][r]));
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = fast_exp2(s_m[w][r] - m);
        n += s_n[w][r] * f;
        v += *reinterpret_cast<const floatx4*>(mb + (w * kPlanRows + r) * OS + ch) * f;
      }
    }
    if (s_np[row_of(r)] == 1) {
      write_row(r, v, n);
    } else {
      parts = true;
      const int p = s_pbase[row_of(r)] + item.ord, hr = head_of(r);
      st_dev4(rs, ((static_cast<uint32_t>(p) * H + hr) * D + ch) * 4u, v[0], v[1], v[2], v[3]);
      if (ch == 0) {
        float* ml = A.ws_ml + (static_cast<size_t>(p) * H + hr) * 2;
        st_dev(ml, m);
        st_dev(ml + 1, n);
      }
    }
  }
  // Partials: the last block to arrive on a row folds them (the exchange
  // protocol of device_common.hpp).
  if (!__syncthreads_or(parts)) return;
  wait_stores();
  __syncthreads();
  if (tid < n_res) {
    bool last = false;
    if (s_np[row_of(tid)] > 1) {
      const int r = item.row_begin + row_of(tid), hr = head_of(tid);
      int32_t* c = A.cnt_layout < 0 ? A.cnt + (static_cast<size_t>(r) * H + hr)
                                    : A.cnt + (static_cast<size_t>(r >> A.cnt_layout) * H + hr) * 32 +
                                          (r & ((1 << A.cnt_layout) - 1));
      last = arrive_last(c, s_np[row_of(tid)]);
    }
    s_last[tid] = last;
  }
  __syncthreads();
  // partials p0, p0 + step, ... below p1 of head hr into (m, n, v), the loads of
  // four in flight together
  auto fold_from = [&](int p0, int step, int p1, int hr, float& m, float& n, floatx4& v) {
    constexpr int NB = 4;
    for (; p0 < p1; p0 += NB * step) {
      float pm[NB], pn[NB];
      float4 x[NB];
#pragma unroll
      for (int k = 0; k < NB; ++k) {
        const int p = min(p0 + k * step, p1 - 1);  // past the end: a valid one, not used
        const float* ml = A.ws_ml + (static_cast<size_t>(p) * H + hr) * 2;
        pm[k] = ld_dev(ml);
        pn[k] = ld_dev(ml + 1);
        x[k] = ld_dev4(rs, ((static_cast<uint32_t>(p) * H + hr) * D + ch) * 4u);
      }
#pragma unroll
      for (int k = 0; k < NB; ++k) {
        if (p0 + k * step >= p1) break;
        const float M = fmaxf(m, pm[k]);
        const float a = fast_exp2(m - M), c = fast_exp2(pm[k] - M);
        n = n * a + pn[k] * c;
        v = v * a + floatx4{x[k].x, x[k].y, x[k].z, x[k].w} * c;
        m = M;
      }
    }
  };
  if (nr > 1 || solo) {  // a result to each group of threads
    for (int r = gi; r < n_res; r += NG) {
      if (!s_last[r]) continue;
      float m = kNegBig, n = 0.f;
      floatx4 v = {0.f, 0.f, 0.f, 0.f};
      const int p0 = s_pbase[row_of(r)];
      fold_from(p0, 1, p0 + s_np[row_of(r)], head_of(r), m, n, v);
      write_row(r, v, n);
    }
  } else if (s_last[0]) {  // one: its partials dealt out to the groups
    float m = kNegBig, n = 0.f;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    fold_from(s_pbase[0] + gi, NG, s_pbase[0] + s_np[0], h0, m, n, v);
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
      write_row(0, o, nn);
    }
  }
}

}  // namespace

hipError_t launch_plan_attention(const PlanArgs& a, hipStream_t stream) {
  if (a.n_items <= 0) return hipSuccess;
  if (a.chunk_stride < 1 || a.chunk_stride > kPlanChunks) return hipErrorInvalidValue;
  const unsigned grid = static_cast<unsigned>(a.n_block_items) * static_cast<unsigned>(a.H) +
                        static_cast<unsigned>(a.n_items - a.n_block_items) * static_cast<unsigned>((a.H + 3) / 4);
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
