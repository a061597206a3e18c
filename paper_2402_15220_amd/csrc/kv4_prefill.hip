// gfx950 (MI355X) prefill attention over a pool held in 4 bits (kv4.hpp), with
// or without a sliding window and sinks.
//
// The last n_q tokens of a sequence of L tokens attend causally: the query at
// position p sees the positions j <= p with j < sinks or j > p - window.
//
// One block of QW KG wavefronts per (tile of 32 QW queries, head, part of the
// tile's keys). The keys that some query of the tile sees are taken as tiles
// of 16 rows of the path's chunks, in order, UK / 16 of them to a unit; tiles
// between the sinks and the first query's window are left out. Codes go from
// memory into registers two units ahead, become fp16 operands on the way into
// one of two LDS buffers, once for all the tile's queries, and one barrier a
// unit tells that a buffer is written and the other one free. Wavefront
// (qw, kg) owns 32 queries and KPW keys of every unit:
//   S^T = K Q^T     32x32x16 matrix ops, K rows as A, q as B (in registers);
//   mask where a unit has a pair that is not seen, online softmax in base 2
//   with a lazy reference maximum;
//   O^T += V^T P^T  P straight from the registers S^T came out in.
//
// Values low + scale * code take up to 15 bits, fp16 holds 11: as fp16 values K
// and V would each add an error the size of P's and of o's own rounding (twice
// the plain form's error in all). So the operands are exact instead: with
// s^ = scale to 8 bits, s^ (code - 8) has at most 11, and with r = scale / s^
// (1 +- 2^-9) and b = low + 8 scale
//   q.k = r_k q.(s^ (code - 8)) + b_k sum(q),
//   p v = (p r_v) (s^ (code - 8)) + p b_v.
// r_k is the factor of the exponent's fma; b_k sum(q) and log2 r_v, which makes
// w = p r_v of p, are one more 16-wide step of the score product (b and sum(q)
// as two fp16 each); sum p = sum w / r_v and sum p b_v = sum w b_v / r_v are the
// first rows of one more channel tile of the O product. P's rounding is left.
//
// What bounds it: issue and latency at two wavefronts a SIMD. Of a 64-query
// block's time (512 queries behind 1,024, 32 heads of 128: one round of 256
// blocks) a quarter goes into turning codes into operands, a third into scores,
// softmax and O, the rest into the start, barriers and the fold. Queries behind
// 1,024 positions: 256 in 26.8 us, 512 in 37.7 (fp16: 24), 576 in 52, 896 in 70;
// 2,048 with a window of 1,024 in 74. A version of four wavefronts that rounded
// values to fp16 and folded parts one after the other took twice as long (82 us for
// 512 queries with their write, now 41.6).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "device_common.hpp"
#include "divide.hpp"
#include "kernels.hpp"
#include "kv4.hpp"

namespace ca {
namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLazyMax = 8.f;
// scores beyond this (log2 units) get their maximum from the exact products:
// r alone could lift P by 2^(score / 2^9)
constexpr float kFarScore = 2000.f;

struct KwpPath {
  int32_t slot[kPrefillInlineChunks];
  int32_t start[kPrefillInlineChunks];
  int32_t end[kPrefillInlineChunks];
};
struct KwpNoPath {};

struct KwpParams {
  const _Float16* q;  // [n_q][H][D]
  _Float16* o;
  const char* kpool;
  const char* vpool;
  int64_t ss, hs;  // bytes
  const int32_t* dpath;  // device path (long paths): slots, starts, ends
  int n_chunks, n_q, H, C, L;
  int window, sinks;
  float qscale;
  float lq, lv;  // q's and V's factors of log2 r_v: 1 / qscale together, lq a power of two
  int n_split;
  float* ws;
  int32_t* cnt;
  int cnt_shift;
  uint32_t ws_bytes;
};

// Granule placement in an fp16 row of LDS: granule c of row r sits at place
// c ^ swz(r), which keeps the reads of one column of 32 rows free of bank
// conflicts.
template <int D>
__device__ __forceinline__ int swz(int r) {
  return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

// Two neighbouring codes of a word, less 8, as fp16 numbers, exactly.
__device__ __forceinline__ half2v codes2(uint32_t w, int pair) {
  const uint32_t x = pair >= 2 ? w >> 8 : w;
  const uint32_t y = pair & 1 ? (x & 0x00f000f0u) | 0x54005400u : (x & 0x000f000fu) | 0x64006400u;
  const _Float16 c = static_cast<_Float16>(pair & 1 ? 72.f : 1032.f);
  return __builtin_bit_cast(half2v, y) - half2v{c, c};
}

// A row's parameters: s^, r, 1 / r and b. A row that stands for NaN has s^ = 0
// and b = NaN. Where 8 s^ or b / r would pass fp16's range (a row over nearly
// all of it, or at its ends), s^ is half and r twice as much.
struct RowPar {
  float s, r, ri, b;
};
constexpr float kWideScale = 8000.f, kFarOff = 32000.f;
__device__ __forceinline__ RowPar row_par(uint32_t w) {
  const half2v p = __builtin_bit_cast(half2v, w);
  const float s = static_cast<float>(p[0]), low = static_cast<float>(p[1]);
  const float b = __builtin_fmaf(8.f, s, low);
  const bool wide = s > kWideScale || __builtin_fabsf(b) > kFarOff;
  const float t = __uint_as_float((__float_as_uint(wide ? 0.5f * s : s) + 0x8000u) & 0xffff0000u);
  RowPar x;
  const bool on = s > 0.f;  // not 0, not NaN
  x.s = on ? t : 0.f;
  x.r = on ? s * __builtin_amdgcn_rcpf(t) : 1.f;
  x.ri = on ? t * __builtin_amdgcn_rcpf(s) : 1.f;
  x.b = b;
  return x;
}

template <int D, int QW, int KG, int KPW, bool INL>
__global__ __launch_bounds__(64 * QW * KG, 2) void kwp_kernel(
    KwpParams P, const std::conditional_t<INL, KwpPath, KwpNoPath> path) {
  constexpr int NT = 64 * QW * KG;     // threads
  constexpr int QR = 32 * QW;          // queries of a tile
  constexpr int UK = KG * KPW;         // keys of a unit
  static_assert(UK == 16 * QW * KG, "a tile of a unit to each wavefront");
  constexpr int ST = UK / 16;          // 16-row tiles of a unit
  constexpr int KS = D / 16;           // 32x32x16 steps over d
  constexpr int DT = D / 32;           // 32-channel tiles of O^T
  constexpr int JT = KPW / 32;         // 32-key tiles of S^T
  constexpr int CW = D / 32;           // code words a thread loads at once
  constexpr int KB = UK * D * 2;       // bytes of K (and of V) of a unit in LDS
  constexpr int RK = 2 * KB, AU = RK + UK * 4, AX = AU + UK * 8;  // factors; extra step; extra rows
  constexpr int BUF = AX + ST * 128;
  constexpr int OST = D + 4;           // merge row stride (floats)
  constexpr int MB = KG > 1 ? (KG - 1) * QR * (OST + 2) * 4 : 0;
  constexpr int LDS = 2 * BUF > MB ? 2 * BUF : MB;
  __shared__ __align__(16) char lds[LDS];
  __shared__ int s_last, s_far[4];  // s_far: a unit with a K row of r = 2
  __shared__ int s_path[INL ? 3 : 1][INL ? (kPrefillInlineChunks + 63) / 64 * 64 : 1];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qw = wv % QW, kg = wv / QW;
  const int l32 = lane & 31, hl = lane >> 5;
  const int H = P.H, n_q = P.n_q, C = P.C, L = P.L;
  const int n_qt = (n_q + QR - 1) / QR;
  // consecutive tiles of a head on one XCD (grid: a multiple of 8), the
  // longest first
  const int per_xcd = static_cast<int>(gridDim.x) / 8;
  const int v = static_cast<int>(blockIdx.x % 8) * per_xcd + static_cast<int>(blockIdx.x / 8);
  if (v >= n_qt * H * P.n_split) return;
  const int part = v % P.n_split, vt = v / P.n_split;
  const int h = vt / n_qt;
  const int q0 = (n_qt - 1 - vt % n_qt) * QR;
  const int qi = q0 + 32 * qw + l32;
  const int shift = L - n_q;
  const int pos = shift + min(qi, n_q - 1);                     // this lane's query
  const int blk_first = shift + q0, blk_last = shift + min(q0 + QR, n_q) - 1;
  const int wav_first = shift + min(q0 + 32 * qw, n_q - 1), wav_last = shift + min(q0 + 32 * qw + 31, n_q - 1);
  const int win = P.window, sinks = P.sinks;

  half8 qf[KS + 1];
#pragma unroll
  for (int s = 0; s < KS; ++s)
    qf[s] = *reinterpret_cast<const half8*>(P.q + (static_cast<size_t>(min(qi, n_q - 1)) * H + h) * D + 16 * s + 8 * hl);

  // Tiles, numbered along the path (chunk * tpc + tile of the chunk):
  // [0, ta) hold the sinks, [tb, te) what the tile's queries see besides.
  const int tpc = (C + 15) >> 4;
  const uint32_t magic = inverse32(tpc);
  auto slot_of = [&](int j) { if constexpr (INL) return path.slot[j]; else return P.dpath[j]; };
  auto start_of = [&](int j) { if constexpr (INL) return path.start[j]; else return P.dpath[P.n_chunks + j]; };
  auto end_of = [&](int j) { if constexpr (INL) return path.end[j]; else return P.dpath[2 * P.n_chunks + j]; };
  const int blk_lo = max(0, blk_first - win + 1);
  int ca = 0, cb = 0, ce = 0;  // chunks that start below the sinks; end at or below blk_lo; start up to blk_last
  int a_start = 0, b_start = 0, e_start = 0;  // starts of chunks ca - 1, cb, ce - 1
  for (int j0 = 0; 64 * j0 < P.n_chunks; ++j0) {
    const int j = min(64 * j0 + lane, P.n_chunks - 1);
    const int w_start = start_of(j), w_end = end_of(j);
    if constexpr (INL) {  // every wavefront the same, and reads what it wrote
      s_path[0][64 * j0 + lane] = slot_of(j);
      s_path[1][64 * j0 + lane] = w_start;
      s_path[2][64 * j0 + lane] = w_end;
    }
    const bool in = 64 * j0 + lane < P.n_chunks;
    const int na = __popcll(__ballot(in && w_start < sinks)), nb = __popcll(__ballot(in && w_end <= blk_lo)),
              ne = __popcll(__ballot(in && w_start <= blk_last));
    if (na > 0) a_start = __builtin_amdgcn_readlane(w_start, na - 1);
    if (cb == 64 * j0 && nb < 64) b_start = __builtin_amdgcn_readlane(w_start, nb);
    if (ne > 0) e_start = __builtin_amdgcn_readlane(w_start, ne - 1);
    ca += na;
    cb += nb;
    ce += ne;
  }
  const int te = (ce - 1) * tpc + min(blk_last - e_start, C - 1) / 16 + 1;  // ce >= 1
  int ta = ca > 0 ? (ca - 1) * tpc + (min(sinks - a_start, C) + 15) / 16 : 0;
  int tb = cb * tpc + max(0, blk_lo - b_start) / 16;
  ta = min(ta, te);
  if (tb < ta) tb = ta;
  const int n_tiles = ta + max(0, te - tb);
  const int n_units_all = (n_tiles + ST - 1) / ST;
  const int u_begin = static_cast<int>(static_cast<int64_t>(n_units_all) * part / P.n_split);
  const int u_end = static_cast<int>(static_cast<int64_t>(n_units_all) * (part + 1) / P.n_split);

  // 64 tiles at a time, one a lane, so that a unit's are v_readlane away.
  int held = -1, t_slot = 0, t_row = 0, t_pos = 0, t_end = 0;
  auto hold = [&](int base) {
    held = base;
    const int i = base + lane;
    const bool in = i < n_tiles;
    const int at = in ? (i < ta ? i : i - ta + tb) : 0;
    int c = divide32(at, tpc, magic);
    c -= c * tpc > at ? 1 : 0;  // of up to 2^26 tiles
    t_row = (at - c * tpc) * 16;
    if constexpr (INL) {
      t_slot = s_path[0][c];
      t_pos = s_path[1][c] + t_row;
      t_end = in ? min(s_path[2][c], blk_last + 1) : 0;
    } else {
      t_slot = slot_of(c);
      t_pos = start_of(c) + t_row;
      t_end = in ? min(end_of(c), blk_last + 1) : 0;
      // wait here, not where the loop reads them
      asm volatile("" : "+v"(t_slot), "+v"(t_pos), "+v"(t_end));
    }
  };
  struct Unit {
    int slot, row, p0, e0;     // of this wavefront's tile (loads, stores)
    int pos[KPW / 16], end[KPW / 16];  // of its keys' tiles; end <= pos: no token
  };
  auto unit_at = [&](int u) {
    Unit d;
    const int base = (u * ST) & ~63, l0 = (u * ST) & 63;
    if (base != held) hold(base);
    d.slot = __builtin_amdgcn_readlane(t_slot, l0 + wv);
    d.row = __builtin_amdgcn_readlane(t_row, l0 + wv);
    d.p0 = __builtin_amdgcn_readlane(t_pos, l0 + wv);
    d.e0 = __builtin_amdgcn_readlane(t_end, l0 + wv);
#pragma unroll
    for (int t = 0; t < KPW / 16; ++t) {
      d.pos[t] = __builtin_amdgcn_readlane(t_pos, l0 + kg * (KPW / 16) + t);
      d.end[t] = __builtin_amdgcn_readlane(t_end, l0 + kg * (KPW / 16) + t);
    }
    return d;
  };

  // One load of everything is a tile a wavefront: K and V words, and the
  // parameters of row lane % 16.
  struct Regs {
    u32x4 k, v;
    uint32_t kr, vr;
  };
  const int par = kv4_rows(C) * (D / 2);
  auto load = [&](const Unit& d, Regs& x) {
    const char* kt = P.kpool + d.slot * P.ss + h * P.hs;
    const char* vt = P.vpool + d.slot * P.ss + h * P.hs;
    const unsigned off = lane * (D / 8);
    const char *kc = kt + d.row * (D / 2), *vc = vt + d.row * (D / 2);
    if constexpr (D == 128) {
      x.k = *reinterpret_cast<const u32x4*>(kc + off);
      x.v = *reinterpret_cast<const u32x4*>(vc + off);
    } else {
      const u32x2 a = *reinterpret_cast<const u32x2*>(kc + off), b = *reinterpret_cast<const u32x2*>(vc + off);
      x.k = u32x4{a[0], a[1], 0, 0};
      x.v = u32x4{b[0], b[1], 0, 0};
    }
    const char *kp = kt + par + d.row * 4, *vp = vt + par + d.row * 4;
    x.kr = *reinterpret_cast<const uint32_t*>(kp + 4u * (lane % 16));
    x.vr = *reinterpret_cast<const uint32_t*>(vp + 4u * (lane % 16));
  };
  auto store = [&](const Unit& d, const Regs& x, int b, int ring) {
    char* buf = lds + b * BUF;
    const int g = lane >> 4, n = lane & 15;
    const int r = 16 * wv + n;    // the lane's row of the unit
    const bool on = d.p0 + n < d.e0;  // what stands behind a chunk's last row is not looked at
    const RowPar k = row_par(on ? x.kr : 0u), w = row_par(on ? x.vr : 0u);
    {  // K: quarter g of row n
      const _Float16 ks = static_cast<_Float16>(k.s);
#pragma unroll
      for (int c = 0; c < CW; ++c) {
        const uint32_t word = x.k[c];
        half8 y;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const half2v z = codes2(word, p) * half2v{ks, ks};
          y[2 * p] = z[0];
          y[2 * p + 1] = z[1];
        }
        *reinterpret_cast<half8*>(buf + r * (D * 2) + 16 * ((g * CW + c) ^ swz<D>(r))) = y;
      }
    }
    // V: tokens 4g .. 4g + 3 of the tile (their s^ from the lanes of those rows)
    // at channels 32 c + 16 e + n, to [tile][channel][groups 0, 2, 1, 3]: a
    // lane of the operand reads groups hl and 2 + hl of its channel at once
    {
      const int vs = __builtin_bit_cast(uint16_t, static_cast<_Float16>(w.s));
      int t4[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) t4[i] = __builtin_amdgcn_ds_bpermute(4 * (4 * g + i), vs);
      const half2v s0 = __builtin_bit_cast(half2v, t4[0] | (t4[1] << 16));
      const half2v s1 = __builtin_bit_cast(half2v, t4[2] | (t4[3] << 16));
      char* vt = buf + KB + wv * (D * 32) + 8 * (((g & 1) << 1) | (g >> 1));
#pragma unroll
      for (int c = 0; c < CW; ++c) {
        const uint32_t word = x.v[c];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const half2v a0 = codes2(word, 2 * e) * s0, a1 = codes2(word, 2 * e + 1) * s1;
          *reinterpret_cast<half4*>(vt + (32 * c + 16 * e + n) * 32) = half4{a0[0], a0[1], a1[0], a1[1]};
        }
      }
    }
    if (g == 0) {
      if (k.r > 1.5f) s_far[ring] = 1;
      *reinterpret_cast<float*>(buf + RK + 4 * r) = P.qscale * k.r;
      // the extra step of the scores, over r_k, by which the product is
      // multiplied: b_k, and log2 r_v; a V row that stands for NaN shows there
      const float kb = k.b * k.ri;
      const _Float16 hi = static_cast<_Float16>(kb);
      const float lr = w.b == w.b ? __builtin_amdgcn_logf(w.r) * P.lv * k.ri : w.b;
      *reinterpret_cast<half4*>(buf + AU + 8 * r) =
          half4{hi, static_cast<_Float16>(kb - static_cast<float>(hi)), static_cast<_Float16>(lr), hi};
    } else if (g == 1) {
      // the extra channel tile's rows: 1 / r_v and b_v / r_v, two halves each, the
      // tokens placed as V's
      const float vb = w.b == w.b ? w.b * w.ri : 0.f;
      const _Float16 h0 = static_cast<_Float16>(w.ri), h1 = static_cast<_Float16>(vb);
      _Float16* ax = reinterpret_cast<_Float16*>(buf + AX + wv * 128) + 4 * (((n >> 2 & 1) << 1) | (n >> 3)) + (n & 3);
      ax[0] = h0;
      ax[16] = static_cast<_Float16>(w.ri - static_cast<float>(h0));
      ax[32] = h1;
      ax[48] = static_cast<_Float16>(vb - static_cast<float>(h1));
    }
  };

  auto read_k = [&](int b, int jt, int s) {
    const int r = kg * KPW + 32 * jt + l32;
    return *reinterpret_cast<const half8*>(lds + b * BUF + r * (D * 2) + 16 * ((2 * s + hl) ^ swz<D>(r)));
  };
  // V^T operand of keys 16 p .. 16 p + 15 of the wavefront's share: element e
  // is key 4 hl + e, then 8 + 4 hl + e - 4, of channel 32 dt + l32
  auto read_v = [&](int b, int p, int dt) {
    const int t = kg * (KPW / 16) + p;
    return *reinterpret_cast<const half8*>(lds + b * BUF + KB + t * (D * 32) + (32 * dt + l32) * 32 + 16 * hl);
  };
  auto read_x = [&](int b, int p) {  // rows past the fourth are not used
    const int t = kg * (KPW / 16) + p;
    return *reinterpret_cast<const half8*>(lds + b * BUF + AX + t * 128 + (l32 & 3) * 32 + 16 * hl);
  };

  Unit cur = unit_at(u_begin), nxt = cur, nx2 = cur;
  Regs ra, rb;
  load(cur, ra);
  nxt = unit_at(min(u_begin + 1, max(u_end, 1) - 1));
  load(nxt, rb);
  if (tid == 0) s_far[0] = 0;
  __syncthreads();

  // q's part of the extra step: sum(q) as two fp16 (of q 2^-8, the query's scores
  // 2^8 back up, where the sum is too large for one), and lq
  bool any_up = false;
  {
    float sum = 0.f, up = 1.f;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += static_cast<float>(qf[s][i]);
    sum += __shfl_xor(sum, 32);
    any_up = __any(fabsf(sum) > 6e4f);
    if (any_up) {
      up = fabsf(sum) > 6e4f ? 256.f : 1.f;
      const float down = 1.f / up;
      sum *= down;
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) qf[s][i] = qf[s][i] * static_cast<_Float16>(down);
    }
    const _Float16 hi = static_cast<_Float16>(sum);
    const _Float16 lo = static_cast<_Float16>(sum - static_cast<float>(hi));
    const _Float16 c = static_cast<_Float16>(P.lq / up);
    const _Float16 z = static_cast<_Float16>(0.f);
    qf[KS] = hl == 0 ? half8{hi, hi, c, lo, z, z, z, z} : half8{z, z, z, z, z, z, z, z};
  }

  float m_run = kNegBig;
  floatx16 acc[DT + 1];  // the last: sum w / r and sum w b / r, in rows 0 .. 3
#pragma unroll
  for (int dt = 0; dt <= DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;

  auto compute = [&](const Unit& d, int b, int ring) {
    const int (&p_)[KPW / 16] = d.pos;
    const int (&e_)[KPW / 16] = d.end;
    bool whole = true, none = true;
#pragma unroll
    for (int t = 0; t < KPW / 16; ++t) {
      whole &= p_[t] + 16 <= e_[t] && p_[t] + 15 <= wav_first && (p_[t] > wav_last - win || p_[t] + 16 <= sinks);
      none &= e_[t] <= p_[t] || p_[t] > wav_last || (p_[t] + 15 <= wav_first - win && p_[t] >= sinks);
    }
    if (none) return;
    floatx16 sa[JT];
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) {
      half8 x;
      const half4 y = *reinterpret_cast<const half4*>(lds + b * BUF + AU + 8 * (kg * KPW + 32 * jt + l32));
      x = __builtin_shufflevector(y, y, 0, 1, 2, 3, 0, 1, 2, 3);  // times zeros of q from the fifth on
      floatx16 z;
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] = 0.f;
      sa[jt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, qf[KS], z, 0, 0, 0);
    }
    // eight operands in flight at a time (left alone, the compiler reads each
    // when it is needed and waits for it)
    constexpr int KH = 8 / JT < KS ? 8 / JT : KS;
    static_assert(KS % KH == 0, "whole groups");
#pragma unroll
    for (int s0 = 0; s0 < KS; s0 += KH) {
      half8 ka[KH][JT];
#pragma unroll
      for (int s = 0; s < KH; ++s)
#pragma unroll
        for (int jt = 0; jt < JT; ++jt) ka[s][jt] = read_k(b, jt, s0 + s);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s < KH; ++s)
#pragma unroll
        for (int jt = 0; jt < JT; ++jt)
          sa[jt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ka[s][jt], qf[s0 + s], sa[jt], 0, 0, 0);
    }
    if (any_up) {
      asm volatile("");
      // the query's 2^8 or 1, from its lane with lq / up (a register of its own
      // would not be left)
      const float up = P.lq / __shfl(static_cast<float>(qf[KS][2]), l32);
#pragma unroll
      for (int jt = 0; jt < JT; ++jt) sa[jt] *= up;
    }
    if (!whole) {
      asm volatile("");
      // min with +inf for a visible pair, -inf for another: integer arithmetic
      // on signs (lane masks of 32 elements would spill the scalar registers)
#pragma unroll
      for (int jt = 0; jt < JT; ++jt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int t = 2 * jt + (r >> 3);
          const int j = p_[t] + 4 * hl + 8 * ((r >> 2) & 1) + (r & 3);
          const int hid = (min(e_[t] - 1, pos) - j) | max(j - (pos - win + 1), sinks - 1 - j);
          sa[jt][r] = fminf(sa[jt][r], __int_as_float((hid & INT32_MIN) | 0x7f800000));
        }
    }
    floatx4 rk[JT * 4];
#pragma unroll
    for (int x = 0; x < JT * 4; ++x)
      rk[x] = *reinterpret_cast<const floatx4*>(lds + b * BUF + RK + 4 * (kg * KPW + 8 * x + 4 * hl));
    auto top = [&]() {
      float c[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int jt = 0; jt < JT; ++jt)
#pragma unroll
        for (int r = 0; r < 16; ++r) c[r & 3] = fmaxf(c[r & 3], sa[jt][r]);
      float a = fmaxf(fmaxf(c[0], c[1]), fmaxf(c[2], c[3])), e = a;
      swap_halves32(a, e);
      return fmaxf(a, e) * P.qscale;
    };
    float mx = top();
    if (__any(fabsf(mx) > kFarScore && mx > -INFINITY) || __builtin_amdgcn_readfirstlane(s_far[ring])) {
      asm volatile("");
      const float f = 1.f / P.qscale;
#pragma unroll
      for (int x = 0; x < JT * 4; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sa[x / 4][4 * (x % 4) + i] *= rk[x][i] * f;
          rk[x][i] = P.qscale;
        }
      mx = top();
    }
    const float mn = mx > m_run + kLazyMax ? mx : m_run;
    if (__any(mn != m_run)) {
      asm volatile("");
      const float al = fast_exp2(m_run - mn);
#pragma unroll
      for (int dt = 0; dt <= DT; ++dt) acc[dt] *= al;
      m_run = mn;
    }
    half8 pb[2 * JT];
#pragma unroll
    for (int jt = 0; jt < JT; ++jt)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        pb[2 * jt + r / 8][r % 8] =
            static_cast<_Float16>(fast_exp2(__builtin_fmaf(sa[jt][r], rk[4 * jt + r / 4][r % 4], -m_run)));
#pragma unroll
    for (int p = 0; p < 2 * JT; ++p) {
      half8 va[DT + 1];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) va[dt] = read_v(b, p, dt);
      va[DT] = read_x(b, p);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int dt = 0; dt <= DT; ++dt)
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(va[dt], pb[p], acc[dt], 0, 0, 0);
    }
  };

  // Unit u is computed from buffer u % 2; the registers unit u came in take
  // unit u + 2. Past the end the last unit is loaded again, so that every step
  // issues the same loads and a wait covers only the registers it needs.
  auto step = [&](int u, Regs& x) {
    const int b = (u - u_begin) & 1, ring = (u - u_begin) & 3;
    store(cur, x, b, ring);
    if (tid == 0) s_far[(ring + 1) & 3] = 0;  // last read three units ago
    nx2 = unit_at(min(u + 2, u_end - 1));
    load(nx2, x);
    __syncthreads();
    if (u < u_end) compute(cur, b, ring);
    cur = nxt;
    nxt = nx2;
  };
  // (an odd last unit is stored twice: a step under a condition would have the
  // compiler keep one register set and move the other one there, loads waited for)
  for (int u = u_begin; u < u_end; u += 2) {
    step(u, ra);
    step(u + 1, rb);
  }
  // rows 0 .. 3 of the extra tile sit in the lower half's first registers
  float n_row = acc[DT][0] + acc[DT][1], base = acc[DT][2] + acc[DT][3];
  n_row = __shfl(n_row, l32);
  base = __shfl(base, l32);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] += base;

  // Fold the key groups, then write o or the part's partial.
  const int r = 32 * qw + l32;  // row inside the tile
  if constexpr (KG > 1) {
    float* ob = reinterpret_cast<float*>(lds);  // [KG - 1][QR][OST]
    float* mb = ob + (KG - 1) * QR * OST;       // [KG - 1][QR][2]
    __syncthreads();
    if (kg > 0) {
      float* at = ob + ((kg - 1) * QR + r) * OST + 4 * hl;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int b = 0; b < 4; ++b)
          *reinterpret_cast<floatx4*>(at + 32 * dt + 8 * b) =
              floatx4{acc[dt][4 * b], acc[dt][4 * b + 1], acc[dt][4 * b + 2], acc[dt][4 * b + 3]};
      if (hl == 0) {
        mb[((kg - 1) * QR + r) * 2] = m_run;
        mb[((kg - 1) * QR + r) * 2 + 1] = n_row;
      }
    }
    __syncthreads();
    if (kg == 0) {
#pragma unroll
      for (int k = 1; k < KG; ++k) {
        const float mo = mb[((k - 1) * QR + r) * 2], no = mb[((k - 1) * QR + r) * 2 + 1];
        const float M = fmaxf(m_run, mo);
        const float a = fast_exp2(m_run - M), c = fast_exp2(mo - M);
        const float* at = ob + ((k - 1) * QR + r) * OST + 4 * hl;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const floatx4 x = *reinterpret_cast<const floatx4*>(at + 32 * dt + 8 * b);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[dt][4 * b + i] = acc[dt][4 * b + i] * a + x[i] * c;
          }
        n_row = n_row * a + no * c;
        m_run = M;
      }
    }
  }
  auto write4 = [&](int row, int ch, const floatx4& x, float inv) {
    half4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = static_cast<_Float16>(x[i] * inv);
    *reinterpret_cast<half4*>(P.o + (static_cast<size_t>(q0 + row) * H + h) * D + ch) = y;
  };
  if (P.n_split == 1) {
    if (kg == 0 && qi < n_q) {
      const float inv = 1.f / n_row;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int b = 0; b < 4; ++b)
          write4(r, 32 * dt + 8 * b + 4 * hl,
                 floatx4{acc[dt][4 * b], acc[dt][4 * b + 1], acc[dt][4 * b + 2], acc[dt][4 * b + 3]}, inv);
    }
    return;
  }
  // Parts: [tile][part] of QR rows of D floats, then QR (m, n) pairs; the
  // exchange protocol of device_common.hpp.
  constexpr uint32_t kPart = (QR * D + 2 * QR) * 4;
  const __amdgpu_buffer_rsrc_t rs = part_rsrc(P.ws, P.ws_bytes);
  if (kg == 0) {
    const uint32_t at = (static_cast<uint32_t>(vt) * P.n_split + part) * kPart;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        st_dev4(rs, at + (r * D + 32 * dt + 8 * b + 4 * hl) * 4u, acc[dt][4 * b], acc[dt][4 * b + 1],
                acc[dt][4 * b + 2], acc[dt][4 * b + 3]);
    if (hl == 0) {
      float* ml = P.ws + at / 4 + QR * D + 2 * r;
      st_dev(ml, m_run);
      st_dev(ml + 1, n_row);
    }
  }
  wait_stores();
  __syncthreads();
  if (tid == 0) s_last = arrive_last(P.cnt + (static_cast<size_t>(vt) << P.cnt_shift), P.n_split);
  __syncthreads();
  if (!s_last) return;
  // four parts of four places (row, four channels) a thread, all their loads in
  // flight together: one after the other, the round trips took 30 us here
  constexpr int IPT = QR * (D / 4) / NT, NI = IPT < 4 ? IPT : 4, NB = 4;
  static_assert(IPT % NI == 0, "places of a thread");
  const int rows = min(QR, n_q - q0);
#pragma unroll 1
  for (int k0 = 0; k0 < IPT; k0 += NI) {
    float m[NI], n[NI];
    floatx4 x[NI];
#pragma unroll
    for (int k = 0; k < NI; ++k) {
      m[k] = kNegBig;
      n[k] = 0.f;
      x[k] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll 1
    for (int p0 = 0; p0 < P.n_split; p0 += NB) {
      float pm[NB][NI], pn[NB][NI];
      float4 y[NB][NI];
#pragma unroll
      for (int p = 0; p < NB; ++p) {
        // past the last part: that one again, not used
        const uint32_t at = (static_cast<uint32_t>(vt) * P.n_split + min(p0 + p, P.n_split - 1)) * kPart;
#pragma unroll
        for (int k = 0; k < NI; ++k) {
          const int i = tid + NT * (k0 + k), row = i / (D / 4), ch = 4 * (i % (D / 4));
          const float* ml = P.ws + at / 4 + QR * D + 2 * row;
          pm[p][k] = ld_dev(ml);
          pn[p][k] = ld_dev(ml + 1);
          y[p][k] = ld_dev4(rs, at + (row * D + ch) * 4u);
        }
      }
#pragma unroll
      for (int p = 0; p < NB; ++p) {
        if (p0 + p >= P.n_split) break;
#pragma unroll
        for (int k = 0; k < NI; ++k) {
          const float M = fmaxf(m[k], pm[p][k]);
          const float f = fast_exp2(m[k] - M), c = fast_exp2(pm[p][k] - M);
          n[k] = n[k] * f + pn[p][k] * c;
          x[k] = x[k] * f + floatx4{y[p][k].x, y[p][k].y, y[p][k].z, y[p][k].w} * c;
          m[k] = M;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < NI; ++k) {
      const int i = tid + NT * (k0 + k), row = i / (D / 4), ch = 4 * (i % (D / 4));
      if (row < rows) write4(row, ch, x[k], 1.f / n[k]);
    }
  }
}

template <int D, int QW, int KG, int KPW>
void launch_wp(const KwpParams& P, const Kv4PrefillArgs& a, hipStream_t stream) {
  const int blocks = (a.n_q + 32 * QW - 1) / (32 * QW) * a.H * a.n_split;
  const dim3 grid(8 * ((blocks + 7) / 8));
  if (a.host_path) {
    KwpPath path;
    for (int j = 0; j < a.n_chunks; ++j) {
      path.slot[j] = a.host_path[j];
      path.start[j] = a.host_path[a.n_chunks + j];
      path.end[j] = a.host_path[2 * a.n_chunks + j];
    }
    kwp_kernel<D, QW, KG, KPW, true><<<grid, 64 * QW * KG, 0, stream>>>(P, path);
  } else {
    kwp_kernel<D, QW, KG, KPW, false><<<grid, 64 * QW * KG, 0, stream>>>(P, KwpNoPath{});
  }
}

}  // namespace

hipError_t launch_kv4_prefill(const Kv4PrefillArgs& a, hipStream_t stream) {
  if (a.n_q <= 0 || a.n_chunks <= 0) return hipSuccess;
  if (a.host_path ? a.n_chunks > kPrefillInlineChunks : !a.path) return hipErrorInvalidValue;
  if (a.n_split < 1 || (a.n_split > 1 && (!a.ws || !a.cnt || a.ws_bytes > 0xFFFFFFF0ull)))
    return hipErrorInvalidValue;
  // lq is a normal fp16 value, exact over 2^8 too; lv log2 r_v (r_v < 2.02) fits
  // fp16 down to scales of 2^-29, and keeps four bits or more up to 2^24 (log2 r_v
  // is at most 2^-8 there but for wide rows, so that these are enough)
  if (!(a.qscale >= 0x1p-29f && a.qscale <= 0x1p24f)) return hipErrorInvalidValue;
  const float lq = std::ldexp(1.f, std::min(std::max(-std::ilogb(a.qscale) - 8, -13), 14));
  const KwpParams P{static_cast<const _Float16*>(a.q), static_cast<_Float16*>(a.o),
                    static_cast<const char*>(a.kpool), static_cast<const char*>(a.vpool), a.ss, a.hs,
                    a.path, a.n_chunks, a.n_q, a.H, a.C, a.L, a.window, a.sinks, a.qscale, lq,
                    1.f / (a.qscale * lq), a.n_split, a.ws, a.cnt, a.cnt_shift,
                    static_cast<uint32_t>(a.ws_bytes)};
  if (a.D == 128 && a.tile_rows == 128) launch_wp<128, 4, 1, 64>(P, a, stream);
  else if (a.D == 128 && a.tile_rows == 64) launch_wp<128, 2, 4, 32>(P, a, stream);
  else if (a.D == 64 && a.tile_rows == 128) launch_wp<64, 4, 1, 64>(P, a, stream);
  else if (a.D == 64 && a.tile_rows == 64) launch_wp<64, 2, 4, 32>(P, a, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace ca
