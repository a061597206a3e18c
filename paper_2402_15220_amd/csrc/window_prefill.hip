// gfx950 (MI355X) prefill attention with a sliding window and sinks, over fp16
// and 4-bit pools, and every prefill call over a 4-bit pool.
//
// The last n_q tokens of a sequence of L tokens attend causally: the query at
// position p sees the positions j <= p with j < sinks or j > p - window.
//
// One block of four wavefronts per (tile of 32 QW queries, head, part of the
// tile's keys). The keys that some query of the tile sees are taken as tiles
// of 16 rows of the path's chunks, in order, UK / 16 of them to a unit; tiles
// between the sinks and the first query's window are left out. A unit goes
// from memory into registers while the one before is computed, and from there
// into one of two LDS buffers (one barrier a unit); codes become fp16 values
// on the way, low + scale * code with one rounding, once for all the tile's
// queries (2^-12 of the value, as where the rows themselves are kept in fp16).
// Wavefront (qw, kg) owns 32 queries and KPW keys of every unit:
//   S^T = K Q^T     32x32x16 matrix ops, K rows as A, q as B (in registers);
//   mask where a unit has a pair that is not seen, online softmax in base 2
//   with a lazy reference maximum;
//   O^T += V^T P^T  P straight from the registers S^T came out in; V^T from
//                   LDS, fp16 rows through ds_read_b64_tr_b16, codes laid out
//                   as the operand when they are written.
// The key groups' states (Eqn 2), and with several parts those of the blocks,
// are folded at the end; the last block of a tile to arrive does the latter.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cstdint>
#include <type_traits>

#include "device_common.hpp"
#include "kernels.hpp"
#include "kv4.hpp"

namespace ca {
namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLazyMax = 8.f;

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
  const int32_t* dslot;  // device path (long paths): slots, starts, ends
  int n_chunks, n_q, H, C, L;
  int window, sinks;
  float qscale;
  int n_split;
  float* ws;
  int32_t* cnt;
  int cnt_shift;
  uint32_t ws_bytes;
};

// Granule placement in an fp16 row of LDS: granule c of row r sits at place
// c ^ swz(r), which keeps the reads of one column of 32 rows and of 64 bytes
// of four rows free of bank conflicts.
template <int D>
__device__ __forceinline__ int swz(int r) {
  return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

template <int S, int D, int QW, int KG, int KPW, bool INL>
__global__ __launch_bounds__(256, 2) void kwp_kernel(KwpParams P,
                                                     const std::conditional_t<INL, KwpPath, KwpNoPath> path) {
  static_assert(QW * KG == 4, "four wavefronts");
  constexpr int QR = 32 * QW;          // queries of a tile
  constexpr int UK = KG * KPW;         // keys of a unit
  constexpr int ST = UK / 16;          // 16-row tiles of a unit
  constexpr int KS = D / 16;           // 32x32x16 steps over d
  constexpr int DT = D / 32;           // 32-channel tiles of O^T
  constexpr int JT = KPW / 32;         // 32-key tiles of S^T
  constexpr int NG = D / 8;            // 16-byte granules of an fp16 row
  constexpr int KB = UK * D * 2;       // bytes of K (and of V) of a unit in LDS
  constexpr int OST = D + 4;           // merge row stride (floats)
  constexpr int MB = KG > 1 ? (KG - 1) * QR * (OST + 2) * 4 : 0;
  constexpr int LDS = 4 * KB > MB ? 4 * KB : MB;
  // staged registers: fp16 granules, or code words and parameters
  constexpr int NL = S == kStoreF16 ? UK * NG / 256 : UK * D / 2 / (4 * D / 32 * 256);
  constexpr int CW = D / 32;           // code words a thread loads at once
  __shared__ __align__(16) char lds[LDS];
  __shared__ int s_last, s_bad[4];

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

  half8 qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s)
    qf[s] = *reinterpret_cast<const half8*>(P.q + (static_cast<size_t>(min(qi, n_q - 1)) * H + h) * D + 16 * s + 8 * hl);

  auto slot_of = [&](int j) { if constexpr (INL) return path.slot[j]; else return P.dslot[j]; };
  auto start_of = [&](int j) { if constexpr (INL) return path.start[j]; else return P.dslot[P.n_chunks + j]; };
  auto end_of = [&](int j) { if constexpr (INL) return path.end[j]; else return P.dslot[2 * P.n_chunks + j]; };

  // Tiles, numbered along the path (chunk * tpc + tile of the chunk):
  // [0, ta) hold the sinks, [tb, te) what the tile's queries see besides.
  const int tpc = (C + 15) >> 4;
  const int blk_lo = max(0, blk_first - win + 1);
  int ca = 0, cb = 0, ce = 0;  // chunks that start below the sinks; end at or below blk_lo; start up to blk_last
  for (int j0 = 0; j0 < P.n_chunks; j0 += 64) {
    const int j = min(j0 + lane, P.n_chunks - 1);
    const int st = start_of(j), en = end_of(j);
    const bool in = j0 + lane < P.n_chunks;
    ca += __popcll(__ballot(in && st < sinks));
    cb += __popcll(__ballot(in && en <= blk_lo));
    ce += __popcll(__ballot(in && st <= blk_last));
  }
  int ta = 0;
  if (ca > 0) ta = (ca - 1) * tpc + (min(sinks - start_of(ca - 1), C) + 15) / 16;
  int tb = cb * tpc + max(0, blk_lo - start_of(min(cb, P.n_chunks - 1))) / 16;
  const int te = (ce - 1) * tpc + min(blk_last - start_of(ce - 1), C - 1) / 16 + 1;  // ce >= 1
  ta = min(ta, te);
  if (tb < ta) tb = ta;
  const int n_tiles = ta + max(0, te - tb);
  const int n_units_all = (n_tiles + ST - 1) / ST;
  const int u_begin = static_cast<int>(static_cast<int64_t>(n_units_all) * part / P.n_split);
  const int u_end = static_cast<int>(static_cast<int64_t>(n_units_all) * (part + 1) / P.n_split);

  struct Unit {
    int slot[ST], row[ST], pos[ST], end[ST];  // end <= pos: no token
  };
  auto unit_at = [&](int u) {
    Unit d;
#pragma unroll
    for (int t = 0; t < ST; ++t) {
      const int i = u * ST + t;
      const bool in = i < n_tiles;
      const int at = in ? (i < ta ? i : i - ta + tb) : 0;
      const int c = at / tpc, r = at - c * tpc;
      d.slot[t] = __builtin_amdgcn_readfirstlane(slot_of(c));
      d.row[t] = __builtin_amdgcn_readfirstlane(r * 16);
      d.pos[t] = __builtin_amdgcn_readfirstlane(start_of(c) + r * 16);
      d.end[t] = __builtin_amdgcn_readfirstlane(in ? min(end_of(c), blk_last + 1) : 0);
    }
    return d;
  };

  u32x4 kr[NL], vr[NL];
  uint32_t kp[NL];
  u32x4 vp[NL];
  // Load i of the block covers RPI rows: fp16, WR neighbouring ones of one
  // 16-row tile a wavefront; 4-bit, a tile a wavefront.
  constexpr int RPI = S == kStoreF16 ? 256 / NG : 64;
  constexpr int WR = RPI / 4;
  auto pick = [&](const int (&x)[ST], int i) {  // the wavefront's tile of load i
    int y = x[i * RPI / 16];
#pragma unroll
    for (int t = 1; t < RPI / 16; ++t) y = wv * WR / 16 == t ? x[i * RPI / 16 + t] : y;
    return y;
  };
  auto load = [&](const Unit& d) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      if constexpr (S == kStoreF16) {
        // the rows of a wavefront's load lie in one 16-row tile
        const int slot = pick(d.slot, i), row = pick(d.row, i);
        const int r = min(row + (wv * WR) % 16 + lane / NG, C - 1);
        const int64_t off = slot * P.ss + h * P.hs;
        const size_t in = static_cast<size_t>(r) * (D * 2) + 16 * (lane % NG);
        kr[i] = *reinterpret_cast<const u32x4*>(P.kpool + off + in);
        vr[i] = *reinterpret_cast<const u32x4*>(P.vpool + off + in);
      } else {
        const int slot = pick(d.slot, i), row = pick(d.row, i);
        const char* kt = P.kpool + slot * P.ss + h * P.hs;
        const char* vt = P.vpool + slot * P.ss + h * P.hs;
        const int pb = kv4_rows(C) * (D / 2);
        const char* kc = kt + row * (D / 2) + lane * (D / 8);
        const char* vc = vt + row * (D / 2) + lane * (D / 8);
        if constexpr (D == 128) {
          kr[i] = *reinterpret_cast<const u32x4*>(kc);
          vr[i] = *reinterpret_cast<const u32x4*>(vc);
        } else {
          const u32x2 a = *reinterpret_cast<const u32x2*>(kc), b = *reinterpret_cast<const u32x2*>(vc);
          kr[i] = u32x4{a[0], a[1], 0, 0};
          vr[i] = u32x4{b[0], b[1], 0, 0};
        }
        kp[i] = *reinterpret_cast<const uint32_t*>(kt + pb + (row + lane % 16) * 4);
        vp[i] = *reinterpret_cast<const u32x4*>(vt + pb + (row + 4 * (lane / 16)) * 4);
      }
    }
  };
  // two neighbouring codes of a word as fp16 numbers, exactly
  auto codes2 = [](uint32_t w, int pair) {
    const uint32_t x = pair >= 2 ? w >> 8 : w;
    const uint32_t y = pair & 1 ? (x & 0x00f000f0u) | 0x54005400u : (x & 0x000f000fu) | 0x64006400u;
    const _Float16 c = pair & 1 ? static_cast<_Float16>(64.f) : static_cast<_Float16>(1024.f);
    return __builtin_bit_cast(half2v, y) - half2v{c, c};
  };
  // Unit d into buffer b. At an edge (a unit of which some query of the tile
  // does not see all), rows past a chunk's end or after the last query become
  // zeros and s_bad[ring] tells of V elements that are not finite.
  auto store = [&](const Unit& d, int b, int ring) {
    char* kl = lds + b * 2 * KB;
    char* vl = kl + KB;
    bool edge = false;
#pragma unroll
    for (int t = 0; t < ST; ++t)
      edge |= d.pos[t] + 16 > d.end[t] || d.pos[t] + 15 > blk_first ||
              (d.pos[t] <= blk_last - win && d.pos[t] + 16 > sinks);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      if constexpr (S == kStoreF16) {
        const int r = i * RPI + wv * WR + lane / NG;  // row of the unit
        const int at = r * (D * 2) + 16 * ((lane % NG) ^ swz<D>(r));
        *reinterpret_cast<u32x4*>(kl + at) = kr[i];
        u32x4 x = vr[i];
        if (edge) {
          if (pick(d.pos, i) + r % 16 >= pick(d.end, i)) x = u32x4{0, 0, 0, 0};
          bool bad = false;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            bad |= ((x[k] & 0x7c00u) == 0x7c00u) || ((x[k] & 0x7c000000u) == 0x7c000000u);
          if (bad) s_bad[ring] = 1;
        }
        *reinterpret_cast<u32x4*>(vl + at) = x;
      } else {
        const int t0 = i * 4 + wv;
        const int p0 = pick(d.pos, i), e0 = pick(d.end, i);
        // K: this thread's quarter of row lane % 16
        const int r = 16 * t0 + lane % 16;
        const half2v kpar = __builtin_bit_cast(half2v, kp[i]);
        const half2v ks = {kpar[0], kpar[0]}, ko = {kpar[1], kpar[1]};
#pragma unroll
        for (int w = 0; w < CW; ++w) {
          const uint32_t word = kr[i][w];
          half8 y;
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const half2v z = __builtin_elementwise_fma(codes2(word, p), ks, ko);
            y[2 * p] = z[0];
            y[2 * p + 1] = z[1];
          }
          const int c = (lane / 16) * CW + w;  // granule of the row
          *reinterpret_cast<half8*>(kl + r * (D * 2) + 16 * (c ^ swz<D>(r))) = y;
        }
        // V: tokens 4g .. 4g + 3 of the tile at channels 32 w + 16 b + n, to
        // [tile][channel][groups 0, 2, 1, 3]: a lane of the operand reads
        // groups hl and 2 + hl of its channel at once
        const int g = lane >> 4, n = lane & 15;
        const uint32_t q0_ = vp[i][0], q1_ = vp[i][1], q2_ = vp[i][2], q3_ = vp[i][3];
        const half2v a0 = __builtin_bit_cast(half2v, q0_), a1 = __builtin_bit_cast(half2v, q1_),
                     a2 = __builtin_bit_cast(half2v, q2_), a3 = __builtin_bit_cast(half2v, q3_);
        const int j0 = p0 + 4 * g;
        const _Float16 z0 = static_cast<_Float16>(0.f);
        const half2v s0 = {j0 < e0 ? a0[0] : z0, j0 + 1 < e0 ? a1[0] : z0};
        const half2v s1 = {j0 + 2 < e0 ? a2[0] : z0, j0 + 3 < e0 ? a3[0] : z0};
        const half2v o0 = {j0 < e0 ? a0[1] : z0, j0 + 1 < e0 ? a1[1] : z0};
        const half2v o1 = {j0 + 2 < e0 ? a2[1] : z0, j0 + 3 < e0 ? a3[1] : z0};
        if (edge) {
          const half2v z = o0 + o1 + s0 + s1;  // NaN where a row stands for NaN
          if (!(z[0] == z[0]) || !(z[1] == z[1])) s_bad[ring] = 1;
        }
        char* vt = vl + t0 * (D * 32) + 8 * (((g & 1) << 1) | (g >> 1));
#pragma unroll
        for (int w = 0; w < CW; ++w) {
          const uint32_t word = vr[i][w];
#pragma unroll
          for (int hb = 0; hb < 2; ++hb) {
            const half2v x = __builtin_elementwise_fma(codes2(word, 2 * hb), s0, o0);
            const half2v y = __builtin_elementwise_fma(codes2(word, 2 * hb + 1), s1, o1);
            *reinterpret_cast<half4*>(vt + (32 * w + 16 * hb + n) * 32) = half4{x[0], x[1], y[0], y[1]};
          }
        }
      }
    }
  };

  auto read_k = [&](int b, int jt, int s) {
    const int r = kg * KPW + 32 * jt + l32;
    return *reinterpret_cast<const half8*>(lds + b * 2 * KB + r * (D * 2) + 16 * ((2 * s + hl) ^ swz<D>(r)));
  };
  // V^T operand of keys 16 p .. 16 p + 15 of the wavefront's share: element e
  // is key 4 hl + e, then 8 + 4 hl + e - 4, of channel 32 dt + l32
  auto read_v = [&](int b, int p, int dt) {
    const char* vl = lds + b * 2 * KB + KB;
    const int t = kg * (KPW / 16) + p;
    if constexpr (S == kStoreF16) {
      const int i16 = lane & 15, sub = (lane >> 4) & 1;
      half4 x[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 16 * t + 8 * e + 4 * hl + (i16 >> 2);
        x[e] = lds_read_tr16(reinterpret_cast<const _Float16*>(
            vl + r * (D * 2) + 16 * ((4 * dt + 2 * sub + ((i16 & 3) >> 1)) ^ swz<D>(r)) + 8 * (i16 & 1)));
      }
      return __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *reinterpret_cast<const half8*>(vl + t * (D * 32) + (32 * dt + l32) * 32 + 16 * hl);
    }
  };

  float m_run = kNegBig, n_run = 0.f;
  floatx16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;

  auto compute = [&](const Unit& d, int b, int ring) {
    bool whole = true, none = true;
#pragma unroll
    for (int t = 0; t < KPW / 16; ++t) {
      int p0 = d.pos[t], e0 = d.end[t];
      if constexpr (KG > 1) {
#pragma unroll
        for (int k = 1; k < KG; ++k) {
          p0 = kg == k ? d.pos[k * (KPW / 16) + t] : p0;
          e0 = kg == k ? d.end[k * (KPW / 16) + t] : e0;
        }
      }
      whole &= p0 + 16 <= e0 && p0 + 15 <= wav_first && (p0 > wav_last - win || p0 + 16 <= sinks);
      none &= e0 <= p0 || p0 > wav_last || (p0 + 15 <= wav_first - win && p0 >= sinks);
    }
    if (none) return;
    // sign bit set: key 16 t + k of the wavefront's share is not seen by this
    // lane's query (integer arithmetic: lane masks of 32 elements would spill
    // the scalar registers)
    int e_[KPW / 16], p_[KPW / 16];
#pragma unroll
    for (int t = 0; t < KPW / 16; ++t) {
      e_[t] = d.end[t];
      p_[t] = d.pos[t];
      if constexpr (KG > 1) {
#pragma unroll
        for (int x = 1; x < KG; ++x) {
          p_[t] = kg == x ? d.pos[x * (KPW / 16) + t] : p_[t];
          e_[t] = kg == x ? d.end[x * (KPW / 16) + t] : e_[t];
        }
      }
    }
    auto unseen = [&](int t, int k) {
      const int j = p_[t] + 4 * hl + k;
      const int a = min(e_[t] - 1, pos) - j;
      const int b = max(j - (pos - win + 1), sinks - 1 - j);
      return a | b;
    };
    floatx16 sa[JT];
#pragma unroll
    for (int jt = 0; jt < JT; ++jt)
#pragma unroll
      for (int i = 0; i < 16; ++i) sa[jt][i] = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int jt = 0; jt < JT; ++jt)
        sa[jt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_k(b, jt, s), qf[s], sa[jt], 0, 0, 0);
    if (!whole) {
#pragma unroll
      for (int jt = 0; jt < JT; ++jt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          sa[jt][r] = fminf(sa[jt][r], __int_as_float((unseen(2 * jt + (r >> 3), 8 * ((r >> 2) & 1) + (r & 3)) &
                                                       INT32_MIN) | 0x7f800000));
    }
    float c[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int jt = 0; jt < JT; ++jt)
#pragma unroll
      for (int r = 0; r < 16; ++r) c[r & 3] = fmaxf(c[r & 3], sa[jt][r]);
    float mx = fmaxf(fmaxf(c[0], c[1]), fmaxf(c[2], c[3]));
    {
      float a = mx, e = mx;
      swap_halves32(a, e);
      mx = fmaxf(a, e) * P.qscale;
    }
    const float mn = mx > m_run + kLazyMax ? mx : m_run;
    if (__any(mn != m_run)) {
      const float al = fast_exp2(m_run - mn);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt] *= al;
      n_run *= al;
      m_run = mn;
    }
    half8 pb[2 * JT];
#pragma unroll
    for (int jt = 0; jt < JT; ++jt)
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const half2v x = {static_cast<_Float16>(fast_exp2(__builtin_fmaf(sa[jt][r], P.qscale, -m_run))),
                          static_cast<_Float16>(fast_exp2(__builtin_fmaf(sa[jt][r + 1], P.qscale, -m_run)))};
        pb[2 * jt + r / 8][r % 8] = x[0];
        pb[2 * jt + r / 8][r % 8 + 1] = x[1];
        n_run = __builtin_amdgcn_fdot2(x, half2v{static_cast<_Float16>(1.f), static_cast<_Float16>(1.f)}, n_run, false);
      }
    if (!whole && __builtin_amdgcn_readfirstlane(s_bad[ring])) {
      // A V element that is not finite (never in ordinary data), in a unit of
      // which some queries do not see all: 0 * V would reach those too. So it
      // counts as 0, and o is NaN for the queries that see it: where the
      // product of "not finite" and "seen" is not zero.
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        floatx16 z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
        for (int p = 0; p < 2 * JT; ++p) {
          half8 x = read_v(b, p, dt), y, w;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const bool bad = !(__builtin_fabsf(static_cast<float>(x[e])) < INFINITY);
            y[e] = static_cast<_Float16>(bad ? 1.f : 0.f);
            x[e] = bad ? static_cast<_Float16>(0.f) : x[e];
            w[e] = static_cast<_Float16>(unseen(p, 8 * (e >> 2) + (e & 3)) < 0 ? 0.f : 1.f);
          }
          z = __builtin_amdgcn_mfma_f32_32x32x16_f16(y, w, z, 0, 0, 0);
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, pb[p], acc[dt], 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] = z[i] > 0.f ? __builtin_nanf("") : acc[dt][i];
      }
      return;
    }
#pragma unroll
    for (int p = 0; p < 2 * JT; ++p)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(read_v(b, p, dt), pb[p], acc[dt], 0, 0, 0);
  };

  // Unit u is computed from buffer u % 2 while unit u + 1 is on its way to the
  // registers; the barrier of a unit also tells that buffer u - 1 is free.
  if (u_begin < u_end) {
    Unit cur = unit_at(u_begin), nxt = cur;
    load(cur);
    if (tid == 0) s_bad[0] = 0;
    __syncthreads();
    for (int u = u_begin; u < u_end; ++u) {
      const int b = (u - u_begin) & 1, ring = (u - u_begin) & 3;
      store(cur, b, ring);
      if (tid == 0) s_bad[(ring + 1) & 3] = 0;  // last read three units ago
      if (u + 1 < u_end) {
        nxt = unit_at(u + 1);
        load(nxt);
      }
      __syncthreads();
      compute(cur, b, ring);
      cur = nxt;
    }
  }

  // Fold the key groups, then write o or the part's partial.
  float n_row = n_run + __shfl_xor(n_run, 32);
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
  const int rows = min(QR, n_q - q0);
  for (int i = tid; i < rows * (D / 4); i += 256) {
    const int row = i / (D / 4), ch = 4 * (i % (D / 4));
    float m = kNegBig, n = 0.f;
    floatx4 x = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < P.n_split; ++p) {
      const uint32_t at = (static_cast<uint32_t>(vt) * P.n_split + p) * kPart;
      const float* ml = P.ws + at / 4 + QR * D + 2 * row;
      const float pm = ld_dev(ml), pn = ld_dev(ml + 1);
      const float4 y = ld_dev4(rs, at + (row * D + ch) * 4u);
      const float M = fmaxf(m, pm);
      const float a = fast_exp2(m - M), c = fast_exp2(pm - M);
      n = n * a + pn * c;
      x = x * a + floatx4{y.x, y.y, y.z, y.w} * c;
      m = M;
    }
    write4(row, ch, x, 1.f / n);
  }
}

template <int S, int D, int QW, int KG, int KPW>
void launch_wp(const KwpParams& P, const WindowPrefillArgs& a, hipStream_t stream) {
  const int blocks = (a.n_q + 32 * QW - 1) / (32 * QW) * a.H * a.n_split;
  const dim3 grid(8 * ((blocks + 7) / 8));
  if (a.host_path) {
    KwpPath path;
    for (int j = 0; j < a.n_chunks; ++j) {
      path.slot[j] = a.host_path[j];
      path.start[j] = a.host_path[a.n_chunks + j];
      path.end[j] = a.host_path[2 * a.n_chunks + j];
    }
    kwp_kernel<S, D, QW, KG, KPW, true><<<grid, 256, 0, stream>>>(P, path);
  } else {
    kwp_kernel<S, D, QW, KG, KPW, false><<<grid, 256, 0, stream>>>(P, KwpNoPath{});
  }
}

template <int S, int D>
hipError_t launch_wp_tile(const KwpParams& P, const WindowPrefillArgs& a, hipStream_t stream) {
  if (a.tile_rows == 128) launch_wp<S, D, 4, 1, 64>(P, a, stream);
  else if (a.tile_rows == 64) launch_wp<S, D, 2, 2, 32>(P, a, stream);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

hipError_t launch_window_prefill(const WindowPrefillArgs& a, hipStream_t stream) {
  if (a.n_q <= 0 || a.n_chunks <= 0) return hipSuccess;
  if (a.host_path ? a.n_chunks > kPrefillInlineChunks : !a.path) return hipErrorInvalidValue;
  if (a.n_split < 1 || (a.n_split > 1 && (!a.ws || !a.cnt || a.ws_bytes > 0xFFFFFFF0ull)))
    return hipErrorInvalidValue;
  const int es = a.store == kStoreF16 ? 2 : 1;
  KwpParams P{static_cast<const _Float16*>(a.q), static_cast<_Float16*>(a.o),
              static_cast<const char*>(a.kpool), static_cast<const char*>(a.vpool), a.ss * es, a.hs * es,
              a.path, a.n_chunks, a.n_q, a.H, a.C, a.L, a.window, a.sinks, a.qscale, a.n_split, a.ws,
              a.cnt, a.cnt_shift, static_cast<uint32_t>(a.ws_bytes)};
  if (a.store == kStoreF16)
    return a.D == 128 ? launch_wp_tile<kStoreF16, 128>(P, a, stream)
                      : a.D == 64 ? launch_wp_tile<kStoreF16, 64>(P, a, stream) : hipErrorInvalidValue;
  if (a.store == kStoreKv4)
    return a.D == 128 ? launch_wp_tile<kStoreKv4, 128>(P, a, stream)
                      : a.D == 64 ? launch_wp_tile<kStoreKv4, 64>(P, a, stream) : hipErrorInvalidValue;
  return hipErrorInvalidValue;
}

}  // namespace ca
