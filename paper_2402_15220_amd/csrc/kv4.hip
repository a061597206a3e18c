// gfx950 (MI355X) K/V writes of a cache held in 4 bits (tile layout: kv4.hpp):
// new rows are quantised as they are stored, split tails are moved code by
// code. 64 tokens of 32 heads of 128 take 4.2 us, 512 6.9 (8.4 MB read, 2.2 MB
// written), 2,048 16.4: two thirds of the rate of a copy, above a launch and a
// round trip of 4 us.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "device_common.hpp"
#include "kernels.hpp"
#include "kv4.hpp"

namespace ca {
namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));

struct Kv4Jobs {
  KvJob job[kKvJobsPerLaunch];
};

// Maximum and minimum over aligned groups of LPR = 8 or 16 lanes.
template <int LPR>
__device__ __forceinline__ void group_range(float& hi, float& lo) {
  hi = fmaxf(hi, dpp<0xB1>(hi));
  lo = fminf(lo, dpp<0xB1>(lo));
  hi = fmaxf(hi, dpp<0x4E>(hi));
  lo = fminf(lo, dpp<0x4E>(lo));
  hi = fmaxf(hi, dpp<0x141>(hi));
  lo = fminf(lo, dpp<0x141>(lo));
  if constexpr (LPR >= 16) {
    hi = fmaxf(hi, dpp<0x140>(hi));
    lo = fminf(lo, dpp<0x140>(lo));
  }
}

// One block per (job, head, share of the job's 16-token blocks). Thread
// (t, e) of the block holds elements 8e .. 8e + 7 of token t; a row is LPR =
// D/8 neighbouring lanes, which find its range by DPP. K words are stored as
// they are formed; V codes are turned over in LDS, byte per code, and words
// of which the job writes only some tokens are merged with what is there. A
// job owns its slot during a launch (the host starts a new launch on a
// conflict), and inside it every 16-token block has one owner, so no two
// threads write one word.
template <int D>
__global__ __launch_bounds__(2 * D) void kv4_write_kernel(Kv4Jobs b, const _Float16* k,
                                                          const _Float16* v, char* kpool, char* vpool,
                                                          int32_t* slot_len, int H, int C, int64_t ss,
                                                          int64_t hs) {
  constexpr int LPR = D / 8;
  __shared__ uint32_t codes[16][D / 4 + 1];  // V codes of a block, a byte each
  const KvJob j = b.job[blockIdx.x];
  const int h = blockIdx.y;
  const int tid = threadIdx.x, t = tid / LPR, e = tid % LPR;
  const int code_bytes = kv4_rows(C) * (D / 2);
  if (j.kind != 2) {
    const size_t dst = static_cast<size_t>(j.dst_slot) * ss + static_cast<size_t>(h) * hs;
    const int first = j.dst_pos & ~15, end = j.dst_pos + j.n;
    for (int b0 = first + 16 * blockIdx.z; b0 < end; b0 += 16 * gridDim.z) {
      const int row = b0 + t;  // destination row
      const bool mine = row >= j.dst_pos && row < end;
      uint32_t kw = 0;            // K: eight codes, element k at nibble kv4_nibble(k)
      uint32_t lo4 = 0, hi4 = 0;  // V: eight codes, a byte each
      uint32_t kp = 0, vp = 0;  // (scale, low)
      if (j.kind == 0) {
        const size_t src = ((static_cast<size_t>(j.src) + (mine ? row - j.dst_pos : 0)) * H + h) * D + 8 * e;
        const uint4 kx = *reinterpret_cast<const uint4*>(k + src);
        const uint4 vx = *reinterpret_cast<const uint4*>(v + src);
        auto quantise = [&](const uint4& raw, float (&c)[8], uint32_t& param) {
          float x[8];
          Elem<_Float16>::unpack(raw, x);
          float hi = x[0], lo = x[0];
#pragma unroll
          for (int i = 1; i < 8; ++i) {
            hi = fmaxf(hi, x[i]);
            lo = fminf(lo, x[i]);
          }
          // NaN where an element is not finite: 0 times it
          float nan = x[0] * 0.f;
#pragma unroll
          for (int i = 1; i < 8; ++i) nan = __builtin_fmaf(x[i], 0.f, nan);
          if (!(nan == 0.f)) hi = INFINITY;  // reaches the whole row through the maximum
          group_range<LPR>(hi, lo);
          const _Float16 s16 = static_cast<_Float16>((hi - lo) / 15.f);
          const float s = static_cast<float>(s16), half = 0.5f * s;
          const float inv = s > 0.f ? 1.f / s : 0.f;
          // the nearest code: the product finds it but for a step at a border,
          // where the residual (exact: few bits) is half a step or more
          float far = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float y = x[i] - lo;
            c[i] = fminf(rintf(y * inv), 15.f);
            far = fmaxf(far, fabsf(__builtin_fmaf(-c[i], s, y)));
          }
          if (far >= half && s > 0.f) {  // decided by the residual, ties to even
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float r = __builtin_fmaf(-c[i], s, x[i] - lo);
              const bool odd = (static_cast<int>(c[i]) & 1) != 0;
              c[i] += r > half || (odd && r == half) ? 1.f : r < -half || (odd && r == -half) ? -1.f : 0.f;
              c[i] = fminf(fmaxf(c[i], 0.f), 15.f);
            }
          }
          half2v p{s16, static_cast<_Float16>(lo)};
          if (!(hi < INFINITY)) {  // a non-finite element: the row stands for NaN
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = 0.f;
            p = half2v{static_cast<_Float16>(__builtin_nanf("")), static_cast<_Float16>(__builtin_nanf(""))};
          }
          param = __builtin_bit_cast(uint32_t, p);
        };
        float c[8];
        quantise(kx, c, kp);
#pragma unroll
        for (int i = 0; i < 8; ++i) kw |= static_cast<uint32_t>(c[i]) << (4 * kv4_nibble(i));
        quantise(vx, c, vp);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          lo4 |= static_cast<uint32_t>(c[i]) << (8 * i);
          hi4 |= static_cast<uint32_t>(c[4 + i]) << (8 * i);
        }
      } else if (mine) {
        const size_t src = static_cast<size_t>(j.src) * ss + static_cast<size_t>(h) * hs;
        const int sr = j.src_pos + row - j.dst_pos;  // source row
        kw = reinterpret_cast<const uint32_t*>(kpool + src)[kv4_k_word(sr, e, D)];
        kp = reinterpret_cast<const uint32_t*>(kpool + src + code_bytes)[sr];
        vp = reinterpret_cast<const uint32_t*>(vpool + src + code_bytes)[sr];
        // elements 8e .. 8e + 7 are channels n0 .. n0 + 7 of tile 2 tp + hb
        const uint32_t* words = reinterpret_cast<const uint32_t*>(vpool + src + static_cast<size_t>(sr & ~15) * (D / 2));
        const int n0 = (8 * e) & 15, tp = e / 4, hb = (e / 2) & 1, gi = sr & 3;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t w = words[(16 * ((sr & 15) >> 2) + n0 + i) * (D / 32) + tp];
          (i < 4 ? lo4 : hi4) |= ((w >> (4 * kv4_nibble(4 * hb + gi))) & 15u) << (8 * (i & 3));
        }
      }
      if (mine) {
        reinterpret_cast<uint32_t*>(kpool + dst)[kv4_k_word(row, e, D)] = kw;
        if (e == 0) {
          reinterpret_cast<uint32_t*>(kpool + dst + code_bytes)[row] = kp;
          reinterpret_cast<uint32_t*>(vpool + dst + code_bytes)[row] = vp;
        }
      }
      codes[t][2 * e] = lo4;
      codes[t][2 * e + 1] = hi4;
      __syncthreads();
      // thread tid forms word tid of the block: group g, channel n, tiles 2 tp, 2 tp + 1
      {
        const int tp = tid % (D / 32), n = tid / (D / 32) % 16, g = tid / (D / 2);
        uint32_t word = 0, mask = 0;
        const unsigned char* byte = reinterpret_cast<const unsigned char*>(codes[4 * g]) + 32 * tp + n;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = b0 + 4 * g + i;
          const bool on = r >= j.dst_pos && r < end;
#pragma unroll
          for (int hb = 0; hb < 2; ++hb) {
            const int sh = 4 * kv4_nibble(4 * hb + i);
            word |= static_cast<uint32_t>(byte[i * (D + 4) + 16 * hb]) << sh;
            mask |= on ? 15u << sh : 0u;
          }
        }
        word &= mask;
        if (mask) {
          uint32_t* at = reinterpret_cast<uint32_t*>(vpool + dst + static_cast<size_t>(b0) * (D / 2)) + tid;
          *at = mask == 0xffffffffu ? word : (*at & ~mask) | word;
        }
      }
      __syncthreads();
    }
  }
  if (h == 0 && blockIdx.z == 0 && tid == 0) slot_len[j.dst_slot] = j.kind == 2 ? j.dst_pos : j.dst_pos + j.n;
}

}  // namespace

hipError_t launch_kv4_jobs(const KvJob* jobs, int n, int H, int D, int C, int64_t ss, int64_t hs,
                           const void* k, const void* v, void* kpool, void* vpool, int32_t* slot_len,
                           hipStream_t stream) {
  if (n <= 0) return hipSuccess;
  if (n > kKvJobsPerLaunch) return hipErrorInvalidValue;
  Kv4Jobs b{};
  int blocks = 1;  // most 16-token blocks of a job
  for (int i = 0; i < n; ++i) {
    b.job[i] = jobs[i];
    if (jobs[i].kind != 2)
      blocks = max(blocks, (jobs[i].dst_pos + jobs[i].n + 15) / 16 - jobs[i].dst_pos / 16);
  }
  const dim3 grid(n, H, blocks < 64 ? blocks : 64);
  auto go = [&](auto kernel, int threads) {
    kernel<<<grid, threads, 0, stream>>>(b, static_cast<const _Float16*>(k), static_cast<const _Float16*>(v),
                                         static_cast<char*>(kpool), static_cast<char*>(vpool), slot_len,
                                         H, C, ss, hs);
  };
  if (D == 128) go(kv4_write_kernel<128>, 256);
  else if (D == 64) go(kv4_write_kernel<64>, 128);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace ca
