// A step's K and V into a KV cache in 4 bits (kv_append4), and rows of it back
// in 16 bits (kv_read4).
#include <algorithm>

#include "kv4_device.cuh"

namespace rs {

namespace {

constexpr int APPEND_LOG = 5, APPEND_UNR = 1, READ_LOG = 5, READ_UNR = 2;   // of a large step: a row's threads, what each has at once

// ------------------------------------------------------------------ 16 values to codes and a scale

template <bool HALF>
__device__ __forceinline__ uint32_t max_nan2(uint32_t a, uint32_t b) {
  uint32_t r;
  if (HALF) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// The codes (8 bytes) and the scale of 16 values in 8 registers.
// scale: max |u| / 6 by the correctly rounded division, so that a quotient in the middle
// of two scales is found in the middle (max |u| has 11 significant bits, a middle 5,
// times 6: at most 8).
// codes: u / scale decides by its place among the middles m = .25, .75, 1.25, 1.75, 2.5,
// 3.5, 5, on which the even code is meant.  x * (1 / scale) is off by two roundings of
// 2^-24, which on a middle could go either way; rounded to 14 significant bits it is m again,
// and beside a middle it stays beside it: x has at most 11 significant bits, m * scale at
// most 7, so that they differ by 2^-11 of x or more.  (A division for each value instead
// would take twice the kernel's instructions.)
template <bool HALF>
__device__ __forceinline__ uint32_t quantise16(const uint32_t* x, float inv_unit, uint2& codes) {
  uint32_t m = x[0] & 0x7FFF7FFFu;
#pragma unroll
  for (int i = 1; i < 8; i++) m = max_nan2<HALF>(m, x[i] & 0x7FFF7FFFu);
  const float2 mm = unpack2<HALF>(max_nan2<HALF>(m, m >> 16));
  const float most = __fdiv_rn(__fmul_rn(mm.x, inv_unit), 6.0f);
  uint16_t s;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %1;" : "=h"(s) : "f"(most));
  const float2 sf = unpack2<true>(scales_f16(s));
  const float f = sf.x > 0.0f ? __fdiv_rn(inv_unit, sf.x) : 0.0f;
  auto quotient = [&](float v) { return __uint_as_float((__float_as_uint(__fmul_rn(v, f)) + 0x200u) & ~0x3FFu); };
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; h++) {
    float t[8];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float2 v = unpack2<HALF>(x[4 * h + i]);
      t[2 * i] = quotient(v.x);
      t[2 * i + 1] = quotient(v.y);
    }
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(w[h]) : "f"(t[0]), "f"(t[1]), "f"(t[2]), "f"(t[3]), "f"(t[4]), "f"(t[5]), "f"(t[6]), "f"(t[7]));
  }
  codes = make_uint2(w[0], w[1]);
  return s & 0xFF;
}

// A row's place in a cache, in bytes from the codes' and the scales' beginnings; the same for K and V.
struct At {
  int64_t codes, scales;
  __device__ At(const rs_kv_cache4& c, int64_t slot) {
    codes = (slot >> 4) * c.stride_block + (slot & 15) * c.stride_token;
    scales = (slot >> 4) * c.scale_block + (slot & 15) * c.scale_token;
  }
};
__device__ __forceinline__ unsigned char* bytes(void* p, int64_t at) { return static_cast<unsigned char*>(p) + at; }

template <bool WIDE>
__device__ __forceinline__ void load16(const uint16_t* src, uint32_t* u) {
  if (WIDE) {
    const uint4 a = __ldcs(reinterpret_cast<const uint4*>(src)), b = __ldcs(reinterpret_cast<const uint4*>(src) + 1);
    u[0] = a.x; u[1] = a.y; u[2] = a.z; u[3] = a.w;
    u[4] = b.x; u[5] = b.y; u[6] = b.z; u[7] = b.w;
  } else {
#pragma unroll
    for (int z = 0; z < 8; z++) u[z] = src[2 * z] | (uint32_t)src[2 * z + 1] << 16;
  }
}

// 2^team_log threads have a row: each UNR groups of 16 elements of K and of V at a time, whose
// loads are on their way together.  (Head sizes are powers of two: a group's head is a shift.)
// Bound: the loads' latency and the instructions, of which a thread's address arithmetic is half; 2 bytes an element are
// read and 9/16 written, and DRAM is busy half of the time (most of what is written stays in L2).  16 001 rows of 8 heads of
// 128 (66 MB in, 18 out): 17.5 us, 4.8 TB/s, where the copy rate would take 12.5; appended and read back 26.8 us, against 41 us where every group of K or V had a thread and a row's address of its own.
template <int D, bool HALF, bool WIDE, int UNR>
__global__ void __launch_bounds__(256) k_kv_append4(rs_kv_cache4 c, const uint16_t* k, const uint16_t* v, int64_t ts, int64_t hs,
                                                    int n_tokens, const int64_t* slots, int team_log, float inv_k, float inv_v) {
  constexpr int G = D / 16;   // groups of a head
  behind_stream();
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x, r = x >> team_log;
  if (r >= n_tokens) return;
  const int64_t slot = slots[r];
  if (slot < 0 || slot >= c.n_blocks * 16) return;
  const At at(c, slot);
  const int team = 1 << team_log, groups = c.n_kv_heads * G;
  for (int p = (int)x & (team - 1); p < groups; p += team * UNR) {
    uint32_t u[UNR][2][8];
#pragma unroll
    for (int i = 0; i < UNR; i++) {
      const int y = p + i * team, h = y / G, e = y % G;
      if (y >= groups) continue;
      const int64_t from = r * ts + h * hs + e * 16;
      load16<WIDE>(k + from, u[i][0]);
      load16<WIDE>(v + from, u[i][1]);
    }
#pragma unroll
    for (int i = 0; i < UNR; i++) {
      const int y = p + i * team, h = y / G, e = y % G;
      if (y >= groups) continue;
      const int64_t code = at.codes + h * c.stride_head + e * 8, scale = at.scales + h * c.scale_head + e;
#pragma unroll
      for (int z = 0; z < 2; z++) {
        uint2 codes;
        const uint32_t s = quantise16<HALF>(u[i][z], z ? inv_v : inv_k, codes);
        *reinterpret_cast<uint2*>(bytes(z ? c.v : c.k, code)) = codes;
        *bytes(z ? c.v_scale : c.k_scale, scale) = (unsigned char)s;
      }
    }
  }
}

// Eight elements from their codes and scale, to dst.
template <bool HALF, bool WIDE>
__device__ __forceinline__ void values8(uint32_t w, uint32_t s, float unit, uint16_t* dst) {
  uint32_t y[4];
  codes_f16(w, y);
  const uint32_t ss = scales_f16(s | s << 8);
#pragma unroll
  for (int z = 0; z < 4; z++) {
    float2 f = unpack2<true>(mul_f16x2(y[z], ss));
    f.x = __fmul_rn(f.x, unit);
    f.y = __fmul_rn(f.y, unit);
    if (HALF) {   // (the largest numbers, not infinity; NaN stays)
      asm("{\n\tmin.NaN.f32 %0, %0, 0f477FE000;\n\tmax.NaN.f32 %0, %0, 0fC77FE000;\n\t}" : "+f"(f.x));
      asm("{\n\tmin.NaN.f32 %0, %0, 0f477FE000;\n\tmax.NaN.f32 %0, %0, 0fC77FE000;\n\t}" : "+f"(f.y));
      asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y[z]) : "f"(f.y), "f"(f.x));
    } else {
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y[z]) : "f"(f.y), "f"(f.x));
    }
  }
  if (WIDE) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(y[0], y[1], y[2], y[3]);
  } else {
#pragma unroll
    for (int z = 0; z < 4; z++) {
      dst[2 * z] = (uint16_t)y[z];
      dst[2 * z + 1] = (uint16_t)(y[z] >> 16);
    }
  }
}

// 2^team_log threads have a row: each UNR pieces of eight elements of K and of V at a time,
// whose loads are on their way together.
// Bound: the instructions (two conversions, a product and a rounding a pair) and the scales' partial sectors beside 9/16 byte
// an element read and 2 written; DRAM is busy 42% of the time, as half of what is written stays in L2.  60 000 rows of 8 heads of 64 (35 MB in, 123 out): 27.5 us,
// 5.75 TB/s (UNR 1: 30.0 us, 4: 32.1 us; a piece a thread with an address of its own: 51 us).
template <int D, bool HALF, bool WIDE, int UNR>
__global__ void __launch_bounds__(256) k_kv_read4(rs_kv_cache4 c, uint16_t* k, uint16_t* v, int64_t ts, int64_t hs, int n_tokens,
                                                  const int64_t* slots, int team_log) {
  constexpr int G = D / 8;   // pieces of a head
  behind_stream();
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x, r = x >> team_log;
  if (r >= n_tokens) return;
  const int64_t slot = slots[r];
  if (slot < 0 || slot >= c.n_blocks * 16) return;
  const At at(c, slot);
  const int team = 1 << team_log, pieces = c.n_kv_heads * G;
  for (int p = (int)x & (team - 1); p < pieces; p += team * UNR) {
    uint32_t w[UNR][2], s[UNR][2];
#pragma unroll
    for (int i = 0; i < UNR; i++) {
      const int y = p + i * team, h = y / G, e = y % G;
      if (y >= pieces) continue;
      const int64_t code = at.codes + h * c.stride_head + e * 4, scale = at.scales + h * c.scale_head + (e >> 1);
#pragma unroll
      for (int z = 0; z < 2; z++) {
        w[i][z] = __ldcs(reinterpret_cast<const uint32_t*>(bytes(z ? c.v : c.k, code)));
        s[i][z] = *bytes(z ? c.v_scale : c.k_scale, scale);
      }
    }
#pragma unroll
    for (int i = 0; i < UNR; i++) {
      const int y = p + i * team, h = y / G, e = y % G;
      if (y >= pieces) continue;
      const int64_t to = r * ts + h * hs + e * 8;
      values8<HALF, WIDE>(w[i][0], s[i][0], c.k_unit, k + to);
      values8<HALF, WIDE>(w[i][1], s[i][1], c.v_unit, v + to);
    }
  }
}

// A kernel for a head size, a type and rows that are aligned or not.
#define KV4_PICK(NAME, UNR) \
  (c.head_dim == 128 ? half ? wide ? NAME<128, true, true, UNR> : NAME<128, true, false, UNR>   \
                            : wide ? NAME<128, false, true, UNR> : NAME<128, false, false, UNR> \
                     : half ? wide ? NAME<64, true, true, UNR> : NAME<64, true, false, UNR>     \
                            : wide ? NAME<64, false, true, UNR> : NAME<64, false, false, UNR>)

// Threads of a row (their logarithm): as many as it has pieces, at most `most` of them.
int team_of(int pieces, int most) {
  int log = 0;
  while ((1 << log) < pieces && log < most) log++;
  return log;
}

bool wide_rows(const void* k, const void* v, int64_t ts, int64_t hs) {
  return ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15) == 0 && ts % 8 == 0 && hs % 8 == 0;
}

}  // namespace

// A small step has a piece of K and V a thread; a large one more, for which the row's address is found once.
cudaError_t launch_kv_append4(const rs_kv_cache4& c, bool half, const void* k, const void* v, int64_t ts, int64_t hs,
                              int n_tokens, const int64_t* slots, int sms, cudaStream_t st) {
  const bool wide = wide_rows(k, v, ts, hs);
  const int groups = c.n_kv_heads * (c.head_dim / 16);
  const bool small = (int64_t)n_tokens * groups <= (int64_t)sms * 1024;
  const int log = team_of(groups, small ? 8 : APPEND_LOG);
  const int64_t threads = (int64_t)n_tokens << log;
  return launch_behind(small ? KV4_PICK(k_kv_append4, 1) : KV4_PICK(k_kv_append4, APPEND_UNR), (unsigned)((threads + 255) / 256), 256, 0, st, c,
                       static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), ts, hs, n_tokens, slots, log, 1.0f / c.k_unit,
                       1.0f / c.v_unit);
}

cudaError_t launch_kv_read4(const rs_kv_cache4& c, bool half, void* k, void* v, int64_t ts, int64_t hs, int n_tokens,
                            const int64_t* slots, int sms, cudaStream_t st) {
  const bool wide = wide_rows(k, v, ts, hs);
  const int pieces = c.n_kv_heads * (c.head_dim / 8);
  const bool small = (int64_t)n_tokens * pieces <= (int64_t)sms * 1024;
  const int log = team_of(pieces, small ? 8 : READ_LOG);
  const int64_t threads = (int64_t)n_tokens << log;
  return launch_behind(small ? KV4_PICK(k_kv_read4, 1) : KV4_PICK(k_kv_read4, READ_UNR), (unsigned)((threads + 255) / 256), 256, 0, st, c,
                       static_cast<uint16_t*>(k), static_cast<uint16_t*>(v), ts, hs, n_tokens, slots, log);
}

}  // namespace rs
