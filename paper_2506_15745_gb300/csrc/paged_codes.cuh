// Rows of a paged cache as values and as codes: where a group's words lie,
// quantising and widening (declared in ipv.h, Codes).
#pragma once

#include <cuda_fp16.h>

#include "paged.cuh"

namespace ipv {

// Where a group's words lie (ipv.h, Codes): lane c of a team holds channels
// 8c..8c+7: word c at 4 bits, words 2c and 2c+1 at 8 bits.
__device__ __forceinline__ int place_u4(int c) { return 2 * (c & 3) + (c >> 2); }
__device__ __forceinline__ int place_u8(int word) { return 4 * (word & 3) + (word >> 2); }

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// 16 bytes that are read once. An ordinary, coherent load: the kernel is there
// before its predecessor, which may be writing these bytes, has ended.
__device__ __forceinline__ uint4 ld_once(const void* p) {
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
  return r;
}

// 2^23 in fp32: 2^23 + u has the integer u in its low bits.
constexpr uint32_t kTwo23 = 0x4B000000u;

__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b) {  // NaN wins
  uint32_t r;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Quantises a lane's CHUNKS chunks of 8 channels of a group (chunks c and c + 4 of
// lane c where there are two) with those of the other lanes of its team, 8 / CHUNKS
// neighbouring ones: codes in w (a word for each chunk at 4 bits, two at 8), the
// group's (step, minimum) in the return value. For whole warps.
template <int FMT, int CHUNKS>
__device__ __forceinline__ uint32_t quantise(const uint4 (&x)[CHUNKS], uint32_t (&w)[2 * CHUNKS]) {
  constexpr int kPairs = 4 * CHUNKS, kValues = 8 * CHUNKS;
  constexpr float kLevels = FMT == kU8 ? 255.0f : 15.0f;
  constexpr uint32_t kSigns = 0x80008000u;
  uint32_t xs[kPairs];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) xs[4 * i] = x[i].x, xs[4 * i + 1] = x[i].y, xs[4 * i + 2] = x[i].z, xs[4 * i + 3] = x[i].w;
  // The group's minimum, and its maximum as the minimum of the negated values, as
  // two halves of one word.
  uint32_t lo2 = xs[0], hi2 = xs[0] ^ kSigns;
#pragma unroll
  for (int i = 1; i < kPairs; ++i) lo2 = min_bf16x2(lo2, xs[i]), hi2 = min_bf16x2(hi2, xs[i] ^ kSigns);
  uint32_t ends = min_bf16x2(__byte_perm(lo2, hi2, 0x5410), __byte_perm(lo2, hi2, 0x7632));
#pragma unroll
  for (int d = 1; d < 8 / CHUNKS; d <<= 1) ends = min_bf16x2(ends, __shfl_xor_sync(0xffffffffu, ends, d));
  const float lo = lo_f(ends), hi = -hi_f(ends);
  if (!(lo >= -kLargest && hi <= kLargest)) {  // NaN too
#pragma unroll
    for (int i = 0; i < 2 * CHUNKS; ++i) w[i] = 0;
    return 0x7FFF7FFFu;  // (NaN, NaN)
  }
  const __half hm = __float2half_rd(lo);
  const float m = __half2float(hm), range = hi - m;
  // The step: range / levels rounded up to fp16. A nearest neighbour of the
  // quotient that is below it (its product with the levels is exact) moves up.
  unsigned short hs = __half_as_ushort(__float2half_rn(range * (1.0f / kLevels)));
  if (fmaf(__half2float(__ushort_as_half(hs)), kLevels, -range) < 0.0f) ++hs;
  const float s = __half2float(__ushort_as_half(hs));
  // u = rint((x - m) / s). Products with a little less and a little more than 1/s
  // (2^-20 of it, more than all roundings) enclose the quotient: where they round
  // to one integer it is the quotient's, and only where they do not is the
  // division done. Adding 1.5 * 2^23 rounds; the integer is in the sum's low bits.
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
  inv = s > 0.0f ? inv : 0.0f;
  const float less = inv * (1.0f - 0x1p-20f), more = inv * (1.0f + 0x1p-20f);
  constexpr float kRound = 12582912.0f;
  uint32_t u[kValues], apart = 0;
#pragma unroll
  for (int i = 0; i < kValues; ++i) {
    const float d = ((i & 1) ? hi_f(xs[i >> 1]) : lo_f(xs[i >> 1])) - m;
    u[i] = __float_as_uint(fmaf(d, less, kRound));
    apart |= u[i] ^ __float_as_uint(fmaf(d, more, kRound));
  }
  if (apart) {
#pragma unroll
    for (int i = 0; i < kValues; ++i)
      u[i] = __float_as_uint((((i & 1) ? hi_f(xs[i >> 1]) : lo_f(xs[i >> 1])) - m) / s + kRound);
  }
  // Words by multiplication: what stands above the codes is the same every time.
  constexpr uint32_t kBits = 0x4B400000u;  // of 1.5 * 2^23
  if (FMT == kU8) {
    constexpr uint32_t kAbove = kBits * 0x01010101u;
#pragma unroll
    for (int i = 0; i < 2 * CHUNKS; ++i)
      w[i] = u[4 * i] + u[4 * i + 1] * 0x100u + u[4 * i + 2] * 0x10000u + u[4 * i + 3] * 0x1000000u - kAbove;
  } else {
    constexpr uint32_t kAbove = kBits * 0x11111111u;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const uint32_t* v = u + 8 * i;
      w[i] = v[0] + v[1] * 0x10u + v[2] * 0x100u + v[3] * 0x1000u + v[4] * 0x10000u + v[5] * 0x100000u + v[6] * 0x1000000u +
             v[7] * 0x10000000u - kAbove;
    }
#pragma unroll
    for (int i = CHUNKS; i < 2 * CHUNKS; ++i) w[i] = 0;
  }
  return hs | (static_cast<uint32_t>(__half_as_ushort(hm)) << 16);
}

// The inverse, rounded once to bf16, or to fp16.
template <int FMT, bool F16>
__device__ __forceinline__ uint4 expand(const uint32_t (&w)[2], uint32_t par) {
  const float s = __half2float(__ushort_as_half(static_cast<unsigned short>(par & 0xFFFFu)));
  const float m = __half2float(__ushort_as_half(static_cast<unsigned short>(par >> 16)));
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (FMT == kU8) {  // a byte under 2^23's exponent
      const float u = __uint_as_float(__byte_perm(w[i >> 2], kTwo23, 0x7650 + (i & 3))) - 8388608.0f;
      f[i] = fmaf(u, s, m);
    } else {  // nibble k in its place stands for 16^k u; the step is taken 16^-k times
      const int k = i & 3;
      const float u = __uint_as_float(((i < 4 ? w[0] : w[0] >> 16) & (15u << (4 * k))) | kTwo23) - 8388608.0f;
      f[i] = fmaf(u, s * (1.0f / (1 << (4 * k))), m);
    }
  }
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (F16)
      asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(o[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
    else
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

}  // namespace ipv
