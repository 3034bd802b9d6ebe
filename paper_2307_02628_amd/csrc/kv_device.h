// Device code that all kernels of the paged cache share: the tokens of a call, pages, codes of 8 and 4 bits.
#pragma once
#include <math.h>

#include <type_traits>

#include "bf16_device.h"
#include "kv_ops.h"

namespace skd {

namespace {

enum { EL_BF16, EL_FP8, EL_FP4 };  // what a page holds: a template parameter of the kernels

struct RowTokens {
  int at, n, past;  // n 0: nothing of this row
};
__device__ inline RowTokens row_tokens(const KvTokens &tk, int r) {
  RowTokens t;
  if (tk.kind == KvTokens::RAGGED) {
    // whatever the arrays hold, no token outside of [0, tokens) is touched
    t.at = min(max(tk.first[r], 0), tk.tokens);
    t.n = min(max(tk.first[r + 1], t.at), tk.tokens) - t.at;
    t.past = tk.past[r];
  } else if (tk.kind == KvTokens::COLUMNS) {
    t.at = r;
    t.n = tk.count;
    t.past = tk.t - tk.past[r];
  } else {
    t.at = tk.first[r];
    t.n = tk.count - tk.past[r];
    t.past = 0;
  }
  // (a past beyond what the call allows for has no pages: positions stay far from the ends of 32 bits)
  t.n = t.past < 0 || t.past > tk.room ? 0 : min(t.n, tk.max_new);
  return t;
}
// The page that holds block `blk` of row r, or -1.
__device__ inline int page_of(const KvView &kv, int r, int blk) {
  const int i = blk / (kv.g.page_tokens >> 5);
  if (i >= kv.g.max_pages) return -1;
  const int page = kv.table[(long)r * kv.g.max_pages + i];
  return page >= 0 && page < kv.pages ? page : -1;
}
// Element (token, column) of a call's values.
__device__ inline long row_index(const KvRows &x, long token, int col) {
  return x.tiles ? d_act_index(token, x.at + col, x.stride) : token * x.stride + x.at + col;
}

// ------------------------------------------------------------------ e4m3 and its power of two
// An 8-bit page holds e4m3 codes, and for every token, kv head and K | V one exponent byte E + 127, E the smallest integer
// from -127 on with max|x| <= 448 * 2^E.  A power of two scales exactly, so the rounding to e4m3 (half a step: 2^-4 of a
// value, or 2^-10 * 2^E below 2^-6 * 2^E) is the only one, a value is restored exactly, and the attention can apply the
// scales to what is in fp32 anyway.  Byte 255: the token's values held an infinity or a NaN, and it reads as NaN.
// Exponent byte of a token whose largest magnitude has the fp32 bits `amax` (255: infinity or NaN among them).
__device__ inline uint32_t kv8_exponent(uint32_t amax) {
  if (amax >= 0x7f800000u) return 255;
  // amax = m * 2^k: 448 = 1.75 * 2^8, so E = k - 8, or k - 7 above 1.75
  const int e = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)(max(e, -127) + 127);
}
__device__ inline float exp2i(int e) { return ldexpf(1.0f, e); }
// four values as codes; 256 * 2^120 would be no finite value: there codes end at 240
__device__ inline uint32_t kv8_pack(float a, float b, float c, float d, uint32_t e) {
  const float inv = exp2i(127 - (int)e), top = e == 247 ? 240.f : 448.f;
  auto y = [&](float x) { return __builtin_amdgcn_fmed3f(x * inv, -top, top); };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y(a), y(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y(c), y(d), w, true);
  return (uint32_t)w;
}
// codes of eight bf16 values
__device__ inline uint2 kv8_codes(uint32x4 x, uint32_t e) {
  if (e == 255) return make_uint2(0, 0);
  return make_uint2(kv8_pack(bf2f(x[0] & 0xffffu), bf2f(x[0] >> 16), bf2f(x[1] & 0xffffu), bf2f(x[1] >> 16), e),
                    kv8_pack(bf2f(x[2] & 0xffffu), bf2f(x[2] >> 16), bf2f(x[3] & 0xffffu), bf2f(x[3] >> 16), e));
}
// largest magnitude of eight bf16 values, as fp32 bits (the bits of magnitudes are ordered as they are, NaN above infinity)
__device__ inline uint32_t max_bits(uint32x4 x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(m, max((x[i] << 16) & 0x7fffffffu, x[i] & 0x7fff0000u));
  return m;
}
template <int LANES>
__device__ inline uint32_t max_over(uint32_t m) {  // over groups of LANES neighbouring lanes
#pragma unroll
  for (int o = 1; o < LANES; o *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  return m;
}
__device__ inline uint32_t max_over_quarters(uint32_t m) {  // over the lanes 16 apart
#pragma unroll
  for (int o = 16; o < 64; o *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  return m;
}
__device__ inline float kv8_value(uint32_t word, int i, float scale) {  // byte i of a word of codes
  const float lo[2] = {__builtin_amdgcn_cvt_f32_fp8(word, 0), __builtin_amdgcn_cvt_f32_fp8(word, 1)};
  const float hi[2] = {__builtin_amdgcn_cvt_f32_fp8(word, 2), __builtin_amdgcn_cvt_f32_fp8(word, 3)};
  return (i < 2 ? lo[i & 1] : hi[i & 1]) * scale;
}
__device__ inline float kv8_scale(uint32_t e) { return e == 255 ? __uint_as_float(0x7fc00000u) : exp2i((int)e - 127); }

// ------------------------------------------------------------------ e2m1 and its power of two
// A 4-bit page holds e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), and for every token, kv head, K | V and 32
// neighbouring elements one exponent byte E + 127, E the smallest integer from -124 on with max|x| <= 6 * 2^E: the smallest code
// is then no subnormal number of bf16 or fp32, and the conversion instructions of gfx950, which take the power of two as an
// operand, are exact.  A value is off by half a step of its code: by a quarter of itself at most down to 2^E, by 2^E / 4 below.
// Byte 255: an infinity or a NaN was among the 32, which read as NaN.
// Exponent byte of 32 values whose largest magnitude has the fp32 bits `amax`.
__device__ inline uint32_t kv4_exponent(uint32_t amax) {
  if (amax >= 0x7f800000u) return 255;
  // amax = m * 2^k: 6 = 1.5 * 2^2, so E = k - 2, or k - 1 above 1.5
  const int e = (int)(amax >> 23) - 127 - 2 + ((amax & 0x7fffffu) > 0x400000u ? 1 : 0);
  return (uint32_t)(max(e, -124) + 127);
}
// The codes of two values in byte SEL of `w`; 4 * 2^126 would be no finite value: there codes end at 3
template <int SEL>
__device__ inline uint32_t kv4_pair(uint32_t w, float a, float b, uint32_t e) {
  const float scale = __uint_as_float(e << 23), top = e == 253 ? 3.0f * 0x1p126f : 3.4028235e38f;
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __builtin_amdgcn_fmed3f(a, -top, top), __builtin_amdgcn_fmed3f(b, -top, top), scale, SEL);
}
// codes of eight bf16 values, the first in the lowest bits
__device__ inline uint32_t kv4_codes(uint32x4 x, uint32_t e) {
  if (e == 255) return 0;
  uint32_t w = kv4_pair<0>(0, bf2f(x[0] & 0xffffu), bf2f(x[0] >> 16), e);
  w = kv4_pair<1>(w, bf2f(x[1] & 0xffffu), bf2f(x[1] >> 16), e);
  w = kv4_pair<2>(w, bf2f(x[2] & 0xffffu), bf2f(x[2] >> 16), e);
  return kv4_pair<3>(w, bf2f(x[3] & 0xffffu), bf2f(x[3] >> 16), e);
}
// The four codes of the low half of `w`, a byte each.
__device__ inline uint32_t spread4(uint32_t w) {
  w = (w | w << 8) & 0x00ff00ffu;
  return (w | w << 4) & 0x0f0f0f0fu;
}
// eight codes of `lo` and of `hi`, one of each in a byte
__device__ inline uint2 kv4_bytes(uint32_t lo, uint32_t hi) {
  return make_uint2(spread4(lo & 0xffffu) | spread4(hi & 0xffffu) << 4, spread4(lo >> 16) | spread4(hi >> 16) << 4);
}
// the values of a byte of codes
__device__ inline floatx2 kv4_values(uint32_t byte, uint32_t e) {
  const float scale = __uint_as_float(e == 255 ? 127u << 23 : e << 23);
  const floatx2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(byte, scale, 0);
  return e == 255 ? floatx2{__uint_as_float(0x7fc00000u), __uint_as_float(0x7fc00000u)} : x;
}

}  // namespace

}  // namespace skd
