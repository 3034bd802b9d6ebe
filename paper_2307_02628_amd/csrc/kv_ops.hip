// The paged cache as an operator: new tokens of ragged rows filed into bf16 or 8-bit pages, read back, and attended to.
//
// An 8-bit page holds e4m3 codes, and for every token, kv head and K | V one exponent byte E + 127, E the smallest integer
// from -127 on with max|x| <= 448 * 2^E.  A power of two scales exactly, so the rounding to e4m3 (half a step: 2^-4 of a
// value, or 2^-10 * 2^E below 2^-6 * 2^E) is the only one, a value is restored exactly, and the attention can apply the
// scales to what is in fp32 anyway.  Byte 255: the token's values held an infinity or a NaN, and it reads as NaN.
#include "kv_ops.h"

#include <math.h>

#include <type_traits>

#include "bf16_device.h"

namespace skd {

namespace {

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
__device__ inline float kv8_value(uint32_t word, int i, float scale) {  // byte i of a word of codes
  const float lo[2] = {__builtin_amdgcn_cvt_f32_fp8(word, 0), __builtin_amdgcn_cvt_f32_fp8(word, 1)};
  const float hi[2] = {__builtin_amdgcn_cvt_f32_fp8(word, 2), __builtin_amdgcn_cvt_f32_fp8(word, 3)};
  return (i < 2 ? lo[i & 1] : hi[i & 1]) * scale;
}
__device__ inline float kv8_scale(uint32_t e) { return e == 255 ? __uint_as_float(0x7fc00000u) : exp2i((int)e - 127); }

// ------------------------------------------------------------------ filing
// A workgroup files the tokens of one row and kv head that lie in one 32-key block.  DH / 8 lanes take a token: 16 bytes of
// K and of V each, largest magnitudes over them; K goes to the page as it is, V^T by way of LDS, where the four keys that
// are neighbours in the page are gathered.  Bound by the bytes of large calls; a block's codes leave as whole words where the
// row fills them, and element by element at the ends of its tokens, so that what other tokens hold there stays.
template <int DH, bool FP8>
__global__ __launch_bounds__(256) void k_kv_append(KvView kv, KvTokens tk, KvRows k, KvRows v, int blocks, uint32_t from) {
  constexpr int LPT = DH / 8, TPP = 256 / LPT;  // lanes a token, tokens a pass
  typedef typename std::conditional<FP8, uint8_t, uint16_t>::type code_t;
  __shared__ __align__(16) code_t sv[32][DH + 8];
  const uint32_t id = from + blockIdx.x;
  const int blk_i = id % blocks, h = id / blocks % kv.g.H, r = id / blocks / kv.g.H;
  const RowTokens t = row_tokens(tk, r);
  const int blk = (t.past >> 5) + blk_i, lo = max(t.past, blk * 32), hi = min(t.past + t.n, blk * 32 + 32);
  if (t.n <= 0 || lo >= hi) return;
  const int page = page_of(kv, r, blk);
  if (page < 0) return;
  unsigned char *pg = kv.pool + (long)page * kv.page_bytes;
  const int slot0 = (blk % (kv.g.page_tokens >> 5)) * 32;
  const int e = (threadIdx.x % LPT) * 8;
  for (int key = threadIdx.x / LPT; key < 32; key += TPP) {
    const int pos = blk * 32 + key;
    if (pos < lo || pos >= hi) continue;
    const long token = t.at + (long)(pos - t.past) * tk.step;
    const uint32x4 kx = *(const uint32x4 *)((const bf16_t *)k.p + row_index(k, token, h * DH + e));
    const uint32x4 vx = *(const uint32x4 *)((const bf16_t *)v.p + row_index(v, token, h * DH + e));
    if constexpr (FP8) {
      const uint32_t ke = kv8_exponent(max_over<LPT>(max_bits(kx))), ve = kv8_exponent(max_over<LPT>(max_bits(vx)));
      *(uint2 *)(pg + kv8_k_off(h, slot0 + key, e, kv.g)) = kv8_codes(kx, ke);
      *(uint2 *)&sv[key][e] = kv8_codes(vx, ve);
      if (e == 0) {
        pg[kv8_exp_off(h, slot0 + key, 0, kv.g)] = (unsigned char)ke;
        pg[kv8_exp_off(h, slot0 + key, 1, kv.g)] = (unsigned char)ve;
      }
    } else {
      *(uint32x4 *)((bf16_t *)pg + kv_k_off(h, slot0 + key, e, kv.g)) = kx;
      *(uint32x4 *)&sv[key][e] = vx;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 8 * DH; i += 256) {  // element el, four keys from key0 on
    const int el = i % DH, key0 = i / DH * 4;
    const int first = blk * 32 + key0;
    code_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = sv[key0 + j][el];
    code_t *to = FP8 ? (code_t *)(pg + kv8_v_off(h, slot0 + key0, el, kv.g)) : (code_t *)pg + kv_v_off(h, slot0 + key0, el, kv.g);
    if (first >= lo && first + 4 <= hi) {
      if constexpr (FP8) *(uint32_t *)to = c[0] | (uint32_t)c[1] << 8 | (uint32_t)c[2] << 16 | (uint32_t)c[3] << 24;
      else *(uint2 *)to = make_uint2(c[0] | (uint32_t)c[1] << 16, c[2] | (uint32_t)c[3] << 16);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (first + j >= lo && first + j < hi) to[j] = c[j];
    }
  }
}

// A few tokens a row (decode steps, drafts): DH / 8 lanes take the key or the value of one token and head.  Hardly any bytes: a
// chain of three round trips (the row's place, its page, the values), so every token has lanes of its own and nothing is shared.
// The tokens of a step for 128 rows of 32 heads of 128, 8 bits: 6.4 us instead of 14.5 by blocks (7.7 with every lane storing the
// eight values that it has read: eight lines of the page for each store of a token and head, now two).
template <int DH, bool FP8>
__global__ __launch_bounds__(256) void k_kv_append_few(KvView kv, KvTokens tk, KvRows k, KvRows v) {
  constexpr int LPT = DH / 8, PER = 256 / LPT;
  const int H = kv.g.H, e = threadIdx.x % LPT * 8;
  const uint32_t unit = blockIdx.x * PER + threadIdx.x / LPT, side = unit / H, token = side / 2;  // [row][token][k | v][head]
  const int h = (int)(unit - side * H), is_v = (int)(side & 1), i = (int)(token % tk.max_new), r = (int)(token / tk.max_new);
  if (r >= kv.rows) return;
  const RowTokens t = row_tokens(tk, r);
  if (i >= t.n) return;
  const KvRows &from = is_v ? v : k;
  const uint32x4 x = *(const uint32x4 *)((const bf16_t *)from.p + row_index(from, t.at + (long)i * tk.step, h * DH + e));
  const int pos = t.past + i, page = page_of(kv, r, pos >> 5);
  if (page < 0) return;
  unsigned char *pg = kv.pool + (long)page * kv.page_bytes;
  const int slot = pos % kv.g.page_tokens;
  // A value's elements lie 16 bytes apart: in one store the lanes take neighbouring ones, through their own wave's part of LDS.
  __shared__ uint32x4 line[256];
  unsigned char *own = (unsigned char *)(line + threadIdx.x / LPT * LPT);
  const int l = threadIdx.x % LPT;
  if constexpr (FP8) {
    const uint32_t ex = kv8_exponent(max_over<LPT>(max_bits(x)));
    const uint2 c = kv8_codes(x, ex);
    if (e == 0) pg[kv8_exp_off(h, slot, is_v, kv.g)] = (unsigned char)ex;
    if (is_v) {
      *(uint2 *)(own + 8 * l) = c;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int j = 0; j < 8; ++j) pg[kv8_v_off(h, slot, l + LPT * j, kv.g)] = own[l + LPT * j];
    } else {
      *(uint2 *)(pg + kv8_k_off(h, slot, e, kv.g)) = c;
    }
  } else if (is_v) {
    *(uint32x4 *)(own + 16 * l) = x;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int j = 0; j < 8; ++j) ((bf16_t *)pg)[kv_v_off(h, slot, l + LPT * j, kv.g)] = ((bf16_t *)own)[l + LPT * j];
  } else {
    *(uint32x4 *)((bf16_t *)pg + kv_k_off(h, slot, e, kv.g)) = x;
  }
}

// ------------------------------------------------------------------ reading back
// A lane takes two pieces of four elements of a token: neighbouring ones where rows are bf16, and where they are fp32 such that
// the lanes' 16-byte stores lie side by side (stores that fill every other 16 bytes of a line, 8 rows of 2048 positions: 196 us
// instead of 108).
template <typename OUT, int DH>
__device__ inline int piece_of(int l, int p) { return sizeof(OUT) == 4 ? p * (DH / 2) + 4 * l : 8 * l + 4 * p; }
template <typename OUT, int DH>
__device__ inline void store_pieces(OUT *row, int l, const float (&x)[8]) {  // (streamed: nothing here reads it again)
  if constexpr (sizeof(OUT) == 4) {
#pragma unroll
    for (int p = 0; p < 2; ++p) __builtin_nontemporal_store(floatx4{x[4 * p], x[4 * p + 1], x[4 * p + 2], x[4 * p + 3]}, (floatx4 *)(row + piece_of<OUT, DH>(l, p)));
  } else {
    __builtin_nontemporal_store(uint32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])}, (uint32x4 *)(row + 8 * l));
  }
}
__device__ inline void decode4(uint32_t w, uint32_t ex, float *x) {
  const float sc = kv8_scale(ex);
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = kv8_value(w, j, sc);
}
__device__ inline void decode4(uint2 w, float *x) {
  x[0] = bf2f(w.x & 0xffffu);
  x[1] = bf2f(w.x >> 16);
  x[2] = bf2f(w.y & 0xffffu);
  x[3] = bf2f(w.y >> 16);
}
// The few tokens of k_kv_append_few the other way.
template <int DH, bool FP8, typename OUT>
__global__ __launch_bounds__(256) void k_kv_read_few(KvView kv, KvTokens tk, KvRows k, KvRows v) {
  constexpr int LPT = DH / 8, PER = 256 / LPT;
  const int H = kv.g.H, l = threadIdx.x % LPT;
  const uint32_t unit = blockIdx.x * PER + threadIdx.x / LPT, side = unit / H, token = side / 2;
  const int h = (int)(unit - side * H), is_v = (int)(side & 1), i = (int)(token % tk.max_new), r = (int)(token / tk.max_new);
  if (r >= kv.rows) return;
  const RowTokens t = row_tokens(tk, r);
  if (i >= t.n) return;
  const int pos = t.past + i, page = page_of(kv, r, pos >> 5);
  if (page < 0) return;
  const unsigned char *pg = kv.pool + (long)page * kv.page_bytes;
  const int slot = pos % kv.g.page_tokens;
  float x[8];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int e = piece_of<OUT, DH>(l, p);
    if constexpr (FP8) {
      uint32_t c = 0;
      if (is_v) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c |= (uint32_t)pg[kv8_v_off(h, slot, e + j, kv.g)] << (8 * j);
      } else {
        c = *(const uint32_t *)(pg + kv8_k_off(h, slot, e, kv.g));
      }
      decode4(c, pg[kv8_exp_off(h, slot, is_v, kv.g)], x + 4 * p);
    } else if (is_v) {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * p + j] = bf2f(((const bf16_t *)pg)[kv_v_off(h, slot, e + j, kv.g)]);
    } else {
      decode4(*(const uint2 *)((const bf16_t *)pg + kv_k_off(h, slot, e, kv.g)), x + 4 * p);
    }
  }
  const KvRows &to = is_v ? v : k;
  store_pieces<OUT, DH>((OUT *)to.p + row_index(to, t.at + (long)i * tk.step, h * DH), l, x);
}

// As above, the other way: a workgroup reads the tokens of a row and kv head that lie in one block.  Bound by the fp32 rows
// that it writes.
template <int DH, bool FP8, typename OUT>
__global__ __launch_bounds__(256) void k_kv_read(KvView kv, KvTokens tk, KvRows k, KvRows v, int blocks, uint32_t from) {
  constexpr int LPT = DH / 8, TPP = 256 / LPT;
  __shared__ float sv[32][DH + 1];
  const uint32_t id = from + blockIdx.x;
  const int blk_i = id % blocks, h = id / blocks % kv.g.H, r = id / blocks / kv.g.H;
  const RowTokens t = row_tokens(tk, r);
  const int blk = (t.past >> 5) + blk_i, lo = max(t.past, blk * 32), hi = min(t.past + t.n, blk * 32 + 32);
  if (t.n <= 0 || lo >= hi) return;
  const int page = page_of(kv, r, blk);
  if (page < 0) return;
  const unsigned char *pg = kv.pool + (long)page * kv.page_bytes;
  const int slot0 = (blk % (kv.g.page_tokens >> 5)) * 32, l = threadIdx.x % LPT;
  // keys are requested ahead of the values' way through LDS
  typename std::conditional<FP8, uint32_t, uint2>::type kw[32 / TPP][2];
  uint32_t ke[32 / TPP];
#pragma unroll
  for (int i = 0; i < 32 / TPP; ++i) {
    const int key = threadIdx.x / LPT + i * TPP;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int e = piece_of<OUT, DH>(l, p);
      if constexpr (FP8) kw[i][p] = *(const uint32_t *)(pg + kv8_k_off(h, slot0 + key, e, kv.g));
      else kw[i][p] = *(const uint2 *)((const bf16_t *)pg + kv_k_off(h, slot0 + key, e, kv.g));
    }
    ke[i] = FP8 ? pg[kv8_exp_off(h, slot0 + key, 0, kv.g)] : 0;
  }
  for (int i = threadIdx.x; i < 8 * DH; i += 256) {
    const int el = i % DH, key0 = i / DH * 4;
    if constexpr (FP8) {
      const uint32_t w = *(const uint32_t *)(pg + kv8_v_off(h, slot0 + key0, el, kv.g));
      const uint32_t x = *(const uint32_t *)(pg + kv8_exp_off(h, slot0 + key0, 1, kv.g));
#pragma unroll
      for (int j = 0; j < 4; ++j) sv[key0 + j][el] = kv8_value(w, j, kv8_scale(x >> (8 * j) & 255u));
    } else {
      const uint2 w = *(const uint2 *)((const bf16_t *)pg + kv_v_off(h, slot0 + key0, el, kv.g));
      sv[key0][el] = bf2f(w.x & 0xffffu);
      sv[key0 + 1][el] = bf2f(w.x >> 16);
      sv[key0 + 2][el] = bf2f(w.y & 0xffffu);
      sv[key0 + 3][el] = bf2f(w.y >> 16);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 32 / TPP; ++i) {
    const int key = threadIdx.x / LPT + i * TPP, pos = blk * 32 + key;
    if (pos < lo || pos >= hi) continue;
    const long token = t.at + (long)(pos - t.past) * tk.step;
    float kx[8], vx[8];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      if constexpr (FP8) decode4(kw[i][p], ke[i], kx + 4 * p);
      else decode4(kw[i][p], kx + 4 * p);
#pragma unroll
      for (int j = 0; j < 4; ++j) vx[4 * p + j] = sv[key][piece_of<OUT, DH>(l, p) + j];
    }
    store_pieces<OUT, DH>((OUT *)k.p + row_index(k, token, h * DH), l, kx);
    store_pieces<OUT, DH>((OUT *)v.p + row_index(v, token, h * DH), l, vx);
  }
}

// ------------------------------------------------------------------ attention
// A query tile is 16 of the R = new * group queries of a row and kv head, in the order (token, head of the group): the 16
// columns of the matrix instructions.  The softmax works in units of log2 against a reference that is raised only by more
// than 8 (weights up to 2^8), denominators come from the matrix cores (a row of ones) and are sums of the rounded weights.
//
// Query i of a row sees positions up to past + i.  In blocks that reach beyond what a tile's first query sees scores are masked by
// selection.  Since 0 * infinity is not 0, that leaves values: beyond the row's last position they are cleared (a page may hold
// anything there); an infinity or NaN that only later queries see makes sums that are not finite, and a wave that ends with such
// sums forms them once more (sums_again), without such values, which are added for the queries that see them.  8-bit values are
// finite, what is not is in their scales, which are selected with the weights.
// The powers of two of 8-bit keys are an operand of the conversion to bf16, those of values multiply the weights: both exact.

// bf16x8 of two words of codes, times the power of two whose exponent byte is `e` (255: NaN)
__device__ inline bf16x8 widen(uint32_t a, uint32_t b, uint32_t e) {
  const float scale = __uint_as_float(e << 23);
  const bf16x2 x[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true)};
  return bf16x8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
}
// fp32 of an exponent byte: byte 0, 2^-127, is a subnormal.  (Weights times such a factor are rounded to multiples of 2^-133, the
// smallest bf16: a value of exponent 0 is off by 2^-134 * 448 = 2^-125 for each key, beside a sum of weights of at least 1.)
__device__ inline float kv8_factor(uint32_t word, int i) {
  const uint32_t e = word >> (8 * i) & 255u;
  return __uint_as_float(e == 255 ? 0x7fc00000u : max(e << 23, 0x00400000u));
}
__device__ inline bf16x8 pack8(const float (&p)[8]) {
  return __builtin_bit_cast(bf16x8, (uint32x4{pack2(p[0], p[1]), pack2(p[2], p[3]), pack2(p[4], p[5]), pack2(p[6], p[7])}));
}
__device__ inline bf16x8 all_ones() {
  bf16x8 x;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (__bf16)1.0f;
  return x;
}
// position (of a block) of element j of a lane's eight
__device__ inline int block_pos(int j, int grp) { return 16 * (j >> 2) + 4 * grp + (j & 3); }

// SHARES: a lane adds up the weights of its own positions (one_sum joins them) instead of the matrix cores all of them, which
// takes 7 registers more: at 4 waves a SIMD they are not there.
template <int DH, bool SHARES>
struct QueryTile {
  floatx4 O[DH / 16], L;  // O[m][i]: element 16 m + 4 (lane / 16) + i of the lane's query (lane % 16)
  float m_ref;
  __device__ void clear() {
    m_ref = -3.0e38f;  // below every score: no weight has been taken
    L = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int m = 0; m < DH / 16; ++m) O[m] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ void relative(const floatx4 (&S)[2], float c, float (&p)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = __builtin_fmaf(S[j >> 2][j & 3], c, -m_ref);
  }
  __device__ static float most(const float (&x)[8]) {
    return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
  }
  __device__ void raise(float bm) {  // the reference to bm, this lane's largest score, if that is above it
    bm = fmaxf(bm, __shfl_xor(bm, 16));  // lanes 16 and 32 apart hold the same query
    bm = fmaxf(bm, __shfl_xor(bm, 32));
    const float m_new = fmaxf(m_ref, bm), alpha = m_new == m_ref ? 1.0f : __builtin_amdgcn_exp2f(m_ref - m_new);
    m_ref = m_new;
    if constexpr (SHARES) L[0] *= alpha;
    else L *= alpha;
#pragma unroll
    for (int m = 0; m < DH / 16; ++m) O[m] *= alpha;
  }
  // The weights of a block from its scores S[tl][i] (position 16 tl + 4 grp + i), rounded to bf16 for the products (by 2^-8 of
  // a weight at most; the denominator adds the rounded ones).  masked: positions from `limit` of the block on have none.
  template <bool FP8>
  __device__ bf16x8 weights(bool masked, floatx4 (&S)[2], float c, int limit, int grp, const float (&vs)[8]) {
    if (masked) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (block_pos(j, 0) >= limit - 4 * grp) S[j >> 2][j & 3] = -INFINITY;
    }
    float p[8];
    relative(S, c, p);
    if (__any(most(p) > 8.0f)) {
      const float x[8] = {S[0][0], S[0][1], S[0][2], S[0][3], S[1][0], S[1][1], S[1][2], S[1][3]};
      raise(most(x) * c);
      relative(S, c, p);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(p[j]);
    bf16x8 pv = pack8(p);
    if constexpr (SHARES) {
#pragma unroll
      for (int j = 0; j < 8; ++j) L[0] += (float)pv[j];
    } else {
      L = __builtin_amdgcn_mfma_f32_16x16x32_bf16(all_ones(), pv, L, 0, 0, 0);
    }
    if constexpr (FP8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] *= vs[j];
      if (masked) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (block_pos(j, 0) >= limit - 4 * grp) p[j] = 0.f;  // (a power of two there may be NaN)
      }
      pv = pack8(p);
    }
    return pv;
  }
  __device__ void one_sum() {
    if constexpr (SHARES) {
      L[0] += __shfl_xor(L[0], 16);
      L[0] += __shfl_xor(L[0], 32);
    }
  }
};
// 1 at positions below `limit`
__device__ inline bf16x8 visible(int limit, int grp) {
  bf16x8 v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (__bf16)(block_pos(j, grp) < limit ? 1.0f : 0.0f);
  return v;
}
// masks of a lane's eight bf16 values: positions below `valid`
struct Keep {
  uint32_t w[4];
  __device__ Keep(int valid, int grp) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = (block_pos(2 * i, grp) < valid ? 0xffffu : 0u) | (block_pos(2 * i + 1, grp) < valid ? 0xffff0000u : 0u);
  }
  __device__ void bf16(uint32x4 &v) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] &= w[i];
  }
  __device__ uint32_t codes(int half) const { return __builtin_amdgcn_perm(w[2 * half + 1], w[2 * half], 0x06040200); }
};
__device__ inline void drop_odd(uint32x4 &v) {  // infinities and NaNs to 0
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t odd = ((v[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
    v[i] &= ~((odd >> 15) * 0xffffu);
  }
}
// Adds to the sums of a tile what the infinities and NaNs of a value fragment are for the queries that see them.
__device__ inline void add_odd(floatx4 &O, const uint32x4 &v, bf16x8 vis) {
  uint32x4 up, down;  // 1 where it is +infinity or NaN, -infinity or NaN
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t u = 0, d = 0;
#pragma unroll
    for (int s = 0; s < 32; s += 16) {
      const uint32_t x = v[i] >> s & 0xffffu;
      if ((x & 0x7f80u) == 0x7f80u) {
        if (x != 0xff80u) u |= 0x3f80u << s;
        if (x != 0x7f80u) d |= 0x3f80u << s;
      }
    }
    up[i] = u;
    down[i] = d;
  }
  const floatx4 z = floatx4{0.f, 0.f, 0.f, 0.f};
  const floatx4 u = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, up), vis, z, 0, 0, 0);
  const floatx4 d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, down), vis, z, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (u[i] > 0.f) O[i] += INFINITY;
    if (d[i] > 0.f) O[i] -= INFINITY;
  }
}

// What a workgroup computes: NQ queries from q0 on of a row and kv head, on one share of their keys.
struct Share {
  RowTokens t;
  int r, h, R, q0;
  int held;        // positions that the cache holds
  int lo, hi;      // blocks
  bool any;
  // Workgroup: [tile, the longest first][row and kv head], `pairs` places for the latter.  Tiles of many queries: of 16 rows and
  // heads of an XCD at a time, so that fewer pages pass through its L2 at once, and the next ones fill the gaps (all of them, 16,
  // 1 at a time, us: 8 prompts of 2048, 32 heads of 128, bf16 428, 411, 440; 512 tokens behind 2048 203, 192, 194; 8 bits 386,
  // 380, 440 and 196, 192, 206; 32 prompts of 512, heads of 64, 8 bits 88, 93, 122).
  static constexpr int TOGETHER = 16;
  template <int NQ>
  __device__ static Share of(const KvAttend &a, int pairs, bool files) {
    Share s;
    const int H = a.kv.g.H, tiles = gridDim.x / pairs, id = blockIdx.x;
    int pair = id % pairs, tile = id / pairs;
    if (NQ == 128 && pairs % 8 == 0) {
      const int at = id / 8, g = at / (tiles * TOGETHER), in = at - g * tiles * TOGETHER, n = min(TOGETHER, pairs / 8 - g * TOGETHER);
      pair = (g * TOGETHER + in % n) * 8 + id % 8;
      tile = in / n;
    }
    const int ri = min(pair / H, a.kv.rows - 1);
    s.h = pair % H;
    s.r = a.order ? a.order[ri] : ri;
    s.t = row_tokens(a.tk, s.r);
    s.R = pair < H * a.kv.rows ? s.t.n * a.group : 0;
    s.q0 = (tiles - 1 - tile) * NQ;
    s.any = s.q0 < s.R;
    s.held = s.t.past + (files ? 0 : s.t.n);
    const int nblk = (min(s.seen(a, min(s.q0 + NQ, s.R) - 1), s.held) + 31) >> 5, per = (nblk + a.splits - 1) / a.splits;
    s.lo = (int)blockIdx.y * per;
    s.hi = min(s.lo + per, nblk);
    return s;
  }
  __device__ int seen(const KvAttend &a, int q) const { return t.past + q / a.group + 1; }  // positions that query q sees
  __device__ long token(const KvAttend &a, int q) const { return t.at + (long)(q / a.group) * a.tk.step; }
  __device__ int head(const KvAttend &a, int q) const { return h * a.group + q % a.group; }
};
template <int DH>
__device__ inline float *part_of(const KvAttend &a, int split, long token, int head) {
  return a.part + (((long)split * a.tk.tokens + token) * a.heads + head) * (DH + 2);
}
template <int DH>
__device__ inline void load_queries(const KvAttend &a, const Share &s, int q, int grp, bf16x8 (&qf)[DH / 32]) {
#pragma unroll
  for (int c = 0; c < DH / 32; ++c) {
    qf[c] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
    if (q < s.R) qf[c] = *(const bf16x8 *)((const bf16_t *)a.q.p + row_index(a.q, s.token(a, q), s.head(a, q) * DH + 32 * c + 8 * grp));
  }
}

// Whether a wave's sums hold an infinity or NaN.
template <int DH, int NT, typename Tile>
__device__ inline bool not_finite_(const Tile (&tile)[NT]) {
  float x = 0.f;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int m = 0; m < DH / 16; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) x = __builtin_fmaf(tile[t].O[m][i], 0.f, x);
  return __any(x != x);
}
template <int DH, typename Tile, int NT>
__device__ inline bool not_finite(const Tile (&tile)[NT]) { return not_finite_<DH, NT, Tile>(tile); }
// The numerators of a wave's tiles again, over blocks first, first + step, ... below end of bf16 pages, against the references
// that the wave has arrived at: values without their infinities and NaNs, which are then added.
template <int DH, typename Tile, int NT>
__device__ __forceinline__ void sums_again(const KvAttend &a, const Share &s, int q0, const int (&limit)[NT], int first, int step, int end, Tile (&tile)[NT]) {
  constexpr int QC = DH / 32, VM = DH / 16;
  const int lane = threadIdx.x & 63, grp = lane >> 4, col = lane & 15, bpp = a.kv.g.page_tokens >> 5;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int m = 0; m < VM; ++m) tile[t].O[m] = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int blk = first; blk < end; blk += step) {
    const int page = page_of(a.kv, s.r, blk);
    if (page < 0) continue;
    const uint32x4 *src = (const uint32x4 *)(a.kv.pool + (long)page * a.kv.page_bytes + ((long)s.h * bpp + blk % bpp) * (128 * DH)) + lane;
    const Keep keep(s.held - blk * 32, grp);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      bf16x8 qf[QC];
      load_queries<DH>(a, s, q0 + 16 * t + col, grp, qf);
      const int lim = limit[t] - blk * 32;
      floatx4 S[2];
#pragma unroll
      for (int tl = 0; tl < 2; ++tl) {
        S[tl] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < QC; ++c) S[tl] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, src[(tl * QC + c) * 64]), qf[c], S[tl], 0, 0, 0);
      }
      float p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        p[j] = block_pos(j, grp) < lim ? __builtin_amdgcn_exp2f(__builtin_fmaf(S[j >> 2][j & 3], a.c, -tile[t].m_ref)) : 0.f;
      const bf16x8 pv = pack8(p), vis = visible(lim, grp);
#pragma unroll
      for (int m = 0; m < VM; ++m) {
        uint32x4 v = src[4 * DH + m * 64], w;
        keep.bf16(v);
        w = v;
        drop_odd(w);
        tile[t].O[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), pv, tile[t].O[m], 0, 0, 0);
        add_odd(tile[t].O[m], v, vis);
        __builtin_amdgcn_sched_barrier(0);  // (one fragment after the other: side by side they take more registers than there are)
      }
    }
  }
}

// Few queries (one or two tiles): a workgroup is NW waves on NT tiles, and a wave takes every NW-th 32-key block, straight from
// the page into the operand registers, with a softmax of its own; the waves' states are joined in LDS, the shares of several
// workgroups by k_kv_merge.  Bound by the bytes of the pages.
template <int DH, bool FP8>
struct KvBlock {
  static constexpr int QC = DH / 32, VM = DH / 16;
  uint32x4 k[FP8 ? QC : 2 * QC], v[FP8 ? VM / 2 : VM];
  uint32_t ke[2], ve[2];  // exponents: of key 16 tl + (lane & 15) (K), of keys 16 tl + 4 (lane >> 4) .. + 3 (V)
};
template <int DH, bool FP8, int NT, int NW>
__global__ __launch_bounds__(NW * 64, NT == 1 ? 4 : 2) void k_kv_attend(KvAttend a, int pairs) {
  constexpr int QC = DH / 32, VM = DH / 16, NQ = 16 * NT;
  // One tile of 128-wide heads keeps its queries in LDS: with them in registers the loop did not fit the 128 of 4 waves a SIMD.
  constexpr bool LDS_Q = NT == 1 && DH == 128;
  __shared__ bf16x8 sh_q[LDS_Q ? QC * 64 : 1];
  __shared__ __align__(16) bf16_t sh_k[DH], sh_v[DH];  // the new token
  extern __shared__ float lds[];                       // [NW][cols][DH + 2]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, grp = lane >> 4, col = lane & 15;
  const bool files = NT == 1 && a.k.p != nullptr;  // (t.n is 1: the token is not in the cache yet)
  const Share s = Share::of<NQ>(a, pairs, files);
  if (!s.any) return;
  const int q0 = s.q0, R = s.R, h = s.h, H = a.kv.g.H, bpp = a.kv.g.page_tokens >> 5;
  // The page that takes the new token, known to the wave that attends to it: without one it is dropped, and nobody sees it.
  const int new_page = files && blockIdx.y == gridDim.y - 1 && wave == NW - 1 ? page_of(a.kv, s.r, s.held >> 5) : -1;
  const bool fresh = new_page >= 0;
  if constexpr (NT == 1) {
    constexpr int LPT = DH / 8;
    if (fresh && lane < 2 * LPT) {
      const KvRows &x = lane < LPT ? a.k : a.v;
      const int e = lane % LPT * 8;
      *(uint32x4 *)&(lane < LPT ? sh_k : sh_v)[e] = *(const uint32x4 *)((const bf16_t *)x.p + row_index(x, s.t.at, h * DH + e));
    }
  }
  bf16x8 qf[NT][QC];
  int limit[NT];                  // positions of the cache that the lane's query sees
  QueryTile<DH, NT == 1> tile[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int q = q0 + 16 * t + col;
    load_queries<DH>(a, s, q, grp, qf[t]);
    limit[t] = q < R ? min(s.seen(a, q), s.held) : 0;
    tile[t].clear();
  }
  if constexpr (LDS_Q) {
    if (wave == 0) {
#pragma unroll
      for (int c = 0; c < QC; ++c) sh_q[c * 64 + lane] = qf[0][c];
    }
    __syncthreads();
  }
  typedef KvBlock<DH, FP8> Block;
  auto load = [&](int page, int ib, Block &b) {
    const unsigned char *pg = a.kv.pool + (long)page * a.kv.page_bytes;
    const long at = (long)h * bpp + ib;
    const uint32x4 *src = (const uint32x4 *)(pg + at * ((FP8 ? 64 : 128) * DH)) + lane;
    constexpr int KF = FP8 ? QC : 2 * QC, VF = FP8 ? VM / 2 : VM;
#pragma unroll
    for (int i = 0; i < KF; ++i) b.k[i] = __builtin_nontemporal_load(&src[i * 64]);
#pragma unroll
    for (int i = 0; i < VF; ++i) b.v[i] = __builtin_nontemporal_load(&src[(KF + i) * 64]);
    if constexpr (FP8) {
      const unsigned char *ex = pg + (long)H * bpp * (64 * DH) + at * 64;
#pragma unroll
      for (int tl = 0; tl < 2; ++tl) {
        b.ke[tl] = ex[16 * tl + col];
        b.ve[tl] = ((const uint32_t *)ex)[8 + 4 * tl + grp];
      }
    }
  };
  // base: first position of the block; valid: positions that the row has
  auto use = [&](auto masked_, int base, Block &b, const int (&lim)[NT], int valid) {
    constexpr bool masked = decltype(masked_)::value;
    floatx4 S[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) S[t][0] = S[t][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < QC; ++c) {
      bf16x8 x[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) x[t] = LDS_Q ? sh_q[c * 64 + lane] : qf[t][c];
#pragma unroll
      for (int tl = 0; tl < 2; ++tl) {
        bf16x8 kf;
        if constexpr (FP8) {
          const uint32x4 w = b.k[tl * (QC / 2) + c / 2];
          kf = widen(w[c % 2 * 2], w[c % 2 * 2 + 1], b.ke[tl]);
        } else {
          kf = __builtin_bit_cast(bf16x8, b.k[tl * QC + c]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t][tl] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, x[t], S[t][tl], 0, 0, 0);
      }
    }
    float vs[8];
    if constexpr (FP8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) vs[j] = kv8_factor(b.ve[j >> 2], j & 3);
    }
    bf16x8 pv[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) pv[t] = tile[t].template weights<FP8>(masked, S[t], a.c, lim[t] - base, grp, vs);
    if (masked) {
      const Keep keep(valid - base, grp);
      if constexpr (FP8) {  // (codes of positions that the row does not have may be NaN)
#pragma unroll
        for (int m = 0; m < VM / 2; ++m) b.v[m] &= uint32x4{keep.codes(0), keep.codes(1), keep.codes(0), keep.codes(1)};
      } else {
#pragma unroll
        for (int m = 0; m < VM; ++m) keep.bf16(b.v[m]);
      }
    }
#pragma unroll
    for (int m = 0; m < VM; ++m) {
      bf16x8 vf;
      if constexpr (FP8) {
        vf = widen(b.v[m / 2][m % 2 * 2], b.v[m / 2][m % 2 * 2 + 1], 127);
      } else {
        vf = __builtin_bit_cast(bf16x8, b.v[m]);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) tile[t].O[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pv[t], tile[t].O[m], 0, 0, 0);
    }
  };
  const int whole = min(s.seen(a, q0), s.held) >> 5;  // blocks before it are seen whole by every query
  // place of the wave's next block, whose page's number is asked for ahead of the use of the one before
  const int32_t *table = a.kv.table + (long)s.r * a.kv.g.max_pages;
  int blk = s.lo + wave, ip = blk / bpp, ib = blk % bpp;
  auto entry = [&]() { return table[min(ip, a.kv.g.max_pages - 1)]; };
  int number = entry();
  auto step = [&](auto masked_) {
    const bool is = number >= 0 && number < a.kv.pages && ip < a.kv.g.max_pages;
    Block b;
    if (is) load(number, ib, b);
    ip += NW / bpp;
    ib += NW % bpp;
    if (ib >= bpp) {
      ib -= bpp;
      ++ip;
    }
    number = entry();
    if (is) use(masked_, blk * 32, b, limit, s.held);
    blk += NW;
  };
  while (blk < min(whole, s.hi)) step(std::false_type());
  while (blk < s.hi) step(std::true_type());
  if constexpr (!FP8) {
    if (__builtin_expect(not_finite<DH>(tile), 0)) sums_again<DH>(a, s, q0, limit, s.lo + wave, NW, s.hi, tile);
  }
  uint32_t ke = 0, ve = 0;  // exponents of the new token
  if constexpr (NT == 1) {
    tile[0].one_sum();
    // The one new token joins the last wave's state: its key as key 0 of a tile, its value by the vector units, four elements of
    // every 16 in a lane.
    if (fresh) {
      if constexpr (FP8) {
        uint32_t km = 0, vm = 0;
#pragma unroll
        for (int i = 0; i < DH / 64; ++i) {
          km = max(km, (uint32_t)(sh_k[lane + 64 * i] & 0x7fff) << 16);
          vm = max(vm, (uint32_t)(sh_v[lane + 64 * i] & 0x7fff) << 16);
        }
        ke = kv8_exponent(max_over<64>(km));
        ve = kv8_exponent(max_over<64>(vm));
      }
      floatx4 S = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < QC; ++c) {
        uint32x4 kx = uint32x4{0, 0, 0, 0};
        if (col == 0) kx = *(const uint32x4 *)&sh_k[32 * c + 8 * grp];
        bf16x8 kf = __builtin_bit_cast(bf16x8, kx);
        if constexpr (FP8) {
          const uint2 w = kv8_codes(kx, ke);
          kf = widen(w.x, w.y, ke);
        }
        S = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, LDS_Q ? sh_q[c * 64 + lane] : qf[0][c], S, 0, 0, 0);
      }
      auto &x = tile[0];
      const float score = __shfl(S[0], col) * a.c, m_new = fmaxf(x.m_ref, score);
      const float alpha = __builtin_amdgcn_exp2f(x.m_ref - m_new), p = __builtin_amdgcn_exp2f(score - m_new);
      x.m_ref = m_new;
      x.L[0] = x.L[0] * alpha + p;
#pragma unroll
      for (int m = 0; m < VM; ++m) {
        const uint2 vx = *(const uint2 *)&sh_v[16 * m + 4 * grp];
        float v[4] = {bf2f(vx.x & 0xffffu), bf2f(vx.x >> 16), bf2f(vx.y & 0xffffu), bf2f(vx.y >> 16)};
        if constexpr (FP8) {
          const uint32_t w = ve == 255 ? 0u : kv8_pack(v[0], v[1], v[2], v[3], ve);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = kv8_value(w, i, kv8_scale(ve));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x.O[m][i] = x.O[m][i] * alpha + p * v[i];
      }
    }
  }
  // the waves' states, a tile at a time
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int first = q0 + 16 * t, cols = min(16, R - first);
    if (cols <= 0) break;
    if (t) __syncthreads();
    if (col < cols) {
      float *mine = lds + ((long)wave * cols + col) * (DH + 2);
#pragma unroll
      for (int m = 0; m < VM; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[16 * m + 4 * grp + i] = tile[t].O[m][i];
      if (grp == 0) {
        mine[DH] = tile[t].m_ref;
        mine[DH + 1] = tile[t].L[0];
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < cols * DH; i += NW * 64) {
      const int e = i % DH, cq = i / DH;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < NW; ++w) M = fmaxf(M, lds[((long)w * cols + cq) * (DH + 2) + DH]);
      float num = 0.f, den = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float *x = lds + ((long)w * cols + cq) * (DH + 2);
        const float f = __builtin_amdgcn_exp2f(x[DH] - M);
        num += f * x[e];
        den += f * x[DH + 1];
      }
      const int q = first + cq, head = s.head(a, q);
      const long token = s.token(a, q);
      if (a.splits == 1) {
        ((bf16_t *)a.o.p)[row_index(a.o, token, head * DH + e)] = (bf16_t)f2bf(den == 0.f ? 0.f : num / den);
      } else {
        float *pp = part_of<DH>(a, blockIdx.y, token, head);
        pp[e] = num;
        if (e == 0) {
          pp[DH] = M;
          pp[DH + 1] = den;
        }
      }
    }
  }
  if constexpr (NT == 1) {
    // The first tile files the new token.  Whoever reads its place meanwhile, in the block around it, discards what is there.
    // (Last of all: a barrier behind the stores would wait for them, 4 us of a step of 32 rows.)
    if (fresh && q0 == 0) {
      const int slot = s.held % a.kv.g.page_tokens;
      unsigned char *pg = a.kv.pool + (long)new_page * a.kv.page_bytes;
      if (lane < DH / 8) {
        const uint32x4 kx = *(const uint32x4 *)&sh_k[8 * lane];
        if constexpr (FP8) *(uint2 *)(pg + kv8_k_off(h, slot, 8 * lane, a.kv.g)) = kv8_codes(kx, ke);
        else *(uint32x4 *)((bf16_t *)pg + kv_k_off(h, slot, 8 * lane, a.kv.g)) = kx;
      }
#pragma unroll
      for (int i = 0; i < DH / 64; ++i) {
        const int e = lane + 64 * i;
        if constexpr (FP8) pg[kv8_v_off(h, slot, e, a.kv.g)] = ve == 255 ? 0 : (unsigned char)kv8_pack(bf2f(sh_v[e]), 0.f, 0.f, 0.f, ve);
        else ((bf16_t *)pg)[kv_v_off(h, slot, e, a.kv.g)] = sh_v[e];
      }
      if (FP8 && lane < 2) pg[kv8_exp_off(h, slot, lane, a.kv.g)] = (unsigned char)(lane ? ve : ke);
    }
  }
}

// Many queries: the waves of a workgroup have two tiles each, 128 queries together, and share the blocks, which a ring of
// stages in LDS holds: filled by LDS-direct loads, one bare barrier for two blocks (8-bit blocks stay codes in LDS, and every wave
// converts what it reads).  Blocks that all queries see whole are taken two at a time with one branch for all weights, the values
// requested before it.  80 KB of stages and up to 256 registers: two workgroups a CU.  Three (168 registers, three stages, a
// block at a time, fragments requested as they are needed): us, 8 rows of 512 new tokens behind 2048, 32 heads of 128, bf16
// 143 -> 136; 2 rows of 1023 behind 8193, 32 queries' and 8 kv heads, 8 bits 404 -> 339.  Bound by the vector units (softmax;
// conversions take two thirds again) and the matrix cores in turns, with two waves a SIMD; four tiles a wave do not fit.
constexpr int rows_stages(int dh, bool fp8) { return fp8 ? 8 : dh == 128 ? 5 : 6; }  // (64: three workgroups, 97 -> 77 us for 32 prompts of 512)
constexpr size_t rows_lds(int dh, bool fp8) { return (size_t)rows_stages(dh, fp8) * (32 * dh * (fp8 ? 2 : 4) + (fp8 ? 256 : 0)); }
template <int DH, bool FP8>
__global__ __launch_bounds__(256, 2) void k_kv_attend_rows(KvAttend a, int pairs) {
  constexpr int QC = DH / 32, VM = DH / 16, NT = 2, NW = 4, NS = rows_stages(DH, FP8), NQ = 16 * NT * NW;
  constexpr int KF = FP8 ? QC : 2 * QC, FR = KF + (FP8 ? VM / 2 : VM), LPW = FR / NW;  // fragments a stage, loads of a wave
  constexpr int STAGE = FR * 64 + (FP8 ? 16 : 0);  // 16-byte pieces; behind 8-bit blocks 256 bytes for their exponents
  extern __shared__ uint32x4 ring[];               // [NS][STAGE]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, grp = lane >> 4, col = lane & 15;
  const Share s = Share::of<NQ>(a, pairs, false);
  if (!s.any) return;
  const int q0 = s.q0 + wave * (16 * NT), R = s.R, h = s.h, H = a.kv.g.H, bpp = a.kv.g.page_tokens >> 5;
  const int whole = s.seen(a, s.q0) >> 5;  // blocks before it are seen whole by every query of the workgroup
  const bool busy = q0 < R;
  const int last = busy ? min((s.seen(a, min(q0 + 16 * NT, R) - 1) + 31) >> 5, s.hi) : 0;
  bf16x8 qf[NT][QC];
  int limit[NT];
  QueryTile<DH, false> tile[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int q = q0 + 16 * t + col;
    limit[t] = q < R ? s.seen(a, q) : 0;
    tile[t].clear();
  }
  // Blocks are requested in order.  Lane l holds page 64 w + l of the row, for the window w of 64 pages that the next block is
  // in, waited for where it is loaded; a block without a page is loaded from page 0 and masked, as is every block from the
  // moment on at which a window has an entry that is no page.
  const int32_t *table = a.kv.table + (long)s.r * a.kv.g.max_pages;
  int ip = s.lo / bpp, ib = s.lo % bpp, pages = 0, window = -1;
  uint32_t none = 0;                               // a bit for each stage: its block has no page
  int into = 0, from = 0, asked = s.lo;            // stages of the next block requested and used; blocks requested
  bool gaps = false;
  const int ip_end = (s.hi + bpp - 1) / bpp;
  const uint32x4 *src = nullptr;                   // this wave's part of the next block
  const unsigned char *ex_src = nullptr;
  bool is = false;
  auto next = [](int stage) { return stage == NS - 1 ? 0 : stage + 1; };
  auto new_page = [&]() {
    if (ip >> 6 != window) {
      window = ip >> 6;
      const int at = window * 64 + lane;
      pages = at < a.kv.g.max_pages ? table[at] : -1;
      asm volatile("" : "+v"(pages));
      gaps |= __any(at >= ip && at < ip_end && (pages < 0 || pages >= a.kv.pages));
    }
    int page = __builtin_amdgcn_readlane(pages, ip & 63);
    is = page >= 0 && page < a.kv.pages;
    if (!is) page = 0;
    const unsigned char *pg = a.kv.pool + (long)page * a.kv.page_bytes;
    const long at = (long)h * bpp + ib;
    src = (const uint32x4 *)(pg + at * ((FP8 ? 64 : 128) * DH)) + wave * LPW * 64;
    ex_src = pg + (long)H * bpp * (64 * DH) + at * 64;
  };
  if (s.lo < s.hi) new_page();
  auto request = [&]() {
    none = (none & ~(1u << into)) | (uint32_t)!is << into;
    uint32x4 *dst = ring + into * STAGE + wave * LPW * 64;
#pragma unroll
    for (int i = 0; i < LPW; ++i)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)&(src + i * 64)[lane],
                                       (__attribute__((address_space(3))) void *)(dst + i * 64), 16, 0, 0);
    if constexpr (FP8)  // every wave, so that all wait for the same number of loads; lanes 16 .. 63 repeat
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(ex_src + 4 * col),
                                       (__attribute__((address_space(3))) void *)(ring + into * STAGE + FR * 64), 4, 0, 0);
    into = next(into);
    ++asked;
    src += FR * 64;
    ex_src += 64;
    if (++ib == bpp) {
      ib = 0;
      if (++ip < ip_end) new_page();
    }
  };
  constexpr int LOADS = LPW + (FP8 ? 1 : 0);
  for (int i = 0; i < NS - 2; ++i)
    if (asked < s.hi) request();
#pragma unroll
  for (int t = 0; t < NT; ++t) load_queries<DH>(a, s, q0 + 16 * t + col, grp, qf[t]);
  wait_vmcnt<0>();  // (waited for inside the loop, the queries would make the compiler wait for the ring as well)
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int c = 0; c < QC; ++c) asm volatile("" : "+v"(qf[t][c]));

  // scores of a block: S[t][tl][i] of position 16 tl + 4 grp + i
  auto scores = [&](int stage, floatx4 (&S)[NT][2]) {
    const uint32x4 *kv = ring + stage * STAGE + lane;
    const unsigned char *ex = (const unsigned char *)(ring + stage * STAGE + FR * 64);
    uint32x4 kw[KF];
#pragma unroll
    for (int i = 0; i < KF; ++i) kw[i] = kv[i * 64];
    const uint32_t ke[2] = {FP8 ? ex[col] : 0u, FP8 ? ex[16 + col] : 0u};
#pragma unroll
    for (int t = 0; t < NT; ++t) S[t][0] = S[t][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < QC; ++c)
#pragma unroll
      for (int tl = 0; tl < 2; ++tl) {
        bf16x8 kf;
        if constexpr (FP8) {
          const uint32x4 w = kw[tl * (QC / 2) + c / 2];
          kf = widen(w[c % 2 * 2], w[c % 2 * 2 + 1], ke[tl]);
        } else {
          kf = __builtin_bit_cast(bf16x8, kw[tl * QC + c]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t][tl] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][c], S[t][tl], 0, 0, 0);
      }
  };
  auto factor_words = [&](int stage, uint32_t (&ve)[2]) {
    const uint32_t *ex = (const uint32_t *)(ring + stage * STAGE + FR * 64);
    ve[0] = ex[8 + grp];
    ve[1] = ex[12 + grp];
  };
  auto add_values = [&](const uint32x4 (&vw)[FR - KF], const bf16x8 (&pv)[NT]) {
#pragma unroll
    for (int m = 0; m < VM; ++m) {
      bf16x8 vf;
      if constexpr (FP8) {
        const uint32x4 w = vw[m / 2];
        vf = widen(w[m % 2 * 2], w[m % 2 * 2 + 1], 127);
      } else {
        vf = __builtin_bit_cast(bf16x8, vw[m]);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) tile[t].O[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pv[t], tile[t].O[m], 0, 0, 0);
    }
  };
  auto values_of = [&](int stage, uint32x4 (&vw)[FR - KF]) {
#pragma unroll
    for (int i = 0; i < FR - KF; ++i) vw[i] = ring[stage * STAGE + (KF + i) * 64 + lane];
  };
  auto use = [&](int blk, bool no_page) {
    const int base = blk * 32;
    floatx4 S[NT][2];
    scores(from, S);
    float vs[8];
    if constexpr (FP8) {
      uint32_t ve[2];
      factor_words(from, ve);
#pragma unroll
      for (int j = 0; j < 8; ++j) vs[j] = kv8_factor(ve[j >> 2], j & 3);
    }
    bf16x8 pv[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) pv[t] = tile[t].template weights<FP8>(true, S[t], a.c, no_page ? 0 : limit[t] - base, grp, vs);
    uint32x4 vw[FR - KF];
    values_of(from, vw);
    add_values(vw, pv);
  };
  // Two blocks that every query sees whole: one branch for all of their weights, so that from there on exponentials and products
  // are formed side by side, and the values are on their way before.
  auto use_two = [&](int one, int two) {
    const int stage[2] = {one, two};
    floatx4 S[2][NT][2];
    uint32_t ve[2][2];
    int power[2][8];  // of the values; 2 rows of 1023 behind 8193, 8 bits, us: by ldexp 338, as factors, 0 for byte 0, 341, as they are 358
    uint32x4 vw[FR - KF];
    bool raise = false;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      __builtin_amdgcn_s_setprio(1);  // (before the other waves' exponentials: 140 -> 136 us)
      scores(stage[u], S[u]);
      __builtin_amdgcn_s_setprio(0);
      if constexpr (FP8) {
        factor_words(stage[u], ve[u]);
#pragma unroll
        for (int j = 0; j < 8; ++j) power[u][j] = (int)(ve[u][j >> 2] >> (8 * (j & 3)) & 255u) - 127;
#pragma unroll
        for (int i = 0; i < 2; ++i) raise |= (((ve[u][i] & 0x7f7f7f7fu) + 0x01010101u) & ve[u][i] & 0x80808080u) != 0;
      }
    }
    values_of(stage[0], vw);
    float p[2][NT][8];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        tile[t].relative(S[u][t], a.c, p[u][t]);
        raise |= tile[t].most(p[u][t]) > 8.0f;
      }
    if (__any(raise)) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float most = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int j = 0; j < 8; ++j) most = fmaxf(most, S[u][t][j >> 2][j & 3]);
        tile[t].raise(most * a.c);
#pragma unroll
        for (int u = 0; u < 2; ++u) tile[t].relative(S[u][t], a.c, p[u][t]);
      }
      if constexpr (FP8)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (power[u][j] == 128) {  // a NaN that all queries see: so are their sums of weights
#pragma unroll
              for (int t = 0; t < NT; ++t) p[u][t][j] = __uint_as_float(0x7fc00000u);
            }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      bf16x8 pv[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int j = 0; j < 8; ++j) p[u][t][j] = __builtin_amdgcn_exp2f(p[u][t][j]);
        pv[t] = pack8(p[u][t]);
        tile[t].L = __builtin_amdgcn_mfma_f32_16x16x32_bf16(all_ones(), pv[t], tile[t].L, 0, 0, 0);
        if constexpr (FP8) {
#pragma unroll
          for (int j = 0; j < 8; ++j) p[u][t][j] = __builtin_ldexpf(p[u][t][j], power[u][j]);
          pv[t] = pack8(p[u][t]);
        }
      }
      add_values(vw, pv);
      if (u == 0) values_of(stage[1], vw);
    }
  };
  // clears what a stage holds from position `valid` of its block on
  auto clear = [&](int valid) {
    const Keep keep(valid, grp);
    for (int m = wave; m < FR - KF; m += NW) {
      uint32x4 &v = ring[from * STAGE + (KF + m) * 64 + lane];
      uint32x4 x = v;
      if constexpr (FP8) x &= uint32x4{keep.codes(0), keep.codes(1), keep.codes(0), keep.codes(1)};
      else keep.bf16(x);
      v = x;
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // waits until the next `n` blocks are there for all waves, and requests others into the stages of those before
  auto open = [&](int blk, int n) {
    const int ahead = asked - blk - n;  // requested behind them
    if (ahead >= 3) wait_vmcnt<3 * LOADS>();
    else if (ahead == 2) wait_vmcnt<2 * LOADS>();
    else if (ahead == 1) wait_vmcnt<LOADS>();
    else wait_vmcnt<0>();
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): this wave's reads of the stages before
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    while (asked < min(s.hi, blk + NS)) request();
  };
  int blk = s.lo;
  for (; blk + 2 <= min(whole, s.hi) && !gaps; blk += 2) {
    open(blk, 2);
    const int second = next(from);
    if (busy) use_two(from, second);
    from = next(second);
  }
  for (; blk < s.hi; ++blk) {
    open(blk, 1);
    const bool no_page = none >> from & 1;
    if (no_page || blk * 32 + 32 > s.held) clear(no_page ? 0 : s.held - blk * 32);
    if (blk < last) use(blk, no_page);
    from = next(from);
  }
  if constexpr (!FP8) {
    if (__builtin_expect(not_finite<DH>(tile), 0)) sums_again<DH>(a, s, q0, limit, s.lo, 1, last, tile);
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int q = q0 + 16 * t + col;
    if (q >= R) continue;
    const auto &x = tile[t];
    const long token = s.token(a, q);
    const int head = s.head(a, q);
    if (a.splits == 1) {
      const float inv = x.L[0] == 0.f ? 0.f : 1.0f / x.L[0];
      bf16_t *o = (bf16_t *)a.o.p;
#pragma unroll
      for (int m = 0; m < VM; ++m)
        *(uint2 *)&o[row_index(a.o, token, head * DH + 16 * m + 4 * grp)] =
            make_uint2(pack2(x.O[m][0] * inv, x.O[m][1] * inv), pack2(x.O[m][2] * inv, x.O[m][3] * inv));
    } else {
      float *pp = part_of<DH>(a, blockIdx.y, token, head);
#pragma unroll
      for (int m = 0; m < VM; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) pp[16 * m + 4 * grp + i] = x.O[m][i];
      if (grp == 0) {
        pp[DH] = x.m_ref;
        pp[DH + 1] = x.L[0];
      }
    }
  }
}

// Joins the shares of a query's keys: a workgroup per query of a row and head.  Every wave weighs the (at most 64) shares, one a
// lane, then 256 / DH groups of threads add up the numerators of theirs.  A chain of three round trips whatever their number.
template <int DH>
__global__ __launch_bounds__(256) void k_kv_merge(KvAttend a, int queries) {
  constexpr int GROUPS = 256 / DH;
  __shared__ float f[64], sum[GROUPS][DH];
  const int H = a.kv.g.H, q = blockIdx.x % queries, h = blockIdx.x / queries % H, r = blockIdx.x / queries / H;
  const RowTokens t = row_tokens(a.tk, r);
  if (q >= t.n * a.group) return;
  const int head = h * a.group + q % a.group, lane = threadIdx.x & 63;
  const long token = t.at + (long)(q / a.group) * a.tk.step, stride = (long)a.tk.tokens * a.heads * (DH + 2);
  const float *x = part_of<DH>(a, 0, token, head);
  float m = -3.0e38f, l = 0.f;
  if (lane < a.splits) {
    m = x[lane * stride + DH];
    l = x[lane * stride + DH + 1];
  }
  float M = m;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) M = fmaxf(M, __shfl_xor(M, o));
  const float w = __builtin_amdgcn_exp2f(m - M);
  const float den = wave_sum_f(lane < a.splits ? w * l : 0.f);
  if (threadIdx.x < 64) f[lane] = w;
  __syncthreads();
  const int e = threadIdx.x % DH, g = threadIdx.x / DH;
  float num = 0.f;
#pragma unroll 8
  for (int s = g; s < a.splits; s += GROUPS) num += f[s] * x[s * stride + e];
  sum[g][e] = num;
  __syncthreads();
  if (g == 0) {
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) num += sum[i][e];
    ((bf16_t *)a.o.p)[row_index(a.o, token, head * DH + e)] = (bf16_t)f2bf(den == 0.f ? 0.f : num / den);
  }
}

// The same for up to 8 shares, of which there are many queries: a wave each, all shares requested at once (two shares of 16384
// queries, 2 rows of 256 tokens behind 500: 44 -> 32 us with the attention, 12 of them a workgroup for each query).
template <int DH>
__global__ __launch_bounds__(256) void k_kv_merge_few(KvAttend a, int queries) {
  constexpr int S = 8, E = DH / 64;
  const int H = a.kv.g.H, lane = threadIdx.x & 63;
  const long id = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int q = (int)(id % queries), h = (int)(id / queries % H), r = (int)(id / queries / H);
  if (r >= a.kv.rows) return;
  const RowTokens t = row_tokens(a.tk, r);
  if (q >= t.n * a.group) return;
  const int head = h * a.group + q % a.group;
  const long token = t.at + (long)(q / a.group) * a.tk.step, stride = (long)a.tk.tokens * a.heads * (DH + 2);
  const float *x = part_of<DH>(a, 0, token, head);
  float m[S], l[S], v[S][E], M = -3.0e38f, den = 0.f, num[E] = {};
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const float *y = x + min(s, a.splits - 1) * stride;
    m[s] = s < a.splits ? y[DH] : -3.0e38f;
    l[s] = s < a.splits ? y[DH + 1] : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) v[s][e] = y[E * lane + e];
  }
#pragma unroll
  for (int s = 0; s < S; ++s) M = fmaxf(M, m[s]);
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const float w = s < a.splits ? __builtin_amdgcn_exp2f(m[s] - M) : 0.f;
    den += w * l[s];
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (s < a.splits) num[e] += w * v[s][e];
  }
  uint32_t o = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) o |= (uint32_t)f2bf(den == 0.f ? 0.f : num[e] / den) << (16 * e);
  bf16_t *to = (bf16_t *)a.o.p + row_index(a.o, token, head * DH + E * lane);
  if constexpr (E == 2) *(uint32_t *)to = o;
  else *to = (bf16_t)o;
}

int blocks_of(const KvTokens &tk) { return (tk.max_new + 31 + 31) / 32; }  // of a row, wherever in a block it begins

}  // namespace

// Workgroups of the kernels for a few tokens, or 0: up to 8 of a row (k_kv_append_few), and a grid that fits.
static unsigned few_groups(const KvView &kv, const KvTokens &tk) {
  const long units = 2L * kv.g.H * tk.max_new * kv.rows, groups = (units * (kv.g.dh / 8) + 255) / 256;
  return tk.max_new <= 8 && launch_fits(groups, 256) ? (unsigned)groups : 0;  // (units, of 8 lanes or more, are in 32 bits then)
}
long kv_blocks(const KvView &kv, const KvTokens &tk) { return (long)blocks_of(tk) * kv.g.H * kv.rows; }
// The kernels for many tokens, a workgroup for each block: f(grid, first block) for as many as a launch has, which is all of them
// but for a row of 100000 tokens among more than a hundred.
template <typename F>
static void each_launch(const KvView &kv, const KvTokens &tk, F f) {
  const long all = kv_blocks(kv, tk);
  for (long from = 0; from < all; from += launch_most(256)) f(dim3((unsigned)std::min(all - from, launch_most(256))), (uint32_t)from);
}
void kv_append(hipStream_t s, const KvView &kv, const KvTokens &tk, const KvRows &k, const KvRows &v) {
  if (const unsigned few = few_groups(kv, tk)) {
    if (kv.g.dh == 64) {
      if (kv.fp8) SKD_LAUNCH((k_kv_append_few<64, true>), dim3(few), dim3(256), 0, s, kv, tk, k, v);
      else SKD_LAUNCH((k_kv_append_few<64, false>), dim3(few), dim3(256), 0, s, kv, tk, k, v);
    } else {
      if (kv.fp8) SKD_LAUNCH((k_kv_append_few<128, true>), dim3(few), dim3(256), 0, s, kv, tk, k, v);
      else SKD_LAUNCH((k_kv_append_few<128, false>), dim3(few), dim3(256), 0, s, kv, tk, k, v);
    }
    return;
  }
  const int blocks = blocks_of(tk);
  each_launch(kv, tk, [&](dim3 grid, uint32_t from) {
    if (kv.g.dh == 64) {
      if (kv.fp8) SKD_LAUNCH((k_kv_append<64, true>), grid, dim3(256), 0, s, kv, tk, k, v, blocks, from);
      else SKD_LAUNCH((k_kv_append<64, false>), grid, dim3(256), 0, s, kv, tk, k, v, blocks, from);
    } else {
      if (kv.fp8) SKD_LAUNCH((k_kv_append<128, true>), grid, dim3(256), 0, s, kv, tk, k, v, blocks, from);
      else SKD_LAUNCH((k_kv_append<128, false>), grid, dim3(256), 0, s, kv, tk, k, v, blocks, from);
    }
  });
}

void kv_read(hipStream_t s, const KvView &kv, const KvTokens &tk, bool bf16, const KvRows &k, const KvRows &v) {
  const int blocks = blocks_of(tk);
  const unsigned few = few_groups(kv, tk);
#define SKD_READ(DH, FP8)                                                                                                     \
  do {                                                                                                                        \
    if (few && bf16) SKD_LAUNCH((k_kv_read_few<DH, FP8, bf16_t>), dim3(few), dim3(256), 0, s, kv, tk, k, v);                    \
    else if (few) SKD_LAUNCH((k_kv_read_few<DH, FP8, float>), dim3(few), dim3(256), 0, s, kv, tk, k, v);                        \
    else each_launch(kv, tk, [&](dim3 grid, uint32_t from) {                                                                  \
      if (bf16) SKD_LAUNCH((k_kv_read<DH, FP8, bf16_t>), grid, dim3(256), 0, s, kv, tk, k, v, blocks, from);                   \
      else SKD_LAUNCH((k_kv_read<DH, FP8, float>), grid, dim3(256), 0, s, kv, tk, k, v, blocks, from);                         \
    });                                                                                                                       \
  } while (0)
  if (kv.g.dh == 64) {
    if (kv.fp8) SKD_READ(64, true);
    else SKD_READ(64, false);
  } else {
    if (kv.fp8) SKD_READ(128, true);
    else SKD_READ(128, false);
  }
#undef SKD_READ
}

// Which kernel and how many shares of the keys: by the most queries that a row and kv head has.
struct AttendPlan {
  int nq;       // queries of a workgroup: 16, 32 or 128
  int waves;    // 16, 32
  int splits;
  long tiles;   // of a row and kv head
  int pairs;    // places for a row and kv head
};
static AttendPlan plan_attend(const KvView &kv, const KvTokens &tk, int heads) {
  AttendPlan p{};
  const long R = (long)tk.max_new * (heads / kv.g.H), blocks = ((long)tk.max_past + tk.max_new + 31) / 32;
  // Up to 16 queries one tile, up to 32 two; beyond, the blocks go through LDS once for all, which 8 bits gain from only with five
  // tiles and more (inputs not in the last-level cache, us.  Two tiles of 16 for 17 .. 32 queries: 16 rows of 2000, 8 kv heads of
  // 128, bf16 31.3, 30.9; 40 rows 70.7, 104.9.  33 .. 64 as two of 32 or through LDS: 8 rows of 1000, 32 heads of 128, bf16 58.7,
  // 35.2, 8 bits 38.7, 38.2; 32 rows of 700, 8 kv heads of 64, bf16 23.4, 19.7, 8 bits 15.2, 22.1; one of 20000, 8 of 128, 8 bits
  // 23.3, 30.5.  65 .. 128: 8 rows of 1000 bf16 107, 38, 8 bits 70, 41.)
  p.nq = R <= 16 ? 16 : R <= (kv.fp8 ? 64 : 32) ? 32 : 128;
  p.tiles = (R + p.nq - 1) / p.nq;
  const long n = (long)kv.g.H * kv.rows, wgs = p.tiles * n;
  // Workgroups go to the eight XCDs in turn.  With a multiple of eight places all tiles of a row and kv head are on one of them
  // and find each other's blocks in its L2 (8 prompts of 2048, 32 heads of 128: 586 us with the tiles next to each other, 441
  // so); a few more places than there are pairs cost less than that gives, many leave XCDs idle.
  p.pairs = (int)n;
  if (p.tiles > 1 && n >= 8 && (n + 7) / 8 * 8 * 20 <= n * 23) p.pairs = (int)((n + 7) / 8 * 8);
  p.splits = 1;
  if (p.nq == 128) {
    // A workgroup for each CU, in shares of 8 blocks at least, of 16 where half of the CUs have one already, and two where shares
    // keep 24 (that rule, without the 16, without the second workgroup, us: one row of 512 behind 8000, 32 heads, 8 kv heads
    // 95, 95, 116; four of 100 behind 3000 47, 47, 54; 512 tokens from nothing, 32 heads of 64 17, 23, 17; one row of 1000 behind
    // 100, 32 heads 36, two workgroups for shares of 16: 48).
    p.waves = 4;
    auto least = [&]() { return wgs * p.splits >= 256 ? 24 : p.splits == 1 && wgs >= 128 ? 16 : 8; };
    while (p.splits < 64 && wgs * p.splits <= 384 && blocks / (2 * p.splits) >= least()) p.splits *= 2;  // (456: the same either way)
  } else {
    // 8 waves a CU, and 16 from 1024 workgroups on, which are narrower then.  (Shares up to 16 waves a CU against this, us: 8 rows of
    // 2000, 32 heads of 128, bf16 45.7, 42.1, 8 bits 28.3, 24.6; one of 32766, 8 kv heads, 8 bits 20.4, 19.6; up to 4: 21.1.)
    // Two tiles that are on half of the CUs already are shared out only if every wave keeps six blocks (shared out all the same, and
    // not, us: 4 rows of 1000 with 20 new tokens, 32 heads 23.3, 20.0; 16 of 2000 with 5, 32 queries' and 8 kv heads 31.7, 31.1; 24 of
    // 3000 with 6 64.9, 50.9; 16 of 500 with 5 17.7, 14.1; against it 16 of 1000 to 2000 with 5, 27.0, 28.5).
    p.waves = p.nq == 16 && wgs >= 1024 ? 4 : 8;
    const int least = p.waves * (p.nq == 32 && wgs >= 128 ? 6 : 1);
    while (p.splits < 64 && wgs * p.waves * p.splits < 2048 && blocks / (2 * p.splits) >= (p.splits == 1 ? least : p.waves)) p.splits *= 2;
  }
  return p;
}
bool kv_attend_fits(const KvView &kv, const KvTokens &tk, int heads) {
  const AttendPlan p = plan_attend(kv, tk, heads);
  return launch_fits(p.tiles * p.pairs, 64 * p.waves);
}
int kv_attend_splits(const KvView &kv, const KvTokens &tk, int heads) { return plan_attend(kv, tk, heads).splits; }
size_t kv_attend_part(const KvView &kv, const KvTokens &tk, int heads, int splits) {
  return splits > 1 ? (size_t)splits * tk.tokens * heads * (kv.g.dh + 2) : 0;
}

template <int DH, bool FP8, int NT, int NW>
static void launch_attend(hipStream_t s, const KvAttend &a, dim3 grid, int pairs) {
  const int cols = std::min(16, a.tk.max_new * a.group);
  const size_t lds = (size_t)NW * cols * (DH + 2) * sizeof(float);
  static std::atomic<uint64_t> done{0};
  if (lds + 8192 > 64 * 1024) (void)allow_lds(done, {(const void *)k_kv_attend<DH, FP8, NT, NW>}, NW * 16 * (DH + 2) * sizeof(float));
  SKD_LAUNCH((k_kv_attend<DH, FP8, NT, NW>), grid, dim3(NW * 64), lds, s, a, pairs);
}
template <int DH, bool FP8>
static void attend(hipStream_t s, const KvAttend &a) {
  const AttendPlan p = plan_attend(a.kv, a.tk, a.heads);
  const dim3 grid((unsigned)(p.tiles * p.pairs), a.splits);
  if (p.nq == 128) {
    static std::atomic<uint64_t> done{0};
    if (rows_lds(DH, FP8) > 64 * 1024) (void)allow_lds(done, {(const void *)k_kv_attend_rows<DH, FP8>}, rows_lds(DH, FP8));
    SKD_LAUNCH((k_kv_attend_rows<DH, FP8>), grid, dim3(256), rows_lds(DH, FP8), s, a, p.pairs);
  } else if (p.nq == 32) {
    launch_attend<DH, FP8, 2, 8>(s, a, grid, p.pairs);
  } else if (p.waves == 4) {
    launch_attend<DH, FP8, 1, 4>(s, a, grid, p.pairs);
  } else {
    launch_attend<DH, FP8, 1, 8>(s, a, grid, p.pairs);
  }
  if (a.splits > 1) {
    const int queries = a.tk.max_new * a.group;
    const long all = (long)queries * a.kv.g.H * a.kv.rows;
    if (a.splits <= 8) SKD_LAUNCH(k_kv_merge_few<DH>, dim3((unsigned)((all + 3) / 4)), dim3(256), 0, s, a, queries);
    else SKD_LAUNCH(k_kv_merge<DH>, dim3((unsigned)all), dim3(256), 0, s, a, queries);
  }
}
void kv_attend(hipStream_t s, const KvAttend &call) {
  KvAttend a = call;
  if (a.k.p && !(a.tk.max_new == 1 && plan_attend(a.kv, a.tk, a.heads).nq == 16)) {  // (one token of few heads: the same launch)
    kv_append(s, a.kv, a.tk, a.k, a.v);
    a.k.p = nullptr;
  }
  if (a.kv.g.dh == 64) a.kv.fp8 ? attend<64, true>(s, a) : attend<64, false>(s, a);
  else a.kv.fp8 ? attend<128, true>(s, a) : attend<128, false>(s, a);
}

}  // namespace skd
