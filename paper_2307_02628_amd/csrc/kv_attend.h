// Kernels of the attention over pages, and their launches, for one kind of page (EL) and with or without changed scores (SC).
#pragma once
#include "kv_device.h"

namespace skd {

// Which kernel and how many shares of the keys: by the most queries that a row and kv head has.
struct AttendPlan {
  int nq;       // queries of a workgroup: 16, 32 or 128
  int waves;    // 16, 32
  int splits;
  long tiles;   // of a row and kv head
  int pairs;    // places for a row and kv head
};

namespace {

enum { SC_MASK = 1, SC_CAP = 2, SC_SLOPES = 4 };  // what of a call's scoring a kernel is made for (no mask, no other)

// ------------------------------------------------------------------ attention
// A query tile is 16 of the R = new * group queries of a row and kv head, in the order (token, head of the group): the 16
// columns of the matrix instructions.  The softmax works in units of log2 against a reference that is raised only by more
// than 8 (weights up to 2^8), denominators come from the matrix cores (a row of ones) and are sums of the rounded weights.
//
// Query i of a row sees positions up to past + i.  In blocks that reach beyond what a tile's first query sees scores are masked by
// selection.  Since 0 * infinity is not 0, that leaves values: beyond the row's last position they are cleared (a page may hold
// anything there); an infinity or NaN that only later queries see makes sums that are not finite, and a wave that ends with such
// sums forms them once more (sums_again), without such values, which are added for the queries that see them.  8-bit values are
// finite where they were filed, what is not is in their scales, which are selected with the weights; with changed scores a position
// that no query sees may never have been filed, so that codes of NaN are looked for (odd_codes).
// The powers of two of 8-bit keys are an operand of the conversion to bf16, those of values multiply the weights: both exact.
// Those of 4-bit keys and values are operands of the conversion (32 elements of a value have one each, so that the weights would
// have to be multiplied for every 32); a value that is not finite is in them, and is added for the queries that see it (odd_exponents).
//
// Changed scores and masks (SC, bits of what a call asks for).  A query sees positions low .. limit - 1 of its own.  The share of
// the distance, over what scores are multiplied by, is where the matrix instructions' sums begin: one instruction a score.  A cap's
// function is applied in place, but for its factor, which takes that place, and for its constant part, which is the same for every position.
// (Its four instructions, two of them of a quarter of the rate, stand in the code as such: with a branch around them, or around
// the share, products and exponentials of two blocks no longer mixed.  8 rows of up to 512 tokens behind 2048, 32 heads of 128, bf16, us
// of short runs: slopes 217, so 162; cap 194, 177; masks alone 156, 144.  Of continued ones, side by side: scores as they are 130, masks
// alone 129, slopes 139 with the nearest blocks first, cap 160, both 175; 8 bits 143, 147, 162, 180, 201; 4 bits 144, 148, 163, 179, 198.)

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
// The power of two of byte i of a word, as the conversions take it: the exponent of an fp32 number whatever its other bits are (255: NaN).
__device__ inline float scale4(uint32_t word, int i) {
  return __uint_as_float(i == 0 ? word << 23 : i == 1 ? word << 15 : i == 2 ? word << 7 : word >> 1);
}
// bf16x8 of a word of eight 4-bit codes
__device__ inline bf16x8 widen4(uint32_t w, float scale) {
  const bf16x2 x[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)};
  return bf16x8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
}
// The two value fragments of 32 elements: byte y of word x is the lane's key 4 x + y, its two codes are of elements 16 apart.
__device__ inline void widen4_values(const uint32_t (&w)[2], const uint32_t (&e)[2], bf16x8 (&f)[2]) {
  uint32_t x[8];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x[4 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], scale4(e[i], 0), 0));
    x[4 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], scale4(e[i], 1), 1));
    x[4 * i + 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], scale4(e[i], 2), 2));
    x[4 * i + 3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i], scale4(e[i], 3), 3));
  }
  uint32x4 lo, hi;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100);
    hi[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302);
  }
  f[0] = __builtin_bit_cast(bf16x8, lo);
  f[1] = __builtin_bit_cast(bf16x8, hi);
}
// 16-byte pieces of a block that a lane takes: keys, values; bytes of a block's codes, and to the next block
constexpr int key_pieces(int dh, int el) { return el == EL_BF16 ? dh / 16 : el == EL_FP8 ? dh / 32 : dh / 64; }
constexpr int value_pieces(int dh, int el) { return key_pieces(dh, el); }
constexpr int block_bytes(int dh, int el) { return el == EL_BF16 ? 128 * dh : el == EL_FP8 ? 64 * dh : 34 * dh; }
// the key fragment of tile tl, elements 32 c .. + 31, of a lane's pieces; e: its exponents
template <int DH, int EL>
__device__ inline bf16x8 key_fragment(const uint32x4 *k, const uint32_t *e, int tl, int c) {
  constexpr int QC = DH / 32;
  if constexpr (EL == EL_FP4) {
    const int f = tl * QC + c;
    return widen4(k[f / 4][f % 4], scale4(e[f / 4], f % 4));
  } else if constexpr (EL == EL_FP8) {
    const uint32x4 w = k[tl * (QC / 2) + c / 2];
    return widen(w[c % 2 * 2], w[c % 2 * 2 + 1], e[tl]);
  } else {
    return __builtin_bit_cast(bf16x8, k[tl * QC + c]);
  }
}

// ------------------------------------------------------------------ changed scores
// cap tanh(x) = cap - 2 cap / (1 + exp(2 x)), here without the constant and times 1 / (2 cap): off by up to 3 * 2^-24 (exponential,
// sum, reciprocal), which for the largest cap, 1024, is 2^-11.4 of a weight, against the 2^-8 of its rounding.  (As a fraction of
// polynomials: 11 instructions and one of a quarter of the rate, instead of 2 and two.)
__device__ inline float capped(float in, float s) { return __builtin_amdgcn_rcpf(-1.0f - __builtin_amdgcn_exp2f(in * s)); }

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

template <bool LOW>
__device__ inline bool hidden(int j, int low, int limit, int grp) {
  const bool behind = block_pos(j, 0) >= limit - 4 * grp;
  return LOW ? behind || block_pos(j, 0) < low - 4 * grp : behind;
}

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
  // a weight at most; the denominator adds the rounded ones).  masked: positions from `limit` of the block on have none, nor (LOW)
  // those before `low`.
  template <bool FP8, bool LOW>
  __device__ bf16x8 weights(bool masked, floatx4 (&S)[2], float c, int low, int limit, int grp, const float (&vs)[8]) {
    if (masked) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (hidden<LOW>(j, low, limit, grp)) S[j >> 2][j & 3] = -INFINITY;
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
          if (hidden<LOW>(j, low, limit, grp)) p[j] = 0.f;  // (a power of two there may be NaN)
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
// 1 at positions from `low` to `limit` - 1
template <bool LOW>
__device__ inline bf16x8 visible(int low, int limit, int grp) {
  bf16x8 v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (__bf16)(hidden<LOW>(j, low, limit, grp) ? 0.0f : 1.0f);
  return v;
}
// Whether masked blocks look for values that are not finite as they come.  (8 bits with scores as they are: the row's last token sees every position
// that the row has, so they were all filed, and what lies behind is cleared.  bf16: sums_again.)
constexpr bool looks(int el, int sc) { return el == EL_FP4 || (el == EL_FP8 && sc); }
__device__ inline uint32_t bytes_of(uint32_t top) { return (top << 1) - (top >> 7); }  // all bits of the bytes whose upper one is set
// 4-bit values of a masked block that are not finite, since 0 is no weight for them, wherever they are: a position that holds NaN, or one
// that nobody wrote.  Of a lane's words of exponents, [group][2], bytes of NaN (and 254, which is never written) are cleared and
// the sums of the queries that see them become NaN; codes with exponent 126 end at 3, as written ones do.  Rare: out of the way of
// everything else.
template <int DH, bool LOW, int NT, int NV, typename Tile>
__device__ inline void odd_exponents(uint32x4 (&v)[NV], uint32_t (&e)[DH / 16], Tile (&tile)[NT], const int (&low)[NT], const int (&limit)[NT]) {
  auto odd = [&](int i) { return ((e[i] & 0x7f7f7f7fu) + 0x03030303u) & e[i] & 0x80808080u; };  // bytes from 253 on
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < DH / 16; ++i) any |= odd(i);
  if (__builtin_expect(!__any(any != 0), 1)) return;
#pragma unroll
  for (int i = 0; i < DH / 16; ++i) {
    if (!__any(odd(i) != 0)) continue;
#pragma unroll 1
    for (int g = 0; g < 4; ++g) {
      const uint32_t b = (uint32_t)__shfl((int)e[i], 16 * g);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int y = 0; y < 4; ++y)
          if ((b >> (8 * y) & 255u) >= 254u && !hidden<LOW>(4 * (i & 1) + y, low[t], limit[t], g)) {
#pragma unroll
            for (int u = 0; u < 2; ++u) tile[t].O[i / 2 * 2 + u] += __uint_as_float(0x7fc00000u);
          }
    }
    const uint32_t w = v[i / 4][i % 4], large = w >> 1 & w >> 2 & 0x11111111u & bytes_of(odd(i));  // of the same keys; codes of 4 and 6
    v[i / 4][i % 4] = (w & ~(large << 1)) | large;
    e[i] &= ~bytes_of(((e[i] & 0x7f7f7f7fu) + 0x02020202u) & e[i] & 0x80808080u);
  }
}
__device__ inline uint32_t over_row(uint32_t x) {  // bits that any of 16 lanes has
  x |= (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xF, 0xF, true);
  x |= (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x124, 0xF, 0xF, true);
  x |= (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x122, 0xF, 0xF, true);
  return x | (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x121, 0xF, 0xF, true);
}
// 8-bit values of a masked block likewise: codes of NaN, which are never filed, are cleared; what is returned says whether there were any, and
// `bad` where: the bytes of the lane's keys 0 .. 3 and 4 .. 7, as their exponents lie, all bits set.
template <int NV>
__device__ inline bool odd_codes(uint32x4 (&v)[NV], uint32_t (&bad)[2]) {
  auto odd = [](uint32_t w) { return (w & 0x7f7f7f7fu) + 0x01010101u; };  // the upper bit of a byte
  bad[0] = bad[1] = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) bad[j & 1] |= odd(v[i][j]);
  if (__builtin_expect(!__any(((bad[0] | bad[1]) & 0x80808080u) != 0), 1)) return false;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) v[i][j] &= ~bytes_of(odd(v[i][j]) & 0x80808080u);
#pragma unroll
  for (int x = 0; x < 2; ++x) bad[x] = bytes_of(over_row(bad[x]) & 0x80808080u);  // (the elements of a key are in 16 lanes)
  return true;
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

// what scores are multiplied by, in units of log2
template <int SC>
__device__ inline float factor(const KvAttend &a) { return SC & SC_CAP ? a.sc.out : a.c; }

// What a workgroup computes: NQ queries from q0 on of a row and kv head, on one share of their keys.
struct Share {
  RowTokens t;
  int r, h, R, q0;
  int held;        // positions that the cache holds
  int lo, hi;      // blocks
  int whole_lo, whole_hi;  // those that every query sees whole
  bool any;
  // Workgroup: [tile, the longest first][row and kv head], `pairs` places for the latter.  Tiles of many queries: of 16 rows and
  // heads of an XCD at a time, so that fewer pages pass through its L2 at once, and the next ones fill the gaps (all of them, 16,
  // 1 at a time, us: 8 prompts of 2048, 32 heads of 128, bf16 428, 411, 440; 512 tokens behind 2048 203, 192, 194; 8 bits 386,
  // 380, 440 and 196, 192, 206; 32 prompts of 512, heads of 64, 8 bits 88, 93, 122).
  static constexpr int TOGETHER = 16;
  template <int NQ, int SC>
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
    s.lo = s.hi = s.whole_lo = s.whole_hi = 0;
    if constexpr (!SC) {
      s.whole_hi = min(s.seen(a, s.q0), s.held) >> 5;
      s.take(a, 0, min(s.seen(a, min(s.q0 + NQ, s.R) - 1), s.held));
    }
    return s;
  }
  // blocks with positions from .. upto - 1, of them this workgroup's share
  __device__ void take(const KvAttend &a, int from, int upto) {
    const int nblk = (upto + 31) >> 5, first = min(from >> 5, nblk), per = (nblk - first + a.splits - 1) / a.splits;
    lo = first + (int)blockIdx.y * per;
    hi = min(lo + per, nblk);
  }
  // SC: the blocks that every query sees whole come first, the others, before and behind them, then: masks are in the code once.
  __device__ int wholes() const { return whole_hi - whole_lo; }
  // LAST_FIRST: of the whole ones the last first, where scores fall with the distance: the nearest have the largest ones, and the
  // reference is not raised again and again (from the first on, and so, us: 8 rows of up to 512 tokens behind 2048, 32 heads of 128, bf16 161,
  // 139, 8 bits 191, 162, 4 bits 184, 163; steps of 32 rows of up to 600 in 4 bits 19.3, 18.2).
  template <bool LAST_FIRST = false>
  __device__ int block(int v) const { return v < wholes() ? (LAST_FIRST ? whole_hi - 1 - v : whole_lo + v) : v < whole_hi - lo ? v - wholes() + lo : v + lo; }
  __device__ int seen(const KvAttend &a, int q) const { return t.past + q / a.group + 1; }  // positions that query q sees
  __device__ long token(const KvAttend &a, int q) const { return t.at + (long)(q / a.group) * a.tk.step; }
  __device__ int head(const KvAttend &a, int q) const { return h * a.group + q % a.group; }
};
// What a lane needs to know of a query: it sees positions low .. limit - 1 of those that the row has (none: 0, 0).
struct Seen {
  int low, limit, pos;
  float slope;  // over what scores are multiplied by
};
// of queries q0 + 16 t + col; the loads are on their way together
template <int SC, int NT>
__device__ inline void see(const KvAttend &a, const Share &s, int q0, Seen (&x)[NT]) {
  const int col = threadIdx.x & 15;
  if constexpr (!SC) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int q = q0 + 16 * t + col;
      x[t] = Seen{0, q < s.R ? s.seen(a, q) : 0, 0, 0.f};
    }
  } else {
    long at[NT];
    int lo[NT], hi[NT];
    float slope[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int q = min(q0 + 16 * t + col, s.R - 1);
      at[t] = s.token(a, q);
      x[t].pos = s.seen(a, q) - 1;
      lo[t] = 0;
      hi[t] = x[t].pos + 1;
      if constexpr (SC & SC_SLOPES) slope[t] = a.sc.slopes[s.head(a, q)];
    }
    if (a.sc.begin) {
#pragma unroll
      for (int t = 0; t < NT; ++t) lo[t] = a.sc.begin[at[t]];
    }
    if (a.sc.end) {
#pragma unroll
      for (int t = 0; t < NT; ++t) hi[t] = a.sc.end[at[t]];
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      lo[t] = max(lo[t], a.sc.window ? max(x[t].pos + 1 - a.sc.window, 0) : 0);
      hi[t] = min(hi[t], s.t.past + s.t.n);
      const bool is = q0 + 16 * t + col < s.R;
      x[t].low = is && lo[t] < hi[t] ? lo[t] : 0;
      x[t].limit = is && lo[t] < hi[t] ? hi[t] : 0;
      x[t].slope = SC & SC_SLOPES && is ? slope[t] * 1.4426950408889634f / factor<SC>(a) : 0.f;
    }
  }
}
// What queries see together: some of them positions from .. upto - 1, each of them all .. any - 1.
struct Span {
  int from, upto, all, any;
  __device__ void join(const Span &x) {
    from = min(from, x.from);
    upto = max(upto, x.upto);
    all = max(all, x.all);
    any = min(any, x.any);
  }
  template <int NT>
  __device__ static Span of(const Share &s, int q0, const Seen (&x)[NT]) {  // of a wave's tiles
    Span r{1 << 30, 0, 0, 1 << 30};
#pragma unroll
    for (int t = 0; t < NT; ++t)
      if (q0 + 16 * t + (int)(threadIdx.x & 15) < s.R) {
        const bool none = x[t].low >= x[t].limit;
        r.join(Span{none ? 1 << 30 : x[t].low, x[t].limit, none ? 1 << 30 : x[t].low, x[t].limit});
      }
    r.join(r.turned<8>());
    r.join(r.turned<4>());
    r.join(r.turned<2>());
    r.join(r.turned<1>());
    return r.uniform();
  }
  template <int N>
  __device__ Span turned() const {  // that of the lane N places on, of 16
    auto of = [](int x) { return __builtin_amdgcn_mov_dpp(x, 0x120 + N, 0xF, 0xF, true); };
    return Span{of(from), of(upto), of(all), of(any)};
  }
  __device__ Span uniform() const {
    auto one = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    return Span{one(from), one(upto), one(all), one(any)};
  }
};
// the blocks of a workgroup whose queries see `x` together
template <int SC>
__device__ inline void take(const KvAttend &a, Share &s, const Span &x) {
  s.take(a, x.from, min(x.upto, s.held));
  // (with slopes: where distances have a sign)
  const int any = min(SC & SC_SLOPES ? min(x.any, s.seen(a, s.q0)) : x.any, s.held);
  s.whole_lo = min(max((x.all + 31) >> 5, s.lo), max(s.hi, s.lo));
  s.whole_hi = max(min(any >> 5, s.hi), s.whole_lo);
}
// Where the scores of a block begin; from: distance of the query from the lane's first position; before: no position lies behind it.
// (A distance is exact up to 2^24, and beyond to 2^-24 of itself.)
template <int SC>
__device__ inline void share_of(bool before, float slope, int from, floatx4 (&S)[2]) {
  if constexpr (SC & SC_SLOPES) {
    const float d = (float)from;
    if (before) {
      const float b = -slope * d;
#pragma unroll
      for (int j = 0; j < 8; ++j) S[j >> 2][j & 3] = __builtin_fmaf(slope, (float)block_pos(j, 0), b);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) S[j >> 2][j & 3] = -slope * __builtin_fabsf(d - (float)block_pos(j, 0));
    }
  } else {
    S[0] = S[1] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
}
// LATE: the share is added at the end, as it is to capped scores (one tile of 128-wide heads has no registers for it before).
template <int SC, bool LATE>
__device__ inline void begin_scores(bool before, const Seen &x, int base, floatx4 (&S)[2]) {
  share_of<LATE || SC & SC_CAP ? 0 : SC>(before, x.slope, x.pos - base, S);
}
template <int SC, bool LATE>
__device__ inline void end_scores(const KvScoring &sc, bool before, const Seen &x, int base, floatx4 (&S)[2]) {
  if constexpr (SC & SC_CAP) {
#pragma unroll
    for (int j = 0; j < 8; ++j) S[j >> 2][j & 3] = capped(sc.in, S[j >> 2][j & 3]);
  }
  if constexpr (SC & SC_SLOPES && (LATE || SC & SC_CAP)) {
    floatx4 B[2];
    float slope = x.slope;
    if constexpr (LATE) asm volatile("" : "+v"(slope), "+v"(S[0]), "+v"(S[1]));  // (not before the products, where registers are few)
    share_of<SC>(before, slope, x.pos - base, B);
    S[0] += B[0];
    S[1] += B[1];
  }
}
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
// The numerators of a wave's tiles again, over blocks first, first + step, ... below end (SC: in their order) of bf16 pages, against the references
// that the wave has arrived at: values without their infinities and NaNs, which are then added.
template <int DH, int SC, bool LAST_FIRST, typename SeenOf, typename Tile, int NT>
__device__ __forceinline__ void sums_again(const KvAttend &a, const Share &s, int q0, SeenOf seen_of, int first, int step, int end, Tile (&tile)[NT]) {
  constexpr int QC = DH / 32, VM = DH / 16;
  const int lane = threadIdx.x & 63, grp = lane >> 4, col = lane & 15, bpp = a.kv.g.page_tokens >> 5;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int m = 0; m < VM; ++m) tile[t].O[m] = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int at = first; at < end; at += step) {
    const int blk = SC ? s.block<LAST_FIRST>(at) : at, page = page_of(a.kv, s.r, blk);
    if (page < 0) continue;
    const uint32x4 *src = (const uint32x4 *)(a.kv.pool + (long)page * a.kv.page_bytes + ((long)s.h * bpp + blk % bpp) * (128 * DH)) + lane;
    const Keep keep(s.held - blk * 32, grp);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      bf16x8 qf[QC];
      load_queries<DH>(a, s, q0 + 16 * t + col, grp, qf);
      const Seen x = seen_of(t);
      const int lim = x.limit - blk * 32, lo = x.low - blk * 32;
      floatx4 S[2];
      begin_scores<SC, true>(false, x, blk * 32 + 4 * grp, S);
#pragma unroll
      for (int tl = 0; tl < 2; ++tl) {
#pragma unroll
        for (int c = 0; c < QC; ++c) S[tl] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, src[(tl * QC + c) * 64]), qf[c], S[tl], 0, 0, 0);
      }
      end_scores<SC, true>(a.sc, false, x, blk * 32 + 4 * grp, S);
      float p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        p[j] = hidden<SC != 0>(j, lo, lim, grp) ? 0.f : __builtin_amdgcn_exp2f(__builtin_fmaf(S[j >> 2][j & 3], factor<SC>(a), -tile[t].m_ref));
      const bf16x8 pv = pack8(p), vis = visible<SC != 0>(lo, lim, grp);
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
// workgroups by k_kv_merge.  Bound by the bytes of the pages; 4 bits by the vector units too (two conversions and a permutation for
// four values; a step of 128 rows of 1024, 32 heads of 128, 75 us: 5.8 TB/s with the vector units at work in 63 % of all cycles).
template <int DH, int EL>
struct KvBlock {
  uint32x4 k[key_pieces(DH, EL)], v[value_pieces(DH, EL)];
  uint32_t ke[2], ve[EL == EL_FP4 ? DH / 16 : 2];  // exponents: of key 16 tl + (lane & 15) (K), of keys 16 tl + 4 (lane >> 4) .. + 3 (V)
};
template <int DH, int EL, int SC, int NT, int NW>
__global__ __launch_bounds__(NW * 64, NT == 1 ? 4 : 2) void k_kv_attend(KvAttend a, int pairs) {
  constexpr bool FP8 = EL == EL_FP8, FP4 = EL == EL_FP4, LOOKS = looks(EL, SC);
  constexpr int QC = DH / 32, VM = DH / 16, NQ = 16 * NT;
  // One tile of 128-wide heads keeps its queries in LDS: with them in registers the loop did not fit the 128 of 4 waves a SIMD.
  constexpr bool LDS_Q = NT == 1 && DH == 128;
  __shared__ bf16x8 sh_q[LDS_Q ? QC * 64 : 1];
  // (and what else is known of a query, if scores are changed)
  __shared__ Seen sh_seen[SC && LDS_Q ? 16 : 1];
  __shared__ int sh_new[16];                           // (whether it sees the new token; of one tile)
  __shared__ __align__(16) bf16_t sh_k[DH], sh_v[DH];  // the new token
  extern __shared__ float lds[];                       // [NW][cols][DH + 2]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, grp = lane >> 4, col = lane & 15;
  const bool files = NT == 1 && a.k.p != nullptr;  // (t.n is 1: the token is not in the cache yet)
  Share s = Share::of<NQ, SC>(a, pairs, files);
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
  Seen seen[NT];                  // of the lane's queries, positions of the cache
  QueryTile<DH, NT == 1> tile[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int q = q0 + 16 * t + col;
    load_queries<DH>(a, s, q, grp, qf[t]);
    tile[t].clear();
  }
  see<SC>(a, s, q0, seen);
  if (SC && NT == 1 && wave == 0 && grp == 0) sh_new[col] = seen[0].low <= s.held && s.held < seen[0].limit;
#pragma unroll
  for (int t = 0; t < NT; ++t) seen[t].limit = min(seen[t].limit, s.held);
  if constexpr (SC) take<SC>(a, s, Span::of(s, q0, seen));
  if constexpr (LDS_Q) {
    if (wave == 0) {
#pragma unroll
      for (int c = 0; c < QC; ++c) sh_q[c * 64 + lane] = qf[0][c];
      if (SC && grp == 0) sh_seen[col] = seen[0];
    }
  }
  if constexpr (LDS_Q || (SC && NT == 1)) __syncthreads();
  typedef KvBlock<DH, EL> Block;
  auto load = [&](int page, int ib, Block &b) {
    const unsigned char *pg = a.kv.pool + (long)page * a.kv.page_bytes;
    const long at = (long)h * bpp + ib;
    const uint32x4 *src = (const uint32x4 *)(pg + at * block_bytes(DH, EL)) + lane;
    constexpr int KF = key_pieces(DH, EL), VF = value_pieces(DH, EL);
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
    if constexpr (FP4) {
      const unsigned char *ex = pg + at * block_bytes(DH, EL) + 32 * DH;
#pragma unroll
      for (int i = 0; i < DH / 64; ++i) b.ke[i] = ((const uint32_t *)(ex + col * (DH / 16)))[i];
#pragma unroll
      for (int i = 0; i < DH / 64; ++i) *(uint32x4 *)&b.ve[4 * i] = ((const uint32x4 *)(ex + DH + grp * (DH / 4)))[i];
    }
  };
  auto seen_of = [&](int t) {
    if constexpr (!SC || !LDS_Q) return seen[t];
    int at = threadIdx.x;
    asm volatile("" : "+v"(at)::"memory");  // (read where it is needed, not kept, nor its place)
    return sh_seen[at & 15];
  };

  // base: first position of the block; valid: positions that the row has
  auto use = [&](auto masked_, int base, Block &b, int valid) {
    constexpr bool masked = decltype(masked_)::value;
    floatx4 S[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) begin_scores<SC, LDS_Q>(!masked, seen_of(t), base + 4 * grp, S[t]);
#pragma unroll
    for (int c = 0; c < QC; ++c) {
      bf16x8 x[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) x[t] = LDS_Q ? sh_q[c * 64 + lane] : qf[t][c];
#pragma unroll
      for (int tl = 0; tl < 2; ++tl) {
        const bf16x8 kf = key_fragment<DH, EL>(b.k, b.ke, tl, c);
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t][tl] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, x[t], S[t][tl], 0, 0, 0);
      }
    }
    if constexpr (FP8 && LOOKS && masked) {  // (positions of such codes hold NaN)
      if (uint32_t bad[2]; odd_codes(b.v, bad)) {
        b.ve[0] |= bad[0];
        b.ve[1] |= bad[1];
      }
    }
    float vs[8];
    if constexpr (FP8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) vs[j] = kv8_factor(b.ve[j >> 2], j & 3);
    }
    bf16x8 pv[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const Seen x = seen_of(t);
      end_scores<SC, LDS_Q>(a.sc, !masked, x, base + 4 * grp, S[t]);
      pv[t] = tile[t].template weights<FP8, SC != 0>(masked, S[t], factor<SC>(a), x.low - base, x.limit - base, grp, vs);
    }
    if constexpr (FP4) {
      if constexpr (masked) {
        int from[NT], to[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const Seen x = seen_of(t);
          from[t] = x.low - base;
          to[t] = x.limit - base;
        }
        odd_exponents<DH, SC != 0, NT>(b.v, b.ve, tile, from, to);
      }
#pragma unroll
      for (int i = 0; i < DH / 32; ++i) {
        bf16x8 vf[2];
        widen4_values({b.v[i / 2][i % 2 * 2], b.v[i / 2][i % 2 * 2 + 1]}, {b.ve[2 * i], b.ve[2 * i + 1]}, vf);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int t = 0; t < NT; ++t) tile[t].O[2 * i + u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[u], pv[t], tile[t].O[2 * i + u], 0, 0, 0);
      }
      return;
    }
    if (masked && !LOOKS) {
      const Keep keep(valid - base, grp);
      if constexpr (FP8) {  // (codes of positions that the row does not have may be NaN)
#pragma unroll
        for (int m = 0; m < VM / 2; ++m) b.v[m] &= uint32x4{keep.codes(0), keep.codes(1), keep.codes(0), keep.codes(1)};
      } else if constexpr (EL == EL_BF16) {
#pragma unroll
        for (int m = 0; m < VM; ++m) keep.bf16(b.v[m]);
      }
    }
#pragma unroll
    for (int m = 0; m < (FP4 ? 0 : VM); ++m) {
      bf16x8 vf{};
      if constexpr (FP8) {
        vf = widen(b.v[m / 2][m % 2 * 2], b.v[m / 2][m % 2 * 2 + 1], 127);
      } else {
        vf = __builtin_bit_cast(bf16x8, b.v[m]);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) tile[t].O[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pv[t], tile[t].O[m], 0, 0, 0);
    }
  };
  // place of the wave's next block, whose page's number is asked for ahead of the use of the one before
  const int32_t *table = a.kv.table + (long)s.r * a.kv.g.max_pages;
  int blk = SC ? wave : s.lo + wave, ip, ib;  // (SC: in their order)
  auto place = [&]() {
    const int b = SC ? s.block<(SC & SC_SLOPES) != 0>(blk) : blk;
    ip = b / bpp;
    ib = b % bpp;
  };
  place();
  auto entry = [&]() { return table[min(ip, a.kv.g.max_pages - 1)]; };
  int number = entry();
  const int end = SC ? s.hi - s.lo : s.hi, masked_from = SC ? s.wholes() : min(s.whole_hi, s.hi);
  // the wave's next block into b, and its first position; negative: it has no page
  auto fetch = [&](Block &b) {
    const bool is = number >= 0 && number < a.kv.pages && ip < a.kv.g.max_pages;
    if (is) load(number, ib, b);
    const int base = is ? (SC ? s.block<(SC & SC_SLOPES) != 0>(blk) : blk) * 32 : -1;
    blk += NW;
    if constexpr (SC) {
      place();
    } else {
      ip += NW / bpp;
      ib += NW % bpp;
      if (ib >= bpp) {
        ib -= bpp;
        ++ip;
      }
    }
    number = entry();
    return base;
  };
  if constexpr (FP4 && NT == 1 && DH == 128 && !SC) {
    // Blocks are small: the next one is on its way while one is used (128 rows of 1024, 32 heads: 83 -> 79 us; one row of 32766, 8 kv
    // heads 15.8 -> 15.1).  Where fewer registers are left, or more queries to compute for, it costs: heads of 64 45 -> 49, two tiles 27.6 -> 28.4.
    // With changed scores, so written, the blocks went through scratch memory: 128 rows of 1023, slopes 96 -> 447, a cap 96 -> 447; 32 rows 30 -> 118.
    Block b;
    int at = blk, base = at < end ? fetch(b) : -1;
    auto step = [&](auto masked_) {
      Block next;
      at = blk;
      const int next_base = at < end ? fetch(next) : -1;
      if (base >= 0) use(masked_, base, b, s.held);
      b = next;
      base = next_base;
    };
    while (at < masked_from) step(std::false_type());
    while (at < end) step(std::true_type());
  } else {
    auto step = [&](auto masked_) {
      Block b;
      const int base = fetch(b);
      if (base >= 0) use(masked_, base, b, s.held);
    };
    while (blk < masked_from) step(std::false_type());
    while (blk < end) step(std::true_type());
  }
  if constexpr (EL == EL_BF16) {
    if (__builtin_expect(not_finite<DH>(tile), 0)) sums_again<DH, SC, (SC & SC_SLOPES) != 0>(a, s, q0, seen_of, SC ? wave : s.lo + wave, NW, SC ? s.hi - s.lo : s.hi, tile);
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
        if constexpr (FP4) {
          const uint32_t e = kv4_exponent(max_over_quarters(max_bits(kx)));
          kf = widen4(kv4_codes(kx, e), scale4(e, 0));
        }
        S = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, LDS_Q ? sh_q[c * 64 + lane] : qf[0][c], S, 0, 0, 0);
      }
      auto &x = tile[0];
      float score = __shfl(S[0], col);
      const bool sees = !SC || sh_new[col];
      if constexpr (SC) {  // (at a distance of 0)
        if constexpr (SC & SC_CAP) score = capped(a.sc.in, score);
        score *= factor<SC>(a);
        if (!sees) score = -INFINITY;
      } else {
        score *= a.c;
      }
      const float m_new = fmaxf(x.m_ref, score);
      const float alpha = __builtin_amdgcn_exp2f(x.m_ref - m_new), p = __builtin_amdgcn_exp2f(score - m_new);
      x.m_ref = m_new;
      x.L[0] = x.L[0] * alpha + p;
      uint32_t e4[DH / 32];
      if constexpr (FP4) {
#pragma unroll
        for (int i = 0; i < DH / 32; ++i) {
          const uint2 lo = *(const uint2 *)&sh_v[32 * i + 4 * grp], hi = *(const uint2 *)&sh_v[32 * i + 16 + 4 * grp];
          e4[i] = kv4_exponent(max_over_quarters(max_bits(uint32x4{lo.x, lo.y, hi.x, hi.y})));
        }
      }
#pragma unroll
      for (int m = 0; m < VM; ++m) {
        const uint2 vx = *(const uint2 *)&sh_v[16 * m + 4 * grp];
        float v[4] = {bf2f(vx.x & 0xffffu), bf2f(vx.x >> 16), bf2f(vx.y & 0xffffu), bf2f(vx.y >> 16)};
        if constexpr (FP8) {
          const uint32_t w = ve == 255 ? 0u : kv8_pack(v[0], v[1], v[2], v[3], ve);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = kv8_value(w, i, kv8_scale(ve));
        }
        if constexpr (FP4) {
          const uint32_t e = e4[m / 2], w = e == 255 ? 0u : kv4_pair<1>(kv4_pair<0>(0, v[0], v[1], e), v[2], v[3], e);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = kv4_values(w >> (4 * (i & 2)) & 255u, e)[i & 1];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (SC) {
            if (!sees) v[i] = 0.f;  // (no 0 x infinity)
          }
          x.O[m][i] = x.O[m][i] * alpha + p * v[i];
        }
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
        else if constexpr (FP4) {
          const uint32_t e = kv4_exponent(max_over<4>(max_bits(kx)));
          *(uint32_t *)(pg + kv4_k_off(h, slot, 8 * lane, a.kv.g)) = kv4_codes(kx, e);
          if (lane % 4 == 0) pg[kv4_k_exp_off(h, slot, lane / 4, a.kv.g)] = (unsigned char)e;
        } else *(uint32x4 *)((bf16_t *)pg + kv_k_off(h, slot, 8 * lane, a.kv.g)) = kx;
      }
      if constexpr (FP4) {
        if (lane < DH / 2) {
          const int e = lane / 16 * 32 + lane % 16;
          const uint32_t lo = sh_v[e], hi = sh_v[e + 16], ex = kv4_exponent(max_over<16>(max((lo << 16) & 0x7fffffffu, (hi << 16) & 0x7fffffffu)));
          pg[kv4_v_off(h, slot, e, a.kv.g)] = ex == 255 ? 0 : (unsigned char)kv4_pair<0>(0, bf2f(lo), bf2f(hi), ex);
          if (lane % 16 == 0) pg[kv4_v_exp_off(h, slot, lane / 16, a.kv.g)] = (unsigned char)ex;
        }
      }
#pragma unroll
      for (int i = 0; i < (FP4 ? 0 : DH / 64); ++i) {
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
// block at a time, fragments requested as they are needed): us of short runs, 8 rows of up to 512 new tokens behind 2048, 32 heads of 128, bf16
// 143 -> 136 (130 of continued ones); 2 rows of 1023 behind 8193, 32 queries' and 8 kv heads, 8 bits 404 -> 339.  Bound by the vector units (softmax;
// conversions take two thirds again) and the matrix cores in turns, with two waves a SIMD; four tiles a wave do not fit.  4 bits, the same 8 rows:
// 144 us (8 bits 143), the vector units at work in 51 % of all cycles, the matrix cores in 25.  What a workgroup with
// changed scores takes before its first block is its rows' place, the ranges of its tokens and a page's number, one after the other; the
// queries come meanwhile (2 prompts of 2047 in windows of 1: 24.7 -> 23.4 us, of which their bytes are 16).
constexpr int rows_stages(int dh, int el) { return el != EL_BF16 ? 8 : dh == 128 ? 5 : 6; }  // (64: three workgroups, 97 -> 77 us for 32 prompts of 512)
constexpr size_t rows_lds(int dh, int el) { return (size_t)rows_stages(dh, el) * ((key_pieces(dh, el) + value_pieces(dh, el)) * 1024 + (el != EL_BF16 ? 256 : 0)); }
template <int DH, int EL, int SC>
__global__ __launch_bounds__(256, SC && DH == 64 ? 3 : 2) void k_kv_attend_rows(KvAttend a, int pairs) {
  constexpr bool FP8 = EL == EL_FP8, FP4 = EL == EL_FP4, LOOKS = looks(EL, SC);
  constexpr int QC = DH / 32, VM = DH / 16, NT = 2, NW = 4, NS = rows_stages(DH, EL), NQ = 16 * NT * NW;
  constexpr int KF = key_pieces(DH, EL), FR = KF + value_pieces(DH, EL), LPW = FR < NW ? 1 : FR / NW;  // fragments a stage, loads of a wave
  constexpr int STAGE = FR * 64 + (FP8 || FP4 ? 16 : 0);  // 16-byte pieces; behind 8- and 4-bit blocks 256 bytes for their exponents
  extern __shared__ uint32x4 ring[];               // [NS][STAGE]
  // 64-wide heads: three workgroups a CU, if what is known of the queries is not kept in registers
  constexpr bool LDS_SEEN = SC && DH == 64;
  __shared__ Seen sh_seen[LDS_SEEN ? NQ : 1];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, grp = lane >> 4, col = lane & 15;
  Share s = Share::of<NQ, SC>(a, pairs, false);
  if (!s.any) return;
  const int q0 = s.q0 + wave * (16 * NT), R = s.R, h = s.h, H = a.kv.g.H, bpp = a.kv.g.page_tokens >> 5;
  const bool busy = q0 < R;
  bf16x8 qf[NT][QC];
  Seen seen[NT];
  QueryTile<DH, false> tile[NT];
  if constexpr (SC) {  // (on their way while the ranges are waited for)
#pragma unroll
    for (int t = 0; t < NT; ++t) load_queries<DH>(a, s, q0 + 16 * t + col, grp, qf[t]);
  }
  see<SC>(a, s, q0, seen);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (LDS_SEEN && grp == 0) sh_seen[wave * (16 * NT) + 16 * t + col] = seen[t];  // (read by this wave alone)
    tile[t].clear();
  }
  auto seen_of = [&](int t) {
    if constexpr (!LDS_SEEN) return seen[t];
    int at = threadIdx.x;
    asm volatile("" : "+v"(at)::"memory");  // (read where it is needed, not kept, nor its place)
    return sh_seen[wave * (16 * NT) + 16 * t + (at & 15)];
  };
  int from_blk = 0, last = 0;  // this wave's blocks
  if constexpr (SC) {
    Span *spans = (Span *)(ring + (NS - 1) * STAGE), mine = Span::of(s, q0, seen);  // (a stage that nothing is requested into before the first barrier of the loop)
    if (lane == 0) spans[wave] = mine;
    __syncthreads();
    Span every = spans[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) every.join(spans[w]);
    take<SC>(a, s, every.uniform());
    from_blk = mine.from >> 5;
    last = min((mine.upto + 31) >> 5, s.hi);
  } else {
    last = busy ? min((s.seen(a, min(q0 + 16 * NT, R) - 1) + 31) >> 5, s.hi) : 0;
  }
  // Blocks are requested in order.  Lane l holds page 64 w + l of the row, for the window w of 64 pages that the next block is
  // in, waited for where it is loaded; a block without a page is loaded from page 0 and masked, as is every block from the
  // moment on at which a window has an entry that is no page.
  const int32_t *table = a.kv.table + (long)s.r * a.kv.g.max_pages;
  constexpr bool BACK = (SC & SC_SLOPES) != 0;     // whole blocks from the last one on
  const int begin = SC ? s.block<BACK>(0) : s.lo;
  int ip = begin / bpp, ib = begin % bpp, pages = 0, window = -1;
  uint32_t none = 0;                               // a bit for each stage: its block has no page
  int into = 0, from = 0, asked = SC ? 0 : s.lo;   // stages of the next block requested and used; blocks requested (SC: in their order)
  int turn = SC ? s.wholes() : 0;                  // SC: the next block that does not follow on the one before
  bool gaps = false;
  const int ip_end = (s.hi + bpp - 1) / bpp, asked_end = SC ? s.hi - s.lo : s.hi;
  const uint32x4 *src = nullptr;                   // this wave's part of the next block
  const unsigned char *ex_src = nullptr;           // its exponents
  bool is = false;
  const int part = FR < NW ? wave % FR : wave * LPW;  // (fewer fragments than waves: two waves load the same one)
  auto next = [](int stage) { return stage == NS - 1 ? 0 : stage + 1; };
  auto new_page = [&]() {
    if (ip >> 6 != window) {
      window = ip >> 6;
      const int at = window * 64 + lane;
      pages = at < a.kv.g.max_pages ? table[at] : -1;
      asm volatile("" : "+v"(pages));
      gaps |= __any(at >= (BACK ? s.lo / bpp : ip) && at < ip_end && (pages < 0 || pages >= a.kv.pages));
    }
    int page = __builtin_amdgcn_readlane(pages, ip & 63);
    is = page >= 0 && page < a.kv.pages;
    if (!is) page = 0;
    const unsigned char *pg = a.kv.pool + (long)page * a.kv.page_bytes;
    const long at = (long)h * bpp + ib;
    src = (const uint32x4 *)(pg + at * block_bytes(DH, EL)) + part * 64;
    ex_src = FP4 ? pg + at * block_bytes(DH, EL) + 32 * DH : pg + (long)H * bpp * (64 * DH) + at * 64;
  };
  if (s.lo < s.hi) new_page();
  auto request = [&]() {
    none = (none & ~(1u << into)) | (uint32_t)!is << into;
    uint32x4 *dst = ring + into * STAGE + part * 64;
#pragma unroll
    for (int i = 0; i < LPW; ++i)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)&(src + i * 64)[lane],
                                       (__attribute__((address_space(3))) void *)(dst + i * 64), 16, 0, 0);
    if constexpr (FP8)  // every wave, so that all wait for the same number of loads; lanes 16 .. 63 repeat
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(ex_src + 4 * col),
                                       (__attribute__((address_space(3))) void *)(ring + into * STAGE + FR * 64), 4, 0, 0);
    if constexpr (FP4)  // (64-wide heads: lanes 32 .. 63 repeat)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(ex_src + 4 * (lane % (DH / 2))),
                                       (__attribute__((address_space(3))) void *)(ring + into * STAGE + FR * 64), 4, 0, 0);
    into = next(into);
    ++asked;
    if constexpr (BACK) {
      const int blk = s.block<true>(asked);
      ip = blk / bpp;
      ib = blk % bpp;
      if (asked < asked_end) new_page();
      return;
    }
    src += block_bytes(DH, EL) / 16;
    ex_src += FP4 ? block_bytes(DH, EL) : 64;
    bool other = ++ib == bpp;  // page
    if (other) {
      ib = 0;
      ++ip;
    }
    if (SC && asked == turn) {  // (behind the whole ones, and where these were)
      const int blk = s.block<BACK>(asked);
      turn = turn == s.wholes() ? s.whole_hi - s.lo : 0;
      ip = blk / bpp;
      ib = blk % bpp;
      other = true;
    }
    if (other && ip < ip_end) new_page();
  };
  constexpr int LOADS = LPW + (FP8 || FP4 ? 1 : 0);
  auto queries_here = [&]() {  // (waited for inside the loop, the queries would make the compiler wait for the ring as well)
    wait_vmcnt<0>();
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < QC; ++c) asm volatile("" : "+v"(qf[t][c]));
  };
  if constexpr (SC) queries_here();
  for (int i = 0; i < NS - 2; ++i)
    if (asked < asked_end) request();
  if constexpr (!SC) {
#pragma unroll
    for (int t = 0; t < NT; ++t) load_queries<DH>(a, s, q0 + 16 * t + col, grp, qf[t]);
    queries_here();
  }

  // scores of a block: S[t][tl][i] of position 16 tl + 4 grp + i
  auto scores = [&](int stage, int base, bool before, floatx4 (&S)[NT][2]) {
    const uint32x4 *kv = ring + stage * STAGE + lane;
    const unsigned char *ex = (const unsigned char *)(ring + stage * STAGE + FR * 64);
    uint32x4 kw[KF];
#pragma unroll
    for (int i = 0; i < KF; ++i) kw[i] = kv[i * 64];
    uint32_t ke[2] = {FP8 ? ex[col] : 0u, FP8 ? ex[16 + col] : 0u};
    if constexpr (FP4) {
#pragma unroll
      for (int i = 0; i < DH / 64; ++i) ke[i] = ((const uint32_t *)(ex + col * (DH / 16)))[i];
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) begin_scores<SC, false>(before, seen_of(t), base + 4 * grp, S[t]);
#pragma unroll
    for (int c = 0; c < QC; ++c)
#pragma unroll
      for (int tl = 0; tl < 2; ++tl) {
        const bf16x8 kf = key_fragment<DH, EL>(kw, ke, tl, c);
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t][tl] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][c], S[t][tl], 0, 0, 0);
      }
  };
  auto factor_words = [&](int stage, uint32_t (&ve)[2]) {
    const uint32_t *ex = (const uint32_t *)(ring + stage * STAGE + FR * 64);
    ve[0] = ex[8 + grp];
    ve[1] = ex[12 + grp];
  };
  auto exponents4 = [&](int stage, uint32_t (&ve)[DH / 16]) {
    const uint32x4 *ex = (const uint32x4 *)((const unsigned char *)(ring + stage * STAGE + FR * 64) + DH + grp * (DH / 4));
#pragma unroll
    for (int i = 0; i < DH / 64; ++i) *(uint32x4 *)&ve[4 * i] = ex[i];
  };
  auto add_values4 = [&](const uint32x4 (&vw)[FR - KF], const uint32_t (&ve)[DH / 16], const bf16x8 (&pv)[NT]) {
#pragma unroll
    for (int i = 0; i < DH / 32; ++i) {
      bf16x8 vf[2];
      widen4_values({vw[i / 2][i % 2 * 2], vw[i / 2][i % 2 * 2 + 1]}, {ve[2 * i], ve[2 * i + 1]}, vf);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int t = 0; t < NT; ++t) tile[t].O[2 * i + u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[u], pv[t], tile[t].O[2 * i + u], 0, 0, 0);
    }
  };
  auto add_values = [&](const uint32x4 (&vw)[FR - KF], const bf16x8 (&pv)[NT]) {
#pragma unroll
    for (int m = 0; m < (FP4 ? 0 : VM); ++m) {
      bf16x8 vf{};
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
    scores(from, base, false, S);
    float vs[8];
    if constexpr (FP8) {
      uint32_t ve[2];
      factor_words(from, ve);
#pragma unroll
      for (int j = 0; j < 8; ++j) vs[j] = kv8_factor(ve[j >> 2], j & 3);
    }
    bf16x8 pv[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const Seen x = seen_of(t);
      end_scores<SC, false>(a.sc, false, x, base + 4 * grp, S[t]);
      pv[t] = tile[t].template weights<FP8, SC != 0>(true, S[t], factor<SC>(a), x.low - base, no_page ? 0 : x.limit - base, grp, vs);
    }
    uint32x4 vw[FR - KF];
    values_of(from, vw);
    int lo[NT], to[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const Seen x = seen_of(t);
      lo[t] = x.low - base;
      to[t] = no_page ? 0 : x.limit - base;
    }
    if constexpr (FP4) {
      uint32_t ve[DH / 16];
      exponents4(from, ve);
      odd_exponents<DH, SC != 0, NT>(vw, ve, tile, lo, to);
      add_values4(vw, ve, pv);
    } else {
      if constexpr (FP8 && LOOKS) {
        if (uint32_t bad[2]; odd_codes(vw, bad)) {
#pragma unroll
          for (int t = 0; t < NT; ++t) {  // (a weight of NaN for a query that sees any)
            bool sees = false;
#pragma unroll
            for (int j = 0; j < 8; ++j) sees |= (bad[j >> 2] >> (8 * (j & 3)) & 255u) && !hidden<SC != 0>(j, lo[t], to[t], grp);
            if (sees) pv[t][0] = (__bf16)__uint_as_float(0x7fc00000u);
          }
        }
      }
      add_values(vw, pv);
    }
  };
  // Two blocks that every query sees whole: one branch for all of their weights, so that from there on exponentials and products
  // are formed side by side, and the values are on their way before.
  auto use_two = [&](int one, int two, int base) {
    constexpr int STEP = BACK ? -32 : 32;  // from one to the other
    const int stage[2] = {one, two};
    const float c = factor<SC>(a);
    floatx4 S[2][NT][2];
    uint32_t ve[2][2];
    int power[2][8];  // of the values; 2 rows of 1023 behind 8193, 8 bits, us: by ldexp 338, as factors, 0 for byte 0, 341, as they are 358
    uint32x4 vw[FR - KF];
    bool raise = false;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      __builtin_amdgcn_s_setprio(1);  // (before the other waves' exponentials: 140 -> 136 us)
      scores(stage[u], base + STEP * u, true, S[u]);
      __builtin_amdgcn_s_setprio(0);
      if constexpr (FP8) {
        factor_words(stage[u], ve[u]);
#pragma unroll
        for (int j = 0; j < 8; ++j) power[u][j] = (int)(ve[u][j >> 2] >> (8 * (j & 3)) & 255u) - 127;
#pragma unroll
        for (int i = 0; i < 2; ++i) raise |= (((ve[u][i] & 0x7f7f7f7fu) + 0x01010101u) & ve[u][i] & 0x80808080u) != 0;
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) end_scores<SC, false>(a.sc, true, seen_of(t), base + STEP * u + 4 * grp, S[u][t]);
    }
    values_of(stage[0], vw);
    float p[2][NT][8];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        tile[t].relative(S[u][t], c, p[u][t]);
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
        tile[t].raise(most * c);
#pragma unroll
        for (int u = 0; u < 2; ++u) tile[t].relative(S[u][t], c, p[u][t]);
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
      if constexpr (FP4) {
        uint32_t e[DH / 16];
        exponents4(stage[u], e);
        add_values4(vw, e, pv);
      } else {
        add_values(vw, pv);
      }
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
      else if constexpr (EL == EL_BF16) keep.bf16(x);
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
    while (asked < min(asked_end, blk + NS)) request();
  };
  auto single = [&](int at) {
    open(at, 1);
    const int blk = SC ? s.block<BACK>(at) : at;
    const bool no_page = none >> from & 1;
    if (!LOOKS && (no_page || blk * 32 + 32 > s.held)) clear(no_page ? 0 : s.held - blk * 32);
    if (blk < last && (!SC || blk >= from_blk)) use(blk, no_page);
    from = next(from);
  };
  auto pair = [&](int at) {
    open(at, 2);
    const int blk = SC ? s.block<BACK>(at) : at;
    const int second = next(from);
    if (busy) use_two(from, second, blk * 32);
    from = next(second);
  };
  int blk = s.lo;
  if constexpr (SC) {
    int v = 0;
    for (; v + 2 <= s.wholes() && !gaps; v += 2) pair(v);
    for (; v < s.hi - s.lo; ++v) single(v);
  } else {
    for (; blk + 2 <= min(s.whole_hi, s.hi) && !gaps; blk += 2) pair(blk);
    for (; blk < s.hi; ++blk) single(blk);
  }
  if constexpr (EL == EL_BF16) {
    if (__builtin_expect(not_finite<DH>(tile), 0)) sums_again<DH, SC, false>(a, s, q0, seen_of, SC ? 0 : s.lo, 1, SC ? s.hi - s.lo : last, tile);
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

template <int DH, int EL, int SC, int NT, int NW>
void launch_attend(hipStream_t s, const KvAttend &a, dim3 grid, int pairs) {
  const int cols = std::min(16, a.tk.max_new * a.group);
  const size_t lds = (size_t)NW * cols * (DH + 2) * sizeof(float);
  static std::atomic<uint64_t> done{0};
  if (lds + 8192 > 64 * 1024) (void)allow_lds(done, {(const void *)k_kv_attend<DH, EL, SC, NT, NW>}, NW * 16 * (DH + 2) * sizeof(float));
  SKD_LAUNCH((k_kv_attend<DH, EL, SC, NT, NW>), grid, dim3(NW * 64), lds, s, a, pairs);
}
template <int DH, int EL, int SC>
void attend_pages(hipStream_t s, const KvAttend &a, const AttendPlan &p) {
  const dim3 grid((unsigned)(p.tiles * p.pairs), a.splits);
  if (p.nq == 128) {
    static std::atomic<uint64_t> done{0};
    if (rows_lds(DH, EL) > 64 * 1024) (void)allow_lds(done, {(const void *)k_kv_attend_rows<DH, EL, SC>}, rows_lds(DH, EL));
    SKD_LAUNCH((k_kv_attend_rows<DH, EL, SC>), grid, dim3(256), rows_lds(DH, EL), s, a, p.pairs);
  } else if (p.nq == 32) {
    launch_attend<DH, EL, SC, 2, 8>(s, a, grid, p.pairs);
  } else if (p.waves == 4) {
    launch_attend<DH, EL, SC, 1, 4>(s, a, grid, p.pairs);
  } else {
    launch_attend<DH, EL, SC, 1, 8>(s, a, grid, p.pairs);
  }
}
template <int EL, int SC>
void attend_elem(hipStream_t s, const KvAttend &a, const AttendPlan &p) {
  if (a.kv.g.dh == 64) attend_pages<64, EL, SC>(s, a, p);
  else attend_pages<128, EL, SC>(s, a, p);
}

}  // namespace

}  // namespace skd
