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
__global__ __launch_bounds__(256) void k_kv_append(KvView kv, KvTokens tk, KvRows k, KvRows v, int blocks) {
  constexpr int LPT = DH / 8, TPP = 256 / LPT;  // lanes a token, tokens a pass
  typedef typename std::conditional<FP8, uint8_t, uint16_t>::type code_t;
  __shared__ __align__(16) code_t sv[32][DH + 8];
  const int blk_i = blockIdx.x % blocks, h = blockIdx.x / blocks % kv.g.H, r = blockIdx.x / blocks / kv.g.H;
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

// ------------------------------------------------------------------ reading back
// As above, the other way: a workgroup reads the tokens of a row and kv head that lie in one block.  Bound by the fp32 rows
// that it writes.
template <int DH, bool FP8, typename OUT>
__global__ __launch_bounds__(256) void k_kv_read(KvView kv, KvTokens tk, KvRows k, KvRows v, int blocks) {
  constexpr int LPT = DH / 8, TPP = 256 / LPT;
  __shared__ float sv[32][DH + 1];
  const int blk_i = blockIdx.x % blocks, h = blockIdx.x / blocks % kv.g.H, r = blockIdx.x / blocks / kv.g.H;
  const RowTokens t = row_tokens(tk, r);
  const int blk = (t.past >> 5) + blk_i, lo = max(t.past, blk * 32), hi = min(t.past + t.n, blk * 32 + 32);
  if (t.n <= 0 || lo >= hi) return;
  const int page = page_of(kv, r, blk);
  if (page < 0) return;
  const unsigned char *pg = kv.pool + (long)page * kv.page_bytes;
  const int slot0 = (blk % (kv.g.page_tokens >> 5)) * 32;
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
  const int e = (threadIdx.x % LPT) * 8;
  for (int key = threadIdx.x / LPT; key < 32; key += TPP) {
    const int pos = blk * 32 + key;
    if (pos < lo || pos >= hi) continue;
    const long token = t.at + (long)(pos - t.past) * tk.step;
    float kx[8], vx[8];
    if constexpr (FP8) {
      const uint2 w = *(const uint2 *)(pg + kv8_k_off(h, slot0 + key, e, kv.g));
      const float sc = kv8_scale(pg[kv8_exp_off(h, slot0 + key, 0, kv.g)]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        kx[j] = kv8_value(w.x, j, sc);
        kx[4 + j] = kv8_value(w.y, j, sc);
      }
    } else {
      const uint32x4 w = *(const uint32x4 *)((const bf16_t *)pg + kv_k_off(h, slot0 + key, e, kv.g));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        kx[2 * j] = bf2f(w[j] & 0xffffu);
        kx[2 * j + 1] = bf2f(w[j] >> 16);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) vx[j] = sv[key][e + j];
    OUT *ko = (OUT *)k.p + row_index(k, token, h * DH + e), *vo = (OUT *)v.p + row_index(v, token, h * DH + e);
    if constexpr (sizeof(OUT) == 4) {
#pragma unroll
      for (int j = 0; j < 8; j += 4) {
        *(floatx4 *)(ko + j) = floatx4{kx[j], kx[j + 1], kx[j + 2], kx[j + 3]};
        *(floatx4 *)(vo + j) = floatx4{vx[j], vx[j + 1], vx[j + 2], vx[j + 3]};
      }
    } else {
      *(uint32x4 *)ko = uint32x4{pack2(kx[0], kx[1]), pack2(kx[2], kx[3]), pack2(kx[4], kx[5]), pack2(kx[6], kx[7])};
      *(uint32x4 *)vo = uint32x4{pack2(vx[0], vx[1]), pack2(vx[2], vx[3]), pack2(vx[4], vx[5]), pack2(vx[6], vx[7])};
    }
  }
}

// ------------------------------------------------------------------ attention
// A query tile is 16 of the R = new * group queries of a row and kv head, in the order (token, head of the group): the 16
// columns of the matrix instructions.  A workgroup is NW waves on one tile and one share of its keys; a wave takes every NW-th
// 32-key block, straight from the page into the operand registers, with a softmax of its own (as k_attention_rows: units of
// log2, a reference that is raised only by more than 8, denominators from the matrix cores); the waves' states are joined in
// LDS, the shares of several workgroups by k_kv_merge.
//
// Query i of a row sees positions up to past + i.  Blocks that reach beyond what the tile's first query sees are masked:
// scores by selection, and since 0 * infinity is not 0, values too: beyond the row's last position they are cleared (a page
// may hold anything there), and an infinity or NaN that only later queries see is kept out of the products and put into the
// sums of those that see it.  8-bit values are finite, what is not is in their scales, which are selected with the weights.
template <int DH, bool FP8>
struct KvBlock {
  static constexpr int QC = DH / 32, VM = DH / 16;
  uint32x4 k[FP8 ? QC : 2 * QC], v[FP8 ? VM / 2 : VM];
  uint32_t ke[2], ve[2];  // exponents: of keys 16 tl + (lane & 15) (K), of keys 16 tl + 4 (lane >> 4) .. + 3 (V)
};
// bf16x8 of two words of codes, times a power of two
__device__ inline bf16x8 widen(uint32_t a, uint32_t b, float scale) {
  const bf16x2 x[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true)};
  return bf16x8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
}

template <int DH, bool FP8, int NW>
__global__ __launch_bounds__(NW * 64, 4) void k_kv_attend(KvAttend a, int tiles) {
  constexpr int QC = DH / 32, VM = DH / 16;
  extern __shared__ float lds[];  // [NW][cols][DH + 2]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, grp = lane >> 4, col = lane & 15;
  const int H = a.kv.g.H, qt = blockIdx.x % tiles, h = blockIdx.x / tiles % H;
  const int ri = blockIdx.x / tiles / H, r = a.order ? a.order[ri] : ri;
  const RowTokens t = row_tokens(a.tk, r);
  const int R = t.n * a.group, q0 = qt * 16;
  if (q0 >= R) return;
  const bool files = a.k.p != nullptr;               // (t.n is 1: the token is not in the cache yet)
  const int held = t.past + (files ? 0 : t.n);       // positions that the cache holds
  const int seen0 = t.past + q0 / a.group + 1;       // positions that the first query of the tile sees
  const int seen1 = min(t.past + min(q0 + 15, R - 1) / a.group + 1, held);  // that the last one sees
  const int mine = q0 + col < R ? t.past + (q0 + col) / a.group + 1 : 0;
  const int nblk = (seen1 + 31) >> 5, per = (nblk + a.splits - 1) / a.splits;
  const int lo = (int)blockIdx.y * per, hi = min(lo + per, nblk);
  const int qi = (q0 + col) / a.group, qh = h * a.group + (q0 + col) % a.group;
  const long q_token = t.at + (long)qi * a.tk.step;

  bf16x8 qf[QC];
#pragma unroll
  for (int c = 0; c < QC; ++c) {
    qf[c] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
    if (q0 + col < R) qf[c] = *(const bf16x8 *)((const bf16_t *)a.q.p + row_index(a.q, q_token, qh * DH + 32 * c + 8 * grp));
  }
  bf16x8 ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
  floatx4 O[VM], L = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int m = 0; m < VM; ++m) O[m] = floatx4{0.f, 0.f, 0.f, 0.f};
  float m_ref = -INFINITY;

  auto load = [&](int blk, int page, KvBlock<DH, FP8> &b) {
    const unsigned char *pg = a.kv.pool + (long)page * a.kv.page_bytes;
    const int bpp = a.kv.g.page_tokens >> 5, ib = blk % bpp;
    if constexpr (FP8) {
      const uint32x4 *src = (const uint32x4 *)(pg + ((long)h * bpp + ib) * (64 * DH)) + lane;
#pragma unroll
      for (int i = 0; i < QC; ++i) b.k[i] = __builtin_nontemporal_load(&src[i * 64]);
#pragma unroll
      for (int i = 0; i < VM / 2; ++i) b.v[i] = __builtin_nontemporal_load(&src[2 * DH + i * 64]);
      const unsigned char *ex = pg + (long)H * bpp * (64 * DH) + ((long)h * bpp + ib) * 64;
#pragma unroll
      for (int tl = 0; tl < 2; ++tl) {
        b.ke[tl] = ((const uint32_t *)ex)[4 * tl + grp];
        b.ve[tl] = ((const uint32_t *)ex)[8 + 4 * tl + grp];
      }
    } else {
      const uint32x4 *src = (const uint32x4 *)(pg + ((long)h * bpp + ib) * (128 * DH)) + lane;
#pragma unroll
      for (int i = 0; i < 2 * QC; ++i) b.k[i] = __builtin_nontemporal_load(&src[i * 64]);
#pragma unroll
      for (int i = 0; i < VM; ++i) b.v[i] = __builtin_nontemporal_load(&src[4 * DH + i * 64]);
    }
  };
  // limit: positions of the block from `base` on that the lane's query sees; clear: those that may hold anything
  auto use = [&](int base, KvBlock<DH, FP8> &b, bool masked, int limit, int valid) {
    floatx4 S[2];
#pragma unroll
    for (int tl = 0; tl < 2; ++tl) {
      S[tl] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < QC; ++c) {
        bf16x8 kf;
        if constexpr (FP8) {
          const uint32x4 w = b.k[tl * (QC / 2) + c / 2];
          kf = widen(w[c % 2 * 2], w[c % 2 * 2 + 1], 1.0f);
        } else {
          kf = __builtin_bit_cast(bf16x8, b.k[tl * QC + c]);
        }
        S[tl] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[c], S[tl], 0, 0, 0);
      }
    }
    // S[tl][i]: position base + 16 tl + 4 grp + i
    float vs[8];
    if constexpr (FP8) {
#pragma unroll
      for (int tl = 0; tl < 2; ++tl)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          S[tl][i] *= kv8_scale(b.ke[tl] >> (8 * i) & 255u);
          vs[tl * 4 + i] = kv8_scale(b.ve[tl] >> (8 * i) & 255u);
        }
    }
    bool ok[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      ok[j] = !masked || base + 16 * (j >> 2) + 4 * grp + (j & 3) < limit;
      if (!ok[j]) S[j >> 2][j & 3] = -INFINITY;
    }
    float bm = fmaxf(fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3])), fmaxf(fmaxf(S[1][0], S[1][1]), fmaxf(S[1][2], S[1][3]))) * a.c;
    if (__any(bm > m_ref + 8.0f)) {
      bm = fmaxf(bm, __shfl_xor(bm, 16));  // lanes 16 and 32 apart hold the same query
      bm = fmaxf(bm, __shfl_xor(bm, 32));
      const float m_new = fmaxf(m_ref, bm);
      const float alpha = m_new == m_ref ? 1.0f : __builtin_amdgcn_exp2f(m_ref - m_new);
      m_ref = m_new;
      L *= alpha;
#pragma unroll
      for (int m = 0; m < VM; ++m) O[m] *= alpha;
    }
    float p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[j >> 2][j & 3], a.c, -m_ref));
      if (!ok[j]) p[j] = 0.f;
    }
    auto pack = [&]() { return __builtin_bit_cast(bf16x8, (uint32x4{pack2(p[0], p[1]), pack2(p[2], p[3]), pack2(p[4], p[5]), pack2(p[6], p[7])})); };
    // the weights are rounded to bf16 for the products (2^-9 of a weight on average); so are those that the denominator adds
    bf16x8 pv = pack();
    L = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pv, L, 0, 0, 0);
    if constexpr (FP8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = ok[j] ? p[j] * vs[j] : 0.f;
      pv = pack();
    }
    uint32_t keep[4];  // bf16: values of positions that the row has
    if (masked) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int pos = base + 16 * (i >> 1) + 4 * grp + 2 * (i & 1);
        keep[i] = (pos < valid ? 0xffffu : 0u) | (pos + 1 < valid ? 0xffff0000u : 0u);
      }
    }
    if constexpr (!FP8) {
      if (masked) {
        uint32_t odd = 0;
#pragma unroll
        for (int m = 0; m < VM; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            b.v[m][i] &= keep[i];
            odd |= ((b.v[m][i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;  // exponents that are all ones
          }
        if (__any(odd != 0)) {
          bf16x8 vis;
#pragma unroll
          for (int j = 0; j < 8; ++j) vis[j] = (__bf16)(ok[j] ? 1.0f : 0.0f);
#pragma unroll
          for (int m = 0; m < VM; ++m) {
            uint32x4 up, down;  // 1 where the value is +infinity or NaN, -infinity or NaN
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t u = 0, dn = 0, w = b.v[m][i];
#pragma unroll
              for (int s = 0; s < 32; s += 16) {
                const uint32_t x = w >> s & 0xffffu;
                if ((x & 0x7f80u) == 0x7f80u) {
                  if (x != 0xff80u) u |= 0x3f80u << s;
                  if (x != 0x7f80u) dn |= 0x3f80u << s;
                  w &= ~(0xffffu << s);
                }
              }
              up[i] = u;
              down[i] = dn;
              b.v[m][i] = w;
            }
            const floatx4 z = floatx4{0.f, 0.f, 0.f, 0.f};
            const floatx4 nu = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, up), vis, z, 0, 0, 0);
            const floatx4 nd = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, down), vis, z, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (nu[i] > 0.f) O[m][i] += INFINITY;
              if (nd[i] > 0.f) O[m][i] -= INFINITY;
            }
          }
        }
      }
    }
#pragma unroll
    for (int m = 0; m < VM; ++m) {
      bf16x8 vf;
      if constexpr (FP8) {
        uint32_t w0 = b.v[m / 2][m % 2 * 2], w1 = b.v[m / 2][m % 2 * 2 + 1];
        if (masked) {  // (codes of positions that the row does not have may be NaN)
          w0 &= __builtin_amdgcn_perm(keep[1], keep[0], 0x06040200);
          w1 &= __builtin_amdgcn_perm(keep[3], keep[2], 0x06040200);
        }
        vf = widen(w0, w1, 1.0f);
      } else {
        vf = __builtin_bit_cast(bf16x8, b.v[m]);
      }
      O[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pv, O[m], 0, 0, 0);
    }
  };
  for (int blk = lo + wave; blk < hi; blk += NW) {
    const int page = page_of(a.kv, r, blk);
    if (page < 0) continue;
    KvBlock<DH, FP8> b;
    load(blk, page, b);
    const bool masked = blk * 32 + 32 > seen0 || blk * 32 + 32 > held;
    use(blk * 32, b, masked, min(mine, held), held);
  }
  if (files && blockIdx.y == gridDim.y - 1 && wave == NW - 1) {
    // The one new token is a block of its own, made from its rows: key 0 of it; and it is filed, by the first tile.  Whoever
    // reads its place meanwhile, in the block around it, discards what is there.
    KvBlock<DH, FP8> b;
    const bool stores = qt == 0;
    const int page = stores ? page_of(a.kv, r, t.past >> 5) : -1;
    unsigned char *pg = page < 0 ? nullptr : a.kv.pool + (long)page * a.kv.page_bytes;
    const int slot = t.past % a.kv.g.page_tokens;
    uint32x4 kx[QC];
    bf16_t vx[VM];
#pragma unroll
    for (int c = 0; c < QC; ++c) {
      kx[c] = uint32x4{0, 0, 0, 0};
      if (col == 0) kx[c] = *(const uint32x4 *)((const bf16_t *)a.k.p + row_index(a.k, t.at, h * DH + 32 * c + 8 * grp));
    }
#pragma unroll
    for (int m = 0; m < VM; ++m) vx[m] = grp == 0 ? ((const bf16_t *)a.v.p)[row_index(a.v, t.at, h * DH + 16 * m + col)] : 0;
    if constexpr (FP8) {
      uint32_t km = 0, vm = 0;
#pragma unroll
      for (int c = 0; c < QC; ++c) km = max(km, max_bits(kx[c]));
#pragma unroll
      for (int m = 0; m < VM; ++m) vm = max(vm, (uint32_t)(vx[m] & 0x7fff) << 16);
      const uint32_t ke = kv8_exponent(max_over<64>(km)), ve = kv8_exponent(max_over<64>(vm));
#pragma unroll
      for (int c = 0; c < QC; ++c) {
        const uint2 w = kv8_codes(kx[c], ke);
        if (c % 2 == 0) b.k[c / 2] = uint32x4{0, 0, 0, 0};
        b.k[c / 2][c % 2 * 2] = w.x;
        b.k[c / 2][c % 2 * 2 + 1] = w.y;
        b.k[QC / 2 + c / 2] = uint32x4{0, 0, 0, 0};
        if (pg && col == 0) *(uint2 *)(pg + kv8_k_off(h, slot, 32 * c + 8 * grp, a.kv.g)) = w;
      }
#pragma unroll
      for (int m = 0; m < VM; ++m) {
        const uint32_t w = ve == 255 ? 0u : (kv8_pack(bf2f(vx[m]), 0.f, 0.f, 0.f, ve) & 255u);
        b.v[m / 2][m % 2 * 2] = w;
        b.v[m / 2][m % 2 * 2 + 1] = 0;
        if (pg && grp == 0) pg[kv8_v_off(h, slot, 16 * m + col, a.kv.g)] = (unsigned char)w;
      }
      b.ke[0] = ke;
      b.ve[0] = ve;
      b.ke[1] = b.ve[1] = 0;
      if (pg && lane < 2) pg[kv8_exp_off(h, slot, lane, a.kv.g)] = (unsigned char)(lane ? ve : ke);
    } else {
#pragma unroll
      for (int c = 0; c < QC; ++c) {
        b.k[c] = kx[c];
        b.k[QC + c] = uint32x4{0, 0, 0, 0};
        if (pg && col == 0) *(uint32x4 *)((bf16_t *)pg + kv_k_off(h, slot, 32 * c + 8 * grp, a.kv.g)) = kx[c];
      }
#pragma unroll
      for (int m = 0; m < VM; ++m) {
        b.v[m] = uint32x4{vx[m], 0, 0, 0};
        if (pg && grp == 0) ((bf16_t *)pg)[kv_v_off(h, slot, 16 * m + col, a.kv.g)] = vx[m];
      }
    }
    use(0, b, true, q0 + col < R ? 1 : 0, 1);
  }
  // O[m][i]: element 16 m + 4 grp + i of query `col`; L, m_ref: its denominator and reference
  const int cols = min(16, R - q0);
  float *mine_o = lds + ((long)wave * cols + col) * (DH + 2);
  if (col < cols) {
#pragma unroll
    for (int m = 0; m < VM; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) mine_o[16 * m + 4 * grp + i] = O[m][i];
    if (grp == 0) {
      mine_o[DH] = m_ref;
      mine_o[DH + 1] = L[0];
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
      const float f = x[DH] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[DH] - M);
      if (f != 0.f || x[DH] != x[DH]) {
        num += f * x[e];
        den += f * x[DH + 1];
      }
    }
    const int qi2 = (q0 + cq) / a.group, head = h * a.group + (q0 + cq) % a.group;
    const long token = t.at + (long)qi2 * a.tk.step;
    if (a.splits == 1) {
      ((bf16_t *)a.o.p)[row_index(a.o, token, head * DH + e)] = (bf16_t)f2bf(den == 0.f ? 0.f : num / den);
    } else {
      float *pp = a.part + (((long)blockIdx.y * a.tk.tokens + token) * a.heads + head) * (DH + 2);
      pp[e] = num;
      if (e == 0) {
        pp[DH] = M;
        pp[DH + 1] = den;
      }
    }
  }
}

// Joins the shares of a query's keys, one workgroup per row, query tile of 16 and kv head as above.
template <int DH>
__global__ __launch_bounds__(256) void k_kv_merge(KvAttend a, int tiles) {
  const int H = a.kv.g.H, qt = blockIdx.x % tiles, h = blockIdx.x / tiles % H, r = blockIdx.x / tiles / H;
  const RowTokens t = row_tokens(a.tk, r);
  const int R = t.n * a.group, q0 = qt * 16, cols = min(16, R - q0);
  for (int i = threadIdx.x; i < cols * DH; i += 256) {
    const int e = i % DH, q = q0 + i / DH, head = h * a.group + q % a.group;
    const long token = t.at + (long)(q / a.group) * a.tk.step, stride = (long)a.tk.tokens * a.heads * (DH + 2);
    const float *x = a.part + (token * a.heads + head) * (DH + 2);
    float M = -INFINITY;
    for (int s = 0; s < a.splits; ++s) M = fmaxf(M, x[s * stride + DH]);
    float num = 0.f, den = 0.f;
    for (int s = 0; s < a.splits; ++s) {
      const float m = x[s * stride + DH], f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
      if (f != 0.f || m != m) {
        num += f * x[s * stride + e];
        den += f * x[s * stride + DH + 1];
      }
    }
    ((bf16_t *)a.o.p)[row_index(a.o, token, head * DH + e)] = (bf16_t)f2bf(den == 0.f ? 0.f : num / den);
  }
}

int blocks_of(const KvTokens &tk) { return (tk.max_new + 31 + 31) / 32; }  // of a row, wherever in a block it begins

}  // namespace

void kv_append(hipStream_t s, const KvView &kv, const KvTokens &tk, const KvRows &k, const KvRows &v) {
  const int blocks = blocks_of(tk);
  const dim3 grid((unsigned)((long)blocks * kv.g.H * kv.rows));
  if (kv.g.dh == 64) {
    if (kv.fp8) SKD_LAUNCH((k_kv_append<64, true>), grid, dim3(256), 0, s, kv, tk, k, v, blocks);
    else SKD_LAUNCH((k_kv_append<64, false>), grid, dim3(256), 0, s, kv, tk, k, v, blocks);
  } else {
    if (kv.fp8) SKD_LAUNCH((k_kv_append<128, true>), grid, dim3(256), 0, s, kv, tk, k, v, blocks);
    else SKD_LAUNCH((k_kv_append<128, false>), grid, dim3(256), 0, s, kv, tk, k, v, blocks);
  }
}

void kv_read(hipStream_t s, const KvView &kv, const KvTokens &tk, bool bf16, const KvRows &k, const KvRows &v) {
  const int blocks = blocks_of(tk);
  const dim3 grid((unsigned)((long)blocks * kv.g.H * kv.rows));
#define SKD_READ(DH, FP8)                                                                                  \
  do {                                                                                                     \
    if (bf16) SKD_LAUNCH((k_kv_read<DH, FP8, bf16_t>), grid, dim3(256), 0, s, kv, tk, k, v, blocks);       \
    else SKD_LAUNCH((k_kv_read<DH, FP8, float>), grid, dim3(256), 0, s, kv, tk, k, v, blocks);             \
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

static long query_tiles(const KvTokens &tk, int group) { return ((long)tk.max_new * group + 15) / 16; }
// Eight waves a workgroup, and as many shares of the keys as give every CU 16 waves; a share has 8 blocks at least.
int kv_attend_splits(const KvView &kv, const KvTokens &tk, int heads) {
  const long wgs = query_tiles(tk, heads / kv.g.H) * kv.g.H * kv.rows, blocks = ((long)tk.max_past + tk.max_new + 31) / 32;
  int splits = 1;
  while (splits < 64 && wgs * splits < 512 && blocks / (2 * splits) >= 8) splits *= 2;
  return splits;
}
size_t kv_attend_part(const KvView &kv, const KvTokens &tk, int heads, int splits) {
  return splits > 1 ? (size_t)splits * tk.tokens * heads * (kv.g.dh + 2) : 0;
}

void kv_attend(hipStream_t s, const KvAttend &a) {
  constexpr int NW = 8;
  const int tiles = (int)query_tiles(a.tk, a.group);
  const dim3 grid((unsigned)((long)tiles * a.kv.g.H * a.kv.rows), a.splits);
  const size_t lds = (size_t)NW * (tiles > 1 ? 16 : a.tk.max_new * a.group) * (a.kv.g.dh + 2) * sizeof(float);
  static std::atomic<uint64_t> done{0};
  const void *all[] = {(const void *)k_kv_attend<64, false, NW>, (const void *)k_kv_attend<64, true, NW>, (const void *)k_kv_attend<128, false, NW>,
                       (const void *)k_kv_attend<128, true, NW>};
  if (lds > 64 * 1024) (void)allow_lds(done, {all[0], all[1], all[2], all[3]}, NW * 16 * 130 * sizeof(float));
  if (a.kv.g.dh == 64) {
    if (a.kv.fp8) SKD_LAUNCH((k_kv_attend<64, true, NW>), grid, dim3(NW * 64), lds, s, a, tiles);
    else SKD_LAUNCH((k_kv_attend<64, false, NW>), grid, dim3(NW * 64), lds, s, a, tiles);
    if (a.splits > 1) SKD_LAUNCH(k_kv_merge<64>, dim3(grid.x), dim3(256), 0, s, a, tiles);
  } else {
    if (a.kv.fp8) SKD_LAUNCH((k_kv_attend<128, true, NW>), grid, dim3(NW * 64), lds, s, a, tiles);
    else SKD_LAUNCH((k_kv_attend<128, false, NW>), grid, dim3(NW * 64), lds, s, a, tiles);
    if (a.splits > 1) SKD_LAUNCH(k_kv_merge<128>, dim3(grid.x), dim3(256), 0, s, a, tiles);
  }
}

}  // namespace skd
