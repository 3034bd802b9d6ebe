// Kernels that file tokens into pages and read them back, and their launches, for one kind of page (EL).
#pragma once
#include "kv_device.h"

namespace skd {

namespace {

// ------------------------------------------------------------------ filing
// A workgroup files the tokens of one row and kv head that lie in one 32-key block.  DH / 8 lanes take a token: 16 bytes of
// K and of V each, largest magnitudes over them; K goes to the page as it is, V^T by way of LDS, where the four keys that
// are neighbours in the page are gathered.  Bound by the bytes of large calls; a block's codes leave as whole words where the
// row fills them, and element by element at the ends of its tokens, so that what other tokens hold there stays.  4 bits: four lanes share an
// exponent, and the lanes of elements 16 apart join their values' codes, two in a byte.  509 tokens of 8 rows, 32 heads of 128: 17 us.
template <int DH, int EL>
__global__ __launch_bounds__(256) void k_kv_append(KvView kv, KvTokens tk, KvRows k, KvRows v, int blocks, uint32_t from) {
  constexpr bool FP8 = EL == EL_FP8, FP4 = EL == EL_FP4;
  constexpr int LPT = DH / 8, TPP = 256 / LPT;  // lanes a token, tokens a pass
  constexpr int CODES = FP4 ? DH / 2 : DH;      // of a token's values: elements, or pairs of them
  typedef typename std::conditional<EL == EL_BF16, uint16_t, uint8_t>::type code_t;
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
    } else if constexpr (FP4) {
      const uint32_t ke = kv4_exponent(max_over<4>(max_bits(kx))), ve = kv4_exponent(max_over<4>(max_bits(vx)));
      *(uint32_t *)(pg + kv4_k_off(h, slot0 + key, e, kv.g)) = kv4_codes(kx, ke);
      const uint32_t low = kv4_codes(vx, ve), high = (uint32_t)__shfl_xor((int)low, 2);
      if (!(e & 16)) *(uint2 *)&sv[key][e / 32 * 16 + e % 32] = kv4_bytes(low, high);
      if (e % 32 == 0) {
        pg[kv4_k_exp_off(h, slot0 + key, e / 32, kv.g)] = (unsigned char)ke;
        pg[kv4_v_exp_off(h, slot0 + key, e / 32, kv.g)] = (unsigned char)ve;
      }
    } else {
      *(uint32x4 *)((bf16_t *)pg + kv_k_off(h, slot0 + key, e, kv.g)) = kx;
      *(uint32x4 *)&sv[key][e] = vx;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 8 * CODES; i += 256) {  // code el, four keys from key0 on
    const int el = i % CODES, key0 = i / CODES * 4;
    const int first = blk * 32 + key0;
    code_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = sv[key0 + j][el];
    code_t *to = FP8   ? (code_t *)(pg + kv8_v_off(h, slot0 + key0, el, kv.g))
                 : FP4 ? (code_t *)(pg + kv4_v_off(h, slot0 + key0, el / 16 * 32 + el % 16, kv.g))
                       : (code_t *)pg + kv_v_off(h, slot0 + key0, el, kv.g);
    if (first >= lo && first + 4 <= hi) {
      if constexpr (FP8 || FP4) *(uint32_t *)to = c[0] | (uint32_t)c[1] << 8 | (uint32_t)c[2] << 16 | (uint32_t)c[3] << 24;
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
template <int DH, int EL>
__global__ __launch_bounds__(256) void k_kv_append_few(KvView kv, KvTokens tk, KvRows k, KvRows v) {
  constexpr bool FP8 = EL == EL_FP8, FP4 = EL == EL_FP4;
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
  } else if constexpr (FP4) {
    const uint32_t ex = kv4_exponent(max_over<4>(max_bits(x))), c = kv4_codes(x, ex), high = (uint32_t)__shfl_xor((int)c, 2);
    if (e % 32 == 0) pg[is_v ? kv4_v_exp_off(h, slot, e / 32, kv.g) : kv4_k_exp_off(h, slot, e / 32, kv.g)] = (unsigned char)ex;
    if (is_v) {
      if (!(e & 16)) *(uint2 *)(own + e / 32 * 16 + e % 32) = kv4_bytes(c, high);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = l + LPT * j;  // pair
        pg[kv4_v_off(h, slot, i / 16 * 32 + i % 16, kv.g)] = own[i];
      }
    } else {
      *(uint32_t *)(pg + kv4_k_off(h, slot, e, kv.g)) = c;
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
__device__ inline void decode4(uint16_t w, uint32_t ex, float *x) {
  const floatx2 a = kv4_values(w & 255u, ex), b = kv4_values(w >> 8, ex);
  x[0] = a[0];
  x[1] = a[1];
  x[2] = b[0];
  x[3] = b[1];
}
__device__ inline void decode4(uint2 w, float *x) {
  x[0] = bf2f(w.x & 0xffffu);
  x[1] = bf2f(w.x >> 16);
  x[2] = bf2f(w.y & 0xffffu);
  x[3] = bf2f(w.y >> 16);
}
// The few tokens of k_kv_append_few the other way.
template <int DH, int EL, typename OUT>
__global__ __launch_bounds__(256) void k_kv_read_few(KvView kv, KvTokens tk, KvRows k, KvRows v) {
  constexpr bool FP8 = EL == EL_FP8, FP4 = EL == EL_FP4;
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
    } else if constexpr (FP4) {
      if (is_v) {
        const uint32_t ex = pg[kv4_v_exp_off(h, slot, e / 32, kv.g)];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * p + j] = kv4_values(pg[kv4_v_off(h, slot, (e & ~16) + j, kv.g)], ex)[(e >> 4) & 1];
      } else {
        decode4(*(const uint16_t *)(pg + kv4_k_off(h, slot, e, kv.g)), pg[kv4_k_exp_off(h, slot, e / 32, kv.g)], x + 4 * p);
      }
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
template <int DH, int EL, typename OUT>
__global__ __launch_bounds__(256) void k_kv_read(KvView kv, KvTokens tk, KvRows k, KvRows v, int blocks, uint32_t from) {
  constexpr bool FP8 = EL == EL_FP8, FP4 = EL == EL_FP4;
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
  typename std::conditional<FP8, uint32_t, typename std::conditional<FP4, uint16_t, uint2>::type>::type kw[32 / TPP][2];
  uint32_t ke[32 / TPP][2];
#pragma unroll
  for (int i = 0; i < 32 / TPP; ++i) {
    const int key = threadIdx.x / LPT + i * TPP;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int e = piece_of<OUT, DH>(l, p);
      if constexpr (FP8) kw[i][p] = *(const uint32_t *)(pg + kv8_k_off(h, slot0 + key, e, kv.g));
      else if constexpr (FP4) kw[i][p] = *(const uint16_t *)(pg + kv4_k_off(h, slot0 + key, e, kv.g));
      else kw[i][p] = *(const uint2 *)((const bf16_t *)pg + kv_k_off(h, slot0 + key, e, kv.g));
      if constexpr (FP4) ke[i][p] = pg[kv4_k_exp_off(h, slot0 + key, e / 32, kv.g)];
    }
    if constexpr (FP8) ke[i][0] = ke[i][1] = pg[kv8_exp_off(h, slot0 + key, 0, kv.g)];
  }
  for (int i = threadIdx.x; i < (FP4 ? 4 : 8) * DH; i += 256) {
    const int el = i % (FP4 ? DH / 2 : DH), key0 = i / (FP4 ? DH / 2 : DH) * 4;
    if constexpr (FP4) {
      const int e = el / 16 * 32 + el % 16;
      const uint32_t w = *(const uint32_t *)(pg + kv4_v_off(h, slot0 + key0, e, kv.g));
      const uint32_t x = *(const uint32_t *)(pg + kv4_v_exp_off(h, slot0 + key0, e / 32, kv.g));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const floatx2 y = kv4_values(w >> (8 * j) & 255u, x >> (8 * j) & 255u);
        sv[key0 + j][e] = y[0];
        sv[key0 + j][e + 16] = y[1];
      }
    } else if constexpr (FP8) {
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
      if constexpr (FP8 || FP4) decode4(kw[i][p], ke[i][p], kx + 4 * p);
      else decode4(kw[i][p], kx + 4 * p);
#pragma unroll
      for (int j = 0; j < 4; ++j) vx[4 * p + j] = sv[key][piece_of<OUT, DH>(l, p) + j];
    }
    store_pieces<OUT, DH>((OUT *)k.p + row_index(k, token, h * DH), l, kx);
    store_pieces<OUT, DH>((OUT *)v.p + row_index(v, token, h * DH), l, vx);
  }
}


int blocks_of(const KvTokens &tk) { return (tk.max_new + 31 + 31) / 32; }  // of a row, wherever in a block it begins

// Workgroups of the kernels for a few tokens, or 0: up to 8 of a row (k_kv_append_few), and a grid that fits.
unsigned few_groups(const KvView &kv, const KvTokens &tk) {
  const long units = 2L * kv.g.H * tk.max_new * kv.rows, groups = (units * (kv.g.dh / 8) + 255) / 256;
  return tk.max_new <= 8 && launch_fits(groups, 256) ? (unsigned)groups : 0;  // (units, of 8 lanes or more, are in 32 bits then)
}
// The kernels for many tokens, a workgroup for each block: f(grid, first block) for as many as a launch has, which is all of them
// but for a row of 100000 tokens among more than a hundred.
template <typename F>
void each_launch(const KvView &kv, const KvTokens &tk, F f) {
  const long all = kv_blocks(kv, tk);
  for (long from = 0; from < all; from += launch_most(256)) f(dim3((unsigned)std::min(all - from, launch_most(256))), (uint32_t)from);
}
template <int DH, int EL>
void append_pages(hipStream_t s, const KvView &kv, const KvTokens &tk, const KvRows &k, const KvRows &v) {
  if (const unsigned few = few_groups(kv, tk)) SKD_LAUNCH((k_kv_append_few<DH, EL>), dim3(few), dim3(256), 0, s, kv, tk, k, v);
  else each_launch(kv, tk, [&](dim3 grid, uint32_t from) { SKD_LAUNCH((k_kv_append<DH, EL>), grid, dim3(256), 0, s, kv, tk, k, v, blocks_of(tk), from); });
}
template <int DH, int EL, typename OUT>
void read_pages(hipStream_t s, const KvView &kv, const KvTokens &tk, const KvRows &k, const KvRows &v) {
  if (const unsigned few = few_groups(kv, tk)) SKD_LAUNCH((k_kv_read_few<DH, EL, OUT>), dim3(few), dim3(256), 0, s, kv, tk, k, v);
  else each_launch(kv, tk, [&](dim3 grid, uint32_t from) { SKD_LAUNCH((k_kv_read<DH, EL, OUT>), grid, dim3(256), 0, s, kv, tk, k, v, blocks_of(tk), from); });
}
template <int EL>
void append_elem(hipStream_t s, const KvView &kv, const KvTokens &tk, const KvRows &k, const KvRows &v) {
  if (kv.g.dh == 64) append_pages<64, EL>(s, kv, tk, k, v);
  else append_pages<128, EL>(s, kv, tk, k, v);
}
template <int EL>
void read_elem(hipStream_t s, const KvView &kv, const KvTokens &tk, bool bf16, const KvRows &k, const KvRows &v) {
  if (kv.g.dh == 64) bf16 ? read_pages<64, EL, bf16_t>(s, kv, tk, k, v) : read_pages<64, EL, float>(s, kv, tk, k, v);
  else bf16 ? read_pages<128, EL, bf16_t>(s, kv, tk, k, v) : read_pages<128, EL, float>(s, kv, tk, k, v);
}

}  // namespace

}  // namespace skd
