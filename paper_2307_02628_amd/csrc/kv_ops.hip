// The paged cache as an operator: new tokens of ragged rows filed into pages of bf16, 8 or 4 bits, read back, and attended to.  Here
// are the kernels for bf16 and 8 bits with scores as they are, what joins shares of the keys, and which kernel a call takes.
#include "kv_attend.h"
#include "kv_file.h"

namespace skd {

// the other kinds: kv_scores*.hip, kv_fp4.hip
void kv_attend_scored_bf16(hipStream_t s, const KvAttend &a, const AttendPlan &p);
void kv_attend_scored_fp8(hipStream_t s, const KvAttend &a, const AttendPlan &p);
void kv_attend_scored_fp4(hipStream_t s, const KvAttend &a, const AttendPlan &p);
void kv_attend_fp4(hipStream_t s, const KvAttend &a, const AttendPlan &p);
void kv_append_fp4(hipStream_t s, const KvView &kv, const KvTokens &tk, const KvRows &k, const KvRows &v);
void kv_read_fp4(hipStream_t s, const KvView &kv, const KvTokens &tk, bool bf16, const KvRows &k, const KvRows &v);

namespace {

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

}  // namespace

long kv_blocks(const KvView &kv, const KvTokens &tk) { return (long)blocks_of(tk) * kv.g.H * kv.rows; }
void kv_append(hipStream_t s, const KvView &kv, const KvTokens &tk, const KvRows &k, const KvRows &v) {
  if (kv.fp4) kv_append_fp4(s, kv, tk, k, v);
  else if (kv.fp8) append_elem<EL_FP8>(s, kv, tk, k, v);
  else append_elem<EL_BF16>(s, kv, tk, k, v);
}
void kv_read(hipStream_t s, const KvView &kv, const KvTokens &tk, bool bf16, const KvRows &k, const KvRows &v) {
  if (kv.fp4) kv_read_fp4(s, kv, tk, bf16, k, v);
  else if (kv.fp8) read_elem<EL_FP8>(s, kv, tk, bf16, k, v);
  else read_elem<EL_BF16>(s, kv, tk, bf16, k, v);
}

static AttendPlan plan_attend(const KvView &kv, const KvTokens &tk, int heads, int window) {
  AttendPlan p{};
  const long R = (long)tk.max_new * (heads / kv.g.H);
  long blocks = ((long)tk.max_past + tk.max_new + 31) / 32;
  // Up to 16 queries one tile, up to 32 two; beyond, the blocks go through LDS once for all, which 8 bits gain from only with five
  // tiles and more (inputs not in the last-level cache, us.  Two tiles of 16 for 17 .. 32 queries: 16 rows of 2000, 8 kv heads of
  // 128, bf16 31.3, 30.9; 40 rows 70.7, 104.9.  33 .. 64 as two of 32 or through LDS: 8 rows of 1000, 32 heads of 128, bf16 58.7,
  // 35.2, 8 bits 38.7, 38.2; 32 rows of 700, 8 kv heads of 64, bf16 23.4, 19.7, 8 bits 15.2, 22.1; one of 20000, 8 of 128, 8 bits
  // 23.3, 30.5.  65 .. 128: 8 rows of 1000 bf16 107, 38, 8 bits 70, 41.  4 bits as 8: 8 rows of 1000, 64 queries 30.8, 35.7, 100 of them
  // 46.3, 37.5; 32 rows of 700, 8 kv heads of 64, 64 queries 15.5, 20.6.)
  p.nq = R <= 16 ? 16 : R <= (kv.fp8 || kv.fp4 ? 64 : 32) ? 32 : 128;
  p.tiles = (R + p.nq - 1) / p.nq;
  // (all that a tile's queries see: a window for its last token and as many positions as the tile has tokens)
  if (window > 0) blocks = std::min(blocks, ((long)window + p.nq / (heads / kv.g.H) + 62) / 32);
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
    // 4 bits are bound by the vector units as much as by bytes: no more than a workgroup a CU (by the rule of the others, and this one, us,
    // 8 kv heads of 128: 24 rows of 1000 14.4, 10.4, of 4000 26.5, 23.8; 12 of 3000 with 5 26.7, 21.8).  Two shares begin where a wave has five
    // blocks, six if that fills half of the CUs, four if scores are changed or tiles are two (one share, two: one row of 1000 9.2, 9.6, with slopes
    // 11.2, 10.1; of 1500 11.6, 10.2; 16 of 1500 12.0, 12.6; 3 of 700 8.6, 10.0, with slopes 9.9, 10.8; 16 of 2000 with 5 20.8, 19.3).
    // Two tiles with changed scores likewise, from four blocks a wave where half of the CUs have one (12 rows of 3000 with 5, 8 kv heads, capped,
    // bf16 34.0, 30.3, 8 bits 29.9, 25.6; 16 of 3000 39.3, 35.1 and 32.7, 27.0).  (One tile of theirs is not: 24 rows of 4000, 8 bits, 39.2, 44.9.)
    const bool one_a_cu = kv.fp4 || (window >= 0 && p.nq == 32);
    int least = p.waves;  // blocks of half a row
    if (kv.fp4) least = p.nq == 32 || window >= 0 ? 2 * p.waves : wgs >= 128 ? 3 * p.waves : 5 * p.waves / 2;
    else if (p.nq == 32 && wgs >= 128) least = (one_a_cu ? 2 : 6) * p.waves;
    auto more = [&]() { return one_a_cu ? wgs * 2 * p.splits <= 256 : wgs * p.waves * p.splits < 2048; };
    while (p.splits < 64 && more() && blocks / (2 * p.splits) >= (p.splits == 1 ? least : p.waves)) p.splits *= 2;
  }
  return p;
}
bool kv_attend_fits(const KvView &kv, const KvTokens &tk, int heads, int window) {
  const AttendPlan p = plan_attend(kv, tk, heads, window);
  return launch_fits(p.tiles * p.pairs, 64 * p.waves);
}
int kv_attend_splits(const KvView &kv, const KvTokens &tk, int heads, int window) { return plan_attend(kv, tk, heads, window).splits; }
size_t kv_attend_part(const KvView &kv, const KvTokens &tk, int heads, int splits) {
  return splits > 1 ? (size_t)splits * tk.tokens * heads * (kv.g.dh + 2) : 0;
}

template <int DH>
static void merge(hipStream_t s, const KvAttend &a) {
  const int queries = a.tk.max_new * a.group;
  const long all = (long)queries * a.kv.g.H * a.kv.rows;
  if (a.splits <= 8) SKD_LAUNCH(k_kv_merge_few<DH>, dim3((unsigned)((all + 3) / 4)), dim3(256), 0, s, a, queries);
  else SKD_LAUNCH(k_kv_merge<DH>, dim3((unsigned)all), dim3(256), 0, s, a, queries);
}
void kv_attend(hipStream_t s, const KvAttend &call) {
  KvAttend a = call;
  const AttendPlan p = plan_attend(a.kv, a.tk, a.heads, a.scored ? a.sc.window : -1);
  if (a.k.p && !(a.tk.max_new == 1 && p.nq == 16)) {  // (one token of few heads: the same launch)
    kv_append(s, a.kv, a.tk, a.k, a.v);
    a.k.p = nullptr;
  }
  if (a.scored) (a.kv.fp4 ? kv_attend_scored_fp4 : a.kv.fp8 ? kv_attend_scored_fp8 : kv_attend_scored_bf16)(s, a, p);
  else if (a.kv.fp4) kv_attend_fp4(s, a, p);
  else if (a.kv.fp8) attend_elem<EL_FP8, 0>(s, a, p);
  else attend_elem<EL_BF16, 0>(s, a, p);
  if (a.splits > 1) a.kv.g.dh == 64 ? merge<64>(s, a) : merge<128>(s, a);
}

}  // namespace skd
