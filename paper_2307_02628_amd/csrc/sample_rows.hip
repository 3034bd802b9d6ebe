// One token a row from fp32 logits, with the row's own temperature, top-k, top-p and min-p and a given uniform number.
//
// With m_i = exp((z_i - max z) / T): kept are the tokens with m_i >= min_p that are among the k largest logits (ties with the k-th
// too), of these the smallest set of largest ones whose mass reaches top_p of theirs (ties with the last too).  All three are
// "z >= threshold", so what is looked for is one threshold, and then the first index whose running mass over the tokens at or
// above it exceeds u times their mass.
//
// Masses are integers in units of 2^-45 (exponentials in 64 bits, to 2^-44), sums of them integers or added in a fixed order in 64
// bits: neither atomics nor the shares of the waves change a draw, and one that 64-bit arithmetic decides comes out the same.
// What lies 32 T below the largest logit has no mass, is never drawn, and is left out from the start.
//
// Two launches.  k_sample_bins, pieces of rows over the whole chip: the piece's largest logit, and by bins of T / 16 (512 and one
// for what is left) how many tokens (rows with top-k or min-p) or how much mass (the others).  It reads the logits once
// and is bound by that.  The bins lie on a grid that all pieces share.  k_sample_pick, a workgroup per row.  Few tokens left by
// top-k or min-p, which is what they are for: the bins say from where on, those tokens go into LDS, and thresholds and token
// are found there by buckets.  Top-p alone: the bin in which the threshold lies, whose values are listed; the piece in which
// the running mass passes the target, and the token in it.  What does not fit into LDS is looked at again instead, ten bits of
// the answer each time.  k_sample_pick is bound by what one CU does: an instruction for each of 131072 tokens is 0.9 us, a barrier
// or a trip to memory 0.3 to 1 us, so four tokens are compared at once, the waves' sums move in registers, and requests go out
// together.
// us (bins + pick), one workgroup per row for everything (six passes over the row) -> this: 128 rows of 131072 with mixed
// parameters 227 -> 60 (21 + 39), one row of 50272 with top-p 75 -> 22 (5 + 17).  1024 bins of T / 32 cost twice the traffic: one
// row 33; shuffles through LDS for the sums and one list for all waves: 25 and 95; the bin of every token computed instead of
// compared with its edges, and the last 64 searched by every wave: 128 rows 70.
#include "sample_rows.h"

#include <float.h>
#include <math.h>

#include "bf16_device.h"

namespace skd {

namespace {

typedef unsigned long long u64;

constexpr int BINS = SAMPLE_BINS, NW = 16, CAP = 8192;  // CAP: tokens that are listed, a wave's share of it by each

__device__ inline uint32_t key_of(float z) {  // ordered as the values are
  const uint32_t b = __float_as_uint(z);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float usable(float z) { return z == z ? z + 0.f : -INFINITY; }  // (-0 as 0)
// Running results of a wave's lanes by moves within the registers (through LDS each of the six steps takes its latency): lanes that
// a step has no other lane for combine with `none`.
template <int CTRL, int ROWS>
__device__ inline uint32_t moved32(uint32_t v, uint32_t none) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS, typename T>
__device__ inline T moved64(T v) {
  const u64 b = __builtin_bit_cast(u64, v);
  return __builtin_bit_cast(T, (u64)moved32<CTRL, ROWS>((uint32_t)b, 0) | (u64)moved32<CTRL, ROWS>((uint32_t)(b >> 32), 0) << 32);
}
template <typename T>
__device__ inline T lane64(T v, int lane) {
  const u64 b = __builtin_bit_cast(u64, v);
  return __builtin_bit_cast(T, (u64)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane) | (u64)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane) << 32);
}
template <typename T>
__device__ inline T wave_scan64(T v) {  // sums of the lanes up to each
  v += moved64<0x111, 0xf>(v);  // 1, 2, 4 and 8 lanes on within each 16; the last of 16 to the next 16, of 32 to the next 32
  v += moved64<0x112, 0xf>(v);
  v += moved64<0x114, 0xf>(v);
  v += moved64<0x118, 0xf>(v);
  v += moved64<0x142, 0xa>(v);
  v += moved64<0x143, 0xc>(v);
  return v;
}
template <typename T>
__device__ inline T wave_sum64(T v) {
  return lane64(wave_scan64(v), 63);
}
__device__ inline uint32_t wave_max(uint32_t v) {
  v = max(v, moved32<0x111, 0xf>(v, 0));
  v = max(v, moved32<0x112, 0xf>(v, 0));
  v = max(v, moved32<0x114, 0xf>(v, 0));
  v = max(v, moved32<0x118, 0xf>(v, 0));
  v = max(v, moved32<0x142, 0xa>(v, 0));
  v = max(v, moved32<0x143, 0xc>(v, 0));
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ inline float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
__device__ inline float uniform(float v) { return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(v))); }
__device__ inline double uniform(double v) {
  const u64 b = __builtin_bit_cast(u64, v);
  return __builtin_bit_cast(double, (u64)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b) | (u64)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32)) << 32);
}
__device__ inline float wave_top(float v) { return value_of(wave_max(key_of(v))); }

// What a row's parameters come to.
struct Params {
  float T, top_p, u;
  int k;
  double log_min;             // log(min_p); 0 from 1 on, -32 where it is off (or below e^-32)
  bool greedy, by_k, by_p;
  bool counts, masses;        // what the bins hold: rows with top-k, all others, both with min-p alone
  __device__ __forceinline__ Params(const SampleRows &a, int b) {
    T = a.temperature ? a.temperature[b] : 1.0f;
    k = a.top_k ? a.top_k[b] : 0;
    top_p = a.top_p ? fmaxf(a.top_p[b], 0.f) : 1.0f;
    if (a.top_p && a.top_p[b] != a.top_p[b]) top_p = 1.0f;
    const float m = a.min_p ? a.min_p[b] : 0.f;
    log_min = uniform(m > 0.f ? fmax(m < 1.f ? log((double)m) : 0.0, -32.0) : -32.0);
    u = fminf(fmaxf(a.u[b], 0.f), 0x1.fffffep-1f);  // (NaN: 0)
    greedy = !(T > 0.f);
    by_k = !greedy && k > 0 && k < a.vocab;
    by_p = !greedy && top_p < 1.f;
    counts = !greedy && (by_k || log_min > -32.0);
    masses = !greedy && !by_k;
  }
  // the smallest float that is not below top + T * log_min
  __device__ __forceinline__ float floor_of(float top) const {
    const double f = (double)top + (double)T * log_min;
    float x = (float)f;
    if ((double)x < f) x = nextafterf(x, INFINITY);
    return fminf(x, top);
  }
};
// Places on the grid of bins, and masses against a largest logit.
struct Grid {
  float s;                    // 16 / T
  double c;                   // 64 log2(e) / T
  const double *tab;          // 2^(i / 64)
  __device__ __forceinline__ Grid(float T, const double *t) : s(uniform((float)(16.0 / (double)T))), c(uniform(64.0 * 1.44269504088896340736 / (double)T)), tab(t) {}
  __device__ float place(float z) const { return floorf(z * s); }
  // (where places overflow, what differs from the largest logit is far below it: NaN is the rest)
  __device__ int bin(float top, float top_place, float z) const { return z == top ? 0 : (int)fminf(top_place - place(z), (float)BINS); }
  // 64 log2 of a mass is split into n + r: 2^(n / 64) from the table, 2^(r / 64) by its series (|r| <= 1/2: the first term left
  // out is below 2^-44); in units of 2^-45, nearest
  __device__ __forceinline__ u64 mass(float z, float top) const {
    const double y = fmax(((double)z - (double)top) * c, -64.0 * 60);
    const double t = y + 0x1.8p52, r = (y - (t - 0x1.8p52)) * (0.69314718055994530942 / 64);
    const int n = (int)(uint32_t)__double_as_longlong(t);
    const double p = 1.0 + r * (1.0 + r * (0.5 + r * (1.0 / 6 + r * (1.0 / 24))));
    const double m = __longlong_as_double(__double_as_longlong(tab[n & 63] * p) + ((long long)(n >> 6) << 52));
    return (u64)(__double_as_longlong(m + 128.0) - __double_as_longlong(128.0));
  }
};
__device__ inline floatx4 load4(const float *z, int at, int end, bool vec) {  // past the end: -infinity
  floatx4 v;
  if (vec && at + 4 <= end) {
    v = *(const floatx4 *)(z + at);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = at + j < end ? z[at + j] : -INFINITY;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = usable(v[j]);
  return v;
}

// PER: tokens of a thread, four neighbouring ones at a time; they stay in registers.
template <int PER>
__global__ __launch_bounds__(256) void k_sample_bins(SampleRows a) {
  __shared__ u64 mass[BINS + 1];
  __shared__ uint32_t count[BINS + 1];
  __shared__ double tab[64];
  __shared__ float tops[4];
  const int tid = threadIdx.x, piece = blockIdx.x % a.pieces, b = blockIdx.x / a.pieces;
  const float *z = a.logits + (long)b * a.stride;
  const bool vec = ((uintptr_t)z & 15) == 0;
  const int begin = piece * (256 * PER), end = min(begin + 256 * PER, a.vocab);
  floatx4 v[PER / 4];
#pragma unroll
  for (int i = 0; i < PER / 4; ++i) v[i] = load4(z, begin + (i * 256 + tid) * 4, end, vec);
  const Params p(a, b);
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < PER / 4; ++i) top = fmaxf(top, fmaxf(fmaxf(v[i][0], v[i][1]), fmaxf(v[i][2], v[i][3])));
  top = wave_top(top);
  if ((tid & 63) == 0) tops[tid >> 6] = top;
  for (int i = tid; i <= BINS; i += 256) {
    mass[i] = 0;
    count[i] = 0;
  }
  if (tid < 64) tab[tid] = exp2(tid / 64.0);
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  SampleBins &out = a.bins[(long)b * a.pieces + piece];
  if (tid == 0) out.top = top;
  if (p.greedy || top == INFINITY || top == -INFINITY) return;
  const Grid g(p.T, tab);
  const float place = g.place(top);
  const float lowest = p.floor_of(top);  // (the row's is not lower)
#pragma unroll
  for (int i = 0; i < PER / 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (v[i][j] >= lowest && v[i][j] > -INFINITY) {
        const int bin = g.bin(top, place, v[i][j]);
        if (p.counts) atomicAdd(&count[bin], 1u);
        if (p.masses) atomicAdd(&mass[bin], g.mass(v[i][j], top));
      }
  __syncthreads();
  if (p.counts)
    for (int i = tid; i <= BINS; i += 256) out.count[i] = count[i];
  if (!p.masses) return;
  u64 all = 0;
  for (int i = tid; i <= BINS; i += 256) {
    out.mass[i] = mass[i];
    all += mass[i];
  }
  all = wave_sum64(all);
  __shared__ u64 sums[4];
  if ((tid & 63) == 0) sums[tid >> 6] = all;
  __syncthreads();
  if (tid == 0) out.all = sums[0] + sums[1] + sums[2] + sums[3];
}

constexpr int PIECES = 128;  // of a row, at most

struct Pick {
  double tab[64];
  double mass[BINS + 1];
  uint32_t count[BINS + 1];
  double scale[PIECES];       // of a piece's masses
  double kept[PIECES];        // masses of its kept tokens
  u64 part[PIECES];           // of those in the threshold's bin
  int shift[PIECES];          // its first bin
  float top[PIECES];
  uint8_t wanted[PIECES];     // a sweep reads it
  float value[CAP];           // listed tokens
  int index[CAP];
  u64 weight[CAP];            // their masses
  int n;
  u64 sum[2][NW];
  int seen[NW];
  uint32_t lo, hi;
  u64 bucket[1024];
  u64 wave_mass[NW];
  int bucket_at;
  u64 bucket_before;
  uint32_t near_key[64];      // the elements of one bucket
  u64 near_mass[64];
  int near_n;
  uint32_t found;
  u64 found_sum;
};

// `v`, so that what is computed from it is computed here: which lanes a step is for takes one comparison, but two scalar registers
// from one step to the next, and together with the rest more than there are.
__device__ inline int now(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// (With a call left to any of the steps all that they share would live in memory: 139 us.)
#define SKD_INLINE __attribute__((always_inline))
__global__ __launch_bounds__(NW * 64) void k_sample_pick(SampleRows a) {
  extern __shared__ unsigned char lds[];
  Pick &sh = *(Pick *)lds;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, b = blockIdx.x, pieces = a.pieces, V = a.vocab;
  const float *z = a.logits + (long)b * a.stride;
  const bool vec = ((uintptr_t)z & 15) == 0;
  const SampleBins *bins = a.bins + (long)b * pieces;
  const int piece_bits = __builtin_ctz((unsigned)a.piece);  // (a power of two)
  const Params p(a, b);
  float top = lane < pieces ? bins[lane].top : -INFINITY;
  if (lane + 64 < pieces) top = fmaxf(top, bins[lane + 64].top);
  top = wave_top(top);
  const bool greedy = p.greedy || top == INFINITY || top == -INFINITY;
  const Grid g(p.T, sh.tab);
  const float place = greedy ? 0.f : g.place(top), lowest = greedy ? top : p.floor_of(top);
  if (tid < 64) sh.tab[tid] = exp2(tid / 64.0);
  if (tid < pieces) {
    const float t = bins[tid].top;
    sh.top[tid] = t;
    sh.shift[tid] = t == -INFINITY ? BINS + 1 : t == top ? 0 : (int)fminf(place - g.place(t), (float)(BINS + 1));
    sh.scale[tid] = t == -INFINITY || greedy ? 0.0 : exp(((double)t - (double)top) / (double)p.T);
    sh.kept[tid] = t == -INFINITY || greedy || !p.masses ? 0.0 : (double)bins[tid].all * sh.scale[tid];
    sh.part[tid] = 0;
  }
  __syncthreads();
  auto answer = [&](int token) {
    a.tokens[b] = token;
    if (a.tokens2) a.tokens2[b] = token;
  };
  // f(logit, index, whether it is one), by whole waves, for the tokens of the wanted pieces from `low` on and below `high`, several
  // requested at a time.  An instruction for every token is 0.9 us at 131072 of them: four are compared at once.
  float low = fmaxf(lowest, -FLT_MAX), high = INFINITY;
  constexpr std::integral_constant<int, 8> at_once{};  // requests in flight; looking again: 2
  constexpr std::integral_constant<int, 2> again{};
  auto sweep = [&](auto f, auto u) SKD_INLINE {
    constexpr int U = decltype(u)::value, STEP = 4 * NW * 64;
    for (int base = 0; base < V; base += U * STEP) {
      floatx4 v[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int at = base + i * STEP + 4 * tid;
        v[i] = floatx4{NAN, NAN, NAN, NAN};
        if (at < V && sh.wanted[at >> piece_bits]) {
          if (vec && at + 4 <= V) {
            v[i] = *(const floatx4 *)(z + at);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = at + j < V ? z[at + j] : NAN;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (__any(fmaxf(fmaxf(v[i][0], v[i][1]), fmaxf(v[i][2], v[i][3])) >= low))
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const bool hit = v[i][j] >= low && v[i][j] < high;
            if (__any(hit)) f(v[i][j] + 0.f, base + i * STEP + 4 * tid + j, hit);
          }
    }
  };
  // The smallest value whose bin is not behind `last`: from where it lies by arithmetic, give or take the roundings of place(), 64
  // candidates at a time.
  auto edge = [&](int last) SKD_INLINE -> float {
    const double w = 1.0 / (double)g.s, z0 = ((double)place - last) * w, m = (fabs((double)place) + BINS) * 0x1p-22 * w;
    const float from = (float)(z0 - m), to = (float)(z0 + m);  // (NaN, infinite: all values)
    uint32_t lo = key_of(from >= -FLT_MAX && from <= top ? from : -FLT_MAX), hi = key_of(to >= -FLT_MAX && to <= top ? to : top);
    while (lo < hi) {
      const uint32_t step = (hi - lo + 63) / 64, k = lo + min(lane * step, hi - lo);
      const u64 hits = __ballot(g.bin(top, place, value_of(k)) <= last);
      if (!hits) {
        lo = min(lo + 63 * step, hi - 1) + 1;
        continue;
      }
      const int l = __ffsll((long long)hits) - 1;
      hi = lo + min(l * step, hi - lo);
      if (l) lo = min(lo + (l - 1) * step + 1, hi);
      else lo = hi;
    }
    return value_of((uint32_t)__builtin_amdgcn_readfirstlane((int)hi)) + 0.f;
  };
  auto bounds = [&](int first, int last) SKD_INLINE {  // low and high for the bins from `first` to `last`
    low = uniform(fmaxf(lowest, last < BINS ? edge(last) : -FLT_MAX));
    high = uniform(first > 0 ? edge(first - 1) : INFINITY);
  };
  // Lists the tokens of the bounds, a wave's in its own part of the list, their masses beside them, and takes their keys into
  // registers; whether all of them fit.  lo, hi: their smallest and largest key.
  bool whole = false;
  constexpr int PER = CAP / (NW * 64);
  uint32_t key[PER];
  const int own_list = wave * (64 * PER);
  auto mass_in = [&](int i) { return sh.weight[own_list + lane + 64 * i]; };
  auto index_of = [&](int i) { return sh.index[own_list + lane + 64 * i]; };
  auto list = [&]() SKD_INLINE {
    __syncthreads();
    if (now(tid) == 0) {
      sh.n = 0;
      sh.lo = 0xffffffffu;
      sh.hi = 0;
    }
    int n = 0;
    __syncthreads();
    sweep([&](float x, int at, bool hit) {
      const u64 hits = __ballot(hit);
      const int to = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(hits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hits, 0));
      if (hit && to < 64 * PER) {
        sh.value[own_list + to] = x;
        sh.index[own_list + to] = at;
      }
      n += __popcll(hits);
    }, at_once);
    if (n && lane == 0) atomicAdd(&sh.n, n <= 64 * PER ? n : CAP + 1);
    __syncthreads();
    whole = sh.n <= CAP;
    uint32_t most = 0, least = 0;     // of key and of ~key
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = lane + 64 * i;
      key[i] = 0;
      if (whole && at < n) {
        key[i] = key_of(sh.value[own_list + at]);
        sh.weight[own_list + at] = g.mass(sh.value[own_list + at], top);
        most = max(most, key[i]);
        least = max(least, ~key[i]);
      }
    }
    if (!whole) {
      most = key_of(high < top ? high : top);
      least = ~key_of(low);
    }
    if (n || !whole) {
      most = wave_max(most);
      least = wave_max(least);
      if (lane == 0) {
        atomicMin(&sh.lo, ~least);
        atomicMax(&sh.hi, most);
      }
    }
    __syncthreads();
  };
  // The listed elements (is(i)) by buckets in an order, their weights added up bucket by bucket: the one in which enough(sum) comes
  // to hold, the sum before it, and its elements' order words and weights in LDS; false where there is none, or too many there.
  auto locate = [&](auto is, auto bucket_of, auto word, auto weight, auto enough) SKD_INLINE -> bool {
    const bool few = sh.n <= 64;
    sh.bucket[tid] = 0;
    if (now(tid) == 0) {
      sh.bucket_at = few ? 0 : 1 << 30;
      sh.bucket_before = 0;
      sh.near_n = 0;
    }
    __syncthreads();
    if (few) {  // one bucket
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (is(i)) {
          const int n = atomicAdd(&sh.near_n, 1);
          sh.near_key[n] = word(i);
          sh.near_mass[n] = weight(i);
        }
      __syncthreads();
      return true;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (is(i)) atomicAdd(&sh.bucket[bucket_of(i)], weight(i));
    __syncthreads();
    const u64 own = sh.bucket[tid], scan = wave_scan64(own);
    if (lane == 63) sh.wave_mass[wave] = scan;
    __syncthreads();
    u64 before = 0;
    for (int w = 0; w < wave; ++w) before += sh.wave_mass[w];
    const u64 hits = __ballot(enough(before + scan));
    if (hits) {
      const int l = __ffsll((long long)hits) - 1;
      if (lane == l) atomicMin(&sh.bucket_at, tid);
    }
    __syncthreads();
    const int at = sh.bucket_at;
    if (at >= 1024) return false;
    if (tid == at) sh.bucket_before = before + scan - own;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (is(i) && bucket_of(i) == at) {
        const int n = atomicAdd(&sh.near_n, 1);
        if (n < 64) {
          sh.near_key[n] = word(i);
          sh.near_mass[n] = weight(i);
        }
      }
    __syncthreads();
    return sh.near_n <= 64;
  };
  // Of the located elements the largest order word (ascending: the smallest) with enough(sum of the weights of those whose word is at
  // least, or at most, as large), and that sum; false: none.  (By one wave: a loop of 64 by all of them takes 5 us.)
  u64 found_sum = 0;
  auto near = [&](bool ascending, auto enough, uint32_t &at) SKD_INLINE -> bool {
    if (wave == 0) {
      const int n = sh.near_n;
      const uint32_t own = lane < n ? sh.near_key[lane] : 0;
      const u64 w = lane < n ? sh.near_mass[lane] : 0;
      u64 sum = sh.bucket_before;
      for (int j = 0; j < n; ++j) {
        const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)own, j);
        const u64 wj = lane64(w, j);
        sum += (ascending ? k <= own : k >= own) ? wj : 0ull;
      }
      const bool ok = lane < n && enough(sum);
      const uint32_t best = wave_max(ok ? ascending ? ~own : own : 0u), word = ascending ? ~best : best;
      const u64 at_word = __ballot(ok && own == word);
      if (lane == 0) {
        sh.found = word;
        sh.near_n = at_word ? 1 : 0;
      }
      if (at_word && lane == __ffsll((long long)at_word) - 1) sh.found_sum = sum;
    }
    __syncthreads();
    at = sh.found;
    found_sum = sh.found_sum;
    return sh.near_n != 0;
  };
  // sum of weight(logit) over the listed tokens, or over what they would be
  auto sum_of = [&](auto weight, int set) SKD_INLINE -> u64 {
    u64 mine = 0;
    if (whole) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (key[i]) mine += weight(value_of(key[i]));
    } else {
      sweep([&](float x, int at, bool hit) {
        if (hit) mine += weight(x);
      }, again);
    }
    mine = wave_sum64(mine);
    if (lane == 0) sh.sum[set][wave] = mine;
    __syncthreads();
    u64 s = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) s += sh.sum[set][w];
    return s;
  };
  // Where there are too many: of the order words word(logit, index) from `first` to `last` the one at which enough(sum of the weights
  // up to it) comes to hold, ten bits of it with every look at the tokens; false: nowhere.
  auto narrow = [&](auto word, auto weight, auto enough, uint32_t first, uint32_t last, uint32_t &at) SKD_INLINE -> bool {
    u64 before = 0;
    while (true) {
      const int shift = max(22 - __clz((int)((last - first) | 1)), 0);
      __syncthreads();
      sh.bucket[tid] = 0;
      if (now(tid) == 0) sh.bucket_at = 1 << 30;
      __syncthreads();
      auto add = [&](float x, int i) {
        const uint32_t w = word(x, i);
        if (w >= first && w <= last) atomicAdd(&sh.bucket[(w - first) >> shift], weight(x));
      };
      if (whole) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (const uint32_t x = (uint32_t)now((int)key[i])) add(value_of(x), index_of(i));
      } else {
        sweep([&](float x, int i, bool hit) {
          if (hit) add(x, i);
        }, again);
      }
      __syncthreads();
      const u64 own = sh.bucket[tid], scan = wave_scan64(own);
      if (lane == 63) sh.wave_mass[wave] = scan;
      __syncthreads();
      u64 run = before;
      for (int w = 0; w < wave; ++w) run += sh.wave_mass[w];
      const u64 hits = __ballot(enough(run + scan));
      if (hits && lane == __ffsll((long long)hits) - 1) atomicMin(&sh.bucket_at, tid);
      __syncthreads();
      const int bucket = sh.bucket_at;
      if (bucket >= 1024) return false;
      if (tid == bucket) sh.bucket_before = run + (scan - own);
      __syncthreads();
      before = sh.bucket_before;
      first += (uint32_t)bucket << shift;
      if (shift == 0) {
        at = first;
        return true;
      }
      last = min(last, first + ((1u << shift) - 1));
    }
  };
  // The largest key among the listed tokens, or what they would be, from which on enough(weight) holds; 0: it does not even for all.
  // summed: found_sum is that weight.
  bool summed = false;
  auto find = [&](auto weight, auto weight_at, auto enough) SKD_INLINE -> uint32_t {
    summed = false;
    if (sh.n == 0) return 0;
    uint32_t at;
    if (whole) {
      const float most = value_of(sh.hi), least = value_of(sh.lo);
      const float s = most > least ? fminf(1023.0f / (most - least), 3.0e38f) : 0.f;
      if (locate([&](int i) { return key[i] != 0; }, [&](int i) { return (int)fminf((most - value_of(key[i])) * s, 1023.0f); }, [&](int i) { return key[i]; },
                 weight_at, enough))
        return (summed = near(false, enough, at)) ? at : 0;
      const bool none = sh.bucket_at >= 1024;
      __syncthreads();
      if (none) return 0;
    }
    return narrow([&](float x, int) { return ~key_of(x); }, weight, enough, ~sh.hi, ~sh.lo, at) ? ~at : 0;
  };
  // First bin up to `last` at which enough(running sum) holds, the sum before it; BINS + 1: none, the sum of them all.
  auto first_bin = [&](const auto *of, int last, auto enough, auto &before) SKD_INLINE -> int {
    typedef typename std::remove_reference<decltype(before)>::type S;
    const S x = tid <= last ? (S)of[tid] : (S)0, scan = wave_scan64(x);
    if (lane == 63) sh.wave_mass[wave] = __builtin_bit_cast(u64, scan);
    if (now(tid) == 0) sh.bucket_at = BINS + 1;
    __syncthreads();
    S run = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      if (w == wave) run = all;
      all += __builtin_bit_cast(S, sh.wave_mass[w]);
    }
    const u64 hits = __ballot(tid <= last && enough(run + scan));
    if (hits && lane == __ffsll((long long)hits) - 1) atomicMin(&sh.bucket_at, tid);
    __syncthreads();
    const int at = sh.bucket_at;
    if (tid == at) sh.bucket_before = __builtin_bit_cast(u64, run + (scan - x));
    __syncthreads();
    before = at <= BINS ? __builtin_bit_cast(S, sh.bucket_before) : all;
    __syncthreads();
    return at;
  };
  auto mass_at = [&](float x) { return g.mass(x, top); };
  // the bins of the row: sums over the pieces of what(piece, bin of the piece)
  static_assert(2 * BINS == NW * 64, "two threads for every bin, each with half of the pieces");
  auto add_bins = [&](auto *to, auto what) SKD_INLINE {
    typedef typename std::remove_reference<decltype(*to)>::type S;
    const int bin = tid % BINS, half = wave / (NW / 2);
    S sum = 0;
    for (int c0 = half; c0 < pieces; c0 += 32) {  // (all requested before the first is used)
      S x[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int c = min(c0 + 2 * j, pieces - 1);
        x[j] = what(c, max(bin - sh.shift[c], 0));
      }
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (c0 + 2 * j < pieces && bin >= sh.shift[c0 + 2 * j]) sum += x[j];
    }
    if (half) ((S *)sh.bucket)[bin] = sum;
    __syncthreads();
    if (!half) to[bin] = sum + ((S *)sh.bucket)[bin];
    __syncthreads();
  };

  const int floor_bin = greedy ? 0 : g.bin(top, place, lowest);
  int bound = floor_bin;              // top-k or min-p: the bin of the k-th, or of the lowest that min-p leaves
  u64 few = 0;                        // tokens up to that bin
  if (p.counts && !greedy) {
    add_bins(sh.count, [&](int c, int i) { return bins[c].count[i]; });
    u64 before = 0;
    if (p.by_k) bound = min(bound, first_bin(sh.count, BINS - 1, [&](u64 n) { return n >= (u64)p.k; }, before));
    if (!p.by_k)
      for (int i = 0; i <= min(bound, BINS - 1); i += 64) few += wave_sum64(i + lane <= min(bound, BINS - 1) ? (u64)sh.count[i + lane] : 0ull);
  }
  if (!greedy && (p.by_k || (p.counts && bound < BINS && few <= CAP))) {
    if (tid < pieces) sh.wanted[tid] = sh.shift[tid] <= bound || (bound == BINS && sh.top[tid] > -INFINITY);
    bounds(0, bound);
    list();
    float cut = lowest;
    if (p.by_k) {
      const uint32_t t = find([](float) { return 1ull; }, [](int) { return 1ull; }, [&](u64 n) { return n >= (u64)p.k; });
      if (t) cut = fmaxf(cut, value_of(t));
    }
    auto kept = [&](int i) { return key[i] != 0 && key[i] >= key_of(cut); };
    auto total_kept = [&]() SKD_INLINE -> u64 {
      if (!whole) return sum_of([&](float x) { return x >= cut ? mass_at(x) : 0ull; }, 0);
      u64 mine = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) mine += kept(i) ? mass_in(i) : 0ull;
      mine = wave_sum64(mine);
      if (lane == 0) sh.sum[0][wave] = mine;
      __syncthreads();
      u64 s = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) s += sh.sum[0][w];
      return s;
    };
    u64 all = total_kept();
    if (p.by_p) {
      const double need = (double)p.top_p * (double)all;
      __syncthreads();
      const uint32_t t = find(mass_at, mass_in, [&](u64 m) { return (double)m >= need; });
      if (t && value_of(t) >= cut) {
        cut = fminf(value_of(t), top);
        if (summed) {
          all = found_sum;
        } else {
          __syncthreads();
          all = total_kept();
        }
      }
    }
    cut = fminf(cut, top);
    const double target = (double)p.u * (double)all;
    // the first index up to which the mass passes the target
    const int shift = max(32 - __clz(V - 1) - 10, 0);
    int token = V - 1;                // (always replaced: the target is below the mass)
    __syncthreads();
    const auto passed = [&](u64 m) { return (double)m > target; };
    uint32_t at;
    bool is;
    if (whole && locate(kept, [&](int i) { return index_of(i) >> shift; }, [&](int i) { return (uint32_t)index_of(i); }, mass_in, passed))
      is = near(true, passed, at);
    else
      is = narrow([&](float, int i) { return (uint32_t)i; }, [&](float x) { return x >= cut ? mass_at(x) : 0ull; }, passed, 0, V - 1, at);
    if (is) token = (int)at;
    if (now(tid) == 0) answer(token);
    return;
  }

  float cut = lowest;                 // keep z >= cut (and above -infinity)
  double target = 0.0;
  if (!greedy) {
    if (p.by_p || p.counts) {
      // ---- top-p alone, or a min-p that leaves many
      add_bins(sh.mass, [&](int c, int i) { return (double)bins[c].mass[i] * sh.scale[c]; });
      int bin = floor_bin;
      auto list_bin = [&]() SKD_INLINE {
        if (tid < pieces) {
          const int i = bin - sh.shift[tid];
          sh.wanted[tid] = sh.top[tid] > -INFINITY && (bin >= BINS || (i >= 0 && bins[tid].mass[i] != 0));
        }
        bounds(bin, bin);
        list();
      };
      double before = 0.0, total;     // masses: of the bins before `bin`, of all that min-p leaves
      if (p.counts) {                 // of the lowest bin only a part
        for (int i = 0; i < bin; i += 64) before += wave_sum64(i + lane < bin ? sh.mass[i + lane] : 0.0);
        list_bin();
        total = before + (double)sum_of(mass_at, 0);
        __syncthreads();
      } else {
        total = lane < pieces ? sh.kept[lane] : 0.0;
        if (lane + 64 < pieces) total += sh.kept[lane + 64];
        total = wave_sum64(total);
      }
      if (p.by_p) {
        const double need = (double)p.top_p * total;
        const int first = first_bin(sh.mass, floor_bin - 1, [&](double m) { return m >= need; }, before);
        if (first < floor_bin || !p.counts) {
          bin = min(first, floor_bin);
          list_bin();
        }
        const uint32_t t = find(mass_at, mass_in, [&](u64 m) { return before + (double)m >= need; });
        if (t) cut = fmaxf(cut, value_of(t));
      }
      cut = fminf(cut, top);
      // kept masses of the pieces: their bins above the cut's, and of that one what is not below the cut
      if (whole) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (key[i] && value_of(key[i]) >= cut) atomicAdd(&sh.part[index_of(i) >> piece_bits], mass_in(i));
      } else {
        sweep([&](float x, int at, bool hit) {
          if (hit && x >= cut) atomicAdd(&sh.part[at >> piece_bits], mass_at(x));
        }, again);
      }
      __syncthreads();
      for (int c = wave; c < pieces; c += NW) {
        double m = 0.0;
        const int most = sh.top[c] == -INFINITY ? 0 : min(bin - sh.shift[c], BINS);
  #pragma unroll 8
      for (int i = lane; i < BINS; i += 64) m += i < most ? (double)bins[c].mass[i] : 0.0;
        m = wave_sum64(m) * sh.scale[c] + (double)sh.part[c];
        if (lane == 0) sh.kept[c] = m;
      }
      __syncthreads();
    }
    double all = lane < pieces ? sh.kept[lane] : 0.0;
    if (lane + 64 < pieces) all += sh.kept[lane + 64];
    target = (double)p.u * wave_sum64(all);
  }
  // ---- the piece in which the running mass passes the target (with rounding, or u = 0, perhaps one behind), and the token
  int piece = 0;
  double run = 0.0;
  if (greedy) {
    while (piece < pieces - 1 && sh.top[piece] != top) ++piece;
  } else {
    for (int c0 = 0; c0 < pieces; c0 += 64) {
      const double m = c0 + lane < pieces ? sh.kept[c0 + lane] : 0.0, scan = wave_scan64(m);
      const u64 hits = __ballot(c0 + lane < pieces && run + scan > target);
      const int at = hits ? __ffsll((long long)hits) - 1 : min(63, pieces - 1 - c0);
      piece = c0 + at;
      if (!hits && piece < pieces - 1) run += lane64(scan, 63);
      else if (at) run += lane64(scan, at - 1);  // (not above the target)
      if (hits) break;
    }
  }
  auto mass_of = [&](float x) -> u64 { return !(x >= cut) || x == -INFINITY ? 0ull : greedy ? 1ull : mass_at(x); };
  int last = 0;                       // the last token that has a mass: what rounding at the very end leaves
  for (; piece < pieces && top > -INFINITY; ++piece) {
    // a wave takes a sixteenth, 256 tokens at a time
    const int begin = piece * a.piece, end = min(begin + a.piece, V), share = a.piece / NW, w0 = begin + wave * share, w1 = min(w0 + share, end);
    u64 mine = 0, own[4];
    int seen = -1;
    for (int at = w0; at < w1; at += 256) {
      const floatx4 v = load4(z, at + 4 * lane, w1, vec);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        own[j] = mass_of(v[j]);
        mine += own[j];
        if (own[j]) seen = at + 4 * lane + j;
      }
    }
    mine = wave_sum64(mine);
    seen = (int)wave_max((uint32_t)(seen + 1)) - 1;
    __syncthreads();
    if (lane == 0) {
      sh.sum[0][wave] = mine;
      sh.seen[wave] = seen;
    }
    __syncthreads();
    double upto = run;
    int win = -1;
    for (int w = 0; w < NW; ++w) {
      last = max(last, sh.seen[w]);
      if (win < 0 && upto + (double)sh.sum[0][w] > target) win = w;
      if (win < 0) upto += (double)sh.sum[0][w];
    }
    if (win < 0) {
      run = upto;
      continue;
    }
    if (wave != win) return;
    u64 before = 0;
    for (int at = w0; at < w1; at += 256) {
      if (share > 256) {  // (a share of 256 is there already)
        const floatx4 v = load4(z, at + 4 * lane, w1, vec);
#pragma unroll
        for (int j = 0; j < 4; ++j) own[j] = mass_of(v[j]);
      }
      const u64 sum = own[0] + own[1] + own[2] + own[3], scan = wave_scan64(sum);
      u64 x = before + scan - sum;
      int found = 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x += own[j];
        if (found == 4 && own[j] && upto + (double)x > target) found = j;
      }
      const u64 hits = __ballot(found < 4);
      if (hits) {
        const int l = __ffsll((long long)hits) - 1;
        last = at + 4 * l + __shfl(found, l);
        break;
      }
      before += lane64(scan, 63);
    }
    if (lane == 0) answer(last);
    return;
  }
  if (now(tid) == 0) answer(last);
}
#undef SKD_INLINE

// Tokens of a thread of k_sample_bins, pieces of 256 times as many: few enough pieces for their bins to be small beside the logits,
// enough of them for the chip (up to 2048 pieces instead of 4096: 128 rows of 131072 61 to 67 us instead of 59 to 60; at least 16
// tokens a thread instead of 8: one row the same).
int per_thread(int rows, int vocab) {
  int per = 8;
  while (per < 64 && (((long)rows * vocab + 256L * per - 1) / (256L * per) > 4096 || (vocab + 256 * per - 1) / (256 * per) > PIECES)) per *= 2;
  return per;
}

}  // namespace

size_t sample_rows_bins(int rows, int vocab) {
  const int piece = 256 * per_thread(rows, vocab);
  return (size_t)rows * ((vocab + piece - 1) / piece);
}

bool sample_rows_fit(int rows, int vocab) { return launch_fits((long)sample_rows_bins(rows, vocab), 256) && launch_fits(rows, NW * 64); }

void sample_rows(hipStream_t s, const SampleRows &call) {
  SampleRows a = call;
  const int per = per_thread(a.rows, a.vocab);
  a.piece = 256 * per;
  a.pieces = (a.vocab + a.piece - 1) / a.piece;
  const dim3 grid((unsigned)a.rows * a.pieces);
  if (per == 8) SKD_LAUNCH(k_sample_bins<8>, grid, dim3(256), 0, s, a);
  else if (per == 16) SKD_LAUNCH(k_sample_bins<16>, grid, dim3(256), 0, s, a);
  else if (per == 32) SKD_LAUNCH(k_sample_bins<32>, grid, dim3(256), 0, s, a);
  else SKD_LAUNCH(k_sample_bins<64>, grid, dim3(256), 0, s, a);
  static std::atomic<uint64_t> done{0};
  (void)allow_lds(done, {(const void *)k_sample_pick}, sizeof(Pick));
  SKD_LAUNCH(k_sample_pick, dim3(a.rows), dim3(NW * 64), sizeof(Pick), s, a);
}

}  // namespace skd
