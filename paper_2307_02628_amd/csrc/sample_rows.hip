// One token a row from fp32 logits, with the row's own temperature, top-k, top-p and min-p and a given uniform number.
//
// With m_i = exp((z_i - max z) / T): kept are the tokens with m_i >= min_p that are among the k largest logits (ties with the k-th
// too), of these the smallest set of largest ones whose mass reaches top_p of theirs (ties with the last too).  All three are
// "z >= threshold", so the kernel looks for one threshold and then for the first index whose running mass over the tokens at or
// above it exceeds u times their mass.
//
// Masses are integers in units of 2^-45 (exponentials in 64 bits, to 2^-44): sums do not depend on their order, so neither
// atomics nor the share of a wave change a draw, and a draw that 64-bit arithmetic decides comes out the same.  What lies
// 32 T below the largest logit has no mass, is never drawn, and is left out from the start.
//
// One workgroup of 16 waves per row, every wave a contiguous piece of it.  Passes over the row: extremes; counts and masses
// by bins of equal width; for top-k and top-p each the values of the bin in which the threshold lies, among which it is found bit
// by bit; running masses.  The row comes from HBM once and from L2 after that.
#include "sample_rows.h"

#include <math.h>

#include "bf16_device.h"

namespace skd {

namespace {

typedef unsigned long long u64;

constexpr int NW = 16, BINS = 2048, CAP = 4096, ROUND = 256;  // ROUND: tokens of a wave at a time

__device__ inline uint32_t key_of(float z) {  // ordered as the values are
  const uint32_t b = __float_as_uint(z);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline u64 shfl_xor64(u64 v, int o) {
  return (u64)(uint32_t)__shfl_xor((int)(uint32_t)v, o) | (u64)(uint32_t)__shfl_xor((int)(uint32_t)(v >> 32), o) << 32;
}
__device__ inline u64 wave_sum64(u64 v) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) v += shfl_xor64(v, o);
  return v;
}

__device__ inline float usable(float z) { return z == z ? z + 0.f : -INFINITY; }  // (-0 as 0)
struct Shared {
  double tab[64];             // 2^(i / 64)
  uint32_t count[BINS];
  u64 mass[BINS];
  float cand[CAP];
  int n_cand;
  u64 part[2][NW];
  float lo[NW], hi[NW];
  u64 run[NW][SAMPLE_ROWS_VOCAB / NW / ROUND];
};

struct Row {
  const float *z;
  int V, begin, end;          // begin, end: this wave's tokens
  bool vec;                   // 16-byte loads
  float top;                  // largest logit
  double c;                   // 64 log2(e) / T
  int lane;

  // f(first token of the lane's four, the four logits); NaN and what lies past the row: -infinity
  template <typename F>
  __device__ void each(F f) const {
    constexpr int U = 4;
    for (int i = begin; i < end; i += U * ROUND) {
      floatx4 v[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int at = i + k * ROUND + 4 * lane;
        if (vec && at + 4 <= end) {
          v[k] = *(const floatx4 *)(z + at);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[k][j] = at + j < end ? z[at + j] : -INFINITY;
        }
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (i + k * ROUND >= end) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[k][j] = usable(v[k][j]);
        f(i + k * ROUND + 4 * lane, v[k]);
      }
    }
  }
  // mass in units of 2^-45; 64 log2 of it is split into n + r: 2^(n / 64) from the table, 2^(r / 64) by its series (|r| <= 1/2:
  // the first term left out is below 2^-44)
  __device__ u64 mass(float x, const double *tab) const {
    if (x == top) return 1ull << 45;
    const double y = fmax(((double)x - (double)top) * c, -64.0 * 60);
    const double t = y + 0x1.8p52, r = (y - (t - 0x1.8p52)) * (0.69314718055994530942 / 64);
    const int n = (int)(uint32_t)__double_as_longlong(t);
    const double p = 1.0 + r * (1.0 + r * (0.5 + r * (1.0 / 6 + r * (1.0 / 24))));
    const double m = __longlong_as_double(__double_as_longlong(tab[n & 63] * p) + ((long long)(n >> 6) << 52));
    return (u64)(__double_as_longlong(m + 128.0) - __double_as_longlong(128.0));
  }
};

__device__ inline u64 block_sum(u64 v, u64 *part, int wave, int lane) {
  v = wave_sum64(v);
  if (lane == 0) part[wave] = v;
  __syncthreads();
  u64 s = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) s += part[w];
  return s;
}

__global__ __launch_bounds__(NW * 64) void k_sample_rows(SampleRows a) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, b = blockIdx.x, V = a.vocab;
  const int piece = (V + NW * ROUND - 1) / (NW * ROUND) * ROUND;
  Row row;
  row.z = a.logits + (long)b * a.stride;
  row.V = V;
  row.begin = min(wave * piece, V);
  row.end = min(row.begin + piece, V);
  row.vec = ((uintptr_t)row.z & 15) == 0;
  row.lane = lane;
  const float T = a.temperature ? a.temperature[b] : 1.0f;
  const int k = a.top_k ? a.top_k[b] : 0;
  const float top_p = a.top_p ? a.top_p[b] : 1.0f, min_p = a.min_p ? a.min_p[b] : 0.f;
  const float u = fminf(fmaxf(a.u[b], 0.f), 0x1.fffffep-1f);  // (NaN: 0)

  // ---- extremes
  float hi = -INFINITY, lo = INFINITY;
  row.each([&](int, floatx4 z) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      hi = fmaxf(hi, z[j]);
      lo = fminf(lo, z[j] == -INFINITY ? INFINITY : z[j]);
    }
  });
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    hi = fmaxf(hi, __shfl_xor(hi, o));
    lo = fminf(lo, __shfl_xor(lo, o));
  }
  if (lane == 0) {
    sh.hi[wave] = hi;
    sh.lo[wave] = lo;
  }
  if (tid < 64) sh.tab[tid] = exp2(tid / 64.0);
  for (int i = tid; i < BINS; i += NW * 64) {
    sh.count[i] = 0;
    sh.mass[i] = 0;
  }
  __syncthreads();
  for (int w = 0; w < NW; ++w) {
    hi = fmaxf(hi, sh.hi[w]);
    lo = fminf(lo, sh.lo[w]);
  }
  row.top = hi;
  // greedy: no temperature, or nothing but the largest has mass
  const bool greedy = !(T > 0.f) || hi == INFINITY || hi == -INFINITY;
  row.c = greedy ? 1.0 : 64.0 * 1.44269504088896340736 / (double)T;
  float floor_ = hi;                      // tokens below have no mass, or too little
  if (!greedy) {
    double f = (double)hi - 32.0 * (double)T;
    if (min_p > 0.f) f = fmax(f, min_p < 1.f ? (double)hi + (double)T * log((double)min_p) : (double)hi);
    // the smallest float that is not below f
    floor_ = (float)f;
    if ((double)floor_ < f) floor_ = nextafterf(floor_, INFINITY);
    floor_ = fminf(fmaxf(floor_, lo), hi);
  }
  uint32_t thr = key_of(floor_);          // keep key >= thr
  const bool by_k = !greedy && k > 0 && k < V, by_p = !greedy && top_p < 1.f;

  if (by_k || by_p) {
    // ---- counts and masses by bins of equal width, the largest logits in bin 0
    const float width = hi - floor_;
    const float s = width > 0.f ? fminf((float)BINS / width, 3.0e38f) : 0.f;
    auto bin_of = [&](float z) { return (int)fminf((hi - z) * s, (float)(BINS - 1)); };
    row.each([&](int, floatx4 z) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (z[j] >= floor_) {
          const int bin = bin_of(z[j]);
          atomicAdd(&sh.count[bin], 1u);
          if (by_p) atomicAdd(&sh.mass[bin], row.mass(z[j], sh.tab));
        }
    });
    __syncthreads();
    // The largest threshold t in the first bin with (weight of the bins before and of its values from t on) reaching a
    // target; `need` says whether a weight does.  Returns the weight of the values above floor_ and at or above t.
    auto find = [&](auto weight_of_bin, auto weight_of, auto need) -> u64 {
      // every wave looks the bins through by itself: 64 at a time
      u64 before = 0;
      int bin = -1;
      for (int i = 0; i < BINS && bin < 0; i += 64) {
        u64 w = weight_of_bin(i + lane);
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
          const u64 other = (u64)(uint32_t)__shfl_up((int)(uint32_t)w, o) | (u64)(uint32_t)__shfl_up((int)(uint32_t)(w >> 32), o) << 32;
          if (lane >= o) w += other;
        }
        const u64 hits = __ballot(need(before + w));
        const int at = hits ? __ffsll((long long)hits) - 1 : 63;
        const u64 upto = (u64)(uint32_t)__shfl((int)(uint32_t)w, at) | (u64)(uint32_t)__shfl((int)(uint32_t)(w >> 32), at) << 32;
        if (hits) {
          bin = i + at;
          before += upto - weight_of_bin(bin);
        } else {
          before += upto;
        }
      }
      if (bin < 0) return before;         // all of them together do not reach it: no cut
      const bool listed = sh.count[bin] <= CAP;
      __syncthreads();
      if (tid == 0) sh.n_cand = 0;
      __syncthreads();
      if (listed)
        row.each([&](int, floatx4 z) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (z[j] >= floor_ && bin_of(z[j]) == bin) sh.cand[atomicAdd(&sh.n_cand, 1)] = z[j];
        });
      __syncthreads();
      constexpr int PER = CAP / (NW * 64);
      uint32_t key[PER];
      u64 w[PER];
      if (listed) {
        const int C = sh.n_cand;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const bool is = tid + i * NW * 64 < C;
          const float z = is ? sh.cand[tid + i * NW * 64] : 0.f;
          key[i] = is ? key_of(z) : 0u;
          w[i] = is ? weight_of(z) : 0ull;
        }
      }
      uint32_t t = 0;
      u64 got = 0;
      for (int bit = 31, set = 0; bit >= 0; --bit, set ^= 1) {
        const uint32_t trial = t | 1u << bit;
        u64 mine = 0;
        if (listed) {
#pragma unroll
          for (int i = 0; i < PER; ++i) mine += key[i] >= trial ? w[i] : 0ull;
        } else {
          row.each([&](int, floatx4 z) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (z[j] >= floor_ && bin_of(z[j]) == bin && key_of(z[j]) >= trial) mine += weight_of(z[j]);
          });
        }
        const u64 sum = before + block_sum(mine, sh.part[set], wave, lane);
        if (need(sum)) {
          t = trial;
          got = sum;
        }
      }
      __syncthreads();
      thr = max(thr, t);
      return got;
    };
    if (by_k) {
      (void)find([&](int i) { return (u64)sh.count[i]; }, [&](float) { return 1ull; }, [&](u64 n) { return n >= (u64)k; });
    }
    if (by_p) {
      // masses of what top-k leaves: bins below the threshold's are dropped, its own is added up again
      u64 total = 0;
      if (by_k) {
        u64 mine = 0;
        row.each([&](int, floatx4 z) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (z[j] >= floor_ && key_of(z[j]) >= thr) mine += row.mass(z[j], sh.tab);
        });
        total = block_sum(mine, sh.part[0], wave, lane);
      } else {
        u64 mine = 0;
        for (int i = tid; i < BINS; i += NW * 64) mine += sh.mass[i];
        total = block_sum(mine, sh.part[0], wave, lane);
      }
      __syncthreads();
      const double target = (double)fmaxf(top_p, 0.f) * (double)total;
      // (values that top-k drops lie below those that reach the target, so they may stay in the bins)
      (void)find([&](int i) { return sh.mass[i]; }, [&](float z) { return row.mass(z, sh.tab); }, [&](u64 m) { return (double)m >= target; });
    }
    thr = min(thr, key_of(hi));
  }

  // ---- running masses in the order of the indices
  auto mass_of = [&](float z) -> u64 { return key_of(z) < thr || z == -INFINITY ? 0ull : greedy ? (z == hi ? 1ull : 0ull) : row.mass(z, sh.tab); };
  u64 mine = 0;
  row.each([&](int at, floatx4 z) {
    u64 m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) m += mass_of(z[j]);
    m = wave_sum64(m);
    if (lane == 0) sh.run[wave][(at - row.begin) / ROUND] = m;
    mine += m;
  });
  if (lane == 0) sh.part[1][wave] = mine;
  __syncthreads();
  u64 all = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) all += sh.part[1][w];
  const double target = greedy ? 0.0 : (double)u * (double)all;
  u64 run = 0;
  int win = NW - 1;
  for (int w = 0; w < NW; ++w) {
    if ((double)(run + sh.part[1][w]) > target) {
      win = w;
      break;
    }
    run += sh.part[1][w];
  }
  if (wave != win) return;
  int token = 0;                          // (a row without a usable logit)
  for (int i = row.begin; i < row.end; i += ROUND) {
    const u64 m = sh.run[wave][(i - row.begin) / ROUND];
    if (!((double)(run + m) > target)) {
      run += m;
      continue;
    }
    u64 own[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = i + 4 * lane + j;
      own[j] = mass_of(at < row.end ? usable(row.z[at]) : -INFINITY);
      sum += own[j];
    }
    u64 upto = sum;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const u64 other = (u64)(uint32_t)__shfl_up((int)(uint32_t)upto, o) | (u64)(uint32_t)__shfl_up((int)(uint32_t)(upto >> 32), o) << 32;
      if (lane >= o) upto += other;
    }
    u64 x = run + upto - sum;
    int found = 4;
#pragma unroll
    for (int j = 3; j >= 0; --j) {
      u64 at = x;
      for (int q = 0; q <= j; ++q) at += own[q];
      if ((double)at > target) found = j;
    }
    const u64 hits = __ballot(found < 4);
    const int l = __ffsll((long long)hits) - 1;
    token = i + 4 * l + __shfl(found, l);
    break;
  }
  if (lane == 0) {
    a.tokens[b] = token;
    if (a.tokens2) a.tokens2[b] = token;
  }
}

}  // namespace

void sample_rows(hipStream_t s, const SampleRows &a) {
  SKD_LAUNCH(k_sample_rows, dim3(a.rows), dim3(NW * 64), 0, s, a);
}

}  // namespace skd
