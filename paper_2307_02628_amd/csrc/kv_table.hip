// Block tables on the device.  A table names pages; a page that no entry names is free, so nothing else has to be kept from call
// to call.  All of it is integer work on a few hundred KB: what counts is the number of launches that have to follow each other.
#include "kv_table.h"

#include <algorithm>

namespace skd {

namespace {

constexpr int PAGE_CHUNKS = 16 * TABLE_CHUNK;  // of pages, whose counts are added up as they are (3 million pages, `over` for more than 1024 chunks: 54 -> 76 us)
__host__ __device__ inline int chunks_of(int n) { return (int)(((long)n + TABLE_CHUNK - 1) / TABLE_CHUNK); }
// Counts of n chunks and, beyond `most` of them, of chunks of chunks (`over`), so that who needs the sum of all before a place reads some
// thousands at most: 2^24 rows are 2^14 chunks, 2^31 pages 2^21.  Atomics add those up, of whole numbers, in any order the same; to a few
// neighbouring places they take 10 to 20 ns each, so that they are for large numbers alone.
struct Counts {
  int32_t *of, *over;
  int n, most;
  __device__ bool far() const { return n > most; }
  __device__ void set(int c, int x) const {
    of[c] = x;
    if (far()) atomicAdd(&over[c / TABLE_CHUNK], x);
  }
};
// Work of an assignment: what a page is to the entries of the new table, before any page is dealt out.
struct AssignWork {
  int32_t *uses;     // [pages]: entries that name it
  int32_t *writes;   // of them those that new tokens go to
  int32_t *loose;    // of them those that hold nothing yet
  Counts needs, copies;  // `need` and `copy` by chunks of rows
  Counts free;       // [chunks of pages]: pages that no entry names
  int32_t *lowest;   // [pages]: the first of those that new tokens go to
  int32_t *soft;     // [chunks]: pages that none names but loose ones
  int32_t *need, *copy;  // [rows]: pages that the row has to get; 1: one of them as a copy
  int32_t *list;     // free pages, ascending, as many as there could be entries for
  __host__ __device__ explicit AssignWork(const KvTable &t) {
    const int chunks = chunks_of(t.pages), row_chunks = chunks_of(t.rows);
    uses = t.work;
    writes = uses + t.pages;
    loose = writes + t.pages;
    needs.over = loose + t.pages;
    copies.over = needs.over + chunks_of(row_chunks);
    free.over = copies.over + chunks_of(row_chunks);
    lowest = free.over + chunks_of(chunks);  // (all before it begins with 0)
    needs.of = lowest + t.pages;
    copies.of = needs.of + row_chunks;
    free.of = copies.of + row_chunks;
    soft = free.of + chunks;
    need = soft + chunks;
    copy = need + t.rows;
    list = copy + t.rows;
    needs.n = copies.n = row_chunks;
    free.n = chunks;
    needs.most = copies.most = TABLE_CHUNK;
    free.most = PAGE_CHUNKS;
  }
};
__host__ __device__ inline long list_of(const KvTable &t) {
  const long entries = (long)t.rows * t.width;
  return entries < t.pages ? entries : t.pages;
}

struct Span {
  int held, upto;   // positions that a row holds, and will have been given pages for
  int first, last;  // entries that tokens to come go to: first .. last - 1
};
__device__ inline Span span_of(const KvTable &t, int r) {
  const long room = (long)t.width * t.page_tokens;  // below 2^30
  Span s;
  s.held = (int)min((long)max(t.len[r], 0), room);
  s.upto = (int)min((long)s.held + max(t.more[r], 0), room);
  s.first = s.held / t.page_tokens;
  s.last = s.upto > s.held ? (s.upto - 1) / t.page_tokens + 1 : s.first;
  return s;
}
__device__ inline bool written(Span s, int i) { return i >= s.first && i < s.last; }

__global__ __launch_bounds__(256) void k_table_fill(int32_t *w, long zero, long top) {
  for (long i = blockIdx.x * 256L + threadIdx.x; i < zero + top; i += gridDim.x * 256L) w[i] = i < zero ? 0 : 0x7fffffff;
}
// The rows in their new order, cut to what they will hold, and what every page is to them.
__global__ __launch_bounds__(256) void k_table_gather(KvTable t) {
  const AssignWork w(t);
  const uint32_t at = blockIdx.x * 256u + threadIdx.x, all = (uint32_t)t.rows * (uint32_t)t.width;
  if (at >= all) return;
  const int r = (int)(at / t.width), i = (int)(at % t.width);
  const int src = t.source ? t.source[r] : r;
  const Span s = span_of(t, r);
  int page = -1;
  if (src >= 0 && src < t.rows && i * t.page_tokens < s.upto) page = t.table[(long)src * t.width + i];
  if (page < 0 || page >= t.pages) page = -1;
  t.out[at] = page;
  if (page < 0) return;
  atomicAdd(&w.uses[page], 1);
  if (written(s, i)) {
    atomicAdd(&w.writes[page], 1);
    atomicMin(&w.lowest[page], (int)at);
    if (i * t.page_tokens >= s.held) atomicAdd(&w.loose[page], 1);
  }
}
// Whether an entry that new tokens go to needs a page of its own: it has none, or one that others name too, unless all of them are
// to be written and it is the first (the others get copies of what it holds before anything is written).
__device__ inline bool fresh(const AssignWork &w, int page, int at) {
  if (page < 0) return true;
  const int n = w.uses[page];
  return !(n == 1 || (n == w.writes[page] && w.lowest[page] == at));
}
__device__ inline int wave_sum_i(int v) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
  return v;
}
// A wave for each row: the pages that it needs; a workgroup for each chunk of pages: the free ones.
__global__ __launch_bounds__(256) void k_table_count(KvTable t, int rows4) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const AssignWork w(t);
  if ((int)blockIdx.x < rows4) {
    const int r = blockIdx.x * 4 + wave;
    if (r >= t.rows) return;
    const Span s = span_of(t, r);
    int n = 0, copy = 0;
    for (int i = s.first + lane; i < s.last; i += 64) {
      const int at = r * t.width + i, page = t.out[at];
      if (!fresh(w, page, at)) continue;
      ++n;
      if (page >= 0 && i * t.page_tokens < s.held) copy = 1;
    }
    n = wave_sum_i(n);
    copy = wave_sum_i(copy);
    if (lane == 0) {
      w.need[r] = n;
      w.copy[r] = copy;
    }
    return;
  }
  __shared__ int sum[2][4];
  const int c = blockIdx.x - rows4;
  int n = 0, soft = 0;
  for (int k = threadIdx.x; k < TABLE_CHUNK; k += 256) {
    const long p = (long)c * TABLE_CHUNK + k;
    if (p >= t.pages) break;
    const int uses = w.uses[p];
    n += uses == 0;
    soft += uses == w.loose[p];
  }
  n = wave_sum_i(n);
  soft = wave_sum_i(soft);
  if (lane == 0) {
    sum[0][wave] = n;
    sum[1][wave] = soft;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    w.free.set(c, sum[0][0] + sum[0][1] + sum[0][2] + sum[0][3]);
    w.soft[c] = sum[1][0] + sum[1][1] + sum[1][2] + sum[1][3];
  }
}
// Sums over the lanes of a wave (none is above the number of pages, or of entries): a lane's part of n values, and all of them.
__device__ inline int part_of(const int32_t *x, int n) {
  int v = 0;
  for (int i = threadIdx.x & 63; i < n; i += 64) v += x[i];
  return v;
}
__device__ inline int sum_of(const int32_t *x, int n) { return wave_sum_i(part_of(x, n)); }
__device__ inline int sum_of(const Counts &c) { return c.far() ? sum_of(c.over, chunks_of(c.n)) : sum_of(c.of, c.n); }
__device__ inline int part_before(const Counts &c, int chunk) {
  const int o = c.far() ? chunk / TABLE_CHUNK : 0;
  return part_of(c.over, o) + part_of(c.of + o * TABLE_CHUNK, chunk - o * TABLE_CHUNK);
}
__device__ inline int sum_before(const Counts &c, int chunk) { return wave_sum_i(part_before(c, chunk)); }
// of all values of which x are counts' own, those before place i
__device__ inline int sum_before(const Counts &c, const int32_t *x, int i) {
  const int chunk = i / TABLE_CHUNK;
  return wave_sum_i(part_before(c, chunk) + part_of(x + (long)chunk * TABLE_CHUNK, i - chunk * TABLE_CHUNK));
}
// Place of each of a chunk's pages for which `is` holds among them, in f(page, place).  256 threads, four pages each.
template <typename Is, typename F>
__device__ inline void each_in_chunk(int c, int pages, Is is, F f) {
  __shared__ int sum[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long p = (long)c * TABLE_CHUNK + threadIdx.x * 4;
  bool has[4];
  int n = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    has[k] = p + k < pages && is(p + k);
    n += has[k];
  }
  int upto = n;  // with this lane
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int x = __shfl_up(upto, o);
    if (lane >= o) upto += x;
  }
  if (lane == 63) sum[wave] = upto;
  __syncthreads();
  int at = upto - n;
  for (int i = 0; i < wave; ++i) at += sum[i];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (p + k < pages) {
      f((int)(p + k), has[k], at);
      at += has[k];
    }
}
// The free pages in ascending order; behind the workgroups of pages one for each chunk of rows: what they need together.
__global__ __launch_bounds__(256) void k_table_list(KvTable t) {
  const AssignWork w(t);
  if ((int)blockIdx.x >= w.free.n) {
    const int c = blockIdx.x - w.free.n, wave = threadIdx.x >> 6;
    if (wave < 2) {
      const int32_t *x = (wave ? w.copy : w.need) + (long)c * TABLE_CHUNK;
      const int all = sum_of(x, min(TABLE_CHUNK, t.rows - c * TABLE_CHUNK));
      if ((threadIdx.x & 63) == 0) (wave ? w.copies : w.needs).set(c, all);
    }
    return;
  }
  const long before = sum_before(w.free, blockIdx.x), room = list_of(t);
  if (before >= room) return;
  each_in_chunk(blockIdx.x, t.pages, [&](long p) { return w.uses[p] == 0; },
                [&](int p, bool is, int at) {
                  if (is && before + at < room) w.list[before + at] = p;
                });
}
// A wave for each row deals its pages out: those that come behind the needs of the rows before it, by their chunks' sums (2^18 rows of one
// page, ms: 0.43, with all rows added up by every row's wave 29; 4096 rows of 16 0.030, 0.048).
__global__ __launch_bounds__(64) void k_table_deal(KvTable t) {
  const int r = blockIdx.x, lane = threadIdx.x;
  if (t.rows == 0) {
    if (lane < 3) t.counts[lane] = 0;
    return;
  }
  const AssignWork w(t);
  const long free = sum_of(w.free), before = sum_before(w.needs, w.need, r), all = sum_of(w.needs);
  const long copies_before = sum_before(w.copies, w.copy, r);
  const bool enough = all <= free;
  const Span s = span_of(t, r);
  long place = before;
  for (int base = s.first; base < s.last; base += 64) {
    const int i = base + lane, at = r * t.width + i;
    const bool in = i < s.last;
    const int page = in ? t.out[at] : -1;
    const bool get = in && fresh(w, page, at), holds = in && i * t.page_tokens < s.held;
    const uint64_t who = __ballot(get);
    if (!enough) {
      if (in && !holds) t.out[at] = -1;
      continue;
    }
    if (get) {
      const int to = w.list[place + __popcll(who & ((1ull << lane) - 1))];
      t.out[at] = to;
      if (page >= 0 && holds) {
        t.copies[2 * copies_before] = page;
        t.copies[2 * copies_before + 1] = to;
      }
    }
    place += __popcll(who);
  }
  const long copies = enough ? sum_of(w.copies) : 0;
  if (lane == 0 && r >= copies) t.copies[2 * (long)r] = t.copies[2 * (long)r + 1] = -1;
  if (r == 0) {
    const long soft = sum_of(w.soft, chunks_of(t.pages));
    if (lane == 0) {
      t.counts[0] = (int)(enough ? t.pages - free + all : t.pages - soft);
      t.counts[1] = (int)(enough ? 0 : all - free);
      t.counts[2] = (int)copies;
    }
  }
}

// A small table by one workgroup: the same steps, what a page is to the entries in LDS, in one launch instead of five (one and five,
// us: 128 rows of 11 of 1384 pages 7.6, 15.6; 128 of 29 of 3148 10.4, 16.4; 64 of 122 of 4096 16.3, 16.0, compacted 7.2, 20.7).
constexpr int ONE_PAGES = 4096, ONE_ENTRIES = 8192;
// Sum over the 1024 threads of those before this one; `all`: over all of them.
__device__ inline int before_in_group(int n, int (&sums)[16], int &all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = n;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int x = __shfl_up(upto, o);
    if (lane >= o) upto += x;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int at = upto - n;
  all = 0;
  for (int i = 0; i < 16; ++i) {
    if (i < wave) at += sums[i];
    all += sums[i];
  }
  return at;
}
__global__ __launch_bounds__(1024) void k_table_assign_one(KvTable t) {
  constexpr int MOST = ONE_ENTRIES / 1024;  // entries of a thread, neighbours: pages are dealt out in their order
  // uses of a page and (upper half) writes to it; loose ones, later the free pages in order; the first that is written to
  __shared__ uint32_t uses[ONE_PAGES];
  __shared__ int loose[ONE_PAGES], lowest[ONE_PAGES], sums[16];
  const int tid = threadIdx.x, all = t.rows * t.width, each = (all + 1023) / 1024;
  for (int p = tid; p < t.pages; p += 1024) {
    uses[p] = 0;
    loose[p] = 0;
    lowest[p] = 0x7fffffff;
  }
  int page[MOST];
  bool write[MOST], holds[MOST];  // tokens to come go there; it holds some already
#pragma unroll
  for (int k = 0; k < MOST; ++k) {
    const int e = tid * each + k;
    page[k] = -1;
    write[k] = holds[k] = false;
    if (k >= each || e >= all) continue;
    const int r = e / t.width, i = e - r * t.width, src = t.source ? t.source[r] : r;
    const Span s = span_of(t, r);
    if (src >= 0 && src < t.rows && i * t.page_tokens < s.upto) page[k] = t.table[src * t.width + i];
    if (page[k] < 0 || page[k] >= t.pages) page[k] = -1;
    write[k] = written(s, i);
    holds[k] = i * t.page_tokens < s.held;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < MOST; ++k) {
    if (page[k] < 0) continue;
    atomicAdd(&uses[page[k]], write[k] ? 0x10001u : 1u);
    if (write[k]) {
      atomicMin(&lowest[page[k]], tid * each + k);
      if (!holds[k]) atomicAdd(&loose[page[k]], 1);
    }
  }
  __syncthreads();
  bool get[MOST];
  int n = 0, c = 0;
#pragma unroll
  for (int k = 0; k < MOST; ++k) {
    get[k] = write[k];
    if (write[k] && page[k] >= 0) {
      const uint32_t u = uses[page[k]], m = u & 0xffffu;
      get[k] = !(m == 1 || (m == u >> 16 && lowest[page[k]] == tid * each + k));
    }
    n += get[k];
    c += get[k] && page[k] >= 0 && holds[k];
  }
  int needed, copies, free, soft = 0;
  int next = before_in_group(n, sums, needed), copy = before_in_group(c, sums, copies);
  // free pages, four a thread
  bool is[ONE_PAGES / 1024];
  n = c = 0;
#pragma unroll
  for (int k = 0; k < ONE_PAGES / 1024; ++k) {
    const int p = tid * (ONE_PAGES / 1024) + k, u = p < t.pages ? (int)(uses[p] & 0xffffu) : -1;
    is[k] = u == 0;
    n += is[k];
    c += u >= 0 && u == loose[p];
  }
  int at = before_in_group(n, sums, free);
  (void)before_in_group(c, sums, soft);
#pragma unroll
  for (int k = 0; k < ONE_PAGES / 1024; ++k)
    if (is[k]) loose[at++] = tid * (ONE_PAGES / 1024) + k;
  __syncthreads();
  const bool enough = needed <= free;
  if (!enough) copies = 0;
#pragma unroll
  for (int k = 0; k < MOST; ++k) {
    const int e = tid * each + k;
    if (k >= each || e >= all) continue;
    int to = page[k];
    if (!enough) {
      if (!holds[k]) to = -1;
    } else if (get[k]) {
      to = loose[next++];
      if (page[k] >= 0 && holds[k]) {
        t.copies[2 * copy] = page[k];
        t.copies[2 * copy++ + 1] = to;
      }
    }
    t.out[e] = to;
  }
  for (int r = tid; r < t.rows; r += 1024)
    if (r >= copies) t.copies[2 * r] = t.copies[2 * r + 1] = -1;
  if (tid == 0) {
    t.counts[0] = enough ? t.pages - free + needed : t.pages - soft;
    t.counts[1] = enough ? 0 : needed - free;
    t.counts[2] = copies;
  }
}

// ------------------------------------------------------------------ pages in use moved to the lowest places
struct CompactWork {
  int32_t *uses, *rank;     // [pages]: 1 if named; place among the pages that move
  Counts used;              // [chunks]
  int32_t *source, *target; // [pages / 2]
  __host__ __device__ explicit CompactWork(const KvTable &t) {
    const int chunks = chunks_of(t.pages);
    uses = t.work;
    used.over = uses + t.pages;
    used.of = used.over + chunks_of(chunks);  // (all before it begins with 0)
    rank = used.of + chunks;
    source = rank + t.pages;
    used.n = chunks;
    used.most = PAGE_CHUNKS;
    target = source + t.pages / 2;
  }
};
__global__ __launch_bounds__(256) void k_table_mark(KvTable t) {
  const CompactWork w(t);
  const uint32_t at = blockIdx.x * 256u + threadIdx.x, all = (uint32_t)t.rows * (uint32_t)t.width;
  if (at >= all) return;
  const int page = t.table[at];
  if (page >= 0 && page < t.pages) w.uses[page] = 1;
}
__global__ __launch_bounds__(256) void k_table_used(KvTable t) {
  const CompactWork w(t);
  __shared__ int sum[4];
  int n = 0;
  for (int k = threadIdx.x; k < TABLE_CHUNK; k += 256) {
    const long p = (long)blockIdx.x * TABLE_CHUNK + k;
    if (p < t.pages) n += w.uses[p];
  }
  n = wave_sum_i(n);
  if ((threadIdx.x & 63) == 0) sum[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) w.used.set(blockIdx.x, sum[0] + sum[1] + sum[2] + sum[3]);
}
// The k-th page in use at or behind the number of all of them goes to the k-th free one before it.
__global__ __launch_bounds__(256) void k_table_rank(KvTable t) {
  const int c = blockIdx.x;
  const CompactWork w(t);
  const int used = sum_of(w.used), below = sum_before(w.used, w.uses, used), before = sum_before(w.used, c);
  each_in_chunk(c, t.pages, [&](long p) { return w.uses[p] != 0; },
                [&](int p, bool is, int at) {
                  at += before;  // pages in use before p
                  if (is && p >= used) {
                    w.rank[p] = at - below;
                    w.source[at - below] = p;
                  }
                  if (!is && p < used) w.target[p - at] = p;
                });
}
__global__ __launch_bounds__(256) void k_table_move(KvTable t) {
  const CompactWork w(t);
  const int used = sum_of(w.used), moved = used - sum_before(w.used, w.uses, used);
  const uint32_t at = blockIdx.x * 256u + threadIdx.x, all = (uint32_t)t.rows * (uint32_t)t.width;
  if (at < all) {
    const int page = t.table[at];
    t.out[at] = page < 0 || page >= t.pages ? -1 : page < used ? page : w.target[w.rank[page]];
  }
  if (at < (uint32_t)t.pages / 2) {
    const bool is = (int)at < moved;
    t.copies[2 * (long)at] = is ? w.source[at] : -1;
    t.copies[2 * (long)at + 1] = is ? w.target[at] : -1;
  }
  if (at == 0) {
    t.counts[0] = used;
    t.counts[1] = 0;
    t.counts[2] = moved;
  }
}

// As k_table_assign_one.
__global__ __launch_bounds__(1024) void k_table_compact_one(KvTable t) {
  __shared__ int used[ONE_PAGES], target[ONE_PAGES / 2], sums[16];
  const int tid = threadIdx.x, all = t.rows * t.width;
  for (int p = tid; p < t.pages; p += 1024) used[p] = 0;
  __syncthreads();
  for (int at = tid; at < all; at += 1024) {
    const int page = t.table[at];
    if (page >= 0 && page < t.pages) used[page] = 1;
  }
  __syncthreads();
  int n = 0, total, moved;
#pragma unroll
  for (int k = 0; k < 4; ++k) n += tid * 4 + k < t.pages && used[tid * 4 + k];
  int at = before_in_group(n, sums, total);  // pages in use before this thread's
  int far = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) far += tid * 4 + k >= total && tid * 4 + k < t.pages && used[tid * 4 + k];
  int rank = before_in_group(far, sums, moved);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int p = tid * 4 + k;
    if (p >= t.pages) continue;
    const bool is = used[p] != 0;
    if (!is && p < total) target[p - at] = p;
    if (is && p >= total) {
      t.copies[2 * rank] = p;
      used[p] = 1 + rank++;
    }
    at += is;
  }
  __syncthreads();
  for (int e = tid; e < all; e += 1024) {
    const int page = t.table[e];
    t.out[e] = page < 0 || page >= t.pages ? -1 : page < total ? page : target[used[page] - 1];
  }
  for (int i = tid; i < t.pages / 2; i += 1024) {
    if (i >= moved) t.copies[2 * i] = -1;
    t.copies[2 * i + 1] = i < moved ? target[i] : -1;
  }
  if (tid < 3) t.counts[tid] = tid == 0 ? total : tid == 1 ? 0 : moved;
}

// ------------------------------------------------------------------ copies of pages
// Workgroups take pieces of 16 KB in turn; a thread has four 16-byte loads on their way.  Bound by the bytes, which are streamed: 37
// pages of 1 MiB 13.1 us (5.9 TB/s), 446 of 256 KiB 40.5 us (5.8 TB/s).
constexpr int COPY_PIECE = 16384;
__global__ __launch_bounds__(256) void k_copy_pages(unsigned char *pool, long page_bytes, int pages, const int32_t *copies, int most, const int32_t *number) {
  typedef __attribute__((__vector_size__(16))) uint32_t piece_t;
  const int n = number ? min(*number, most) : most;
  const long pieces = (page_bytes + COPY_PIECE - 1) / COPY_PIECE;
  for (long id = blockIdx.x; id < n * pieces; id += gridDim.x) {
    const long which = id / pieces, at = (id - which * pieces) * COPY_PIECE;
    const int from = copies[2 * which], to = copies[2 * which + 1];
    if (from < 0 || from >= pages || to < 0 || to >= pages || from == to) continue;
    const piece_t *src = (const piece_t *)(pool + (long)from * page_bytes + at);
    piece_t *dst = (piece_t *)(pool + (long)to * page_bytes + at);
    const int left = (int)min((long)COPY_PIECE, page_bytes - at) / 16;
    piece_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((int)threadIdx.x + 256 * i < left) x[i] = __builtin_nontemporal_load(&src[threadIdx.x + 256 * i]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((int)threadIdx.x + 256 * i < left) __builtin_nontemporal_store(x[i], &dst[threadIdx.x + 256 * i]);
  }
}

bool by_one(const KvTable &t) { return t.pages <= ONE_PAGES && (long)t.rows * t.width <= ONE_ENTRIES; }
unsigned groups_for(long n) { return (unsigned)std::max(1L, (n + 255) / 256); }

}  // namespace

// words of work that begin with 0
static size_t assign_zeros(const KvTable &t) { return 3 * (size_t)t.pages + 2 * (size_t)chunks_of(chunks_of(t.rows)) + chunks_of(chunks_of(t.pages)); }
static size_t compact_zeros(const KvTable &t) { return (size_t)t.pages + chunks_of(chunks_of(t.pages)); }
bool kv_table_fits(const KvTable &t) {
  const long entries = (long)t.rows * t.width;
  return entries < 1L << 31 && launch_fits((long)t.rows + chunks_of(t.pages), 256);
}
size_t kv_assign_words(const KvTable &t) {
  return assign_zeros(t) + t.pages + 2 * (size_t)chunks_of(t.pages) + 2 * (size_t)chunks_of(t.rows) + 2 * (size_t)t.rows + (size_t)list_of(t);
}
size_t kv_compact_words(const KvTable &t) { return compact_zeros(t) + t.pages + chunks_of(t.pages) + 2 * (size_t)(t.pages / 2); }

void kv_assign(hipStream_t s, const KvTable &t) {
  const int chunks = chunks_of(t.pages), rows4 = (t.rows + 3) / 4;
  const long entries = (long)t.rows * t.width;
  if (by_one(t)) {
    SKD_LAUNCH(k_table_assign_one, dim3(1), dim3(1024), 0, s, t);
    return;
  }
  SKD_LAUNCH(k_table_fill, dim3(std::min(groups_for(4L * t.pages), 1024u)), dim3(256), 0, s, t.work, (long)assign_zeros(t), (long)t.pages);
  SKD_LAUNCH(k_table_gather, dim3(groups_for(entries)), dim3(256), 0, s, t);
  SKD_LAUNCH(k_table_count, dim3(rows4 + chunks), dim3(256), 0, s, t, rows4);
  SKD_LAUNCH(k_table_list, dim3(chunks + chunks_of(t.rows)), dim3(256), 0, s, t);
  SKD_LAUNCH(k_table_deal, dim3(std::max(t.rows, 1)), dim3(64), 0, s, t);
}
void kv_compact(hipStream_t s, const KvTable &t) {
  const int chunks = chunks_of(t.pages);
  const long entries = (long)t.rows * t.width;
  if (by_one(t)) {
    SKD_LAUNCH(k_table_compact_one, dim3(1), dim3(1024), 0, s, t);
    return;
  }
  SKD_LAUNCH(k_table_fill, dim3(std::min(groups_for(t.pages), 1024u)), dim3(256), 0, s, t.work, (long)compact_zeros(t), 0L);
  SKD_LAUNCH(k_table_mark, dim3(groups_for(entries)), dim3(256), 0, s, t);
  SKD_LAUNCH(k_table_used, dim3(chunks), dim3(256), 0, s, t);
  SKD_LAUNCH(k_table_rank, dim3(chunks), dim3(256), 0, s, t);
  SKD_LAUNCH(k_table_move, dim3(groups_for(std::max(entries, (long)t.pages / 2))), dim3(256), 0, s, t);
}
void kv_copy_pages(hipStream_t s, unsigned char *pool, long page_bytes, int pages, const int32_t *copies, int most, const int32_t *number) {
  const long pieces = (page_bytes + COPY_PIECE - 1) / COPY_PIECE;
  const unsigned groups = (unsigned)((__int128)most * pieces < 2048 ? most * pieces : 2048);  // (8 a CU)
  SKD_LAUNCH(k_copy_pages, dim3(groups), dim3(256), 0, s, pool, page_bytes, pages, copies, most, number);
}

}  // namespace skd
