// Block tables of the paged cache on the device (kv_table.hip): the next table of a batch, pages in use moved together, pages copied.
#pragma once
#include "kv_ops.h"

namespace skd {

constexpr int TABLE_CHUNK = 1024;  // pages whose free ones a workgroup counts

struct KvTable {
  const int32_t *table;   // [rows][width]
  int rows, width, page_tokens, pages;
  const int32_t *source, *len, *more;  // [rows]; source null: every row itself
  int32_t *out;           // [rows][width]; may be `table` where every row is itself
  int32_t *copies;        // [rows][2], of compaction [pages / 2][2]: from, to; -1, -1 behind the last
  int32_t *counts;        // [3]: pages in use, pages missing, copies
  int32_t *work;
};
bool kv_table_fits(const KvTable &t);         // in a launch each, and entries in 32 bits
size_t kv_assign_words(const KvTable &t);     // of work
size_t kv_compact_words(const KvTable &t);
void kv_assign(hipStream_t s, const KvTable &t);
void kv_compact(hipStream_t s, const KvTable &t);
void kv_copy_pages(hipStream_t s, unsigned char *pool, long page_bytes, int pages, const int32_t *copies, int most, const int32_t *number);

}  // namespace skd
