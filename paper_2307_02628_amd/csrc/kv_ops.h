// Launch interface of the paged cache as an operator (kv_ops.hip): tokens of any rows filed into pages of bf16, 8 or 4
// bits, read back and attended to.  Used by the C entry points skd_kv_* and by the engine.
#pragma once
#include "skd_kernels.h"

namespace skd {

int hip_failed(hipError_t e);  // notes the error for skd_last_hip_error; what an entry point returns

struct KvView {
  KvGeom g;                 // H: kv heads; page_elems unused
  bool fp8, fp4;            // neither: bf16
  int pages, rows;
  long page_bytes;
  unsigned char *pool;
  const int32_t *table;     // [rows][g.max_pages]
};

// Which tokens a call is about: the i-th new token of row r is token at(r) + i * step, at position past(r) + i.
struct KvTokens {
  enum Kind {
    RAGGED,                 // at = first[r], new = first[r + 1] - first[r], past = past[r]
    COLUMNS,                // at = r, new = count (0 while the column is padding), past = t - past[r]; step = rows
    PROMPT                  // at = first[r], new = count - past[r], past = 0
  } kind;
  const int32_t *first, *past;
  int tokens, count, t, step;
  int max_new, max_past;    // what the grid is made for
  int room;                 // positions that a row's pages hold, below 2^30
};

// Values of one kind of a call's tokens: [token][heads][dh] with `stride` elements from token to token, or (tiles) columns
// `at` .. of activation tiles of `stride` columns.
struct KvRows {
  void *p;
  long stride;
  int at;
  bool tiles;
};

// Blocks of 32 positions that filing and reading back look at (a call's must be below 2^31): of every row and kv head as many as a
// row's new tokens may lie in.
long kv_blocks(const KvView &kv, const KvTokens &tk);
// k, v (bf16) of the tokens into their pages
void kv_append(hipStream_t s, const KvView &kv, const KvTokens &tk, const KvRows &k, const KvRows &v);
// the pages' values of the tokens, fp32 or bf16 rows
void kv_read(hipStream_t s, const KvView &kv, const KvTokens &tk, bool bf16, const KvRows &k, const KvRows &v);

// What becomes of a score s = scale * q . k, in units of log 2, and which positions a token sees.
struct KvScoring {
  bool capped;
  float in, out;            // capped: q . k becomes -out / (1 + 2^(in q . k))
  const float *slopes;      // [heads] or null
  int window;               // 0: none
  const int32_t *begin, *end;  // [tokens] or null
};

struct KvAttend {
  KvView kv;
  KvTokens tk;
  int heads, group;         // query heads, of them to a kv head
  float c;                  // scores -> log2 of the weights
  bool scored;              // sc is what it goes by
  KvScoring sc;
  KvRows q, o, k, v;        // bf16; k.p null: the cache holds the new tokens, else they are filed first
  const int32_t *order;     // rows in the order of their dispatch, or null (scored: null)
  int splits;               // of the keys of a query tile
  float *part;              // splits > 1: [splits][tokens * heads][dh + 2]: numerators, maximum, denominator
};
// window: of changed scores, 0 where they have none; -1: scores as they are
bool kv_attend_fits(const KvView &kv, const KvTokens &tk, int heads, int window = -1);  // in a launch; rows x kv heads must be below 2^31 before
int kv_attend_splits(const KvView &kv, const KvTokens &tk, int heads, int window = -1);
size_t kv_attend_part(const KvView &kv, const KvTokens &tk, int heads, int splits);  // floats
void kv_attend(hipStream_t s, const KvAttend &a);

}  // namespace skd
