// Draws with parameters per row (sample_rows.hip).  Used by skd_sample and by the engine's sampling head.
#pragma once
#include "skd_kernels.h"

namespace skd {

constexpr int SAMPLE_ROWS_VOCAB = 1 << 18;  // masses are counted in units of 2^-45 of the largest, their sum in 63 bits
constexpr int SAMPLE_BINS = 512;

struct SampleBins {           // of a piece of a row; [rows][pieces]
  uint64_t mass[SAMPLE_BINS + 1];
  uint32_t count[SAMPLE_BINS + 1];
  float top;                  // largest logit of the piece
  uint64_t all;               // mass of the piece
};

struct SampleRows {
  const float *logits;
  long stride;
  int rows, vocab;
  // [rows]; null: 1, off, off, off
  const float *temperature;
  const int32_t *top_k;
  const float *top_p, *min_p;
  const float *u;             // [rows]
  int32_t *tokens, *tokens2;  // tokens2: second destination, or null
  SampleBins *bins;           // sample_rows_bins(rows, vocab) of them
  int piece, pieces;          // set by sample_rows: tokens of a piece
};
size_t sample_rows_bins(int rows, int vocab);
bool sample_rows_fit(int rows, int vocab);  // in a launch each
void sample_rows(hipStream_t s, const SampleRows &a);

}  // namespace skd
