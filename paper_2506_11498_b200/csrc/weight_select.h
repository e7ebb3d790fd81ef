// The selection by accumulated weight, for the entry point and the cache that keeps rows by it.
#pragma once

#include "lrsa_internal.h"

namespace lrsa {

constexpr int kSelectSeqs = 16;   // sequences of a launch
struct WeightSelectArgs {
  const float* weight;   // [B*Hkv][row]
  const float* ring;     // when not null, positions below ring_below are here: [B*Hkv][ring_len], position p at (p - ring_first) % ring_len
  int ring_below, ring_first, ring_len;
  int32_t* idx;          // [B*Hkv][Wtot][K]
  int* status;           // cleared when not null
  long long row;
  int L, K, Wtot, n;     // n sequences, with item0[n] windows over all (batch, KV head) pairs
  int item0[kSelectSeqs + 1];
  int windows[kSelectSeqs], first[kSelectSeqs];    // per pair; token of window 0 in the row
  int woff[kSelectSeqs], emit0[kSelectSeqs];       // first window in idx; position of window 0
};
int launch_weight_select(const WeightSelectArgs& a, cudaStream_t st);

}  // namespace lrsa
