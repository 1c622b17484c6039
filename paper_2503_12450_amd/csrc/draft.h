// Launchers of what decides about drafted tokens: probabilities of logits, and
// which of a tree's tokens they accept.
#pragma once

#include "common.h"

namespace marcache {

constexpr int kMaxVocab = 1 << 20;

struct VerifyArgs {
  const void* p;      // [m, vocab]: probabilities; greedy: anything of the same order
  const void* draft;  // [m, vocab], nullable: probabilities that a row's children were drawn from
  const int32_t* q_start;
  const int32_t* parent;
  const int32_t* tokens;
  const float* random;  // null: greedy
  int32_t* path;
  int32_t* kept;
  int32_t* next;
  void* ws;
  long ld_p, ld_draft;
  int m, n_seqs, vocab;
};

hipError_t launch_probabilities(int dtype, const void* logits, long ld, const float* temperature, int m, int vocab,
                                float* out, long ld_out, hipStream_t st);
hipError_t launch_verify(int dtype, const VerifyArgs& a, hipStream_t st);
size_t verify_workspace(int m, int n_seqs, int vocab);

}  // namespace marcache
