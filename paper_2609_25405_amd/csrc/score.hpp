// Scores of tokens: kernel arguments and the launcher.
#pragma once

#include "common.hpp"
#include "orthrus/score.h"

namespace orthrus {

struct Score {
    const float *logits;
    int64_t stride;
    int rows, vocab, n_top;
    const int32_t *tokens;
    float *logprob, *entropy;
    int32_t *rank, *top_ids;
    float *top_logprobs;
    char *ws;
};
// most slices of a row, each a workgroup; 1: no workspace and no merge launch
int score_slices(int vocab);
size_t score_bytes(int rows, int vocab, int n_top);
hipError_t launch_score(const Score &a, hipStream_t s);

}  // namespace orthrus
