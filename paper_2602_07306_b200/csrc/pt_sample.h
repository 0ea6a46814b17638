// Sampling from logits (pt_sample.cu), shared with the generate loop.
#pragma once
#include "pt_internal.h"

namespace pt {

struct SampleP {
    const void* logits;                   // [n][row_stride] fp32 or bf16
    int64_t row_stride;
    int vocab;
    const float* u;                       // [n]
    const float* temperature;             // [n]; null: 1
    const int32_t* top_k;                 // [n]; null: off
    const float* top_p;                   // [n]; null: off
    const float* min_p;                   // [n]; null: off
    int32_t* token;                       // [n], may be null
    int32_t* token2; int64_t token2_stride;   // a second place for the token, may be null
    float* prob; int64_t prob_stride;     // may be null
};

int sample_vocab_limit();
pt_status launch_sample(const SampleP& p, int64_t n, bool bf16, cudaStream_t st);

}  // namespace pt
