// Launcher interface of the rules on logits (logits.cu), called by the C ABI
// (api_decode.cu) after validation.
#pragma once

#include "decode.cuh"

namespace starq {

struct LogitsArgs {
    const void* X; int ldx; int dtype; int T; int V;
    const int32_t* seq_start; int B; int max_new;
    starq_logits_rules r;            // zeros: no rules
    void* Y; int ldy;                // the logits under the rules (kind -1),
    int kind;                        // or a starq_confidence and
    int32_t* token; float* confidence; float* lse;
    unsigned* status;
};
cudaError_t launch_logits(const LogitsArgs& a, cudaStream_t s);

}  // namespace starq
