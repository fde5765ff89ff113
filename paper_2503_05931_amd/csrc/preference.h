// What the preference loss's kernels (preference.hip) and their host side (aed_train.hip) share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace aed {

struct PreferenceArgs {
    const void* logits;
    int64_t row_stride;  // elements
    const int32_t* labels;
    const float* ref;
    float *loss, *ratio;
    float2* lse;              // [rows]: maximum, log of the sum of exponentials relative to it
    float* gain;              // [rows]: log-probability of the label less the reference's
    int32_t* arrived;         // workgroups, 0 between calls
    const int32_t* seq_of;    // [rows]
    const int32_t* seq_start;  // [2 pairs + 1]
    const float* d_loss;
    void* d_logits;
    int64_t d_row_stride;
    int rows, pairs, vocab;
    float beta, smoothing;
};

hipError_t launch_preference_forward(const PreferenceArgs& a, bool bf16, hipStream_t s);
hipError_t launch_preference_backward(const PreferenceArgs& a, bool bf16, hipStream_t s);

}  // namespace aed
