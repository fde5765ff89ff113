// What the kernels on rows of logits (sample.hip, top_logits.hip, distill.hip) and their host side (aed_vocab.hip) share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace aed {

constexpr int kMostTop = 128;           // entries of a row's list
constexpr int kMostVocab = 1 << 18;     // sums of as many weights stay in 64 bits (sample.hip); a bit for each takes 32 KB of LDS (distill.hip)
constexpr float kLeftOut = 0x1.fffffep127f;
constexpr int kMostRows = (1 << 22) - 1;  // a launch has less than 2^32 threads, a row at most 1024

// Rows of logits
struct LogitRows {
    const void* data;
    int64_t stride;  // elements
    int rows, vocab;
};

struct SampleArgs {
    LogitRows z;
    const float* uniforms;
    float temperature, top_p, min_p;  // of all rows; by row where the pointers are not null
    int top_k;
    const float *temperatures, *top_ps, *min_ps;
    const int32_t* top_ks;
    int32_t* tokens;
    float* logp;
    int weight_bits;  // weights are whole multiples of 2^-weight_bits
};

struct TopArgs {
    LogitRows z;
    float *values, *rest;
    int32_t* ids;
    int top;
    float scale;  // 1 / temperature, times log2 e
    float temperature;
};

struct DistillArgs {
    LogitRows z;
    const float *values, *rest, *weights;
    const int32_t* ids;
    float *loss, *row_loss;
    float* stats;  // [rows][top + 2]: what p outside of the list is made of (distill.hip), then by entry the gradient by its id (kLeftOut: left out)
    const float* d_loss;
    void* d_logits;
    int64_t d_stride;
    int top;
    float temperature, scale, scale_low;  // scale_d's float below, and what it lacks, above 0
    double scale_d, factor;               // log2 e / temperature; temperature^2 ln 2
};

hipError_t launch_sample(const SampleArgs& a, bool bf16, hipStream_t s);
hipError_t launch_top(const TopArgs& a, bool bf16, hipStream_t s);
hipError_t launch_distill_forward(const DistillArgs& a, bool bf16, hipStream_t s);
hipError_t launch_distill_backward(const DistillArgs& a, bool bf16, hipStream_t s);

}  // namespace aed
