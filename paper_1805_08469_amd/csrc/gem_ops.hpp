// gem_ops.hpp -- pieces shared by the host side and the kernels of the worker's
// operators (scores of logits, distillation, the gated recurrence).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/gem.h"

namespace gemk {

// Keeps the detail of a failed HIP call for gem_last_error (gem_api.cpp).
void note_hip_error(const char* file, const char* what, hipError_t e, int line);

// Scratch that every handle has, ahead of what gem_scan_scratch asks for.
constexpr int64_t kFixedScratch = int64_t{8} << 20;

// Tokens between two kept states of a recurrence.
constexpr int kStateTokens = 8;

// Rows of logits, and what a launch over them needs.
struct LogitArgs {
    const void* z;
    int64_t stride;        // elements between rows
    int64_t rows;
    int32_t vocab;
    float scale;           // log2(e) / temperature
    float inv_t;           // 1 / temperature
};

struct ScoreArgs {
    LogitArgs l;
    const int32_t* tokens; // [rows][n_tokens]
    int32_t n_tokens;
    int32_t top_k;
    gem_scores out;
};

struct DistillArgs {
    LogitArgs l;
    const int32_t* ids;    // [rows][k]
    const float* lp;       // [rows][k]
    int32_t k;
    int32_t tail;
    const float* weight;   // [rows] or null
    float* loss;           // [rows] or null
    void* grad;            // rows x vocab, or null: the loss alone
    int64_t grad_stride;
};

struct ScanArgs {
    gem_scan s;            // strides filled in
    void* y;
    int64_t y_stride;
    float* h_last;
    float* states;
};

struct ScanBackArgs {
    gem_scan s;
    const float* states;
    const void* dy;
    int64_t dy_stride;
    const float* dh_last;
    void* dx;
    int64_t dx_stride;
    void* dgate;
    int64_t dgate_stride;
    float* dh0;
};

// What a handle gives a launch.
struct OpsDevice {
    int32_t cus;             // compute units
    void* scratch;           // kFixedScratch bytes
    void* scan;              // scan_bytes bytes
    int64_t scan_bytes;
};

hipError_t launch_scores(const ScoreArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream);
hipError_t launch_distill(const DistillArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream);
int64_t scan_rows(int64_t tokens, int64_t channels);
int64_t scan_bytes(int64_t tokens, int64_t channels);            // of a launch
int64_t scan_scratch_bytes(int64_t tokens, int64_t channels);    // of it and of any smaller one
hipError_t launch_scan_forward(const ScanArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream);
hipError_t launch_scan_backward(const ScanBackArgs& a, bool bf16, const OpsDevice& d, hipStream_t stream);

}  // namespace gemk
