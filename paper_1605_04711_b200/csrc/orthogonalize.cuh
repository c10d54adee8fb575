// What the two paths of the orthogonalised updates share: the coefficients of a step and the small path's interface.
#pragma once

#include <stdint.h>

#include "common.cuh"

namespace twn_detail {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr int kNsMaxItems = 32;

struct NsSource {
    const void *G;               // the update; NULL for Muon, whose update is
    const float *dW;             //   V, or dW + momentum V (look ahead), with
    float *V;                    //   V = momentum V + dW
    void *O;
    int m, n;                    // shorter and longer side
    float out_scale;
    uint8_t g_bf16, o_bf16, tall, vec_in, vec_out;
};

// Matrices of at most kNsSmallM x kNsSmallN in at most kNsSmallSteps steps: one launch, a cluster of blocks for each.
constexpr int kNsSmallM = 128, kNsSmallN = 8192, kNsSmallSteps = 5;
constexpr size_t kNsSmallScratch = 64 * 1024;
struct NsSmallItem {
    NsSource src;
    uint16_t *scratch;           // kNsSmallScratch bytes, 16-byte aligned
};
struct NsSmallParams {
    NsSmallItem item[kNsMaxItems];
    int count, steps, look_ahead;
    float momentum, eps;
    int32_t *status;
};
int ns_small(const NsSmallParams &P, cudaStream_t s);

}  // namespace twn_detail
