// Launchers of the operators for learning cells by gradient: softmax cross entropy over the centroids
// (softmax_loss.hip), rows grouped by cell and back (group_rows.hip), gradient clipping (clip_grads.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

static inline int type_bytes(int dtype) { return dtype == VLQ_F32 ? 4 : 2; }

// ---- softmax_loss.hip ----
struct LossArgs {
    int dtype;
    const void *x, *c;
    int64_t n;
    int d, k;
    const float *bias; // or NULL
    float scale;
    const int32_t *label;
    float *loss;       // forward
    float *stats;      // [n x 2], written forward, read backward
    const float *grad; // backward: [n]
    void *dx, *dc;     // backward, each may be NULL
    float *dbias;
    void *ws;
};
size_t loss_workspace(int dtype, int64_t n, int d, int k, bool backward);
int launch_softmax_loss(const LossArgs &a, hipStream_t st);          // 0 or a hipError_t
int launch_softmax_loss_backward(const LossArgs &a, hipStream_t st); // 0 or a hipError_t
