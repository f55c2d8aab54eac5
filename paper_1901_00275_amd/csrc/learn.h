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

// ---- group_rows.hip ---- (each returns 0 or a hipError_t)
size_t group_workspace(int64_t pairs, int cells);
int launch_group_rows(const int32_t *cell, int64_t pairs, int cells, int64_t *off, int32_t *place, int32_t *source, void *ws,
                      hipStream_t st);
int launch_gather_rows(int dtype, const void *x, int64_t n, int w, int d, const int32_t *source, void *y, hipStream_t st);
int launch_combine_rows(int dtype, const void *y, int64_t n, int w, int d, const int32_t *place, const float *weight, void *out,
                        hipStream_t st);
int launch_combine_rows_backward(int dtype, const void *dout, const void *y, int64_t n, int w, int d, const int32_t *place,
                                 const float *weight, void *dy, float *dweight, hipStream_t st);

// ---- clip_grads.hip ----
size_t clip_workspace(int tensors, const int64_t *counts);
int launch_clip_grads(int tensors, const int *dtypes, const int64_t *counts, const void *const *in, float max_norm,
                      void *const *out, float *norm, void *ws, hipStream_t st);
