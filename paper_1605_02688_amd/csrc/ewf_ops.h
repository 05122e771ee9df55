// The operators of sequence models: what the host side (ewf_ops.cpp) hands to the kernels (ewf_norm.hip,
// ewf_act8.hip, ewf_recurrence.hip).  Strides are in elements.
#pragma once

#include <cstddef>
#include <cstdint>

#include "ewf.h"

struct ihipStream_t;

namespace ewf {

// Where row r of a tensor begins: the rows are at most two axes, n1 the extent of the inner one.
struct RowStride { int64_t outer = 0, inner = 0; };

struct Rows {
    uint32_t rows = 0;
    uint32_t n1 = 1;                     // rows == n1: one axis, RowStride::inner alone counts
    int32_t cols = 0;
};

constexpr int kKeepBlock = 32;           // elements that share a scale

struct NormLaunch {
    Rows r;
    int dtype, param_dtype, code_dtype;
    float eps;
    const void *x, *weight, *bias, *dy;
    void *y, *dx, *dweight, *dbias;
    float *mean, *rstd;
    uint8_t *codes, *scales;
    RowStride sx, sy, smean, srstd, scodes, sscales, sdy, sdx;
    float *partials;                     // backward: [blocks][2][padded cols]
    int blocks;                          // backward: workgroups that leave a partial
    int padded;                          // backward: cols rounded up
};

struct ActLaunch {
    Rows r;
    int dtype, code_dtype;
    int act;
    const void *x, *dy;
    void *y, *dx;
    uint8_t *codes, *scales;
    RowStride sx, sy, scodes, sscales, sdy, sdx;
};

struct RecTensor { void *p = nullptr; int64_t batch = 0, step = 0; };

struct RecLaunch {
    int64_t batch, steps, channels;
    int dtype;
    RecTensor u, v, w, h, dh, du, dv, dw;
    RecTensor h0, last, dlast, dh0;      // float32, step unused
    const int32_t *lengths;
    int64_t lengths_stride;
    void *workspace;
};

// ---- kernels' launchers (device translation units).  They launch on `stream` and report nothing: the caller asks the runtime.
void launch_layer_norm(const NormLaunch &a, int units, ihipStream_t *stream);
// Chooses the backward pass's workgroups: fills blocks and padded.
void plan_layer_norm_grad(NormLaunch &a, int units);
void launch_layer_norm_grad(const NormLaunch &a, ihipStream_t *stream);
void launch_activation(const ActLaunch &a, ihipStream_t *stream);
void launch_activation_grad(const ActLaunch &a, ihipStream_t *stream);
void launch_read8(const ActLaunch &a, ihipStream_t *stream);
size_t recurrence_workspace(const RecLaunch &a, bool backward, int units);
void launch_recurrence(const RecLaunch &a, bool backward, int units, ihipStream_t *stream);

}  // namespace ewf
