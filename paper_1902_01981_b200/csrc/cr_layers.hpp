// Launch wrappers of the layer kernels: group norm and dropout (cr_layers.cu), 8-bit integer product (cr_int8.cu).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "cr_kernels.hpp"

namespace cr {

// Element types and activations; the values are those of cr_elem_t and cr_act_t.
enum { kElemF32 = 0, kElemBF16 = 1, kElemF16 = 2 };
enum { kActNone = 0, kActRelu = 1, kActSilu = 2 };
inline int elem_bytes(int elem) { return elem == kElemF32 ? 4 : 2; }

// Dropout: `threshold` of 65536 values of a 16-bit number are dropped, the others scaled by `scale`; `key` is the
// finished seed, `offset` the index of the first element.
struct DropSpec {
    unsigned long long key = 0;
    unsigned long long offset = 0;
    uint32_t threshold = 0;   // 0: nothing is dropped
    float scale = 1.f;
};
DropSpec make_drop(double p, uint64_t seed, int64_t offset);

struct GroupNormArgs {
    const void *x = nullptr;       // [samples][positions][ld_x], channels innermost
    const void *dy = nullptr;      // backward
    void *y = nullptr;             // forward: y, backward: dx (may be null)
    const float *gamma = nullptr;  // [channels] or null: ones
    const float *beta = nullptr;   // [channels] or null: zeros
    float *mean = nullptr;         // [samples][groups]: written by the forward pass, read by the backward pass
    float *rstd = nullptr;
    float *dgamma = nullptr;       // backward: [partitions][ld_param], may be null
    float *dbeta = nullptr;
    int64_t samples = 0, positions = 0;
    int64_t ld_x = 0, ld_dy = 0, ld_y = 0, ld_param = 0;
    int64_t partitions = 1;
    int channels = 0, groups = 0;
    int elem = 0, act = 0;
    float eps = 0.f;
    DropSpec drop;
    float *workspace = nullptr;
    int *status = nullptr;            // the plan's status word and the bound of every device-side wait
    unsigned long long wait_ns = 0;
    int device = 0;
};

// Whether all rows of the tensors are whole 16-byte vectors (dy, y may be null).
bool group_norm_vector_rows(const GroupNormArgs &a);
// Workspace in bytes, from the sizes and from whether the rows are such vectors.
size_t group_norm_workspace_bytes(int64_t samples, int64_t positions, int channels, int groups, int elem, bool vectors);
size_t group_norm_backward_workspace_bytes(int64_t samples, int64_t positions, int channels, int groups, int elem, bool vectors);
cudaError_t launch_group_norm(const GroupNormArgs &a, const DeviceInfo &dev, cudaStream_t stream, int64_t *launches);
cudaError_t launch_group_norm_backward(const GroupNormArgs &a, const DeviceInfo &dev, cudaStream_t stream, int64_t *launches);

// The one-pass forms (cr_group_norm.cu), for vector rows: whether an item fits a cluster, for the backward pass with the
// rows of sums it leaves for a sample (0: no).  The backward one leaves the sums of dz (sum1) and dz xhat (sum2) of each
// sample's channels in that many rows of ld_sum, or in one (`whole`, which takes an item that one CTA holds: two rows).
bool group_norm_on_chip(int64_t samples, int64_t positions, int channels, int groups, int elem);
int group_norm_backward_on_chip(int64_t samples, int64_t positions, int channels, int groups, int elem);
cudaError_t launch_group_norm_on_chip(const GroupNormArgs &a, cudaStream_t stream, int64_t *launches);
cudaError_t launch_group_norm_grad_on_chip(const GroupNormArgs &a, float *sum1, float *sum2, int64_t ld_sum, bool whole, cudaStream_t stream,
                                           int64_t *launches);

// y = residual + dropout(x) over [rows][cols] with row strides; residual may be null.
cudaError_t launch_dropout(const void *x, const void *residual, void *y, int64_t rows, int64_t cols, int64_t ld_x,
                           int64_t ld_r, int64_t ld_y, int elem, const DropSpec &drop, const DeviceInfo &dev,
                           cudaStream_t stream, int64_t *launches);

// q[r][:] = rint(x[r][:] * 127 / max|x[r][:]|), scale[r] = max|x[r][:]| / 127.
cudaError_t launch_quantize_rows(const void *x, int64_t rows, int64_t cols, int64_t ld_x, int elem, int8_t *q, int64_t ld_q,
                                 float *scale, const DeviceInfo &dev, cudaStream_t stream, int64_t *launches);

struct Int8ProductArgs {
    const int8_t *x = nullptr;       // [tokens][ld_x]
    const int8_t *w = nullptr;       // [outer][ld_w]
    const float *x_scale = nullptr;  // [tokens]
    const float *w_scale = nullptr;  // [outer]
    const float *bias = nullptr;     // [outer] or null
    void *y = nullptr;               // [tokens][ld_y]
    int64_t tokens = 0, outer = 0, inner = 0;
    int64_t ld_x = 0, ld_w = 0, ld_y = 0;
    int elem = 0;
    int device = 0;
};
cudaError_t launch_int8_product(const Int8ProductArgs &a, int *status, const DeviceInfo &dev, const Tuning &tune,
                                EncodeTiledFn encode, cudaStream_t stream, int64_t *launches);

}  // namespace cr
