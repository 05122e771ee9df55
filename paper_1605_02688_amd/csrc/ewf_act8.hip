// Activations whose argument is kept in 8 bits for the backward pass: element-wise, one pass each way.
#include "ewf_ops_device.h"

namespace ewf {

namespace {

constexpr float kLog2E = 1.44269504f;

// 1 / (1 + 2^(-x log2 e)) with native exp2 and reciprocal: relative error 2^-24 (2 + |x|) or so
EWF_OPS_DEV float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-x * kLog2E)); }

template <int ACT>
EWF_OPS_DEV float act_value(float x)
{
    if constexpr (ACT == EWF_RELU) return x > 0.f ? x : x != x ? x : 0.f;
    else if constexpr (ACT == EWF_ACT_TANH) return tanhf(x);
    else if constexpr (ACT == EWF_ACT_SIGMOID) return sigmoid(x);
    else if constexpr (ACT == EWF_SILU) return x * sigmoid(x);
    else if constexpr (ACT == EWF_GELU) return x * (0.5f + 0.5f * erff(x * 0.70710678f));
    else return x;
}

// d act / dx.  A NaN argument (a block without a finite scale) gives NaN for every activation.
template <int ACT>
EWF_OPS_DEV float act_slope(float x)
{
    if constexpr (ACT == EWF_RELU) return x > 0.f ? 1.f : x != x ? x : 0.f;
    else if constexpr (ACT == EWF_ACT_TANH) { const float t = tanhf(x); return fmaf(-t, t, 1.f); }
    else if constexpr (ACT == EWF_ACT_SIGMOID) { const float p = sigmoid(x); return p * sigmoid(-x); }
    else if constexpr (ACT == EWF_SILU) { const float p = sigmoid(x); return fmaf(x * p, sigmoid(-x), p); }
    else if constexpr (ACT == EWF_GELU) {
        const float density = 0.39894228f * __builtin_amdgcn_exp2f(x * x * (-0.5f * kLog2E));
        return fmaf(x, density, 0.5f + 0.5f * erff(x * 0.70710678f));
    } else return x == x ? 1.f : x;
}

// A lane takes a vector of V elements; 32 / V lanes share a scale, so a row takes a whole number of such groups.
// item / per_row is a product with mul = ceil(2^(31 + s) / per_row), 2^s >= per_row > 2^(s-1): mul is less than 2^s / per_row
// too large, which for item < 2^31 does not reach the next whole number.
struct Items {
    uint32_t row0, count, per_row, mul, shift;
};
struct Place { uint32_t row; int c; };

EWF_OPS_DEV Place place(uint32_t item, const Items &i, int V)
{
    const uint32_t row = (uint32_t)((uint64_t)item * i.mul >> i.shift);
    return {i.row0 + row, (int)(item - row * i.per_row) * V};
}

template <typename T, int ACT>
__global__ void __launch_bounds__(256) k_act(ActLaunch a, Items items)
{
    constexpr int V = Vec16<T>::V;
    typedef typename T::raw raw;
    const uint32_t item = blockIdx.x * 256 + threadIdx.x;
    const bool live = item < items.count;                    // (all lanes of a scale's group or none)
    const Place at = live ? place(item, items, V) : Place{0, 0};
    const int cols = live ? a.r.cols : 0, c = at.c;
    u32x4 x = {0u, 0u, 0u, 0u};
    if (c < cols) x = load_part<T>((const raw *)a.x + row_offset(a.r, at.row, a.sx), c, cols, a.nt);
    float f[V];
#pragma unroll
    for (int e = 0; e < V; e++) f[e] = element<T>(x, e);
    if (a.codes)
        keep_part<V>(a.codes + row_offset(a.r, at.row, a.scodes), a.scales + row_offset(a.r, at.row, a.sscales), c, cols, f,
                     a.code_dtype == EWF_E4M3);
    if (a.y && c < cols) {
#pragma unroll
        for (int e = 0; e < V; e++) f[e] = act_value<ACT>(f[e]);
        store_part<T>((raw *)a.y + row_offset(a.r, at.row, a.sy), c, cols, pack16<T>(f), a.nt);
    }
}

// dx = dy act'(x8); without dy: x8 itself.
template <typename T, int ACT>
__global__ void __launch_bounds__(256) k_act_grad(ActLaunch a, Items items)
{
    constexpr int V = Vec16<T>::V;
    typedef typename T::raw raw;
    const uint32_t item = blockIdx.x * 256 + threadIdx.x;
    if (item >= items.count) return;
    const Place at = place(item, items, V);
    const int cols = a.r.cols, c = at.c;
    if (c >= cols) return;
    u32x4 dy = {0u, 0u, 0u, 0u};
    if (a.dy) dy = load_part<T>((const raw *)a.dy + row_offset(a.r, at.row, a.sdy), c, cols, a.nt);
    const u32x2 code = load_codes<V>(a.codes + row_offset(a.r, at.row, a.scodes), c, cols);
    const uint32_t byte = a.scales[row_offset(a.r, at.row, a.sscales) + c / kKeepBlock];
    float f[V];
    decode_part<V>(code, byte, a.code_dtype == EWF_E4M3, f);
    if (a.dy) {
#pragma unroll
        for (int e = 0; e < V; e++) f[e] = element<T>(dy, e) * act_slope<ACT>(f[e]);
    }
    store_part<T>((raw *)a.dx + row_offset(a.r, at.row, a.sdx), c, cols, pack16<T>(f), a.nt);
}

template <typename T, int ACT, bool GRAD>
void run(const ActLaunch &a, hipStream_t stream)
{
    constexpr int V = Vec16<T>::V;
    Items i{};
    i.per_row = (uint32_t)(((int64_t)a.r.cols + kKeepBlock - 1) / kKeepBlock) * (kKeepBlock / V);
    uint32_t s = 0;
    while (((uint64_t)1 << s) < i.per_row) s++;
    i.shift = 31 + s;
    i.mul = (uint32_t)((((uint64_t)1 << i.shift) + i.per_row - 1) / i.per_row);
    // launches of fewer than 2^31 items each
    const uint32_t most = 0x7fffff00u / i.per_row;
    for (uint32_t row = 0; row < a.r.rows; row += i.count / i.per_row) {
        i.row0 = row;
        i.count = (a.r.rows - row < most ? a.r.rows - row : most) * i.per_row;
        const dim3 grid((i.count + 255) / 256);
        if constexpr (GRAD) hipLaunchKernelGGL((k_act_grad<T, ACT>), grid, dim3(256), 0, stream, a, i);
        else hipLaunchKernelGGL((k_act<T, ACT>), grid, dim3(256), 0, stream, a, i);
    }
}

template <typename T, bool GRAD>
void run_act(const ActLaunch &a, hipStream_t stream)
{
    switch (a.act) {
    case EWF_RELU: return run<T, EWF_RELU, GRAD>(a, stream);
    case EWF_ACT_TANH: return run<T, EWF_ACT_TANH, GRAD>(a, stream);
    case EWF_ACT_SIGMOID: return run<T, EWF_ACT_SIGMOID, GRAD>(a, stream);
    case EWF_SILU: return run<T, EWF_SILU, GRAD>(a, stream);
    case EWF_GELU: return run<T, EWF_GELU, GRAD>(a, stream);
    default: return run<T, EWF_IDENTITY, GRAD>(a, stream);
    }
}

template <bool GRAD>
void run_type(const ActLaunch &a, hipStream_t stream)
{
    if (a.dtype == EWF_F32) run_act<F32, GRAD>(a, stream);
    else if (a.dtype == EWF_F16) run_act<F16, GRAD>(a, stream);
    else run_act<BF16, GRAD>(a, stream);
}

}  // namespace

void launch_activation(const ActLaunch &a, hipStream_t stream) { run_type<false>(a, stream); }
void launch_activation_grad(const ActLaunch &a, hipStream_t stream) { run_type<true>(a, stream); }
void launch_read8(const ActLaunch &a, hipStream_t stream) { run_type<true>(a, stream); }

}  // namespace ewf
