// Activations whose argument is kept in 8 bits for the backward pass: element-wise, one pass each way.
//
// A lane takes one 16-byte vector and a workgroup of 256 a contiguous piece; two or four vectors a lane are slower (bfloat16 [8192,
// 8192], both passes, 117, 122 and 128 us), as for a plain copy.  Memory bounds them: forward 6.4 TB/s, backward, which
// reads three streams for two written, 5.2.
#include "ewf_ops_device.h"

namespace ewf {

namespace {

// The normal distribution function, to its own precision on both sides of zero (1 + erf loses what lies below -3 in 16 bits already), and
// e = exp(-x^2 / 2).  Below zero, with a = -x: e t P(t), t = 1 / (1 + 0.35 a), P the polynomial of degree 8 whose largest relative
// error up to a = 13.5, where float32 ends, is least (3.2e-8; fitted to erfc in 64 bits).  The square's rounding costs x^2 / 2 units: at
// -9, 4e-6.  Both passes of gelu, bfloat16 [8192, 8192], take 134 us, with the device library's erf 153, with its erfc 198.
struct Normal { float below, e; };
EWF_OPS_DEV Normal normal(float x)
{
    const float a = fminf(fabsf(x), 16.f);              // (both are 0 there; a NaN goes on in x)
    const float e = __builtin_amdgcn_exp2f(a * a * (-0.5f * kLog2E)), t = recip<F32>(fmaf(0.35f, a, 1.f));
    float p = -0.0291258656f;
    p = fmaf(p, t, 0.143872231f);
    p = fmaf(p, t, -0.255504578f);
    p = fmaf(p, t, 0.158929303f);
    p = fmaf(p, t, -0.0229371525f);
    p = fmaf(p, t, 0.105432943f);
    p = fmaf(p, t, 0.119852431f);
    p = fmaf(p, t, 0.139859080f);
    p = fmaf(p, t, 0.139621571f);
    const float tail = e * (t * p);
    return {x < 0.f ? tail : 1.f - tail, e};
}

template <typename T, int ACT>
EWF_OPS_DEV float act_value(float x)
{
    if constexpr (ACT == EWF_RELU) return x > 0.f ? x : x != x ? x : 0.f;
    else if constexpr (ACT == EWF_ACT_TANH) return tanhf(x);
    else if constexpr (ACT == EWF_ACT_SIGMOID) return sigmoid<T>(x);
    else if constexpr (ACT == EWF_SILU) return x * sigmoid<T>(x);
    else if constexpr (ACT == EWF_GELU) return x * normal(x).below;
    else return x;
}

// d act / dx.  A NaN argument (a block without a finite scale) gives NaN for every activation.  That of tanh is 4 f (1 - f), f the
// sigmoid of 2 x, small numbers that 1 - tanh^2 would lose.  The slopes of silu and gelu are 0
// and 1 in float32 long before +-128 (their distance is less than 2^-118 there): farther arguments, up to the infinities that
// the largest floats' codes stand for in 32 bits, are taken as those, because x times a gate that is only nearly shut is not small for them.
template <typename T, int ACT>
EWF_OPS_DEV float act_slope(float x)
{
    if constexpr (ACT == EWF_SILU || ACT == EWF_GELU) x = x < -128.f ? -128.f : x > 128.f ? 128.f : x;
    if constexpr (ACT == EWF_RELU) return x > 0.f ? 1.f : x != x ? x : 0.f;
    else if constexpr (ACT == EWF_ACT_TANH) { float p, m; gate<T>(2.f * x, p, m); return 4.f * (p * m); }
    else if constexpr (ACT == EWF_ACT_SIGMOID) { float p, m; gate<T>(x, p, m); return p * m; }
    else if constexpr (ACT == EWF_SILU) { float p, m; gate<T>(x, p, m); return fmaf(x * p, m, p); }
    else if constexpr (ACT == EWF_GELU) {
        const Normal n = normal(x);
        return fmaf(x * 0.39894228f, n.e, n.below);
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

template <typename T, int ACT, int U>
__global__ void __launch_bounds__(256) k_act(ActLaunch a, Items items)
{
    constexpr int V = Vec16<T>::V;
    typedef typename T::raw raw;
    Place at[U];
    u32x4 x[U];
    const int cols = a.r.cols;
#pragma unroll
    for (int i = 0; i < U; i++) {
        const uint32_t item = (blockIdx.x * U + i) * 256 + threadIdx.x;
        at[i] = item < items.count ? place(item, items, V) : Place{items.row0, cols};    // (all lanes of a scale's group or none)
        x[i] = u32x4{0u, 0u, 0u, 0u};
        if (at[i].c < cols) x[i] = load_part<T>((const raw *)a.x + row_offset(a.r, at[i].row, a.sx), at[i].c, cols);
    }
#pragma unroll
    for (int i = 0; i < U; i++) {
        const int c = at[i].c;
        float f[V];
#pragma unroll
        for (int e = 0; e < V; e++) f[e] = element<T>(x[i], e);
        if (a.codes)
            keep_part<V>(a.codes + row_offset(a.r, at[i].row, a.scodes), a.scales + row_offset(a.r, at[i].row, a.sscales), c, cols, f,
                         a.code_dtype == EWF_E4M3);
        if (a.y && c < cols) {
#pragma unroll
            for (int e = 0; e < V; e++) f[e] = act_value<T, ACT>(f[e]);
            store_part<T>((raw *)a.y + row_offset(a.r, at[i].row, a.sy), c, cols, pack16<T>(f));
        }
    }
}

// dx = dy act'(x8); without dy: x8 itself.
template <typename T, int ACT, int U>
__global__ void __launch_bounds__(256) k_act_grad(ActLaunch a, Items items)
{
    constexpr int V = Vec16<T>::V;
    typedef typename T::raw raw;
    Place at[U];
    u32x4 dy[U];
    u32x2 code[U];
    uint32_t byte[U];
    const int cols = a.r.cols;
#pragma unroll
    for (int i = 0; i < U; i++) {
        const uint32_t item = (blockIdx.x * U + i) * 256 + threadIdx.x;
        at[i] = item < items.count ? place(item, items, V) : Place{items.row0, cols};
        dy[i] = u32x4{0u, 0u, 0u, 0u};
        code[i] = u32x2{0u, 0u};
        byte[i] = 0;
        const int c = at[i].c;
        if (c < cols) {
            if (a.dy) dy[i] = load_part<T>((const raw *)a.dy + row_offset(a.r, at[i].row, a.sdy), c, cols);
            code[i] = load_codes<V>(a.codes + row_offset(a.r, at[i].row, a.scodes), c, cols);
            byte[i] = a.scales[row_offset(a.r, at[i].row, a.sscales) + c / kKeepBlock];
        }
    }
#pragma unroll
    for (int i = 0; i < U; i++) {
        const int c = at[i].c;
        if (c >= cols) continue;
        float f[V];
        decode_part<V>(code[i], byte[i], a.code_dtype == EWF_E4M3, f);
        if (a.dy) {
#pragma unroll
            for (int e = 0; e < V; e++) f[e] = element<T>(dy[i], e) * act_slope<T, ACT>(f[e]);
        }
        store_part<T>((raw *)a.dx + row_offset(a.r, at[i].row, a.sdx), c, cols, pack16<T>(f));
    }
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
    const uint32_t most = 0x7ffff000u / i.per_row;
    for (uint32_t row = 0; row < a.r.rows; row += i.count / i.per_row) {
        i.row0 = row;
        i.count = (a.r.rows - row < most ? a.r.rows - row : most) * i.per_row;
        constexpr uint32_t U = 1, per = 256 * U;
        const dim3 grid((i.count + per - 1) / per);
        if constexpr (GRAD) hipLaunchKernelGGL((k_act_grad<T, ACT, U>), grid, dim3(256), 0, stream, a, i);
        else hipLaunchKernelGGL((k_act<T, ACT, U>), grid, dim3(256), 0, stream, a, i);
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
