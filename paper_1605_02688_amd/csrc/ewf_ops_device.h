// Device-side helpers that the operators' kernels share (gfx950, wavefronts of 64): 16-byte accesses at
// element alignment, conversions, sums over groups of lanes, and the 8-bit form of a block of 32 elements.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "ewf_ops.h"

namespace ewf {

#define EWF_OPS_DEV __device__ __forceinline__

// ------------------------------------------------------------------ storage types

struct F32 { typedef float raw; static constexpr int code = EWF_F32; };
struct F16 { typedef uint16_t raw; static constexpr int code = EWF_F16; };
struct BF16 { typedef uint16_t raw; static constexpr int code = EWF_BF16; };

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
// the same at element alignment: the memory instructions of this target take any address
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef u32x4 u32x4_a1 __attribute__((aligned(1)));
typedef u32x2 u32x2_a4 __attribute__((aligned(4)));
typedef u32x2 u32x2_a1 __attribute__((aligned(1)));
typedef unsigned int u32_a2 __attribute__((aligned(2)));
typedef unsigned int u32_a1 __attribute__((aligned(1)));

template <typename T> struct Vec16;                     // 16 bytes of T
template <> struct Vec16<F32> { static constexpr int V = 4; typedef u32x4_a4 at; };
template <> struct Vec16<F16> { static constexpr int V = 8; typedef u32x4_a2 at; };
template <> struct Vec16<BF16> { static constexpr int V = 8; typedef u32x4_a2 at; };

template <typename T>
EWF_OPS_DEV u32x4 load16(const typename T::raw *p)
{
    return *reinterpret_cast<const typename Vec16<T>::at *>(p);
}

template <typename T>
EWF_OPS_DEV void store16(typename T::raw *p, u32x4 v)
{
    *reinterpret_cast<typename Vec16<T>::at *>(p) = v;
}

EWF_OPS_DEV float bits_to_float(uint32_t b) { return __builtin_bit_cast(float, b); }
EWF_OPS_DEV uint32_t float_to_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

// a word of two halves <-> two floats
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <typename T> EWF_OPS_DEV float half_lo(uint32_t w);
template <typename T> EWF_OPS_DEV float half_hi(uint32_t w);
template <> EWF_OPS_DEV float half_lo<BF16>(uint32_t w) { return bits_to_float(w << 16); }
template <> EWF_OPS_DEV float half_hi<BF16>(uint32_t w) { return bits_to_float(w & 0xffff0000u); }
template <> EWF_OPS_DEV float half_lo<F16>(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w).x; }
template <> EWF_OPS_DEV float half_hi<F16>(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w).y; }

// to nearest, ties to even: the one rounding that a result of this type has
template <typename T> EWF_OPS_DEV uint32_t pack_halves(float lo, float hi);
template <> EWF_OPS_DEV uint32_t pack_halves<BF16>(float lo, float hi)
{
    f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
template <> EWF_OPS_DEV uint32_t pack_halves<F16>(float lo, float hi)
{
    f16x2 v = {(_Float16)lo, (_Float16)hi};
    return __builtin_bit_cast(uint32_t, v);
}

// Element e of a 16-byte vector as float; `e` is a constant wherever this is used.
template <typename T>
EWF_OPS_DEV float element(const u32x4 &v, int e)
{
    if constexpr (sizeof(typename T::raw) == 4) return bits_to_float(v[e]);
    else return (e & 1) ? half_hi<T>(v[e >> 1]) : half_lo<T>(v[e >> 1]);
}

template <typename T>
EWF_OPS_DEV u32x4 pack16(const float *f)
{
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (sizeof(typename T::raw) == 4) v[i] = float_to_bits(f[i]);
        else v[i] = pack_halves<T>(f[2 * i], f[2 * i + 1]);
    }
    return v;
}

template <typename T> EWF_OPS_DEV float load1(const typename T::raw *p)
{
    if constexpr (sizeof(typename T::raw) == 4) return *p;
    else return half_lo<T>(*p);
}
template <typename T> EWF_OPS_DEV void store1(typename T::raw *p, float f)
{
    if constexpr (sizeof(typename T::raw) == 4) *p = f;
    else *p = (uint16_t)pack_halves<T>(f, 0.f);
}

// The 16-byte vector whose elements e >= s are v[e - ...] moved down by s elements (zeros above): a row's
// last whole vector made into the vector that the row's end cuts.
template <typename T>
EWF_OPS_DEV u32x4 move_down(u32x4 v, int s)
{
    const int words = sizeof(typename T::raw) == 4 ? s : s >> 1;
    if (words & 2) v = u32x4{v[2], v[3], 0u, 0u};
    if (words & 1) v = u32x4{v[1], v[2], v[3], 0u};
    if (words & 4) v = u32x4{0u, 0u, 0u, 0u};
    if (sizeof(typename T::raw) == 2 && (s & 1))
        v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
    return v;
}

// Elements c .. c + V - 1 of a row of `cols` elements, zeros behind its end, in two steps: the access, and what makes the
// vector of it, which waits for the access.  Rows that a vector is CUT by the end of: that vector's lane reads the row's last
// whole vector -- one access as every other, in flight with them -- and moves it down by what it began too early.
template <typename T, bool CUT = true>
EWF_OPS_DEV u32x4 fetch_part(const typename T::raw *row, int c, int cols)
{
    constexpr int V = Vec16<T>::V;
    u32x4 r = {0u, 0u, 0u, 0u};
    if (!CUT || cols % V == 0) return c < cols ? load16<T>(row + c) : r;
    if (cols >= V) return c < cols ? load16<T>(row + (c <= cols - V ? c : cols - V)) : r;
#pragma unroll
    for (int e = 0; e < V; e++)
        if (c + e < cols) {
            if constexpr (sizeof(typename T::raw) == 4) r[e] = float_to_bits(row[c + e]);
            else r[e >> 1] |= (uint32_t)row[c + e] << ((e & 1) * 16);
        }
    return r;
}

template <typename T, bool CUT = true>
EWF_OPS_DEV u32x4 settle_part(u32x4 v, int c, int cols)
{
    constexpr int V = Vec16<T>::V;
    if (!CUT || cols % V == 0 || cols < V) return v;
    const int early = c - (cols - V);
    return move_down<T>(v, early < 0 ? 0 : early < V ? early : V);
}

template <typename T, bool CUT = true>
EWF_OPS_DEV u32x4 load_part(const typename T::raw *row, int c, int cols)
{
    return settle_part<T, CUT>(fetch_part<T, CUT>(row, c, cols), c, cols);
}

template <typename T, bool CUT = true>
EWF_OPS_DEV void store_part(typename T::raw *row, int c, int cols, u32x4 v)
{
    constexpr int V = Vec16<T>::V;
    if (!CUT || c + V <= cols) { store16<T>(row + c, v); return; }
#pragma unroll
    for (int e = 0; e < V; e++)
        if (c + e < cols) {
            if constexpr (sizeof(typename T::raw) == 4) row[c + e] = bits_to_float(v[e]);
            else row[c + e] = (uint16_t)(v[e >> 1] >> ((e & 1) * 16));
        }
}

// Parameters: the tensors' type, or float32.  Zeros behind the end.
template <typename T, bool CUT = true>
EWF_OPS_DEV void load_params(const void *p, bool f32, int c, int cols, float *out)
{
    constexpr int V = Vec16<T>::V;
    if (f32) {
#pragma unroll
        for (int q = 0; q < V; q += 4) {
            u32x4 w = load_part<F32, CUT>((const float *)p, c + q, cols);
#pragma unroll
            for (int e = 0; e < 4; e++) out[q + e] = element<F32>(w, e);
        }
    } else {
        u32x4 w = load_part<T, CUT>((const typename T::raw *)p, c, cols);
#pragma unroll
        for (int e = 0; e < V; e++) out[e] = element<T>(w, e);
    }
}

EWF_OPS_DEV int64_t row_offset(const Rows &r, uint32_t row, const RowStride &s)
{
    if (r.rows == r.n1) return (int64_t)row * s.inner;
    const uint32_t o = row / r.n1;
    return (int64_t)o * s.outer + (int64_t)(row - o * r.n1) * s.inner;
}

// ------------------------------------------------------------------ sums over groups of lanes

template <int CTRL>
EWF_OPS_DEV uint32_t lane_move(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;    // within quads, 8 and 16 lanes

// The sum over the L lanes of a group (a power of two, aligned), in every lane of it.  Every lane adds the same
// two numbers at each step, so all hold the same bits.
template <int L>
EWF_OPS_DEV float group_sum(float x)
{
    if constexpr (L >= 2) x += bits_to_float(lane_move<kSwap1>(float_to_bits(x)));
    if constexpr (L >= 4) x += bits_to_float(lane_move<kSwap2>(float_to_bits(x)));
    if constexpr (L >= 8) x += bits_to_float(lane_move<kHalfMirror>(float_to_bits(x)));
    if constexpr (L >= 16) x += bits_to_float(lane_move<kMirror>(float_to_bits(x)));
    if constexpr (L >= 32) x += __shfl_xor(x, 16);
    if constexpr (L >= 64) x += __shfl_xor(x, 32);
    return x;
}

// ------------------------------------------------------------------ sigmoids

constexpr float kLog2E = 1.44269504f;

// e = 2^(-u log2 e) = exp(-u) and f = 1 / (1 + e), by the type that results are stored as.  float32: the product's rounding and what
// float32 drops of log2 e correct e to first order, one Newton step the reciprocal: f and 1 - f are off by at most 4.6 times 2^-24 (2^25
// arguments up to 86).  16 bits: the native operations alone, off by about |u| times 2^-24, at most 2^-18 of a gate that is not shut, where half
// a step of float16 is 2^-11.
template <typename T>
EWF_OPS_DEV float exp_neg(float u)
{
    const float t = -u * kLog2E, e = __builtin_amdgcn_exp2f(t);
    if constexpr (sizeof(typename T::raw) == 2) return e;
    const float r = fmaf(-u, 1.92596299e-8f, fmaf(-u, kLog2E, -t));
    return e * __builtin_amdgcn_fmed3f(fmaf(r, 0.693147182f, 1.f), 0.5f, 2.f);     // (the median drops the NaN of infinite u)
}

template <typename T>
EWF_OPS_DEV float recip(float y)                        // y finite, from 1
{
    const float r = __builtin_amdgcn_rcpf(y);
    if constexpr (sizeof(typename T::raw) == 2) return r;
    return fmaf(fmaf(-y, r, 1.f), r, r);
}

// f = sigmoid(u) and 1 - f = e f, small ones relative to themselves.  A gate of less than 2^-126 counts as zero and its complement
// as one, where e f would be infinity times zero; a NaN stays one.
template <typename T>
EWF_OPS_DEV void gate(float u, float &f, float &g)
{
    const float e = exp_neg<T>(u);
    const bool shut = e > 0x1p126f;
    const float h = recip<T>(1.f + e);
    f = shut ? 0.f : h;
    g = shut ? 1.f : e * h;
}

template <typename T>
EWF_OPS_DEV float sigmoid(float x)
{
    if constexpr (sizeof(typename T::raw) == 2) return recip<T>(1.f + exp_neg<T>(x));        // (e may overflow: zero)
    float f, g;
    gate<T>(x, f, g);
    return f;
}

// ------------------------------------------------------------------ 8 bits

// Magnitudes are compared as their bits, which rank NaN above infinity above every number.
template <int L>
EWF_OPS_DEV uint32_t group_max(uint32_t x)
{
    uint32_t y;
    if constexpr (L >= 2) { y = lane_move<kSwap1>(x); x = x > y ? x : y; }
    if constexpr (L >= 4) { y = lane_move<kSwap2>(x); x = x > y ? x : y; }
    if constexpr (L >= 8) { y = lane_move<kHalfMirror>(x); x = x > y ? x : y; }
    return x;
}

// The scale's byte for a block whose largest magnitude has these bits.  L 2^k reaches m 2^E iff m <= 127/64
// (k = E - 6) or 448/256 (k = E - 8): adding what is missing to the next power of two carries into the
// exponent exactly where the mantissa is above that.
EWF_OPS_DEV uint32_t scale_byte(uint32_t top, bool e4m3)
{
    if (top >= 0x7f800000u) return 255;
    const uint32_t e = (top + (e4m3 ? 0x1fffffu : 0x1ffffu)) >> 23;
    const uint32_t less = e4m3 ? 8 : 6;
    return e > less ? e - less : 1;
}

// Four codes of elements already divided by the block's unit (an exact step), rounded to nearest even.
EWF_OPS_DEV uint32_t encode4(float a, float b, float c, float d, bool e4m3)
{
    if (e4m3) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    }
    // 1.5 2^23: the sum's last bit is worth one, its low byte is the whole number in two's complement
    constexpr float kRound = 12582912.f;
    const uint32_t p = float_to_bits(a + kRound), q = float_to_bits(b + kRound), r = float_to_bits(c + kRound), s = float_to_bits(d + kRound);
    const uint32_t pq = __builtin_amdgcn_perm(q, p, 0x0c0c0400u), rs = __builtin_amdgcn_perm(s, r, 0x04000c0cu);
    return pq | rs;
}

EWF_OPS_DEV void decode4(uint32_t w, bool e4m3, float unit, float *out)
{
    if (e4m3) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        out[0] = lo.x * unit; out[1] = lo.y * unit; out[2] = hi.x * unit; out[3] = hi.y * unit;
    } else {
        out[0] = (float)(int8_t)w * unit;
        out[1] = (float)(int8_t)(w >> 8) * unit;
        out[2] = (float)(int8_t)(w >> 16) * unit;
        out[3] = (float)(int8_t)(w >> 24) * unit;
    }
}

// 2^k of a scale's byte; byte 255 is an infinity, and 0 times that is NaN.
EWF_OPS_DEV float scale_unit(uint32_t byte) { return bits_to_float(byte << 23); }

// Writes the V elements f (zeros behind the row's end) of a lane as codes, and once a block its scale.  A block of 32
// is 32 / V neighbouring lanes, all of which take part; c is a multiple of V.
template <int V, bool CUT = true>
EWF_OPS_DEV void keep_part(uint8_t *codes, uint8_t *scales, int c, int cols, const float *f, bool e4m3)
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < V; e++) {
        const uint32_t m = float_to_bits(f[e]) & 0x7fffffffu;
        top = top > m ? top : m;
    }
    top = group_max<kKeepBlock / V>(top);
    const uint32_t byte = scale_byte(top, e4m3);
    const float per = bits_to_float((254u - byte) << 23);              // 2^-k
    uint32_t w[V / 4];
#pragma unroll
    for (int q = 0; q < V / 4; q++) {
        w[q] = encode4(f[4 * q] * per, f[4 * q + 1] * per, f[4 * q + 2] * per, f[4 * q + 3] * per, e4m3);
        if (byte == 255) w[q] = 0;
    }
    if (c + V <= cols) {
        if constexpr (V == 8) *reinterpret_cast<u32x2_a1 *>(codes + c) = u32x2{w[0], w[1]};
        else *reinterpret_cast<u32_a1 *>(codes + c) = w[0];
    } else if constexpr (CUT) {
#pragma unroll
        for (int e = 0; e < V; e++)
            if (c + e < cols) codes[c + e] = (uint8_t)(w[e >> 2] >> ((e & 3) * 8));
    }
    if (c < cols && c % kKeepBlock == 0) scales[c / kKeepBlock] = (uint8_t)byte;
}

// The raw codes of a lane's V elements: zeros behind the row's end.
template <int V, bool CUT = true>
EWF_OPS_DEV u32x2 load_codes(const uint8_t *codes, int c, int cols)
{
    u32x2 w = {0u, 0u};
    if (c + V <= cols) {
        if constexpr (V == 8) w = *reinterpret_cast<const u32x2_a1 *>(codes + c);
        else w[0] = *reinterpret_cast<const u32_a1 *>(codes + c);
    } else if constexpr (CUT) {
#pragma unroll
        for (int e = 0; e < V; e++)
            if (c + e < cols) w[e >> 2] |= (uint32_t)codes[c + e] << ((e & 3) * 8);
    }
    return w;
}

template <int V>
EWF_OPS_DEV void decode_part(u32x2 w, uint32_t byte, bool e4m3, float *out)
{
    const float unit = scale_unit(byte);
#pragma unroll
    for (int q = 0; q < V / 4; q++) decode4(w[q], e4m3, unit, out + 4 * q);
}

}  // namespace ewf
