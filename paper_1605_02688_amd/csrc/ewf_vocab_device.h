// What the operators over rows of logits share: rows as vectors, and their sums.
//
// With c = scale log2 e a logit x stands for 2^(c x).  A thread adds e = 2^(c x - m), and for the entropy e (c x - m), about a whole number m that lags
// behind: it moves only where a logit is 2^8 beyond it, so that moves are rare, exact, and e cannot overflow; c x - m is one multiply-add with one
// rounding.  Threads' sums are moved to a common m and added in a fixed order, and come out about the row's largest logit.  Points lie from -2^22 on:
// lower, c x has no fraction left and a point made of it is off by more powers of two than e has (masks of -1e10 and the like), and beside a larger logit
// nothing is left of what lies there.  A row whose largest logit is beyond 2^22 (or leaves float32, as the type's lowest number) is swept again about that.
#pragma once

#include <algorithm>
#include <type_traits>

#include "ewf_ops_device.h"

namespace ewf {

namespace {

typedef unsigned long long u64;

constexpr float kLn2 = 0.693147181f;
constexpr float kInf = __builtin_huge_valf();
constexpr float kFloor = -1e4f;          // powers of two below which nothing is left; products with it stay finite

template <typename T> constexpr uint32_t kNothing = 0xff80ff80u;        // a word of minus infinities
template <> constexpr uint32_t kNothing<F16> = 0xfc00fc00u;
template <> constexpr uint32_t kNothing<F32> = 0xff800000u;

// A row on the grid of `grid` (the address that decides: the results' where there are any): whole 16-byte vectors from element `head` on, which begins a
// unit of LINE bytes, and at most kEdges elements on its two edges.  Results begin on cache lines (128 bytes): a copy of 400 MB whose
// wavefronts' accesses do not takes 5 % longer.
constexpr int kLine = 128, kEdges = 72;
template <typename T, int LINE = 16>
struct Span {
    static constexpr int V = Vec16<T>::V;
    int cols, head, nvec;
    EWF_OPS_DEV Span(const void *grid, int cols) : cols(cols)
    {
        const int over = (int)((uintptr_t)grid & (LINE - 1)) / (int)sizeof(typename T::raw);
        head = over ? LINE / (int)sizeof(typename T::raw) - over : 0;
        head = head < cols ? head : cols;
        nvec = (cols - head) / V;
    }
    EWF_OPS_DEV int edges() const { return cols - nvec * V; }
    EWF_OPS_DEV int edge(int i) const { return i < head ? i : i + nvec * V; }
    EWF_OPS_DEV int edge_of(int c) const { return c < head ? c : c - nvec * V; }       // (an element that is on one)
    EWF_OPS_DEV bool inside(int c) const { return c >= head && c < head + nvec * V; }
};

// Vector j + lane of a row, at any alignment (j the same for all lanes: the address is a scalar and 32 bits of a lane's); STREAM: past the caches.
template <typename T, bool STREAM>
EWF_OPS_DEV u32x4 load_vector(const typename T::raw *first, int j, uint32_t lane)
{
    const typename Vec16<T>::at *from = (const typename Vec16<T>::at *)((const char *)first + (int64_t)j * 16 + lane * 16u);
    return STREAM ? __builtin_nontemporal_load(from) : *from;
}

// Gradients are written past the caches: of 47 MB, copied, 15.9 us for 21.4; of 400 MB 139 for 144.
template <typename T>
EWF_OPS_DEV void store_vector(typename T::raw *first, int j, uint32_t lane, const float *f)
{
    __builtin_nontemporal_store(pack16<T>(f), (u32x4 *)((char *)first + (int64_t)j * 16 + lane * 16u));
}

// The largest of L lanes, in every one.
template <int L>
EWF_OPS_DEV float group_most(float x)
{
    x = fmaxf(x, bits_to_float(lane_move<kSwap1>(float_to_bits(x))));
    x = fmaxf(x, bits_to_float(lane_move<kSwap2>(float_to_bits(x))));
    x = fmaxf(x, bits_to_float(lane_move<kHalfMirror>(float_to_bits(x))));
    x = fmaxf(x, bits_to_float(lane_move<kMirror>(float_to_bits(x))));
    if constexpr (L >= 32) x = fmaxf(x, __shfl_xor(x, 16));
    if constexpr (L >= 64) x = fmaxf(x, __shfl_xor(x, 32));
    return x;
}
EWF_OPS_DEV float wave_max(float x) { return group_most<64>(x); }

// A number that all lanes have, as a scalar.
EWF_OPS_DEV float scalar(float x) { return bits_to_float((uint32_t)__builtin_amdgcn_readfirstlane((int)float_to_bits(x))); }

// A row's place on the (at most two) axes that rows have.
struct RowAt { uint32_t outer, inner; };
EWF_OPS_DEV RowAt row_at(const Rows &r, uint32_t row)
{
    if (r.rows == r.n1) return {0, row};
    const uint32_t o = row / r.n1;
    return {o, row - o * r.n1};
}
EWF_OPS_DEV int64_t at(const RowAt &row, const RowStride &s) { return (int64_t)row.outer * s.outer + (int64_t)row.inner * s.inner; }

// The lowest point.
constexpr float kLowest = -0x1p22f;

// Sums of a thread: s of the e, w of e times their exponent, about m, which moves for a logit above `limit`; peak is the largest logit.
struct Sums {
    float m = kLowest, limit = -kInf, s = 0.f, w = 0.f, peak = -kInf;
};

// Moves the point from `from` to `to` powers of two, upwards (sums of nothing move anywhere).  The product is rounded here and not contracted into the
// sum over lanes behind it, which would add a rounded and an unrounded number: lanes would then hold different sums.
template <bool ENT>
EWF_OPS_DEV void move(Sums &a, float from, float to)
{
#pragma clang fp contract(off)
    const float d = __builtin_amdgcn_fmed3f(from - to, kFloor, 0.f), r = __builtin_amdgcn_exp2f(d);
    if (ENT) a.w = r * fmaf(a.s, d, a.w);
    a.s *= r;
}

// Adds n logits whose largest is `top`; lag = 8 / c.
template <bool ENT, int n>
EWF_OPS_DEV void add(Sums &a, const float *x, float top, float c, float lag)
{
    a.peak = fmaxf(a.peak, top);
    if (__any(top > a.limit)) {
        const float to = fmaxf(a.m, rintf(top * c));
        move<ENT>(a, a.m, to);
        a.m = to;
        a.limit = fmaxf(a.limit, top + lag);
    }
    float w = 0.f;
#pragma unroll
    for (int e = 0; e < n; e++) {
        const float t = fmaf(x[e], c, -a.m), p = __builtin_amdgcn_exp2f(t);
        a.s += p;
        if (ENT) w = fmaf(p, t, w);
    }
    if (ENT && __any(w != w)) {          // (a minus infinity: 0 times that)
        w = 0.f;
#pragma unroll
        for (int e = 0; e < n; e++) {
            const float t = fmaf(x[e], c, -a.m);
            w = fmaf(__builtin_amdgcn_exp2f(t), fmaxf(t, kFloor), w);
        }
    }
    if (ENT) a.w += w;
}

// (the compiler takes the largest of three only after a canonicalising step for each operand; a NaN loses either way)
EWF_OPS_DEV float max3(float a, float b, float c)
{
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}

template <int V>
EWF_OPS_DEV float max_of(const float *x)
{
    float m = max3(x[0], x[1], x[2]);
#pragma unroll
    for (int e = 3; e + 1 < V; e += 2) m = max3(m, x[e], x[e + 1]);
    return V % 2 ? m : max3(m, x[V - 1], x[V - 1]);
}

// A whole number of powers of two near a largest logit: what sums of a wavefront are brought to (threads' points are no further up).
EWF_OPS_DEV float point_of(float peak, float c) { return fmaxf(rintf(peak * c), kLowest); }
// Whether a row whose largest logit this is cannot be summed about such a point: whole numbers and c x have to keep their fractions.
EWF_OPS_DEV bool beyond(float peak, float c) { return fabsf(peak) < kInf && !(fabsf(peak * c) < 0x1p22f); }

// 2^(c (x - ref) - off) of logits x, one multiply-add each: as 2^rest 2^(c x - k), k a whole number.  Rows beyond that (see above) as it is written.
struct Exponent {
    float c, k, ref, off, rest;
    bool as_is;
    EWF_OPS_DEV Exponent() {}
    EWF_OPS_DEV Exponent(float ref, float off, float c) : c(c), ref(scalar(ref)), off(scalar(off))
    {
        const float a = rintf(ref * c), b = rintf(off);
        as_is = beyond(ref, c);
        k = scalar(as_is ? 0.f : a + b);
        rest = scalar(as_is ? 0.f : fmaf(-ref, c, a) + (b - off));
    }
    // the exponents, but for `rest`
    template <int V>
    EWF_OPS_DEV void of(const float *x, float *t) const
    {
        if (as_is)
#pragma unroll
            for (int e = 0; e < V; e++) t[e] = (x[e] - ref) * c - off;
        else
#pragma unroll
            for (int e = 0; e < V; e++) t[e] = fmaf(x[e], c, -k);
    }
};

// A wavefront's sums, in every lane, about its point.
template <bool ENT>
EWF_OPS_DEV Sums wave_sums(Sums a, float c)
{
    a.peak = wave_max(a.peak);
    move<ENT>(a, a.m, point_of(a.peak, c));
    a.s = group_sum<64>(a.s);
    if (ENT) a.w = group_sum<64>(a.w);
    return a;
}

// Those of W wavefronts, left in LDS, in every lane, about their point.
template <int W, bool ENT>
EWF_OPS_DEV Sums joined_sums(const float *peak, const float *s, const float *w, float c)
{
    const int from = threadIdx.x & 15;
    Sums a;
    const float own = from < W ? peak[from] : -kInf;
    a.s = from < W ? s[from] : 0.f;
    if (ENT) a.w = from < W ? w[from] : 0.f;
    a.peak = group_most<16>(own);
    move<ENT>(a, point_of(own, c), point_of(a.peak, c));
    a.s = group_sum<16>(a.s);
    if (ENT) a.w = group_sum<16>(a.w);
    return a;
}

// From their point to the largest logit: at most half a power of two.
template <bool ENT>
EWF_OPS_DEV void settle(Sums &a, float c)
{
    if (a.peak == -kInf) return;
    const float d = fmaf(-a.peak, c, point_of(a.peak, c)), r = __builtin_amdgcn_exp2f(d);
    if (ENT) a.w = r * fmaf(a.s, d, a.w);
    a.s *= r;
}

// The sums of N threads, in every thread, about the row's largest logit.
template <int N, bool ENT>
EWF_OPS_DEV Sums workgroup_sums(Sums a, float c, float *lds)        // lds: 3 * 16 words
{
    a = wave_sums<ENT>(a, c);
    if (N > 64) {
        if ((threadIdx.x & 63) == 0) { lds[threadIdx.x >> 6] = a.peak; lds[16 + (threadIdx.x >> 6)] = a.s; if (ENT) lds[32 + (threadIdx.x >> 6)] = a.w; }
        __syncthreads();
        a = joined_sums<N / 64, ENT>(lds, lds + 16, lds + 32, c);
    }
    settle<ENT>(a, c);
    return a;
}

// ------------------------------------------------------------------ launches

template <typename F>
void by_type(int dtype, F &&f)
{
    if (dtype == EWF_F32) f.template operator()<F32>();
    else if (dtype == EWF_F16) f.template operator()<F16>();
    else f.template operator()<BF16>();
}

// Launches of at most 2^31 threads.
template <typename F>
void by_rows(VocabLaunch a, int64_t blocks_per_row, int threads, F &&launch)
{
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 31) / threads / blocks_per_row);
    for (int64_t row = 0; row < a.r.rows; row += most) {
        const int64_t rows = std::min<int64_t>(most, a.r.rows - row);
        a.row0 = (uint32_t)row;
        a.rows = (uint32_t)rows;
        launch(a, dim3((unsigned)(rows * blocks_per_row)), (unsigned)rows);
    }
}

inline int vectors(const VocabLaunch &a) { return (a.r.cols + (a.dtype == EWF_F32 ? 4 : 8) - 1) / (a.dtype == EWF_F32 ? 4 : 8); }

}  // namespace

}  // namespace ewf
