// Operators over rows of logits: log probabilities of given tokens with entropy and the largest alternatives, the loss against a
// teacher's top logits, and the gradients of both.
//
// With c = scale log2 e a logit x stands for 2^(c x).  A thread adds e = 2^(c x - m), and for the entropy e (c x - m), about a whole number m that lags
// behind: it moves only where a logit is 2^8 beyond it, so that moves are rare, exact, and e cannot overflow; c x - m is one multiply-add with one
// rounding.  Threads' sums are moved to a common m and added in a fixed order, and come out about the row's largest logit.  Where c x itself leaves float32
// (rows of the type's lowest or largest numbers) a row is swept again about its largest.
#include <algorithm>
#include <type_traits>

#include "ewf_ops_device.h"

#ifndef NTBITS
#define NTBITS 0
#endif
namespace ewf {

namespace {

typedef unsigned long long u64;

constexpr float kLn2 = 0.693147181f;
constexpr float kInf = __builtin_huge_valf();
constexpr float kFloor = -1e4f;          // powers of two below which nothing is left; products with it stay finite
constexpr int kCandidates = 512;         // logits that a row's last selection ranks

template <typename T> constexpr uint32_t kNothing = 0xff80ff80u;        // a word of minus infinities
template <> constexpr uint32_t kNothing<F16> = 0xfc00fc00u;
template <> constexpr uint32_t kNothing<F32> = 0xff800000u;

// A row on the 16-byte grid of `grid` (the address that decides: the results' where there are any): whole vectors from element `head` on,
// and at most 2 V - 2 elements on its two edges.
constexpr int kEdges = 16;
template <typename T>
struct Span {
    static constexpr int V = Vec16<T>::V, LINE = 16;
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

// A row's place on the (at most two) axes that rows have.
struct RowAt { uint32_t outer, inner; };
EWF_OPS_DEV RowAt row_at(const Rows &r, uint32_t row)
{
    if (r.rows == r.n1) return {0, row};
    const uint32_t o = row / r.n1;
    return {o, row - o * r.n1};
}
EWF_OPS_DEV int64_t at(const RowAt &row, const RowStride &s) { return (int64_t)row.outer * s.outer + (int64_t)row.inner * s.inner; }

// Sums of a thread: s of the e, w of e times their exponent, about m, which moves for a logit above `limit`; peak is the largest logit.
struct Sums {
    float m = -1e38f, limit = -kInf, s = 0.f, w = 0.f, peak = -kInf;
};

// Moves the point from `from` to `to` powers of two, upwards (sums of nothing move anywhere).
template <bool ENT>
EWF_OPS_DEV void move(Sums &a, float from, float to)
{
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

// A whole number of powers of two near a largest logit: what sums of a wavefront are brought to.
EWF_OPS_DEV float point_of(float peak, float c) { return peak == -kInf ? 0.f : rintf(peak * c); }
// Whether a row whose largest logit this is cannot be summed about such a point.
EWF_OPS_DEV bool beyond(float peak, float c) { return fabsf(peak) < kInf && !(fabsf(peak * c) < 0x1p100f); }

// The sums of N threads, in every thread, about the row's largest logit.
template <int N, bool ENT>
EWF_OPS_DEV Sums workgroup_sums(Sums a, float c, float *lds)        // lds: 3 * 16 words
{
    constexpr int W = N / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    a.peak = wave_max(a.peak);
    float m = point_of(a.peak, c);
    move<ENT>(a, a.m, m);
    a.s = group_sum<64>(a.s);
    if (ENT) a.w = group_sum<64>(a.w);
    if (W > 1) {
        if (lane == 0) { lds[wave] = a.peak; lds[16 + wave] = a.s; if (ENT) lds[32 + wave] = a.w; }
        __syncthreads();
        const int from = lane & 15;
        const float part = from < W ? lds[from] : -kInf;
        a.s = from < W ? lds[16 + from] : 0.f;
        if (ENT) a.w = from < W ? lds[32 + from] : 0.f;
        a.peak = group_most<16>(part);
        m = point_of(a.peak, c);
        move<ENT>(a, point_of(part, c), m);
        a.s = group_sum<16>(a.s);
        if (ENT) a.w = group_sum<16>(a.w);
    }
    if (a.peak != -kInf) {
        const float d = fmaf(-a.peak, c, m), r = __builtin_amdgcn_exp2f(d);       // (at most half a power of two)
        if (ENT) a.w = r * fmaf(a.s, d, a.w);
        a.s *= r;
    }
    return a;
}

// ------------------------------------------------------------------ the largest

// Floats in their order as whole numbers, -0 as +0.  A key is this over the complement of a place, so that keys are ranked by value and,
// among equals, by the lowest place; 0 is no key (minus infinity is none either).
EWF_OPS_DEV uint32_t ordered(float x)
{
    const uint32_t b = float_to_bits(x + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
EWF_OPS_DEV float unordered(uint32_t k) { return bits_to_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
EWF_OPS_DEV u64 key_of(float x, uint32_t at) { return x > -kInf ? (u64)ordered(x) << 32 | (uint32_t)~at : 0; }

// The largest logits of pieces of a row: a piece is what kPieceLanes lanes (a cache line) take in kPieceTrips trips.
constexpr int kPieceLanes = 8, kPieceTrips = 4;
constexpr int kBins = 1024, kBinShift = 16, kChosen = 320;

template <int N>
struct TopLds {
    uint32_t bins[kBins];
    alignas(16) u64 found[kCandidates];
    int chosen[N > 64 ? kChosen : 1], hits[N > 64 ? kCandidates : 1], nchosen, nhits, nfound;
    int bin, upto, before, total;
};

// Where a bin is kept: a lane's 16 are 64 apart.
EWF_OPS_DEV int bin_at(uint32_t bin) { return (int)((bin & 15) << 6 | bin >> 4); }

// Of bins that count numbers from the largest down: the first bin with which there are k of them, how many there are up to its end and before
// it; all of them.  One wavefront.
template <int N>
EWF_OPS_DEV void find_bin(TopLds<N> &l, int k)
{
    const int lane = threadIdx.x & 63;
    int sum = 0;
#pragma unroll
    for (int i = 0; i < 16; i++) sum += l.bins[i * 64 + lane];
    auto up_to = [&](int v, int lanes) {
#pragma unroll
        for (int d = 1; d < lanes; d *= 2) {
            const int u = __shfl_up(v, d);
            v += (lane & (lanes - 1)) >= d ? u : 0;
        }
        return v;
    };
    const int upto = up_to(sum, 64);                     // of this lane's bins and those before
    const u64 reach = __ballot(upto >= k);
    const int at = reach ? __builtin_ctzll(reach) : 63, had = __shfl(upto - sum, at), all = __shfl(upto, 63);
    const int mine = l.bins[(lane & 15) * 64 + at], within = had + up_to(mine, 16);
    const uint32_t ends = (uint32_t)__ballot(within >= k) & 0xffff;
    const int in = ends ? __builtin_ctz(ends) : 15;
    if (lane == in) { l.bin = at * 16 + in; l.before = within - mine; l.upto = within; l.total = all; }
}

// The k-th largest of the lanes' numbers, k up to 64, as ordered() has it, 0 where fewer are above minus infinity: bit by bit.
EWF_OPS_DEV uint32_t kth_of_lanes(float x, int k)
{
    const uint32_t v = x > -kInf ? ordered(x) : 0;
    uint32_t at = 0;
    for (int bit = 31; bit >= 0; bit--) {
        const uint32_t next = at | 1u << bit;
        if (__popcll(__ballot(v >= next)) >= k) at = next;
    }
    return at;
}

// Collects the k largest logits of a row, and perhaps some that are smaller, in found[]: returns how many.  peak: the largest, a number.  pieces: the
// largest of each of the row's pieces, per_part in each part of `per` vectors, of which a thread has the first ones in `mine` (minus infinity
// behind the last); or null.
//
// Logits are counted by their distance below the peak in steps of 2^kBinShift of their order (1/128 of a power of two): the bins that have k of
// them give a bound, and what reaches it is collected and ranked.  With pieces, those are counted in the logits' place: k pieces whose largest reach a
// bound hold k logits that do, and no others can.  A single wavefront takes its lanes' largest for that.
constexpr int kOwnPieces = 4;
template <typename T, int N>
EWF_OPS_DEV int largest(TopLds<N> &l, const typename T::raw *row, const Span<T> &s, const float *pieces, const float *mine, float edge, int parts, int per_part,
                        int per, float peak, int k)
{
    constexpr int V = Vec16<T>::V, W = N / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t top = ordered(peak);
    const typename T::raw *first = row + s.head;
    auto clear_bins = [&] {
        for (int i = tid; i < kBins; i += N) l.bins[i] = 0;
        if (tid == 0) l.nchosen = l.nhits = l.nfound = 0;
        __syncthreads();
    };
    auto count_in = [&](uint32_t bin) { atomicAdd(&l.bins[bin_at(bin < kBins - 1 ? bin : kBins - 1)], 1u); };
    auto find = [&] {
        __syncthreads();
        if (tid < 64) find_bin(l, k);
        __syncthreads();
    };
    // the number that a bin's end stands for, 0 where it has none
    auto end_of = [&](uint32_t bin) { return bin == kBins - 1 || bin + 1 > top >> kBinShift ? 0u : top - ((bin + 1) << kBinShift) + 1; };
    uint32_t bound = 0;
    auto collect = [&](float x, int at) {
        const u64 key = key_of(x, at);
        if (key && (uint32_t)(key >> 32) >= bound) {
            const int i = atomicAdd(&l.nfound, 1);
            if (i < kCandidates) l.found[i] = key;
        }
    };
    // all logits of the row (what follows them is no hurry's: one access at a time)
    auto sweep = [&](auto &&each) {
        for (int j = tid; j < s.nvec; j += N) {
            const u32x4 v = load16<T>(first + (int64_t)j * V);
#pragma unroll
            for (int e = 0; e < V; e++) each(element<T>(v, e), s.head + j * V + e);
        }
        if (tid < s.edges()) each(edge, s.edge(tid));
    };
    auto floor_of = [&](uint32_t bound) { return bound > ordered(-kInf) ? unordered(bound) : -kInf; };      // (below minus infinity lie NaN)
    bool collected = false;
    if constexpr (N == 64) {
        if (s.nvec <= 256 && k <= 64) {
            u32x4 v[4];
            float most = edge;
#pragma unroll
            for (int u = 0; u < 4; u++) {
                v[u] = u32x4{kNothing<T>, kNothing<T>, kNothing<T>, kNothing<T>};
                if (tid + u * N < s.nvec) v[u] = load16<T>(first + (int64_t)(tid + u * N) * V);
            }
#pragma unroll
            for (int u = 0; u < 4; u++)
#pragma unroll
                for (int e = 0; e < V; e++) most = fmaxf(most, element<T>(v[u], e));
            bound = kth_of_lanes(most, k);
            if (bound) {
                const float floor = unordered(bound);
                if (tid == 0) l.nfound = 0;
                __syncthreads();
#pragma unroll
                for (int u = 0; u < 4; u++)
#pragma unroll
                    for (int e = 0; e < V; e++)
                        if (element<T>(v[u], e) >= floor) collect(element<T>(v[u], e), s.head + (tid + u * N) * V + e);
                if (tid < s.edges()) collect(edge, s.edge(tid));
                __syncthreads();
                collected = l.nfound <= kCandidates;
                __syncthreads();
            }
        }
    } else if (pieces) {
        const int n = parts * per_part;
        auto each_piece = [&](auto &&each) {
#pragma unroll
            for (int i = 0; i < kOwnPieces; i++) each(mine[i], i * N + tid);
            for (int i = kOwnPieces * N + tid; i < n; i += N) each(pieces[i], i);
        };
        clear_bins();
        each_piece([&](float x, int) { if (x > -kInf) count_in((top - ordered(x)) >> kBinShift); });
        find();
        if (l.total >= k && l.upto <= kChosen && end_of(l.bin)) {
            bound = end_of(l.bin);
            const float floor = floor_of(bound);
            each_piece([&](float x, int i) { if (x >= floor) l.chosen[atomicAdd(&l.nchosen, 1)] = i; });
            if (tid < s.edges()) collect(edge, s.edge(tid));
            __syncthreads();
            // half a wavefront takes a piece
            constexpr int U = 4;
            static_assert(kPieceLanes * kPieceTrips == 32, "");
            const int half = lane >> 5, trip = (lane >> 3) & 3, in_line = lane & 7, nchosen = l.nchosen;
            for (int c0 = 2 * wave + half; c0 - half < nchosen; c0 += 2 * U * W) {
                u32x4 v[U];
                int j[U];
#pragma unroll
                for (int u = 0; u < U; u++) {
                    const int c = c0 + u * 2 * W, i = l.chosen[c < nchosen ? c : 0];
                    const int part = parts == 1 ? 0 : i / per_part, q = i - part * per_part, end = (part + 1) * per < s.nvec ? (part + 1) * per : s.nvec;
                    j[u] = part * per + (q / 32 * kPieceTrips + trip) * 256 + q % 32 * kPieceLanes + in_line;
                    if (c >= nchosen || j[u] >= end) j[u] = -1;
                    v[u] = u32x4{kNothing<T>, kNothing<T>, kNothing<T>, kNothing<T>};
                    if (j[u] >= 0) v[u] = load16<T>(first + (int64_t)j[u] * V);
                }
#pragma unroll
                for (int u = 0; u < U; u++) {
                    float x[V];
#pragma unroll
                    for (int e = 0; e < V; e++) x[e] = element<T>(v[u], e);
                    if (j[u] >= 0 && max_of<V>(x) >= floor) {
                        const int h = atomicAdd(&l.nhits, 1);
                        if (h < kCandidates) l.hits[h] = j[u];
                    }
                }
            }
            __syncthreads();
            const int hits = l.nhits;
            if (hits <= kCandidates)
                for (int i = tid; i < hits * V; i += N) {
                    const int c = s.head + l.hits[i / V] * V + i % V;
                    collect(load1<T>(row + c), c);
                }
            __syncthreads();
            collected = hits <= kCandidates && l.nfound <= kCandidates;
            __syncthreads();
        }
    }
    if (!collected) {
        clear_bins();
        sweep([&](float x, int) { if (x > -kInf) count_in((top - ordered(x)) >> kBinShift); });
        find();
        const bool all = l.total <= k;
        bound = all ? 0 : end_of(l.bin);
        if (all || (bound && l.upto <= kCandidates)) {
            sweep(collect);
            __syncthreads();
        } else {
            // many equal or nearly equal ones, or a few far above all others: the k-th value digit by digit
            uint32_t value = 0;
            int need = k;
            for (int shift : {22, 12, 2, 0}) {
                const int bits = shift ? 10 : 2;
                clear_bins();
                sweep([&](float x, int) {
                    const uint32_t d = top - ordered(x);
                    if (x > -kInf && (shift == 22 || d >> (shift + bits) == value)) atomicAdd(&l.bins[bin_at(d >> shift & ((1u << bits) - 1))], 1u);
                });
                __syncthreads();
                if (tid < 64) find_bin(l, need);
                __syncthreads();
                value = value << bits | (uint32_t)l.bin;
                need -= l.before;
                __syncthreads();
            }
            // what is larger, and the first `need` that are equal
            const uint32_t kth = top - value;
            bound = kth + 1;
            clear_bins();
            sweep(collect);
            __syncthreads();
            int *counts = (int *)l.bins;                 // of a window's threads
            int had = 0;
            for (int c0 = 0; c0 < s.cols && had < need; c0 += N * V) {
                int c = c0 + tid * V, mine = 0;
                bool equal[V];
#pragma unroll
                for (int e = 0; e < V; e++) {
                    const float x = c + e < s.cols ? load1<T>(row + c + e) : -kInf;
                    equal[e] = x > -kInf && ordered(x) == kth;
                    mine += equal[e] ? 1 : 0;
                }
                int upto = mine;
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const int v = __shfl_up(upto, d);
                    upto += lane >= d ? v : 0;
                }
                if (lane == 63) counts[wave] = upto;
                __syncthreads();
                int place = had + upto - mine;
                for (int w = 0; w < W; w++) {
                    if (w < wave) place += counts[w];
                    had += counts[w];
                }
#pragma unroll
                for (int e = 0; e < V; e++)
                    if (equal[e]) {
                        if (place < need) l.found[atomicAdd(&l.nfound, 1)] = (u64)kth << 32 | (uint32_t)~(c + e);
                        place++;
                    }
                __syncthreads();
            }
        }
    }
    const int n = l.nfound;
    for (int i = n + tid; i < (n + 7) / 8 * 8; i += N) l.found[i] = 0;
    __syncthreads();
    return n;
}

// A key's place among n: the number of larger ones.
EWF_OPS_DEV int place_of(const u64 *found, int n, u64 key)
{
    int place = 0;
    for (int q = 0; q < n; q += 8)
#pragma unroll
        for (int e = 0; e < 8; e++) place += found[q + e] > key ? 1 : 0;
    return place;
}

// ------------------------------------------------------------------ a row's results

// Writes what a row's sums give, and its alternatives from nfound keys among which they are.
template <int N>
EWF_OPS_DEV void finish_logprobs(const VocabLaunch &a, const RowAt &row, const Sums &sum, float token_logit, const u64 *found, int nfound)
{
    const bool none = sum.peak == -kInf && sum.s == 0.f;
    const float logsum = none ? -kInf : logf(sum.s);
    const bool nan = !none && !(sum.s < kInf);           // a NaN or an infinity among the logits
    const float bad = __builtin_nanf("");
    if (threadIdx.x == 0) {
        if (a.logprob) a.logprob[at(row, a.slogprob)] = nan ? bad : none ? -kInf : fmaf(token_logit - sum.peak, a.scale, -logsum);
        if (a.peak) a.peak[at(row, a.speak)] = nan ? bad : sum.peak;
        if (a.logsum) a.logsum[at(row, a.slogsum)] = nan ? bad : logsum;
        if (a.entropy) a.entropy[at(row, a.sentropy)] = nan ? bad : none ? 0.f : logsum - kLn2 * (sum.w / sum.s);
    }
    if (a.top) {
        float *value = a.top_values + at(row, a.stop_values);
        int32_t *index = a.top_indices + at(row, a.stop_indices);
        for (int i = threadIdx.x; i < nfound; i += N) {
            const u64 key = found[i];
            const int place = place_of(found, nfound, key);
            if (place >= a.top) continue;
            value[place] = fmaf(unordered((uint32_t)(key >> 32)) - sum.peak, a.scale, -logsum);
            index[place] = (int32_t)~(uint32_t)key;
        }
        for (int i = nfound + threadIdx.x; i < a.top; i += N) { value[i] = nan ? bad : -kInf; index[i] = -1; }
    }
}

// A row without a token: zeros, and no alternatives.
template <int N>
EWF_OPS_DEV void padding_logprobs(const VocabLaunch &a, const RowAt &row)
{
    if (threadIdx.x == 0) {
        if (a.logprob) a.logprob[at(row, a.slogprob)] = 0.f;
        if (a.peak) a.peak[at(row, a.speak)] = 0.f;
        if (a.logsum) a.logsum[at(row, a.slogsum)] = 0.f;
        if (a.entropy) a.entropy[at(row, a.sentropy)] = 0.f;
    }
    if (a.top) {
        float *value = a.top_values + at(row, a.stop_values);
        int32_t *index = a.top_indices + at(row, a.stop_indices);
        for (int i = threadIdx.x; i < a.top; i += N) { value[i] = -kInf; index[i] = -1; }
    }
}

EWF_OPS_DEV bool is_padding(const VocabLaunch &a, const RowAt &row, int &token)
{
    token = -1;
    if (!a.tokens) return false;
    token = a.tokens[at(row, a.stokens)];
    return (uint32_t)token >= (uint32_t)a.r.cols;
}

// ------------------------------------------------------------------ a teacher's entries

// The entries of a row in LDS.  An entry inside the row's vectors is in the list of the thread that takes its vector (thread = vector mod N),
// one on an edge in the list of that edge's thread, with no trip.
template <int N>
struct Entries {
    int head[N];                                        // last entry of each thread's list, -1
    int next[kMaxTop], index[kMaxTop], trip[kMaxTop], owner[kMaxTop];
    float q[kMaxTop], logq[kMaxTop], logit[kMaxTop], grad[kMaxTop];
    int edge[kEdges];                                   // an entry on each edge element, -1
    float tail_q, total_q;                              // 1 - sum q; sum q
    int live;                                           // entries that exist
    float gradient[4];                                  // of the logits that no entry names (see Slope)
};

template <int N>
EWF_OPS_DEV void clear(Entries<N> &l)
{
    l.head[threadIdx.x] = -1;
    if (threadIdx.x < kEdges) l.edge[threadIdx.x] = -1;
}

EWF_OPS_DEV float load_teacher(const VocabLaunch &a, int64_t at)
{
    if (a.teacher_dtype == EWF_F32) return ((const float *)a.teacher_values)[at];
    const uint32_t h = ((const uint16_t *)a.teacher_values)[at];
    return a.teacher_dtype == EWF_BF16 ? half_lo<BF16>(h) : half_lo<F16>(h);
}

// Reads and ranks a row's entries: one wavefront, two entries a lane, after clear() and a barrier.  The vectors of this workgroup are j0 .. j1 - 1 (thread
// (j - j0) mod N takes vector j); `edges`: and the edges.
template <typename T, int N>
EWF_OPS_DEV void read_entries(Entries<N> &l, const VocabLaunch &a, const RowAt &row, const typename T::raw *logits, const Span<T> &s, int j0, int j1, bool edges)
{
    constexpr int V = Vec16<T>::V;
    const int lane = threadIdx.x;
    const int64_t values = at(row, a.steacher_values), indices = at(row, a.steacher_indices);
    int c[2];
    float v[2], x[2];
    bool live[2];
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int i = h * 64 + lane;
        c[h] = i < a.entries ? a.teacher_indices[indices + i] : -1;
        v[h] = i < a.entries ? load_teacher(a, values + i) : 0.f;
        live[h] = (uint32_t)c[h] < (uint32_t)s.cols;
    }
    const int some = __popcll(__ballot(live[0])) + __popcll(__ballot(live[1]));
#pragma unroll
    for (int h = 0; h < 2; h++) {
        x[h] = live[h] ? load1<T>(logits + c[h]) : 0.f;
        v[h] = live[h] ? v[h] * a.teacher_scale : -kInf;
    }
    float q[2], tail = 0.f, total;
    if (a.with_tail) {
        q[0] = expf(v[0]); q[1] = expf(v[1]);
        total = group_sum<64>(q[0] + q[1]);
        tail = fmaxf(1.f - total, 0.f);
        if (!(total < kInf)) tail = total - total;      // (a NaN stays one)
    } else {
        const float top = wave_max(fmaxf(v[0], v[1])), m = top == -kInf ? 0.f : top;
        q[0] = expf(v[0] - m); q[1] = expf(v[1] - m);
        const float sum = group_sum<64>(q[0] + q[1]), log_sum = logf(sum);
#pragma unroll
        for (int h = 0; h < 2; h++) {
            q[h] = sum == 0.f ? 0.f : q[h] / sum;
            v[h] = v[h] - m - log_sum;
        }
        total = sum == 0.f ? 0.f : sum < kInf ? 1.f : sum - sum;
    }
    if (lane == 0) { l.tail_q = tail; l.total_q = total; l.live = some; }
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int i = h * 64 + lane;
        l.index[i] = live[h] ? c[h] : -1;
        l.q[i] = live[h] ? q[h] : 0.f;
        l.logq[i] = v[h];
        l.logit[i] = x[h];
        if (!live[h]) continue;
        const int j = s.inside(c[h]) ? (c[h] - s.head) / V : -1;
        l.trip[i] = -1;
        int owner;
        if (j < 0) {
            const int e = s.edge_of(c[h]);
            owner = (uint32_t)e % N;
            if (edges) l.edge[e] = i;                   // (of several that are the same one, any: they have the same gradient)
        } else {
            owner = (uint32_t)j % N;
            if (j >= j0 && j < j1) { owner = (j - j0) % N; l.trip[i] = (j - j0) / N; }
        }
        l.owner[i] = owner;
        l.next[i] = atomicExch(&l.head[owner], i);
    }
}

// Behind a barrier: the probabilities of all entries with entry i's index, in the entries' order, and whether it is the first of them.
template <int N>
EWF_OPS_DEV float same_index(const Entries<N> &l, int i, int entries, bool &first)
{
    const int c = l.index[i];
    first = true;
    if (c < 0) return 0.f;
    bool again = false;
    for (int k = l.head[l.owner[i]]; k >= 0; k = l.next[k]) {
        if (k == i || l.index[k] != c) continue;
        again = true;
        first = first && k > i;
    }
    if (!again) return l.q[i];
    float q = 0.f;
    for (int k = 0; k < entries; k++) q += l.index[k] == c ? l.q[k] : 0.f;
    return q;
}

// The gradient of a logit x that no entry names is coef 2^(c (x - ref) - off), that of an entry factor (mass 2^(c (x - ref) - logsum2) - q).
struct Slope { float ref, off, coef, logsum2, mass, factor; };

EWF_OPS_DEV bool tail_counts(float tail, float logsum) { return tail - logsum >= -126.f * kLn2; }

EWF_OPS_DEV Slope slope_of(const VocabLaunch &a, float peak, float logsum, float tail, float tail_q, float total_q, float weight)
{
    Slope g;
    g.factor = weight * a.scale;
    g.ref = peak;
    g.logsum2 = g.off = logsum * kLog2E;
    g.mass = total_q;
    g.coef = g.factor * total_q;
    if (a.with_tail && tail_counts(tail, logsum) && tail_q > 0.f) {
        // m p - q_t p / p_t, as p / p_t (m p_t - q_t): the first is at most 1
        g.mass = total_q + tail_q;
        g.off = tail * kLog2E;
        g.coef = g.factor * fmaf(g.mass, expf(tail - logsum), -tail_q);
    }
    if (peak == -kInf) { g.ref = g.off = g.logsum2 = 0.f; g.coef = 0.f; }       // (a student without a logit: p = 0)
    return g;
}

// Behind the row's sums (of all logits, or with a tail of those that no entry names) and a barrier: one wavefront writes the loss and the
// statistics, and with `slope` what the gradients need.
template <int N>
EWF_OPS_DEV void finish_distill(const VocabLaunch &a, Entries<N> &l, const RowAt &row, Sums sum, bool slope, Slope &g)
{
    const int lane = threadIdx.x & 63;
    bool first[2];
    float all[2], x[2];
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int i = h * 64 + lane;
        all[h] = same_index(l, i, a.entries, first[h]);
        first[h] = first[h] && l.index[i] >= 0;
        x[h] = l.logit[i];
    }
    float peak = sum.peak, total = sum.s, tail = -kInf;
    if (a.with_tail) {
        peak = wave_max(fmaxf(peak, fmaxf(first[0] ? x[0] : -kInf, first[1] ? x[1] : -kInf)));
        const float ref = peak == -kInf ? 0.f : peak;
        float e = 0.f;
#pragma unroll
        for (int h = 0; h < 2; h++) e += first[h] ? __builtin_amdgcn_exp2f((x[h] - ref) * a.c) : 0.f;
        e = group_sum<64>(e);
        if (sum.s != 0.f) tail = fmaf(sum.peak - ref, a.scale, logf(sum.s));
        total = e + (sum.peak == -kInf ? 0.f : sum.s * __builtin_amdgcn_exp2f((sum.peak - ref) * a.c));
    }
    const bool none = total == 0.f;
    const float logsum = none ? -kInf : logf(total);
    const bool nan = !none && !(total < kInf);
    float loss = 0.f;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int i = h * 64 + lane;
        const float q = l.q[i], logp = none ? -kInf : fmaf(x[h] - peak, a.scale, -logsum);
        if (l.index[i] >= 0 && q != 0.f) loss += q * (l.logq[i] - logp);
    }
    loss = group_sum<64>(loss);
    const float tail_q = l.tail_q, bad = __builtin_nanf("");
    if (a.with_tail && tail_q != 0.f && (tail_counts(tail, logsum) || tail_q != tail_q)) loss += tail_q * (logf(tail_q) - (tail - logsum));
    if (lane == 0) {
        if (a.loss) a.loss[at(row, a.sloss)] = nan ? bad : loss;
        if (a.peak) a.peak[at(row, a.speak)] = nan ? bad : peak;
        if (a.logsum) a.logsum[at(row, a.slogsum)] = nan ? bad : logsum;
        if (a.tail) a.tail[at(row, a.stail)] = nan ? bad : tail;
    }
    if (!slope) return;
    const float weight = a.dloss ? a.dloss[at(row, a.sdloss)] : 1.f;
    g = slope_of(a, nan ? bad : peak, nan ? bad : logsum, tail, tail_q, l.total_q, weight);
#pragma unroll
    for (int h = 0; h < 2; h++)
        l.grad[h * 64 + lane] = g.factor * fmaf(g.mass, __builtin_amdgcn_exp2f(fmaf(x[h] - g.ref, a.c, -g.logsum2)), -all[h]);
    if (lane == 0) { l.gradient[0] = g.ref; l.gradient[1] = g.off; l.gradient[2] = g.coef; }
}

EWF_OPS_DEV void padding_distill(const VocabLaunch &a, const RowAt &row)
{
    if (threadIdx.x) return;
    if (a.loss) a.loss[at(row, a.sloss)] = 0.f;
    if (a.peak) a.peak[at(row, a.speak)] = 0.f;
    if (a.logsum) a.logsum[at(row, a.slogsum)] = 0.f;
    if (a.tail) a.tail[at(row, a.stail)] = 0.f;
}

// ------------------------------------------------------------------ sums over rows

enum { kLogprobs = 0, kDistill = 1, kDistillTail = 2 };

// The sums of a row that cannot be taken about a whole number of powers of two (see beyond): about its largest logit, element by element.
template <typename T, int N, int KIND, typename L>
EWF_OPS_DEV void sum_again(const VocabLaunch &a, const typename T::raw *p, const Span<T> &s, int j0, int j1, bool edges, const L &entries, float *lds,
                                       Sums &sum)
{
    constexpr int V = Vec16<T>::V;
    const int tid = threadIdx.x, end = s.head + j1 * V;
    float total = 0.f, weighted = 0.f;
    for (int c = s.head + j0 * V + tid; c < end + (edges ? s.edges() : 0); c += N) {
        const int at = c < end ? c : s.edge(c - end);
        float x = load1<T>(p + at);
        if constexpr (KIND == kDistillTail)
            for (int k = 0; k < a.entries; k++) x = entries.index[k] == at ? -kInf : x;
        const float t = fmaxf((x - sum.peak) * a.c, kFloor), e = __builtin_amdgcn_exp2f(t);
        total += x == x ? e : x;
        weighted = fmaf(e, t, weighted);
    }
    total = group_sum<64>(total);
    weighted = group_sum<64>(weighted);
    __syncthreads();
    if ((tid & 63) == 0) { lds[tid >> 6] = total; lds[16 + (tid >> 6)] = weighted; }
    __syncthreads();
    sum.s = group_sum<16>((tid & 15) < N / 64 ? lds[tid & 15] : 0.f);
    sum.w = group_sum<16>((tid & 15) < N / 64 ? lds[16 + (tid & 15)] : 0.f);
}

// A workgroup takes rows, or parts of rows (a.splits of each), one after the other, the next one's first vectors in flight while it finishes.  Where rows
// have parts or alternatives are asked for it leaves sums and, TOP, the largest of their pieces in the workspace.
template <typename T, int N, bool ENT, bool TOP, int KIND, bool STREAM>
__global__ void __launch_bounds__(N) k_rows(VocabLaunch a)
{
    typedef typename T::raw raw;
    constexpr int V = Vec16<T>::V, U = kPieceTrips;
    __shared__ float sums[48];
    __shared__ typename std::conditional<KIND != kLogprobs, Entries<N>, int>::type entries;
    const int tid = threadIdx.x;
    const bool parts = a.parts != nullptr;
    const uint32_t splits = (uint32_t)a.splits, items = a.rows * splits;

    struct Item { RowAt row; uint32_t part; const raw *p; int token, j0, j1; bool edges; };
    auto item_at = [&](uint32_t i) {
        Item t;
        const uint32_t row = splits == 1 ? i : i / splits, split = i - row * splits;
        t.part = i;
        t.edges = split == 0;
        t.row = row_at(a.r, a.row0 + row);
        t.p = (const raw *)a.logits + at(t.row, a.slogits);
        const Span<T> s(t.p, a.r.cols);
        const int per = splits == 1 ? s.nvec : (s.nvec + (int)splits - 1) / (int)splits;
        t.j0 = (int)split * per < s.nvec ? (int)split * per : s.nvec;
        t.j1 = t.j0 + per < s.nvec ? t.j0 + per : s.nvec;
        return t;
    };
    // the first item from i on that is no padding (whose results it writes)
    auto next_item = [&](uint32_t &i, Item &t) {
        for (; i < items; i += gridDim.x) {
            t = item_at(i);
            if constexpr (KIND == kLogprobs) {
                if (is_padding(a, t.row, t.token)) {
                    if (!parts) padding_logprobs<N>(a, t.row);
                    continue;
                }
            }
            return true;
        }
        return false;
    };
    // vector j of an item (behind its end: the last one, left out later)
    auto fetch = [&](const Item &t, const raw *first, int j) {
        const u32x4 *from = (const u32x4 *)((const char *)first + (uint32_t)(j < t.j1 ? j : t.j1 - 1) * 16u);
        return STREAM ? __builtin_nontemporal_load(from) : *from;
    };
    uint32_t i = blockIdx.x;
    Item t;
    u32x4 v[U];
    bool more = next_item(i, t);
    auto begin = [&](const Item &t) {
        const raw *first = t.p + Span<T>(t.p, a.r.cols).head;
        if (t.j0 < t.j1)
#pragma unroll
            for (int u = 0; u < U; u++) v[u] = fetch(t, first, t.j0 + tid + u * N);
    };
    if (more) begin(t);
    while (more) {
        const Span<T> s(t.p, a.r.cols);
        const int j0 = t.j0, j1 = t.j1;
        const bool edges = t.edges;
        const RowAt row = t.row;
        const raw *p = t.p;
        float edge = -kInf;
        if (edges && tid < s.edges()) edge = load1<T>(p + s.edge(tid));
        float token_logit = 0.f;
        if (KIND == kLogprobs && !parts && t.token >= 0) token_logit = load1<T>(p + t.token);
        bool live = true;
        if constexpr (KIND != kLogprobs)
            if (KIND == kDistillTail || !parts) {
                clear(entries);
                __syncthreads();
                if (tid < 64) read_entries<T>(entries, a, row, p, s, j0, j1, edges);
                __syncthreads();
                live = entries.live != 0;
            }
        if constexpr (KIND == kDistillTail)
            if (edges && tid < kEdges && entries.edge[tid] >= 0) edge = -kInf;
        int hit = 0x7fffffff;                                // the next of this thread's trips that holds an entry
        auto next_hit = [&](int from) {
            hit = 0x7fffffff;
            if constexpr (KIND == kDistillTail)
                for (int k = entries.head[tid]; k >= 0; k = entries.next[k])
                    if (entries.trip[k] >= from && entries.trip[k] < hit) hit = entries.trip[k];
        };
        next_hit(0);
        Sums sum;
        float most_of_piece = -kInf;
        auto take = [&](const u32x4 &v, int trip) {
            float x[V];
#pragma unroll
            for (int e = 0; e < V; e++) x[e] = element<T>(v, e);
            if constexpr (KIND == kDistillTail)
                if (hit == trip) {
                    for (int k = entries.head[tid]; k >= 0; k = entries.next[k]) {
                        const int at = entries.trip[k] == trip ? (entries.index[k] - s.head) % V : V;
#pragma unroll
                        for (int e = 0; e < V; e++) x[e] = e == at ? -kInf : x[e];
                    }
                    next_hit(trip + 1);
                }
            const float most = max_of<V>(x);
            if (TOP) most_of_piece = fmaxf(most_of_piece, most);
            add<ENT, V>(sum, x, most, a.c, a.lag);
        };
        uint32_t ni = i + gridDim.x;
        Item nt;
        const bool nmore = next_item(ni, nt);
        float *pieces = TOP ? a.pieces + (int64_t)t.part * a.pieces_per_part + tid / kPieceLanes : nullptr;
        int pieces_left = TOP ? a.pieces_per_part : 0;
        auto end_of_pieces = [&] {
            if constexpr (TOP) {
                static_assert(U == kPieceTrips && N == 256, "");
                float m = most_of_piece;
                m = fmaxf(m, bits_to_float(lane_move<kSwap1>(float_to_bits(m))));
                m = fmaxf(m, bits_to_float(lane_move<kSwap2>(float_to_bits(m))));
                m = fmaxf(m, bits_to_float(lane_move<kHalfMirror>(float_to_bits(m))));
                if (tid % kPieceLanes == 0) *pieces = m;
                pieces += N / kPieceLanes;
                pieces_left -= N / kPieceLanes;
                most_of_piece = -kInf;
            }
        };
        // each vector's registers take the next block's, or the next item's first, as soon as it is done
        if (live && j0 < j1) {
            const raw *first = p + s.head;
            int j = j0 + tid, trip = 0;
            for (; j - tid + U * N < j1; j += U * N, trip += U) {
#pragma unroll
                for (int u = 0; u < U; u++) {
                    take(v[u], trip + u);
                    v[u] = fetch(t, first, j + (U + u) * N);
                }
                end_of_pieces();
            }
#pragma unroll
            for (int u = 0; u < U; u++)
                if (__any(j + u * N < j1)) {
                    if (j + u * N >= j1) v[u] = u32x4{kNothing<T>, kNothing<T>, kNothing<T>, kNothing<T>};
                    take(v[u], trip + u);
                }
            end_of_pieces();
        }
        while (pieces_left > 0) end_of_pieces();          // (rows that begin in a vector have fewer, and a row's last part)
        if (nmore) begin(nt);
        if (live) {
            add<ENT, 1>(sum, &edge, edge, a.c, a.lag);
            sum = workgroup_sums<N, ENT>(sum, a.c, sums);
            if (beyond(sum.peak, a.c)) sum_again<T, N, KIND>(a, p, s, j0, j1, edges, entries, sums, sum);
            if (parts) {
                if (tid == 0) {
                    float *out = a.parts + (int64_t)t.part * 4;
                    out[0] = sum.peak; out[1] = sum.s; out[2] = sum.w;
                }
            } else if constexpr (KIND == kLogprobs) {
                finish_logprobs<N>(a, row, sum, token_logit, nullptr, 0);
            } else if (tid < 64) {
                Slope g;
                finish_distill(a, entries, row, sum, false, g);
            }
        } else if (!parts) padding_distill(a, row);
        if (N > 64 || KIND != kLogprobs) __syncthreads();          // (LDS is the next item's)
        i = ni;
        t = nt;
        more = nmore;
    }
}

// Joins the parts of a row.
template <typename T, int N, bool TOP, int KIND>
__global__ void __launch_bounds__(N, TOP && N > 64 ? 8 : 1) k_join(VocabLaunch a)
{
    typedef typename T::raw raw;
    __shared__ typename std::conditional<KIND != kLogprobs, Entries<N>, int>::type entries;
    __shared__ typename std::conditional<TOP, TopLds<N>, int>::type top;
    const RowAt row = row_at(a.r, a.row0 + blockIdx.x);
    const raw *p = (const raw *)a.logits + at(row, a.slogits);
    const int tid = threadIdx.x, lane = tid & 63, splits = a.splits;
    const int64_t part = (int64_t)blockIdx.x * splits;
    const Span<T> s(p, a.r.cols);
    // (all loads that do not wait for another)
    const float *pieces = TOP && a.pieces ? a.pieces + part * a.pieces_per_part : nullptr;
    float mine[kOwnPieces], edge = -kInf;
    if constexpr (TOP) {
#pragma unroll
        for (int i = 0; i < kOwnPieces; i++) mine[i] = pieces && i * N + tid < splits * a.pieces_per_part ? pieces[i * N + tid] : -kInf;
        if (tid < s.edges()) edge = load1<T>(p + s.edge(tid));
    }
    Sums sum;
    if (lane < splits) {
        const float *in = a.parts + (part + lane) * 4;
        sum.peak = in[0]; sum.s = in[1]; sum.w = in[2];
    }
    int token = 0;
    if constexpr (KIND == kLogprobs) {
        if (is_padding(a, row, token)) { padding_logprobs<N>(a, row); return; }
    } else {
        clear(entries);
        __syncthreads();
        if (tid < 64) read_entries<T>(entries, a, row, p, s, 0, 0, false);
        __syncthreads();
        if (entries.live == 0) { padding_distill(a, row); return; }
    }
    const float token_logit = KIND == kLogprobs && token >= 0 ? load1<T>(p + token) : 0.f;
    const float peak = wave_max(sum.peak);
    move<true>(sum, (sum.peak - peak) * a.c, 0.f);
    sum.s = group_sum<64>(sum.s);
    sum.w = group_sum<64>(sum.w);
    sum.peak = peak;
    const u64 *found = nullptr;
    int nfound = 0;
    if constexpr (TOP) {
        if (fabsf(peak) < kInf && sum.s < kInf)
            nfound = largest<T, N>(top, p, s, pieces, mine, edge, splits, a.pieces_per_part, (s.nvec + splits - 1) / splits, peak, a.top);
        found = top.found;
    }
    if constexpr (KIND == kLogprobs) finish_logprobs<N>(a, row, sum, token_logit, found, nfound);
    else if (tid < 64) {
        Slope g;
        finish_distill(a, entries, row, sum, false, g);
    }
}

// ------------------------------------------------------------------ gradients from saved statistics

constexpr int kGradThreads = 256;

// Writes vector j of a row, whose elements are f.
template <typename T>
EWF_OPS_DEV void store_vector(typename T::raw *out, const Span<T> &s, int j, const float *f, int nt = 0)
{
    u32x4 *to = (u32x4 *)(out + s.head) + j;
    if (NTBITS & 4) __builtin_nontemporal_store(pack16<T>(f), to);
    else *to = pack16<T>(f);
}
template <typename T>
EWF_OPS_DEV u32x4 load_vector(const typename T::raw *p, const Span<T> &s, int j, int nt)
{
    const typename Vec16<T>::at *from = (const typename Vec16<T>::at *)(p + s.head) + j;
    return NTBITS & 2 ? __builtin_nontemporal_load(from) : *from;
}

// One workgroup a piece of U vectors a thread of a row.  dx_j = c (g ([j = token] - p_j) - h p_j (log p_j + entropy))
template <typename T, bool ENT, int U>
__global__ void __launch_bounds__(kGradThreads) k_logprobs_grad(VocabLaunch a)
{
    typedef typename T::raw raw;
    constexpr int V = Vec16<T>::V, N = kGradThreads;
    const uint32_t pieces = (uint32_t)a.splits, piece = blockIdx.x % pieces;
    const RowAt row = row_at(a.r, a.row0 + blockIdx.x / pieces);
    const raw *p = (const raw *)a.logits + at(row, a.slogits);
    raw *out = (raw *)a.dlogits + at(row, a.sdlogits);
    const Span<T> s(out, a.r.cols);
    const int tid = threadIdx.x, j0 = (int)piece * (U * N) + tid;
    const bool edge = piece == 0 && tid < s.edges();
    int token;
    if (is_padding(a, row, token)) {
        const float zero[V] = {};
#pragma unroll
        for (int u = 0; u < U; u++)
            if (j0 + u * N < s.nvec) store_vector<T>(out, s, j0 + u * N, zero);
        if (edge) store1<T>(out + s.edge(tid), 0.f);
        return;
    }
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        v[u] = u32x4{0u, 0u, 0u, 0u};
        if (j0 + u * N < s.nvec) v[u] = load_vector<T>(p, s, j0 + u * N, 0);
    }
    const float x = edge ? load1<T>(p + s.edge(tid)) : 0.f;
    const float peak = a.peak[at(row, a.speak)], logsum = a.logsum[at(row, a.slogsum)];
    const float g = a.dlogprob ? a.dlogprob[at(row, a.sdlogprob)] * a.scale : 0.f;
    const float h = ENT ? a.dentropy[at(row, a.sdentropy)] * a.scale : 0.f, H = ENT ? a.entropy[at(row, a.sentropy)] : 0.f;
    const bool none = peak == -kInf;                     // (no logit at all: no gradient)
    const float ref = none ? 0.f : peak, off = none ? 0.f : logsum * kLog2E;
    const float A = none ? 0.f : -g - (ENT ? h * H : 0.f), B = none ? 0.f : -h * kLn2, hot = none ? 0.f : g;
    auto slope = [&](float x, int c) {
        const float t = fmaf(x - ref, a.c, -off), q = __builtin_amdgcn_exp2f(t);
        return fmaf(q, ENT ? fmaf(B, fmaxf(t, kFloor), A) : A, c == token ? hot : 0.f);
    };
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int j = j0 + u * N, c = s.head + j * V;
        if (j >= s.nvec) continue;
        float f[V];
#pragma unroll
        for (int e = 0; e < V; e++) f[e] = slope(element<T>(v[u], e), c + e);
        store_vector<T>(out, s, j, f, 0);
    }
    if (edge) store1<T>(out + s.edge(tid), slope(x, s.edge(tid)));
}

// The entries' gradients into a vector that holds some.
template <int V, int N>
EWF_OPS_DEV void put_entries(const Entries<N> &l, int trip, int head, float *f)
{
    for (int k = l.head[threadIdx.x]; k >= 0; k = l.next[k]) {
        if (l.trip[k] != trip) continue;
        const int at = (l.index[k] - head) % V;
        const float g = l.grad[k];
#pragma unroll
        for (int e = 0; e < V; e++) f[e] = e == at ? g : f[e];
    }
}

template <int N>
EWF_OPS_DEV uint32_t trips_with_entries(const Entries<N> &l)
{
    uint32_t m = 0;
    for (int k = l.head[threadIdx.x]; k >= 0; k = l.next[k])
        if (l.trip[k] >= 0) m |= 1u << l.trip[k];
    return m;
}

template <typename T, int U>
__global__ void __launch_bounds__(kGradThreads) k_distill_grad(VocabLaunch a)
{
    typedef typename T::raw raw;
    constexpr int V = Vec16<T>::V, N = kGradThreads;
    __shared__ Entries<N> l;
    const uint32_t pieces = (uint32_t)a.splits, piece = blockIdx.x % pieces;
    const RowAt row = row_at(a.r, a.row0 + blockIdx.x / pieces);
    const raw *p = (const raw *)a.logits + at(row, a.slogits);
    raw *out = (raw *)a.dlogits + at(row, a.sdlogits);
    const Span<T> s(out, a.r.cols);
    const int tid = threadIdx.x, begin = (int)piece * (U * N), j0 = begin + tid;
    const int end = begin + U * N < s.nvec ? begin + U * N : s.nvec;
    const bool edge = piece == 0 && tid < s.edges();
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        v[u] = u32x4{0u, 0u, 0u, 0u};
        if (j0 + u * N < end) v[u] = load_vector<T>(p, s, j0 + u * N, 0);
    }
    const float x = edge ? load1<T>(p + s.edge(tid)) : 0.f;
    clear(l);
    __syncthreads();
    if (tid < 64) read_entries<T>(l, a, row, p, s, begin, end, piece == 0);
    __syncthreads();
    const float peak = a.peak[at(row, a.speak)], logsum = a.logsum[at(row, a.slogsum)];
    const float tail = a.with_tail ? a.tail[at(row, a.stail)] : 0.f;
    const float weight = a.dloss ? a.dloss[at(row, a.sdloss)] : 1.f;
    Slope g = slope_of(a, peak, logsum, tail, l.tail_q, l.total_q, weight);
    const bool padding = l.live == 0;
    if (tid < a.entries) {
        bool first;
        const float q = same_index(l, tid, a.entries, first);
        l.grad[tid] = g.factor * fmaf(g.mass, __builtin_amdgcn_exp2f(fmaf(l.logit[tid] - g.ref, a.c, -g.logsum2)), -q);
    }
    __syncthreads();
    const uint32_t held = trips_with_entries(l);
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int j = j0 + u * N;
        if (j >= end) continue;
        float f[V];
#pragma unroll
        for (int e = 0; e < V; e++) f[e] = g.coef * __builtin_amdgcn_exp2f(fmaf(element<T>(v[u], e) - g.ref, a.c, -g.off));
        if (held >> u & 1) put_entries<V>(l, u, s.head, f);
        if (padding)
#pragma unroll
            for (int e = 0; e < V; e++) f[e] = 0.f;
        store_vector<T>(out, s, j, f, 0);
    }
    if (edge) {
        const int k = l.edge[tid];
        const float f = k >= 0 ? l.grad[k] : g.coef * __builtin_amdgcn_exp2f(fmaf(x - g.ref, a.c, -g.off));
        store1<T>(out + s.edge(tid), padding ? 0.f : f);
    }
}

// ------------------------------------------------------------------ loss and gradient, the row held

// One workgroup a row, NV vectors a thread in registers: the logits are read once.
template <typename T, int N, int NV>
__global__ void __launch_bounds__(N) k_distill_held(VocabLaunch a)
{
    typedef typename T::raw raw;
    constexpr int V = Vec16<T>::V;
    __shared__ float sums[48];
    __shared__ Entries<N> l;
    const RowAt row = row_at(a.r, a.row0 + blockIdx.x);
    const raw *p = (const raw *)a.logits + at(row, a.slogits);
    raw *out = (raw *)a.dlogits + at(row, a.sdlogits);
    const Span<T> s(out, a.r.cols);
    const int tid = threadIdx.x;
    const bool edge = tid < s.edges();
    u32x4 v[NV];
#pragma unroll
    for (int u = 0; u < NV; u++) {
        v[u] = u32x4{kNothing<T>, kNothing<T>, kNothing<T>, kNothing<T>};
        if (tid + u * N < s.nvec) v[u] = load_vector<T>(p, s, tid + u * N, 0);
    }
    float x = edge ? load1<T>(p + s.edge(tid)) : -kInf;
    clear(l);
    __syncthreads();
    if (tid < 64) read_entries<T>(l, a, row, p, s, 0, s.nvec, true);
    __syncthreads();
    if (l.live == 0) {
        padding_distill(a, row);
        const float zero[V] = {};
#pragma unroll
        for (int u = 0; u < NV; u++)
            if (tid + u * N < s.nvec) store_vector<T>(out, s, tid + u * N, zero);
        if (edge) store1<T>(out + s.edge(tid), 0.f);
        return;
    }
    const uint32_t held = trips_with_entries(l);
    const int on_edge = tid < kEdges ? l.edge[tid] : -1;
    if (a.with_tail) {
        // the entries are left out of the sums: their logits are held apart, and their gradients replace what becomes of these
#pragma unroll
        for (int u = 0; u < NV; u++)
            if (held >> u & 1) {
                float f[V];
#pragma unroll
                for (int e = 0; e < V; e++) f[e] = element<T>(v[u], e);
                for (int k = l.head[tid]; k >= 0; k = l.next[k]) {
                    if (l.trip[k] != u) continue;
                    const int at = (l.index[k] - s.head) % V;
#pragma unroll
                    for (int e = 0; e < V; e++) f[e] = e == at ? -kInf : f[e];
                }
                v[u] = pack16<T>(f);
            }
        if (on_edge >= 0) x = -kInf;
    }
    // the workgroup's largest, then the sums about it
    float most = x;
#pragma unroll
    for (int u = 0; u < NV; u++) {
        float f[V];
#pragma unroll
        for (int e = 0; e < V; e++) f[e] = element<T>(v[u], e);
        most = fmaxf(most, max_of<V>(f));
    }
    Sums sum;
    sum.peak = most;
    constexpr int W = N / 64;
    float peak = wave_max(most);
    if (W > 1) {
        if ((tid & 63) == 0) sums[tid >> 6] = peak;
        __syncthreads();
        peak = wave_max((tid & 63) < W ? sums[tid & 63] : -kInf);
    }
    const float ref = peak == -kInf ? 0.f : peak;
    float total = edge ? __builtin_amdgcn_exp2f((x - ref) * a.c) : 0.f;
#pragma unroll
    for (int u = 0; u < NV; u++)
#pragma unroll
        for (int e = 0; e < V; e++) total += __builtin_amdgcn_exp2f((element<T>(v[u], e) - ref) * a.c);
    total = group_sum<64>(total);
    if (W > 1) {
        if ((tid & 63) == 0) sums[16 + (tid >> 6)] = total;
        __syncthreads();
        total = group_sum<16>((tid & 63) < W ? sums[16 + (tid & 63)] : 0.f);
        total = __shfl(total, 0);
    }
    if (tid < 64) {
        sum.peak = peak; sum.s = total;
        Slope g;
        finish_distill(a, l, row, sum, true, g);
    }
    __syncthreads();
    const float from = l.gradient[0], off = l.gradient[1], coef = l.gradient[2];
#pragma unroll
    for (int u = 0; u < NV; u++) {
        const int j = tid + u * N;
        if (j >= s.nvec) continue;
        float f[V];
#pragma unroll
        for (int e = 0; e < V; e++) f[e] = coef * __builtin_amdgcn_exp2f(fmaf(element<T>(v[u], e) - from, a.c, -off));
        if (held >> u & 1) put_entries<V>(l, u, s.head, f);
        store_vector<T>(out, s, j, f, 0);
    }
    if (edge) store1<T>(out + s.edge(tid), on_edge >= 0 ? l.grad[on_edge] : coef * __builtin_amdgcn_exp2f(fmaf(x - from, a.c, -off)));
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

int vectors(const VocabLaunch &a) { return (a.r.cols + (a.dtype == EWF_F32 ? 4 : 8) - 1) / (a.dtype == EWF_F32 ? 4 : 8); }

template <typename T, int N, bool ENT, bool TOP, int KIND>
void run_rows(const VocabLaunch &a, hipStream_t stream)
{
    constexpr bool kLong = N > 64;
    by_rows(a, a.splits, N, [&](VocabLaunch b, dim3 grid, unsigned rows) {
        if (b.parts) b.parts += (int64_t)b.row0 * b.splits * 4;          // (all launches' parts are apart)
        if (b.pieces) b.pieces += (int64_t)b.row0 * b.splits * b.pieces_per_part;
        grid.x = std::min(grid.x, (unsigned)b.resident);
        if (kLong && b.stream) hipLaunchKernelGGL((k_rows<T, N, ENT, TOP && kLong, KIND, kLong>), grid, dim3(N), 0, stream, b);
        else hipLaunchKernelGGL((k_rows<T, N, ENT, TOP && kLong, KIND, false>), grid, dim3(N), 0, stream, b);
        constexpr int J = TOP && kLong ? 256 : 64;
        if (b.parts) hipLaunchKernelGGL((k_join<T, J, TOP, KIND>), dim3(rows), dim3(J), 0, stream, b);
    });
}

template <typename T, int N>
void run_kind(const VocabLaunch &a, hipStream_t stream)
{
    if (a.entries) {
        if (a.with_tail) run_rows<T, N, false, false, kDistillTail>(a, stream);
        else run_rows<T, N, false, false, kDistill>(a, stream);
    } else if (a.top) {
        if (a.entropy) run_rows<T, N, true, true, kLogprobs>(a, stream);
        else run_rows<T, N, false, true, kLogprobs>(a, stream);
    } else {
        if (a.entropy) run_rows<T, N, true, false, kLogprobs>(a, stream);
        else run_rows<T, N, false, false, kLogprobs>(a, stream);
    }
}

struct RunRows {
    const VocabLaunch &a;
    hipStream_t stream;
    template <typename T> void operator()() const
    {
        if (a.threads == 64) run_kind<T, 64>(a, stream);
        else run_kind<T, 256>(a, stream);
    }
};

constexpr int kLogprobsGradVectors = 4, kDistillGradVectors = 8;

struct RunLogprobsGrad {
    VocabLaunch a;
    hipStream_t stream;
    template <typename T> void operator()()
    {
        constexpr int U = kLogprobsGradVectors;
        const int pieces = std::max(1, (vectors(a) + U * kGradThreads - 1) / (U * kGradThreads));
        a.splits = pieces;
        by_rows(a, pieces, kGradThreads, [&](const VocabLaunch &b, dim3 grid, unsigned) {
            if (b.dentropy) hipLaunchKernelGGL((k_logprobs_grad<T, true, U>), grid, dim3(kGradThreads), 0, stream, b);
            else hipLaunchKernelGGL((k_logprobs_grad<T, false, U>), grid, dim3(kGradThreads), 0, stream, b);
        });
    }
};

struct RunDistillGrad {
    VocabLaunch a;
    hipStream_t stream;
    template <typename T> void operator()()
    {
        constexpr int U = kDistillGradVectors;
        const int pieces = std::max(1, (vectors(a) + U * kGradThreads - 1) / (U * kGradThreads));
        a.splits = pieces;
        by_rows(a, pieces, kGradThreads, [&](const VocabLaunch &b, dim3 grid, unsigned) {
            hipLaunchKernelGGL((k_distill_grad<T, U>), grid, dim3(kGradThreads), 0, stream, b);
        });
    }
};

struct RunHeld {
    const VocabLaunch &a;
    hipStream_t stream;
    template <typename T, int N, int NV> void go() const
    {
        by_rows(a, 1, N, [&](const VocabLaunch &b, dim3 grid, unsigned) {
            hipLaunchKernelGGL((k_distill_held<T, N, NV>), grid, dim3(N), 0, stream, b);
        });
    }
    template <typename T> void operator()() const
    {
        const int n = vectors(a);
        if (n <= 64) go<T, 64, 1>();
        else if (n <= 128) go<T, 64, 2>();
        else if (n <= 256) go<T, 64, 4>();
        else if (n <= 512) go<T, 256, 2>();
        else if (n <= 1024) go<T, 256, 4>();
        else if (n <= 2048) go<T, 256, 8>();
        else if (n <= 4096) go<T, 1024, 4>();
        else if (n <= 8192) go<T, 1024, 8>();
        else if (n <= 12288) go<T, 1024, 12>();
        else go<T, 1024, 16>();
    }
};

}  // namespace

void plan_vocab(VocabLaunch &a, int units)
{
    const int n = vectors(a);
    a.held = a.entries && a.dlogits && n <= kHeldVectors;
    a.threads = n <= 256 ? 64 : 256;
    // few rows are shared by workgroups that take 1024 vectors at least, where a second launch costs less than what it saves: one row of 131072 float32
    // takes 20 us whole, 7.7 in 32 parts; eight rows of 50257 bfloat16 8.1 us whole (and 8.1 in 6 parts), with 20 alternatives, which need the
    // second launch anyway, 17.3 and 12.2
    a.splits = 1;
    if (a.r.rows < (uint32_t)units && n >= (a.top ? 2048 : 12288))
        a.splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(64, n / 1024), (2 * units + a.r.rows - 1) / a.r.rows));
    // (the largest a row can have: its vectors begin at its first whole 16 bytes)
    if (a.top && a.threads == 256) a.pieces_per_part = ((n + a.splits - 1) / a.splits + kPieceTrips * 256 - 1) / (kPieceTrips * 256) * (256 / kPieceLanes);
    // workgroups that stay: as many as share the rows evenly
    const int64_t room = (int64_t)units * 2048 / a.threads, items = (int64_t)a.r.rows * a.splits, each = (items + room - 1) / room;
    a.resident = each ? (int)((items + each - 1) / each) : 0;
    // logits that the memory-side cache cannot keep pass it by: bfloat16 [4096, 32768] 51.7 us, passing 45.6; [2048, 32768] 27.2 and 24.7; [1024, 32768] 14.3 and 15.7
    a.stream = (int64_t)a.r.rows * a.r.cols * (a.dtype == EWF_F32 ? 4 : 2) >= (int64_t)128 << 20;
}

void launch_token_logprobs(const VocabLaunch &a, hipStream_t stream) { by_type(a.dtype, RunRows{a, stream}); }
void launch_token_logprobs_grad(const VocabLaunch &a, hipStream_t stream) { by_type(a.dtype, RunLogprobsGrad{a, stream}); }
void launch_distill_grad(const VocabLaunch &a, hipStream_t stream) { by_type(a.dtype, RunDistillGrad{a, stream}); }
void launch_distill(const VocabLaunch &a, hipStream_t stream)
{
    if (a.held) return by_type(a.dtype, RunHeld{a, stream});
    by_type(a.dtype, RunRows{a, stream});
    if (a.dlogits) launch_distill_grad(a, stream);
}

}  // namespace ewf
