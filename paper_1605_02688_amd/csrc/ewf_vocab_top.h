// The largest logits of a row, in a fixed order.
#pragma once

#include "ewf_vocab_device.h"

namespace ewf {

namespace {

// Floats in their order as whole numbers, -0 as +0.  A key is this over the complement of a place, so that keys are ranked by value and,
// among equals, by the lowest place; 0 is no key (minus infinity is none either).
EWF_OPS_DEV uint32_t ordered(float x)
{
    const uint32_t b = float_to_bits(x + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
EWF_OPS_DEV float unordered(uint32_t k) { return bits_to_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
EWF_OPS_DEV u64 key_of(float x, uint32_t at) { return x > -kInf ? (u64)ordered(x) << 32 | (uint32_t)~at : 0; }

// The largest logits of pieces of a row: a piece is what kPieceLanes lanes (a cache line) take in kPieceTrips trips.  Threads' own largest in
// their place name vectors that lie in lines of their own, which brings nearly all of a row back: [2048, 131072] with 64 alternatives 190 us, 117 so.
constexpr int kPieceLanes = 8, kPieceTrips = 4;
constexpr int kCandidates = 512;         // logits that a row's last selection ranks
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
            each_piece([&](float x, int i) { if (x > -kInf && x >= floor) l.chosen[atomicAdd(&l.nchosen, 1)] = i; });        // (l.upto of them)
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

}  // namespace

}  // namespace ewf
