// The sums of rows of logits: one kernel for log probabilities and for a teacher's entries.
#pragma once

#include "ewf_vocab_entries.h"
#include "ewf_vocab_top.h"

namespace ewf {

namespace {

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

enum { kLogprobs = 0, kDistill = 1, kDistillTail = 2 };

// The sums of a row that cannot be taken about a whole number of powers of two (see beyond): about its largest logit, element by element; with a
// `tail` of what no entry names, which is looked for among all entries at each logit: right, and slow.  Losses and gradients of bfloat16 [2048, 131072] against 64 entries
// take 3.7 ms where all that no entry names is -1e30, and 7.7 where all logits are beyond 2^22 and the gradients look for them too, for 210 us.
template <typename T, int N, typename S, typename L>
EWF_OPS_DEV void sum_again(const VocabLaunch &a, const typename T::raw *p, const S &s, int j0, int j1, bool edges, bool tail, const L &entries, float *lds,
                           Sums &sum)
{
    constexpr int V = Vec16<T>::V;
    const int tid = threadIdx.x, end = s.head + j1 * V;
    float total = 0.f, weighted = 0.f;
    for (int c = s.head + j0 * V + tid; c < end + (edges ? s.edges() : 0); c += N) {
        const int at = c < end ? c : s.edge(c - end);
        float x = load1<T>(p + at);
        if constexpr (!std::is_same<L, int>::value)
            if (tail)
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

// A workgroup takes rows, or parts of rows (a.splits of each), one after the other; a vector's registers take the next vector as soon as it is summed, the
// last ones the next row's first, which are in flight while this row is finished.
//
// Memory bounds it: bfloat16 [2048, 131072] 84 us (6.4 TB/s), [4096, 50257] 68 to 72 (6.0), float32 [1280, 10000] 11.1, with 7 vector instructions a logit of
// which one is the exponential.  On the way (bfloat16 [4096, 50257]): a row a workgroup, sums about a logit 79.7; loads past the caches 75.7; the largest
// of three by one instruction, and vectors taken in turn rather than copied from a second set, 71.7.  Six or eight vectors in flight: 68 and 70 there,
// but float32 [1280, 10000] 11.6 and 12.1; half as many workgroups 73.1 and 13.6.  Rows that begin on cache lines: no change.
// Where rows have parts or alternatives are asked for it leaves sums and, TOP, the largest of their pieces in the workspace.
template <typename T, int N, bool ENT, bool TOP, int KIND, int K, bool STREAM>
__global__ void __launch_bounds__(N) k_rows(VocabLaunch a)
{
    typedef typename T::raw raw;
    constexpr int V = Vec16<T>::V, U = kPieceTrips;
    __shared__ float sums[48];
    __shared__ typename std::conditional<KIND != kLogprobs, Entries<N, K>, int>::type entries;
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
                if (tid < 64) take_entries<T>(entries, a, row, p, s, j0, j1, edges);
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
                    each_entry<V>(entries, trip, s.head, [&](int at, int) {
#pragma unroll
                        for (int e = 0; e < V; e++) x[e] = e == at ? -kInf : x[e];
                    });
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
            if (beyond(sum.peak, a.c)) sum_again<T, N>(a, p, s, j0, j1, edges, KIND == kDistillTail, entries, sums, sum);
            if (parts) {
                if (tid == 0) {
                    float *out = a.parts + (int64_t)t.part * 4;
                    out[0] = sum.peak; out[1] = sum.s; out[2] = sum.w;
                }
            } else if constexpr (KIND == kLogprobs) {
                finish_logprobs<N>(a, row, sum, token_logit, nullptr, 0);
            } else if (tid < 64) {
                const Stats r = stats_of(a, entries, sum);
                finish_distill(a, entries, row, r);
                if (a.prepared) prepare_gradients(a, entries, row, r, prepared_row(a, t.part));
            }
        } else if (!parts) {
            padding_distill(a, row, tid);
            if (a.prepared && tid == 0) prepared_row(a, t.part)->padding = 1;
        }
        if (N > 64 || KIND != kLogprobs) __syncthreads();          // (LDS is the next item's)
        i = ni;
        t = nt;
        more = nmore;
    }
}

// Joins the parts of a row, and finds its alternatives: 2048 rows of 131072 bfloat16 with 64 of them in 23 to 27 us (84 MB of pieces' lines read again), one row in 6 to 8,
// a chain of loads that wait for each other (parts, pieces, the chosen pieces, their vectors).  Within the first kernel the choice took 80 us more there than sums alone:
// its registers leave one workgroup a compute unit, which loads nothing meanwhile.
template <typename T, int N, bool TOP, int KIND, int K>
__global__ void __launch_bounds__(N, TOP && N > 64 ? 8 : 1) k_join(VocabLaunch a)
{
    typedef typename T::raw raw;
    __shared__ typename std::conditional<KIND != kLogprobs, Entries<N, K>, int>::type entries;
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
        if (tid < 64) take_entries<T>(entries, a, row, p, s, 0, 0, false);
        __syncthreads();
        if (entries.live == 0) {
            padding_distill(a, row, tid);
            if (a.prepared && tid == 0) prepared_row(a, blockIdx.x)->padding = 1;
            return;
        }
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
        const Stats r = stats_of(a, entries, sum);
        finish_distill(a, entries, row, r);
        if (a.prepared) prepare_gradients(a, entries, row, r, prepared_row(a, blockIdx.x));
    }
}

template <typename T, int N, bool ENT, bool TOP, int KIND, int K = 0>
void run_rows(const VocabLaunch &a, hipStream_t stream)
{
    constexpr bool kLong = N > 64;
    by_rows(a, a.splits, N, [&](VocabLaunch b, dim3 grid, unsigned rows) {
        if (b.parts) b.parts += (int64_t)b.row0 * b.splits * 4;          // (all launches' parts are apart)
        if (b.pieces) b.pieces += (int64_t)b.row0 * b.splits * b.pieces_per_part;
        if (b.prepared) b.prepared = (char *)b.prepared + b.row0 * prepared_bytes(b.entries);
        grid.x = std::min(grid.x, (unsigned)b.resident);
        if (kLong && b.stream) hipLaunchKernelGGL((k_rows<T, N, ENT, TOP && kLong, KIND, K, kLong>), grid, dim3(N), 0, stream, b);
        else hipLaunchKernelGGL((k_rows<T, N, ENT, TOP && kLong, KIND, K, false>), grid, dim3(N), 0, stream, b);
        constexpr int J = TOP && kLong ? 256 : 64;
        if (b.parts) hipLaunchKernelGGL((k_join<T, J, TOP, KIND, K>), dim3(rows), dim3(J), 0, stream, b);
    });
}

}  // namespace

}  // namespace ewf
