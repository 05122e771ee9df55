// A teacher's entries of a row, and what a loss against them makes of the row's sums.
#pragma once

#include <cstddef>

#include "ewf_vocab_device.h"

namespace ewf {

namespace {

// The entries of a row in LDS.  An entry inside the row's vectors is in the list of the thread that takes its vector (thread = vector mod N),
// one on an edge in the list of that edge's thread, with no trip.  K, 64 or 128, is what a row can have: with 64 of them a lane has one, and LDS lets more
// workgroups share a compute unit (bfloat16 [16384, 1000], 20 entries: 35 us, with room for 128 always 39).
template <int N, int K>
struct Entries {
    int head[N];                                        // last entry of each thread's list, -1
    int next[K], index[K], trip[K];
    float q[K], logq[K], logit[K];
    float all[K];                                       // of all entries with the same index
    int edge[kEdges];                                   // an entry on each edge element, -1
    float tail_q, total_q;                              // 1 - sum q; sum q
    float peak, sum;                                    // of the logits that they name: the largest, the sum about it
    int live;                                           // entries that exist
};

EWF_OPS_DEV float load_teacher(const VocabLaunch &a, int64_t at)
{
    if (a.teacher_dtype == EWF_F32) return ((const float *)a.teacher_values)[at];
    const uint32_t h = ((const uint16_t *)a.teacher_values)[at];
    return a.teacher_dtype == EWF_BF16 ? half_lo<BF16>(h) : half_lo<F16>(h);
}

// LDS that one wavefront writes and reads itself.
EWF_OPS_DEV void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// A wavefront reads a row's entries, one or two a lane: indices and values, then the logits that they name ...
template <int K>
struct RawEntries { int c[K / 64]; float v[K / 64], x[K / 64]; };

template <int K>
EWF_OPS_DEV void read_entries(RawEntries<K> &r, const VocabLaunch &a, const RowAt &row)
{
    const int64_t values = at(row, a.steacher_values), indices = at(row, a.steacher_indices);
#pragma unroll
    for (int h = 0; h < K / 64; h++) {
        const int i = h * 64 + (threadIdx.x & 63);
        r.c[h] = i < a.entries ? a.teacher_indices[indices + i] : -1;
        r.v[h] = i < a.entries ? load_teacher(a, values + i) : 0.f;
    }
}

template <typename T, int K>
EWF_OPS_DEV void read_logits(RawEntries<K> &r, const VocabLaunch &a, const typename T::raw *logits)
{
#pragma unroll
    for (int h = 0; h < K / 64; h++) r.x[h] = (uint32_t)r.c[h] < (uint32_t)a.r.cols ? load1<T>(logits + r.c[h]) : 0.f;
}

// q = e^(v - m), their sum
template <int H>
EWF_OPS_DEV float exponentials(const float *v, float m, float *q)
{
    float sum = 0.f;
#pragma unroll
    for (int h = 0; h < H; h++) sum += q[h] = expf(v[h] - m);
    return sum;
}

// ... and ranks them; the others see them behind a barrier.  The vectors of this workgroup are j0 .. j1 - 1 (thread (j - j0) mod N takes vector j);
// `edges`: and the edges.
template <typename T, int N, int K, typename S>
EWF_OPS_DEV void rank_entries(Entries<N, K> &l, const RawEntries<K> &r, const VocabLaunch &a, const S &s, int j0, int j1, bool edges)
{
    constexpr int V = Vec16<T>::V;
    constexpr int H = K / 64;
    const int lane = threadIdx.x & 63;
    const int *c = r.c;
    const float *x = r.x;
    float v[H];
    bool live[H];
    int some = 0;
    for (int i = lane; i < N; i += 64) l.head[i] = -1;
    for (int i = lane; i < kEdges; i += 64) l.edge[i] = -1;
#pragma unroll
    for (int h = 0; h < H; h++) {
        live[h] = (uint32_t)c[h] < (uint32_t)s.cols;
        v[h] = live[h] ? r.v[h] * a.teacher_scale : -kInf;
        some += __popcll(__ballot(live[h]));
    }
    float q[H], tail = 0.f, total;
    if (a.with_tail) {
        total = group_sum<64>(exponentials<H>(v, 0.f, q));
        tail = fmaxf(1.f - total, 0.f);
        if (!(total < kInf)) tail = total - total;      // (a NaN stays one)
    } else {
        const float top = wave_max(fmaxf(v[0], v[H - 1])), m = top == -kInf ? 0.f : top;
        const float sum = group_sum<64>(exponentials<H>(v, m, q)), log_sum = logf(sum);
#pragma unroll
        for (int h = 0; h < H; h++) {
            q[h] = sum == 0.f ? 0.f : q[h] / sum;
            v[h] = v[h] - m - log_sum;
        }
        total = sum == 0.f ? 0.f : sum < kInf ? 1.f : sum - sum;
    }
    if (lane == 0) { l.tail_q = tail; l.total_q = total; l.live = some; }
    wave_fence();
    int owner[H];
#pragma unroll
    for (int h = 0; h < H; h++) {
        const int i = h * 64 + lane;
        l.index[i] = live[h] ? c[h] : -1;
        l.q[i] = live[h] ? q[h] : 0.f;
        l.logq[i] = v[h];
        l.logit[i] = x[h];
        owner[h] = 0;
        if (!live[h]) continue;
        const int j = s.inside(c[h]) ? (c[h] - s.head) / V : -1;
        int trip = -1;
        if (j < 0) {
            const int e = s.edge_of(c[h]);
            owner[h] = (uint32_t)e % N;
            if (edges) l.edge[e] = i;                   // (of several that are the same one, any: they have the same gradient)
        } else {
            owner[h] = (uint32_t)j % N;
            if (j >= j0 && j < j1) { owner[h] = (j - j0) % N; trip = (j - j0) / N; }
        }
        l.trip[i] = trip;
        l.next[i] = atomicExch(&l.head[owner[h]], i);
    }
    wave_fence();
    // entries of the same index are in the same list; their probabilities are added in the entries' order
    bool first[H];
#pragma unroll
    for (int h = 0; h < H; h++) {
        const int i = h * 64 + lane;
        bool again = false;
        first[h] = live[h];
        for (int k = live[h] ? l.head[owner[h]] : -1; k >= 0; k = l.next[k]) {
            if (k == i || l.index[k] != c[h]) continue;
            again = true;
            first[h] = first[h] && k > i;
        }
        float all = live[h] ? q[h] : 0.f;
        if (again) {
            all = 0.f;
            for (int k = 0; k < a.entries; k++) all += l.index[k] == c[h] ? l.q[k] : 0.f;
        }
        l.all[i] = all;
    }
    const float peak = wave_max(fmaxf(first[0] ? x[0] : -kInf, first[H - 1] ? x[H - 1] : -kInf)), ref = peak == -kInf ? 0.f : peak;
    float e = 0.f;
#pragma unroll
    for (int h = 0; h < H; h++) e += first[h] ? __builtin_amdgcn_exp2f((x[h] - ref) * a.c) : 0.f;
    e = group_sum<64>(e);
    if (lane == 0) { l.peak = peak; l.sum = e; }
}

template <typename T, int N, int K, typename S>
EWF_OPS_DEV void take_entries(Entries<N, K> &l, const VocabLaunch &a, const RowAt &row, const typename T::raw *logits, const S &s, int j0, int j1, bool edges)
{
    RawEntries<K> r;
    read_entries(r, a, row);
    read_logits<T>(r, a, logits);
    rank_entries<T>(l, r, a, s, j0, j1, edges);
}

EWF_OPS_DEV bool tail_counts(float tail, float logsum) { return tail - logsum >= -126.f * kLn2; }

// A row's statistics from its sums: of all logits, or with a tail of those that no entry names.
struct Stats { float peak, logsum, tail; };

template <int N, int K>
EWF_OPS_DEV Stats stats_of(const VocabLaunch &a, const Entries<N, K> &l, const Sums &sum)
{
    Stats r = {sum.peak, 0.f, -kInf};
    float total = sum.s;
    if (a.with_tail) {
        r.peak = fmaxf(sum.peak, l.peak);
        const float ref = r.peak == -kInf ? 0.f : r.peak;
        if (sum.s != 0.f) r.tail = fmaf(sum.peak - ref, a.scale, logf(sum.s));
        total = (sum.peak == -kInf ? sum.s : sum.s * __builtin_amdgcn_exp2f((sum.peak - ref) * a.c)) +
                (l.peak == -kInf ? l.sum : l.sum * __builtin_amdgcn_exp2f((l.peak - ref) * a.c));
    }
    r.logsum = total == 0.f ? -kInf : logf(total);
    if (!(total < kInf)) r.peak = r.logsum = r.tail = __builtin_nanf("");       // a NaN or an infinity among the logits
    return r;
}

// Writes the loss and the statistics: one wavefront.
template <int N, int K>
EWF_OPS_DEV void finish_distill(const VocabLaunch &a, const Entries<N, K> &l, const RowAt &row, const Stats &r)
{
    const int lane = threadIdx.x & 63;
    const bool none = r.logsum == -kInf;
    float loss = 0.f;
#pragma unroll
    for (int h = 0; h < K / 64; h++) {
        const int i = h * 64 + lane;
        const float q = l.q[i], logp = none ? -kInf : fmaf(l.logit[i] - r.peak, a.scale, -r.logsum);
        if (l.index[i] >= 0 && q != 0.f) loss += q * (l.logq[i] - logp);
    }
    loss = group_sum<64>(loss);
    const float tail_q = l.tail_q;
    if (a.with_tail && tail_q != 0.f && (tail_counts(r.tail, r.logsum) || tail_q != tail_q)) loss += tail_q * (logf(tail_q) - (r.tail - r.logsum));
    if (lane == 0) {
        if (a.loss) a.loss[at(row, a.sloss)] = r.peak == r.peak ? loss : r.peak;
        if (a.peak) a.peak[at(row, a.speak)] = r.peak;
        if (a.logsum) a.logsum[at(row, a.slogsum)] = r.logsum;
        if (a.tail) a.tail[at(row, a.stail)] = r.tail;
    }
}

EWF_OPS_DEV void padding_distill(const VocabLaunch &a, const RowAt &row, int thread)
{
    if (thread) return;
    if (a.loss) a.loss[at(row, a.sloss)] = 0.f;
    if (a.peak) a.peak[at(row, a.speak)] = 0.f;
    if (a.logsum) a.logsum[at(row, a.slogsum)] = 0.f;
    if (a.tail) a.tail[at(row, a.stail)] = 0.f;
}

// The gradients of a row: of a logit that no entry names, coef 2^t, t as `rest` has it without its own rest; of an entry, factor (mass p - q).
struct Slope {
    Exponent rest, p;
    float coef, mass, factor;
    EWF_OPS_DEV Slope() {}
    template <int N, int K>
    EWF_OPS_DEV Slope(const VocabLaunch &a, const Entries<N, K> &l, const Stats &r, float weight)
        : rest(ref(r), off(a, l, r) * kLog2E, a.c), p(ref(r), r.peak == -kInf ? 0.f : r.logsum * kLog2E, a.c)
    {
        factor = scalar(weight * a.scale);
        mass = scalar(l.total_q);
        coef = factor * mass;
        if (with_rest(a, l, r)) {
            // m p - q_t p / p_t, as p / p_t (m p_t - q_t): the first is at most 1
            mass = scalar(mass + l.tail_q);
            coef = factor * fmaf(mass, expf(r.tail - r.logsum), -l.tail_q);
        }
        coef = scalar(r.peak == -kInf ? 0.f : coef * __builtin_amdgcn_exp2f(rest.rest));        // (a student without a logit: p = 0)
    }
    template <int N, int K>
    EWF_OPS_DEV float entry(const Entries<N, K> &l, int k) const
    {
        float t;
        p.of<1>(&l.logit[k], &t);
        return factor * fmaf(mass, __builtin_amdgcn_exp2f(t + p.rest), -l.all[k]);
    }
private:
    static EWF_OPS_DEV float ref(const Stats &r) { return r.peak == -kInf ? 0.f : r.peak; }
    template <int N, int K>
    static EWF_OPS_DEV bool with_rest(const VocabLaunch &a, const Entries<N, K> &l, const Stats &r)
    {
        return a.with_tail && tail_counts(r.tail, r.logsum) && l.tail_q > 0.f;
    }
    template <int N, int K>
    static EWF_OPS_DEV float off(const VocabLaunch &a, const Entries<N, K> &l, const Stats &r)
    {
        return r.peak == -kInf ? 0.f : with_rest(a, l, r) ? r.tail : r.logsum;
    }
};

// What a row's gradients need, in the workspace: of 32 bytes, then the entries.
struct Prepared {
    struct Entry { int index; float grad; };
    float ref, off, coef;
    int padding, unused[4];
    Entry entry[1];
    EWF_OPS_DEV Exponent exponent(float c) const { return Exponent(ref, off, c); }
};
static_assert(offsetof(Prepared, entry) == kPreparedBytes && sizeof(Prepared::Entry) == kPreparedEntryBytes, "");
inline __host__ __device__ size_t prepared_bytes(int entries) { return kPreparedBytes + (size_t)entries * kPreparedEntryBytes; }

EWF_OPS_DEV Prepared *prepared_row(const VocabLaunch &a, uint32_t in_launch) { return (Prepared *)((char *)a.prepared + in_launch * prepared_bytes(a.entries)); }

// One wavefront; the same gradient stands at each entry of an index.
template <int N, int K>
EWF_OPS_DEV void prepare_gradients(const VocabLaunch &a, const Entries<N, K> &l, const RowAt &row, const Stats &r, Prepared *to)
{
    const Slope g(a, l, r, a.dloss ? a.dloss[at(row, a.sdloss)] : 1.f);
    const int lane = threadIdx.x & 63;
    if (lane == 0) {
        to->ref = g.rest.ref;
        to->off = g.rest.off;
        to->coef = g.coef;
        to->padding = l.live == 0;
    }
    for (int i = lane; i < a.entries; i += 64) to->entry[i] = {l.index[i], l.index[i] >= 0 ? g.entry(l, i) : 0.f};
}

// The trips of this thread that hold entries, as bits.
template <int N, int K>
EWF_OPS_DEV uint32_t trips_with_entries(const Entries<N, K> &l)
{
    uint32_t m = 0;
    for (int k = l.head[threadIdx.x]; k >= 0; k = l.next[k])
        if (l.trip[k] >= 0) m |= 1u << l.trip[k];
    return m;
}

// Calls to(e, k) for the elements e of this thread's vector of a trip that entries k name.
template <int V, int N, int K, typename F>
EWF_OPS_DEV void each_entry(const Entries<N, K> &l, int trip, int head, F &&to)
{
    for (int k = l.head[threadIdx.x]; k >= 0; k = l.next[k])
        if (l.trip[k] == trip) to((l.index[k] - head) % V, k);
}

}  // namespace

}  // namespace ewf
