// Operators over rows of logits: log probabilities of given tokens with entropy and the largest alternatives, the loss against a
// teacher's top logits, and the gradients of both.
//
// A row's statistics are kept about a point m that lags behind the largest logit seen: with t = c (x - m) in powers of two (c = scale log2 e) a
// thread adds e = 2^t and, for the entropy, e t; it moves m only where a logit is 2^8 beyond it, so that the moves are rare and e cannot
// overflow.  Threads' sums are then moved to the row's largest logit and added in a fixed order.
#include <algorithm>
#include <type_traits>

#include "ewf_ops_device.h"

namespace ewf {

namespace {

typedef unsigned long long u64;

constexpr float kLn2 = 0.693147181f;
constexpr float kInf = __builtin_huge_valf();
constexpr float kLowest = -3.40282347e38f;
constexpr float kFloor = -1e4f;          // powers of two below which nothing is left; products with it stay finite
constexpr int kCandidates = 1024;        // alternatives that a row's last selection ranks

template <typename T> constexpr uint32_t kNothing = 0xff80ff80u;        // a word of minus infinities
template <> constexpr uint32_t kNothing<F16> = 0xfc00fc00u;
template <> constexpr uint32_t kNothing<F32> = 0xff800000u;

// A row on the 16-byte grid of `grid` (the address that decides: the results' where there are any): whole vectors from element `head` on,
// and at most 2 V - 2 elements on its two edges.
template <typename T>
struct Span {
    static constexpr int V = Vec16<T>::V;
    int cols, head, nvec;
    EWF_OPS_DEV Span(const void *grid, int cols) : cols(cols)
    {
        const int over = (int)((uintptr_t)grid & 15) / (int)sizeof(typename T::raw);
        head = over ? V - over : 0;
        head = head < cols ? head : cols;
        nvec = (cols - head) / V;
    }
    EWF_OPS_DEV int edges() const { return cols - nvec * V; }
    EWF_OPS_DEV int edge(int i) const { return i < head ? i : i + nvec * V; }
    EWF_OPS_DEV int edge_of(int c) const { return c < head ? c : c - nvec * V; }       // (an element that is on one)
    EWF_OPS_DEV bool inside(int c) const { return c >= head && c < head + nvec * V; }
};

EWF_OPS_DEV float wave_max(float x)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

// Sums of a thread, a workgroup or a row.  e's sum s and e t's sum w are about m; peak is the largest logit.
struct Sums {
    float m = kLowest, s = 0.f, w = 0.f, peak = -kInf;
};

// Moves upwards (sums of nothing move anywhere).
template <bool ENT>
EWF_OPS_DEV void move_to(Sums &a, float m, float c)
{
    const float d = __builtin_amdgcn_fmed3f((a.m - m) * c, kFloor, 0.f), r = __builtin_amdgcn_exp2f(d);
    if (ENT) a.w = r * fmaf(a.s, d, a.w);
    a.s *= r;
    a.m = m;
}

// Adds n logits whose largest is `top`.
template <bool ENT, int n>
EWF_OPS_DEV void add(Sums &a, const float *x, float top, float c, float lag)
{
    a.peak = fmaxf(a.peak, top);
    if (__any(top > a.m + lag)) move_to<ENT>(a, fmaxf(a.m, top), c);
#pragma unroll
    for (int e = 0; e < n; e++) {
        const float t = (x[e] - a.m) * c, p = __builtin_amdgcn_exp2f(t);
        a.s += p;
        if (ENT) a.w = fmaf(p, fmaxf(t, kFloor), a.w);
    }
}

template <int V>
EWF_OPS_DEV float max_of(const float *x)
{
    float m = x[0];
#pragma unroll
    for (int e = 1; e < V; e++) m = fmaxf(m, x[e]);
    return m;
}

// The sums of N threads, in every thread, about the row's largest logit (0 where that is minus infinity).
template <int N, bool ENT>
EWF_OPS_DEV Sums workgroup_sums(Sums a, float c, float *lds)        // lds: 3 * 16 words
{
    constexpr int W = N / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float peak = wave_max(a.peak);
    if (W > 1) {
        if (lane == 0) lds[wave] = peak;
        __syncthreads();
        peak = wave_max(lane < W ? lds[lane] : -kInf);
    }
    move_to<ENT>(a, peak == -kInf ? 0.f : peak, c);
    a.s = group_sum<64>(a.s);
    if (ENT) a.w = group_sum<64>(a.w);
    if (W > 1) {
        if (lane == 0) { lds[16 + wave] = a.s; if (ENT) lds[32 + wave] = a.w; }
        __syncthreads();
        a.s = group_sum<16>(lane < W ? lds[16 + lane] : 0.f);
        a.s = __shfl(a.s, 0);
        if (ENT) { a.w = group_sum<16>(lane < W ? lds[32 + lane] : 0.f); a.w = __shfl(a.w, 0); }
    }
    a.peak = peak;
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

// The bound that exactly k of n keys (different ones; n at most 64 R) reach, or 1 where there are no more than k.  One wavefront.
// Bits from the top, values first, until the count is met: one look at all keys each.
template <int R>
EWF_OPS_DEV u64 kth_largest(const u64 *keys, int n, int k)
{
    const int lane = threadIdx.x & 63;
    uint32_t hi[R], lo[R];
    int some = 0;
#pragma unroll
    for (int r = 0; r < R; r++) {
        const u64 v = r * 64 + lane < n ? keys[r * 64 + lane] : 0;
        hi[r] = (uint32_t)(v >> 32);
        lo[r] = (uint32_t)v;
        some += __popcll(__ballot(hi[r] != 0));
    }
    if (some <= k) return 1;
    uint32_t at = 0;
    for (int bit = 31; bit >= 0; bit--) {
        const uint32_t next = at | 1u << bit;
        int count = 0;
#pragma unroll
        for (int r = 0; r < R; r++) count += __popcll(__ballot(hi[r] >= next));
        if (count >= k) at = next;
        if (count == k) return (u64)at << 32;
    }
    int over = 0;
#pragma unroll
    for (int r = 0; r < R; r++) over += __popcll(__ballot(hi[r] > at));
    uint32_t low = 0;
    for (int bit = 31; bit >= 0; bit--) {
        const uint32_t next = low | 1u << bit;
        int count = over;
#pragma unroll
        for (int r = 0; r < R; r++) count += __popcll(__ballot(hi[r] == at && lo[r] >= next));
        if (count >= k) low = next;
        if (count == k) break;
    }
    return (u64)at << 32 | low;
}

struct Best {
    float value = -kInf;
    int vec = 0;
};

template <int N>
struct TopLds {
    u64 keys[N], found[kCandidates], bound;
    int chosen[N], nchosen, nfound, count[2];
};

// Writes the k largest logits of the vectors j0 .. j1 - 1 of a row and of its edges (where `edges`) to found[], as keys in descending order,
// and 0 behind the last.  best: of each thread, the largest logit of its vectors j0 + thread, + N ... and the first vector that has it.
//
// The k largest lie in the k threads whose best are largest: each other thread's elements have k larger ones before them.  Those
// threads' vectors are read a second time, by all threads, and what reaches the k-th best is collected.
template <typename T, int N>
EWF_OPS_DEV void largest(TopLds<N> &l, const typename T::raw *row, const Span<T> &s, int j0, int j1, bool edges, float edge, const Best &best, int k)
{
    constexpr int V = Vec16<T>::V, U = 4;
    const int tid = threadIdx.x;
    const u64 mine = key_of(best.value, best.vec);
    l.keys[tid] = mine;
    if (tid == 0) l.nchosen = l.nfound = 0;
    __syncthreads();
    if (tid < 64) {
        const u64 b = kth_largest<N / 64>(l.keys, N, k);
        if (tid == 0) l.bound = b;
    }
    __syncthreads();
    const u64 bound = l.bound;
    // the same bound for elements: the last of the vector that it names
    u64 least = bound;
    if ((uint32_t)bound > 1) {
        const u64 last = (u64)(uint32_t)~(uint32_t)bound * V + V - 1 + s.head;
        least = (bound & 0xffffffff00000000ull) | (uint32_t)~(uint32_t)(last < 0xffffffffu ? last : 0xffffffffu);
    }
    auto collect = [&](float x, int at) {
        const u64 key = key_of(x, at);
        if (key >= least && key) {
            const int i = atomicAdd(&l.nfound, 1);
            if (i < kCandidates) l.found[i] = key;
        }
    };
    if (mine >= bound && mine) l.chosen[atomicAdd(&l.nchosen, 1)] = tid;
    if (edges && tid < s.edges()) collect(edge, s.edge(tid));
    __syncthreads();
    const int nchosen = l.nchosen, trips = (j1 - j0 + N - 1) / N, items = nchosen * trips;
    auto sweep = [&](auto &&each) {
        for (int i0 = tid; i0 < items; i0 += U * N) {
            u32x4 v[U];
            int j[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int i = i0 + u * N;
                j[u] = i < items ? j0 + (i / nchosen) * N + l.chosen[i % nchosen] : j1;
                v[u] = u32x4{kNothing<T>, kNothing<T>, kNothing<T>, kNothing<T>};
                if (j[u] < j1) v[u] = load16<T>(row + s.head + (int64_t)j[u] * V);
            }
#pragma unroll
            for (int u = 0; u < U; u++)
#pragma unroll
                for (int e = 0; e < V; e++) each(element<T>(v[u], e), s.head + j[u] * V + e);
        }
    };
    sweep(collect);
    __syncthreads();
    int n = l.nfound;
    if (n > kCandidates) {
        // (more than fit, as where logits repeat with the threads' period: the k-th key bit by bit, a sweep for each)
        u64 at = 0;
        for (int bit = 63; bit >= 0; bit--) {
            const u64 next = at | 1ull << bit;
            int count = 0;
            auto ask = [&](float x, int p) { const u64 key = key_of(x, p); count += key >= next && key ? 1 : 0; };
            sweep(ask);
            if (edges && tid < s.edges()) ask(edge, s.edge(tid));
            if (tid == 0) l.count[bit & 1] = 0;
            __syncthreads();
            if (count) atomicAdd(&l.count[bit & 1], count);
            __syncthreads();
            if (l.count[bit & 1] >= k) at = next;
        }
        if (tid == 0) l.nfound = 0;
        least = at;
        __syncthreads();
        if (edges && tid < s.edges()) collect(edge, s.edge(tid));
        sweep(collect);
        __syncthreads();
        n = l.nfound;
    }
    if (n > 2 * k + 64) {
        // ranking takes n looks a key: fewer keys first
        if (tid < 64) {
            const u64 b = kth_largest<kCandidates / 64>(l.found, n, k);
            if (tid == 0) { l.bound = b; l.nchosen = 0; }
        }
        __syncthreads();
        u64 keep[kCandidates / N > 0 ? kCandidates / N : 1];
#pragma unroll
        for (int i = 0; i < (int)(sizeof(keep) / sizeof(u64)); i++) keep[i] = i * N + tid < n ? l.found[i * N + tid] : 0;
        const u64 b = l.bound;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < (int)(sizeof(keep) / sizeof(u64)); i++)
            if (keep[i] >= b && keep[i]) l.found[atomicAdd(&l.nchosen, 1)] = keep[i];
        __syncthreads();
        n = l.nchosen;
    }
    // each key's place is the number of larger ones
    constexpr int M = (2 * 128 + 64 + N - 1) / N;
    u64 key[M];
    int place[M];
#pragma unroll
    for (int i = 0; i < M; i++) { key[i] = i * N + tid < n ? l.found[i * N + tid] : 0; place[i] = 0; }
    for (int q = 0; q < n; q++) {
        const u64 other = l.found[q];
#pragma unroll
        for (int i = 0; i < M; i++) place[i] += other > key[i] ? 1 : 0;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < M; i++)
        if (key[i] && place[i] < k) l.found[place[i]] = key[i];
    for (int i = n + tid; i < k; i += N) l.found[i] = 0;
    __syncthreads();
}

// ------------------------------------------------------------------ a row's results

// Writes what a row's sums give.  w is that of e t about the peak.
template <int N>
EWF_OPS_DEV void finish_logprobs(const VocabLaunch &a, uint32_t row, const Sums &sum, float token_logit, const u64 *found)
{
    const bool none = sum.peak == -kInf && sum.s == 0.f;
    const float logsum = none ? -kInf : logf(sum.s);
    const bool nan = !none && !(sum.s < kInf);           // a NaN or an infinity among the logits
    const float bad = __builtin_nanf("");
    if (threadIdx.x == 0) {
        if (a.logprob) a.logprob[row_offset(a.r, row, a.slogprob)] = nan ? bad : none ? -kInf : fmaf(token_logit - sum.peak, a.scale, -logsum);
        if (a.peak) a.peak[row_offset(a.r, row, a.speak)] = nan ? bad : sum.peak;
        if (a.logsum) a.logsum[row_offset(a.r, row, a.slogsum)] = nan ? bad : logsum;
        if (a.entropy) a.entropy[row_offset(a.r, row, a.sentropy)] = nan ? bad : none ? 0.f : logsum - kLn2 * (sum.w / sum.s);
    }
    if (a.top) {
        float *value = a.top_values + row_offset(a.r, row, a.stop_values);
        int32_t *index = a.top_indices + row_offset(a.r, row, a.stop_indices);
        for (int i = threadIdx.x; i < a.top; i += N) {
            const u64 key = found[i];
            value[i] = nan ? bad : key ? fmaf(unordered((uint32_t)(key >> 32)) - sum.peak, a.scale, -logsum) : -kInf;
            index[i] = nan || !key ? -1 : (int32_t)~(uint32_t)key;
        }
    }
}

// A row without a token: zeros, and no alternatives.
template <int N>
EWF_OPS_DEV void padding_logprobs(const VocabLaunch &a, uint32_t row)
{
    if (threadIdx.x == 0) {
        if (a.logprob) a.logprob[row_offset(a.r, row, a.slogprob)] = 0.f;
        if (a.peak) a.peak[row_offset(a.r, row, a.speak)] = 0.f;
        if (a.logsum) a.logsum[row_offset(a.r, row, a.slogsum)] = 0.f;
        if (a.entropy) a.entropy[row_offset(a.r, row, a.sentropy)] = 0.f;
    }
    if (a.top) {
        float *value = a.top_values + row_offset(a.r, row, a.stop_values);
        int32_t *index = a.top_indices + row_offset(a.r, row, a.stop_indices);
        for (int i = threadIdx.x; i < a.top; i += N) { value[i] = -kInf; index[i] = -1; }
    }
}

EWF_OPS_DEV bool is_padding(const VocabLaunch &a, uint32_t row, int &token)
{
    token = -1;
    if (!a.tokens) return false;
    token = a.tokens[row_offset(a.r, row, a.stokens)];
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
    int edge[16];                                       // an entry on each edge element, -1
    float tail_q, total_q;                              // 1 - sum q; sum q
    int live;                                           // entries that exist
    float gradient[4];                                  // of the logits that no entry names (see Slope)
};

template <int N>
EWF_OPS_DEV void clear(Entries<N> &l)
{
    l.head[threadIdx.x] = -1;
    if (threadIdx.x < 16) l.edge[threadIdx.x] = -1;
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
EWF_OPS_DEV void read_entries(Entries<N> &l, const VocabLaunch &a, uint32_t row, const typename T::raw *logits, const Span<T> &s, int j0, int j1, bool edges)
{
    constexpr int V = Vec16<T>::V;
    const int lane = threadIdx.x;
    const int64_t values = row_offset(a.r, row, a.steacher_values), indices = row_offset(a.r, row, a.steacher_indices);
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
            owner = s.edge_of(c[h]) & 15;
            if (edges) l.edge[owner] = i;               // (of several that are the same one, any: they have the same gradient)
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
EWF_OPS_DEV void finish_distill(const VocabLaunch &a, Entries<N> &l, uint32_t row, Sums sum, bool slope, Slope &g)
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
        move_to<false>(sum, ref, a.c);
        total = sum.s + e;
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
        if (a.loss) a.loss[row_offset(a.r, row, a.sloss)] = nan ? bad : loss;
        if (a.peak) a.peak[row_offset(a.r, row, a.speak)] = nan ? bad : peak;
        if (a.logsum) a.logsum[row_offset(a.r, row, a.slogsum)] = nan ? bad : logsum;
        if (a.tail) a.tail[row_offset(a.r, row, a.stail)] = nan ? bad : tail;
    }
    if (!slope) return;
    const float weight = a.dloss ? a.dloss[row_offset(a.r, row, a.sdloss)] : 1.f;
    g = slope_of(a, nan ? bad : peak, nan ? bad : logsum, tail, tail_q, l.total_q, weight);
#pragma unroll
    for (int h = 0; h < 2; h++)
        l.grad[h * 64 + lane] = g.factor * fmaf(g.mass, __builtin_amdgcn_exp2f(fmaf(x[h] - g.ref, a.c, -g.logsum2)), -all[h]);
    if (lane == 0) { l.gradient[0] = g.ref; l.gradient[1] = g.off; l.gradient[2] = g.coef; }
}

EWF_OPS_DEV void padding_distill(const VocabLaunch &a, uint32_t row)
{
    if (threadIdx.x) return;
    if (a.loss) a.loss[row_offset(a.r, row, a.sloss)] = 0.f;
    if (a.peak) a.peak[row_offset(a.r, row, a.speak)] = 0.f;
    if (a.logsum) a.logsum[row_offset(a.r, row, a.slogsum)] = 0.f;
    if (a.tail) a.tail[row_offset(a.r, row, a.stail)] = 0.f;
}

// ------------------------------------------------------------------ sums over rows

enum { kLogprobs = 0, kDistill = 1, kDistillTail = 2 };

// One workgroup a row, or one of a.splits that share it and leave their sums and their largest in the workspace.
template <typename T, int N, bool ENT, bool TOP, int KIND>
__global__ void __launch_bounds__(N) k_rows(VocabLaunch a)
{
    typedef typename T::raw raw;
    constexpr int V = Vec16<T>::V, U = 4;
    __shared__ float sums[48];
    __shared__ typename std::conditional<TOP, TopLds<N>, int>::type top;
    __shared__ typename std::conditional<KIND != kLogprobs, Entries<N>, int>::type entries;
    const int tid = threadIdx.x;
    const uint32_t block = blockIdx.x, splits = (uint32_t)a.splits;
    const uint32_t row = a.row0 + block / splits, split = block - block / splits * splits;
    const raw *p = (const raw *)a.logits + row_offset(a.r, row, a.slogits);
    const Span<T> s(p, a.r.cols);
    const int per = (s.nvec + (int)splits - 1) / (int)splits;
    const int j0 = (int)split * per < s.nvec ? (int)split * per : s.nvec, j1 = j0 + per < s.nvec ? j0 + per : s.nvec;
    const bool edges = split == 0;
    int token = 0;
    if constexpr (KIND == kLogprobs) {
        if (is_padding(a, row, token)) {
            if (splits == 1) padding_logprobs<N>(a, row);
            return;
        }
    } else if (KIND == kDistillTail || splits == 1) {
        clear(entries);
        __syncthreads();
        if (tid < 64) read_entries<T>(entries, a, row, p, s, j0, j1, edges);
        __syncthreads();
        if (entries.live == 0) {
            if (splits == 1) padding_distill(a, row);
            return;
        }
    }
    float token_logit = 0.f;
    if (KIND == kLogprobs && splits == 1 && token >= 0) token_logit = load1<T>(p + token);
    Sums sum;
    Best best;
    float edge = -kInf;
    if (edges && tid < s.edges()) edge = load1<T>(p + s.edge(tid));
    if constexpr (KIND == kDistillTail)
        if (edges && tid < 16 && entries.edge[tid] >= 0) edge = -kInf;
    int hit = 0x7fffffff;                                // the next of this thread's trips that holds an entry
    auto next_hit = [&](int from) {
        hit = 0x7fffffff;
        if constexpr (KIND == kDistillTail)
            for (int k = entries.head[tid]; k >= 0; k = entries.next[k])
                if (entries.trip[k] >= from && entries.trip[k] < hit) hit = entries.trip[k];
    };
    next_hit(0);
    const raw *first = p + s.head;
    for (int j = j0 + tid, trip = 0; j - tid < j1; j += U * N, trip += U) {
        u32x4 v[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            v[u] = u32x4{kNothing<T>, kNothing<T>, kNothing<T>, kNothing<T>};
            if (j + u * N < j1) v[u] = load16<T>(first + (int64_t)(j + u * N) * V);
        }
        float x[U * V];
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int e = 0; e < V; e++) x[u * V + e] = element<T>(v[u], e);
        if constexpr (KIND == kDistillTail)
            if (hit < trip + U) {
                for (int k = entries.head[tid]; k >= 0; k = entries.next[k]) {
                    const int at = (entries.trip[k] - trip) * V + (entries.index[k] - s.head) % V;
                    if (entries.trip[k] < trip) continue;
#pragma unroll
                    for (int e = 0; e < U * V; e++) x[e] = e == at ? -kInf : x[e];
                }
                next_hit(trip + U);
            }
        float most[U], over = -kInf;
#pragma unroll
        for (int u = 0; u < U; u++) {
            most[u] = max_of<V>(x + u * V);
            if (TOP && most[u] > best.value) { best.value = most[u]; best.vec = j + u * N; }
            over = fmaxf(over, most[u]);
        }
        add<ENT, U * V>(sum, x, over, a.c, a.lag);
    }
    add<ENT, 1>(sum, &edge, edge, a.c, a.lag);
    sum = workgroup_sums<N, ENT>(sum, a.c, sums);
    if constexpr (TOP) largest<T, N>(top, p, s, j0, j1, edges, edge, best, a.top);
    if (splits > 1) {
        const int64_t part = (int64_t)(row - a.row0) * splits + split;
        if (tid == 0) {
            float *out = a.parts + part * 4;
            out[0] = sum.peak; out[1] = sum.s; out[2] = sum.w;
        }
        if constexpr (TOP)
            for (int i = tid; i < a.top; i += N) a.part_keys[part * a.top + i] = top.found[i];
        return;
    }
    if constexpr (KIND == kLogprobs) {
        const u64 *found = nullptr;
        if constexpr (TOP) found = top.found;
        finish_logprobs<N>(a, row, sum, token_logit, found);
    } else if (tid < 64) {
        Slope g;
        finish_distill(a, entries, row, sum, false, g);
    }
}

// Joins the parts of a row.
template <typename T, int N, bool TOP, int KIND>
__global__ void __launch_bounds__(N) k_join(VocabLaunch a)
{
    typedef typename T::raw raw;
    __shared__ typename std::conditional<KIND != kLogprobs, Entries<N>, int>::type entries;
    __shared__ u64 keys[TOP ? kMaxJoin : 1], found[TOP ? kMaxTop : 1];
    const uint32_t row = a.row0 + blockIdx.x;
    const raw *p = (const raw *)a.logits + row_offset(a.r, row, a.slogits);
    const int tid = threadIdx.x, lane = tid & 63, splits = a.splits;
    int token = 0;
    if constexpr (KIND == kLogprobs) {
        if (is_padding(a, row, token)) { padding_logprobs<N>(a, row); return; }
    } else {
        const Span<T> s(p, a.r.cols);
        clear(entries);
        __syncthreads();
        if (tid < 64) read_entries<T>(entries, a, row, p, s, 0, 0, false);
        __syncthreads();
        if (entries.live == 0) { padding_distill(a, row); return; }
    }
    const float token_logit = KIND == kLogprobs && token >= 0 ? load1<T>(p + token) : 0.f;
    const int64_t part = (int64_t)blockIdx.x * splits;
    Sums sum;
    sum.m = 0.f;
    if (lane < splits) {
        const float *in = a.parts + (part + lane) * 4;
        sum.peak = in[0]; sum.s = in[1]; sum.w = in[2];
        sum.m = sum.peak == -kInf ? 0.f : sum.peak;
    }
    const float peak = wave_max(sum.peak);
    move_to<true>(sum, peak == -kInf ? 0.f : peak, a.c);
    sum.s = group_sum<64>(sum.s);
    sum.w = group_sum<64>(sum.w);
    sum.peak = peak;
    if constexpr (TOP) {
        // the parts' lists descend: a key's place is the number of larger ones in each
        const int k = a.top, n = splits * k;
        for (int i = tid; i < n; i += N) keys[i] = a.part_keys[part * k + i];
        for (int i = tid; i < k; i += N) found[i] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += N) {
            const u64 key = keys[i];
            int place = 0;
            for (int q = 0; q < splits && key && place < k; q++) {
                int lo = 0, hi = k;
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (keys[q * k + mid] > key) lo = mid + 1; else hi = mid;
                }
                place += lo;
            }
            if (key && place < k) found[place] = key;
        }
        __syncthreads();
    }
    if constexpr (KIND == kLogprobs) finish_logprobs<N>(a, row, sum, token_logit, found);
    else if (tid < 64) {
        Slope g;
        finish_distill(a, entries, row, sum, false, g);
    }
}

// ------------------------------------------------------------------ gradients from saved statistics

constexpr int kGradThreads = 256;

// Writes vector j of a row, whose elements are f.
template <typename T>
EWF_OPS_DEV void store_vector(typename T::raw *out, const Span<T> &s, int j, const float *f)
{
    store16<T>(out + s.head + (int64_t)j * Vec16<T>::V, pack16<T>(f));
}

// One workgroup a piece of U vectors a thread of a row.  dx_j = c (g ([j = token] - p_j) - h p_j (log p_j + entropy))
template <typename T, bool ENT, int U>
__global__ void __launch_bounds__(kGradThreads) k_logprobs_grad(VocabLaunch a)
{
    typedef typename T::raw raw;
    constexpr int V = Vec16<T>::V, N = kGradThreads;
    const uint32_t pieces = (uint32_t)a.splits, row = a.row0 + blockIdx.x / pieces, piece = blockIdx.x - blockIdx.x / pieces * pieces;
    const raw *p = (const raw *)a.logits + row_offset(a.r, row, a.slogits);
    raw *out = (raw *)a.dlogits + row_offset(a.r, row, a.sdlogits);
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
        if (j0 + u * N < s.nvec) v[u] = load16<T>(p + s.head + (int64_t)(j0 + u * N) * V);
    }
    const float x = edge ? load1<T>(p + s.edge(tid)) : 0.f;
    const float peak = a.peak[row_offset(a.r, row, a.speak)], logsum = a.logsum[row_offset(a.r, row, a.slogsum)];
    const float g = a.dlogprob ? a.dlogprob[row_offset(a.r, row, a.sdlogprob)] * a.scale : 0.f;
    const float h = ENT ? a.dentropy[row_offset(a.r, row, a.sdentropy)] * a.scale : 0.f, H = ENT ? a.entropy[row_offset(a.r, row, a.sentropy)] : 0.f;
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
        store_vector<T>(out, s, j, f);
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
    const uint32_t pieces = (uint32_t)a.splits, row = a.row0 + blockIdx.x / pieces, piece = blockIdx.x - blockIdx.x / pieces * pieces;
    const raw *p = (const raw *)a.logits + row_offset(a.r, row, a.slogits);
    raw *out = (raw *)a.dlogits + row_offset(a.r, row, a.sdlogits);
    const Span<T> s(out, a.r.cols);
    const int tid = threadIdx.x, begin = (int)piece * (U * N), j0 = begin + tid;
    const int end = begin + U * N < s.nvec ? begin + U * N : s.nvec;
    const bool edge = piece == 0 && tid < s.edges();
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        v[u] = u32x4{0u, 0u, 0u, 0u};
        if (j0 + u * N < end) v[u] = load16<T>(p + s.head + (int64_t)(j0 + u * N) * V);
    }
    const float x = edge ? load1<T>(p + s.edge(tid)) : 0.f;
    clear(l);
    __syncthreads();
    if (tid < 64) read_entries<T>(l, a, row, p, s, begin, end, piece == 0);
    __syncthreads();
    const float peak = a.peak[row_offset(a.r, row, a.speak)], logsum = a.logsum[row_offset(a.r, row, a.slogsum)];
    const float tail = a.with_tail ? a.tail[row_offset(a.r, row, a.stail)] : 0.f;
    const float weight = a.dloss ? a.dloss[row_offset(a.r, row, a.sdloss)] : 1.f;
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
        store_vector<T>(out, s, j, f);
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
    const uint32_t row = a.row0 + blockIdx.x;
    const raw *p = (const raw *)a.logits + row_offset(a.r, row, a.slogits);
    raw *out = (raw *)a.dlogits + row_offset(a.r, row, a.sdlogits);
    const Span<T> s(out, a.r.cols);
    const int tid = threadIdx.x;
    const bool edge = tid < s.edges();
    u32x4 v[NV];
#pragma unroll
    for (int u = 0; u < NV; u++) {
        v[u] = u32x4{kNothing<T>, kNothing<T>, kNothing<T>, kNothing<T>};
        if (tid + u * N < s.nvec) v[u] = load16<T>(p + s.head + (int64_t)(tid + u * N) * V);
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
    const int on_edge = tid < 16 ? l.edge[tid] : -1;
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
        sum.peak = peak; sum.m = ref; sum.s = total;
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
        store_vector<T>(out, s, j, f);
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
        a.row0 = (uint32_t)row;
        const int64_t rows = std::min<int64_t>(most, a.r.rows - row);
        launch(a, dim3((unsigned)(rows * blocks_per_row)), (unsigned)rows);
    }
}

int vectors(const VocabLaunch &a) { return (a.r.cols + (a.dtype == EWF_F32 ? 4 : 8) - 1) / (a.dtype == EWF_F32 ? 4 : 8); }

template <typename T, int N, bool ENT, bool TOP, int KIND>
void run_rows(const VocabLaunch &a, hipStream_t stream)
{
    by_rows(a, a.splits, N, [&](VocabLaunch b, dim3 grid, unsigned rows) {
        if (b.splits > 1) {      // (all launches' parts are apart)
            b.parts += (int64_t)b.row0 * b.splits * 4;
            if (TOP) b.part_keys += (int64_t)b.row0 * b.splits * b.top;
        }
        hipLaunchKernelGGL((k_rows<T, N, ENT, TOP, KIND>), grid, dim3(N), 0, stream, b);
        if (b.splits > 1) hipLaunchKernelGGL((k_join<T, TOP ? 1024 : 64, TOP, KIND>), dim3(rows), dim3(TOP ? 1024 : 64), 0, stream, b);
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
        else if (a.threads == 256) run_kind<T, 256>(a, stream);
        else run_kind<T, 1024>(a, stream);
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
    a.threads = n <= 256 ? 64 : a.r.rows < (uint32_t)units ? 1024 : 256;
    a.splits = 1;
    if (a.r.rows < (uint32_t)units && n > 32768) {
        a.splits = (int)std::min<int64_t>(std::min<int64_t>(64, n / 8192), (2 * units + a.r.rows - 1) / a.r.rows);
        if (a.top) a.splits = std::min(a.splits, kMaxJoin / a.top);
    }
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
