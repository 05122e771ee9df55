// The loss of a student's logits against a teacher's entries, and its gradient, by itself or in the loss's own sweep.
#include "ewf_vocab_rows.h"

namespace ewf {

namespace {

// One wavefront a row: what the gradients of a row need, from the statistics that the loss has saved.  4096 rows of 32 entries take 8 to 9 us; the kernel below would
// have to do it for each piece of a row (102 us in place of 91 for both).
template <typename T, int K>
__global__ void __launch_bounds__(64) k_distill_prepare(VocabLaunch a)
{
    typedef typename T::raw raw;
    __shared__ Entries<64, K> l;
    const RowAt row = row_at(a.r, a.row0 + blockIdx.x);
    const raw *p = (const raw *)a.logits + at(row, a.slogits);
    const Stats r = {a.peak[at(row, a.speak)], a.logsum[at(row, a.slogsum)], a.with_tail ? a.tail[at(row, a.stail)] : 0.f};
    take_entries<T>(l, a, row, p, Span<T>(p, a.r.cols), 0, 0, false);
    __syncthreads();
    prepare_gradients(a, l, row, r, prepared_row(a, blockIdx.x));
}

constexpr int kGradThreads = 256, kGradVectors = 2;

// One workgroup a piece of a row: the element-wise gradient, and the entries' that lie in it, each in the list of the thread that takes its vector
// or its edge.  bfloat16 [4096, 32768] 80 to 82 us, 6.6 TB/s.
template <typename T, bool STREAM>
__global__ void __launch_bounds__(kGradThreads) k_distill_grad(VocabLaunch a)
{
    typedef typename T::raw raw;
    constexpr int V = Vec16<T>::V, N = kGradThreads, U = kGradVectors;
    __shared__ int head[N], next[kMaxTop], index[kMaxTop];
    __shared__ float grad[kMaxTop];
    const uint32_t pieces = (uint32_t)a.splits, piece = blockIdx.x % pieces, in_launch = blockIdx.x / pieces;
    const RowAt row = row_at(a.r, a.row0 + in_launch);
    const raw *p = (const raw *)a.logits + at(row, a.slogits);
    raw *out = (raw *)a.dlogits + at(row, a.sdlogits);
    const Span<T, kLine> s(out, a.r.cols);
    const int tid = threadIdx.x, begin = (int)piece * (U * N), end = begin + U * N < s.nvec ? begin + U * N : s.nvec;
    const bool edge = piece == 0 && tid < s.edges();
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        v[u] = u32x4{0u, 0u, 0u, 0u};
        if (begin + u * N + tid < end) v[u] = load_vector<T, STREAM>(p + s.head, begin + u * N, tid);
    }
    const float x = edge ? load1<T>(p + s.edge(tid)) : 0.f;
    const Prepared *prepared = prepared_row(a, in_launch);
    const bool padding = prepared->padding;              // (then nothing else is there)
    const Prepared::Entry e = tid < a.entries && !padding ? prepared->entry[tid] : Prepared::Entry{-1, 0.f};
    const Exponent t = prepared->exponent(a.c);
    const float coef = prepared->coef;
    head[tid] = -1;
    __syncthreads();
    if (e.index >= 0) {
        const int j = s.inside(e.index) ? (e.index - s.head) / V - begin : -1;
        const int owner = j >= 0 ? (j < U * N ? j % N : -1) : s.inside(e.index) || piece ? -1 : s.edge_of(e.index);
        index[tid] = e.index;
        grad[tid] = e.grad;
        if (owner >= 0) next[tid] = atomicExch(&head[owner], tid);
    }
    __syncthreads();
    const int list = head[tid];
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int j = begin + u * N + tid;
        if (j >= end) continue;
        float f[V], q[V];
#pragma unroll
        for (int i = 0; i < V; i++) f[i] = element<T>(v[u], i);
        t.of<V>(f, q);
#pragma unroll
        for (int i = 0; i < V; i++) f[i] = coef * __builtin_amdgcn_exp2f(q[i]);
        for (int k = list; k >= 0; k = next[k]) {
            const int at = index[k] - s.head - j * V;    // (another vector's, or an edge's: outside)
            const float g = grad[k];
#pragma unroll
            for (int i = 0; i < V; i++) f[i] = i == at ? g : f[i];
        }
        if (padding)
#pragma unroll
            for (int i = 0; i < V; i++) f[i] = 0.f;
        store_vector<T>(out + s.head, begin + u * N, tid, f);
    }
    if (edge) {
        float q;
        t.of<1>(&x, &q);
        q = coef * __builtin_amdgcn_exp2f(q);
        for (int k = list; k >= 0; k = next[k]) q = index[k] == s.edge(tid) ? grad[k] : q;
        store1<T>(out + s.edge(tid), padding ? 0.f : q);
    }
}

// A workgroup holds a row in registers, NV vectors a thread, and takes rows one after the other: logits are read once, a vector's registers
// take the next row's as soon as its gradients are written.  Between the two barriers of a row its sums are taken as its vectors arrive; the
// next row's entries are read behind them.
//
// Memory bounds it where several rows share a compute unit: bfloat16 [4096, 50257] (two) 163 us, 5.1 TB/s; in one workgroup of 1024 threads 190, in two sweeps 200.
// Shorter rows by single wavefronts wait for their entries, which only other rows hide: [8192, 7000] 62 us, 3.7 TB/s; [16384, 1000] 35, 1.9.
// A row of more than 8192 vectors has a compute unit to itself, and no register is free for the next one from its last vector's arrival to its first
// gradients; the first half of the next row comes into the cache meanwhile: [2048, 131072] 212 us (5.1 TB/s), without that 232 (without any arithmetic either 207,
// without the stores 143), with a quarter 222, the whole row 239 (the compute units of one cache have 8 MB of rows, twice what it keeps), from the sums' begin
// on 220; float32 [1280, 50257] 95 and 105; below 8192 vectors no gain.  Tried there: the next row's sums begun amid this one's gradients 267 (a wait
// for a load waits for the stores before it), loads before stores, entries ranked behind the gradients, plain loads or stores: no gain.  Registers hold a row with nothing
// spilled only if logits are unpacked twice.
template <typename T, int N, int NV, int K, bool STREAM>
__global__ void __launch_bounds__(N, NV > 8 ? 4 : 1) k_distill_held(VocabLaunch a)
{
    typedef typename T::raw raw;
    constexpr int V = Vec16<T>::V, W = N / 64, LINE = N > 64 ? kLine : 16;
    typedef Span<T, LINE> RowSpan;
    __shared__ float parts[2][2][16];
    __shared__ Entries<N, K> lists[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t i = blockIdx.x;
    RowAt row = row_at(a.r, a.row0 + i);
    const raw *p = (const raw *)a.logits + at(row, a.slogits);
    raw *out = (raw *)a.dlogits + at(row, a.sdlogits);
    RowSpan s(out, a.r.cols);
    u32x4 v[NV];
    float x;
    auto fetch = [&](u32x4 &v, const raw *p, const RowSpan &s, int u) {
        if (u * N + tid < s.nvec) v = load_vector<T, STREAM>(p + s.head, u * N, tid);
        else v = u32x4{kNothing<T>, kNothing<T>, kNothing<T>, kNothing<T>};
    };
#pragma unroll
    for (int u = 0; u < NV; u++) fetch(v[u], p, s, u);
    x = tid < s.edges() ? load1<T>(p + s.edge(tid)) : -kInf;
    if (tid < 64) take_entries<T>(lists[0], a, row, p, s, 0, s.nvec, true);
    for (int turn = 0;; turn ^= 1) {
        const Entries<N, K> &l = lists[turn];
        __syncthreads();
        const bool padding = l.live == 0;
        const uint32_t held = trips_with_entries(l);
        const int on_edge = tid < s.edges() ? l.edge[tid] : -1;
        // the next row, its entries on their way while this one's sums are taken
        const uint32_t next = i + gridDim.x;
        const bool more = next < a.rows;
        const RowAt nrow = row_at(a.r, a.row0 + (more ? next : i));
        const raw *np = (const raw *)a.logits + at(nrow, a.slogits);
        raw *nout = (raw *)a.dlogits + at(nrow, a.sdlogits);
        const RowSpan ns(nout, a.r.cols);
        RawEntries<K> entries;
        const bool reader = more && tid < 64;
        if (reader) read_entries(entries, a, nrow);
        Sums sum;
#pragma unroll
        for (int u = 0; u < NV; u++) {
            if (__any(u * N + tid < s.nvec)) {
                float f[V];
#pragma unroll
                for (int e = 0; e < V; e++) f[e] = element<T>(v[u], e);
                if (a.with_tail && held >> u & 1)       // (what no entry names: the entries' own sum is taken with them)
                    each_entry<V>(l, u, s.head, [&](int at, int) {
#pragma unroll
                        for (int e = 0; e < V; e++) f[e] = e == at ? -kInf : f[e];
                    });
                add<false, V>(sum, f, max_of<V>(f), a.c, a.lag);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // (logits are unpacked again below: kept unpacked they would not fit)
#pragma unroll
        for (int u = 0; u < NV; u++) asm volatile("" : "+v"(v[u]));
        if (reader) read_logits<T>(entries, a, np);
        // (one element of each cache line)
        raw ahead = {};
        if (N == 1024 && more && tid * 16 < ns.nvec) ahead = *(const raw *)((const char *)(np + ns.head) + tid * 128);
        const float own = a.with_tail && on_edge >= 0 ? -kInf : x;
        add<false, 1>(sum, &own, own, a.c, a.lag);
        sum = wave_sums<false>(sum, a.c);
        if (W > 1) {
            if (lane == 0) { parts[turn][0][wave] = sum.peak; parts[turn][1][wave] = sum.s; }
            __syncthreads();
            sum = joined_sums<W, false>(parts[turn][0], parts[turn][1], nullptr, a.c);
        }
        settle<false>(sum, a.c);
        if (beyond(sum.peak, a.c)) sum_again<T, N>(a, p, s, 0, s.nvec, true, a.with_tail, l, &parts[turn][0][0], sum);
        Stats r = stats_of(a, l, sum);
        r = {scalar(r.peak), scalar(r.logsum), scalar(r.tail)};
        if (wave == W - 1) {
            if (!padding) finish_distill(a, l, row, r);
            else if (lane == 0) {
                a.loss[at(row, a.sloss)] = 0.f;
                if (a.peak) a.peak[at(row, a.speak)] = 0.f;
                if (a.logsum) a.logsum[at(row, a.slogsum)] = 0.f;
                if (a.tail) a.tail[at(row, a.stail)] = 0.f;
            }
        }
        const Slope g(a, l, r, a.dloss ? a.dloss[at(row, a.sdloss)] : 1.f);
        if (reader) rank_entries<T>(lists[turn ^ 1], entries, a, ns, 0, ns.nvec, true);
        float coef = g.coef, point = g.rest.k;
        if (padding) {                                   // (whatever its logits are)
            coef = point = 0.f;
#pragma unroll
            for (int u = 0; u < NV; u++) v[u] = u32x4{0u, 0u, 0u, 0u};
        }
        if (g.rest.as_is)                                // (the type's lowest or largest numbers: element by element, before the entries')
            for (int c = s.head + tid; c < s.head + s.nvec * V; c += N) {
                const float y = load1<T>(p + c);
                float t;
                g.rest.template of<1>(&y, &t);
                t = g.coef * __builtin_amdgcn_exp2f(t);
                for (int k = 0; k < a.entries; k++)
                    if (l.index[k] == c) t = g.entry(l, k);
                store1<T>(out + c, padding ? 0.f : t);
            }
#pragma unroll
        for (int u = 0; u < NV; u++) {
            const int j = u * N + tid;
            if (j < s.nvec && !g.rest.as_is) {
                float f[V];
#pragma unroll
                for (int e = 0; e < V; e++) f[e] = element<T>(v[u], e);
#pragma unroll
                for (int e = 0; e < V; e++) f[e] = coef * __builtin_amdgcn_exp2f(fmaf(f[e], a.c, -point));
                store_vector<T>(out + s.head, u * N, tid, f);
            }
            if (more) fetch(v[u], np, ns, u);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (N == 1024) asm volatile("" :: "v"((int)*(const uint16_t *)&ahead));
        // the entries' gradients, each by the thread that wrote its vector (and after that: a thread's stores keep their order)
        for (int k = g.rest.as_is ? -1 : l.head[tid]; k >= 0; k = l.next[k])
            if (l.trip[k] >= 0) store1<T>(out + l.index[k], g.entry(l, k));
        if (tid < s.edges()) {
            float t;
            g.rest.template of<1>(&x, &t);
            store1<T>(out + s.edge(tid), padding ? 0.f : on_edge >= 0 ? g.entry(l, on_edge) : g.coef * __builtin_amdgcn_exp2f(t));
        }
        if (!more) return;
        x = tid < ns.edges() ? load1<T>(np + ns.edge(tid)) : -kInf;
        i = next;
        row = nrow;
        p = np;
        out = nout;
        s = ns;
    }
}

struct RunRows {
    const VocabLaunch &a;
    hipStream_t stream;
    template <typename T, int N, int K> void go() const
    {
        if (a.with_tail) run_rows<T, N, false, false, kDistillTail, K>(a, stream);
        else run_rows<T, N, false, false, kDistill, K>(a, stream);
    }
    template <typename T, int K> void run() const
    {
        if (a.threads == 64) go<T, 64, K>();
        else go<T, 256, K>();
    }
    template <typename T> void operator()() const
    {
        if (a.entries <= 64) run<T, 64>();
        else run<T, kMaxTop>();
    }
};

struct RunPrepare {
    const VocabLaunch &a;
    hipStream_t stream;
    template <typename T> void operator()() const
    {
        by_rows(a, 1, 64, [&](VocabLaunch b, dim3 grid, unsigned) {
            b.prepared = (char *)b.prepared + b.row0 * prepared_bytes(b.entries);
            if (b.entries <= 64) hipLaunchKernelGGL((k_distill_prepare<T, 64>), grid, dim3(64), 0, stream, b);
            else hipLaunchKernelGGL((k_distill_prepare<T, kMaxTop>), grid, dim3(64), 0, stream, b);
        });
    }
};

struct RunGrad {
    VocabLaunch a;
    hipStream_t stream;
    template <typename T> void operator()()
    {
        a.splits = std::max(1, (vectors(a) + kGradVectors * kGradThreads - 1) / (kGradVectors * kGradThreads));
        by_rows(a, a.splits, kGradThreads, [&](VocabLaunch b, dim3 grid, unsigned) {
            b.prepared = (char *)b.prepared + b.row0 * prepared_bytes(b.entries);
            if (b.stream) hipLaunchKernelGGL((k_distill_grad<T, true>), grid, dim3(kGradThreads), 0, stream, b);
            else hipLaunchKernelGGL((k_distill_grad<T, false>), grid, dim3(kGradThreads), 0, stream, b);
        });
    }
};

struct RunHeld {
    const VocabLaunch &a;
    hipStream_t stream;
    template <typename T, int N, int NV, int K> void go() const
    {
        by_rows(a, 1, N, [&](const VocabLaunch &b, dim3 grid, unsigned) {
            grid.x = std::min(grid.x, (unsigned)b.resident);
            if (N > 64 && b.stream) hipLaunchKernelGGL((k_distill_held<T, N, NV, K, (N > 64)>), grid, dim3(N), 0, stream, b);
            else hipLaunchKernelGGL((k_distill_held<T, N, NV, K, false>), grid, dim3(N), 0, stream, b);
        });
    }
    template <typename T, int K> void run() const
    {
        const int n = vectors(a);
        if (a.threads == 64) {
            if (n <= 64) go<T, 64, 1, K>();
            else if (n <= 128) go<T, 64, 2, K>();
            else if (n <= 256) go<T, 64, 4, K>();
            else if (n <= 512) go<T, 64, 8, K>();
            else go<T, 64, 16, K>();
        } else if (n <= 512) go<T, 256, 2, K>();
        else if (n <= 1024) go<T, 256, 4, K>();
        else if (n <= 2048) go<T, 256, 8, K>();
        else if (n <= 4096) go<T, 256, 16, K>();
        else if (n <= 6144) go<T, 512, 12, K>();
        else if (n <= 8192) go<T, 512, 16, K>();
        else if (n <= 12288) go<T, 1024, 12, K>();
        else go<T, 1024, 16, K>();
    }
    template <typename T> void operator()() const
    {
        if (a.entries <= 64) run<T, 64>();
        else run<T, kMaxTop>();
    }
};

}  // namespace

void launch_distill_grad(const VocabLaunch &a, hipStream_t stream)
{
    by_type(a.dtype, RunPrepare{a, stream});
    by_type(a.dtype, RunGrad{a, stream});
}

void launch_distill(const VocabLaunch &a, hipStream_t stream)
{
    if (a.held) return by_type(a.dtype, RunHeld{a, stream});
    by_type(a.dtype, RunRows{a, stream});                   // (prepares the gradients too)
    if (a.dlogits) by_type(a.dtype, RunGrad{a, stream});
}

}  // namespace ewf
