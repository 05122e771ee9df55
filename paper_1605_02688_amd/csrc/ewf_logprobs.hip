// Log probabilities of given tokens with entropy and the largest alternatives, and their gradient; the plan of all operators over rows of logits.
#include "ewf_vocab_rows.h"

namespace ewf {

namespace {

constexpr int kGradThreads = 256, kGradVectors = 2;

// One workgroup a piece of a row, element-wise, so that memory bounds it: bfloat16 [4096, 50257] 128 us (6.4 TB/s; a copy of these bytes 126), float16
// [750, 33279] 17.5.  Pieces of 8 KB: a copy takes 126 to 131 us with one to four vectors a thread, 192 with eight.
//     dx_j = scale (g ([j = token] - p_j) - h p_j (log p_j + entropy))
template <typename T, bool ENT, bool STREAM>
__global__ void __launch_bounds__(kGradThreads) k_logprobs_grad(VocabLaunch a)
{
    typedef typename T::raw raw;
    constexpr int V = Vec16<T>::V, N = kGradThreads, U = kGradVectors;
    const uint32_t pieces = (uint32_t)a.splits, piece = blockIdx.x % pieces;
    const RowAt row = row_at(a.r, a.row0 + blockIdx.x / pieces);
    const raw *p = (const raw *)a.logits + at(row, a.slogits);
    raw *out = (raw *)a.dlogits + at(row, a.sdlogits);
    const Span<T, kLine> s(out, a.r.cols);
    const int tid = threadIdx.x, begin = (int)piece * (U * N), j0 = begin + tid;
    const bool edge = piece == 0 && tid < s.edges();
    int token;
    if (is_padding(a, row, token)) {
        const float zero[V] = {};
#pragma unroll
        for (int u = 0; u < U; u++)
            if (j0 + u * N < s.nvec) store_vector<T>(out + s.head, begin + u * N, tid, zero);
        if (edge) store1<T>(out + s.edge(tid), 0.f);
        return;
    }
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        v[u] = u32x4{0u, 0u, 0u, 0u};
        if (j0 + u * N < s.nvec) v[u] = load_vector<T, STREAM>(p + s.head, begin + u * N, tid);
    }
    const float x = edge ? load1<T>(p + s.edge(tid)) : 0.f;
    const float peak = a.peak[at(row, a.speak)], logsum = a.logsum[at(row, a.slogsum)];
    const float g = a.dlogprob ? a.dlogprob[at(row, a.sdlogprob)] * a.scale : 0.f;
    const float h = ENT ? a.dentropy[at(row, a.sdentropy)] * a.scale : 0.f, H = ENT ? a.entropy[at(row, a.sentropy)] : 0.f;
    const bool none = peak == -kInf;                     // (no logit at all: no gradient)
    const Exponent e(none ? 0.f : peak, none ? 0.f : logsum * kLog2E, a.c);
    // p = r 2^t, log p = (t + rest) ln 2
    const float r = none ? 0.f : __builtin_amdgcn_exp2f(e.rest), hot = none ? 0.f : g;
    const float A = r * (-g - (ENT ? h * fmaf(e.rest, kLn2, H) : 0.f)), B = r * -h * kLn2;
    auto slope = [&](float t) {
        const float q = __builtin_amdgcn_exp2f(t);
        return q * (ENT ? fmaf(B, fmaxf(t, kFloor), A) : A);
    };
    // (of another piece's token: no vector of this one)
    const int in = token - s.head, token_vec = s.inside(token) ? in / V : -1, token_at = in % V;
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int j = j0 + u * N;
        if (j >= s.nvec) continue;
        float f[V], t[V];
#pragma unroll
        for (int i = 0; i < V; i++) f[i] = element<T>(v[u], i);
        e.of<V>(f, t);
#pragma unroll
        for (int i = 0; i < V; i++) f[i] = slope(t[i]);
        if (j == token_vec)
#pragma unroll
            for (int i = 0; i < V; i++) f[i] += i == token_at ? hot : 0.f;
        store_vector<T>(out + s.head, begin + u * N, tid, f);
    }
    if (edge) {
        float t;
        e.of<1>(&x, &t);
        store1<T>(out + s.edge(tid), slope(t) + (s.edge(tid) == token ? hot : 0.f));
    }
}

template <typename T, int N>
void run_kind(const VocabLaunch &a, hipStream_t stream)
{
    if (a.top) {
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

struct RunGrad {
    VocabLaunch a;
    hipStream_t stream;
    template <typename T, bool ENT> void go()
    {
        const int pieces = std::max(1, (vectors(a) + kGradVectors * kGradThreads - 1) / (kGradVectors * kGradThreads));
        a.splits = pieces;
        by_rows(a, pieces, kGradThreads, [&](const VocabLaunch &b, dim3 grid, unsigned) {
            if (b.stream) hipLaunchKernelGGL((k_logprobs_grad<T, ENT, true>), grid, dim3(kGradThreads), 0, stream, b);
            else hipLaunchKernelGGL((k_logprobs_grad<T, ENT, false>), grid, dim3(kGradThreads), 0, stream, b);
        });
    }
    template <typename T> void operator()()
    {
        if (a.dentropy) go<T, true>();
        else go<T, false>();
    }
};

}  // namespace

// Workgroups of a compute unit that hold rows of n vectors: as many as their registers (and for one wavefront's up to 256 vectors their LDS) leave room for:
// one more of 256 threads, which does not fit, has to wait for the others to end (bfloat16 [4096, 10000] 54.8 us for 46.9).  32 in place of 16 wavefronts of their own:
// [16384, 2000] 45.5 for 48.
static int held_workgroups(int threads, int n, int entries)
{
    if (threads == 64) return n <= 256 && entries <= 64 ? 32 : 16;
    return n <= 2048 ? 5 : n <= 4096 ? 4 : n <= 8192 ? 2 : 1;
}

void plan_vocab(VocabLaunch &a, int units)
{
    const int n = vectors(a);
    // however few the rows are: losses first and gradients behind them, which parts of rows may share, take longer (20 entries and a tail, one row of 8192 vectors 14.0 us held
    // and 18.9 apart in bfloat16, 10.8 and 16.3 in float32; 32 rows of 12288 17.2 and 19.3, 13.8 and 18.2; 128 of 16384 21.0 and 30.6, 17.3 and 28.5), but for up to 32 rows of
    // 16384 vectors of 16 bits (19 to 20 and 16 to 19)
    a.held = a.entries && a.dlogits && a.loss && n <= kHeldVectors;
    // a wavefront a row where there are wavefronts for all compute units, bfloat16: [16384, 2048] 19.4 us, on 256 threads 40.9; [16384, 4096] 31.7 and 52.7;
    // [8192, 12000] 39.2 and 43.7; but [4096, 32768] 50.5 and 45.8, [600, 16000] 9.4 and 8.2.  Alternatives of rows above 256 vectors need the 256 threads' pieces.
    a.threads = n <= 256 || (!a.top && n <= 2048 && a.r.rows >= (uint32_t)(4 * units)) ? 64 : 256;
    // few rows are shared by workgroups that take 1024 vectors at least, where a second launch costs less than what it saves: one row of 131072 float32
    // takes 20 us whole, 7.7 in 32 parts; eight rows of 50257 bfloat16 8.1 us whole (and 8.1 in 6 parts), with 20 alternatives, which need the
    // second launch anyway, 17.3 and 12.2
    a.splits = 1;
    // a wavefront holds a row where each SIMD has more than one (bfloat16, 20 entries: [2048, 2000] 12.7 us, [1500, 2000] 12.1, on 256 threads 12.8 and 14.4; but
    // [1024, 2000] 11.4 and 9.8, [64, 2000] 9.9 and 7.5), a long one two: [8192, 4000] 38 and 55, [8192, 7000] 62 and 73, [2048, 4000] 16.8 and 18.3,
    // [2048, 7000] 22.1 and 22.2, but [1024, 4000] 14.5 and 10.9
    if (a.held) a.threads = n <= 64 || (n <= 256 && a.r.rows > (uint32_t)(4 * units)) || (n <= 1024 && a.r.rows >= (uint32_t)(8 * units)) ? 64 : 256;
    if (a.r.rows < (uint32_t)units && n >= (a.top ? 2048 : 12288) && !a.held && (a.loss || !a.dlogits))
        a.splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(64, n / 1024), (2 * units + a.r.rows - 1) / a.r.rows));
    // (the largest a row can have: its vectors begin at its first whole 16 bytes)
    if (a.top && a.threads == 256) a.pieces_per_part = ((n + a.splits - 1) / a.splits + kPieceTrips * 256 - 1) / (kPieceTrips * 256) * (256 / kPieceLanes);
    // workgroups that stay: as many as share the rows evenly
    const int64_t room = (int64_t)units * (a.held ? held_workgroups(a.threads, n, a.entries) : 2048 / a.threads), items = (int64_t)a.r.rows * a.splits, each = (items + room - 1) / room;
    a.resident = each ? (int)((items + each - 1) / each) : 0;
    // logits that the memory-side cache cannot keep pass it by: bfloat16 [4096, 32768] 51.7 us, passing 45.6; [2048, 32768] 27.2 and 24.7; [1024, 32768] 14.3 and 15.7
    a.stream = (int64_t)a.r.rows * a.r.cols * (a.dtype == EWF_F32 ? 4 : 2) >= (int64_t)128 << 20;
}

void launch_token_logprobs(const VocabLaunch &a, hipStream_t stream) { by_type(a.dtype, RunRows{a, stream}); }
void launch_token_logprobs_grad(const VocabLaunch &a, hipStream_t stream) { by_type(a.dtype, RunGrad{a, stream}); }

}  // namespace ewf
