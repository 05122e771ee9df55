// Layer normalisation, forward and backward.
//
// Forward: mean, then the mean square of what is left of it, from the row in registers: two sums in turn, because a
// sum of squares about zero loses the variance of rows far from it.  Backward: with g = dy weight and n the normalised
// row, dx = rstd (g - mean(g) - n mean(g n)); two sums along the row, and down the columns the sums of dy n and dy.
// Memory bounds both: bfloat16 [16384, 4096] forward 50 us for 268 MB (without its sums 51), backward 72 us for 403 MB and
// 4 for the fold of the column sums.
#include "ewf_ops_device.h"

namespace ewf {

namespace {

// A row is held by TPR threads, NV vectors of 16 bytes each: vector j of thread t begins at element
// (j TPR + t) V.  A workgroup holds G = threads / TPR rows at once.
constexpr int kThreads = 512;
template <int TPR> struct Held {
    static constexpr int threads = TPR > kThreads ? TPR : kThreads;
    static constexpr int groups = threads / TPR;
    static constexpr int waves = threads / 64;
};

// The sum over a row's threads, in each of them; two calls in turn need two arrays.
template <int TPR>
EWF_OPS_DEV float row_sum(float x, float *lds)
{
    if constexpr (TPR <= 64) return group_sum<TPR>(x);
    else {
        constexpr int W = TPR / 64;
        x = group_sum<64>(x);
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) lds[wave] = x;
        __syncthreads();
        const float *mine = lds + wave / W * W;
        float s = mine[0];
#pragma unroll
        for (int i = 1; i < W; i++) s += mine[i];
        return s;
    }
}

// Vector j of thread t once its access is there; vectors that lie inside the row in all threads are whole.
template <typename T, bool CUT, int TPR>
EWF_OPS_DEV u32x4 settle(u32x4 v, int j, int t, int cols)
{
    if (CUT && (j + 1) * TPR * Vec16<T>::V > cols) v = settle_part<T, CUT>(v, (j * TPR + t) * Vec16<T>::V, cols);
    return v;
}

// ------------------------------------------------------------------ forward

template <typename T, int TPR, int NV, bool CUT, bool KEPT>
__global__ void __launch_bounds__(Held<TPR>::threads) k_norm(NormLaunch a)
{
    constexpr int V = Vec16<T>::V, G = Held<TPR>::groups;
    typedef typename T::raw raw;
    __shared__ float red[2][Held<TPR>::waves];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, cols = a.r.cols;
    const bool pf32 = a.param_dtype == EWF_F32, e4m3 = a.code_dtype == EWF_E4M3;
    float w[NV][V], b[NV][V];
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * TPR + t) * V;
#pragma unroll
        for (int e = 0; e < V; e++) { w[j][e] = 1.f; b[j][e] = 0.f; }
        if (a.weight) load_params<T, CUT>(a.weight, pf32, c, cols, w[j]);
        if (a.bias) load_params<T, CUT>(a.bias, pf32, c, cols, b[j]);
    }
    u32x4 next[NV];
    auto fetch = [&](uint32_t row) {
        const raw *p = (const raw *)a.x + row_offset(a.r, row, a.sx);
#pragma unroll
        for (int j = 0; j < NV; j++) next[j] = fetch_part<T, CUT>(p, (j * TPR + t) * V, cols);
    };
#pragma unroll
    for (int j = 0; j < NV; j++) next[j] = u32x4{0u, 0u, 0u, 0u};
    uint32_t base = blockIdx.x * G;
    if (base + g < a.r.rows) fetch(base + g);
    // (the same number of trips in every thread of a workgroup: row_sum synchronises it)
    for (; base < a.r.rows; base += gridDim.x * G) {
        const uint32_t row = base + g;
        const bool live = row < a.r.rows;
        float f[NV][V], s = 0.f;                         // the elements; less the mean
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const u32x4 x = settle<T, CUT, TPR>(next[j], j, t, cols);
#pragma unroll
            for (int e = 0; e < V; e++) { f[j][e] = element<T>(x, e); s += f[j][e]; }        // (zeros behind the row's end)
        }
        const uint64_t then = (uint64_t)row + (uint64_t)gridDim.x * G;
        if (then < a.r.rows) fetch((uint32_t)then);      // in flight during this row
        const float mean = row_sum<TPR>(s, red[0]) / (float)cols;
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * TPR + t) * V;
            float part = 0.f;
#pragma unroll
            for (int e = 0; e < V; e++) {
                f[j][e] -= mean;
                if (!CUT || c + e < cols) part = fmaf(f[j][e], f[j][e], part);
            }
            if (!CUT && c >= cols) part = 0.f;
            q += part;
        }
        const float rstd = 1.f / sqrtf(row_sum<TPR>(q, red[1]) / (float)cols + a.eps);
        const int end = live ? cols : 0;
        const uint32_t at = live ? row : 0;
        raw *y = (raw *)a.y + row_offset(a.r, at, a.sy);
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * TPR + t) * V;
            float n[V], o[V];
#pragma unroll
            for (int e = 0; e < V; e++) {
                n[e] = f[j][e] * rstd;
                o[e] = fmaf(n[e], w[j][e], b[j][e]);
            }
            if (c < end) store_part<T, CUT>(y, c, end, pack16<T>(o));
            if constexpr (KEPT) {
                if (CUT || c >= end)
#pragma unroll
                    for (int e = 0; e < V; e++) n[e] = c + e < end ? n[e] : 0.f;
                keep_part<V, CUT>(a.codes + row_offset(a.r, at, a.scodes), a.scales + row_offset(a.r, at, a.sscales), c, end, n, e4m3);
            }
        }
        if (live && t == 0) {
            if (a.mean) a.mean[row_offset(a.r, row, a.smean)] = mean;
            if (a.rstd) a.rstd[row_offset(a.r, row, a.srstd)] = rstd;
        }
    }
}

// Rows that no workgroup holds: three sweeps over a row, the second and third mostly from the caches.
constexpr int kLongThreads = 1024;

template <typename T>
__global__ void __launch_bounds__(kLongThreads) k_norm_long(NormLaunch a)
{
    constexpr int V = Vec16<T>::V;
    constexpr int64_t step = (int64_t)kLongThreads * V;
    typedef typename T::raw raw;
    __shared__ float red[2][kLongThreads / 64];
    const int cols = a.r.cols;
    const bool pf32 = a.param_dtype == EWF_F32, e4m3 = a.code_dtype == EWF_E4M3;
    for (uint32_t row = blockIdx.x; row < a.r.rows; row += gridDim.x) {
        const raw *x = (const raw *)a.x + row_offset(a.r, row, a.sx);
        raw *y = (raw *)a.y + row_offset(a.r, row, a.sy);
        uint8_t *codes = a.codes + row_offset(a.r, row, a.scodes), *scales = a.scales + row_offset(a.r, row, a.sscales);
        float s = 0.f, q = 0.f;
        for (int64_t at = 0; at < cols; at += step) {
            const u32x4 v = load_part<T>(x, (int)(at + threadIdx.x * V), cols);
            float part = 0.f;
#pragma unroll
            for (int e = 0; e < V; e++) part += element<T>(v, e);
            s += part;
        }
        const float mean = row_sum<kLongThreads>(s, red[0]) / (float)cols;
        for (int64_t at = 0; at < cols; at += step) {
            const int c = (int)(at + threadIdx.x * V);
            const u32x4 v = load_part<T>(x, c, cols);
            float part = 0.f;
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float d = element<T>(v, e) - mean;
                if (c + e < cols) part = fmaf(d, d, part);
            }
            q += part;
        }
        const float rstd = 1.f / sqrtf(row_sum<kLongThreads>(q, red[1]) / (float)cols + a.eps);
        for (int64_t at = 0; at < cols; at += step) {
            const int c = (int)(at + threadIdx.x * V);
            const u32x4 v = load_part<T>(x, c, cols);
            float n[V], o[V], w[V], b[V];
#pragma unroll
            for (int e = 0; e < V; e++) { w[e] = 1.f; b[e] = 0.f; }
            if (a.weight) load_params<T>(a.weight, pf32, c, cols, w);
            if (a.bias) load_params<T>(a.bias, pf32, c, cols, b);
#pragma unroll
            for (int e = 0; e < V; e++) {
                n[e] = (element<T>(v, e) - mean) * rstd;
                o[e] = fmaf(n[e], w[e], b[e]);
            }
            if (c < cols) store_part<T>(y, c, cols, pack16<T>(o));
            if (a.codes) {
#pragma unroll
                for (int e = 0; e < V; e++) n[e] = c + e < cols ? n[e] : 0.f;
                keep_part<V>(codes, scales, c, cols, n, e4m3);
            }
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row_offset(a.r, row, a.smean)] = mean;
            if (a.rstd) a.rstd[row_offset(a.r, row, a.srstd)] = rstd;
        }
    }
}

// ------------------------------------------------------------------ backward

// The normalised elements n of a lane's vector: from x, or from 8 bits.
template <typename T>
EWF_OPS_DEV void normalised(const NormLaunch &a, u32x4 x, float mean, float rstd, u32x2 code, uint32_t byte, float *n)
{
    constexpr int V = Vec16<T>::V;
    if (a.codes) decode_part<V>(code, byte, a.code_dtype == EWF_E4M3, n);
    else {
#pragma unroll
        for (int e = 0; e < V; e++) n[e] = (element<T>(x, e) - mean) * rstd;
    }
}

// One sweep over dy and x: a workgroup takes rows in turn and its threads keep their columns' sums for dweight and
// dbias in registers; what remains across workgroups is one partial per workgroup, folded by k_norm_finish.
// Rows that are cut: registers for two workgroups a unit, up to 512 threads of two vectors (without the bound: float16 from 8 bits [20011,
// 1001] 33.9 us and 44.9, [61060, 25] 18.6 and 25.8; from x bfloat16 [8192, 4001] 44.6 and 51.4).  What does not fit spills: in 16 bits from
// codes 2 to 8 registers, on 512 threads 20 (float16 [8192, 7001] writes 165 MB for 143), from x at most 4.  Workgroups of 1024
// threads hold 128 registers a thread whatever is asked for: whole rows spill 8 to 10 (bfloat16 [8192, 16384] 248 us, 336 MB written for 302),
// cut ones 73 from x and 220 to 234 from codes (float16 [143, 14170] 17 and 25 us, 37 and 61 MB written for 20).
template <typename T, int TPR, int NV, bool CUT, bool KEPT>
__global__ void __launch_bounds__(Held<TPR>::threads, CUT && NV == 2 && TPR <= kThreads ? 4 : 1) k_norm_grad(NormLaunch a)
{
    constexpr int V = Vec16<T>::V, G = Held<TPR>::groups;
    typedef typename T::raw raw;
    __shared__ float red[2][Held<TPR>::waves];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, cols = a.r.cols;
    const bool sums = a.partials != nullptr;
    float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
    for (int j = 0; j < NV; j++) {
#pragma unroll
        for (int e = 0; e < V; e++) { w[j][e] = 1.f; dw[j][e] = 0.f; db[j][e] = 0.f; }
        if (a.weight) load_params<T, CUT>(a.weight, a.param_dtype == EWF_F32, (j * TPR + t) * V, cols, w[j]);
    }
    // (workgroups of 1024 threads have 128 registers a thread, which do not hold a second row)
    constexpr bool kAhead = TPR < 1024;
    struct Row {
        u32x4 dy[NV], x[NV];
        u32x2 code[NV];
        uint32_t byte[NV];
        float mean, rstd;
    } next;
    auto fetch = [&](uint32_t row) {
        const raw *pd = (const raw *)a.dy + row_offset(a.r, row, a.sdy);
        next.rstd = a.rstd[row_offset(a.r, row, a.srstd)];
        next.mean = 0.f;
        if constexpr (KEPT) {
            const uint8_t *pc = a.codes + row_offset(a.r, row, a.scodes), *ps = a.scales + row_offset(a.r, row, a.sscales);
#pragma unroll
            for (int j = 0; j < NV; j++) {
                const int c = (j * TPR + t) * V;
                next.dy[j] = fetch_part<T, CUT>(pd, c, cols);
                next.code[j] = load_codes<V, CUT>(pc, c, cols);
                next.byte[j] = c < cols ? ps[c / kKeepBlock] : 0;
            }
        } else {
            const raw *px = (const raw *)a.x + row_offset(a.r, row, a.sx);
            next.mean = a.mean[row_offset(a.r, row, a.smean)];
#pragma unroll
            for (int j = 0; j < NV; j++) {
                next.dy[j] = fetch_part<T, CUT>(pd, (j * TPR + t) * V, cols);
                next.x[j] = fetch_part<T, CUT>(px, (j * TPR + t) * V, cols);
            }
        }
    };
    uint32_t base = blockIdx.x * G;
    if (kAhead && base + g < a.r.rows) fetch(base + g);
    for (; base < a.r.rows; base += gridDim.x * G) {
        const uint32_t row = base + g;
        const bool live = row < a.r.rows;
        if (!kAhead && live) fetch(row);
        Row now = next;
        if constexpr (CUT)
#pragma unroll
            for (int j = 0; j < NV; j++) {
                now.dy[j] = settle<T, CUT, TPR>(now.dy[j], j, t, cols);
                if constexpr (!KEPT) now.x[j] = settle<T, CUT, TPR>(now.x[j], j, t, cols);
            }
        const uint64_t then = (uint64_t)row + (uint64_t)gridDim.x * G;
        if (kAhead && then < a.r.rows) fetch((uint32_t)then);   // in flight during this row
        const float rstd = now.rstd;
        // g = dy weight and n = c unit, from 8 bits as they stand (unit 1), from x with c = x - mean and unit = rstd, which is multiplied
        // in outside the row's sum: behind the row's end dy is zero, but -mean rstd may be infinite where the row's own n are not (rows
        // of one value beyond 10^36).  No sum leaves the range by it: where c passes 2^64 the forward pass's squares overflow.
        // c and g are kept for the second half, or, where rows are cut, computed again (kernels of rows that are cut need the
        // registers: float16 [20011, 1001] 40 us and 58, where two workgroups share a unit and where they do not; bfloat16
        // [16384, 4096], kept, 77, computed again, 80)
        const float unit = KEPT ? 1.f : rstd;
        float gr[NV][V], c[NV][V], s1 = 0.f, s2 = 0.f;
        auto elements = [&](int j) {
            if constexpr (KEPT) decode_part<V>(now.code[j], now.byte[j], a.code_dtype == EWF_E4M3, c[j]);
#pragma unroll
            for (int e = 0; e < V; e++) {
                if constexpr (!KEPT) c[j][e] = element<T>(now.x[j], e) - now.mean;
                gr[j][e] = element<T>(now.dy[j], e) * w[j][e];
            }
        };
        if (live) {
#pragma unroll
            for (int j = 0; j < NV; j++) {
                elements(j);
#pragma unroll
                for (int e = 0; e < V; e++) {
                    const float d = element<T>(now.dy[j], e);
                    s1 += gr[j][e];
                    s2 = fmaf(gr[j][e], c[j][e], s2);
                    dw[j][e] = fmaf(d * unit, c[j][e], dw[j][e]);
                    db[j][e] += d;
                }
            }
        }
        const float m1 = row_sum<TPR>(s1, red[0]) / (float)cols;
        const float m2 = row_sum<TPR>(s2 * unit, red[1]) / (float)cols * unit;
        if (!live) continue;
        raw *dx = (raw *)a.dx + row_offset(a.r, row, a.sdx);
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int at = (j * TPR + t) * V;
            float o[V];
            if constexpr (CUT) elements(j);
#pragma unroll
            for (int e = 0; e < V; e++) o[e] = rstd * fmaf(-c[j][e], m2, gr[j][e] - m1);
            if (at < cols) store_part<T, CUT>(dx, at, cols, pack16<T>(o));
        }
    }
    if (!sums) return;
    // rows of the same workgroup, in the order of their threads: lanes of a wavefront first, then wavefronts
    if constexpr (TPR < 64) {
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int e = 0; e < V; e++)
#pragma unroll
                for (int m = TPR; m < 64; m *= 2) { dw[j][e] += __shfl_xor(dw[j][e], m); db[j][e] += __shfl_xor(db[j][e], m); }
    }
    float *mine = a.partials + (size_t)blockIdx.x * 2 * a.padded;
    if constexpr (G == 1) {
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * TPR + t) * V;
            if (c < a.padded)
#pragma unroll
                for (int e = 0; e < V; e += 4) {
                    store16<F32>(mine + c + e, pack16<F32>(&dw[j][e]));
                    store16<F32>(mine + a.padded + c + e, pack16<F32>(&db[j][e]));
                }
        }
    } else {
        constexpr int L = TPR < 64 ? TPR : 64;                      // lanes of a wavefront with columns of their own
        constexpr int groups = TPR <= 64 ? Held<TPR>::waves : G;   // rows left
        __shared__ float sum[NV * TPR * V];
        const int who = TPR <= 64 ? (int)(threadIdx.x >> 6) : g;
        const bool holds = (int)(threadIdx.x & 63) < L;
        for (int part = 0; part < 2; part++) {
            for (int turn = 0; turn < groups; turn++) {
                __syncthreads();
                if (who == turn && holds) {
#pragma unroll
                    for (int j = 0; j < NV; j++)
#pragma unroll
                        for (int e = 0; e < V; e++) {
                            const int c = (j * TPR + t) * V + e;
                            const float add = part ? db[j][e] : dw[j][e];
                            sum[c] = turn ? sum[c] + add : add;
                        }
                }
            }
            __syncthreads();
            for (int c = threadIdx.x; c < a.padded; c += Held<TPR>::threads) mine[part * a.padded + c] = sum[c];
        }
    }
}

// Rows that no workgroup holds: dx row by row in two sweeps, the sums column by column in a sweep of their own.
template <typename T>
__global__ void __launch_bounds__(kLongThreads) k_norm_grad_long(NormLaunch a)
{
    constexpr int V = Vec16<T>::V;
    constexpr int64_t step = (int64_t)kLongThreads * V;
    typedef typename T::raw raw;
    __shared__ float red[2][kLongThreads / 64];
    const int cols = a.r.cols;
    for (uint32_t row = blockIdx.x; row < a.r.rows; row += gridDim.x) {
        const raw *pd = (const raw *)a.dy + row_offset(a.r, row, a.sdy);
        const raw *px = (const raw *)a.x + row_offset(a.r, row, a.sx);
        const uint8_t *pc = a.codes + row_offset(a.r, row, a.scodes), *ps = a.scales + row_offset(a.r, row, a.sscales);
        raw *dx = (raw *)a.dx + row_offset(a.r, row, a.sdx);
        const float mean = a.codes ? 0.f : a.mean[row_offset(a.r, row, a.smean)], rstd = a.rstd[row_offset(a.r, row, a.srstd)];
        float gr[V], n[V];
        auto part = [&](int64_t at) {
            const int c = (int)(at + threadIdx.x * V);
            const u32x4 dy = load_part<T>(pd, c, cols);
            u32x4 x = {0u, 0u, 0u, 0u};
            u32x2 code = {0u, 0u};
            uint32_t byte = 0;
            if (!a.codes) x = load_part<T>(px, c, cols);
            else if (c < cols) { code = load_codes<V>(pc, c, cols); byte = ps[c / kKeepBlock]; }
            float w[V];
#pragma unroll
            for (int e = 0; e < V; e++) w[e] = 1.f;
            if (a.weight) load_params<T>(a.weight, a.param_dtype == EWF_F32, c, cols, w);
            normalised<T>(a, x, mean, rstd, code, byte, n);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const bool in = c + e < cols;
                gr[e] = in ? element<T>(dy, e) * w[e] : 0.f;
                n[e] = in ? n[e] : 0.f;
            }
            return c;
        };
        float s1 = 0.f, s2 = 0.f;
        for (int64_t at = 0; at < cols; at += step) {
            part(at);
            float p1 = 0.f, p2 = 0.f;
#pragma unroll
            for (int e = 0; e < V; e++) { p1 += gr[e]; p2 = fmaf(gr[e], n[e], p2); }
            s1 += p1;
            s2 += p2;
        }
        const float m1 = row_sum<kLongThreads>(s1, red[0]) / (float)cols, m2 = row_sum<kLongThreads>(s2, red[1]) / (float)cols;
        for (int64_t at = 0; at < cols; at += step) {
            const int c = part(at);
            float o[V];
#pragma unroll
            for (int e = 0; e < V; e++) o[e] = rstd * fmaf(-n[e], m2, gr[e] - m1);
            if (c < cols) store_part<T>(dx, c, cols, pack16<T>(o));
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) k_norm_grad_columns(NormLaunch a)
{
    constexpr int V = Vec16<T>::V;
    typedef typename T::raw raw;
    const int cols = a.r.cols, c = (int)((blockIdx.y * 256 + threadIdx.x) * V);
    if (c >= a.padded) return;
    float dw[V], db[V];
#pragma unroll
    for (int e = 0; e < V; e++) dw[e] = db[e] = 0.f;
    for (uint32_t row = blockIdx.x; row < a.r.rows; row += gridDim.x) {
        const u32x4 dy = load_part<T>((const raw *)a.dy + row_offset(a.r, row, a.sdy), c, cols);
        u32x4 x = {0u, 0u, 0u, 0u};
        u32x2 code = {0u, 0u};
        uint32_t byte = 0;
        float mean = 0.f;
        if (!a.codes) {
            x = load_part<T>((const raw *)a.x + row_offset(a.r, row, a.sx), c, cols);
            mean = a.mean[row_offset(a.r, row, a.smean)];
        } else if (c < cols) {
            code = load_codes<V>(a.codes + row_offset(a.r, row, a.scodes), c, cols);
            byte = a.scales[row_offset(a.r, row, a.sscales) + c / kKeepBlock];
        }
        float n[V];
        normalised<T>(a, x, mean, a.rstd[row_offset(a.r, row, a.srstd)], code, byte, n);
#pragma unroll
        for (int e = 0; e < V; e++) {
            const float d = element<T>(dy, e);
            if (c + e < cols) dw[e] = fmaf(d, n[e], dw[e]);
            db[e] += d;
        }
    }
    float *mine = a.partials + (size_t)blockIdx.x * 2 * a.padded;
#pragma unroll
    for (int e = 0; e < V; e += 4) {
        store16<F32>(mine + c + e, pack16<F32>(&dw[e]));
        store16<F32>(mine + a.padded + c + e, pack16<F32>(&db[e]));
    }
}

// Folds the workgroups' partials: 64 columns a workgroup, its wavefronts take the partials in turn.
constexpr int kFinishWaves = 16;

template <typename T>
__global__ void __launch_bounds__(kFinishWaves * 64) k_norm_finish(NormLaunch a)
{
    __shared__ float part[kFinishWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t at = (int64_t)blockIdx.x * 64 + lane, wide = 2 * (int64_t)a.padded;
    float s = 0.f;
    if (at < wide) {
        const float *p = a.partials + at;
        int k = wave;
        for (; k + 7 * kFinishWaves < a.blocks; k += 8 * kFinishWaves) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = p[(int64_t)(k + i * kFinishWaves) * wide];
            s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
        for (; k < a.blocks; k += kFinishWaves) s += p[(int64_t)k * wide];
    }
    part[wave][lane] = s;
    __syncthreads();
    if (wave || at >= wide) return;
    s = part[0][lane];
#pragma unroll
    for (int i = 1; i < kFinishWaves; i++) s += part[i][lane];
    const bool bias = at >= a.padded;
    const int64_t c = bias ? at - a.padded : at;
    void *out = bias ? a.dbias : a.dweight;
    if (!out || c >= a.r.cols) return;
    if (a.param_dtype == EWF_F32) ((float *)out)[c] = s;
    else store1<T>((typename T::raw *)out + c, s);
}

// ------------------------------------------------------------------ which kernel

// Threads and vectors a thread of a row.
struct RowShape { int threads, vectors; };

// The fewest vectors that hold the row, by 8 (the lanes that share a scale, at most) to 1024 threads of two, or 32 to 512
// threads of three (0: none do).  bfloat16 rows on T threads of three vectors and on 2 T of two, us: forward [16384, 4608] 61 and 66,
// [16384, 1400] 18.9 and 21.1, [16384, 6144] 77.6 and 77.7.  Backward three vectors take registers for their sums: worth it where two
// vectors of twice the threads would stand half empty ([16384, 4608] 86 and 98; [16384, 6144] 120 and 111, [16384, 1400] 35 and 33) and
// where that would be 1024 threads, whose registers do not hold two ([8192, 12000] 120 and 206); rows that are cut have none left
// over (float16 [20011, 1301] 82 and 67).
RowShape row_shape(int cols, int V, bool backward, bool kept)
{
    const int need = (cols + V - 1) / V;
    for (int tpr = 8; tpr <= 1024; tpr *= 2) {
        if (need <= 2 * tpr) return {tpr, 2};
        if (need > 3 * tpr || tpr < 32 || tpr > 512) continue;
        const bool cut = cols % V != 0;
        if (backward ? tpr == 512 || (2 * need <= 5 * tpr && !cut) : !cut && !kept) return {tpr, 3};
    }
    return {0, 0};
}

// Calls f<T, threads, vectors>() for the row's shape; false where no workgroup holds it.
template <typename T, typename F>
bool with_shape(F &&f, int cols, bool backward, bool kept)
{
    const RowShape s = row_shape(cols, Vec16<T>::V, backward, kept);
    switch (s.threads * 4 + s.vectors) {
#define EWF_ROW(TPR, NV) case TPR * 4 + NV: return f.template operator()<T, TPR, NV>(), true;
    EWF_ROW(8, 2) EWF_ROW(16, 2) EWF_ROW(32, 2) EWF_ROW(32, 3) EWF_ROW(64, 2) EWF_ROW(64, 3) EWF_ROW(128, 2) EWF_ROW(128, 3)
    EWF_ROW(256, 2) EWF_ROW(256, 3) EWF_ROW(512, 2) EWF_ROW(512, 3) EWF_ROW(1024, 2)
#undef EWF_ROW
    }
    return false;
}

template <typename F>
void with_type(F &&f, int dtype)
{
    if (dtype == EWF_F32) f.template operator()<F32>();
    else if (dtype == EWF_F16) f.template operator()<F16>();
    else f.template operator()<BF16>();
}

uint32_t at_most(uint64_t n, uint32_t cap) { return (uint32_t)(n < cap ? n : cap); }

template <bool CUT>
struct Forward {
    const NormLaunch &a;
    int units;
    hipStream_t stream;
    template <typename T, int TPR, int NV> void operator()() const
    {
        constexpr int G = Held<TPR>::groups;
        const dim3 grid(at_most(((uint64_t)a.r.rows + G - 1) / G, 2 * (uint32_t)units)), block(Held<TPR>::threads);
        if (a.codes) hipLaunchKernelGGL((k_norm<T, TPR, NV, CUT, true>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((k_norm<T, TPR, NV, CUT, false>), grid, block, 0, stream, a);
    }
    template <typename T> void operator()() const
    {
        if (with_shape<T>(*this, a.r.cols, false, a.codes)) return;
        hipLaunchKernelGGL(k_norm_long<T>, dim3(at_most(a.r.rows, 4096)), dim3(kLongThreads), 0, stream, a);
    }
};

template <bool CUT>
struct Backward {
    const NormLaunch &a;
    hipStream_t stream;
    template <typename T, int TPR, int NV> void operator()() const
    {
        const dim3 grid(a.blocks), block(Held<TPR>::threads);
        if (a.codes) hipLaunchKernelGGL((k_norm_grad<T, TPR, NV, CUT, true>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((k_norm_grad<T, TPR, NV, CUT, false>), grid, block, 0, stream, a);
    }
    template <typename T> void operator()() const
    {
        if (a.r.rows && !with_shape<T>(*this, a.r.cols, true, a.codes)) {
            // (the sums first: dx may lie over dy or x)
            const int per = 256 * Vec16<T>::V;
            if (a.partials)
                hipLaunchKernelGGL(k_norm_grad_columns<T>, dim3(a.blocks, (a.padded + per - 1) / per), dim3(256), 0, stream, a);
            hipLaunchKernelGGL(k_norm_grad_long<T>, dim3(at_most(a.r.rows, 4096)), dim3(kLongThreads), 0, stream, a);
        }
        if (a.dweight || a.dbias)
            hipLaunchKernelGGL(k_norm_finish<T>, dim3((2 * (uint64_t)a.padded + 63) / 64), dim3(kFinishWaves * 64), 0, stream, a);
    }
};

// Rows that end inside a vector of 16 bytes have kernels of their own.
bool is_cut(const NormLaunch &a) { return a.r.cols % (a.dtype == EWF_F32 ? 4 : 8) != 0; }

}  // namespace

void launch_layer_norm(const NormLaunch &a, int units, hipStream_t stream) 
{
    if (is_cut(a)) with_type(Forward<true>{a, units, stream}, a.dtype);
    else with_type(Forward<false>{a, units, stream}, a.dtype);
}

void plan_layer_norm_grad(NormLaunch &a, int units)
{
    const int V = a.dtype == EWF_F32 ? 4 : 8;
    a.padded = (a.r.cols + 7) / 8 * 8;
    const int tpr = row_shape(a.r.cols, V, true, a.codes).threads;
    const int groups = tpr == 0 || tpr > kThreads ? 1 : kThreads / tpr;
    const uint64_t trips = ((uint64_t)a.r.rows + groups - 1) / groups;
    // One workgroup of 512 threads for each unit, two where rows are cut (its kernels have the registers for two): bfloat16
    // [16384, 4096] 77 and 83 us, [16384, 1024] 26.6 and 28.7; float16 [20011, 1001] 53 and 40.  More leave more partials.
    const uint64_t most = tpr == 0 ? 64 : tpr <= kThreads && is_cut(a) ? 2 * units : units;
    // the fewest that take no more rows each: 513 trips by 512 workgroups are two trips for the longest, and by 257 as well
    const uint64_t each = (trips + most - 1) / most;
    a.blocks = each ? (int)((trips + each - 1) / each) : 0;
}

void launch_layer_norm_grad(const NormLaunch &a, hipStream_t stream) 
{
    if (is_cut(a)) with_type(Backward<true>{a, stream}, a.dtype);
    else with_type(Backward<false>{a, stream}, a.dtype);
}

}  // namespace ewf
