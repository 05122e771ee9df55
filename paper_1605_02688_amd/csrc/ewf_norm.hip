// Layer normalisation, forward and backward.
#include "ewf_ops_device.h"

namespace ewf {

namespace {

// A row is held by TPR threads, NV vectors of 16 bytes each: vector j of thread t begins at element
// (j TPR + t) V.  Workgroups of 256 threads (1024 where a row needs them) hold G = threads / TPR rows at once.
template <int TPR> struct Shape {
    static constexpr int threads = TPR > 256 ? TPR : 256;
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

// ------------------------------------------------------------------ forward

template <typename T, int TPR, int NV>
__global__ void __launch_bounds__(Shape<TPR>::threads) k_norm(NormLaunch a)
{
    constexpr int V = Vec16<T>::V, G = Shape<TPR>::groups;
    typedef typename T::raw raw;
    __shared__ float red[2][Shape<TPR>::waves];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, cols = a.r.cols;
    const bool pf32 = a.param_dtype == EWF_F32, e4m3 = a.code_dtype == EWF_E4M3;
    float w[NV][V], b[NV][V];
#pragma unroll
    for (int j = 0; j < NV; j++) {
        const int c = (j * TPR + t) * V;
#pragma unroll
        for (int e = 0; e < V; e++) { w[j][e] = 1.f; b[j][e] = 0.f; }
        if (a.weight) load_params<T>(a.weight, pf32, c, cols, w[j]);
        if (a.bias) load_params<T>(a.bias, pf32, c, cols, b[j]);
    }
    u32x4 x[NV];
    auto fetch = [&](uint32_t row) {
        const raw *p = (const raw *)a.x + row_offset(a.r, row, a.sx);
#pragma unroll
        for (int j = 0; j < NV; j++) x[j] = load_part<T>(p, (j * TPR + t) * V, cols, a.nt);
    };
    uint32_t base = blockIdx.x * G;
    if (base + g < a.r.rows) fetch(base + g);
    // (the same number of trips in every thread of a workgroup: row_sum synchronises it)
    for (; base < a.r.rows; base += gridDim.x * G) {
        const uint32_t row = base + g;
        const bool live = row < a.r.rows;
        float s = 0.f;
        u32x4 now[NV];
#pragma unroll
        for (int j = 0; j < NV; j++) {
            now[j] = live ? x[j] : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int e = 0; e < V; e++) s += element<T>(now[j], e);
        }
        const uint64_t next = (uint64_t)row + (uint64_t)gridDim.x * G;
        if (next < a.r.rows) fetch((uint32_t)next);      // in flight during this row's sums
        const float mean = row_sum<TPR>(s, red[0]) / (float)cols;
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * TPR + t) * V;
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float d = element<T>(now[j], e) - mean;
                if (c + e < cols) q = fmaf(d, d, q);
            }
        }
        const float rstd = 1.f / sqrtf(row_sum<TPR>(q, red[1]) / (float)cols + a.eps);
        raw *y = (raw *)a.y + (live ? row_offset(a.r, row, a.sy) : 0);
        uint8_t *codes = a.codes + (live ? row_offset(a.r, row, a.scodes) : 0);
        uint8_t *scales = a.scales + (live ? row_offset(a.r, row, a.sscales) : 0);
        const int end = live ? cols : 0;
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * TPR + t) * V;
            float n[V], o[V];
#pragma unroll
            for (int e = 0; e < V; e++) {
                n[e] = (element<T>(now[j], e) - mean) * rstd;
                o[e] = fmaf(n[e], w[j][e], b[j][e]);
            }
            if (c < end) store_part<T>(y, c, end, pack16<T>(o), a.nt);
            if (a.codes) {
#pragma unroll
                for (int e = 0; e < V; e++) n[e] = c + e < end ? n[e] : 0.f;
                keep_part<V>(codes, scales, c, end, n, e4m3);
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
            const u32x4 v = load_part<T>(x, (int)(at + threadIdx.x * V), cols, false);
            float part = 0.f;
#pragma unroll
            for (int e = 0; e < V; e++) part += element<T>(v, e);
            s += part;
        }
        const float mean = row_sum<kLongThreads>(s, red[0]) / (float)cols;
        for (int64_t at = 0; at < cols; at += step) {
            const int c = (int)(at + threadIdx.x * V);
            const u32x4 v = load_part<T>(x, c, cols, false);
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
            const u32x4 v = load_part<T>(x, c, cols, false);
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
            if (c < cols) store_part<T>(y, c, cols, pack16<T>(o), a.nt);
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
template <typename T, int TPR, int NV>
__global__ void __launch_bounds__(Shape<TPR>::threads) k_norm_grad(NormLaunch a)
{
    constexpr int V = Vec16<T>::V, G = Shape<TPR>::groups;
    typedef typename T::raw raw;
    __shared__ float red[2][Shape<TPR>::waves];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, cols = a.r.cols;
    const bool sums = a.partials != nullptr;
    float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
    for (int j = 0; j < NV; j++) {
#pragma unroll
        for (int e = 0; e < V; e++) { w[j][e] = 1.f; dw[j][e] = 0.f; db[j][e] = 0.f; }
        if (a.weight) load_params<T>(a.weight, a.param_dtype == EWF_F32, (j * TPR + t) * V, cols, w[j]);
    }
    u32x4 dy[NV], x[NV];
    u32x2 code[NV];
    uint32_t byte[NV];
    float mean = 0.f, rstd = 0.f;
    auto fetch = [&](uint32_t row) {
        const raw *pd = (const raw *)a.dy + row_offset(a.r, row, a.sdy);
#pragma unroll
        for (int j = 0; j < NV; j++) dy[j] = load_part<T>(pd, (j * TPR + t) * V, cols, a.nt);
        if (a.codes) {
            const uint8_t *pc = a.codes + row_offset(a.r, row, a.scodes), *ps = a.scales + row_offset(a.r, row, a.sscales);
#pragma unroll
            for (int j = 0; j < NV; j++) {
                const int c = (j * TPR + t) * V;
                code[j] = load_codes<V>(pc, c, cols);
                byte[j] = c < cols ? ps[c / kKeepBlock] : 0;
            }
        } else {
            const raw *px = (const raw *)a.x + row_offset(a.r, row, a.sx);
#pragma unroll
            for (int j = 0; j < NV; j++) x[j] = load_part<T>(px, (j * TPR + t) * V, cols, a.nt);
            mean = a.mean[row_offset(a.r, row, a.smean)];
        }
        rstd = a.rstd[row_offset(a.r, row, a.srstd)];
    };
    for (uint32_t base = blockIdx.x * G; base < a.r.rows; base += gridDim.x * G) {
        const uint32_t row = base + g;
        const bool live = row < a.r.rows;
        if (live) fetch(row);
        const int end = live ? cols : 0;
        float n[NV][V], s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * TPR + t) * V;
            normalised<T>(a, x[j], mean, rstd, code[j], byte[j], n[j]);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const bool in = c + e < end;
                const float d = in ? element<T>(dy[j], e) : 0.f, ne = in ? n[j][e] : 0.f, gr = d * w[j][e];
                n[j][e] = ne;
                s1 += gr;
                s2 = fmaf(gr, ne, s2);
                dw[j][e] = fmaf(d, ne, dw[j][e]);
                db[j][e] += d;
            }
        }
        const float m1 = row_sum<TPR>(s1, red[0]) / (float)cols;
        const float m2 = row_sum<TPR>(s2, red[1]) / (float)cols;
        raw *dx = (raw *)a.dx + (live ? row_offset(a.r, row, a.sdx) : 0);
#pragma unroll
        for (int j = 0; j < NV; j++) {
            const int c = (j * TPR + t) * V;
            float o[V];
#pragma unroll
            for (int e = 0; e < V; e++) o[e] = rstd * (fmaf(-n[j][e], m2, element<T>(dy[j], e) * w[j][e] - m1));
            if (c < end) store_part<T>(dx, c, end, pack16<T>(o), a.nt);
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
                    store16<F32>(mine + c + e, pack16<F32>(&dw[j][e]), false);
                    store16<F32>(mine + a.padded + c + e, pack16<F32>(&db[j][e]), false);
                }
        }
    } else {
        constexpr int L = TPR < 64 ? TPR : 64;                      // lanes of a wavefront with columns of their own
        constexpr int groups = TPR <= 64 ? Shape<TPR>::waves : G;   // rows left
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
            for (int c = threadIdx.x; c < a.padded; c += Shape<TPR>::threads) mine[part * a.padded + c] = sum[c];
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
            const u32x4 dy = load_part<T>(pd, c, cols, false);
            u32x4 x = {0u, 0u, 0u, 0u};
            u32x2 code = {0u, 0u};
            uint32_t byte = 0;
            if (!a.codes) x = load_part<T>(px, c, cols, false);
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
            if (c < cols) store_part<T>(dx, c, cols, pack16<T>(o), a.nt);
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
        const u32x4 dy = load_part<T>((const raw *)a.dy + row_offset(a.r, row, a.sdy), c, cols, false);
        u32x4 x = {0u, 0u, 0u, 0u};
        u32x2 code = {0u, 0u};
        uint32_t byte = 0;
        float mean = 0.f;
        if (!a.codes) {
            x = load_part<T>((const raw *)a.x + row_offset(a.r, row, a.sx), c, cols, false);
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
        store16<F32>(mine + c + e, pack16<F32>(&dw[e]), false);
        store16<F32>(mine + a.padded + c + e, pack16<F32>(&db[e]), false);
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
        for (; k + 3 * kFinishWaves < a.blocks; k += 4 * kFinishWaves) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] = p[(int64_t)(k + i * kFinishWaves) * wide];
            s += (v[0] + v[1]) + (v[2] + v[3]);
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

// The threads of a row: the fewest that hold it in four vectors each (0: none do).  At least the 32 / V lanes
// that share a scale.
int row_threads(int cols, int V, int most)
{
    const int need = (cols + V - 1) / V;
    for (int tpr : {kKeepBlock / V, 16, 64, 256}) if (need <= 4 * tpr) return tpr;
    return need <= most * 1024 ? 1024 : 0;
}

template <typename F, typename T, int TPR>
bool with_vectors(F &&f, int need, int most)
{
    if (need <= TPR) return f.template operator()<T, TPR, 1>(), true;
    if (need <= 2 * TPR) return f.template operator()<T, TPR, 2>(), true;
    if (need <= 4 * TPR && most >= 4) return f.template operator()<T, TPR, 4>(), true;
    return false;
}

// Calls f<T, TPR, NV>() for the row's shape; false where no workgroup holds it.
template <typename T, typename F>
bool with_shape(F &&f, int cols, int most)
{
    constexpr int V = Vec16<T>::V;
    const int need = (cols + V - 1) / V;
    switch (row_threads(cols, V, most)) {
    case kKeepBlock / V: return with_vectors<F, T, kKeepBlock / V>(f, need, 4);
    case 16: return with_vectors<F, T, 16>(f, need, 4);
    case 64: return with_vectors<F, T, 64>(f, need, 4);
    case 256: return with_vectors<F, T, 256>(f, need, 4);
    case 1024: return with_vectors<F, T, 1024>(f, need, most);
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

// Workgroups of 1024 threads have 128 registers a thread: what they hold of a row in the backward pass (the
// elements, the parameters and two sums each) must fit those.
int grad_vectors(int dtype) { return dtype == EWF_F32 ? 4 : 2; }

uint32_t at_most(uint64_t n, uint32_t cap) { return (uint32_t)(n < cap ? n : cap); }

struct Forward {
    const NormLaunch &a;
    hipStream_t stream;
    template <typename T, int TPR, int NV> void operator()() const
    {
        constexpr int G = Shape<TPR>::groups;
        const uint32_t blocks = at_most(((uint64_t)a.r.rows + G - 1) / G, 2048);
        hipLaunchKernelGGL((k_norm<T, TPR, NV>), dim3(blocks), dim3(Shape<TPR>::threads), 0, stream, a);
    }
    template <typename T> void operator()() const
    {
        if (with_shape<T>(*this, a.r.cols, 4)) return;
        hipLaunchKernelGGL(k_norm_long<T>, dim3(at_most(a.r.rows, 4096)), dim3(kLongThreads), 0, stream, a);
    }
};

struct Backward {
    const NormLaunch &a;
    hipStream_t stream;
    template <typename T, int TPR, int NV> void operator()() const
    {
        hipLaunchKernelGGL((k_norm_grad<T, TPR, NV>), dim3(a.blocks), dim3(Shape<TPR>::threads), 0, stream, a);
    }
    template <typename T> void operator()() const
    {
        if (a.r.rows && !with_shape<T>(*this, a.r.cols, grad_vectors(a.dtype))) {
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

}  // namespace

void launch_layer_norm(const NormLaunch &a, hipStream_t stream) { with_type(Forward{a, stream}, a.dtype); }

void plan_layer_norm_grad(NormLaunch &a, int units)
{
    const int V = a.dtype == EWF_F32 ? 4 : 8;
    a.padded = (a.r.cols + 7) / 8 * 8;
    const int tpr = row_threads(a.r.cols, V, grad_vectors(a.dtype));
    const int groups = tpr == 0 ? 1 : tpr > 256 ? 1 : 256 / tpr;
    const uint64_t trips = ((uint64_t)a.r.rows + groups - 1) / groups;
    a.blocks = (int)at_most(trips, (uint32_t)(tpr == 0 ? 64 : tpr > 256 ? units : 4 * units));
}

void launch_layer_norm_grad(const NormLaunch &a, hipStream_t stream) { with_type(Backward{a, stream}, a.dtype); }

}  // namespace ewf
