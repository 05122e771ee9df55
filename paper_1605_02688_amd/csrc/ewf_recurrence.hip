// Gated linear recurrence over time and its backward pass.
//
// A step is the map s -> f s + b of a channel's state, and maps compose: (F, B) after (f, b) is (F f, F b + B).
// Forward, in time:  s = h, f = f_t, b = i_t v_t, h_t = s.  Backward, against time:  with s_t = f_t G_t, what step t
// hands to step t - 1, G_t = dh_t + s_(t+1) and s_t = f_t s_(t+1) + f_t dh_t.  f lies in [0, 1], so that products of
// f never overflow whatever their number.
#include "ewf_ops_device.h"

namespace ewf {

namespace {

constexpr float kLog2E = 1.44269504f;
constexpr int kStrip = 64;               // channels of a workgroup: two a lane, 32 lanes

struct Pair { float x, y; };

// f = sigmoid(u) and 1 - f, both to within a few units in the last place: e = 2^(-u log2 e), f = 1 / (1 + e),
// 1 - f = e f.  e is kept finite (a gate of less than 2^-126 counts as that); a NaN stays one.
EWF_OPS_DEV void gate(float u, float &f, float &g)
{
    float e = __builtin_amdgcn_exp2f(-u * kLog2E);
    e = e > 0x1p126f ? 0x1p126f : e;
    f = __builtin_amdgcn_rcpf(1.f + e);
    g = e * f;
}

// Two neighbouring channels as they are stored: one word of halves, or two floats.
template <typename T> struct Two;
template <> struct Two<F32> {
    u32x2 w;
    EWF_OPS_DEV float x() const { return bits_to_float(w[0]); }
    EWF_OPS_DEV float y() const { return bits_to_float(w[1]); }
};
template <> struct Two<F16> {
    uint32_t w;
    EWF_OPS_DEV float x() const { return half_lo<F16>(w); }
    EWF_OPS_DEV float y() const { return half_hi<F16>(w); }
};
template <> struct Two<BF16> {
    uint32_t w;
    EWF_OPS_DEV float x() const { return half_lo<BF16>(w); }
    EWF_OPS_DEV float y() const { return half_hi<BF16>(w); }
};

template <typename T>
EWF_OPS_DEV Two<T> load_two(const typename T::raw *p)
{
    if constexpr (sizeof(typename T::raw) == 4) return {*reinterpret_cast<const u32x2_a4 *>(p)};
    else return {*reinterpret_cast<const u32_a2 *>(p)};
}

template <typename T>
EWF_OPS_DEV void store_two(typename T::raw *p, float x, float y)
{
    if constexpr (sizeof(typename T::raw) == 4) *reinterpret_cast<u32x2_a4 *>(p) = u32x2{float_to_bits(x), float_to_bits(y)};
    else *reinterpret_cast<u32_a2 *>(p) = pack_halves<T>(x, y);
}

// A lane's channels c and c + 1 of `channels`.  At the last channels a lane reads the pair that ends there, and drops
// what is not its own; lanes behind the end read it too and write nothing.
struct Lane {
    int64_t from;        // channel that a load begins at
    int have;            // channels that are the lane's own: 0, 1 or 2
    bool second;         // the lane's one channel is the second of the pair it reads
    bool single;         // there is one channel in all: element loads
};

EWF_OPS_DEV Lane lane_at(int64_t c, int64_t channels)
{
    Lane l;
    l.have = c + 1 < channels ? 2 : c < channels ? 1 : 0;
    l.single = channels == 1;
    l.from = l.have == 2 ? c : l.single ? 0 : channels - 2;
    l.second = l.have == 1 && !l.single;
    return l;
}

template <typename T>
EWF_OPS_DEV Two<T> load_edge(const typename T::raw *p, const Lane &l)
{
    Two<T> r;
    if (l.single) {
        if constexpr (sizeof(typename T::raw) == 4) r.w = u32x2{float_to_bits(*p), 0u};
        else r.w = *p;
    } else {
        r = load_two<T>(p);
        if constexpr (sizeof(typename T::raw) == 4) r.w[0] = l.second ? r.w[1] : r.w[0];
        else r.w = l.second ? r.w >> 16 : r.w;
    }
    return r;
}

template <typename T>
EWF_OPS_DEV void store_edge(typename T::raw *p, int have, float x, float y)
{
    if (have == 2) store_two<T>(p, x, y);
    else if (have == 1) store1<T>(p, x);
}

EWF_OPS_DEV Pair load_state(const RecTensor &t, int64_t b, const Lane &l)
{
    Pair s = {0.f, 0.f};
    if (!t.p) return s;
    const Two<F32> v = load_edge<F32>((const float *)t.p + b * t.batch + l.from, l);
    return {v.x(), v.y()};
}

EWF_OPS_DEV void store_state(const RecTensor &t, int64_t b, int64_t c, int have, Pair s)
{
    if (t.p) store_edge<F32>((float *)t.p + b * t.batch + c, have, s.x, s.y);
}

template <typename T>
EWF_OPS_DEV typename T::raw *at(const RecTensor &t, int64_t b, int64_t step, int64_t c)
{
    return (typename T::raw *)t.p + b * t.batch + step * t.step + c;
}

EWF_OPS_DEV int64_t sequence_length(const RecLaunch &a, int64_t b)
{
    if (!a.lengths) return a.steps;
    const int64_t n = a.lengths[b * a.lengths_stride];
    return n < 0 ? 0 : n > a.steps ? a.steps : n;
}

// The gradients of one element.
template <bool TIED>
EWF_OPS_DEV void gradients(float G, float f, float one_less_f, float i, float one_less_i, float before, float v, float &du, float &dv, float &dw)
{
    dv = G * i;
    if constexpr (TIED) du = G * (before - v) * (f * one_less_f);
    else {
        du = G * before * (f * one_less_f);
        dw = dv * v * one_less_i;
    }
}

// ------------------------------------------------------------------ few steps: a lane walks through time

template <typename T, bool TIED>
__global__ void __launch_bounds__(64) k_rec_walk(RecLaunch a)
{
    const uint32_t pairs = (uint32_t)((a.channels + 1) / 2), all = pairs * (uint32_t)a.batch;
    const uint32_t id = blockIdx.x * 64 + threadIdx.x;
    if (id >= all) return;
    const int64_t b = id / pairs, c = (int64_t)(id - (uint32_t)b * pairs) * 2;
    const Lane l = lane_at(c, a.channels);
    const int64_t len = sequence_length(a, b);
    Pair s = load_state(a.h0, b, l);
    for (int64_t t = 0; t < len; t++) {
        const Two<T> u = load_edge<T>(at<T>(a.u, b, t, l.from), l), v = load_edge<T>(at<T>(a.v, b, t, l.from), l);
        float f0, g0, f1, g1;
        gate(u.x(), f0, g0);
        gate(u.y(), f1, g1);
        if constexpr (!TIED) {
            const Two<T> w = load_edge<T>(at<T>(a.w, b, t, l.from), l);
            float less;
            gate(w.x(), g0, less);
            gate(w.y(), g1, less);
        }
        s = {fmaf(f0, s.x, g0 * v.x()), fmaf(f1, s.y, g1 * v.y())};
        store_edge<T>(at<T>(a.h, b, t, c), l.have, s.x, s.y);
    }
    store_state(a.last, b, c, l.have, s);
}

template <typename T, bool TIED>
__global__ void __launch_bounds__(64) k_rec_walk_grad(RecLaunch a)
{
    const uint32_t pairs = (uint32_t)((a.channels + 1) / 2), all = pairs * (uint32_t)a.batch;
    const uint32_t id = blockIdx.x * 64 + threadIdx.x;
    if (id >= all) return;
    const int64_t b = id / pairs, c = (int64_t)(id - (uint32_t)b * pairs) * 2;
    const Lane l = lane_at(c, a.channels);
    const int64_t len = sequence_length(a, b);
    const Pair h0 = load_state(a.h0, b, l);
    Pair s = load_state(a.dlast, b, l);
    for (int64_t t = len - 1; t >= 0; t--) {
        const Two<T> u = load_edge<T>(at<T>(a.u, b, t, l.from), l), v = load_edge<T>(at<T>(a.v, b, t, l.from), l);
        const Two<T> dh = load_edge<T>(at<T>(a.dh, b, t, l.from), l);
        Pair before = h0;
        if (t > 0) {
            const Two<T> h = load_edge<T>(at<T>(a.h, b, t - 1, l.from), l);
            before = {h.x(), h.y()};
        }
        float f0, g0, f1, g1, i0, j0, i1, j1;
        gate(u.x(), f0, g0);
        gate(u.y(), f1, g1);
        i0 = g0; j0 = f0; i1 = g1; j1 = f1;
        if constexpr (!TIED) {
            const Two<T> w = load_edge<T>(at<T>(a.w, b, t, l.from), l);
            gate(w.x(), i0, j0);
            gate(w.y(), i1, j1);
        }
        const Pair G = {dh.x() + s.x, dh.y() + s.y};
        float du0, dv0, dw0, du1, dv1, dw1;
        gradients<TIED>(G.x, f0, g0, i0, j0, before.x, v.x(), du0, dv0, dw0);
        gradients<TIED>(G.y, f1, g1, i1, j1, before.y, v.y(), du1, dv1, dw1);
        store_edge<T>(at<T>(a.du, b, t, c), l.have, du0, du1);
        store_edge<T>(at<T>(a.dv, b, t, c), l.have, dv0, dv1);
        if constexpr (!TIED) store_edge<T>(at<T>(a.dw, b, t, c), l.have, dw0, dw1);
        s = {f0 * G.x, f1 * G.y};
    }
    store_state(a.dh0, b, c, l.have, s);
}

// ------------------------------------------------------------------ tiles of steps
//
// A workgroup of W wavefronts takes kStrip channels of a sequence and W x 2 x R steps at a time.  A lane holds two
// channels and R consecutive steps in registers, the two halves of a wavefront one run of R steps after the
// other.  A lane composes its steps (the map of all of them, and the state at each of them if the tile began at zero),
// the maps are composed across halves by a lane exchange and across wavefronts through LDS, and with the state that
// its run begins at a lane finishes its results: F_r s + (state from zero).

template <typename T, bool BACK> struct Raw;            // a lane's operands at one step, as stored
template <typename T> struct Raw<T, false> { Two<T> u, v, w; };
template <typename T> struct Raw<T, true> { Two<T> u, v, w, h, dh; };

template <typename T, bool TIED, bool BACK, int R, int W>
struct Tile {
    static constexpr int kSteps = W * 2 * R;
    const RecLaunch &a;
    int64_t b, c, len;
    Lane l;
    bool whole_strip;
    int first;                                          // of this lane's steps within a tile
    Pair h0;                                            // BACK: the state before the first step

    EWF_OPS_DEV Tile(const RecLaunch &a_, int64_t strip, int64_t b_) : a(a_), b(b_)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        c = strip * kStrip + (lane & 31) * 2;
        len = sequence_length(a, b);
        l = lane_at(c, a.channels);
        whole_strip = strip * kStrip + kStrip <= a.channels;
        first = (wave * 2 + (lane >> 5)) * R;
        if constexpr (BACK) h0 = load_state(a.h0, b, l);
    }

    // The time of the k-th step of the walk: backwards it begins at the sequence's end.
    EWF_OPS_DEV int64_t time(int64_t k) const { return BACK ? len - 1 - k : k; }

    // Every step of the tile from k0 on exists, and so does the state before it in memory.
    EWF_OPS_DEV bool whole(int64_t k0) const { return whole_strip && k0 + kSteps <= len - (BACK ? 1 : 0); }

    EWF_OPS_DEV void load(int64_t k0, Raw<T, BACK> (&raw)[R]) const
    {
        if (whole(k0)) {
            const int64_t t = time(k0 + first), s = BACK ? -1 : 1;
            const typename T::raw *pu = at<T>(a.u, b, t, c), *pv = at<T>(a.v, b, t, c), *pw = nullptr, *ph = nullptr, *pd = nullptr;
            if constexpr (!TIED) pw = at<T>(a.w, b, t, c);
            if constexpr (BACK) { ph = at<T>(a.h, b, t - 1, c); pd = at<T>(a.dh, b, t, c); }
#pragma unroll
            for (int r = 0; r < R; r++) {
                raw[r].u = load_two<T>(pu + r * s * a.u.step);
                raw[r].v = load_two<T>(pv + r * s * a.v.step);
                if constexpr (!TIED) raw[r].w = load_two<T>(pw + r * s * a.w.step);
                if constexpr (BACK) {
                    raw[r].h = load_two<T>(ph + r * s * a.h.step);
                    raw[r].dh = load_two<T>(pd + r * s * a.dh.step);
                }
            }
            return;
        }
#pragma unroll
        for (int r = 0; r < R; r++) {
            // (steps that do not exist read one that does; compose() leaves them out)
            int64_t k = k0 + first + r;
            k = k < len ? k : len - 1;
            const int64_t t = time(k);
            raw[r].u = load_edge<T>(at<T>(a.u, b, t, l.from), l);
            raw[r].v = load_edge<T>(at<T>(a.v, b, t, l.from), l);
            if constexpr (!TIED) raw[r].w = load_edge<T>(at<T>(a.w, b, t, l.from), l);
            if constexpr (BACK) {
                raw[r].h = load_edge<T>(at<T>(a.h, b, t > 0 ? t - 1 : 0, l.from), l);
                raw[r].dh = load_edge<T>(at<T>(a.dh, b, t, l.from), l);
            }
        }
    }
};

struct Map { float F0, B0, F1, B1; };                   // of a lane's two channels

EWF_OPS_DEV Pair apply(const Map &m, const Pair &s) { return {fmaf(m.F0, s.x, m.B0), fmaf(m.F1, s.y, m.B1)}; }

template <typename T, bool TIED, bool BACK, int R, int W>
__global__ void __launch_bounds__(W * 64) k_rec_march(RecLaunch a)
{
    typedef Tile<T, TIED, BACK, R, W> Tl;
    __shared__ Map totals[2][W][32];
    const uint32_t strips = (uint32_t)((a.channels + kStrip - 1) / kStrip), jobs = strips * (uint32_t)a.batch;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool later = lane >= 32;
    for (uint32_t job = blockIdx.x; job < jobs; job += gridDim.x) {
        const uint32_t b = job / strips;
        Tl tile(a, job - b * strips, b);
        __syncthreads();                                    // (the arrays of the job before are read)
        Pair carry = load_state(BACK ? a.dlast : a.h0, b, tile.l);
        Raw<T, BACK> raw[R];
        if (tile.len > 0) tile.load(0, raw);
        int buf = 0;
        for (int64_t k0 = 0; k0 < tile.len; k0 += Tl::kSteps, buf ^= 1) {
            const bool whole = k0 + Tl::kSteps <= tile.len;
            float F[R][2], S[R][2];                         // the map's factor up to (BACK: before) a step; the state there from zero
            float f[R][2], g[R][2], i[R][2], j[R][2], v[R][2], before[R][2];
            float P0 = 1.f, P1 = 1.f, s0 = 0.f, s1 = 0.f;
    #pragma unroll
            for (int r = 0; r < R; r++) {
                const int64_t k = k0 + tile.first + r;
                const bool live = whole || k < tile.len;
                gate(raw[r].u.x(), f[r][0], g[r][0]);
                gate(raw[r].u.y(), f[r][1], g[r][1]);
                if constexpr (!TIED) {
                    gate(raw[r].w.x(), i[r][0], j[r][0]);
                    gate(raw[r].w.y(), i[r][1], j[r][1]);
                } else {
                    i[r][0] = g[r][0]; i[r][1] = g[r][1]; j[r][0] = f[r][0]; j[r][1] = f[r][1];
                }
                v[r][0] = raw[r].v.x(); v[r][1] = raw[r].v.y();
                if constexpr (!BACK) {
                    if (live) {
                        s0 = fmaf(f[r][0], s0, i[r][0] * v[r][0]);
                        s1 = fmaf(f[r][1], s1, i[r][1] * v[r][1]);
                        P0 *= f[r][0];
                        P1 *= f[r][1];
                    }
                    F[r][0] = P0; F[r][1] = P1;
                    S[r][0] = s0; S[r][1] = s1;
                } else {
                    before[r][0] = raw[r].h.x(); before[r][1] = raw[r].h.y();
                    if (k == tile.len - 1) { before[r][0] = tile.h0.x; before[r][1] = tile.h0.y; }
                    F[r][0] = P0; F[r][1] = P1;
                    S[r][0] = s0 + raw[r].dh.x(); S[r][1] = s1 + raw[r].dh.y();
                    if (live) {
                        s0 = f[r][0] * S[r][0];
                        s1 = f[r][1] * S[r][1];
                        P0 *= f[r][0];
                        P1 *= f[r][1];
                    }
                }
            }
            // the next tile's operands are in flight during the rest
            if (k0 + Tl::kSteps < tile.len) tile.load(k0 + Tl::kSteps, raw);
            // across the halves of the wavefront
            const Map own = {P0, s0, P1, s1};
            const Map other = {__shfl_xor(P0, 32), __shfl_xor(s0, 32), __shfl_xor(P1, 32), __shfl_xor(s1, 32)};
            if (later)
                totals[buf][wave][lane - 32] = Map{own.F0 * other.F0, fmaf(own.F0, other.B0, own.B0), own.F1 * other.F1, fmaf(own.F1, other.B1, own.B1)};
            __syncthreads();
            // across the wavefronts, in every one of them (two arrays in turn: one barrier a tile)
            Pair at_wave = carry;
    #pragma unroll
            for (int q = 0; q < W; q++) {
                if (q == wave) at_wave = carry;
                carry = apply(totals[buf][q][lane & 31], carry);
            }
            const Pair from = later ? apply(other, at_wave) : at_wave;
    #pragma unroll
            for (int r = 0; r < R; r++) {
                const int64_t k = k0 + tile.first + r;
                if (!(whole || k < tile.len)) continue;
                const int64_t t = tile.time(k);
                const float G0 = fmaf(F[r][0], from.x, S[r][0]), G1 = fmaf(F[r][1], from.y, S[r][1]);
                if constexpr (!BACK) store_edge<T>(at<T>(a.h, b, t, tile.c), tile.l.have, G0, G1);
                else {
                    float du0, dv0, dw0, du1, dv1, dw1;
                    gradients<TIED>(G0, f[r][0], g[r][0], i[r][0], j[r][0], before[r][0], v[r][0], du0, dv0, dw0);
                    gradients<TIED>(G1, f[r][1], g[r][1], i[r][1], j[r][1], before[r][1], v[r][1], du1, dv1, dw1);
                    store_edge<T>(at<T>(a.du, b, t, tile.c), tile.l.have, du0, du1);
                    store_edge<T>(at<T>(a.dv, b, t, tile.c), tile.l.have, dv0, dv1);
                    if constexpr (!TIED) store_edge<T>(at<T>(a.dw, b, t, tile.c), tile.l.have, dw0, dw1);
                }
            }
        }
        if (wave == 0 && !later) store_state(BACK ? a.dh0 : a.last, b, tile.c, tile.l.have, carry);
    }
}

// ------------------------------------------------------------------ which kernel

constexpr uint32_t kMostJobs = 1 << 20;  // workgroups of a launch; further strips are taken in turn
constexpr int kWalkSteps = 16;           // up to here a lane walks through time by itself

template <typename T, bool TIED>
void run(const RecLaunch &a, bool backward, hipStream_t stream)
{
    if (a.steps <= kWalkSteps) {
        // (fewer than 2^31 lanes: batch x channels is)
        const dim3 grid((uint32_t)(((uint64_t)((a.channels + 1) / 2) * a.batch + 63) / 64));
        if (backward) hipLaunchKernelGGL((k_rec_walk_grad<T, TIED>), grid, dim3(64), 0, stream, a);
        else hipLaunchKernelGGL((k_rec_walk<T, TIED>), grid, dim3(64), 0, stream, a);
        return;
    }
    const uint64_t jobs = (uint64_t)((a.channels + kStrip - 1) / kStrip) * a.batch;
    const dim3 grid((uint32_t)(jobs < kMostJobs ? jobs : kMostJobs));
    if (backward) hipLaunchKernelGGL((k_rec_march<T, TIED, true, 4, 8>), grid, dim3(512), 0, stream, a);
    else hipLaunchKernelGGL((k_rec_march<T, TIED, false, 8, 8>), grid, dim3(512), 0, stream, a);
}

template <typename T>
void run_type(const RecLaunch &a, bool backward, hipStream_t stream)
{
    if (a.w.p) run<T, false>(a, backward, stream);
    else run<T, true>(a, backward, stream);
}

}  // namespace

size_t recurrence_workspace(const RecLaunch &, bool, int) { return 0; }

void launch_recurrence(const RecLaunch &a, bool backward, int, hipStream_t stream)
{
    if (a.dtype == EWF_F32) run_type<F32>(a, backward, stream);
    else if (a.dtype == EWF_F16) run_type<F16>(a, backward, stream);
    else run_type<BF16>(a, backward, stream);
}

}  // namespace ewf
