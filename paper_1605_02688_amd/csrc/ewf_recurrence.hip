// Gated linear recurrence over time and its backward pass.
//
// A step is the map s -> f s + b of a channel's state, and maps compose: (F, B) after (f, b) is (F f, F b + B).
// Forward, in time:  s = h, f = f_t, b = i_t v_t, h_t = s.  Backward, against time:  with s_t = f_t G_t, what step t
// hands to step t - 1, G_t = dh_t + s_(t+1) and s_t = f_t s_(t+1) + f_t dh_t.  f lies in [0, 1], so that products of
// f never overflow whatever their number.
#include "ewf_ops_device.h"

namespace ewf {

void aux_fill_zero(void *ptr, size_t nbytes, hipStream_t stream);

namespace {

// ------------------------------------------------------------------ a lane's channels
//
// A lane takes C neighbouring channels, 8 bytes of them.  Where fewer are left it reads the last C of the row and drops
// what is not its own; lanes behind the end read those too, and write nothing.

template <typename T> constexpr int kWidth = 8 / (int)sizeof(typename T::raw);

struct Lane {
    int from;            // channel that a load begins at
    int have;            // channels that are the lane's own
};

template <typename T>
EWF_OPS_DEV Lane lane_at(int c, int channels)
{
    constexpr int C = kWidth<T>;
    Lane l;
    l.have = channels - c;
    l.have = l.have < 0 ? 0 : l.have > C ? C : l.have;
    l.from = c + C <= channels ? c : channels >= C ? channels - C : 0;
    return l;
}

template <typename T> struct Eight {
    u32x2 w;
    EWF_OPS_DEV float operator[](int e) const
    {
        if constexpr (sizeof(typename T::raw) == 4) return bits_to_float(w[e]);
        else return (e & 1) ? half_hi<T>(w[e >> 1]) : half_lo<T>(w[e >> 1]);
    }
    // Drops the first n elements; zeros move in behind.
    EWF_OPS_DEV void move_down(int n)
    {
        const uint64_t x = __builtin_bit_cast(uint64_t, w);
        w = __builtin_bit_cast(u32x2, n < kWidth<T> ? x >> (n * (64 / kWidth<T>)) : (uint64_t)0);
    }
};

typedef u32x2 u32x2_a2 __attribute__((aligned(2)));
template <typename T> struct EightAt { typedef u32x2_a2 at; };
template <> struct EightAt<F32> { typedef u32x2_a4 at; };

template <typename T>
EWF_OPS_DEV Eight<T> load_eight(const typename T::raw *p) { return {*reinterpret_cast<const typename EightAt<T>::at *>(p)}; }

// Rows of fewer than C channels, element by element: those behind the last are copies of it, and nobody's.
template <typename T>
EWF_OPS_DEV Eight<T> load_few(const typename T::raw *p, int channels)
{
    constexpr int C = kWidth<T>;
    uint64_t w = 0;
#pragma unroll
    for (int e = 0; e < C; e++) {
        const typename T::raw x = p[e < channels ? e : channels - 1];
        if constexpr (C == 2) w |= (uint64_t)float_to_bits(x) << (e * 32);
        else w |= (uint64_t)x << (e * 16);
    }
    return {__builtin_bit_cast(u32x2, w)};
}

template <typename T>
EWF_OPS_DEV void store_eight(typename T::raw *p, const float *f)
{
    u32x2 w;
    if constexpr (sizeof(typename T::raw) == 4) w = u32x2{float_to_bits(f[0]), float_to_bits(f[1])};
    else w = u32x2{pack_halves<T>(f[0], f[1]), pack_halves<T>(f[2], f[3])};
    *reinterpret_cast<typename EightAt<T>::at *>(p) = w;
}

template <typename T>
EWF_OPS_DEV void store_edge(typename T::raw *p, int have, const float *f)
{
    if (have == kWidth<T>) { store_eight<T>(p, f); return; }
#pragma unroll
    for (int e = 0; e < kWidth<T>; e++)
        if (e < have) store1<T>(p + e, f[e]);
}

EWF_OPS_DEV float load_state(const RecTensor &t, int64_t b, int c) { return t.p ? ((const float *)t.p)[b * t.batch + c] : 0.f; }
EWF_OPS_DEV void store_state(const RecTensor &t, int64_t b, int c, float s)
{
    if (t.p) ((float *)t.p)[b * t.batch + c] = s;
}

EWF_OPS_DEV int sequence_length(const RecLaunch &a, int64_t b)
{
    if (!a.lengths) return (int)a.steps;
    const int n = a.lengths[b * a.lengths_stride];
    return n < 0 ? 0 : n > a.steps ? (int)a.steps : n;
}

// One element's gradients from G, the gradient of its state; `f` and `before` are its gate and the state before it.  Returns what the
// step hands to the one before.  Gates first: a product that a shut gate makes small does not overflow on the way.
template <typename T, bool TIED>
EWF_OPS_DEV float gradients(float G, float u, float w, float v, float before, float &du, float &dv, float &dw)
{
    float f, g;
    gate<T>(u, f, g);
    if constexpr (TIED) {
        dv = G * g;
        du = dv * (f + f) * fmaf(0.5f, before, -0.5f * v);        // (halves: states of both signs may lie further apart than float32 reaches)
    } else {
        float i, j;
        gate<T>(w, i, j);
        dv = G * i;
        dw = dv * j * v;
        du = G * (f * g) * before;
    }
    return f * G;
}

// ------------------------------------------------------------------ few steps: a lane walks through time

// CUT: rows that end inside a lane's channels.
template <typename T, bool TIED, bool BACK, bool CUT>
__global__ void __launch_bounds__(64) k_rec_walk(RecLaunch a)
{
    constexpr int C = kWidth<T>;
    typedef typename T::raw raw;
    const int channels = (int)a.channels;
    const uint32_t lanes = (uint32_t)(channels + C - 1) / C, id = blockIdx.x * 64 + threadIdx.x;
    if (id >= lanes * (uint32_t)a.batch) return;
    const int64_t b = id / lanes;
    const int c = (int)(id - (uint32_t)b * lanes) * C;
    const Lane l = lane_at<T>(c, channels);
    const int len = sequence_length(a, b);
    auto load = [&](const RecTensor &x, int64_t t) {
        const raw *p = (const raw *)x.p + b * x.batch + t * x.step + l.from;
        return CUT && channels < C ? load_few<T>(p, channels) : load_eight<T>(p);
    };
    auto store = [&](const RecTensor &x, int64_t t, const float *f) {
        raw *p = (raw *)x.p + b * x.batch + t * x.step + c;
        if constexpr (CUT) store_edge<T>(p, l.have, f);
        else store_eight<T>(p, f);
    };
    const int drop = c - l.from;
    auto settle = [&](Eight<T> x) {
        if constexpr (CUT) x.move_down(drop);
        return x;
    };
    float s[C];
#pragma unroll
    for (int e = 0; e < C; e++) s[e] = e < l.have ? load_state(BACK ? a.dlast : a.h0, b, c + e) : 0.f;
    // (the operands of kAhead steps are read together: bfloat16 [128, 16, 2048] forward and backward 7.3 and 13.5 us; eight, 7.1 and 13.8)
    constexpr int kAhead = 4;
    if constexpr (!BACK) {
        for (int t0 = 0; t0 < len; t0 += kAhead) {
            Eight<T> u[kAhead], v[kAhead], w[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; k++) {
                const int t = t0 + k;
                if (t >= len) break;
                u[k] = load(a.u, t);
                v[k] = load(a.v, t);
                if constexpr (!TIED) w[k] = load(a.w, t);
            }
#pragma unroll
            for (int k = 0; k < kAhead; k++) {
                if (t0 + k >= len) break;
                u[k] = settle(u[k]);
                v[k] = settle(v[k]);
                if constexpr (!TIED) w[k] = settle(w[k]);
#pragma unroll
                for (int e = 0; e < C; e++) {
                    float f, i, less;
                    gate<T>(u[k][e], f, i);
                    if constexpr (!TIED) gate<T>(w[k][e], i, less);
                    s[e] = fmaf(f, s[e], i * v[k][e]);
                }
                store(a.h, t0 + k, s);
            }
        }
    } else {
        for (int t0 = len - 1; t0 >= 0; t0 -= kAhead) {
            Eight<T> u[kAhead], v[kAhead], w[kAhead], h[kAhead], dh[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; k++) {
                const int t = t0 - k;
                if (t < 0) break;
                u[k] = load(a.u, t);
                v[k] = load(a.v, t);
                dh[k] = load(a.dh, t);
                if constexpr (!TIED) w[k] = load(a.w, t);
                h[k] = load(a.h, t > 0 ? t - 1 : 0);
            }
#pragma unroll
            for (int k = 0; k < kAhead; k++) {
                const int t = t0 - k;
                if (t < 0) break;
                u[k] = settle(u[k]);
                v[k] = settle(v[k]);
                dh[k] = settle(dh[k]);
                h[k] = settle(h[k]);
                if constexpr (!TIED) w[k] = settle(w[k]);
                float du[C], dv[C], dw[C];
#pragma unroll
                for (int e = 0; e < C; e++) {
                    float before = h[k][e];
                    if (t == 0) before = e < l.have ? load_state(a.h0, b, c + e) : 0.f;
                    s[e] = gradients<T, TIED>(dh[k][e] + s[e], u[k][e], TIED ? 0.f : w[k][e], v[k][e], before, du[e], dv[e], dw[e]);
                }
                store(a.du, t, du);
                store(a.dv, t, dv);
                if constexpr (!TIED) store(a.dw, t, dw);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < C; e++)
        if (e < l.have) store_state(BACK ? a.dh0 : a.last, b, c + e, s[e]);
}

// ------------------------------------------------------------------ tiles of steps
//
// A workgroup of W wavefronts takes a strip of L x C channels of a sequence and W x G x R steps at a time, G = 64 / L.
// A lane holds R consecutive steps in registers, the G groups of a wavefront one run of R steps after the other.  A
// lane composes its steps to one map; the maps are composed across groups by lane exchanges and across wavefronts
// through LDS, by one thread for each channel, which also keeps the channel's state; and from the state that its run
// begins at a lane walks its steps a second time.

struct Map { float F, B; };
EWF_OPS_DEV Map after(const Map &m, const Map &n) { return {m.F * n.F, fmaf(m.F, n.B, m.B)}; }     // m after n
EWF_OPS_DEV float apply(const Map &m, float s) { return fmaf(m.F, s, m.B); }

template <typename T, bool BACK> struct Raw;            // a lane's operands at one step, as stored
template <typename T> struct Raw<T, false> { Eight<T> u, v, w; };
template <typename T> struct Raw<T, true> { Eight<T> u, v, w, h, dh; };

// The rows of one tensor that a lane reads or writes, one after the other: an address that all lanes of a wavefront share, and
// offsets of 32 bits to it (the host refuses steps that are further apart).  Reads stay between the first and the last
// step that exists: steps that do not are read from there, and composing leaves them out.
// FEW: rows of fewer than C channels.
template <typename T, bool BACK, bool FEW>
struct Rows {
    char *base;
    int at, step, lowest, highest;                      // bytes
    int few;                                            // FEW: the channels

    EWF_OPS_DEV Eight<T> load() const
    {
        const int off = BACK ? (at > lowest ? at : lowest) : (at < highest ? at : highest);
        const typename T::raw *p = (const typename T::raw *)(base + (uint32_t)off);
        if constexpr (FEW) return load_few<T>(p, few);
        else return load_eight<T>(p);
    }
    EWF_OPS_DEV typename T::raw *pointer() const { return (typename T::raw *)(base + (uint32_t)at); }
    EWF_OPS_DEV void next() { at += BACK ? -step : step; }
};

template <typename T, bool TIED, bool BACK, int L, int R, int W, bool FEW = false>
struct Tile {
    static constexpr int C = kWidth<T>, G = 64 / L, kSteps = W * G * R, kStrip = L * C, size = sizeof(typename T::raw);
    static_assert(kStrip <= W * 64, "one thread for each channel of a strip");
    static_assert(G * R <= 32, "a wavefront's steps span less than 2^31 bytes");
    const RecLaunch &a;
    int b, c0, len, channels;                           // sequence, first channel
    int place, group, wave;                             // of the lane in its row; of its run in the wavefront
    bool whole_strip;
    Lane l;

    EWF_OPS_DEV Tile(const RecLaunch &a_, int strip, int b_) : a(a_), b(b_), c0(strip * kStrip)
    {
        channels = (int)a.channels;
        place = threadIdx.x % L;
        group = threadIdx.x % 64 / L;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        len = __builtin_amdgcn_readfirstlane(sequence_length(a, b));
        l = lane_at<T>(channel(), channels);
        whole_strip = c0 + kStrip <= channels;
    }

    EWF_OPS_DEV int channel() const { return c0 + C * place; }
    // The time of the k-th step of the walk: backwards it begins at the sequence's end.
    EWF_OPS_DEV int time(int k) const { return BACK ? len - 1 - k : k; }
    // The first step of a lane's R in the tile that begins at step k0.
    EWF_OPS_DEV int first(int k0) const { return k0 + (wave * G + group) * R; }
    // The earliest time of the wavefront's steps that exist (a wavefront without any reads the last that does).
    EWF_OPS_DEV int earliest(int k0) const
    {
        const int k = k0 + wave * G * R + (BACK ? G * R - 1 : 0);
        return time(k < len ? k : len - 1);
    }

    // `before` of the tensor: its rows one step earlier.
    EWF_OPS_DEV Rows<T, BACK, FEW> rows(const RecTensor &x, int k0, bool read, bool before = false) const
    {
        const int t0 = earliest(k0), shift = before ? 1 : 0;
        const int base = t0 >= shift ? t0 - shift : 0;                                  // (uniform)
        int rel = BACK ? len - 1 - first(k0) - shift - base : group * R;               // of the lane's first step
        if (BACK && rel < 0) rel = 0;                                                   // (all its rows are read at the earliest)
        const int more = len - 1 - base;
        const int edge = FEW ? 0 : channels - C < c0 ? channels - C : c0;                         // (uniform: reads of the last channels begin there)
        const int from = read ? edge : c0, c = (read ? l.from - edge : C * place) * size;
        Rows<T, BACK, FEW> r;
        r.base = (char *)x.p + (b * x.batch + base * x.step + from) * size;
        r.step = (int)(x.step * size);
        r.at = rel * r.step + c;
        r.lowest = c;
        r.highest = (more < G * R - 1 ? more : G * R - 1) * r.step + c;
        r.few = channels;
        return r;
    }

    EWF_OPS_DEV void load(int k0, Raw<T, BACK> (&raw)[R]) const
    {
        auto fetch = [&](const RecTensor &x, bool before, Eight<T> Raw<T, BACK>::*to) {
            auto p = rows(x, k0, true, before);
#pragma unroll
            for (int r = 0; r < R; r++) { raw[r].*to = p.load(); p.next(); }
        };
        fetch(a.u, false, &Raw<T, BACK>::u);
        fetch(a.v, false, &Raw<T, BACK>::v);
        if constexpr (!TIED) fetch(a.w, false, &Raw<T, BACK>::w);
        if constexpr (BACK) {
            fetch(a.dh, false, &Raw<T, BACK>::dh);
            fetch(a.h, true, &Raw<T, BACK>::h);
        }
        if (!FEW && !whole_strip) {
            const int drop = channel() - l.from;
#pragma unroll
            for (int r = 0; r < R; r++) {
                raw[r].u.move_down(drop);
                raw[r].v.move_down(drop);
                if constexpr (!TIED) raw[r].w.move_down(drop);
                if constexpr (BACK) { raw[r].h.move_down(drop); raw[r].dh.move_down(drop); }
            }
        }
    }

    // What a lane keeps of its steps between the two walks: forward the steps' maps; backward the operands, from which
    // the gates are computed a second time (bfloat16 [8, 4096, 2048] 176 us; with the gates kept, 218.  Forward the second
    // computation costs more than the registers it saves: 108 and 100).
    static constexpr bool kMaps = !BACK;
    struct Maps { float f[R][C], b[R][C]; };

    EWF_OPS_DEV void step_map(const Raw<T, BACK> &x, int e, float &f, float &b) const
    {
        if constexpr (BACK) {
            f = sigmoid<T>(x.u[e]);
            b = f * x.dh[e];
        } else {
            float i, less;
            gate<T>(x.u[e], f, i);
            if constexpr (!TIED) gate<T>(x.w[e], i, less);
            b = i * x.v[e];
        }
    }

    // Composes a lane's steps to one map a channel.
    EWF_OPS_DEV void compose(int k0, const Raw<T, BACK> (&raw)[R], Maps &maps, Map (&m)[C]) const
    {
        const bool all = len - k0 >= kSteps;
        const int from = first(k0);
#pragma unroll
        for (int e = 0; e < C; e++) m[e] = {1.f, 0.f};
#pragma unroll
        for (int r = 0; r < R; r++) {
#pragma unroll
            for (int e = 0; e < C; e++) {
                float f, x;
                step_map(raw[r], e, f, x);
                if (!all && from + r >= len) { f = 1.f; x = 0.f; }
                m[e] = after({f, x}, m[e]);
                if constexpr (kMaps) { maps.f[r][e] = f; maps.b[r][e] = x; }
            }
        }
    }

    // The maps of the groups before a lane's own, composed; m becomes the map of the wavefront in its last group.
    EWF_OPS_DEV void across_groups(Map (&m)[C], Map (&before)[C]) const
    {
#pragma unroll
        for (int e = 0; e < C; e++) {
            Map own = m[e];
#pragma unroll
            for (int d = 1; d < G; d *= 2) {
                const Map prev = {__shfl_up(own.F, d * L), __shfl_up(own.B, d * L)};
                if (group >= d) own = after(own, prev);
            }
            before[e] = {1.f, 0.f};
            if constexpr (G > 1) {
                const Map prev = {__shfl_up(own.F, L), __shfl_up(own.B, L)};
                if (group > 0) before[e] = prev;
            }
            m[e] = own;
        }
    }

    // Walks a lane's steps from the states s that they begin at, and writes its results.
    EWF_OPS_DEV void finish(int k0, const Raw<T, BACK> (&raw)[R], const Maps &maps, float (&s)[C]) const
    {
        const int from = first(k0);
        auto put = [&](Rows<T, BACK, FEW> &p, int r, const float *f) {
            if (from + r < len) {
                if (whole_strip) store_eight<T>(p.pointer(), f);
                else store_edge<T>(p.pointer(), l.have, f);
            }
            p.next();
        };
        if constexpr (!BACK) {
            auto ph = rows(a.h, k0, false);
#pragma unroll
            for (int r = 0; r < R; r++) {
#pragma unroll
                for (int e = 0; e < C; e++) {
                    float f, b;
                    if constexpr (kMaps) { f = maps.f[r][e]; b = maps.b[r][e]; }
                    else step_map(raw[r], e, f, b);
                    s[e] = fmaf(f, s[e], b);
                }
                put(ph, r, s);
            }
        } else {
            auto pu = rows(a.du, k0, false), pv = rows(a.dv, k0, false), pw = rows(TIED ? a.du : a.dw, k0, false);
#pragma unroll
            for (int r = 0; r < R; r++) {
                const Raw<T, true> &x = raw[r];
                float du[C], dv[C], dw[C];
#pragma unroll
                for (int e = 0; e < C; e++) {
                    float state = x.h[e];
                    if (from + r == len - 1) state = e < l.have ? load_state(a.h0, b, channel() + e) : 0.f;
                    s[e] = gradients<T, TIED>(x.dh[e] + s[e], x.u[e], TIED ? 0.f : x.w[e], x.v[e], state, du[e], dv[e], dw[e]);
                }
                put(pu, r, du);
                put(pv, r, dv);
                if constexpr (!TIED) put(pw, r, dw);
            }
        }
    }
};

// ------------------------------------------------------------------ one workgroup for a strip: tile after tile

template <typename T, bool TIED, bool BACK, int L, int R, int W>
__global__ void __launch_bounds__(W * 64) k_rec_march(RecLaunch a)
{
    typedef Tile<T, TIED, BACK, L, R, W> Tl;
    constexpr int C = Tl::C;
    __shared__ Map totals[W][Tl::kStrip];
    __shared__ float states[W][Tl::kStrip];             // that a wavefront's steps begin at
    const uint32_t strips = ((uint32_t)a.channels + Tl::kStrip - 1) / Tl::kStrip, jobs = strips * (uint32_t)a.batch;
    for (uint32_t job = blockIdx.x; job < jobs; job += gridDim.x) {
        const uint32_t b = job / strips;
        const Tl tile(a, job - b * strips, b);
        const int mine = tile.c0 + threadIdx.x;         // the channel whose state this thread keeps
        const bool keeps = threadIdx.x < Tl::kStrip && mine < tile.channels;
        float state = keeps ? load_state(BACK ? a.dlast : a.h0, b, mine) : 0.f;
        Raw<T, BACK> raw[R];
        if (tile.len > 0) tile.load(0, raw);
        for (int k0 = 0; k0 < tile.len; k0 += Tl::kSteps) {
            typename Tl::Maps maps;
            Map m[C], before[C];
            Raw<T, BACK> now[R];
#pragma unroll
            for (int r = 0; r < R; r++) now[r] = raw[r];
            // the next tile's operands are in flight during all of this one
            if (tile.len - k0 > Tl::kSteps) tile.load(k0 + Tl::kSteps, raw);
            tile.compose(k0, now, maps, m);
            tile.across_groups(m, before);
            if (tile.group == Tl::G - 1)
#pragma unroll
                for (int e = 0; e < C; e++) totals[tile.wave][tile.place * C + e] = m[e];
            __syncthreads();
            if (threadIdx.x < Tl::kStrip) {
#pragma unroll
                for (int q = 0; q < W; q++) {
                    states[q][threadIdx.x] = state;
                    state = apply(totals[q][threadIdx.x], state);
                }
            }
            __syncthreads();
            float s[C];
#pragma unroll
            for (int e = 0; e < C; e++) s[e] = apply(before[e], states[tile.wave][tile.place * C + e]);
            tile.finish(k0, now, maps, s);
        }
        if (keeps) store_state(BACK ? a.dh0 : a.last, b, mine, state);
    }
}

// ------------------------------------------------------------------ chains of tiles
//
// Many steps: a workgroup takes one tile, and the tiles of a strip of channels form a chain.  Every tile's map is published
// as soon as it is known, and the state behind it as soon as that is: a tile finds the state that it begins at by
// composing the maps of the tiles before it, back to the nearest whose state is known.  The operands are read once and no
// tile waits for another's loads.
//
// A channel's record in the workspace is one 64-bit word, written and read by single atomic accesses that need no order among
// each other: the map's B or the state in the upper half, the map's F below, whose two upper bits are
// free (F lies in [0, 1]) and say what the word holds.  The words are zero when the kernel begins.
//
// The wait ends: a workgroup draws its place in the chain when it runs, so that all tiles before it belong to workgroups
// that run or are done, and it publishes its own map before it waits; the first tile waits for none, and each next one
// only for words that workgroups publish without waiting, or after a wait that has ended.  Where a caller breaks the
// rule that overlapping calls have workspaces of their own, words can be lost: a wait is given up after kMostLooks
// looks (seconds; a tile takes microseconds), and the channel's states from there on are NaN.  The looks are counted by the wavefront
// that waits: while its queue is held back it does not look either.  A place that is not one of the
// chain's is not taken: whatever the workspace holds, every access is in bounds.

constexpr uint32_t kMapBit = 1u << 30, kStateBit = 1u << 31;

// (a factor that is NaN becomes a map that yields NaN)
EWF_OPS_DEV uint64_t map_word(const Map &m)
{
    const bool sound = m.F == m.F;
    return (uint64_t)float_to_bits(sound ? m.B : m.F) << 32 | (sound ? float_to_bits(m.F) : 0u) | kMapBit;
}
EWF_OPS_DEV uint64_t state_word(float s) { return (uint64_t)float_to_bits(s) << 32 | kStateBit; }
EWF_OPS_DEV bool is_empty(uint64_t w) { return (uint32_t)w < kMapBit; }

EWF_OPS_DEV void publish(uint64_t *p, uint64_t w) { __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
EWF_OPS_DEV uint64_t look(const uint64_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The state that the tile at `place` (not the first) of a channel begins at; `record` is the tile's own, `back` what two
// neighbouring tiles' records are apart.  Back to the nearest known state, then from it through the maps in the order of
// the tiles: the operations are those by which the tiles in between find their own states, so that the result has the same
// bits wherever the search ends.  Four records are looked at together: their loads overlap (eight and sixteen cost
// more traffic than they save).
constexpr int kLook = 4;
constexpr int kMostLooks = 1 << 22;

EWF_OPS_DEV float search(const uint64_t *record, int64_t back, int place)
{
    constexpr uint64_t kNone = (uint64_t)0x7fc00000u << 32 | kStateBit;    // before the first tile, which publishes a state: never reached
    uint64_t w[kLook];
    int from = place - 1, looks = 0;
    for (bool known = false; ; from -= kLook) {
#pragma unroll
        for (int q = 0; q < kLook; q++) w[q] = from >= q ? look(record - (place - from + q) * back) : kNone;
#pragma unroll
        for (int q = 0; q < kLook; q++) {
            if (known) break;
            while (is_empty(w[q])) {
                if (++looks > kMostLooks) return bits_to_float(0x7fc00000u);
                __builtin_amdgcn_s_sleep(1);
                w[q] = look(record - (place - from + q) * back);
            }
            known = (uint32_t)w[q] & kStateBit;
        }
        if (known) break;
    }
    float s = 0.f;
    for (;;) {
#pragma unroll
        for (int q = kLook - 1; q >= 0; q--) {          // (what precedes the nearest known state is replaced by it)
            const float value = bits_to_float((uint32_t)(w[q] >> 32));
            s = (uint32_t)w[q] & kStateBit ? value : fmaf(bits_to_float((uint32_t)w[q] & ~kMapBit), s, value);
        }
        from += kLook;
        if (from > place - 1) return s;
#pragma unroll
        for (int q = 0; q < kLook; q++) w[q] = look(record - (place - from + q) * back);
    }
}

// (backward: registers for four wavefronts on each of a unit's four SIMDs, two workgroups; with two gates the wide tile then spills 9
// (float32), 13 (float16) and 19 (bfloat16) registers, and the second workgroup is worth more: bfloat16 [8, 4096, 2048] 249 us, 545 MB
// written for 420, and 264.  Forward long tiles have 224 registers in 16 bits, 163 in float32: one workgroup a unit, which loads nothing while it
// searches)
template <typename T, bool TIED, bool BACK, int L, int R, int W, bool FEW>
__global__ void __launch_bounds__(W * 64, BACK ? 4 : 1) k_rec_chain(RecLaunch a, uint32_t chains, uint32_t tiles)
{
    typedef Tile<T, TIED, BACK, L, R, W, FEW> Tl;
    constexpr int C = Tl::C;
    __shared__ Map totals[W][Tl::kStrip];
    __shared__ float states[W][Tl::kStrip];
    __shared__ uint32_t drawn;
    const uint32_t strips = ((uint32_t)a.channels + Tl::kStrip - 1) / Tl::kStrip, jobs = chains * tiles;
    uint64_t *records = (uint64_t *)a.workspace;
    uint32_t *counters = (uint32_t *)(records + (uint64_t)chains * tiles * Tl::kStrip);
    const int64_t back = (int64_t)chains * Tl::kStrip;
    for (uint32_t job = blockIdx.x; job < jobs; job += gridDim.x) {
        const uint32_t chain = job % chains, b = chain / strips;
        uint32_t place = 0;
        __syncthreads();                                // (the arrays of the job before are read)
        if (tiles > 1 && threadIdx.x == 0) drawn = __hip_atomic_fetch_add(counters + chain, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const Tl tile(a, chain - b * strips, b);        // (reads the sequence's length while the place is drawn)
        if (tiles > 1) {
            __syncthreads();
            place = __builtin_amdgcn_readfirstlane(drawn);
            if (place >= tiles) continue;               // (only where another call has written into the workspace)
        }
        const int k0 = (int)place * Tl::kSteps;
        if (k0 >= tile.len && place) continue;          // (no step: nobody looks for this tile)
        Raw<T, BACK> raw[R];
        typename Tl::Maps maps;
        Map m[C], before[C];
        if (tile.len > 0) {
            tile.load(k0, raw);
            tile.compose(k0, raw, maps, m);
            tile.across_groups(m, before);
            if (tile.group == Tl::G - 1)
#pragma unroll
                for (int e = 0; e < C; e++) totals[tile.wave][tile.place * C + e] = m[e];
        }
        __syncthreads();
        if (threadIdx.x < Tl::kStrip) {
            const int mine = tile.c0 + threadIdx.x;
            const bool exists = mine < tile.channels;
            Map part[W], all = {1.f, 0.f};
            if (tile.len > 0)
#pragma unroll
                for (int q = 0; q < W; q++) {
                    part[q] = totals[q][threadIdx.x];
                    all = after(part[q], all);
                }
            uint64_t *record = records + (uint64_t)place * back + (uint64_t)chain * Tl::kStrip + threadIdx.x;
            float state;
            if (place) {
                publish(record, map_word(all));
                state = search(record, back, (int)place);
            } else state = exists ? load_state(BACK ? a.dlast : a.h0, b, mine) : 0.f;
            const float end = apply(all, state);
            if (tile.len - k0 > Tl::kSteps) publish(record, state_word(end));
            else if (exists) store_state(BACK ? a.dh0 : a.last, b, mine, end);
            if (tile.len > 0)
#pragma unroll
                for (int q = 0; q < W; q++) {
                    states[q][threadIdx.x] = state;
                    state = apply(part[q], state);
                }
        }
        __syncthreads();
        if (tile.len == 0) continue;
        float s[C];
#pragma unroll
        for (int e = 0; e < C; e++) s[e] = apply(before[e], states[tile.wave][tile.place * C + e]);
        tile.finish(k0, raw, maps, s);
    }
}

// ------------------------------------------------------------------ which kernel

constexpr uint32_t kMostJobs = 1 << 20;  // workgroups of a launch; further jobs are taken in turn

// Lanes a row, steps a lane, wavefronts.
template <int L_, int R_, int W_> struct Shape { static constexpr int L = L_, R = R_, W = W_, steps = W_ * (64 / L_) * R_; };
typedef Shape<8, 4, 8> Slim;             // 64 bytes, 256 steps
typedef Shape<16, 4, 8> Narrow;          // 128 bytes of a row, 128 steps
typedef Shape<32, 16, 8> Long;           // 256 bytes, 256 steps
typedef Shape<64, 8, 8> Wide;            // 512 bytes, 64 steps

enum class How { Walk, March, Slim, Small, Large };

struct Plan {
    How how = How::Walk;
    uint64_t chains = 0, tiles = 1;
    size_t bytes = 0;
};

template <typename S>
void cut(const RecLaunch &a, How how, Plan &p)
{
    const int64_t strip = S::L * (a.dtype == EWF_F32 ? 2 : 4);
    p.how = how;
    p.chains = (uint64_t)((a.channels + strip - 1) / strip) * a.batch;
    p.tiles = how == How::March ? 1 : (uint64_t)((a.steps + S::steps - 1) / S::steps);
    p.bytes = p.tiles > 1 ? (p.chains * p.tiles * strip * 8 + p.chains * 4 + 15) / 16 * 16 : 0;
}

// A shape's strips fit rows that fill two thirds of them.
template <typename S>
bool filled(const RecLaunch &a)
{
    const int64_t strip = S::L * (a.dtype == EWF_F32 ? 2 : 4);
    return a.channels * 3 >= (a.channels + strip - 1) / strip * strip * 2;
}

// Few steps: a lane walks through time by itself, at up to 1 us for four steps; tiles cost what their number does.  bfloat16, us,
// forward and backward, walk / the better tiles: [32, 16, 1024] (512 strips of 128 bytes) 6.4, 8.6 / 6.7, 8.9; [16, 24, 2048]
// (512) 7.2, 11.4 / 6.4, 9.1; [64, 32, 2048] (2048) 9.4, 18.0 / 15.8, 16.4; [128, 48, 2048] (4096) 16.8, 30.1 / 30.5, 33.9.  Rows that
// are cut are walked more slowly: [2, 13, 74] 7.2, 10.7 / 6.3, 7.6.
bool is_walked(const RecLaunch &a, int units)
{
    const int64_t strip = a.dtype == EWF_F32 ? 32 : 64, strips = (a.channels + strip - 1) / strip * a.batch, times = strips / (4 * (int64_t)units);
    const bool cut = a.channels % (a.dtype == EWF_F32 ? 2 : 4) != 0;
    return a.steps <= (cut ? 8 : 16) * (times < 1 ? 1 : times > 3 ? 3 : times);
}

// Rows of up to 64 bytes: slim tiles (bfloat16 [36, 34737, 26], us, forward and backward, slim / narrow / large / march: 67,
// 137 / 115, 203 / 220, 565 / 732; [256, 4096, 26] 54, 111 / 89, 167 / 175, 465 / 91).
// Forward, us, march / chains of long tiles / chains of narrow tiles, bfloat16 [8, 4096, 2048] (256 strips of 64 channels)
// 91 / 105 / 121, [16, 512, 1024] (256) 13.0 / 15.3 / -, [3, 4096, 2048] (96) 73 / 44 / 48, [1, 65536, 1024] (16) 1047 / 103 / -: a
// workgroup for a strip where there is one for nearly each unit, tiles where there are fewer.  Long tiles, of which fewer
// search, where there is one for each unit ([4, 2048, 1024], 256 of them, 16.6 / 18.2; [2, 512, 2048], 64, 11.8 / 10.8).
// Backward, wide tiles / narrow ones: [8, 4096, 2048] 176 / 206, [3, 4096, 2048] (1536 wide tiles) 77 / 82, [4, 2048, 1024] (512)
// 34.1 / 32.8, float16 [5, 1237, 1000] (400) 30.9 / 23.0; sequences that one wide tile holds ([32, 64, 2048]) 14.5 / 19.0.
// Where rows leave a part of them empty, [20, 8000, 160 | 200 | 300], long / narrow 62 / 49, 67 / 70, 104 / 103, wide / narrow
// 103 / 97, 110 / 145, 202 / 196.
Plan plan_of(const RecLaunch &a, bool backward, int units)
{
    Plan p;
    if (is_walked(a, units)) return p;
    if (a.channels <= (a.dtype == EWF_F32 ? 16 : 32)) {
        cut<Slim>(a, How::Slim, p);
        return p;
    }
    if (!backward) {
        cut<Narrow>(a, How::March, p);
        if (p.chains * 8 >= (uint64_t)units * 7) return p;
        cut<Long>(a, How::Large, p);
        if (filled<Long>(a) && p.chains * p.tiles >= (uint64_t)units) return p;
    } else {
        cut<Wide>(a, How::Large, p);
        if (filled<Wide>(a) && (p.chains * p.tiles >= 4 * (uint64_t)units || p.tiles == 1)) return p;
    }
    cut<Narrow>(a, How::Small, p);
    return p;
}

template <typename T, bool TIED, bool BACK, typename S, bool FEW = false>
void run_chain(const RecLaunch &a, const Plan &p, hipStream_t stream)
{
    if (p.bytes) aux_fill_zero(a.workspace, p.bytes, stream);
    const uint64_t jobs = p.chains * p.tiles;
    hipLaunchKernelGGL((k_rec_chain<T, TIED, BACK, S::L, S::R, S::W, FEW>), dim3((uint32_t)(jobs < kMostJobs ? jobs : kMostJobs)), dim3(S::W * 64), 0, stream, a,
                       (uint32_t)p.chains, (uint32_t)p.tiles);
}

template <typename T, bool TIED, bool BACK>
void run(const RecLaunch &a, const Plan &p, hipStream_t stream)
{
    constexpr int C = kWidth<T>;
    switch (p.how) {
    case How::Walk: {
        // (fewer than 2^31 lanes: batch x channels is)
        const dim3 grid((uint32_t)(((uint64_t)((a.channels + C - 1) / C) * a.batch + 63) / 64));
        if (a.channels % C) hipLaunchKernelGGL((k_rec_walk<T, TIED, BACK, true>), grid, dim3(64), 0, stream, a);
        else hipLaunchKernelGGL((k_rec_walk<T, TIED, BACK, false>), grid, dim3(64), 0, stream, a);
        return;
    }
    case How::March:
        if constexpr (!BACK)
            hipLaunchKernelGGL((k_rec_march<T, TIED, false, Narrow::L, Narrow::R, Narrow::W>), dim3((uint32_t)(p.chains < kMostJobs ? p.chains : kMostJobs)),
                               dim3(Narrow::W * 64), 0, stream, a);
        return;
    case How::Slim:
        if (a.channels < C) return run_chain<T, TIED, BACK, Slim, true>(a, p, stream);
        return run_chain<T, TIED, BACK, Slim>(a, p, stream);
    case How::Small: return run_chain<T, TIED, BACK, Narrow>(a, p, stream);
    case How::Large:
        if constexpr (BACK) return run_chain<T, TIED, true, Wide>(a, p, stream);
        else return run_chain<T, TIED, false, Long>(a, p, stream);
    }
}

template <typename T>
void run_type(const RecLaunch &a, bool backward, const Plan &p, hipStream_t stream)
{
    if (a.w.p) { if (backward) run<T, false, true>(a, p, stream); else run<T, false, false>(a, p, stream); }
    else { if (backward) run<T, true, true>(a, p, stream); else run<T, true, false>(a, p, stream); }
}

}  // namespace

size_t recurrence_workspace(const RecLaunch &a, bool backward, int units) { return plan_of(a, backward, units).bytes; }

void launch_recurrence(const RecLaunch &a, bool backward, int units, hipStream_t stream)
{
    const Plan p = plan_of(a, backward, units);
    if (a.dtype == EWF_F32) run_type<F32>(a, backward, p, stream);
    else if (a.dtype == EWF_F16) run_type<F16>(a, backward, p, stream);
    else run_type<BF16>(a, backward, p, stream);
}

}  // namespace ewf
