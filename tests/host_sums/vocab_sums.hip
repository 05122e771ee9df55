// The sums that the operators over a vocabulary take of a row of logits, by the library's own functions in a host program: a thread each of the
// lanes, which the points of a row's wavefronts and of the row join in 64 bits.  Reads scale, lanes, a wavefront's lanes and logits a lane and the logits, lane after
// lane, and prints peak, whether the row has to be swept again, and the sums about the peak.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>
#include <vector>

#undef __device__
#define __device__ __attribute__((host)) __attribute__((device))
static inline float host_exp2(float x) { return x < -126.f ? 0.f : std::exp2(x); }          // (the native one has no smaller results)
static inline float host_med3(float a, float b, float c) { return std::fmax(std::fmin(std::fmax(a, b), c), std::fmin(a, b)); }
#define __builtin_amdgcn_exp2f host_exp2
#define __builtin_amdgcn_fmed3f host_med3
#define __any(x) (x)
#define rintf std::rint
#define fmaxf std::fmax
#define fmaf std::fma
#define fabsf std::fabs
#include "ewf_vocab_device.h"

using namespace ewf;

int main()
{
    float scale;
    int lanes, wave, each;
    while (std::scanf("%a %d %d %d", &scale, &lanes, &wave, &each) == 4) {
        const float c = scale * 1.44269504f, lag = 8.f / c;
        std::vector<Sums> threads(lanes);
        for (Sums &t : threads)
            for (int i = 0; i < each; i++) {
                float x;
                if (std::scanf("%a", &x) != 1) return 1;
                add<true, 1>(t, &x, x, c, lag);
            }
        Sums row;
        for (const Sums &t : threads) row.peak = std::fmax(row.peak, t.peak);
        double s = 0, w = 0;
        for (int first = 0; first < lanes; first += wave) {
            Sums joined;
            double ws = 0, ww = 0;
            for (int i = first; i < first + wave; i++) joined.peak = std::fmax(joined.peak, threads[i].peak);
            for (int i = first; i < first + wave; i++) {
                Sums t = threads[i];
                move<true>(t, t.m, point_of(joined.peak, c));
                ws += t.s;
                ww += t.w;
            }
            joined.s = (float)ws;
            joined.w = (float)ww;
            move<true>(joined, point_of(joined.peak, c), point_of(row.peak, c));
            s += joined.s;
            w += joined.w;
        }
        row.s = (float)s;
        row.w = (float)w;
        settle<true>(row, c);
        std::printf("%a %d %a %a\n", row.peak, (int)beyond(row.peak, c), row.s, row.w);
    }
    return 0;
}
