// Rotary positions: pairs of a head's numbers are turned by position * frequency.
#include "token_internal.h"

namespace laplex {

namespace {

constexpr int kRotaryThreads = 256;

// cos and sin of position * frequency.  The product passes what fp32 holds (position 10^6 at one radian per position leaves
// 0.06 radians): it is formed and brought below a turn in fp64, and only the rest is rounded.
__device__ __forceinline__ void turn_of(int64_t position, float frequency, float magnitude, bool inverse, float* c, float* s)
{
    const double turns = (double)position * (double)frequency * 0.15915494309189533577;      // 1 / (2 pi)
    const float rest = (float)((turns - rint(turns)) * 2.0);                                  // in half turns, [-1, 1]
    float sn, cs;
    sincospif(rest, &sn, &cs);
    *c = cs * magnitude;
    *s = (inverse ? -sn : sn) * magnitude;
}

// one thread per (token, pair or number that passes through): all heads
template <typename T>
__global__ void __launch_bounds__(kRotaryThreads)
k_rotary(RotaryArgs A)
{
    const int units = A.half + (A.dim - 2 * A.half);
    const int64_t total = A.tokens * units;
    for (int64_t i = (int64_t)blockIdx.x * kRotaryThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kRotaryThreads) {
        const int64_t token = i / units;
        const int unit = (int)(i - token * units);
        const T* x = static_cast<const T*>(A.x) + token * A.ldx;
        T* y = static_cast<T*>(A.y) + token * A.ldy;
        if (unit < A.half) {
            const int first = A.interleaved ? 2 * unit : unit, second = A.interleaved ? first + 1 : unit + A.half;
            float c, s;
            turn_of(A.positions[token], A.frequencies[unit], A.magnitude, A.inverse, &c, &s);
            for (int h = 0; h < A.heads; ++h) {
                const float u = to_float(x[h * A.dim + first]), v = to_float(x[h * A.dim + second]);
                y[h * A.dim + first] = (T)(u * c - v * s);
                y[h * A.dim + second] = (T)(v * c + u * s);
            }
        } else {
            const int at = unit + A.half;
            for (int h = 0; h < A.heads; ++h) y[h * A.dim + at] = x[h * A.dim + at];
        }
    }
}

__global__ void k_rotary_frequencies(float* out, int64_t pairs, double base, int scaling, double factor, double context, double low,
                                     double high)
{
    const double kTurn = 6.28318530717958647693;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < pairs; i += (int64_t)gridDim.x * blockDim.x) {
        const double part = (double)i / (double)pairs;
        if (scaling == 2 && pairs > 1) base *= pow(factor, (double)pairs / (double)(pairs - 1));
        double f = pow(base, -part);
        if (scaling == 1) f /= factor;
        if (scaling == 3) {
            double keep = (context * f / kTurn - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f = f * keep + f / factor * (1.0 - keep);
        }
        out[i] = (float)f;
        if (scaling == 2 && pairs > 1) base /= pow(factor, (double)pairs / (double)(pairs - 1));
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& A, hipStream_t st)
{
    const int64_t total = A.tokens * (A.dim - A.half);
    int64_t blocks = (total + kRotaryThreads - 1) / kRotaryThreads;
    if (blocks > (1 << 20)) blocks = 1 << 20;
    profile_before("rotary", st);
    if (A.bf16) hipLaunchKernelGGL((k_rotary<__bf16>), dim3((unsigned)blocks), dim3(kRotaryThreads), 0, st, A);
    else hipLaunchKernelGGL((k_rotary<float>), dim3((unsigned)blocks), dim3(kRotaryThreads), 0, st, A);
    profile_after("rotary", st);
    return hipGetLastError();
}

hipError_t launch_rotary_frequencies(float* out, int64_t pairs, double base, int scaling, double factor, double context,
                                     double low, double high, hipStream_t st)
{
    const int64_t blocks = (pairs + 63) / 64;
    hipLaunchKernelGGL(k_rotary_frequencies, dim3((unsigned)(blocks < 1024 ? blocks : 1024)), dim3(64), 0, st, out, pairs, base, scaling,
                       factor, context, low, high);
    return hipGetLastError();
}

}  // namespace laplex
