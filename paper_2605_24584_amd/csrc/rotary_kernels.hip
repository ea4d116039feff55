// Rotary positions: pairs of a head's numbers are turned by position * frequency.  Memory bound: a read and a write per number.
// A workgroup takes a few tokens, forms their cosines and sines once, in LDS, for all heads, and then streams the heads in pieces of 16 bytes.
// 16384 tokens, 32 heads of 128 bf16 numbers: 43 us for 268 MB (6.2 TB/s); 50021 tokens, 18 heads of 80 fp32 numbers, 36 of them turned in neighbouring
// pairs: 111 us for 576 MB (5.2 TB/s; pair by pair 133); 64 tokens of 32 heads 2.9 us, a launch.
#include "token_internal.h"

namespace laplex {

namespace {

constexpr int kRotaryThreads = 256;
constexpr int64_t kRotaryMaxBlocks = int64_t(1) << 22;      // (a grid holds fewer than 2^32 threads)

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

// n / by for n < 2^31 by a product (by >= 1)
struct Divisor {
    uint32_t factor, shift;
    Divisor() = default;
    explicit Divisor(uint32_t by) : factor(0), shift(0)
    {
        while (shift < 31 && (uint64_t(1) << shift) < by) ++shift;
        factor = (uint32_t)(((uint64_t(1) << 32) * ((uint64_t(1) << shift) - by)) / by + 1);
    }
    __device__ __forceinline__ uint32_t of(uint32_t n) const { return (__umulhi(n, factor) + n) >> shift; }
};

struct RotaryTiles {
    RotaryArgs A;
    int tile;                        // tokens of a workgroup
    int pairs, rest;                 // units of a head: those that turn, those that pass through
    Divisor token, head;             // by the units of a token, of a head
};

template <typename T, int VEC> struct Vec { typedef T type __attribute__((ext_vector_type(VEC))); };
template <typename T> struct Vec<T, 1> { typedef T type; };

template <typename T, int VEC>
__device__ __forceinline__ void load_vec(float* out, const T* p)
{
    const typename Vec<T, VEC>::type v = *reinterpret_cast<const typename Vec<T, VEC>::type*>(p);
    if constexpr (VEC == 1) out[0] = to_float(v);
    else
#pragma unroll
        for (int i = 0; i < VEC; ++i) out[i] = to_float((T)v[i]);
}
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T* p, const float* in)
{
    typename Vec<T, VEC>::type v;
    if constexpr (VEC == 1) v = (T)in[0];
    else
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = (T)in[i];
    *reinterpret_cast<typename Vec<T, VEC>::type*>(p) = v;
}

// A unit is VEC pairs, VEC numbers from either half of what is turned; INTERLEAVED: the pairs of VEC numbers side by side (of two, if VEC is one).
template <typename T, int VEC, bool INTERLEAVED>
__global__ void __launch_bounds__(kRotaryThreads)
k_rotary(RotaryTiles R)
{
    extern __shared__ float2 table[];                  // [tile][half]
    const RotaryArgs& A = R.A;
    const uint32_t per_head = R.pairs + R.rest, per_token = per_head * A.heads;
    for (int64_t token0 = (int64_t)blockIdx.x * R.tile; token0 < A.tokens; token0 += (int64_t)gridDim.x * R.tile) {
        const int tokens = A.tokens - token0 < R.tile ? (int)(A.tokens - token0) : R.tile;
        for (int i = threadIdx.x; i < tokens * A.half; i += kRotaryThreads) {
            const int t = i / A.half;
            float c, s;
            turn_of(A.positions[token0 + t], A.frequencies[i - t * A.half], A.magnitude, A.inverse, &c, &s);
            table[i] = float2{c, s};
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < per_token * tokens; i += kRotaryThreads) {
            const uint32_t t = R.token.of(i), in_token = i - t * per_token, h = R.head.of(in_token), unit = in_token - h * per_head;
            const T* x = static_cast<const T*>(A.x) + (token0 + t) * A.ldx + h * A.dim;
            T* y = static_cast<T*>(A.y) + (token0 + t) * A.ldy + h * A.dim;
            if (unit < (uint32_t)R.pairs) {
                if constexpr (INTERLEAVED) {
                    constexpr int PAIRS = VEC > 1 ? VEC / 2 : 1, PIECE = VEC > 1 ? VEC : 1;
                    const float2* turns = table + t * A.half + unit * PAIRS;
                    const int first = 2 * unit * PAIRS;
                    float u[2 * PAIRS];
                    load_vec<T, PIECE>(u, x + first);
                    if (VEC == 1) load_vec<T, PIECE>(u + 1, x + first + 1);
#pragma unroll
                    for (int j = 0; j < PAIRS; ++j) {
                        const float2 w = turns[j];
                        const float p = u[2 * j], q = u[2 * j + 1];
                        u[2 * j] = p * w.x - q * w.y;
                        u[2 * j + 1] = q * w.x + p * w.y;
                    }
                    store_vec<T, PIECE>(y + first, u);
                    if (VEC == 1) store_vec<T, PIECE>(y + first + 1, u + 1);
                } else {
                    const float2* turns = table + t * A.half + unit * VEC;
                    const int first = unit * VEC, second = first + A.half;
                    float u[VEC], v[VEC];
                    load_vec<T, VEC>(u, x + first);
                    load_vec<T, VEC>(v, x + second);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float2 w = turns[j];
                        const float p = u[j], q = v[j];
                        u[j] = p * w.x - q * w.y;
                        v[j] = q * w.x + p * w.y;
                    }
                    store_vec<T, VEC>(y + first, u);
                    store_vec<T, VEC>(y + second, v);
                }
            } else {
                const int at = 2 * A.half + (unit - R.pairs) * VEC;
                *reinterpret_cast<typename Vec<T, VEC>::type*>(y + at) = *reinterpret_cast<const typename Vec<T, VEC>::type*>(x + at);
            }
        }
        __syncthreads();                               // the table may be written again
    }
}

__global__ void k_rotary_frequencies(float* out, int64_t pairs, double base, int scaling, double factor, double context, double low,
                                     double high)
{
    const double kTurn = 6.28318530717958647693;
    if (scaling == 2 && pairs > 1) base *= pow(factor, (double)pairs / (double)(pairs - 1));
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < pairs; i += (int64_t)gridDim.x * blockDim.x) {
        const double part = (double)i / (double)pairs;
        double f = pow(base, -part);
        if (scaling == 1) f /= factor;
        if (scaling == 3) {
            double keep = (context * f / kTurn - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f = f * keep + f / factor * (1.0 - keep);
        }
        out[i] = (float)f;
    }
}

}  // namespace

namespace {

template <typename T, int VEC>
void rotary_with(const RotaryTiles& R, dim3 grid, size_t lds, hipStream_t st)
{
    if (R.A.interleaved) hipLaunchKernelGGL((k_rotary<T, VEC, true>), grid, dim3(kRotaryThreads), lds, st, R);
    else hipLaunchKernelGGL((k_rotary<T, VEC, false>), grid, dim3(kRotaryThreads), lds, st, R);
}

template <typename T>
void rotary_of(const RotaryTiles& R, int vec, dim3 grid, size_t lds, hipStream_t st)
{
    if (vec * sizeof(T) == 16) rotary_with<T, 16 / sizeof(T)>(R, grid, lds, st);
    else if (vec * sizeof(T) == 8) rotary_with<T, 8 / sizeof(T)>(R, grid, lds, st);
    else rotary_with<T, 1>(R, grid, lds, st);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& A, hipStream_t st)
{
    // in place the numbers that pass through are there
    const bool copies = A.x != A.y || A.ldx != A.ldy;
    if (A.half == 0 && !copies) return hipSuccess;
    const int size = A.bf16 ? 2 : 4, rest = A.dim - 2 * A.half;
    // the widest pieces that every row, head and part of a head is a whole number of
    int vec = 16 / size;
    const auto fits = [&](int v) {
        const int64_t bytes = (int64_t)v * size;
        return reinterpret_cast<uintptr_t>(A.x) % bytes == 0 && reinterpret_cast<uintptr_t>(A.y) % bytes == 0 && A.ldx * size % bytes == 0 &&
               A.ldy * size % bytes == 0 && A.dim % v == 0 && (A.interleaved ? 2 * A.half : A.half) % v == 0;
    };
    if (!fits(vec)) vec /= 2;
    if (!fits(vec)) vec = 1;
    RotaryTiles R{};
    R.A = A;
    R.pairs = A.interleaved && vec > 1 ? 2 * A.half / vec : A.half / vec;
    R.rest = copies ? rest / vec : 0;
    const int64_t units = (int64_t)(R.pairs + R.rest) * A.heads;
    R.head = Divisor((uint32_t)(R.pairs + R.rest));
    R.token = Divisor((uint32_t)units);
    // about four units a thread, as long as there are tokens for two thousand workgroups; the table at most 16 KB
    int64_t tile = (4 * kRotaryThreads + units - 1) / units;
    if (tile > A.tokens / 2048) tile = A.tokens / 2048;
    if (A.half && tile > 2048 / A.half) tile = 2048 / A.half;
    if (tile > 1024) tile = 1024;
    if (tile < 1) tile = 1;
    R.tile = (int)tile;
    const int64_t tiles = (A.tokens + tile - 1) / tile;
    const dim3 grid((unsigned)(tiles < kRotaryMaxBlocks ? tiles : kRotaryMaxBlocks));
    const size_t lds = (size_t)tile * A.half * sizeof(float2);
    profile_before("rotary", st);
    if (A.bf16) rotary_of<__bf16>(R, vec, grid, lds, st);
    else rotary_of<float>(R, vec, grid, lds, st);
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
