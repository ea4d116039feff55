// Layer norm of rows and its gradient.
//
//   mean = sum x / w,  rstd = (sum (x - mean)^2 / w + eps)^(-1/2),  hat = (x - mean) rstd,  y = hat weight + bias
//   g = gy weight:  gx = rstd (g - sum g / w - hat sum (g hat) / w),   gweight = sum over rows of gy hat,   gbias = sum over rows of gy
//
// Rows of up to kThreads * kMost pieces of eight (bf16) or four numbers are held in registers: x is read once, and the squares are summed about the mean and not as a
// difference of two sums.  A row belongs to `lanes` threads, a power of two: to part of a wavefront, a wavefront, or the workgroup.
// The gradient's workgroups take a range of rows each and keep the sums of their columns in registers; they are written once for each
// workgroup (k_norm_parts) and added up in order by a second launch, so that the same call gives the same bits.  Longer rows are read again instead of held
// (k_norm_*_long), and their columns are summed by a launch of their own.
//
// What bounds it: HBM.  In bf16 32768 rows of 4096: forward 135 us (4.0 TB/s), gradient 190 (4.2) and 7 for the join; 524288 rows of 128: 58 (4.6 TB/s) and 96 (4.2).  In fp32 (with the join)
// 211 (5.1) and 341 (4.7), 124 (4.3) and 181 (4.4).  Rows that are not held, or barely, are far from that: 8192 x 16384 in bf16 274 (2.0) and 557 (1.5; the gradient's eight pieces a thread leave 196
// bytes a lane in scratch and one wavefront a SIMD), in fp32, not held, 359 (3.0) and 700 (2.3); 2048 x 100000 in bf16 456 (1.8) and 1075 (1.1), of which the 819 MB of columns' sums are a part.  Weights held in registers
// over a workgroup's rows, and not read again for each, took both directions of 32768 x 4096 from 517 to 332 us.  Reading the next row ahead is no faster: other workgroups of the compute unit do so.
#include "token_internal.h"

namespace laplex {

namespace {

constexpr int kThreads = 256;
constexpr int kMost = 8;                 // pieces of a row that a thread holds

template <typename T> struct Piece;
template <> struct Piece<float> { static constexpr int N = 4; typedef float type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Piece<__bf16> { static constexpr int N = 8; typedef __bf16 type __attribute__((ext_vector_type(8), aligned(2))); };

// numbers at .. at + N - 1 of a row of `width`; zeros in the place of those that do not exist
template <typename T>
__device__ __forceinline__ void load_piece(float* out, const T* row, int64_t at, int64_t width)
{
    constexpr int N = Piece<T>::N;
    if (at + N <= width) {
        const typename Piece<T>::type v = *reinterpret_cast<const typename Piece<T>::type*>(row + at);
#pragma unroll
        for (int e = 0; e < N; ++e) out[e] = (float)v[e];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) out[e] = at + e < width ? to_float(row[at + e]) : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void store_piece(T* row, int64_t at, int64_t width, const float* v)
{
    constexpr int N = Piece<T>::N;
    if (at + N <= width) {
        typename Piece<T>::type w;
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = (T)v[e];
        *reinterpret_cast<typename Piece<T>::type*>(row + at) = w;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (at + e < width) row[at + e] = (T)v[e];
    }
}

// a weight's numbers that go with a piece of either type (fp32, as they lie; `otherwise` where there is no weight)
template <int N>
__device__ __forceinline__ void load_weight(float* out, const float* w, int64_t at, int64_t width, float otherwise)
{
#pragma unroll
    for (int e = 0; e < N; ++e) out[e] = otherwise;
    if (!w) return;
#pragma unroll
    for (int e = 0; e < N; e += 4) load_piece<float>(out + e, w, at + e, width);
}

// Sums over the `lanes` threads of a row; over the workgroup through `side`, one barrier per call, two sides in turn.
template <int M, int LANES>
__device__ __forceinline__ void row_sums(float (&v)[M], float (*side)[M])
{
#pragma unroll
    for (int step = 1; step < (LANES < 64 ? LANES : 64); step <<= 1)
#pragma unroll
        for (int i = 0; i < M; ++i) v[i] += __shfl_xor(v[i], step);
    if (LANES > 64) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < M; ++i) side[threadIdx.x >> 6][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < M; ++i) v[i] = (side[0][i] + side[1][i]) + (side[2][i] + side[3][i]);
    }
}

__device__ __forceinline__ float inverse_root(float variance, float eps) { return 1.0f / sqrtf(variance + eps); }

template <typename T, int LANES, int COUNT>
__global__ void __launch_bounds__(kThreads)
k_norm(NormArgs A)
{
    constexpr int N = Piece<T>::N, ROWS = kThreads / LANES;
    __shared__ float side[2][kThreads / 64][1];
    const int lane = threadIdx.x % LANES;
    const float width = (float)A.width;
    float w[COUNT][N], b[COUNT][N];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        load_weight<N>(w[i], A.weight, (int64_t)(i * LANES + lane) * N, A.width, 1.0f);
        load_weight<N>(b[i], A.bias, (int64_t)(i * LANES + lane) * N, A.width, 0.0f);
    }
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < A.rows; first += (int64_t)gridDim.x * ROWS) {
        const int64_t row = first + threadIdx.x / LANES;
        const bool live = row < A.rows;
        const T* const x = static_cast<const T*>(A.x) + (live ? row : A.rows - 1) * A.ldx;
        float v[COUNT][N], sum[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < COUNT; ++i) load_piece<T>(v[i], x, (int64_t)(i * LANES + lane) * N, A.width);
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) sum[0] += v[i][e];
        row_sums<1, LANES>(sum, side[0]);
        const float mean = sum[0] / width;      // (divided, not multiplied by 1 / width: rows of one number again and again have exactly it for a mean where their sum is exact)
        sum[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                v[i][e] -= mean;
                const float w = (int64_t)(i * LANES + lane) * N + e < A.width ? v[i][e] : 0.0f;
                sum[0] += w * w;
            }
        row_sums<1, LANES>(sum, side[1]);
        const float rstd = inverse_root(sum[0] / width, A.eps);
        if (!live) continue;
        if (lane == 0) {
            if (A.mean_out) A.mean_out[row] = mean;
            if (A.rstd_out) A.rstd_out[row] = rstd;
        }
        T* const y = static_cast<T*>(A.y) + row * A.ldy;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int64_t at = (int64_t)(i * LANES + lane) * N;
            if (at >= A.width) continue;
#pragma unroll
            for (int e = 0; e < N; ++e) v[i][e] = fmaf(v[i][e] * rstd, w[i][e], b[i][e]);
            store_piece<T>(y, at, A.width, v[i]);
        }
    }
}

// Rows that are not held: a workgroup reads its row three times.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_long(NormArgs A)
{
    constexpr int N = Piece<T>::N;
    __shared__ float side[2][kThreads / 64][1];
    const int64_t step = (int64_t)kThreads * N;
    const float width = (float)A.width;
    for (int64_t row = blockIdx.x; row < A.rows; row += gridDim.x) {
        const T* const x = static_cast<const T*>(A.x) + row * A.ldx;
        float v[N], sum[1] = {0.0f};
        for (int64_t at = (int64_t)threadIdx.x * N; at < A.width; at += step) {
            load_piece<T>(v, x, at, A.width);
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < N; ++e) s += v[e];
            sum[0] += s;
        }
        row_sums<1, kThreads>(sum, side[0]);
        const float mean = sum[0] / width;      // (divided, not multiplied by 1 / width: rows of one number again and again have exactly it for a mean where their sum is exact)
        sum[0] = 0.0f;
        for (int64_t at = (int64_t)threadIdx.x * N; at < A.width; at += step) {
            load_piece<T>(v, x, at, A.width);
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < N; ++e) s += at + e < A.width ? (v[e] - mean) * (v[e] - mean) : 0.0f;
            sum[0] += s;
        }
        row_sums<1, kThreads>(sum, side[1]);
        const float rstd = inverse_root(sum[0] / width, A.eps);
        if (threadIdx.x == 0) {
            if (A.mean_out) A.mean_out[row] = mean;
            if (A.rstd_out) A.rstd_out[row] = rstd;
        }
        T* const y = static_cast<T*>(A.y) + row * A.ldy;
        for (int64_t at = (int64_t)threadIdx.x * N; at < A.width; at += step) {
            float w[N], b[N];
            load_piece<T>(v, x, at, A.width);
            load_weight<N>(w, A.weight, at, A.width, 1.0f);
            load_weight<N>(b, A.bias, at, A.width, 0.0f);
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] = fmaf((v[e] - mean) * rstd, w[e], b[e]);
            store_piece<T>(y, at, A.width, w);
        }
    }
}

// The gradient.  A workgroup takes rows blockIdx.x * ROWS + r, then those gridDim.x * ROWS further on; parts[workgroup][2][width] <- its rows' sums.
template <typename T, int LANES, int COUNT>
__global__ void __launch_bounds__(kThreads)
k_norm_parts(NormBackwardArgs A)
{
    constexpr int N = Piece<T>::N, ROWS = kThreads / LANES;
    __shared__ float side[2][kThreads / 64][2];
    __shared__ float columns[LANES < kThreads ? ROWS : 1][LANES < kThreads ? LANES * N : 1];
    const int lane = threadIdx.x % LANES, r = threadIdx.x / LANES;
    const float width = (float)A.width;
    float w[COUNT][N], gw[COUNT][N], gb[COUNT][N];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        load_weight<N>(w[i], A.weight, (int64_t)(i * LANES + lane) * N, A.width, 1.0f);
#pragma unroll
        for (int e = 0; e < N; ++e) gw[i][e] = gb[i][e] = 0.0f;
    }
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < A.rows; first += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const int64_t row = first + r < A.rows ? first + r : A.rows - 1;
        const bool live = first + r < A.rows;
        const T* const x = static_cast<const T*>(A.x) + row * A.ldx;
        const T* const gy = static_cast<const T*>(A.gy) + row * A.ldgy;
        float hat[COUNT][N], g[COUNT][N], sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            load_piece<T>(hat[i], x, (int64_t)(i * LANES + lane) * N, A.width);
            load_piece<T>(g[i], gy, (int64_t)(i * LANES + lane) * N, A.width);
        }
        const float mean = A.mean[row], rstd = A.rstd[row];
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                hat[i][e] = (hat[i][e] - mean) * rstd;
                const float t = live ? g[i][e] : 0.0f;         // (rows behind the last are the last one again)
                if (A.gweight) gw[i][e] = fmaf(t, live ? hat[i][e] : 0.0f, gw[i][e]);
                gb[i][e] += t;
                g[i][e] *= w[i][e];
                sum[0] += g[i][e];
                sum[1] = fmaf(g[i][e], hat[i][e], sum[1]);
            }
        if (!A.gx) continue;
        row_sums<2, LANES>(sum, side[turn]);
        const float c1 = sum[0] / width, c2 = sum[1] / width;
        if (!live) continue;
        T* const gx = static_cast<T*>(A.gx) + row * A.ldgx;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int64_t at = (int64_t)(i * LANES + lane) * N;
#pragma unroll
            for (int e = 0; e < N; ++e) g[i][e] = rstd * (g[i][e] - c1 - hat[i][e] * c2);
            if (at < A.width) store_piece<T>(gx, at, A.width, g[i]);
        }
    }
    if (!A.parts) return;
    float* const parts = A.parts + (int64_t)blockIdx.x * 2 * A.width;
    const auto write = [&](float (&sums)[COUNT][N], float* out) {
        if (LANES < kThreads) {
            // the rows of the workgroup, in order
            for (int i = 0; i < COUNT; ++i) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < N; ++e) columns[LANES < kThreads ? r : 0][LANES < kThreads ? lane * N + e : 0] = sums[i][e];
                __syncthreads();
                for (int c = threadIdx.x; c < LANES * N; c += kThreads) {
                    float s = 0.0f;
                    for (int k = 0; k < ROWS; ++k) s += columns[LANES < kThreads ? k : 0][LANES < kThreads ? c : 0];
                    const int64_t at = (int64_t)i * LANES * N + c;
                    if (at < A.width) out[at] = s;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const int64_t at = (int64_t)(i * LANES + lane) * N;
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (at + e < A.width) out[at + e] = sums[i][e];
            }
        }
    };
    if (A.gweight) write(gw, parts);
    if (A.gbias) write(gb, parts + A.width);
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_backward_long(NormBackwardArgs A)
{
    constexpr int N = Piece<T>::N;
    __shared__ float side[2][kThreads / 64][2];
    const int64_t step = (int64_t)kThreads * N;
    const float width = (float)A.width;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < A.rows; row += gridDim.x, turn ^= 1) {
        const T* const x = static_cast<const T*>(A.x) + row * A.ldx;
        const T* const gy = static_cast<const T*>(A.gy) + row * A.ldgy;
        T* const gx = static_cast<T*>(A.gx) + row * A.ldgx;
        const float mean = A.mean[row], rstd = A.rstd[row];
        float v[N], g[N], w[N], sum[2] = {0.0f, 0.0f};
        const auto load = [&](int64_t at) {
            load_piece<T>(v, x, at, A.width);
            load_piece<T>(g, gy, at, A.width);
            load_weight<N>(w, A.weight, at, A.width, 1.0f);
#pragma unroll
            for (int e = 0; e < N; ++e) { v[e] = (v[e] - mean) * rstd; g[e] *= w[e]; }
        };
        for (int64_t at = (int64_t)threadIdx.x * N; at < A.width; at += step) {
            load(at);
            float s = 0.0f, t = 0.0f;
#pragma unroll
            for (int e = 0; e < N; ++e) { s += g[e]; t = fmaf(g[e], v[e], t); }
            sum[0] += s; sum[1] += t;
        }
        row_sums<2, kThreads>(sum, side[turn]);
        const float c1 = sum[0] / width, c2 = sum[1] / width;
        for (int64_t at = (int64_t)threadIdx.x * N; at < A.width; at += step) {
            load(at);
#pragma unroll
            for (int e = 0; e < N; ++e) g[e] = rstd * (g[e] - c1 - v[e] * c2);
            store_piece<T>(gx, at, A.width, g);
        }
    }
}

// Columns' sums of long rows: a workgroup takes kThreads columns of the rows blockIdx.y, + gridDim.y, ...
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_norm_columns_long(NormBackwardArgs A)
{
    const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (c >= A.width) return;
    float gw = 0.0f, gb = 0.0f;
    for (int64_t row = blockIdx.y; row < A.rows; row += gridDim.y) {
        const float g = to_float(static_cast<const T*>(A.gy)[row * A.ldgy + c]);
        const float hat = (to_float(static_cast<const T*>(A.x)[row * A.ldx + c]) - A.mean[row]) * A.rstd[row];
        gw = fmaf(g, hat, gw);
        gb += g;
    }
    float* const parts = A.parts + (int64_t)blockIdx.y * 2 * A.width;
    parts[c] = gw;
    parts[A.width + c] = gb;
}

// gweight, gbias <- the parts' sums: 32 columns of a workgroup, eight threads each.
__global__ void __launch_bounds__(kThreads)
k_norm_join(const float* parts, int64_t count, int64_t width, float* gweight, float* gbias)
{
    __shared__ float side[kThreads / 32][32];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float* const out = blockIdx.y ? gbias : gweight;
    if (!out) return;
    const float* const from = parts + (blockIdx.y ? width : 0) + c;
    float s = 0.0f;
    if (c < width) {
        int64_t p = group;
        for (; p + 7 * 8 < count; p += 64) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = from[(p + i * 8) * 2 * width];
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
        for (; p < count; p += 8) s += from[p * 2 * width];
    }
    side[group][lane] = s;
    __syncthreads();
    if (group == 0 && c < width) {
        float all = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) all += side[i][lane];
        out[c] = all;
    }
}

// threads of a row and pieces of each, by the width: part of a wavefront, a wavefront with one piece a thread or, if `two`, with two, or the workgroup
struct Plan { int lanes, count; };

Plan plan_of(int64_t pieces, bool two)
{
    for (int lanes = 1; lanes <= 64; lanes *= 2)
        if (pieces <= lanes) return {lanes, 1};
    if (two && pieces <= 128) return {64, 2};
    for (int count = 1; count <= kMost; count *= 2)
        if (pieces <= (int64_t)kThreads * count) return {kThreads, count};
    return {0, 0};
}

// Forward, workgroups that go over the rows with the weights in registers: us with 1024 / 2048 / 4096 / one for each row, bf16: 32768 rows of 4096 132 / 136 / 133 / 152, 524288 of 128
// 77 / 69 / 68 / 63, 65536 of 1024 71 / 74 / 72 / 72, 16384 of 8192 204 / 207 / 210 / 222; fp32, the same rows: 219 / 211 / 207 / 195, 114 / 120 / 118 / 122, 122 / 110 / 110 / 125,
// 214 / 205 / 203 / 212.  2048 and 4096 are alike within 2 %; each of the others loses a tenth somewhere.  Backward, workgroups that keep sums of columns, 512 / 1024 / 2048: 32768 of 4096 396 / 321 / 349, 524288 of 128 219 / 166 / 177; each has two turns at least where there are
// more than 256, since it writes as much as a row of sums: 1024 of 8192 in 512 / 1024 parts 63 / 87.
constexpr int64_t kForwardWorkgroups = 2048, kPartWorkgroups = 1024, kLeastParts = 256, kMostWorkgroups = int64_t(1) << 22;      // (a grid holds fewer than 2^32 threads)

unsigned workgroups(int64_t wanted) { return (unsigned)(wanted < kMostWorkgroups ? wanted : kMostWorkgroups); }

int64_t pieces_of(bool bf16, int64_t width) { return bf16 ? (width + 7) / 8 : (width + 3) / 4; }

int64_t parts_of(const Plan& P, int64_t rows)
{
    const int64_t at_once = P.lanes ? kThreads / P.lanes : 1, all = (rows + at_once - 1) / at_once;
    const int64_t some = all / 2 > kLeastParts ? all / 2 : all < kLeastParts ? all : kLeastParts;
    return some < kPartWorkgroups ? some : kPartWorkgroups;
}

template <typename T, int LANES, int COUNT>
hipError_t forward_with(const NormArgs& A, hipStream_t st)
{
    constexpr int ROWS = kThreads / LANES;
    hipLaunchKernelGGL((k_norm<T, LANES, COUNT>), dim3((unsigned)((A.rows + ROWS - 1) / ROWS < kForwardWorkgroups ? (A.rows + ROWS - 1) / ROWS : kForwardWorkgroups)), dim3(kThreads), 0, st, A);
    return hipGetLastError();
}

template <typename T, int LANES, int COUNT>
hipError_t backward_with(const NormBackwardArgs& A, int64_t parts, hipStream_t st)
{
    hipLaunchKernelGGL((k_norm_parts<T, LANES, COUNT>), dim3((unsigned)parts), dim3(kThreads), 0, st, A);
    return hipGetLastError();
}

#define NORM_PLANS(call)                                                                                                          \
    do {                                                                                                                          \
        if (P.lanes == kThreads)                                                                                                  \
            return P.count == 1 ? call(kThreads, 1) : P.count == 2 ? call(kThreads, 2) : P.count == 4 ? call(kThreads, 4) : call(kThreads, 8); \
        if (P.lanes == 64) return P.count == 1 ? call(64, 1) : call(64, 2);                                                       \
        return P.lanes == 32 ? call(32, 1) : P.lanes == 16 ? call(16, 1) : P.lanes == 8 ? call(8, 1) : P.lanes == 4 ? call(4, 1) : P.lanes == 2 ? call(2, 1) : call(1, 1); \
    } while (0)

template <typename T>
hipError_t forward_of(const NormArgs& A, const Plan& P, hipStream_t st)
{
    if (P.lanes == 0) {
        hipLaunchKernelGGL((k_norm_long<T>), dim3(workgroups(A.rows)), dim3(kThreads), 0, st, A);
        return hipGetLastError();
    }
#define NORM_CALL(lanes, count) forward_with<T, lanes, count>(A, st)
    NORM_PLANS(NORM_CALL);
#undef NORM_CALL
}

template <typename T>
hipError_t backward_of(const NormBackwardArgs& A, const Plan& P, int64_t parts, hipStream_t st)
{
    if (P.lanes == 0) {
        // (the columns first: gx may take the place of gy)
        if (A.parts)
            hipLaunchKernelGGL((k_norm_columns_long<T>), dim3((unsigned)((A.width + kThreads - 1) / kThreads), (unsigned)parts), dim3(kThreads), 0, st, A);
        if (A.gx) hipLaunchKernelGGL((k_norm_backward_long<T>), dim3(workgroups(A.rows)), dim3(kThreads), 0, st, A);
        return hipGetLastError();
    }
#define NORM_CALL(lanes, count) backward_with<T, lanes, count>(A, parts, st)
    NORM_PLANS(NORM_CALL);
#undef NORM_CALL
}

}  // namespace

size_t norm_workspace(int64_t rows, int64_t width)
{
    // (of either type, and of any number of rows up to these)
    int64_t most = 0;
    for (int bf16 = 0; bf16 < 2; ++bf16) {
        const int64_t parts = parts_of(plan_of(pieces_of(bf16 != 0, width), true), rows);
        most = parts > most ? parts : most;
    }
    return (size_t)most * 2 * (size_t)width * sizeof(float);
}

hipError_t launch_norm(const NormArgs& A, hipStream_t st)
{
    // Rows of two pieces a lane: a wavefront for a row where there are rows for all of them (no barrier), else the workgroup.  us, rows of 1024 in bf16, wavefront / workgroup:
    // 64 rows 7.2 / 6.4, 512 7.4 / 6.5, 1024 7.7 / 7.5, 2048 8.6 / 8.8, 4096 10.2 / 11.7, 32768 41 / 48.
    const Plan P = plan_of(pieces_of(A.bf16, A.width), A.rows >= 2048);
    profile_before("norm", st);
    const hipError_t e = A.bf16 ? forward_of<__bf16>(A, P, st) : forward_of<float>(A, P, st);
    profile_after("norm", st);
    return e;
}

hipError_t launch_norm_backward(const NormBackwardArgs& A, hipStream_t st)
{
    // (wavefront / workgroup for rows of two pieces a lane: 8192 of 1024 in bf16 38 / 48 us)
    const Plan P = plan_of(pieces_of(A.bf16, A.width), true);
    const int64_t parts = parts_of(P, A.rows);
    if (A.rows > 0) {
        profile_before("norm_backward", st);
        const hipError_t e = A.bf16 ? backward_of<__bf16>(A, P, parts, st) : backward_of<float>(A, P, parts, st);
        profile_after("norm_backward", st);
        if (e != hipSuccess) return e;
    }
    if (!A.gweight && !A.gbias) return hipSuccess;
    profile_before("norm_join", st);
    hipLaunchKernelGGL(k_norm_join, dim3((unsigned)((A.width + 31) / 32), 2), dim3(kThreads), 0, st, A.parts, parts, A.width, A.gweight, A.gbias);
    profile_after("norm_join", st);
    return hipGetLastError();
}

}  // namespace laplex
