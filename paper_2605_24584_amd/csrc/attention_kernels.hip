// Linear attention with a decay for each head: the causal Laplace kernel exp(-rate (t - s)), s <= t, over token positions,
// weighted by (q_t . k_s).
#include "token_internal.h"

namespace laplex {

namespace {

constexpr int kStepThreads = 256;

__device__ __forceinline__ float rate_of(const float* rates, int h)
{
    return fminf(rates[h], 1.0e30f);      // an infinite rate: nothing but the token itself, and 0 * rate stays 0
}

__device__ __forceinline__ void sequence_rows(const int64_t* starts, int64_t tokens, int64_t sequences, int64_t b, int64_t* begin, int64_t* count)
{
    if (!starts) { *count = tokens / sequences; *begin = b * *count; return; }
    int64_t lo = starts[b], hi = starts[b + 1];                       // whatever they hold, no row outside the matrices is touched
    lo = lo < 0 ? 0 : lo > tokens ? tokens : lo;
    hi = hi < lo ? lo : hi > tokens ? tokens : hi;
    *begin = lo; *count = hi - lo;
}

// The recurrence S <- l S + k v^T token by token: 16 columns of one head of one sequence, 16 lanes of a wavefront share a
// column, each with every 16th row of it.
template <typename T>
__global__ void __launch_bounds__(256)
k_attention_recurrent(AttentionArgs A)
{
    const Walk W = A.walk[blockIdx.z];
    const int slices = (W.dv + 15) / 16;
    const int64_t b = blockIdx.x / slices;
    const int slice = blockIdx.x % slices, h = blockIdx.y;
    if (b >= A.sequences) return;
    const int part = threadIdx.x & 15, col = slice * 16 + (threadIdx.x >> 4);
    const float rate = rate_of(A.rates, h), decay = expf(-rate);
    int64_t begin, count;
    sequence_rows(A.starts, A.tokens, A.sequences, b, &begin, &count);
    const bool live = col < W.dv;
    float S[16];
    const int64_t at = (b * A.heads + h) * (int64_t)W.dk * W.dv;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int row = i * 16 + part;
        S[i] = 0.0f;
        if (W.state_in && live && row < W.dk)
            S[i] = W.in_scale * W.state_in[at + (W.transposed ? (int64_t)col * W.dk + row : (int64_t)row * W.dv + col)];
    }
    for (int64_t u = 0; u < count; ++u) {
        const int64_t t = begin + (W.reverse ? count - 1 - u : u);
        const T* q = static_cast<const T*>(W.q) + t * W.ldq + (int64_t)h * W.dk;
        const T* k = static_cast<const T*>(W.k) + t * W.ldk + (int64_t)h * W.dk;
        const float v = live ? to_float(static_cast<const T*>(W.v)[t * W.ldv + (int64_t)h * W.dv + col]) : 0.0f;
        const float d = (u == 0 && W.lead == 0) ? 1.0f : decay;
        float o = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = i * 16 + part;
            if (row < W.dk) {
                S[i] = S[i] * d + to_float(k[row]) * v;
                o += S[i] * to_float(q[row]);
            }
        }
#pragma unroll
        for (int m = 8; m >= 1; m >>= 1) o += __shfl_xor(o, m);
        if (W.out && live && part == 0) static_cast<T*>(W.out)[t * W.ldo + (int64_t)h * W.dv + col] = (T)(o * W.out_scale);
    }
    if (W.state_out && live) {
        const float d = (W.lead == 0 && count > 0) ? decay : 1.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = i * 16 + part;
            if (row < W.dk) W.state_out[at + (int64_t)row * W.dv + col] = W.last_scale * (S[i] * d);
        }
    }
}

// One token for every sequence: a workgroup per (sequence, head), a thread per column and part of the rows.
template <typename T>
__global__ void __launch_bounds__(kStepThreads)
k_attention_step(AttentionStepArgs A)
{
    const int64_t b = blockIdx.x;
    const int h = blockIdx.y;
    const float decay = expf(-rate_of(A.rates, h));
    const T* q = static_cast<const T*>(A.q) + b * A.ldq + (int64_t)h * A.dk;
    const T* k = static_cast<const T*>(A.k) + b * A.ldk + (int64_t)h * A.dk;
    const T* v = static_cast<const T*>(A.v) + b * A.ldv + (int64_t)h * A.dv;
    float* S = A.state + (b * A.heads + h) * (int64_t)A.dk * A.dv;
    for (int col = threadIdx.x; col < A.dv; col += kStepThreads) {
        const float vc = to_float(v[col]);
        float o = 0.0f;
        for (int row = 0; row < A.dk; ++row) {
            const float s = S[(int64_t)row * A.dv + col] * decay + to_float(k[row]) * vc;
            S[(int64_t)row * A.dv + col] = s;
            o += to_float(q[row]) * s;
        }
        static_cast<T*>(A.y)[b * A.ldy + (int64_t)h * A.dv + col] = (T)(A.scale * o);
    }
}

}  // namespace

size_t attention_workspace(bool, int64_t, int64_t, int, int, int) { return 0; }

hipError_t launch_attention(const AttentionArgs& A, hipStream_t st)
{
    int most = 0;
    for (int w = 0; w < A.walks; ++w) most = A.walk[w].dv > most ? A.walk[w].dv : most;
    const dim3 grid((unsigned)(A.sequences * ((most + 15) / 16)), (unsigned)A.heads, (unsigned)A.walks);
    profile_before("attention", st);
    if (A.bf16) hipLaunchKernelGGL((k_attention_recurrent<__bf16>), grid, dim3(256), 0, st, A);
    else hipLaunchKernelGGL((k_attention_recurrent<float>), grid, dim3(256), 0, st, A);
    profile_after("attention", st);
    return hipGetLastError();
}

hipError_t launch_attention_step(const AttentionStepArgs& A, hipStream_t st)
{
    const dim3 grid((unsigned)A.sequences, (unsigned)A.heads);
    profile_before("attention_step", st);
    if (A.bf16) hipLaunchKernelGGL((k_attention_step<__bf16>), grid, dim3(kStepThreads), 0, st, A);
    else hipLaunchKernelGGL((k_attention_step<float>), grid, dim3(kStepThreads), 0, st, A);
    profile_after("attention_step", st);
    return hipGetLastError();
}

}  // namespace laplex
