// Log probabilities, entropy and the likeliest alternatives over logits y[k][batch], and the gradient into the logits.
#include "token_internal.h"

namespace laplex {

namespace {

// A logit as a whole number in the order of the values: -0 equals +0, NaN comes before all numbers.
__device__ __forceinline__ uint32_t order_of(float v)
{
    if (v != v) return 0xFFFFFFFFu;
    const uint32_t bits = __float_as_uint(v + 0.0f);
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

// one workgroup per column: three passes over its rows, then one pass per alternative
template <typename T>
__global__ void __launch_bounds__(256)
k_logprob_column(LogprobArgs A)
{
    __shared__ float red[256], red2[256];
    __shared__ unsigned long long key[256];
    const int64_t t = blockIdx.x;
    const T* y = static_cast<const T*>(A.y) + t;
    const int x = threadIdx.x;
    float m = -INFINITY;
    for (int64_t i = x; i < A.k; i += 256) m = fmaxf(m, to_float(y[i * A.ldy]));
    red[x] = m;
    __syncthreads();
    for (int s = 128; s >= 1; s >>= 1) { if (x < s) red[x] = fmaxf(red[x], red[x + s]); __syncthreads(); }
    m = red[0];
    __syncthreads();
    const float base = m == -INFINITY ? 0.0f : m;
    float sum = 0.0f, away = 0.0f;
    for (int64_t i = x; i < A.k; i += 256) {
        const float d = (to_float(y[i * A.ldy]) - base) * A.tau, e = expf(d);
        sum += e;
        away += e > 0.0f ? e * d : 0.0f;
    }
    red[x] = sum; red2[x] = away;
    __syncthreads();
    for (int s = 128; s >= 1; s >>= 1) { if (x < s) { red[x] += red[x + s]; red2[x] += red2[x + s]; } __syncthreads(); }
    sum = red[0]; away = red2[0];
    const float log_sum = logf(sum);
    if (x == 0) {
        if (A.lse) A.lse[t] = base * A.tau + log_sum;
        if (A.entropy) A.entropy[t] = sum == 0.0f ? 0.0f : log_sum - away / sum;
        if (A.logp) {
            const int64_t target = A.targets[t];
            float out = 0.0f;
            if (target >= 0 && target < A.k) out = sum == 0.0f ? -INFINITY : (to_float(y[target * A.ldy]) - base) * A.tau - log_sum;
            A.logp[t] = out;
        }
    }
    unsigned long long below = ~0ull;
    for (int r = 0; r < A.top; ++r) {
        unsigned long long best = 0;
        for (int64_t i = x; i < A.k; i += 256) {
            const unsigned long long mine = ((unsigned long long)order_of(to_float(y[i * A.ldy])) << 32) | (uint32_t)(0xFFFFFFFFu - (uint32_t)i);
            if (mine < below && mine > best) best = mine;
        }
        __syncthreads();
        key[x] = best;
        __syncthreads();
        for (int s = 128; s >= 1; s >>= 1) { if (x < s) key[x] = key[x] > key[x + s] ? key[x] : key[x + s]; __syncthreads(); }
        below = key[0];
        if (x == 0) {
            const int64_t id = (int64_t)(0xFFFFFFFFu - (uint32_t)below);
            A.top_ids[r * A.batch + t] = id;
            A.top_logp[r * A.batch + t] = sum == 0.0f ? -INFINITY : (to_float(y[id * A.ldy]) - base) * A.tau - log_sum;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256)
k_logprob_backward(LogprobBackwardArgs A)
{
    const int64_t total = A.k * A.batch;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / A.batch, t = i - r * A.batch;
        const float lse = A.lse[t], logp = to_float(static_cast<const T*>(A.y)[r * A.ldy + t]) * A.tau - lse;
        const float p = lse == -INFINITY ? 0.0f : expf(logp);
        float g = 0.0f;
        if (A.glogp) {
            const int64_t target = A.targets[t];
            if (target >= 0 && target < A.k) g += A.glogp[t] * ((r == target && lse != -INFINITY ? 1.0f : 0.0f) - p);
        }
        if (A.gentropy && p > 0.0f) g -= A.gentropy[t] * (p * (logp + A.entropy[t]));
        if (A.glse) g += A.glse[t] * p;
        if (p != p) g = p;
        static_cast<T*>(A.gy)[r * A.ldgy + t] = (T)(A.tau * g);
    }
}

}  // namespace

size_t logprob_workspace(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_logprob(const LogprobArgs& A, hipStream_t st)
{
    profile_before("logprob", st);
    if (A.bf16) hipLaunchKernelGGL((k_logprob_column<__bf16>), dim3((unsigned)A.batch), dim3(256), 0, st, A);
    else hipLaunchKernelGGL((k_logprob_column<float>), dim3((unsigned)A.batch), dim3(256), 0, st, A);
    profile_after("logprob", st);
    return hipGetLastError();
}

hipError_t launch_logprob_backward(const LogprobBackwardArgs& A, hipStream_t st)
{
    const int64_t blocks = (A.k * A.batch + 255) / 256;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536));
    profile_before("logprob_backward", st);
    if (A.bf16) hipLaunchKernelGGL((k_logprob_backward<__bf16>), grid, dim3(256), 0, st, A);
    else hipLaunchKernelGGL((k_logprob_backward<float>), grid, dim3(256), 0, st, A);
    profile_after("logprob_backward", st);
    return hipGetLastError();
}

}  // namespace laplex
