// Log probabilities, entropy and the likeliest alternatives over logits y[k][batch] (a row per vocabulary entry), and the
// gradient into the logits.
//
// Per column, with m = max y, d = y - m:   s = sum exp(tau d),  w = sum d exp(tau d);
//   lse = tau m + log s,   entropy = log s - tau w / s,   logp = tau (y - m) - log s.
// One pass over the logits (k_logprob_rows): a thread holds (m, s, w) of up to four neighbouring columns and takes groups of kGroup consecutive
// rows; the running maximum and the rescaling cost it one more exponential per group.  A second launch (k_logprob_finish), a
// wavefront per column, brings the parts together.
//
// Alternatives: the pass also writes the maximum of every group (1 / kGroup of what it reads).  Values are ordered by size and, of
// equal ones, by row.  A value among the `top` largest lies in one of the `top` groups with the largest maxima (ties: the first
// ones): otherwise each of those holds a value before it.  So the second launch picks among groups of groups, opens those,
// picks groups, opens those, and picks rows: a few hundred values per column instead of k.
#include "token_internal.h"

namespace laplex {

namespace {

constexpr int kGroup = 16;            // rows whose maximum is kept
constexpr int kSuper = 8;             // groups that are looked at together first
constexpr int kPick = 16;             // values per lane that a choice is made among
constexpr int kDirect = 64 * kPick;   // rows that need no groups
constexpr int kRowThreads = 256;

// ----------------------------------------------------------------------------
// Up to four neighbouring logits; rows need not be aligned to more than one.
// ----------------------------------------------------------------------------
template <typename T, int VEC> struct Lane;
template <> struct Lane<float, 1> { typedef float type; };
template <> struct Lane<__bf16, 1> { typedef __bf16 type; };
template <> struct Lane<float, 4> { typedef float type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Lane<__bf16, 4> { typedef __bf16 type __attribute__((ext_vector_type(4), aligned(2))); };

__device__ __forceinline__ float part(float v, int) { return v; }
__device__ __forceinline__ float part(__bf16 v, int) { return (float)v; }
__device__ __forceinline__ float part(Lane<float, 4>::type v, int c) { return v[c]; }
__device__ __forceinline__ float part(Lane<__bf16, 4>::type v, int c) { return (float)v[c]; }

// `have` of the VEC columns at p exist
template <typename T, int VEC>
__device__ __forceinline__ void load_columns(float* out, const T* p, int have)
{
    if (have >= VEC) {
        const typename Lane<T, VEC>::type v = *reinterpret_cast<const typename Lane<T, VEC>::type*>(p);
#pragma unroll
        for (int c = 0; c < VEC; ++c) out[c] = part(v, c);
    } else {
#pragma unroll
        for (int c = 0; c < VEC; ++c) out[c] = c < have ? to_float(p[c]) : -INFINITY;
    }
}

struct Stats { float m, s, w; };      // maximum, sum exp(tau (y - m)), sum (y - m) exp(tau (y - m))

__device__ __forceinline__ float exp_of(float d, float c) { return __builtin_amdgcn_exp2f(d * c); }      // c = tau / log 2

// brings the sums of `a` to the maximum m >= a.m (a maximum of -inf: there is nothing in them)
__device__ __forceinline__ void rebase(Stats& a, float m, float c)
{
    const float d = a.m == -INFINITY ? 0.0f : a.m - m;
    const float e = exp_of(d, c);
    a.w = e > 0.0f ? (a.w + d * a.s) * e : (a.s != a.s ? a.s : 0.0f);
    a.s = a.s * e;
    a.m = m;
}

__device__ __forceinline__ Stats join(Stats a, Stats b, float c)
{
    const float m = fmaxf(a.m, b.m);
    rebase(a, m, c);
    rebase(b, m, c);
    return Stats{m, a.s + b.s, a.w + b.w};
}

// ----------------------------------------------------------------------------
// The pass over the logits.  lanes_log2: 2^that lanes across the columns, the rest of the workgroup across groups of rows.
// parts[(part * 3 + {m, s, w}) * batch + column].
// ----------------------------------------------------------------------------
struct RowsArgs {
    const void* y;
    int64_t ldy, k, batch;
    float c;
    int lanes_log2, turns;            // groups of rows per thread
    int64_t slabs;
    float *parts, *maxima;
};

template <typename T, int VEC, bool TOP>
__global__ void __launch_bounds__(kRowThreads)
k_logprob_rows(RowsArgs A)
{
    __shared__ Stats side[kRowThreads / 64][64][VEC];
    const int lanes = 1 << A.lanes_log2, x = threadIdx.x, column_lane = x & (lanes - 1), row_lane = x >> A.lanes_log2;
    const int row_lanes = kRowThreads >> A.lanes_log2;
    const int64_t slab = blockIdx.x % A.slabs, block = blockIdx.x / A.slabs;
    const int64_t t = (slab * lanes + column_lane) * VEC;
    const int have = A.batch - t >= VEC ? VEC : A.batch > t ? (int)(A.batch - t) : 0;
    Stats st[VEC];
#pragma unroll
    for (int c = 0; c < VEC; ++c) st[c] = Stats{-INFINITY, 0.0f, 0.0f};
    if (have > 0) {
        for (int n = 0; n < A.turns; ++n) {
            const int64_t group = (block * A.turns + n) * row_lanes + row_lane, row = group * kGroup;
            if (row >= A.k) break;
            const T* p = static_cast<const T*>(A.y) + row * A.ldy + t;
            const int rows = A.k - row < kGroup ? (int)(A.k - row) : kGroup;
            float v[kGroup][VEC];
            if (rows == kGroup) {
#pragma unroll
                for (int i = 0; i < kGroup; ++i) load_columns<T, VEC>(v[i], p + i * A.ldy, have);
            } else {
#pragma unroll
                for (int i = 0; i < kGroup; ++i) {
                    if (i < rows) load_columns<T, VEC>(v[i], p + i * A.ldy, have);
                    else
#pragma unroll
                        for (int c = 0; c < VEC; ++c) v[i][c] = -INFINITY;
                }
            }
#pragma unroll
            for (int c = 0; c < VEC; ++c) {
                float m = v[0][c];
                bool nan = m != m;
#pragma unroll
                for (int i = 1; i < kGroup; ++i) {
                    m = fmaxf(m, v[i][c]);
                    if (TOP) nan = nan || v[i][c] != v[i][c];
                }
                if (TOP && c < have) A.maxima[group * A.batch + t + c] = nan ? NAN : m;
                rebase(st[c], fmaxf(st[c].m, m), A.c);
                const float base = st[c].m == -INFINITY ? 0.0f : st[c].m;
                float s = 0.0f, w = 0.0f;
#pragma unroll
                for (int i = 0; i < kGroup; ++i) {
                    const float d = v[i][c] - base, e = exp_of(d, A.c);
                    s += e;
                    w += e > 0.0f ? d * e : 0.0f;
                }
                st[c].s += s;
                st[c].w += w;
            }
        }
    }
    // over the rows of a wavefront, then over the wavefronts
#pragma unroll
    for (int c = 0; c < VEC; ++c)
        for (int step = lanes; step < 64; step <<= 1) {
            const Stats other{__shfl_xor(st[c].m, step), __shfl_xor(st[c].s, step), __shfl_xor(st[c].w, step)};
            st[c] = join(st[c], other, A.c);
        }
    // (a wavefront holds min(64, lanes) columns' lanes)
#pragma unroll
    for (int c = 0; c < VEC; ++c) side[x >> 6][x & 63][c] = st[c];
    __syncthreads();
    if (x < lanes && have > 0) {
        float* const out = A.parts + block * 3 * A.batch + t;
#pragma unroll
        for (int c = 0; c < VEC; ++c) {
            Stats all = side[0][x][c];
            for (int wave = 1; wave < kRowThreads / 64; ++wave) all = join(all, side[wave][x][c], A.c);
            if (c < have) { out[c] = all.m; out[A.batch + c] = all.s; out[2 * A.batch + c] = all.w; }
        }
    }
}

// ----------------------------------------------------------------------------
// A wavefront chooses the `want` largest of up to 64 N values: keys in the order of the values, key[r] of lane l is value
// 64 r + l, and of equal ones the first are taken; key 0: no value.
// ----------------------------------------------------------------------------

// A logit as a whole number in the order of the values: -0 equals +0, NaN comes before all numbers; never 0.
__device__ __forceinline__ uint32_t order_of(float v)
{
    if (v != v) return 0xFFFFFFFFu;
    const uint32_t bits = __float_as_uint(v + 0.0f);
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

// what lanes of the wavefront have written to LDS is there for the others
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// chosen[0 .. count) <- numbers of the chosen values, ascending; keys[] <- their keys (may be null).  Returns count (uniform).
__device__ __forceinline__ int choose(const uint32_t (&key)[kPick], int used, int want, int* chosen, uint32_t* keys)
{
    const int lane = threadIdx.x & 63;
    const uint64_t below = (1ull << lane) - 1ull;
    // the largest bound that `want` values reach, bit by bit
    uint32_t bound = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t trial = bound | (1u << bit);
        int count = 0;
#pragma unroll
        for (int r = 0; r < kPick; ++r)
            if (r < used) count += __popcll(__ballot(key[r] >= trial));
        if (count >= want) bound = trial;
    }
    int above = 0;
#pragma unroll
    for (int r = 0; r < kPick; ++r)
        if (r < used) above += __popcll(__ballot(key[r] > bound));
    int equal = bound == 0 ? 0 : want - above, count = 0;      // how many of those at the bound are taken
#pragma unroll
    for (int r = 0; r < kPick; ++r)
        if (r < used) {
            const uint64_t same = __ballot(key[r] == bound);
            const bool mine = key[r] > bound || (key[r] == bound && __popcll(same & below) < equal);
            equal -= __popcll(same);
            equal = equal < 0 ? 0 : equal;
            const uint64_t all = __ballot(mine);
            if (mine) {
                const int at = count + __popcll(all & below);
                chosen[at] = r * 64 + lane;
                if (keys) keys[at] = key[r];
            }
            count += __popcll(all);
        }
    wave_sync();
    return count;
}

struct FinishArgs {
    LogprobArgs L;
    const float *parts, *maxima;
    int64_t part_count, groups;
    float c;
};

constexpr int kFinishWaves = 4;
constexpr int kMaxTop = 64;

template <typename T>
__global__ void __launch_bounds__(kFinishWaves * 64)
k_logprob_finish(FinishArgs F)
{
    __shared__ int list_a[kFinishWaves][kMaxTop], list_b[kFinishWaves][kMaxTop];
    __shared__ uint32_t stage[kFinishWaves][kDirect];      // keys on their way into the registers
    __shared__ uint32_t keys_a[kFinishWaves][kMaxTop], best_key[kFinishWaves][2 * kMaxTop], best_row[kFinishWaves][2 * kMaxTop];
    const LogprobArgs& A = F.L;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t = (int64_t)blockIdx.x * kFinishWaves + wave;
    if (t >= A.batch) return;                        // (nothing below is for the whole workgroup)
    const T* const y = static_cast<const T*>(A.y) + t;

    Stats st{-INFINITY, 0.0f, 0.0f};
    for (int64_t p = lane; p < F.part_count; p += 64) {
        const float* const at = F.parts + p * 3 * A.batch + t;
        st = join(st, Stats{at[0], at[A.batch], at[2 * A.batch]}, F.c);
    }
    for (int step = 32; step >= 1; step >>= 1) {
        const Stats other{__shfl_xor(st.m, step), __shfl_xor(st.s, step), __shfl_xor(st.w, step)};
        st = join(st, other, F.c);
    }
    const bool empty = st.m == -INFINITY && st.s == 0.0f;
    const float log_sum = logf(st.s);
    auto logp_of = [&](float v) { return empty ? -INFINITY : (v - st.m) * A.tau - log_sum; };
    if (lane == 0) {
        if (A.lse) A.lse[t] = empty ? -INFINITY : st.m * A.tau + log_sum;
        if (A.entropy) A.entropy[t] = empty ? 0.0f : log_sum - A.tau * (st.w / st.s);
        if (A.logp) {
            const int64_t target = A.targets[t];
            A.logp[t] = target >= 0 && target < A.k ? logp_of(to_float(y[target * A.ldy])) : 0.0f;
        }
    }
    if (A.top == 0) return;

    int *const la = list_a[wave], *const lb = list_b[wave];
    uint32_t *const ka = keys_a[wave], *const bk = best_key[wave], *const br = best_row[wave];
    uint32_t* const sk = stage[wave];
    int best = 0;                                    // values chosen so far, by row, in bk and br
    auto take = [&](uint32_t (&key)[kPick], int used) {
        wave_sync();
#pragma unroll
        for (int r = 0; r < kPick; ++r) key[r] = r < used ? sk[r * 64 + lane] : 0;
        wave_sync();
    };
    const int want = A.top;
    uint32_t key[kPick];
    // stretches of kDirect rows, or of kDirect groups of groups
    const int64_t span = A.k <= kDirect ? kDirect : (int64_t)kDirect * kSuper * kGroup;
    for (int64_t first = 0; first < A.k; first += span) {
        int used, count;
        if (A.k > kDirect) {
            const int64_t group0 = first / kGroup, left = F.groups - group0;
            const float* const maxima = F.maxima + group0 * A.batch + t;
            const int supers = (int)((left + kSuper - 1) / kSuper < kDirect ? (left + kSuper - 1) / kSuper : kDirect);
            used = (supers + 63) / 64;
#pragma unroll 2
            for (int r = 0; r < used; ++r) {
                const int64_t g = (int64_t)(r * 64 + lane) * kSuper;
                float v[kSuper];
#pragma unroll
                for (int i = 0; i < kSuper; ++i) v[i] = g + i < left ? maxima[(g + i) * A.batch] : -INFINITY;
                uint32_t most = 0;
#pragma unroll
                for (int i = 0; i < kSuper; ++i) { const uint32_t o = order_of(v[i]); most = o > most ? o : most; }
                sk[r * 64 + lane] = g < left ? most : 0;
            }
            take(key, used);
            count = choose(key, used, want, la, nullptr);
            const int groups = count * kSuper;
            used = (groups + 63) / 64;
#pragma unroll 4
            for (int n = lane; n < used * 64; n += 64) {
                const int64_t g = n < groups ? (int64_t)la[n / kSuper] * kSuper + n % kSuper : left;
                sk[n] = g < left ? order_of(maxima[g * A.batch]) : 0;
            }
            take(key, used);
            count = choose(key, used, want, lb, nullptr);
            for (int n = lane; n < count; n += 64) lb[n] = la[lb[n] / kSuper] * kSuper + lb[n] % kSuper;
            wave_sync();
            const int rows = count * kGroup;
            used = (rows + 63) / 64;
#pragma unroll 4
            for (int n = lane; n < used * 64; n += 64) {
                const int64_t row = n < rows ? first + (int64_t)lb[n / kGroup] * kGroup + n % kGroup : A.k;
                sk[n] = row < A.k ? order_of(to_float(y[row * A.ldy])) : 0;
            }
        } else {
            used = (int)((A.k + 63) / 64);
#pragma unroll 4
            for (int n = lane; n < used * 64; n += 64) sk[n] = n < A.k ? order_of(to_float(y[n * A.ldy])) : 0;
        }
        take(key, used);
        count = choose(key, used, want, la, ka);
        for (int n = lane; n < count; n += 64) {
            const int c = la[n];
            br[best + n] = (uint32_t)(A.k > kDirect ? first + (int64_t)lb[c / kGroup] * kGroup + c % kGroup : c);
            bk[best + n] = ka[n];
        }
        wave_sync();
        best += count;
        if (best > want) {                           // more than one stretch: the earlier one's rows come first
#pragma unroll
            for (int r = 0; r < kPick; ++r) key[r] = r < 2 && r * 64 + lane < best ? bk[r * 64 + lane] : 0;
            best = choose(key, 2, want, la, ka);
            const uint32_t row = lane < best ? br[la[lane]] : 0;
            wave_sync();
            if (lane < best) { br[lane] = row; bk[lane] = ka[lane]; }
            wave_sync();
        }
    }
    if (lane < best) {
        const uint32_t mine = bk[lane], row = br[lane];
        int rank = 0;
        for (int n = 0; n < best; ++n) rank += bk[n] > mine || (bk[n] == mine && n < lane);
        A.top_ids[rank * A.batch + t] = row;
        A.top_logp[rank * A.batch + t] = logp_of(to_float(y[row * A.ldy]));
    }
}

// ----------------------------------------------------------------------------
// gy = tau p ( glse - glogp - gentropy (log p + entropy) ) + tau glogp at the target.  One read and one write per logit.
// ----------------------------------------------------------------------------
struct BackwardArgs {
    LogprobBackwardArgs B;
    int lanes_log2, turns;
    int64_t slabs;
};

constexpr int kBackRows = 8;

template <typename T, int VEC>
__global__ void __launch_bounds__(kRowThreads)
k_logprob_backward(BackwardArgs F)
{
    const LogprobBackwardArgs& A = F.B;
    const int lanes = 1 << F.lanes_log2, x = threadIdx.x, column_lane = x & (lanes - 1), row_lane = x >> F.lanes_log2;
    const int row_lanes = kRowThreads >> F.lanes_log2;
    const int64_t slab = blockIdx.x % F.slabs, block = blockIdx.x / F.slabs;
    const int64_t t = (slab * lanes + column_lane) * VEC;
    const int have = A.batch - t >= VEC ? VEC : A.batch > t ? (int)(A.batch - t) : 0;
    if (have == 0) return;
    float lse[VEC], one[VEC], logs[VEC], hit[VEC];
    int64_t target[VEC];
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
        const int64_t at = t + (c < have ? c : 0);
        lse[c] = A.lse[at];
        target[c] = -1; hit[c] = 0.0f;
        one[c] = A.glse ? A.glse[at] : 0.0f;
        logs[c] = 0.0f;
        if (A.glogp) {
            const int64_t given = A.targets[at];
            if (given >= 0 && given < A.k) { hit[c] = A.glogp[at]; one[c] -= hit[c]; target[c] = given; }
        }
        if (A.gentropy) { logs[c] = -A.gentropy[at]; one[c] += logs[c] * A.entropy[at]; }
        if (lse[c] == -INFINITY) { lse[c] = 0.0f; target[c] = -1; }      // nothing but -inf: p is 0 everywhere
    }
    for (int n = 0; n < F.turns; ++n) {
        const int64_t row0 = ((block * F.turns + n) * row_lanes + row_lane) * kBackRows;
        if (row0 >= A.k) break;
        const T* p = static_cast<const T*>(A.y) + row0 * A.ldy + t;
        T* g = static_cast<T*>(A.gy) + row0 * A.ldgy + t;
        float v[kBackRows][VEC];
#pragma unroll
        for (int i = 0; i < kBackRows; ++i)
            if (row0 + i < A.k) load_columns<T, VEC>(v[i], p + i * A.ldy, have);
#pragma unroll
        for (int i = 0; i < kBackRows; ++i) {
            if (row0 + i >= A.k) break;
            typename Lane<T, VEC>::type out;
#pragma unroll
            for (int c = 0; c < VEC; ++c) {
                const float logp = fmaf(v[i][c], A.tau, -lse[c]), q = expf(logp);
                float r = q == 0.0f ? 0.0f : q * fmaf(logs[c], logp, one[c]);
                if (row0 + i == target[c]) r += hit[c];
                if constexpr (VEC == 1) out = (T)(A.tau * r);
                else out[c] = (T)(A.tau * r);
            }
            if (have >= VEC) *reinterpret_cast<typename Lane<T, VEC>::type*>(g + i * A.ldgy) = out;
            else if constexpr (VEC > 1) {
#pragma unroll
                for (int c = 0; c < VEC; ++c)
                    if (c < have) g[i * A.ldgy + c] = out[c];
            }
        }
    }
}

// Lanes across the columns, and how often a thread takes rows: about kTarget workgroups, if there are rows for them.
struct Shape {
    int vec, lanes_log2, turns;
    int64_t slabs, blocks;
};

Shape shape_of(int64_t k, int64_t batch, int rows, int64_t target)
{
    Shape S;
    S.vec = batch >= 4 ? 4 : 1;
    const int64_t wide = (batch + S.vec - 1) / S.vec;
    S.lanes_log2 = 0;
    while (S.lanes_log2 < 6 && (int64_t(1) << S.lanes_log2) < wide) ++S.lanes_log2;
    S.slabs = (wide + (int64_t(1) << S.lanes_log2) - 1) >> S.lanes_log2;
    const int64_t row_lanes = kRowThreads >> S.lanes_log2, turn = row_lanes * rows, all = (k + turn - 1) / turn;
    int64_t blocks = target / S.slabs;
    blocks = blocks < 1 ? 1 : blocks > all ? all : blocks;
    S.turns = (int)((all + blocks - 1) / (blocks ? blocks : 1));
    if (S.turns < 1) S.turns = 1;
    S.blocks = (all + S.turns - 1) / S.turns;
    return S;
}

constexpr int64_t kRowsTarget = 1024, kBackTarget = 4096;

struct Plan {
    Shape rows;
    int64_t groups;
    size_t off_maxima, total;
};

Plan plan_of(int64_t k, int64_t batch, int64_t top)
{
    Plan P;
    P.rows = shape_of(k, batch, kGroup, kRowsTarget);
    P.groups = top > 0 && k > kDirect ? (k + kGroup - 1) / kGroup : 0;
    P.off_maxima = ((size_t)P.rows.blocks * 3 * batch * sizeof(float) + 255) / 256 * 256;
    P.total = P.off_maxima + (size_t)P.groups * batch * sizeof(float);
    return P;
}

template <typename T, int VEC>
void rows_with(const RowsArgs& R, bool top, const Plan& P, hipStream_t st)
{
    const dim3 grid((unsigned)(P.rows.blocks * P.rows.slabs));
    if (top) hipLaunchKernelGGL((k_logprob_rows<T, VEC, true>), grid, dim3(kRowThreads), 0, st, R);
    else hipLaunchKernelGGL((k_logprob_rows<T, VEC, false>), grid, dim3(kRowThreads), 0, st, R);
}

}  // namespace

size_t logprob_workspace(int64_t k, int64_t batch, int64_t top) { return batch ? plan_of(k, batch, top).total : 0; }

hipError_t launch_logprob(const LogprobArgs& A, hipStream_t st)
{
    const Plan P = plan_of(A.k, A.batch, A.top);
    RowsArgs R{};
    R.y = A.y; R.ldy = A.ldy; R.k = A.k; R.batch = A.batch; R.c = A.tau * 1.44269504088896340736f;
    R.lanes_log2 = P.rows.lanes_log2; R.turns = P.rows.turns; R.slabs = P.rows.slabs;
    R.parts = reinterpret_cast<float*>(A.ws); R.maxima = reinterpret_cast<float*>(A.ws + P.off_maxima);
    if (A.k > 0) {
        profile_before("logprob_rows", st);
        if (A.bf16) { if (P.rows.vec == 4) rows_with<__bf16, 4>(R, P.groups > 0, P, st); else rows_with<__bf16, 1>(R, P.groups > 0, P, st); }
        else { if (P.rows.vec == 4) rows_with<float, 4>(R, P.groups > 0, P, st); else rows_with<float, 1>(R, P.groups > 0, P, st); }
        profile_after("logprob_rows", st);
    }
    FinishArgs F{};
    F.L = A; F.parts = R.parts; F.maxima = R.maxima; F.part_count = A.k > 0 ? P.rows.blocks : 0; F.groups = P.groups; F.c = R.c;
    const dim3 grid((unsigned)((A.batch + kFinishWaves - 1) / kFinishWaves));
    profile_before("logprob_finish", st);
    if (A.bf16) hipLaunchKernelGGL((k_logprob_finish<__bf16>), grid, dim3(kFinishWaves * 64), 0, st, F);
    else hipLaunchKernelGGL((k_logprob_finish<float>), grid, dim3(kFinishWaves * 64), 0, st, F);
    profile_after("logprob_finish", st);
    return hipGetLastError();
}

hipError_t launch_logprob_backward(const LogprobBackwardArgs& A, hipStream_t st)
{
    const Shape S = shape_of(A.k, A.batch, kBackRows, kBackTarget);
    BackwardArgs F{};
    F.B = A; F.lanes_log2 = S.lanes_log2; F.turns = S.turns; F.slabs = S.slabs;
    const dim3 grid((unsigned)(S.blocks * S.slabs));
    profile_before("logprob_backward", st);
    if (A.bf16) {
        if (S.vec == 4) hipLaunchKernelGGL((k_logprob_backward<__bf16, 4>), grid, dim3(kRowThreads), 0, st, F);
        else hipLaunchKernelGGL((k_logprob_backward<__bf16, 1>), grid, dim3(kRowThreads), 0, st, F);
    } else {
        if (S.vec == 4) hipLaunchKernelGGL((k_logprob_backward<float, 4>), grid, dim3(kRowThreads), 0, st, F);
        else hipLaunchKernelGGL((k_logprob_backward<float, 1>), grid, dim3(kRowThreads), 0, st, F);
    }
    profile_after("logprob_backward", st);
    return hipGetLastError();
}

}  // namespace laplex
