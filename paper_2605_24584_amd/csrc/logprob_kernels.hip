// Log probabilities, entropy and the likeliest alternatives over logits y[k][batch] (a row per vocabulary entry), and the
// gradient into the logits.
//
// Per column, with m = max y, x = tau (y - m) / log 2:   s = sum 2^x,  w = sum x 2^x;
//   lse = tau m + log s,   entropy = log s - log 2 w / s,   logp = tau (y - m) - log s.
// One pass over the logits (k_logprob_rows): a thread holds (m, s, w) of up to four neighbouring columns and takes groups of kGroup consecutive
// rows; the running maximum and the rescaling cost it one more exponential per group.  A second launch (k_logprob_finish), a
// wavefront per column, brings the parts together.  All sums are fp32, a few hundred rows to a part.
//
// Alternatives: the pass also writes the maximum of every group (1 / kGroup of what it reads).  Values are ordered by size and, of
// equal ones, by row.  The second launch takes the maxima of groups of groups and finds a bound that at least `top` of them reach: every value among
// the `top` largest reaches it too.  Groups of groups that reach it are opened, then groups, then rows, each level's loads together, and what is left
// (little more than `top` values) is put in order by counting what comes before each.  Where many values are equal more may reach the bound than there
// is room for; then the first `top` of each level are chosen, one level after the other: a value among the `top` largest lies in one of the `top`
// groups with the largest maxima (ties: the first ones), since otherwise each of those holds a value before it.
//
// The pass and the gradient are bound by memory: 32000 x 4099 fp32 95 to 105 us for 0.52 GB read (5.2 TB/s), the gradient 200 to 220 us for 1.05 GB.  The second
// launch is bound by latency, three or four dependent rounds of loads: 32000 x 1 with the 8 likeliest 8.4 us (the pass 4.7), 32000 x 256 with 20 18.5 us (12), none
// asked for 7.4 us.  (A form that extracted the alternatives level by level took 40 and 59 us.)
#include "token_internal.h"

namespace laplex {

namespace {

constexpr int kGroupBits = 4, kGroup = 1 << kGroupBits;      // rows whose maximum is kept
constexpr int kSuperBits = 3, kSuper = 1 << kSuperBits;      // groups that are looked at together first
constexpr int kPick = 16;             // values per lane that a choice is made among
constexpr int kDirect = 64 * kPick;   // rows that need no groups
constexpr int kRowThreads = 256, kRowThreadsFew = 64;   // of a workgroup; where those would leave compute units without one

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

struct Stats { float m, s, w; };      // maximum, sum 2^x, sum x 2^x

// c of x = c (y - m): tau / log 2, or the largest number: with an infinite one the maximum itself would give 0 * inf.  (From tau = 2.3e38 on, where logits that are not equal differ by
// less than 1e-36 or have probability 0.)
__host__ __device__ __forceinline__ float rate_of(float tau)
{
    const float c = tau * 1.44269504088896340736f;
    return c < 3.402823466e38f ? c : 3.402823466e38f;
}

// brings the sums of `a` to the maximum m >= a.m (a maximum of -inf: there is nothing in them)
__device__ __forceinline__ void rebase(Stats& a, float m, float c)
{
    const float x = a.m == -INFINITY ? 0.0f : (a.m - m) * c;
    const float e = __builtin_amdgcn_exp2f(x);
    a.w = e > 0.0f ? (a.w + x * a.s) * e : (a.s != a.s ? a.s : 0.0f);
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

template <typename T, int VEC, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS)
k_logprob_rows(RowsArgs A)
{
    __shared__ Stats side[THREADS / 64][64][VEC];
    const int lanes = 1 << A.lanes_log2, x = threadIdx.x, column_lane = x & (lanes - 1), row_lane = x >> A.lanes_log2;
    const int row_lanes = THREADS >> A.lanes_log2;
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
                    const float x = (v[i][c] - base) * A.c, e = __builtin_amdgcn_exp2f(x);
                    s += e;
                    w += e > 0.0f ? x * e : 0.0f;
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
            for (int wave = 1; wave < THREADS / 64; ++wave) all = join(all, side[wave][x][c], A.c);
            if (c < have) { out[c] = all.m; out[A.batch + c] = all.s; out[2 * A.batch + c] = all.w; }
        }
    }
}

// ----------------------------------------------------------------------------
// A wavefront chooses the `want` largest of up to 64 N values: keys in the order of the values, and of equal ones the first are
// taken; key 0: no value.
// ----------------------------------------------------------------------------

// A logit as a whole number in the order of the values: -0 equals +0, NaN comes before all numbers; never 0.
__device__ __forceinline__ uint32_t order_of(float v)
{
    if (v != v) return 0xFFFFFFFFu;
    const uint32_t bits = __float_as_uint(v + 0.0f);
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}
// and back (NaN is some NaN)
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// what lanes of the wavefront have written to LDS is there for the others
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The largest bound, a multiple of 2^LOW, that at least `want` of the keys reach (0: there are fewer keys but 0), two bits at a time.
template <int N, int LOW>
__device__ __forceinline__ uint32_t bound_of(const uint32_t (&key)[N], int want)
{
    uint32_t bound = 0;
#pragma unroll 1
    for (int bit = 30; bit >= LOW; bit -= 2) {
        const uint32_t low = bound | (1u << bit), mid = bound | (2u << bit), high = bound | (3u << bit);
        int at_low = 0, at_mid = 0, at_high = 0;
#pragma unroll
        for (int r = 0; r < N; ++r) {
            at_low += __popcll(__ballot(key[r] >= low));
            at_mid += __popcll(__ballot(key[r] >= mid));
            at_high += __popcll(__ballot(key[r] >= high));
        }
        bound = at_high >= want ? high : at_mid >= want ? mid : at_low >= want ? low : bound;
    }
    return bound;
}

// chosen[0 .. count) <- numbers of the chosen values, ascending; keys[] <- their keys (may be null).  Returns count (uniform).
template <int N>
__device__ __forceinline__ int choose_among(const uint32_t* stage, int want, int* chosen, uint32_t* keys)
{
    const int lane = threadIdx.x & 63;
    const uint64_t below = (1ull << lane) - 1ull;
    uint32_t key[N];
#pragma unroll
    for (int r = 0; r < N; ++r) key[r] = stage[r * 64 + lane];
    const uint32_t bound = bound_of<N, 0>(key, want);
    int above = 0;
#pragma unroll
    for (int r = 0; r < N; ++r) above += __popcll(__ballot(key[r] > bound));
    int equal = bound == 0 ? 0 : want - above, count = 0;      // how many of those at the bound are taken
#pragma unroll
    for (int r = 0; r < N; ++r) {
        const uint64_t same = __ballot(key[r] == bound);
        const bool mine = key[r] > bound || (key[r] == bound && __popcll(same & below) < equal);
        equal -= __popcll(same);
        equal = equal < 0 ? 0 : equal;
        const uint64_t all = __ballot(mine);
        if (mine) {
            const int at = count + __popcll(all & below);
            chosen[at] = r * 64 + lane;
            keys[at] = key[r];
        }
        count += __popcll(all);
    }
    wave_sync();
    return count;
}

// `used` times 64 keys in `stage` (room for kDirect; what lies behind those is overwritten)
__device__ __forceinline__ int choose(uint32_t* stage, int used, int want, int* chosen, uint32_t* keys)
{
    const int lane = threadIdx.x & 63;
    const int padded = used <= 1 ? 1 : used <= 2 ? 2 : used <= 4 ? 4 : used <= 8 ? 8 : kPick;
    for (int n = used * 64 + lane; n < padded * 64; n += 64) stage[n] = 0;
    wave_sync();
    switch (padded) {
        case 1: return choose_among<1>(stage, want, chosen, keys);
        case 2: return choose_among<2>(stage, want, chosen, keys);
        case 4: return choose_among<4>(stage, want, chosen, keys);
        case 8: return choose_among<8>(stage, want, chosen, keys);
        default: return choose_among<kPick>(stage, want, chosen, keys);
    }
}

// A bound that at least `want` of `used` times 64 keys in `stage` reach, and few more: the upper halves of the keys alone are looked at.  At least 1.
template <int N>
__device__ __forceinline__ uint32_t coarse_among(const uint32_t* stage, int want)
{
    uint32_t key[N];
#pragma unroll
    for (int r = 0; r < N; ++r) key[r] = stage[r * 64 + (threadIdx.x & 63)];
    const uint32_t bound = bound_of<N, 16>(key, want);
    return bound ? bound : 1u;
}
__device__ __forceinline__ uint32_t coarse(uint32_t* stage, int used, int want)
{
    const int padded = used <= 4 ? 4 : kPick;
    for (int n = used * 64 + (threadIdx.x & 63); n < padded * 64; n += 64) stage[n] = 0;
    wave_sync();
    return padded == 4 ? coarse_among<4>(stage, want) : coarse_among<kPick>(stage, want);
}

struct FinishArgs {
    LogprobArgs L;
    const float *parts, *maxima;
    int64_t part_count, groups;
    float c;
};

constexpr int kChiplets = 8;
constexpr int kFinishThreads = 256;
constexpr int kAhead = 4;               // parts that a lane has asked for at a time
constexpr int kMaxTop = 64, kOpen = 128, kFound = 192;      // groups that are opened; values among which the places are given: kMaxTop and 128 new ones

// COLS columns of a workgroup are read together, and finished by a wavefront each.
template <typename T, bool TOP, int COLS>
__global__ void __launch_bounds__(kFinishThreads)
k_logprob_finish(FinishArgs F)
{
    __shared__ Stats side[kFinishThreads][COLS];
    const LogprobArgs& A = F.L;
    const int x = threadIdx.x, lane = x & 63, wave = x >> 6;
    // neighbouring columns share lines: they go to one chiplet (workgroups are dealt to the chiplets in turn)
    const int64_t t0 = ((int64_t)(blockIdx.x % kChiplets) * (gridDim.x / kChiplets) + blockIdx.x / kChiplets) * COLS, t = t0 + wave;
    if (t0 >= A.batch) return;
    const int have = A.batch - t0 < COLS ? (int)(A.batch - t0) : COLS;

    // groups of groups: what the first level of each column's choice is made among (asked for before the parts are waited for)
    constexpr int kSpan = TOP ? kDirect : 4;
    __shared__ __attribute__((aligned(16))) uint32_t stage[COLS][kSpan];      // keys on their way into the registers
    const int64_t all_supers = (F.groups + kSuper - 1) / kSuper;
    const int supers = TOP && A.k > kDirect ? (int)(all_supers < kDirect ? all_supers : kDirect) : 0;
    float v[2][kSuper][COLS];
    const auto ask = [&](int n0) {
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int i = 0; i < kSuper; ++i) {
                const int n = n0 + a * kFinishThreads;
                if (n < supers && n * kSuper + i < F.groups)
                    load_columns<float, COLS>(v[a][i], F.maxima + (int64_t)(n * kSuper + i) * A.batch + t0, have);
            }
    };
    const auto put = [&](int n0) {
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const int n = n0 + a * kFinishThreads;
            if (n < supers)
#pragma unroll
                for (int c = 0; c < COLS; ++c) {
                    uint32_t most = 0;
#pragma unroll
                    for (int i = 0; i < kSuper; ++i) { const uint32_t o = n * kSuper + i < F.groups ? order_of(v[a][i][c]) : 0; most = o > most ? o : most; }
                    stage[c][n] = most;
                }
        }
    };
    if (TOP) ask(x);
    {
        Stats st[COLS];
#pragma unroll
        for (int c = 0; c < COLS; ++c) st[c] = Stats{-INFINITY, 0.0f, 0.0f};
        for (int64_t p0 = x; p0 < F.part_count; p0 += kFinishThreads * kAhead) {
            float m[kAhead][COLS], s[kAhead][COLS], w[kAhead][COLS];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int64_t p = p0 + i * kFinishThreads;
                if (p < F.part_count) {
                    const float* const at = F.parts + p * 3 * A.batch + t0;
                    load_columns<float, COLS>(m[i], at, have);
                    load_columns<float, COLS>(s[i], at + A.batch, have);
                    load_columns<float, COLS>(w[i], at + 2 * A.batch, have);
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (p0 + i * kFinishThreads < F.part_count)
#pragma unroll
                    for (int c = 0; c < COLS; ++c) st[c] = join(st[c], Stats{m[i][c], s[i][c], w[i][c]}, F.c);
        }
#pragma unroll
        for (int c = 0; c < COLS; ++c) side[x][c] = st[c];
    }
    if (TOP) {
        put(x);
        for (int n = x + 2 * kFinishThreads; n < supers; n += 2 * kFinishThreads) { ask(n); put(n); }
    }
    __syncthreads();
    if (wave >= COLS || t >= A.batch) return;        // (nothing below is for the whole workgroup)
    const T* const y = static_cast<const T*>(A.y) + t;

    // the column's maximum, then every lane's sums brought to it, then their sum
    constexpr int kShares = kFinishThreads / 64;
    Stats some[kShares], st{-INFINITY, 0.0f, 0.0f};
#pragma unroll
    for (int n = 0; n < kShares; ++n) { some[n] = side[n * 64 + lane][wave]; st.m = fmaxf(st.m, some[n].m); }
    for (int step = 32; step >= 1; step >>= 1) st.m = fmaxf(st.m, __shfl_xor(st.m, step));
#pragma unroll
    for (int n = 0; n < kShares; ++n) {
        rebase(some[n], st.m, F.c);
        st.s += some[n].s;
        st.w += some[n].w;
    }
    for (int step = 32; step >= 1; step >>= 1) { st.s += __shfl_xor(st.s, step); st.w += __shfl_xor(st.w, step); }
    const bool empty = st.m == -INFINITY && st.s == 0.0f;
    const float log_sum = logf(st.s);
    auto logp_of = [&](float v) { return empty ? -INFINITY : (v - st.m) * A.tau - log_sum; };
    if (lane == 0) {
        if (A.lse) A.lse[t] = empty ? -INFINITY : st.m * A.tau + log_sum;
        if (A.entropy) A.entropy[t] = empty ? 0.0f : log_sum - 0.69314718055994530942f * (st.w / st.s);
        if (A.logp) {
            const int64_t target = A.targets[t];
            A.logp[t] = target >= 0 && target < A.k ? logp_of(to_float(y[target * A.ldy])) : 0.0f;
        }
    }
    if constexpr (TOP) {
        __shared__ int lists[COLS][2][kMaxTop], open[COLS][2][kOpen];
        __shared__ uint32_t keys[COLS][kMaxTop];
        __shared__ __attribute__((aligned(16))) uint32_t found_key[COLS][kFound], found_row[COLS][kFound];
        uint32_t *const fk = found_key[wave], *const fr = found_row[wave], *const sk = stage[wave];
        int *const ol = open[wave][0], *const op = open[wave][1];
        int best = 0;                                  // fk, fr [0, best): the largest so far, in their order
        const int want = A.top;
        const uint64_t below = (1ull << lane) - 1ull;
        // stretches of kDirect groups of groups
        const int64_t span = (int64_t)kDirect * kSuper * kGroup;
        for (int64_t first = 0; first < A.k; first += span) {
            const int64_t left = A.k - first < span ? A.k - first : span, groups = (left + kGroup - 1) / kGroup;
            const float* const maxima = F.maxima + first / kGroup * A.batch + t;
            const T* const rows = y + first * A.ldy;
            const bool direct = A.k <= kDirect;
            const auto group_value = [&](int g) { return maxima[(int64_t)g * A.batch]; };
            const auto row_value = [&](int r) { return to_float(rows[(int64_t)r * A.ldy]); };
            // (all loads below are of places that exist, whether their values are kept or not: none of them waits for the one before)
            const auto super_key = [&](int n) {
                float v[kSuper];
#pragma unroll
                for (int i = 0; i < kSuper; ++i) v[i] = group_value(n * kSuper + i < groups ? n * kSuper + i : (int)groups - 1);
                uint32_t most = 0;
#pragma unroll
                for (int i = 0; i < kSuper; ++i) { const uint32_t o = order_of(v[i]); most = o > most ? o : most; }
                return most;
            };
            // sk[n] <- the key of value(number(n)), n < total, or 0 where the number reaches the limit: eight of a lane's loads at a time
            const auto gather = [&](int total, int64_t limit, auto number, auto value) {
                for (int n0 = lane; n0 < total; n0 += 64 * 8) {
                    int id[8];
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) id[i] = number(n0 + i * 64 < total ? n0 + i * 64 : total - 1);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = value(id[i] < limit ? id[i] : (int)limit - 1);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (n0 + i * 64 < total) sk[n0 + i * 64] = id[i] < limit ? order_of(v[i]) : 0;
                }
                wave_sync();
            };
            // keys of the groups of groups (the first stretch's are there), or of the rows where they are few
            const int whole = direct ? (int)left : (int)((groups + kSuper - 1) / kSuper);
            if (direct) {
                gather(whole, left, [](int n) { return n; }, row_value);
            } else if (first > 0) {
                for (int n = lane; n < whole; n += 64) sk[n] = super_key(n);
            }
            const int used = (whole + 63) / 64;
            for (int n = whole + lane; n < used * 64; n += 64) sk[n] = 0;
            // What reaches a bound that `want` of them reach: those are opened, and again what reaches it.  Where many values are equal it may be more
            // than there is room for.
            const uint32_t bound = coarse(sk, used, want);
            int found = best;
            bool fits = true;
            if (direct) {
                for (int n = lane; n < used * 64; n += 64) {
                    const uint32_t k = sk[n];
                    const uint64_t all = __ballot(k >= bound);
                    const int at = found + __popcll(all & below);
                    if (k >= bound && at < kFound) { fk[at] = k; fr[at] = (uint32_t)n; }
                    found += __popcll(all);
                }
            } else {
                int listed = 0, opened = 0;
                for (int n = lane; n < used * 64; n += 64) {
                    const bool in = sk[n] >= bound;
                    const uint64_t all = __ballot(in);
                    const int at = listed + __popcll(all & below);
                    if (in && at < kOpen) ol[at] = n;
                    listed += __popcll(all);
                }
                wave_sync();
                fits = listed <= kOpen;
                // (all loads of a level at a time, then what of it is kept)
                for (int n0 = 0; fits && n0 < listed * kSuper; n0 += kDirect) {
                    const int some = listed * kSuper - n0 < kDirect ? listed * kSuper - n0 : kDirect;
                    gather(some, groups, [&](int n) { return ol[(n0 + n) >> kSuperBits] * kSuper + (n & (kSuper - 1)); }, group_value);
                    for (int n = lane; n < (some + 63) / 64 * 64; n += 64) {
                        const bool in = n < some && sk[n] >= bound;
                        const uint64_t all = __ballot(in);
                        const int at = opened + __popcll(all & below);
                        if (in && at < kOpen) op[at] = ol[(n0 + n) >> kSuperBits] * kSuper + (n & (kSuper - 1));
                        opened += __popcll(all);
                    }
                    wave_sync();
                }
                fits = fits && opened <= kOpen;
                for (int n0 = 0; fits && n0 < opened * kGroup; n0 += kDirect) {
                    const int some = opened * kGroup - n0 < kDirect ? opened * kGroup - n0 : kDirect;
                    gather(some, left, [&](int n) { return op[(n0 + n) >> kGroupBits] * kGroup + (n & (kGroup - 1)); }, row_value);
                    for (int n = lane; n < (some + 63) / 64 * 64; n += 64) {
                        const uint32_t k = n < some ? sk[n] : 0;
                        const uint64_t all = __ballot(k >= bound);
                        const int at = found + __popcll(all & below);
                        if (k >= bound && at < kFound) { fk[at] = k; fr[at] = (uint32_t)(first + op[(n0 + n) >> kGroupBits] * kGroup + (n & (kGroup - 1))); }
                        found += __popcll(all);
                    }
                    wave_sync();
                }
            }
            if (!fits || found > kFound) {
                // Level by level, the `want` first ones of each: no more than that are ever held.
                int *const ids = lists[wave][0], *const chosen = lists[wave][1];
                int count = 0;
#pragma unroll 1
                for (int level = direct ? 2 : 0; level < 3; ++level) {
                    // what is opened (bits of its size), how many there are, and the limit of their numbers
                    const bool all = level == 0 || direct;
                    const int bits = level == 1 ? kSuperBits : kGroupBits;
                    const int64_t limit = level == 1 ? groups : left;
                    const int candidates = all ? whole : count << bits;
                    const auto number = [&](int n) { return all ? n : (ids[n >> bits] << bits) + (n & ((1 << bits) - 1)); };
#pragma unroll 4
                    for (int n = lane; n < candidates; n += 64) {
                        const int id = number(n);
                        sk[n] = level == 0 ? super_key(id) : id >= limit ? 0 : order_of(level == 1 ? group_value(id) : row_value(id));
                    }
                    const int some = (candidates + 63) / 64;
                    for (int n = candidates + lane; n < some * 64; n += 64) sk[n] = 0;
                    count = choose(sk, some, want, chosen, keys[wave]);
                    const int id = lane < count ? number(chosen[lane]) : 0;
                    wave_sync();
                    if (lane < count) ids[lane] = id;
                    wave_sync();
                }
                if (lane < count) { fr[best + lane] = (uint32_t)(first + ids[lane]); fk[best + lane] = keys[wave][lane]; }
                found = best + count;
            }
            wave_sync();
            // the places of all that was found, those of earlier stretches among it
            for (int n = found + lane; n < (found + 63) / 64 * 64; n += 64) { fk[n] = 0; fr[n] = 0xFFFFFFFFu; }
            wave_sync();
            uint32_t k[kFound / 64], row[kFound / 64];
            int place[kFound / 64];
#pragma unroll
            for (int i = 0; i < kFound / 64; ++i) {
                place[i] = kFound;
                if (i * 64 >= found) continue;
                k[i] = fk[i * 64 + lane];
                row[i] = fr[i * 64 + lane];
                int before = 0;
#pragma unroll 2
                for (int j = 0; j < found; j += 4) {
                    const uint4 ok = *reinterpret_cast<const uint4*>(fk + j), orow = *reinterpret_cast<const uint4*>(fr + j);
                    before += (ok.x > k[i] || (ok.x == k[i] && orow.x < row[i])) + (ok.y > k[i] || (ok.y == k[i] && orow.y < row[i])) +
                              (ok.z > k[i] || (ok.z == k[i] && orow.z < row[i])) + (ok.w > k[i] || (ok.w == k[i] && orow.w < row[i]));
                }
                if (i * 64 + lane < found) place[i] = before;
            }
            wave_sync();
#pragma unroll
            for (int i = 0; i < kFound / 64; ++i)
                if (place[i] < want) { fk[place[i]] = k[i]; fr[place[i]] = row[i]; }
            best = found < want ? found : want;
            wave_sync();
        }
        if (lane < best) {
            A.top_ids[lane * A.batch + t] = fr[lane];
            A.top_logp[lane * A.batch + t] = logp_of(value_of(fk[lane]));
        }
    }
}

// ----------------------------------------------------------------------------
// gy = tau p ( glse - glogp - gentropy (log p + entropy) ) + tau glogp at the target.  One read and one write per logit.
//
// log p = tau y - lse is off by the rounding of lse, which is nothing beside the other roundings up to |lse| = kPlainLse, 6e-5 of p at 1000, and all there is to
// p in a column of nothing but the type's lowest value.  Columns beyond that are left to workgroups of their own, in front of the others in the same launch: they
// take the column's maximum and sum anew and use log p = tau (y - m) - log s.  Where there are none such a workgroup ends after a look at lse, and the gradient
// takes what it took without them; where all columns are far (32000 x 1 / 256 / 4099 fp32) 56 / 118 / 900 us instead of 8 / 17 / 205.
// ----------------------------------------------------------------------------
struct BackwardArgs {
    LogprobBackwardArgs B;
    int lanes_log2, turns;
    int64_t slabs;
    int far_lanes_log2;
    int64_t far_blocks;
};

// Rows of a thread at a time: 16 bytes of each are on their way at once.  32000 x 256 fp32, 4 / 8 / 16 rows: 22.9 / 19.1 / 17.0 us, 32000 x 4099: 260 / 217 / 197.
// The gradient is streamed past the caches: left there its lines are written back while the next call reads (32000 x 2048, the next forward call
// 79 -> 55 us, this one 92 -> 88; 32000 x 4099, rows that are aligned to nothing, 143 -> 101 and 197 -> 210).
constexpr int kBackRows = 16;

constexpr float kPlainLse = 64.0f;
__device__ __forceinline__ bool is_far(float lse) { return fabsf(lse) > kPlainLse; }      // (a NaN is not: p is NaN either way)

// What the rows of up to VEC neighbouring columns have in common: log p = tau (y - from) - less.
template <int VEC>
struct Columns {
    float from[VEC], less[VEC], one[VEC], logs[VEC], hit[VEC];
    int64_t target[VEC];
};

template <typename T, int VEC, bool FAR>
__device__ __forceinline__ void gradient_rows(const LogprobBackwardArgs& A, const Columns<VEC>& C, int64_t row0, int64_t t, int have)
{
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
            const float logp = fmaf(FAR ? v[i][c] - C.from[c] : v[i][c], A.tau, -C.less[c]), q = expf(logp);
            float r = q == 0.0f ? 0.0f : q * fmaf(C.logs[c], logp, C.one[c]);
            if (row0 + i == C.target[c]) r += C.hit[c];
            if constexpr (VEC == 1) out = (T)(A.tau * r);
            else out[c] = (T)(A.tau * r);
        }
        if (have >= VEC) __builtin_nontemporal_store(out, reinterpret_cast<typename Lane<T, VEC>::type*>(g + i * A.ldgy));
        else if constexpr (VEC > 1) {
#pragma unroll
            for (int c = 0; c < VEC; ++c)
                if (c < have) g[i * A.ldgy + c] = out[c];
        }
    }
}

// `less` is lse, `from` 0; true if some column is far.
template <int VEC>
__device__ __forceinline__ bool load_common(const LogprobBackwardArgs& A, Columns<VEC>& C, int64_t t, int have)
{
    bool far = false;
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
        const int64_t at = t + (c < have ? c : 0);
        C.from[c] = 0.0f;
        C.less[c] = A.lse[at];
        far = far || is_far(C.less[c]);
        C.target[c] = -1; C.hit[c] = 0.0f;
        C.one[c] = A.glse ? A.glse[at] : 0.0f;
        C.logs[c] = 0.0f;
        if (A.glogp) {
            const int64_t given = A.targets[at];
            if (given >= 0 && given < A.k) { C.hit[c] = A.glogp[at]; C.one[c] -= C.hit[c]; C.target[c] = given; }
        }
        if (A.gentropy) { C.logs[c] = -A.gentropy[at]; C.one[c] += C.logs[c] * A.entropy[at]; }
    }
    return far;
}

template <typename T, int VEC>
__device__ __forceinline__ void far_columns(const BackwardArgs& F, int64_t block)
{
    __shared__ Stats side[kRowThreads / 64][64][VEC];
    const LogprobBackwardArgs& A = F.B;
    const int lanes = 1 << F.far_lanes_log2, x = threadIdx.x, column_lane = x & (lanes - 1), row_lane = x >> F.far_lanes_log2;
    const int row_lanes = kRowThreads >> F.far_lanes_log2;
    block = block % kChiplets * (F.far_blocks / kChiplets) + block / kChiplets;      // (neighbouring columns share lines)
    const int64_t t = (block * lanes + column_lane) * VEC;
    const int have = A.batch - t >= VEC ? VEC : A.batch > t ? (int)(A.batch - t) : 0;
    Columns<VEC> C;
    const bool mine = have > 0 && load_common(A, C, t, have);
    if (!__syncthreads_or(mine)) return;
    const float c2 = rate_of(A.tau);
    Stats st[VEC];
#pragma unroll
    for (int c = 0; c < VEC; ++c) st[c] = Stats{-INFINITY, 0.0f, 0.0f};
    if (mine)
        for (int64_t row0 = (int64_t)row_lane * kBackRows; row0 < A.k; row0 += (int64_t)row_lanes * kBackRows) {
            const T* const p = static_cast<const T*>(A.y) + row0 * A.ldy + t;
            float v[kBackRows][VEC];
#pragma unroll
            for (int i = 0; i < kBackRows; ++i) {
                if (row0 + i < A.k) load_columns<T, VEC>(v[i], p + i * A.ldy, have);
                else
#pragma unroll
                    for (int c = 0; c < VEC; ++c) v[i][c] = -INFINITY;
            }
#pragma unroll
            for (int c = 0; c < VEC; ++c) {
                float m = v[0][c];
#pragma unroll
                for (int i = 1; i < kBackRows; ++i) m = fmaxf(m, v[i][c]);
                rebase(st[c], fmaxf(st[c].m, m), c2);
                const float base = st[c].m == -INFINITY ? 0.0f : st[c].m;
#pragma unroll
                for (int i = 0; i < kBackRows; ++i) st[c].s += __builtin_amdgcn_exp2f((v[i][c] - base) * c2);
            }
        }
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
        for (int step = lanes; step < 64; step <<= 1)
            st[c] = join(st[c], Stats{__shfl_xor(st[c].m, step), __shfl_xor(st[c].s, step), 0.0f}, c2);
        side[x >> 6][x & 63][c] = st[c];
    }
    __syncthreads();
    if (!mine) return;
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
        if (!is_far(C.less[c])) continue;
        Stats all = side[0][column_lane][c];
        for (int wave = 1; wave < kRowThreads / 64; ++wave) all = join(all, side[wave][column_lane][c], c2);
        const bool empty = all.m == -INFINITY && all.s == 0.0f;            // nothing but -inf: p is 0 everywhere
        C.from[c] = empty ? 0.0f : all.m;
        C.less[c] = empty ? 0.0f : logf(all.s);
        if (empty) C.target[c] = -1;
    }
    for (int64_t row0 = (int64_t)row_lane * kBackRows; row0 < A.k; row0 += (int64_t)row_lanes * kBackRows) gradient_rows<T, VEC, true>(A, C, row0, t, have);
}

template <typename T, int VEC>
__global__ void __launch_bounds__(kRowThreads)
k_logprob_backward(BackwardArgs F)
{
    if (blockIdx.x < F.far_blocks) {
        far_columns<T, VEC>(F, blockIdx.x);
        return;
    }
    const LogprobBackwardArgs& A = F.B;
    const int lanes = 1 << F.lanes_log2, x = threadIdx.x, column_lane = x & (lanes - 1), row_lane = x >> F.lanes_log2;
    const int row_lanes = kRowThreads >> F.lanes_log2;
    const int64_t id = blockIdx.x - F.far_blocks, slab = id % F.slabs, block = id / F.slabs;
    const int64_t t = (slab * lanes + column_lane) * VEC;
    const int have = A.batch - t >= VEC ? VEC : A.batch > t ? (int)(A.batch - t) : 0;
    if (have == 0) return;
    Columns<VEC> C;
    if (load_common(A, C, t, have)) return;
    for (int n = 0; n < F.turns; ++n) {
        const int64_t row0 = ((block * F.turns + n) * row_lanes + row_lane) * kBackRows;
        if (row0 >= A.k) break;
        gradient_rows<T, VEC, false>(A, C, row0, t, have);
    }
}

constexpr int64_t kFewWorkgroups = 256;      // compute units

// Lanes across the columns, and how often a thread takes rows: about `target` workgroups, if there are rows for them.  few: smaller ones, where others would leave compute
// units without one.
struct Shape {
    int vec, lanes_log2, turns, threads;
    int64_t slabs, blocks;
};

Shape shape_of(int64_t k, int64_t batch, int rows, int64_t target, bool few)
{
    Shape S;
    S.threads = kRowThreads;
    S.vec = batch >= 4 ? 4 : 1;
    const int64_t wide = (batch + S.vec - 1) / S.vec;
    S.lanes_log2 = 0;
    while (S.lanes_log2 < 6 && (int64_t(1) << S.lanes_log2) < wide) ++S.lanes_log2;
    S.slabs = (wide + (int64_t(1) << S.lanes_log2) - 1) >> S.lanes_log2;
    if (few && S.slabs * ((k * (int64_t(1) << S.lanes_log2)) / (kRowThreads * rows)) < kFewWorkgroups) S.threads = kRowThreadsFew;
    const int64_t row_lanes = S.threads >> S.lanes_log2, turn = row_lanes * rows, all = (k + turn - 1) / turn;
    int64_t blocks = target / S.slabs;
    blocks = blocks < 1 ? 1 : blocks > all ? all : blocks;
    S.turns = (int)((all + blocks - 1) / (blocks ? blocks : 1));
    if (S.turns < 1) S.turns = 1;
    S.blocks = (all + S.turns - 1) / S.turns;
    return S;
}

// Workgroups: for the pass over the logits two a compute unit (32000 x 2048, 256 / 512 / 1024 / 8192 of them: 69 / 68 / 79 / 66 us and a last launch of 7.0 / 7.4 / 8.0 /
// 11.3; with one column or few the parts of more would cost more than they gain); for the gradient one turn each, up to what a grid holds with room to spare.
constexpr int64_t kRowsTarget = 512, kBackTarget = int64_t(1) << 20;

struct Plan {
    Shape rows;
    int64_t groups;
    size_t off_maxima, total;
};

Plan plan_of(int64_t k, int64_t batch, int64_t top)
{
    Plan P;
    P.rows = shape_of(k, batch, kGroup, kRowsTarget, true);
    P.groups = top > 0 && k > kDirect ? (k + kGroup - 1) / kGroup : 0;
    P.off_maxima = ((size_t)P.rows.blocks * 3 * batch * sizeof(float) + 255) / 256 * 256;
    P.total = P.off_maxima + (size_t)P.groups * batch * sizeof(float);
    return P;
}

template <typename T, int VEC>
void rows_with(const RowsArgs& R, bool top, const Plan& P, hipStream_t st)
{
    const dim3 grid((unsigned)(P.rows.blocks * P.rows.slabs)), block(P.rows.threads);
    if (P.rows.threads == kRowThreadsFew) {
        if (top) hipLaunchKernelGGL((k_logprob_rows<T, VEC, true, kRowThreadsFew>), grid, block, 0, st, R);
        else hipLaunchKernelGGL((k_logprob_rows<T, VEC, false, kRowThreadsFew>), grid, block, 0, st, R);
    } else {
        if (top) hipLaunchKernelGGL((k_logprob_rows<T, VEC, true, kRowThreads>), grid, block, 0, st, R);
        else hipLaunchKernelGGL((k_logprob_rows<T, VEC, false, kRowThreads>), grid, block, 0, st, R);
    }
}

template <typename T, int COLS>
void finish_with(const FinishArgs& F, hipStream_t st)
{
    const int64_t blocks = (F.L.batch + COLS - 1) / COLS;
    const dim3 grid((unsigned)((blocks + kChiplets - 1) / kChiplets * kChiplets)), block(kFinishThreads);
    if (F.L.top > 0) hipLaunchKernelGGL((k_logprob_finish<T, true, COLS>), grid, block, 0, st, F);
    else hipLaunchKernelGGL((k_logprob_finish<T, false, COLS>), grid, block, 0, st, F);
}

}  // namespace

size_t logprob_workspace(int64_t k, int64_t batch, int64_t top) { return batch ? plan_of(k, batch, top).total : 0; }

hipError_t launch_logprob(const LogprobArgs& A, hipStream_t st)
{
    const Plan P = plan_of(A.k, A.batch, A.top);
    RowsArgs R{};
    R.y = A.y; R.ldy = A.ldy; R.k = A.k; R.batch = A.batch; R.c = rate_of(A.tau);
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
    profile_before("logprob_finish", st);
    if (A.bf16) { if (P.rows.vec == 4) finish_with<__bf16, 4>(F, st); else finish_with<__bf16, 1>(F, st); }
    else { if (P.rows.vec == 4) finish_with<float, 4>(F, st); else finish_with<float, 1>(F, st); }
    profile_after("logprob_finish", st);
    return hipGetLastError();
}

hipError_t launch_logprob_backward(const LogprobBackwardArgs& A, hipStream_t st)
{
    const Shape S = shape_of(A.k, A.batch, kBackRows, kBackTarget, false);
    BackwardArgs F{};
    F.B = A; F.lanes_log2 = S.lanes_log2; F.turns = S.turns; F.slabs = S.slabs;
    // 64 bytes of fp32 rows side by side, if that leaves every compute unit a workgroup
    F.far_lanes_log2 = S.vec == 4 && A.batch >= 16 * kFewWorkgroups ? 2 : 0;
    const int64_t far_columns = S.vec << F.far_lanes_log2;
    F.far_blocks = ((A.batch + far_columns - 1) / far_columns + kChiplets - 1) / kChiplets * kChiplets;
    const dim3 grid((unsigned)(F.far_blocks + S.blocks * S.slabs));
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
