// Verification of drafted tokens against the target's probabilities, over logits y[k][batch] (a row per vocabulary entry).
//
//   p = softmax(tau y), q = softmax(draft_tau z) of a column, q = 1 of the draft itself where there is no z.  Column c of a sequence judges its c-th draft x:  kept while chance * q(x) < p(x).
//   At the first draft that is refused the next token is drawn from max(p - q, 0), after the last one from p:  the first row whose running sum of
//   weights passes next_chance * (their sum).
//
// Whole numbers come out, and a comparison turns on the last bits of what is compared: everything that is summed or compared is in 64 bits, the
// exponentials among it.  2^f, |f| <= 1/2, is its Taylor series up to f^13 (the next term is below 2^-57 of the result).
//
// Four launches: k_verify_rows reads both matrices once, and leaves maximum and sum of every column and part of the rows (and, for the greedy rule, the place of
// the maximum); k_verify_judge, a wavefront per column, joins them and judges the draft; k_verify_left sums what is left of the refused columns over the same
// parts of the rows; k_verify_draw, a workgroup per sequence, finds the part and then the row.  The second reading takes the refused columns alone.
//
// What bounds it: 64-bit vector instructions, some 43 a logit, not memory.  32000 rows x 1001 columns in fp32 with the drafts' logits: rows 95 us (0.26 GB: 2.7 TB/s), left 32, draw 15,
// judge 12, the call 138; 60001 x 576 in bf16, certain drafts: rows 55, draw 16 (1 of it for the draft's part, summed again), judge 7, the call 68.  Five columns of 32000 cost the four
// launches and the draw's two searches: 26 us.  (Times at parts, workgroups and sequences side by side below are of single calls with all caches filled with other data, 10 to 25 us more.)
// Two columns a lane, and several parts a workgroup in k_verify_left, were no faster.
#include "token_internal.h"

namespace laplex {

namespace {

constexpr int kThreads = 256;
constexpr int kGroup = 8;                 // rows that a thread has asked for at a time
// Parts of the rows (us with 64 / 128 / 256: 60001 rows x 576 columns in bf16 94 / 80 / 76, 32000 x 40 52 / 42 / 41, x 2048 292 / 285 / 302), workgroups that are enough for a matrix
// (1024 to 8192 are alike) and columns of a workgroup (32 / 64: 32000 x 1000 and their drafts' 164 / 166).
constexpr int kMaxParts = 256, kWorkgroups = 4096, kSlab = 64;

// 2^(c d), d <= 0 and c d finite; 0 below 2^-1074.  (The rest is written as one operation, so that the same numbers give the same bits wherever this is used.)
__device__ __forceinline__ double power_in_range(double d, double c)
{
    const double n = __builtin_rint(d * c), f = fma(d, c, -n);
    double s = 0x1.816193166d0f9p-40;                          // log(2)^13 / 13!, then 12, ...
    s = fma(s, f, 0x1.c3bd650fc2986p-36);
    s = fma(s, f, 0x1.e8cac7351bb25p-32);
    s = fma(s, f, 0x1.e4cf5158b8ecap-28);
    s = fma(s, f, 0x1.b5253d395e7c4p-24);
    s = fma(s, f, 0x1.62c0223a5c824p-20);
    s = fma(s, f, 0x1.ffcbfc588b0c7p-17);
    s = fma(s, f, 0x1.430912f86c787p-13);
    s = fma(s, f, 0x1.5d87fe78a6731p-10);
    s = fma(s, f, 0x1.3b2ab6fba4e77p-7);
    s = fma(s, f, 0x1.c6b08d704a0c0p-5);
    s = fma(s, f, 0x1.ebfbdff82c58fp-3);
    s = fma(s, f, 0x1.62e42fefa39efp-1);
    s = fma(s, f, 1.0);
    return __builtin_ldexp(s, (int)n);
}

// 2^(c (y - m)) of a logit below the maximum m, which is finite or -inf (then there is nothing but -inf)
__device__ __forceinline__ double weight_of(float y, float m, double c)
{
    const double d = (double)y - (m == -INFINITY ? 0.0 : (double)m);
    return d * c < -1100.0 ? 0.0 : power_in_range(d, c);      // (NaN for NaN)
}

struct Sum { float m; double s; };        // maximum and sum of 2^(c (y - m)); s is NaN where a logit is NaN or +inf

__device__ __forceinline__ Sum join(Sum a, Sum b, double c)
{
    const float m = fmaxf(a.m, b.m);
    const double x = a.m == m ? a.s : a.s * weight_of(a.m, m, c), y = b.m == m ? b.s : b.s * weight_of(b.m, m, c);
    return Sum{m, x + y};
}

__device__ __forceinline__ double shuffle(double v, int step)
{
    const long long b = __double_as_longlong(v);
    const int lo = __shfl_xor((int)b, step), hi = __shfl_xor((int)(b >> 32), step);
    return __longlong_as_double(((long long)hi << 32) | (uint32_t)lo);
}

// ----------------------------------------------------------------------------
// The pass over a matrix: 2^lanes_log2 lanes across the columns, the rest of the workgroup across groups of rows; a part is a range of consecutive rows.
// ----------------------------------------------------------------------------
template <typename T, bool PLACE>
__global__ void __launch_bounds__(kThreads)
k_verify_rows(VerifyArgs A)
{
    __shared__ Sum side[kThreads / 64][64];
    __shared__ int64_t side_at[kThreads / 64][PLACE ? 64 : 1];
    const int lanes = 1 << A.lanes_log2, x = threadIdx.x, column_lane = x & (lanes - 1), row_lane = x >> A.lanes_log2, row_lanes = kThreads >> A.lanes_log2;
    const int64_t slab = blockIdx.x, part = blockIdx.y;
    const int which = blockIdx.z;
    const int64_t ld = which ? A.ldz : A.ldy, t = slab * lanes + column_lane;
    const T* const y = static_cast<const T*>(which ? A.z : A.y) + t;
    const double c = which ? A.draft_c : A.c;
    const float far = (float)(1200.0 / c);
    const int64_t first = part * A.part_rows + (int64_t)row_lane * kGroup, step = (int64_t)row_lanes * kGroup;
    const int64_t end = (part + 1) * A.part_rows < A.k ? (part + 1) * A.part_rows : A.k;
    Sum st{-INFINITY, 0.0};
    // Logits further below the maximum than reach weigh 0.  An fp32 difference may be the maximum itself again (large logits, large c): there is a reach only
    // where its own weight is 0, below 2^-1074.
    float reach = -INFINITY;
    int64_t place = INT64_MAX;
    float ahead[kGroup];                               // the next rows are on their way while these are summed
    const auto ask = [&](int64_t row) {
        const T* const p = y + row * ld;
        const int rows = end - row < kGroup ? (int)(end - row) : kGroup;
#pragma unroll
        for (int i = 0; i < kGroup; ++i) ahead[i] = to_float(p[(i < rows ? i : 0) * ld]);
    };
    if (t < A.batch && first < end) {
        ask(first);
        for (int64_t row = first; row < end; row += step) {
            const int rows = end - row < kGroup ? (int)(end - row) : kGroup;
            float v[kGroup], m = -INFINITY;
            bool bad = false;                          // NaN or +inf
#pragma unroll
            for (int i = 0; i < kGroup; ++i) v[i] = i < rows ? ahead[i] : -INFINITY;
            if (row + step < end) ask(row + step);
#pragma unroll
            for (int i = 0; i < kGroup; ++i) {
                bad = bad || !(v[i] < INFINITY);
                if (PLACE && v[i] > m && v[i] > st.m) place = row + i;
                m = fmaxf(m, v[i]);
            }
            if (m > st.m) {
                st.s *= weight_of(st.m, m, c);
                st.m = m;
                reach = m - far;
                if (!(((double)m - (double)reach) * c >= 1100.0)) reach = -INFINITY;
            }
            // What is so far below the maximum that its weight is 0 is brought nearer, to where it is still 0: no further test in 64 bits.
            if (reach > -INFINITY) {
#pragma unroll
                for (int i = 0; i < kGroup; ++i) st.s += power_in_range((double)fmaxf(v[i], reach) - (double)st.m, c);
            } else {
#pragma unroll
                for (int i = 0; i < kGroup; ++i) st.s += weight_of(v[i], st.m, c);
            }
            if (bad) st.s = NAN;
        }
    }
    const auto both = [&](Sum& a, int64_t& at, Sum b, int64_t bt) {
        if (PLACE) at = b.m > a.m || (b.m == a.m && bt < at) ? bt : at;
        a = join(a, b, c);
    };
    for (int step = lanes; step < 64; step <<= 1) {
        const Sum other{__shfl_xor(st.m, step), shuffle(st.s, step)};
        int64_t at = 0;
        if (PLACE) at = __double_as_longlong(shuffle(__longlong_as_double(place), step));
        both(st, place, other, at);
    }
    side[x >> 6][x & 63] = st;
    if (PLACE) side_at[x >> 6][PLACE ? x & 63 : 0] = place;
    __syncthreads();
    if (x < lanes && t < A.batch) {
        Sum all = side[0][x];
        int64_t at = PLACE ? side_at[0][PLACE ? x : 0] : 0;
        for (int w = 1; w < kThreads / 64; ++w) both(all, at, side[w][x], PLACE ? side_at[w][PLACE ? x : 0] : 0);
        const int64_t to = (which * A.parts + part) * A.batch + t;
        A.part_max[to] = all.m;
        A.part_sum[to] = all.s;
        if (PLACE) A.part_place[to] = at;
    }
}

__device__ __forceinline__ int64_t start_of(const VerifyArgs& A, int64_t b)
{
    if (!A.starts) return A.sequences > 0 ? A.batch / A.sequences * b : 0;
    const int64_t v = A.starts[b];                       // whatever it holds, no column outside the matrices is touched
    return v < 0 ? 0 : v > A.batch ? A.batch : v;
}

// The sequence that column t belongs to, or -1; by a wavefront.
__device__ __forceinline__ int64_t sequence_of(const VerifyArgs& A, int64_t t, int64_t& end)
{
    int64_t lo = 0, hi = A.sequences;                    // the last sequence that begins at t or before it, 64 candidates at a time
    if (!A.starts) {
        lo = t / (A.batch / A.sequences);
    } else {
        const int lane = threadIdx.x & 63;
        while (hi - lo > 1) {
            const int64_t step = (hi - lo + 63) / 64, c = lo + lane * step;
            const uint64_t votes = __ballot(c < hi && start_of(A, c) <= t);
            const int at = votes ? 63 - __builtin_clzll(votes) : 0;
            lo += at * step;
            hi = lo + step < hi ? lo + step : hi;
        }
    }
    end = start_of(A, lo + 1);
    return start_of(A, lo) <= t && t < end ? lo : -1;
}

// One wavefront per column: joins its parts, and judges its draft.
template <typename T, bool PLACE>
__global__ void __launch_bounds__(kThreads)
k_verify_judge(VerifyArgs A)
{
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (t >= A.batch) return;
    int64_t end = 0;
    if (sequence_of(A, t, end) < 0) {
        if (lane == 0) {
            VerifyColumn none{};
            none.mode = kVerifyNone;
            A.columns[t] = none;
            if (A.logp) A.logp[t] = 0.0f;
        }
        return;
    }
    // the parts of both matrices: the largest maximum first, then every part's sum once
    constexpr int N = kMaxParts / 64;
    float m[2][N];
    double s[2][N];
    int64_t at[N];
    const int matrices = A.z ? 2 : 1;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int64_t p = n * 64 + lane, from = (which * A.parts + p) * A.batch + t;
            const bool there = which < matrices && p < A.parts;
            m[which][n] = there ? A.part_max[from] : -INFINITY;
            s[which][n] = there ? A.part_sum[from] : 0.0;
            if (PLACE && which == 0) at[n] = there ? A.part_place[from] : INT64_MAX;
        }
    Sum sum[2];
    int64_t place = INT64_MAX;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float most = m[which][0];
#pragma unroll
        for (int n = 1; n < N; ++n) most = fmaxf(most, m[which][n]);
        for (int step = 1; step < 64; step <<= 1) most = fmaxf(most, __shfl_xor(most, step));
        double all = 0.0;
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (m[which][n] > -INFINITY || s[which][n] != 0.0) all += s[which][n] * weight_of(m[which][n], most, which ? A.draft_c : A.c);
        for (int step = 1; step < 64; step <<= 1) all += shuffle(all, step);
        sum[which] = Sum{most, all};
    }
    if (PLACE) {
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (m[0][n] == sum[0].m && at[n] < place) place = at[n];
        for (int step = 1; step < 64; step <<= 1) {
            const int64_t other = __double_as_longlong(shuffle(__longlong_as_double(place), step));
            place = other < place ? other : place;
        }
    }
    if (lane != 0) return;
    const bool fine = sum[0].s > 0.0, draft_fine = !A.z || sum[1].s > 0.0;      // not of a NaN, +inf or nothing but -inf
    const int64_t x = A.drafts ? A.drafts[t] : -1;
    const bool last = t + 1 == end, given = !last && x >= 0 && x < A.k;
    bool kept = false;
    float logp = 0.0f;
    if (given) {
        const float yx = to_float(static_cast<const T*>(A.y)[x * A.ldy + t]);
        const double px = fine ? weight_of(yx, sum[0].m, A.c) / sum[0].s : NAN;
        logp = !fine ? NAN : (float)(A.tau * ((double)yx - (double)sum[0].m) - log(sum[0].s));
        if (PLACE) {
            kept = fine && x == place;
        } else {
            double qx = 1.0;
            if (A.z) qx = draft_fine ? weight_of(to_float(static_cast<const T*>(A.z)[x * A.ldz + t]), sum[1].m, A.draft_c) / sum[1].s : NAN;
            kept = A.chances[t] * qx < px;               // (not where one of them is NaN)
        }
    }
    if (A.logp) A.logp[t] = logp;
    VerifyColumn out;
    out.m = sum[0].m; out.draft_m = sum[1].m; out.s = sum[0].s; out.draft_s = sum[1].s; out.place = place;
    // how the next token is drawn if it is drawn here: not at all, from p, from what is left of p
    out.kept = kept;
    out.mode = !fine ? kVerifyNone : PLACE ? kVerifyPlace : !given || !draft_fine ? kVerifyAll : A.z ? kVerifyLeft : kVerifyOthers;
    A.columns[t] = out;
}

// The columns at which `1 << log2` sequences from b0 on draw their next tokens: drawn[i] <- the first one whose draft is not kept; -1: the sequence has no
// columns, or does not exist.  By the whole workgroup.
__device__ __forceinline__ void find_drawn(const VerifyArgs& A, int64_t b0, int log2, int* drawn)
{
    const int x = threadIdx.x, i = x & ((1 << log2) - 1);
    const bool there = b0 + i < A.sequences;
    const int begin = there ? (int)start_of(A, b0 + i) : 0, end = there ? (int)start_of(A, b0 + i + 1) : 0;
    if (x < 1 << log2) drawn[x] = INT32_MAX;
    __syncthreads();
    // (the last column has no draft: it is never kept)
    for (int t = begin + (x >> log2); t < end; t += kThreads >> log2)
        if (!A.columns[t].kept) {
            atomicMin(&drawn[i], t);
            break;
        }
    __syncthreads();
    if (x < 1 << log2 && drawn[x] == INT32_MAX) drawn[x] = -1;
    __syncthreads();
}

// share, draft_share: one over the columns' sums.  Both products are rounded before they are compared: a difference with one product exact would hold the other one's rounding
// where both are alike, and such rows could be drawn.
__device__ __forceinline__ double left_of(const VerifyArgs& A, const VerifyColumn& C, double share, double draft_share, float y, float z)
{
#pragma clang fp contract(off)
    const double p = weight_of(y, C.m, A.c) * share, q = weight_of(z, C.draft_m, A.draft_c) * draft_share, d = p - q;
    return d > 0.0 ? d : 0.0;
}

// What is left of the refused columns, summed over each part of the rows: 2^seq_log2 sequences side by side (their columns share lines), the rest of the
// workgroup across the rows.  left[part][sequence].
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_verify_left(VerifyArgs A)
{
    __shared__ VerifyColumn of[16];
    __shared__ int drawn[16];
    __shared__ double side[kThreads];
    const int width = 1 << A.seq_log2, x = threadIdx.x;
    const int64_t b0 = (int64_t)blockIdx.x * width;
    find_drawn(A, b0, A.seq_log2, drawn);
    const int mine = x & (width - 1), rows = kThreads >> A.seq_log2;
    if (x < width) {
        if (drawn[x] >= 0) of[x] = A.columns[drawn[x]];
        if (drawn[x] >= 0 && of[x].mode != kVerifyLeft) drawn[x] = -1;
    }
    __syncthreads();
    const int64_t t = drawn[mine], part = blockIdx.y, end = (part + 1) * A.part_rows < A.k ? (part + 1) * A.part_rows : A.k;
    VerifyColumn C{};
    if (t >= 0) C = of[mine];
    const double share = 1.0 / C.s, draft_share = 1.0 / C.draft_s;
    const T* const y = static_cast<const T*>(A.y) + (t >= 0 ? t : 0);
    const T* const z = static_cast<const T*>(A.z) + (t >= 0 ? t : 0);
    double sum = 0.0;
    if (t >= 0)
        for (int64_t r0 = part * A.part_rows + (x >> A.seq_log2); r0 < end; r0 += 8 * rows) {
            float p[8], q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t r = r0 + i * rows < end ? r0 + i * rows : r0;
                p[i] = to_float(y[r * A.ldy]);
                q[i] = to_float(z[r * A.ldz]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (r0 + i * rows < end) sum += left_of(A, C, share, draft_share, p[i], q[i]);
        }
    side[x] = sum;
    __syncthreads();
    if (x < width && t >= 0) {
        double all = 0.0;
        for (int i = 0; i < rows; ++i) all += side[i * width + x];
        A.left[part * A.sequences + b0 + x] = all;
    }
}

// Running sums over the workgroup's threads: v's own included.  By wavefronts, then over them.
__device__ __forceinline__ double running(double v, double* side, double& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int step = 1; step < 64; step <<= 1) {
        const long long bits = __double_as_longlong(v);
        const int lo = __shfl_up((int)bits, step), hi = __shfl_up((int)(bits >> 32), step);
        if (lane >= step) v += __longlong_as_double(((long long)hi << 32) | (uint32_t)lo);
    }
    __syncthreads();
    if (lane == 63) side[wave] = v;
    __syncthreads();
    double before = 0.0;
    total = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) before += side[w];
        total += side[w];
    }
    return before + v;
}

// One workgroup per sequence: how many drafts are kept, and the next token.
template <typename T>
__global__ void __launch_bounds__(kThreads)
k_verify_draw(VerifyArgs A)
{
    __shared__ int drawn, shared, last_some;
    __shared__ double side[kThreads / 64];
    __shared__ double found_before;
    const int x = threadIdx.x;
    const int64_t b = blockIdx.x;
    find_drawn(A, b, 0, &drawn);
    const int64_t t = drawn;
    VerifyColumn C{};
    C.mode = kVerifyNone;
    if (t >= 0) C = A.columns[t];
    if (x == 0) A.accepted[b] = t >= 0 ? t - start_of(A, b) : 0;
    if (C.mode == kVerifyNone || C.mode == kVerifyPlace) {
        if (x == 0) {
            A.next[b] = C.mode == kVerifyNone ? -1 : C.place;
            if (A.next_logp)
                A.next_logp[b] = C.mode == kVerifyNone ? 0.0f : (float)(-log(C.s));      // the largest logit's
        }
        return;
    }
    const int64_t draft = C.mode == kVerifyOthers ? A.drafts[t] : -1;
    const double share = 1.0 / C.s, draft_share = 1.0 / C.draft_s;
    const double chance = A.next_chances[b];
    int mode = C.mode;
    // The weight of a row.  A part may be chosen only where one of its rows has some weight: a part's weight is the sum of these numbers, or no less than the largest of them and 0
    // if that is.  (So p is not divided by its sum here: of the smallest weights that would leave 0 in the rows, though not in a part's sum.)
    const auto row_weight = [&](int64_t r) {
        const float y = to_float(static_cast<const T*>(A.y)[r * A.ldy + t]);
        if (mode == kVerifyLeft) return left_of(A, C, share, draft_share, y, to_float(static_cast<const T*>(A.z)[r * A.ldz + t]));
        return mode == kVerifyOthers && r == draft ? 0.0 : weight_of(y, C.m, A.c);
    };
    // The draft's part of the rows, without the draft, is summed again: a difference would hold the rounding of what is taken away.
    const int64_t drafted = draft >= 0 ? draft / A.part_rows : -1;
    double others = 0.0;
    if (drafted >= 0) {
        const int64_t begin = drafted * A.part_rows, end = begin + A.part_rows < A.k ? begin + A.part_rows : A.k;
        double some = 0.0;
        for (int64_t r = begin + x; r < end; r += kThreads) some += row_weight(r);
        running(some, side, others);
    }
    // the weights of the parts of the rows: a thread each
    const auto part_weight = [&]() {
        if (x >= A.parts) return 0.0;
        if (mode == kVerifyLeft) return A.left[x * A.sequences + b];
        if (mode == kVerifyOthers && x == drafted) return others;
        return A.part_sum[x * A.batch + t] * weight_of(A.part_max[x * A.batch + t], C.m, A.c);
    };
    double total, mine = part_weight(), sum = running(mine, side, total);
    if (!(total > 0.0)) {                                 // nothing is left where it is refused: by rounding alone
        mode = kVerifyAll;
        mine = part_weight();
        sum = running(mine, side, total);
    }
    const double bar = chance * total;
    // the first thread whose running sum passes the bar and who has some weight; of none, the last one with some
    const auto first = [&](bool past, bool some) {
        if (x == 0) { shared = kThreads; last_some = 0; }
        __syncthreads();
        if (past && some) atomicMin(&shared, x);
        if (some) atomicMax(&last_some, x);
        __syncthreads();
        const int at = shared < kThreads ? shared : last_some;
        __syncthreads();
        return at;
    };
    const int part = first(sum > bar, mine > 0.0);
    if (x == part) found_before = sum - mine;
    __syncthreads();
    // within it every thread takes some consecutive rows
    const int64_t begin = part * A.part_rows, end = begin + A.part_rows < A.k ? begin + A.part_rows : A.k;
    const int64_t each = (end - begin + kThreads - 1) / kThreads, r0 = begin + x * each, r1 = r0 + each < end ? r0 + each : end;
    double rows = 0.0;
    for (int64_t r = r0; r < r1; ++r) rows += row_weight(r);
    double in_part;
    sum = running(rows, side, in_part);
    const int thread = first(found_before + sum > bar, rows > 0.0);
    if (x == thread) {
        double run = found_before + (sum - rows);
        int64_t next = -1;
        for (int64_t r = r0; r < r1; ++r) {
            const double w = row_weight(r);
            if (!(w > 0.0)) continue;
            next = r;
            run += w;
            if (run > bar) break;
        }
        A.next[b] = next;
        if (A.next_logp)
            A.next_logp[b] = next < 0 ? 0.0f : (float)(A.tau * ((double)to_float(static_cast<const T*>(A.y)[next * A.ldy + t]) - (double)C.m) - log(C.s));
    }
}

struct Plan { int lanes_log2; int64_t slabs, part_rows, parts; };

Plan plan_of(int64_t k, int64_t batch)
{
    Plan P;
    P.lanes_log2 = 0;
    while (P.lanes_log2 < 6 && (1 << P.lanes_log2) < batch) ++P.lanes_log2;
    P.slabs = (batch + (1 << P.lanes_log2) - 1) >> P.lanes_log2;
    const int64_t at_once = (int64_t)(kThreads >> P.lanes_log2) * kGroup;
    int64_t parts = (k + at_once - 1) / at_once;
    if (parts > kMaxParts) parts = kMaxParts;
    if (parts > 1 && parts * P.slabs > kWorkgroups) parts = kWorkgroups / P.slabs > 1 ? kWorkgroups / P.slabs : 1;
    P.part_rows = (k + parts - 1) / parts;
    P.part_rows = (P.part_rows + at_once - 1) / at_once * at_once;
    P.parts = (k + P.part_rows - 1) / P.part_rows;
    return P;
}

size_t aligned(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

// For either rule, with the drafts' logits or without.
size_t verify_workspace(int64_t k, int64_t batch, int64_t sequences)
{
    if (k == 0 || batch == 0 || sequences == 0) return 0;
    const int64_t columns = kMaxParts * batch, enough = (int64_t)kWorkgroups * kSlab + batch, most = columns < enough ? columns : enough;      // parts times columns
    return aligned(2 * most * 8) + aligned(2 * most * 4) + aligned(most * 8) + aligned(batch * sizeof(VerifyColumn)) + aligned(kMaxParts * sequences * 8);
}

// No columns, or no sequences: no sequence has a next token, no column a draft.
__global__ void __launch_bounds__(kThreads)
k_verify_none(VerifyArgs A)
{
    for (int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x; b < A.sequences; b += (int64_t)gridDim.x * kThreads) {
        A.accepted[b] = 0;
        A.next[b] = -1;
        if (A.next_logp) A.next_logp[b] = 0.0f;
    }
    if (A.logp)
        for (int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x; t < A.batch; t += (int64_t)gridDim.x * kThreads) A.logp[t] = 0.0f;
}

template <typename T>
static hipError_t launch_verify_of(const VerifyArgs& A, const Plan& P, hipStream_t st)
{
    const dim3 grid((unsigned)P.slabs, (unsigned)P.parts, A.z ? 2 : 1), block(kThreads);
    const bool place = A.part_place != nullptr;
    profile_before("verify_rows", st);
    if (place) hipLaunchKernelGGL((k_verify_rows<T, true>), grid, block, 0, st, A);
    else hipLaunchKernelGGL((k_verify_rows<T, false>), grid, block, 0, st, A);
    profile_after("verify_rows", st);
    const dim3 columns((unsigned)((A.batch + kThreads / 64 - 1) / (kThreads / 64)));
    profile_before("verify_judge", st);
    if (place) hipLaunchKernelGGL((k_verify_judge<T, true>), columns, block, 0, st, A);
    else hipLaunchKernelGGL((k_verify_judge<T, false>), columns, block, 0, st, A);
    profile_after("verify_judge", st);
    if (A.z) {
        profile_before("verify_left", st);
        hipLaunchKernelGGL((k_verify_left<T>), dim3((unsigned)((A.sequences + (1 << A.seq_log2) - 1) >> A.seq_log2), (unsigned)P.parts), block, 0, st, A);
        profile_after("verify_left", st);
    }
    profile_before("verify_draw", st);
    hipLaunchKernelGGL((k_verify_draw<T>), dim3((unsigned)A.sequences), block, 0, st, A);
    profile_after("verify_draw", st);
    return hipGetLastError();
}

hipError_t launch_verify(const VerifyArgs& given, hipStream_t st)
{
    VerifyArgs A = given;
    if (A.batch == 0 || A.sequences == 0) {
        const int64_t most = A.batch > A.sequences ? A.batch : A.sequences;
        hipLaunchKernelGGL(k_verify_none, dim3((unsigned)((most + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, A);
        return hipGetLastError();
    }
    const Plan P = plan_of(A.k, A.batch);
    A.lanes_log2 = P.lanes_log2; A.part_rows = P.part_rows; A.parts = P.parts;
    // (us with 1 / 4 / 8 / 16 sequences side by side: 512 of 4 columns 895 / 386 / 292 / 302, 200 of 5 324 / 178 / 164 / 166, 8 of 5 62 / 43 / 41 / 41)
    A.seq_log2 = 0;
    while (A.seq_log2 < 4 && (1 << A.seq_log2) < A.sequences) ++A.seq_log2;
    char* at = A.ws;
    const auto take = [&](size_t bytes) { char* const here = at; at += aligned(bytes); return here; };
    A.part_sum = reinterpret_cast<double*>(take(2 * P.parts * A.batch * 8));
    A.part_max = reinterpret_cast<float*>(take(2 * P.parts * A.batch * 4));
    if (A.greedy) A.part_place = reinterpret_cast<int64_t*>(take(P.parts * A.batch * 8));
    A.columns = reinterpret_cast<VerifyColumn*>(take(A.batch * sizeof(VerifyColumn)));
    A.left = reinterpret_cast<double*>(take(P.parts * A.sequences * 8));
    return A.bf16 ? launch_verify_of<__bf16>(A, P, st) : launch_verify_of<float>(A, P, st);
}

}  // namespace laplex
