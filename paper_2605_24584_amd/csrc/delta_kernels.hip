// Linear attention by the gated delta rule.  Per head, with l_t = exp(-rates_t) and the state S (dk x dv):
//   S <- l_t S,   u_t = beta_t (v_t - S^T k_t),   S <- S + k_t u_t^T,   y_t = scale S^T q_t.
//
// In chunks of C tokens, with G_i = -(rates_1 + .. + rates_i) inside the chunk, D_ij = exp(G_i - G_j), gamma_i = exp(G_i), tail_j = exp(G_C - G_j), the state S0
// that enters the chunk and q, k, v, u as rows:
//   A_ij = beta_i D_ij k_i.k_j (j < i),   T = (1 + A)^-1,   U = T beta (V - gamma K S0)
//   Y = scale (gamma Q S0 + P U),  P_ij = D_ij q_i.k_j (j <= i),     S_C = gamma_C S0 + (tail K)^T U
// and backwards, from the gradient G of S_C:
//   dU = scale P^T gY + tail K G,   dR = T^T dU,   gV = beta dR,   dS0 = gamma_C G + scale (gamma Q)^T gY - (beta gamma K)^T dR
//   N = scale D (gY U^T) (j <= i),  M = -beta D (dR U^T) (j < i)
//   gQ = N K + scale gamma gY S0^T,   gK = N^T Q + (M + M^T) K - beta gamma dR S0^T + tail U G^T
//   gbeta_i = dR_i.(v_i - gamma_i S0^T k_i) + sum_j M_ij k_i.k_j / beta_i,    and what goes to the decays from the same sums (k_delta_gradients).
//
// In chunks k_delta_prepare forms T for every chunk and head, all chunks at once.  k_delta_walk goes over the chunks of a sequence with the state in
// accumulator registers: a wavefront owns 16 columns of the state, of U and of the results, and since an accumulator (a pair of them in bf16) IS a fragment of the
// next product over the same rows, neither the state nor U passes through memory on its way from product to product.  k_delta_back is the walk from the last chunk
// to the first, with the gradient of the state.  k_delta_gradients forms what is left of the gradients, all chunks at once, from the states, U, G and dR that the two
// walks have written.  Long sequences are cut into stretches of chunks: a walk of all stretches at once finds what each does to a state (S -> turned S + added), k_delta_carry
// joins these in order, and the walks then start from the stretches' own states.  k_delta_tokens takes sequences of a few tokens one token at a time.
//
// What bounds it (us, bf16, heads of 128): products that wait for one another with one or two wavefronts on a SIMD, as many vector instructions beside them (splits into
// parts, decays), and in the gradients LDS, of which a workgroup takes all.  8 x 4096 tokens of 16 heads, trained: prepare 105, walk 517, back 483, gradients 908 (the recurrence's operations and bytes
// would take 220).  There memory has a part in it too: the walks write states, their gradients, U and dR, 1.6 GB, and the gradients read them (counted: 0.95 GB written by the
// walk, 0.81 by the walk back); there and back they would take 650 of the 1942 at a copy's rate.  4 x 2048 of 16: prepare 40, stretches 94, carry 21, walk 84.  65536 of 8: 136, 350, 122,
// 274.  256 sequences of up to 5 tokens, token by token: 124 with the caches filled with other data before (114 among other calls), which is 0.54 GB of states at 4.4 TB/s.
// Scratch (bytes a lane): the walk with results 44 (128 numbers, 8 wavefronts) and 28 (256), prepare 36 in bf16 up to 128 numbers, gradients 8 (96 numbers, bf16), tokens 12 (8 rows a
// thread).
// Chunks of half as many tokens make the walks slower (4 x 2048 268 -> 350, 8 x 4096 trained 2120 -> 3390): a chunk's waits stay, and there are twice as many.  Sixteen wavefronts for the gradients
// spill.  Fragments asked for a step ahead took 8 x 4096 from 2120 to 2030, 65536 from 963 to 925.
//
// Numbers: sums, states and everything from which states come are fp32 numbers; in bf16 they enter products as sums of three bf16 numbers (exactly; of the nine
// products of two such sums the three below 2^-24 are left out).  What only goes into a result that is rounded to bf16 enters as two (16 bits).  The
// G_i are summed in 64 bits, since differences of far sums are what counts.
#include "token_tiles.h"

namespace laplex {

namespace {

constexpr int kPrepareThreads = 256;
constexpr int64_t kRows = 32768;          // sequences or chunks along a grid's second axis
constexpr int64_t kPays = 3;              // sequences of more stretches are cut into them (see cut_of)

// ----------------------------------------------------------------------------
// Sequences, and the chunks of sequences: sequence b has the chunks first_chunk(b), ...: at least as many as its rows need, whatever its length.
// ----------------------------------------------------------------------------
__device__ __forceinline__ int64_t start_of(const DeltaArgs& A, int64_t b)
{
    if (!A.starts) return A.each * b;
    const int64_t v = A.starts[b];                     // whatever it holds, no row outside the matrices is touched
    return v < 0 ? 0 : v > A.tokens ? A.tokens : v;
}

__device__ __forceinline__ int64_t count_of(const DeltaArgs& A, int64_t b, int64_t begin)
{
    const int64_t end = start_of(A, b + 1), count = end > begin ? end - begin : 0;
    if (!A.lengths) return count;
    const int64_t n = A.lengths[b];
    return n < 0 ? 0 : n < count ? n : count;
}

// Sequences are cut into units of so many tokens (chunks, or stretches of chunks): sequence b has those from first_unit(b) on, at least as many as its rows need.
__device__ __forceinline__ int64_t first_unit(const DeltaArgs& A, int64_t b, int64_t begin, int64_t size, int64_t per_sequence)
{
    return A.starts ? (uint32_t)begin / (uint32_t)size + b : b * per_sequence;
}

template <int C>
__device__ __forceinline__ int64_t first_chunk(const DeltaArgs& A, int64_t b, int64_t begin) { return first_unit(A, b, begin, C, A.per_sequence); }

// a whole number that all lanes hold
__device__ __forceinline__ int64_t uniform(int64_t v)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)v), hi = __builtin_amdgcn_readfirstlane((int)(v >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

// The unit with this number: its sequence and its number there.  By a wavefront.
struct Unit { int64_t b, index, begin, count; };      // begin, count: the sequence's rows
__device__ __forceinline__ Unit find_unit(const DeltaArgs& A, int64_t unit, int64_t size, int64_t per_sequence)
{
    int64_t lo = 0;
    if (A.starts) {
        // the last sequence whose first unit is at most this one: 64 candidates at a time
        int64_t hi = A.sequences;
        const int lane = threadIdx.x & 63;
        while (hi - lo > 1) {
            const int64_t step = (uint32_t)(hi - lo + 63) / 64u, c = lo + lane * step;
            const uint64_t votes = __ballot(c < hi && first_unit(A, c, start_of(A, c), size, per_sequence) <= unit);
            const int at = votes ? 63 - __builtin_clzll(votes) : 0;
            lo += at * step;
            hi = lo + step < hi ? lo + step : hi;
        }
    } else {
        lo = (uint32_t)unit / (uint32_t)per_sequence;
    }
    Unit u;
    u.b = uniform(lo);
    u.begin = uniform(start_of(A, u.b));
    u.count = uniform(count_of(A, u.b, u.begin));
    u.index = uniform(unit - first_unit(A, u.b, u.begin, size, per_sequence));
    return u;
}

// The chunk with this number: its first row and how many rows it has (0: there is none).
template <int C>
__device__ __forceinline__ void find_chunk(const DeltaArgs& A, int64_t chunk, int64_t& row, int& valid)
{
    const Unit u = find_unit(A, chunk, C, A.per_sequence);
    const int64_t at = u.index * C;
    row = u.begin + at;
    valid = at >= 0 && at < u.count ? (u.count - at < C ? (int)(u.count - at) : C) : 0;
}

// Of sequences with several stretches each has a place in the workspace.  They are numbered like the stretches, but for b, where no more than
// begin / (stretch + 1) sequences before this one can have several: however many short sequences are packed, there are at most two places for `stretch` tokens.
__device__ __forceinline__ int64_t first_place(const DeltaArgs& A, int64_t b, int64_t begin)
{
    if (!A.starts) return b * A.stretches;
    const int64_t several = (uint32_t)begin / (uint32_t)(A.stretch + 1);
    return (uint32_t)begin / (uint32_t)A.stretch + (b < several ? b : several);
}

// The stretch with this number, [lo, hi) of its sequence's tokens; a sequence of up to kPays of them is one.
struct Stretch {
    int64_t b, begin, lo, hi, index, place;
    bool there, last, several;        // several: its sequence has more than one
};
__device__ __forceinline__ Stretch find_stretch(const DeltaArgs& A, int64_t slot)
{
    const Unit u = find_unit(A, slot, A.stretch, A.stretches);
    Stretch s;
    s.b = u.b; s.begin = u.begin; s.index = u.index;
    s.several = u.count > kPays * A.stretch;
    s.lo = s.several ? u.index * A.stretch : 0;
    s.there = u.index == 0 || (s.several && u.index > 0 && s.lo < u.count);
    s.hi = s.several && s.lo + A.stretch < u.count ? s.lo + A.stretch : u.count;
    s.last = s.hi == u.count;
    s.place = first_place(A, s.b, s.begin) + s.index;
    return s;
}

// ----------------------------------------------------------------------------
// Geometry, and what a chunk and head leave in the workspace.
// ----------------------------------------------------------------------------
template <typename T, int DK>
struct Sizes {
    static constexpr int E = Num<T>::E, K = Num<T>::K, R = Patch<T>::R;
    static constexpr int C = (DK > 128 ? 32 : 64) * 2 / (int)sizeof(T);
    static constexpr int CT = C / 16, DT = DK / 16, KD = DK / K, KC = C / K;
    static constexpr int ROW = (DK * (int)sizeof(T) / 16 + 7) / 8 * 8, SEQ = C * (int)sizeof(T) / 16;      // slots of a row of numbers, of tokens
    static constexpr int kBytesRows = C * ROW * 16, kBytesTurned = DK * SEQ * 16, kBytesMap = C * SEQ * 16;
    static constexpr int PARTS = sizeof(T) == 2 ? 3 : 1, SOME = sizeof(T) == 2 ? 2 : 1;                    // of an fp32 number: all 24 bits, 16
    static constexpr int TILES = CT * (CT + 1) / 2;
    // numbers of a chunk and head: T and scale P (tiles on and below the diagonal, rows of 16), then what follows
    static constexpr int kP = TILES * 256, kBeta = 2 * kP, kGamma = kBeta + C, kTail = kGamma + C, kHigh = kTail + C, kLow = kHigh + C, kWhole = kLow + C, kBad = kWhole + 2,
                         kNumbers = kWhole + 4;
};

__device__ __forceinline__ int tile_at(int i, int j) { return i * (i + 1) / 2 + j; }

// Fragments of fp32 numbers in accumulators, as sums of PARTS fragments
template <typename T, int PARTS>
__device__ __forceinline__ void parts_of(const float* x, typename Num<T>::frag* out)
{
    if constexpr (sizeof(T) == 2) {
        if constexpr (PARTS == 3) split3(x, out[0], out[1], out[2]);
        else split2(x, out[0], out[1]);
    } else {
        out[0] = f32x4{x[0], x[1], x[2], x[3]};
    }
}

// fragment m of accumulators that hold rows 16 t + 4 g .. + 3 each
template <typename T>
__device__ __forceinline__ void numbers_of(const f32x4* acc, int m, float* x)
{
#pragma unroll
    for (int e = 0; e < Num<T>::E; ++e) x[e] = sizeof(T) == 2 ? acc[2 * m + (e >> 2)][e & 3] : acc[m][e];
}

// a (exact) times a sum of parts; of two sums of three parts; of two sums of two
template <int PARTS, typename F>
__device__ __forceinline__ f32x4 mma_exact(F a, const F* b, f32x4 c)
{
#pragma unroll
    for (int p = PARTS - 1; p >= 0; --p) c = mma(a, b[p], c);
    return c;
}
template <int PARTS, typename F>
__device__ __forceinline__ f32x4 mma_parts(const F* a, const F* b, f32x4 c)
{
#pragma unroll
    for (int s = PARTS - 1; s >= 0; --s)
#pragma unroll
        for (int p = 0; p <= s; ++p) c = mma(a[p], b[s - p], c);
    return c;
}

// Where four tokens or numbers 4 p .. + 3 of a row lie: quads of 32 bf16 numbers in the order 0 4 1 5 2 6 3 7, which is a pair of accumulators'.
template <typename T, int SLOTS>
__device__ __forceinline__ int quad_at(int row, int p)
{
    if (sizeof(T) == 2) return 16 * slot_at<SLOTS>(row, (p >> 3) * 4 + (p & 3)) + 8 * ((p >> 2) & 1);
    return 16 * slot_at<SLOTS>(row, p);
}

// The patch's columns as rows, tokens along the slots in that order.  (The permutation of row 4 piece + e is that of row 4 piece, changed by e alone.)
template <typename T, int SLOTS>
__device__ __forceinline__ void put_turned(char* tile, const Patch<T>& p, int first, int piece)
{
    const int quad = first >> 2, slot = sizeof(T) == 2 ? (quad >> 3) * 4 + (quad & 3) : quad, low = slot ^ twist<SLOTS>(piece * 4);
    char* const at = tile + piece * 4 * SLOTS * 16 + (sizeof(T) == 2 ? 8 * ((quad >> 2) & 1) : (first & 2) * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        char* const to = at + e * SLOTS * 16 + 16 * (low ^ (SLOTS >= 8 ? e : (e >> 1)));
        if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x4*>(to) = bf16x4{p.r[0][e], p.r[1][e], p.r[2][e], p.r[3][e]};
        else *reinterpret_cast<f32x2*>(to) = f32x2{p.r[0][e], p.r[1][e]};
    }
}

// four fp32 numbers as PARTS quads, `size` bytes apart
template <typename T, int PARTS>
__device__ __forceinline__ void put_parts(char* at, int size, f32x4 v)
{
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<f32x4*>(at) = v;
    } else {
        f32x4 r = v;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            if (p + 1 < PARTS || PARTS == 3) {
                *reinterpret_cast<u32x2*>(at + p * size) = u32x2{__builtin_amdgcn_perm(__float_as_uint(r[1]), __float_as_uint(r[0]), 0x07060302u),
                                                                  __builtin_amdgcn_perm(__float_as_uint(r[3]), __float_as_uint(r[2]), 0x07060302u)};
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] -= upper(r[e]);
            } else {
                *reinterpret_cast<bf16x4*>(at + p * size) = bf16x4{(__bf16)r[0], (__bf16)r[1], (__bf16)r[2], (__bf16)r[3]};
            }
        }
    }
}

// How a matrix is read: kSome a number at a time, kWide four at a time, kWhole so where all of them exist.
enum { kSome, kWide, kWhole };
__device__ __forceinline__ int how(bool wide, bool whole) { return !wide ? kSome : whole ? kWhole : kWide; }

// Accumulators to rows of `stride` numbers from base on, which all lanes share: rows 16 t + 4 g + r, column col.
template <int TILES>
__device__ __forceinline__ void store_tiles(float* base, const f32x4* acc, int stride, int g, int col)
{
    const uint32_t at = 4 * g * stride + col;
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) *reinterpret_cast<float*>(reinterpret_cast<char*>(base) + (at + (16 * t + r) * stride) * 4u) = acc[t][r];
}

template <typename T>
__device__ __forceinline__ void put_number(char* at, T v) { *reinterpret_cast<T*>(at) = v; }

// A patch of R rows of four numbers, whatever their alignment; others in the place of those that do not exist (keep_patch makes zeros of them).
template <typename T>
__device__ __forceinline__ void load_patch(Patch<T>& p, const T* base, int64_t stride, int first, int valid, int at, int width, int how)
{
    if (how == kWhole) load_wide<T, false>(p, base, stride, first, valid, at, width);
    else if (how == kWide) load_wide<T, true>(p, base, stride, first, valid, at, width);
    else load_some(p, base, stride, first, valid, at, width);
}

// numbers that are not finite become zeros
__device__ __forceinline__ void clean_patch(Patch<float>& p)
{
#pragma unroll
    for (int i = 0; i < Patch<float>::R; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) p.r[i][e] = finite_bits(p.r[i][e]) ? p.r[i][e] : 0.0f;
}
__device__ __forceinline__ void clean_patch(Patch<__bf16>& p)
{
#pragma unroll
    for (int i = 0; i < Patch<__bf16>::R; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) p.r[i][e] = finite_bits((float)p.r[i][e]) ? p.r[i][e] : (__bf16)0.0f;
}
// the first row of a patch that holds such a number
template <typename T>
__device__ __forceinline__ int odd_row(const Patch<T>& p)
{
#pragma unroll
    for (int i = 0; i < Patch<T>::R; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!finite_bits((float)p.r[i][e])) return i;
    return 0;
}

__device__ __forceinline__ float decay_of(float high_i, float low_i, float high_j, float low_j) { return expf((high_i - high_j) + (low_i - low_j)); }

// ----------------------------------------------------------------------------
// T and the decays of every chunk and head.  A workgroup takes a chunk and a head of keys, and the heads of values that share it one after the other.
// T by blocks of 16: those on the diagonal by substitution, a lane to a column; T_ij = -T_ii sum_{j <= m < i} A_im T_mj, a wavefront to a column of blocks.
// ----------------------------------------------------------------------------
template <typename T, int DK>
__global__ void __launch_bounds__(kPrepareThreads, 4)
k_delta_prepare(DeltaArgs A)
{
    typedef Sizes<T, DK> Z;
    constexpr int C = Z::C, CT = Z::CT, R = Z::R, WAVES = kPrepareThreads / 64, PAD = C + 4;
    // the keys and queries, and in their place, when their products are formed, A and the inverses of its blocks
    constexpr int kMap = C * PAD * 4, kDiagonal = CT * 16 * 20 * 4, kBytes = 2 * Z::kBytesRows > kMap + kDiagonal ? 2 * Z::kBytesRows : kMap + kDiagonal;
    __shared__ __attribute__((aligned(16))) char lds[kBytes];
    char *const Ks = lds, *const Qs = lds + Z::kBytesRows;
    float* const map = reinterpret_cast<float*>(lds);
    float (*const diagonal)[16][20] = reinterpret_cast<float (*)[16][20]>(lds + kMap);
    __shared__ double G[C];
    __shared__ float beta[C];
    __shared__ int odd_key, odd;
    const int x = threadIdx.x, lane = x & 63, wave = __builtin_amdgcn_readfirstlane(x >> 6), r16 = lane & 15, g = lane >> 4;
    const int64_t chunk = (int64_t)blockIdx.z * kRows + blockIdx.y;
    if (chunk >= A.chunks) return;
    int64_t row;
    int valid;
    find_chunk<C>(A, chunk, row, valid);
    if (valid == 0) return;
    const int kh = blockIdx.x, group = A.heads / A.key_heads;
    if (x == 0) odd_key = C;
    __syncthreads();
    const T* const k = static_cast<const T*>(A.k) + row * A.ldk + (int64_t)kh * A.dk;
    const int64_t near = INT32_MAX / (int64_t)(C * sizeof(T)) - DK;
    const bool wide = (A.wide & 2) && A.ldk < near, wide_q = (A.wide & 1) && A.ldq < near;
    const T* const q = static_cast<const T*>(A.q) + row * A.ldq + (int64_t)kh * A.dk;
    for (int p = x; p < (C / R) * (DK / 4); p += kPrepareThreads) {
        const int piece = p % (DK / 4), first = (p / (DK / 4)) * R;
        Patch<T> patch, query;
        load_patch(patch, k, A.ldk, first, valid, piece * 4, A.dk, wide);
        load_patch(query, q, A.ldq, first, valid, piece * 4, A.dk, wide_q);
        keep_patch(query, first, valid, piece * 4, A.dk);
        put_rows<Z::ROW>(Qs, query, first, piece);
        keep_patch(patch, first, valid, piece * 4, A.dk);
        if (!finite_patch(patch)) {
            atomicMin(&odd_key, first + odd_row(patch));
            clean_patch(patch);
        }
        put_rows<Z::ROW>(Ks, patch, first, piece);
    }
    __syncthreads();
    // k_i . k_j and q_i . k_j: a lane holds rows 4 g .. + 3 and column r16 of a tile
    constexpr int NT = (Z::TILES + WAVES - 1) / WAVES;
    f32x4 kk[NT], qk[NT];
    const Reader<Z::ROW> rows(r16, g);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int tile = n * WAVES + wave;
        int it = 0, jt = tile;
        while (jt > it) { jt -= it + 1; ++it; }
        kk[n] = qk[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (it < CT)
#pragma unroll
            for (int m = 0; m < Z::KD; ++m) {
                const typename Num<T>::frag kf = get<T>(Ks, rows.at(jt, m));
                kk[n] = mma(get<T>(Ks, rows.at(it, m)), kf, kk[n]);
                qk[n] = mma(get<T>(Qs, rows.at(it, m)), kf, qk[n]);
            }
    }
    for (int e = 0; e < group; ++e) {
        const int h = kh * group + e;
        float* const out = A.maps + (chunk * A.heads + h) * Z::kNumbers;
        __syncthreads();
        if (x == 0) odd = odd_key;
        __syncthreads();
        if (wave == 0) {
            // sums of the rates in 64 bits.  A rate from 1e5 on leaves nothing (e^-104 is 0 in fp32), and keeps the differences behind it exact.
            float rate = 0.0f, b = 0.0f;
            if (lane < valid) {
                rate = A.rates[(row + lane) * A.ldr + h];
                b = A.beta[(row + lane) * A.ldb + h];
            }
            if (!(rate > -INFINITY) || !finite_bits(b)) { atomicMin(&odd, lane); rate = b = 0.0f; }
            double sum = rate < 1.0e5f ? -(double)rate : -1.0e5;
            for (int step = 1; step < 64; step <<= 1) {
                const long long bits = __double_as_longlong(sum);
                const int lo = __shfl_up((int)bits, step), hi = __shfl_up((int)(bits >> 32), step);
                if (lane >= step) sum += __longlong_as_double(((long long)hi << 32) | (uint32_t)lo);
            }
            if (lane < C) {
                G[lane] = sum;
                beta[lane] = b;
            }
        }
        __syncthreads();
        if (x < C) {
            const double mine = G[x], all = G[C - 1];
            const float high = (float)mine;
            out[Z::kBeta + x] = beta[x];
            out[Z::kGamma + x] = (float)exp(mine);
            out[Z::kTail + x] = (float)exp(all - mine);
            out[Z::kHigh + x] = high;
            out[Z::kLow + x] = (float)(mine - (double)high);
            if (x == 0) {
                const double whole = exp(all);
                out[Z::kWhole] = (float)whole;
                out[Z::kWhole + 1] = (float)(whole - (double)(float)whole);
                reinterpret_cast<int*>(out)[Z::kBad] = odd;
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int tile = n * WAVES + wave;
            int it = 0, jt = tile;
            while (jt > it) { jt -= it + 1; ++it; }
            if (it < CT)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * it + 4 * g + r, j = 16 * jt + r16;
                    const float d = j <= i ? expf((float)(G[i] - G[j])) : 0.0f;
                    map[i * PAD + j] = j < i ? beta[i] * d * kk[n][r] : 0.0f;
                    out[Z::kP + tile * 256 + (4 * g + r) * 16 + r16] = j <= i ? A.scale * d * qk[n][r] : 0.0f;
                }
        }
        __syncthreads();
        if (wave == 0 && lane < C) {
            const int b = lane >> 4, c = lane & 15;
            float t[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float s = i == c ? 1.0f : 0.0f;
#pragma unroll
                for (int m = 0; m < i; ++m) s = fmaf(-map[(16 * b + i) * PAD + 16 * b + m], t[m], s);
                t[i] = s;
                diagonal[b][i][c] = s;
            }
        }
        __syncthreads();
        for (int j = wave; j < CT; j += WAVES) {
            f32x4 X[CT];
#pragma unroll
            for (int i = 0; i < CT; ++i) {
                if (i < j) continue;
                if (i == j) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) X[i][r] = diagonal[i][4 * g + r][r16];
                } else {
                    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int m = 0; m < i; ++m)
                        if (m >= j) s = mma(*reinterpret_cast<const f32x4*>(&map[(16 * i + r16) * PAD + 16 * m + 4 * g]), X[m], s);
                    s = mma(*reinterpret_cast<const f32x4*>(&diagonal[i][r16][4 * g]), s, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
                    X[i] = -s;
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) out[tile_at(i, j) * 256 + (4 * g + r) * 16 + r16] = X[i][r];
            }
        }
    }
}

// ----------------------------------------------------------------------------
// The walk over the chunks of a sequence.
// ----------------------------------------------------------------------------
template <typename T, int DK, int WAVES, bool OUT>
struct WalkLds {
    typedef Sizes<T, DK> Z;
    static constexpr int COLS = 16 * WAVES;
    static constexpr int kTurned = 0, kMap = kTurned + Z::kBytesTurned, kKeys = kMap + Z::PARTS * Z::kBytesMap, kValues = kKeys + Z::kBytesRows;
    static constexpr int kQueries = kValues + COLS * Z::SEQ * 16, kP = kQueries + Z::kBytesRows;
    static constexpr int kBytes = OUT ? kP + Z::SOME * Z::kBytesMap : kQueries;
};

enum { kResults, kKeep, kStates };      // with results; what gradients need alone; what a stretch does to the state, for the stretches behind it

template <typename T, int DK, int WAVES, int MODE>
__global__ void __launch_bounds__(64 * WAVES)
k_delta_walk(DeltaArgs A)
{
    typedef Sizes<T, DK> Z;
    constexpr bool OUT = MODE == kResults, STATES = MODE == kStates;
    typedef WalkLds<T, DK, WAVES, OUT> L;
    typedef typename Num<T>::frag frag;
    typedef typename Num<T>::quad quad;
    constexpr int C = Z::C, R = Z::R, ROW = Z::ROW, SEQ = Z::SEQ, CT = Z::CT, DT = Z::DT, KD = Z::KD, KC = Z::KC, THREADS = 64 * WAVES, COLS = L::COLS;
    __shared__ __attribute__((aligned(16))) char lds[L::kBytes];
    __shared__ __attribute__((aligned(16))) float beta[C], gamma[C], tail[C], whole[2];
    __shared__ int odd[2];
    char *const Kt = lds + L::kTurned, *const Ts = lds + L::kMap, *const Ks = lds + L::kKeys, *const Vt = lds + L::kValues, *const Qs = lds + L::kQueries, *const Ps = lds + L::kP;

    // STATES: the first half of a head's workgroups sum up what the stretch adds to the state, the second half how it turns the state that enters it: the columns of a unit matrix
    const int parts = STATES ? 2 : 1, slice = blockIdx.x % A.slices, part = blockIdx.x / A.slices % parts, h = blockIdx.x / (A.slices * parts), col0 = slice * COLS;
    const int64_t slot = (int64_t)blockIdx.z * kRows + blockIdx.y;
    if (slot >= A.slots || col0 >= (part ? A.dk : (A.dv + Z::K - 1) / Z::K * Z::K)) return;      // (k_delta_gradients reads whole fragments of columns)
    const Stretch s = find_stretch(A, slot);
    if (!s.there || (STATES && (!s.several || (s.last && !(part && A.training))))) return;
    const int64_t b = s.b, begin = s.begin, count = s.hi, chunk0 = first_chunk<C>(A, b, begin);
    const int x = threadIdx.x, lane = x & 63, wave = __builtin_amdgcn_readfirstlane(x >> 6), r16 = lane & 15, g = lane >> 4;
    const int kh = h / (A.heads / A.key_heads), col = col0 + 16 * wave + r16;
    for (int i = x; i < Z::PARTS * Z::kBytesMap / 16; i += THREADS) reinterpret_cast<f32x4*>(Ts)[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (OUT)
        for (int i = x; i < Z::SOME * Z::kBytesMap / 16; i += THREADS) reinterpret_cast<f32x4*>(Ps)[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (x < 2) odd[x] = C;

    // the state: rows 16 t + 4 g .. + 3, column col
    f32x4 S[DT];
    float* const entering = A.added + (s.place * A.heads + h) * (int64_t)DK * DK + col;      // (of several stretches the first one's, too: another workgroup may already write the last state in its place)
    const int64_t state_at = (b * A.heads + h) * (int64_t)A.dk * A.dv;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * t + 4 * g + r;
            if (STATES) S[t][r] = part && row == col && col < A.dk ? 1.0f : 0.0f;      // (nothing behind dk: no key takes of it what rates below 0 add)
            else if (s.several) S[t][r] = col < A.dv ? entering[row * DK] : 0.0f;
            else S[t][r] = A.state_in && row < A.dk && col < A.dv ? A.state_in[state_at + (int64_t)row * A.dv + col] : 0.0f;
        }

    const int64_t near = INT32_MAX / (int64_t)(C * sizeof(T)) - DK;
    const bool wq = (A.wide & 1) && A.ldq < near, wk = (A.wide & 2) && A.ldk < near, wv = (A.wide & 4) && A.ldv < near, wo = A.wide & 8;
    constexpr int kRowPatches = (C / R) * (DK / 4), kColPatches = (C / R) * (COLS / 4);
    constexpr int NR = (kRowPatches + THREADS - 1) / THREADS, NV = (kColPatches + THREADS - 1) / THREADS, NM = (Z::TILES * 64 + THREADS - 1) / THREADS;
    Patch<T> pq[NR], pk[NR], pv[NV];
    f32x4 pt[NM], pp[NM];
    float pn[3], pw = 0.0f;
    int pb = C;
    const auto load = [&](int64_t at) {
        const int y = here(x);                         // (formed anew for each chunk, as everything below: places kept from before the loop would fill the registers)
        const int valid = (int)(count - at < C ? count - at : C);
        const int64_t row = begin + at;
        const int hq = how(wq, valid == C && A.dk == DK), hk = how(wk, valid == C && A.dk == DK), hv = how(wv, valid == C && col0 + COLS <= A.dv);
        const T* const q = static_cast<const T*>(A.q) + row * A.ldq + (int64_t)kh * A.dk;
        const T* const k = static_cast<const T*>(A.k) + row * A.ldk + (int64_t)kh * A.dk;
        const T* const v = static_cast<const T*>(A.v) + row * A.ldv + (int64_t)h * A.dv;
        const float* const numbers = A.maps + ((chunk0 + at / C) * A.heads + h) * Z::kNumbers;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int p = y + i * THREADS, first = (p / (DK / 4)) * R, piece = (p % (DK / 4)) * 4;
            if (kRowPatches % THREADS == 0 || p < kRowPatches) {
                if (OUT) load_patch(pq[i], q, A.ldq, first, valid, piece, A.dk, hq);
                load_patch(pk[i], k, A.ldk, first, valid, piece, A.dk, hk);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = y + i * THREADS;
            if ((kColPatches % THREADS == 0 || p < kColPatches) && part == 0)
                load_patch(pv[i], v, A.ldv, (p / (COLS / 4)) * R, valid, col0 + (p % (COLS / 4)) * 4, A.dv, hv);
        }
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            const int p = y + i * THREADS;
            if (Z::TILES % WAVES == 0 || i * WAVES + wave < Z::TILES) {
                pt[i] = reinterpret_cast<const f32x4*>(numbers)[p];
                if (OUT) pp[i] = reinterpret_cast<const f32x4*>(numbers + Z::kP)[p];
            }
        }
        if (y < C) {
#pragma unroll
            for (int i = 0; i < 3; ++i) pn[i] = numbers[Z::kBeta + i * C + y];
        }
        if (y < 2) pw = numbers[Z::kWhole + y];
        if (x == 0) pb = reinterpret_cast<const int*>(numbers)[Z::kBad];
    };
    if (s.lo < count) load(s.lo);
    __syncthreads();

    int turn = 0;
    for (int64_t at = s.lo; at < count; at += C, turn ^= 1) {
        const int valid = (int)(count - at < C ? count - at : C);
        const int y = here(x), l = here(lane), r16 = l & 15, g = l >> 4;
        const int64_t row = begin + at, chunk = chunk0 + at / C;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int p = y + i * THREADS, first = (p / (DK / 4)) * R, piece = p % (DK / 4);
            if (kRowPatches % THREADS == 0 || p < kRowPatches) {
                if (OUT) {
                    if (!(valid == C && A.dk == DK)) keep_patch(pq[i], first, valid, piece * 4, A.dk);
                    put_rows<ROW>(Qs, pq[i], first, piece);
                }
                if (!(valid == C && A.dk == DK)) keep_patch(pk[i], first, valid, piece * 4, A.dk);
                if (!finite_patch(pk[i])) clean_patch(pk[i]);
                put_rows<ROW>(Ks, pk[i], first, piece);
                put_turned<T, SEQ>(Kt, pk[i], first, piece);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = y + i * THREADS, first = (p / (COLS / 4)) * R, piece = p % (COLS / 4);
            if ((kColPatches % THREADS == 0 || p < kColPatches) && part == 0) {
                if (!(valid == C && col0 + COLS <= A.dv)) keep_patch(pv[i], first, valid, col0 + piece * 4, A.dv);
                if (!finite_patch(pv[i])) {
                    atomicMin(&odd[turn], first + odd_row(pv[i]));
                    clean_patch(pv[i]);
                }
                put_turned<T, SEQ>(Vt, pv[i], first, piece);
            }
        }
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            const int tile = i * WAVES + wave;         // (a wavefront takes a tile)
            if (Z::TILES % WAVES == 0 || tile < Z::TILES) {
                int it = 0, jt = tile;
                while (jt > it) { jt -= it + 1; ++it; }
                const int to = quad_at<T, SEQ>(16 * it + (l >> 2), 4 * jt + (l & 3));
                put_parts<T, Z::PARTS>(Ts + to, Z::kBytesMap, pt[i]);
                if (OUT) put_parts<T, Z::SOME>(Ps + to, Z::kBytesMap, pp[i]);
            }
        }
        if (y < C) { beta[y] = pn[0]; gamma[y] = pn[1]; tail[y] = pn[2]; }
        if (y < 2) whole[y] = pw;
        if (x == 0 && pb < C) atomicMin(&odd[turn], pb);
        __syncthreads();

        const int bad = odd[turn];                     // from this token on there is nothing but NaN
        const Reader<ROW> rows(r16, g);
        const Reader<SEQ> columns(r16, g);
        if (!STATES && A.states_out) store_tiles<DT>(A.states_out + (chunk * A.heads + h) * (int64_t)DK * DK, S, DK, g, col);
        f32x4 U[CT], O[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) U[t] = O[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        // K S and Q S: rows of tokens 16 t + 4 g .. + 3, column col, of the one, the other way round of the other
        // (fragments are asked for a step ahead of their products, here and below: the compiler would ask for each where it is needed, and wait)
        frag kf[2][CT], qf[2][CT];
        const auto ask_rows = [&](int m) {
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                kf[m & 1][t] = get<T>(Ks, rows.at(t, m));
                if (OUT) qf[m & 1][t] = get<T>(Qs, rows.at(t, m));
            }
        };
        ask_rows(0);
#pragma unroll
        for (int m = 0; m < KD; ++m) {
            if (m + 1 < KD) ask_rows(m + 1);
            __builtin_amdgcn_sched_barrier(0);
            float xs[Z::E];
            numbers_of<T>(S, m, xs);
            frag sf[Z::PARTS];
            parts_of<T, Z::PARTS>(xs, sf);
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                U[t] = mma_exact<Z::PARTS>(kf[m & 1][t], sf, U[t]);
                if (OUT)
#pragma unroll
                    for (int p = Z::SOME - 1; p >= 0; --p) O[t] = mma(sf[p], qf[m & 1][t], O[t]);
            }
        }
        frag tf[2][KC][Z::PARTS];
        const auto ask_map = [&](int t) {
#pragma unroll
            for (int m = 0; m < KC; ++m)
#pragma unroll
                for (int p = 0; p < Z::PARTS; ++p)
                    if (16 * t + 15 >= m * Z::K) tf[t & 1][m][p] = get<T>(Ts + p * Z::kBytesMap, columns.at(t, m));
        };
        ask_map(0);
        __builtin_amdgcn_sched_barrier(0);
        if (at + C < count) load(at + C);
        // R = beta (V - gamma K S), U = T R
        frag Rf[KC][Z::PARTS];
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            quad v;
            if (STATES && part)
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = (T)0.0f;
            else
                v = *reinterpret_cast<const quad*>(Vt + quad_at<T, SEQ>(16 * wave + r16, 4 * t + g));
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + 4 * g + r;
                U[t][r] = beta[i] * ((float)v[r] - gamma[i] * U[t][r]);
            }
            if (OUT) O[t] *= A.scale * gamma[16 * t + r16];
        }
#pragma unroll
        for (int m = 0; m < KC; ++m) {
            __builtin_amdgcn_sched_barrier(0);
            float xs[Z::E];
            numbers_of<T>(U, m, xs);
            parts_of<T, Z::PARTS>(xs, Rf[m]);
        }
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            if (t + 1 < CT) ask_map(t + 1);
            __builtin_amdgcn_sched_barrier(0);
            U[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int m = 0; m < KC; ++m)
                if (16 * t + 15 >= m * Z::K) U[t] = mma_parts<Z::PARTS>(tf[t & 1][m], Rf[m], U[t]);
        }
        if (!STATES && A.u_out) store_tiles<CT>(A.u_out + (chunk * A.heads + h) * (int64_t)C * DK, U, DK, g, col);
        if (OUT) {
#pragma unroll
            for (int m = 0; m < KC; ++m) {
                frag pf[2][Z::SOME];
                const int t0 = m * Z::K / 16;          // rows above this block see none of it
#pragma unroll
                for (int p = 0; p < Z::SOME; ++p) pf[0][p] = get<T>(Ps + p * Z::kBytesMap, columns.at(t0, m));
                __builtin_amdgcn_sched_barrier(0);
                float xs[Z::E];
                numbers_of<T>(U, m, xs);
                frag uf[Z::SOME];
                parts_of<T, Z::SOME>(xs, uf);
#pragma unroll
                for (int t = t0; t < CT; ++t) {
                    if (t + 1 < CT)
#pragma unroll
                        for (int p = 0; p < Z::SOME; ++p) pf[(t + 1 - t0) & 1][p] = get<T>(Ps + p * Z::kBytesMap, columns.at(t + 1, m));
                    __builtin_amdgcn_sched_barrier(0);
                    O[t] = mma_parts<Z::SOME>(uf, pf[(t - t0) & 1], O[t]);
                }
            }
            T* const out = static_cast<T*>(A.y) + row * A.ldy + (int64_t)h * A.dv;
            const int n = col0 + 16 * wave + 4 * g;
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                const int i = 16 * t + r16;
                if (i >= valid) continue;
                quad w;
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = (T)(i < bad ? O[t][r] : NAN);
                T* const to = out + i * A.ldy + n;
                if (wo) {
                    if (n < A.dv) *reinterpret_cast<quad*>(to) = w;
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (n + r < A.dv) to[r] = w[r];
                }
            }
        }
        // the state at the chunk's end; its decay in two numbers, since the same rounding in every chunk would add up
        const float d = bad < C ? NAN : whole[0], rest = whole[1];
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = fmaf(S[t][r], d, S[t][r] * rest);
#pragma unroll
        for (int m = 0; m < KC; ++m) {
            frag cf[2];
            cf[0] = get<T>(Kt, columns.at(0, m));
            cf[1] = get<T>(Kt, columns.at(1, m));
            __builtin_amdgcn_sched_barrier(0);
            float xs[Z::E];
            numbers_of<T>(U, m, xs);
#pragma unroll
            for (int e = 0; e < Z::E; ++e) xs[e] *= tail[m * Z::K + (sizeof(T) == 2 ? 16 * (e >> 2) + 4 * g + (e & 3) : 4 * g + e)];
            frag part[Z::PARTS];
            parts_of<T, Z::PARTS>(xs, part);
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                const frag k = cf[t & 1];
                if (t + 2 < DT) cf[t & 1] = get<T>(Kt, columns.at(t + 2, m));
                __builtin_amdgcn_sched_barrier(0);
                S[t] = mma_exact<Z::PARTS>(k, part, S[t]);
            }
        }
        __syncthreads();                               // the tiles may be written again
        if (x == 0) odd[turn] = C;
    }
    if (STATES) {
        float* const to = (part ? A.turned : A.added) + (s.place * A.heads + h) * (int64_t)DK * DK + col;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) to[(16 * t + 4 * g + r) * DK] = S[t][r];
    } else if (A.state_out && s.last)
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + 4 * g + r;
                if (row < A.dk && col < A.dv) A.state_out[state_at + (int64_t)row * A.dv + col] = S[t][r];
            }
}

// ----------------------------------------------------------------------------
// The walk back: the gradient G of the state, from the last chunk to the first.  Leaves G of every chunk's end, and dR.
// ----------------------------------------------------------------------------
template <typename T, int DK, int WAVES>
struct BackLds {
    typedef Sizes<T, DK> Z;
    static constexpr int COLS = 16 * WAVES;
    static constexpr int kKeysTurned = 0, kQueriesTurned = kKeysTurned + Z::kBytesTurned, kKeys = kQueriesTurned + Z::kBytesTurned;
    static constexpr int kValues = kKeys + Z::kBytesRows, kMap = kValues + COLS * Z::SEQ * 16, kP = kMap + Z::PARTS * Z::kBytesMap, kBytes = kP + Z::PARTS * Z::kBytesMap;
};

template <typename T, int DK, int WAVES, bool STATES>
__global__ void __launch_bounds__(64 * WAVES)
k_delta_back(DeltaArgs A)
{
    typedef Sizes<T, DK> Z;
    typedef BackLds<T, DK, WAVES> L;
    typedef typename Num<T>::frag frag;
    constexpr int C = Z::C, R = Z::R, ROW = Z::ROW, SEQ = Z::SEQ, CT = Z::CT, DT = Z::DT, KD = Z::KD, KC = Z::KC, THREADS = 64 * WAVES, COLS = L::COLS;
    __shared__ __attribute__((aligned(16))) char lds[L::kBytes];
    __shared__ __attribute__((aligned(16))) float beta[C], gamma[C], tail[C], whole[2];
    char *const Kt = lds + L::kKeysTurned, *const Qt = lds + L::kQueriesTurned, *const Ks = lds + L::kKeys, *const Yt = lds + L::kValues,
         *const Ts = lds + L::kMap, *const Ps = lds + L::kP;

    const int slice = blockIdx.x % A.slices, h = blockIdx.x / A.slices, col0 = slice * COLS;
    const int64_t slot = (int64_t)blockIdx.z * kRows + blockIdx.y;
    if (slot >= A.slots || col0 >= (A.dv + Z::K - 1) / Z::K * Z::K) return;
    const Stretch s = find_stretch(A, slot);
    if (!s.there || (STATES && (!s.several || s.index == 0))) return;
    const int64_t b = s.b, begin = s.begin, count = s.hi, chunk0 = first_chunk<C>(A, b, begin);
    const int x = threadIdx.x, lane = x & 63, wave = __builtin_amdgcn_readfirstlane(x >> 6), r16 = lane & 15, g = lane >> 4;
    const int kh = h / (A.heads / A.key_heads), col = col0 + 16 * wave + r16;
    for (int i = x; i < 2 * Z::PARTS * Z::kBytesMap / 16; i += THREADS) reinterpret_cast<f32x4*>(Ts)[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    f32x4 S[DT];
    float* const entering = A.added_back + (s.place * A.heads + h) * (int64_t)DK * DK + col;
    const int64_t state_at = (b * A.heads + h) * (int64_t)A.dk * A.dv;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * t + 4 * g + r;
            if (STATES) S[t][r] = 0.0f;
            else if (s.several) S[t][r] = col < A.dv ? entering[row * DK] : 0.0f;
            else S[t][r] = A.gstate_out && row < A.dk && col < A.dv ? A.gstate_out[state_at + (int64_t)row * A.dv + col] : 0.0f;
        }
    const int64_t near = INT32_MAX / (int64_t)(C * sizeof(T)) - DK;
    const bool wq = (A.wide & 1) && A.ldq < near, wk = (A.wide & 2) && A.ldk < near, wy = (A.wide & 16) && A.ldgy < near;
    constexpr int kRowPatches = (C / R) * (DK / 4), kColPatches = (C / R) * (COLS / 4);
    constexpr int NR = (kRowPatches + THREADS - 1) / THREADS, NV = (kColPatches + THREADS - 1) / THREADS, NM = (Z::TILES * 64 + THREADS - 1) / THREADS;
    Patch<T> pq[NR], pk[NR], pv[NV];
    f32x4 pt[NM], pp[NM];
    float pn[3], pw = 0.0f;
    const auto load = [&](int64_t at) {
        const int y = here(x);                         // (formed anew for each chunk, as everything below: places kept from before the loop would fill the registers)
        const int valid = (int)(count - at < C ? count - at : C);
        const int64_t row = begin + at;
        const int hq = how(wq, valid == C && A.dk == DK), hk = how(wk, valid == C && A.dk == DK), hy = how(wy, valid == C && col0 + COLS <= A.dv);
        const T* const q = static_cast<const T*>(A.q) + row * A.ldq + (int64_t)kh * A.dk;
        const T* const k = static_cast<const T*>(A.k) + row * A.ldk + (int64_t)kh * A.dk;
        const T* const gy = static_cast<const T*>(A.gy) + row * A.ldgy + (int64_t)h * A.dv;
        const float* const numbers = A.maps + ((chunk0 + at / C) * A.heads + h) * Z::kNumbers;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int p = y + i * THREADS, first = (p / (DK / 4)) * R, piece = (p % (DK / 4)) * 4;
            if (kRowPatches % THREADS == 0 || p < kRowPatches) {
                load_patch(pq[i], q, A.ldq, first, valid, piece, A.dk, hq);
                load_patch(pk[i], k, A.ldk, first, valid, piece, A.dk, hk);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = y + i * THREADS;
            if (kColPatches % THREADS == 0 || p < kColPatches)
                load_patch(pv[i], gy, A.ldgy, (p / (COLS / 4)) * R, valid, col0 + (p % (COLS / 4)) * 4, A.dv, hy);
        }
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            const int p = y + i * THREADS;
            if (Z::TILES % WAVES == 0 || i * WAVES + wave < Z::TILES) {
                pt[i] = reinterpret_cast<const f32x4*>(numbers)[p];
                pp[i] = reinterpret_cast<const f32x4*>(numbers + Z::kP)[p];
            }
        }
        if (y < C) {
#pragma unroll
            for (int i = 0; i < 3; ++i) pn[i] = numbers[Z::kBeta + i * C + y];
        }
        if (y < 2) pw = numbers[Z::kWhole + y];
    };
    const int64_t last = count > s.lo ? s.lo + (count - 1 - s.lo) / C * C : -1;
    if (last >= 0) load(last);
    __syncthreads();
    for (int64_t at = last; at >= s.lo; at -= C) {
        const int valid = (int)(count - at < C ? count - at : C);
        const int y = here(x), l = here(lane), r16 = l & 15, g = l >> 4;
        const int64_t chunk = chunk0 + at / C;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int p = y + i * THREADS, first = (p / (DK / 4)) * R, piece = p % (DK / 4);
            if (kRowPatches % THREADS == 0 || p < kRowPatches) {
                if (!(valid == C && A.dk == DK)) {
                    keep_patch(pq[i], first, valid, piece * 4, A.dk);
                    keep_patch(pk[i], first, valid, piece * 4, A.dk);
                }
                put_rows<ROW>(Ks, pk[i], first, piece);
                put_turned<T, SEQ>(Qt, pq[i], first, piece);
                put_turned<T, SEQ>(Kt, pk[i], first, piece);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = y + i * THREADS, first = (p / (COLS / 4)) * R, piece = p % (COLS / 4);
            if (kColPatches % THREADS == 0 || p < kColPatches) {
                if (!(valid == C && col0 + COLS <= A.dv)) keep_patch(pv[i], first, valid, col0 + piece * 4, A.dv);
                put_turned<T, SEQ>(Yt, pv[i], first, piece);
            }
        }
        // T and P turned: row j, tokens i along the slots
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            const int tile = i * WAVES + wave;         // (a wavefront takes a tile)
            if (Z::TILES % WAVES == 0 || tile < Z::TILES) {
                int it = 0, jt = tile;
                while (jt > it) { jt -= it + 1; ++it; }
                const int token = 16 * it + (l >> 2);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    char* const to = Ts + quad_at<T, SEQ>(16 * jt + 4 * (l & 3) + e, token >> 2) + (token & 3) * (int)sizeof(T);
                    float v = pt[i][e], w = pp[i][e];
#pragma unroll
                    for (int part = 0; part < Z::PARTS; ++part) {
                        const float up = sizeof(T) == 2 ? upper(v) : v, wp = sizeof(T) == 2 ? upper(w) : w;
                        put_number<T>(to + part * Z::kBytesMap, (T)up);
                        put_number<T>(to + (Ps - Ts) + part * Z::kBytesMap, (T)wp);
                        v -= up;
                        w -= wp;
                    }
                }
            }
        }
        if (y < C) { beta[y] = pn[0]; gamma[y] = pn[1]; tail[y] = pn[2]; }
        if (y < 2) whole[y] = pw;
        __syncthreads();
        const Reader<ROW> rows(r16, g);
        const Reader<SEQ> columns(r16, g);
        Reader<SEQ> values(r16, g);
        values.base += wave * 16 * SEQ * 16;
        values.low ^= ((2 * wave) & Reader<SEQ>::kMask) * 16;
        if (!STATES) store_tiles<DT>(A.gstates + (chunk * A.heads + h) * (int64_t)DK * DK, S, DK, g, col);
        // tail K G
        f32x4 U[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) U[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        frag kf[2][CT];
        const auto ask_rows = [&](int m) {
#pragma unroll
            for (int t = 0; t < CT; ++t) kf[m & 1][t] = get<T>(Ks, rows.at(t, m));
        };
        ask_rows(0);
#pragma unroll
        for (int m = 0; m < KD; ++m) {
            if (m + 1 < KD) ask_rows(m + 1);
            __builtin_amdgcn_sched_barrier(0);
            float xs[Z::E];
            numbers_of<T>(S, m, xs);
            frag sf[Z::PARTS];
            parts_of<T, Z::PARTS>(xs, sf);
#pragma unroll
            for (int t = 0; t < CT; ++t) U[t] = mma_exact<Z::PARTS>(kf[m & 1][t], sf, U[t]);
        }
        // a map's fragments of row t, from the blocks that hold tokens behind it
        frag tf[2][KC][Z::PARTS];
        const auto ask_map = [&](const char* map, int t) {
#pragma unroll
            for (int m = 0; m < KC; ++m)
#pragma unroll
                for (int p = 0; p < Z::PARTS; ++p)
                    if (m * Z::K + Z::K > 16 * t) tf[t & 1][m][p] = get<T>(map + p * Z::kBytesMap, columns.at(t, m));
        };
        frag yf[KC];
#pragma unroll
        for (int m = 0; m < KC; ++m) yf[m] = get<T>(Yt, values.at(0, m));
        ask_map(Ps, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (at - C >= s.lo) load(at - C);
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) U[t][r] *= tail[16 * t + 4 * g + r];
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            if (t + 1 < CT) ask_map(Ps, t + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int m = 0; m < KC; ++m)
                if (m * Z::K + Z::K > 16 * t)
#pragma unroll
                    for (int p = Z::PARTS - 1; p >= 0; --p) U[t] = mma(tf[t & 1][m][p], yf[m], U[t]);
        }
        ask_map(Ts, 0);
        // dR = T^T dU
        frag Uf[KC][Z::PARTS];
#pragma unroll
        for (int m = 0; m < KC; ++m) {
            __builtin_amdgcn_sched_barrier(0);
            float xs[Z::E];
            numbers_of<T>(U, m, xs);
            parts_of<T, Z::PARTS>(xs, Uf[m]);
        }
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            if (t + 1 < CT) ask_map(Ts, t + 1);
            __builtin_amdgcn_sched_barrier(0);
            U[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int m = 0; m < KC; ++m)
                if (m * Z::K + Z::K > 16 * t) U[t] = mma_parts<Z::PARTS>(tf[t & 1][m], Uf[m], U[t]);
        }
        if (!STATES) store_tiles<CT>(A.r_out + (chunk * A.heads + h) * (int64_t)C * DK, U, DK, g, col);
        const float d = whole[0], rest = whole[1];
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = fmaf(S[t][r], d, S[t][r] * rest);
#pragma unroll
        for (int m = 0; m < KC; ++m) {
            frag cf[2];
            cf[0] = get<T>(Qt, columns.at(0, m));
            cf[1] = get<T>(Kt, columns.at(0, m));
            __builtin_amdgcn_sched_barrier(0);
            float xs[Z::E], ys[Z::E];
            numbers_of<T>(U, m, xs);
#pragma unroll
            for (int e = 0; e < Z::E; ++e) {
                const int i = m * Z::K + (sizeof(T) == 2 ? 16 * (e >> 2) + 4 * g + (e & 3) : 4 * g + e);
                xs[e] *= -beta[i] * gamma[i];
                ys[e] = (float)yf[m][e] * (A.scale * gamma[i]);
            }
            frag rf[Z::PARTS], gf[Z::PARTS];
            parts_of<T, Z::PARTS>(xs, rf);
            parts_of<T, Z::PARTS>(ys, gf);
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                const frag q = cf[0], k = cf[1];
                if (t + 1 < DT) {
                    cf[0] = get<T>(Qt, columns.at(t + 1, m));
                    cf[1] = get<T>(Kt, columns.at(t + 1, m));
                }
                __builtin_amdgcn_sched_barrier(0);
                S[t] = mma_exact<Z::PARTS>(q, gf, S[t]);
                S[t] = mma_exact<Z::PARTS>(k, rf, S[t]);
            }
        }
        __syncthreads();
    }
    if (STATES) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) entering[(16 * t + 4 * g + r) * DK] = S[t][r];
    } else if (A.gstate_in && s.index == 0)
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + 4 * g + r;
                if (row < A.dk && col < A.dv) A.gstate_in[state_at + (int64_t)row * A.dv + col] = S[t][r];
            }
}

// ----------------------------------------------------------------------------
// The states that enter the stretches of a sequence that has several, in the places of what the stretches add: S_(n+1) = turned_n S_n + added_n from state_in on, or, back,
// G_(n-1) = turned_n^T G_n + added_n from gstate_out on.  A workgroup to 16 columns, on the fp32 matrix instructions whatever the type: a wavefront forms every fourth 16 rows, and hands them
// to the others through LDS, since a step waits for the one before (65536 tokens of 8 heads of 128, 32 steps: 204 us with 16 columns to a wavefront, 122 so).
// ----------------------------------------------------------------------------
constexpr int kCarryWaves = 4;

template <int DK, bool BACK>
__global__ void __launch_bounds__(64 * kCarryWaves)
k_delta_carry(DeltaArgs A)
{
    constexpr int DT = DK / 16, THREADS = 64 * kCarryWaves, PAD = DK + 4;
    constexpr int ROWS = DK > 192 ? 64 : DK > 128 ? 80 : DK, BLOCKS = (DK + ROWS - 1) / ROWS, N = (ROWS * DK / 4 + THREADS - 1) / THREADS;
    __shared__ __attribute__((aligned(16))) float M[ROWS * PAD];
    __shared__ f32x4 formed[DT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    // (a head's workgroups are `heads` apart: where that is a multiple of 8 they share an L2, and `turned` in it)
    const int h = blockIdx.x % A.heads, col0 = blockIdx.x / A.heads * 16, col = col0 + r16;
    const int64_t b = (int64_t)blockIdx.z * kRows + blockIdx.y;
    if (b >= A.sequences) return;
    const int64_t begin = start_of(A, b), count = count_of(A, b, begin);
    if (count <= kPays * A.stretch || col0 >= A.dv) return;
    const int64_t stretches = (count + A.stretch - 1) / A.stretch, place = first_place(A, b, begin), step = (int64_t)A.heads * DK * DK;
    const float* const given = BACK ? A.gstate_out : A.state_in;
    float* const added = (BACK ? A.added_back : A.added) + (place * A.heads + h) * (int64_t)DK * DK;
    const float* const turned = A.turned + (place * A.heads + h) * (int64_t)DK * DK;
    f32x4 S[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * t + 4 * g + r;
            S[t][r] = given && row < A.dk && col < A.dv ? given[(b * A.heads + h) * (int64_t)A.dk * A.dv + (int64_t)row * A.dv + col] : 0.0f;
        }
    // blocks of rows of `turned` go through LDS; the next one is on its way meanwhile
    f32x4 ahead[N];
    const auto ask = [&](int64_t n, int block) {
        const f32x4* const from = reinterpret_cast<const f32x4*>(turned + n * step + block * ROWS * DK);
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const int at = c * THREADS + threadIdx.x, row = at / (DK / 4), column = at % (DK / 4) * 4;
            ahead[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};  // (no workgroup has written the columns behind dk)
            if (at < ROWS * DK / 4 && block * ROWS + row < DK && column < (A.dk + 15) / 16 * 16) ahead[c] = from[at];
        }
    };
    const auto number = [&](int64_t i) { return BACK ? stretches - 1 - i : i; };
    ask(number(0), 0);
    for (int64_t i = 0; i < stretches; ++i) {
        const int64_t n = number(i);
        float* const here = added + n * step + col;
        const bool last = i + 1 == stretches;
        f32x4 next[DT];
#pragma unroll
        for (int t = 0; t < DT; ++t)
            if (t % kCarryWaves == wave)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float* const at = here + (16 * t + 4 * g + r) * DK;
                    next[t][r] = last ? 0.0f : *at;
                    *at = S[t][r];
                }
        if (last) break;
#pragma unroll
        for (int block = 0; block < BLOCKS; ++block) {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const int at = c * THREADS + threadIdx.x, row = at / (DK / 4), column = at % (DK / 4) * 4;
                if (at < ROWS * DK / 4) *reinterpret_cast<f32x4*>(&M[row * PAD + column]) = ahead[c];
            }
            __syncthreads();
            if (block + 1 < BLOCKS) ask(n, block + 1);
            else if (i + 2 < stretches) ask(number(i + 1), 0);
            // rows of the block are results ahead, what is summed over back
            if constexpr (BACK) {
#pragma unroll
                for (int c = 0; c < DT; ++c)
                    if (c % kCarryWaves == wave)
#pragma unroll
                        for (int a = 0; a < ROWS / 16; ++a) {
                            if (block * (ROWS / 16) + a >= DT) continue;
                            f32x4 f;
#pragma unroll
                            for (int r = 0; r < 4; ++r) f[r] = M[(16 * a + 4 * g + r) * PAD + 16 * c + r16];
                            next[c] = mma(f, S[block * (ROWS / 16) + a], next[c]);
                        }
            } else {
#pragma unroll
                for (int a = 0; a < ROWS / 16; ++a) {
                    const int mine = block * (ROWS / 16) + a;
                    if (mine < DT && mine % kCarryWaves == wave)
#pragma unroll
                        for (int c = 0; c < DT; ++c) next[mine] = mma(*reinterpret_cast<const f32x4*>(&M[(16 * a + r16) * PAD + 16 * c + 4 * g]), S[c], next[mine]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < DT; ++t)
            if (t % kCarryWaves == wave) formed[t][lane] = next[t];
        __syncthreads();
#pragma unroll
        for (int t = 0; t < DT; ++t) S[t] = formed[t][lane];
    }
}

// ----------------------------------------------------------------------------
// What is left of the gradients: a workgroup takes a chunk and a head of keys, a wavefront 16 numbers of a head of keys (or twice 16), and the
// heads of values that share them one after the other, so that their gradients are summed in its registers.
// With X1 = S0 gY^T, X2 = S0 dR^T, X3 = G U^T (numbers of a key x tokens) and the rows and columns of the maps:
//   dG_i = sum_j (in_ij) - sum_j (in_ji) + scale gamma_i q_i.X1_i - beta_i gamma_i k_i.X2_i - tail_i k_i.X3_i,     in = N (q k) + M (k k)
//   and, of the chunk's whole decay,  sum_i tail_i k_i.X3_i + gamma_C <S0, G>;   grates_t = -(sum_{i >= t} dG_i + that).
// ----------------------------------------------------------------------------
template <typename T, int DK>
struct GradientLds {
    typedef Sizes<T, DK> Z;
    static constexpr int kKeys = 0, kQueries = kKeys + Z::kBytesRows, kY = kQueries + Z::kBytesRows, kU = kY + Z::kBytesRows, kR = kU + Z::PARTS * Z::kBytesRows,
                         kBytes = kR + Z::PARTS * Z::kBytesRows;
    // over U and R, when they are done with
    static constexpr int kKeysTurned = kU, kQueriesTurned = kKeysTurned + Z::kBytesTurned, kN = kQueriesTurned + Z::kBytesTurned, kNt = kN + Z::SOME * Z::kBytesMap,
                         kM = kNt + Z::SOME * Z::kBytesMap, kEnd = kM + Z::SOME * Z::kBytesMap;
    static constexpr int kAll = kBytes > kEnd ? kBytes : kEnd;
};

template <typename T, int DK, int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
k_delta_gradients(DeltaArgs A)
{
    typedef Sizes<T, DK> Z;
    typedef GradientLds<T, DK> L;
    typedef typename Num<T>::frag frag;
    typedef typename Num<T>::quad quad;
    constexpr int C = Z::C, R = Z::R, ROW = Z::ROW, SEQ = Z::SEQ, CT = Z::CT, DT = Z::DT, KD = Z::KD, KC = Z::KC, THREADS = 64 * WAVES, NT = DT / WAVES;
    static_assert(DT % WAVES == 0, "every wavefront has as many tiles");
    constexpr int NM = (Z::TILES + WAVES - 1) / WAVES;
    __shared__ __attribute__((aligned(16))) char lds[L::kAll];
    __shared__ __attribute__((aligned(16))) float beta[C], gamma[C], tail[C], high[C], low[C], whole;
    __shared__ float row_in[CT][C], col_in[CT][C], row_kk[CT][C], dots[WAVES][3][C], rv[C], state_dot[WAVES];
    char *const Ks = lds + L::kKeys, *const Qs = lds + L::kQueries, *const Ys = lds + L::kY, *const Us = lds + L::kU, *const Rs = lds + L::kR;
    char *const Kt = lds + L::kKeysTurned, *const Qt = lds + L::kQueriesTurned, *const Ns = lds + L::kN, *const Nt = lds + L::kNt, *const Ms = lds + L::kM;

    const int64_t chunk = (int64_t)blockIdx.z * kRows + blockIdx.y;
    if (chunk >= A.chunks) return;
    int64_t row;
    int valid;
    find_chunk<C>(A, chunk, row, valid);
    if (valid == 0) return;
    const int x = threadIdx.x, lane = x & 63, wave = __builtin_amdgcn_readfirstlane(x >> 6), r16 = lane & 15, g = lane >> 4;
    const int kh = blockIdx.x, group = A.heads / A.key_heads, kdv = (A.dv + Z::K - 1) / Z::K;
    const int64_t near = INT32_MAX / (int64_t)(C * sizeof(T)) - DK;
    const bool wq = (A.wide & 1) && A.ldq < near, wk = (A.wide & 2) && A.ldk < near, wy = (A.wide & 16) && A.ldgy < near, wv = A.wide & 4, wg = A.wide & 128;
    const T* const q = static_cast<const T*>(A.q) + row * A.ldq + (int64_t)kh * A.dk;
    const T* const k = static_cast<const T*>(A.k) + row * A.ldk + (int64_t)kh * A.dk;
    const int hy = how(wy, valid == C && A.dv == DK), hq = how(wq, valid == C && A.dk == DK), hk = how(wk, valid == C && A.dk == DK);
    constexpr int kPatches = (C / R) * (DK / 4);
    for (int p = x; p < kPatches; p += THREADS) {
        const int piece = p % (DK / 4), first = (p / (DK / 4)) * R;
        Patch<T> a, c;
        load_patch(a, q, A.ldq, first, valid, piece * 4, A.dk, hq);
        load_patch(c, k, A.ldk, first, valid, piece * 4, A.dk, hk);
        keep_patch(a, first, valid, piece * 4, A.dk);
        keep_patch(c, first, valid, piece * 4, A.dk);
        put_rows<ROW>(Qs, a, first, piece);
        put_rows<ROW>(Ks, c, first, piece);
    }
    f32x4 gq[NT][CT], gk[NT][CT];          // numbers 16 t + 4 g .. + 3 of the key, token 16 t + r16
#pragma unroll
    for (int a = 0; a < NT; ++a)
#pragma unroll
        for (int t = 0; t < CT; ++t) gq[a][t] = gk[a][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // The rows that a head reads, all asked for at once.  (For the next head while this one's last products run they would not fit the registers.)
    constexpr int PIECES = DK <= 64 ? 16 : DK <= 128 ? 32 : 64, NP = (kPatches + THREADS - 1) / THREADS, NU = (C * PIECES + THREADS - 1) / THREADS;      // (PIECES threads of a wavefront have a token)
    constexpr int AHEAD = DK / Z::K % 4 == 0 ? 4 : DK / Z::K % 3 == 0 ? 3 : 2;   // fragments of a row of the states
    Patch<T> py[NP];
    f32x4 pu[NU], pr[NU], s4[AHEAD][Z::E / 4], g4[AHEAD][Z::E / 4];
    const auto ask_state = [&](f32x4 (&to)[AHEAD][Z::E / 4], const float* states, int64_t of, int a, int m0) {
        const float* const from = states + of * (int64_t)DK * DK + (16 * (a * WAVES + wave) + r16) * DK + 4 * g;
#pragma unroll
        for (int m = 0; m < AHEAD; ++m)
#pragma unroll
            for (int c = 0; c < Z::E / 4; ++c) {
                to[m][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};      // (behind those no workgroup of the walks has written)
                if (m0 + m < kdv) to[m][c] = *reinterpret_cast<const f32x4*>(from + (m0 + m) * Z::K + 16 * c);
            }
    };
    const auto ask = [&](int h) {
        const int64_t of = chunk * A.heads + h;
        const T* const gy = static_cast<const T*>(A.gy) + row * A.ldgy + (int64_t)h * A.dv;
        const float* const u = A.u_out + of * (int64_t)C * DK;
        const float* const dr = A.r_out + of * (int64_t)C * DK;
        const int y = here(x);
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            const int p = y + n * THREADS;
            if (kPatches % THREADS == 0 || p < kPatches) load_patch(py[n], gy, A.ldgy, (p / (DK / 4)) * R, valid, p % (DK / 4) * 4, A.dv, hy);
        }
#pragma unroll
        for (int n = 0; n < NU; ++n) {
            const int p = y + n * THREADS, at = p % PIECES * 4, i = p / PIECES;
            pu[n] = pr[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (i >= C || at >= kdv * Z::K) continue;
            pu[n] = *reinterpret_cast<const f32x4*>(u + i * DK + at);
            pr[n] = *reinterpret_cast<const f32x4*>(dr + i * DK + at);
        }
    };
    for (int e = 0; e < group; ++e) {
        const int h = kh * group + e;
        const int64_t of = chunk * A.heads + h;
        const float* const numbers = A.maps + of * Z::kNumbers;
        // (formed anew for each head: places kept from before the loop would fill the registers)
        const int x = here(threadIdx.x), lane = x & 63, r16 = lane & 15, g = lane >> 4;
        const T* const v = static_cast<const T*>(A.v) + row * A.ldv + (int64_t)h * A.dv;
        quad pv[NU];
        ask(h);
#pragma unroll
        for (int n = 0; n < NU; ++n) {
            const int p = x + n * THREADS, at = p % PIECES * 4, i = p / PIECES;
#pragma unroll
            for (int c = 0; c < 4; ++c) pv[n][c] = (T)0.0f;
            if (i >= valid || at >= A.dv) continue;
            if (wv) {
                pv[n] = *reinterpret_cast<const quad*>(v + i * A.ldv + at);
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (at + c < A.dv) pv[n][c] = v[i * A.ldv + at + c];
            }
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            const int p = x + n * THREADS, piece = p % (DK / 4), first = (p / (DK / 4)) * R;
            if (kPatches % THREADS == 0 || p < kPatches) {
                keep_patch(py[n], first, valid, piece * 4, A.dv);
                put_rows<ROW>(Ys, py[n], first, piece);
            }
        }
        // U and dR; gv, and dR . v of every token, on the way
#pragma unroll
        for (int n = 0; n < NU; ++n) {
            const int p = x + n * THREADS, piece = p % PIECES, i = p / PIECES, at = 4 * piece;
            float s = 0.0f;
            if (i < C && piece < DK / 4) {
                if (i < valid && at < A.dv) {
                    T* const gv = static_cast<T*>(A.gv) + (row + i) * A.ldgv + (int64_t)h * A.dv + at;
                    const float bi = numbers[Z::kBeta + i];
                    quad g4;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        s = fmaf(pr[n][c], (float)pv[n][c], s);
                        g4[c] = (T)(bi * pr[n][c]);
                    }
                    if (A.gv && wg) {
                        *reinterpret_cast<quad*>(gv) = g4;
                    } else if (A.gv) {
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (at + c < A.dv) gv[c] = g4[c];
                    }
                }
                put_parts<T, Z::PARTS>(Us + quad_at<T, ROW>(i, piece), Z::kBytesRows, pu[n]);
                put_parts<T, Z::PARTS>(Rs + quad_at<T, ROW>(i, piece), Z::kBytesRows, pr[n]);
            }
            for (int step = 1; step < PIECES; step <<= 1) s += __shfl_xor(s, step);
            if (piece == 0 && i < C) rv[i] = s;
        }
        ask_state(s4, A.states_out, of, 0, 0);         // (on its way while the maps are formed)
        if (x < C) {
            beta[x] = numbers[Z::kBeta + x]; gamma[x] = numbers[Z::kGamma + x]; tail[x] = numbers[Z::kTail + x];
            high[x] = numbers[Z::kHigh + x]; low[x] = numbers[Z::kLow + x];
        }
        if (x == 0) whole = numbers[Z::kWhole];
        for (int i = x; i < CT * C; i += THREADS) (&row_in[0][0])[i] = (&col_in[0][0])[i] = (&row_kk[0][0])[i] = 0.0f;
        __syncthreads();

        const Reader<ROW> rows(r16, g);
        const Reader<SEQ> columns(r16, g);
        // the maps: a lane holds rows i = 16 it + 4 g .. + 3 and column j = 16 jt + r16 of a tile
        f32x4 N[NM], M[NM];
#pragma unroll
        for (int n = 0; n < NM; ++n) {
            const int tile = n * WAVES + wave;
            int it = 0, jt = tile;
            while (jt > it) { jt -= it + 1; ++it; }
            N[n] = M[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (it >= CT) continue;
            f32x4 qk = {0.0f, 0.0f, 0.0f, 0.0f}, kk = qk;
#pragma unroll 2
            for (int m = 0; m < DK / Z::K; ++m) {
                frag uf[Z::PARTS], rf[Z::PARTS];
#pragma unroll
                for (int p = 0; p < Z::PARTS; ++p) {
                    uf[p] = get<T>(Us + p * Z::kBytesRows, rows.at(jt, m));
                    rf[p] = get<T>(Rs + p * Z::kBytesRows, rows.at(it, m));
                }
                N[n] = mma_exact<Z::PARTS>(get<T>(Ys, rows.at(it, m)), uf, N[n]);
                M[n] = mma_parts<Z::PARTS>(rf, uf, M[n]);
            }
#pragma unroll
            for (int m = 0; m < KD; ++m) {
                if (m % 2 == 0) __builtin_amdgcn_sched_barrier(0);
                const frag kf = get<T>(Ks, rows.at(jt, m));
                qk = mma(get<T>(Qs, rows.at(it, m)), kf, qk);
                kk = mma(get<T>(Ks, rows.at(it, m)), kf, kk);
            }
            const int j = 16 * jt + r16;
            float col = 0.0f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * it + 4 * g + r;
                const float d = j <= i ? decay_of(high[i], low[i], high[j], low[j]) : 0.0f;
                N[n][r] = j <= i ? A.scale * d * N[n][r] : 0.0f;
                const float bare = j < i ? -d * M[n][r] : 0.0f;
                M[n][r] = beta[i] * bare;
                float kk_sum = bare * kk[r], in = N[n][r] * qk[r] + beta[i] * kk_sum;
                col += in;
#pragma unroll
                for (int step = 1; step < 16; step <<= 1) { kk_sum += __shfl_xor(kk_sum, step); in += __shfl_xor(in, step); }
                if (r16 == 0) { row_in[jt][i] = in; row_kk[jt][i] = kk_sum; }
            }
            col += __shfl_xor(col, 16);
            col += __shfl_xor(col, 32);
            if (g == 0) col_in[it][j] = col;
        }

        // X1, X2, X3 of the wavefront's numbers of a key and the tokens, one tile of numbers after the other
        float state_sum = 0.0f, q1[CT], k2[CT], k3[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) q1[t] = k2[t] = k3[t] = 0.0f;
#pragma unroll
        for (int a = 0; a < NT; ++a) {
            const int t0 = a * WAVES + wave;
            f32x4 X1[CT], X2[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t) X1[t] = X2[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
            for (int m0 = 0; m0 < DK / Z::K; m0 += AHEAD) {
                if (a > 0 || m0 > 0) ask_state(s4, A.states_out, of, a, m0);
                ask_state(g4, A.gstates, of, a, m0);
#pragma unroll
                for (int n = 0; n < AHEAD; ++n) {
                    const int m = m0 + n;
                    float xs[Z::E];
#pragma unroll
                    for (int c = 0; c < Z::E; ++c) xs[c] = s4[n][c >> 2][c & 3];
                    frag sf[Z::PARTS];
                    parts_of<T, Z::PARTS>(xs, sf);
#pragma unroll
                    for (int t = 0; t < CT; ++t) {
                        __builtin_amdgcn_sched_barrier(0);
                        const frag yf = get<T>(Ys, rows.at(t, m));
                        frag rf[Z::PARTS];
#pragma unroll
                        for (int p = 0; p < Z::PARTS; ++p) rf[p] = get<T>(Rs + p * Z::kBytesRows, rows.at(t, m));
#pragma unroll
                        for (int p = Z::PARTS - 1; p >= 0; --p) X1[t] = mma(sf[p], yf, X1[t]);
                        X2[t] = mma_parts<Z::PARTS>(sf, rf, X2[t]);
                    }
                }
#pragma unroll
                for (int n = 0; n < AHEAD; ++n)
#pragma unroll
                    for (int c = 0; c < Z::E; ++c) state_sum = fmaf(s4[n][c >> 2][c & 3], g4[n][c >> 2][c & 3], state_sum);
            }
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                const int i = 16 * t + r16;
                const quad q4 = *reinterpret_cast<const quad*>(Qs + quad_at<T, ROW>(i, 4 * t0 + g)), k4 = *reinterpret_cast<const quad*>(Ks + quad_at<T, ROW>(i, 4 * t0 + g));
                const float c1 = A.scale * gamma[i], c2 = beta[i] * gamma[i];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    q1[t] = fmaf((float)q4[r], X1[t][r], q1[t]);
                    k2[t] = fmaf((float)k4[r], X2[t][r], k2[t]);
                    gq[a][t][r] = fmaf(c1, X1[t][r], gq[a][t][r]);
                    gk[a][t][r] = fmaf(-c2, X2[t][r], gk[a][t][r]);
                }
            }
            f32x4 X3[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t) X3[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
            for (int m0 = 0; m0 < DK / Z::K; m0 += AHEAD) {
                if (DK / Z::K > AHEAD) ask_state(g4, A.gstates, of, a, m0);
#pragma unroll
                for (int n = 0; n < AHEAD; ++n) {
                    const int m = m0 + n;
                    float xs[Z::E];
#pragma unroll
                    for (int c = 0; c < Z::E; ++c) xs[c] = g4[n][c >> 2][c & 3];
                    frag gf[Z::PARTS];
                    parts_of<T, Z::PARTS>(xs, gf);
#pragma unroll
                    for (int t = 0; t < CT; ++t) {
                        __builtin_amdgcn_sched_barrier(0);
                        frag uf[Z::PARTS];
#pragma unroll
                        for (int p = 0; p < Z::PARTS; ++p) uf[p] = get<T>(Us + p * Z::kBytesRows, rows.at(t, m));
                        X3[t] = mma_parts<Z::PARTS>(gf, uf, X3[t]);
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                const int i = 16 * t + r16;
                const quad k4 = *reinterpret_cast<const quad*>(Ks + quad_at<T, ROW>(i, 4 * t0 + g));
                const float c3 = tail[i];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    k3[t] = fmaf((float)k4[r], X3[t][r], k3[t]);
                    gk[a][t][r] = fmaf(c3, X3[t][r], gk[a][t][r]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const int i = 16 * t + r16;
#pragma unroll
            for (int step = 16; step < 64; step <<= 1) {
                q1[t] += __shfl_xor(q1[t], step);
                k2[t] += __shfl_xor(k2[t], step);
                k3[t] += __shfl_xor(k3[t], step);
            }
            if (g == 0) { dots[wave][0][i] = q1[t]; dots[wave][1][i] = k2[t]; dots[wave][2][i] = k3[t]; }
        }
        for (int step = 1; step < 64; step <<= 1) state_sum += __shfl_xor(state_sum, step);
        if (lane == 0) state_dot[wave] = state_sum;
        __syncthreads();                               // U and dR are done with

        for (int p = x; p < kPatches; p += THREADS) {
            const int piece = p % (DK / 4), first = (p / (DK / 4)) * R;
            Patch<T> a, c;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                a.r[r] = *reinterpret_cast<const quad*>(Qs + quad_at<T, ROW>(first + r, piece));
                c.r[r] = *reinterpret_cast<const quad*>(Ks + quad_at<T, ROW>(first + r, piece));
            }
            put_turned<T, SEQ>(Qt, a, first, piece);
            put_turned<T, SEQ>(Kt, c, first, piece);
        }
        for (int i = x; i < 3 * Z::SOME * Z::kBytesMap / 16; i += THREADS) reinterpret_cast<f32x4*>(Ns)[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NM; ++n) {
            const int tile = n * WAVES + wave;
            int it = 0, jt = tile;
            while (jt > it) { jt -= it + 1; ++it; }
            if (it >= CT) continue;
            const int i = 16 * it + 4 * g, j = 16 * jt + r16;
            put_parts<T, Z::SOME>(Nt + quad_at<T, SEQ>(j, i >> 2), Z::kBytesMap, N[n]);
            const auto single = [&](char* map, int r0, int token, float v) {
                char* const to = map + quad_at<T, SEQ>(r0, token >> 2) + (token & 3) * (int)sizeof(T);
                if constexpr (sizeof(T) == 4) {
                    put_number<T>(to, v);
                } else {
                    put_number<T>(to, (T)upper(v));
                    put_number<T>(to + Z::kBytesMap, (T)(v - upper(v)));
                }
            };
#pragma unroll
            for (int r = 0; r < 4; ++r) single(Ns, i + r, j, N[n][r]);
            if (it == jt) {
                // both halves of a tile on the diagonal
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (j < i + r) { single(Ms, i + r, j, M[n][r]); single(Ms, j, i + r, M[n][r]); }
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) single(Ms, i + r, j, M[n][r]);
                put_parts<T, Z::SOME>(Ms + quad_at<T, SEQ>(j, i >> 2), Z::kBytesMap, M[n]);
            }
        }
        // decays and weights of the tokens
        if (wave == 0) {
            const int i = lane < C ? lane : C - 1;
            float in = 0.0f, kk_sum = 0.0f, d1 = 0.0f, d2 = 0.0f, d3 = 0.0f, all = 0.0f;
            for (int t = 0; t < CT; ++t) {
                in += row_in[t][i];
                kk_sum += row_kk[t][i];
            }
            for (int t = 0; t < CT; ++t) in -= col_in[t][i];
            for (int w = 0; w < WAVES; ++w) {
                d1 += dots[w][0][i];
                d2 += dots[w][1][i];
                d3 += dots[w][2][i];
                all += state_dot[w];
            }
            const float late = lane < C ? tail[i] * d3 : 0.0f, taken = gamma[i] * d2;
            float dg = lane < C ? in + A.scale * gamma[i] * d1 - beta[i] * taken - late : 0.0f, lates = late;
            for (int step = 1; step < 64; step <<= 1) {
                const float other = __shfl_down(dg, step);
                if (lane + step < 64) dg += other;
                lates += __shfl_xor(lates, step);
            }
            if (lane < valid) {
                if (A.grates) A.grates[(row + lane) * A.ldgr + h] = -(dg + (lates + whole * all));
                if (A.gbeta) A.gbeta[(row + lane) * A.ldgb + h] = rv[i] - taken + kk_sum;
            }
        }
        __syncthreads();
#pragma unroll
        for (int a = 0; a < NT; ++a) {
            const int t0 = a * WAVES + wave;
#pragma unroll
            for (int m = 0; m < KC; ++m) {
                const frag kf = get<T>(Kt, columns.at(t0, m)), qf = get<T>(Qt, columns.at(t0, m));
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int p = Z::SOME - 1; p >= 0; --p) {
                        if (16 * t + 15 >= m * Z::K) gq[a][t] = mma(kf, get<T>(Ns + p * Z::kBytesMap, columns.at(t, m)), gq[a][t]);
                        if (m * Z::K + Z::K > 16 * t) gk[a][t] = mma(qf, get<T>(Nt + p * Z::kBytesMap, columns.at(t, m)), gk[a][t]);
                        gk[a][t] = mma(kf, get<T>(Ms + p * Z::kBytesMap, columns.at(t, m)), gk[a][t]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int a = 0; a < NT; ++a) {
        const int n = 16 * (a * WAVES + wave) + 4 * g;
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const int i = 16 * t + r16;
            if (i >= valid) continue;
            const auto write = [&](void* base, int64_t ld, bool wide, f32x4 v) {
                if (!base) return;
                T* const to = static_cast<T*>(base) + (row + i) * ld + (int64_t)kh * A.dk + n;
                quad w;
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = (T)v[r];
                if (wide) {
                    if (n < A.dk) *reinterpret_cast<quad*>(to) = w;
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (n + r < A.dk) to[r] = w[r];
                }
            };
            write(A.gq, A.ldgq, A.wide & 32, gq[a][t]);
            write(A.gk, A.ldgk, A.wide & 64, gk[a][t]);
        }
    }
}

// ----------------------------------------------------------------------------
// A few tokens of every sequence: the state in registers, token after token.  With e = S^T k and f = S^T q of the decayed state,
//   u = beta (v - e),   y = scale (f + (k . q) u),   S <- S + k u^T:
// both sums go over the state at once.  256 sequences of up to 5 tokens, 16 heads of 128: 124 us, 110 for the states' way through memory alone.  A workgroup takes a slice of the columns: `lanes` times VEC of them, the rest of its threads the rows.
// ----------------------------------------------------------------------------
constexpr int kTokenThreads = 256;

constexpr int kTokenBlock = 8;            // tokens whose rows are read together

template <typename T, int VEC, int DEPTH>
__global__ void __launch_bounds__(kTokenThreads, DEPTH * VEC > 32 ? 2 : DEPTH > 4 ? 4 : 5)
k_delta_tokens(DeltaArgs A, int lanes_log2, int slices)
{
    constexpr int WAVES = kTokenThreads / 64, COLS = 16 * VEC;
    __shared__ __attribute__((aligned(16))) float qs[kTokenBlock][256], ks[kTokenBlock][256], vs[kTokenBlock][COLS], high[kTokenBlock], low[kTokenBlock], weight[kTokenBlock], product[kTokenBlock];
    __shared__ float side[2][WAVES][16][2 * VEC];
    typedef float vec __attribute__((ext_vector_type(VEC), aligned(VEC == 4 ? 16 : 4)));
    const int x = threadIdx.x, lanes = 1 << lanes_log2, r0 = (x >> lanes_log2) * DEPTH, lane = x & (lanes - 1), cols = lanes * VEC;      // a thread has DEPTH rows, one behind the other
    const int h = blockIdx.x / slices, col0 = blockIdx.x % slices * cols, kh = h / (A.heads / A.key_heads), col = col0 + lane * VEC;
    const int64_t b = (int64_t)blockIdx.z * kRows + blockIdx.y;
    if (b >= A.sequences) return;
    const int64_t begin = start_of(A, b), count = count_of(A, b, begin);
    if (count == 0 && A.state_in == A.state_out) return;
    const bool live = col < A.dv;
    const int64_t at = (b * A.heads + h) * (int64_t)A.dk * A.dv + col;
    vec S[DEPTH];
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
        S[i] = vec(0.0f);
        if (A.state_in && live && r0 + i < A.dk) S[i] = *reinterpret_cast<const vec*>(A.state_in + at + (int64_t)(r0 + i) * A.dv);
    }
    for (int64_t n0 = 0; n0 < count; n0 += kTokenBlock) {
        const int some = (int)(count - n0 < kTokenBlock ? count - n0 : kTokenBlock);
        if (n0 > 0) __syncthreads();
        for (int n = 0; n < some; ++n) {
            const int64_t row = begin + n0 + n;
            if (x >= A.dk) {
                qs[n][x] = ks[n][x] = 0.0f;
            } else {
                qs[n][x] = to_float(static_cast<const T*>(A.q)[row * A.ldq + (int64_t)kh * A.dk + x]);
                ks[n][x] = to_float(static_cast<const T*>(A.k)[row * A.ldk + (int64_t)kh * A.dk + x]);
            }
            if (x < cols) vs[n][x] = col0 + x < A.dv ? to_float(static_cast<const T*>(A.v)[row * A.ldv + (int64_t)h * A.dv + col0 + x]) : 0.0f;
        }
        if (x < some) {
            // the decay in two numbers: rounded to one it could be off the same way at every token
            const int64_t row = begin + n0 + x;
            const double exact = exp(-(double)A.rates[row * A.ldr + h]);
            high[x] = (float)exact;
            low[x] = (float)(exact - (double)(float)exact);
            weight[x] = A.beta[row * A.ldb + h];
        }
        __syncthreads();
        for (int n = x >> 6; n < some; n += WAVES) {
            float p = 0.0f;
            for (int r = x & 63; r < A.dk; r += 64) p = fmaf(ks[n][r], qs[n][r], p);
            for (int step = 1; step < 64; step <<= 1) p += __shfl_xor(p, step);
            if ((x & 63) == 0) product[n] = p;
        }
#pragma unroll 1
        for (int n = 0; n < some; ++n) {
            const float hi = high[n], lo = low[n];
            float e[VEC], f[VEC], kr[DEPTH], qr[DEPTH];
#pragma unroll
            for (int i = 0; i < DEPTH; i += 4) {
                // (rows behind the last are zeros)
                const f32x4 k4 = *reinterpret_cast<const f32x4*>(&ks[n][(r0 + i) & 255]), q4 = *reinterpret_cast<const f32x4*>(&qs[n][(r0 + i) & 255]);
#pragma unroll
                for (int r = 0; r < 4; ++r) { kr[i + r] = r0 + i < 256 ? k4[r] : 0.0f; qr[i + r] = r0 + i < 256 ? q4[r] : 0.0f; }
            }
#pragma unroll
            for (int c = 0; c < VEC; ++c) e[c] = f[c] = 0.0f;
#pragma unroll
            for (int i = 0; i < DEPTH; ++i)
#pragma unroll
                for (int c = 0; c < VEC; ++c) {
                    S[i][c] = fmaf(S[i][c], hi, S[i][c] * lo);
                    e[c] = fmaf(kr[i], S[i][c], e[c]);
                    f[c] = fmaf(qr[i], S[i][c], f[c]);
                }
            for (int step = lanes; step < 64; step <<= 1)
#pragma unroll
                for (int c = 0; c < VEC; ++c) { e[c] += __shfl_xor(e[c], step); f[c] += __shfl_xor(f[c], step); }
            if ((x & 63) < lanes)
#pragma unroll
                for (int c = 0; c < VEC; ++c) { side[n & 1][x >> 6][x & 63][2 * c] = e[c]; side[n & 1][x >> 6][x & 63][2 * c + 1] = f[c]; }
            __syncthreads();
            float u[VEC];
#pragma unroll
            for (int c = 0; c < VEC; ++c) {
                float es = 0.0f, fs = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) { es += side[n & 1][w][lane][2 * c]; fs += side[n & 1][w][lane][2 * c + 1]; }
                u[c] = weight[n] * (vs[n][lane * VEC + c] - es);
                f[c] = A.scale * fmaf(product[n], u[c], fs);
            }
            if (r0 == 0 && live) {
                T* const y = static_cast<T*>(A.y) + (begin + n0 + n) * A.ldy + (int64_t)h * A.dv + col;
#pragma unroll
                for (int c = 0; c < VEC; ++c) y[c] = (T)f[c];
            }
#pragma unroll
            for (int i = 0; i < DEPTH; ++i)
#pragma unroll
                for (int c = 0; c < VEC; ++c) S[i][c] = fmaf(kr[i], u[c], S[i][c]);
        }
    }
    if (A.state_out && live)
#pragma unroll
        for (int i = 0; i < DEPTH; ++i)
            if (r0 + i < A.dk) *reinterpret_cast<vec*>(A.state_out + at + (int64_t)(r0 + i) * A.dv) = S[i];
}

// ----------------------------------------------------------------------------
// Launches.
// ----------------------------------------------------------------------------
int padded_of(int dk, int dv)
{
    const int most = dk > dv ? dk : dv;
    return most <= 64 ? 64 : most <= 96 ? 96 : most <= 128 ? 128 : most <= 192 ? 192 : 256;
}
int tokens_of_chunk(bool bf16, int padded) { return (padded > 128 ? 32 : 64) / (bf16 ? 1 : 2); }

int64_t chunks_of(int64_t tokens, int64_t sequences, int c, bool equal)
{
    return equal ? sequences * ((sequences > 0 ? tokens / sequences + c - 1 : 0) / c) : tokens / c + sequences;
}

// Sequences of no more tokens than this go token by token, where all are of equal lengths (packed ones are as long as the device's numbers say, and go in chunks).  us of
// single calls, of which one of next to no work takes 9, token by token / in chunks, heads of 128: 256 sequences of 16 heads, 2 tokens 132 / 340, 5 185 / 334, 8 241 / 334,
// 16 393 / 336; 4 sequences 10.9 / 45, 16 / 44, 21 / 44, 35 / 44.
constexpr int64_t kFewTokens = 12;

size_t aligned(size_t v) { return (v + 255) / 256 * 256; }

struct Parts { size_t maps, states, u, gstates, r, added, turned, added_back, all; };

Parts layout_of(bool bf16, int64_t chunks, int64_t places, int heads, int dk, int dv, bool training)
{
    const int d = padded_of(dk, dv), c = tokens_of_chunk(bf16, d), ct = c / 16;
    const size_t each = (size_t)chunks * heads * sizeof(float), numbers = (size_t)(ct * (ct + 1) * 256 + 5 * c + 4), state = (size_t)places * heads * d * d * sizeof(float);
    Parts L{};
    const auto take = [&](size_t bytes) { const size_t at = L.all; L.all += aligned(bytes); return at; };
    L.maps = take(each * numbers);
    L.added = take(state);
    L.turned = take(state);
    if (training) {
        L.added_back = take(state);
        L.states = take(each * d * d);
        L.u = take(each * c * d);
        L.gstates = take(each * d * d);
        L.r = take(each * c * d);
    }
    return L;
}

// How sequences are cut into stretches.
struct Cut { bool cut; int64_t stretch, per_sequence, slots, places; };

// A workgroup of a walk takes most of a compute unit's LDS, so 256 of them fill the card: us with stretches for 128 / 256 / 512, 16 heads of 128 in bf16: 1 x 65536 tokens of 8
// heads 1047 / 979 / 1145, 4 x 2048 247 / 227 / 278, 2 x 4096 for training 812 / 730 / 880; in fp32 256 / 512: 4 x 2048 437 / 471, 8 x 4096 for training 3203 / 4085.  Packed sequences of uneven
// lengths leave places, and two workgroups of fp32 numbers fit a compute unit: 256 / 512 in fp32, over four draws of the lengths: 24 sequences of 30011 tokens, 6 heads of 96 and 80, for training
// 1782 / 1690, their results alone 695 / 649; 16 of 32768, 16 heads of 128 1722 / 1550; 8 of 32768 for training 5559 / 4600; 12 of 20000, 8 heads of 64 358 / 291, for training 850 / 725; 40 of
// 50000, 4 heads of 128 901 / 888; 4 of 9000, 16 heads of 96 536 / 461; 10 of 30000, 4 heads of 256 2067 / 1717.  In bf16 16 of 32768 780 / 837, 8 of 32768 for training 2695 / 2737.
// Stretches of at least 2 / 4 / 8 chunks: 1 x 1024 123 / 112 / 132, 1 x 4096 222 / 222 / 203.
// A cut costs the maps from state to state besides, about twice the work, and pays for sequences of more than three stretches (kPays).  Cut / whole: 1 x 512 (two stretches) 99 / 82, 8 x 4096 for
// training (two) 2169 / 1958, 1 x 1024 (four) 112 / 133, 4 x 2048 (four) 231 / 248, 1 x 65536 927 / 6689.  Packed, kPays 1 / 2 / 3 over eight draws of the lengths: 24 of 30011 in fp32 for
// training 1542 / 1557 / 1598, 16 of 32768 in bf16 820 / 777 / 733: one number for both, which costs the one 4 % and gives the other 11 %.
constexpr int64_t kLeastChunks = 4;
int64_t workgroups_of(bool bf16, bool equal) { return bf16 || equal ? 256 : 512; }

// By the sizes alone: of packed sequences the kernels see which ones are long enough.
Cut cut_of(bool bf16, int64_t tokens, int64_t sequences, int heads, int dk, int dv, bool equal)
{
    const int d = padded_of(dk, dv), c = tokens_of_chunk(bf16, d), slices = d > 128 ? 2 : 1;
    const int64_t longest = equal ? (sequences > 0 ? tokens / sequences : 0) : tokens;
    const int64_t units = (int64_t)heads * slices * tokens, wanted = workgroups_of(bf16, equal);
    Cut P;
    P.stretch = ((units + wanted - 1) / wanted + c - 1) / c * c;
    if (P.stretch < kLeastChunks * c) P.stretch = kLeastChunks * c;
    P.cut = longest > kPays * P.stretch;
    if (!P.cut) P.stretch = longest + 1;               // (more than all tokens: so an empty sequence behind the last token has its place too)
    P.per_sequence = 1;
    if (equal && P.cut) P.per_sequence = (longest + P.stretch - 1) / P.stretch;
    P.slots = !P.cut ? sequences : equal ? sequences * P.per_sequence : tokens / P.stretch + sequences;
    const int64_t several = tokens / (P.stretch + 1);
    P.places = !P.cut ? 0 : equal ? P.slots : tokens / P.stretch + (sequences < several ? sequences : several);
    return P;
}

bool allows(const void* p, int64_t ld, int d, int size, int bytes)
{
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * size % bytes == 0 && d * size % bytes == 0;
}

dim3 grid_of(int64_t across, int64_t rows)
{
    const int64_t deep = (rows + kRows - 1) / kRows;
    return dim3((unsigned)across, (unsigned)(deep > 1 ? kRows : rows), (unsigned)deep);
}

enum { kRunResults, kRunKeep, kRunStates, kRunBack, kRunBackStates };

// WAVES: wavefronts of a walk's workgroup, 16 columns of the state each
template <typename T, int DK, int WAVES>
hipError_t walks_with(const DeltaArgs& A, int what, hipStream_t st)
{
    const dim3 grid = grid_of((int64_t)A.heads * A.slices, A.slots), twice = grid_of((int64_t)A.heads * A.slices * 2, A.slots), block(64 * WAVES);
    const char* const names[] = {"delta_walk", "delta_walk", "delta_states", "delta_back", "delta_back_states"};
    profile_before(names[what], st);
    if (what == kRunResults) hipLaunchKernelGGL((k_delta_walk<T, DK, WAVES, kResults>), grid, block, 0, st, A);
    else if (what == kRunKeep) hipLaunchKernelGGL((k_delta_walk<T, DK, WAVES, kKeep>), grid, block, 0, st, A);
    else if (what == kRunStates) hipLaunchKernelGGL((k_delta_walk<T, DK, WAVES, kStates>), twice, block, 0, st, A);
    else if (what == kRunBack) hipLaunchKernelGGL((k_delta_back<T, DK, WAVES, false>), grid, block, 0, st, A);
    else hipLaunchKernelGGL((k_delta_back<T, DK, WAVES, true>), grid, block, 0, st, A);
    profile_after(names[what], st);
    return hipGetLastError();
}

template <int DK>
hipError_t carry_with(const DeltaArgs& A, bool back, hipStream_t st)
{
    const dim3 grid = grid_of((int64_t)A.heads * (DK / 16), A.sequences), block(64 * kCarryWaves);
    profile_before("delta_carry", st);
    if (back) hipLaunchKernelGGL((k_delta_carry<DK, true>), grid, block, 0, st, A);
    else hipLaunchKernelGGL((k_delta_carry<DK, false>), grid, block, 0, st, A);
    profile_after("delta_carry", st);
    return hipGetLastError();
}

template <typename T, int DK, int ACROSS>
hipError_t run_with(DeltaArgs A, bool cut, hipStream_t st)
{
    const dim3 chunks = grid_of(A.key_heads, A.chunks);
    // Half as many columns of a workgroup where all compute units have room for twice the workgroups: us, half / whole columns, sequences of 128 tokens and 16 heads of 128: 4 of them
    // 41 / 49, 8 45 / 50, 12 63 / 51.
    const bool narrow = A.slots * A.heads * (DK / (16 * ACROSS)) * 2 <= 256;
    A.slices = DK / (16 * ACROSS) * (narrow ? 2 : 1);
    const auto walks = [&](int what) { return narrow ? walks_with<T, DK, ACROSS / 2>(A, what, st) : walks_with<T, DK, ACROSS>(A, what, st); };
    hipError_t e = hipSuccess;
    if (A.forward || !A.saved) {
        if (A.chunks > 0) {
            profile_before("delta_prepare", st);
            hipLaunchKernelGGL((k_delta_prepare<T, DK>), chunks, dim3(kPrepareThreads), 0, st, A);
            profile_after("delta_prepare", st);
        }
        if (cut) e = walks(kRunStates);
        if (cut && e == hipSuccess) e = carry_with<DK>(A, false, st);
        if (e == hipSuccess) e = walks(A.forward ? kRunResults : kRunKeep);
    }
    if (A.forward || e != hipSuccess) return e;
    if (cut) e = walks(kRunBackStates);
    if (cut && e == hipSuccess) e = carry_with<DK>(A, true, st);
    if (e == hipSuccess) e = walks(kRunBack);
    if (e == hipSuccess && A.chunks > 0 && (A.gq || A.gk || A.gv || A.grates || A.gbeta)) {
        profile_before("delta_gradients", st);
        hipLaunchKernelGGL((k_delta_gradients<T, DK, ACROSS>), chunks, dim3(64 * ACROSS), 0, st, A);
        profile_after("delta_gradients", st);
        e = hipGetLastError();
    }
    return e;
}

template <typename T>
hipError_t run_of(const DeltaArgs& A, bool cut, int padded, hipStream_t st)
{
    if (padded == 64) return run_with<T, 64, 4>(A, cut, st);
    if (padded == 96) return run_with<T, 96, 6>(A, cut, st);
    if (padded == 128) return run_with<T, 128, 8>(A, cut, st);
    if (padded == 192) return run_with<T, 192, 6>(A, cut, st);
    return run_with<T, 256, 8>(A, cut, st);
}

template <typename T, int VEC>
hipError_t tokens_with(const DeltaArgs& A, int lanes_log2, int slices, hipStream_t st)
{
    const dim3 grid = grid_of((int64_t)A.heads * slices, A.sequences), block(kTokenThreads);
    const int rows = kTokenThreads >> lanes_log2, depth = (A.dk + rows - 1) / rows;
    profile_before("delta_tokens", st);
    if (depth <= 4) hipLaunchKernelGGL((k_delta_tokens<T, VEC, 4>), grid, block, 0, st, A, lanes_log2, slices);
    else if (depth <= 8) hipLaunchKernelGGL((k_delta_tokens<T, VEC, 8>), grid, block, 0, st, A, lanes_log2, slices);
    else hipLaunchKernelGGL((k_delta_tokens<T, VEC, 16>), grid, block, 0, st, A, lanes_log2, slices);
    profile_after("delta_tokens", st);
    return hipGetLastError();
}

}  // namespace

// For up to so many tokens and sequences, of equal lengths or not, of heads and sizes like these.
size_t delta_workspace(bool bf16, int64_t tokens, int64_t sequences, int heads, int dk, int dv, bool training)
{
    if (heads == 0) return 0;
    // of equal lengths or packed, and cut into stretches of no fewer than so many tokens
    const int d = padded_of(dk, dv), c = tokens_of_chunk(bf16, d);
    const int64_t by_size = tokens / (kLeastChunks * c), by_work = workgroups_of(bf16, false) / ((int64_t)heads * (d > 128 ? 2 : 1)) + 1, several = by_size < by_work ? by_size : by_work;
    return layout_of(bf16, tokens / c + sequences, several > 0 ? several + (sequences < several ? sequences : several) : 0, heads, dk, dv, training).all;
}

hipError_t launch_delta_tokens(const DeltaArgs& given, hipStream_t st)
{
    DeltaArgs A = given;
    A.each = !A.starts && A.sequences > 0 ? A.tokens / A.sequences : 0;
    const bool aligned4 = A.dv % 4 == 0 && reinterpret_cast<uintptr_t>(A.state_in) % 16 == 0 && reinterpret_cast<uintptr_t>(A.state_out) % 16 == 0;
    const int vec = aligned4 ? 4 : 1, wide = (A.dv + vec - 1) / vec;
    // at most 16 lanes: 16 rows of the state for every thread then.  us with 8 / 16 lanes, 16 heads of 128: 64 sequences of 1 token 38 / 41, 128 of 1 63 / 64, 256 of 5 210 / 181.
    int lanes_log2 = 0;
    const int most = A.sequences * A.heads >= 1024 ? 4 : 3;
    while (lanes_log2 < most && (1 << lanes_log2) < wide) ++lanes_log2;
    const int slices = (wide + (1 << lanes_log2) - 1) >> lanes_log2;
    if (A.bf16) return vec == 4 ? tokens_with<__bf16, 4>(A, lanes_log2, slices, st) : tokens_with<__bf16, 1>(A, lanes_log2, slices, st);
    return vec == 4 ? tokens_with<float, 4>(A, lanes_log2, slices, st) : tokens_with<float, 1>(A, lanes_log2, slices, st);
}

hipError_t launch_delta(const DeltaArgs& given, hipStream_t st)
{
    DeltaArgs A = given;
    if (A.forward && !A.saved && !A.starts && A.tokens <= A.sequences * kFewTokens) return launch_delta_tokens(A, st);
    const int padded = padded_of(A.dk, A.dv), c = tokens_of_chunk(A.bf16, padded), size = A.bf16 ? 2 : 4;
    const bool training = !A.forward || A.saved;
    A.each = !A.starts && A.sequences > 0 ? A.tokens / A.sequences : 0;
    A.per_sequence = (A.each + c - 1) / c;
    A.chunks = chunks_of(A.tokens, A.sequences, c, A.starts == nullptr);
    const Cut P = cut_of(A.bf16, A.tokens, A.sequences, A.heads, A.dk, A.dv, A.starts == nullptr);
    A.stretch = P.stretch; A.stretches = P.per_sequence; A.slots = P.slots; A.training = training;
    const Parts L = layout_of(A.bf16, A.chunks, P.places, A.heads, A.dk, A.dv, training);
    A.maps = reinterpret_cast<float*>(A.ws + L.maps);
    A.added = reinterpret_cast<float*>(A.ws + L.added);
    A.turned = reinterpret_cast<float*>(A.ws + L.turned);
    if (training) {
        A.added_back = reinterpret_cast<float*>(A.ws + L.added_back);
        A.states_out = reinterpret_cast<float*>(A.ws + L.states);
        A.u_out = reinterpret_cast<float*>(A.ws + L.u);
        A.gstates = reinterpret_cast<float*>(A.ws + L.gstates);
        A.r_out = reinterpret_cast<float*>(A.ws + L.r);
    }
    A.wide = (allows(A.q, A.ldq, A.dk, size, 4 * size) ? 1 : 0) | (allows(A.k, A.ldk, A.dk, size, 4 * size) ? 2 : 0) | (allows(A.v, A.ldv, A.dv, size, 4 * size) ? 4 : 0) |
             (allows(A.y, A.ldy, A.dv, size, 4 * size) ? 8 : 0) | (allows(A.gy, A.ldgy, A.dv, size, 4 * size) ? 16 : 0) |
             (allows(A.gq, A.ldgq, A.dk, size, 4 * size) ? 32 : 0) | (allows(A.gk, A.ldgk, A.dk, size, 4 * size) ? 64 : 0) |
             (allows(A.gv, A.ldgv, A.dv, size, 4 * size) ? 128 : 0);
    return A.bf16 ? run_of<__bf16>(A, P.cut, padded, st) : run_of<float>(A, P.cut, padded, st);
}

}  // namespace laplex
