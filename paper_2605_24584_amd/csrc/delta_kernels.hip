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
// Four kernels.  k_delta_prepare forms T for every chunk and head, all chunks at once.  k_delta_walk goes over the chunks of a sequence with the state in
// accumulator registers: a wavefront owns 16 columns of the state, of U and of the results, and since an accumulator (a pair of them in bf16) IS a fragment of the
// next product over the same rows, neither the state nor U passes through memory on its way from product to product.  k_delta_back is the walk from the last chunk
// to the first, with the gradient of the state.  k_delta_gradients forms what is left of the gradients, all chunks at once, from the states, U, G and dR that the two
// walks have written.
//
// Numbers: sums, states and everything from which states come are fp32 numbers; in bf16 they enter products as sums of three bf16 numbers (exactly; of the nine
// products of two such sums the three below 2^-24 are left out).  What only goes into a result that is rounded to bf16 enters as two (16 bits).  The
// G_i are summed in 64 bits, since differences of far sums are what counts.
#include "token_tiles.h"

namespace laplex {

namespace {

constexpr int kPrepareThreads = 256;
constexpr int64_t kRows = 32768;          // sequences or chunks along a grid's second axis

// ----------------------------------------------------------------------------
// Sequences, and the chunks of sequences: sequence b has the chunks first_chunk(b), ...: at least as many as its rows need, whatever its length.
// ----------------------------------------------------------------------------
__device__ __forceinline__ int64_t start_of(const DeltaArgs& A, int64_t b)
{
    if (!A.starts) return A.sequences > 0 ? A.tokens / A.sequences * b : 0;
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

template <int C>
__device__ __forceinline__ int64_t first_chunk(const DeltaArgs& A, int64_t b, int64_t begin)
{
    return A.starts ? begin / C + b : b * A.per_sequence;
}

// The chunk with this number: its first row and how many rows it has (0: there is none).  By a wavefront.
template <int C>
__device__ __forceinline__ void find_chunk(const DeltaArgs& A, int64_t chunk, int64_t& row, int& valid)
{
    int64_t lo = 0;
    if (A.starts) {
        // the last sequence whose first chunk is at most this one: 64 candidates at a time
        int64_t hi = A.sequences;
        const int lane = threadIdx.x & 63;
        while (hi - lo > 1) {
            const int64_t step = (hi - lo + 63) / 64, c = lo + lane * step;
            const uint64_t votes = __ballot(c < hi && first_chunk<C>(A, c, start_of(A, c)) <= chunk);
            const int at = votes ? 63 - __builtin_clzll(votes) : 0;
            lo += at * step;
            hi = lo + step < hi ? lo + step : hi;
        }
    } else {
        lo = chunk / A.per_sequence;
    }
    const int64_t begin = start_of(A, lo), count = count_of(A, lo, begin), at = (chunk - first_chunk<C>(A, lo, begin)) * C;
    row = begin + at;
    valid = at >= 0 && at < count ? (count - at < C ? (int)(count - at) : C) : 0;
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
    // numbers of a chunk and head: T (tiles on and below the diagonal, rows of 16), then what follows
    static constexpr int kT = TILES * 256;
    static constexpr int kBeta = kT, kGamma = kT + C, kTail = kT + 2 * C, kHigh = kT + 3 * C, kLow = kT + 4 * C, kWhole = kT + 5 * C, kBad = kWhole + 2, kNumbers = kT + 5 * C + 4;
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

// The patch's columns as rows, tokens along the slots in that order.
template <typename T, int SLOTS>
__device__ __forceinline__ void put_turned(char* tile, const Patch<T>& p, int first, int piece)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        char* const at = tile + quad_at<T, SLOTS>(piece * 4 + e, first >> 2);
        if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x4*>(at) = bf16x4{p.r[0][e], p.r[1][e], p.r[2][e], p.r[3][e]};
        else *reinterpret_cast<f32x2*>(at + (first & 2) * 4) = f32x2{p.r[0][e], p.r[1][e]};
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

template <typename T>
__device__ __forceinline__ void put_number(char* at, T v) { *reinterpret_cast<T*>(at) = v; }

// A patch of R rows of four numbers, whatever their alignment; zeros in the place of those that do not exist.
template <typename T>
__device__ __forceinline__ void load_patch(Patch<T>& p, const T* base, int64_t stride, int first, int valid, int at, int width, bool wide)
{
    if (wide) load_wide<T, true>(p, base, stride, first, valid, at, width);
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
__global__ void __launch_bounds__(kPrepareThreads)
k_delta_prepare(DeltaArgs A)
{
    typedef Sizes<T, DK> Z;
    constexpr int C = Z::C, CT = Z::CT, R = Z::R, WAVES = kPrepareThreads / 64, PAD = C + 4;
    __shared__ __attribute__((aligned(16))) char Ks[Z::kBytesRows];
    __shared__ __attribute__((aligned(16))) float map[C * PAD], diagonal[CT][16][20];
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
    const bool wide = (A.wide & 2) && A.ldk < near;
    for (int p = x; p < (C / R) * (DK / 4); p += kPrepareThreads) {
        const int piece = p % (DK / 4), first = (p / (DK / 4)) * R;
        Patch<T> patch;
        load_patch(patch, k, A.ldk, first, valid, piece * 4, A.dk, wide);
        keep_patch(patch, first, valid, piece * 4, A.dk);
        if (!finite_patch(patch)) {
            atomicMin(&odd_key, first + odd_row(patch));
            clean_patch(patch);
        }
        put_rows<Z::ROW>(Ks, patch, first, piece);
    }
    __syncthreads();
    // k_i . k_j: a lane holds rows 4 g .. + 3 and column r16 of a tile
    constexpr int NT = (Z::TILES + WAVES - 1) / WAVES;
    f32x4 kk[NT];
    const Reader<Z::ROW> rows(r16, g);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int tile = n * WAVES + wave;
        int it = 0, jt = tile;
        while (jt > it) { jt -= it + 1; ++it; }
        kk[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (it < CT)
#pragma unroll
            for (int m = 0; m < Z::KD; ++m) kk[n] = mma(get<T>(Ks, rows.at(it, m)), get<T>(Ks, rows.at(jt, m)), kk[n]);
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
                    map[i * PAD + j] = j < i ? beta[i] * expf((float)(G[i] - G[j])) * kk[n][r] : 0.0f;
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

template <typename T, int DK, int WAVES, bool OUT>
__global__ void __launch_bounds__(64 * WAVES)
k_delta_walk(DeltaArgs A)
{
    typedef Sizes<T, DK> Z;
    typedef WalkLds<T, DK, WAVES, OUT> L;
    typedef typename Num<T>::frag frag;
    typedef typename Num<T>::quad quad;
    constexpr int C = Z::C, R = Z::R, ROW = Z::ROW, SEQ = Z::SEQ, CT = Z::CT, DT = Z::DT, KD = Z::KD, KC = Z::KC, THREADS = 64 * WAVES, COLS = L::COLS;
    __shared__ __attribute__((aligned(16))) char lds[L::kBytes];
    __shared__ float beta[C], gamma[C], tail[C], high[C], low[C], whole[2];
    __shared__ int odd[2];
    char *const Kt = lds + L::kTurned, *const Ts = lds + L::kMap, *const Ks = lds + L::kKeys, *const Vt = lds + L::kValues, *const Qs = lds + L::kQueries, *const Ps = lds + L::kP;

    const int slice = blockIdx.x % A.slices, h = blockIdx.x / A.slices, col0 = slice * COLS;
    const int64_t b = (int64_t)blockIdx.z * kRows + blockIdx.y;
    if (b >= A.sequences || col0 >= A.dv) return;
    const int64_t begin = start_of(A, b), count = count_of(A, b, begin), chunk0 = first_chunk<C>(A, b, begin);
    const int x = threadIdx.x, lane = x & 63, wave = __builtin_amdgcn_readfirstlane(x >> 6), r16 = lane & 15, g = lane >> 4;
    const int kh = h / (A.heads / A.key_heads), col = col0 + 16 * wave + r16;
    for (int i = x; i < Z::PARTS * Z::kBytesMap / 16; i += THREADS) reinterpret_cast<f32x4*>(Ts)[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (OUT)
        for (int i = x; i < Z::SOME * Z::kBytesMap / 16; i += THREADS) reinterpret_cast<f32x4*>(Ps)[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (x < 2) odd[x] = C;

    // the state: rows 16 t + 4 g .. + 3, column col
    f32x4 S[DT];
    const int64_t state_at = (b * A.heads + h) * (int64_t)A.dk * A.dv;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * t + 4 * g + r;
            S[t][r] = A.state_in && row < A.dk && col < A.dv ? A.state_in[state_at + (int64_t)row * A.dv + col] : 0.0f;
        }

    const int64_t near = INT32_MAX / (int64_t)(C * sizeof(T)) - DK;
    const bool wq = (A.wide & 1) && A.ldq < near, wk = (A.wide & 2) && A.ldk < near, wv = (A.wide & 4) && A.ldv < near, wo = A.wide & 8;
    constexpr int kRowPatches = (C / R) * (DK / 4), kColPatches = (C / R) * (COLS / 4);
    constexpr int NR = (kRowPatches + THREADS - 1) / THREADS, NV = (kColPatches + THREADS - 1) / THREADS, NM = (Z::TILES * 64 + THREADS - 1) / THREADS;
    Patch<T> pq[NR], pk[NR], pv[NV];
    f32x4 pt[NM];
    float pn[5], pw = 0.0f;
    int pb = C;
    const auto load = [&](int64_t at) {
        const int valid = (int)(count - at < C ? count - at : C);
        const int64_t row = begin + at;
        const T* const q = static_cast<const T*>(A.q) + row * A.ldq + (int64_t)kh * A.dk;
        const T* const k = static_cast<const T*>(A.k) + row * A.ldk + (int64_t)kh * A.dk;
        const T* const v = static_cast<const T*>(A.v) + row * A.ldv + (int64_t)h * A.dv;
        const float* const numbers = A.maps + ((chunk0 + at / C) * A.heads + h) * Z::kNumbers;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int p = x + i * THREADS, first = (p / (DK / 4)) * R, piece = (p % (DK / 4)) * 4;
            if (kRowPatches % THREADS == 0 || p < kRowPatches) {
                if (OUT) load_patch(pq[i], q, A.ldq, first, valid, piece, A.dk, wq);
                load_patch(pk[i], k, A.ldk, first, valid, piece, A.dk, wk);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = x + i * THREADS;
            if (kColPatches % THREADS == 0 || p < kColPatches)
                load_patch(pv[i], v, A.ldv, (p / (COLS / 4)) * R, valid, col0 + (p % (COLS / 4)) * 4, A.dv, wv);
        }
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            const int p = x + i * THREADS;
            if ((Z::TILES * 64) % THREADS == 0 || p < Z::TILES * 64) pt[i] = reinterpret_cast<const f32x4*>(numbers)[p];
        }
        if (x < C) {
#pragma unroll
            for (int i = 0; i < 5; ++i) pn[i] = numbers[Z::kBeta + i * C + x];
        }
        if (x < 2) pw = numbers[Z::kWhole + x];
        if (x == 0) pb = reinterpret_cast<const int*>(numbers)[Z::kBad];
    };
    if (count > 0) load(0);
    __syncthreads();

    int turn = 0;
    for (int64_t at = 0; at < count; at += C, turn ^= 1) {
        const int valid = (int)(count - at < C ? count - at : C);
        const int64_t row = begin + at, chunk = chunk0 + at / C;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int p = x + i * THREADS, first = (p / (DK / 4)) * R, piece = p % (DK / 4);
            if (kRowPatches % THREADS == 0 || p < kRowPatches) {
                if (OUT) {
                    keep_patch(pq[i], first, valid, piece * 4, A.dk);
                    put_rows<ROW>(Qs, pq[i], first, piece);
                }
                keep_patch(pk[i], first, valid, piece * 4, A.dk);
                if (!finite_patch(pk[i])) clean_patch(pk[i]);
                put_rows<ROW>(Ks, pk[i], first, piece);
                put_turned<T, SEQ>(Kt, pk[i], first, piece);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = x + i * THREADS, first = (p / (COLS / 4)) * R, piece = p % (COLS / 4);
            if (kColPatches % THREADS == 0 || p < kColPatches) {
                keep_patch(pv[i], first, valid, col0 + piece * 4, A.dv);
                if (!finite_patch(pv[i])) {
                    atomicMin(&odd[turn], first + odd_row(pv[i]));
                    clean_patch(pv[i]);
                }
                put_turned<T, SEQ>(Vt, pv[i], first, piece);
            }
        }
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            const int p = x + i * THREADS;
            if ((Z::TILES * 64) % THREADS == 0 || p < Z::TILES * 64) {
                const int tile = p >> 6;
                int it = 0, jt = tile;
                while (jt > it) { jt -= it + 1; ++it; }
                put_parts<T, Z::PARTS>(Ts + quad_at<T, SEQ>(16 * it + ((p & 63) >> 2), 4 * jt + (p & 3)), Z::kBytesMap, pt[i]);
            }
        }
        if (x < C) { beta[x] = pn[0]; gamma[x] = pn[1]; tail[x] = pn[2]; high[x] = pn[3]; low[x] = pn[4]; }
        if (x < 2) whole[x] = pw;
        if (x == 0 && pb < C) atomicMin(&odd[turn], pb);
        if (at + C < count) load(at + C);
        __syncthreads();

        const int bad = odd[turn];                     // from this token on there is nothing but NaN
        const Reader<ROW> rows(r16, g);
        const Reader<SEQ> columns(r16, g);
        if (A.states_out) {
            float* const to = A.states_out + (chunk * A.heads + h) * (int64_t)DK * DK + col;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) to[(16 * t + 4 * g + r) * DK] = S[t][r];
        }
        if (OUT) {
            // P, tiles on and below the diagonal dealt to the wavefronts: a lane holds P[i][j .. j + 3]
#pragma unroll
            for (int n = 0; n < (Z::TILES + WAVES - 1) / WAVES; ++n) {
                const int tile = n * WAVES + wave;
                int it = 0, jt = tile;
                while (jt > it) { jt -= it + 1; ++it; }
                if (it < CT) {
                    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int m = 0; m < KD; ++m) acc = mma(get<T>(Ks, rows.at(jt, m)), get<T>(Qs, rows.at(it, m)), acc);
                    const int i = 16 * it + r16, j = 16 * jt + 4 * g;
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[r] = j + r <= i ? acc[r] * decay_of(high[i], low[i], high[j + r], low[j + r]) : 0.0f;
                    put_parts<T, Z::SOME>(Ps + quad_at<T, SEQ>(i, j >> 2), Z::kBytesMap, acc);
                }
            }
        }
        f32x4 U[CT], O[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) U[t] = O[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        // K S and Q S: rows of tokens 16 t + 4 g .. + 3, column col, of the one, the other way round of the other
#pragma unroll
        for (int m = 0; m < KD; ++m) {
            float xs[Z::E];
            numbers_of<T>(S, m, xs);
            frag sf[Z::PARTS];
            parts_of<T, Z::PARTS>(xs, sf);
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                U[t] = mma_exact<Z::PARTS>(get<T>(Ks, rows.at(t, m)), sf, U[t]);
                if (OUT) {
                    const frag qf = get<T>(Qs, rows.at(t, m));
#pragma unroll
                    for (int p = Z::SOME - 1; p >= 0; --p) O[t] = mma(sf[p], qf, O[t]);
                }
            }
        }
        // R = beta (V - gamma K S), U = T R
        frag Rf[KC][Z::PARTS];
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            const quad v = *reinterpret_cast<const quad*>(Vt + quad_at<T, SEQ>(16 * wave + r16, 4 * t + g));
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + 4 * g + r;
                U[t][r] = beta[i] * ((float)v[r] - gamma[i] * U[t][r]);
            }
            if (OUT) O[t] *= gamma[16 * t + r16];
        }
#pragma unroll
        for (int m = 0; m < KC; ++m) {
            float xs[Z::E];
            numbers_of<T>(U, m, xs);
            parts_of<T, Z::PARTS>(xs, Rf[m]);
        }
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            U[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int m = 0; m < KC; ++m)
                if (16 * t + 15 >= m * Z::K) {
                    frag tf[Z::PARTS];
#pragma unroll
                    for (int p = 0; p < Z::PARTS; ++p) tf[p] = get<T>(Ts + p * Z::kBytesMap, columns.at(t, m));
                    U[t] = mma_parts<Z::PARTS>(tf, Rf[m], U[t]);
                }
        }
        if (A.u_out) {
            float* const to = A.u_out + (chunk * A.heads + h) * (int64_t)C * DK + col;
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) to[(16 * t + 4 * g + r) * DK] = U[t][r];
        }
        if (OUT) {
            __syncthreads();                           // P is there
#pragma unroll
            for (int m = 0; m < KC; ++m) {
                float xs[Z::E];
                numbers_of<T>(U, m, xs);
                frag uf[Z::SOME];
                parts_of<T, Z::SOME>(xs, uf);
#pragma unroll
                for (int t = 0; t < CT; ++t)
                    if (16 * t + 15 >= m * Z::K) {
                        frag pf[Z::SOME];
#pragma unroll
                        for (int p = 0; p < Z::SOME; ++p) pf[p] = get<T>(Ps + p * Z::kBytesMap, columns.at(t, m));
                        O[t] = mma_parts<Z::SOME>(uf, pf, O[t]);
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
                for (int r = 0; r < 4; ++r) w[r] = (T)(i < bad ? O[t][r] * A.scale : NAN);
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
        const float d = whole[0], rest = whole[1];
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = bad < C ? NAN : fmaf(S[t][r], d, S[t][r] * rest);
#pragma unroll
        for (int m = 0; m < KC; ++m) {
            float xs[Z::E];
            numbers_of<T>(U, m, xs);
#pragma unroll
            for (int e = 0; e < Z::E; ++e) xs[e] *= tail[m * Z::K + (sizeof(T) == 2 ? 16 * (e >> 2) + 4 * g + (e & 3) : 4 * g + e)];
            frag part[Z::PARTS];
            parts_of<T, Z::PARTS>(xs, part);
#pragma unroll
            for (int t = 0; t < DT; ++t) S[t] = mma_exact<Z::PARTS>(get<T>(Kt, columns.at(t, m)), part, S[t]);
        }
        __syncthreads();                               // the tiles may be written again
        if (x == 0) odd[turn] = C;
    }
    if (A.state_out)
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
    static constexpr int kKeysTurned = 0, kQueriesTurned = kKeysTurned + Z::kBytesTurned, kKeys = kQueriesTurned + Z::kBytesTurned, kQueries = kKeys + Z::kBytesRows;
    static constexpr int kValues = kQueries + Z::kBytesRows, kMap = kValues + COLS * Z::SEQ * 16, kP = kMap + Z::PARTS * Z::kBytesMap, kBytes = kP + Z::PARTS * Z::kBytesMap;
};

template <typename T, int DK, int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
k_delta_back(DeltaArgs A)
{
    typedef Sizes<T, DK> Z;
    typedef BackLds<T, DK, WAVES> L;
    typedef typename Num<T>::frag frag;
    constexpr int C = Z::C, R = Z::R, ROW = Z::ROW, SEQ = Z::SEQ, CT = Z::CT, DT = Z::DT, KD = Z::KD, KC = Z::KC, THREADS = 64 * WAVES, COLS = L::COLS;
    __shared__ __attribute__((aligned(16))) char lds[L::kBytes];
    __shared__ float beta[C], gamma[C], tail[C], high[C], low[C], whole[2];
    char *const Kt = lds + L::kKeysTurned, *const Qt = lds + L::kQueriesTurned, *const Ks = lds + L::kKeys, *const Qs = lds + L::kQueries, *const Yt = lds + L::kValues,
         *const Ts = lds + L::kMap, *const Ps = lds + L::kP;

    const int slice = blockIdx.x % A.slices, h = blockIdx.x / A.slices, col0 = slice * COLS;
    const int64_t b = (int64_t)blockIdx.z * kRows + blockIdx.y;
    if (b >= A.sequences || col0 >= A.dv) return;
    const int64_t begin = start_of(A, b), count = count_of(A, b, begin), chunk0 = first_chunk<C>(A, b, begin);
    const int x = threadIdx.x, lane = x & 63, wave = __builtin_amdgcn_readfirstlane(x >> 6), r16 = lane & 15, g = lane >> 4;
    const int kh = h / (A.heads / A.key_heads), col = col0 + 16 * wave + r16;
    for (int i = x; i < 2 * Z::PARTS * Z::kBytesMap / 16; i += THREADS) reinterpret_cast<f32x4*>(Ts)[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    f32x4 S[DT];
    const int64_t state_at = (b * A.heads + h) * (int64_t)A.dk * A.dv;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * t + 4 * g + r;
            S[t][r] = A.gstate_out && row < A.dk && col < A.dv ? A.gstate_out[state_at + (int64_t)row * A.dv + col] : 0.0f;
        }
    const int64_t near = INT32_MAX / (int64_t)(C * sizeof(T)) - DK;
    const bool wq = (A.wide & 1) && A.ldq < near, wk = (A.wide & 2) && A.ldk < near, wy = (A.wide & 16) && A.ldgy < near;
    constexpr int kRowPatches = (C / R) * (DK / 4), kColPatches = (C / R) * (COLS / 4);
    constexpr int NR = (kRowPatches + THREADS - 1) / THREADS, NV = (kColPatches + THREADS - 1) / THREADS, NM = (Z::TILES * 64 + THREADS - 1) / THREADS;
    Patch<T> pq[NR], pk[NR], pv[NV];
    f32x4 pt[NM];
    float pn[5], pw = 0.0f;
    const auto load = [&](int64_t at) {
        const int valid = (int)(count - at < C ? count - at : C);
        const int64_t row = begin + at;
        const T* const q = static_cast<const T*>(A.q) + row * A.ldq + (int64_t)kh * A.dk;
        const T* const k = static_cast<const T*>(A.k) + row * A.ldk + (int64_t)kh * A.dk;
        const T* const gy = static_cast<const T*>(A.gy) + row * A.ldgy + (int64_t)h * A.dv;
        const float* const numbers = A.maps + ((chunk0 + at / C) * A.heads + h) * Z::kNumbers;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int p = x + i * THREADS, first = (p / (DK / 4)) * R, piece = (p % (DK / 4)) * 4;
            if (kRowPatches % THREADS == 0 || p < kRowPatches) {
                load_patch(pq[i], q, A.ldq, first, valid, piece, A.dk, wq);
                load_patch(pk[i], k, A.ldk, first, valid, piece, A.dk, wk);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = x + i * THREADS;
            if (kColPatches % THREADS == 0 || p < kColPatches)
                load_patch(pv[i], gy, A.ldgy, (p / (COLS / 4)) * R, valid, col0 + (p % (COLS / 4)) * 4, A.dv, wy);
        }
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            const int p = x + i * THREADS;
            if ((Z::TILES * 64) % THREADS == 0 || p < Z::TILES * 64) pt[i] = reinterpret_cast<const f32x4*>(numbers)[p];
        }
        if (x < C) {
#pragma unroll
            for (int i = 0; i < 5; ++i) pn[i] = numbers[Z::kBeta + i * C + x];
        }
        if (x < 2) pw = numbers[Z::kWhole + x];
    };
    const int64_t last = count > 0 ? (count - 1) / C * C : -1;
    if (count > 0) load(last);
    __syncthreads();
    for (int64_t at = last; at >= 0; at -= C) {
        const int valid = (int)(count - at < C ? count - at : C);
        const int64_t chunk = chunk0 + at / C;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int p = x + i * THREADS, first = (p / (DK / 4)) * R, piece = p % (DK / 4);
            if (kRowPatches % THREADS == 0 || p < kRowPatches) {
                keep_patch(pq[i], first, valid, piece * 4, A.dk);
                keep_patch(pk[i], first, valid, piece * 4, A.dk);
                put_rows<ROW>(Qs, pq[i], first, piece);
                put_rows<ROW>(Ks, pk[i], first, piece);
                put_turned<T, SEQ>(Qt, pq[i], first, piece);
                put_turned<T, SEQ>(Kt, pk[i], first, piece);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = x + i * THREADS, first = (p / (COLS / 4)) * R, piece = p % (COLS / 4);
            if (kColPatches % THREADS == 0 || p < kColPatches) {
                keep_patch(pv[i], first, valid, col0 + piece * 4, A.dv);
                put_turned<T, SEQ>(Yt, pv[i], first, piece);
            }
        }
        // T turned: row j, tokens i along the slots
#pragma unroll
        for (int i = 0; i < NM; ++i) {
            const int p = x + i * THREADS;
            if ((Z::TILES * 64) % THREADS == 0 || p < Z::TILES * 64) {
                const int tile = p >> 6;
                int it = 0, jt = tile;
                while (jt > it) { jt -= it + 1; ++it; }
                const int token = 16 * it + ((p & 63) >> 2);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    char* const to = Ts + quad_at<T, SEQ>(16 * jt + 4 * (p & 3) + e, token >> 2) + (token & 3) * (int)sizeof(T);
                    float v = pt[i][e];
#pragma unroll
                    for (int part = 0; part < Z::PARTS; ++part) {
                        const float up = sizeof(T) == 2 ? upper(v) : v;
                        put_number<T>(to + part * Z::kBytesMap, (T)up);
                        v -= up;
                    }
                }
            }
        }
        if (x < C) { beta[x] = pn[0]; gamma[x] = pn[1]; tail[x] = pn[2]; high[x] = pn[3]; low[x] = pn[4]; }
        if (x < 2) whole[x] = pw;
        if (at >= C) load(at - C);
        __syncthreads();
        const Reader<ROW> rows(r16, g);
        const Reader<SEQ> columns(r16, g);
        Reader<SEQ> values(r16, g);
        values.base += wave * 16 * SEQ * 16;
        values.low ^= ((2 * wave) & Reader<SEQ>::kMask) * 16;
        float* const to_state = A.gstates + (chunk * A.heads + h) * (int64_t)DK * DK + col;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) to_state[(16 * t + 4 * g + r) * DK] = S[t][r];
        // P turned: row j, four tokens i
#pragma unroll
        for (int n = 0; n < (Z::TILES + WAVES - 1) / WAVES; ++n) {
            const int tile = n * WAVES + wave;
            int it = 0, jt = tile;
            while (jt > it) { jt -= it + 1; ++it; }
            if (it < CT) {
                f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int m = 0; m < KD; ++m) acc = mma(get<T>(Qs, rows.at(it, m)), get<T>(Ks, rows.at(jt, m)), acc);
                const int i = 16 * it + 4 * g, j = 16 * jt + r16;
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[r] = j <= i + r ? acc[r] * A.scale * decay_of(high[i + r], low[i + r], high[j], low[j]) : 0.0f;
                put_parts<T, Z::PARTS>(Ps + quad_at<T, SEQ>(j, i >> 2), Z::kBytesMap, acc);
            }
        }
        // tail K G
        f32x4 U[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) U[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int m = 0; m < KD; ++m) {
            float xs[Z::E];
            numbers_of<T>(S, m, xs);
            frag sf[Z::PARTS];
            parts_of<T, Z::PARTS>(xs, sf);
#pragma unroll
            for (int t = 0; t < CT; ++t) U[t] = mma_exact<Z::PARTS>(get<T>(Ks, rows.at(t, m)), sf, U[t]);
        }
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) U[t][r] *= tail[16 * t + 4 * g + r];
        __syncthreads();                               // P is there
#pragma unroll
        for (int m = 0; m < KC; ++m) {
            const frag yf = get<T>(Yt, values.at(0, m));
#pragma unroll
            for (int t = 0; t < CT; ++t)
                if (m * Z::K + Z::K > 16 * t)
#pragma unroll
                    for (int p = Z::PARTS - 1; p >= 0; --p) U[t] = mma(get<T>(Ps + p * Z::kBytesMap, columns.at(t, m)), yf, U[t]);
        }
        // dR = T^T dU
        frag Uf[KC][Z::PARTS];
#pragma unroll
        for (int m = 0; m < KC; ++m) {
            float xs[Z::E];
            numbers_of<T>(U, m, xs);
            parts_of<T, Z::PARTS>(xs, Uf[m]);
        }
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            U[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int m = 0; m < KC; ++m)
                if (m * Z::K + Z::K > 16 * t) {
                    frag tf[Z::PARTS];
#pragma unroll
                    for (int p = 0; p < Z::PARTS; ++p) tf[p] = get<T>(Ts + p * Z::kBytesMap, columns.at(t, m));
                    U[t] = mma_parts<Z::PARTS>(tf, Uf[m], U[t]);
                }
        }
        float* const to_r = A.r_out + (chunk * A.heads + h) * (int64_t)C * DK + col;
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) to_r[(16 * t + 4 * g + r) * DK] = U[t][r];
        const float d = whole[0], rest = whole[1];
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = fmaf(S[t][r], d, S[t][r] * rest);
#pragma unroll
        for (int m = 0; m < KC; ++m) {
            const frag yf = get<T>(Yt, values.at(0, m));
            float xs[Z::E], ys[Z::E];
            numbers_of<T>(U, m, xs);
#pragma unroll
            for (int e = 0; e < Z::E; ++e) {
                const int i = m * Z::K + (sizeof(T) == 2 ? 16 * (e >> 2) + 4 * g + (e & 3) : 4 * g + e);
                xs[e] *= -beta[i] * gamma[i];
                ys[e] = (float)yf[e] * (A.scale * gamma[i]);
            }
            frag rf[Z::PARTS], gf[Z::PARTS];
            parts_of<T, Z::PARTS>(xs, rf);
            parts_of<T, Z::PARTS>(ys, gf);
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                S[t] = mma_exact<Z::PARTS>(get<T>(Qt, columns.at(t, m)), gf, S[t]);
                S[t] = mma_exact<Z::PARTS>(get<T>(Kt, columns.at(t, m)), rf, S[t]);
            }
        }
        __syncthreads();
    }
    if (A.gstate_in)
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + 4 * g + r;
                if (row < A.dk && col < A.dv) A.gstate_in[state_at + (int64_t)row * A.dv + col] = S[t][r];
            }
}

// ----------------------------------------------------------------------------
// What is left of the gradients: a workgroup takes a chunk and a head of keys, a wavefront 16 numbers of a head of keys (or twice 16), and the heads of values
// that share them one after the other, so that their gradients are summed in its registers.
// With X1 = S0 gY^T, X2 = S0 dR^T, X3 = G U^T (numbers of a key x tokens) and the rows and columns of the maps:
//   dG_i = sum_j (in_ij) - sum_j (in_ji) + scale gamma_i q_i.X1_i - beta_i gamma_i k_i.X2_i - tail_i k_i.X3_i,     in = N (q k) + M (k k)
//   and, of the chunk's whole decay,  sum_i tail_i k_i.X3_i + gamma_C <S0, G>;   grates_t = -(sum_{i >= t} dG_i + that).
// ----------------------------------------------------------------------------
template <typename T, int DK, int WAVES>
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
    typedef GradientLds<T, DK, WAVES> L;
    typedef typename Num<T>::frag frag;
    typedef typename Num<T>::quad quad;
    constexpr int C = Z::C, R = Z::R, ROW = Z::ROW, SEQ = Z::SEQ, CT = Z::CT, DT = Z::DT, KD = Z::KD, KC = Z::KC, THREADS = 64 * WAVES, NT = DT / WAVES;
    static_assert(DT % WAVES == 0, "every wavefront has as many tiles");
    constexpr int NM = (Z::TILES + WAVES - 1) / WAVES;
    __shared__ __attribute__((aligned(16))) char lds[L::kAll];
    __shared__ float beta[C], gamma[C], tail[C], high[C], low[C], whole;
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
    const bool wq = (A.wide & 1) && A.ldq < near, wk = (A.wide & 2) && A.ldk < near, wy = (A.wide & 16) && A.ldgy < near;
    const T* const q = static_cast<const T*>(A.q) + row * A.ldq + (int64_t)kh * A.dk;
    const T* const k = static_cast<const T*>(A.k) + row * A.ldk + (int64_t)kh * A.dk;
    constexpr int kPatches = (C / R) * (DK / 4);
    for (int p = x; p < kPatches; p += THREADS) {
        const int piece = p % (DK / 4), first = (p / (DK / 4)) * R;
        Patch<T> a, c;
        load_patch(a, q, A.ldq, first, valid, piece * 4, A.dk, wq);
        load_patch(c, k, A.ldk, first, valid, piece * 4, A.dk, wk);
        keep_patch(a, first, valid, piece * 4, A.dk);
        keep_patch(c, first, valid, piece * 4, A.dk);
        put_rows<ROW>(Qs, a, first, piece);
        put_rows<ROW>(Ks, c, first, piece);
    }
    const Reader<ROW> rows(r16, g);
    const Reader<SEQ> columns(r16, g);
    f32x4 gq[NT][CT], gk[NT][CT];          // numbers 16 t + 4 g .. + 3 of the key, token 16 tt + r16
#pragma unroll
    for (int a = 0; a < NT; ++a)
#pragma unroll
        for (int t = 0; t < CT; ++t) gq[a][t] = gk[a][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    for (int e = 0; e < group; ++e) {
        const int h = kh * group + e;
        const int64_t of = chunk * A.heads + h;
        const T* const gy = static_cast<const T*>(A.gy) + row * A.ldgy + (int64_t)h * A.dv;
        const float* const numbers = A.maps + of * Z::kNumbers;
        const float* const u = A.u_out + of * (int64_t)C * DK;
        const float* const dr = A.r_out + of * (int64_t)C * DK;
        __syncthreads();
        for (int p = x; p < kPatches; p += THREADS) {
            const int piece = p % (DK / 4), first = (p / (DK / 4)) * R;
            Patch<T> a;
            load_patch(a, gy, A.ldgy, first, valid, piece * 4, A.dv, wy);
            keep_patch(a, first, valid, piece * 4, A.dv);
            put_rows<ROW>(Ys, a, first, piece);
        }
        for (int p = x; p < C * DK / 4; p += THREADS) {
            const int piece = p % (DK / 4), i = p / (DK / 4);
            if (piece * 4 >= kdv * Z::K) continue;     // (columns that no workgroup of the walks has written)
            put_parts<T, Z::PARTS>(Us + quad_at<T, ROW>(i, piece), Z::kBytesRows, *reinterpret_cast<const f32x4*>(u + i * DK + piece * 4));
            put_parts<T, Z::PARTS>(Rs + quad_at<T, ROW>(i, piece), Z::kBytesRows, *reinterpret_cast<const f32x4*>(dr + i * DK + piece * 4));
        }
        if (x < C) {
            beta[x] = numbers[Z::kBeta + x]; gamma[x] = numbers[Z::kGamma + x]; tail[x] = numbers[Z::kTail + x];
            high[x] = numbers[Z::kHigh + x]; low[x] = numbers[Z::kLow + x];
        }
        if (x == 0) whole = numbers[Z::kWhole];
        for (int i = x; i < CT * C; i += THREADS) (&row_in[0][0])[i] = (&col_in[0][0])[i] = (&row_kk[0][0])[i] = 0.0f;
        // gv, and dR . v of every token
        for (int i = wave; i < valid; i += WAVES) {
            const T* const v = static_cast<const T*>(A.v) + (row + i) * A.ldv + (int64_t)h * A.dv;
            T* const gv = A.gv ? static_cast<T*>(A.gv) + (row + i) * A.ldgv + (int64_t)h * A.dv : nullptr;
            const float bi = numbers[Z::kBeta + i];
            float s = 0.0f;
            for (int c = lane; c < A.dv; c += 64) {
                const float r = dr[i * DK + c];
                s = fmaf(r, to_float(v[c]), s);
                if (gv) gv[c] = (T)(bi * r);
            }
            for (int step = 1; step < 64; step <<= 1) s += __shfl_xor(s, step);
            if (lane == 0) rv[i] = s;
        }
        __syncthreads();

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
            for (int m = 0; m < kdv; ++m) {
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

        // X1, X2, X3 of the wavefront's numbers of a key, one tile after the other
        float state_sum = 0.0f, q1[CT], k2[CT], k3[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) q1[t] = k2[t] = k3[t] = 0.0f;
#pragma unroll
        for (int a = 0; a < NT; ++a) {
            const int t0 = a * WAVES + wave;
            f32x4 X1[CT], X2[CT], X3[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t) X1[t] = X2[t] = X3[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            const float* const s0 = A.states_out + of * (int64_t)DK * DK + (16 * t0 + r16) * DK;
            const float* const gs = A.gstates + of * (int64_t)DK * DK + (16 * t0 + r16) * DK;
            for (int m = 0; m < kdv; ++m) {
                float xs[Z::E], ys[Z::E];
#pragma unroll
                for (int c = 0; c < Z::E; c += 4) {
                    const int at = m * Z::K + 4 * c + 4 * g;
                    const f32x4 a4 = *reinterpret_cast<const f32x4*>(s0 + at), b4 = *reinterpret_cast<const f32x4*>(gs + at);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        xs[c + r] = a4[r];
                        ys[c + r] = b4[r];
                        state_sum = fmaf(a4[r], b4[r], state_sum);
                    }
                }
                frag sf[Z::PARTS], gf[Z::PARTS];
                parts_of<T, Z::PARTS>(xs, sf);
                parts_of<T, Z::PARTS>(ys, gf);
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    const frag yf = get<T>(Ys, rows.at(t, m));
#pragma unroll
                    for (int p = Z::PARTS - 1; p >= 0; --p) X1[t] = mma(sf[p], yf, X1[t]);
                    frag uf[Z::PARTS], rf[Z::PARTS];
#pragma unroll
                    for (int p = 0; p < Z::PARTS; ++p) {
                        uf[p] = get<T>(Us + p * Z::kBytesRows, rows.at(t, m));
                        rf[p] = get<T>(Rs + p * Z::kBytesRows, rows.at(t, m));
                    }
                    X2[t] = mma_parts<Z::PARTS>(sf, rf, X2[t]);
                    X3[t] = mma_parts<Z::PARTS>(gf, uf, X3[t]);
                }
            }
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                const int i = 16 * t + r16;
                const quad q4 = *reinterpret_cast<const quad*>(Qs + quad_at<T, ROW>(i, 4 * t0 + g)), k4 = *reinterpret_cast<const quad*>(Ks + quad_at<T, ROW>(i, 4 * t0 + g));
                const float c1 = A.scale * gamma[i], c2 = beta[i] * gamma[i], c3 = tail[i];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    q1[t] = fmaf((float)q4[r], X1[t][r], q1[t]);
                    k2[t] = fmaf((float)k4[r], X2[t][r], k2[t]);
                    k3[t] = fmaf((float)k4[r], X3[t][r], k3[t]);
                    gq[a][t][r] = fmaf(c1, X1[t][r], gq[a][t][r]);
                    gk[a][t][r] = fmaf(-c2, X2[t][r], fmaf(c3, X3[t][r], gk[a][t][r]));
                }
            }
        }
#pragma unroll
        for (int t = 0; t < CT; ++t) {
#pragma unroll
            for (int step = 16; step < 64; step <<= 1) {
                q1[t] += __shfl_xor(q1[t], step);
                k2[t] += __shfl_xor(k2[t], step);
                k3[t] += __shfl_xor(k3[t], step);
            }
            if (g == 0) { dots[wave][0][16 * t + r16] = q1[t]; dots[wave][1][16 * t + r16] = k2[t]; dots[wave][2][16 * t + r16] = k3[t]; }
        }
        for (int step = 1; step < 64; step <<= 1) state_sum += __shfl_xor(state_sum, step);
        if (lane == 0) state_dot[wave] = state_sum;
        __syncthreads();                               // U and dR are done with

        for (int p = x; p < kPatches; p += THREADS) {
            const int piece = p % (DK / 4), first = (p / (DK / 4)) * R;
            Patch<T> a, c;
            load_patch(a, q, A.ldq, first, valid, piece * 4, A.dk, wq);
            load_patch(c, k, A.ldk, first, valid, piece * 4, A.dk, wk);
            keep_patch(a, first, valid, piece * 4, A.dk);
            keep_patch(c, first, valid, piece * 4, A.dk);
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
                for (int t = 0; t < CT; ++t)
#pragma unroll
                    for (int p = Z::SOME - 1; p >= 0; --p) {
                        if (16 * t + 15 >= m * Z::K) gq[a][t] = mma(kf, get<T>(Ns + p * Z::kBytesMap, columns.at(t, m)), gq[a][t]);
                        if (m * Z::K + Z::K > 16 * t) gk[a][t] = mma(qf, get<T>(Nt + p * Z::kBytesMap, columns.at(t, m)), gk[a][t]);
                        gk[a][t] = mma(kf, get<T>(Ms + p * Z::kBytesMap, columns.at(t, m)), gk[a][t]);
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
// both sums go over the state at once.  A workgroup takes a slice of the columns: `lanes` times VEC of them, the rest of its threads the rows.
// ----------------------------------------------------------------------------
constexpr int kTokenThreads = 256;

template <typename T, int VEC, int DEPTH>
__global__ void __launch_bounds__(kTokenThreads)
k_delta_tokens(DeltaArgs A, int lanes_log2, int slices)
{
    constexpr int WAVES = kTokenThreads / 64;
    __shared__ float qs[2][256], ks[2][256], side[2][WAVES][64][2 * VEC], products[2][WAVES];
    typedef float vec __attribute__((ext_vector_type(VEC), aligned(VEC == 4 ? 16 : 4)));
    const int x = threadIdx.x, lanes = 1 << lanes_log2, rows = kTokenThreads >> lanes_log2, r0 = x >> lanes_log2;
    const int h = blockIdx.x / slices, slice = blockIdx.x % slices, kh = h / (A.heads / A.key_heads), col = (slice * lanes + (x & (lanes - 1))) * VEC;
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
        if (A.state_in && live && r0 + i * rows < A.dk) S[i] = *reinterpret_cast<const vec*>(A.state_in + at + (int64_t)(r0 + i * rows) * A.dv);
    }
    for (int64_t n = 0; n < count; ++n) {
        const int turn = (int)(n & 1);
        const int64_t row = begin + n;
        float kq = 0.0f;
        if (x < A.dk) {
            const float qx = to_float(static_cast<const T*>(A.q)[row * A.ldq + (int64_t)kh * A.dk + x]), kx = to_float(static_cast<const T*>(A.k)[row * A.ldk + (int64_t)kh * A.dk + x]);
            qs[turn][x] = qx;
            ks[turn][x] = kx;
            kq = qx * kx;
        }
        const float rate = A.rates[row * A.ldr + h], beta = A.beta[row * A.ldb + h];
        float v[VEC];
#pragma unroll
        for (int c = 0; c < VEC; ++c) v[c] = live ? to_float(static_cast<const T*>(A.v)[row * A.ldv + (int64_t)h * A.dv + col + c]) : 0.0f;
        // the decay in two numbers: rounded to one it could be off the same way at every token
        const double exact = exp(-(double)rate);
        const float hi = (float)exact, lo = (float)(exact - (double)hi);
        for (int step = 1; step < 64; step <<= 1) kq += __shfl_xor(kq, step);
        if ((x & 63) == 0) products[turn][x >> 6] = kq;
        __syncthreads();
        float e[VEC], f[VEC];
#pragma unroll
        for (int c = 0; c < VEC; ++c) e[c] = f[c] = 0.0f;
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            const int r = r0 + i * rows;
            if (r < A.dk) {
                const float kr = ks[turn][r], qr = qs[turn][r];
#pragma unroll
                for (int c = 0; c < VEC; ++c) {
                    S[i][c] = fmaf(S[i][c], hi, S[i][c] * lo);
                    e[c] = fmaf(kr, S[i][c], e[c]);
                    f[c] = fmaf(qr, S[i][c], f[c]);
                }
            }
        }
        for (int step = lanes; step < 64; step <<= 1)
#pragma unroll
            for (int c = 0; c < VEC; ++c) { e[c] += __shfl_xor(e[c], step); f[c] += __shfl_xor(f[c], step); }
        if ((x & 63) < lanes)
#pragma unroll
            for (int c = 0; c < VEC; ++c) { side[turn][x >> 6][x & 63][2 * c] = e[c]; side[turn][x >> 6][x & 63][2 * c + 1] = f[c]; }
        __syncthreads();
        const int column = x & (lanes - 1);
        float u[VEC];
        const float product = (products[turn][0] + products[turn][1]) + (products[turn][2] + products[turn][3]);
#pragma unroll
        for (int c = 0; c < VEC; ++c) {
            float es = 0.0f, fs = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) { es += side[turn][w][column][2 * c]; fs += side[turn][w][column][2 * c + 1]; }
            u[c] = beta * (v[c] - es);
            f[c] = A.scale * fmaf(product, u[c], fs);
        }
        if (A.y && r0 == 0 && live) {
            T* const y = static_cast<T*>(A.y) + row * A.ldy + (int64_t)h * A.dv + col;
#pragma unroll
            for (int c = 0; c < VEC; ++c) y[c] = (T)f[c];
        }
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            const int r = r0 + i * rows;
            if (r < A.dk)
#pragma unroll
                for (int c = 0; c < VEC; ++c) S[i][c] = fmaf(ks[turn][r], u[c], S[i][c]);
        }
    }
    if (A.state_out && live)
#pragma unroll
        for (int i = 0; i < DEPTH; ++i)
            if (r0 + i * rows < A.dk) *reinterpret_cast<vec*>(A.state_out + at + (int64_t)(r0 + i * rows) * A.dv) = S[i];
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

size_t aligned(size_t v) { return (v + 255) / 256 * 256; }

struct Parts { size_t maps, states, u, gstates, r, all; };

Parts layout_of(bool bf16, int64_t chunks, int heads, int dk, int dv, bool training)
{
    const int d = padded_of(dk, dv), c = tokens_of_chunk(bf16, d), ct = c / 16;
    const size_t each = (size_t)chunks * heads * sizeof(float), numbers = (size_t)(ct * (ct + 1) / 2 * 256 + 5 * c + 4);
    Parts L{};
    L.maps = 0;
    L.all = aligned(each * numbers);
    if (training) {
        const auto take = [&](size_t bytes) { const size_t at = L.all; L.all += aligned(bytes); return at; };
        L.states = take(each * d * d);
        L.u = take(each * c * d);
        L.gstates = take(each * d * d);
        L.r = take(each * c * d);
    }
    return L;
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

template <typename T, int DK, int WAVES>
hipError_t run_with(DeltaArgs A, hipStream_t st)
{
    const dim3 sequences = grid_of((int64_t)A.heads * A.slices, A.sequences), chunks = grid_of(A.key_heads, A.chunks), block(64 * WAVES);
    if (A.forward || !A.saved) {
        if (A.chunks > 0) {
            profile_before("delta_prepare", st);
            hipLaunchKernelGGL((k_delta_prepare<T, DK>), chunks, dim3(kPrepareThreads), 0, st, A);
            profile_after("delta_prepare", st);
        }
        profile_before("delta_walk", st);
        if (A.forward) hipLaunchKernelGGL((k_delta_walk<T, DK, WAVES, true>), sequences, block, 0, st, A);
        else hipLaunchKernelGGL((k_delta_walk<T, DK, WAVES, false>), sequences, block, 0, st, A);
        profile_after("delta_walk", st);
    }
    if (!A.forward) {
        profile_before("delta_back", st);
        hipLaunchKernelGGL((k_delta_back<T, DK, WAVES>), sequences, block, 0, st, A);
        profile_after("delta_back", st);
        if (A.chunks > 0 && (A.gq || A.gk || A.gv || A.grates || A.gbeta)) {
            profile_before("delta_gradients", st);
            hipLaunchKernelGGL((k_delta_gradients<T, DK, WAVES>), chunks, block, 0, st, A);
            profile_after("delta_gradients", st);
        }
    }
    return hipGetLastError();
}

template <typename T>
hipError_t run_of(const DeltaArgs& A, int padded, hipStream_t st)
{
    if (padded == 64) return run_with<T, 64, 4>(A, st);
    if (padded == 96) return run_with<T, 96, 6>(A, st);
    if (padded == 128) return run_with<T, 128, 8>(A, st);
    if (padded == 192) return run_with<T, 192, 6>(A, st);
    return run_with<T, 256, 8>(A, st);
}

template <typename T, int VEC>
hipError_t tokens_with(const DeltaArgs& A, int lanes_log2, int slices, hipStream_t st)
{
    const dim3 grid = grid_of((int64_t)A.heads * slices, A.sequences), block(kTokenThreads);
    const int rows = kTokenThreads >> lanes_log2, depth = (A.dk + rows - 1) / rows;
    profile_before("delta_tokens", st);
    if (depth <= 4) hipLaunchKernelGGL((k_delta_tokens<T, VEC, 4>), grid, block, 0, st, A, lanes_log2, slices);
    else hipLaunchKernelGGL((k_delta_tokens<T, VEC, 16>), grid, block, 0, st, A, lanes_log2, slices);
    profile_after("delta_tokens", st);
    return hipGetLastError();
}

}  // namespace

// For up to so many tokens and sequences, of equal lengths or not, of heads and sizes like these.
size_t delta_workspace(bool bf16, int64_t tokens, int64_t sequences, int heads, int dk, int dv, bool training)
{
    const int c = tokens_of_chunk(bf16, padded_of(dk, dv));
    return layout_of(bf16, tokens / c + sequences, heads, dk, dv, training).all;
}

hipError_t launch_delta_tokens(const DeltaArgs& A, hipStream_t st)
{
    const bool aligned4 = A.dv % 4 == 0 && reinterpret_cast<uintptr_t>(A.state_in) % 16 == 0 && reinterpret_cast<uintptr_t>(A.state_out) % 16 == 0;
    const int vec = aligned4 ? 4 : 1, wide = (A.dv + vec - 1) / vec;
    // at most 16 lanes: 16 rows of the state for every thread then
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
    const int padded = padded_of(A.dk, A.dv), c = tokens_of_chunk(A.bf16, padded), size = A.bf16 ? 2 : 4;
    const bool training = !A.forward || A.saved;
    A.slices = padded > 128 ? 2 : 1;
    A.per_sequence = !A.starts && A.sequences > 0 ? (A.tokens / A.sequences + c - 1) / c : 0;
    A.chunks = chunks_of(A.tokens, A.sequences, c, A.starts == nullptr);
    const Parts L = layout_of(A.bf16, A.chunks, A.heads, A.dk, A.dv, training);
    A.maps = reinterpret_cast<float*>(A.ws + L.maps);
    if (training) {
        A.states_out = reinterpret_cast<float*>(A.ws + L.states);
        A.u_out = reinterpret_cast<float*>(A.ws + L.u);
        A.gstates = reinterpret_cast<float*>(A.ws + L.gstates);
        A.r_out = reinterpret_cast<float*>(A.ws + L.r);
    }
    A.wide = (allows(A.q, A.ldq, A.dk, size, 4 * size) ? 1 : 0) | (allows(A.k, A.ldk, A.dk, size, 4 * size) ? 2 : 0) | (allows(A.v, A.ldv, A.dv, size, 4 * size) ? 4 : 0) |
             (allows(A.y, A.ldy, A.dv, size, 4 * size) ? 8 : 0) | (allows(A.gy, A.ldgy, A.dv, size, 4 * size) ? 16 : 0) |
             (allows(A.gq, A.ldgq, A.dk, size, 4 * size) ? 32 : 0) | (allows(A.gk, A.ldgk, A.dk, size, 4 * size) ? 64 : 0);
    return A.bf16 ? run_of<__bf16>(A, padded, st) : run_of<float>(A, padded, st);
}

}  // namespace laplex
