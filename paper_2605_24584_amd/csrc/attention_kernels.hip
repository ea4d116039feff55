// Linear attention with a decay for each head: the causal Laplace kernel exp(-rate (t - s)), s <= t, over token positions,
// weighted by (q_t . k_s):  y_t = sum_{s <= t} l^(t-s) (q_t . k_s) v_s + l^(t+1) q_t S0,  l = exp(-rate).
//
// A walk (token_internal.h) is computed in chunks of C tokens with the state S (dk x dv) carried from chunk to chunk:
//   inside a chunk   P_ij = l^(i-j) (q_i . k_j), j <= i;     out_i = l^(i+lead) q_i S + sum_j P_ij v_j
//   and its end      S <- l^C S + sum_j l^(C-j-lead) k_j v_j^T
// All four products run on the matrix cores.  A workgroup of four, six or eight wavefronts walks one head of one stretch of a sequence; a
// wavefront owns 16 columns of the result and of the state, which stays in its accumulator registers from the first chunk to
// the last: as it leaves an accumulator a pair of tiles IS a fragment of the product q S (over the state's rows in a
// permuted order, which the rows of q in LDS share), so the state does not pass through memory.  (32 columns a wavefront, four of them: 249 registers
// instead of 128 and no faster.)
//
// Sequences that are long and few are cut into stretches: one launch forms what each stretch adds to the state (k_attention_walk<STATES>, which
// reads k and v alone), one brings these together in order (k_attention_carry), and then all stretches are walked at once.
//
// Numbers: bf16 q, k, v and results; sums and states are fp32.  What goes from one product into the next is not rounded to the type: P, and the state for the
// product q S, are the sum of two bf16 numbers (16 bits, where the result is rounded to 8: it is rounded once, whatever the lengths), and what goes into a state
// that can be asked for is not rounded at all: l^d v is the sum of three bf16 numbers, exactly, so a state is an fp32 sum of exact products.  fp32 runs on
// the fp32 matrix instructions.
//
// What bounds it: a chunk of 64 bf16 tokens of a head of 128 takes a compute unit 5.1 to 5.3 us with two workgroups on it; its LDS reads alone would
// take 2.1, its vector instructions 2.1, its matrix products 1.3: as they are, they hardly overlap.  us of the walk / states / carry (on average over calls, between
// which the walk of a long sequence varies most): 4 x 2048 tokens, 16 heads of 128, bf16 51 / 24 / 11; one of 65536, 8 heads 167 to 189 / 82 / 28; 8 x 4096, 16 heads
// 163 / 67 / 11, its gradients 501 uncut (3.2 TB/s: three walks, each with three matrices read and one written); 24 sequences of 1250 on average, 6 heads of 96 x 80, fp32
// 143 / 54 / 13, its gradients 380 to 420 / 120 / 21.
#include "token_internal.h"

namespace laplex {

namespace {

constexpr int kStepThreads = 256;

__device__ __forceinline__ float rate_of(const float* rates, int h)
{
    const float r = rates[h];
    return r > 1.0e30f ? 1.0e30f : r;     // an infinite rate: nothing but the token itself, and 0 * rate stays 0.  NaN stays NaN
}

__device__ __forceinline__ int64_t start_of(const int64_t* starts, int64_t tokens, int64_t sequences, int64_t b)
{
    if (!starts) return sequences > 0 ? tokens / sequences * b : 0;
    const int64_t v = starts[b];                       // whatever it holds, no row outside the matrices is touched
    return v < 0 ? 0 : v > tokens ? tokens : v;
}

// ----------------------------------------------------------------------------
// Fragments: 16 bytes of a row, K numbers of the contraction per step of the matrix cores (16 x 16 results; lane l holds
// row or column l % 16 and the numbers of group l / 16; of a result, column l % 16 and rows 4 (l / 16) .. + 3).
// ----------------------------------------------------------------------------
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

template <typename T> struct Num;
template <> struct Num<float> {
    typedef f32x4 frag;
    typedef f32x4 quad;                  // four numbers
    static constexpr int E = 4, K = 16;
};
template <> struct Num<__bf16> {
    typedef bf16x8 frag;
    typedef bf16x4 quad;
    static constexpr int E = 8, K = 32;
};

__device__ __forceinline__ f32x4 mma(f32x4 a, f32x4 b, f32x4 c)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// A tile in LDS: rows of SLOTS times 16 bytes.  The slots of a row are permuted by its number, so that eight lanes that read
// the same slot of eight rows, or write a column's pieces of eight rows, meet eight different groups of banks.
template <int SLOTS>
__device__ __forceinline__ int twist(int row)
{
    return SLOTS >= 8 ? (row ^ (row >> 3)) & 7 : ((row >> 1) ^ (row >> 3)) & 3;
}
template <int SLOTS>
__device__ __forceinline__ int slot_at(int row, int slot) { return row * SLOTS + (slot ^ twist<SLOTS>(row)); }

// Keeps the compiler from forming everything that follows from v outside the loop over chunks, where it would fill the registers.
__device__ __forceinline__ int here(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// a value that all lanes hold
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }

// A lane's part of the place of slot 4 m + g of row 16 t + r16: the rest of the permutation depends on t and m alone.
template <int SLOTS>
struct Reader {
    static constexpr int kMask = SLOTS >= 8 ? 7 : 3;
    int base, low;
    __device__ __forceinline__ Reader(int r16, int g) : base(r16 * SLOTS * 16), low((g ^ twist<SLOTS>(r16)) * 16) {}
    __device__ __forceinline__ int at(int t, int m) const
    {
        const int fixed = (4 * m ^ 2 * t) & kMask;
        return base + (low ^ (fixed * 16)) + ((4 * m) & ~kMask) * 16 + t * 16 * SLOTS * 16;
    }
};

// R rows of four numbers each
template <typename T>
struct Patch {
    static constexpr int R = sizeof(T) == 2 ? 4 : 2;
    typename Num<T>::quad r[R];
};

// Rows first .. first + R - 1 of a chunk of `valid` rows from `base` on, numbers at .. at + 3 of `width`, which may be read four at a time and lie
// within 2^31 bytes of the chunk's lowest row.  CLAMP: where some do not exist others are read in their place (no branch, so that nothing waits for the loads
// here), and keep_patch zeroes them before they are used.
template <typename T, bool CLAMP>
__device__ __forceinline__ void load_wide(Patch<T>& out, const T* base, int64_t stride, int first, int valid, int at, int width)
{
    typedef typename Num<T>::quad quad;
    const bool down = stride < 0;                      // an unsigned 32-bit place from the row that lies lowest
    const char* const low = reinterpret_cast<const char*>(down ? base + stride * (valid - 1) : base);
    const uint32_t step = (uint32_t)((down ? -stride : stride) * (int)sizeof(T));
    if (CLAMP) at = at < width - 4 ? at : width - 4;
    const uint32_t place = (down ? valid - 1 - first : first) * step + at * (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < Patch<T>::R; ++i) {
        if (CLAMP) {
            const int row = first + i < valid ? first + i : valid - 1;
            out.r[i] = *reinterpret_cast<const quad*>(low + ((down ? valid - 1 - row : row) * step + at * (int)sizeof(T)));
        } else {
            out.r[i] = *reinterpret_cast<const quad*>(low + (down ? place - i * step : place + i * step));
        }
    }
}
__device__ __forceinline__ void keep_patch(Patch<float>& p, int first, int valid, int at, int width)
{
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (first + i >= valid || at + e >= width) p.r[i][e] = 0.0f;
}
__device__ __forceinline__ void keep_patch(Patch<__bf16>& p, int first, int valid, int at, int width)
{
    const int n = width - at;                          // numbers that exist
    const uint32_t m0 = n >= 2 ? 0xFFFFFFFFu : n == 1 ? 0xFFFFu : 0, m1 = n >= 4 ? 0xFFFFFFFFu : n == 3 ? 0xFFFFu : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u32x2 v = __builtin_bit_cast(u32x2, p.r[i]);
        p.r[i] = __builtin_bit_cast(bf16x4, first + i < valid ? u32x2{v[0] & m0, v[1] & m1} : u32x2{0, 0});
    }
}

// Rows of any alignment, width and distance, a number at a time; as above, others in the place of those that do not exist.
template <typename T>
__device__ __forceinline__ void load_some(Patch<T>& out, const T* base, int64_t stride, int first, int valid, int at, int width)
{
#pragma unroll
    for (int i = 0; i < Patch<T>::R; ++i) {
        const T* const p = base + (first + i < valid ? first + i : valid - 1) * stride;
#pragma unroll
        for (int e = 0; e < 4; ++e) out.r[i][e] = p[at + e < width ? at + e : width - 1];
    }
    if constexpr (sizeof(T) == 2) {
        // Put together here, where that waits for the loads of a patch: 16-bit numbers take a register each until then.
#pragma unroll
        for (int i = 0; i < Patch<T>::R; ++i) {
            u32x2 v = __builtin_bit_cast(u32x2, out.r[i]);
            v[0] = here(v[0]); v[1] = here(v[1]);
            out.r[i] = __builtin_bit_cast(typename Num<T>::quad, v);
        }
    }
}

// Rows as they are, numbers along the slots (first: a multiple of R, piece: which four numbers).  In bf16 the quads of 32 numbers lie in the order
// 0 4 1 5 2 6 3 7: group g of a fragment then holds numbers 4 g .. + 3 and 16 + 4 g .. + 3, which are the rows of a pair of accumulator
// tiles that the group holds.
template <int SLOTS>
__device__ __forceinline__ void put_rows(char* tile, const Patch<__bf16>& p, int first, int piece)
{
    const int low = here(((piece >> 3) * 4 + (piece & 3)) ^ twist<SLOTS>(first));
    char* const at = tile + first * SLOTS * 16 + 8 * ((piece >> 2) & 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<bf16x4*>(at + i * SLOTS * 16 + 16 * (low ^ i)) = p.r[i];
}
template <int SLOTS>
__device__ __forceinline__ void put_rows(char* tile, const Patch<float>& p, int first, int piece)
{
    const int low = here(piece ^ twist<SLOTS>(first));
    char* const at = tile + first * SLOTS * 16;
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<f32x4*>(at + i * SLOTS * 16 + 16 * (low ^ i)) = p.r[i];
}

// The patch's columns as rows, tokens along the slots.
template <int SLOTS>
__device__ __forceinline__ void put_columns(char* tile, const Patch<__bf16>& p, int first, int piece)
{
    const int low = here((first >> 3) ^ twist<SLOTS>(piece * 4));
    char* const at = tile + piece * 4 * SLOTS * 16 + 8 * ((first >> 2) & 1);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bf16x4 v = {p.r[0][e], p.r[1][e], p.r[2][e], p.r[3][e]};
        *reinterpret_cast<bf16x4*>(at + e * SLOTS * 16 + 16 * (low ^ (SLOTS >= 8 ? e : (e >> 1)))) = v;
    }
}
template <int SLOTS>
__device__ __forceinline__ void put_columns(char* tile, const Patch<float>& p, int first, int piece)
{
    const int low = here((first >> 2) ^ twist<SLOTS>(piece * 4));
    char* const at = tile + piece * 4 * SLOTS * 16 + 8 * ((first >> 1) & 1);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const f32x2 v = {p.r[0][e], p.r[1][e]};
        *reinterpret_cast<f32x2*>(at + e * SLOTS * 16 + 16 * (low ^ (SLOTS >= 8 ? e : (e >> 1)))) = v;
    }
}

template <typename T>
__device__ __forceinline__ typename Num<T>::frag get(const char* tile, int place)
{
    return *reinterpret_cast<const typename Num<T>::frag*>(tile + place);
}

// x = hi + mid + lo, exactly: bf16 holds 8 bits, so three of them hold all 24 of an fp32 number.  The upper half of an fp32 number is a bf16 one.
__device__ __forceinline__ float upper(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }
__device__ __forceinline__ bf16x8 uppers(const float* x)
{
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_amdgcn_perm(__float_as_uint(x[2 * e + 1]), __float_as_uint(x[2 * e]), 0x07060302u);
    return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ void split3(const float* x, bf16x8& hi, bf16x8& mid, bf16x8& lo)
{
    float r[8], q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        r[e] = x[e] - upper(x[e]);
        q[e] = r[e] - upper(r[e]);
    }
    hi = uppers(x); mid = uppers(r); lo = uppers(q);
}

// x = hi + mid but for 2^-15 of x
__device__ __forceinline__ void split2(const float* x, bf16x8& hi, bf16x8& mid)
{
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = x[e] - upper(x[e]);
    hi = uppers(x);
#pragma unroll
    for (int e = 0; e < 8; ++e) mid[e] = (__bf16)r[e];
}

__device__ __forceinline__ void split2(f32x4 x, bf16x4& hi, bf16x4& mid)
{
    hi = __builtin_bit_cast(bf16x4, u32x2{__builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302u),
                                          __builtin_amdgcn_perm(__float_as_uint(x[3]), __float_as_uint(x[2]), 0x07060302u)});
#pragma unroll
    for (int e = 0; e < 4; ++e) mid[e] = (__bf16)(x[e] - upper(x[e]));
}

__device__ __forceinline__ bool finite_bits(float v) { return (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u; }
__device__ __forceinline__ bool finite_patch(const Patch<float>& p)
{
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) { const uint32_t v = __float_as_uint(p.r[i][e]) & 0x7F800000u; most = v > most ? v : most; }
    return most != 0x7F800000u;
}
__device__ __forceinline__ bool finite_patch(const Patch<__bf16>& p)
{
    uint32_t odd = 0;                                  // an exponent of ones carries into the sign's place
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u32x2 v = __builtin_bit_cast(u32x2, p.r[i]);
        odd |= ((v[0] & 0x7F807F80u) + 0x00800080u) | ((v[1] & 0x7F807F80u) + 0x00800080u);
    }
    return (odd & 0x80008000u) == 0;
}

// ----------------------------------------------------------------------------
// Which stretch of which sequence: sequences are cut into stretches of `stretch` tokens (a multiple of every C), each with a slot.  Of equal lengths
// every sequence has its slots; otherwise sequence b has those from start / stretch + b on: at least one, and as many as it has stretches, and a
// slot beyond those has nothing to do.
//
// A sequence of several stretches has a place in the workspace for the state that enters each.  They are numbered like the slots, but for b, where no more than
// start / (stretch + 1) sequences before this one can have several: however many short sequences are packed, there are at most two places for `stretch` tokens.
// ----------------------------------------------------------------------------
constexpr int64_t kSlotRows = 32768;      // slots along a grid's second axis

struct Stretch {
    int64_t b;                        // sequence
    int64_t begin, count;             // its rows
    int64_t lo, hi;                   // tokens of the stretch, in the order of the walk
    bool there, last;
    int64_t index;
};

__device__ __forceinline__ int64_t first_slot(const AttentionArgs& A, int64_t b, int64_t begin)
{
    return A.starts ? (uint32_t)begin / (uint32_t)A.stretch + b : b * A.per_sequence;
}

__device__ __forceinline__ int64_t first_place(const AttentionArgs& A, int64_t b, int64_t begin)
{
    if (!A.starts) return b * A.per_sequence;
    const int64_t several = (uint32_t)begin / (uint32_t)(A.stretch + 1);
    return (uint32_t)begin / (uint32_t)A.stretch + (b < several ? b : several);
}

// The stretch with this slot, or (PLACES) the one with this place, if there is one.
template <bool PLACES>
__device__ __forceinline__ Stretch find_stretch(const AttentionArgs& A, int64_t slot)
{
    const auto first = [&](int64_t b, int64_t begin) { return PLACES ? first_place(A, b, begin) : first_slot(A, b, begin); };
    Stretch s;
    int64_t lo = 0;
    if (A.starts) {
        // the last sequence whose first one is at most this one: 64 candidates at a time
        int64_t hi = A.sequences;                      // in [lo, hi)
        const int lane = threadIdx.x & 63;
        while (hi - lo > 1) {
            const int64_t step = (hi - lo + 63) / 64;
            const int64_t c = lo + lane * step;
            const bool mine = c < hi && first(c, start_of(A.starts, A.tokens, A.sequences, c)) <= slot;
            const uint64_t votes = __ballot(mine);
            const int at = votes ? 63 - __builtin_clzll(votes) : 0;
            lo += at * step;
            hi = lo + step < hi ? lo + step : hi;
        }
    } else {
        lo = slot / A.per_sequence;
    }
    s.b = lo;
    s.begin = start_of(A.starts, A.tokens, A.sequences, lo);
    const int64_t end = start_of(A.starts, A.tokens, A.sequences, lo + 1);
    s.count = end > s.begin ? end - s.begin : 0;
    s.index = slot - first(lo, s.begin);
    s.lo = s.index * A.stretch;
    s.there = s.index >= 0 && (s.lo < s.count || s.index == 0);
    s.hi = s.lo + A.stretch < s.count ? s.lo + A.stretch : s.count;
    s.last = s.hi == s.count;
    return s;
}

// A number of the initial state, not yet scaled; of one that does not exist, another one.
__device__ __forceinline__ float state_value(const Walk& W, int64_t at, int row, int col)
{
    const int down = W.transposed ? 1 : W.dv, along = W.transposed ? W.dk : 1;
    return W.state_in[at + (row < W.dk ? row : W.dk - 1) * down + (col < W.dv ? col : W.dv - 1) * along];
}

// Where a set's state has row `row` and column `col`, in numbers from its first: pieces of four rows, as the accumulators hold them.
template <int DK, int COLS>
__device__ __forceinline__ int set_place(int row, int col)
{
    return (col / COLS) * DK * COLS + ((((col % COLS) / 16) * (DK / 16) + row / 16) * 64 + (row % 16) / 4 * 16 + col % 16) * 4 + row % 4;
}

// Sizes of a walk's kernel: DK the padded rows of the state; every wavefront has a tile of 16 columns.
template <typename T, int DK, int WAVES>
struct Geometry {
    static constexpr int E = Num<T>::E, K = Num<T>::K, R = Patch<T>::R, THREADS = 64 * WAVES;
    static constexpr int C = (DK > 128 ? 32 : 64) * 2 / (int)sizeof(T);      // tokens of a chunk
    static constexpr int COLS = 16 * WAVES;                                      // columns of a workgroup
    static constexpr int ROW = (DK * (int)sizeof(T) / 16 + 7) / 8 * 8, SEQ = C * (int)sizeof(T) / 16;   // slots of a row of numbers (a multiple of 8: they are permuted by eights), of tokens
    static constexpr int CT = C / 16, DT = DK / 16, KD = DK / K, KC = C / K;
    static constexpr int kBytesRows = C * ROW * 16, kBytesK = DK * SEQ * 16, kBytesV = COLS * SEQ * 16;
    // bf16: P's second part is kept beside the first.  Of rows below 32 it lies 32 tokens further along where a row has 64 (they see none of those), of the others, and
    // where a row has 32, 32 rows further down.
    static constexpr int kBytesP = (C + (sizeof(T) == 2 ? 32 : 0)) * SEQ * 16;
    static constexpr int kLds = 2 * kBytesRows + kBytesK + kBytesV + kBytesP;
};

enum { kWalk, kStates };      // kStates: only what a stretch adds to the state, for the stretches behind it (U below)

template <typename T, int DK, int WAVES, int MODE>
__global__ void __launch_bounds__(64 * WAVES, (MODE == kStates && sizeof(T) == 4 ? (DK > 128 ? 4 : DK > 96 ? 5 : 6) : DK > 128 ? 2 : DK > 96 ? 4 : DK > 64 && sizeof(T) == 4 ? 5 : 3))      // as many as LDS and the state leave room for
k_attention_walk(AttentionArgs A)
{
    typedef Geometry<T, DK, WAVES> G;
    constexpr bool STATES = MODE == kStates;
    typedef typename Num<T>::frag frag;
    typedef typename Num<T>::quad quad;
    constexpr int E = G::E, C = G::C, R = G::R, ROW = G::ROW, SEQ = G::SEQ, CT = G::CT, DT = G::DT, KD = G::KD, KC = G::KC, THREADS = G::THREADS;
    __shared__ __attribute__((aligned(16))) char lds[STATES ? G::kBytesK + G::kBytesV : G::kLds];
    __shared__ float power[C + 1], weight[C];          // l^d (times inner, where it is used for the weights alone), and the weights of the chunk's tokens in the state
    __shared__ int odd[2];
    char* const Kt = lds;                              // [DK][C]
    char* const Vt = Kt + G::kBytesK;                  // [COLS][C]
    char* const Qs = Vt + G::kBytesV;                  // [C][DK], as Ks
    char* const Ks = Qs + G::kBytesRows;
    char* const Ps = Ks + G::kBytesRows;               // [C][C], and its second part

    // heads side by side: the slots that have nothing to do are then spread over the chiplets, which take workgroups in turn
    const int walks = STATES ? A.sets : A.walks, walk = blockIdx.z % walks, slice = blockIdx.x % A.slices, h = blockIdx.x / A.slices, col0 = slice * G::COLS;
    const int64_t slot = (int64_t)(blockIdx.z / walks) * kSlotRows + blockIdx.y;
    const Walk W = STATES ? A.states[walk] : A.walk[walk];
    if (slot >= (STATES ? A.places : A.slots) || col0 >= W.dv) return;
    const Stretch s = find_stretch<STATES>(A, slot);
    if (!s.there || (STATES && s.last)) return;

    const int x = threadIdx.x, lane = x & 63, wave = __builtin_amdgcn_readfirstlane(x >> 6), r16 = lane & 15, g = lane >> 4;
    const double rate = (double)rate_of(A.rates, h);
    const float inner = uniform(W.inner);
    for (int d = x; d <= C; d += THREADS) power[d] = STATES ? (float)exp(-rate * d) * inner : (float)exp(-rate * d);
    if (!STATES)
        for (int i = x; i < G::kBytesP / 16; i += THREADS) reinterpret_cast<f32x4*>(Ps)[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (x < 2) odd[x] = 0;
    // A chunk's decay as an fp32 number and what its rounding leaves out, in parts of it: the same rounding in every chunk would add up, so the
    // next number up or down is taken whenever what has been left out reaches half of their distance.  The last chunk may be shorter.
    const double full_decay = exp(-rate * C);
    const float decay = uniform((float)full_decay), end_decay = uniform((float)exp(-rate * (int)((s.hi - s.lo) % C)));
    // (twice the smallest number at least: half of that is not 0)
    const float ulp = uniform(fmaxf(__uint_as_float(__float_as_uint(decay) + 1) - decay, 2.8e-45f)), rest = uniform((float)(full_decay - (double)decay));
    float left = 0.0f;

    const int64_t back = W.reverse ? -1 : 1;
    const int64_t first_row = s.begin + (W.reverse ? s.count - 1 - s.lo : s.lo);
    const int64_t sq = back * W.ldq, sk = back * W.ldk, sv = back * W.ldv;
    const int64_t near = INT32_MAX / (int64_t)(C * sizeof(T)) - DK;      // rows further apart need 64-bit places
    const int flags = STATES ? A.states_wide[walk] : A.wide[walk];
    const bool wide = (flags & 7) == 7 && W.ldq < near && W.ldk < near && W.ldv < near, wo = flags & 8;
    const bool whole = wide && W.dk == DK && col0 + G::COLS <= W.dv, whole_out = W.out && wo && col0 + G::COLS <= W.dv;

    // the state: rows 16 t + 4 g .. + 3, columns col0 + 16 wave + r16
    f32x4 S[DT];
    const int col = col0 + 16 * wave + r16;
    const int64_t state_at = (s.b * A.heads + h) * (int64_t)W.dk * W.dv;
    constexpr int kPieces = DK * G::COLS / 4;
    const int64_t place = STATES ? slot : first_place(A, s.b, s.begin) + s.index;
    f32x4* const set = reinterpret_cast<f32x4*>(A.ws) + (((int64_t)(STATES ? walk : W.set) * A.places + place) * A.heads + h) * A.slices * kPieces;
    f32x4* const U = set + (int64_t)slice * kPieces + wave * DT * 64 + lane;
    // (of several stretches the first one's state, too, comes from U: another workgroup may already write the last state, in its place)
    const bool several = s.count > A.stretch;
    const bool from_set = !STATES && several && (s.index > 0 || W.state_in), from_given = !STATES && !several && W.state_in;
    // One branch for all loads of a kind, and others in the place of what does not exist: nothing waits for one of them before the next is asked for.
    if (from_set && !W.set_transposed) {
#pragma unroll
        for (int t = 0; t < DT; ++t) S[t] = U[t * 64];
    } else if (from_set) {
        // row `col` and columns 16 t + 4 g .. + 3 of the set
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = reinterpret_cast<const float*>(set)[set_place<DK, G::COLS>(col, 16 * t + 4 * g + r)];
    } else if (from_given) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = state_value(W, state_at, 16 * t + 4 * g + r, col);
    } else {
#pragma unroll
        for (int t = 0; t < DT; ++t) S[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const float scale = from_given ? 1.0f / W.last_scale : 1.0f;
    if ((from_set && W.set_transposed) || from_given)
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = col < W.dv && 16 * t + 4 * g + r < W.dk ? scale * S[t][r] : 0.0f;

    // a chunk's patches
    constexpr int kRowPatches = (C / R) * (DK / 4), kColPatches = (C / R) * (G::COLS / 4);
    constexpr int NR = (kRowPatches + THREADS - 1) / THREADS, NV = (kColPatches + THREADS - 1) / THREADS;
    Patch<T> pq[NR], pk[NR], pv[NV];
    const T* q = static_cast<const T*>(W.q) + first_row * W.ldq + (int64_t)h * W.dk;       // the first row of the chunk that is loaded next
    const T* k = static_cast<const T*>(W.k) + first_row * W.ldk + (int64_t)h * W.dk;
    const T* v = static_cast<const T*>(W.v) + first_row * W.ldv + (int64_t)h * W.dv;
    auto load = [&](int64_t u) {
        const int valid = (int)(s.hi - u < C ? s.hi - u : C), y = here(x);
        auto each = [&](auto rows_of, auto columns_of) {
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const int p = y + i * THREADS;
                if (kRowPatches % THREADS == 0 || p < kRowPatches) rows_of(i, (p / (DK / 4)) * R, (p % (DK / 4)) * 4);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int p = y + i * THREADS;
                if (kColPatches % THREADS == 0 || p < kColPatches) columns_of(i, (p / (G::COLS / 4)) * R, col0 + (p % (G::COLS / 4)) * 4);
            }
        };
        // (one branch for all: a wait for the loads of one matrix where the other branch has its own would hold up the next one's)
        if (whole && valid == C)
            each([&](int i, int row, int at) {
                     if (!STATES) load_wide<T, false>(pq[i], q, sq, row, C, at, DK);
                     load_wide<T, false>(pk[i], k, sk, row, C, at, DK);
                 },
                 [&](int i, int row, int at) { load_wide<T, false>(pv[i], v, sv, row, C, at, W.dv); });
        else if (wide)
            each([&](int i, int row, int at) {
                     if (!STATES) load_wide<T, true>(pq[i], q, sq, row, valid, at, W.dk);
                     load_wide<T, true>(pk[i], k, sk, row, valid, at, W.dk);
                 },
                 [&](int i, int row, int at) { load_wide<T, true>(pv[i], v, sv, row, valid, at, W.dv); });
        else
            each([&](int i, int row, int at) {
                     if (!STATES) load_some(pq[i], q, sq, row, valid, at, W.dk);
                     load_some(pk[i], k, sk, row, valid, at, W.dk);
                 },
                 [&](int i, int row, int at) { load_some(pv[i], v, sv, row, valid, at, W.dv); });
        q += C * sq; k += C * sk; v += C * sv;
    };
    if (s.lo < s.hi) load(s.lo);
    __syncthreads();                                   // the powers are there
    T* out = static_cast<T*>(W.out) + first_row * W.ldo + (int64_t)h * W.dv + col0 + 16 * wave;      // the chunk's first row
    const int64_t so = back * W.ldo;

    int turn = 0;
    for (int64_t u = s.lo; u < s.hi; u += C, turn ^= 1) {
        const int valid = (int)(s.hi - u < C ? s.hi - u : C);
        bool fine = true;
        const int y = here(x);
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int p = y + i * THREADS;
            if (kRowPatches % THREADS == 0 || p < kRowPatches) {
                const int piece = p % (DK / 4), row = (p / (DK / 4)) * R;
                if (!(whole && valid == C)) {
                    if (!STATES) keep_patch(pq[i], row, valid, piece * 4, W.dk);
                    keep_patch(pk[i], row, valid, piece * 4, W.dk);
                }
                if (!STATES) { put_rows<ROW>(Qs, pq[i], row, piece); put_rows<ROW>(Ks, pk[i], row, piece); }
                put_columns<SEQ>(Kt, pk[i], row, piece);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int p = y + i * THREADS;
            if (kColPatches % THREADS == 0 || p < kColPatches) {
                const int piece = p % (G::COLS / 4), row = (p / (G::COLS / 4)) * R;
                if (!(whole && valid == C)) keep_patch(pv[i], row, valid, col0 + piece * 4, W.dv);
                put_columns<SEQ>(Vt, pv[i], row, piece);
                if (!STATES) fine = fine && finite_patch(pv[i]);
            }
        }
        if (!STATES && !fine) odd[turn] = 1;
        if (u == s.lo || valid < C)
            if (x < C) weight[x] = STATES ? power[x < valid ? valid - x - W.lead : 0] : power[x < valid ? valid - x - W.lead : 0] * inner;
        if (u + C < s.hi) load(u + C);
        __syncthreads();

        const int l = here(lane), r16 = l & 15, g = l >> 4;
        const Reader<ROW> rows(r16, g);
        const Reader<SEQ> columns(r16, g);
        Reader<SEQ> values(r16, g);                    // the columns of this wavefront
        values.base += wave * 16 * SEQ * 16;
        values.low ^= ((2 * wave) & Reader<SEQ>::kMask) * 16;
        if (!STATES) {
            // P: tiles on and below the diagonal, dealt to the wavefronts; as it leaves the accumulator a lane holds P[i][j .. j + 3]
#pragma unroll
            for (int n = 0; n < (CT * (CT + 1) / 2 + WAVES - 1) / WAVES; ++n) {
                const int tile = n * WAVES + wave;
                int it = 0, jt = tile;
                while (jt > it) { jt -= it + 1; ++it; }
                if (it < CT) {
                    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int m = 0; m < KD; ++m) acc = mma(get<T>(Ks, rows.at(jt, m)), get<T>(Qs, rows.at(it, m)), acc);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int d = 16 * (it - jt) + r16 - 4 * g - r;
                        acc[r] = d >= 0 ? acc[r] * power[d < 0 ? 0 : d] * inner : 0.0f;
                    }
                    const int j = 16 * jt + 4 * g;
                    const auto put = [&](int row, int j, quad w) {
                        *reinterpret_cast<quad*>(Ps + 16 * slot_at<SEQ>(row + r16, j / E) + (j % E) * (int)sizeof(T)) = w;
                    };
                    if constexpr (sizeof(T) == 2) {
                        quad hi, mid;
                        split2(acc, hi, mid);
                        put(16 * it, j, hi);
                        const bool along = KC == 2 && it < 2;
                        put(along ? 16 * it : 16 * it + 32, along ? j + 32 : j, mid);
                    } else {
                        put(16 * it, j, acc);
                    }
                }
            }
            // q S, weighted by the rows
            f32x4 O[CT];
#pragma unroll
            for (int t = 0; t < CT; ++t)
                O[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int m = 0; m < KD; ++m) {
                if (m % 2 == 0) __builtin_amdgcn_sched_barrier(0);     // (all steps' fragments at once do not fit the registers)
                constexpr int TERMS = sizeof(T) == 2 ? 2 : 1;
                frag sf[TERMS];
                if constexpr (sizeof(T) == 2) {
                    float xs[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) xs[e] = S[2 * m + (e >> 2)][e & 3];
                    split2(xs, sf[0], sf[1]);
                } else {
                    sf[0] = S[m];
                }
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    const frag qf = get<T>(Qs, rows.at(t, m));
#pragma unroll
                    for (int p = 0; p < TERMS; ++p) O[t] = mma(sf[p], qf, O[t]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < CT; ++t) {
                const float ahead = power[16 * t + r16 + W.lead];
                O[t] *= ahead;
            }
            __syncthreads();                           // P is there
            const bool slow = odd[turn] != 0;          // a value of v is not finite: 0 * v of the tokens behind a row must not reach it
            if (x == 0) odd[turn ^ 1] = 0;
#pragma unroll
            for (int m = 0; m < KC; ++m) {
                frag vf = get<T>(Vt, values.at(0, m));
                if (slow)
#pragma unroll
                    for (int e = 0; e < E; ++e) vf[e] = finite_bits((float)vf[e]) ? vf[e] : (T)0.0f;
#pragma unroll
                for (int t = 0; t < CT; ++t)
                    if (16 * t + 15 >= m * G::K) {
                        const frag pf = get<T>(Ps, columns.at(t, m));
                        O[t] = mma(vf, pf, O[t]);
                        if constexpr (sizeof(T) == 2) {
                            const bool along = KC == 2 && t < 2;
                            O[t] = mma(vf, get<T>(Ps, columns.at(along ? t : t + 2, along ? 1 : m)), O[t]);
                        }
                    }
            }
            if (slow)
                for (int j = 0; j < C; ++j) {
                    const int i0 = here(r16), n0 = here(wave * 16 + 4 * g);
                    float p[CT];
#pragma unroll
                    for (int t = 0; t < CT; ++t)
                        p[t] = (float)*reinterpret_cast<const T*>(Ps + 16 * slot_at<SEQ>(16 * t + i0, j / E) + (j % E) * (int)sizeof(T));
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float vj = (float)*reinterpret_cast<const T*>(Vt + 16 * slot_at<SEQ>(n0 + r, j / E) + (j % E) * (int)sizeof(T));
#pragma unroll
                        for (int t = 0; t < CT; ++t)
                            if (!finite_bits(vj) && 16 * t + i0 >= j) O[t][r] += vj * p[t];
                    }
                }
            const auto result = [&](int t) {
                quad w;
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = (T)(O[t][r] * W.out_scale);
                return w;
            };
            if (whole_out && valid == C) {
#pragma unroll
                for (int t = 0; t < CT; ++t)
                    *reinterpret_cast<quad*>(out + (16 * t + r16) * so + 4 * g) = result(t);
            } else if (W.out) {
#pragma unroll
                for (int t = 0; t < CT; ++t)
                    if (16 * t + r16 < valid) {
                        const int n = col0 + 16 * wave + 4 * g;
                        T* const at = out + (16 * t + r16) * so + 4 * g;
                        const quad w = result(t);
                        if (wo) {
                            if (n < W.dv) *reinterpret_cast<quad*>(at) = w;
                        } else {
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (n + r < W.dv) at[r] = w[r];
                        }
                    }
            }
            out += C * so;
        }
        // the state at the chunk's end
        float d = decay;
        left += rest;
        if (left >= 0.5f * ulp) { d = decay + ulp; left -= ulp; }
        else if (left <= -0.5f * ulp) { d = decay - ulp; left += ulp; }
        if (valid < C) d = end_decay;
#pragma unroll
        for (int t = 0; t < DT; ++t)
            S[t] *= d;
#pragma unroll
        for (int m = 0; m < KC; ++m) {
            __builtin_amdgcn_sched_barrier(0);
            float w[E];
#pragma unroll
            for (int e = 0; e < E; ++e) w[e] = weight[(4 * m + g) * E + e];
            const frag vf = get<T>(Vt, values.at(0, m));
            float xs[E];
#pragma unroll
            for (int e = 0; e < E; ++e) xs[e] = w[e] * (float)vf[e];
            constexpr int TERMS = sizeof(T) == 2 ? 3 : 1;
            frag part[TERMS];
            if constexpr (sizeof(T) == 2) {
                // all 24 bits where the state can be asked for, 16 where it only goes on into results of 8
                if (W.exact) split3(xs, part[0], part[1], part[2]);
                else split2(xs, part[0], part[1]);
            } else part[0] = f32x4{xs[0], xs[1], xs[2], xs[3]};
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                const frag kf = get<T>(Kt, columns.at(t, m));
#pragma unroll
                for (int p = 0; p < TERMS; ++p)
                    if (p < 2 || W.exact) S[t] = mma(kf, part[p], S[t]);
            }
        }
        __syncthreads();                               // the tiles may be written again
    }

#pragma unroll
    for (int t = 0; t < DT; ++t) {
        if (STATES) U[t * 64] = S[t];
        else if (W.state_out && s.last) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + 4 * g + r;
                if (col < W.dv && row < W.dk) W.state_out[state_at + (int64_t)row * W.dv + col] = W.last_scale * S[t][r];
            }
        }
    }
}

// What enters the stretches: carry_n = l^stretch carry_(n-1) + U_(n-1), carry_0 = the initial state, in the places of the U.
// A thread per four rows of a column of the state, for every sequence; or, where there are fewer places than sequences, for every place, of which a sequence's first
// one has something to do (4096 sequences of 16 tokens, 16 heads: 1.3 ms to look at each).
template <int DK, int COLS>
__global__ void __launch_bounds__(256)
k_attention_carry(AttentionArgs A)
{
    constexpr int kPieces = DK * COLS / 4, kBlocks = (kPieces + 255) / 256;
    const Walk W = A.states[blockIdx.z];
    const bool by_place = A.places < A.sequences;
    for (int64_t block = blockIdx.x; block < (by_place ? A.places : A.sequences) * A.slices * kBlocks; block += gridDim.x) {
        int64_t b = block / (A.slices * kBlocks);
        if (by_place) {
            const Stretch s = find_stretch<true>(A, b);
            if (s.index != 0 || s.count <= A.stretch) continue;
            b = s.b;
        }
        const int rest = (int)(block % (A.slices * kBlocks)), slice = rest / kBlocks, piece = (rest % kBlocks) * 256 + threadIdx.x;
        const int h = blockIdx.y, col0 = slice * COLS;
        if (col0 >= W.dv || piece >= kPieces) continue;
        constexpr int DT = DK / 16;
        const int lane = piece & 63, t = (piece >> 6) % DT, wave = piece / (64 * DT);
        const int64_t begin = start_of(A.starts, A.tokens, A.sequences, b), end = start_of(A.starts, A.tokens, A.sequences, b + 1);
        const int64_t count = end > begin ? end - begin : 0, stretches = (count + A.stretch - 1) / A.stretch;
        const int64_t place = first_place(A, b, begin);
        if (stretches < 2 || place + stretches > A.places) continue;
        const double d = exp(-(double)rate_of(A.rates, h) * (double)A.stretch);
        const float hi = (float)d, lo = (float)(d - (double)hi);
        f32x4 carry = {0.0f, 0.0f, 0.0f, 0.0f};
        if (W.state_in) {
            const int col = col0 + wave * 16 + (lane & 15);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * t + 4 * (lane >> 4) + r;
                const float v = state_value(W, (b * A.heads + h) * (int64_t)W.dk * W.dv, row, col);
                carry[r] = col < W.dv && row < W.dk ? (1.0f / W.last_scale) * v : 0.0f;
            }
        }
        const int64_t step = (int64_t)A.heads * A.slices * kPieces;
        f32x4* U = reinterpret_cast<f32x4*>(A.ws) + ((((int64_t)blockIdx.z * A.places + place) * A.heads + h) * A.slices + slice) * kPieces + piece;
        f32x4 next = U[0];
        if (W.state_in) U[0] = carry;
        for (int64_t n = 1; n < stretches; ++n) {
#pragma unroll
            for (int r = 0; r < 4; ++r) carry[r] = fmaf(carry[r], hi, fmaf(carry[r], lo, next[r]));
            if (n + 1 < stretches) next = U[n * step];
            U[n * step] = carry;
        }
    }
}

// One token for every sequence: the state is read and written once, everything else is a few hundred numbers.  A workgroup takes `lanes` times VEC columns of one
// state, a lane VEC of them, the rest of the lanes its rows.  256 sequences of 16 heads of 128 x 128: 88 us for 0.54 GB (6.1 TB/s); one sequence 4.0 us.
template <typename T, int VEC>
__global__ void __launch_bounds__(kStepThreads)
k_attention_step(AttentionStepArgs A, int lanes_log2, int slices)
{
    constexpr int kAhead = 4;                          // rows that a thread has asked for at a time
    __shared__ float qs[256], ks[256], side[kStepThreads / 64][64][VEC];
    const int x = threadIdx.x, lanes = 1 << lanes_log2, rows = kStepThreads >> lanes_log2;
    const int64_t b = blockIdx.x / slices;
    const int slice = blockIdx.x % slices, h = blockIdx.y, col = (slice * lanes + (x & (lanes - 1))) * VEC;
    // the decay in two floats: rounded to one it would be off the same way at every token
    const double exact = exp(-(double)rate_of(A.rates, h));
    const float hi = (float)exact, lo = (float)(exact - (double)hi);
    if (x < A.dk) {
        qs[x] = to_float(static_cast<const T*>(A.q)[b * A.ldq + (int64_t)h * A.dk + x]);
        ks[x] = to_float(static_cast<const T*>(A.k)[b * A.ldk + (int64_t)h * A.dk + x]);
    }
    const bool live = col < A.dv;
    float v[VEC], o[VEC];
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
        v[c] = live ? to_float(static_cast<const T*>(A.v)[b * A.ldv + (int64_t)h * A.dv + col + c]) : 0.0f;
        o[c] = 0.0f;
    }
    __syncthreads();
    typedef float vec __attribute__((ext_vector_type(VEC)));
    float* const S = A.state + (b * A.heads + h) * (int64_t)A.dk * A.dv + col;
    if (live)
        for (int r0 = x >> lanes_log2; r0 < A.dk; r0 += kAhead * rows) {
            vec s[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (r0 + i * rows < A.dk) s[i] = *reinterpret_cast<const vec*>(S + (int64_t)(r0 + i * rows) * A.dv);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int r = r0 + i * rows;
                if (r < A.dk) {
#pragma unroll
                    for (int c = 0; c < VEC; ++c) {
                        s[i][c] = fmaf(s[i][c], hi, fmaf(s[i][c], lo, ks[r] * v[c]));
                        o[c] = fmaf(qs[r], s[i][c], o[c]);
                    }
                    *reinterpret_cast<vec*>(S + (int64_t)r * A.dv) = s[i];
                }
            }
        }
    for (int step = lanes; step < 64; step <<= 1)
#pragma unroll
        for (int c = 0; c < VEC; ++c) o[c] += __shfl_xor(o[c], step);
#pragma unroll
    for (int c = 0; c < VEC; ++c) side[x >> 6][x & 63][c] = o[c];
    __syncthreads();
    if (x < lanes && live) {
        T* const y = static_cast<T*>(A.y) + b * A.ldy + (int64_t)h * A.dv + col;
#pragma unroll
        for (int c = 0; c < VEC; ++c)
            y[c] = (T)(A.scale * ((side[0][x][c] + side[1][x][c]) + (side[2][x][c] + side[3][x][c])));
    }
}

struct Plan {
    int dk, cols, slices;              // padded rows of the state, columns of a workgroup, workgroups side by side
    int64_t stretch, per_sequence, slots, places;
    bool cut;                          // some sequence may have more than one stretch
};

constexpr int64_t kPackedWorkgroups = 2048, kLeastStretch = 64;

// By the sizes alone.  walks: 1 for the forward call, 3 for the backward one, also where not all gradients are wanted (what one of them is must not
// depend on the others).
Plan plan_of(bool bf16, int64_t tokens, int64_t sequences, int heads, int dk, int dv, int walks, bool equal)
{
    Plan P;
    const int most = dk > dv ? dk : dv;
    P.dk = most <= 64 ? 64 : most <= 96 ? 96 : most <= 128 ? 128 : most <= 192 ? 192 : 256;
    P.cols = P.dk == 64 ? 64 : P.dk == 96 || P.dk == 192 ? 96 : 128;
    P.slices = (most + P.cols - 1) / P.cols;
    const int64_t longest = equal && sequences > 0 ? tokens / sequences : tokens;
    // Two workgroups for every compute unit, where cutting is worth its two further launches and the second read of k and v: not where whole sequences
    // give every compute unit one or nearly (a stretch would be half a sequence or more).  Of unknown lengths four times as many, since the longest
    // stretch is what the others wait for.  us, stretches of 256 / 512 / 1024 / 2048 / whole sequences: 4 x 2048 tokens, 16 heads 92 / 92 / 142 / - / 186; 65536
    // tokens, 8 heads 371 / 292 / 253 / 297 / 5810; 8 x 4096, 16 heads 310 / 261 / 230 / 285 / 381, their gradients 749 / 651 / 596 / 564 / 502; 24 sequences of
    // 1250 tokens on average, 6 heads, fp32 226 / 232 / 355 / 503 / 674, their gradients 473 / 509 / 677 / 940 / 783.
    const int64_t work = tokens * heads * P.slices * walks, workgroups = equal ? 512 : kPackedWorkgroups;
    P.stretch = (work + 64 * workgroups - 1) / (64 * workgroups) * 64;
    // At least 256 tokens, or the states that pass through memory cost more than the walks.  Where even those leave compute units without a workgroup the
    // time is that of one workgroup's stretch, twice, and of the chain of states over the stretches: shorter ones, the more so the shorter the sequence.
    // us, stretches of 256 / 128 / 64, one sequence, bf16, a head of 128: 384 tokens 42 / 29 / 25; 1024 46 / 31 / 26; 4096 50 / 39 / 40; 16384 64 / 67 / 96;
    // fp32 83 / 50 / 34; 86 / 52 / 37; 90 / 60 / 51; 103 / 87 / 106.  Sequences of a few tokens on average need none of it.
    int64_t least = 256;
    if (work < 256 * 256 && tokens >= 64 * sequences) least = longest <= 2048 ? kLeastStretch : longest <= 8192 ? 128 : 256;
    if (P.stretch < least) P.stretch = least;
    // (192 tokens whole / in stretches of 64: bf16 23 / 22 us, their gradients 21 / 22; fp32 44 / 33 and 42 / 33)
    P.cut = longest > 2 * P.stretch && longest > (bf16 ? 256 : 128);
    if (!P.cut) P.stretch = longest < 64 ? 64 : (longest + 63) / 64 * 64;
    P.per_sequence = equal ? (longest + P.stretch - 1) / P.stretch : 0;
    if (equal && P.per_sequence < 1) P.per_sequence = 1;
    P.slots = equal ? sequences * P.per_sequence : tokens / P.stretch + sequences;
    const int64_t several = tokens / (P.stretch + 1);
    P.places = !P.cut ? 0 : equal ? P.slots : tokens / P.stretch + (sequences < several ? sequences : several);
    return P;
}

bool allows(const void* p, int64_t ld, int d, int size, int bytes)
{
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * size % bytes == 0 && d * size % bytes == 0;
}

template <typename T, int DK, int WAVES>
hipError_t walk_with(const AttentionArgs& A, const Plan& P, hipStream_t st)
{
    const int64_t deep = (P.slots + kSlotRows - 1) / kSlotRows;
    const dim3 grid((unsigned)(A.heads * P.slices), (unsigned)(deep > 1 ? kSlotRows : P.slots), (unsigned)(deep * A.walks));
    if (P.cut) {
        const int64_t places_deep = (P.places + kSlotRows - 1) / kSlotRows;
        const dim3 sets_grid(grid.x, (unsigned)(places_deep > 1 ? kSlotRows : P.places), (unsigned)(places_deep * A.sets));
        profile_before("attention_states", st);
        hipLaunchKernelGGL((k_attention_walk<T, DK, WAVES, kStates>), sets_grid, dim3(64 * WAVES), 0, st, A);
        profile_after("attention_states", st);
        profile_before("attention_carry", st);
        const int64_t blocks = (P.places < A.sequences ? P.places : A.sequences) * P.slices * ((DK * 16 * WAVES / 4 + 255) / 256), most = int64_t(1) << 22;      // (a grid holds fewer than 2^32 threads)
        hipLaunchKernelGGL((k_attention_carry<DK, 16 * WAVES>), dim3((unsigned)(blocks < most ? blocks : most), (unsigned)A.heads, (unsigned)A.sets),
                           dim3(256), 0, st, A);
        profile_after("attention_carry", st);
    }
    profile_before("attention_walk", st);
    hipLaunchKernelGGL((k_attention_walk<T, DK, WAVES, kWalk>), grid, dim3(64 * WAVES), 0, st, A);
    profile_after("attention_walk", st);
    return hipGetLastError();
}

template <typename T>
hipError_t walk_of(const AttentionArgs& A, const Plan& P, hipStream_t st)
{
    if (P.dk == 64) return walk_with<T, 64, 4>(A, P, st);
    if (P.dk == 96) return walk_with<T, 96, 6>(A, P, st);
    if (P.dk == 128) return walk_with<T, 128, 8>(A, P, st);
    if (P.dk == 192) return walk_with<T, 192, 6>(A, P, st);
    return walk_with<T, 256, 8>(A, P, st);
}

}  // namespace

// For any number of tokens and sequences up to these, the forward and the backward call, lengths that are equal or not: a stretch has at least kLeastStretch tokens and
// at least work / kPackedWorkgroups, so that there are at most `most` whole ones, and a place more for each sequence of several.
size_t attention_workspace(int64_t tokens, int64_t sequences, int heads, int dk, int dv)
{
    size_t bytes = 0;
    for (int walks = 1; walks <= 3 && heads > 0 && tokens > 128; walks += 2) {
        const Plan P = plan_of(false, tokens, sequences, heads, dk, dv, walks, false);
        const int64_t by_work = kPackedWorkgroups / ((int64_t)heads * P.slices * walks), most = tokens / kLeastStretch < by_work ? tokens / kLeastStretch : by_work;
        const size_t here = (size_t)(walks > 1 ? 2 : 1) * (most + (sequences < most ? sequences : most)) * heads * P.slices * P.dk * P.cols * sizeof(float);
        bytes = here > bytes ? here : bytes;
    }
    return bytes;
}

hipError_t launch_attention(const AttentionArgs& given, hipStream_t st)
{
    AttentionArgs A = given;
    const Plan P = plan_of(A.bf16, A.tokens, A.sequences, A.heads, A.walk[0].dk, A.walk[0].dv, A.backward ? 3 : 1, A.starts == nullptr);
    A.stretch = P.stretch; A.per_sequence = P.per_sequence; A.slots = P.slots; A.places = P.places; A.slices = P.slices;
    const int size = A.bf16 ? 2 : 4;
    const auto flags = [&](const Walk& W) {
        return (allows(W.q, W.ldq, W.dk, size, 4 * size) ? 1 : 0) | (allows(W.k, W.ldk, W.dk, size, 4 * size) ? 2 : 0) |
               (allows(W.v, W.ldv, W.dv, size, 4 * size) ? 4 : 0) | (allows(W.out, W.ldo, W.dv, size, 4 * size) ? 8 : 0);
    };
    for (int w = 0; w < A.walks; ++w) A.wide[w] = flags(A.walk[w]);
    for (int w = 0; w < A.sets; ++w) A.states_wide[w] = flags(A.states[w]);
    return A.bf16 ? walk_of<__bf16>(A, P, st) : walk_of<float>(A, P, st);
}

hipError_t launch_attention_step(const AttentionStepArgs& A, hipStream_t st)
{
    const int vec = A.dv % 4 == 0 && reinterpret_cast<uintptr_t>(A.state) % 16 == 0 ? 4 : 1;
    const int wide = (A.dv + vec - 1) / vec;
    // few states: narrower slices of them, so that more compute units take part
    const int most = A.sequences * A.heads >= 1024 ? 6 : 3;
    int lanes_log2 = 0;
    while (lanes_log2 < most && (1 << lanes_log2) < wide) ++lanes_log2;
    const int slices = (wide + (1 << lanes_log2) - 1) >> lanes_log2;
    const dim3 grid((unsigned)(A.sequences * slices), (unsigned)A.heads), block(kStepThreads);
    profile_before("attention_step", st);
    if (A.bf16) {
        if (vec == 4) hipLaunchKernelGGL((k_attention_step<__bf16, 4>), grid, block, 0, st, A, lanes_log2, slices);
        else hipLaunchKernelGGL((k_attention_step<__bf16, 1>), grid, block, 0, st, A, lanes_log2, slices);
    } else {
        if (vec == 4) hipLaunchKernelGGL((k_attention_step<float, 4>), grid, block, 0, st, A, lanes_log2, slices);
        else hipLaunchKernelGGL((k_attention_step<float, 1>), grid, block, 0, st, A, lanes_log2, slices);
    }
    profile_after("attention_step", st);
    return hipGetLastError();
}

}  // namespace laplex
