// Tiles for the products of a chunk of tokens: fragments of rows for the matrix cores, their places in LDS, reading rows of any alignment, and fp32 numbers as
// sums of bf16 ones (attention_kernels.hip, delta_kernels.hip).
#pragma once

#include "token_internal.h"

namespace laplex {

namespace {

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

}  // namespace

}  // namespace laplex
