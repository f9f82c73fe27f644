// What the 8-bit operators with a scale for each block of 128 share: element types, the format's
// conversions, and the layout of 8-bit weights.
#ifndef SLIM_BLOCK_FP8_H
#define SLIM_BLOCK_FP8_H

#include "slim_internal.h"

namespace slim {

constexpr int kBlk = 128;                     // values to a scale, inputs to a weight tile
constexpr float kFp8Max = 448.0f;             // largest value of E4M3
constexpr float kTopFloor = 0x1p-100f;        // a block's largest magnitude counts as this much at least
constexpr int kMaxK = 1 << 22;                // a tile of 256 rows stays below 2^31 bytes
constexpr int kWTileRows = 64, kWTileBytes = kWTileRows * kBlk;

inline int blocks_of(int k) { return (int)(((int64_t)k + kBlk - 1) / kBlk); }
inline int wtile_rows(int n) { return (int)(((int64_t)n + kWTileRows - 1) / kWTileRows); }

// Byte of weight (o, i), both inside one tile of 64 rows x 128 inputs.  A tile is four fragments of
// V_MFMA_F32_16X16X128_F8F6F4's A operand (2 KiB, each two loads of 64 lanes x 16 bytes).  Row 4 g + r of fragment t is row
// 16 g + 4 t + r of the tile, so that a lane, which holds rows 4 g .. 4 g + 3 of a fragment's results, has 16 consecutive
// rows after the four.
__host__ __device__ inline uint32_t wtile_place(uint32_t o, uint32_t i)
{
    const uint32_t g = o >> 4, t = (o >> 2) & 3u, r = o & 3u, h = i >> 6, q = (i >> 4) & 3u, b = i & 15u;
    return t * 2048u + h * 1024u + (q * 16u + 4u * g + r) * 16u + b;
}

struct F16 {
    typedef _Float16 type;
};
struct BF16 {
    typedef __bf16 type;
};
struct F32 {
    typedef float type;
};

// `count` elements of a row that need not be aligned to more than an element, as one access (the memory pipeline
// takes any address).
template <class T, int N>
struct Piece {
    typedef typename T::type vec __attribute__((ext_vector_type(N)));
    struct __attribute__((packed, aligned(sizeof(typename T::type)))) place {
        vec v;
    };
    static __device__ __forceinline__ vec load(const typename T::type *p) { return reinterpret_cast<const place *>(p)->v; }
    static __device__ __forceinline__ void store(typename T::type *p, vec v) { reinterpret_cast<place *>(p)->v = v; }
    // past the caches' turn: for what is not read again soon and would only put out what is
    static __device__ __forceinline__ void store_streaming(typename T::type *p, vec v)
    {
        typedef vec any __attribute__((aligned(sizeof(typename T::type))));
        __builtin_nontemporal_store(v, reinterpret_cast<any *>(p));
    }
};

// N elements of a row from `at` on in 32 bits, zero from element `len` on.
template <class T, int N>
__device__ __forceinline__ void load_piece(const typename T::type *row, int at, int len, float (&v)[N])
{
    if (at + N <= len) {
        const auto x = Piece<T, N>::load(row + at);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (float)x[e];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = at + e < len ? (float)row[at + e] : 0.f;
    }
}
template <class T, int N, bool STREAMING = false>
__device__ __forceinline__ void store_piece(typename T::type *row, int at, int len, const float (&v)[N])
{
    if (at + N <= len) {
        typename Piece<T, N>::vec x;
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = (typename T::type)v[e];
        if constexpr (STREAMING)
            Piece<T, N>::store_streaming(row + at, x);
        else
            Piece<T, N>::store(row + at, x);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (at + e < len) row[at + e] = (typename T::type)v[e];
    }
}

// Magnitudes are compared as whole numbers: the order of their bits is theirs, with a NaN above everything, so that a
// block that holds one has a NaN for its scale.
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

template <int N>
__device__ __forceinline__ uint32_t top_of(const float (&v)[N])
{
    uint32_t t = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) t = max(t, magnitude_bits(v[e]));
    return t;
}

__device__ __forceinline__ float floored_top(uint32_t bits)
{
    return __builtin_bit_cast(float, max(bits, __builtin_bit_cast(uint32_t, kTopFloor)));
}

// Four codes: nearest value of the format, ties to even (the conversion instruction).  |v| is at most kFp8Max up to a rounding of
// the product that made it, and what is that near above it still rounds to it; a NaN becomes the format's.
__device__ __forceinline__ uint32_t four_fp8(float v0, float v1, float v2, float v3)
{
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v2, v3, __builtin_amdgcn_cvt_pk_fp8_f32(v0, v1, 0, false), true);
}

}  // namespace slim
#endif
