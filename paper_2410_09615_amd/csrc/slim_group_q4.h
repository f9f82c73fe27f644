// What the operators on 4-bit weights with a scale for each group of inputs share: the layout of the codes, and codes as numbers.
#ifndef SLIM_GROUP_Q4_H
#define SLIM_GROUP_Q4_H

#include "slim_block_fp8.h"

namespace slim {

// Codes are kept in blocks of 16 rows x 128 inputs (1 KiB), row block major.  Piece (q, r) of a block, 16 bytes at (16 q + r) * 16, is what a
// lane holds of the four 16 x 16 x 32 products over the block's inputs: its dword j has inputs 32 j + 8 q .. + 7 of row r.  Inputs 2 i and
// 2 i + 1 of a dword are its nibbles i and i + 4, so that shifting by 4 i and masking leaves the two as 16-bit halves.
constexpr int kGq4Rows = 16, kGq4Cols = 128, kGq4Block = 1024;
// Whether weights are streamed (slim_group_q4_stream.hip): for up to 48 tokens, and on small layers for some more, a workgroup for each 48 of them.  us streamed / in tiles: 64 tokens on
// 4096 x 4096 12.5 / 18.5, on 5120 x 5120 17.9 / 19.2, on 4096 x 11008 26.2 / 22.9; gated 64 on 4096 x 4096 18.1 / 20.8, on 5120 x 5120 28.8 / 22.7; 144 on 1024 x 4096 8.6 / 16.3, on 4096 x 4096 22.9 / 22.1.
inline bool gq4_streamed(int n, int k, int m, bool gated)
{
    const int64_t weights = (int64_t)n * k * (gated ? 2 : 1);
    return m <= 48 || (m <= 96 && weights <= 34 << 20) || (m <= 192 && weights <= 8 << 20);
}
constexpr int kGq4Sym = 8;                    // the zero point of symmetric weights

inline int gq4_row_blocks(int n) { return (int)(((int64_t)n + kGq4Rows - 1) / kGq4Rows); }
inline int gq4_col_blocks(int k) { return (int)(((int64_t)k + kGq4Cols - 1) / kGq4Cols); }
inline int gq4_groups(int k, int shift) { return (int)(((int64_t)k + (1 << shift) - 1) >> shift); }
// 5, 6, 7 for groups of 32, 64, 128; -1 for others
inline int gq4_shift(int group) { return group == 32 ? 5 : group == 64 ? 6 : group == 128 ? 7 : -1; }

inline bool half_dtype(int32_t d) { return d == SLIM_F16 || d == SLIM_BF16; }
inline bool whole_elements(const void *p, int32_t d) { return (reinterpret_cast<uintptr_t>(p) & (d == SLIM_F32 ? 3u : 1u)) == 0; }

// One layer's weights as the kernels take them.
struct Gq4Weights {
    const uint8_t *codes;
    const half_t *scales;     // [n][groups]
    const uint8_t *zeros;     // the same, or null: kGq4Sym throughout
};

// The layer is what its sizes say it has to be; sets shift.
inline int gq4_check(const slim_group_q4_layer *l, int *shift)
{
    if (!l || !l->codes || !l->scales) return SLIM_ERR_NULL;
    if (slim_group_q4_sizes(l->n, l->k, l->group, nullptr, nullptr, nullptr) != SLIM_OK) return SLIM_ERR_SHAPE;
    if (!aligned16(l->codes) || (reinterpret_cast<uintptr_t>(l->scales) & 1u)) return SLIM_ERR_ALIGN;
    *shift = gq4_shift(l->group);
    return SLIM_OK;
}
inline Gq4Weights gq4_weights(const slim_group_q4_layer *l)
{
    return Gq4Weights{l->codes, reinterpret_cast<const half_t *>(l->scales), l->zeros};
}

// 1024 as two fp16 numbers: or'd onto a nibble it makes 1024 + c.  The same 15 binades lower: (1024 + c) 2^-15, where numbers are as far apart as whole ones are here, 2^-15.
constexpr uint32_t kGq4Bias = 0x64006400u, kGq4BiasLow = 0x28002800u;
constexpr float kGq4Low = 0x1p-15f;

// Constants that the compiler has to keep in registers: an instruction takes no two of them as literals.
struct Gq4Masks {
    uint32_t low, high, bias;
    half2_t sixteenth;
    __device__ __forceinline__ explicit Gq4Masks(uint32_t b = kGq4Bias) : bias(b)
    {
        low = 0x000f000fu;
        high = 0x00f000f0u;
        sixteenth = half2_t{(half_t)0.0625f, (half_t)0.0625f};
        asm volatile("" : "+s"(low), "+s"(high), "+v"(bias), "+v"(sixteenth));
    }
};

// Nibble E (0 .. 3) of both halves of a dword in fp16: 1024 + c of an even one, 1024 + 16 c of an odd one (the bits of 1024 set beside it): a shift per two nibbles.
template <int E>
__device__ __forceinline__ half2_t gq4_biased(uint32_t d, const Gq4Masks &k)
{
    return __builtin_bit_cast(half2_t, ((E < 2 ? d : d >> 8) & (E % 2 ? k.high : k.low)) | k.bias);
}
// 1024 + z of two zero points in fp16 (up to 1024 the steps there are 1)
__device__ __forceinline__ half2_t gq4_biased_zeros(uint32_t z0, uint32_t z1, uint32_t bias = kGq4Bias) { return __builtin_bit_cast(half2_t, (z1 << 16 | z0) + bias); }

// c - z of nibble E of both halves, exactly; z: 1024 + the zero points.
template <int E>
__device__ __forceinline__ half2_t gq4_less_zeros(uint32_t d, const Gq4Masks &k, half2_t z, half2_t z_sixteenth)
{
    const half2_t c = gq4_biased<E>(d, k);
    return E % 2 ? __builtin_elementwise_fma(c, k.sixteenth, -z_sixteenth) : c - z;
}

// ---- scales that fp16 weights cannot have ----
// (c - z) s reaches 255 x 65504, fp16 ends at 65504.  Where weights are rounded to fp16, groups whose scale is 256 or more are left out (a scale of 0; below that values stay below 256 x 255 =
// 65280), and where a workgroup has met one it goes over its share once more for those alone, with weights and inputs as sums of two bf16 numbers (16 bits of a weight, all 11 of an input), whose
// four products are added to the same sums.  Scales that are not finite stay with the others.  What it costs where there are none: six instructions for four scales, and a barrier
// (77 tokens' gradients through 5003 x 4100 24.5 -> 25.0 us, others within 1 %); where each row has one: 128 tokens on 4096 x 4096 20 -> 110 us, 4096 tokens 132 -> 813, their gradients 137 -> 1022.
__device__ __forceinline__ bool gq4_large(uint32_t h) { return (h & 0x7fffu) - 0x5c00u < 0x2000u; }             // 256 to 65504, as bits of fp16
// the scale if it is one of these (rest) or if it is none, and 0 otherwise
__device__ __forceinline__ uint32_t gq4_scale_of(uint32_t h, bool rest) { return gq4_large(h) == rest ? h : 0u; }
// whether one of the four scales is large or not finite
__device__ __forceinline__ bool gq4_any_large(uint2_t s)
{
    return ((((s[0] & 0x7fff7fffu) + 0x24002400u) | ((s[1] & 0x7fff7fffu) + 0x24002400u)) & 0x80008000u) != 0;
}
constexpr int kGq4Flags = 64;                                                   // bytes of LDS behind the windows: one number for each wavefront
// Whether any of the workgroup's `waves` wavefronts has it.
__device__ __forceinline__ bool gq4_any_wave(bool mine, uint8_t *flags, int wave, int waves)
{
    uint32_t *const f = reinterpret_cast<uint32_t *>(flags);
    const bool any = __ballot(mine) != 0;
    if ((threadIdx.x & (kWave - 1)) == 0) f[wave] = any;
    __syncthreads();
    uint32_t all = 0;
    for (int i = 0; i < waves; ++i) all |= f[i];
    return __builtin_amdgcn_readfirstlane((int)all) != 0;
}

// What turns codes into values (c - z) s, for the two halves (of one group or of two).
//   fp16: c - z exactly, and one rounding of the product to fp16 (of scales below 256).
//   bf16: (1024 + c) s - (1024 + z) s by one fused operation in binary32, exact since a code, a zero point and a scale have 23 bits between them; one rounding.
template <class T>
struct Gq4Pair;
template <>
struct Gq4Pair<F16> {
    half2_t s, z, z16;
    __device__ __forceinline__ Gq4Pair(half_t s0, uint32_t z0, half_t s1, uint32_t z1)
        : s{s0, s1}, z(gq4_biased_zeros(z0, z1)), z16(z - half2_t{(half_t)960.f, (half_t)960.f})
    {
    }
    template <int E>
    __device__ __forceinline__ uint32_t value(uint32_t d, const Gq4Masks &k) const
    {
        return __builtin_bit_cast(uint32_t, gq4_less_zeros<E>(d, k, z, z16) * s);
    }
};
template <>
struct Gq4Pair<BF16> {
    float s0, s1, c0, c1, o0, o1;                 // scales; what an even nibble's value lacks, and an odd one's
    __device__ __forceinline__ Gq4Pair(half_t a, uint32_t z0, half_t b, uint32_t z1) : s0((float)a), s1((float)b)
    {
        c0 = -(float)(1024u + z0) * s0;
        c1 = -(float)(1024u + z1) * s1;
        o0 = -(float)(64u + z0) * s0;
        o1 = -(float)(64u + z1) * s1;
    }
    template <int E>
    __device__ __forceinline__ uint32_t value(uint32_t d, const Gq4Masks &k) const
    {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        const half2_t h = gq4_biased<E>(d, k);
        const float f = E % 2 ? 0.0625f : 1.f;
        bf2 v;
        v[0] = (__bf16)__builtin_fmaf((float)h[0], s0 * f, E % 2 ? o0 : c0);
        v[1] = (__bf16)__builtin_fmaf((float)h[1], s1 * f, E % 2 ? o1 : c1);
        return __builtin_bit_cast(uint32_t, v);
    }
};

// A value at any address.
template <class V>
struct __attribute__((packed, aligned(1))) Gq4Any {
    V v;
};

template <class T>
struct Gq4Vec {
    typedef typename T::type E;
    typedef E v8 __attribute__((ext_vector_type(8)));
};

__device__ __forceinline__ float16_t gq4_mma32(Gq4Vec<F16>::v8 a, Gq4Vec<F16>::v8 b, float16_t c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float16_t gq4_mma32(Gq4Vec<BF16>::v8 a, Gq4Vec<BF16>::v8 b, float16_t c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float4_t gq4_mma16(Gq4Vec<F16>::v8 a, Gq4Vec<F16>::v8 b, float4_t c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float4_t gq4_mma16(Gq4Vec<BF16>::v8 a, Gq4Vec<BF16>::v8 b, float4_t c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// The first (0) or second (1) bf16 number of the two whose sum is v to 16 bits, as bits; of 8 fp16 numbers.
__device__ __forceinline__ uint32_t gq4_part_of(float v, int part)
{
    const uint32_t first = __builtin_bit_cast(uint32_t, v) & 0xffff0000u;
    return part ? (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)(v - __builtin_bit_cast(float, first))) : first >> 16;
}
__device__ __forceinline__ Gq4Vec<BF16>::v8 gq4_part_of(Gq4Vec<F16>::v8 v, int part)
{
    uint4_t out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = gq4_part_of((float)v[2 * e], part) | gq4_part_of((float)v[2 * e + 1], part) << 16;
    return __builtin_bit_cast(Gq4Vec<BF16>::v8, out);
}

// The 16-byte pieces of an LDS row of 64 values are put in another order in each of eight rows, so that the lanes of a read or write find all banks; the
// order is the same 32 rows on.
__device__ __forceinline__ uint32_t gq4_turn(uint32_t row) { return (row & 7u) ^ (row >> 3 & 3u); }

// A barrier for what is in LDS: unlike __syncthreads() it does not wait for loads that are under way to registers.
__device__ __forceinline__ void gq4_lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}

// ---- products whose inputs are shared by several workgroups ----
// Where there are fewer tiles than compute units, `splits` workgroups take a share each of what a tile sums over, and leave their sums in binary32: part[split][m][ld], of a gated block G's
// and then U's, 2 m rows.  gq4_launch_finish adds them in order and rounds.
struct Gq4Split {
    float *part;             // null: one workgroup has it all
    int splits, ld;
};
constexpr int kGq4Reads = 4 << 20;           // bytes that the memory system moves in about a microsecond
inline int gq4_part_ld(int outs) { return (int)(((int64_t)outs + 7) / 8 * 8); }
inline int64_t gq4_part_bytes(int splits, int m, int outs, bool gated) { return splits > 1 ? (int64_t)splits * m * gq4_part_ld(outs) * (gated ? 8 : 4) : 0; }

// A tile's shape: outputs and tokens, workgroups to a compute unit, the time (us) of a step of 64 inputs with few and with all compute units at work.
struct Gq4Shape {
    int outs, toks, per_cu;
    float few, all;
};
struct Gq4Plan {
    int shape, splits;
};
// The shape and number of splits with the least of rounds x (steps x time + 5 us) and what sums left in memory cost.
template <int N>
inline Gq4Plan gq4_plan(const Gq4Shape (&shapes)[N], int outs, int m, int steps, bool gated)
{
    const double cus = device_info().cus;
    Gq4Plan best{0, 1};
    double least = 0;
    for (int i = 0; i < N; ++i) {
        const Gq4Shape &s = shapes[i];
        const double tiles = (double)(((int64_t)outs * (gated ? 2 : 1) + s.outs - 1) / s.outs) * (double)(((int64_t)m + s.toks - 1) / s.toks);
        for (int splits = 1; splits <= 16 && (splits == 1 || (tiles * splits <= cus * s.per_cu && splits * 8 <= steps)); ++splits) {
            const double slots = cus * s.per_cu, rounds = __builtin_ceil(tiles * splits / slots), busy = tiles * splits / slots;
            const double step = busy <= 0.5 ? s.few : busy >= 1 ? s.all : s.few + (s.all - s.few) * (busy - 0.5) * 2;
            double time = rounds * (((steps + splits - 1) / splits) * step + 5);
            if (splits > 1) time += 4 + (2.0 * (double)gq4_part_bytes(splits, m, outs, gated) + 2.0 * m * outs) / kGq4Reads;
            if ((i == 0 && splits == 1) || time < least) {
                least = time;
                best = Gq4Plan{i, splits};
            }
        }
    }
    return best;
}

int gq4_launch_finish(const Gq4Split &p, int m, int outs, bool gated, void *const (&y)[3], const int64_t (&y_ld)[3], int32_t dtype, hipStream_t st);

// sigma(g) = 1 / (1 + exp(-g)) as a product of two factors, exp(-|g| / 2) each below 0: what silu is multiplied by may be as large as sigma is small, and each of the two is in binary32's range as long
// as a result in bf16 is (1 / (1 + exp(-g)) itself is 0 from -88.7 on, where silu(g) u has values down to -190).  An exponential of a quarter, squared twice: the instruction gives no subnormal numbers.
struct Gq4Sigma {
    float s, h;
    __device__ __forceinline__ explicit Gq4Sigma(float g)
    {
        const float quarter = __expf(-0.25f * __builtin_fabsf(g)), half = quarter * quarter;
        h = g < 0.f ? half : 1.f;
        s = h / (1.f + half * half);
    }
};
// silu(g) u
__device__ __forceinline__ float gq4_gated(float g, float u)
{
    const Gq4Sigma sigma(g);
    return (g * sigma.s) * (sigma.h * u);
}

}  // namespace slim
#endif
