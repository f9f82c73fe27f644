// 4-bit weights with a scale, and where asked for a zero point, for each group of 32, 64 or 128 inputs of a row: quantization, layout and its
// inverse, the values that codes stand for; and the gradient of a gated activation.
//
//   symmetric:         s = fp16(max |w| / 7),  z = 8,              c = clamp(rint(w / s), -8, 7) + 8
//   with zero points:  s = fp16((hi - lo) / 15),  z = rint(-lo / s),  c = clamp(rint(w / s) + z, 0, 15),   lo = min(w, 0), hi = max(w, 0)
//   value = (c - z) s
// Quotients in binary32.  All of these are bound by memory: quantization 4096 x 4096 fp16 13.1 us (3.2 TB/s; its 42 MB come from the last-level cache, all wavefronts
// are there at once, and the life of one is a load, a reduction, codes and a store: instructions count, 17.7 us with a conversion, shift and two clamps per code and three for what is not finite), 10007 x 5003 fp32 with zero points in groups of 32 80 us (2.8 TB/s, rows at odd multiples of 4 bytes); values 10.0 and 56 us (4.2 TB/s); the activation's gradient,
// 4096 x 11008 bf16, 73 to 78 us (5.8 to 6.2 TB/s).  The scale is rounded to fp16 before the codes are made, so codes are the nearest ones to the scale that is kept.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "slim_group_q4.h"

namespace slim {

struct Gq4QuantArgs {
    const void *W;
    int64_t ld;
    int n, k, cb, kg;
    int64_t blocks;
    uint8_t *codes;
    half_t *scales;
    uint8_t *zeros;
};

// Smallest / largest over the four lanes that hold a row's pieces.
__device__ __forceinline__ float over_four(float v, bool larger)
{
#pragma unroll
    for (int off = 1; off <= 2; off <<= 1) {
        const float o = __shfl_xor(v, off, kWave);
        v = larger ? fmaxf(v, o) : fminf(v, o);
    }
    return v;
}
__device__ __forceinline__ uint32_t over_four(uint32_t v)
{
    v |= (uint32_t)__shfl_xor((int)v, 1, kWave);
    return v | (uint32_t)__shfl_xor((int)v, 2, kWave);
}

// a / b to the nearest, given 1 / b to the nearest: the product with it is within a step of the quotient, what it lacks is exact in one fused operation, and adding that times 1 / b rounds once
// (Markstein's theorem; b is an fp16 number from 2^-24 to 65504, and quotients too small for it to hold are far below the 1/2 that a code begins at).  Three instructions where a division
// takes ten (3.5 us of 4096 x 4096 in fp16).
__device__ __forceinline__ float nearest_quotient(float a, float b, float inverse)
{
    const float q = a * inverse;
    return __builtin_fmaf(__builtin_fmaf(-q, b, a), inverse, q);
}

// A wavefront takes a block of 16 rows x 128 inputs; lane (r, q) = (lane / 4, lane % 4) the inputs 32 j + 8 q .. + 7 of row r, which are its piece of
// the layout.  Bound by memory.
template <class T, int SHIFT, bool ZEROS>
__global__ __launch_bounds__(256) void gq4_quant_kernel(Gq4QuantArgs a)
{
    constexpr int PER = 1 << (SHIFT - 5), GROUPS = 4 / PER;          // pieces per group, groups per block
    const int lane = (int)threadIdx.x & (kWave - 1), r = lane >> 2, q = lane & 3;
    const int64_t block = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    if (block >= a.blocks) return;
    const int rb = (int)(block / a.cb), cb = (int)(block % a.cb), row = rb * kGq4Rows + r;
    const bool there = row < a.n;
    const typename T::type *W = static_cast<const typename T::type *>(a.W) + (int64_t)(there ? row : a.n - 1) * a.ld;
    float w[4][8];
#pragma unroll
    for (int j = 0; j < 4; ++j) load_piece<T, 8>(W, cb * kGq4Cols + 32 * j + 8 * q, a.k, w[j]);
    uint4_t out;
    uint16_t __attribute__((ext_vector_type(GROUPS))) kept;
    uint8_t __attribute__((ext_vector_type(GROUPS))) points;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        float lo = 0.f, hi = 0.f, span;
        uint32_t odd;                                                // an infinity or a NaN among them
        if constexpr (ZEROS) {
            float none = 0.f;                                        // 0 w is a NaN for those alone
#pragma unroll
            for (int j = g * PER; j < (g + 1) * PER; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    lo = fminf(lo, w[j][e]);
                    hi = fmaxf(hi, w[j][e]);
                    none = __builtin_fmaf(w[j][e], 0.f, none);
                }
            lo = over_four(lo, false);
            hi = over_four(hi, true);
            odd = over_four((uint32_t)(none != 0.f));
            span = hi - lo;
        } else {
            uint32_t most = 0;                                       // (magnitudes as bits: those are larger than any number's)
#pragma unroll
            for (int j = g * PER; j < (g + 1) * PER; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = max(most, magnitude_bits(w[j][e]));
            most = max(most, (uint32_t)__shfl_xor((int)most, 1, kWave));
            most = max(most, (uint32_t)__shfl_xor((int)most, 2, kWave));
            odd = most >= 0x7f800000u;
            span = __builtin_bit_cast(float, most);
        }
        half_t s16 = (half_t)(span / (ZEROS ? 15.f : 7.f));
        if ((float)s16 == 0.f) s16 = span == 0.f ? (half_t)1.f : __builtin_bit_cast(half_t, (uint16_t)1);
        if ((float)s16 > 65504.f) s16 = (half_t)65504.f;
        const float s = (float)s16;
        const float inverse = 1.f / s;
        const float z = ZEROS ? fminf(fmaxf(__builtin_rintf(nearest_quotient(-lo, s, inverse)), 0.f), 15.f) : (float)kGq4Sym;
        // rint(q) by adding 1.5 2^23, which leaves it in the low bits (what is too large for that is beyond the clamp too); z and the bits of 1.5 2^23 come in once for a dword's eight.
        constexpr float kWhole = 12582912.f;
        const float least = kWhole - z, largest = kWhole + 15.f - z;
        const uint32_t rest = (uint32_t)z * 0x11111111u - 0x11111111u * 0x4b400000u;
#pragma unroll
        for (int j = g * PER; j < (g + 1) * PER; ++j) {
            uint32_t d = rest;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float c = __builtin_amdgcn_fmed3f(nearest_quotient(w[j][e], s, inverse) + kWhole, least, largest);
                d += __builtin_bit_cast(uint32_t, c) << (4 * ((e >> 1) + 4 * (e & 1)));
            }
            const int left = a.k - (cb * kGq4Cols + 32 * j + 8 * q);    // inputs there are from the piece's first on; the codes past them are 0
            if (left < 8) {
                uint32_t there = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) there |= (e < left ? 15u : 0u) << (4 * ((e >> 1) + 4 * (e & 1)));
                d &= there;
            }
            out[j] = odd ? 0u : d;
        }
        kept[g] = odd ? (uint16_t)0x7e00 : __builtin_bit_cast(uint16_t, s16);
        if constexpr (ZEROS) points[g] = odd ? (uint8_t)0 : (uint8_t)z;
    }
    // a row's groups by one store where all are there
    if (q == 0 && there) {
        const int64_t at = (int64_t)row * a.kg + cb * GROUPS;
        if ((cb + 1) * GROUPS <= a.kg) {
            reinterpret_cast<Gq4Any<decltype(kept)> *>(a.scales + at)->v = kept;
            if constexpr (ZEROS) reinterpret_cast<Gq4Any<decltype(points)> *>(a.zeros + at)->v = points;
        } else {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
                if (cb * GROUPS + g < a.kg) {
                    a.scales[at + g] = __builtin_bit_cast(half_t, (uint16_t)kept[g]);
                    if constexpr (ZEROS) a.zeros[at + g] = points[g];
                }
        }
    }
    if (!there) out = uint4_t{0, 0, 0, 0};
    *reinterpret_cast<uint4_t *>(a.codes + block * kGq4Block + (q * 16 + r) * 16) = out;
}

// Row-major codes, a byte each, to the layout (TILE) and back.
template <bool TILE>
__global__ __launch_bounds__(256) void gq4_retile_kernel(const uint8_t *in, int64_t ld, int n, int k, int cb, int64_t blocks, uint8_t *out)
{
    const int lane = (int)threadIdx.x & (kWave - 1), r = lane >> 2, q = lane & 3;
    for (int64_t block = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave; block < blocks; block += (int64_t)gridDim.x * 4) {
        const int row = (int)(block / cb) * kGq4Rows + r, c0 = (int)(block % cb) * kGq4Cols;
        const int64_t at = block * kGq4Block + (q * 16 + r) * 16;
        uint4_t v = {0, 0, 0, 0};
        if constexpr (!TILE) v = *reinterpret_cast<const uint4_t *>(in + at);
        if (row < n) {
            const int64_t base = (int64_t)row * ld;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int c = c0 + 32 * j + 8 * q + e, bit = 4 * ((e >> 1) + 4 * (e & 1));
                    if (c < k) {
                        if constexpr (TILE)
                            v[j] |= (in[base + c] & 15u) << bit;
                        else
                            out[base + c] = (uint8_t)((v[j] >> bit) & 15u);
                    }
                }
        }
        if constexpr (TILE) *reinterpret_cast<uint4_t *>(out + at) = v;
    }
}

// The values that codes stand for, rounded once to the type asked for.
template <class T, int SHIFT>
__global__ __launch_bounds__(256) void gq4_values_kernel(Gq4Weights w, int n, int k, int cb, int kg, int64_t blocks, typename T::type *out, int64_t ld)
{
    const int lane = (int)threadIdx.x & (kWave - 1), r = lane >> 2, q = lane & 3;
    const int64_t block = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    if (block >= blocks) return;
    const int row = (int)(block / cb) * kGq4Rows + r, b = (int)(block % cb);
    if (row >= n) return;
    const uint4_t v = *reinterpret_cast<const uint4_t *>(w.codes + block * kGq4Block + (q * 16 + r) * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c0 = b * kGq4Cols + 32 * j + 8 * q;
        if (c0 >= k) return;
        const int64_t g = (int64_t)row * kg + (c0 >> SHIFT);
        const float s = (float)w.scales[g];
        const int z = w.zeros ? (int)w.zeros[g] : kGq4Sym;
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)((int)((v[j] >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15u) - z) * s;
        store_piece<T, 8>(out + (int64_t)row * ld, c0, k, f);
    }
}

struct Gq4ActArgs {
    const void *dH, *G, *U;
    void *dG, *dU;
    int64_t h_ld, g_ld, u_ld, dg_ld, du_ld, pieces;
    int n, row_pieces;
};

// dU = dH silu(G),  dG = dH U sigma(G) (1 + G (1 - sigma(G))); a thread has 8 values of a row at a time.  dG may be G, dU may be U.
template <class T>
__global__ __launch_bounds__(256) void gq4_act_backward_kernel(Gq4ActArgs a)
{
    typedef typename T::type E;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / a.row_pieces;
        const int at = (int)(i % a.row_pieces) * 8;
        float h[8], g[8], u[8];
        load_piece<T, 8>(static_cast<const E *>(a.dH) + row * a.h_ld, at, a.n, h);
        load_piece<T, 8>(static_cast<const E *>(a.G) + row * a.g_ld, at, a.n, g);
        load_piece<T, 8>(static_cast<const E *>(a.U) + row * a.u_ld, at, a.n, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // (a G that overflowed when it was kept has the limits: at -inf both gradients are 0, at inf silu's is 1)
            constexpr float kMost = 3.402823466e38f;
            const Gq4Sigma sigma(g[e]);
            const float low = fmaxf(g[e], -kMost);
            u[e] = (sigma.s * (1.f + fminf(low, kMost) * (1.f - sigma.s * sigma.h)) * h[e]) * (sigma.h * u[e]);
            h[e] = (low * sigma.s) * (sigma.h * h[e]);
        }
        store_piece<T, 8>(static_cast<E *>(a.dG) + row * a.dg_ld, at, a.n, u);
        store_piece<T, 8>(static_cast<E *>(a.dU) + row * a.du_ld, at, a.n, h);
    }
}

// Sums of several workgroups, added in order; a thread has 8 of a token's results at a time.
template <class T, bool GATED>
__global__ __launch_bounds__(256) void gq4_finish_kernel(Gq4Split p, int m, int outs, int64_t pieces, void *y0, void *y1, void *y2, int64_t ld0, int64_t ld1, int64_t ld2)
{
    typedef typename T::type E;
    const int per_row = p.ld / 8;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per_row;
        const int at = (int)(i % per_row) * 8;
        float v[GATED ? 2 : 1][8];
#pragma unroll
        for (int u = 0; u < (GATED ? 2 : 1); ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] = 0.f;
        for (int z = 0; z < p.splits; ++z)
#pragma unroll
            for (int u = 0; u < (GATED ? 2 : 1); ++u) {
                const float4_t *q = reinterpret_cast<const float4_t *>(p.part + (((int64_t)z * (GATED ? 2 : 1) + u) * m + row) * p.ld + at);
                const float4_t a = q[0], b = q[1];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[u][e] += a[e];
                    v[u][4 + e] += b[e];
                }
            }
        if constexpr (GATED) {
            float h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = gq4_gated(v[0][e], v[1][e]);
            store_piece<T, 8>(static_cast<E *>(y0) + row * ld0, at, outs, h);
            if (y1) store_piece<T, 8>(static_cast<E *>(y1) + row * ld1, at, outs, v[0]);
            if (y2) store_piece<T, 8>(static_cast<E *>(y2) + row * ld2, at, outs, v[1]);
        } else
            store_piece<T, 8>(static_cast<E *>(y0) + row * ld0, at, outs, v[0]);
    }
}

int gq4_launch_finish(const Gq4Split &p, int m, int outs, bool gated, void *const (&y)[3], const int64_t (&y_ld)[3], int32_t dtype, hipStream_t st)
{
    const int64_t pieces = (int64_t)m * (p.ld / 8), groups = (pieces + 255) / 256;
    const dim3 grid((unsigned)(groups < 8192 ? groups : 8192)), threads(256);
    auto launch = [&](auto type, auto g) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_finish_kernel<decltype(type), decltype(g)::value>), grid, threads, 0, st, p, m, outs, pieces, y[0], y[1], y[2], y_ld[0],
                           y_ld[1], y_ld[2]);
    };
    if (dtype == SLIM_F16)
        gated ? launch(F16{}, std::true_type{}) : launch(F16{}, std::false_type{});
    else
        gated ? launch(BF16{}, std::true_type{}) : launch(BF16{}, std::false_type{});
    return hip_status(hipGetLastError());
}

template <class T, bool ZEROS>
static void launch_quant(const Gq4QuantArgs &a, int shift, hipStream_t st)
{
    const dim3 grid((unsigned)((a.blocks + 3) / 4)), threads(256);
    if (shift == 5)
        hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_quant_kernel<T, 5, ZEROS>), grid, threads, 0, st, a);
    else if (shift == 6)
        hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_quant_kernel<T, 6, ZEROS>), grid, threads, 0, st, a);
    else
        hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_quant_kernel<T, 7, ZEROS>), grid, threads, 0, st, a);
}
template <class T>
static void launch_values(const Gq4Weights &w, int n, int k, int shift, void *out, int64_t ld, hipStream_t st)
{
    const int cb = gq4_col_blocks(k), kg = gq4_groups(k, shift);
    const int64_t blocks = (int64_t)gq4_row_blocks(n) * cb;
    const dim3 grid((unsigned)((blocks + 3) / 4)), threads(256);
    typename T::type *o = static_cast<typename T::type *>(out);
    if (shift == 5)
        hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_values_kernel<T, 5>), grid, threads, 0, st, w, n, k, cb, kg, blocks, o, ld);
    else if (shift == 6)
        hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_values_kernel<T, 6>), grid, threads, 0, st, w, n, k, cb, kg, blocks, o, ld);
    else
        hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_values_kernel<T, 7>), grid, threads, 0, st, w, n, k, cb, kg, blocks, o, ld);
}

// The gated activation's gradient, for slim_group_q4_gated_backward (arguments checked there).
int gq4_launch_act_backward(const void *dH, int64_t h_ld, const void *G, int64_t g_ld, const void *U, int64_t u_ld, int32_t m, int32_t n, void *dG,
                            int64_t dg_ld, void *dU, int64_t du_ld, int32_t dtype, hipStream_t st)
{
    Gq4ActArgs a{dH, G, U, dG, dU, h_ld, g_ld, u_ld, dg_ld, du_ld, 0, n, (int)(((int64_t)n + 7) / 8)};
    a.pieces = (int64_t)m * a.row_pieces;
    const int64_t groups = (a.pieces + 255) / 256;
    const dim3 grid((unsigned)(groups < 8192 ? groups : 8192)), threads(256);
    if (dtype == SLIM_F16)
        hipLaunchKernelGGL(gq4_act_backward_kernel<F16>, grid, threads, 0, st, a);
    else
        hipLaunchKernelGGL(gq4_act_backward_kernel<BF16>, grid, threads, 0, st, a);
    return hip_status(hipGetLastError());
}

}  // namespace slim

using namespace slim;

extern "C" int slim_group_q4_sizes(int32_t n, int32_t k, int32_t group, size_t *codes_bytes, size_t *scales_bytes, size_t *zeros_bytes)
{
    const int shift = gq4_shift(group);
    if (n < 1 || k < 1 || k > kMaxK || n > (1 << 30) || shift < 0) return SLIM_ERR_SHAPE;
    const int64_t blocks = (int64_t)gq4_row_blocks(n) * gq4_col_blocks(k);
    if (blocks > INT32_MAX) return SLIM_ERR_SHAPE;
    if (codes_bytes) *codes_bytes = (size_t)blocks * kGq4Block;
    if (scales_bytes) *scales_bytes = (size_t)n * gq4_groups(k, shift) * sizeof(half_t);
    if (zeros_bytes) *zeros_bytes = (size_t)n * gq4_groups(k, shift);
    return SLIM_OK;
}

// A launch has fewer than 2^32 threads: 64 to each block of codes where they are made or read back.
static bool gq4_has_threads(int n, int k) { return (int64_t)gq4_row_blocks(n) * gq4_col_blocks(k) <= (1 << 26) - 4; }

extern "C" int slim_group_q4_weight(const void *W, int64_t ld, int32_t dtype, int32_t n, int32_t k, int32_t group, uint8_t *codes, slim_half *scales,
                                    uint8_t *zeros, void *stream)
{
    if (!W || !codes || !scales) return SLIM_ERR_NULL;
    if (slim_group_q4_sizes(n, k, group, nullptr, nullptr, nullptr) != SLIM_OK || ld < k || (!half_dtype(dtype) && dtype != SLIM_F32) || !gq4_has_threads(n, k)) return SLIM_ERR_SHAPE;
    if (!whole_elements(W, dtype) || !aligned16(codes) || (reinterpret_cast<uintptr_t>(scales) & 1u)) return SLIM_ERR_ALIGN;
    const int shift = gq4_shift(group);
    const Gq4QuantArgs a{W, ld, n, k, gq4_col_blocks(k), gq4_groups(k, shift), (int64_t)gq4_row_blocks(n) * gq4_col_blocks(k), codes,
                         reinterpret_cast<half_t *>(scales), zeros};
    hipStream_t st = static_cast<hipStream_t>(stream);
    auto launch = [&](auto type) {
        typedef decltype(type) T;
        if (zeros)
            launch_quant<T, true>(a, shift, st);
        else
            launch_quant<T, false>(a, shift, st);
    };
    if (dtype == SLIM_F32)
        launch(F32{});
    else if (dtype == SLIM_F16)
        launch(F16{});
    else
        launch(BF16{});
    return hip_status(hipGetLastError());
}

template <bool TILE>
static int gq4_retile(const uint8_t *in, uint8_t *out, int64_t ld, int32_t n, int32_t k, void *stream)
{
    if (!in || !out) return SLIM_ERR_NULL;
    if (slim_group_q4_sizes(n, k, 128, nullptr, nullptr, nullptr) != SLIM_OK || ld < k) return SLIM_ERR_SHAPE;
    if (!aligned16(TILE ? out : in)) return SLIM_ERR_ALIGN;
    const int cb = gq4_col_blocks(k);
    const int64_t blocks = (int64_t)gq4_row_blocks(n) * cb, groups = (blocks + 3) / 4;
    hipLaunchKernelGGL(gq4_retile_kernel<TILE>, dim3((unsigned)(groups < (1 << 20) ? groups : 1 << 20)), dim3(256), 0, static_cast<hipStream_t>(stream), in, ld,
                       n, k, cb, blocks, out);
    return hip_status(hipGetLastError());
}

extern "C" int slim_group_q4_tile(const uint8_t *in, int64_t ld, int32_t n, int32_t k, uint8_t *codes, void *stream)
{
    return gq4_retile<true>(in, codes, ld, n, k, stream);
}

extern "C" int slim_group_q4_untile(const uint8_t *codes, int32_t n, int32_t k, uint8_t *out, int64_t ld, void *stream)
{
    return gq4_retile<false>(codes, out, ld, n, k, stream);
}

extern "C" int slim_group_q4_values(const slim_group_q4_layer *layer, void *out, int64_t ld, int32_t dtype, void *stream)
{
    if (!out) return SLIM_ERR_NULL;
    int shift;
    const int status = gq4_check(layer, &shift);
    if (status != SLIM_OK) return status;
    if (ld < layer->k || (!half_dtype(dtype) && dtype != SLIM_F32) || !gq4_has_threads(layer->n, layer->k)) return SLIM_ERR_SHAPE;
    if (!whole_elements(out, dtype)) return SLIM_ERR_ALIGN;
    const Gq4Weights w = gq4_weights(layer);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == SLIM_F32)
        launch_values<F32>(w, layer->n, layer->k, shift, out, ld, st);
    else if (dtype == SLIM_F16)
        launch_values<F16>(w, layer->n, layer->k, shift, out, ld, st);
    else
        launch_values<BF16>(w, layer->n, layer->k, shift, out, ld, st);
    return hip_status(hipGetLastError());
}
