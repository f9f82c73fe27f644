// 8-bit quantization with a scale for each block of 128: of a layer's inputs, 128 inputs of a token to a scale, where they are
// made (the norm that adds the residual; the gated activation), and of weights, 128 x 128 to a scale.
//
//   code = E4M3(z * (448 / top)),  value = code * scale,  scale = top / 448,  top = max |z| of the block (2^-100 at least)
//
// The norm's output is y = z rstd with z = h gain, h = x + residual and rstd = 1 / sqrt(mean(h^2) + eps): y's codes are z's, since rstd
// multiplies top too, and only the scale, top / 448 * rstd, waits for the sum over the row.  So a row's codes do not depend
// on the order of that sum, and they are on their way while it is made.
#include <hip/hip_runtime.h>

#include "slim_block_fp8.h"

namespace slim {

// Largest of the 16 lanes that hold a block (8 values each); every lane gets it.
__device__ __forceinline__ uint32_t block_top(uint32_t t)
{
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x128, 0xf, 0xf, true));     // row_ror:8
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x124, 0xf, 0xf, true));
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x122, 0xf, 0xf, true));
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x121, 0xf, 0xf, true));
    return t;
}

// Codes of 8 values, given their block's top.
__device__ __forceinline__ uint2_t eight_codes(const float (&z)[8], float top)
{
    const float inv = kFp8Max / top;
    uint2_t c;
    c[0] = four_fp8(z[0] * inv, z[1] * inv, z[2] * inv, z[3] * inv);
    c[1] = four_fp8(z[4] * inv, z[5] * inv, z[6] * inv, z[7] * inv);
    return c;
}

struct NormArgs {
    const void *X, *res, *gain;
    void *H, *Y;
    int64_t x_ld, res_ld, h_ld, y_ld;
    uint8_t *codes;
    float *scales;
    int m, k, kb;
    float eps;
    bool gain32;
};

// A piece of 8 elements of a row as they are stored, zeros from element `len` on.
template <class T>
__device__ __forceinline__ typename Piece<T, 8>::vec raw_piece(const typename T::type *row, int at, int len)
{
    if (at + 8 <= len) return Piece<T, 8>::load(row + at);
    typename Piece<T, 8>::vec v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = at + e < len ? row[at + e] : (typename T::type)0.f;
    return v;
}
// h of one piece of 8.
template <class T>
__device__ __forceinline__ void norm_load(const NormArgs &a, int64_t row, int at, float (&h)[8])
{
    typedef typename T::type E;
    load_piece<T>(static_cast<const E *>(a.X) + row * a.x_ld, at, a.k, h);
    if (a.res) {
        float r[8];
        load_piece<T>(static_cast<const E *>(a.res) + row * a.res_ld, at, a.k, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] += r[e];
    }
}
template <class T>
__device__ __forceinline__ void gain_piece(const NormArgs &a, int at, float (&g)[8])
{
    if (!a.gain) {
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = 1.0f;
    } else if (a.gain32) {
        load_piece<F32>(static_cast<const float *>(a.gain), at, a.k, g);
    } else {
        load_piece<T>(static_cast<const typename T::type *>(a.gain), at, a.k, g);
    }
}

// A row per workgroup, NV pieces of 8 values per lane, held in registers from the one read to the last write (more rows than
// workgroups fit into a grid are walked).  LONG: rows that do not fit so are read twice, the sum first.
// Bound by memory: 4096 x 8192 in fp16 with a residual moves 236 MB in 46 us, 5.1 TB/s (a large copy: 5.15); 1777 x 5003 in bf16, whose rows begin
// at odd elements, 80 MB in 18.8 us (13 % of it for that).  H, which nothing reads soon, is stored past the caches' turn (49.4 and 19.5 us without that); the codes are not:
// it would be 44.8 here and 9 us more in the product that reads them (the feed-forward part of 4096 x 11008 at 512 tokens 108 -> 117 us).  One row of 8192 takes 3.7 us: the launch, one read, the sum across
// wavefronts, one write.  Workgroups that stay and walk the rows with the next row's loads under way, 2 to 32 of them per compute unit, took 48 to 57 us.
// 1 / sqrt and not the approximation: once per row.
template <class T, int NV, bool LONG>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs a)
{
    typedef typename T::type E;
    typedef typename Piece<T, 8>::vec V;
    __shared__ float red[2][16];
    const int kp = a.kb * kBlk, step = 8 * (int)blockDim.x, waves = (int)blockDim.x / kWave, first = 8 * (int)threadIdx.x;
    int turn = 0;

    // 1 / root mean square of a row from this lane's share of its squares' sum
    auto factor = [&](float s) {
        s = wave_sum(s);
        if (waves > 1) {
            // (two sets in turn: a wavefront that is a row ahead does not overwrite what another still reads)
            if ((threadIdx.x & (kWave - 1)) == 0) red[turn][threadIdx.x / kWave] = s;
            __syncthreads();
            s = 0.f;
            for (int w = 0; w < waves; ++w) s += red[turn][w];
            turn ^= 1;
        }
        return 1.0f / sqrtf(s / (float)a.k + a.eps);
    };
    // codes of a piece, and what its scale is but for the row's factor (every lane of the block returns it)
    auto encode = [&](int64_t row, int at, const float(&z)[8]) {
        const float top = floored_top(block_top(top_of(z)));
        *reinterpret_cast<uint2_t *>(a.codes + row * kp + at) = eight_codes(z, top);
        return top / kFp8Max;
    };
    auto finish = [&](int64_t row, int at, float sc, float rstd, float(&z)[8]) {
        if ((threadIdx.x & 15) == 0) a.scales[row * a.kb + at / kBlk] = sc * rstd;
        if (a.Y) {
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] *= rstd;
            store_piece<T>(static_cast<E *>(a.Y) + row * a.y_ld, at, a.k, z);
        }
    };

    if constexpr (!LONG) {
        for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x) {
            // all loads first, as they are stored
            V x[NV], r[NV];
#pragma unroll
            for (int p = 0; p < NV; ++p) {
                const int at = first + p * step;
                if (at < kp) {
                    x[p] = raw_piece<T>(static_cast<const E *>(a.X) + row * a.x_ld, at, a.k);
                    if (a.res) r[p] = raw_piece<T>(static_cast<const E *>(a.res) + row * a.res_ld, at, a.k);
                }
            }
            float z[NV][8], sc[NV], sum = 0.f;
#pragma unroll
            for (int p = 0; p < NV; ++p) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    z[p][e] = (float)x[p][e];
                    if (a.res) z[p][e] += (float)r[p][e];
                }
            }
#pragma unroll
            for (int p = 0; p < NV; ++p) {
                const int at = first + p * step;
                sc[p] = 0.f;
                if (at < kp) {
                    float g[8];
                    gain_piece<T>(a, at, g);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum += z[p][e] * z[p][e];
                    if (a.H) store_piece<T, 8, true>(static_cast<E *>(a.H) + row * a.h_ld, at, a.k, z[p]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[p][e] *= g[e];
                    sc[p] = encode(row, at, z[p]);
                }
            }
            const float rstd = factor(sum);
#pragma unroll
            for (int p = 0; p < NV; ++p)
                if (first + p * step < kp) finish(row, first + p * step, sc[p], rstd, z[p]);
        }
    } else {
        for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x) {
            float h[8], g[8], sum = 0.f;
            for (int at = first; at < kp; at += step) {
                norm_load<T>(a, row, at, h);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += h[e] * h[e];
            }
            const float rstd = factor(sum);
            for (int at = first; at < kp; at += step) {
                norm_load<T>(a, row, at, h);            // (H or Y may be X or the residual: a piece is read and written by one lane, here last)
                if (a.H) store_piece<T, 8, true>(static_cast<E *>(a.H) + row * a.h_ld, at, a.k, h);
                gain_piece<T>(a, at, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[e] *= g[e];
                finish(row, at, encode(row, at, h), rstd, h);
            }
        }
    }
}

struct ActArgs {
    const void *G, *U;
    int64_t g_ld, u_ld;
    uint8_t *codes;
    float *scales;
    int64_t pieces;       // of 8 values, all rows
    int k, kb;
};

// 16 lanes per block.  A lane takes one piece per round; nothing is shared between blocks, so the largest of a block is found in registers and the
// values are read once.  Bound by memory: 2048 x 11008 in bf16, gated, moves 114 MB in 23 us, 5.0 TB/s (a large copy: 5.15); 16 x 13824 takes
// 3.0 us, a launch and one dependent access.  exp and the division in 32 bits; the result is rounded once, to its code.
// (Codes stored past the caches' turn: 23 us, and as much more in the product that reads them at 512 tokens.)
template <class T, bool SILU>
__global__ __launch_bounds__(256) void act_kernel(ActArgs a)
{
    typedef typename T::type E;
    const int per_row = a.kb * 16;
    for (int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x; p < a.pieces; p += (int64_t)gridDim.x * 256) {
        const int64_t row = p / per_row;
        const int at = 8 * (int)(p - row * per_row);
        float v[8];
        load_piece<T>(static_cast<const E *>(a.G) + row * a.g_ld, at, a.k, v);
        if constexpr (SILU) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = v[e] / (1.0f + __expf(-v[e]));
        }
        if (a.U) {
            float u[8];
            load_piece<T>(static_cast<const E *>(a.U) + row * a.u_ld, at, a.k, u);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= u[e];
        }
        const float top = floored_top(block_top(top_of(v)));
        *reinterpret_cast<uint2_t *>(a.codes + p * 8) = eight_codes(v, top);
        if ((threadIdx.x & 15) == 0) a.scales[p / 16] = top / kFp8Max;
    }
}

// Place of a 16-byte piece of a pair of tiles in LDS: a row's pieces, 256 bytes apart, go to different banks.
__device__ __forceinline__ uint32_t wtile_lds(uint32_t place)
{
    const uint32_t piece = place >> 4;
    return ((piece ^ ((piece >> 4) & 7u)) << 4) | (place & 15u);
}

// One workgroup per 128 x 128 weights: in registers while their largest is found (so they are read once), then through LDS into the order of the tiles.
// VEC values of 16 bytes per lane and load.  Bound by memory: 28672 x 8192 in bf16 moves 705 MB in 123 us, 5.7 TB/s (a large copy: 5.15, half of it
// writes; here a third); 4096 x 4096 in fp32 84 MB in 14.2 us.  The codes are stored past the caches' turn (128 and 14.4 us without; loads so are slower, 16 us the second).
template <class T>
__global__ __launch_bounds__(256) void weight_kernel(const typename T::type *W, int64_t ld, int n, int k, int kb, uint8_t *codes, float *scales)
{
    constexpr int VEC = 16 / sizeof(typename T::type), LANES = kBlk / VEC, ROWS = 256 / LANES, PASSES = kBlk / ROWS;
    __shared__ __align__(16) uint8_t tile[2 * kWTileBytes];
    __shared__ uint32_t red[4];
    const int bk = (int)(blockIdx.x % (unsigned)kb), bn = (int)(blockIdx.x / (unsigned)kb);
    const int c = (int)threadIdx.x % LANES * VEC, r0 = (int)threadIdx.x / LANES;
    float v[PASSES][VEC];
    uint32_t t = 0;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int64_t o = (int64_t)bn * kBlk + p * ROWS + r0;
        if (o < n) {
            load_piece<T>(W + o * ld, bk * kBlk + c, k, v[p]);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[p][e] = 0.f;
        }
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) t = max(t, top_of(v[p]));
    t = block_top(t);
    t = max(t, (uint32_t)__shfl_xor((int)t, 16, kWave));
    t = max(t, (uint32_t)__shfl_xor((int)t, 32, kWave));
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = t;
    __syncthreads();
    const float top = floored_top(max(max(red[0], red[1]), max(red[2], red[3])));
    const float inv = kFp8Max / top;
    if (threadIdx.x == 0) scales[blockIdx.x] = top / kFp8Max;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const uint32_t o = (uint32_t)(p * ROWS + r0);
        const uint32_t at = (o >> 6) * (uint32_t)kWTileBytes + wtile_place(o & 63u, (uint32_t)c);
#pragma unroll
        for (int e = 0; e < VEC; e += 4)
            *reinterpret_cast<uint32_t *>(tile + wtile_lds(at + e)) =
                four_fp8(v[p][e] * inv, v[p][e + 1] * inv, v[p][e + 2] * inv, v[p][e + 3] * inv);
    }
    __syncthreads();
    const int tiles = bn * 2 + 1 < (n + kWTileRows - 1) / kWTileRows ? 2 : 1;     // of 64 rows in this block
    for (int u = 0; u < tiles; ++u) {
        uint8_t *out = codes + ((int64_t)(bn * 2 + u) * kb + bk) * kWTileBytes;
#pragma unroll
        for (int s = 0; s < kWTileBytes / 4096; ++s) {
            const uint32_t at = (uint32_t)s * 4096u + threadIdx.x * 16u;
            __builtin_nontemporal_store(*reinterpret_cast<const uint4_t *>(tile + wtile_lds((uint32_t)u * kWTileBytes + at)), reinterpret_cast<uint4_t *>(out + at));
        }
    }
}

// Row-major codes to tiles (TILE), or back: one lane per piece of 16 inputs of a row of the padded matrix.  Once per layer, so no more than right.
template <bool TILE>
__global__ __launch_bounds__(256) void retile_kernel(const uint8_t *in, int64_t ld, int n, int k, int kb, int64_t pieces, uint8_t *out)
{
    const int per_row = kb * 8;
    for (int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x; p < pieces; p += (int64_t)gridDim.x * 256) {
        const int64_t o = p / per_row;
        const int i = 16 * (int)(p - o * per_row);
        const int64_t at = ((o >> 6) * kb + (i >> 7)) * kWTileBytes + wtile_place((uint32_t)(o & 63), (uint32_t)(i & 127));
        if constexpr (TILE) {
            uint4_t v = {0, 0, 0, 0};
            if (o < n) {
                const uint8_t *row = in + o * ld;
                if (i + 16 <= k) {
                    __builtin_memcpy(&v, row + i, 16);
                } else {
                    for (int e = 0; i + e < k; ++e) v[e >> 2] |= (uint32_t)row[i + e] << (8 * (e & 3));
                }
            }
            *reinterpret_cast<uint4_t *>(out + at) = v;
        } else if (o < n) {
            const uint4_t v = *reinterpret_cast<const uint4_t *>(in + at);
            uint8_t *row = out + o * ld;
            if (i + 16 <= k) {
                __builtin_memcpy(row + i, &v, 16);
            } else {
                for (int e = 0; i + e < k; ++e) row[i + e] = (uint8_t)(v[e >> 2] >> (8 * (e & 3)));
            }
        }
    }
}

static bool element_aligned(const void *p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == SLIM_F32 ? 3u : 1u)) == 0; }
static bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
static bool half_type(int dtype) { return dtype == SLIM_F16 || dtype == SLIM_BF16; }

template <class T, int NV, bool LONG>
static void launch_norm(const NormArgs &a, int threads, hipStream_t st)
{
    const unsigned grid = (unsigned)(a.m < (1 << 20) ? a.m : 1 << 20);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_kernel<T, NV, LONG>), dim3(grid), dim3((unsigned)threads), 0, st, a);
}

// Pieces per lane: one, the shortest way through a row (1 x 8192: 3.8 us, with two 4.0, with four 5.3); two where that would take more than
// half of a compute unit's wavefronts for one row and there are rows for all of them (4096 x 8192: 59 us with one, 48 with two, 51 with four;
// 512 x 8192: 9.0, 8.4, 9.2; 4096 x 4096 and 333 x 4100 are faster with one); more only where the row asks for them.
template <class T>
static void launch_norm_of(const NormArgs &a, hipStream_t st)
{
    const int pieces = a.kb * 16;
    auto threads = [&](int nv) { return (pieces + nv * kWave - 1) / (nv * kWave) * kWave; };
    if (pieces <= 512 || (pieces <= 1024 && a.m <= device_info().cus))
        launch_norm<T, 1, false>(a, threads(1), st);
    else if (pieces <= 2048)
        launch_norm<T, 2, false>(a, threads(2), st);
    else if (pieces <= 4096)
        launch_norm<T, 4, false>(a, threads(4), st);
    else
        launch_norm<T, 1, true>(a, 1024, st);
}

template <class T>
static void launch_weight(const void *W, int64_t ld, int n, int k, uint8_t *codes, float *scales, hipStream_t st)
{
    const int kb = blocks_of(k);
    hipLaunchKernelGGL(weight_kernel<T>, dim3((unsigned)((int64_t)blocks_of(n) * kb)), dim3(256), 0, st,
                       static_cast<const typename T::type *>(W), ld, n, k, kb, codes, scales);
}

}  // namespace slim

using namespace slim;

extern "C" int slim_block_fp8_sizes(int32_t m, int32_t k, size_t *codes_bytes, size_t *scales_bytes)
{
    if (m < 1 || k < 1 || k > kMaxK) return SLIM_ERR_SHAPE;
    if (codes_bytes) *codes_bytes = (size_t)m * blocks_of(k) * kBlk;
    if (scales_bytes) *scales_bytes = (size_t)m * blocks_of(k) * sizeof(float);
    return SLIM_OK;
}

extern "C" int slim_block_fp8_weight_sizes(int32_t n, int32_t k, size_t *codes_bytes, size_t *scales_bytes)
{
    if (n < 1 || k < 1 || k > kMaxK || (int64_t)blocks_of(n) * blocks_of(k) > INT32_MAX) return SLIM_ERR_SHAPE;
    if (codes_bytes) *codes_bytes = (size_t)wtile_rows(n) * blocks_of(k) * kWTileBytes;
    if (scales_bytes) *scales_bytes = (size_t)blocks_of(n) * blocks_of(k) * sizeof(float);
    return SLIM_OK;
}

extern "C" int slim_block_fp8_norm(const void *X, int64_t x_ld, const void *residual, int64_t residual_ld, const void *gain,
                                   int32_t gain_dtype, int32_t dtype, int32_t m, int32_t k, float eps, void *H, int64_t h_ld, void *Y,
                                   int64_t y_ld, uint8_t *codes, float *scales, void *stream)
{
    if (!X || !codes || !scales) return SLIM_ERR_NULL;
    if (m < 1 || k < 1 || k > kMaxK || !half_type(dtype) || (gain && gain_dtype != dtype && gain_dtype != SLIM_F32) || !(eps >= 0.f))
        return SLIM_ERR_SHAPE;
    if (x_ld < k || (residual && residual_ld < k) || (H && h_ld < k) || (Y && y_ld < k)) return SLIM_ERR_SHAPE;
    if (!element_aligned(X, dtype) || !element_aligned(residual, dtype) || !element_aligned(gain, gain_dtype) || !element_aligned(H, dtype) ||
        !element_aligned(Y, dtype) || !aligned16(codes) || !aligned4(scales))
        return SLIM_ERR_ALIGN;
    const NormArgs a{X, residual, gain, H, Y, x_ld, residual_ld, h_ld, y_ld, codes, scales, m, k, blocks_of(k), eps, gain_dtype == SLIM_F32};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == SLIM_F16)
        launch_norm_of<F16>(a, st);
    else
        launch_norm_of<BF16>(a, st);
    return hip_status(hipGetLastError());
}

extern "C" int slim_block_fp8_act(const void *G, int64_t g_ld, const void *U, int64_t u_ld, int32_t act, int32_t dtype, int32_t m, int32_t k,
                                  uint8_t *codes, float *scales, void *stream)
{
    if (!G || !codes || !scales) return SLIM_ERR_NULL;
    if (m < 1 || k < 1 || k > kMaxK || !half_type(dtype) || (act != SLIM_ACT_NONE && act != SLIM_ACT_SILU)) return SLIM_ERR_SHAPE;
    if (g_ld < k || (U && u_ld < k)) return SLIM_ERR_SHAPE;
    if (!element_aligned(G, dtype) || !element_aligned(U, dtype) || !aligned16(codes) || !aligned4(scales)) return SLIM_ERR_ALIGN;
    const int kb = blocks_of(k);
    const ActArgs a{G, U, g_ld, u_ld, codes, scales, (int64_t)m * kb * 16, k, kb};
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t groups = (a.pieces + 255) / 256;
    const dim3 grid((unsigned)(groups < 8192 ? groups : 8192)), threads(256);
    if (dtype == SLIM_F16) {
        if (act == SLIM_ACT_SILU)
            hipLaunchKernelGGL(HIP_KERNEL_NAME(act_kernel<F16, true>), grid, threads, 0, st, a);
        else
            hipLaunchKernelGGL(HIP_KERNEL_NAME(act_kernel<F16, false>), grid, threads, 0, st, a);
    } else {
        if (act == SLIM_ACT_SILU)
            hipLaunchKernelGGL(HIP_KERNEL_NAME(act_kernel<BF16, true>), grid, threads, 0, st, a);
        else
            hipLaunchKernelGGL(HIP_KERNEL_NAME(act_kernel<BF16, false>), grid, threads, 0, st, a);
    }
    return hip_status(hipGetLastError());
}

extern "C" int slim_block_fp8_weight(const void *W, int64_t ld, int32_t dtype, int32_t n, int32_t k, uint8_t *codes, float *scales, void *stream)
{
    if (!W || !codes || !scales) return SLIM_ERR_NULL;
    if (slim_block_fp8_weight_sizes(n, k, nullptr, nullptr) != SLIM_OK || ld < k || (!half_type(dtype) && dtype != SLIM_F32)) return SLIM_ERR_SHAPE;
    if (!element_aligned(W, dtype) || !aligned16(codes) || !aligned4(scales)) return SLIM_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == SLIM_F32)
        launch_weight<F32>(W, ld, n, k, codes, scales, st);
    else if (dtype == SLIM_F16)
        launch_weight<F16>(W, ld, n, k, codes, scales, st);
    else
        launch_weight<BF16>(W, ld, n, k, codes, scales, st);
    return hip_status(hipGetLastError());
}

template <bool TILE>
static int retile(const uint8_t *in, uint8_t *out, int64_t ld, int32_t n, int32_t k, void *stream)
{
    if (!in || !out) return SLIM_ERR_NULL;
    if (slim_block_fp8_weight_sizes(n, k, nullptr, nullptr) != SLIM_OK || ld < k) return SLIM_ERR_SHAPE;
    if (!aligned16(TILE ? out : in)) return SLIM_ERR_ALIGN;
    const int kb = blocks_of(k);
    const int64_t pieces = (int64_t)wtile_rows(n) * kWTileRows * kb * 8;
    const int64_t groups = (pieces + 255) / 256;
    hipLaunchKernelGGL(retile_kernel<TILE>, dim3((unsigned)(groups < (1 << 20) ? groups : 1 << 20)), dim3(256), 0,
                       static_cast<hipStream_t>(stream), in, ld, n, k, kb, pieces, out);
    return hip_status(hipGetLastError());
}

extern "C" int slim_block_fp8_tile(const uint8_t *in, int64_t ld, int32_t n, int32_t k, uint8_t *codes, void *stream)
{
    return retile<true>(in, codes, ld, n, k, stream);
}

extern "C" int slim_block_fp8_untile(const uint8_t *codes, int32_t n, int32_t k, uint8_t *out, int64_t ld, void *stream)
{
    return retile<false>(codes, out, ld, n, k, stream);
}
