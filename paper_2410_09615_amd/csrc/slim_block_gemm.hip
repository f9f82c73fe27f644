// Product of 8-bit inputs and 8-bit weights, a scale for each 128 inputs of a token and each 128 x 128 weights:
//   Y[t][o] = sum over blocks b of  xs[t][b] ws[o / 128][b] * sum over the block's inputs i of X[t][i] W[o][i].
// A block's inner sum starts from zero and is added to the fp32 accumulator with the product of the two scales, and each result
// is rounded once.  The weights are the A operand of the matrix instructions (rows of a result tile), the tokens the B operand (columns):
// a lane's results all have its token's scale.
//
// The inner sum is one V_MFMA_F32_16X16X128_F8F6F4, or, EXACT, four V_MFMA_F32_16X16X32_F16 on the codes as fp16 numbers (which they are
// exactly).  The 8-bit instruction aligns the eight products of a piece of 8 inputs with the largest of them and cuts what
// is more than 13 bits below it (measured with single products; between pieces, and in the 16-bit instruction, nothing above 2^-23 is lost).
// On blocks as they are quantized here that is 1.5e-5 to 8e-5 of a result (2-norm), below the 2.1e-4 of its rounding to fp16
// and far below what 8-bit codes carry; results in fp32 are asked for to be better than that, and the 16-bit instructions are
// half as fast.  So results in fp32 are EXACT, as is the kernel for few tokens, which waits for memory either way.
#include <hip/hip_runtime.h>

#include "slim_block_fp8.h"
#include "slim_mma.h"

namespace slim {

typedef int int8v_t __attribute__((ext_vector_type(8)));

struct BlockGemmArgs {
    const uint8_t *W;        // tiles of 64 x 128
    const float *ws;         // [row blocks][kb]
    const uint8_t *X;        // [m][128 kb]
    const float *xs;         // [m][kb]
    void *Y;
    int64_t y_ld;
    int n, m, kb, tiles_o, tiles_t;
};

// The 32 codes of a row or token that a lane holds of a block: as they are, or as fp16 numbers.
template <bool EXACT>
struct Codes;
template <>
struct Codes<false> {
    uint4_t h[2];
    __device__ __forceinline__ Codes() {}
    __device__ __forceinline__ Codes(uint4_t h0, uint4_t h1) : h{h0, h1} {}
};
template <>
struct Codes<true> {
    half8_t c[4];
    __device__ __forceinline__ Codes() {}
    __device__ __forceinline__ Codes(uint4_t h0, uint4_t h1)
    {
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const uint32_t v = d < 4 ? h0[d] : h1[d - 4];
            const half2_t lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)v, 1.0f, false);
            const half2_t hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)v, 1.0f, true);
            c[d / 2][4 * (d & 1)] = lo[0];
            c[d / 2][4 * (d & 1) + 1] = lo[1];
            c[d / 2][4 * (d & 1) + 2] = hi[0];
            c[d / 2][4 * (d & 1) + 3] = hi[1];
        }
    }
};

__device__ __forceinline__ float4_t block_product(const Codes<true> &a, const Codes<true> &b)
{
    float4_t p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 4; ++c) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.c[c], b.c[c], p, 0, 0, 0);
    return p;
}

__device__ __forceinline__ float4_t block_product(const Codes<false> &x, const Codes<false> &y)
{
    const uint4_t a0 = x.h[0], a1 = x.h[1], b0 = y.h[0], b1 = y.h[1];
    const int8v_t a = {(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
    const int8v_t b = {(int)b0[0], (int)b0[1], (int)b0[2], (int)b0[3], (int)b1[0], (int)b1[1], (int)b1[2], (int)b1[3]};
    // (format 0 of both operands is E4M3; without scales of its own)
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, float4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}

// ---- few tokens: the weights are streamed once, each wavefront of a workgroup a share of the blocks ----
// FR fragments of 16 rows and TB tiles of 16 tokens per workgroup.  Wavefront w takes blocks w, w + S, ...; the S partial results meet in LDS
// and are added in order.
template <int FR, int TB, class T>
__global__ __launch_bounds__(1024) void block_stream_kernel(BlockGemmArgs a)
{
    extern __shared__ __align__(16) float4_t part[];       // [S][FR * TB][64]
    constexpr int U = FR * TB >= 8 ? 1 : FR * TB >= 4 ? 2 : 4;
    const int S = (int)blockDim.x / kWave, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x & (kWave - 1);
    const int f0 = (int)blockIdx.x * FR, rt = f0 >> 2, t0 = f0 & 3, j = lane & 15, q = lane >> 4;
    const uint32_t kp = (uint32_t)a.kb * kBlk;
    const uint8_t *W = a.W + (int64_t)rt * a.kb * kWTileBytes + t0 * 2048 + lane * 16;
    const float *ws = a.ws + (int64_t)(rt >> 1) * a.kb;
    const rsrc_t xd = make_rsrc(a.X, (uint32_t)a.m * kp), sd = make_rsrc(a.xs, (uint32_t)a.m * (uint32_t)a.kb * 4u);

    float4_t acc[FR][TB];
#pragma unroll
    for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int t = 0; t < TB; ++t) acc[f][t] = float4_t{0.f, 0.f, 0.f, 0.f};

    for (int b0 = w; b0 < a.kb; b0 += S * U) {
        uint4_t wv[U][FR][2], xv[U][TB][2];
        float s[U][TB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int b = b0 + u * S;
            // blocks past the end: the last one again, with scale zero (a NaN among its codes is in the result anyway)
            const int bc = b < a.kb ? b : a.kb - 1;
#pragma unroll
            for (int f = 0; f < FR; ++f)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    wv[u][f][h] = *reinterpret_cast<const uint4_t *>(W + (int64_t)bc * kWTileBytes + f * 2048 + h * 1024);
            const float wsb = b < a.kb ? ws[bc] : 0.f;
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                const uint32_t row = (uint32_t)(t * 16 + j);
#pragma unroll
                for (int h = 0; h < 2; ++h) xv[u][t][h] = load16(xd, row * kp + (uint32_t)q * 16u, (uint32_t)bc * kBlk + (uint32_t)h * 64u);
                const uint32_t sv = __builtin_amdgcn_raw_buffer_load_b32(sd, (int)((row * (uint32_t)a.kb + (uint32_t)bc) * 4u), 0, 0);
                s[u][t] = __builtin_bit_cast(float, sv) * wsb;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Codes<true> x[TB];
#pragma unroll
            for (int t = 0; t < TB; ++t) x[t] = Codes<true>(xv[u][t][0], xv[u][t][1]);
#pragma unroll
            for (int f = 0; f < FR; ++f) {
                const Codes<true> wf(wv[u][f][0], wv[u][f][1]);
#pragma unroll
                for (int t = 0; t < TB; ++t) {
                    const float4_t p = block_product(wf, x[t]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[f][t][r] = __builtin_fmaf(p[r], s[u][t], acc[f][t][r]);
                }
            }
        }
    }
#pragma unroll
    for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int t = 0; t < TB; ++t) part[(w * FR * TB + f * TB + t) * kWave + lane] = acc[f][t];
    __syncthreads();
    for (int i = w; i < FR * TB; i += S) {
        float4_t v = part[i * kWave + lane];
        for (int z = 1; z < S; ++z) v += part[(z * FR * TB + i) * kWave + lane];
        const int tok = (i % TB) * 16 + j, o = rt * kWTileRows + 16 * q + 4 * (t0 + i / TB);
        if (tok < a.m) {
            const float y[4] = {v[0], v[1], v[2], v[3]};
            store_piece<T>(static_cast<typename T::type *>(a.Y) + tok * a.y_ld, o, a.n, y);
        }
    }
}

// ---- many tokens: tiles through LDS ----
// A workgroup of WR x WT wavefronts has a tile of 16 AF WR rows x 16 BF WT tokens; STAGES buffers of 128 inputs are
// filled by loads that write LDS directly, STAGES - 1 blocks ahead.  A wavefront waits until no more of its loads are under way than the later
// blocks' pieces, which its pieces of this one are not among; the barrier after it makes that everyone's.  The tokens' scales are
// fetched for four blocks at a time (they are next to one another), into two buffers of their own, with the pieces of the first of
// the four: a wait that leaves out of account that those are more loads ends the later for it, never sooner.
template <int WR, int WT, int AF, int BF, int STAGES, bool EXACT, class T>
__global__ __launch_bounds__(WR *WT *kWave, 2) void block_tile_kernel(BlockGemmArgs a)
{
    constexpr int WAVES = WR * WT, BM = 16 * AF * WR, BN = 16 * BF * WT;
    constexpr int WB = BM * kBlk, XB = BN * kBlk, SL = (BN + 63) / 64, SB = SL * 1024, STAGE = WB + XB, SCALES = STAGES * STAGE;
    constexpr int WL = WB / 1024 / WAVES, XL = XB / 1024 / WAVES, LOADS = WL + XL;
    static_assert(WL * WAVES * 1024 == WB && XL * WAVES * 1024 == XB && BM % kWTileRows == 0 && AF % 4 == 0, "tile");
    static_assert(AF * 16 == 64 || (AF * 16) % kBlk == 0, "a wavefront's rows have one scale per block");
    static_assert(SL <= WAVES && STAGES <= 4, "scales");
    extern __shared__ __align__(16) uint8_t lds[];
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x & (kWave - 1);
    const int wr = w % WR, wt = w / WR, j = lane & 15, q = lane >> 4;
    const int gx = a.tiles_o * a.tiles_t;
    const int qx = gx % kDies == 0 ? ((int)blockIdx.x % kDies) * (gx / kDies) + (int)blockIdx.x / kDies : (int)blockIdx.x;
    const int tile = blocked_tile(qx, a.tiles_o, a.tiles_t);
    const int o0 = tile % a.tiles_o * BM, tok0 = tile / a.tiles_o * BN;
    const uint32_t kp = (uint32_t)a.kb * kBlk;
    const int rows = min(BM, (a.n - o0 + kWTileRows - 1) / kWTileRows * kWTileRows), toks = min(BN, a.m - tok0);
    const rsrc_t wd = make_rsrc(a.W + (int64_t)o0 * kp, (uint32_t)rows * kp);
    const rsrc_t xd = make_rsrc(a.X + (int64_t)tok0 * kp, (uint32_t)toks * kp);
    const rsrc_t sd = make_rsrc(a.xs + (int64_t)tok0 * a.kb, (uint32_t)toks * (uint32_t)a.kb * 4u);
    // rows past the layer's last block of 128 are zeros: any scale will do
    const int rb = min((o0 + wr * AF * 16) / kBlk, (a.n - 1) / kBlk);
    const float *ws = a.ws + (int64_t)rb * a.kb;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;

    // this wavefront's shares of a block: pieces of a KiB of the weight tiles, and groups of eight tokens whose eight 16-byte pieces are put in another
    // order in each of eight rows, so that a fragment's reads find all banks
    uint32_t woff[WL], xoff[XL];
#pragma unroll
    for (int i = 0; i < WL; ++i) {
        const int piece = w * WL + i;
        woff[i] = (uint32_t)(piece / 8) * (uint32_t)a.kb * kWTileBytes + (uint32_t)(piece % 8) * 1024u + (uint32_t)lane * 16u;
    }
#pragma unroll
    for (int i = 0; i < XL; ++i) xoff[i] = (uint32_t)((w * XL + i) * 8 + lane / 8) * kp + (uint32_t)((lane & 7) ^ (lane / 8)) * 16u;
    const uint32_t soff = (uint32_t)(w * 64 + lane) * (uint32_t)a.kb * 4u;
    auto fetch = [&](int b) {
        const uint32_t base = lds0 + (uint32_t)(b % STAGES) * STAGE;
#pragma unroll
        for (int i = 0; i < WL; ++i) load_to_lds(wd, woff[i], (uint32_t)b * kWTileBytes, base + (uint32_t)(w * WL + i) * 1024u);
#pragma unroll
        for (int i = 0; i < XL; ++i) load_to_lds(xd, xoff[i], (uint32_t)b * kBlk, base + WB + (uint32_t)(w * XL + i) * 1024u);
        if ((b & 3) == 0 && w < SL) load_to_lds(sd, soff + (uint32_t)b * 4u, 0u, lds0 + SCALES + (uint32_t)(b >> 2 & 1) * SB + (uint32_t)w * 1024u);
    };

    float4_t acc[AF][BF];
#pragma unroll
    for (int i = 0; i < AF; ++i)
#pragma unroll
        for (int t = 0; t < BF; ++t) acc[i][t] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < STAGES - 1; ++b)
        if (b < a.kb) fetch(b);

    for (int b = 0; b < a.kb; ++b) {
        const float wsb = ws[b];
        if (b + STAGES - 2 < a.kb)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"((STAGES - 2) * LOADS) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" : : : "memory");
        // (everyone is past block b - 1, whose buffer this fills)
        if (b + STAGES - 1 < a.kb) fetch(b + STAGES - 1);
        const uint8_t *base = lds + (b % STAGES) * STAGE;
        Codes<EXACT> x[BF];
        float s[BF];
#pragma unroll
        for (int t = 0; t < BF; ++t) {
            const int tok = (wt * BF + t) * 16 + j;
            const uint8_t *row = base + WB + tok * kBlk;
            x[t] = Codes<EXACT>(*reinterpret_cast<const uint4_t *>(row + ((q ^ (tok & 7)) * 16)),
                                *reinterpret_cast<const uint4_t *>(row + (((4 + q) ^ (tok & 7)) * 16)));
            s[t] = *reinterpret_cast<const float *>(lds + SCALES + (b >> 2 & 1) * SB + tok * 16 + (b & 3) * 4) * wsb;
        }
#pragma unroll
        for (int i = 0; i < AF; ++i) {
            const uint8_t *frag = base + (wr * AF + i) * 2048 + lane * 16;
            const Codes<EXACT> wf(*reinterpret_cast<const uint4_t *>(frag), *reinterpret_cast<const uint4_t *>(frag + 1024));
#pragma unroll
            for (int t = 0; t < BF; ++t) {
                const float4_t p = block_product(wf, x[t]);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][t][r] = __builtin_fmaf(p[r], s[t], acc[i][t][r]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < BF; ++t) {
        const int tok = tok0 + (wt * BF + t) * 16 + j;
        if (tok < a.m) {
            typename T::type *row = static_cast<typename T::type *>(a.Y) + tok * a.y_ld;
#pragma unroll
            for (int u = 0; u < AF / 4; ++u) {
                float y[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) y[e] = acc[4 * u + e / 4][t][e % 4];
                const int o = o0 + (wr * AF / 4 + u) * kWTileRows + 16 * q;
                if constexpr (sizeof(typename T::type) == 4) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const float z[4] = {y[e], y[e + 1], y[e + 2], y[e + 3]};
                        store_piece<T>(row, o + e, a.n, z);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 16; e += 8) {
                        const float z[8] = {y[e], y[e + 1], y[e + 2], y[e + 3], y[e + 4], y[e + 5], y[e + 6], y[e + 7]};
                        store_piece<T>(row, o + e, a.n, z);
                    }
                }
            }
        }
    }
}

template <int FR, int TB, class T>
static void launch_stream(const BlockGemmArgs &a, hipStream_t st)
{
    const int most = FR * TB >= 16 ? 4 : FR * TB >= 8 ? 8 : 16;          // 64 KiB of partial results at most
    const int waves = a.kb < most ? a.kb : most;
    const unsigned grid = (unsigned)(wtile_rows(a.n) * 4 / FR);
    hipLaunchKernelGGL(HIP_KERNEL_NAME(block_stream_kernel<FR, TB, T>), dim3(grid), dim3((unsigned)(waves * kWave)),
                       (size_t)waves * FR * TB * kWave * sizeof(float4_t), st, a);
}

template <int WR, int WT, int AF, int BF, int STAGES, bool EXACT, class T>
static int launch_tile(BlockGemmArgs a, hipStream_t st)
{
    constexpr int BM = 16 * AF * WR, BN = 16 * BF * WT, LDS = STAGES * (BM + BN) * kBlk + (BN + 63) / 64 * 2048;
    a.tiles_o = (int)(((int64_t)a.n + BM - 1) / BM);
    a.tiles_t = (int)(((int64_t)a.m + BN - 1) / BN);
    const int64_t tiles = (int64_t)a.tiles_o * a.tiles_t;
    if (tiles * (WR * WT * kWave) > UINT32_MAX) return SLIM_ERR_SHAPE;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(block_tile_kernel<WR, WT, AF, BF, STAGES, EXACT, T>), dim3((unsigned)tiles), dim3(WR * WT * kWave), LDS, st, a);
    return SLIM_OK;
}

template <class T>
static int launch_block_gemm(const BlockGemmArgs &a, hipStream_t st)
{
    if (a.m <= 16) {
        if (a.n <= 8192)
            launch_stream<1, 1, T>(a, st);
        else
            launch_stream<4, 1, T>(a, st);
        return SLIM_OK;
    }
    if (a.m <= 64) {
        if (a.m <= 32)
            launch_stream<2, 2, T>(a, st);
        else
            launch_stream<2, 4, T>(a, st);
        return SLIM_OK;
    }
    constexpr bool EXACT = sizeof(typename T::type) == 4;
    if constexpr (!EXACT)
        if ((int64_t)((a.n + 255) / 256) * ((a.m + 255) / 256) >= 256) return launch_tile<2, 4, 8, 4, 2, false, T>(a, st);
    return launch_tile<2, 2, 4, 4, 2, EXACT, T>(a, st);
}

}  // namespace slim

using namespace slim;

extern "C" int slim_block_fp8_gemm_workspace(int32_t n, int32_t k, int32_t m, size_t *bytes)
{
    if (!bytes) return SLIM_ERR_NULL;
    if (slim_block_fp8_weight_sizes(n, k, nullptr, nullptr) != SLIM_OK || m < 1) return SLIM_ERR_SHAPE;
    *bytes = 256;
    return SLIM_OK;
}

extern "C" int slim_block_fp8_gemm(const slim_block_fp8_layer *layer, const uint8_t *X, const float *x_scales, int32_t m, void *Y, int64_t y_ld,
                                   int32_t dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!layer || !layer->codes || !layer->scales || !X || !x_scales || !Y || !workspace) return SLIM_ERR_NULL;
    size_t need;
    const int status = slim_block_fp8_gemm_workspace(layer->n, layer->k, m, &need);
    if (status != SLIM_OK) return status;
    if (y_ld < layer->n || (dtype != SLIM_F16 && dtype != SLIM_BF16 && dtype != SLIM_F32)) return SLIM_ERR_SHAPE;
    auto off = [](const void *p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; };
    if (off(layer->codes, 16) || off(layer->scales, 4) || off(X, 16) || off(x_scales, 4) || off(workspace, 16) || off(Y, dtype == SLIM_F32 ? 4 : 2))
        return SLIM_ERR_ALIGN;
    if (workspace_bytes < need) return SLIM_ERR_WORKSPACE;
    BlockGemmArgs a{layer->codes, layer->scales, X, x_scales, Y, y_ld, layer->n, m, blocks_of(layer->k), 0, 0};
    hipStream_t st = static_cast<hipStream_t>(stream);
    int rc;
    if (dtype == SLIM_F16)
        rc = launch_block_gemm<F16>(a, st);
    else if (dtype == SLIM_BF16)
        rc = launch_block_gemm<BF16>(a, st);
    else
        rc = launch_block_gemm<F32>(a, st);
    return rc != SLIM_OK ? rc : hip_status(hipGetLastError());
}
