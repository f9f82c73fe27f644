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
// half as fast.  So results in fp32 are EXACT, as is the kernel for few tokens: for layers larger than the last-level cache, where it waits for memory, that
// costs nothing; on smaller ones the conversions to fp16 are what bounds it (block_stream_kernel).
#include <hip/hip_runtime.h>

#include "slim_block_fp8.h"
#include "slim_mma.h"

namespace slim {

typedef int int8v_t __attribute__((ext_vector_type(8)));

// fp32 behind a uniform address, read by scalar loads
typedef __attribute__((address_space(4))) const float scalar_float;

struct BlockGemmArgs {
    const uint8_t *W;        // tiles of 64 x 128
    const float *ws;         // [row blocks][kb]
    const uint8_t *X;        // [m][128 kb]
    const float *xs;         // [m][kb]
    void *Y;
    int64_t y_ld;
    int n, m, kb, tiles_o, tiles_t;
    bool whole_lines;        // every row of Y begins at a multiple of 64 bytes
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

// N load instructions of 64 x 16 bytes that write LDS, a KiB apart both in memory and in LDS: to byte lds_byte + AT (uniform) on, in lane order.
// The compiler does not see the loads: the caller waits for them.
template <int N, int AT>
__device__ __forceinline__ void load_run_to_lds(rsrc_t r, uint32_t lane_off, uint32_t uniform_off, uint32_t lds_byte)
{
    static_assert(N == 1 || N == 2 || N == 4, "run");
    if constexpr (N == 1)
        asm volatile("s_add_u32 m0, %3, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds"
                     :
                     : "v"(lane_off), "s"(r), "s"(uniform_off), "s"(lds_byte), "n"(AT)
                     : "memory", "scc", "m0");
    else if constexpr (N == 2)
        asm volatile("s_add_u32 m0, %3, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds\n\t"
                     "buffer_load_dwordx4 %0, %1, %2 offen offset:1024 lds"
                     :
                     : "v"(lane_off), "s"(r), "s"(uniform_off), "s"(lds_byte), "n"(AT)
                     : "memory", "scc", "m0");
    else
        asm volatile("s_add_u32 m0, %3, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds\n\t"
                     "buffer_load_dwordx4 %0, %1, %2 offen offset:1024 lds\n\t"
                     "buffer_load_dwordx4 %0, %1, %2 offen offset:2048 lds\n\t"
                     "buffer_load_dwordx4 %0, %1, %2 offen offset:3072 lds"
                     :
                     : "v"(lane_off), "s"(r), "s"(uniform_off), "s"(lds_byte), "n"(AT)
                     : "memory", "scc", "m0");
}

// ---- few tokens: the weights are streamed once, each wavefront of a workgroup a share of the blocks ----
// FR fragments of 16 rows and TB tiles of 16 tokens per workgroup of S wavefronts, a run of blocks per wavefront.  A wavefront is a
// pipeline of its own: D blocks' operands of its share are under way to its own part of LDS (loads that write LDS; the tokens' as eight rows of
// 128 bytes per load, in the order of block_tile_kernel's: as a fragment needs them, 16 rows of 64, they take more than twice the time).
// The S partial results meet in LDS and are added in order.
// Bound by memory where the layer is large: 28672 x 8192 at 16 tokens 44 us, 5.3 TB/s, and 42 to 44 with the products left out.  Layers that fit the
// last-level cache are bound by what a wavefront issues, conversions to fp16 first: 5120 x 5120 at 48 tokens 9.7 us on 160 of 256 compute units (more
// workgroups of fewer fragments convert the tokens more often, the times are at launch_stream_of); 4096 x 4096 at one token 5.3 us, of which a launch is 3.
constexpr int kStreamDepth = 2;             // blocks under way per wavefront

constexpr size_t stream_lds(int fr, int tb, int waves)
{
    const size_t ring = (size_t)waves * (kStreamDepth * (fr + tb) * 2048 + 2048), sums = (size_t)waves * fr * tb * kWave * sizeof(float4_t);
    return ring > sums ? ring : sums;
}

template <int FR, int TB>
struct StreamLds {
    static constexpr int stage = (FR + TB) * 2048, scales = 2048;         // per wavefront: of a block; of twice four blocks
};

template <int FR, int TB, int D, int THREADS, class T>
__global__ __launch_bounds__(THREADS) void block_stream_kernel(BlockGemmArgs a)
{
    typedef StreamLds<FR, TB> Lds;
    constexpr int LOADS = 2 * (FR + TB), RUN = FR > 1 ? 4 : 2;
    extern __shared__ __align__(16) uint8_t lds[];
    const int S = (int)blockDim.x / kWave, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x & (kWave - 1);
    const int f0 = (int)blockIdx.x * FR, rt = f0 >> 2, t0 = f0 & 3, j = lane & 15, q = lane >> 4;
    const uint32_t kp = (uint32_t)a.kb * kBlk;
    const rsrc_t wd = make_rsrc(a.W + (int64_t)rt * a.kb * kWTileBytes, (uint32_t)a.kb * kWTileBytes);
    const rsrc_t xd = make_rsrc(a.X, (uint32_t)a.m * kp), sd = make_rsrc(a.xs, (uint32_t)a.m * (uint32_t)a.kb * 4u);
    const scalar_float *ws = (const scalar_float *)(a.ws + (int64_t)(rt >> 1) * a.kb);
    const int share = (a.kb + S - 1) / S, first = w * share, count = min(share, a.kb - first);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    const uint32_t ring = (uint32_t)w * (D * Lds::stage), scales = (uint32_t)S * (D * Lds::stage) + (uint32_t)w * Lds::scales;

    uint32_t xoff[2 * TB];
#pragma unroll
    for (int i = 0; i < 2 * TB; ++i) xoff[i] = (uint32_t)(8 * i + lane / 8) * kp + (uint32_t)((lane & 7) ^ (lane / 8)) * 16u;
    const uint32_t woff = (uint32_t)t0 * 2048u + (uint32_t)lane * 16u, soff = (uint32_t)lane * (uint32_t)a.kb * 4u;
    // The operands of the share's block i (past its end nothing: offsets out of range; the number of loads under way is what counts).
    auto fetch = [&](int i, int slot) {
        const uint32_t out = i < count ? 0u : 0x80000000u, b = i < count ? (uint32_t)(first + i) : 0u;
        const uint32_t base = lds0 + ring + (uint32_t)slot * Lds::stage;
        if ((i & 3) == 0) load_to_lds(sd, (soff + b * 4u) | out, 0u, lds0 + scales + (uint32_t)(i >> 2 & 1) * 1024u);
#pragma unroll
        for (int f = 0; f < 2 * FR; f += RUN) load_run_to_lds<RUN, 0>(wd, (woff + (uint32_t)f * 1024u) | out, b * kWTileBytes, base + (uint32_t)f * 1024u);
#pragma unroll
        for (int t = 0; t < 2 * TB; ++t) load_to_lds(xd, xoff[t] | out, b * kBlk, base + (uint32_t)(2 * FR + t) * 1024u);
    };
    float4_t acc[FR][TB];
#pragma unroll
    for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int t = 0; t < TB; ++t) acc[f][t] = float4_t{0.f, 0.f, 0.f, 0.f};
    if (count > 0) {
#pragma unroll
        for (int i = 0; i < D; ++i) fetch(i, i);
    }
    // (the rows' scale comes by a scalar load, a block ahead: those are counted apart from the loads to LDS)
    float wsb, next_wsb = ws[min(first, a.kb - 1)];
    for (int i = 0, slot = 0; i < count; ++i) {
        wsb = next_wsb;
        next_wsb = ws[min(first + i + 1, a.kb - 1)];
        asm volatile("s_waitcnt vmcnt(%0)" : : "n"((D - 1) * LOADS) : "memory");
        const uint8_t *base = lds + ring + slot * Lds::stage;
        uint4_t wv[FR][2], xv[TB][2];
        float s[TB];
#pragma unroll
        for (int f = 0; f < FR; ++f)
#pragma unroll
            for (int h = 0; h < 2; ++h) wv[f][h] = *reinterpret_cast<const uint4_t *>(base + (2 * f + h) * 1024 + lane * 16);
#pragma unroll
        for (int t = 0; t < TB; ++t) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                xv[t][h] = *reinterpret_cast<const uint4_t *>(base + FR * 2048 + (16 * t + j) * kBlk + (((4 * h + q) ^ (j & 7)) * 16));
            s[t] = *reinterpret_cast<const float *>(lds + scales + (i >> 2 & 1) * 1024 + (16 * t + j) * 16 + (i & 3) * 4) * wsb;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
        fetch(i + D, slot);
        slot = slot + 1 < D ? slot + 1 : 0;
        Codes<true> x[TB];
#pragma unroll
        for (int t = 0; t < TB; ++t) x[t] = Codes<true>(xv[t][0], xv[t][1]);
#pragma unroll
        for (int f = 0; f < FR; ++f) {
            const Codes<true> wf(wv[f][0], wv[f][1]);
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                const float4_t p = block_product(wf, x[t]);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[f][t][r] = __builtin_fmaf(p[r], s[t], acc[f][t][r]);
            }
        }
    }
    // (nothing is under way into LDS, and no one reads operands there, when the sums go in)
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    __syncthreads();
    float4_t *part = reinterpret_cast<float4_t *>(lds);                   // [S][FR * TB][64]
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
// A workgroup of WR x WT wavefronts has a tile of 16 AF WR rows x 16 BF WT tokens.  STAGES buffers of one block each are
// filled by loads that write LDS directly.  There is one barrier per block, TAIL row fragments before its end, when a wavefront has read all it
// needs of the block: past it everyone's pieces of the next block are there (each has waited for its own), so that the next
// block's first fragments are read during the last products of this one, and this block's buffer is free to be filled.
// The tokens' scales are fetched for 16 blocks at a time (64 bytes of a token's row), into two buffers of their own, ahead of the pieces of
// the first of the 16.  A wavefront waits until no more of its loads are under way than the pieces of later blocks; that some of
// those may be scales makes it wait longer, never shorter.
// Results leave through LDS, so that a store instruction writes whole lines of a token's row.
// 28672 x 8192 at 4096 tokens takes 760 to 782 us from card to card, 2.53 PFLOP/s (671 us for the library's product with one scale in all): power holds the clock at 1.65 GHz,
// the matrix pipes are busy 68 % of it; without the scaled additions, 4 of a lane's instructions per product, it would be 661, without
// loads 595.  10007 x 4100 at 333 tokens in fp32 (EXACT) takes 35.3 us, matrix pipes 32 % busy: its 128 conversions and 64 additions per 64 products
// of a wavefront take about as long to issue as the products, and hide behind them only in part (without the conversions 26.7 us, without the
// additions 25.7, without the products 26.4, without loads 32.7); a conversion and an addition placed by hand after every product, or two chains of
// products in turn, were no faster (36.4, 37.5).
// KG = 2: two such groups of wavefronts share the tile, each with half of the blocks and buffers of its own, and their sums are added at the end: where
// there are few tiles, twice the loads are under way, and a SIMD has two wavefronts with the larger share of the tile.
template <int BM, int BN, int STAGES>
struct TileLds {
    static constexpr int stage = (BM + BN) * kBlk, scales = STAGES * stage, chunk = BN * 64, bytes = scales + 2 * chunk;
};

template <int KG, int WR, int WT, int AF, int BF, int STAGES, bool EXACT, class T>
__global__ __launch_bounds__(KG *WR *WT *kWave, 2) void block_tile_kernel(BlockGemmArgs a)
{
    typedef typename T::type E;
    constexpr int WAVES = WR * WT, BM = 16 * AF * WR, BN = 16 * BF * WT, TAIL = 2;
    constexpr int WB = BM * kBlk, XB = BN * kBlk;
    constexpr int WL = WB / 1024 / WAVES, XL = XB / 1024 / WAVES, SL = BN / 16 / WAVES, LOADS = WL + XL;
    constexpr int RUN = EXACT && WL >= 4 ? 4 : WL < 4 ? WL : 1, WU = WL / RUN, UNITS = WU + XL;          // loads of weights in one go, and units of loads per block
    typedef TileLds<BM, BN, STAGES> Lds;
    static_assert(WL * WAVES * 1024 == WB && XL * WAVES * 1024 == XB && SL * WAVES * 16 == BN && BM % kWTileRows == 0 && AF % 4 == 0, "tile");
    static_assert(AF * 16 == 64 || (AF * 16) % kBlk == 0, "a wavefront's rows have one scale per block");
    static_assert(STAGES >= 2 && STAGES <= 8 && (int)(BM * BN * sizeof(E)) <= Lds::scales, "buffers");
    extern __shared__ __align__(16) uint8_t lds[];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x & (kWave - 1);
    const int group = wave / WAVES, w = wave % WAVES;
    const int wr = w % WR, wt = w / WR, j = lane & 15, q = lane >> 4;
    const int gx = a.tiles_o * a.tiles_t;
    const int qx = gx % kDies == 0 ? ((int)blockIdx.x % kDies) * (gx / kDies) + (int)blockIdx.x / kDies : (int)blockIdx.x;
    const int tile = blocked_tile(qx, a.tiles_o, a.tiles_t);
    const int o0 = tile % a.tiles_o * BM, tok0 = tile / a.tiles_o * BN;
    const uint32_t kp = (uint32_t)a.kb * kBlk;
    const int rows = min(BM, (a.n - o0 + kWTileRows - 1) / kWTileRows * kWTileRows), toks = min(BN, a.m - tok0);
    const uint8_t *wbase = a.W + (int64_t)o0 * kp, *xbase = a.X + (int64_t)tok0 * kp;
    const rsrc_t sd = make_rsrc(a.xs + (int64_t)tok0 * a.kb, (uint32_t)toks * (uint32_t)a.kb * 4u);
    // rows past the layer's last block of 128 are zeros: any scale will do
    const int rb = min((o0 + wr * AF * 16) / kBlk, (a.n - 1) / kBlk);
    const float *ws = a.ws + (int64_t)rb * a.kb;
    uint8_t *const own = lds + group * Lds::bytes;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)own;
    // the group's blocks: count from `first` on; the second group may have one less than the first (none where there is one block only)
    const int turns = (a.kb + KG - 1) / KG, first = group * turns, count = min(turns, a.kb - first);

    // this wavefront's shares of a block: a run of KiB of the weight tiles, and groups of eight tokens whose eight 16-byte pieces are put in another
    // order in each of eight rows, so that a fragment's reads find all banks
    uint32_t woff[WU], xoff[XL], soff[SL];
#pragma unroll
    for (int i = 0; i < WU; ++i) {
        const int piece = w * WL + i * RUN;
        woff[i] = (uint32_t)(piece / 8) * (uint32_t)a.kb * kWTileBytes + (uint32_t)(piece % 8) * 1024u + (uint32_t)lane * 16u;
    }
#pragma unroll
    for (int i = 0; i < XL; ++i) xoff[i] = (uint32_t)((w * XL + i) * 8 + lane / 8) * kp + (uint32_t)((lane & 7) ^ (lane / 8)) * 16u;
#pragma unroll
    for (int i = 0; i < SL; ++i)
        soff[i] = (uint32_t)((w * SL + i) * 16 + lane / 4) * (uint32_t)a.kb * 4u + (uint32_t)((lane & 3) ^ (lane >> 4)) * 16u;
    auto fetch_scales = [&](int b) {
#pragma unroll
        for (int i = 0; i < SL; ++i)
            load_to_lds(sd, soff[i] + (uint32_t)(first + b) * 4u, 0u, lds0 + Lds::scales + (uint32_t)(b >> 4 & 1) * Lds::chunk + (uint32_t)(w * SL + i) * 1024u);
    };
    // Unit `u` of this wavefront's share of the group's block b.  Past the last block nothing is read (from a buffer of no length; zeros): the number of
    // loads under way is the same everywhere.  The uniform offset is then 0: whether the range check leaves it out or takes it off the buffer's length, 0
    // bytes from there on are no bytes, and no address is one of a neighbour's block or past the operand.
    auto fetch_unit = [&](auto uc, int b, int buffer) {
        constexpr int u = decltype(uc)::value;
        const uint32_t base = lds0 + (uint32_t)buffer * Lds::stage;
        const bool there = b < count;
        const uint32_t block = there ? (uint32_t)(first + b) : 0u;
        if constexpr (u < WU) {
            const rsrc_t d = make_rsrc(wbase, there ? (uint32_t)rows * kp : 0u);
            load_run_to_lds<RUN, u * RUN * 1024>(d, woff[u], block * kWTileBytes, base + (uint32_t)(w * WL) * 1024u);
        } else {
            const rsrc_t d = make_rsrc(xbase, there ? (uint32_t)toks * kp : 0u);
            load_run_to_lds<1, WB + (u - WU) * 1024>(d, xoff[u - WU], block * kBlk, base + (uint32_t)(w * XL) * 1024u);
        }
    };

    // The rows' scales of 64 blocks, one per lane.  They are waited for where they are loaded: a wait of the compiler's inside the loop would be
    // for all the loads under way, which it does not know of.
    float row_scales;
    auto fetch_row_scales = [&](int b) {
        row_scales = ws[min(first + b + lane, a.kb - 1)];
        asm volatile("" : "+v"(row_scales));
    };
    fetch_row_scales(0);

    const int xrow = (wt * BF * 16 + j) * kBlk, xp0 = (q ^ (j & 7)) * 16, xp1 = ((4 + q) ^ (j & 7)) * 16;
    auto load_x = [&](int buffer, int t) {
        const uint8_t *row = own + buffer * Lds::stage + WB + xrow + t * 16 * kBlk;
        return Codes<false>(*reinterpret_cast<const uint4_t *>(row + xp0), *reinterpret_cast<const uint4_t *>(row + xp1));
    };
    auto load_w = [&](int buffer, int i) {
        const uint8_t *frag = own + buffer * Lds::stage + (wr * AF + i) * 2048 + lane * 16;
        return Codes<false>(*reinterpret_cast<const uint4_t *>(frag), *reinterpret_cast<const uint4_t *>(frag + 1024));
    };
    auto load_scale = [&](int b, int t) {
        return *reinterpret_cast<const float *>(own + Lds::scales + (b >> 4 & 1) * Lds::chunk + ((wt * BF + t) * 16 + j) * 64 +
                                                ((b >> 2 & 3) ^ (j >> 2)) * 16 + (b & 3) * 4);
    };

    float4_t acc[AF][BF];
#pragma unroll
    for (int i = 0; i < AF; ++i)
#pragma unroll
        for (int t = 0; t < BF; ++t) acc[i][t] = float4_t{0.f, 0.f, 0.f, 0.f};
    // Row fragments in registers: two in turn, and the last TAIL, which are all read before the barrier, in their own.
    constexpr int MAIN = AF - TAIL, WBUF = TAIL > 1 ? 2 + TAIL : 2;
    auto place = [](int i) { return i < MAIN || TAIL == 1 ? i % 2 : 2 + i - MAIN; };
    Codes<false> x[BF], wv[WBUF];
    float s[BF], wsb;
    // EXACT: what is being multiplied as fp16 numbers, made of the codes when the products begin (by then they are there); or, of AHEAD tokens' tiles,
    // among the last products of the block before, a tile after its codes were asked for.  With one group: 1024 tokens on 11008 x 4096 89.3 -> 86.9 us,
    // 4096 tokens on 8192 x 8192 470 -> 458.  With two, whose wavefronts fill in for each other, it loses 1 %.
    constexpr int AHEAD = KG == 1 ? BF - 1 : 0;
    Codes<true> xh[EXACT ? BF : 1], wh[EXACT ? TAIL : 1];
    auto product = [&](int i, int t) {
        if constexpr (EXACT)
            return block_product(wh[i < MAIN ? 0 : i - MAIN], xh[t]);
        else
            return block_product(wv[place(i)], x[t]);
    };
    // The products of a block in order: fragment by fragment, the last TAIL token tile by token tile.  Each is added LAG products later, when the matrix
    // pipe has it ready.
    constexpr int SLOTS = AF * BF, LAG = EXACT ? 2 : 3;
    // A block's loads are asked for a few at a time between the products, EARLY units of them in the tail that follows the barrier and the others in the
    // next block: all at once they held the wavefronts up behind one another, 600 of 3170 cycles per block of 256 x 256.
    constexpr int SPREAD = SLOTS >= 2 * UNITS ? 2 : 1, EARLY = UNITS < (TAIL * BF + SPREAD - 1) / SPREAD ? UNITS : (TAIL * BF + SPREAD - 1) / SPREAD;
    static_assert((UNITS - EARLY) * SPREAD <= MAIN * BF, "every unit has its place");
    auto row_of = [](int n) { return n < MAIN * BF ? n / BF : MAIN + (n - MAIN * BF) % TAIL; };
    auto token_of = [](int n) { return n < MAIN * BF ? n % BF : (n - MAIN * BF) / TAIL; };
    float4_t p[LAG + 1];
    auto add = [&](auto nc) {
        constexpr int n = decltype(nc)::value, i = row_of(n), t = token_of(n);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[i][t][r] = __builtin_fmaf(p[n % (LAG + 1)][r], s[t], acc[i][t][r]);
    };

#pragma unroll
    for (int b = 0; b < STAGES - 1; ++b) {
        if (b == 0) fetch_scales(0);
        static_for<UNITS>([&](auto uc) { fetch_unit(uc, b, b); });
    }
    static_for<EARLY>([&](auto uc) { fetch_unit(uc, STAGES - 1, STAGES - 1); });
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
    wsb = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, row_scales), 0));
#pragma unroll
    for (int t = 0; t < BF; ++t) {
        x[t] = load_x(0, t);
        s[t] = load_scale(0, t) * wsb;
    }
    wv[0] = load_w(0, 0);
    if constexpr (EXACT) {
#pragma unroll
        for (int t = 0; t < AHEAD; ++t) xh[t] = Codes<true>(x[t].h[0], x[t].h[1]);
    }

    for (int b = 0, buffer = 0; b < count; ++b) {
        const int after = buffer + 1 < STAGES ? buffer + 1 : 0, before = buffer > 0 ? buffer - 1 : STAGES - 1;
        static_for<MAIN * BF>([&](auto nc) {
            constexpr int n = decltype(nc)::value, i = row_of(n), t = token_of(n);
            if constexpr (t == 0) {
                if constexpr (i + 1 < MAIN || TAIL == 1) wv[place(i + 1)] = load_w(buffer, i + 1);
                if constexpr (TAIL > 1 && i >= MAIN - TAIL) wv[place(i + TAIL)] = load_w(buffer, i + TAIL);
                if constexpr (EXACT) wh[0] = Codes<true>(wv[place(i)].h[0], wv[place(i)].h[1]);
            }
            if constexpr (EXACT && i == 0 && t >= AHEAD) xh[t] = Codes<true>(x[t].h[0], x[t].h[1]);
            if constexpr (n % SPREAD == 0 && EARLY + n / SPREAD < UNITS)
                fetch_unit(std::integral_constant<int, EARLY + n / SPREAD>{}, b + STAGES - 1, before);
            if constexpr (n >= LAG) add(std::integral_constant<int, n - LAG>{});
            p[n % (LAG + 1)] = product(i, t);
            if constexpr (!EXACT || n % 2 == 1) __builtin_amdgcn_sched_barrier(0);
        });
        // The sums so far are made here: the compiler would put them off past the barrier, and spill the products.
#pragma unroll
        for (int i = 0; i < MAIN; ++i)
#pragma unroll
            for (int t = 0; t < BF; ++t) asm volatile("" : "+v"(acc[i][t]));
        if (((b + 1) & (kWave - 1)) == 0) fetch_row_scales(b + 1);
        wsb = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, row_scales), (b + 1) & (kWave - 1)));
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"((STAGES - 2) * LOADS) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" : : : "memory");
        if (((b + STAGES) & 15) == 0) fetch_scales(b + STAGES);
        // (past the last block what is read is an older one's, and is not used)
        float sn[BF];
#pragma unroll
        for (int t = 0; t < BF; ++t) sn[t] = load_scale(b + 1, t);
        wv[0] = load_w(after, 0);
        if constexpr (EXACT) {
#pragma unroll
            for (int i = 0; i < TAIL; ++i) wh[i] = Codes<true>(wv[place(MAIN + i)].h[0], wv[place(MAIN + i)].h[1]);
        }
        __builtin_amdgcn_sched_barrier(0);
        static_for<TAIL * BF>([&](auto nc) {
            constexpr int n = MAIN * BF + decltype(nc)::value, i = row_of(n), t = token_of(n);
            if constexpr ((n - MAIN * BF) % SPREAD == 0 && (n - MAIN * BF) / SPREAD < EARLY)
                fetch_unit(std::integral_constant<int, (n - MAIN * BF) / SPREAD>{}, b + STAGES, buffer);
            p[n % (LAG + 1)] = product(i, t);
            if constexpr (i == AF - 1) x[t] = load_x(after, t);
            if constexpr (EXACT && i == AF - 1 && t > 0 && t <= AHEAD) xh[t - 1] = Codes<true>(x[t - 1].h[0], x[t - 1].h[1]);
            if constexpr (n >= LAG) add(std::integral_constant<int, n - LAG>{});        // (64 x 64: the third product is the tail's first)
            if constexpr (!EXACT || n % 2 == 1) __builtin_amdgcn_sched_barrier(0);
        });
        static_for<LAG>([&](auto nc) { add(std::integral_constant<int, SLOTS - LAG + decltype(nc)::value>{}); });
#pragma unroll
        for (int t = 0; t < BF; ++t) s[t] = sn[t] * wsb;
        buffer = after;
    }
    // A group with a block less has nothing to multiply in the last turn, where the other meets its barrier once more.  (Not zeros with a scale of 0: that
    // times an infinite scale of the rows' last block is a NaN, and what is not there need not be zeros.)
    if (KG > 1 && count < turns) __builtin_amdgcn_s_barrier();

    // Results stream past the caches where their rows begin at multiples of 64 bytes; otherwise the ends of a tile's rows are parts of lines, which are better
    // put together in the L2.  (2171 x 7424 and x 7442 in fp32 on 166 inputs: 17.6 and 27.8 us streaming, 20.0 and 21.2 cached; 4096 x 11008 on 512: 65 and 85.)
    // Results to LDS: a row of BM per token, its 16-byte pieces in another order in each of up to 16 rows; from there a piece per lane and store.
    constexpr int PIECE = 16 / sizeof(E), PER_ROW = BM / PIECE, TURN = (PER_ROW < 16 ? PER_ROW : 16) - 1;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
    if constexpr (KG > 1) {
        float4_t *part = reinterpret_cast<float4_t *>(lds);          // [SLOTS][WAVES][64]
        if (group == 1) {
#pragma unroll
            for (int n = 0; n < SLOTS; ++n) part[(n * WAVES + w) * kWave + lane] = acc[n / BF][n % BF];
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int n = 0; n < SLOTS; ++n) acc[n / BF][n % BF] += part[(n * WAVES + w) * kWave + lane];
        }
        __syncthreads();
    }
    if (group == 0)
#pragma unroll
    for (int t = 0; t < BF; ++t) {
        const int tok = (wt * BF + t) * 16 + j;
#pragma unroll
        for (int u = 0; u < AF / 4; ++u)
#pragma unroll
            for (int e = 0; e < 16; e += PIECE) {
                typedef E vec __attribute__((ext_vector_type(PIECE)));
                vec v;
#pragma unroll
                for (int z = 0; z < PIECE; ++z) v[z] = (E)acc[4 * u + (e + z) / 4][t][(e + z) % 4];
                const int c = ((wr * AF / 4 + u) * kWTileRows + 16 * q + e) / PIECE;
                *reinterpret_cast<vec *>(lds + (tok * PER_ROW + (c ^ (tok & TURN))) * 16) = v;
            }
    }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < toks * PER_ROW; i += KG * WAVES * kWave) {
        const int tok = i / PER_ROW, c = i % PER_ROW, o = o0 + c * PIECE;
        if (o < a.n) {
            typedef E vec __attribute__((ext_vector_type(PIECE)));
            const vec v = *reinterpret_cast<const vec *>(lds + (tok * PER_ROW + (c ^ (tok & TURN))) * 16);
            E *row = static_cast<E *>(a.Y) + (int64_t)(tok0 + tok) * a.y_ld;
            if (o + PIECE <= a.n) {
                if (a.whole_lines)
                    Piece<T, PIECE>::store_streaming(row + o, v);
                else
                    Piece<T, PIECE>::store(row + o, v);
            } else {
#pragma unroll
                for (int z = 0; z < PIECE; ++z)
                    if (o + z < a.n) row[o + z] = v[z];
            }
        }
    }
}

// As many fragments per workgroup as leave 160 workgroups for 256 compute units: the tokens are read once per workgroup, and four fragments are a whole tile
// of weights.  us with one / two / four fragments: 28672 x 8192 at 16 tokens 49 / 51 / 45, at 64 tokens 96 / 72 / 58; 8192 x 8192 at 64 tokens 23 / 19 / 22;
// 5120 x 5120 at 48 tokens 11.9 / 9.9 / 13.8; 4096 x 4096 at 32 tokens 6.9 / 7.3 / 9.2.  Two fragments are not worth it for up to 16 tokens
// (8192 x 8192: 12.2 / 15.1 / 13.0).
// Four wavefronts, two blocks under way each: more of either was slower for 28672 x 8192 at one token (41 us with 4 or 8 wavefronts of one
// fragment, 52 with 16; three or four blocks under way 44 to 50).  Eight where there are fewer workgroups than compute units.
struct StreamPlan {
    int fragments, waves, workgroups;
};
static StreamPlan plan_stream(int n, int kb, int tb)
{
    const DeviceInfo dev = device_info();
    const int all = wtile_rows(n) * 4, enough = dev.cus * 5 / 8;
    StreamPlan p;
    p.fragments = all >= 4 * enough ? 4 : tb > 1 && all >= 2 * enough ? 2 : 1;
    p.waves = p.fragments == 1 && all < dev.cus ? 8 : 4;
    while (p.waves > 1 && stream_lds(p.fragments, tb, p.waves) > dev.lds) p.waves /= 2;
    if (p.waves > kb) p.waves = kb;
    p.workgroups = all / p.fragments;
    return p;
}

template <int FR, int TB, class T>
static void launch_stream(const BlockGemmArgs &a, const StreamPlan &p, hipStream_t st)
{
    hipLaunchKernelGGL(HIP_KERNEL_NAME(block_stream_kernel<FR, TB, kStreamDepth, 8 * kWave, T>), dim3((unsigned)p.workgroups),
                       dim3((unsigned)(p.waves * kWave)), stream_lds(FR, TB, p.waves), st, a);
}

template <int TB, class T>
static void launch_stream_of(const BlockGemmArgs &a, hipStream_t st)
{
    const StreamPlan p = plan_stream(a.n, a.kb, TB);
    if (p.fragments == 4) {
        launch_stream<4, TB, T>(a, p, st);
        return;
    }
    if constexpr (TB > 1)
        if (p.fragments == 2) {
            launch_stream<2, TB, T>(a, p, st);
            return;
        }
    launch_stream<1, TB, T>(a, p, st);
}

// Tiles of block_tile_kernel: rows, tokens, threads, workgroups per compute unit (by LDS), and the time per block of 128 inputs with every compute unit
// at work and with at most half of them (less power, less traffic).  The times (us) are those of one to three rounds on 128 to
// 4096 tokens, 4096 to 28672 rows and 4096 to 11008 inputs; a call takes rounds * (blocks * time + 3) or so, and the tile with the least of that
// is taken.  us so, with the tiles in their order (the one taken in brackets):
//   128 tokens, 4096 x 4096      41  27  19  15  12.0 [10.4]
//   256 tokens, 5120 x 5120      52  33  23 [18] 18  23
//   333 tokens, 10007 x 4100     46  29 [22] 31  31  39
//   512 tokens, 4096 x 11008    104  64  43 [35] 38  41
//   700 tokens, 4096 x 4096      43  28 [19] 29  25  28
//   1000 tokens, 8192 x 8192     80 [63] 77 105 108 125
//   1024 tokens, 11008 x 4096   [46] 60  60  83  78  97
// 256 x 256 is bound by power.  What bounds the smaller tiles was not measured: a block of 64 x 128 takes 0.40 us, 960 cycles, of which a wavefront's 8 products
// and 32 additions are under 400, and its 24.6 KB arrive at 61 GB/s per compute unit (64 x 64: 68, 128 x 128: 53).
struct TileShape {
    int rows, toks, threads, per_cu;
    float full, half;
};
constexpr TileShape kTiles[] = {{256, 256, 512, 1, 1.7f, 1.3f},   {256, 128, 512, 1, 1.0f, 0.8f},  {128, 128, 512, 1, 0.62f, 0.5f},
                                {64, 128, 256, 1, 0.40f, 0.38f}, {64, 64, 256, 2, 0.45f, 0.33f}, {64, 64, 512, 1, 0.24f, 0.24f}};
// (with results in fp32: 128 x 128, the same by two groups, 64 x 128 and 64 x 64 by two groups; 128 tokens on 4096 x 4096: 37, 31, 23, [16]; 256 tokens on
// 5120 x 5120: 45, 37, [28], 35; 333 tokens on 10007 x 4100: 40, [36], 48, 61; 1024 tokens on 11008 x 4096: [87], 94, 131, 154)
constexpr TileShape kExactTiles[] = {{128, 128, 256, 2, 1.31f, 1.1f}, {128, 128, 512, 1, 0.97f, 0.92f}, {64, 128, 512, 1, 0.64f, 0.64f}, {64, 64, 512, 1, 0.42f, 0.42f}};

template <int SHAPE, int KG, int WR, int WT, int AF, int BF, int STAGES, bool EXACT, class T>
static int launch_tile(BlockGemmArgs a, hipStream_t st)
{
    constexpr int BM = 16 * AF * WR, BN = 16 * BF * WT;
    constexpr size_t LDS = (size_t)KG * TileLds<BM, BN, STAGES>::bytes;
    constexpr TileShape shape = EXACT ? kExactTiles[SHAPE] : kTiles[SHAPE];
    static_assert(shape.rows == BM && shape.toks == BN && shape.threads == KG * WR * WT * kWave && shape.per_cu * LDS <= 160 * 1024, "the table's tile");
    static_assert(KG <= 2 && LDS <= 160 * 1024 && (KG == 1 || (size_t)BM * BN * 4 <= LDS), "LDS");
    a.tiles_o = (int)(((int64_t)a.n + BM - 1) / BM);
    a.tiles_t = (int)(((int64_t)a.m + BN - 1) / BN);
    const int64_t tiles = (int64_t)a.tiles_o * a.tiles_t;
    if (tiles * (KG * WR * WT * kWave) > UINT32_MAX) return SLIM_ERR_SHAPE;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(block_tile_kernel<KG, WR, WT, AF, BF, STAGES, EXACT, T>), dim3((unsigned)tiles), dim3(KG * WR * WT * kWave), LDS,
                       st, a);
    return SLIM_OK;
}

static int plan_tile(int n, int kb, int m, bool exact)
{
    const TileShape *shapes = exact ? kExactTiles : kTiles;
    const int count = exact ? (int)(sizeof kExactTiles / sizeof kExactTiles[0]) : (int)(sizeof kTiles / sizeof kTiles[0]);
    const double cus = device_info().cus;
    int best = 0;
    double least = 0;
    for (int i = 0; i < count; ++i) {
        const TileShape &t = shapes[i];
        const double tiles = (double)(((int64_t)n + t.rows - 1) / t.rows) * (double)(((int64_t)m + t.toks - 1) / t.toks);
        const double rounds = __builtin_ceil(tiles / (cus * t.per_cu));
        const double time = rounds * (kb * (2 * tiles <= cus * t.per_cu ? t.half : t.full) + 3.0);
        if (i == 0 || time < least) {
            least = time;
            best = i;
        }
    }
    return best;
}

template <class T>
static int launch_block_gemm(const BlockGemmArgs &a, hipStream_t st)
{
    switch ((a.m + 15) / 16) {
    case 1: launch_stream_of<1, T>(a, st); return SLIM_OK;
    case 2: launch_stream_of<2, T>(a, st); return SLIM_OK;
    case 3: launch_stream_of<3, T>(a, st); return SLIM_OK;
    case 4: launch_stream_of<4, T>(a, st); return SLIM_OK;
    default: break;
    }
    constexpr bool EXACT = sizeof(typename T::type) == 4;
    const int shape = plan_tile(a.n, a.kb, a.m, EXACT);
    if constexpr (EXACT) {
        switch (shape) {
        case 0: return launch_tile<0, 1, 2, 2, 4, 4, 2, true, T>(a, st);
        case 1: return launch_tile<1, 2, 2, 2, 4, 4, 2, true, T>(a, st);
        case 2: return launch_tile<2, 2, 1, 4, 4, 2, 2, true, T>(a, st);
        default: return launch_tile<3, 2, 1, 4, 4, 1, 4, true, T>(a, st);
        }
    } else {
        switch (shape) {
        case 0: return launch_tile<0, 1, 2, 4, 8, 4, 2, false, T>(a, st);
        case 1: return launch_tile<1, 1, 4, 2, 4, 4, 3, false, T>(a, st);
        case 2: return launch_tile<2, 1, 2, 4, 4, 2, 4, false, T>(a, st);
        case 3: return launch_tile<3, 1, 1, 4, 4, 2, 4, false, T>(a, st);
        case 4: return launch_tile<4, 1, 1, 4, 4, 1, 4, false, T>(a, st);
        default: return launch_tile<5, 2, 1, 4, 4, 1, 4, false, T>(a, st);
        }
    }
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

// What slim_block_fp8_gemm would launch (no launch, no device access but for its number of compute units).
extern "C" int slim_block_fp8_gemm_plan(int32_t n, int32_t k, int32_t m, int32_t dtype, int32_t *out)
{
    if (!out) return SLIM_ERR_NULL;
    if (slim_block_fp8_weight_sizes(n, k, nullptr, nullptr) != SLIM_OK || m < 1 || (dtype != SLIM_F16 && dtype != SLIM_BF16 && dtype != SLIM_F32))
        return SLIM_ERR_SHAPE;
    const int kb = blocks_of(k);
    if (m <= 64) {
        const int tb = (m + 15) / 16;
        const StreamPlan p = plan_stream(n, kb, tb);
        const int32_t plan[6] = {0, 16 * p.fragments, 16 * tb, p.waves * kWave, p.workgroups, 1};
        for (int i = 0; i < 6; ++i) out[i] = plan[i];
        return SLIM_OK;
    }
    const bool exact = dtype == SLIM_F32;
    const int shape = plan_tile(n, kb, m, exact);
    const TileShape &t = exact ? kExactTiles[shape] : kTiles[shape];
    const int64_t tiles = (((int64_t)n + t.rows - 1) / t.rows) * (((int64_t)m + t.toks - 1) / t.toks);
    if (tiles * t.threads > UINT32_MAX) return SLIM_ERR_SHAPE;
    const int32_t plan[6] = {1, t.rows, t.toks, t.threads, (int32_t)tiles, exact ? 1 : 0};
    for (int i = 0; i < 6; ++i) out[i] = plan[i];
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
    BlockGemmArgs a{layer->codes, layer->scales, X, x_scales, Y, y_ld, layer->n, m, blocks_of(layer->k), 0, 0, false};
    a.whole_lines = (reinterpret_cast<uintptr_t>(Y) & 63u) == 0 && y_ld * (dtype == SLIM_F32 ? 4 : 2) % 64 == 0;
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
