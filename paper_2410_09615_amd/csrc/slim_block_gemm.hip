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
// A workgroup of WR x WT wavefronts has a tile of 16 AF WR rows x 16 BF WT tokens.  STAGES buffers of one block each are
// filled by loads that write LDS directly.  There is one barrier per block, TAIL row fragments before its end, when a wavefront has read all it
// needs of the block: past it everyone's pieces of the next block are there (each has waited for its own), so that the next
// block's first fragments are read during the last products of this one, and this block's buffer is free to be filled.
// The tokens' scales are fetched for 16 blocks at a time (64 bytes of a token's row), into two buffers of their own, ahead of the pieces of
// the first of the 16.  A wavefront waits until no more of its loads are under way than the pieces of later blocks; that some of
// those may be scales makes it wait longer, never shorter.
// Results leave through LDS, so that a store instruction writes whole lines of a token's row.
template <int BM, int BN, int STAGES>
struct TileLds {
    static constexpr int stage = (BM + BN) * kBlk, scales = STAGES * stage, chunk = BN * 64, bytes = scales + 2 * chunk;
};

template <int WR, int WT, int AF, int BF, int STAGES, bool EXACT, class T>
__global__ __launch_bounds__(WR *WT *kWave, 2) void block_tile_kernel(BlockGemmArgs a)
{
    typedef typename T::type E;
    constexpr int WAVES = WR * WT, BM = 16 * AF * WR, BN = 16 * BF * WT, TAIL = AF / 4;
    constexpr int WB = BM * kBlk, XB = BN * kBlk;
    constexpr int WL = WB / 1024 / WAVES, XL = XB / 1024 / WAVES, SL = BN / 16 / WAVES, LOADS = WL + XL;
    typedef TileLds<BM, BN, STAGES> Lds;
    static_assert(WL * WAVES * 1024 == WB && XL * WAVES * 1024 == XB && SL * WAVES * 16 == BN && BM % kWTileRows == 0 && AF % 4 == 0, "tile");
    static_assert(AF * 16 == 64 || (AF * 16) % kBlk == 0, "a wavefront's rows have one scale per block");
    static_assert(STAGES >= 2 && STAGES <= 8 && (int)(BM * BN * sizeof(E)) <= Lds::scales, "buffers");
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
    uint32_t woff[WL], xoff[XL], soff[SL];
#pragma unroll
    for (int i = 0; i < WL; ++i) {
        const int piece = w * WL + i;
        woff[i] = (uint32_t)(piece / 8) * (uint32_t)a.kb * kWTileBytes + (uint32_t)(piece % 8) * 1024u + (uint32_t)lane * 16u;
    }
#pragma unroll
    for (int i = 0; i < XL; ++i) xoff[i] = (uint32_t)((w * XL + i) * 8 + lane / 8) * kp + (uint32_t)((lane & 7) ^ (lane / 8)) * 16u;
#pragma unroll
    for (int i = 0; i < SL; ++i) soff[i] = (uint32_t)((w * SL + i) * 16 + lane / 4) * (uint32_t)a.kb * 4u + (uint32_t)((lane & 3) ^ (lane >> 4)) * 16u;
    auto fetch_scales = [&](int b) {
#pragma unroll
        for (int i = 0; i < SL; ++i)
            load_to_lds(sd, soff[i] + (uint32_t)b * 4u, 0u, lds0 + Lds::scales + (uint32_t)(b >> 4 & 1) * Lds::chunk + (uint32_t)(w * SL + i) * 1024u);
    };
    // Piece `i` of this wavefront's of block b.  Past the last block nothing is read (an offset out of the buffer's range gives zeros): the number of
    // loads under way is the same everywhere.
    auto fetch_piece = [&](auto ic, int b, int buffer) {
        constexpr int i = decltype(ic)::value;
        const uint32_t base = lds0 + (uint32_t)buffer * Lds::stage, out = b < a.kb ? 0u : 0x80000000u, bb = b < a.kb ? (uint32_t)b : 0u;
        if constexpr (i < WL)
            load_to_lds(wd, woff[i] | out, bb * kWTileBytes, base + (uint32_t)(w * WL + i) * 1024u);
        else
            load_to_lds(xd, xoff[i - WL] | out, bb * kBlk, base + WB + (uint32_t)(w * XL + i - WL) * 1024u);
    };

    // The rows' scales of 64 blocks, one per lane.  They are waited for where they are loaded: a wait of the compiler's inside the loop would be
    // for all the loads under way, which it does not know of.
    float row_scales;
    auto fetch_row_scales = [&](int b) {
        row_scales = ws[min(b + lane, a.kb - 1)];
        asm volatile("" : "+v"(row_scales));
    };
    fetch_row_scales(0);

    const int xrow = (wt * BF * 16 + j) * kBlk, xp0 = (q ^ (j & 7)) * 16, xp1 = ((4 + q) ^ (j & 7)) * 16;
    auto load_x = [&](int buffer, int t) {
        const uint8_t *row = lds + buffer * Lds::stage + WB + xrow + t * 16 * kBlk;
        return Codes<EXACT>(*reinterpret_cast<const uint4_t *>(row + xp0), *reinterpret_cast<const uint4_t *>(row + xp1));
    };
    auto load_w = [&](int buffer, int i) {
        const uint8_t *frag = lds + buffer * Lds::stage + (wr * AF + i) * 2048 + lane * 16;
        return Codes<EXACT>(*reinterpret_cast<const uint4_t *>(frag), *reinterpret_cast<const uint4_t *>(frag + 1024));
    };
    auto load_scale = [&](int b, int t) {
        return *reinterpret_cast<const float *>(lds + Lds::scales + (b >> 4 & 1) * Lds::chunk + ((wt * BF + t) * 16 + j) * 64 +
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
    Codes<EXACT> x[BF], wv[WBUF];
    float s[BF], wsb;
    // The products of a block in order: fragment by fragment, the last TAIL token tile by token tile.  Each is added LAG products later, when the matrix
    // pipe has it ready.
    constexpr int SLOTS = AF * BF, LAG = EXACT ? 1 : 3;
    // A block's pieces are asked for one at a time between the products, EARLY of them in the tail that follows the barrier and the others in the
    // next block: all at once they held the wavefronts up behind one another, 600 of 3170 cycles per block of 256 x 256.
    constexpr int SPREAD = 2, EARLY = TAIL * BF / SPREAD;
    static_assert(EARLY <= LOADS && (LOADS - EARLY) * SPREAD <= MAIN * BF, "every piece has its place");
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
        static_for<LOADS>([&](auto ic) { fetch_piece(ic, b, b); });
    }
    static_for<EARLY>([&](auto ic) { fetch_piece(ic, STAGES - 1, STAGES - 1); });
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

    for (int b = 0, buffer = 0; b < a.kb; ++b) {
        const int after = buffer + 1 < STAGES ? buffer + 1 : 0, before = buffer > 0 ? buffer - 1 : STAGES - 1;
        static_for<MAIN * BF>([&](auto nc) {
            constexpr int n = decltype(nc)::value, i = row_of(n), t = token_of(n);
            if constexpr (t == 0) {
                if constexpr (i + 1 < MAIN || TAIL == 1) wv[place(i + 1)] = load_w(buffer, i + 1);
                if constexpr (TAIL > 1 && i >= MAIN - TAIL) wv[place(i + TAIL)] = load_w(buffer, i + TAIL);
            }
            if constexpr (n % SPREAD == 0 && EARLY + n / SPREAD < LOADS)
                fetch_piece(std::integral_constant<int, EARLY + n / SPREAD>{}, b + STAGES - 1, before);
            p[n % (LAG + 1)] = block_product(wv[place(i)], x[t]);
            if constexpr (n >= LAG) add(std::integral_constant<int, n - LAG>{});
            __builtin_amdgcn_sched_barrier(0);
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
        __builtin_amdgcn_sched_barrier(0);
        static_for<TAIL * BF>([&](auto nc) {
            constexpr int n = MAIN * BF + decltype(nc)::value, i = row_of(n), t = token_of(n);
            if constexpr ((n - MAIN * BF) % SPREAD == 0)
                fetch_piece(std::integral_constant<int, (n - MAIN * BF) / SPREAD>{}, b + STAGES, buffer);
            p[n % (LAG + 1)] = block_product(wv[place(i)], x[t]);
            if constexpr (i == AF - 1) x[t] = load_x(after, t);
            add(std::integral_constant<int, n - LAG>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        static_for<LAG>([&](auto nc) { add(std::integral_constant<int, SLOTS - LAG + decltype(nc)::value>{}); });
#pragma unroll
        for (int t = 0; t < BF; ++t) s[t] = sn[t] * wsb;
        buffer = after;
    }

    // Results to LDS: a row of BM per token, its 16-byte pieces in another order in each of 16 rows; from there a piece per lane and store.
    constexpr int PIECE = 16 / sizeof(E), PER_ROW = BM / PIECE;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
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
                *reinterpret_cast<vec *>(lds + (tok * PER_ROW + (c ^ (tok & 15))) * 16) = v;
            }
    }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < toks * PER_ROW; i += WAVES * kWave) {
        const int tok = i / PER_ROW, c = i % PER_ROW, o = o0 + c * PIECE;
        if (o < a.n) {
            typedef E vec __attribute__((ext_vector_type(PIECE)));
            const vec v = *reinterpret_cast<const vec *>(lds + (tok * PER_ROW + (c ^ (tok & 15))) * 16);
            E *row = static_cast<E *>(a.Y) + (int64_t)(tok0 + tok) * a.y_ld;
            if (o + PIECE <= a.n) {
                Piece<T, PIECE>::store_streaming(row + o, v);
            } else {
#pragma unroll
                for (int z = 0; z < PIECE; ++z)
                    if (o + z < a.n) row[o + z] = v[z];
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
    constexpr int BM = 16 * AF * WR, BN = 16 * BF * WT;
    constexpr size_t LDS = TileLds<BM, BN, STAGES>::bytes;
    a.tiles_o = (int)(((int64_t)a.n + BM - 1) / BM);
    a.tiles_t = (int)(((int64_t)a.m + BN - 1) / BN);
    const int64_t tiles = (int64_t)a.tiles_o * a.tiles_t;
    if (tiles * (WR * WT * kWave) > UINT32_MAX) return SLIM_ERR_SHAPE;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(block_tile_kernel<WR, WT, AF, BF, STAGES, EXACT, T>), dim3((unsigned)tiles), dim3(WR * WT * kWave), LDS,
                       st, a);
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
