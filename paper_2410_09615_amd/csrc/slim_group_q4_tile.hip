// Products with 4-bit weights that have a scale for each group of inputs, for many tokens: tiles through LDS.
//   plain       Y = X W^T
//   gated       H = silu(X Wg^T) * (X Wu^T), and where asked for G = X Wg^T and U = X Wu^T
//   transposed  dX = sum of dY_i W_i over one or two layers
// A workgroup has a tile of BT tokens x BO outputs and goes over the inputs 64 at a time.  Codes become numbers of the inputs' type, (c - z) s rounded
// once to it, on their way into LDS, so that they are converted once per workgroup; the inputs go there as they are.  Products are summed in binary32 by
// the 32 x 32 x 16 matrix instructions, the weights as their A operand, and each result is rounded once.
#include <hip/hip_runtime.h>

#include "slim_group_q4.h"
#include "slim_mma.h"

namespace slim {

enum Gq4Mode { kGq4Plain, kGq4Gated, kGq4Transposed };

struct Gq4TileArgs {
    Gq4Weights w[2];
    const void *x[2];
    int64_t x_ld[2];
    void *y[3];              // plain, transposed: the result; gated: H, G, U (G and U may be null)
    int64_t y_ld[3];
    int n, k, m, cb, rb, kg; // the layer: rows, inputs; blocks of inputs, blocks of rows, groups of a row
    int terms;               // layers that a transposed product goes over
    int tiles_o, tiles_t;
};

// The 16-byte pieces of an LDS row of 64 values are put in another order in each of eight rows, so that the lanes of a read or write find all banks; the
// order is the same 32 rows on.
__device__ __forceinline__ uint32_t gq4_turn(uint32_t row) { return (row & 7u) ^ (row >> 3 & 3u); }

// How the loop over the inputs is laid out.  KG groups of WR x WT wavefronts take turns at pieces of 64 inputs, each with two buffers of its own in LDS.  While a
// piece is multiplied from one buffer, the next one goes from registers into the other, codes becoming numbers on the way, and the one after that is asked for from
// memory into the registers that this frees: every quarter of a piece's products (16 inputs) has a quarter of that work beside it.  One barrier per piece.
// Inputs that end inside a piece are left for last and taken without that overlap.
template <class T, int MODE, int SHIFT, int KG, int WR, int WT, int AF, int BF>
__global__ __launch_bounds__(KG *WR *WT *kWave, 2) void gq4_tile_kernel(Gq4TileArgs a)
{
    typedef typename T::type E;
    typedef typename Gq4Vec<T>::v8 vec8;
    constexpr int THREADS = WR * WT * kWave, BO = 32 * AF * WR, BT = 32 * BF * WT, STAGE = (BO + BT) * 128;
    constexpr bool TRANS = MODE == kGq4Transposed, GATED = MODE == kGq4Gated;
    constexpr int XTASKS = BT * 8 / THREADS, WTASKS = BO * (TRANS ? 2 : 4) / THREADS, PARTS = TRANS ? 4 : 2;      // (codes come in dwords: of four rows, of two quarters)
    static_assert(XTASKS * THREADS == BT * 8 && WTASKS * THREADS == BO * (TRANS ? 2 : 4) && (!GATED || AF % 2 == 0) && (!TRANS || BO % 128 == 0), "tile");
    extern __shared__ __align__(16) uint8_t lds[];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x & (kWave - 1);
    const int group = KG > 1 ? wave / (WR * WT) : 0, gw = KG > 1 ? wave % (WR * WT) : wave, tid = gw * kWave + lane;
    const int wr = gw % WR, wt = gw / WR;
    const int gx = a.tiles_o * a.tiles_t;
    const int qx = gx % kDies == 0 ? ((int)blockIdx.x % kDies) * (gx / kDies) + (int)blockIdx.x / kDies : (int)blockIdx.x;
    const int tile = blocked_tile(qx, a.tiles_o, a.tiles_t);
    const int o0 = tile % a.tiles_o * (GATED ? BO / 2 : BO), t0 = tile / a.tiles_o * BT;
    const int len = TRANS ? a.n : a.k, outs = TRANS ? a.k : a.n;                 // what is summed over; results of a token
    const int whole = len / 64, terms = TRANS ? a.terms : 1, steps = whole * terms;
    uint8_t *const own = lds + group * (2 * STAGE);

    // ---- where this thread's share of a piece lies: uniform bases, and 32 bits from there on ----
    uint32_t x_at[XTASKS], w_at[WTASKS], s_at[WTASKS];
    const uint8_t *codes[WTASKS];
    const half_t *scales[WTASKS];
    const uint8_t *zeros[WTASKS];
#pragma unroll
    for (int i = 0; i < XTASKS; ++i) {
        const int task = tid + i * THREADS;
        x_at[i] = (uint32_t)min(task >> 3, a.m - 1 - t0);                        // (times the row's length, which a term has its own of)
    }
    auto weights = [&](int term) {
#pragma unroll
        for (int i = 0; i < WTASKS; ++i) {
            const int b = gw + i * (WR * WT);                                     // the block of 16 x 128 this wavefront has a part of
            if constexpr (!TRANS) {
                const int r = lane & 15, rb = min(GATED ? o0 / 16 + (b >> 2) * 2 + (b & 1) : o0 / 16 + b, a.rb - 1);
                const Gq4Weights &w = GATED && (b & 2) ? a.w[1] : a.w[0];
                codes[i] = w.codes + (int64_t)rb * a.cb * kGq4Block;
                w_at[i] = (uint32_t)lane * 16u;
                scales[i] = w.scales + (int64_t)rb * kGq4Rows * a.kg;
                zeros[i] = w.zeros ? w.zeros + (int64_t)rb * kGq4Rows * a.kg : nullptr;
                s_at[i] = (uint32_t)min(r, a.n - 1 - rb * kGq4Rows) * (uint32_t)a.kg;
            } else {
                const int j = lane & 3, p = lane >> 2 & 3, q = lane >> 4, rl = b & 3, cb = min(o0 / 128 + (b >> 2), a.cb - 1);
                const Gq4Weights &w = a.w[term];
                codes[i] = w.codes + ((int64_t)rl * a.cb + cb) * kGq4Block;
                w_at[i] = (uint32_t)((q * 16 + 4 * p) * 16 + j * 4);
                scales[i] = w.scales + (int64_t)rl * kGq4Rows * a.kg;
                zeros[i] = w.zeros ? w.zeros + (int64_t)rl * kGq4Rows * a.kg : nullptr;
                s_at[i] = (uint32_t)(4 * p) * (uint32_t)a.kg + (uint32_t)min((cb * 128 + 32 * j) >> SHIFT, a.kg - 1);
            }
        }
    };

    vec8 xv[XTASKS];
    uint32_t wv[WTASKS][PARTS], zv[WTASKS][PARTS];
    half_t sv[WTASKS][PARTS];
    // of the term's inputs from `at` on: task i of the tokens, task i of the weights
    auto fetch_x = [&](int i, int term, int at) {
        const uint8_t *base = static_cast<const uint8_t *>(term ? a.x[1] : a.x[0]);
        const int64_t ld = term ? a.x_ld[1] : a.x_ld[0];
        base += ((int64_t)t0 * ld + at) * 2;
        xv[i] = Piece<T, 8>::load(reinterpret_cast<const E *>(base + (x_at[i] * (uint32_t)ld + (uint32_t)(tid & 7) * 8u) * 2u));
    };
    auto fetch_w = [&](int i, int at) {
        if constexpr (!TRANS) {
            const uint2_t d = *reinterpret_cast<const uint2_t *>(codes[i] + ((int64_t)(at >> 7) * kGq4Block + (at & 64) / 8) + w_at[i]);
            wv[i][0] = d[0];
            wv[i][1] = d[1];
#pragma unroll
            for (int j = 0; j < (SHIFT == 5 ? 2 : 1); ++j) {
                const int gi = (at + 32 * j) >> SHIFT;
                sv[i][j] = *(scales[i] + gi + s_at[i]);
                zv[i][j] = zeros[i] ? (uint32_t) * (zeros[i] + gi + s_at[i]) : (uint32_t)kGq4Sym;
            }
        } else {
            const uint8_t *c = codes[i] + (int64_t)(at >> 4) * a.cb * kGq4Block;
            const half_t *s = scales[i] + (int64_t)at * a.kg;
            const uint8_t *z = zeros[i] + (int64_t)at * a.kg;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                wv[i][e] = *reinterpret_cast<const uint32_t *>(c + 16 * e + w_at[i]);
                sv[i][e] = *(s + (int64_t)e * a.kg + s_at[i]);
                zv[i][e] = zeros[i] ? (uint32_t) * (z + (int64_t)e * a.kg + s_at[i]) : (uint32_t)kGq4Sym;
            }
        }
    };
    // ---- into LDS ----
    uint32_t xl_at[XTASKS];
#pragma unroll
    for (int i = 0; i < XTASKS; ++i) {
        const uint32_t row = (uint32_t)(tid + i * THREADS) >> 3;
        xl_at[i] = BO * 128u + row * 128u + (((uint32_t)tid & 7u) ^ gq4_turn(row)) * 16u;
    }
    auto put_x = [&](int i, uint8_t *to) { *reinterpret_cast<vec8 *>(to + xl_at[i]) = xv[i]; };
    // quarter `h` of a weight task: forward a half of dword h / 2's work is not worth splitting: dword h / 2 at even h; transposed inputs 2 h and 2 h + 1 of the four rows
    auto put_w = [&](int i, int h, uint8_t *to) {
        const uint32_t b = (uint32_t)(gw + i * (WR * WT));
        if constexpr (!TRANS) {
            if (h & 1) return;
            const int j = h / 2, js = SHIFT == 5 ? j : 0;
            const uint32_t q = (uint32_t)lane >> 4, row = b * 16 + (lane & 15);
            const Gq4Pair<T> value(sv[i][js], zv[i][js], sv[i][js], zv[i][js]);
            uint4_t v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = value(wv[i][j] >> (4 * e));
            *reinterpret_cast<uint4_t *>(to + row * 128 + ((4u * j + q) ^ gq4_turn(row)) * 16) = v;
        } else {
            const uint32_t j = lane & 3, p = lane >> 2 & 3, q = lane >> 4, piece = (b & 3) * 2 + (p >> 1);
            const Gq4Pair<T> v01(sv[i][0], zv[i][0], sv[i][1], zv[i][1]), v23(sv[i][2], zv[i][2], sv[i][3], zv[i][3]);
#pragma unroll
            for (int e = 2 * h; e < 2 * h + 2; ++e) {
                const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;          // the nibbles of input e of both rows, as halves
                const uint32_t d01 = __builtin_amdgcn_perm(wv[i][1], wv[i][0], sel), d23 = __builtin_amdgcn_perm(wv[i][3], wv[i][2], sel);
                const uint32_t col = (b >> 2) * 128 + 32 * j + 8 * q + e;
                const uint2_t v = {v01(d01 >> (4 * (e >> 1))), v23(d23 >> (4 * (e >> 1)))};
                *reinterpret_cast<uint2_t *>(to + col * 128 + (piece ^ gq4_turn(col)) * 16 + (p & 1) * 8) = v;
            }
        }
    };

    float16_t acc[AF][BF];
#pragma unroll
    for (int i = 0; i < AF; ++i)
#pragma unroll
        for (int t = 0; t < BF; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][t][e] = 0.f;

    const uint32_t fr = (uint32_t)lane & 31u, fh = (uint32_t)lane >> 5, turned = (fh ^ gq4_turn(fr)) * 16u;
    const uint32_t wl_at = (uint32_t)(wr * AF * 32) * 128u + fr * 128u, xl_from = (uint32_t)(BO + wt * BF * 32) * 128u + fr * 128u;
    auto read = [&](const uint8_t *from, int kk, vec8 (&af)[AF], vec8 (&bf)[BF]) {
#pragma unroll
        for (int i = 0; i < AF; ++i) af[i] = *reinterpret_cast<const vec8 *>(from + wl_at + (turned ^ (uint32_t)kk * 32u) + i * 4096);
#pragma unroll
        for (int t = 0; t < BF; ++t) bf[t] = *reinterpret_cast<const vec8 *>(from + xl_from + (turned ^ (uint32_t)kk * 32u) + t * 4096);
    };
    auto multiply = [&](const vec8 (&af)[AF], const vec8 (&bf)[BF]) {
#pragma unroll
        for (int t = 0; t < BF; ++t)
#pragma unroll
            for (int i = 0; i < AF; ++i) acc[i][t] = gq4_mma32(af[i], bf[t], acc[i][t]);
    };

    // Step s of the group is piece group + s KG of all terms' whole ones.  (Past the last the last is fetched again, and not used.)
    const int turns = (steps + KG - 1) / KG, mine = (steps - group + KG - 1) / KG;
    auto place = [&](int s, int &term, int &at) {
        const int step = min(group + s * KG, steps - 1);
        term = TRANS && step >= whole ? 1 : 0;
        at = (step - term * whole) * 64;
    };
    int loaded = 0;                                                              // the term whose weights' bases are held
    weights(0);
    auto use_term = [&](int term) {
        if (TRANS && term != loaded) {
            weights(term);
            loaded = term;
        }
    };
    if (steps > 0) {
        int term, at;
        place(0, term, at);
        use_term(term);
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) fetch_x(i, term, at);
#pragma unroll
        for (int i = 0; i < WTASKS; ++i) fetch_w(i, at);
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) put_x(i, own);
#pragma unroll
        for (int i = 0; i < WTASKS; ++i)
#pragma unroll
            for (int h = 0; h < 4; ++h) put_w(i, h, own);
        place(1, term, at);
        use_term(term);
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) fetch_x(i, term, at);
#pragma unroll
        for (int i = 0; i < WTASKS; ++i) fetch_w(i, at);
        __syncthreads();
        for (int s = 0; s < turns; ++s) {
            uint8_t *const from = own + (s & 1) * STAGE, *const to = own + (~s & 1) * STAGE;
            place(s + 2, term, at);
            use_term(term);
            if (s < mine) {
                vec8 af[2][AF], bf[2][BF];
                read(from, 0, af[0], bf[0]);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                    if (kk < 3) read(from, kk + 1, af[(kk + 1) & 1], bf[(kk + 1) & 1]);
#pragma unroll
                    for (int i = 0; i < XTASKS; ++i)
                        if (i * 4 / XTASKS == kk) {
                            put_x(i, to);
                            fetch_x(i, term, at);
                        }
#pragma unroll
                    for (int i = 0; i < WTASKS; ++i) {
                        put_w(i, kk, to);
                        if (kk == 3) fetch_w(i, at);
                    }
                    multiply(af[kk & 1], bf[kk & 1]);
                }
            }
            __syncthreads();
        }
    }
    if (len % 64) {
        const int at = whole * 64;
        for (int term = 0; term < terms; ++term) {
            __syncthreads();
            if (group == 0) {
                use_term(term);
                const E *x = static_cast<const E *>(term ? a.x[1] : a.x[0]);
                const int64_t ld = term ? a.x_ld[1] : a.x_ld[0];
#pragma unroll
                for (int i = 0; i < XTASKS; ++i) {
                    const E *row = x + ((int64_t)t0 + x_at[i]) * ld;
                    const int c = at + (tid & 7) * 8;
#pragma unroll
                    for (int e = 0; e < 8; ++e) xv[i][e] = c + e < len ? row[c + e] : (E)0.f;
                    put_x(i, own);
                }
#pragma unroll
                for (int i = 0; i < WTASKS; ++i) {
                    if constexpr (!TRANS) {
                        const uint2_t d = *reinterpret_cast<const uint2_t *>(codes[i] + ((int64_t)(at >> 7) * kGq4Block + (at & 64) / 8) + w_at[i]);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int gi = min((at + 32 * j) >> SHIFT, a.kg - 1);
                            wv[i][j] = d[j];
                            sv[i][j] = *(scales[i] + gi + s_at[i]);
                            zv[i][j] = zeros[i] ? (uint32_t) * (zeros[i] + gi + s_at[i]) : (uint32_t)kGq4Sym;
                        }
                    } else {
                        const int rl = (gw + i * (WR * WT)) & 3, p = lane >> 2 & 3, block = min((at >> 4) + rl, a.rb - 1) - rl;
                        const uint8_t *c = codes[i] + (int64_t)block * a.cb * kGq4Block;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int row = at + rl * 16 + 4 * p + e, up = min(row, a.n - 1) - rl * 16 - 4 * p;      // rows from the lane's own of the first blocks
                            wv[i][e] = *reinterpret_cast<const uint32_t *>(c + 16 * e + w_at[i]);
                            sv[i][e] = row < a.n ? scales[i][(int64_t)up * a.kg + s_at[i]] : (half_t)0.f;            // (rows past the last are no terms of the sum)
                            zv[i][e] = zeros[i] ? (uint32_t)zeros[i][(int64_t)up * a.kg + s_at[i]] : (uint32_t)kGq4Sym;
                        }
                    }
#pragma unroll
                    for (int h = 0; h < 4; ++h) put_w(i, h, own);
                }
            }
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                    vec8 af[AF], bf[BF];
                    read(own, kk, af, bf);
                    multiply(af, bf);
                }
            }
        }
    }
    if constexpr (KG > 1) {
        // the groups' sums, added in order: group 1 .. hand theirs to group 0
        float16_t *part = reinterpret_cast<float16_t *>(lds);
        for (int g = 1; g < KG; ++g) {
            __syncthreads();
            if (group == g) {
#pragma unroll
                for (int i = 0; i < AF; ++i)
#pragma unroll
                    for (int t = 0; t < BF; ++t) part[(i * BF + t) * THREADS + tid] = acc[i][t];
            }
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int i = 0; i < AF; ++i)
#pragma unroll
                    for (int t = 0; t < BF; ++t) acc[i][t] += part[(i * BF + t) * THREADS + tid];
            }
        }
    }

    // Results leave through LDS, so that a store writes whole pieces of a token's row.
    constexpr int OUT = GATED ? BO / 2 : BO, PER_ROW = OUT / 8, TURN = (PER_ROW < 16 ? PER_ROW : 16) - 1;
    typedef E vec4 __attribute__((ext_vector_type(4)));
    auto leave = [&](void *y, int64_t y_ld, auto &&value) {
        __syncthreads();
        if (KG == 1 || group == 0)
#pragma unroll
        for (int i = 0; i < AF; i += GATED ? 2 : 1)
#pragma unroll
            for (int t = 0; t < BF; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    vec4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = (E)value(i, t, 4 * g + e);
                    const int tok = (wt * BF + t) * 32 + (lane & 31), c = ((GATED ? (wr * AF + i) / 2 : wr * AF + i) * 32 + 8 * g) / 8;
                    *reinterpret_cast<vec4 *>(lds + (tok * PER_ROW + (c ^ (tok & TURN))) * 16 + (lane >> 5) * 8) = v;
                }
        __syncthreads();
        const int toks = min(BT, a.m - t0);
        for (int i = (int)threadIdx.x; i < toks * PER_ROW; i += KG * THREADS) {
            const int tok = i / PER_ROW, c = i % PER_ROW, o = o0 + c * 8;
            if (o < outs) {
                const vec8 v = *reinterpret_cast<const vec8 *>(lds + (tok * PER_ROW + (c ^ (tok & TURN))) * 16);
                E *row = static_cast<E *>(y) + (int64_t)(t0 + tok) * y_ld;
                if (o + 8 <= outs)
                    Piece<T, 8>::store(row + o, v);
                else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (o + e < outs) row[o + e] = v[e];
                }
            }
        }
    };
    if constexpr (GATED) {
        leave(a.y[0], a.y_ld[0], [&](int i, int t, int e) {
            const float g = acc[i][t][e];
            return g * gq4_sigma(g) * acc[i + 1][t][e];
        });
        if (a.y[1]) leave(a.y[1], a.y_ld[1], [&](int i, int t, int e) { return acc[i][t][e]; });
        if (a.y[2]) leave(a.y[2], a.y_ld[2], [&](int i, int t, int e) { return acc[i + 1][t][e]; });
    } else
        leave(a.y[0], a.y_ld[0], [&](int i, int t, int e) { return acc[i][t][e]; });
}

template <class T, int MODE, int SHIFT, int KG, int WR, int WT, int AF, int BF>
static int launch_gq4_tile(Gq4TileArgs a, hipStream_t st)
{
    constexpr int THREADS = KG * WR * WT * kWave, BO = 32 * AF * WR, BT = 32 * BF * WT;
    constexpr size_t LDS = 2 * (size_t)KG * (BO + BT) * 128;
    static_assert(LDS <= 160 * 1024 && (size_t)BO * BT * (KG > 1 ? 4 : 2) <= LDS, "LDS");
    const int outs = MODE == kGq4Transposed ? a.k : a.n, wide = MODE == kGq4Gated ? BO / 2 : BO;
    a.tiles_o = (int)(((int64_t)outs + wide - 1) / wide);
    a.tiles_t = (int)(((int64_t)a.m + BT - 1) / BT);
    const int64_t tiles = (int64_t)a.tiles_o * a.tiles_t;
    if (tiles * THREADS > UINT32_MAX) return SLIM_ERR_SHAPE;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_tile_kernel<T, MODE, SHIFT, KG, WR, WT, AF, BF>), dim3((unsigned)tiles), dim3(THREADS), LDS, st, a);
    return SLIM_OK;
}

template <class T, int MODE, int SHIFT>
static int launch_gq4_shape(const Gq4TileArgs &a, hipStream_t st)
{
    int shape = a.m > 256 ? 0 : 2;
    if (const char *e = getenv("GQ4_T")) shape = atoi(e);
    switch (shape) {
    case 0: return launch_gq4_tile<T, MODE, SHIFT, 1, 4, 2, 2, 4>(a, st);     // 256 x 256
    case 1: return launch_gq4_tile<T, MODE, SHIFT, 1, 4, 2, 2, 2>(a, st);     // 256 x 128
    case 2: return launch_gq4_tile<T, MODE, SHIFT, 1, 2, 2, 2, 2>(a, st);     // 128 x 128
    case 3: return launch_gq4_tile<T, MODE, SHIFT, 2, 2, 2, 2, 1>(a, st);     // 128 x 64, two groups
    default: return launch_gq4_tile<T, MODE, SHIFT, 2, 2, 2, 2, 2>(a, st);    // 128 x 128, two groups
    }
}

template <int MODE>
static int launch_gq4(const Gq4TileArgs &a, int shift, int32_t dtype, hipStream_t st)
{
    auto of = [&](auto type) {
        typedef decltype(type) T;
        return shift == 5 ? launch_gq4_shape<T, MODE, 5>(a, st) : shift == 6 ? launch_gq4_shape<T, MODE, 6>(a, st) : launch_gq4_shape<T, MODE, 7>(a, st);
    };
    const int rc = dtype == SLIM_F16 ? of(F16{}) : of(BF16{});
    return rc != SLIM_OK ? rc : hip_status(hipGetLastError());
}

int gq4_launch_act_backward(const void *dH, int64_t h_ld, const void *G, int64_t g_ld, const void *U, int64_t u_ld, int32_t m, int32_t n, void *dG,
                            int64_t dg_ld, void *dU, int64_t du_ld, int32_t dtype, hipStream_t st);

// Weights are streamed for up to so many tokens (whose row stride leaves a token within 32 bits of the first).
static bool gq4_few(int m, int64_t x_ld) { return m <= kGq4Few && x_ld < (1 << 24); }
int gq4_launch_stream(const slim_group_q4_layer *layer, const slim_group_q4_layer *up, int shift, const void *X, int64_t x_ld, int32_t m, void *const (&y)[3],
                      const int64_t (&y_ld)[3], int32_t dtype, hipStream_t st);

static Gq4TileArgs gq4_args(const slim_group_q4_layer *l, int shift, int m)
{
    Gq4TileArgs a{};
    a.w[0] = gq4_weights(l);
    a.n = l->n;
    a.k = l->k;
    a.m = m;
    a.cb = gq4_col_blocks(l->k);
    a.rb = gq4_row_blocks(l->n);
    a.kg = gq4_groups(l->k, shift);
    a.terms = 1;
    return a;
}

// Both layers of a gated block: of one shape and group.
static int gq4_check_pair(const slim_group_q4_layer *gate, const slim_group_q4_layer *up, int *shift)
{
    const int one = gq4_check(gate, shift), two = gq4_check(up, shift);
    if (one == SLIM_ERR_NULL || two == SLIM_ERR_NULL) return SLIM_ERR_NULL;
    if (one == SLIM_ERR_SHAPE || two == SLIM_ERR_SHAPE || gate->n != up->n || gate->k != up->k || gate->group != up->group) return SLIM_ERR_SHAPE;
    return one != SLIM_OK ? one : two;
}

}  // namespace slim

using namespace slim;

extern "C" int slim_group_q4_gemm(const slim_group_q4_layer *layer, const void *X, int64_t x_ld, int32_t m, void *Y, int64_t y_ld, int32_t dtype,
                                  void *stream)
{
    if (!X || !Y) return SLIM_ERR_NULL;
    int shift;
    const int status = gq4_check(layer, &shift);
    if (status == SLIM_ERR_NULL || status == SLIM_ERR_SHAPE) return status;
    if (m < 1 || !half_dtype(dtype) || x_ld < layer->k || y_ld < layer->n) return SLIM_ERR_SHAPE;
    if (status != SLIM_OK || !whole_elements(X, dtype) || !whole_elements(Y, dtype)) return SLIM_ERR_ALIGN;
    Gq4TileArgs a = gq4_args(layer, shift, m);
    a.x[0] = X;
    a.x_ld[0] = x_ld;
    a.y[0] = Y;
    a.y_ld[0] = y_ld;
    if (gq4_few(m, x_ld)) return gq4_launch_stream(layer, nullptr, shift, X, x_ld, m, a.y, a.y_ld, dtype, static_cast<hipStream_t>(stream));
    return launch_gq4<kGq4Plain>(a, shift, dtype, static_cast<hipStream_t>(stream));
}

extern "C" int slim_group_q4_gemm_t(const slim_group_q4_layer *layer, const void *dY, int64_t dy_ld, int32_t m, void *dX, int64_t dx_ld, int32_t dtype,
                                    void *stream)
{
    if (!dY || !dX) return SLIM_ERR_NULL;
    int shift;
    const int status = gq4_check(layer, &shift);
    if (status == SLIM_ERR_NULL || status == SLIM_ERR_SHAPE) return status;
    if (m < 1 || !half_dtype(dtype) || dy_ld < layer->n || dx_ld < layer->k) return SLIM_ERR_SHAPE;
    if (status != SLIM_OK || !whole_elements(dY, dtype) || !whole_elements(dX, dtype)) return SLIM_ERR_ALIGN;
    Gq4TileArgs a = gq4_args(layer, shift, m);
    a.x[0] = dY;
    a.x_ld[0] = dy_ld;
    a.y[0] = dX;
    a.y_ld[0] = dx_ld;
    return launch_gq4<kGq4Transposed>(a, shift, dtype, static_cast<hipStream_t>(stream));
}

extern "C" int slim_group_q4_gated(const slim_group_q4_layer *gate, const slim_group_q4_layer *up, const void *X, int64_t x_ld, int32_t m, void *H,
                                   int64_t h_ld, void *G, int64_t g_ld, void *U, int64_t u_ld, int32_t dtype, void *stream)
{
    if (!X || !H) return SLIM_ERR_NULL;
    int shift;
    const int status = gq4_check_pair(gate, up, &shift);
    if (status == SLIM_ERR_NULL || status == SLIM_ERR_SHAPE) return status;
    if (m < 1 || !half_dtype(dtype) || x_ld < gate->k || h_ld < gate->n || (G && g_ld < gate->n) || (U && u_ld < gate->n)) return SLIM_ERR_SHAPE;
    if (status != SLIM_OK || !whole_elements(X, dtype) || !whole_elements(H, dtype) || !whole_elements(G, dtype) || !whole_elements(U, dtype)) return SLIM_ERR_ALIGN;
    Gq4TileArgs a = gq4_args(gate, shift, m);
    a.w[1] = gq4_weights(up);
    a.x[0] = X;
    a.x_ld[0] = x_ld;
    a.y[0] = H;
    a.y_ld[0] = h_ld;
    a.y[1] = G;
    a.y_ld[1] = g_ld;
    a.y[2] = U;
    a.y_ld[2] = u_ld;
    if (gq4_few(m, x_ld)) return gq4_launch_stream(gate, up, shift, X, x_ld, m, a.y, a.y_ld, dtype, static_cast<hipStream_t>(stream));
    return launch_gq4<kGq4Gated>(a, shift, dtype, static_cast<hipStream_t>(stream));
}

extern "C" int slim_group_q4_gated_backward(const slim_group_q4_layer *gate, const slim_group_q4_layer *up, const void *dH, int64_t dh_ld, const void *G,
                                            int64_t g_ld, const void *U, int64_t u_ld, int32_t m, void *dG, int64_t dg_ld, void *dU, int64_t du_ld,
                                            void *dX, int64_t dx_ld, int32_t dtype, void *stream)
{
    if (!dH || !G || !U || !dG || !dU || !dX) return SLIM_ERR_NULL;
    int shift;
    const int status = gq4_check_pair(gate, up, &shift);
    if (status == SLIM_ERR_NULL || status == SLIM_ERR_SHAPE) return status;
    const int n = gate->n;
    if (m < 1 || !half_dtype(dtype) || dh_ld < n || g_ld < n || u_ld < n || dg_ld < n || du_ld < n || dx_ld < gate->k || dG == dU) return SLIM_ERR_SHAPE;
    if (status != SLIM_OK) return status;
    for (const void *p : {dH, G, U, (const void *)dG, (const void *)dU, (const void *)dX})
        if (!whole_elements(p, dtype)) return SLIM_ERR_ALIGN;
    Gq4TileArgs a = gq4_args(gate, shift, m);
    a.w[1] = gq4_weights(up);
    a.terms = 2;
    a.x[0] = dG;
    a.x_ld[0] = dg_ld;
    a.x[1] = dU;
    a.x_ld[1] = du_ld;
    a.y[0] = dX;
    a.y_ld[0] = dx_ld;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int rc = gq4_launch_act_backward(dH, dh_ld, G, g_ld, U, u_ld, m, n, dG, dg_ld, dU, du_ld, dtype, st);
    return rc != SLIM_OK ? rc : launch_gq4<kGq4Transposed>(a, shift, dtype, st);
}
