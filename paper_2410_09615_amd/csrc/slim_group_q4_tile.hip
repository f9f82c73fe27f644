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

// The 16-byte pieces of an LDS row of 64 values are put in another order in each of eight rows, so that the lanes of a read or write find all banks.
__device__ __forceinline__ uint32_t gq4_turn(uint32_t row) { return (row ^ (row >> 3)) & 7u; }

template <class T, int MODE, int SHIFT, int WR, int WT, int AF, int BF>
__global__ __launch_bounds__(WR *WT *kWave, 2) void gq4_tile_kernel(Gq4TileArgs a)
{
    typedef typename T::type E;
    typedef typename Gq4Vec<T>::v8 vec8;
    constexpr int THREADS = WR * WT * kWave, BO = 32 * AF * WR, BT = 32 * BF * WT, STAGE = (BO + BT) * 128;
    constexpr bool TRANS = MODE == kGq4Transposed, GATED = MODE == kGq4Gated;
    constexpr int XTASKS = BT * 8 / THREADS, WTASKS = BO * (TRANS ? 2 : 4) / THREADS;
    static_assert(XTASKS * THREADS == BT * 8 && WTASKS * THREADS == BO * (TRANS ? 2 : 4) && (!GATED || AF % 2 == 0) && (!TRANS || BO % 128 == 0), "tile");
    extern __shared__ __align__(16) uint8_t lds[];
    const int tid = (int)threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int wr = wave % WR, wt = wave / WR;
    const int gx = a.tiles_o * a.tiles_t;
    const int qx = gx % kDies == 0 ? ((int)blockIdx.x % kDies) * (gx / kDies) + (int)blockIdx.x / kDies : (int)blockIdx.x;
    const int tile = blocked_tile(qx, a.tiles_o, a.tiles_t);
    const int o0 = tile % a.tiles_o * (GATED ? BO / 2 : BO), t0 = tile / a.tiles_o * BT;
    const int len = TRANS ? a.n : a.k, outs = TRANS ? a.k : a.n;                 // what is summed over; results of a token
    const int per_term = (len + 63) / 64, steps = TRANS ? per_term * a.terms : per_term;

    uint4_t xv[XTASKS];
    uint32_t wv[WTASKS][TRANS ? 4 : 2];
    half_t sv[WTASKS][TRANS ? 4 : 2];
    uint32_t zv[WTASKS][TRANS ? 4 : 2];

    auto fetch = [&](int step) {
        const int term = TRANS && step >= per_term ? 1 : 0, at = (step - term * per_term) * 64;
        const E *x = static_cast<const E *>(term ? a.x[1] : a.x[0]);
        const int64_t x_ld = term ? a.x_ld[1] : a.x_ld[0];
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) {
            const int task = tid + i * THREADS, c = at + (task & 7) * 8;
            const E *row = x + (int64_t)min(t0 + (task >> 3), a.m - 1) * x_ld;
            if (c + 8 <= len)
                xv[i] = __builtin_bit_cast(uint4_t, Piece<T, 8>::load(row + c));
            else {
                vec8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = c + e < len ? row[c + e] : (E)0.f;
                xv[i] = __builtin_bit_cast(uint4_t, v);
            }
        }
#pragma unroll
        for (int i = 0; i < WTASKS; ++i) {
            const int task = tid + i * THREADS, b = task / kWave, l = task % kWave;
            if constexpr (!TRANS) {
                const int r = l & 15;
                const int rb = min(GATED ? o0 / 16 + (b >> 2) * 2 + (b & 1) : o0 / 16 + b, a.rb - 1);
                const Gq4Weights &w = GATED && (b & 2) ? a.w[1] : a.w[0];
                const uint2_t d = *reinterpret_cast<const uint2_t *>(w.codes + ((int64_t)rb * a.cb + (at >> 7)) * kGq4Block + l * 16 + (at & 64) / 8);
                wv[i][0] = d[0];
                wv[i][1] = d[1];
                const int64_t g = (int64_t)min(rb * 16 + r, a.n - 1) * a.kg;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (j == 1 && SHIFT > 5) {
                        sv[i][1] = sv[i][0];
                        zv[i][1] = zv[i][0];
                    } else {
                        const int gi = min((at + 32 * j) >> SHIFT, a.kg - 1);
                        sv[i][j] = w.scales[g + gi];
                        zv[i][j] = w.zeros ? w.zeros[g + gi] : kGq4Sym;
                    }
                }
            } else {
                const int j = l & 3, p = l >> 2 & 3, q = l >> 4, rl = b & 3;
                const int rb = min((at >> 4) + rl, a.rb - 1), cb = min(o0 / 128 + (b >> 2), a.cb - 1);
                const Gq4Weights &w = term ? a.w[1] : a.w[0];
                const uint32_t *d = reinterpret_cast<const uint32_t *>(w.codes + ((int64_t)rb * a.cb + cb) * kGq4Block) + (q * 16 + 4 * p) * 4 + j;
                const int gi = min((cb * 128 + 32 * j) >> SHIFT, a.kg - 1);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = at + rl * 16 + 4 * p + e;
                    const int64_t g = (int64_t)min(row, a.n - 1) * a.kg + gi;
                    wv[i][e] = d[4 * e];
                    sv[i][e] = row < a.n ? w.scales[g] : (half_t)0.f;        // (rows past the last are no terms of the sum, whatever their scale)
                    zv[i][e] = w.zeros ? w.zeros[g] : kGq4Sym;
                }
            }
        }
    };
    auto stage = [&](int buffer) {
        uint8_t *wl = lds + buffer * STAGE, *xl = wl + BO * 128;
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) {
            const uint32_t task = (uint32_t)(tid + i * THREADS), row = task >> 3;
            *reinterpret_cast<uint4_t *>(xl + row * 128 + ((task & 7u) ^ gq4_turn(row)) * 16) = xv[i];
        }
#pragma unroll
        for (int i = 0; i < WTASKS; ++i) {
            const uint32_t task = (uint32_t)(tid + i * THREADS), b = task / kWave, l = task % kWave;
            if constexpr (!TRANS) {
                const uint32_t q = l >> 4, row = b * 16 + (l & 15);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const Gq4Pair<T> value(sv[i][j], zv[i][j], sv[i][j], zv[i][j]);
                    uint4_t v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = value(wv[i][j] >> (4 * e));
                    *reinterpret_cast<uint4_t *>(wl + row * 128 + ((4u * j + q) ^ gq4_turn(row)) * 16) = v;
                }
            } else {
                const uint32_t j = l & 3, p = l >> 2 & 3, q = l >> 4, piece = (b & 3) * 2 + (p >> 1);
                const Gq4Pair<T> v01(sv[i][0], zv[i][0], sv[i][1], zv[i][1]), v23(sv[i][2], zv[i][2], sv[i][3], zv[i][3]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;      // the nibbles of input e of both rows, as halves
                    const uint32_t d01 = __builtin_amdgcn_perm(wv[i][1], wv[i][0], sel), d23 = __builtin_amdgcn_perm(wv[i][3], wv[i][2], sel);
                    const uint32_t col = (b >> 2) * 128 + 32 * j + 8 * q + e;
                    const uint2_t v = {v01(d01 >> (4 * (e >> 1))), v23(d23 >> (4 * (e >> 1)))};
                    *reinterpret_cast<uint2_t *>(wl + col * 128 + (piece ^ gq4_turn(col)) * 16 + (p & 1) * 8) = v;
                }
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

    fetch(0);
    for (int step = 0; step < steps; ++step) {
        const int buffer = step & 1;
        stage(buffer);
        if (step + 1 < steps) fetch(step + 1);
        __syncthreads();
        const uint8_t *wl = lds + buffer * STAGE, *xl = wl + BO * 128;
        const uint32_t r = (uint32_t)lane & 31u, half = (uint32_t)lane >> 5;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            vec8 af[AF], bf[BF];
#pragma unroll
            for (int i = 0; i < AF; ++i) {
                const uint32_t row = (uint32_t)(wr * AF + i) * 32u + r;
                af[i] = *reinterpret_cast<const vec8 *>(wl + row * 128 + ((2u * kk + half) ^ gq4_turn(row)) * 16);
            }
#pragma unroll
            for (int t = 0; t < BF; ++t) {
                const uint32_t row = (uint32_t)(wt * BF + t) * 32u + r;
                bf[t] = *reinterpret_cast<const vec8 *>(xl + row * 128 + ((2u * kk + half) ^ gq4_turn(row)) * 16);
            }
#pragma unroll
            for (int i = 0; i < AF; ++i)
#pragma unroll
                for (int t = 0; t < BF; ++t) acc[i][t] = gq4_mma32(af[i], bf[t], acc[i][t]);
        }
    }

    // Results leave through LDS, so that a store writes whole pieces of a token's row.
    constexpr int OUT = GATED ? BO / 2 : BO, PER_ROW = OUT / 8, TURN = (PER_ROW < 16 ? PER_ROW : 16) - 1;
    typedef E vec4 __attribute__((ext_vector_type(4)));
    auto leave = [&](void *y, int64_t y_ld, auto &&value) {
        __syncthreads();
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
        for (int i = tid; i < toks * PER_ROW; i += THREADS) {
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

template <class T, int MODE, int SHIFT, int WR, int WT, int AF, int BF>
static int launch_gq4_tile(Gq4TileArgs a, hipStream_t st)
{
    constexpr int THREADS = WR * WT * kWave, BO = 32 * AF * WR, BT = 32 * BF * WT;
    constexpr size_t LDS = 2 * (size_t)(BO + BT) * 128;
    static_assert(LDS <= 160 * 1024 && (size_t)BO * BT * 2 <= LDS, "LDS");
    const int outs = MODE == kGq4Transposed ? a.k : a.n, wide = MODE == kGq4Gated ? BO / 2 : BO;
    a.tiles_o = (int)(((int64_t)outs + wide - 1) / wide);
    a.tiles_t = (int)(((int64_t)a.m + BT - 1) / BT);
    const int64_t tiles = (int64_t)a.tiles_o * a.tiles_t;
    if (tiles * THREADS > UINT32_MAX) return SLIM_ERR_SHAPE;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_tile_kernel<T, MODE, SHIFT, WR, WT, AF, BF>), dim3((unsigned)tiles), dim3(THREADS), LDS, st, a);
    return SLIM_OK;
}

template <class T, int MODE, int SHIFT>
static int launch_gq4_shape(const Gq4TileArgs &a, hipStream_t st)
{
    if (a.m > 256) return launch_gq4_tile<T, MODE, SHIFT, 4, 2, 2, 4>(a, st);
    return launch_gq4_tile<T, MODE, SHIFT, 2, 2, 2, 2>(a, st);
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
