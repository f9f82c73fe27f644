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

// Per group of wavefronts: two buffers of a piece's weights and tokens, two windows of scales and zero points.
template <int MODE, int KG, int BO, int BT>
struct Gq4TileLds {
    static constexpr int table = MODE == kGq4Transposed ? 8 * 64 * 3 : BO * 24, bytes = KG * (2 * (BO + BT) * 128 + 2 * table);
};

// How the loop over the inputs is laid out.  KG groups of WR x WT wavefronts take turns at pieces of 64 inputs, each with two buffers of its own in LDS.  While a
// piece is multiplied from one buffer, the next one goes from registers into the other, codes becoming numbers on the way, and the one after that is asked for from
// memory into the registers that this frees: every quarter of a piece's products (16 inputs) has a quarter of that work beside it.  One barrier per piece.
// Inputs that end inside a piece are left for last and taken without that overlap.
template <class T, int MODE, int SHIFT, int KG, int P, int WR, int WT, int AF, int BF>
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
    const Gq4Masks masks;
    constexpr int TABLE = Gq4TileLds<MODE, KG, BO, BT>::table;
    uint8_t *const own = lds + group * (2 * STAGE + 2 * TABLE), *const tables = own + 2 * STAGE;

    // ---- where this thread's share of a piece lies: uniform bases, and 32 bits from there on ----
    uint32_t x_at[XTASKS];
    const uint8_t *codes[WTASKS];
#pragma unroll
    for (int i = 0; i < XTASKS; ++i) x_at[i] = (uint32_t)min((tid + i * THREADS) >> 3, a.m - 1 - t0);      // (times the row's length, which a term has its own of)
    const uint32_t w_at = TRANS ? (uint32_t)(((lane >> 4) * 16 + 4 * (lane >> 2 & 3)) * 16 + (lane & 3) * 4) : (uint32_t)lane * 16u;
    auto weights = [&](int term) {
#pragma unroll
        for (int i = 0; i < WTASKS; ++i) {
            const int b = gw + i * (WR * WT);                                     // the block of 16 x 128 this wavefront has a part of
            if constexpr (!TRANS) {
                const int rb = min(GATED ? o0 / 16 + (b >> 2) * 2 + (b & 1) : o0 / 16 + b, a.rb - 1);
                codes[i] = (GATED && (b & 2) ? a.w[1].codes : a.w[0].codes) + (int64_t)rb * a.cb * kGq4Block;
            } else {
                const int cb = min(o0 / 128 + (b >> 2), a.cb - 1);
                codes[i] = (term ? a.w[1].codes : a.w[0].codes) + ((int64_t)(b & 3) * a.cb + cb) * kGq4Block;
            }
        }
    };

    struct Piece64 {                                                             // a thread's share of a piece, in registers
        vec8 x[XTASKS];
        uint32_t w[WTASKS][PARTS];
    };
    Piece64 pieces[P];
    // of the term's inputs from `at` on: task i of the tokens, task i of the weights
    auto fetch_x = [&](Piece64 &v, int i, int term, int at) {
        const uint8_t *base = static_cast<const uint8_t *>(term ? a.x[1] : a.x[0]);
        const int64_t ld = term ? a.x_ld[1] : a.x_ld[0];
        base += ((int64_t)t0 * ld + at) * 2;
        v.x[i] = Piece<T, 8>::load(reinterpret_cast<const E *>(base + (x_at[i] * (uint32_t)ld + (uint32_t)(tid & 7) * 8u) * 2u));
    };
    auto fetch_w = [&](Piece64 &v, int i, int at) {
        if constexpr (!TRANS) {
            const uint2_t d = *reinterpret_cast<const uint2_t *>(codes[i] + ((int64_t)(at >> 7) * kGq4Block + (at & 64) / 8) + w_at);
            v.w[i][0] = d[0];
            v.w[i][1] = d[1];
        } else {
            const uint8_t *c = codes[i] + (int64_t)(at >> 4) * a.cb * kGq4Block;
#pragma unroll
            for (int e = 0; e < 4; ++e) v.w[i][e] = *reinterpret_cast<const uint32_t *>(c + 16 * e + w_at);
        }
    };
    // ---- scales and zero points: windows of them in LDS, two, filled one ahead ----
    // Where each lane fetches the scale of its own row, neighbouring lanes ask the memory pipeline for different lines, which takes four times as long as when they share
    // one: so eight groups of a row are fetched by eight lanes (forward; a window is 8 groups of the tile's rows), or those of the tile's columns (transposed; a window is
    // the 64 rows of a piece).  Forward the table is [row][8 groups], transposed [group][64 rows].
    constexpr int SPAN = TRANS ? (BO >> SHIFT) : 8, ITEMS = ((TRANS ? 64 : BO) * SPAN + THREADS - 1) / THREADS;
    static_assert(SPAN <= 8, "window");
    struct Window {
        half_t s[ITEMS];
        uint32_t z[ITEMS];
        int term;
    };
    Window ahead;
    // forward: window w; transposed: rows from `at` on of the term's layer
    auto load_window = [&](int w, int term, int at) {
        ahead.term = term;
        const int wave_row = gw * kWave / SPAN;                                  // (a wavefront's items of one i are of one layer)
        int own_tid = tid;                                                       // (made anew here each time: kept over the loop, what follows from it takes too many registers)
        asm volatile("" : "+v"(own_tid));
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int item = own_tid + i * THREADS, row = item / SPAN, g = item % SPAN;
            const Gq4Weights &l = TRANS ? (term ? a.w[1] : a.w[0]) : (GATED && (i * THREADS / SPAN + wave_row & 32) ? a.w[1] : a.w[0]);
            int local = row, from = 8 * w + g, first = o0;                       // rows from the first one there
            if constexpr (TRANS) {
                first = at;
                from = (o0 >> SHIFT) + g;
            } else if constexpr (GATED)
                local = (row >> 6) * 32 + (row & 31);
            const uint8_t *scales = reinterpret_cast<const uint8_t *>(l.scales + (int64_t)first * a.kg);
            const uint8_t *zeros = l.zeros ? l.zeros + (int64_t)first * a.kg : scales;      // (symmetric: what is read of the scales instead is not used)
            const uint32_t place = (uint32_t)min(local, a.n - 1 - first) * (uint32_t)a.kg + (uint32_t)min(from, a.kg - 1);
            ahead.s[i] = *reinterpret_cast<const half_t *>(scales + place * 2u);
            ahead.z[i] = *(zeros + place);
            if constexpr (BO * BT >= 256 * 256) __builtin_amdgcn_sched_barrier(0);          // (one after the other: no registers are left)
        }
    };
    // the first `there` rows of a transposed window are there: the others are no terms of the sum
    auto put_window = [&](int w, int there) {
        uint8_t *const t = tables + (w & 1) * TABLE;
        int own_tid = tid;
        asm volatile("" : "+v"(own_tid));
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int item = own_tid + i * THREADS, row = item / SPAN, g = item % SPAN;
            if (TRANS && item >= 64 * SPAN) continue;
            const bool points = TRANS ? (ahead.term ? a.w[1].zeros : a.w[0].zeros) != nullptr : (GATED && (row & 32) ? a.w[1].zeros : a.w[0].zeros) != nullptr;
            const uint8_t z = points ? (uint8_t)ahead.z[i] : (uint8_t)kGq4Sym;
            if constexpr (TRANS) {
                *reinterpret_cast<half_t *>(t + (g * 64 + row) * 2) = row < there ? ahead.s[i] : (half_t)0.f;
                t[8 * 64 * 2 + g * 64 + row] = z;
            } else {
                *reinterpret_cast<half_t *>(t + row * 24 + g * 2) = ahead.s[i];
                t[row * 24 + 16 + g] = z;
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
    // (a group with a step less than others multiplies by zeros in the last turn: with a branch around its loads the compiler would wait for all of them each time)
    auto put_x = [&](const Piece64 &v, int i, uint8_t *to, bool there) {
        *reinterpret_cast<uint4_t *>(to + xl_at[i]) = there ? __builtin_bit_cast(uint4_t, v.x[i]) : uint4_t{0, 0, 0, 0};
    };
    // A quarter of a weight task: forward, dword h / 2 (at even h); transposed, inputs 2 h and 2 h + 1 of the four rows.  Inputs from `at` on, window w.
    auto put_w = [&](const Piece64 &v, int i, int h, uint8_t *to, int at, int w) {
        const uint32_t b = (uint32_t)(gw + i * (WR * WT));
        const uint8_t *const t = tables + (w & 1) * TABLE;
        if constexpr (!TRANS) {
            if (h & 1) return;
            const int j = h / 2;
            const uint32_t q = (uint32_t)lane >> 4, row = b * 16 + (lane & 15), g = (uint32_t)(at + 32 * j) >> SHIFT & 7u;
            const half_t sc = *reinterpret_cast<const half_t *>(t + row * 24 + g * 2);
            const uint32_t z = t[row * 24 + 16 + g];
            const Gq4Pair<T> value(sc, z, sc, z);
            uint4_t out;
            static_for<4>([&](auto e) { out[decltype(e)::value] = value.template value<decltype(e)::value>(v.w[i][j], masks); });
            *reinterpret_cast<uint4_t *>(to + row * 128 + ((4u * j + q) ^ gq4_turn(row)) * 16) = out;
        } else {
            const uint32_t j = lane & 3, p = lane >> 2 & 3, q = lane >> 4, piece = (b & 3) * 2 + (p >> 1), g = ((b >> 2) * 128 + 32 * j) >> SHIFT;
            typedef half_t half4v __attribute__((ext_vector_type(4)));
            const half4v sc = *reinterpret_cast<const half4v *>(t + (g * 64 + (b & 3) * 16 + 4 * p) * 2);
            const uint32_t z = *reinterpret_cast<const uint32_t *>(t + 8 * 64 * 2 + g * 64 + (b & 3) * 16 + 4 * p);
            const Gq4Pair<T> v01(sc[0], z & 255u, sc[1], z >> 8 & 255u), v23(sc[2], z >> 16 & 255u, sc[3], z >> 24);
            static_for<8>([&](auto ec) {
                constexpr int e = decltype(ec)::value;
                if (e / 2 != h) return;
                const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;          // the nibbles of input e of both rows, as halves
                const uint32_t d01 = __builtin_amdgcn_perm(v.w[i][1], v.w[i][0], sel), d23 = __builtin_amdgcn_perm(v.w[i][3], v.w[i][2], sel);
                const uint32_t col = (b >> 2) * 128 + 32 * j + 8 * q + e;
                const uint2_t out = {v01.template value<e / 2>(d01, masks), v23.template value<e / 2>(d23, masks)};
                *reinterpret_cast<uint2_t *>(to + col * 128 + (piece ^ gq4_turn(col)) * 16 + (p & 1) * 8) = out;
            });
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
    // The window of step s, whose inputs are from `at` on: of the eight groups there, or of the step's rows.
    auto window_of = [&](int s, int at) { return TRANS ? s : at >> (SHIFT + 3); };
    auto load_window_of = [&](int w) {
        int term = 0, at = 0;
        if constexpr (TRANS) place(w, term, at);
        load_window(w, term, at);
    };
    if (steps > 0) {
        int term, at, put_at;
        load_window_of(0);
        place(0, term, at);
        use_term(term);
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) fetch_x(pieces[0], i, term, at);
#pragma unroll
        for (int i = 0; i < WTASKS; ++i) fetch_w(pieces[0], i, at);
        put_window(0, 64);
        load_window_of(1);
        put_window(1, 64);
        load_window_of(2);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) put_x(pieces[0], i, own, KG == 1 || mine > 0);
#pragma unroll
        for (int i = 0; i < WTASKS; ++i)
#pragma unroll
            for (int h = 0; h < 4; ++h) put_w(pieces[0], i, h, own, at, 0);
#pragma unroll
        for (int n = 1; n <= P; ++n) {
            place(n, term, at);
            use_term(term);
#pragma unroll
            for (int i = 0; i < XTASKS; ++i) fetch_x(pieces[n % P], i, term, at);
#pragma unroll
            for (int i = 0; i < WTASKS; ++i) fetch_w(pieces[n % P], i, at);
        }
        int window = 0;
        gq4_lds_barrier();
        vec8 af[2][AF], bf[2][BF];
        read(own, 0, af[0], bf[0]);
        for (int s = 0; s < turns;) {
#pragma unroll
            for (int n = 1; n <= P; ++n) {
                uint8_t *const from = own + (s & 1) * STAGE, *const to = own + (~s & 1) * STAGE;
                Piece64 &next = pieces[n % P];
                place(s + 1, term, put_at);
                if (window_of(s + 1, put_at) != window) {
                    window = window_of(s + 1, put_at);
                    put_window(window + 1, 64);
                    load_window_of(window + 2);
                }
                place(s + 1 + P, term, at);
                use_term(term);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                    // The barrier stands before the last quarter's products: past it the next piece is in LDS, and its first operands are read beside them.
                    if (kk == 3) gq4_lds_barrier();
                    read(kk < 3 ? from : to, (kk + 1) & 3, af[(kk + 1) & 1], bf[(kk + 1) & 1]);
#pragma unroll
                    for (int i = 0; i < XTASKS; ++i)
                        if (i * 3 / XTASKS == kk) {
                            put_x(next, i, to, KG == 1 || s + 1 < mine);
                            fetch_x(next, i, term, at);
                        }
#pragma unroll
                    for (int i = 0; i < WTASKS; ++i) {
#pragma unroll
                        for (int h = 0; h < 4; ++h)
                            if ((i * 4 + h) * 3 / (WTASKS * 4) == kk) put_w(next, i, h, to, put_at, window);
                        if (kk == 3) fetch_w(next, i, at);
                    }
                    multiply(af[kk & 1], bf[kk & 1]);
                    if constexpr (AF * BF >= 8) {
#pragma unroll
                        for (int i = 0; i < AF * BF; ++i) {
                            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);       // a product
                            __builtin_amdgcn_sched_group_barrier(0x080, 2, 0);       // LDS
                            __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);       // vector instructions
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                if (++s >= turns) break;
            }
        }
    }
    if (len % 64) {
        const int at = whole * 64, w = window_of(0, at);
        for (int term = 0; term < terms; ++term) {
            if (TRANS && term != loaded) {
                weights(term);
                loaded = term;
            }
            load_window(w, term, at);
            __syncthreads();                                                     // (nobody reads from LDS any more)
            put_window(w, len - at);
            __syncthreads();
            if (group == 0) {
                const E *x = static_cast<const E *>(term ? a.x[1] : a.x[0]);
                const int64_t ld = term ? a.x_ld[1] : a.x_ld[0];
                Piece64 &v = pieces[0];
#pragma unroll
                for (int i = 0; i < XTASKS; ++i) {
                    const E *row = x + ((int64_t)t0 + x_at[i]) * ld;
                    const int c = at + (tid & 7) * 8;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v.x[i][e] = c + e < len ? row[c + e] : (E)0.f;
                    put_x(v, i, own, true);
                }
#pragma unroll
                for (int i = 0; i < WTASKS; ++i) {
                    int from = at;
                    if constexpr (TRANS) {                                       // (blocks of rows past the last are not there)
                        const int rl = (gw + i * (WR * WT)) & 3;
                        from = (min((at >> 4) + rl, a.rb - 1) - rl) * 16;
                    }
                    fetch_w(v, i, from);
#pragma unroll
                    for (int h = 0; h < 4; ++h) put_w(v, i, h, own, at, w);
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

template <class T, int MODE, int SHIFT, int KG, int P, int WR, int WT, int AF, int BF>
static int launch_gq4_tile(Gq4TileArgs a, hipStream_t st)
{
    constexpr int THREADS = KG * WR * WT * kWave, BO = 32 * AF * WR, BT = 32 * BF * WT;
    constexpr size_t LDS = Gq4TileLds<MODE, KG, BO, BT>::bytes;
    static_assert(LDS <= 160 * 1024 && (size_t)BO * BT * (KG > 1 ? 4 : 2) <= LDS, "LDS");
    const int outs = MODE == kGq4Transposed ? a.k : a.n, wide = MODE == kGq4Gated ? BO / 2 : BO;
    a.tiles_o = (int)(((int64_t)outs + wide - 1) / wide);
    a.tiles_t = (int)(((int64_t)a.m + BT - 1) / BT);
    const int64_t tiles = (int64_t)a.tiles_o * a.tiles_t;
    if (tiles * THREADS > UINT32_MAX) return SLIM_ERR_SHAPE;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_tile_kernel<T, MODE, SHIFT, KG, P, WR, WT, AF, BF>), dim3((unsigned)tiles), dim3(THREADS), LDS, st, a);
    return SLIM_OK;
}

template <class T, int MODE, int SHIFT>
static int launch_gq4_shape(const Gq4TileArgs &a, hipStream_t st)
{
    int shape = a.m > 256 ? 0 : 2;
    if (const char *e = getenv("GQ4_T")) shape = atoi(e);
    switch (shape) {
    case 0: return launch_gq4_tile<T, MODE, SHIFT, 1, 1, 4, 2, 2, 4>(a, st);     // 256 x 256
    case 1: return launch_gq4_tile<T, MODE, SHIFT, 1, 2, 4, 2, 2, 2>(a, st);     // 256 x 128
    case 2: return launch_gq4_tile<T, MODE, SHIFT, 2, 2, 2, 2, 2, 2>(a, st);     // 128 x 128, two groups
    case 3: return launch_gq4_tile<T, MODE, SHIFT, 2, 4, 2, 2, 2, 1>(a, st);     // 128 x 64, two groups
    case 4: return launch_gq4_tile<T, MODE, SHIFT, 3, 3, 2, 1, 2, 1>(a, st);     // 128 x 32, three groups
    default: break;
    }
    if constexpr (MODE != kGq4Transposed) return launch_gq4_tile<T, MODE, SHIFT, 4, 3, 1, 2, 2, 1>(a, st);    // 64 x 64, four groups
    return launch_gq4_tile<T, MODE, SHIFT, 3, 3, 2, 1, 2, 1>(a, st);
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

int gq4_launch_rows(const slim_group_q4_layer *layer, const slim_group_q4_layer *up, int shift, const void *X, int64_t x_ld, int32_t m, void *const (&y)[3],
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
    return gq4_launch_rows(layer, nullptr, shift, X, x_ld, m, a.y, a.y_ld, dtype, static_cast<hipStream_t>(stream));
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
    return gq4_launch_rows(gate, up, shift, X, x_ld, m, a.y, a.y_ld, dtype, static_cast<hipStream_t>(stream));
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
