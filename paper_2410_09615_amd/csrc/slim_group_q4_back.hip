// Gradients through frozen 4-bit weights that have a scale for each group of inputs:  dX = sum of dY_i W_i over one layer or the two of a gated block.
// What is summed over are a layer's rows, so a lane's codes, which are inputs of one row, have to change places: a thread takes the same eight inputs of four rows, and a byte permutation
// of two rows' dwords leaves pairs (row, row + 1) of one input side by side.  Codes become numbers of the gradients' type, (c - z) s rounded once to it, on their way into LDS.  Products
// are summed in binary32 by the 32 x 32 x 16 matrix instructions, the weights as their A operand, and each result is rounded once.  In fp16 groups whose scale makes weights beyond 65504 are left
// to a turn of their own (gq4_large).
#include <hip/hip_runtime.h>

#include "slim_group_q4.h"
#include "slim_mma.h"

namespace slim {

struct Gq4BackArgs {
    Gq4Weights w[2];
    const void *x[2];        // dY of each layer
    int64_t x_ld[2];
    void *y;
    int64_t y_ld;
    int n, k, m, cb, rb, kg; // a layer: rows, inputs; blocks of inputs, blocks of rows, groups of a row
    int terms;               // layers
    int tiles_o, tiles_t;
    Gq4Split split;
};

// Per group of wavefronts: two buffers of a piece's weights and gradients, two windows of scales and zero points.
template <int KG, int BO, int BT>
struct Gq4BackLds {
    static constexpr int stage = (BO + BT) * 128, table = 8 * 64 * 3, bytes = KG * 2 * (stage + table);
};

// A workgroup has a tile of BT tokens x BO inputs and goes over the layers' rows 64 at a time.  KG groups of WR x WT wavefronts take turns at those pieces, each with two buffers of its own
// in LDS.  While a piece is multiplied from one, the next one goes from registers into the other, and the one P further is asked for from memory into the registers that this frees: beside
// each quarter of a piece's products (16 rows) stands a part of that work.  Rows that do not fill a piece are left for last and taken without that overlap.
// Many tokens (256 x 256): 4096 through 8192 x 8192 in fp16 500 to 522 us from card to card, 1.05 to 1.10 PFLOP/s; through 2 x 11008 x 4096 in bf16 732 to 763 us with the activation's gradient (73 to 78), matrix pipes 58 % busy at 1.74 GHz.  LDS
// carries 256 KiB for a piece's 256 products, about as long as they take, and the two overlap in part: without products 336 us of the 500, without stores to LDS 290.  (Half of the wavefronts at
// products while the others store, in turn: 599 us.)  Smaller tiles are bound by the chain between two barriers, read, convert, store: 1.3 us a turn on 128 x 128 whose products take 0.2.
template <class T, int SHIFT, int KG, int P, int WR, int WT, int AF, int BF>
__global__ __launch_bounds__(KG *WR *WT *kWave, 2) void gq4_back_kernel(Gq4BackArgs a)
{
    typedef typename T::type E;
    typedef typename Gq4Vec<T>::v8 vec8;
    constexpr int THREADS = WR * WT * kWave, BO = 32 * AF * WR, BT = 32 * BF * WT;
    typedef Gq4BackLds<KG, BO, BT> Lds;
    constexpr int STAGE = Lds::stage, TABLE = Lds::table, XTASKS = BT * 8 / THREADS, WTASKS = BO * 2 / THREADS;
    static_assert(XTASKS * THREADS == BT * 8 && WTASKS * THREADS == BO * 2 && BO % 128 == 0 && AF % 2 == 0, "tile");
    extern __shared__ __align__(16) uint8_t lds[];
    const Gq4Masks masks;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x & (kWave - 1);
    const int group = KG > 1 ? wave / (WR * WT) : 0, gw = KG > 1 ? wave % (WR * WT) : wave, tid = gw * kWave + lane;
    const int wr = gw % WR, wt = gw / WR;
    const int gx = a.tiles_o * a.tiles_t;
    const int qx = gx % kDies == 0 ? ((int)blockIdx.x % kDies) * (gx / kDies) + (int)blockIdx.x / kDies : (int)blockIdx.x;
    const int tile = blocked_tile(qx, a.tiles_o, a.tiles_t);
    const int o0 = tile % a.tiles_o * BO, t0 = tile / a.tiles_o * BT;
    // this workgroup's share of the steps
    const int whole = a.n / 64, share = (whole * a.terms + a.split.splits - 1) / a.split.splits, begin = (int)blockIdx.y * share, steps = min(share, whole * a.terms - begin);
    uint8_t *const own = lds + group * (2 * STAGE + 2 * TABLE), *const tables = own + 2 * STAGE;

    // ---- where this thread's share of a piece lies: uniform bases, and 32 bits from there on.  Lane (q, p, j) of block b has rows 4 p .. 4 p + 3, inputs 32 j + 8 q .. + 7. ----
    const uint32_t lj = (uint32_t)lane & 3u, lp = (uint32_t)lane >> 2 & 3u, lq = (uint32_t)lane >> 4;
    uint32_t x_at[XTASKS], xl_at[XTASKS], wl_at[WTASKS];
    const uint8_t *codes[WTASKS];
#pragma unroll
    for (int i = 0; i < XTASKS; ++i) {
        const uint32_t row = (uint32_t)(tid + i * THREADS) >> 3;
        x_at[i] = (uint32_t)min((int)row, a.m - 1 - t0);                         // (times the row's length, which a layer has its own of)
        xl_at[i] = BO * 128u + row * 128u + (((uint32_t)tid & 7u) ^ gq4_turn(row)) * 16u;
    }
    const uint32_t w_at = (lq * 16u + 4u * lp) * 16u + lj * 4u;
#pragma unroll
    for (int i = 0; i < WTASKS; ++i) {
        // Input e of the lane's eight: 128 e bytes on, its 16-byte pieces in another order: e ^ q ^ 4 (j % 2), so that a store of 64 lanes, whose inputs are all 128 bytes or more apart,
        // finds all banks (with gq4_turn's e ^ q half of them: 37 % of LDS's cycles were waits on 256 x 256, now 17 %).
        const uint32_t b = (uint32_t)(gw + i * (WR * WT)), col = (b >> 2) * 128u + 32u * lj + 8u * lq;
        wl_at[i] = col * 128u + (((b & 3u) * 2u + (lp >> 1)) ^ lq ^ (lj & 1u) * 4u) * 16u + (lp & 1u) * 8u;
    }
    auto weights = [&](int term) {
#pragma unroll
        for (int i = 0; i < WTASKS; ++i) {
            const int b = gw + i * (WR * WT), cb = min(o0 / 128 + (b >> 2), a.cb - 1);
            codes[i] = (term ? a.w[1].codes : a.w[0].codes) + ((int64_t)(b & 3) * a.cb + cb) * kGq4Block;
        }
    };

    struct Share {                                                               // a thread's share of a piece, in registers
        vec8 x[XTASKS];
        uint32_t w[WTASKS][4];
    };
    Share pieces[P];
    // of the term's rows from `at` on
    auto fetch_x = [&](Share &v, int i, int term, int at) {
        const uint8_t *base = static_cast<const uint8_t *>(term ? a.x[1] : a.x[0]);
        const int64_t ld = term ? a.x_ld[1] : a.x_ld[0];
        base += ((int64_t)t0 * ld + at) * 2;
        v.x[i] = Piece<T, 8>::load(reinterpret_cast<const E *>(base + (x_at[i] * (uint32_t)ld + (uint32_t)(tid & 7) * 8u) * 2u));
    };
    auto fetch_w = [&](Share &v, int i, int at) {
        const uint8_t *c = codes[i] + (int64_t)(at >> 4) * a.cb * kGq4Block;
#pragma unroll
        for (int e = 0; e < 4; ++e) v.w[i][e] = *reinterpret_cast<const uint32_t *>(c + 16 * e + w_at);
    };
    // ---- scales and zero points: a window is those of a piece's 64 rows for the tile's inputs, [group][64 rows] in LDS; two, filled one ahead ----
    constexpr int SPAN = BO >> SHIFT, ITEMS = (64 * SPAN + THREADS - 1) / THREADS;
    static_assert(SPAN <= 8, "window");
    struct Window {
        half_t s[ITEMS];
        uint32_t z[ITEMS];
        int term;
    };
    Window ahead;
    auto load_window = [&](int term, int at) {
        ahead.term = term;
        int own_tid = tid;                                                       // (made anew here each time: kept over the loop, what follows from it takes too many registers)
        asm volatile("" : "+v"(own_tid));
        const Gq4Weights &l = term ? a.w[1] : a.w[0];
        const uint8_t *scales = reinterpret_cast<const uint8_t *>(l.scales + (int64_t)at * a.kg);
        const uint8_t *zeros = l.zeros ? l.zeros + (int64_t)at * a.kg : scales;         // (symmetric: what is read of the scales instead is not used)
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int item = own_tid + i * THREADS, row = item / SPAN, g = item % SPAN;
            const uint32_t place = (uint32_t)min(row, a.n - 1 - at) * (uint32_t)a.kg + (uint32_t)min((o0 >> SHIFT) + g, a.kg - 1);
            ahead.s[i] = *reinterpret_cast<const half_t *>(scales + place * 2u);
            ahead.z[i] = *(zeros + place);
        }
    };
    // the first `there` rows are there: the others are no terms of the sum
    bool large = false;                                                          // (fp16) whether there was a scale whose group is left out: gq4_large
    auto put_window = [&](int w, int there, bool rest) {
        uint8_t *const t = tables + (w & 1) * TABLE;
        int own_tid = tid;
        asm volatile("" : "+v"(own_tid));
        const bool points = (ahead.term ? a.w[1].zeros : a.w[0].zeros) != nullptr;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int item = own_tid + i * THREADS, row = item / SPAN, g = item % SPAN;
            if (item >= 64 * SPAN) continue;
            uint32_t h = row < there ? __builtin_bit_cast(uint16_t, ahead.s[i]) : 0;
            if constexpr (__is_same(T, F16)) {
                large |= gq4_large(h);
                h = gq4_scale_of(h, rest);
            }
            *reinterpret_cast<uint16_t *>(t + (g * 64 + row) * 2) = (uint16_t)h;
            t[8 * 64 * 2 + g * 64 + row] = points ? (uint8_t)ahead.z[i] : (uint8_t)kGq4Sym;
        }
    };
    // the scales and zero points of a weight task's four rows
    typedef half_t half4v __attribute__((ext_vector_type(4)));
    struct Scales {
        half4v s[WTASKS];
        uint32_t z[WTASKS];
    };
    auto read_scales = [&](Scales &v, int w) {
        const uint8_t *const t = tables + (w & 1) * TABLE;
#pragma unroll
        for (int i = 0; i < WTASKS; ++i) {
            const uint32_t b = (uint32_t)(gw + i * (WR * WT)), at = (((b >> 2) * 128u + 32u * lj) >> SHIFT) * 64u + (b & 3u) * 16u + 4u * lp;
            v.s[i] = *reinterpret_cast<const half4v *>(t + at * 2);
            v.z[i] = *reinterpret_cast<const uint32_t *>(t + 8 * 64 * 2 + at);
        }
    };
    // ---- into LDS ----
    // (a group with a step less than others multiplies by zeros in the last turn: with a branch around its loads the compiler would wait for all of them each time)
    auto put_x = [&](const Share &v, int i, uint8_t *to, bool there) {
        *reinterpret_cast<uint4_t *>(to + xl_at[i]) = there ? __builtin_bit_cast(uint4_t, v.x[i]) : uint4_t{0, 0, 0, 0};
    };
    // inputs 2 h and 2 h + 1 of a weight task
    auto put_w = [&](const Share &v, const Scales &sc, int i, auto hc, uint8_t *to) {
        constexpr int h = decltype(hc)::value;
        const Gq4Pair<T> v01(sc.s[i][0], sc.z[i] & 255u, sc.s[i][1], sc.z[i] >> 8 & 255u), v23(sc.s[i][2], sc.z[i] >> 16 & 255u, sc.s[i][3], sc.z[i] >> 24);
        static_for<2>([&](auto ec) {
            constexpr int e = 2 * h + decltype(ec)::value;
            const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;              // the nibbles of input e of both rows, as halves
            const uint32_t d01 = __builtin_amdgcn_perm(v.w[i][1], v.w[i][0], sel), d23 = __builtin_amdgcn_perm(v.w[i][3], v.w[i][2], sel);
            const uint2_t out = {v01.template value<h>(d01, masks), v23.template value<h>(d23, masks)};
            *reinterpret_cast<uint2_t *>(to + (wl_at[i] ^ (uint32_t)(e * 16)) + e * 128) = out;
        });
    };

    // (fp16) a weight task's first or second part, of scales that fp16 weights cannot have
    auto put_w_rest = [&](const Share &v, const Scales &sc, int i, int part, uint8_t *to) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t b[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int c = (int)(v.w[i][r] >> (4 * (e >> 1) + 16 * (e & 1)) & 15u), z = (int)(sc.z[i] >> (8 * r) & 255u);
                b[r] = gq4_part_of((float)(c - z) * (float)sc.s[i][r], part);
            }
            *reinterpret_cast<uint2_t *>(to + (wl_at[i] ^ (uint32_t)(e * 16)) + e * 128) = uint2_t{b[0] | b[1] << 16, b[2] | b[3] << 16};
        }
    };

    float16_t acc[AF][BF];
#pragma unroll
    for (int i = 0; i < AF; ++i)
#pragma unroll
        for (int t = 0; t < BF; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][t][e] = 0.f;

    const uint32_t fr = (uint32_t)lane & 31u, turned = ((uint32_t)lane >> 5 ^ gq4_turn(fr)) * 16u;
    const uint32_t wl_from = (uint32_t)(wr * AF * 32) * 128u + fr * 128u, xl_from = (uint32_t)(BO + wt * BF * 32) * 128u + fr * 128u;
    auto read = [&](const uint8_t *from, int kk, vec8 (&af)[AF], vec8 (&bf)[BF]) {
#pragma unroll
        for (int i = 0; i < AF; ++i) af[i] = *reinterpret_cast<const vec8 *>(from + wl_from + (turned ^ (uint32_t)(kk * 32 ^ (i & 1) * 64)) + i * 4096);
#pragma unroll
        for (int t = 0; t < BF; ++t) bf[t] = *reinterpret_cast<const vec8 *>(from + xl_from + (turned ^ (uint32_t)kk * 32u) + t * 4096);
    };
    auto multiply = [&](const vec8 (&af)[AF], const vec8 (&bf)[BF]) {
#pragma unroll
        for (int t = 0; t < BF; ++t)
#pragma unroll
            for (int i = 0; i < AF; ++i) acc[i][t] = gq4_mma32(af[i], bf[t], acc[i][t]);
    };

    // Step s of the group is piece group + s KG of the share.  (Past the last the last is fetched again, and not used.)
    const int turns = (steps + KG - 1) / KG, mine = (steps - group + KG - 1) / KG;
    auto place = [&](int s, int &term, int &at) {
        const int step = begin + min(group + s * KG, steps - 1);
        term = step >= whole ? 1 : 0;
        at = (step - term * whole) * 64;
    };
    int loaded = 0;                                                              // the layer whose codes' places are held
    weights(0);
    auto use_term = [&](int term) {
        if (term != loaded) {
            weights(term);
            loaded = term;
        }
    };
    auto load_window_of = [&](int s) {
        int term, at;
        place(s, term, at);
        load_window(term, at);
    };
    auto fetch = [&](Share &v, int s) {
        int term, at;
        place(s, term, at);
        use_term(term);
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) fetch_x(v, i, term, at);
#pragma unroll
        for (int i = 0; i < WTASKS; ++i) fetch_w(v, i, at);
    };
    if (steps > 0) {
        Scales sc;
        load_window_of(0);
        fetch(pieces[0], 0);
        put_window(0, 64, false);
        load_window_of(1);
        put_window(1, 64, false);
        load_window_of(2);
        __syncthreads();
        read_scales(sc, 0);
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) put_x(pieces[0], i, own, KG == 1 || mine > 0);
#pragma unroll
        for (int i = 0; i < WTASKS; ++i) static_for<4>([&](auto h) { put_w(pieces[0], sc, i, h, own); });
#pragma unroll
        for (int n = 1; n <= P; ++n) fetch(pieces[n % P], n);
        read_scales(sc, 1);
        gq4_lds_barrier();
        vec8 af[2][AF], bf[2][BF];
        read(own, 0, af[0], bf[0]);
        for (int s = 0; s < turns;) {
#pragma unroll
            for (int n = 1; n <= P; ++n) {
                uint8_t *const from = own + (s & 1) * STAGE, *const to = own + (~s & 1) * STAGE;
                Share &next = pieces[n % P];
                int term, at;
                place(s + 1 + P, term, at);
                use_term(term);
                static_for<4>([&](auto kkc) {
                    constexpr int kk = decltype(kkc)::value;
                    // The barrier stands before the last quarter's products: past it the next piece is in LDS, and its first operands are read beside them.
                    if constexpr (kk == 3) gq4_lds_barrier();
                    read(kk < 3 ? from : to, (kk + 1) & 3, af[(kk + 1) & 1], bf[(kk + 1) & 1]);
                    // (the window of step s + 1, in registers by now, is left by all; that of s + 2 is there, and the one after it takes its place past the barrier)
                    if constexpr (kk == 0) {
                        put_window(s, 64, false);
                        load_window_of(s + 3);
                    }
                    if constexpr (kk == 3) read_scales(sc, s);
#pragma unroll
                    for (int i = 0; i < XTASKS; ++i)
                        if (i * 3 / XTASKS == kk) {
                            put_x(next, i, to, KG == 1 || s + 1 < mine);
                            fetch_x(next, i, term, at);
                        }
                    static_for<4 * WTASKS>([&](auto ihc) {
                        constexpr int ih = decltype(ihc)::value;
                        if constexpr (ih * 3 / (WTASKS * 4) == kk) put_w(next, sc, ih / 4, std::integral_constant<int, ih % 4>{}, to);
                    });
                    if constexpr (kk == 3) {
#pragma unroll
                        for (int i = 0; i < WTASKS; ++i) fetch_w(next, i, at);
                    }
                    multiply(af[kk & 1], bf[kk & 1]);
#pragma unroll
                    for (int i = 0; i < AF * BF; ++i) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                          // a product,
                        __builtin_amdgcn_sched_group_barrier(0x002, AF * BF >= 8 ? 5 : 10, 0);      // and vector instructions that it takes the time of
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
                if (++s >= turns) break;
            }
        }
    }
    // ---- pieces without overlap, by the first group of wavefronts ----
    const int tails = a.n % 64 && (int)blockIdx.y == a.split.splits - 1 ? a.terms : 0;
    // a piece's inputs element by element, and its codes
    auto stage_x = [&](Share &v, int term, int at, auto &&of) {
        const E *x = static_cast<const E *>(term ? a.x[1] : a.x[0]);
        const int64_t ld = term ? a.x_ld[1] : a.x_ld[0];
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) {
            const E *row = x + ((int64_t)t0 + x_at[i]) * ld;
            const int c = at + (tid & 7) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) v.x[i][e] = c + e < a.n ? of(row[c + e]) : (E)0.f;
            put_x(v, i, own, true);
        }
    };
    auto stage_w = [&](Share &v, int i, int at) {
        const int rl = (gw + i * (WR * WT)) & 3;
        fetch_w(v, i, (min((at >> 4) + rl, a.rb - 1) - rl) * 16);                // (blocks of rows past the last are not there)
    };
    // rows that do not fill a piece, of each layer
    for (int term = 0; term < tails; ++term) {
        const int at = whole * 64;
        use_term(term);
        load_window(term, at);
        __syncthreads();                                                         // (nobody reads from LDS any more)
        put_window(0, a.n - at, false);
        __syncthreads();
        if (group == 0) {
            Share &v = pieces[0];
            Scales sc;
            read_scales(sc, 0);
            stage_x(v, term, at, [](E e) { return e; });
#pragma unroll
            for (int i = 0; i < WTASKS; ++i) {
                stage_w(v, i, at);
                static_for<4>([&](auto h) { put_w(v, sc, i, h, own); });
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
    if constexpr (__is_same(T, F16)) {
        // groups that were left out: pieces of the share, and what does not fill one
        if (gq4_any_wave(large, lds + Lds::bytes, wave, KG * WR * WT)) {
            const int full = max(steps, 0);
            for (int p = 0; p < full + tails; ++p) {
                const int term = p < full ? (begin + p >= whole ? 1 : 0) : p - full, at = p < full ? (begin + p - term * whole) * 64 : whole * 64;
                use_term(term);
                load_window(term, at);
                __syncthreads();
                put_window(0, min(64, a.n - at), true);
                for (int part = 0; part < 2; ++part) {
                    __syncthreads();
                    if (group == 0) {
                        Share &v = pieces[0];
                        Scales sc;
                        read_scales(sc, 0);
                        // (an infinite input has had its part: times the scales that are 0 now it would be a NaN)
                        if (part == 0) stage_x(v, term, at, [](E e) { return __builtin_isfinite((float)e) ? e : (E)0.f; });
#pragma unroll
                        for (int i = 0; i < WTASKS; ++i) {
                            stage_w(v, i, at);
                            put_w_rest(v, sc, i, part, own);
                        }
                    }
                    __syncthreads();
                    if (group == 0) {
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) {
                            vec8 af[AF], bf[BF];
                            read(own, kk, af, bf);
#pragma unroll
                            for (int t = 0; t < BF; ++t)
#pragma unroll
                                for (int other = 0; other < 2; ++other) {
                                    const Gq4Vec<BF16>::v8 x = gq4_part_of(bf[t], other);
#pragma unroll
                                    for (int i = 0; i < AF; ++i) acc[i][t] = gq4_mma32(__builtin_bit_cast(Gq4Vec<BF16>::v8, af[i]), x, acc[i][t]);
                                }
                        }
                    }
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

    // (uniform: all of a workgroup or none)
    if (a.split.part) {
        if (KG == 1 || group == 0)
#pragma unroll
            for (int i = 0; i < AF; ++i)
#pragma unroll
                for (int t = 0; t < BF; ++t) {
                    const int tok = t0 + (wt * BF + t) * 32 + (lane & 31), o = o0 + (wr * AF + i) * 32 + 4 * (lane >> 5);
                    float *const row = a.split.part + ((int64_t)blockIdx.y * a.m + tok) * a.split.ld + o;
                    if (tok < a.m)
#pragma unroll
                        for (int g = 0; g < 4; ++g)
                            if (o + 8 * g < a.split.ld)
                                *reinterpret_cast<float4_t *>(row + 8 * g) = float4_t{acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
                }
        return;
    }

    // Results leave through LDS, so that a store writes whole pieces of a token's row.
    constexpr int PER_ROW = BO / 8, TURN = (PER_ROW < 16 ? PER_ROW : 16) - 1;
    typedef E vec4 __attribute__((ext_vector_type(4)));
    __syncthreads();
    if (KG == 1 || group == 0)
#pragma unroll
        for (int i = 0; i < AF; ++i)
#pragma unroll
            for (int t = 0; t < BF; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    vec4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = (E)acc[i][t][4 * g + e];
                    const int tok = (wt * BF + t) * 32 + (lane & 31), c = (wr * AF + i) * 4 + g;
                    *reinterpret_cast<vec4 *>(lds + (tok * PER_ROW + (c ^ (tok & TURN))) * 16 + (lane >> 5) * 8) = v;
                }
    __syncthreads();
    const int toks = min(BT, a.m - t0);
    for (int i = (int)threadIdx.x; i < toks * PER_ROW; i += KG * THREADS) {
        const int tok = i / PER_ROW, c = i % PER_ROW, o = o0 + c * 8;
        if (o < a.k) {
            const vec8 v = *reinterpret_cast<const vec8 *>(lds + (tok * PER_ROW + (c ^ (tok & TURN))) * 16);
            E *row = static_cast<E *>(a.y) + (int64_t)(t0 + tok) * a.y_ld;
            if (o + 8 <= a.k)
                Piece<T, 8>::store(row + o, v);
            else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (o + e < a.k) row[o + e] = v[e];
            }
        }
    }
}

// Inputs and tokens of a tile, workgroups per compute unit, us per step of 64 rows.
constexpr Gq4Shape kBackShapes[] = {{256, 256, 1, 1.44f, 2.0f}, {256, 128, 1, 1.12f, 1.4f}, {128, 128, 1, 0.65f, 0.78f}, {128, 64, 1, 0.55f, 0.62f}};

static Gq4Plan gq4_plan_back(int n, int k, int m, int terms)
{
    return gq4_plan(kBackShapes, k, m, n / 64 * terms, false);
}
void gq4_back_plan(int n, int k, int m, int terms, int32_t *out)
{
    const Gq4Plan p = gq4_plan_back(n, k, m, terms);
    out[1] = kBackShapes[p.shape].outs;
    out[2] = kBackShapes[p.shape].toks;
    out[3] = p.splits;
}
int64_t gq4_back_workspace(int n, int k, int m, int terms) { return gq4_part_bytes(gq4_plan_back(n, k, m, terms).splits, m, k, false); }

template <class T, int SHIFT, int SHAPE, int KG, int P, int WR, int WT, int AF, int BF>
static int launch_gq4_back_of(Gq4BackArgs a, hipStream_t st)
{
    constexpr int THREADS = KG * WR * WT * kWave, BO = 32 * AF * WR, BT = 32 * BF * WT;
    constexpr size_t RING = Gq4BackLds<KG, BO, BT>::bytes + kGq4Flags, SUMS = (size_t)BO * BT * (KG > 1 ? 4 : 2), LDS = RING > SUMS ? RING : SUMS;
    static_assert(LDS * kBackShapes[SHAPE].per_cu <= 160 * 1024 && kBackShapes[SHAPE].outs == BO && kBackShapes[SHAPE].toks == BT, "the table's tile");
    a.tiles_o = (int)(((int64_t)a.k + BO - 1) / BO);
    a.tiles_t = (int)(((int64_t)a.m + BT - 1) / BT);
    const int64_t tiles = (int64_t)a.tiles_o * a.tiles_t;
    if (tiles * THREADS > UINT32_MAX) return SLIM_ERR_SHAPE;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_back_kernel<T, SHIFT, KG, P, WR, WT, AF, BF>), dim3((unsigned)tiles, (unsigned)a.split.splits), dim3(THREADS), LDS, st, a);
    return SLIM_OK;
}

template <class T, int SHIFT>
static int launch_gq4_back_shape(const Gq4BackArgs &a, int shape, hipStream_t st)
{
    switch (shape) {
    case 0: return launch_gq4_back_of<T, SHIFT, 0, 1, 1, 4, 2, 2, 4>(a, st);
    case 1: return launch_gq4_back_of<T, SHIFT, 1, 1, 2, 4, 2, 2, 2>(a, st);
    case 2: return launch_gq4_back_of<T, SHIFT, 2, 2, 2, 2, 2, 2, 2>(a, st);
    default: return launch_gq4_back_of<T, SHIFT, 3, 2, 3, 2, 2, 2, 1>(a, st);
    }
}

// dX of one layer (second null) or two, of one shape; any number of tokens (arguments are checked where this is called).
int gq4_launch_back(const slim_group_q4_layer *one, const slim_group_q4_layer *second, int shift, const void *dY, int64_t ld, const void *dY2, int64_t ld2, int32_t m, void *dX,
                    int64_t dx_ld, int32_t dtype, void *workspace, hipStream_t st)
{
    const int terms = second ? 2 : 1;
    const Gq4Plan plan = gq4_plan_back(one->n, one->k, m, terms);
    Gq4BackArgs a{};
    a.split = Gq4Split{plan.splits > 1 ? static_cast<float *>(workspace) : nullptr, plan.splits, gq4_part_ld(one->k)};
    a.w[0] = gq4_weights(one);
    if (second) a.w[1] = gq4_weights(second);
    a.x[0] = dY;
    a.x_ld[0] = ld;
    a.x[1] = dY2;
    a.x_ld[1] = ld2;
    a.y = dX;
    a.y_ld = dx_ld;
    a.n = one->n;
    a.k = one->k;
    a.m = m;
    a.cb = gq4_col_blocks(one->k);
    a.rb = gq4_row_blocks(one->n);
    a.kg = gq4_groups(one->k, shift);
    a.terms = terms;
    auto of = [&](auto type) {
        typedef decltype(type) T;
        return shift == 5 ? launch_gq4_back_shape<T, 5>(a, plan.shape, st) : shift == 6 ? launch_gq4_back_shape<T, 6>(a, plan.shape, st) : launch_gq4_back_shape<T, 7>(a, plan.shape, st);
    };
    const int rc = dtype == SLIM_F16 ? of(F16{}) : of(BF16{});
    if (rc != SLIM_OK) return rc;
    if (plan.splits > 1) {
        void *const y[3] = {dX, nullptr, nullptr};
        const int64_t y_ld[3] = {dx_ld, 0, 0};
        return gq4_launch_finish(a.split, m, one->k, false, y, y_ld, dtype, st);
    }
    return hip_status(hipGetLastError());
}

}  // namespace slim
