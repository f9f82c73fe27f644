// Products with 4-bit weights that have a scale for each group of inputs, for more tokens than are streamed for (slim_group_q4_stream.hip):
//   plain  Y = X W^T,     gated  H = silu(X Wg^T) * (X Wu^T), and where asked for G = X Wg^T and U = X Wu^T
// A workgroup has a tile of BT tokens x BO rows of weights.  The tokens go through LDS; the weights do not: a wavefront has its own 64 rows, and a lane's 16 bytes of a
// block of the layout are its operand of four 32 x 32 x 16 products once codes are numbers of the inputs' type, (c - z) s rounded once to it: the matrix instructions take 16 bits, and a scale
// has 11 of them.  (Scales on the sums, as for few tokens, would take a second set of accumulators and, in groups of 32, as many additions as the products take cycles.)  With
// weights through LDS too it carries 256 KiB for a product's 256 x 256 x 64 instead of 160, and they take turns (a tile of 256 x 256, since replaced by two of 256 x 128 per compute unit: 4096 tokens on
// 8192 x 8192 504 us with, 491 without).
// Products are summed in binary32, each result is rounded once.  In fp16 groups whose scale makes weights beyond 65504 are left to a turn of their own (gq4_large).
// Bound by power where there are many tokens: 4096 on 2 x 28672 x 8192 gated 3.30 to 3.55 ms from card to card, 1.08 to 1.17 PFLOP/s, matrix pipes 68 to 72 % busy at 1.5 GHz (the library's product of two fp16
// matrices of 8192 x 8192: 1.34 PFLOP/s).  With few tiles by what a wavefront issues and waits for between two barriers: a step of 64 inputs takes 0.85 us on 256 x 128 with one workgroup per
// compute unit, 0.5 on 256 x 64, 0.3 on 128 x 64 (the times at kRowShapes), where its products alone would take 0.43, 0.21 and 0.11; 333 tokens on 10007 x 4100 in groups of 32 53 to 55 us.
// What is put between the products is placed by hand (a product, then vector instructions for its time): on 256 x 128 left to the compiler 4096 tokens on 8192 x 8192 take 556 us, 502 so, 1024 on
// 11008 x 4096 115 and 106 (the smaller tiles are as fast either way).
#include <hip/hip_runtime.h>

#include "slim_group_q4.h"
#include "slim_mma.h"

namespace slim {

// Rows and tokens of a tile, workgroups per compute unit, us per step of 64 inputs (of the slope between 4096 and 11008 inputs, and of 8192 x 8192 at 4096 tokens).
constexpr Gq4Shape kRowShapes[] = {{256, 128, 2, 0.85f, 1.9f}, {256, 64, 1, 0.5f, 0.65f}, {128, 64, 1, 0.3f, 0.38f}};

static Gq4Plan gq4_plan_rows(int n, int k, int m, bool gated)
{
    return gq4_plan(kRowShapes, n, m, 2 * (k / kGq4Cols), gated);
}
void gq4_rows_plan(int n, int k, int m, bool gated, int32_t *out)
{
    const Gq4Plan p = gq4_plan_rows(n, k, m, gated);
    out[1] = kRowShapes[p.shape].outs;
    out[2] = kRowShapes[p.shape].toks;
    out[3] = p.splits;
}
int64_t gq4_rows_workspace(int n, int k, int m, bool gated) { return gq4_part_bytes(gq4_plan_rows(n, k, m, gated).splits, m, n, gated); }

struct Gq4RowsArgs {
    Gq4Weights w[2];
    const void *x;
    int64_t x_ld;
    void *y[3];              // plain: the result; gated: H, G, U (G and U may be null)
    int64_t y_ld[3];
    int n, k, m, cb, rb, kg; // the layer: rows, inputs; blocks of inputs, blocks of rows, groups of a row
    int tiles_o, tiles_t;
    Gq4Split split;
};

// Per group of wavefronts: two buffers of a step's tokens, two windows of scales and zero points (8 groups of each row).
template <int KG, int BO, int BT>
struct Gq4RowsLds {
    static constexpr int stage = BT * 128, table = BO * 24, bytes = KG * 2 * (stage + table);
};

// A step is half a block of 128 inputs: 16 of each 32, so that a lane's 16 bytes of codes are all it needs of a block of rows.  KG groups of WR wavefronts share the steps, a run
// of them each.  Weights of RW steps and tokens of RX are in registers or on their way there; tokens go into one buffer of LDS while the other is multiplied from.
template <class T, bool GATED, int SHIFT, int KG, int WR, int BF, int RX, int RW>
__global__ __launch_bounds__(KG *WR *kWave, 2) void gq4_rows_kernel(Gq4RowsArgs a)
{
    typedef typename T::type E;
    typedef typename Gq4Vec<T>::v8 vec8;
    constexpr int AF = 2, THREADS = WR * kWave, BO = 32 * AF * WR, BT = 32 * BF, UNROLL = RW;
    constexpr int NG = kGq4Cols >> SHIFT, PER = 4 / NG;                       // groups per block, products of a step per group
    typedef Gq4RowsLds<KG, BO, BT> Lds;
    constexpr int STAGE = Lds::stage, TABLE = Lds::table, XTASKS = BT * 8 / THREADS, ITEMS = BO * 2 / THREADS;
    static_assert(XTASKS * THREADS == BT * 8 && ITEMS * THREADS == BO * 2 && RW % RX == 0 && RW % 2 == 0, "tile");
    extern __shared__ __align__(16) uint8_t lds[];
    const Gq4Masks masks;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x & (kWave - 1);
    const int group = KG > 1 ? wave / WR : 0, wr = KG > 1 ? wave % WR : wave, tid = wr * kWave + lane;
    const int gx = a.tiles_o * a.tiles_t;
    const int qx = gx % kDies == 0 ? ((int)blockIdx.x % kDies) * (gx / kDies) + (int)blockIdx.x / kDies : (int)blockIdx.x;
    const int tile = blocked_tile(qx, a.tiles_o, a.tiles_t);
    const int o0 = tile % a.tiles_o * (GATED ? BO / 2 : BO), t0 = tile / a.tiles_o * BT, outs = a.n;
    // this workgroup's share of the steps, and its groups' of that
    const int whole = a.k / kGq4Cols, share = (2 * whole + a.split.splits - 1) / a.split.splits, begin = (int)blockIdx.y * share, end = min(begin + share, 2 * whole);
    const int steps = end - begin, turns = (steps + KG - 1) / KG, first = begin + group * turns, last = max(min(first + turns, end) - 1, 0);
    uint8_t *const own = lds + group * (2 * STAGE + 2 * TABLE), *const tables = own + 2 * STAGE;

    // ---- weights: lane (half, row of 32) of row tile i ----
    const uint8_t *codes[AF];
    uint32_t w_at[AF];
#pragma unroll
    for (int i = 0; i < AF; ++i) {
        const Gq4Weights &l = GATED && i == 1 ? a.w[1] : a.w[0];
        const int rb0 = GATED ? o0 / 16 + wr * 2 : o0 / 16 + (wr * AF + i) * 2, rb = min(rb0, a.rb - 1);
        codes[i] = l.codes + (int64_t)rb * a.cb * kGq4Block;
        w_at[i] = (uint32_t)min(lane >> 4 & 1, a.rb - 1 - rb) * (uint32_t)a.cb * kGq4Block + (uint32_t)((lane >> 5) * 16 + (lane & 15)) * 16u;
    }
    struct Codes {
        uint4_t c[AF];
    };
    auto fetch_w = [&](Codes &v, int step) {
        const int64_t at = (int64_t)(step >> 1) * kGq4Block + (step & 1) * 512;
#pragma unroll
        for (int i = 0; i < AF; ++i) v.c[i] = *reinterpret_cast<const uint4_t *>(codes[i] + at + w_at[i]);
    };
    // ---- tokens: piece p of a row's step is inputs 32 (p / 2) + 16 (step % 2) + 8 (p % 2) of the block ----
    uint32_t x_at[XTASKS], xl_at[XTASKS];
#pragma unroll
    for (int i = 0; i < XTASKS; ++i) {
        const uint32_t row = (uint32_t)(tid + i * THREADS) >> 3, p = (uint32_t)tid & 7u;
        x_at[i] = ((uint32_t)min((int)row, a.m - 1 - t0) * (uint32_t)a.x_ld + (p >> 1) * 32u + (p & 1u) * 8u) * 2u;
        xl_at[i] = row * 128u + (p ^ gq4_turn(row)) * 16u;
    }
    struct Tokens {
        vec8 x[XTASKS];
    };
    const uint8_t *const xbase = static_cast<const uint8_t *>(a.x) + (int64_t)t0 * a.x_ld * 2;
    auto fetch_x = [&](Tokens &v, int i, int step) {
        const uint8_t *base = xbase + ((int64_t)(step >> 1) * kGq4Cols + (step & 1) * 16) * 2;
        v.x[i] = Piece<T, 8>::load(reinterpret_cast<const E *>(base + x_at[i]));
    };
    // (a group with a step less than others multiplies by zeros in the last turns: with a branch around its loads the compiler would wait for all of them each time)
    auto put_x = [&](const Tokens &v, int i, uint8_t *to, bool there) {
        *reinterpret_cast<uint4_t *>(to + xl_at[i]) = there ? __builtin_bit_cast(uint4_t, v.x[i]) : uint4_t{0, 0, 0, 0};
    };
    // ---- scales and zero points: windows of 8 groups of the tile's rows in LDS, two, filled one ahead ----
    // Where each lane fetches the scale of its own row every step, neighbouring lanes ask the memory pipeline for different lines, which takes four times as long as when they share one.
    // A thread fetches four groups of a row.  Near a row's end they are fetched from four before the end and moved down to their places.
    struct Window {
        uint2_t s[ITEMS];
        uint32_t z[ITEMS];
    };
    Window ahead;
    auto load_window = [&](int w) {
        const int wave_row = wr * 32;                                         // (a wavefront's items of one i are of one layer)
        int own_tid = tid;                                                    // (made anew here each time: kept over the loop, what follows from it takes too many registers)
        asm volatile("" : "+v"(own_tid));
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int item = own_tid + i * THREADS, row = item / 2, g = 8 * w + 4 * (item % 2), from = max(min(g, a.kg - 4), 0);
            const Gq4Weights &l = GATED && ((i * (THREADS / 2) + wave_row) & 32) ? a.w[1] : a.w[0];
            const int local = GATED ? (row >> 6) * 32 + (row & 31) : row;
            const uint8_t *scales = reinterpret_cast<const uint8_t *>(l.scales + (int64_t)o0 * a.kg);
            const uint8_t *zeros = l.zeros ? l.zeros + (int64_t)o0 * a.kg : scales;          // (symmetric: what is read of the scales instead is not used)
            const uint32_t place = (uint32_t)min(local, a.n - 1 - o0) * (uint32_t)a.kg + (uint32_t)from;
            if (a.kg >= 4) {
                ahead.s[i] = reinterpret_cast<const Gq4Any<uint2_t> *>(scales + place * 2u)->v;
                ahead.z[i] = reinterpret_cast<const Gq4Any<uint32_t> *>(zeros + place)->v;
            } else {
                ahead.s[i] = uint2_t{0, 0};
                ahead.z[i] = 0;
#pragma unroll
                for (int e = 0; e < 3; ++e) {
                    const uint32_t at = place + (uint32_t)min(e, a.kg - 1);
                    ahead.s[i][e / 2] |= (uint32_t) * reinterpret_cast<const uint16_t *>(scales + at * 2u) << (16 * (e & 1));
                    ahead.z[i] |= (uint32_t)zeros[at] << (8 * e);
                }
            }
        }
    };
    bool large = false;                                                        // (fp16) whether there was a scale whose group is left out: gq4_large
    auto put_window = [&](int w, bool rest) {
        uint8_t *const t = tables + (w & 1) * TABLE;
        int own_tid = tid;
        asm volatile("" : "+v"(own_tid));
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int item = own_tid + i * THREADS, row = item / 2, g = 8 * w + 4 * (item % 2), down = g - max(min(g, a.kg - 4), 0);
            const bool points = (GATED && (row & 32) ? a.w[1].zeros : a.w[0].zeros) != nullptr;
            if constexpr (__is_same(T, F16)) {
                if (rest || gq4_any_large(ahead.s[i])) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t at = 16 * (e & 1), h = ahead.s[i][e / 2] >> at & 0xffffu;
                        large |= gq4_large(h);
                        ahead.s[i][e / 2] = (ahead.s[i][e / 2] & ~(0xffffu << at)) | gq4_scale_of(h, rest) << at;
                    }
                }
            }
            // (groups that are not there, whose places get anything, may be all four)
            const uint64_t s = (uint64_t)ahead.s[i][1] << 32 | ahead.s[i][0];
            *reinterpret_cast<uint64_t *>(t + row * 24 + (item % 2) * 8) = s >> (16 * (down & 3));
            *reinterpret_cast<uint32_t *>(t + row * 24 + 16 + (item % 2) * 4) = points ? ahead.z[i] >> (8 * (down & 3)) : 0x01010101u * kGq4Sym;
        }
    };
    auto window_of = [&](int step) { return step >> (SHIFT - 3); };            // a block has NG groups, a window 8: two steps a block

    float16_t acc[AF][BF];
#pragma unroll
    for (int i = 0; i < AF; ++i)
#pragma unroll
        for (int t = 0; t < BF; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][t][e] = 0.f;

    const uint32_t fr = (uint32_t)lane & 31u, turned = ((uint32_t)lane >> 5 ^ gq4_turn(fr)) * 16u;
    const uint32_t xl_from = fr * 128u, s_from = ((uint32_t)(wr * AF * 32) + fr) * 24u;
    auto read = [&](const uint8_t *from, int kk, vec8 (&bf)[BF]) {
#pragma unroll
        for (int t = 0; t < BF; ++t) bf[t] = *reinterpret_cast<const vec8 *>(from + xl_from + (turned ^ (uint32_t)kk * 32u) + t * 4096);
    };
    // a step's scales and zero points of the lane's rows, as they are in the table
    struct Scales {
        uint32_t s[AF][(NG + 1) / 2], z[AF];
    };
    auto read_scales = [&](Scales &v, int step) {
        const uint8_t *const t = tables + (window_of(step) & 1) * TABLE + s_from;
        const uint32_t g = (uint32_t)(step >> 1) * NG & 7u;
#pragma unroll
        for (int i = 0; i < AF; ++i) {
            const uint8_t *const at = t + i * 32 * 24;
            if constexpr (NG == 1) {
                v.s[i][0] = *reinterpret_cast<const uint16_t *>(at + g * 2);
                v.z[i] = at[16 + g];
            } else if constexpr (NG == 2) {
                v.s[i][0] = *reinterpret_cast<const uint32_t *>(at + g * 2);
                v.z[i] = *reinterpret_cast<const uint16_t *>(at + 16 + g);
            } else {
                const uint2_t d = *reinterpret_cast<const uint2_t *>(at + g * 2);
                v.s[i][0] = d[0];
                v.s[i][1] = d[1];
                v.z[i] = *reinterpret_cast<const uint32_t *>(at + 16 + g);
            }
        }
    };
    // numbers of dword kk of the codes
    auto number = [&](const Codes &v, const Scales &sc, auto kkc, vec8 (&af)[AF]) {
        constexpr int kk = decltype(kkc)::value, g = kk / PER;
#pragma unroll
        for (int i = 0; i < AF; ++i) {
            const half_t s16 = __builtin_bit_cast(half_t, (uint16_t)(sc.s[i][g / 2] >> (16 * (g & 1))));
            const uint32_t z = NG == 1 ? sc.z[i] : sc.z[i] >> (8 * g) & 255u;
            const Gq4Pair<T> value(s16, z, s16, z);
            uint4_t out;
            static_for<4>([&](auto e) { out[decltype(e)::value] = value.template value<decltype(e)::value>(v.c[i][kk], masks); });
            af[i] = __builtin_bit_cast(vec8, out);
        }
    };
    auto multiply = [&](const vec8 (&af)[AF], const vec8 (&bf)[BF]) {
#pragma unroll
        for (int t = 0; t < BF; ++t)
#pragma unroll
            for (int i = 0; i < AF; ++i) acc[i][t] = gq4_mma32(af[i], bf[t], acc[i][t]);
    };
    // (fp16) the first or second part of the numbers of dword kk, of scales that fp16 weights cannot have
    auto number_rest = [&](const Codes &v, const Scales &sc, auto kkc, int part, Gq4Vec<BF16>::v8 (&af)[AF]) {
        constexpr int kk = decltype(kkc)::value, g = kk / PER;
#pragma unroll
        for (int i = 0; i < AF; ++i) {
            const float s = (float)__builtin_bit_cast(half_t, (uint16_t)(sc.s[i][g / 2] >> (16 * (g & 1))));
            const int z = (int)(NG == 1 ? sc.z[i] : sc.z[i] >> (8 * g) & 255u);
            uint4_t out;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t d = v.c[i][kk] >> (4 * e);
                out[e] = gq4_part_of((float)((int)(d & 15u) - z) * s, part) | gq4_part_of((float)((int)(d >> 16 & 15u) - z) * s, part) << 16;
            }
            af[i] = __builtin_bit_cast(Gq4Vec<BF16>::v8, out);
        }
    };

    if (steps > 0) {
        // (past the group's last step the last is fetched again; a group without steps has the layer's first)
        Codes w[RW];
        Tokens x[RX];
        auto step_of = [&](int s) { return min(first + s, last); };
        const int mine = min(turns, end - first);
        int window = window_of(step_of(0));
        load_window(window);
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) fetch_x(x[0], i, step_of(0));
#pragma unroll
        for (int i = 0; i < RW; ++i) fetch_w(w[i], step_of(i));
        put_window(window, false);
        load_window(window + 1);
        put_window(window + 1, false);
        load_window(window + 2);
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) put_x(x[0], i, own, KG == 1 || mine > 0);
#pragma unroll
        for (int i = 1; i <= RX; ++i)
#pragma unroll
            for (int z = 0; z < XTASKS; ++z) fetch_x(x[i % RX], z, step_of(i));
        gq4_lds_barrier();
        vec8 af[2][AF], bf[2][BF];
        Scales sc[2];
        read(own, 0, bf[0]);
        read_scales(sc[0], step_of(0));
        number(w[0], sc[0], std::integral_constant<int, 0>{}, af[0]);
        for (int s = 0; s < turns;) {
#pragma unroll
            for (int n = 0; n < UNROLL; ++n) {
                uint8_t *const from = own + (s & 1) * STAGE, *const to = own + (~s & 1) * STAGE;
                const int step = step_of(s), after = step_of(s + 1);
                Tokens &next = x[(n + 1) % RX];
                // The windows of this step's and the next one's groups are there.  Where this one's is a new one, nobody reads from the one before it any more (that was before the last
                // barrier), and the one after it takes its place; a window has four steps at least.
                if (window_of(step) != window) {
                    window = window_of(step);
                    put_window(window + 1, false);
                    load_window(window + 2);
                }
                static_for<4>([&](auto kkc) {
                    constexpr int kk = decltype(kkc)::value;
                    // The barrier stands before the last quarter's products: past it the next step's tokens are in LDS, and its first operands are made beside them.
                    if constexpr (kk == 3) gq4_lds_barrier();
                    read(kk < 3 ? from : to, (kk + 1) & 3, bf[(kk + 1) & 1]);
                    if constexpr (kk == 1) read_scales(sc[(n + 1) & 1], after);
#pragma unroll
                    for (int i = 0; i < XTASKS; ++i)
                        if (i * 3 / XTASKS == kk) {
                            put_x(next, i, to, KG == 1 || s + 1 < mine);
                            fetch_x(next, i, step_of(s + 1 + RX));
                        }
                    if constexpr (kk == 3) {
                        fetch_w(w[n], step_of(s + RW));
                        number(w[(n + 1) % RW], sc[(n + 1) & 1], std::integral_constant<int, 0>{}, af[0]);
                    } else
                        number(w[n], sc[n & 1], std::integral_constant<int, kk + 1>{}, af[(kk + 1) & 1]);
                    multiply(af[kk & 1], bf[kk & 1]);
#pragma unroll
                    for (int i = 0; i < AF * BF; ++i) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                  // a product,
                        __builtin_amdgcn_sched_group_barrier(0x002, BF >= 4 ? 4 : 8, 0);    // and vector instructions that it takes the time of
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
                if (++s >= turns) break;
            }
        }
    }
    // ---- steps without overlap, by the first group of wavefronts ----
    const int tail = whole < a.cb && (int)blockIdx.y == a.split.splits - 1 ? 2 : 0;
    // a step's tokens, element by element
    auto stage_x = [&](int step, auto &&of) {
        const int left = a.k - (step >> 1) * kGq4Cols;
#pragma unroll
        for (int i = 0; i < XTASKS; ++i) {
            const int row = (tid + i * THREADS) >> 3, p = tid & 7, c = 32 * (p >> 1) + 16 * (step & 1) + 8 * (p & 1);
            const E *at = static_cast<const E *>(a.x) + (int64_t)min(t0 + row, a.m - 1) * a.x_ld + (int64_t)(step >> 1) * kGq4Cols + c;
            Tokens v;
#pragma unroll
            for (int z = 0; z < 8; ++z) v.x[i][z] = c + z < left ? of(at[z]) : (E)0.f;
            put_x(v, i, own, true);
        }
    };
    if (tail) {
        // inputs that end inside a block: its two halves
        const int w = window_of(2 * whole);
        load_window(w);
        __syncthreads();                                                      // (nobody reads from LDS any more)
        put_window(w, false);
        for (int e = 0; e < 2; ++e) {
            __syncthreads();
            if (group == 0) stage_x(2 * whole + e, [](E v) { return v; });
            __syncthreads();
            if (group == 0) {
                Codes v;
                fetch_w(v, 2 * whole + e);
                Scales sc;
                read_scales(sc, 2 * whole + e);
                static_for<4>([&](auto kkc) {
                    vec8 af[AF], bf[BF];
                    read(own, decltype(kkc)::value, bf);
                    number(v, sc, kkc, af);
                    multiply(af, bf);
                });
            }
        }
    }
    if constexpr (__is_same(T, F16)) {
        // groups that were left out
        if (gq4_any_wave(large, lds + Lds::bytes, wave, KG * WR)) {
            for (int step = min(begin, end); step < end + tail; ++step) {
                const int w = window_of(step);
                load_window(w);
                __syncthreads();
                put_window(w, true);
                // (an infinite token has had its part: times the scales that are 0 now it would be a NaN)
                if (group == 0) stage_x(step, [](E v) { return __builtin_isfinite((float)v) ? v : (E)0.f; });
                __syncthreads();
                if (group == 0) {
                    Codes v;
                    fetch_w(v, step);
                    Scales sc;
                    read_scales(sc, step);
                    static_for<4>([&](auto kkc) {
                        vec8 bf[BF];
                        read(own, decltype(kkc)::value, bf);
#pragma unroll
                        for (int part = 0; part < 2; ++part) {
                            Gq4Vec<BF16>::v8 af[AF];
                            number_rest(v, sc, kkc, part, af);
#pragma unroll
                            for (int t = 0; t < BF; ++t)
#pragma unroll
                                for (int other = 0; other < 2; ++other) {
                                    const Gq4Vec<BF16>::v8 x = gq4_part_of(bf[t], other);
#pragma unroll
                                    for (int i = 0; i < AF; ++i) acc[i][t] = gq4_mma32(af[i], x, acc[i][t]);
                                }
                        }
                    });
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
                    const int tok = t0 + t * 32 + (lane & 31), o = o0 + (GATED ? (wr * AF + i) / 2 : wr * AF + i) * 32 + 4 * (lane >> 5);
                    float *const row = a.split.part + (((int64_t)blockIdx.y * (GATED ? 2 : 1) + (GATED ? i & 1 : 0)) * a.m + tok) * a.split.ld + o;
                    if (tok < a.m)
#pragma unroll
                        for (int g = 0; g < 4; ++g)
                            if (o + 8 * g < a.split.ld)
                                *reinterpret_cast<float4_t *>(row + 8 * g) = float4_t{acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
                }
        return;
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
                    const int tok = t * 32 + (lane & 31), c = ((GATED ? (wr * AF + i) / 2 : wr * AF + i) * 32 + 8 * g) / 8;
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
        leave(a.y[0], a.y_ld[0], [&](int i, int t, int e) { return gq4_gated(acc[i][t][e], acc[i + 1][t][e]); });
        if (a.y[1]) leave(a.y[1], a.y_ld[1], [&](int i, int t, int e) { return acc[i][t][e]; });
        if (a.y[2]) leave(a.y[2], a.y_ld[2], [&](int i, int t, int e) { return acc[i + 1][t][e]; });
    } else
        leave(a.y[0], a.y_ld[0], [&](int i, int t, int e) { return acc[i][t][e]; });
}

template <class T, bool GATED, int SHIFT, int SHAPE, int KG, int WR, int BF, int RX, int RW>
static int launch_gq4_rows_of(Gq4RowsArgs a, hipStream_t st)
{
    constexpr int THREADS = KG * WR * kWave, BO = 64 * WR, BT = 32 * BF;
    constexpr size_t OUT = (size_t)BO * BT * 2 / (GATED ? 2 : 1), SUMS = KG > 1 ? (size_t)BO * BT * 4 : 0, RING = Gq4RowsLds<KG, BO, BT>::bytes + kGq4Flags;
    constexpr size_t LDS = RING > OUT ? (RING > SUMS ? RING : SUMS) : OUT > SUMS ? OUT : SUMS;
    static_assert(LDS * kRowShapes[SHAPE].per_cu <= 160 * 1024 && kRowShapes[SHAPE].outs == BO && kRowShapes[SHAPE].toks == BT, "the table's tile");
    const int wide = GATED ? BO / 2 : BO;
    a.tiles_o = (int)(((int64_t)a.n + wide - 1) / wide);
    a.tiles_t = (int)(((int64_t)a.m + BT - 1) / BT);
    const int64_t tiles = (int64_t)a.tiles_o * a.tiles_t;
    if (tiles * THREADS > UINT32_MAX) return SLIM_ERR_SHAPE;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_rows_kernel<T, GATED, SHIFT, KG, WR, BF, RX, RW>), dim3((unsigned)tiles, (unsigned)a.split.splits), dim3(THREADS), LDS, st, a);
    return SLIM_OK;
}

template <class T, bool GATED, int SHIFT>
static int launch_gq4_rows_shape(const Gq4RowsArgs &a, int shape, hipStream_t st)
{
    switch (shape) {
    case 0: return launch_gq4_rows_of<T, GATED, SHIFT, 0, 1, 4, 4, 1, 2>(a, st);
    case 1: return launch_gq4_rows_of<T, GATED, SHIFT, 1, 2, 4, 2, 2, 2>(a, st);
    default: return launch_gq4_rows_of<T, GATED, SHIFT, 2, 4, 2, 2, 2, 2>(a, st);
    }
}

// Any number of tokens (arguments are checked where this is called); up: null for a plain product.
int gq4_launch_rows(const slim_group_q4_layer *layer, const slim_group_q4_layer *up, int shift, const void *X, int64_t x_ld, int32_t m, void *const (&y)[3],
                    const int64_t (&y_ld)[3], int32_t dtype, void *workspace, hipStream_t st)
{
    const Gq4Plan plan = gq4_plan_rows(layer->n, layer->k, m, up != nullptr);
    Gq4RowsArgs a{};
    a.split = Gq4Split{plan.splits > 1 ? static_cast<float *>(workspace) : nullptr, plan.splits, gq4_part_ld(layer->n)};
    a.w[0] = gq4_weights(layer);
    if (up) a.w[1] = gq4_weights(up);
    a.x = X;
    a.x_ld = x_ld;
    for (int i = 0; i < 3; ++i) {
        a.y[i] = y[i];
        a.y_ld[i] = y_ld[i];
    }
    a.n = layer->n;
    a.k = layer->k;
    a.m = m;
    a.cb = gq4_col_blocks(layer->k);
    a.rb = gq4_row_blocks(layer->n);
    a.kg = gq4_groups(layer->k, shift);
    auto of = [&](auto type, auto gated) {
        typedef decltype(type) T;
        constexpr bool GATED = decltype(gated)::value;
        return shift == 5 ? launch_gq4_rows_shape<T, GATED, 5>(a, plan.shape, st) : shift == 6 ? launch_gq4_rows_shape<T, GATED, 6>(a, plan.shape, st) : launch_gq4_rows_shape<T, GATED, 7>(a, plan.shape, st);
    };
    int rc;
    if (dtype == SLIM_F16)
        rc = up ? of(F16{}, std::true_type{}) : of(F16{}, std::false_type{});
    else
        rc = up ? of(BF16{}, std::true_type{}) : of(BF16{}, std::false_type{});
    if (rc != SLIM_OK) return rc;
    if (plan.splits > 1) return gq4_launch_finish(a.split, m, layer->n, up != nullptr, a.y, a.y_ld, dtype, st);
    return hip_status(hipGetLastError());
}

}  // namespace slim
