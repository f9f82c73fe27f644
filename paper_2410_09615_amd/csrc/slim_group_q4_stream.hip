// Products with 4-bit weights that have a scale for each group of inputs, for up to 48 tokens (small layers: 192, in chunks of up to 48): the weights are streamed once, from memory to registers.
//   plain  Y = X W^T,     gated  H = silu(X Wg^T) * (X Wu^T)
// A workgroup has FR blocks of 16 rows (of a gated pair half are gate's, half up's) and all tokens; its wavefronts share the inputs, blocks of 128 each.
// A lane's 16 bytes of a block are its operand of four 16 x 16 x 32 products, once codes are numbers: c - z, exactly, in the inputs' type.  A group's
// products start from zero and are added to the binary32 sums with its scale, so that a result is rounded once and nothing before it is.
// The wavefronts' sums meet in LDS and are added in order.
// Bound by memory in fp16 where the layer is large: 28672 x 8192 at one token 24.0 us, 5.0 TB/s (a large copy 5.15), 2 x 28672 x 8192 gated 49, at 16 tokens 28.4.  In bf16 a pair of codes takes five instructions
// instead of two and a half: one token 31 us, 16 tokens 34 to 36, vector instructions 60 % of the cycles.  With 48 tokens by what is issued and by the tokens' way through the L2, which every
// workgroup takes (13824 x 5120 gated, bf16, groups of 64: 424 MB of tokens to 77 of weights, 39 us).  4096 x 4096 at one token: the call's host time, 5 us (kernel 5).
#include <hip/hip_runtime.h>

#include "slim_group_q4.h"
#include "slim_mma.h"

namespace slim {

struct Gq4StreamArgs {
    Gq4Weights w[2];
    const void *x;
    int64_t x_ld;
    void *y[3];
    int64_t y_ld[3];
    int n, k, m, cb, rb, kg;
};

// c - z of the eight codes of a dword, exactly, in the inputs' type; in bf16 times 2^-15 (of masks and zero points that are biased so), so that a group's sum of products, at most 128 terms with
// |c - z| up to 255, is smaller than its largest input and stays in range wherever the result does: with whole numbers tokens of 2^121 have sums beyond binary32.  (fp16's tokens end at 2^16.)
template <class T>
constexpr uint32_t kGq4StreamBias = __is_same(T, F16) ? kGq4Bias : kGq4BiasLow;
template <class T>
constexpr float kGq4StreamLow = __is_same(T, F16) ? 1.f : kGq4Low;
template <class T>
__device__ __forceinline__ typename Gq4Vec<T>::v8 gq4_whole(uint32_t d, const Gq4Masks &k, half2_t z0, half2_t z1)
{
    uint4_t v;
    static_for<4>([&](auto ec) {
        const half2_t c = gq4_less_zeros<decltype(ec)::value>(d, k, z0, z1);
        if constexpr (__is_same(T, F16))
            v[decltype(ec)::value] = __builtin_bit_cast(uint32_t, c);
        else                                                          // (whole numbers below 256 times 2^-15: their first 16 bits in binary32)
            v[decltype(ec)::value] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, (float)c[1]), __builtin_bit_cast(uint32_t, (float)c[0]), 0x07060302u);
    });
    return __builtin_bit_cast(typename Gq4Vec<T>::v8, v);
}

// Orders a wavefront's writes to LDS before its reads of what other lanes wrote: its LDS instructions are executed in order.
__device__ __forceinline__ void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// What a wavefront has of LDS: a block's tokens, and for each block of rows 32 groups' scales and zero points.
template <int FR, int TB>
struct Gq4StreamLds {
    static constexpr int scale_row = 80, zero_row = 40, table = 16 * (scale_row + zero_row), scales = TB * 4096, bytes = scales + FR * table;
};

// XI: loads of four tokens each; TB: tiles of 16 tokens; D: blocks' weights under way and in use.
template <class T, bool GATED, int SHIFT, int FR, int XI, int D, int THREADS>
__global__ __launch_bounds__(THREADS) void gq4_stream_kernel(Gq4StreamArgs a)
{
    typedef typename T::type E;
    typedef typename Gq4Vec<T>::v8 vec8;
    constexpr int TB = (XI + 3) / 4, NG = kGq4Cols >> SHIFT, PER = 4 / NG;               // groups per block, products per group
    extern __shared__ __align__(16) uint8_t lds[];
    const int S = (int)blockDim.x / kWave, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x & (kWave - 1);
    const int r = lane & 15, q = lane >> 4;
    const int t0 = (int)blockIdx.y * (16 * TB), toks = min(16 * TB, a.m - t0);          // this workgroup's tokens
    const uint8_t *const xbase = static_cast<const uint8_t *>(a.x) + (int64_t)t0 * a.x_ld * 2;
    constexpr int PAIRS = GATED ? FR / 2 : FR;
    const int rb0 = (int)blockIdx.x * PAIRS;
    const int whole = a.k / kGq4Cols, share = (whole + S - 1) / S, first = w * share, end = min(first + share, whole);
    const Gq4Masks masks(kGq4StreamBias<T>);

    typedef Gq4StreamLds<FR, TB> Lds;
    uint8_t *const own = lds + w * Lds::bytes;
    const uint8_t *codes[FR], *zeros[FR];
    const half_t *scales[FR];
    uint32_t row_at[FR];                                              // the lane's row among the groups of its 16 rows
#pragma unroll
    for (int f = 0; f < FR; ++f) {
        const Gq4Weights &l = GATED && f >= PAIRS ? a.w[1] : a.w[0];
        const int rb = min(rb0 + (GATED ? f % PAIRS : f), a.rb - 1);
        const int64_t at = (int64_t)rb * kGq4Rows * a.kg;
        codes[f] = l.codes + (int64_t)rb * a.cb * kGq4Block;
        scales[f] = l.scales + at;
        zeros[f] = l.zeros ? l.zeros + at : nullptr;
        row_at[f] = (uint32_t)min(r, a.n - 1 - rb * kGq4Rows) * (uint32_t)a.kg;
    }
    // Inputs are fetched as they lie, 16 lanes to the 256 bytes of a token's block, and put in LDS, each wavefront its own, from where a product's operand is read: as
    // the operand needs them, neighbouring lanes would ask for different tokens.  A token's 16 pieces of 16 bytes are in another order in each of 16 rows.
    uint32_t x_at[XI];
#pragma unroll
    for (int i = 0; i < XI; ++i) x_at[i] = ((uint32_t)min(4 * i + q, toks - 1) * (uint32_t)a.x_ld + 8u * (uint32_t)r) * 2u;

    struct Stage {
        uint4_t c[FR];
    };
    struct Tokens {
        vec8 v[XI];
    };
    // Scales and zero points come 32 groups of a row at a time, lane (r, q) the eight from 8 q on, and are read from LDS too, for the same reason.
    struct Run {
        uint4_t s[FR];
        uint2_t z[FR];
    };
    auto load_run = [&](Run &run, int g0) {
        const int at = g0 + 8 * q;
#pragma unroll
        for (int f = 0; f < FR; ++f) {
            run.s[f] = uint4_t{0, 0, 0, 0};
            run.z[f] = uint2_t{0x01010101u * kGq4Sym, 0x01010101u * kGq4Sym};
            if (at + 8 <= a.kg) {
                run.s[f] = reinterpret_cast<const Gq4Any<uint4_t> *>(scales[f] + (row_at[f] + (uint32_t)at))->v;
                if (zeros[f]) run.z[f] = reinterpret_cast<const Gq4Any<uint2_t> *>(zeros[f] + (row_at[f] + (uint32_t)at))->v;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (at + e < a.kg) {
                        run.s[f][e / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, scales[f][row_at[f] + (uint32_t)(at + e)]) << (16 * (e & 1));
                        if (zeros[f])
                            run.z[f][e / 4] = (run.z[f][e / 4] & ~(255u << (8 * (e & 3)))) | (uint32_t)zeros[f][row_at[f] + (uint32_t)(at + e)] << (8 * (e & 3));
                    }
            }
        }
    };
    auto put_run = [&](const Run &run) {
#pragma unroll
        for (int f = 0; f < FR; ++f) {
            *reinterpret_cast<uint4_t *>(own + Lds::scales + f * Lds::table + r * Lds::scale_row + q * 16) = run.s[f];
            *reinterpret_cast<uint2_t *>(own + Lds::scales + f * Lds::table + 16 * Lds::scale_row + r * Lds::zero_row + q * 8) = run.z[f];
        }
        wave_lds_order();
    };
    auto load_x = [&](Tokens &x, int b) {
        const uint8_t *base = xbase + (int64_t)b * (kGq4Cols * 2);
#pragma unroll
        for (int i = 0; i < XI; ++i) x.v[i] = Piece<T, 8>::load(reinterpret_cast<const E *>(base + x_at[i]));
    };
    auto load = [&](Stage &st, int b) {
#pragma unroll
        for (int f = 0; f < FR; ++f) st.c[f] = *reinterpret_cast<const uint4_t *>(codes[f] + (int64_t)b * kGq4Block + (uint32_t)lane * 16u);
    };
    float4_t acc[FR][TB];
#pragma unroll
    for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int t = 0; t < TB; ++t) acc[f][t] = float4_t{0.f, 0.f, 0.f, 0.f};
    auto put_x = [&](const Tokens &x) {
#pragma unroll
        for (int i = 0; i < XI; ++i) *reinterpret_cast<vec8 *>(own + (4 * i + q) * 256 + (r ^ ((4 * i + q) & 15)) * 16) = x.v[i];
        wave_lds_order();
    };
    // a block's products; its first group is the run's group `at`
    auto use = [&](const Stage &st, int at) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            float4_t p[FR][TB];
            float s[FR];
            half2_t z0[FR], z1[FR];
#pragma unroll
            for (int f = 0; f < FR; ++f) {
                const uint8_t *table = own + Lds::scales + f * Lds::table;
                s[f] = (float)*reinterpret_cast<const half_t *>(table + r * Lds::scale_row + (at + g) * 2) * (1.f / kGq4StreamLow<T>);
                const uint32_t zp = table[16 * Lds::scale_row + r * Lds::zero_row + at + g];
                z0[f] = gq4_biased_zeros(zp, zp, kGq4StreamBias<T>);
                z1[f] = z0[f] - half2_t{(half_t)(960.f * kGq4StreamLow<T>), (half_t)(960.f * kGq4StreamLow<T>)};
#pragma unroll
                for (int t = 0; t < TB; ++t) p[f][t] = float4_t{0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll
            for (int j = g * PER; j < (g + 1) * PER; ++j) {
                vec8 xf[TB];
#pragma unroll
                for (int t = 0; t < TB; ++t) xf[t] = *reinterpret_cast<const vec8 *>(own + (16 * t + r) * 256 + ((4 * j + q) ^ r) * 16);
#pragma unroll
                for (int f = 0; f < FR; ++f) {
                    const vec8 wv = gq4_whole<T>(st.c[f][j], masks, z0[f], z1[f]);
#pragma unroll
                    for (int t = 0; t < TB; ++t) p[f][t] = gq4_mma16(xf[t], wv, p[f][t]);
                }
                // (with so many tokens there is no room in registers for the next products' operands)
                if constexpr (XI >= 12 && FR > 1) __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int f = 0; f < FR; ++f)
#pragma unroll
                for (int t = 0; t < TB; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[f][t][e] = __builtin_fmaf(p[f][t][e], s[f], acc[f][t][e]);
        }
        wave_lds_order();
    };
    constexpr int RUN = 32 / NG;                                      // blocks of a run
    Stage st[D];
    Tokens x;
    Run run;
    if (first < end) {
        load_run(run, first * NG);
        load_x(x, first);
#pragma unroll
        for (int i = 0; i < D - 1; ++i) load(st[i], min(first + i, end - 1));
        for (int b = first, at = 0;;) {
            bool more = true;
#pragma unroll
            for (int i = 0; i < D; ++i) {
                if (at == 0) {
                    put_run(run);
                    if (b + RUN < end) load_run(run, (b + RUN) * NG);
                }
                // (Loads come back in order: the tokens of the next block are asked for before weights that are wanted later.  Past the share's last block it is
                // fetched again.)
                put_x(x);
                load_x(x, min(b + 1, end - 1));
                __builtin_amdgcn_sched_barrier(0);
                load(st[(i + D - 1) % D], min(b + D - 1, end - 1));
                __builtin_amdgcn_sched_barrier(0);
                use(st[i], at * NG);
                at = at + 1 < RUN ? at + 1 : 0;
                if (++b >= end) {
                    more = false;
                    break;
                }
            }
            if (!more) break;
        }
    }
    // inputs that end inside a block
    if (whole < a.cb && w == S - 1) {
        const int left = a.k - whole * kGq4Cols;
        load_run(run, whole * NG);
        load(st[0], whole);
        const uint8_t *base = xbase + (int64_t)whole * (kGq4Cols * 2);
#pragma unroll
        for (int i = 0; i < XI; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) x.v[i][e] = 8 * r + e < left ? reinterpret_cast<const E *>(base + x_at[i])[e] : (E)0.f;
        put_run(run);
        put_x(x);
        use(st[0], 0);
    }

    __syncthreads();                                                  // (the sums go where the tokens were)
    float4_t *part = reinterpret_cast<float4_t *>(lds);               // [S][FR * TB][64]
#pragma unroll
    for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int t = 0; t < TB; ++t) part[(w * FR * TB + f * TB + t) * kWave + lane] = acc[f][t];
    __syncthreads();
    for (int i = (int)threadIdx.x / kWave; i < PAIRS * TB; i += S) {
        const int f = i / TB, t = i % TB, row = (rb0 + f) * kGq4Rows + r;
        float4_t v = {0.f, 0.f, 0.f, 0.f}, u = v;
        for (int z = 0; z < S; ++z) {
            v += part[(z * FR * TB + i) * kWave + lane];
            if constexpr (GATED) u += part[(z * FR * TB + PAIRS * TB + i) * kWave + lane];
        }
        if (row < a.n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t tok = t0 + 16 * t + 4 * q + e;
                if (tok < a.m) {
                    if constexpr (GATED) {
                        static_cast<E *>(a.y[0])[tok * a.y_ld[0] + row] = (E)gq4_gated(v[e], u[e]);
                        if (a.y[1]) static_cast<E *>(a.y[1])[tok * a.y_ld[1] + row] = (E)v[e];
                        if (a.y[2]) static_cast<E *>(a.y[2])[tok * a.y_ld[2] + row] = (E)u[e];
                    } else
                        static_cast<E *>(a.y[0])[tok * a.y_ld[0] + row] = (E)v[e];
                }
            }
        }
    }
}

// Two blocks of rows to a workgroup (a gated pair has two in any case) read the tokens half as often, but leave half as many workgroups: what takes less
// of rounds x (blocks + half a block per 16 tokens).  us with one / two: 4096 x 4096 at 16 tokens 5.0 / 6.5, 48 8.6 / 10.2; 8192 x 8192 at 16 10.8 / 9.6, 48 21.0 / 15.4;
// 11008 x 4096 at 16 8.1 / 8.8, 48 17.3 / 14.8; 28672 x 8192 at 16 36.6 / 28.4, 48 80 / 52.
// Wavefronts: as many as have 2700 blocks of weights at work, 10 per compute unit (with three under way each, 32 KiB), two at least: more have shorter shares.  us with
// 2 / 4 / 8: 28672 x 8192 at one token 24.0 / 25.0 / 26.3 (two blocks of rows), 8192 x 28672 at one 46 / 31 / 26, 11008 x 4096 at 4 7.8 / 6.7 / 7.8, 4096 x 4096 at 16 6.9 / 5.1 / 5.0.
struct Gq4StreamPlan {
    int blocks, waves, workgroups;
};
static Gq4StreamPlan gq4_plan_stream(int rb, int cb, int tb, bool gated)
{
    const int cus = device_info().cus;
    auto cost = [&](int blocks) { return ((rb + blocks * cus - 1) / (blocks * cus)) * (2 * blocks + tb); };
    Gq4StreamPlan p;
    p.blocks = gated || cost(2) <= cost(1) ? 2 : 1;
    p.workgroups = gated ? rb : (rb + p.blocks - 1) / p.blocks;
    p.waves = 2;
    const int64_t all = gated ? 2 * (int64_t)rb : rb;
    while (p.waves < 8 && all * p.waves * 256 < (int64_t)2700 * cus && p.waves * 2 <= cb) p.waves *= 2;
    const size_t bytes = (p.blocks == 2 ? Gq4StreamLds<2, 1>::bytes : Gq4StreamLds<1, 1>::bytes) + (size_t)(tb - 1) * 4096;
    while (p.waves > 1 && p.waves * bytes > device_info().lds) p.waves /= 2;
    return p;
}

// of a call's tokens: workgroups for so many each, up to 48 and as alike as can be
static int gq4_stream_chunks(int m) { return (m + 47) / 48; }
static int gq4_stream_tiles(int m) { return ((m + gq4_stream_chunks(m) - 1) / gq4_stream_chunks(m) + 15) / 16; }

void gq4_stream_plan(int n, int k, int m, bool gated, int32_t *out)
{
    const Gq4StreamPlan p = gq4_plan_stream(gq4_row_blocks(n), gq4_col_blocks(k), gq4_stream_tiles(m), gated);
    out[1] = p.blocks * kGq4Rows;
    out[2] = m <= 4 ? 4 : 16 * gq4_stream_tiles(m);
    out[3] = p.waves;
}

template <class T, bool GATED, int SHIFT, int FR, int XI>
static void launch_gq4_stream_of(const Gq4StreamArgs &a, const Gq4StreamPlan &p, hipStream_t st)
{
    constexpr int TB = (XI + 3) / 4, D = XI >= 12 ? 2 : 3, THREADS = 512;
    constexpr size_t LDS = Gq4StreamLds<FR, TB>::bytes;
    static_assert(LDS == Gq4StreamLds<FR, 1>::bytes + (TB - 1) * 4096 && (size_t)FR * TB * kWave * 16 <= LDS, "LDS");
    hipLaunchKernelGGL(HIP_KERNEL_NAME(gq4_stream_kernel<T, GATED, SHIFT, FR, XI, D, THREADS>), dim3((unsigned)p.workgroups, (unsigned)((a.m + 16 * TB - 1) / (16 * TB))), dim3((unsigned)(p.waves * kWave)),
                       p.waves * LDS, st, a);
}

template <class T, bool GATED, int SHIFT, int XI>
static void launch_gq4_stream_tb(const Gq4StreamArgs &a, hipStream_t st)
{
    const Gq4StreamPlan p = gq4_plan_stream(a.rb, a.cb, XI <= 4 ? 1 : XI / 4, GATED);
    if constexpr (!GATED)
        if (p.blocks == 1) return launch_gq4_stream_of<T, GATED, SHIFT, 1, XI>(a, p, st);
    launch_gq4_stream_of<T, GATED, SHIFT, 2, XI>(a, p, st);
}

template <class T, bool GATED, int SHIFT>
static void launch_gq4_stream_shift(const Gq4StreamArgs &a, hipStream_t st)
{
    if (a.m <= 4) return launch_gq4_stream_tb<T, GATED, SHIFT, 1>(a, st);
    switch (gq4_stream_tiles(a.m)) {
    case 1: return launch_gq4_stream_tb<T, GATED, SHIFT, 4>(a, st);
    case 2: return launch_gq4_stream_tb<T, GATED, SHIFT, 8>(a, st);
    default: return launch_gq4_stream_tb<T, GATED, SHIFT, 12>(a, st);
    }
}

template <class T, bool GATED>
static void launch_gq4_stream_type(const Gq4StreamArgs &a, int shift, hipStream_t st)
{
    if (shift == 5)
        launch_gq4_stream_shift<T, GATED, 5>(a, st);
    else if (shift == 6)
        launch_gq4_stream_shift<T, GATED, 6>(a, st);
    else
        launch_gq4_stream_shift<T, GATED, 7>(a, st);
}

// Few tokens (gq4_streamed; checked, as all arguments are, where this is called); up: null for a plain product.
int gq4_launch_stream(const slim_group_q4_layer *layer, const slim_group_q4_layer *up, int shift, const void *X, int64_t x_ld, int32_t m, void *const (&y)[3],
                      const int64_t (&y_ld)[3], int32_t dtype, hipStream_t st)
{
    Gq4StreamArgs a{};
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
    if (dtype == SLIM_F16) {
        if (up)
            launch_gq4_stream_type<F16, true>(a, shift, st);
        else
            launch_gq4_stream_type<F16, false>(a, shift, st);
    } else {
        if (up)
            launch_gq4_stream_type<BF16, true>(a, shift, st);
        else
            launch_gq4_stream_type<BF16, false>(a, shift, st);
    }
    return hip_status(hipGetLastError());
}

}  // namespace slim
