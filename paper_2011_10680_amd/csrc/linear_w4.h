// Linear layer with 4-bit weights and a scale for each group of them, for the few rows of a decoding step: one projection, or the two of a
// gated feed-forward block with the activation and the product.
//
//   y[m,n] = sum_g s[n,g] * ( sum_{k in g} x[m,k] u[n,k]  -  (16 + z[n,g]) * sum_{k in g} x[m,k] ),   u = 16 + nibble
//
// The matrix instruction takes 16 outputs x 32 weights from one register of packed nibbles per lane: a shift, and one
// three-operand bit operation put two nibbles into the mantissas of two 16-bit floats of value 16 + nibble (exact in both
// types; a signed nibble is its offset form with zero point 8), so a weight costs one vector operation and no conversion.
// The zero point and the 16 leave through the sum of x over the group, which one product with a matrix of ones gives for
// all outputs.  Group sums and totals are 32-bit; nothing is rounded before the result.
//
// Bound by the weights' bytes for some rows (13 of 16384 x 8192, groups of 64 with zero points: 20.8 us, 74 MB at 3.5 TB/s, half of the
// waves' time waiting), by a launch and one chain of loads for one row of a small layer (1000 x 2048: 4.2 us, of which an empty launch
// is 2.6), and by the vector pipe beyond 32 rows, where a weight is expanded again for every tile of rows.  A wave reads 16 bytes per lane (four lanes cover 64 bytes of one output's row), and a 4 x 4
// exchange between its quarters turns the four registers into four operands of 32 consecutive weights each, so that a group
// of 32 has a matrix instruction of its own.  The waves of a workgroup take every W-th 128 weights of the same outputs and
// add up in LDS: one output's reduction is shared by the whole workgroup, and few outputs still fill the chip.  The scales of the
// workgroup's outputs are brought into LDS first, in rows as they lie (read by each lane where it needs them, two bytes here and there,
// they took the 13 rows from 25 to 30 us).
#pragma once
#include "lm.h"
#include "lm_launch.h"

namespace hawq {

namespace {

constexpr int kScaleBytes = 64 * 1024;       // of LDS for the scales of a segment of the reduction

template <class T> struct Nibbles;
template <> struct Nibbles<F16> {            // 16 + u: 0x4C00 | u << 6
    static constexpr uint32_t mask = 0x03C003C0u, base = 0x4C004C00u, sign = 0x02000200u, one = 0x3C003C00u;
    template <int I> static __device__ __forceinline__ uint32_t shift(uint32_t d) { return I == 0 ? d << 6 : I == 1 ? d << 2 : I == 2 ? d >> 2 : d >> 6; }
};
template <> struct Nibbles<BF16> {           // 0x4180 | u << 3
    static constexpr uint32_t mask = 0x00780078u, base = 0x41804180u, sign = 0x00400040u, one = 0x3F803F80u;
    template <int I> static __device__ __forceinline__ uint32_t shift(uint32_t d) { return I == 0 ? d << 3 : I == 1 ? d >> 1 : I == 2 ? d >> 5 : d >> 9; }
};

// operand of eight weights: nibbles (0,4), (1,5), (2,6), (3,7); base: Nibbles<T>::base ^ (sign where the weights are signed)
template <class T>
__device__ __forceinline__ typename T::v8 expand(uint32_t d, uint32_t mask, uint32_t base) {
    v4u r;
    r.x = (Nibbles<T>::template shift<0>(d) & mask) ^ base;
    r.y = (Nibbles<T>::template shift<1>(d) & mask) ^ base;
    r.z = (Nibbles<T>::template shift<2>(d) & mask) ^ base;
    r.w = (Nibbles<T>::template shift<3>(d) & mask) ^ base;
    return __builtin_bit_cast(typename T::v8, r);
}

// eight consecutive values of x in the same order
template <class T>
__device__ __forceinline__ typename T::v8 ordered(v4u d) {
    v4u r;
    r.x = __builtin_amdgcn_perm(d.z, d.x, 0x05040100u);
    r.y = __builtin_amdgcn_perm(d.z, d.x, 0x07060302u);
    r.z = __builtin_amdgcn_perm(d.w, d.y, 0x05040100u);
    r.w = __builtin_amdgcn_perm(d.w, d.y, 0x07060302u);
    return __builtin_bit_cast(typename T::v8, r);
}

// register j of the wave's quarter c <-> register c of its quarter j
__device__ __forceinline__ void exchange_quarters(v4u &d) {
    const v2u a = __builtin_amdgcn_permlane32_swap(d.x, d.z, false, false), b = __builtin_amdgcn_permlane32_swap(d.y, d.w, false, false);
    const v2u e = __builtin_amdgcn_permlane16_swap(a.x, b.x, false, false), f = __builtin_amdgcn_permlane16_swap(a.y, b.y, false, false);
    d.x = e.x; d.y = e.y; d.z = f.x; d.w = f.y;
}

// An output by the formula as it stands, one weight after the other, in 64 bits, whose range no product of three leaves: where x times
// 31 leaves that of 32 bits, or x or a scale is infinite, the two sums of the fast form do, and their difference says nothing.
template <class T>
__device__ __forceinline__ double plain_output(const LinearW4Args &a, int m, int64_t n) {
    typedef typename T::elem E;
    const E *x = (const E *)a.x + m * a.x_stride, *s = (const E *)a.scales + n * a.groups;
    const uint8_t *w = a.w + n * (a.K >> 1);
    double v = 0;
    for (int g = 0; g < a.groups; ++g) {
        const int zero = a.zeros ? a.zeros[n * a.groups + g] : 0, end = (int)min((int64_t)(g + 1) * a.group, (int64_t)a.K);
        const double scale = (double)(float)s[g];
        for (int k = g * a.group; k < end; ++k) {
            const int q = w[k >> 1] >> (4 * (k & 1)) & 15;
            v += (double)(float)x[k] * (double)((a.zeros || q < 8 ? q : q - 16) - zero) * scale;
        }
    }
    return v;
}

// g / (1 + exp(-t)) by exp(-|t|), which is 1 at most.  Its argument is a product with log2(e) and what rounding that left out (2 units in the last
// place; the product alone would be off by 30).  The instruction has no results below 2^-126, where g times it still is a number: such ones are taken
// times 2^64, and 1 + exp(-|t|) is 1 there.
__device__ __forceinline__ float gate_of(float g, float t) {
    const float v = -fabsf(t), p = v * 1.44269504f, rest = fmaf(v, 1.92596303e-8f, fmaf(v, 1.44269504f, -p));
    const bool far = p < -64.f;
    float e = __builtin_amdgcn_exp2f(far ? p + 64.f : p);
    e = p > -256.f ? fmaf(e, rest * 0.693147181f, e) : e;
    const float r = __builtin_amdgcn_rcpf(far ? 1.f : 1.f + e);
    return t < 0 ? g * e * (far ? 0x1p-64f : r) : g * r;
}

// The gate's activation.  The normal distribution's tail is taken by itself, not as a difference from 1.
__device__ __forceinline__ float activated(float g, int kind) {
    if (kind == HAWQ_SILU) return gate_of(g, g);
    if (kind == HAWQ_GELU) return 0.5f * g * erfcf(g * -0.70710678118654752f);
    if (kind == HAWQ_GELU_TANH) return gate_of(g, 1.5957691216057308f * (g + 0.044715f * g * g * g));      // (1 + tanh(t / 2)) / 2 = 1 / (1 + exp(-t))
    return g > 0.f || g != g ? g : 0.f;
}

// RT, MT: 16-output and 16-row tiles of a wave.  PIECES: parts of 128 weights with a scale of their own.  ALIGN: bytes the rows of w
// are read in (16, 4; 1: also x element by element).  ZEROS: unsigned weights with zero points.  GATED: half of the tiles are outputs of
// the gate, the other half the same outputs of the second projection, and what is stored is act(gate) * second.
template <class T, int RT, int MT, int PIECES, int ALIGN, bool ZEROS, bool GATED>
__global__ __launch_bounds__(512) void linear_w4(LinearW4Args a, FastDiv by_group) {
    typedef typename T::elem E;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, r = lane & 15, c = lane >> 4;
    constexpr int OUT = GATED ? RT / 2 : RT;       // tiles of outputs
    const int n0 = blockIdx.x * (16 * OUT), m0 = blockIdx.y * (16 * MT);
    // scales of a segment of the reduction: [group][scale, scale * (16 + zero point)][outputs], fours of outputs swizzled by the group
    constexpr int R = 16 * RT, SEG = kScaleBytes / (8 * R);
    float *scale = (float *)lds;
    auto swizzled = [&](int group, int row) { return row ^ ((group << 2) & (R - 1)); };
    uint32_t mask = Nibbles<T>::mask, base = Nibbles<T>::base ^ (ZEROS ? 0u : Nibbles<T>::sign);
    asm("" : "+s"(mask));                          // (registers: as literals the two operations would not be one instruction)
    asm("" : "+v"(base));
    const typename T::v8 ones = __builtin_bit_cast(typename T::v8, v4u{Nibbles<T>::one, Nibbles<T>::one, Nibbles<T>::one, Nibbles<T>::one});

    // Offsets of this lane's rows of w, one for each tile, from the workgroup's first row, and of its rows of x (rows past the last one:
    // the last one again).
    uint32_t w_row[RT];
    std::conditional_t<ALIGN == 1, int64_t, uint32_t> x_row[MT];
    const int64_t first = (int64_t)n0;
    for (int t = 0; t < RT; ++t) {
        w_row[t] = (uint32_t)min(16 * (t % OUT) + r, a.N - 1 - n0) * (uint32_t)(a.K >> 1);
    }
    for (int i = 0; i < MT; ++i) x_row[i] = min(16 * i + r, a.M - 1 - m0) * (decltype(x_row[0] + 0))a.x_stride;
    const uint8_t *w0 = a.w + first * (a.K >> 1), *z0 = ZEROS ? a.zeros + first * a.groups : nullptr;
    const uint8_t *w1 = GATED ? w0 + a.up * (a.K >> 1) : nullptr, *z1 = GATED && ZEROS ? z0 + a.up * a.groups : nullptr;
    const E *s0 = (const E *)a.scales + first * a.groups, *s1 = GATED ? s0 + a.up * a.groups : nullptr, *x0 = (const E *)a.x + (int64_t)m0 * a.x_stride;

    // x of more than 16 rows would not fit beside the next step's: it is read where it is used, from the caches
    constexpr bool X_AHEAD = MT == 1;
    struct Stage {
        v4u w[RT], x[X_AHEAD ? 1 : 0][4];
    };
    // No branches around loads: behind one the compiler no longer knows which loads are under way and waits for all of them.  What lies
    // past the end of the reduction is read from its last whole piece, and x is zero there.
    auto load_x = [&](int k0, int i, v4u (&x)[4]) {
        for (int j = 0; j < 4; ++j) {
            const int k = k0 + 32 * j + 8 * c;
            if constexpr (ALIGN > 1) {
                x[j] = *(const v4u *)(x0 + (x_row[i] + (uint32_t)min(k, a.K - 8)));
            } else {
                for (int e = 0; e < 4; ++e) {
                    const uint16_t *p = (const uint16_t *)x0 + (x_row[i] + (uint32_t)min(k + 2 * e, a.K - 2));
                    x[j][e] = p[0] | (uint32_t)p[1] << 16;
                }
            }
        }
    };
    // the 128 weights from k0 on: 32 of this lane's rows from k0 + 32 c on
    auto load = [&](int k0, Stage &g) {
        const int kw = k0 + 32 * c;
        for (int t = 0; t < RT; ++t) {
            const uint8_t *from = GATED && t >= OUT ? w1 : w0;
            if constexpr (ALIGN == 16) {
                g.w[t] = *(const v4u *)(from + (w_row[t] + (uint32_t)(min(kw, a.K - 32) >> 1)));
            } else if constexpr (ALIGN == 4) {
                for (int j = 0; j < 4; ++j) g.w[t][j] = *(const uint32_t *)(from + (w_row[t] + (uint32_t)(min(kw + 8 * j, a.K - 8) >> 1)));
            } else {
                for (int j = 0; j < 4; ++j) {
                    uint32_t d = 0;
                    for (int i = 0; i < 4; ++i) d |= (uint32_t)from[w_row[t] + (uint32_t)(min(kw + 8 * j + 2 * i, a.K - 2) >> 1)] << (8 * i);
                    g.w[t][j] = d;
                }
            }
        }
        if constexpr (X_AHEAD) load_x(k0, 0, g.x[0]);
    };

    v4f acc[RT][MT];
    for (int t = 0; t < RT; ++t)
        for (int i = 0; i < MT; ++i) acc[t][i] = v4f{0, 0, 0, 0};

    auto use = [&](int k0, int g0, Stage &now) {
        v4u xs[MT][4];
        for (int i = 0; i < MT; ++i) {
            if constexpr (X_AHEAD) for (int j = 0; j < 4; ++j) xs[i][j] = now.x[0][j];
            else load_x(k0, i, xs[i]);
            if (k0 + 128 > a.K)
                for (int j = 0; j < 4; ++j)
                    for (int e = 0; e < 4; ++e)
                        if (k0 + 32 * j + 8 * c + 2 * e >= a.K) xs[i][j][e] = 0;
        }
        for (int t = 0; t < RT; ++t) exchange_quarters(now.w[t]);
        typename T::v8 xv[MT][4];
        float sum[MT][PIECES];                                      // (every row of the product with ones is the same)
        for (int i = 0; i < MT; ++i)
            for (int p = 0; p < PIECES; ++p) {
                v4f t{0, 0, 0, 0};
                for (int j = p * 4 / PIECES; j < (p + 1) * 4 / PIECES; ++j) {
                    xv[i][j] = ordered<T>(xs[i][j]);
                    t = T::mfma16(ones, xv[i][j], t);
                }
                sum[i][p] = t[0];
            }
        int group[PIECES];                                          // of the segment
        for (int p = 0; p < PIECES; ++p) group[p] = (int)fdiv((uint32_t)min(k0 + p * (128 / PIECES), a.K - 1), by_group) - g0;
        for (int t = 0; t < RT; ++t)
            for (int p = 0; p < PIECES; ++p) {
                v4f part[MT];
                for (int i = 0; i < MT; ++i) part[i] = v4f{0, 0, 0, 0};
                for (int j = p * 4 / PIECES; j < (p + 1) * 4 / PIECES; ++j) {
                    const typename T::v8 wv = expand<T>(now.w[t][j], mask, base);
                    for (int i = 0; i < MT; ++i) part[i] = T::mfma16(wv, xv[i][j], part[i]);
                }
                const float *at = scale + group[p] * (2 * R) + swizzled(group[p], 16 * t + 4 * c);
                const v4f sc = *(const v4f *)at, sz = *(const v4f *)(at + R);
                for (int i = 0; i < MT; ++i)
                    for (int e = 0; e < 4; ++e) acc[t][i][e] = fmaf(sc[e], part[i][e], fmaf(-sz[e], sum[i][p], acc[t][i][e]));
            }
    };
    for (int g0 = 0; g0 < a.groups; g0 += SEG) {
        const int n_groups = min(SEG, a.groups - g0), last = (min(a.K, (g0 + n_groups) * a.group) + 127) >> 7;     // (SEG groups are whole steps)
        int step = ((g0 * a.group) >> 7) + wave;
        Stage even, odd;
        load(min(step, last - 1) << 7, even);
        if (g0 > 0) __syncthreads();
        for (int row = wave; row < R; row += waves) {
            const E *scales = GATED && row >= 16 * OUT ? s1 : s0;
            const uint8_t *zeros = GATED && row >= 16 * OUT ? z1 : z0;
            for (int g = lane; g < n_groups; g += 64) {
                const uint32_t i = (uint32_t)min(row % (16 * OUT), a.N - 1 - n0) * (uint32_t)a.groups + g0 + g;
                const float sc = (float)scales[i];
                float *at = scale + g * (2 * R) + swizzled(g, row);
                at[0] = sc;
                at[R] = sc * (float)(16 + (ZEROS ? zeros[i] : 8));
            }
        }
        __syncthreads();
        for (; step < last;) {
            load(min(step + waves, last - 1) << 7, odd);
            use(step << 7, g0, even);
            step += waves;
            if (step >= last) break;
            load(min(step + waves, last - 1) << 7, even);
            use(step << 7, g0, odd);
            step += waves;
        }
    }

    // the waves' parts of 16 rows of y at a time: [wave][row][16 RT outputs, four more to spread the rows over the banks]
    constexpr int kRow = 16 * RT + 4;
    float *red = (float *)lds;
    E *y = (E *)a.y;
    for (int i = 0; i < MT; ++i) {
        __syncthreads();
        for (int t = 0; t < RT; ++t) *(v4f *)(red + (wave * 16 + r) * kRow + 16 * t + 4 * c) = acc[t][i];
        __syncthreads();
        // output n of the tile, that of the second projection at n + 16 OUT; as the formula stands where it is not finite
        auto sum_of = [&](int m, int n, int64_t row) {
            float v = 0;
            for (int k = 0; k < waves; ++k) v += red[(k * 16 + m) * kRow + n];
            const float bias = a.bias ? (float)((const E *)a.bias)[row] : 0.f;
            if (fabsf(v) < INFINITY) return a.bias ? v + bias : v;
            return (float)(plain_output<T>(a, m0 + 16 * i + m, row) + (double)bias);
        };
        for (int e = threadIdx.x; e < 256 * OUT; e += blockDim.x) {
            const int m = e / (16 * OUT), n = e % (16 * OUT);
            if (m0 + 16 * i + m >= a.M || n0 + n >= a.N) continue;
            float v = sum_of(m, n, n0 + n);
            if constexpr (GATED) v = activated(v, a.activation) * sum_of(m, n + 16 * OUT, a.up + n0 + n);
            y[(int64_t)(m0 + 16 * i + m) * a.y_stride + n0 + n] = (E)v;
        }
    }
}

template <class T, int RT, int MT, int PIECES, int ALIGN, bool GATED>
hawq_status launch(const LinearW4Args &all, hipStream_t s) {
    LinearW4Args a = all;
    const int steps = (a.K + 127) / 128, waves = steps < 8 ? steps : 8;
    const int segment = kScaleBytes / (8 * 16 * RT);
    const size_t scales = (size_t)(a.groups < segment ? a.groups : segment) * 16 * RT * 8, sums = (size_t)waves * 16 * (16 * RT + 4) * 4;
    const size_t lds = scales > sums ? scales : sums;
    // as many outputs and rows at a time as a launch holds (more than millions of either)
    constexpr int OUT = GATED ? RT / 2 : RT;
    const int64_t n_most = most_blocks(64 * waves) * (16 * OUT), m_most = kMostAlong * (16 * MT);
    for (int64_t n = 0; n < all.N; n += n_most)
        for (int64_t m = 0; m < all.M; m += m_most) {
            a.N = (int32_t)(all.N - n < n_most ? all.N - n : n_most);
            a.M = (int32_t)(all.M - m < m_most ? all.M - m : m_most);
            a.x = (const uint16_t *)all.x + m * all.x_stride;
            a.w = all.w + n * (all.K >> 1);
            a.scales = (const uint16_t *)all.scales + n * all.groups;
            a.zeros = all.zeros ? all.zeros + n * all.groups : nullptr;
            a.bias = all.bias ? (const uint16_t *)all.bias + n : nullptr;
            a.y = (uint16_t *)all.y + m * all.y_stride + n;
            const dim3 grid((unsigned)(((int64_t)a.N + 16 * OUT - 1) / (16 * OUT)), (unsigned)(((int64_t)a.M + 16 * MT - 1) / (16 * MT)));
            if (a.zeros) linear_w4<T, RT, MT, PIECES, ALIGN, true, GATED><<<grid, 64 * waves, lds, s>>>(a, fast_div((uint32_t)a.group));
            else linear_w4<T, RT, MT, PIECES, ALIGN, false, GATED><<<grid, 64 * waves, lds, s>>>(a, fast_div((uint32_t)a.group));
            const hawq_status st = check_launch();
            if (st != HAWQ_OK) return st;
        }
    return HAWQ_OK;
}

}  // namespace

}  // namespace hawq
