// Linear layer with 4-bit weights and a scale for each group of them, for the few rows of a decoding step.
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
__device__ __forceinline__ double plain_output(const LinearW4Args &a, int m, int n) {
    typedef typename T::elem E;
    const E *x = (const E *)a.x + m * a.x_stride, *s = (const E *)a.scales + (int64_t)n * a.groups;
    const uint8_t *w = a.w + (int64_t)n * (a.K >> 1);
    double v = 0;
    for (int g = 0; g < a.groups; ++g) {
        const int zero = a.zeros ? a.zeros[(int64_t)n * a.groups + g] : 0, end = (int)min((int64_t)(g + 1) * a.group, (int64_t)a.K);
        const double scale = (double)(float)s[g];
        for (int k = g * a.group; k < end; ++k) {
            const int q = w[k >> 1] >> (4 * (k & 1)) & 15;
            v += (double)(float)x[k] * (double)((a.zeros || q < 8 ? q : q - 16) - zero) * scale;
        }
    }
    return v;
}

// RT, MT: 16-output and 16-row tiles of a wave.  PIECES: parts of 128 weights with a scale of their own.  ALIGN: bytes the rows of w
// are read in (16, 4; 1: also x element by element).  ZEROS: unsigned weights with zero points.
template <class T, int RT, int MT, int PIECES, int ALIGN, bool ZEROS>
__global__ __launch_bounds__(512) void linear_w4(LinearW4Args a, FastDiv by_group) {
    typedef typename T::elem E;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, r = lane & 15, c = lane >> 4;
    const int n0 = blockIdx.x * (16 * RT), m0 = blockIdx.y * (16 * MT);
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
        w_row[t] = (uint32_t)min(16 * t + r, a.N - 1 - n0) * (uint32_t)(a.K >> 1);
    }
    for (int i = 0; i < MT; ++i) x_row[i] = min(16 * i + r, a.M - 1 - m0) * (decltype(x_row[0] + 0))a.x_stride;
    const uint8_t *w0 = a.w + first * (a.K >> 1), *z0 = ZEROS ? a.zeros + first * a.groups : nullptr;
    const E *s0 = (const E *)a.scales + first * a.groups, *x0 = (const E *)a.x + (int64_t)m0 * a.x_stride;

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
            if constexpr (ALIGN == 16) {
                g.w[t] = *(const v4u *)(w0 + (w_row[t] + (uint32_t)(min(kw, a.K - 32) >> 1)));
            } else if constexpr (ALIGN == 4) {
                for (int j = 0; j < 4; ++j) g.w[t][j] = *(const uint32_t *)(w0 + (w_row[t] + (uint32_t)(min(kw + 8 * j, a.K - 8) >> 1)));
            } else {
                for (int j = 0; j < 4; ++j) {
                    uint32_t d = 0;
                    for (int i = 0; i < 4; ++i) d |= (uint32_t)w0[w_row[t] + (uint32_t)(min(kw + 8 * j + 2 * i, a.K - 2) >> 1)] << (8 * i);
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
        for (int row = wave; row < R; row += waves)
            for (int g = lane; g < n_groups; g += 64) {
                const uint32_t i = (uint32_t)min(row, a.N - 1 - n0) * (uint32_t)a.groups + g0 + g;
                const float sc = (float)s0[i];
                float *at = scale + g * (2 * R) + swizzled(g, row);
                at[0] = sc;
                at[R] = sc * (float)(16 + (ZEROS ? z0[i] : 8));
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
        for (int e = threadIdx.x; e < 256 * RT; e += blockDim.x) {
            const int m = e / (16 * RT), n = e % (16 * RT);
            float v = 0;
            for (int k = 0; k < waves; ++k) v += red[(k * 16 + m) * kRow + n];
            if (m0 + 16 * i + m < a.M && n0 + n < a.N) {
                const float bias = a.bias ? (float)((const E *)a.bias)[n0 + n] : 0.f;
                if (fabsf(v) < INFINITY) v = a.bias ? v + bias : v;
                else v = (float)(plain_output<T>(a, m0 + 16 * i + m, n0 + n) + (double)bias);
                y[(int64_t)(m0 + 16 * i + m) * a.y_stride + n0 + n] = (E)v;
            }
        }
    }
}

template <class T, int RT, int MT, int PIECES, int ALIGN>
hawq_status launch(const LinearW4Args &all, hipStream_t s) {
    LinearW4Args a = all;
    const int steps = (a.K + 127) / 128, waves = steps < 8 ? steps : 8;
    const int segment = kScaleBytes / (8 * 16 * RT);
    const size_t scales = (size_t)(a.groups < segment ? a.groups : segment) * 16 * RT * 8, sums = (size_t)waves * 16 * (16 * RT + 4) * 4;
    const size_t lds = scales > sums ? scales : sums;
    // as many outputs and rows at a time as a launch holds (more than millions of either)
    const int64_t n_most = most_blocks(64 * waves) * (16 * RT), m_most = kMostAlong * (16 * MT);
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
            const dim3 grid((unsigned)(((int64_t)a.N + 16 * RT - 1) / (16 * RT)), (unsigned)(((int64_t)a.M + 16 * MT - 1) / (16 * MT)));
            if (a.zeros) linear_w4<T, RT, MT, PIECES, ALIGN, true><<<grid, 64 * waves, lds, s>>>(a, fast_div((uint32_t)a.group));
            else linear_w4<T, RT, MT, PIECES, ALIGN, false><<<grid, 64 * waves, lds, s>>>(a, fast_div((uint32_t)a.group));
            const hawq_status st = check_launch();
            if (st != HAWQ_OK) return st;
        }
    return HAWQ_OK;
}

// Tiles of a workgroup: a larger one reads x fewer times and has more to do for every 128 weights, and what does not come out even
// over the 256 compute units waits for its last round.  The times are those of a workgroup alone on its unit (K = 4096, groups of 128,
// us; the smaller forms leave room for a second one, which the rounds do not count); times the rounds they order the measured ones right, as for 30 rows of 4096 outputs 13.4 / 10.5 / 14.6 (16, 32, 64 outputs, 16
// rows) and 13.5 / 18.3 (32, 64 outputs, 32 rows), for 64 rows of 8192 (K = 8192) 81 / 53 / 42, 41 / 31 and 45 (64 outputs, 64 rows).
struct Tiles { int rt, mt; float us; };
constexpr Tiles kTiles[] = {{1, 1, 8.0f}, {2, 1, 10.0f}, {4, 1, 14.5f}, {2, 2, 13.5f}, {4, 2, 18.3f}, {4, 4, 27.5f}};

// the best of the forms whose bit is set in `forms`
int best_tiles(const LinearW4Args &a, unsigned forms) {
    int best = -1;
    double least = 0;
    for (int i = 0; i < 6; ++i) {
        if (!(forms >> i & 1)) continue;
        const Tiles &t = kTiles[i];
        const int64_t blocks = ((int64_t)a.N + 16 * t.rt - 1) / (16 * t.rt) * (((int64_t)a.M + 16 * t.mt - 1) / (16 * t.mt));
        const double us = t.us * (double)((blocks + 255) / 256);
        if (best < 0 || us < least) best = i, least = us;
    }
    return best;
}

template <class T, int PIECES, int ALIGN>
hawq_status pick_tiles(const LinearW4Args &a, hipStream_t s) {
    // Rows of w that are not read in whole vectors have the first and the fourth form only.  Read in 4 bytes they go by the best of all six,
    // its rows at least (8192 outputs of K = 4104: 13 rows 14.1 us in the first form, 15.7 in the fourth), element by element, where
    // x costs more, by the better of the two (K = 4096: 72 and 57).
    const int best = best_tiles(a, ALIGN == 1 ? 0x09 : 0x3f);
    if constexpr (ALIGN == 16) {
        if (best == 1) return launch<T, 2, 1, PIECES, ALIGN>(a, s);
        if (best == 2) return launch<T, 4, 1, PIECES, ALIGN>(a, s);
        if (best == 4) return launch<T, 4, 2, PIECES, ALIGN>(a, s);
        if (best == 5) return launch<T, 4, 4, PIECES, ALIGN>(a, s);
    }
    return best >= 3 ? launch<T, 2, 2, PIECES, ALIGN>(a, s) : launch<T, 1, 1, PIECES, ALIGN>(a, s);
}

template <class T, int ALIGN>
hawq_status pick_pieces(const LinearW4Args &a, hipStream_t s) {
    return a.group % 128 == 0 ? pick_tiles<T, 1, ALIGN>(a, s) : a.group % 64 == 0 ? pick_tiles<T, 2, ALIGN>(a, s) : pick_tiles<T, 4, ALIGN>(a, s);
}

template <class T>
hawq_status pick_align(const LinearW4Args &a, hipStream_t s) {
    const bool x16 = ((uintptr_t)a.x & 15) == 0 && a.x_stride % 8 == 0 && a.x_stride < (1 << 25);      // (32-bit offsets inside 64 rows)
    if (x16 && a.K % 32 == 0 && ((uintptr_t)a.w & 15) == 0) return pick_pieces<T, 16>(a, s);
    if (x16 && a.K % 8 == 0 && ((uintptr_t)a.w & 3) == 0) return pick_pieces<T, 4>(a, s);
    return pick_pieces<T, 1>(a, s);
}

}  // namespace

hawq_status launch_linear_w4(const LinearW4Args &a, hipStream_t s) { return a.dtype == HAWQ_F16 ? pick_align<F16>(a, s) : pick_align<BF16>(a, s); }

}  // namespace hawq
