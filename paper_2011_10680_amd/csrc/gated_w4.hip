// The first half of a gated feed-forward block from 4-bit weights, act(x Wg^T) * (x Wu^T): for few rows the linear layer's kernel with both
// projections in a workgroup (linear_w4.h), for whole prompts the kernel below.
//
// Prompt kernel.  A workgroup of eight waves takes 128 rows and 128 outputs, a wave 64 rows and the 32 + 32 columns of its outputs' two
// projections, so that gate and second projection of an output meet in one lane and only their product is stored.  As in linear_w4.h a
// weight is 16 + nibble in the mantissa of a 16-bit float, and a group's part is scaled in 32 bits:
//   g[m,n] = sum_g s[n,g] * ( sum_k x[m,k] u[n,k] )  -  sum_g ( s[n,g] (16 + z[n,g]) ) * ( sum_{k in g} x[m,k] )
// The second term is a matrix product with the groups as its axis: the sums of x (a launch of their own leaves them in the workspace) as
// three bf16 parts, 24 bits, and s (16 + z), which has 16 bits at most, as two, five products of parts for a group, 16 to an instruction's two
// groups.  It costs the matrix pipe a sixteenth (groups of 128) to a quarter (32); subtracted by the vector pipe it would cost that as much as the scaling.
// It is taken off first, for 64 groups at a time, so that a running sum is as large as it and rounds to 2^-24 of that: with x of mean 3 and spread 1 the sums
// are off by 8 10^-6 (K = 4096, groups of 128), 1.6 10^-5 (groups of 32) or 2 10^-5 (K = 65536) of their size, where the form for few rows has 3 to 5 10^-7;
// under the rounding of the type, 2^-11 or 2^-8.  Group by group it would need the sums of x beside the steps' tiles in LDS, which are 146 of 160 KB.
//
// x comes into LDS by direct loads, 64 inputs at a time in four arrays in turn, weights 128 inputs at a time in two; pieces are swizzled so that
// the operand reads are free of bank conflicts.  Two exchanges between a wave's halves give each operand register eight consecutive inputs.  The
// two waves of a SIMD run half a step apart, so that one reads and expands (vector pipe) while the other multiplies (matrix pipe).
//
// Bound by the two pipes: 2049 rows of 8192 x 4096 (bf16, groups of 128, zero points) take 273 us, 1010 TFLOP/s, of which the sums of x are 5 and
// the last row's launch 13; the matrix pipe works half of the kernel's time, the vector pipe 0.57.  A library's bf16 product of 8192 cubed reaches
// 1210 to 1485 here.  On the way: the form for few rows 1297 us, a tile of 128 x 128 541, three steps under way and scales in LDS 385, wider
// tiles of a wave and a group of 128 scaled once 366, waves in turn 313, the last row by the form for few 273.
// 13 rows of 12288 x 4096 take 17.6 us (55 MB of codes, scales and zero points: 10.7 at the rate of a large copy).
#include "linear_w4.h"

namespace hawq {

namespace {

constexpr int kRows = 128, kOuts = 128, kStep = 64, kThreads = 512;
// Of the prompt kernel: a row's sums in LDS, 32-bit offsets, a launch of all tiles of rows.
constexpr int kMostInputs = 1 << 16, kMostXStride = 1 << 22, kMostTall = 1 << 29;

// v as three bf16 parts, each the one below its rest's (towards zero), and the operand {1, 1, 2, 2, 3, 0, 0, 0} of them
__device__ __forceinline__ v4u three_parts(float v) {
    const uint32_t a = __float_as_uint(v) & 0xFFFF0000u;
    const float r = v - __uint_as_float(a);
    const uint32_t b = __float_as_uint(r) & 0xFFFF0000u, c = __float_as_uint(r - __uint_as_float(b)) & 0xFFFF0000u;
    return v4u{a | a >> 16, b | b >> 16, c >> 16, 0u};
}
// {1, 2, 1, 2, 1, 0, 0, 0} of two parts
__device__ __forceinline__ v4u two_parts(float v) {
    const uint32_t a = __float_as_uint(v) & 0xFFFF0000u, b = __float_as_uint(v - __uint_as_float(a)) & 0xFFFF0000u;
    return v4u{a >> 16 | b, a >> 16 | b, a >> 16, 0u};
}

// sums of x over the groups of a row, in parts: [M][groups] of 16 bytes
template <class T>
__global__ __launch_bounds__(256) void group_sums(LinearW4Args a) {
    typedef typename T::elem E;
    __shared__ float piece[kMostInputs / 32];
    const int64_t m = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (m >= a.M) return;
    const E *x = (const E *)a.x + m * a.x_stride;
    for (int k = 8 * threadIdx.x; k < ((a.K + 511) & ~511); k += 2048) {       // (whole waves: lanes past the end add zero)
        float v = 0;
        if (k < a.K) {
            const typename T::v8 d = *(const typename T::v8 *)(x + k);
            for (int e = 0; e < 8; ++e) v += (float)d[e];
        }
        v += __shfl_xor(v, 1);
        v += __shfl_xor(v, 2);
        if ((threadIdx.x & 3) == 0 && k < a.K) piece[k >> 5] = v;
    }
    __syncthreads();
    v4u *out = (v4u *)a.sums + m * a.groups;
    for (int g = threadIdx.x; g < a.groups; g += 256) {
        float v = 0;
        for (int p = g * (a.group >> 5); p < min((g + 1) * (a.group >> 5), a.K >> 5); ++p) v += piece[p];
        out[g] = three_parts(v);
    }
}

// Operand of eight weights in their order: byte i holds two, and a product with 2^a + 2^b puts them where the mantissas are.
template <class T>
__device__ __forceinline__ typename T::v8 expand_in_order(uint32_t d, uint32_t mask, uint32_t base) {
    constexpr uint32_t by = std::is_same<T, F16>::value ? 0x40040u : 0x8008u;
    v4u r;
    for (int i = 0; i < 4; ++i) r[i] = (__umul24(d >> (8 * i) & 255u, by) & mask) ^ base;
    return __builtin_bit_cast(typename T::v8, r);
}

constexpr int kBlock = 2 * kStep, kGroups = 64;  // inputs whose weights are fetched together; groups whose scales are in LDS at once
constexpr int kSide = 4;                         // row tiles side by side in the order of the tiles

// Scales and zero points of a workgroup's columns: rows of 33 and 17 words, so that a column's scale and its neighbours' lie in different
// banks.  unread: a direct load goes there once, since the compiler has a read of LDS that no direct load has written to wait for all that
// are under way, and the scales' would wait for the next steps' x.
template <class E, bool ZEROS>
struct Side {
    E scale[2 * kOuts][kGroups + 2];
    uint8_t zero[ZEROS ? 2 * kOuts : 1][kGroups + 4];
    uint32_t unread[64];
};

// PARTS: how often a group's part of 128 inputs is scaled: 1, 2 or 4 times, for groups of multiples of 128, 64 and 32
template <class T, int PARTS, bool ZEROS>
__global__ __launch_bounds__(kThreads, 2) void gated_prompt(LinearW4Args a, FastDiv by_group, int m_tiles, int tiles, int first_n) {
    typedef typename T::elem E;
    __shared__ __align__(1024) char x0[kRows * kStep * 2], x1[kRows * kStep * 2], x2[kRows * kStep * 2], x3[kRows * kStep * 2], w0[kOuts * kBlock], w1[kOuts * kBlock];
    __shared__ __align__(16) Side<E, ZEROS> lds;
    auto &scale = lds.scale;
    auto &zero = lds.zero;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    // An XCD's workgroups at one time are some tiles of rows by some of outputs: 4 by 8 read 4 MB of x and 4 of w, 16 by 2 would read 17.
    const int id = (int)xcd_remap(blockIdx.x, tiles), set = id / (kSide * (tiles / m_tiles)), in_set = id - set * kSide * (tiles / m_tiles), side = min(kSide, m_tiles - set * kSide);
    const int m0 = (set * kSide + in_set % side) * kRows, n0 = first_n + in_set / side * kOuts;
    const int wm = (wave >> 2) * 64, wn = (wave & 3) * 32, n = min(n0 + wn + col, a.N - 1);
    uint32_t mask = Nibbles<T>::mask, base = Nibbles<T>::base ^ (ZEROS ? 0u : Nibbles<T>::sign);
    asm("" : "+s"(mask));
    asm("" : "+v"(base));
    // row of w, scales, zeros of column c of the workgroup, the second projection's behind the gate's
    auto row_of = [&](int c) { return min(n0 + (c & (kOuts - 1)), a.N - 1) + (c >= kOuts ? a.up : 0); };

    // Direct loads, a kilobyte of a wave at a time.  x: lane -> a row and a piece of 16 bytes; piece p of row r lies at p ^ (r / 2 & 7), so that
    // 16 rows' reads meet every bank once.  Weights of a block: lane -> a column and a piece of its 64 bytes, piece p of column c at p ^ (c / 4 & 3).
    const int x_row = wave * 8 + (lane >> 3), x_piece = (lane & 7) ^ (x_row >> 1 & 7);
    const uint32_t x_off = (uint32_t)x_row * (uint32_t)a.x_stride * 2 + x_piece * 16;
    const int rows = min(kRows, a.M - m0);
    const E *x = (const E *)a.x + (int64_t)m0 * a.x_stride;
    auto fetch_x = [&](int k, char *to) {        // (rows and inputs past the last: zeros)
        const int k0 = min(k, a.K - 32);
        const __amdgpu_buffer_rsrc_t rx = scalar_rsrc(x + k0, (uint32_t)(((rows - 1) * a.x_stride + a.K - k0) * 2));
        const uint32_t off = k + 8 * x_piece < a.K ? x_off : 0x80000000u;
        for (int i = 0; i < 2; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (__attribute__((address_space(3))) void *)(to + i * 8192 + wave * 1024), 16, (int)(off + (uint32_t)(i * 64) * (uint32_t)a.x_stride * 2), 0, 0, 0);
    };
    const int last_c = min(kOuts, a.N - n0) - 1, w_row = a.K >> 1, w_col = wave * 32 + (lane >> 2) & (kOuts - 1);      // (a wave's 32 columns are of one projection)
    const uint8_t *w = a.w + (n0 + (wave >= 4 ? a.up : 0)) * w_row;
    const int w_piece = (lane & 3) ^ (lane >> 4 & 3);
    auto fetch_w = [&](int k, char *to) {        // (columns past the last: the last one's; inputs past the last: whatever there is)
        const int k0 = min(k, a.K - 32);
        const __amdgpu_buffer_rsrc_t rw = scalar_rsrc(w + (k0 >> 1), (uint32_t)(last_c * w_row + w_row - (k0 >> 1)));
        for (int i = 0; i < 2; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (__attribute__((address_space(3))) void *)(to + wave * 2048 + i * 1024), 16,
                                                     (int)((uint32_t)min(w_col + 16 * i, last_c) * (uint32_t)w_row + 16 * w_piece), 0, 0, 0);
    };

    v16f acc[2][2];                              // [rows][projection]
    for (int i = 0; i < 2; ++i)
        for (int t = 0; t < 2; ++t)
            for (int e = 0; e < 16; ++e) acc[i][t][e] = 0;
    int x_at[4];                                 // operand reads: pieces 2 half + (0, 1) of the row's first and second 32 inputs
    for (int p = 0; p < 4; ++p) x_at[p] = (wm + col) * 128 + (((4 * (p >> 1) + 2 * half + (p & 1)) ^ (col >> 1 & 7)) << 4);
    int w_at[2];                                 // pieces half and 2 + half of the column's 64 bytes
    for (int s = 0; s < 2; ++s) w_at[s] = (wn + col) * 64 + (((2 * s + half) ^ (col >> 2 & 3)) << 4);
    // Operands of the 64 inputs from k on, the first or second of a block's two steps, and their products.
    constexpr int PIECES = PARTS == 4 ? 2 : 1;
    typename T::v8 wv[2][4], xv[2][4];
    float sc[2][PIECES];
    v16f part[2][2];
    auto read = [&](auto second, int k, int g0, const char *xs, const char *ws) {
        v4u d[2];
        for (int t = 0; t < 2; ++t) d[t] = *(const v4u *)(ws + w_at[decltype(second)::value] + t * kOuts * 64);
        for (int p = 0; p < PIECES; ++p) {
            const int g = (int)fdiv((uint32_t)min(k + 32 * p, a.K - 1), by_group) - g0;
            for (int t = 0; t < 2; ++t) sc[t][p] = (float)scale[t * kOuts + wn + col][g];
        }
        for (int i = 0; i < 2; ++i)
            for (int p = 0; p < 4; ++p) xv[i][p] = *(const typename T::v8 *)(xs + x_at[p] + i * 32 * 128);
        for (int t = 0; t < 2; ++t) {
            const v2u u = __builtin_amdgcn_permlane32_swap(d[t].x, d[t].z, false, false), v = __builtin_amdgcn_permlane32_swap(d[t].y, d[t].w, false, false);
            wv[t][0] = expand_in_order<T>(u.x, mask, base);
            wv[t][1] = expand_in_order<T>(v.x, mask, base);
            wv[t][2] = expand_in_order<T>(u.y, mask, base);
            wv[t][3] = expand_in_order<T>(v.y, mask, base);
        }
    };
    auto multiply = [&](auto second) {
        constexpr bool kSecond = decltype(second)::value;
        for (int t = 0; t < 2; ++t)
            for (int p = 0; p < PIECES; ++p)
                for (int i = 0; i < 2; ++i) {
                    v16f &sum = part[i][t];
                    if (PARTS > 1 || !kSecond)
                        for (int e = 0; e < 16; ++e) sum[e] = 0;
                    for (int j = p * 4 / PIECES; j < (p + 1) * 4 / PIECES; ++j) sum = T::mfma32(xv[i][j], wv[t][j], sum);
                    if (PARTS > 1 || kSecond)
                        for (int e = 0; e < 16; ++e) acc[i][t][e] = fmaf(sc[t][p], sum[e], acc[i][t][e]);
                }
    };
    // No more than so many loads under way, and LDS done with; LDS alone.  (Instructions that the compiler counts with, and a line that nothing
    // in memory crosses.)
    auto wait_for = [](auto loads) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(decltype(loads)::value | 0x70);
        asm volatile("" ::: "memory");
    };
    auto wait_lds = [] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xC07F);
        asm volatile("" ::: "memory");
    };
    for (int g0 = 0; g0 < a.groups; g0 += kGroups) {
        const int n_groups = min(kGroups, a.groups - g0), first = g0 * a.group, last = (int)min((int64_t)first + (int64_t)n_groups * a.group, (int64_t)a.K);
        const int blocks = (last - first + kBlock - 1) / kBlock;
        __syncthreads();
        // The second term, sixteen groups at a time: their sums in the places of a step's x and a block's weights that are not needed yet, eight
        // groups to a row of 128 bytes.
        for (int q0 = 0; q0 < n_groups; q0 += 32) {
            v4u in[8];                           // of 32 groups
            for (int i = 0; i < 8; ++i) {
                const int r = x_row + 64 * (i & 1), g = g0 + q0 + 8 * (i >> 1) + x_piece;
                in[i] = ((const v4u *)a.sums)[(int64_t)min(m0 + r, a.M - 1) * a.groups + min(g, a.groups - 1)];
                if (g >= a.groups) in[i] = v4u{0, 0, 0, 0};
            }
            // a thread brings sixteen scales and zero points of a column to LDS
            const int c = threadIdx.x >> 1, g1 = q0 + 16 * (threadIdx.x & 1);
            const int64_t row = row_of(c) * a.groups + g0;
            if (q0 + 32 <= n_groups) {
                typedef uint32_t at2 __attribute__((ext_vector_type(4), aligned(2)));
                typedef uint32_t at1 __attribute__((ext_vector_type(4), aligned(1)));
                const v4u lo = *(const at2 *)((const E *)a.scales + row + g1), hi = *(const at2 *)((const E *)a.scales + row + g1 + 8);
                v4u z{0, 0, 0, 0};
                if (ZEROS) z = *(const at1 *)(a.zeros + row + g1);
                for (int e = 0; e < 4; ++e) {
                    ((uint32_t *)&scale[c][g1])[e] = lo[e];
                    ((uint32_t *)&scale[c][g1])[4 + e] = hi[e];
                    if (ZEROS) ((uint32_t *)&zero[c][g1])[e] = z[e];
                }
            } else {
                for (int e = 0; e < 16; ++e) scale[c][g1 + e] = ((const E *)a.scales)[row + min(g1 + e, n_groups - 1)];
                if (ZEROS)
                    for (int e = 0; e < 16; ++e) zero[c][g1 + e] = a.zeros[row + min(g1 + e, n_groups - 1)];
            }
            auto bring = [&](const v4u *sums) {
                for (int i = 0; i < 4; ++i) *(v4u *)((i < 2 ? x3 : w1) + (i & 1) * 8192 + threadIdx.x * 16) = sums[i];
            };
            bring(in);
            if (q0 == 0) {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(scalar_rsrc(w, 4), (__attribute__((address_space(3))) void *)lds.unread, 4, 0, 0, 0, 0);
                fetch_w(first, w0);
                fetch_x(first, x0);
                fetch_x(first + kStep, x1);
                fetch_x(first + kBlock, x2);
            }
            auto subtract = [&](int g1, const char *from) {
                for (int q = 0; q < 4; ++q) {
                    const int g = g1 + 2 * q + half;
                    BF16::v8 xs[2], ws[2];
                    for (int i = 0; i < 2; ++i) xs[i] = *(const BF16::v8 *)(from + (wm + 32 * i + col) * 128 + (((2 * q + half) ^ (col >> 1 & 7)) << 4));
                    for (int t = 0; t < 2; ++t) {
                        const int c = t * kOuts + wn + col;
                        ws[t] = __builtin_bit_cast(BF16::v8, two_parts(-(float)scale[c][g] * (float)(16 + (ZEROS ? zero[c][g] : 8))));
                    }
                    for (int i = 0; i < 2; ++i)
                        for (int t = 0; t < 2; ++t) acc[i][t] = BF16::mfma32(xs[i], ws[t], acc[i][t]);
                }
            };
            for (int s = 0; s < 32 && q0 + s < n_groups; s += 16) {
                if (s > 0) bring(in + 4);
                wait_lds();
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                subtract(q0 + s, x3);
                if (q0 + s + 8 < n_groups) subtract(q0 + s + 8, w1);
                wait_lds();
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }
        }
        wait_for(std::integral_constant<int, 4>());
        __builtin_amdgcn_s_barrier();            // (w0 and x0 have landed)
        asm volatile("" ::: "memory");
        // Steps of 64 inputs, x three steps ahead and the weights of a block two.  The two waves of a SIMD take turns, half a step apart: while
        // one reads and expands its operands the other multiplies.  Before the second barrier of a step a wave's loads for the next one have
        // landed: no more than those behind them are under way.  What is fetched takes the place of what all waves have read.  (Past the end
        // zeros are fetched: with loads in a branch the compiler would wait for all of them.)
        auto turn = [&](auto allowed, auto second, int k, const char *xs, const char *ws, char *x_to, char *w_to) {
            __builtin_amdgcn_s_barrier();        // (__syncthreads would wait for all loads)
            asm volatile("" ::: "memory");
            if (!decltype(second)::value) fetch_w(k + kBlock, w_to);
            fetch_x(k + 3 * kStep, x_to);
            __builtin_amdgcn_sched_barrier(0);   // (else they are put off to the products' end)
            read(second, k, g0, xs, ws);
            __builtin_amdgcn_sched_barrier(0);
            wait_for(allowed);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_setprio(1);
            multiply(second);
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
        };
        typedef std::integral_constant<int, 4> Four;
        typedef std::integral_constant<int, 6> Six;
        if (wave >= 4) __builtin_amdgcn_s_barrier();
        for (int k = first; k < last; k += 2 * kBlock) {
            turn(Six(), std::false_type(), k, x0, w0, x3, w1);
            turn(Four(), std::true_type(), k + kStep, x1, w0, x0, nullptr);
            if (k + kBlock >= last) break;
            turn(Six(), std::false_type(), k + kBlock, x2, w1, x1, w0);
            turn(Four(), std::true_type(), k + kBlock + kStep, x3, w1, x2, nullptr);
        }
        if (wave < 4) __builtin_amdgcn_s_barrier();
        wait_for(std::integral_constant<int, 0>());
    }

    const bool inside = n0 + wn + col < a.N;
    float bias[2] = {0, 0};
    if (a.bias)
        for (int t = 0; t < 2; ++t) bias[t] = (float)((const E *)a.bias)[n + t * a.up];
    uint32_t bad = 0;
    auto finish = [&](auto act) {
        for (int i = 0; i < 2; ++i)
            for (int e = 0; e < 16; ++e) {
                const int m = m0 + wm + 32 * i + 8 * (e >> 2) + 4 * half + (e & 3);
                const float g = acc[i][0][e], u = acc[i][1][e];
                if (inside && m < a.M) {
                    if (!(fabsf(g) < INFINITY) || !(fabsf(u) < INFINITY)) bad |= 1u << (16 * i + e);
                    ((E *)a.y)[m * a.y_stride + n] = (E)(act(g + bias[0]) * (u + bias[1]));
                }
            }
    };
    if (a.activation == HAWQ_SILU) finish([](float v) { return activated(v, HAWQ_SILU); });
    else if (a.activation == HAWQ_GELU) finish([](float v) { return activated(v, HAWQ_GELU); });
    else if (a.activation == HAWQ_GELU_TANH) finish([](float v) { return activated(v, HAWQ_GELU_TANH); });
    else finish([](float v) { return activated(v, HAWQ_RELU); });
    for (; bad; bad &= bad - 1) {                // as the formula stands where a sum is not finite
        const int b = __builtin_ctz(bad), e = b & 15, m = m0 + wm + 32 * (b >> 4) + 8 * (e >> 2) + 4 * half + (e & 3);
        float v[2];
        for (int t = 0; t < 2; ++t) v[t] = (float)(plain_output<T>(a, m, n + t * a.up) + (double)bias[t]);
        ((E *)a.y)[m * a.y_stride + n] = (E)(activated(v[0], a.activation) * v[1]);
    }
}

// Time of a form in us: `at` for the launch, `in` for every 4096 inputs of the first workgroups, one to each of the 256 compute units, and `more` and
// `begin` for every 256 after them.  Fitted to 150 calls of 1 to 800 rows, 512 to 16384 outputs and 256 to 11008 inputs, in groups of 128
// (off by a sixteenth at the median): the form chosen by it took 1.02 times the best one's time in the mean, 1.2 times at most.  Larger forms
// begin whole rounds, small ones share a unit.
struct Form { int rows, outputs; float at, in, more, begin; bool rounds; };
constexpr Form kForms[] = {{16, 16, 5.6f, 3.6f, 6.1f, 1.2f, false}, {16, 32, 7.9f, 5.9f, 10.1f, 3.2f, false}, {32, 16, 6.2f, 5.8f, 8.6f, 1.0f, false},
                           {32, 32, 9.1f, 8.0f, 13.3f, 4.0f, true}, {64, 32, 11.1f, 11.9f, 21.6f, 4.4f, true}};
constexpr Form kPrompt = {kRows, kOuts, 13.2f, 46.9f, 49.7f, 12.0f, true};
constexpr float kScaledTwice = 1.25f, kScaledFour = 1.6f;      // groups of 64 and 32 (8192 x 4096, 256 rows: 63, 74 and 99 us)
float time_of(const Form &f, const LinearW4Args &a) {
    const int64_t blocks = ((int64_t)a.N + f.outputs - 1) / f.outputs * (((int64_t)a.M + f.rows - 1) / f.rows);
    const float k = (float)a.K / 4096.f, rounds = f.rounds ? (float)((blocks + 255) / 256) : (float)blocks / 256.f;
    return f.at + f.in * k + (rounds > 1 ? rounds - 1 : 0.f) * (f.more * k + f.begin);
}
// the best of the forms whose bit is set; up to 16 rows the first (one row of 12288 outputs 16.5 us, the second 22.4)
int best_form(const LinearW4Args &a, unsigned forms) {
    int best = 0;
    if (a.M > 16)
        for (int i = 1; i < 5; ++i)
            if ((forms >> i & 1) && time_of(kForms[i], a) < time_of(kForms[best], a)) best = i;
    return best;
}

template <class T, int PIECES, int ALIGN>
hawq_status pick_tiles(const LinearW4Args &a, hipStream_t s) {
    const int best = best_form(a, ALIGN == 16 ? 0x1f : 0x05);
    if constexpr (ALIGN == 16) {
        if (best == 1) return launch<T, 4, 1, PIECES, ALIGN, true>(a, s);
        if (best == 3) return launch<T, 4, 2, PIECES, ALIGN, true>(a, s);
        if (best == 4) return launch<T, 4, 4, PIECES, ALIGN, true>(a, s);
    }
    return best == 2 ? launch<T, 2, 2, PIECES, ALIGN, true>(a, s) : launch<T, 2, 1, PIECES, ALIGN, true>(a, s);
}

template <class T, int ALIGN>
hawq_status pick_pieces(const LinearW4Args &a, hipStream_t s) {
    return a.group % 128 == 0 ? pick_tiles<T, 1, ALIGN>(a, s) : a.group % 64 == 0 ? pick_tiles<T, 2, ALIGN>(a, s) : pick_tiles<T, 4, ALIGN>(a, s);
}

template <class T>
hawq_status few_rows(const LinearW4Args &a, hipStream_t s) {
    const bool x16 = ((uintptr_t)a.x & 15) == 0 && a.x_stride % 8 == 0 && a.x_stride < (1 << 25);      // (32-bit offsets inside 64 rows)
    if (x16 && a.K % 32 == 0 && ((uintptr_t)a.w & 15) == 0) return pick_pieces<T, 16>(a, s);
    if (x16 && a.K % 8 == 0 && ((uintptr_t)a.w & 3) == 0) return pick_pieces<T, 4>(a, s);
    return pick_pieces<T, 1>(a, s);
}

// What the prompt kernel takes by its sizes (the workspace goes by them alone), and by its addresses.
bool prompt_sized(const LinearW4Args &a) {
    if (a.M <= 16 || a.M > kMostTall || a.K > kMostInputs || a.x_stride > kMostXStride || a.K % 32 != 0 || a.x_stride % 8 != 0) return false;
    const float more = a.group % 128 == 0 ? 1.f : a.group % 64 == 0 ? kScaledTwice : kScaledFour;
    return more * time_of(kPrompt, a) < time_of(kForms[best_form(a, 0x1f)], a);
}
bool prompt_placed(const LinearW4Args &a) { return ((uintptr_t)a.x & 15) == 0 && ((uintptr_t)a.w & 15) == 0; }

template <class T>
hawq_status prompt(const LinearW4Args &all, hipStream_t s) {
    LinearW4Args a = all;
    // Rows past the last whole tile, up to 16, go by the form for few where their tiles would begin another round of the 256 compute units.
    const int64_t n_tiles = ((int64_t)a.N + kOuts - 1) / kOuts, rest = a.M % kRows;
    const auto rounds = [&](int64_t m_tiles) { return (m_tiles * n_tiles + 255) / 256; };
    if (rest > 0 && rest <= 16 && rounds(a.M / kRows + 1) > rounds(a.M / kRows)) a.M -= (int32_t)rest;
    const Grid rows = spread(a.M, 1, 256);
    group_sums<T><<<dim3((unsigned)rows.x, (unsigned)rows.y), 256, 0, s>>>(a);
    hawq_status st = check_launch();
    if (st != HAWQ_OK) return st;
    const int64_t m_tiles = ((int64_t)a.M + kRows - 1) / kRows, at_once = most_blocks(kThreads) / m_tiles;
    const FastDiv by_group = fast_div((uint32_t)a.group);
    for (int64_t n = 0; n < n_tiles; n += at_once) {                     // as many outputs as a launch holds
        const int tiles = (int)(m_tiles * (n_tiles - n < at_once ? n_tiles - n : at_once)), first_n = (int)n * kOuts;
        const auto go = [&](auto parts) {
            constexpr int PARTS = decltype(parts)::value;
            if (a.zeros) gated_prompt<T, PARTS, true><<<dim3((unsigned)tiles), kThreads, 0, s>>>(a, by_group, (int)m_tiles, tiles, first_n);
            else gated_prompt<T, PARTS, false><<<dim3((unsigned)tiles), kThreads, 0, s>>>(a, by_group, (int)m_tiles, tiles, first_n);
        };
        if (a.group % 128 == 0) go(std::integral_constant<int, 1>());
        else if (a.group % 64 == 0) go(std::integral_constant<int, 2>());
        else go(std::integral_constant<int, 4>());
        st = check_launch();
        if (st != HAWQ_OK) return st;
    }
    if (a.M == all.M) return HAWQ_OK;
    LinearW4Args last = all;
    last.M = all.M - a.M;
    last.x = (const uint16_t *)all.x + (int64_t)a.M * a.x_stride;
    last.y = (uint16_t *)all.y + (int64_t)a.M * a.y_stride;
    return few_rows<T>(last, s);
}

}  // namespace

size_t gated_w4_workspace(const LinearW4Args &a) { return prompt_sized(a) ? (size_t)a.M * a.groups * 16 : 0; }

hawq_status launch_gated_w4(const LinearW4Args &a, hipStream_t s) {
    if (prompt_sized(a) && prompt_placed(a)) return a.dtype == HAWQ_F16 ? prompt<F16>(a, s) : prompt<BF16>(a, s);
    return a.dtype == HAWQ_F16 ? few_rows<F16>(a, s) : few_rows<BF16>(a, s);
}

}  // namespace hawq
