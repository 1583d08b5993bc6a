// The first half of a gated feed-forward block from 4-bit weights, act(x Wg^T) * (x Wu^T): for few rows the linear layer's kernel with both
// projections in a workgroup (linear_w4.h), for whole prompts the kernel below.
//
// Prompt kernel.  A workgroup of four waves takes 128 rows and 64 outputs, a wave 64 rows and the 32 + 32 columns of its outputs' two
// projections, so that gate and second projection of an output meet in one lane and only their product is stored.  As in linear_w4.h a
// weight is 16 + nibble in the mantissa of a 16-bit float, and a group's part is scaled in 32 bits:
//   g[m,n] = sum_g s[n,g] * ( sum_k x[m,k] u[n,k] )  -  sum_g ( s[n,g] (16 + z[n,g]) ) * ( sum_{k in g} x[m,k] )
// The second term is a matrix product with the groups as its axis: the sums of x (a launch of their own leaves them in the workspace) as
// three bf16 parts, 24 bits, and s (16 + z), which has 16 bits at most, as two, five products of parts for a group, 16 to an instruction's two
// groups.  It costs the matrix pipe a sixteenth (groups of 128) to a quarter (32); subtracted by the vector pipe it would cost that as much as the scaling.
//
// x comes into LDS by direct loads, 64 inputs at a time in two arrays in turn, pieces swizzled by the row so that the operand reads are free
// of bank conflicts; weights go from memory to the wave's registers, 16 bytes a lane, and two exchanges between the wave's halves give each
// operand register eight consecutive inputs.
#include "linear_w4.h"

namespace hawq {

namespace {

constexpr int kRows = 128, kOuts = 64, kStep = 64;
constexpr int kMostInputs = 1 << 16, kMostXStride = 1 << 22;       // of the prompt kernel: 32-bit offsets, a row's sums in LDS

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

constexpr int kStage = (kRows * 2 + 2 * kOuts / 2) * kStep, kGroups = 64;      // bytes of x and w of a step; groups whose scales are in LDS at once

// PIECES: groups of 32 inputs (2) or of multiples of 64 (1)
template <class T, int PIECES, bool ZEROS>
__global__ __launch_bounds__(256, 2) void gated_prompt(LinearW4Args a, FastDiv by_group, int m_tiles, int tiles, int first_n) {
    typedef typename T::elem E;
    __shared__ __align__(1024) char stage0[kStage], stage1[kStage], stage2[kStage];
    __shared__ __align__(16) E scale[kGroups][2 * kOuts];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const int id = (int)xcd_remap(blockIdx.x, tiles), m0 = id % m_tiles * kRows, n0 = first_n + id / m_tiles * kOuts;
    const int wm = (wave >> 1) * 64, wn = (wave & 1) * 32, n = min(n0 + wn + col, a.N - 1);
    uint32_t mask = Nibbles<T>::mask, base = Nibbles<T>::base ^ (ZEROS ? 0u : Nibbles<T>::sign);
    asm("" : "+s"(mask));
    asm("" : "+v"(base));
    // row of w, scales, zeros of column c of the workgroup, the second projection's behind the gate's
    auto row_of = [&](int c) { return min(n0 + (c & (kOuts - 1)), a.N - 1) + (c >= kOuts ? a.up : 0); };

    // direct loads of x: lane -> a row and a piece of 16 bytes of the wave's kilobyte; piece p of row r lies at p ^ (r & 7).  Of w: 16 bytes of
    // a column's 32.
    const int lrow = wave * 8 + (lane >> 3), lpiece = (lane & 7) ^ (lrow & 7);
    const uint32_t x_off = (uint32_t)lrow * (uint32_t)a.x_stride * 2 + lpiece * 16;
    const int rows = min(kRows, a.M - m0);
    const E *x = (const E *)a.x + (int64_t)m0 * a.x_stride;
    const int first_c = wave * 32 & (kOuts - 1), last_c = min(kOuts, a.N - n0) - 1, w_row = a.K >> 1;      // (a wave's 32 columns are of one projection)
    const uint8_t *w = a.w + (n0 + (wave >= 2 ? a.up : 0)) * w_row;
    const uint32_t w_off = (uint32_t)min(first_c + (lane >> 1), last_c) * (uint32_t)w_row + 16 * (lane & 1);
    constexpr int kLoads = 5;                    // of a wave for a step
    auto fetch = [&](int k0, char *to) {
        const __amdgpu_buffer_rsrc_t rx = scalar_rsrc(x + k0, (uint32_t)(((rows - 1) * a.x_stride + a.K - k0) * 2));      // (rows past the last: zeros)
        const uint32_t off = k0 + 8 * lpiece < a.K ? x_off : 0x80000000u;
        for (int i = 0; i < 4; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (__attribute__((address_space(3))) void *)(to + i * 4096 + wave * 1024), 16, (int)(off + (uint32_t)(i * 32) * (uint32_t)a.x_stride * 2), 0, 0, 0);
        const __amdgpu_buffer_rsrc_t rw = scalar_rsrc(w + (k0 >> 1), (uint32_t)(last_c * w_row + w_row - (k0 >> 1)));
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (__attribute__((address_space(3))) void *)(to + kRows * kStep * 2 + wave * 1024), 16, (int)w_off, 0, 0, 0);
    };

    v16f acc[2][2];                              // [rows][projection]
    for (int i = 0; i < 2; ++i)
        for (int t = 0; t < 2; ++t)
            for (int e = 0; e < 16; ++e) acc[i][t][e] = 0;
    {
        const v4u *sums[2];
        for (int i = 0; i < 2; ++i) sums[i] = (const v4u *)a.sums + (int64_t)min(m0 + wm + 32 * i + col, a.M - 1) * a.groups;
        const E *s[2];
        const uint8_t *z[2] = {nullptr, nullptr};
        for (int t = 0; t < 2; ++t) {
            s[t] = (const E *)a.scales + (n + t * a.up) * a.groups;
            if (ZEROS) z[t] = a.zeros + (n + t * a.up) * a.groups;
        }
        for (int q = 0; q < a.groups; q += 2) {
            const int g = min(q + half, a.groups - 1);
            const uint32_t there = q + half < a.groups ? ~0u : 0u;
            v4u xs[2], ws[2];
            for (int i = 0; i < 2; ++i) xs[i] = sums[i][g] & there;
            for (int t = 0; t < 2; ++t) ws[t] = two_parts(-(float)s[t][g] * (float)(16 + (ZEROS ? z[t][g] : 8))) & there;
            for (int i = 0; i < 2; ++i)
                for (int t = 0; t < 2; ++t) acc[i][t] = BF16::mfma32(__builtin_bit_cast(BF16::v8, xs[i]), __builtin_bit_cast(BF16::v8, ws[t]), acc[i][t]);
        }
    }

    int x_at[4];                                 // operand reads: pieces 2 half + (0, 1) of the row's first and second 32 inputs
    for (int p = 0; p < 4; ++p) x_at[p] = (wm + col) * 128 + (((4 * (p >> 1) + 2 * half + (p & 1)) ^ (col & 7)) << 4);
    const int w_at = kRows * kStep * 2 + (wn + col) * 32 + half * 16;
    auto use = [&](int k0, int g0, const char *at) {
        typename T::v8 wv[2][4], xv[2][4];
        for (int i = 0; i < 2; ++i)
            for (int p = 0; p < 4; ++p) xv[i][p] = *(const typename T::v8 *)(at + x_at[p] + i * 32 * 128);
        float sc[2][PIECES];
        for (int p = 0; p < PIECES; ++p) {
            const int g = (int)fdiv((uint32_t)min(k0 + 32 * p, a.K - 1), by_group) - g0;
            for (int t = 0; t < 2; ++t) sc[t][p] = (float)scale[g][t * kOuts + wn + col];
        }
        for (int t = 0; t < 2; ++t) {
            const v4u d = *(const v4u *)(at + w_at + t * kOuts * 32);
            const v2u u = __builtin_amdgcn_permlane32_swap(d.x, d.z, false, false), v = __builtin_amdgcn_permlane32_swap(d.y, d.w, false, false);
            wv[t][0] = expand_in_order<T>(u.x, mask, base);
            wv[t][1] = expand_in_order<T>(v.x, mask, base);
            wv[t][2] = expand_in_order<T>(u.y, mask, base);
            wv[t][3] = expand_in_order<T>(v.y, mask, base);
        }
        for (int t = 0; t < 2; ++t)
            for (int i = 0; i < 2; ++i)
                for (int p = 0; p < PIECES; ++p) {
                    v16f part;
                    for (int e = 0; e < 16; ++e) part[e] = 0;
                    for (int j = p * 4 / PIECES; j < (p + 1) * 4 / PIECES; ++j) part = T::mfma32(xv[i][j], wv[t][j], part);
                    for (int e = 0; e < 16; ++e) acc[i][t][e] = fmaf(sc[t][p], part[e], acc[i][t][e]);
                }
    };
    for (int g0 = 0; g0 < a.groups; g0 += kGroups) {
        const int n_groups = min(kGroups, a.groups - g0), first = g0 * a.group, last = (int)min((int64_t)first + (int64_t)n_groups * a.group, (int64_t)a.K);
        __syncthreads();
        for (int i = threadIdx.x; i < n_groups * 2 * kOuts; i += 256) {
            const int c = i & (2 * kOuts - 1), g = i / (2 * kOuts);
            scale[g][c] = ((const E *)a.scales)[row_of(c) * a.groups + g0 + g];
        }
        fetch(first, stage0);
        fetch(min(first + kStep, a.K - 32), stage1);
        // Three steps in turn: what the step needs has landed when no more than the next one's loads are under way; the one two ahead then
        // takes the place of the step before, which all waves have left behind.  (Past the end the last inputs are fetched again: with loads in
        // a branch the compiler would wait for all of them.)
        auto turn = [&](int k, const char *now, char *then) {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLoads) : "memory");
            __builtin_amdgcn_s_barrier();        // (__syncthreads would wait for the next step's loads too)
            asm volatile("" ::: "memory");
            fetch(min(k + 2 * kStep, a.K - 32), then);
            use(k, g0, now);
        };
        for (int k = first; k < last; k += 3 * kStep) {
            turn(k, stage0, stage2);
            if (k + kStep >= last) break;
            turn(k + kStep, stage1, stage0);
            if (k + 2 * kStep >= last) break;
            turn(k + 2 * kStep, stage2, stage1);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
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

template <class T>
bool whole_rows(const LinearW4Args &a) { return ((uintptr_t)a.x & 15) == 0 && a.x_stride % 8 == 0 && a.K % 32 == 0 && ((uintptr_t)a.w & 15) == 0; }

bool prompt_sized(const LinearW4Args &a) { return a.M > 128 && a.K <= kMostInputs && a.x_stride <= kMostXStride && a.K % 32 == 0 && a.x_stride % 8 == 0; }

template <class T>
hawq_status launch_prompt(const LinearW4Args &a, hipStream_t s) {
    const Grid rows = spread(a.M, 1, 256);
    group_sums<T><<<dim3((unsigned)rows.x, (unsigned)rows.y), 256, 0, s>>>(a);
    hawq_status st = check_launch();
    if (st != HAWQ_OK) return st;
    const int64_t m_tiles = ((int64_t)a.M + kRows - 1) / kRows, n_tiles = ((int64_t)a.N + kOuts - 1) / kOuts, at_once = most_blocks(256) / m_tiles;
    const FastDiv by_group = fast_div((uint32_t)a.group);
    for (int64_t n = 0; n < n_tiles; n += at_once) {                     // as many outputs as a launch holds
        const int tiles = (int)(m_tiles * (n_tiles - n < at_once ? n_tiles - n : at_once)), first_n = (int)n * kOuts;
        if (a.group % 64 == 0) {
            if (a.zeros) gated_prompt<T, 1, true><<<dim3((unsigned)tiles), 256, 0, s>>>(a, by_group, (int)m_tiles, tiles, first_n);
            else gated_prompt<T, 1, false><<<dim3((unsigned)tiles), 256, 0, s>>>(a, by_group, (int)m_tiles, tiles, first_n);
        } else {
            if (a.zeros) gated_prompt<T, 2, true><<<dim3((unsigned)tiles), 256, 0, s>>>(a, by_group, (int)m_tiles, tiles, first_n);
            else gated_prompt<T, 2, false><<<dim3((unsigned)tiles), 256, 0, s>>>(a, by_group, (int)m_tiles, tiles, first_n);
        }
        st = check_launch();
        if (st != HAWQ_OK) return st;
    }
    return HAWQ_OK;
}

template <class T, int PIECES, int ALIGN>
hawq_status pick_tiles(const LinearW4Args &a, hipStream_t s) {
    return a.M > 16 ? launch<T, 2, 2, PIECES, ALIGN, true>(a, s) : launch<T, 2, 1, PIECES, ALIGN, true>(a, s);
}

template <class T, int ALIGN>
hawq_status pick_pieces(const LinearW4Args &a, hipStream_t s) {
    return a.group % 128 == 0 ? pick_tiles<T, 1, ALIGN>(a, s) : a.group % 64 == 0 ? pick_tiles<T, 2, ALIGN>(a, s) : pick_tiles<T, 4, ALIGN>(a, s);
}

template <class T>
hawq_status pick_align(const LinearW4Args &a, hipStream_t s) {
    if (prompt_sized(a) && whole_rows<T>(a)) return launch_prompt<T>(a, s);
    const bool x16 = ((uintptr_t)a.x & 15) == 0 && a.x_stride % 8 == 0 && a.x_stride < (1 << 25);      // (32-bit offsets inside 64 rows)
    if (x16 && a.K % 32 == 0 && ((uintptr_t)a.w & 15) == 0) return pick_pieces<T, 16>(a, s);
    if (x16 && a.K % 8 == 0 && ((uintptr_t)a.w & 3) == 0) return pick_pieces<T, 4>(a, s);
    return pick_pieces<T, 1>(a, s);
}

}  // namespace

size_t gated_w4_workspace(const LinearW4Args &a) { return prompt_sized(a) ? (size_t)a.M * a.groups * 16 : 0; }

hawq_status launch_gated_w4(const LinearW4Args &a, hipStream_t s) { return a.dtype == HAWQ_F16 ? pick_align<F16>(a, s) : pick_align<BF16>(a, s); }

}  // namespace hawq
