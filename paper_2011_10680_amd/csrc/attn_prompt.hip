// Causal attention over packed prompts: y[i] = sum_{j <= i} p_ij v_j, p = softmax of scale * q_i . k_j, in one pass over the
// keys with a running maximum and sum.
//
// Matrix-core kernel.  A workgroup of four waves takes 128 queries of one head of one sequence, a wave 32 of them.  Scores are
// computed transposed, S^T = K Q^T (keys down the accumulator's registers, a query per lane), so that a query's maximum and
// sum are a lane's own values and one exchange between the wave's halves, and the 16-bit probabilities are, register for
// register, the operand of O^T = V^T P^T: the keys of a register group only come in an order (8 b + 4 half + j) that V^T is
// read in too.  Nothing of S or P passes through LDS.  Keys and values of 64 tokens at a time come into LDS by direct loads,
// two tiles in turn, rows swizzled so that both the row reads of K and the transposing reads of V are free of bank conflicts;
// V^T's operand comes from the transposing LDS read, four keys of one element per lane.
//
// Masked probabilities are exact zeros, but 0 * infinity in V would not be: a row whose result is NaN is computed again by
// the plain path, which leaves unseen values out.  So is a row with scores of millions.
//
// Bound by the matrix and vector pipes together: an exponential, a maximum and a sum for every 256 operations of a 128-element
// head.  32 heads on 8 of 128 elements, bf16, prompts of 8192, 5000 and 8001 tokens: 1.20 ms, 1060 TFLOP/s, matrix pipes busy
// for 0.57 and vector pipes for 0.50 of the time (a large library product of the type reaches 1485); 12 prompts of 1 to 2048
// tokens: 193 us, 745 TFLOP/s, where workgroups live for some ten tiles, their start and end cost a fifth, and keys past the
// diagonal inside a tile an eighth more products.  Half as many workgroups of eight waves, three or four tiles in LDS, a score product
// ahead of the tile before and raised wave priorities measured no faster or slower.
#include "attn_any.h"
#include "lm_launch.h"

namespace hawq {

namespace {

constexpr int kRows = 128, kKeys = 64;

template <class T>
__device__ __forceinline__ KeyRow prompt_key(const AttnPromptArgs &a, int64_t row, int hk) {
    typedef typename T::elem E;
    return {(const E *)a.k + row * a.k_token + hk * a.k_head, (const E *)a.v + row * a.v_token + hk * a.v_head, 1.f, 1.f, false};
}

// any head dimension, stride and alignment: a wave per query
template <class T>
__global__ __launch_bounds__(64) void attn_prompt_any(AttnPromptArgs a) {
    typedef typename T::elem E;
    __shared__ float q_lds[256];
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (id >= (int64_t)a.total * a.q_heads) return;
    const int h = (int)(id / a.total), row = (int)(id - (int64_t)h * a.total), hk = h / (a.q_heads / a.kv_heads);
    int from = 0, to = 0;
    // the sequence that holds the row: the last one that begins at or before it (empty ones in between hold nothing)
    int lo = 0, hi = a.n_seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.starts[mid] <= row) lo = mid; else hi = mid - 1;
    }
    sequence_rows(a.starts, lo, a.total, from, to);
    if (row < from || row >= to) return;
    store_row<T>(attend_row<T>((const E *)a.q + row * a.q_token + h * a.q_head, a.head_dim, a.scale, 0, row - from + 1, q_lds,
                               [&](int j) { return prompt_key<T>(a, from + j, hk); }, [](int) { return true; }),
                 (E *)a.y + row * a.y_token + h * a.y_head, a.head_dim);
}

// The sequence and the 128 queries of tile `tile`.  Every wave looks for itself.
//
// Up to 64 sequences the tiles are in falling order of their place in their sequence, whatever the sequence: the longest rows begin
// first and the last workgroups to begin are the shortest.  A lane holds a sequence's number of tiles; the tiles at place p or
// later number the sum of max(n - p, 0), and bisection finds the place whose tiles include this one.  More sequences are short ones
// in the main: they follow one another, each from its end.
__device__ __forceinline__ bool find_tile(const AttnPromptArgs &a, int tile, int &from, int &to, int &q0) {
    const int lane = threadIdx.x & 63;
    if (a.n_seqs <= 64) {
        int f = 0, t = 0;
        if (lane < a.n_seqs) sequence_rows(a.starts, lane, a.total, f, t);
        const int n = (t - f + kRows - 1) / kRows;
        int lo = 0, hi = max_of_lanes(n);                                   // tiles at place lo or later: more than `tile`; at hi or later: none
        if (sum_of_lanes(n) <= tile) return false;
        int past = 0;                                                       // tiles at place lo + 1 or later
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1, m = sum_of_lanes(max(n - mid, 0));
            if (m > tile) lo = mid; else hi = mid, past = m;
        }
        // of the sequences with a tile at this place, the (tile - past)-th
        uint64_t here = __ballot(n > lo);
        for (int skip = tile - past; skip > 0; --skip) here &= here - 1;
        const int l = __builtin_ctzll(here);
        from = __builtin_amdgcn_readlane(f, l);
        to = __builtin_amdgcn_readlane(t, l);
        q0 = lo * kRows;
        return true;
    }
    int before = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        int f = 0, t = 0;
        if (b0 + lane < a.n_seqs) sequence_rows(a.starts, b0 + lane, a.total, f, t);
        const int n = (t - f + kRows - 1) / kRows;
        const int upto = sum_up_to_lane(n);
        const uint64_t past = __ballot(before + upto > tile);
        if (past) {
            const int l = __builtin_ctzll(past);
            from = __builtin_amdgcn_readlane(f, l);
            to = __builtin_amdgcn_readlane(t, l);
            q0 = (before + __builtin_amdgcn_readlane(upto, l) - 1 - tile) * kRows;
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// DT: 32-element tiles of the head dimension (2: up to 64, LDS rows of 128 bytes; 3, 4: up to 96 and 128, rows of 256)
template <class T, int DT>
__global__ __launch_bounds__(256, 2) void attn_prompt(AttnPromptArgs a, float by_log2e, uint32_t negate) {
    typedef typename T::elem E;
    constexpr int KS = 2 * DT, PITCH = DT == 2 ? 128 : 256, TILE = kKeys * PITCH, LOADS = TILE / 4096;
    __shared__ __align__(1024) char k_even[TILE], v_even[TILE], k_odd[TILE], v_odd[TILE];
    __shared__ float q_lds[4][256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;

    // heads that share keys run on one XCD (workgroups go to the eight in turn), the tiles of all heads side by side
    int h = blockIdx.x % a.q_heads;
    int tile = blockIdx.x / a.q_heads;
    if (blockIdx.y > 0) tile += blockIdx.y * (gridDim.x / a.q_heads);           // (a second division, where there is need of it)
    if (a.q_heads % 8 == 0) h = (h & 7) * (a.q_heads / 8) + (h >> 3);
    const int hk = h / (a.q_heads / a.kv_heads);
    int from, to, q0;
    if (!find_tile(a, tile, from, to, q0)) return;
    from = __builtin_amdgcn_readfirstlane(from);                                // (the same in every lane: the compiler does not see it)
    to = __builtin_amdgcn_readfirstlane(to);
    q0 = __builtin_amdgcn_readfirstlane(q0);
    const int len = to - from, qw = q0 + 32 * wave, q_at = qw + col;            // the wave's first query, this lane's
    const E *kp = (const E *)a.k + from * a.k_token + hk * a.k_head, *vp = (const E *)a.v + from * a.v_token + hk * a.v_head;

    // the swizzle: 16-byte piece c of row r lies at piece c ^ f(r)
    auto f = [](int r) { return PITCH == 256 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r << 1) & 4) | ((r >> 2) & 3); };

    // direct loads: lane -> byte 16 lane of the wave's kilobyte, that is a row and a piece; pieces past the head's elements are zeros
    const int lrow = (wave * 1024 + lane * 16) / PITCH, lpiece = ((lane * 16 % PITCH) >> 4) ^ f(lrow);
    constexpr int kStep = 4096 / PITCH;                                         // rows from one of a wave's loads to its next
    const bool inside = lpiece * 8 < a.head_dim;
    const uint32_t k_off = inside ? (uint32_t)(lrow * a.k_token * 2 + lpiece * 16) : 0x80000000u, v_off = inside ? (uint32_t)(lrow * a.v_token * 2 + lpiece * 16) : 0x80000000u;
    auto fetch = [&](int j0, char *kt, char *vt) {
        const int last = min(kKeys, len - j0) - 1;                              // last row of the tile: what lies past it is zeros
        const __amdgpu_buffer_rsrc_t rk = scalar_rsrc(kp + j0 * a.k_token, (uint32_t)((last * a.k_token + a.head_dim) * 2));
        const __amdgpu_buffer_rsrc_t rv = scalar_rsrc(vp + j0 * a.v_token, (uint32_t)((last * a.v_token + a.head_dim) * 2));
        for (int i = 0; i < LOADS; ++i) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (__attribute__((address_space(3))) void *)(kt + i * 4096 + wave * 1024), 16, (int)(k_off + (uint32_t)(i * kStep * a.k_token * 2)), 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (__attribute__((address_space(3))) void *)(vt + i * 4096 + wave * 1024), 16, (int)(v_off + (uint32_t)(i * kStep * a.v_token * 2)), 0, 0, 0);
        }
    };
    const int n_tiles = (min(len, q0 + kRows) + kKeys - 1) / kKeys;
    fetch(0, k_even, v_even);

    // queries: operand B, 8 elements at 16 s + 8 half of this lane's query (past the last one: the last one's, not stored)
    typename T::v8 q[KS];
    {
        const E *p = (const E *)a.q + (from + min(q_at, len - 1)) * a.q_token + h * a.q_head;
        for (int s = 0; s < KS; ++s) {
            const int d = 16 * s + 8 * half;
            v4u x = d < a.head_dim ? *(const v4u *)(p + d) : v4u{0, 0, 0, 0};
            x ^= negate;
            q[s] = __builtin_bit_cast(typename T::v8, x);
        }
    }

    // addresses of the operand reads inside a tile
    int k_at[KS], v_at[DT][2];
    for (int s = 0; s < KS; ++s) k_at[s] = col * PITCH + (((2 * s + half) ^ f(col)) << 4);
    for (int t = 0; t < DT; ++t)
        for (int b = 0; b < 2; ++b) {
            const int row = 8 * b + 4 * half + ((lane >> 2) & 3), piece = 4 * t + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
            v_at[t][b] = row * PITCH + ((piece ^ f(row)) << 4) + (lane & 1) * 8;
        }

    v16f o[DT];
    for (int t = 0; t < DT; ++t)
        for (int e = 0; e < 16; ++e) o[t][e] = 0;
    float m = -INFINITY, total = 0;      // the maximum the weights refer to (in units of the scores), this half's sum of weights

    auto compute = [&](int j0, const char *kt, const char *vt) {
        if (j0 > qw + 31) return;
        v16f sc[2];
        for (int t = 0; t < 2; ++t)
            for (int e = 0; e < 16; ++e) sc[t][e] = 0;
        // (six of K's operands on their way before the first product, else each waits for its own: 1070 instead of 1045 TFLOP/s)
        __builtin_amdgcn_sched_barrier(0);
        for (int s = 0; s < KS; ++s)
            for (int t = 0; t < 2; ++t) sc[t] = T::mfma32(*(const typename T::v8 *)(kt + k_at[s] + 32 * t * PITCH), q[s], sc[t]);
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
        for (int i = 0; i < 2 * KS - 6; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, 6, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (j0 + kKeys - 1 > qw)
            for (int t = 0; t < 2; ++t)
                for (int e = 0; e < 16; ++e)
                    if (j0 + 32 * t + 8 * (e >> 2) + 4 * half + (e & 3) > q_at) sc[t][e] = -INFINITY;
        float top = -INFINITY;
        for (int t = 0; t < 2; ++t)
            for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[t][e]);
        {
            const v2u x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(x.x), __uint_as_float(x.y));
        }
        // the weights refer to an earlier maximum until one of the wave's queries has outgrown it by 2^8: powers of two cost no
        // precision, and most tiles then leave o alone.  They are rounded to T for the product (its operands are of 16 bits), from 2^lift on
        if (__any(top * by_log2e > m * by_log2e + 8.f)) {
            const float next = fmaxf(m, top), keep = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - next) * by_log2e);
            m = next;
            total *= keep;
            for (int t = 0; t < DT; ++t)
                for (int e = 0; e < 16; ++e) o[t][e] *= keep;
        }
        const float off = m == -INFINITY ? 0.f : fmaf(-m, by_log2e, T::lift);
        for (int t = 0; t < 2; ++t) {
            typename T::v8 p[2];
            float sum;          // (of 16 keys before it meets the total: many small weights one by one would be lost beside a large one)
            for (int e = 0; e < 16; ++e) {
                const float w = __builtin_amdgcn_exp2f(fmaf(sc[t][e], by_log2e, off));
                sum = e == 0 ? w : sum + w;
                p[e >> 3][e & 7] = (E)w;
            }
            total += sum;
            for (int s = 0; s < 2; ++s)
                for (int d = 0; d < DT; ++d) {
                    typedef short v4s __attribute__((ext_vector_type(4)));
                    typedef short v8s __attribute__((ext_vector_type(8)));
                    const char *at = vt + (32 * t + 16 * s) * PITCH;
                    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(at + v_at[d][0]));
                    const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(at + v_at[d][1]));
                    const v8s both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    o[d] = T::mfma32(__builtin_bit_cast(typename T::v8, both), p[s], o[d]);
                }
        }
    };
    for (int j = 0; j < n_tiles; j += 2) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (j + 1 < n_tiles) fetch((j + 1) * kKeys, k_odd, v_odd);
        compute(j * kKeys, k_even, v_even);
        if (j + 1 >= n_tiles) break;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (j + 2 < n_tiles) fetch((j + 2) * kKeys, k_even, v_even);
        compute((j + 1) * kKeys, k_odd, v_odd);
    }

    // the halves hold the elements 8 b + 4 half + j of every 32
    {
        const v2u x = __builtin_amdgcn_permlane32_swap(__float_as_uint(total), __float_as_uint(total), false, false);
        total = __uint_as_float(x.x) + __uint_as_float(x.y);
    }
    const float by = 1.f / total;
    // (a maximum of millions: its own weight is 2 to the power of what rounding it left out, which may be beyond any float)
    bool bad = fabsf(m) * by_log2e > 0x1p22f && m > -INFINITY;
    for (int t = 0; t < DT; ++t)
        for (int e = 0; e < 16; ++e) {
            o[t][e] = total == 0.f ? 0.f : o[t][e] * by;
            bad |= o[t][e] != o[t][e];
        }
    if (q_at < len) {
        E *y = (E *)a.y + (from + q_at) * a.y_token + h * a.y_head;
        for (int t = 0; t < DT; ++t)
            for (int b = 0; b < 4; ++b) {
                const int d = 32 * t + 8 * b + 4 * half;
                if (d < a.head_dim) {
                    typename T::v4 r;
                    for (int e = 0; e < 4; ++e) r[e] = (E)o[t][4 * b + e];
                    *(typename T::v4 *)(y + d) = r;
                }
            }
    }
    const uint64_t lanes = __ballot(bad && q_at < len);
    for (uint32_t rows = (uint32_t)lanes | (uint32_t)(lanes >> 32); rows; rows &= rows - 1) {
        const int i = qw + __builtin_ctz(rows);
        const int64_t row = from + i;
        store_row<T>(attend_row<T>((const E *)a.q + row * a.q_token + h * a.q_head, a.head_dim, a.scale, 0, i + 1, q_lds[wave],
                                   [&](int j) { return prompt_key<T>(a, from + j, hk); }, [](int) { return true; }),
                     (E *)a.y + row * a.y_token + h * a.y_head, a.head_dim);
    }
}

// Rows that are read and written in whole vectors, tiles of 64 rows inside 31-bit offsets.
bool matrix_form(const AttnPromptArgs &a) {
    const int64_t loads = a.q_token | a.q_head | a.k_token | a.k_head | a.v_token | a.v_head;
    return a.head_dim % 8 == 0 && a.head_dim <= 128 && loads % 8 == 0 && (a.y_token | a.y_head) % 4 == 0 &&
           (((uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v) & 15) == 0 && ((uintptr_t)a.y & 7) == 0 && a.k_token < (1 << 23) && a.v_token < (1 << 23);
}

template <class T>
hawq_status launch(const AttnPromptArgs &a, hipStream_t s) {
    const int64_t tiles = ((int64_t)a.total + kRows - 1) / kRows + a.n_seqs;
    const Grid g = spread(tiles, a.q_heads, 256);
    if (matrix_form(a) && g.x > 0 && tiles <= INT32_MAX) {
        // q . k times a negative scale is (-q) . k times its magnitude; a scale of 0 is as good as the smallest number
        const float c = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1.2e-38f);
        const uint32_t negate = a.scale < 0 ? 0x80008000u : 0u;
        const dim3 grid((unsigned)g.x, (unsigned)g.y);
        if (a.head_dim <= 64) attn_prompt<T, 2><<<grid, 256, 0, s>>>(a, c, negate);
        else if (a.head_dim <= 96) attn_prompt<T, 3><<<grid, 256, 0, s>>>(a, c, negate);
        else attn_prompt<T, 4><<<grid, 256, 0, s>>>(a, c, negate);
        return check_launch();
    }
    const Grid each = spread((int64_t)a.total * a.q_heads, 1, 64);
    if (each.x == 0) return HAWQ_ERR_UNSUPPORTED;
    attn_prompt_any<T><<<dim3((unsigned)each.x, (unsigned)each.y), 64, 0, s>>>(a);
    return check_launch();
}

}  // namespace

hawq_status launch_attn_prompt(const AttnPromptArgs &a, hipStream_t s) { return a.dtype == HAWQ_F16 ? launch<F16>(a, s) : launch<BF16>(a, s); }

}  // namespace hawq
