// Low-rank adapters of the rows' own beside a projection that all rows share.
//
//   y[m,n] = base[m,n] + s_i * sum_j b[i,n,j] h[m,j],   h[m,j] = sum_k a[i,j,k] x[m,k],   i = adapter[m]
//
// Two launches, a product each, both on the matrix cores: the inner one reads x once and shares K out to workgroups where there are few
// rows (their parts of h lie in the workspace, in 32 bits), the outer one adds the parts up and passes over base and y.  A tile of rows is
// taken once for every adapter that occurs in it, and a column of the product is kept where the row has that adapter: rows of any order are
// served, and those of one adapter share its reading as far as they lie in one tile.
//
// h stays at 32 bits' worth: the matrix instruction takes 16-bit operands, so h goes in as two parts, hi = T(h) and lo = T(h - hi), which
// hold 2^-18 of it (bf16) or 2^-22 (f16, after a power of two for each row that brings its largest to 2^13: a half neither overflows nor
// loses lo's last bits there).  The second product costs nothing beside the bytes of y.  A sum that the two parts leave infinite or no number is
// taken once more from h itself, by its own lane (5003 rows of NaN 0.5 ms, of infinities 1.3).
//
// Few rows are bound by two launches and the loads' latency (one row of 768 x 256 7.7 us, 48 rows of 6144 x 4096 over twelve adapters 15), many
// by bytes on their way: 5003 rows of 4096 x 4096 take 55 us from the caches and 70 to 74 from memory, the inner product 26 of them (47 MB; a lane
// has 312 registers, 332 where elements are read one by one, so that a compute unit has four waves; what lies past K is put to zero where it is
// loaded, so that a step's loads have landed before the products of the step in front of it end) and the outer one 31 (120 MB, 3.9 TB/s, 32 MB of
// them the inner sums' parts, one read after the other by every XCD; a tile's outputs on one XCD read fewer and took 33).
#include "lm.h"
#include "lm_launch.h"

namespace hawq {

namespace {

constexpr int kSteps = 64;                       // k of a step
// Waves that share K out in a workgroup of the inner product: more leave fewer parts to add up (48 rows over twelve adapters 15.1 us with 8, 16.9
// with 4), and a wave of 64 rows has registers for few beside it (5003 rows: 69 and 60).
constexpr int waves_of(int mt) { return mt == 1 ? 8 : 4; }
constexpr int kRanks = 128;                      // ranks of the outer product that are staged at once

struct Plan {
    int mt, slots, splits;                       // 16-row tiles of a workgroup, its grid's share of the adapters of a tile, parts of K
};

// the row's adapter, -1: none, or one without ranks
__device__ __forceinline__ int rank_of(const AdaptersArgs &a, int i) { return min(max(a.ranks[i], 0), a.max_rank); }
__device__ __forceinline__ int adapter_of(const AdaptersArgs &a, int m, int *rank) {
    const int i = a.adapter[m], r = i >= 0 && i < a.n_adapters ? rank_of(a, i) : 0;
    *rank = r;
    return r > 0 ? i : -1;
}

// f(adapter, rank, rows) for the slot's share of what occurs in the tile's rows (bit m: row m0 + m); none: also for rows without one, as -1.
// Every lane of every wave of the workgroup gets the same.
template <int MT, class F>
__device__ __forceinline__ void each_adapter(const AdaptersArgs &a, int m0, int slot, int slots, bool none, F &&f) {
    const int lane = threadIdx.x & 63, n = min(16 * MT, a.M - m0);
    int rank = 0, mine = -2;
    if (lane < n) mine = adapter_of(a, m0 + lane, &rank);
    uint64_t left = __ballot(none ? mine >= -1 : mine >= 0);
    for (int at = 0; left; ++at) {
        const int first = __builtin_ctzll(left), id = __builtin_amdgcn_readlane(mine, first);
        const uint64_t rows = __ballot(mine == id);
        left &= ~rows;
        if (at % slots == slot) f(id, __builtin_amdgcn_readlane(rank, first), rows);
    }
}

// eight elements from k on, zero from K on
template <class T, bool VECTOR>
__device__ __forceinline__ typename T::v8 load8(const typename T::elem *p, int k, int K) {
    if constexpr (VECTOR) {
        v4u d = *(const v4u *)(p + min(k, K - 8));
        if (k >= K) d = v4u{0, 0, 0, 0};
        return __builtin_bit_cast(typename T::v8, d);
    } else {
        const uint16_t *u = (const uint16_t *)p;
        v4u d;
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = u[min(k + 2 * i, K - 1)], hi = u[min(k + 2 * i + 1, K - 1)];
            d[i] = (k + 2 * i < K ? lo : 0) | (k + 2 * i + 1 < K ? hi << 16 : 0);
        }
        return __builtin_bit_cast(typename T::v8, d);
    }
}

// Ranks rb .. rb + 16 NT - 1 of the rows' inner sums over the workgroup's part of K.
template <class T, int MT, int NT, bool VECTOR>
__device__ __forceinline__ void inner_tile(const AdaptersArgs &a, int m0, int id, int rank, int rb, uint64_t rows, int first, int sharers, float *h, float *red) {
    typedef typename T::elem E;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, c = lane >> 4;
    const E *x[MT], *row[NT];
    for (int i = 0; i < MT; ++i) x[i] = (const E *)a.x + min(m0 + 16 * i + r, a.M - 1) * a.x_stride;
    for (int t = 0; t < NT; ++t) row[t] = (const E *)a.a + id * a.a_adapter + min(rb + 16 * t + r, rank - 1) * a.a_row;
    v4f acc[MT][NT];
    for (int i = 0; i < MT; ++i)
        for (int t = 0; t < NT; ++t) acc[i][t] = v4f{0, 0, 0, 0};
    struct Stage {
        typename T::v8 x[MT][2], a[NT][2];
    };
    auto load = [&](int step, Stage &g) {
        for (int s = 0; s < 2; ++s) {
            const int k = step * kSteps + 32 * s + 8 * c;
            for (int i = 0; i < MT; ++i) g.x[i][s] = load8<T, VECTOR>(x[i], k, a.K);
            for (int t = 0; t < NT; ++t) g.a[t][s] = load8<T, VECTOR>(row[t], k, a.K);
        }
    };
    auto use = [&](const Stage &g) {
        for (int s = 0; s < 2; ++s)
            for (int i = 0; i < MT; ++i)
                for (int t = 0; t < NT; ++t) acc[i][t] = T::mfma16(g.a[t][s], g.x[i][s], acc[i][t]);
    };
    // (a wave's steps side by side: 55 us for 5003 rows over four adapters, one apart from the next by all waves 57)
    const int all = (a.K + kSteps - 1) / kSteps, each = (all + sharers - 1) / sharers;
    const int64_t begin = (int64_t)(first + wave) * each;
    if (begin < all) {
        int step = (int)begin;
        const int last = min(all, step + each);
        Stage even, odd;
        load(step, even);
        for (;;) {
            load(min(step + 1, last - 1), odd);
            use(even);
            if (++step >= last) break;
            load(min(step + 1, last - 1), even);
            use(odd);
            if (++step >= last) break;
        }
    }
    constexpr int kRow = 16 * NT + 4;
    __syncthreads();
    for (int i = 0; i < MT; ++i)
        for (int t = 0; t < NT; ++t) *(v4f *)(red + ((wave * MT + i) * 16 + r) * kRow + 16 * t + 4 * c) = acc[i][t];
    __syncthreads();
    for (int e = threadIdx.x; e < 64 * NT * MT; e += 64 * waves_of(MT)) {
        const int m = e / (4 * NT), j = e % (4 * NT) * 4;
        v4f v{0, 0, 0, 0};
        for (int w = 0; w < waves_of(MT); ++w) v += *(const v4f *)(red + (w * MT * 16 + m) * kRow + j);
        if (rows >> m & 1)
            for (int f = 0; f < 4; ++f)
                if (rb + j + f < rank) h[(int64_t)(m0 + m) * a.max_rank + rb + j + f] = v[f];
    }
}

template <class T, int MT, bool VECTOR>
__global__ __launch_bounds__(64 * waves_of(MT)) void inner(AdaptersArgs a, int slots, int splits) {
    __shared__ __align__(16) float red[waves_of(MT) * MT * 16 * 68];
    const int64_t tile = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (tile * (16 * MT) >= a.M) return;
    const int m0 = (int)tile * (16 * MT), slot = blockIdx.z % slots, split = blockIdx.z / slots;
    float *h = a.h + (int64_t)split * a.M * a.max_rank;
    each_adapter<MT>(a, m0, slot, slots, false, [&](int id, int rank, uint64_t rows) {
        for (int rb = 0; rb < rank; rb += 64) {
            const int tiles = (rank - rb + 15) / 16;
            if (tiles == 1) inner_tile<T, MT, 1, VECTOR>(a, m0, id, rank, rb, rows, waves_of(MT) * split, waves_of(MT) * splits, h, red);
            else if (tiles == 2) inner_tile<T, MT, 2, VECTOR>(a, m0, id, rank, rb, rows, waves_of(MT) * split, waves_of(MT) * splits, h, red);
            else inner_tile<T, MT, 4, VECTOR>(a, m0, id, rank, rb, rows, waves_of(MT) * split, waves_of(MT) * splits, h, red);
        }
    });
}

// A sum over the ranks as the formula stands.  That of the two parts of h differs from it where b is infinite (the second part may be 0, or of
// the other sign), and where h is a number of 32 bits that rounds to an infinite one of the type.
template <class T>
__device__ __forceinline__ float plain_outer(const AdaptersArgs &a, int m, const typename T::elem *b, int rank, int splits) {
    double v = 0;
#pragma unroll 1
    for (int j = 0; j < rank && v == v; ++j) {      // (no number stays none)
        const float *p = a.h + (int64_t)m * a.max_rank + j;
        float h = 0;
        for (int s = 0; s < splits; ++s) h += p[(int64_t)s * a.M * a.max_rank];
        v += (double)(float)b[j] * (double)h;
    }
    return (float)v;
}

// 64 outputs of a wave at a time: tile t of its product has outputs n0 + 16 c + 4 t + e where the instruction has rows 4 c + e, so that a lane
// ends with 16 outputs that lie side by side.
template <class T, int MT, bool VECTOR, bool ROWS>
__global__ __launch_bounds__(256) void outer(AdaptersArgs a, int slots, int splits, int chunks, int along, int passes, bool copy) {
    typedef typename T::elem E;
    constexpr int kRow = kRanks + 8;
    __shared__ __align__(16) E parts[2][16 * MT][kRow];
    __shared__ float unit[16 * MT];                     // the power of two that a row's h was divided by
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, c = lane >> 4;
    const int64_t tile = (int64_t)blockIdx.y * along + blockIdx.x / chunks;
    if (tile * (16 * MT) >= a.M) return;
    const int m0 = (int)tile * (16 * MT), chunk = blockIdx.x % chunks;
    // of this thread: a row of h, and which eighths of it
    constexpr int kSub = 256 / (16 * MT);
    const int sm = threadIdx.x / kSub, sub = threadIdx.x % kSub;
    const float *h_row = a.h + (int64_t)min(m0 + sm, a.M - 1) * a.max_rank;
    auto inner_sums = [&](int j, int rank, float (&v)[8]) {
        for (int e = 0; e < 8; ++e) v[e] = 0;
        for (int s = 0; s < splits; ++s) {
            const float *p = h_row + (int64_t)s * a.M * a.max_rank + j;
            if constexpr (VECTOR) {
                const v4f lo = *(const v4f *)p, hi = *(const v4f *)(p + 4);
                for (int e = 0; e < 4; ++e) v[e] += lo[e], v[4 + e] += hi[e];
            } else {
                for (int e = 0; e < 8; ++e) v[e] += p[min(e, rank - 1 - j)];
            }
        }
        for (int e = 0; e < 8; ++e)
            if (j + e >= rank) v[e] = 0;
    };
    each_adapter<MT>(a, m0, blockIdx.z, slots, copy, [&](int id, int rank, uint64_t rows) {
        const bool mine = rows >> sm & 1;
        float down = 1.f;
        if (std::is_same<T, F16>::value && id >= 0) {
            float top = 0;
            for (int j = 8 * sub; mine && j < rank; j += 8 * kSub) {
                float v[8];
                inner_sums(j, rank, v);
                for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]) < INFINITY ? fabsf(v[e]) : 0.f);
            }
            for (int d = kSub >> 1; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
            const int p = min(max((int)(__builtin_bit_cast(uint32_t, top) >> 23) - 127 - 13, -100), 114);
            down = __builtin_bit_cast(float, (uint32_t)(127 - p) << 23);
            __syncthreads();
            if (sub == 0) unit[sm] = __builtin_bit_cast(float, (uint32_t)(127 + p) << 23);
        }
        const float scale = id >= 0 ? a.scales[id] : 0.f;
        const E *b = (const E *)a.b + (int64_t)max(id, 0) * a.b_adapter;
        for (int p = 0; p < passes; ++p) {
            const int n0 = ((chunk * passes + p) * 4 + wave) * 64;
            const int n = n0 + 16 * c;
            typename T::v8 ahead[ROWS ? MT : 1][2];      // base, on its way under the products
            if (ROWS)
                for (int i = 0; i < MT; ++i)
                    for (int q = 0; q < 2; ++q)
                        if (n + 16 <= a.N && (rows >> (16 * i + r) & 1)) ahead[i][q] = *(const typename T::v8 *)((const E *)a.base + (m0 + 16 * i + r) * a.base_stride + n + 8 * q);
            v4f acc[MT][4];
            for (int i = 0; i < MT; ++i)
                for (int t = 0; t < 4; ++t) acc[i][t] = v4f{0, 0, 0, 0};
            for (int j0 = 0; j0 < rank; j0 += kRanks) {
                if (p == 0 || rank > kRanks) {
                    __syncthreads();
                    for (int j = 8 * sub; j < min(rank - j0 + 31 & ~31, kRanks); j += 8 * kSub) {
                        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                        if (mine && j0 + j < rank) inner_sums(j0 + j, rank, v);
                        typename T::v8 hi, lo;
                        for (int e = 0; e < 8; ++e) {
                            const float d = v[e] * down;
                            hi[e] = (E)d;
                            lo[e] = fabsf((float)hi[e]) < INFINITY ? (E)(d - (float)hi[e]) : (E)0.f;
                        }
                        *(typename T::v8 *)&parts[0][sm][j] = hi;
                        *(typename T::v8 *)&parts[1][sm][j] = lo;
                    }
                    __syncthreads();
                }
                if (n0 >= a.N) continue;
                for (int s = 0; s < min((rank - j0 + 31) / 32, kRanks / 32); ++s) {
                    typename T::v8 bv[4];
                    for (int t = 0; t < 4; ++t) {
                        const E *row = b + min(n0 + 16 * (r >> 2) + 4 * t + (r & 3), a.N - 1) * a.b_row;
                        const int j = j0 + 32 * s + 8 * c;
                        if constexpr (VECTOR) {
                            v4u d = *(const v4u *)(row + min(j, a.max_rank - 8));
                            if (j + 8 > rank)
                                for (int e = 0; e < 4; ++e) d[e] = j + 2 * e + 1 < rank ? d[e] : j + 2 * e < rank ? d[e] & 0xffffu : 0u;
                            bv[t] = __builtin_bit_cast(typename T::v8, d);
                        } else {
                            bv[t] = load8<T, false>(row, j, rank);
                        }
                    }
                    for (int i = 0; i < MT; ++i)
                        for (int part = 0; part < 2; ++part) {
                            const typename T::v8 hv = *(const typename T::v8 *)&parts[part][16 * i + r][32 * s + 8 * c];
                            for (int t = 0; t < 4; ++t) acc[i][t] = T::mfma16(bv[t], hv, acc[i][t]);
                        }
                }
            }
            if (n >= a.N) continue;
            for (int i = 0; i < MT; ++i) {
                const int m = m0 + 16 * i + r;
                if (!(rows >> (16 * i + r) & 1)) continue;
                float none = 0;                          // 0, or no number where a sum is not finite
                for (int t = 0; t < 4; ++t)
                    for (int e = 0; e < 4; ++e) none = fmaf(acc[i][t][e], 0.f, none);
                const E *base = (const E *)a.base + m * a.base_stride + n;
                E *y = (E *)a.y + m * a.y_stride + n;
                const float up = std::is_same<T, F16>::value && id >= 0 ? unit[16 * i + r] : 1.f;
                auto sum = [&](E v, float add) { return id >= 0 ? (E)((float)v + scale * add * up) : v; };
                if (ROWS && n + 16 <= a.N && none == 0) {
                    for (int q = 0; q < 2; ++q) {
                        typename T::v8 v = ahead[ROWS ? i : 0][q];
                        for (int e = 0; e < 8; ++e) v[e] = sum(v[e], acc[i][2 * q + (e >> 2)][e & 3]);
                        *(typename T::v8 *)(y + 8 * q) = v;
                    }
                } else {
                    for (int e = 0; e < min(16, a.N - n); ++e) {
                        float add = 0;
                        for (int t = 0; t < 4; ++t)
                            for (int f = 0; f < 4; ++f) add = e == 4 * t + f ? acc[i][t][f] : add;
                        if (!(fabsf(add) < INFINITY)) add = plain_outer<T>(a, m, b + (n + e) * a.b_row, rank, splits) / up;
                        y[e] = sum(base[e], add);
                    }
                }
            }
        }
    });
}

Plan plan(const AdaptersArgs &a) {
    Plan p;
    // A tile of 64 rows reads an adapter a fourth as often and is taken once for all that occur in it, one of 16 has more beside it (4096 x 4096,
    // us, 16 and 64 rows: one adapter of rank 64 at a time 29 and 43 for 600 rows, 56 and 60 for 2500, 89 and 70 for 5000; of rank 16 mixed
    // 48 and 75, 85 and 95)
    p.mt = a.M >= 4096 ? 4 : 1;
    const int64_t tiles = ((int64_t)a.M + 16 * p.mt - 1) / (16 * p.mt), each = waves_of(p.mt) * kSteps, steps = (a.K + each - 1) / each;
    p.slots = p.mt == 4 ? 1 : a.n_adapters < 16 ? (a.n_adapters > 0 ? a.n_adapters : 1) : 16;
    const int64_t wanted = (p.mt == 1 ? 256 : 512) / (tiles * (p.slots < 4 ? p.slots : 4)), most = steps < 16 ? steps : 16;
    p.splits = (int)(wanted < 1 ? 1 : wanted < most ? wanted : most);
    return p;
}

template <class T, int MT>
hawq_status launch(const AdaptersArgs &a, const Plan &p, hipStream_t s) {
    const int64_t tiles = ((int64_t)a.M + 16 * MT - 1) / (16 * MT);
    const auto eights = [](int64_t strides, uintptr_t pointers) { return strides % 8 == 0 && pointers % 16 == 0; };
    if (a.n_adapters > 0) {
        const Grid g = spread(tiles, 1, 64 * waves_of(MT));
        if (g.x == 0) return HAWQ_ERR_UNSUPPORTED;
        const dim3 grid((unsigned)g.x, (unsigned)g.y, (unsigned)(p.slots * p.splits));
        if (eights(a.K | a.x_stride | a.a_adapter | a.a_row, (uintptr_t)a.x | (uintptr_t)a.a)) inner<T, MT, true><<<grid, 64 * waves_of(MT), 0, s>>>(a, p.slots, p.splits);
        else inner<T, MT, false><<<grid, 64 * waves_of(MT), 0, s>>>(a, p.slots, p.splits);
        const hawq_status st = check_launch();
        if (st != HAWQ_OK) return st;
    }
    const bool copy = a.y != a.base;
    const int slots = MT == 4 ? 1 : p.slots + 1;
    // outputs of a workgroup: 256 at a time, more where there are workgroups enough
    int passes = 1;
    while (passes < 8 && tiles * slots * (((int64_t)a.N + 512 * passes - 1) / (512 * passes)) >= 512) passes *= 2;
    const int64_t chunks = ((int64_t)a.N + 256 * passes - 1) / (256 * passes);
    const Grid g = spread(tiles, chunks, 256);
    if (g.x == 0) return HAWQ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)g.x, (unsigned)g.y, (unsigned)slots);
    const bool vector = eights(a.max_rank | a.b_adapter | a.b_row, (uintptr_t)a.b), rows = eights(a.base_stride | a.y_stride, (uintptr_t)a.base | (uintptr_t)a.y);
    const int along = (int)(g.x / chunks);
    if (vector && rows) outer<T, MT, true, true><<<grid, 256, 0, s>>>(a, slots, p.splits, (int)chunks, along, passes, copy);
    else if (vector) outer<T, MT, true, false><<<grid, 256, 0, s>>>(a, slots, p.splits, (int)chunks, along, passes, copy);
    else outer<T, MT, false, false><<<grid, 256, 0, s>>>(a, slots, p.splits, (int)chunks, along, passes, copy);
    return check_launch();
}

}  // namespace

size_t adapters_workspace(const AdaptersArgs &a) { return ((size_t)a.M * a.max_rank * 4 * plan(a).splits + 15) & ~(size_t)15; }

hawq_status launch_adapters(const AdaptersArgs &a, hipStream_t s) {
    const Plan p = plan(a);
    if (a.dtype == HAWQ_F16) return p.mt == 4 ? launch<F16, 4>(a, p, s) : launch<F16, 1>(a, p, s);
    return p.mt == 4 ? launch<BF16, 4>(a, p, s) : launch<BF16, 1>(a, p, s);
}

}  // namespace hawq
