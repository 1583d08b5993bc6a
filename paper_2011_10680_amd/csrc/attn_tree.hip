// Attention of drafted tokens over a paged cache and over one another.
//
// Matrix-core kernel.  The rows that share a key head (drafts x heads of the group) are taken 16 or 32 to a workgroup, whose
// waves walk over the cache 32 keys at a time, each wave every W-th of these chunks, and join their running maxima, sums and
// outputs in LDS at the end; a long cache is shared out to several workgroups, whose parts a second launch joins.  As in prompt
// attention the scores are computed transposed, S^T = K Q^T and O^T = V^T P^T: K's operand is read from memory straight into
// registers, P's is the accumulator of S^T as it is, V comes through the wave's own LDS and its transposing read.  Keys are
// looked up in the block table one chunk ahead of their loads, and loaded one chunk ahead of their use.
//
// An 8-bit cache's codes become 16-bit floats exactly; a key's scale multiplies its score.  A value's scale would drive f16
// weights below their range, so its logarithm joins the exponent instead: the stored weight is exp2(s + log2 vs - m) with the
// maximum m taken of that sum, and the sum of weights adds it divided by vs.  (Drafts have no scale: beside one a cached weight is lower by
// its vs, which the 2^7 that halves begin with make up for.)
//
// Bound by the cache's bytes where there are many, by the chain of dependent loads (lengths, table, keys) where there are few.
// 32 heads on 8 of 128 elements, bf16: 32 requests of one token over 500 to 16384 in 8 bits 132 us with the join, 571 MB of codes and
// scales at 4.6 TB/s in the kernel itself; the same in 16 bits 216.  7 requests of 1 to 64 drafts over caches of 0 to 4097 tokens of 16 bits 29 us,
// 5.4 of them the join.  8 heads on one of 64, one token over 611: 8.9 us, three chunks a wave.  (Two chunks on their way instead of one
// measured 139, 34.5 and 9.9: a wave has few chunks, and what it loads beyond them costs more.)
//
// Rows whose result is NaN are computed again by the plain path: 0 times an unseen infinity, a value's scale that is not 0 and below 2^-90.  So are
// rows with scores of thousands (millions over 16 bits).
#include "attn_any.h"
#include "lm_launch.h"

namespace hawq {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// One request and head of keys as a sequence of positions: cached tokens, then from position `pad` on the drafts.
template <class T>
struct TreeKeys {
    typedef typename T::elem E;
    const AttnTreeArgs &a;
    int hk, from, drafts, cached, pad;
    const int32_t *table;

    __device__ __forceinline__ TreeKeys(const AttnTreeArgs &args, int b, int head) : a(args), hk(head) {
        int to;
        sequence_rows(a.starts, b, a.total, from, to);
        drafts = min(to - from, a.max_drafts);
        cached = min(max(a.cached[b], 0), a.max_cached);
        pad = cached;
        table = a.table + (int64_t)b * a.table_stride;
    }
    __device__ __forceinline__ TreeKeys(const AttnTreeArgs &args, const TreeKeys &k) : a(args), hk(k.hk), from(k.from), drafts(k.drafts), cached(k.cached), pad(k.pad), table(k.table) {}
    __device__ __forceinline__ bool on_a_page(int j) const { return (uint32_t)table[fdiv((uint32_t)j, a.cache.by_page)] < (uint32_t)a.cache.n_pages; }
    __device__ __forceinline__ uint64_t mask(int t) const { return a.mask ? a.mask[from + t] : t == 63 ? ~0ull : (2ull << t) - 1; }
    __device__ __forceinline__ KeyRow operator()(int j) const {
        if (j >= pad) {
            const int64_t r = from + j - pad;
            return {(const E *)a.k + r * a.k_token + hk * a.k_head, (const E *)a.v + r * a.v_token + hk * a.v_head, 1.f, 1.f, false};
        }
        const bool codes = a.cache.dtype == HAWQ_S8;
        const int i = (int)fdiv((uint32_t)j, a.cache.by_page), at = j - i * a.cache.page, size = codes ? 1 : 2;
        const int64_t p = table[i], e = p * a.cache.page_stride + at * a.cache.token_stride + hk * a.cache.head_stride;
        const int64_t f = (p * a.cache.page + at) * a.kv_heads + hk;
        return {(const char *)a.cache.k + e * size, (const char *)a.cache.v + e * size, codes ? a.cache.ks[f] : 1.f, codes ? a.cache.vs[f] : 1.f, codes};
    }
    __device__ __forceinline__ bool visible(int j, uint64_t seen) const {
        return j < pad ? j < cached && on_a_page(j) : j - pad < drafts && (seen >> (j - pad) & 1) != 0;
    }
    __device__ __forceinline__ RowSums attend(int t, int h, int begin, int end, float *q_lds) const {
        const uint64_t seen = mask(t);
        return attend_row<T>((const E *)a.q + (int64_t)(from + t) * a.q_token + h * a.q_head, a.head_dim, a.scale, begin, end, q_lds, *this,
                             [&](int j) { return visible(j, seen); });
    }
    __device__ __forceinline__ E *out(int t, int h) const { return (E *)a.y + (int64_t)(from + t) * a.y_token + h * a.y_head; }
};

// any head dimension, stride and alignment: a wave per row
template <class T>
__global__ __launch_bounds__(64) void attn_tree_any(AttnTreeArgs a) {
    __shared__ float q_lds[256];
    const int t = blockIdx.x, h = blockIdx.y;
    const TreeKeys<T> keys(a, blockIdx.z, h / (a.q_heads / a.kv_heads));
    if (t >= keys.drafts) return;
    store_row<T>(keys.attend(t, h, 0, keys.cached + keys.drafts, q_lds), keys.out(t, h), a.head_dim);
}

struct TreePlan {
    int32_t rows;              // rows of a workgroup: 16, 32
    int32_t row_tiles;         // workgroups over a request's rows
    int32_t waves;             // its waves
    int32_t chunks, splits;    // chunks of 32 keys of a workgroup (listed: at least), workgroups over a request's chunks at most
    FastDiv by_group;          // heads of a group
    FastDiv by_heads, by_units;   // heads of keys, these times row tiles
    int32_t listed;            // workgroups take what work there is in turn, else one workgroup for all that might be
    int32_t blocks;
    int64_t parts;             // partial rows there is room for
};

constexpr int kChunk = 32;
constexpr int kPartRows = 32;     // of an item, where the work is listed

TreePlan tree_plan(const AttnTreeArgs &a) {
    TreePlan p;
    const int group = a.q_heads / a.kv_heads;
    const int64_t rows = (int64_t)a.max_drafts * group;
    p.rows = rows <= 16 ? 16 : 32;
    p.row_tiles = (int32_t)((rows + p.rows - 1) / p.rows);
    p.by_group = fast_div((uint32_t)group);
    p.by_heads = fast_div((uint32_t)a.kv_heads);
    p.by_units = fast_div((uint32_t)(a.kv_heads * p.row_tiles));
    const int64_t most = ((int64_t)a.max_cached + kChunk - 1) / kChunk + (a.max_drafts + kChunk - 1) / kChunk, one = (int64_t)a.n_seqs * a.kv_heads * p.row_tiles;
    // caches of up to 1024 tokens are not shared out (no second launch): a workgroup has eight waves where there are few of them
    p.waves = p.rows == 16 && most <= 33 && one <= 256 ? 8 : 4;
    if (most <= 33 && (p.waves == 8 || one >= 256)) {
        p.chunks = (int32_t)most;
        p.splits = 1;
        p.parts = p.listed = 0;
        p.blocks = one > most_blocks(64 * p.waves) ? 0 : (int32_t)one;      // (0: more than a launch holds)
        return p;
    }
    // At least two chunks for a wave.  With 32 rows and up to 64 requests the kernel itself sizes the parts; else enough workgroups for
    // every compute unit some times over, since the requests are of unequal length.
    int64_t chunks = p.rows > 16 && a.n_seqs <= 64 ? 1 : (most * one + 4095) / 4096;
    if (chunks > most) chunks = most;       // (many requests over long caches: past 32 bits)
    chunks = (chunks + p.waves - 1) / p.waves * p.waves;
    p.chunks = (int32_t)(chunks < 2 * p.waves ? 2 * p.waves : chunks);
    p.splits = (int32_t)((most + p.chunks - 1) / p.chunks);
    const int64_t all = one * p.splits, resident = 512;
    p.listed = p.rows > 16 && a.n_seqs <= 64 && all > resident && p.splits > 1;
    p.blocks = p.listed ? (int32_t)resident : all > most_blocks(64 * p.waves) ? 0 : (int32_t)all;
    if (p.blocks == 0) p.splits = 1;
    p.parts = p.splits == 1 ? 0 : p.listed ? resident * kPartRows : (int64_t)a.total * a.q_heads * p.splits;
    return p;
}

// Partial sums: a part of a row is head_dim floats; then for each the maximum (powers of two) and the sum of weights.  Parts lie as
// [row][q head][split], or, listed, as [item][row of the tile]: wherever a request is shared out there are no more items than workgroups,
// so that the room does not grow with the rows and lengths there might be.  A request's items: [row tile][key head][split].
__device__ __forceinline__ float *stats_of(const AttnTreeArgs &a, const TreePlan &p) { return a.partial + p.parts * a.head_dim; }
// behind them, listed: the chunks of a part, then the first item of every request
__device__ __forceinline__ int *list_of(const AttnTreeArgs &a, const TreePlan &p) { return (int *)(stats_of(a, p) + p.parts * 2); }

typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));

// eight codes as T, exactly
template <class T>
__device__ __forceinline__ typename T::v8 from_codes(uint32_t lo, uint32_t hi) {
    typename T::v8 r;
    asm("" : "+v"(lo), "+v"(hi));        // (else the bytes are split where they are loaded, a register each)
    for (int i = 0; i < 4; ++i) {
        r[i] = (typename T::elem)(float)(int8_t)(lo >> (8 * i));
        r[4 + i] = (typename T::elem)(float)(int8_t)(hi >> (8 * i));
    }
    return r;
}

__device__ __forceinline__ float max_of_quarters(float v) {
    v2u x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(x.x), __uint_as_float(x.y));
    x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x.x), __uint_as_float(x.y));
}
__device__ __forceinline__ float sum_of_quarters(float v) {
    v2u x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(x.x) + __uint_as_float(x.y);
    x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(x.x) + __uint_as_float(x.y);
}
__device__ __forceinline__ int64_t shfl64(int64_t v, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__shfl((int)v, lane) | (uint64_t)(uint32_t)__shfl((int)(v >> 32), lane) << 32);
}

// CODES: 8-bit cache.  WHOLE: every 16 keys of a chunk lie in one page.  DT: 32-element parts of the head dimension (2, 4).
// NT: 16-row tiles.  W: waves.
template <class T, bool CODES, bool WHOLE, int DT, int NT, int W>
__global__ __launch_bounds__(64 * W, 2) void attn_tree(AttnTreeArgs a, TreePlan p, float by_log2e, uint32_t negate) {
    typedef typename T::elem E;
    constexpr int PITCH = DT == 2 ? 128 : 256, D16 = 2 * DT, DP = 32 * DT, TILE = kChunk * PITCH, V_LOADS = TILE / 1024;
    // Maxima (powers of two) beyond which steps of a float are too coarse for what is added to them: a scale's logarithm, which the sum of
    // weights does not see rounded (at 2^12 by 2^-12), the 2^7 of halves.  Such rows go to the plain path.
    constexpr float kMostTop = CODES ? 0x1p12f : T::lift > 0 ? 0x1p22f : INFINITY;
    constexpr int RED = 16 * (DP + 4) * 4 > TILE ? 16 * (DP + 4) * 4 : TILE;       // a wave's part of 16 rows, when the waves join
    __shared__ __align__(1024) char v_even[W * RED], v_odd[CODES ? 16 : W * TILE];   // (codes pass through registers: one buffer)
    __shared__ float scales[W][2][kChunk], stat[W][2][16 * NT], joined[2][16 * NT], q_lds[W][256];
    __shared__ uint32_t bad;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane >> 4, r = lane & 15;
    const int group = a.q_heads / a.kv_heads;
    // Work: key heads, row tiles, then parts of the cache of one request after the other.  Listed, a lane knows the work of the requests
    // up to its own, and a part is as many chunks as give every workgroup one.
    const bool listed = NT > 1 && p.listed;      // (16 rows: shorter parts and no list measured 141 us where lists took 157, decode of 32 requests)
    int chunks = p.chunks, upto = 0, my_tiles = 1, my_work = 0;
    if (listed) {
        int my_chunks = 0;
        if (lane < a.n_seqs) {
            int from, to;
            sequence_rows(a.starts, lane, a.total, from, to);
            const int drafts = min(to - from, a.max_drafts), cached = min(max(a.cached[lane], 0), a.max_cached);
            my_tiles = (drafts * group + 16 * NT - 1) / (16 * NT);
            my_chunks = drafts > 0 ? (cached + kChunk - 1) / kChunk + (drafts + kChunk - 1) / kChunk : 0;
        }
        float all = (float)a.kv_heads * (float)my_tiles * (float)my_chunks;
        for (int d = 32; d > 0; d >>= 1) all += __shfl_xor(all, d);
        chunks = max(chunks, __builtin_amdgcn_readfirstlane(first_chunks(all, gridDim.x, W)));
        for (;; chunks += (chunks / 8 + W) / W * W) {
            my_work = a.kv_heads * my_tiles * ((my_chunks + chunks - 1) / chunks);
            if (sum_of_lanes(my_work) <= (int)gridDim.x || !__any(my_chunks > chunks)) break;
        }
        upto = sum_up_to_lane(my_work);
        if (blockIdx.x == 0 && wave == 0) {
            int *list = list_of(a, p);
            if (lane == 0) list[0] = chunks;
            if (lane < a.n_seqs) list[1 + lane] = upto - my_work;
        }
    }
    const int n_items = listed ? __builtin_amdgcn_readlane(upto, 63) : gridDim.x;
    for (int item = blockIdx.x; item < n_items; item += gridDim.x) {
    // Workgroups go to the eight XCDs in turn.  Eight parts at a time are dealt out so that the heads and row tiles of a part follow one
    // another on one XCD: they share lines (a token's scales, rows of less than a line, for row tiles all) that only its L2 then fetches.
    int b = 0, id = item, n_here = gridDim.x, tiles = p.row_tiles;
    if (listed) {
        b = __builtin_ctzll(__ballot(upto > item));
        n_here = __builtin_amdgcn_readlane(my_work, b);
        id -= __builtin_amdgcn_readlane(upto, b) - n_here;
        tiles = __builtin_amdgcn_readlane(my_tiles, b);
    }
    const int units = a.kv_heads * tiles;
    auto by_units = [&](int x) { return listed ? x / units : (int)fdiv((uint32_t)x, p.by_units); };
    const int eights = by_units(id >> 3), in = id - eights * 8 * units;
    const bool dealt = (eights + 1) * 8 * (int64_t)units <= n_here;
    int split = dealt ? eights * 8 + (in & 7) : by_units(id);
    const int unit = dealt ? in >> 3 : id - split * units, tile = (int)fdiv((uint32_t)unit, p.by_heads), hk = unit - tile * a.kv_heads;
    if (!listed) {
        b = split / p.splits;
        split -= b * p.splits;
    }
    TreeKeys<T> keys(a, b, hk);
    const int n_rows = keys.drafts * group, row0 = tile * 16 * NT;
    const int cached_chunks = (keys.cached + kChunk - 1) / kChunk, n_chunks = cached_chunks + (keys.drafts + kChunk - 1) / kChunk;
    const int first = split * chunks, last = min(n_chunks, first + chunks);
    if (row0 >= n_rows || first >= last) break;                    // (not listed: the only item)
    keys.pad = cached_chunks * kChunk;

    // queries: operand B; d of lane, step s: 32 s + 8 c, with codes 64 (s / 2) + 16 c + 8 (s % 2) (16 codes are one load)
    typename T::v8 q[NT][DT];
    uint64_t mask[NT];
    for (int n = 0; n < NT; ++n) {
        const int row = min(row0 + 16 * n + r, n_rows - 1), t = (int)fdiv((uint32_t)row, p.by_group), h = hk * group + row - t * group;
        const E *at = (const E *)a.q + (int64_t)(keys.from + t) * a.q_token + h * a.q_head;
        mask[n] = keys.mask(t);
        for (int s = 0; s < DT; ++s) {
            const int d = CODES ? 64 * (s >> 1) + 16 * c + 8 * (s & 1) : 32 * s + 8 * c;
            v4u x = d < a.head_dim ? *(const v4u *)(at + d) : v4u{0, 0, 0, 0};
            x ^= negate;
            q[n][s] = __builtin_bit_cast(typename T::v8, x);
        }
    }

    // swizzle of V's rows in LDS: 16-byte piece i of row x lies at piece i ^ f(x)
    auto f = [](int x) { return PITCH == 256 ? (x & 7) << 1 : (x & 6); };
    const int v_base = (4 * c + ((lane >> 2) & 3)) * PITCH + ((f(4 * c + ((lane >> 2) & 3)) | ((lane >> 1) & 1)) << 4) + (lane & 1) * 8;

    struct Chunk {
        v4u k[2][CODES ? DT / 2 : DT], v[CODES ? V_LOADS / 2 : 1];
        float ks, vs;
        uint32_t seen;
    };
    // The pages of a chunk's keys: that of this lane's key (lane & 31), or, WHOLE, those of the two tiles of 16 keys.  Only looked up
    // here; a key past the last one is the last one, not seen.
    struct Place {
        int chunk, page[WHOLE ? 2 : 1];
    };
    const Fixed<int32_t> table = (Fixed<int32_t>)keys.table;
    const int size = CODES ? 1 : 2;
    auto key_of = [&](int chunk, int t) {                                             // first key of a tile, or this lane's key
        const int j = chunk * kChunk + (WHOLE ? 16 * t : (lane & 31));
        return WHOLE ? max(min(j, keys.cached - 1), 0) & ~15 : min(j, keys.cached - 1);
    };
    auto look_up = [&](int chunk, Place &g) {
        g.chunk = chunk;
        for (int t = 0; t < (WHOLE ? 2 : 1); ++t) g.page[t] = table[fdiv((uint32_t)key_of(chunk, t), a.cache.by_page)];
    };
    // the lanes' loads: K a key and 16 bytes a lane; V a row's pieces side by side (past the head's elements: the first piece -- K's
    // meet zeros in q, V's are not stored)
    constexpr int K_LOADS = CODES ? DT / 2 : DT, LANES = CODES ? PITCH / 32 : PITCH / 16, N_V = CODES ? V_LOADS / 2 : V_LOADS, V_ROWS = 64 / LANES;
    int k_piece[K_LOADS], v_piece[V_LOADS > 1 && PITCH == 256 && !CODES ? 2 : 1];
    for (int s = 0; s < K_LOADS; ++s) {
        const int d = CODES ? 64 * s + 16 * c : 32 * s + 8 * c;
        k_piece[s] = d < a.head_dim ? d : 0;
    }
    for (int i = 0; i < (int)(sizeof(v_piece) / sizeof(int)); ++i) {
        const int d = CODES ? lane % LANES * 16 : ((lane % LANES) ^ f(i * V_ROWS + lane / LANES)) * 8;
        v_piece[i] = d < a.head_dim ? d : 0;
    }
    const Global<char> k_cache = (Global<char>)a.cache.k, v_cache = (Global<char>)a.cache.v;
    const int token_bytes = (int)a.cache.token_stride * size;                         // (WHOLE)
    auto load_cached = [&](const Place &w, Chunk &g, char *vt) {
        // elements from the cache's start and places of the scales, of a tile or of this lane's key
        int64_t at[WHOLE ? 2 : 1], scale[WHOLE ? 2 : 1];
        bool ok[WHOLE ? 2 : 1];
        for (int t = 0; t < (WHOLE ? 2 : 1); ++t) {
            const int i = key_of(w.chunk, t), place = i - (int)fdiv((uint32_t)i, a.cache.by_page) * a.cache.page;
            ok[t] = (uint32_t)w.page[t] < (uint32_t)a.cache.n_pages;
            const int64_t page = ok[t] ? w.page[t] : 0;
            at[t] = (page * a.cache.page_stride + place * a.cache.token_stride + hk * a.cache.head_stride) * size;
            scale[t] = (page * a.cache.page + place) * a.kv_heads + hk;
        }
        if constexpr (WHOLE) {
            g.seen = 0;
            for (int t = 0; t < 2; ++t) {
                const int n = min(keys.cached - (w.chunk * kChunk + 16 * t), 16);
                if (ok[t] && n > 0) g.seen |= (n == 16 ? 0xffffu : (1u << n) - 1) << (16 * t);
            }
        } else {
            g.seen = (uint32_t)__ballot(ok[0] && w.chunk * kChunk + (lane & 31) < keys.cached);
        }
        // row of a tile -> the row read: the last one seen where the tile is not full
        auto row_of = [&](int t, int row) {
            const uint32_t seen = g.seen >> (16 * t) & 0xffffu;
            return seen == 0xffffu ? row : min(row, 31 - __builtin_clz(seen | 1u));
        };
        if constexpr (CODES) {
            const int64_t i = WHOLE ? ((lane & 16) ? scale[1] : scale[0]) + (int64_t)row_of((lane >> 4) & 1, lane & 15) * a.kv_heads : scale[0];
            g.ks = a.cache.ks[i];
            g.vs = a.cache.vs[i];
        }
        for (int t = 0; t < 2; ++t) {
            if constexpr (WHOLE) {
                const uint32_t row = (uint32_t)(row_of(t, r) * token_bytes);
                for (int s = 0; s < K_LOADS; ++s) g.k[t][s] = *(Global<v4u>)(k_cache + at[t] + (row + k_piece[s] * size));
            } else {
                const int64_t key = shfl64(at[0], 16 * t + r);
                for (int s = 0; s < K_LOADS; ++s) g.k[t][s] = *(Global<v4u>)(k_cache + key + k_piece[s] * size);
            }
        }
        for (int i = 0; i < N_V; ++i) {
            const int row = i * V_ROWS + lane / LANES, piece = v_piece[i % (int)(sizeof(v_piece) / sizeof(int))] * size;
            Global<char> from;
            if constexpr (WHOLE) {
                const int t = i / (N_V / 2);
                from = v_cache + at[t] + (uint32_t)(row_of(t, row - 16 * t) * token_bytes + piece);
            } else from = v_cache + shfl64(at[0], row) + piece;
            if constexpr (CODES) g.v[i] = *(Global<v4u>)from;
            else __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)(vt + i * 1024), 16, 0, 0);
        }
    };

    v4f o[NT][D16];
    float m[NT], total[NT];
    for (int n = 0; n < NT; ++n) {
        m[n] = -INFINITY;
        total[n] = 0;
        for (int d = 0; d < D16; ++d) o[n][d] = v4f{0, 0, 0, 0};
    }

    // scores in sc (times c = scale log2 e where WEIGHTED: times the key's own factor too), 32 keys' values in vt
    auto join = [&](v4f (&sc)[2][NT], auto weighted, const float *vlog, const float *vinv, const char *vt) {
        constexpr bool WEIGHTED = decltype(weighted)::value;
        typename T::v8 pv[NT];
        float lv[2][4], iv[2][4];
        if constexpr (WEIGHTED)
            for (int t = 0; t < 2; ++t) {
                *(v4f *)lv[t] = *(const v4f *)(vlog + 16 * t + 4 * c);
                *(v4f *)iv[t] = *(const v4f *)(vinv + 16 * t + 4 * c);
            }
        for (int n = 0; n < NT; ++n) {
            float top = -INFINITY;
            for (int t = 0; t < 2; ++t)
                for (int e = 0; e < 4; ++e) {
                    if constexpr (WEIGHTED) sc[t][n][e] += lv[t][e];
                    top = fmaxf(top, sc[t][n][e]);
                }
            top = max_of_quarters(top);
            if (__any(top > m[n] + 8.f)) {       // (as in prompt attention: powers of two up to 2^8 over the maximum do no harm)
                const float next = fmaxf(m[n], top), keep = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[n] - next);
                m[n] = next;
                total[n] *= keep;
                for (int d = 0; d < D16; ++d) o[n][d] *= keep;
            }
            const float off = m[n] == -INFINITY ? 0.f : m[n] - T::lift;
            float sum = 0;      // (of the lane's 8 keys before it meets the total, as in prompt attention)
            for (int t = 0; t < 2; ++t)
                for (int e = 0; e < 4; ++e) {
                    const float w = __builtin_amdgcn_exp2f(sc[t][n][e] - off);
                    if constexpr (WEIGHTED) sum = fmaf(w, iv[t][e], sum);
                    else sum += w;
                    pv[n][4 * t + e] = (E)w;
                }
            total[n] += sum;
        }
        for (int d = 0; d < D16; ++d) {
            const char *at = vt + (v_base ^ (d << 5));
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)at);
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(at + 16 * PITCH));
            const v8s both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            for (int n = 0; n < NT; ++n) o[n][d] = T::mfma16(__builtin_bit_cast(typename T::v8, both), pv[n], o[n][d]);
        }
    };

    auto use_cached = [&](Chunk &g, char *vt) {
        float *vlog = scales[wave][0], *vinv = scales[wave][1];
        float kf[2][4];
        if constexpr (CODES) {
            __builtin_amdgcn_wave_barrier();
            const bool mine = g.seen >> (lane & 31) & 1;                             // (a key that is not seen has no scale)
            if (lane < kChunk) vlog[lane] = mine ? g.ks * by_log2e : 0.f;
            __builtin_amdgcn_wave_barrier();
            for (int t = 0; t < 2; ++t) *(v4f *)kf[t] = *(const v4f *)(vlog + 16 * t + 4 * c);
            __builtin_amdgcn_wave_barrier();
            // a row of zeros (scale 0) counts with a scale that leaves its weight in the sum; other scales below that (and NaN) make the rows
            // that see them NaN, for the plain path
            const float v = mine ? fmaxf(g.vs, 0x1p-90f) : 1.f;
            if (lane < kChunk) {
                vlog[lane] = mine && !(g.vs >= 0x1p-90f || g.vs == 0.f) ? __builtin_nanf("") : __builtin_amdgcn_logf(v);
                vinv[lane] = 1.f / v;
            }
            // V's codes to LDS as T
            constexpr int LANES = PITCH / 32;
            for (int i = 0; i < V_LOADS / 2; ++i) {
                const int row = i * (64 / LANES) + lane / LANES, piece = lane % LANES * 2;
                *(typename T::v8 *)(vt + row * PITCH + ((piece ^ f(row)) << 4)) = from_codes<T>(g.v[i].x, g.v[i].y);
                *(typename T::v8 *)(vt + row * PITCH + (((piece + 1) ^ f(row)) << 4)) = from_codes<T>(g.v[i].z, g.v[i].w);
            }
            __builtin_amdgcn_wave_barrier();
        }
        v4f sc[2][NT];
        for (int t = 0; t < 2; ++t) {
            for (int n = 0; n < NT; ++n) sc[t][n] = v4f{0, 0, 0, 0};
            for (int s = 0; s < DT; ++s) {
                typename T::v8 k;
                if constexpr (CODES) k = (s & 1) ? from_codes<T>(g.k[t][s >> 1].z, g.k[t][s >> 1].w) : from_codes<T>(g.k[t][s >> 1].x, g.k[t][s >> 1].y);
                else k = __builtin_bit_cast(typename T::v8, g.k[t][s]);
                for (int n = 0; n < NT; ++n) sc[t][n] = T::mfma16(k, q[n][s], sc[t][n]);
            }
            for (int n = 0; n < NT; ++n)
                for (int e = 0; e < 4; ++e) sc[t][n][e] *= CODES ? kf[t][e] : by_log2e;
        }
        if (g.seen != 0xffffffffu)
            for (int t = 0; t < 2; ++t)
                for (int e = 0; e < 4; ++e)
                    if (!(g.seen >> (16 * t + 4 * c + e) & 1))
                        for (int n = 0; n < NT; ++n) sc[t][n][e] = -INFINITY;
        join(sc, std::integral_constant<bool, CODES>{}, vlog, vinv, vt);
    };

    // a chunk of drafts: rows of k and v in T, seen as the masks say
    auto use_drafts = [&](int chunk, char *vt) {
        const int j0 = (chunk - cached_chunks) * kChunk;
        constexpr int LANES = PITCH / 16;
        for (int i = 0; i < V_LOADS; ++i) {
            const int row = i * (64 / LANES) + lane / LANES, piece = lane % LANES;
            const int64_t at = keys.from + min(j0 + row, keys.drafts - 1);
            const v4u x = *(const v4u *)((const E *)a.v + at * a.v_token + hk * a.v_head + (piece * 8 < a.head_dim ? piece * 8 : 0));
            *(v4u *)(vt + row * PITCH + ((piece ^ f(row)) << 4)) = x;
        }
        __builtin_amdgcn_wave_barrier();
        v4f sc[2][NT];
        for (int t = 0; t < 2; ++t) {
            for (int n = 0; n < NT; ++n) sc[t][n] = v4f{0, 0, 0, 0};
            const E *at = (const E *)a.k + (int64_t)(keys.from + min(j0 + 16 * t + r, keys.drafts - 1)) * a.k_token + hk * a.k_head;
            for (int s = 0; s < DT; ++s) {
                const int d = CODES ? 64 * (s >> 1) + 16 * c + 8 * (s & 1) : 32 * s + 8 * c;
                const v4u k = *(const v4u *)(at + (d < a.head_dim ? d : 0));
                for (int n = 0; n < NT; ++n) sc[t][n] = T::mfma16(__builtin_bit_cast(typename T::v8, k), q[n][s], sc[t][n]);
            }
            for (int n = 0; n < NT; ++n)
                for (int e = 0; e < 4; ++e) {
                    const int j = j0 + 16 * t + 4 * c + e;
                    sc[t][n][e] = j < keys.drafts && (mask[n] >> j & 1) ? sc[t][n][e] * by_log2e : -INFINITY;
                }
        }
        join(sc, std::false_type{}, nullptr, nullptr, vt);
    };

    {
        char *ve = v_even + wave * RED, *vo = CODES ? ve : v_odd + wave * TILE;
        const int end = min(last, cached_chunks);
        int chunk = first + wave;
        if (chunk < end) {
            // Loads are issued without a branch around them (behind one the compiler waits for all that may be under way): a wave's last
            // chunk is loaded once more, from the caches.
            Place place;
            Chunk even, odd;
            look_up(chunk, place);
            load_cached(place, even, ve);
            look_up(chunk + W < end ? chunk + W : chunk, place);
            for (;;) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // all of this chunk has landed; what is issued next is the following one's
                load_cached(place, odd, vo);
                look_up(chunk + 2 * W < end ? chunk + 2 * W : chunk, place);
                use_cached(even, ve);
                chunk += W;
                if (chunk >= end) break;
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                load_cached(place, even, ve);
                look_up(chunk + 2 * W < end ? chunk + 2 * W : chunk, place);
                use_cached(odd, vo);
                chunk += W;
                if (chunk >= end) break;
            }
            if constexpr (!CODES) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // (the chunk loaded once more may land where the drafts and the sums go)
        }
        for (; chunk < last; chunk += W) use_drafts(chunk, ve);
    }

    // From here on the arguments are read again where they are needed: held through the loop they would not fit the scalar registers.
    Fixed<char> kernel_arguments = (Fixed<char>)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(kernel_arguments));
    const AttnTreeArgs &late = *(const AttnTreeArgs *)kernel_arguments;
    const TreeKeys<T> rest(late, keys);

    // the waves join: each row's maximum and sum, then 16 rows' outputs at a time
    for (int n = 0; n < NT; ++n) {
        total[n] = sum_of_quarters(total[n]);
        if (c == 0) {
            stat[wave][0][16 * n + r] = m[n];
            stat[wave][1][16 * n + r] = total[n];
        }
    }
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    if (threadIdx.x < 16 * NT) {
        float top = -INFINITY, sum = 0;
        for (int w = 0; w < W; ++w) top = fmaxf(top, stat[w][0][threadIdx.x]);
        for (int w = 0; w < W; ++w) {
            const float mw = stat[w][0][threadIdx.x];
            sum += mw == top ? stat[w][1][threadIdx.x] : stat[w][1][threadIdx.x] * __builtin_amdgcn_exp2f(mw - top);
        }
        joined[0][threadIdx.x] = top;
        joined[1][threadIdx.x] = sum;
        if (fabsf(top) > kMostTop && top > -INFINITY) atomicOr(&bad, 1u << threadIdx.x);
    }
    __syncthreads();
    const bool whole = n_chunks <= chunks;
    const int item_part = listed && !whole ? (item - id + unit * ((n_chunks + chunks - 1) / chunks) + split) * kPartRows : 0;
    auto part_at = [&](int row, int t, int h) { return listed ? (int64_t)(item_part + row - row0) : ((int64_t)(rest.from + t) * late.q_heads + h) * p.splits + split; };
    float *red = (float *)v_even;
    constexpr int ROW = DP + 4;
    for (int n = 0; n < NT; ++n) {
        const float top = joined[0][16 * n + r], keep = m[n] == top ? 1.f : __builtin_amdgcn_exp2f(m[n] - top);
        for (int d = 0; d < D16; ++d) *(v4f *)(red + wave * (RED / 4) + r * ROW + 16 * d + 4 * c) = o[n][d] * keep;
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * (DP / 4); e += 64 * W) {
            const int i = e / (DP / 4), d = e % (DP / 4) * 4, row = row0 + 16 * n + i;
            if (row >= n_rows || d >= late.head_dim) continue;
            v4f v{0, 0, 0, 0};
            for (int w = 0; w < W; ++w) v += *(const v4f *)(red + w * (RED / 4) + i * ROW + d);
            const float sum = joined[1][16 * n + i], any = v.x + v.y + v.z + v.w + sum;
            const int t = (int)fdiv((uint32_t)row, p.by_group), h = hk * group + row - t * group;
            if (any != any) atomicOr(&bad, 1u << (16 * n + i));
            if (whole) {
                const float by = 1.f / sum;
                typename T::v4 y;
                for (int k = 0; k < 4; ++k) y[k] = (E)(sum == 0.f ? 0.f : v[k] * by);
                *(typename T::v4 *)(rest.out(t, h) + d) = y;
            } else {
                const int64_t at = part_at(row, t, h);
                *(v4f *)(late.partial + at * late.head_dim + d) = v;
                if (d == 0) *(float2 *)(stats_of(late, p) + 2 * at) = make_float2(joined[0][16 * n + i] - T::lift, sum);
            }
        }
        __syncthreads();
    }
    // rows with a NaN, or scores too large, once more, the plain way
    int nth = 0;
        for (uint32_t left = bad; left; left &= left - 1, ++nth) {
            const int row = row0 + __builtin_ctz(left);
            if (nth % W != wave || row >= n_rows) continue;
            const int t = (int)fdiv((uint32_t)row, p.by_group), h = hk * group + row - t * group;
            const RowSums s = rest.attend(t, h, first * kChunk, last * kChunk, q_lds[wave]);
            if (whole) {
                store_row<T>(s, rest.out(t, h), late.head_dim);
            } else {
                const int64_t i = part_at(row, t, h);
                for (int k = 0; k < 4; ++k)
                    if (lane + 64 * k < late.head_dim) late.partial[i * late.head_dim + lane + 64 * k] = s.total == 0.f ? 0.f : s.o[k];
                if (lane < 2) stats_of(late, p)[2 * i + lane] = lane ? s.total : s.m * kLog2e;
            }
        }
    if (!listed) break;
    __syncthreads();
    }
}

// one wave per row: the parts of a request that was shared out
template <class T>
__global__ __launch_bounds__(256) void attn_tree_join(AttnTreeArgs a, TreePlan p) {
    typedef typename T::elem E;
    const int lane = threadIdx.x & 63, h = blockIdx.x * 4 + (threadIdx.x >> 6), t = blockIdx.y, b = blockIdx.z;
    if (h >= a.q_heads) return;
    const TreeKeys<T> keys(a, b, 0);
    const int n_chunks = (keys.cached + kChunk - 1) / kChunk + (keys.drafts + kChunk - 1) / kChunk;
    const int *list = list_of(a, p);
    const int chunks = p.listed ? list[0] : p.chunks;
    if (t >= keys.drafts || n_chunks <= chunks) return;
    const int n = (n_chunks + chunks - 1) / chunks;
    int64_t first = ((int64_t)(keys.from + t) * a.q_heads + h) * p.splits;      // this row's parts: from here on,
    int step = 1;                                                               // this far apart
    if (p.listed) {
        const int hk = (int)fdiv((uint32_t)h, p.by_group), group = a.q_heads / a.kv_heads, row = t * group + h - hk * group;
        first = (int64_t)(list[1 + b] + (row / kPartRows * a.kv_heads + hk) * n) * kPartRows + row % kPartRows;
        step = kPartRows;
    }
    const float *stats = stats_of(a, p) + 2 * first, *part = a.partial + first * a.head_dim;
    float top = -INFINITY, sum = 0;
    float2 o = make_float2(0, 0);
    for (int s = lane; s < n; s += 64) top = fmaxf(top, stats[2 * s * step]);
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const int two = min(2 * lane, a.head_dim - 2);      // this lane's elements (past the last: the last ones, not stored)
    for (int s0 = 0; s0 < n; s0 += 64) {       // 64 parts' weights, a lane each; then their outputs, the loads of eight in flight
        const int s = s0 + lane;
        float w = 0;
        if (s < n) {
            const float *at = stats + 2 * s * step;
            w = at[0] == top ? 1.f : __builtin_amdgcn_exp2f(at[0] - top);
            sum += w * at[1];
        }
        const int here = min(64, n - s0);
        for (int i = 0; i < here; i += 8) {
            float2 x[8];
            for (int k = 0; k < 8; ++k) x[k] = *(const float2 *)(part + (int64_t)(s0 + min(i + k, here - 1)) * step * a.head_dim + two);
            for (int k = 0; k < 8; ++k) {
                const float wi = __shfl(w, min(i + k, 63));        // (0 past the last part)
                if (i + k < here) {
                    o.x += wi * x[k].x;
                    o.y += wi * x[k].y;
                }
            }
        }
    }
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if (2 * lane >= a.head_dim) return;
    const float by = 1.f / sum;
    *(typename T::v2 *)(keys.out(t, h) + two) = typename T::v2{(E)(sum == 0.f ? 0.f : o.x * by), (E)(sum == 0.f ? 0.f : o.y * by)};
}

// Rows read in whole vectors.  (Pointers are 0 where only the workspace is asked for.)
bool matrix_form(const AttnTreeArgs &a) {
    const bool codes = a.cache.dtype == HAWQ_S8;
    const int64_t rows = a.q_token | a.q_head | a.k_token | a.k_head | a.v_token | a.v_head, cache = a.cache.page_stride | a.cache.token_stride | a.cache.head_stride;
    return a.head_dim <= 128 && a.head_dim % (codes ? 16 : 8) == 0 && rows % 8 == 0 && (a.y_token | a.y_head) % 4 == 0 && ((uintptr_t)a.y & 7) == 0 && cache % (codes ? 16 : 8) == 0 &&
           (((uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.cache.k | (uintptr_t)a.cache.v) & 15) == 0;
}

template <class T, bool CODES, bool WHOLE, int DT>
void launch_rows(const AttnTreeArgs &a, const TreePlan &p, hipStream_t s) {
    const unsigned blocks = (unsigned)p.blocks;
    const float c = fmaxf(fabsf(a.scale) * kLog2e, 1.2e-38f);       // (a negative scale: -q; zero: as good as the smallest number)
    const uint32_t negate = a.scale < 0 ? 0x80008000u : 0u;
    if (p.waves == 8) attn_tree<T, CODES, WHOLE, DT, 1, 8><<<blocks, 512, 0, s>>>(a, p, c, negate);
    else if (p.rows == 16) attn_tree<T, CODES, WHOLE, DT, 1, 4><<<blocks, 256, 0, s>>>(a, p, c, negate);
    else attn_tree<T, CODES, WHOLE, DT, 2, 4><<<blocks, 256, 0, s>>>(a, p, c, negate);
}

template <class T, bool CODES>
void launch_form(const AttnTreeArgs &a, const TreePlan &p, hipStream_t s) {
    // 16 keys from a multiple of 16 on share a page; their rows lie within 31-bit offsets of the first
    if (a.cache.page % 16 == 0 && a.cache.token_stride < (1 << 25)) {
        if (a.head_dim <= 64) launch_rows<T, CODES, true, 2>(a, p, s);
        else launch_rows<T, CODES, true, 4>(a, p, s);
    } else if (a.head_dim <= 64) launch_rows<T, CODES, false, 2>(a, p, s);
    else launch_rows<T, CODES, false, 4>(a, p, s);
}

template <class T>
hawq_status launch(const AttnTreeArgs &a, hipStream_t s) {
    const TreePlan p = tree_plan(a);
    if (!matrix_form(a) || p.blocks == 0) {
        attn_tree_any<T><<<dim3((unsigned)a.max_drafts, (unsigned)a.q_heads, (unsigned)a.n_seqs), 64, 0, s>>>(a);
        return check_launch();
    }
    if (a.cache.dtype == HAWQ_S8) launch_form<T, true>(a, p, s);
    else launch_form<T, false>(a, p, s);
    if (p.splits > 1) attn_tree_join<T><<<dim3((unsigned)(a.q_heads + 3) / 4, (unsigned)a.max_drafts, (unsigned)a.n_seqs), 256, 0, s>>>(a, p);
    return check_launch();
}

}  // namespace

size_t attn_tree_workspace(const AttnTreeArgs &a) {
    const TreePlan p = tree_plan(a);
    return p.splits > 1 ? (size_t)p.parts * (a.head_dim + 2) * sizeof(float) + (p.listed ? 65 * sizeof(int) : 0) : 0;
}

hawq_status launch_attn_tree(const AttnTreeArgs &a, hipStream_t s) { return a.dtype == HAWQ_F16 ? launch<F16>(a, s) : launch<BF16>(a, s); }

}  // namespace hawq
