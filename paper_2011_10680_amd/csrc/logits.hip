// What a server does to the logits before it chooses: penalties for tokens that occurred, biases, grammar masks.
//
// Two things are done to a row.  Its logits are copied with the mask applied, eight to a thread (in place: only what the mask takes away).  And
// the tokens that occurred or are listed are counted in LDS, one word a token (bit 31: occurred; bits 24 to 30: its place in a short list of
// biases; below: how often the model wrote it), whose logits are then written again.  Integer counts and maxima: the order of the atomics does not
// matter.
//
// Few logits go through one launch: a workgroup copies a part of the vocabulary and counts the tokens that fall into it, words lying by token.
// Many go through two: a copy that waits for nothing but the mask, and a workgroup for each row, whose words lie by a hash of the token,
// so that the row's tokens are read once.  Rows with more tokens or longer lists than that holds go part by part there, too, all parts in one
// workgroup (a row of 128001 in place: 9999 tokens 20 us, 10001 50, 131072 465; by a workgroup for each part, where it is copied, 11, 11 and 93).
//
// Bound by the logits' bytes for many rows, by a chain of loads (request, lengths, tokens, logits) and a launch for few.  Measured: 256 x 128001
// 57 us from memory, 43 from the caches, of which the copy is 27 (4.9 TB/s) and the tokens 16; 171 x 64000 27.5 and 18; one row of 32000 6, twice
// an empty launch.  Words checked in order instead of by token, in one launch: 256 x 128001 64 us and more from the caches, the copy's loop no
// longer in the instruction cache.
#include "lm.h"
#include "lm_launch.h"

namespace hawq {

namespace {

constexpr uint32_t kOccurred = 0x80000000u, kPlaces = 0x7F000000u, kListed = 1u << 24, kCount = 0x00FFFFFFu;
constexpr int kFewBiases = 127;                  // whose places a word holds
constexpr int kPartThreads = 512, kAhead = 4;    // eights of a thread that are loaded before the request is looked for, one after the other (each in a branch)
// Logits from which tokens are counted in a launch of their own: 171 x 64000 take 18.5 us in one launch and 20.9 in two, 256 x 128001 61 and 43.
constexpr int64_t kApart = 1 << 24;
constexpr int kRowThreads = 1024, kSlots = 16384, kMostHashed = 10000;

// The request whose rows t belongs to, -1: none.  64 places at a time: the chain of loads is one or two long, up to 2^24 requests four.
__device__ __forceinline__ int request_of(const LogitsArgs &a, int t) {
    if (!a.starts) return t;
    const int lane = threadIdx.x & 63;
    int low = 0, high = a.n_seqs;                // the first request that ends behind t is in [low, high), or high itself where that is known to
    bool known = false;
    while (low < high) {
        const int step = (int)(((int64_t)high - low + 63) / 64);
        const int at = (int)min((int64_t)low + (int64_t)lane * step + step, (int64_t)high) - 1;
        const uint64_t ends = __ballot(a.starts[at + 1] > t);
        if (!ends) {
            if (!known) return -1;
            low = high;
            break;
        }
        known = true;
        const int first = __builtin_ctzll(ends);
        high = (int)min((int64_t)low + (int64_t)first * step + step, (int64_t)high) - 1;
        low = (int)min((int64_t)low + (int64_t)first * step, (int64_t)high);
    }
    low = __builtin_amdgcn_readfirstlane(low);
    return known && a.starts[low] <= t ? low : -1;
}

// the larger of a word's place and this one, beside whatever else changes the word
__device__ __forceinline__ void highest(uint32_t *word, uint32_t place) {
    uint32_t had = *(volatile uint32_t *)word;
    while ((had >> 24 & 127u) < place) {
        const uint32_t now = atomicCAS(word, had, (had & ~kPlaces) | place << 24);
        if (now == had) return;
        had = now;
    }
}

template <class T, int THREADS>
struct Row {
    typedef typename T::elem E;
    const E *x;
    E *y;
    float r, presence, frequency;
    const int32_t *bias_ids, *past, *drafts;
    const float *bias_values;
    const uint32_t *allowed;                     // nullptr: everything
    uint64_t sees;                               // of 64 drafts; all ones without a mask
    int biases, len, prompt, seen;               // numbers of listed, past and drafted tokens
    bool counts;
    int32_t listed, draft, head[4];              // this thread's first listed, drafted and past tokens

    // what is known of row t of request b, all at once: every load that waits for another costs a microsecond
    __device__ __forceinline__ void load(const LogitsArgs &a, int t, int b) {
        x = (const E *)a.x + t * a.x_stride;
        y = (E *)a.y + t * a.y_stride;
        const int64_t p = 3 * (int64_t)b;
        r = a.penalties ? a.penalties[p] : 1.f;
        presence = a.penalties ? a.penalties[p + 1] : 0.f;
        frequency = a.penalties ? a.penalties[p + 2] : 0.f;
        const int first = a.n_bias > 0 ? min(max(a.bias_starts[b], 0), a.n_bias) : 0;
        biases = a.n_bias > 0 ? min(max(a.bias_starts[b + 1], first), a.n_bias) - first : 0;
        bias_ids = a.bias_ids + first;
        bias_values = a.bias_values + first;
        len = a.past_stride > 0 ? min(max(a.past_lens[b], 0), a.past_stride) : 0;
        prompt = a.past_stride > 0 && a.prompt_lens ? a.prompt_lens[b] : 0;
        past = a.past + (int64_t)b * a.past_stride;
        int from = t, to = t + 1;
        if (a.drafts && a.starts) sequence_rows(a.starts, b, a.total, from, to);
        drafts = a.drafts ? a.drafts + from : nullptr;
        sees = a.drafts && a.mask ? a.mask[t] : ~0ull;
        seen = !a.drafts ? 0 : a.mask ? min(to - from, 64) : t + 1 - from;
        const int row = a.n_allowed == 0 ? -1 : a.allowed_row ? a.allowed_row[t] : t;
        allowed = row >= 0 && row < a.n_allowed ? a.allowed + row * a.allowed_stride : nullptr;
        counts = r != 1.f || presence != 0.f || frequency != 0.f;
        if (!counts) len = seen = 0;
        listed = biases > 0 ? bias_ids[min((int)threadIdx.x, biases - 1)] : -1;
        draft = seen > 0 ? drafts[min((int)threadIdx.x, seen - 1)] : -1;
        for (int i = 0; i < 4; ++i) head[i] = len > 0 ? past[min((int)threadIdx.x + i * THREADS, len - 1)] : -1;
    }

    // f(token, entry of the list or -1, whether the model wrote it) of this thread's share of all
    template <class F>
    __device__ __forceinline__ void each(F &&f) const {
        for (int i = threadIdx.x; i < biases; i += THREADS) f(i < THREADS ? listed : bias_ids[i], i, false);
        for (int i = threadIdx.x; i < seen; i += THREADS) f(sees >> (i & 63) & 1 ? i < THREADS ? draft : drafts[i] : -1, -1, true);      // (-1 is no token)
        // (four tokens on their way at a time)
        for (int i0 = threadIdx.x; i0 < len; i0 += 4 * THREADS) {
            int32_t token[4];
            for (int i = 0; i < 4; ++i) token[i] = i0 < THREADS ? head[i] : past[min(i0 + i * THREADS, len - 1)];
            for (int i = 0; i < 4; ++i)
                if (i0 + i * THREADS < len) f(token[i], -1, i0 + i * THREADS >= prompt);
        }
    }

    // the logits of tokens v[i] with words c[i], 0: none; place: entries of the list and 1, 0: not in it (in a row with a mask the mask's words are
    // read in branches, one after the other)
    template <int N>
    __device__ __forceinline__ void again(const int (&v)[N], const uint32_t (&c)[N], const uint32_t (&place)[N]) const {
        E l[N];
        float bias[N];
        uint32_t kept[N];
        for (int i = 0; i < N; ++i) {
            const int at = c[i] ? v[i] : 0;
            l[i] = x[at];
            kept[i] = c[i] ? allowed ? allowed[at >> 5] >> (at & 31) & 1 : 1 : 0;
            bias[i] = place[i] ? bias_values[place[i] - 1] : 0.f;
        }
        for (int i = 0; i < N; ++i) {
            float n = (float)l[i];
            if (c[i] & kOccurred) n = n > 0 ? n / r : n * r;
            if (c[i] & kCount) n = n - frequency * (float)(c[i] & kCount) - presence;
            if (place[i]) n += bias[i];
            if (kept[i]) y[v[i]] = (E)n;
        }
    }

    // The tokens v0 .. v0 + n - 1 by words of their own, count[n], and where the list is long place[n], cleared before and seen by all.
    // Whoever counted a token takes its word away afterwards: the first one writes the token's logit again.
    __device__ __forceinline__ void settle(int v0, int n, uint32_t *count, uint32_t *place) const {
        const bool places = biases > kFewBiases;
        each([&](int32_t token, int entry, bool written) {
            const uint32_t at = (uint32_t)token - (uint32_t)v0;
            if (at >= (uint32_t)n) return;
            if (entry >= 0) {
                if (places) atomicMax(place + at, (uint32_t)entry + 1), atomicOr(count + at, kListed);
                else highest(count + at, (uint32_t)entry + 1);
            } else {
                if (written) atomicAdd(count + at, 1u);
                atomicOr(count + at, kOccurred);
            }
        });
        __syncthreads();
        auto take = [&](auto &token) {
            constexpr int N = sizeof(token) / sizeof(token[0]);
            bool any = false;
            for (int i = 0; i < N; ++i) any |= (uint32_t)token[i] - (uint32_t)v0 < (uint32_t)n;
            if (!any) return;
            uint32_t c[N], l[N];
            for (int i = 0; i < N; ++i) {
                const uint32_t at = (uint32_t)token[i] - (uint32_t)v0;
                c[i] = at < (uint32_t)n ? atomicExch(count + at, 0u) : 0u;
            }
            for (int i = 0; i < N; ++i) l[i] = !(c[i] & kPlaces) ? 0u : places ? place[(uint32_t)token[i] - (uint32_t)v0] : c[i] >> 24 & 127u;
            again(token, c, l);
        };
        for (int i = threadIdx.x; i < biases; i += THREADS) {
            const int32_t token[1] = {i < THREADS ? listed : bias_ids[i]};
            take(token);
        }
        for (int i = threadIdx.x; i < seen; i += THREADS) {
            const int32_t token[1] = {i < THREADS ? draft : drafts[i]};
            take(token);
        }
        for (int i0 = threadIdx.x; i0 < len; i0 += 4 * THREADS) {
            int32_t token[4];                    // (past the last one: that one again)
            for (int i = 0; i < 4; ++i) token[i] = i0 < THREADS ? head[i] : past[min(i0 + i * THREADS, len - 1)];
            take(token);
        }
    }
};

// n words, a multiple of four
template <int THREADS>
__device__ __forceinline__ void clear(uint32_t *words, int n) {
    for (int i = threadIdx.x; i < n / 4; i += THREADS) ((v4u *)words)[i] = v4u{0, 0, 0, 0};
}

// IN_PLACE: y is x, and what does not change is neither read nor written.  WORDS: tokens are counted here, too.
template <class T, bool IN_PLACE, bool WORDS>
__global__ __launch_bounds__(kPartThreads) void logits_part(LogitsArgs a, int part) {
    typedef typename T::elem E;
    typedef uint32_t Eight __attribute__((ext_vector_type(4), aligned(2)));      // (rows of x lie at any element)
    extern __shared__ __align__(16) uint32_t words[];
    const int t = (int)((int64_t)blockIdx.z * gridDim.y + blockIdx.y);
    if (t >= a.total) return;
    const int v0 = blockIdx.x * part, n = min(part, a.vocab - v0);
    // eights that lie at multiples of 16 bytes in y; the first may begin before v0, the last end past the part
    E *const y = (E *)a.y + t * a.y_stride + v0;
    const E *const x = (const E *)a.x + t * a.x_stride + v0;
    const int off = (int)((uintptr_t)y >> 1 & 7), eights = (n + off + 7) >> 3;
    auto whole = [&](int k) { return 8 * k >= off && 8 * k + 8 - off <= n; };
    Eight ahead[kAhead];
    if (!IN_PLACE)
        for (int i = 0; i < kAhead; ++i) {
            const int k = threadIdx.x + i * kPartThreads;
            if (k < eights && whole(k)) ahead[i] = *(const Eight *)(x + (8 * k - off));
        }
    const int b = request_of(a, t);
    if (b < 0) return;
    Row<T, kPartThreads> row;
    row.load(a, t, b);
    if (WORDS) clear<kPartThreads>(words, part + 16);
    const uint32_t *const allowed = row.allowed;
    auto copy = [&](int k, Eight d) {
        const int at = 8 * k - off;              // of the eight's first element in the part
        if (!whole(k)) {
#pragma unroll 1
            for (int i = max(at, 0); i < min(at + 8, n); ++i) {
                const bool kept = !allowed || (allowed[(v0 + i) >> 5] >> ((v0 + i) & 31) & 1);
                if (!IN_PLACE || !kept) y[i] = kept ? x[i] : (E)-INFINITY;
            }
            return;
        }
        uint32_t bits = 255u;
        if (allowed) {
            const int v = v0 + at, s = v & 31;
            bits = allowed[v >> 5] >> s;
            if (s > 24) bits |= allowed[(v >> 5) + 1] << (32 - s);
            bits &= 255u;
        }
        if (IN_PLACE) {
            if (bits == 255u) return;
            if (bits != 0) d = *(const Eight *)(x + at);
        }
        typename T::v8 e = __builtin_bit_cast(typename T::v8, (v4u)d);
        if (bits != 255u)
            for (int i = 0; i < 8; ++i)
                if (!(bits >> i & 1)) e[i] = (E)-INFINITY;
        *(v4u *)(y + at) = __builtin_bit_cast(v4u, e);
    };
    if (!IN_PLACE || allowed) {
        for (int i = 0; i < kAhead; ++i) {
            const int k = threadIdx.x + i * kPartThreads;
            if (k < eights) copy(k, ahead[i]);
        }
        for (int k = threadIdx.x + kAhead * kPartThreads; k < eights; k += kPartThreads) {
            Eight d{0, 0, 0, 0};
            if (!IN_PLACE && whole(k)) d = *(const Eight *)(x + (8 * k - off));
            copy(k, d);
        }
    }
    if (!WORDS || (!row.counts && row.biases == 0)) return;
    // Words are cleared for all.  (__syncthreads would wait for the copy here, too, which has until the tokens are counted: it is what comes between
    // counting and writing again.)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int half = row.biases > kFewBiases ? part / 2 + 4 : part;              // a long list's places share the words
    for (int first = 0; first < n; first += half) {
        if (first > 0) {
            __syncthreads();
            clear<kPartThreads>(words, part + 16);
            __syncthreads();
        }
        row.settle(v0 + first, min(half, n - first), words, words + half);
    }
}

// The tokens of one row, behind its copy.
template <class T>
__global__ __launch_bounds__(kRowThreads) void logits_row(LogitsArgs a) {
    extern __shared__ __align__(16) uint32_t words[];
    const int t = (int)((int64_t)blockIdx.y * gridDim.x + blockIdx.x);
    if (t >= a.total) return;
    const int b = request_of(a, t);
    if (b < 0) return;
    Row<T, kRowThreads> row;
    row.load(a, t, b);
    const int64_t tokens = (int64_t)row.len + row.seen + row.biases;
    if (tokens == 0) return;
    if (tokens > kMostHashed || row.biases > kFewBiases) {
        for (int64_t v = 0; v < a.vocab; v += kSlots) {
            __syncthreads();
            clear<kRowThreads>(words, 2 * kSlots);
            __syncthreads();
            row.settle((int)v, (int)min((int64_t)kSlots, a.vocab - v), words, words + kSlots);
        }
        return;
    }
    // slots of a token and a word, half as many again as tokens or more: 4096, 8192 or 16384
    uint32_t *const key = words, *const count = words + kSlots;
    const int bits = tokens <= 2700 ? 12 : tokens <= 5400 ? 13 : 14, slots = 1 << bits;
    clear<kRowThreads>(key, slots);
    clear<kRowThreads>(count, slots);
    __syncthreads();
    row.each([&](int32_t token, int entry, bool written) {
        if ((uint32_t)token >= (uint32_t)a.vocab) return;
        const uint32_t product = (uint32_t)token * 2654435761u;      // (2^32 by the golden ratio)
        // (odd steps reach every slot, of which there are more than tokens; steps of a token's own: the slots beside one another that a history
        // may have been made for fill up no faster than others)
        uint32_t at = product >> (32 - bits);
        const uint32_t on = product >> 6 | 1u;
        for (;;) {
            const uint32_t had = atomicCAS(key + at, 0u, (uint32_t)token + 1);
            if (had == 0 || had == (uint32_t)token + 1) break;
            at = (at + on) & (slots - 1);
        }
        if (entry >= 0) {
            highest(count + at, (uint32_t)entry + 1);
        } else {
            if (written) atomicAdd(count + at, 1u);
            atomicOr(count + at, kOccurred);
        }
    });
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < slots / 4; i += kRowThreads) {
        const v4u k = ((const v4u *)key)[i], c = ((const v4u *)count)[i];
        const int v[4] = {(int)k.x - 1, (int)k.y - 1, (int)k.z - 1, (int)k.w - 1};      // (an empty slot's word is 0)
        const uint32_t words_of[4] = {c.x, c.y, c.z, c.w}, places[4] = {c.x >> 24 & 127u, c.y >> 24 & 127u, c.z >> 24 & 127u, c.w >> 24 & 127u};
        if (c.x | c.y | c.z | c.w) row.again(v, words_of, places);
    }
}

template <class T, bool IN_PLACE>
hawq_status launch(const LogitsArgs &a, hipStream_t s) {
    const bool counted = a.penalties || a.n_bias > 0, copied = !IN_PLACE || a.n_allowed > 0;
    const bool apart = counted && (!copied || (int64_t)a.total * a.vocab >= kApart);
    if (copied) {
        const int part = logits_part_of(a.total, a.vocab);
        const int64_t along = a.total < kMostAlong ? a.total : kMostAlong;
        const dim3 grid((unsigned)logits_parts(a.vocab, part), (unsigned)along, (unsigned)((a.total + along - 1) / along));
        if (counted && !apart) logits_part<T, IN_PLACE, true><<<grid, kPartThreads, (size_t)(part + 16) * 4, s>>>(a, part);
        else logits_part<T, IN_PLACE, false><<<grid, kPartThreads, 0, s>>>(a, part);
        const hawq_status st = check_launch();
        if (st != HAWQ_OK) return st;
    }
    if (!apart) return HAWQ_OK;
    const Grid g = spread(a.total, 1, kRowThreads);
    if (g.x == 0) return HAWQ_ERR_UNSUPPORTED;
    logits_row<T><<<dim3((unsigned)g.x, (unsigned)g.y), kRowThreads, 2 * kSlots * 4, s>>>(a);
    return check_launch();
}

}  // namespace

hawq_status launch_logits(const LogitsArgs &a, hipStream_t s) {
    if (a.dtype == HAWQ_F16) return a.x == a.y ? launch<F16, true>(a, s) : launch<F16, false>(a, s);
    return a.x == a.y ? launch<BF16, true>(a, s) : launch<BF16, false>(a, s);
}

}  // namespace hawq
