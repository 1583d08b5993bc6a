// What a server does to the logits before it chooses: penalties for tokens that occurred, biases, grammar masks.
//
// A workgroup takes a part of the vocabulary for one row.  It copies the part with the mask applied, eight logits to a thread, in place only
// what the mask takes away; that waits for nothing but the mask.  Meanwhile it counts the past tokens of the row's request that fall into the
// part in LDS, one word a token (bit 31: occurred; bits 24 to 30: its place in a short list of biases; below: how often the model wrote it), and
// the drafted tokens that the row sees.  Whoever counted a token then takes its word away: the first one writes the token's logit again.  With a
// long list the part is counted in two halves, the second half of LDS holding the places.  Integer counts and maxima: the order of the atomics
// does not matter.
//
// Bound by the logits' bytes for many rows, by a chain of loads (request, lengths, tokens) and a launch for few.
#include "lm.h"
#include "lm_launch.h"

namespace hawq {

namespace {

constexpr uint32_t kOccurred = 0x80000000u, kPlace = 0x7F000000u, kCount = 0x00FFFFFFu;
constexpr int kThreads = 512, kAhead = 4;        // eights of a thread on their way while the tokens are counted
constexpr int kFewBiases = 127, kTokens = 4;     // tokens of a thread under way

// The request whose rows t belongs to, -1: none.  64 places at a time: the lengths' chain of loads is one or two long.
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

// the larger of a word's place (bits 24 to 30) and this one, beside whatever else changes the word
__device__ __forceinline__ void highest(uint32_t *word, uint32_t place) {
    uint32_t had = *(volatile uint32_t *)word;
    while ((had >> 24 & 127u) < place) {
        const uint32_t now = atomicCAS(word, had, (had & ~kPlace) | place << 24);
        if (now == had) return;
        had = now;
    }
}

// IN_PLACE: y is x, and what does not change is neither read nor written.
template <class T, bool IN_PLACE>
__global__ __launch_bounds__(kThreads) void logits_part(LogitsArgs a, int part) {
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
            const int k = threadIdx.x + i * kThreads;
            if (k < eights && whole(k)) ahead[i] = *(const Eight *)(x + (8 * k - off));
        }
    const int b = request_of(a, t);
    if (b < 0) return;
    // what is known of the request, all at once: every load that waits for another costs a microsecond
    const int64_t pen = 3 * (int64_t)b;
    const float r = a.penalties ? a.penalties[pen] : 1.f, presence = a.penalties ? a.penalties[pen + 1] : 0.f, frequency = a.penalties ? a.penalties[pen + 2] : 0.f;
    const int first_bias = a.n_bias > 0 ? min(max(a.bias_starts[b], 0), a.n_bias) : 0, last_bias = a.n_bias > 0 ? min(max(a.bias_starts[b + 1], first_bias), a.n_bias) : 0;
    const int len = a.past_stride > 0 ? min(max(a.past_lens[b], 0), a.past_stride) : 0, prompt = a.past_stride > 0 && a.prompt_lens ? a.prompt_lens[b] : 0;
    const int mask_row = a.n_allowed == 0 ? -1 : a.allowed_row ? a.allowed_row[t] : t;
    int from = t, to = t + 1;
    if (a.drafts && a.starts) sequence_rows(a.starts, b, a.total, from, to);
    const uint64_t sees = a.drafts && a.mask ? a.mask[t] : ~0ull;
    const int seen = !a.drafts ? 0 : a.mask ? min(to - from, 64) : t + 1 - from;
    const bool counts = r != 1.f || presence != 0.f || frequency != 0.f, biases = last_bias > first_bias;
    const uint32_t *const allowed = mask_row >= 0 && mask_row < a.n_allowed ? a.allowed + mask_row * a.allowed_stride : nullptr;
    const int32_t *const past = a.past + (int64_t)b * a.past_stride;
    const int32_t listed = biases ? a.bias_ids[min(first_bias + (int)threadIdx.x, last_bias - 1)] : -1, draft = seen > 0 ? a.drafts[from + min((int)threadIdx.x, seen - 1)] : -1;
    // this thread's tokens from i0 on, -1 past the last; the first ones
    struct Tokens { int32_t id[kTokens]; };
    auto read = [&](int i0) {
        Tokens k;
        for (int i = 0; i < kTokens; ++i) {
            const int p = i0 + i * kThreads + (int)threadIdx.x;
            k.id[i] = past[min(p, len - 1)];
            if (p >= len) k.id[i] = -1;
        }
        return k;
    };
    Tokens head;
    if (counts && len > 0) head = read(0);
    auto may = [&](int v) { return !allowed || (allowed[v >> 5] >> (v & 31) & 1); };
    auto copy = [&](int k, Eight d) {
        const int at = 8 * k - off;              // of the eight's first element in the part
        if (!whole(k)) {
            for (int i = max(at, 0); i < min(at + 8, n); ++i) {
                const bool kept = may(v0 + i);
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
    if (!IN_PLACE || allowed)
        for (int i = 0; i < kAhead; ++i) {
            const int k = threadIdx.x + i * kThreads;
            if (k < eights) copy(k, ahead[i]);
        }
    if (!IN_PLACE || allowed)
        for (int k = threadIdx.x + kAhead * kThreads; k < eights; k += kThreads) {
            Eight d{0, 0, 0, 0};
            if (!IN_PLACE && whole(k)) d = *(const Eight *)(x + (8 * k - off));
            copy(k, d);
        }
    if (!counts && !biases) return;

    const bool places = last_bias - first_bias > kFewBiases;
    const int per = places ? (part + 1) >> 1 : part;
    uint32_t *const count = words, *const place = words + per;              // place: i + 1 for entry i of the list
    for (int first = 0; first < n; first += per) {
        const int some = min(per, n - first);                               // tokens v0 + first and on
        for (int i = threadIdx.x; i < (part + 4) / 4; i += kThreads) ((v4u *)words)[i] = v4u{0, 0, 0, 0};
        __syncthreads();
        auto place_of = [&](int32_t token) { return (uint32_t)token - (uint32_t)(v0 + first); };      // below `some` if it is one of these
        // bit i: token i is one of these
        auto hits_of = [&](const Tokens &k) {
            uint32_t hits = 0;
            for (int i = 0; i < kTokens; ++i) hits |= place_of(k.id[i]) < (uint32_t)some ? 1u << i : 0u;
            return hits;
        };
        auto tally = [&](const Tokens &k, int i0) {
            const uint32_t hits = hits_of(k);
            if (hits)
                for (int i = 0; i < kTokens; ++i)
                    if (hits >> i & 1) {
                        uint32_t *const word = count + place_of(k.id[i]);
                        if (i0 + i * kThreads + (int)threadIdx.x >= prompt) atomicAdd(word, 1u);
                        atomicOr(word, kOccurred);
                    }
        };
        // the logit of a token whose word c was taken away
        auto again = [&](uint32_t at, uint32_t c) {
            const int e = first + (int)at;
            const E l = x[e];
            const float bias = c & kPlace ? a.bias_values[first_bias + (int)(places ? place[at] : c >> 24 & 127u) - 1] : 0.f;
            if (!may(v0 + e)) return;
            float v = (float)l;
            if (c & kOccurred) v = v > 0 ? v / r : v * r;
            if (c & kCount) v = v - frequency * (float)(c & kCount) - presence;
            if (c & kPlace) v += bias;
            y[e] = (E)v;
        };
        auto settle = [&](const Tokens &k) {
            const uint32_t hits = hits_of(k);
            if (hits) {
                uint32_t c[kTokens];
                for (int i = 0; i < kTokens; ++i) c[i] = hits >> i & 1 ? atomicExch(count + place_of(k.id[i]), 0u) : 0u;
                for (int i = 0; i < kTokens; ++i)
                    if (c[i]) again(place_of(k.id[i]), c[i]);
            }
        };
        auto settle_one = [&](int32_t token) {
            const uint32_t at = place_of(token), c = at < (uint32_t)some ? atomicExch(count + at, 0u) : 0u;
            if (c) again(at, c);
        };
        for (int i = threadIdx.x; i < last_bias - first_bias; i += kThreads) {
            const uint32_t at = place_of(i < kThreads ? listed : a.bias_ids[first_bias + i]);
            if (at >= (uint32_t)some) continue;
            if (places) atomicMax(place + at, (uint32_t)i + 1), atomicOr(count + at, 1u << 24);
            else highest(count + at, (uint32_t)i + 1);
        }
        if (counts) {
            for (int i = threadIdx.x; i < seen; i += kThreads) {
                const uint32_t at = place_of(i < kThreads ? draft : a.drafts[from + i]);
                if (at < (uint32_t)some && (!a.mask || (sees >> i & 1))) {
                    atomicAdd(count + at, 1u);
                    atomicOr(count + at, kOccurred);
                }
            }
            if (len > 0) tally(head, 0);
            for (int i0 = kTokens * kThreads; i0 < len; i0 += kTokens * kThreads) tally(read(i0), i0);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < last_bias - first_bias; i += kThreads) settle_one(i < kThreads ? listed : a.bias_ids[first_bias + i]);
        if (counts) {
            for (int i = threadIdx.x; i < seen; i += kThreads) settle_one(i < kThreads ? draft : a.drafts[from + i]);
            if (len > 0) settle(head);
            for (int i0 = kTokens * kThreads; i0 < len; i0 += kTokens * kThreads) settle(read(i0));
        }
        if (first + per < n) __syncthreads();
    }
}

}  // namespace

hawq_status launch_logits(const LogitsArgs &a, hipStream_t s) {
    // parts of 16384 tokens, smaller ones where that gives the 256 compute units less than four each
    int part = 16384;
    while (part > 1024 && (int64_t)a.total * ((a.vocab + part - 1) / part) < 1024) part /= 2;
    const int64_t along = a.total < kMostAlong ? a.total : kMostAlong;
    const dim3 grid((unsigned)(((int64_t)a.vocab + part - 1) / part), (unsigned)along, (unsigned)((a.total + along - 1) / along));
    const size_t lds = (size_t)(part + 32) * 4;
    const bool in_place = a.x == a.y;
    if (a.dtype == HAWQ_F16) {
        if (in_place) logits_part<F16, true><<<grid, kThreads, lds, s>>>(a, part);
        else logits_part<F16, false><<<grid, kThreads, lds, s>>>(a, part);
    } else {
        if (in_place) logits_part<BF16, true><<<grid, kThreads, lds, s>>>(a, part);
        else logits_part<BF16, false><<<grid, kThreads, lds, s>>>(a, part);
    }
    return check_launch();
}

}  // namespace hawq
