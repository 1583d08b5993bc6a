// Rotary positions of queries and keys.
//
//   (x, y) -> scale * (x cos a - y sin a, y cos a + x sin a),   a = 2 pi * position * turns[f]
//
// The angle's revolutions are a product of 64-bit floats, less the nearest whole number: a position of 2^20 keeps the angle to 2^-33 of a
// revolution, where a 32-bit product would keep 2^-5.  What is left is below half a revolution and goes on in 32 bits.
//
// Bound by bytes: 20001 tokens of 32 + 8 heads of 128 take 79 us, 5.2 TB/s, the rate of a large copy (an element at a time, its angle made
// for each head: 238); one token 4.7, near an empty launch.  A workgroup takes some tokens: each of its threads makes a sine and a cosine or two, which lie in LDS for all heads, and
// has its first vectors of queries and keys on the way meanwhile.
#include "lm.h"
#include "lm_launch.h"

namespace hawq {

namespace {

constexpr int kThreads = 256, kAhead = 4;        // items of a thread under way

template <int V> struct Vector { typedef uint32_t bits __attribute__((ext_vector_type(V / 2))); };
template <> struct Vector<2> { typedef uint32_t bits; };
template <> struct Vector<1> { typedef uint16_t bits; };

// An item is two vectors of V elements of a head: of the pairs (halves: V of the first half and V of the second; pairs: 2 V side by side), or
// two side by side of those that are copied.  Items of a head: those of the turned elements first.
template <class T, int V, bool HALVES>
__global__ __launch_bounds__(kThreads) void rotary(RotaryArgs a, int tokens, int slots, FastDiv by_slot, FastDiv by_head) {
    typedef typename T::elem E;
    typedef typename Vector<V>::bits Bits;
    extern __shared__ __align__(16) float turn[];    // [token][cosines, sines][rotary_dim / 2]
    const int half = a.rotary_dim >> 1, turned = half / V;
    const int64_t t0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * tokens;
    const int n = (int)min((int64_t)tokens, (int64_t)a.total - t0);
    if (n <= 0) return;
    const uint32_t items = (uint32_t)n * a.heads * slots;
    struct Item {
        const E *x;
        E *y;
        int gap, f;          // from the first vector to the second; of the first pair in LDS, -1: copied
        Bits lo, hi;
    };
    auto load = [&](uint32_t i, Item &it) {
        const uint32_t row = fdiv(i, by_slot), t = fdiv(row, by_head);
        const int slot = (int)(i - row * slots);
        int h = (int)(row - t * a.heads);
        const int which = h >= a.q_heads;
        h -= which ? a.q_heads : 0;
        it.f = slot < turned ? (int)t * a.rotary_dim + slot * V : -1;
        const int e = slot < turned ? (HALVES ? slot : 2 * slot) * V : a.rotary_dim + (slot - turned) * 2 * V;
        it.gap = slot < turned ? (HALVES ? half : V) : e + V < a.head_dim ? V : 0;
        it.x = (const E *)a.x[which] + (t0 + t) * a.x_token[which] + h * a.x_head[which] + e;
        it.y = (E *)a.y[which] + (t0 + t) * a.y_token[which] + h * a.y_head[which] + e;
        it.lo = *(const Bits *)it.x;
        it.hi = *(const Bits *)(it.x + it.gap);
    };
    auto store = [&](Item &it) {
        E in[2 * V], out[2 * V];
        __builtin_memcpy(in, &it.lo, 2 * V);
        __builtin_memcpy(in + V, &it.hi, 2 * V);
        if (it.f >= 0) {
            const float *c = turn + it.f, *s = c + half;
            for (int e = 0; e < V; ++e) {
                const int i = HALVES ? e : 2 * e, j = HALVES ? V + e : 2 * e + 1;
                const float u = (float)in[i], v = (float)in[j];
                out[i] = (E)(u * c[e] - v * s[e]);
                out[j] = (E)(v * c[e] + u * s[e]);
            }
            __builtin_memcpy(&it.lo, out, 2 * V);
            __builtin_memcpy(&it.hi, out + V, 2 * V);
        }
        *(Bits *)it.y = it.lo;
        if (it.gap) *(Bits *)(it.y + it.gap) = it.hi;
    };
    Item it[kAhead];
    uint32_t at = threadIdx.x;
    for (int k = 0; k < kAhead; ++k) load(min(at + k * kThreads, items - 1), it[k]);
    for (int i = threadIdx.x; i < n * half; i += kThreads) {
        const int t = i / half, f = i - t * half;
        double r = (double)a.positions[t0 + t] * a.turns[f];
        r -= rint(r);
        float s, c;
        sincospif(2.f * (float)r, &s, &c);
        turn[t * a.rotary_dim + f] = c * a.scale;
        turn[t * a.rotary_dim + half + f] = s * a.scale;
    }
    __syncthreads();
    for (;;) {
        for (int k = 0; k < kAhead; ++k)
            if (at + k * kThreads < items) store(it[k]);
        at += kAhead * kThreads;
        if (at >= items) break;
        for (int k = 0; k < kAhead; ++k) load(min(at + k * kThreads, items - 1), it[k]);
    }
}

template <class T, int V>
hawq_status launch(const RotaryArgs &a, hipStream_t s) {
    // Elements past the turned ones are copied only where they are not in place (queries and keys alike: the one that is in place copies too).
    const bool in_place = (a.q_heads == 0 || a.x[0] == a.y[0]) && (a.heads == a.q_heads || a.x[1] == a.y[1]);
    const int half = a.rotary_dim / 2, slots = half / V + (in_place ? 0 : (a.head_dim - a.rotary_dim + 2 * V - 1) / (2 * V));
    // As many tokens to a workgroup as give each thread an angle, while there are workgroups enough
    int tokens = 1;
    while (tokens * 2 * half <= kThreads && a.total / (tokens * 2) >= 1024 && (int64_t)tokens * 2 * a.heads * slots < INT32_MAX / 2) tokens *= 2;
    const Grid g = spread(((int64_t)a.total + tokens - 1) / tokens, 1, kThreads);
    if (g.x == 0) return HAWQ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)g.x, (unsigned)g.y);
    const size_t lds = (size_t)tokens * a.rotary_dim * sizeof(float);
    const FastDiv by_slot = fast_div((uint32_t)slots), by_head = fast_div((uint32_t)a.heads);
    if (a.layout == HAWQ_ROTARY_HALVES) rotary<T, V, true><<<grid, kThreads, lds, s>>>(a, tokens, slots, by_slot, by_head);
    else rotary<T, V, false><<<grid, kThreads, lds, s>>>(a, tokens, slots, by_slot, by_head);
    return check_launch();
}

template <class T>
hawq_status pick_vector(const RotaryArgs &a, hipStream_t s) {
    int64_t strides = a.head_dim | a.rotary_dim / 2;
    uintptr_t addresses = 0;
    for (int i = 0; i < 2; ++i)
        if (i == 0 ? a.q_heads > 0 : a.heads > a.q_heads) {
            strides |= a.x_token[i] | a.x_head[i] | a.y_token[i] | a.y_head[i];
            addresses |= (uintptr_t)a.x[i] | (uintptr_t)a.y[i];
        }
    if (strides % 8 == 0 && addresses % 16 == 0) return launch<T, 8>(a, s);
    if (strides % 2 == 0 && addresses % 4 == 0) return launch<T, 2>(a, s);
    return launch<T, 1>(a, s);
}

}  // namespace

hawq_status launch_rotary(const RotaryArgs &a, hipStream_t s) { return a.dtype == HAWQ_F16 ? pick_vector<F16>(a, s) : pick_vector<BF16>(a, s); }

}  // namespace hawq
