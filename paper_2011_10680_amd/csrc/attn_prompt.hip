// Causal attention over packed prompts.
#include "attn_any.h"

namespace hawq {

namespace {

template <class T>
__global__ __launch_bounds__(64) void attn_prompt_any(AttnPromptArgs a) {
    typedef typename T::elem E;
    __shared__ float q_lds[256];
    const int row = blockIdx.x, h = blockIdx.y, hk = h / (a.q_heads / a.kv_heads);
    int from = 0, to = 0;
    // the sequence that holds the row: the last one that begins at or before it (empty ones in between hold nothing)
    int lo = 0, hi = a.n_seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.starts[mid] <= row) lo = mid; else hi = mid - 1;
    }
    sequence_rows(a.starts, lo, a.total, from, to);
    if (row < from || row >= to) return;
    attend_row<T>((const E *)a.q + row * a.q_token + h * a.q_head, (E *)a.y + row * a.y_token + h * a.y_head, a.head_dim, a.scale, row - from + 1, q_lds,
                  [&](int j) -> KeyRow { return {(const E *)a.k + (from + j) * a.k_token + hk * a.k_head, (const E *)a.v + (from + j) * a.v_token + hk * a.v_head, 1.f, 1.f, false}; },
                  [](int) { return true; });
}

}  // namespace

hawq_status launch_attn_prompt(const AttnPromptArgs &a, hipStream_t s) {
    if (a.q_heads > 65535) return HAWQ_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)a.total, (unsigned)a.q_heads);
    if (a.dtype == HAWQ_F16) attn_prompt_any<F16><<<grid, 64, 0, s>>>(a);
    else attn_prompt_any<BF16><<<grid, 64, 0, s>>>(a);
    return check_launch();
}

}  // namespace hawq
