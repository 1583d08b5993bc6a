"""Argument checks of rotary positions, gated projections, adapters and logits processing, on the host: a refused call has a code and enqueues
nothing (there is no GPU to enqueue to)."""
import ctypes

import pytest

OK, NULL, SHAPE, DTYPE, RANGE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4, 6, 8
P = ctypes.c_void_p(4096)
Q = ctypes.c_void_p(8192)
ODD = ctypes.c_void_p(4097)
TWO = ctypes.c_void_p(4098)
FOUR = ctypes.c_void_p(4100)


@pytest.fixture(scope="module")
def lib():
    import paper_2011_10680_amd as hawq
    from paper_2011_10680_amd import build
    if build.is_stale():
        build.build()
    return hawq.load_library()


def test_rotary(lib):
    import paper_2011_10680_amd as hawq
    base = dict(total=5, q_heads=4, kv_heads=2, head_dim=64, rotary_dim=32, layout=hawq.ROTARY_HALVES, dtype=hawq.BF16, scale=1.0, q_token=256, q_head=64, k_token=128, k_head=64,
                yq_token=256, yq_head=64, yk_token=128, yk_head=64)

    def call(**kw):
        args = [kw.pop(n, v) for n, v in (("q", P), ("k", P), ("positions", P), ("turns", P), ("yq", Q), ("yk", Q))]
        return lib.hawq_rotary(ctypes.byref(hawq.RotaryDesc(**dict(base, **kw))), *args, None)
    assert lib.hawq_rotary(None, *[P] * 6, None) == NULL
    assert call(total=0, q=None, yq=None) == OK and call(q_heads=0, kv_heads=0, q=None) == OK
    assert call(total=0, q=None, yq=None, q_token=512) == OK
    for name in ("q", "k", "positions", "turns", "yq", "yk"):
        assert call(**{name: None}) == NULL, name
    for kw in (dict(total=-1), dict(q_heads=-1), dict(kv_heads=-1), dict(head_dim=0), dict(head_dim=257), dict(rotary_dim=0), dict(rotary_dim=31), dict(rotary_dim=66), dict(q_token=-1),
               dict(k_head=-1), dict(yq_token=255), dict(yq_head=63), dict(yk_token=0), dict(k_token=1 << 41), dict(q=Q, q_token=512), dict(yk=P, yk_head=65, yk_token=256)):
        assert call(**kw) == SHAPE, kw
    for dt in (hawq.S8, 7):
        assert call(dtype=dt) == DTYPE
    for kw in (dict(scale=float("nan")), dict(scale=float("inf")), dict(layout=2), dict(layout=-1)):
        assert call(**kw) == RANGE, kw
    for kw in (dict(q=ODD), dict(yk=ODD), dict(positions=TWO), dict(turns=FOUR), dict(q_heads=65536, q_token=1 << 23, yq_token=1 << 23)):
        assert call(**kw) == UNSUPPORTED, kw


def test_gated(lib):
    import paper_2011_10680_amd as hawq
    base = dict(M=1, N=16, K=64, group=32, x_dtype=hawq.F16, w_dtype=hawq.S4, activation=hawq.SILU, x_stride=64, y_stride=16)

    def call(x=P, w=P, scales=P, zeros=None, bias=None, y=P, workspace=P, bytes=1 << 40, **kw):
        return lib.hawq_gated_w4(ctypes.byref(hawq.GatedW4Desc(**dict(base, **kw))), x, w, scales, zeros, bias, y, workspace, bytes, None)
    assert lib.hawq_gated_w4(None, *[P] * 7, 0, None) == NULL
    assert call(M=0) == OK and call(M=0, x=None, y=None) == OK
    for name in ("x", "w", "scales", "y"):
        assert call(**{name: None}) == NULL, name
    for kw in (dict(M=-1), dict(N=0), dict(N=(1 << 30) + 1, y_stride=1 << 31), dict(K=0), dict(K=63), dict(group=0), dict(group=48), dict(group=-32), dict(x_stride=63), dict(y_stride=15),
               dict(x_stride=-1), dict(x_stride=1 << 41)):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(x_dtype=hawq.S8), dict(x_dtype=9), dict(w_dtype=hawq.S8), dict(zeros=P)):
        assert call(**kw) == DTYPE, kw
    assert call(activation=-1) == RANGE and call(activation=4) == RANGE
    assert call(w_dtype=hawq.U4) == NULL
    for name in ("x", "scales", "bias", "y"):
        assert call(**{name: ODD}) == UNSUPPORTED, name
    assert call(K=(1 << 25) + 2, x_stride=1 << 26) == UNSUPPORTED
    assert hawq.hawq_gated_w4_workspace_bytes(hawq.GatedW4Desc(**dict(base, M=-1))) == 0
    wide = dict(base, M=4000, N=4096, K=4096, x_stride=4096, y_stride=4096)
    need = hawq.hawq_gated_w4_workspace_bytes(hawq.GatedW4Desc(**wide))
    for M in ((1 << 29) + 1, (1 << 31) - 4096):         # more rows than a launch of the prompts' form has workgroups for
        assert hawq.hawq_gated_w4_workspace_bytes(hawq.GatedW4Desc(**dict(wide, M=M, x_stride=0))) == 0
    if need:
        assert call(bytes=need - 1, **wide) == WORKSPACE and call(workspace=None, **wide) == NULL and call(workspace=ctypes.c_void_p(4104), **wide) == UNSUPPORTED


def test_adapters(lib):
    import paper_2011_10680_amd as hawq
    base = dict(M=4, N=16, K=64, n_adapters=2, max_rank=8, dtype=hawq.BF16, x_stride=64, base_stride=16, y_stride=16, a_adapter=512, a_row=64, b_adapter=128, b_row=8)
    names = ("x", "a", "b", "ranks", "scales", "adapter", "base", "y", "workspace")

    def call(bytes=1 << 40, **kw):
        args = [kw.pop(n, Q if n == "y" else P) for n in names]
        return lib.hawq_adapters(ctypes.byref(hawq.AdaptersDesc(**dict(base, **kw))), *args, bytes, None)
    assert lib.hawq_adapters(None, *[P] * 9, 0, None) == NULL
    assert call(M=0, x=None, base=None, y=None, y_stride=32) == OK
    for name in names:
        assert call(**{name: None}) == NULL, name
    for kw in (dict(M=-1), dict(N=0), dict(K=0), dict(n_adapters=-1), dict(max_rank=0), dict(x_stride=63), dict(base_stride=15), dict(y_stride=15), dict(y_stride=0), dict(a_row=63),
               dict(b_row=7), dict(a_adapter=-1), dict(b_adapter=1 << 41), dict(y=P, y_stride=32)):
        assert call(**kw) == SHAPE, kw
    assert call(dtype=hawq.S32) == DTYPE
    for kw in (dict(x=ODD), dict(a=ODD), dict(b=ODD), dict(base=ODD), dict(y=ODD), dict(ranks=TWO), dict(scales=TWO), dict(adapter=TWO), dict(workspace=ctypes.c_void_p(4104)),
               dict(max_rank=(1 << 16) + 1, b_row=1 << 17)):
        assert call(**kw) == UNSUPPORTED, kw
    need = hawq.hawq_adapters_workspace_bytes(hawq.AdaptersDesc(**base))
    assert need > 0 and call(bytes=need - 1) == WORKSPACE
    assert hawq.hawq_adapters_workspace_bytes(hawq.AdaptersDesc(**dict(base, K=-1))) == 0


def test_logits(lib):
    import paper_2011_10680_amd as hawq
    base = dict(n_seqs=2, total=5, vocab=100, dtype=hawq.F16, past_stride=9, n_bias=3, n_allowed=2, allowed_stride=4, x_stride=100, y_stride=104)
    names = ("x", "past", "past_lens", "prompt_lens", "starts", "drafts", "mask", "penalties", "bias_starts", "bias_ids", "bias_values", "allowed", "allowed_row", "y")

    def call(**kw):
        args = [kw.pop(n, Q if n == "y" else P) for n in names]
        return lib.hawq_logits(ctypes.byref(hawq.LogitsDesc(**dict(base, **kw))), *args, None)
    assert lib.hawq_logits(None, *[P] * 15) == NULL
    assert call(n_seqs=0) == OK and call(total=0, x=None, y=None) == OK
    for name in ("x", "y", "past", "past_lens", "bias_starts", "bias_ids", "bias_values", "allowed"):
        assert call(**{name: None}) == NULL, name
    for kw in (dict(n_seqs=-1), dict(total=-1), dict(vocab=0), dict(past_stride=-1), dict(n_bias=-1), dict(n_allowed=-1), dict(x_stride=99), dict(y_stride=99), dict(y_stride=0),
               dict(allowed_stride=3), dict(starts=None), dict(allowed_row=None), dict(y=P)):
        assert call(**kw) == SHAPE, kw
    assert call(dtype=hawq.S8) == DTYPE
    for kw in (dict(x=ODD), dict(y=ODD), dict(past=TWO), dict(past_lens=TWO), dict(prompt_lens=TWO), dict(starts=TWO), dict(drafts=TWO), dict(mask=FOUR), dict(penalties=TWO),
               dict(bias_starts=TWO), dict(bias_ids=TWO), dict(bias_values=TWO), dict(allowed=TWO), dict(allowed_row=TWO)):
        assert call(**kw) == UNSUPPORTED, kw
