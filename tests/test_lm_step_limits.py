"""Where rotary positions, gated projections, adapters and logits processing end, on the host: one more than the largest is refused, with nothing enqueued."""
import ctypes

import pytest

NULL, UNSUPPORTED, WORKSPACE = 1, 6, 8
P, Q = ctypes.c_void_p(4096), ctypes.c_void_p(8192)
MOST = (1 << 31) - 4096


@pytest.fixture(scope="module")
def hawq():
    import paper_2011_10680_amd as hawq
    from paper_2011_10680_amd import build
    if build.is_stale():
        build.build()
    hawq.load_library()
    return hawq


@pytest.mark.parametrize("change", [dict(total=1 << 23), dict(past_stride=1 << 23), dict(vocab=MOST + 1, x_stride=1 << 31, y_stride=1 << 31)])
def test_logits(hawq, change):
    base = dict(n_seqs=2, total=5, vocab=100, dtype=hawq.F16, past_stride=9, n_bias=0, n_allowed=0, allowed_stride=0, x_stride=100, y_stride=104)
    d = hawq.LogitsDesc(**dict(base, **change))
    assert hawq.load_library().hawq_logits(ctypes.byref(d), P, P, P, P, P, P, P, P, None, None, None, None, None, Q, None) == UNSUPPORTED


@pytest.mark.parametrize("change", [dict(M=MOST + 1), dict(N=MOST + 1, base_stride=1 << 31, y_stride=1 << 31), dict(K=MOST + 1, x_stride=1 << 31, a_row=1 << 31)])
def test_adapters(hawq, change):
    base = dict(M=4, N=16, K=64, n_adapters=2, max_rank=8, dtype=hawq.BF16, x_stride=64, base_stride=16, y_stride=16, a_adapter=512, a_row=64, b_adapter=128, b_row=8)
    d = hawq.AdaptersDesc(**dict(base, **change))
    assert hawq.hawq_adapters_workspace_bytes(d) == 0
    assert hawq.load_library().hawq_adapters(ctypes.byref(d), P, P, P, P, P, P, P, Q, P, 1 << 60, None) == UNSUPPORTED


def test_gated(hawq):
    base = dict(M=4000, N=4096, K=4096, group=128, x_dtype=hawq.F16, w_dtype=hawq.S4, activation=hawq.SILU, x_stride=4096, y_stride=4096)

    def call(workspace=P, bytes=1 << 60, **kw):
        return hawq.load_library().hawq_gated_w4(ctypes.byref(hawq.GatedW4Desc(**dict(base, **kw))), P, P, P, None, None, Q, workspace, bytes, None)
    need = hawq.hawq_gated_w4_workspace_bytes(hawq.GatedW4Desc(**base))
    assert need > 0                                    # (else the three calls below would be made)
    assert call(bytes=need - 1) == WORKSPACE and call(workspace=None) == NULL and call(workspace=ctypes.c_void_p(4104)) == UNSUPPORTED
    assert call(M=MOST + 1) == UNSUPPORTED
