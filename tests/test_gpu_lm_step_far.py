"""Rotary positions, gated projections, adapters and logits with rows that lie more than 2^31 elements apart or behind: the same as with rows side by side.
Other strides may take another form of a kernel, so a result may be rounded the other way: a step of the type."""
import pytest

pytestmark = pytest.mark.gpu


def _far(t, stride):
    """A copy of t [rows, ...] with its rows `stride` elements apart; what lies between is whatever the memory held."""
    import torch
    out = torch.empty((t.shape[0] - 1) * stride + t[0].numel(), dtype=t.dtype, device="cuda").as_strided(t.shape, (stride,) + t.stride()[1:])
    out.copy_(t)
    return out


@pytest.mark.parametrize("tokens,stride", [(3, (1 << 31) + 8), (3, (1 << 31) + 2), (2, (1 << 32) + 1), (70, 1 << 25)])
@pytest.mark.parametrize("in_place", [False, True])
def test_rotary(tokens, stride, in_place):
    import torch
    import paper_2011_10680_amd as hawq
    q, k = torch.randn((tokens, 2, 64), device="cuda").half(), torch.randn((tokens, 1, 64), device="cuda").half()
    pos, turns = torch.arange(tokens, dtype=torch.int32, device="cuda") * 77, torch.rand(16, dtype=torch.float64, device="cuda")

    def run(q, k, yq, yk):
        d = hawq.RotaryDesc(total=tokens, q_heads=2, kv_heads=1, head_dim=64, rotary_dim=32, layout=hawq.ROTARY_HALVES, dtype=hawq.F16, scale=1.0, q_token=q.stride(0), q_head=64,
                            k_token=k.stride(0), k_head=64, yq_token=yq.stride(0), yq_head=64, yk_token=yk.stride(0), yk_head=64)
        hawq.hawq_rotary(d, q, k, pos, turns, yq, yk)
        torch.cuda.synchronize()
        return yq, yk
    want = run(q, k, torch.empty_like(q), torch.empty_like(k))
    fq, fk = _far(q, stride), _far(k, stride)
    got = run(fq, fk, *((fq, fk) if in_place else (_far(torch.zeros_like(q), stride), _far(torch.zeros_like(k), stride))))
    for g, v in zip(got, want):                  # (a step of f16; where the two products cancel, 32 bits' steps of values up to 8)
        assert torch.allclose(g.float(), v.float(), rtol=2 ** -10, atol=2 ** -20)


@pytest.mark.parametrize("M,N,K,x_stride,y_stride", [(3, 48, 256, (1 << 31) + 8, (1 << 31) + 1), (20, 100, 64, 1 << 27, 1 << 27), (300, 9000, 512, 1 << 22, (1 << 23) + 1),
                                                     (1040, 2113, 160, 1 << 21, 1 << 21)])
def test_gated(M, N, K, x_stride, y_stride):
    import torch
    import paper_2011_10680_amd as hawq
    x, w = torch.randn((M, K), device="cuda").half(), torch.randint(0, 256, (2 * N, K // 2), dtype=torch.uint8, device="cuda")
    scales = torch.rand((2 * N, -(-K // 128)), device="cuda").half() / 50

    def run(x, y):
        d = hawq.GatedW4Desc(M=M, N=N, K=K, group=128, x_dtype=hawq.F16, w_dtype=hawq.S4, activation=hawq.SILU, x_stride=x.stride(0), y_stride=y.stride(0))
        n = hawq.hawq_gated_w4_workspace_bytes(d)
        hawq.hawq_gated_w4(d, x, w, scales, None, None, y, torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
        torch.cuda.synchronize()
        return y
    want = run(x, torch.empty((M, N), dtype=torch.float16, device="cuda")).float()
    got = run(_far(x, x_stride), _far(torch.zeros((M, N), dtype=torch.float16, device="cuda"), y_stride)).float()
    # Two roundings to f16, and sums in another order: up to 512 steps of 2^-24 of a running sum of 2 x 512 terms of 31 |x| |s|, 0.25 in the mean, make
    # 0.008 of g or u, times the other (5 at most) 0.04; the largest of millions of products of two such is 10 or more.
    assert torch.allclose(got, want, rtol=2 ** -9, atol=4e-3 * float(want.abs().max()))


@pytest.mark.parametrize("M,x_stride,y_stride", [(3, (1 << 31) + 8, (1 << 31) + 8), (3, (1 << 31) + 1, (1 << 32) + 3), (70, 1 << 25, 1 << 25), (4100, 1 << 20, 1 << 20)])
@pytest.mark.parametrize("in_place", [False, True])
def test_adapters(M, x_stride, y_stride, in_place):
    import torch
    import paper_2011_10680_amd as hawq
    N, K, n, R = 100, 72, 3, 16
    x, base = torch.randn((M, K), device="cuda").bfloat16(), torch.randn((M, N), device="cuda").bfloat16()
    a, b = torch.randn((n, R, K), device="cuda").bfloat16(), torch.randn((n, N, R), device="cuda").bfloat16()
    ranks, scales = torch.tensor([16, 3, 9], dtype=torch.int32, device="cuda"), torch.rand(n, device="cuda")
    adapter = torch.randint(-1, n, (M,), device="cuda").int()

    def run(x, base, y, a, b):
        d = hawq.AdaptersDesc(M=M, N=N, K=K, n_adapters=n, max_rank=R, dtype=hawq.BF16, x_stride=x.stride(0), base_stride=base.stride(0), y_stride=y.stride(0), a_adapter=a.stride(0),
                              a_row=a.stride(1), b_adapter=b.stride(0), b_row=b.stride(1))
        hawq.hawq_adapters(d, x, a, b, ranks, scales, adapter, base, y, torch.empty(hawq.hawq_adapters_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        return y
    want = run(x, base, torch.empty_like(base), a, b)
    far = _far(base, y_stride)
    got = run(_far(x, x_stride), far, far if in_place else _far(torch.zeros_like(base), y_stride), *((_far(a, x_stride), _far(b, x_stride)) if M == 3 else (a, b)))
    assert torch.allclose(got.float(), want.float(), rtol=2 ** -7, atol=2 ** -12)      # (a step of bf16, 32 bits' steps of values up to 500)


@pytest.mark.parametrize("n,stride,past_stride,allowed_stride", [(3, (1 << 31) + 8, 20, 1 << 30), (3, (1 << 31) + 1, 20, 64), (300, 1 << 23, (1 << 23) - 1, 64)])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("masks", [0, 3])
def test_logits(n, stride, past_stride, allowed_stride, in_place, masks):
    import torch
    import paper_2011_10680_amd as hawq
    V, most = 1500, 20
    i32 = dict(dtype=torch.int32, device="cuda")
    x, past, lens = torch.randn((n, V), device="cuda").bfloat16(), torch.randint(0, V, (n, most), **i32), torch.randint(0, most + 1, (n,), **i32)
    penalties = torch.tensor([[1.5, 0.25, 0.125]] * n, device="cuda")
    allowed, row = torch.randint(-2 ** 31, 2 ** 31 - 1, (3, 47), **i32), torch.randint(-1, 3, (n,), **i32)

    def run(x, y, past, allowed):
        d = hawq.LogitsDesc(n_seqs=n, total=n, vocab=V, dtype=hawq.BF16, past_stride=past.stride(0), n_bias=0, n_allowed=masks, allowed_stride=allowed.stride(0), x_stride=x.stride(0),
                            y_stride=y.stride(0))
        hawq.hawq_logits(d, x, past, lens, None, None, None, None, penalties, None, None, None, allowed if masks else None, row if masks else None, y)
        torch.cuda.synchronize()
        return y
    want = run(x, torch.empty_like(x), past, allowed)
    far = _far(x, stride)
    got = run(far, far if in_place else _far(torch.zeros_like(x), stride), _far(past, past_stride), _far(allowed, allowed_stride))
    assert torch.equal(got, want)
