"""hawq_rotary on the GPU against the definition in 64 bits."""
import numpy as np
import pytest

import lm_step_reference as ref

pytestmark = pytest.mark.gpu


def _turns(R, base=10000.0):
    return base ** (-np.arange(R // 2) * 2.0 / R) / (2 * np.pi)


def _run(total, H, KV, D, R, layout, dtype, far=5000, scale=1.0, pad=0, at=0, in_place=False, heads_first=False, positions=None, seed=0):
    import torch
    import paper_2011_10680_amd as hawq
    dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    r = np.random.default_rng(seed)
    turns = _turns(R)
    pos = r.integers(0, far, size=total) if positions is None else np.asarray(positions)
    x, y, want, bounds, kw = [], [], [], [], {}
    for name, h in (("q", H), ("k", KV)):
        v = torch.from_numpy(r.normal(size=(total, h, D)).astype(np.float32)).to(dt)
        # a slice with other values around it that are neither read into a result nor written over
        shape = (h, total, D + pad) if heads_first else (total, h, D + pad)
        whole = torch.full((at + total * h * (D + pad) + 8,), float("nan"), dtype=dt, device="cuda")
        d = whole[at:at + total * h * (D + pad)].view(shape)
        d = (d.transpose(0, 1) if heads_first else d)[..., :D]
        d.copy_(v)
        out = torch.full((total, h, D + pad), 7.0, dtype=dt, device="cuda")
        o = d if in_place else out[..., :D]
        x.append(d)
        y.append((o, whole if in_place else out, v, h))
        for n, t in ((name, d), ("y" + name, o)):
            kw[n + "_token"], kw[n + "_head"] = t.stride(0), t.stride(1)
        w, size = ref.rotary(v.double().numpy(), pos, turns, layout, float(np.float32(scale)))
        want.append(w)
        bounds.append(ref.rotary_bound(w, size, pos, turns, dtype))
    desc = hawq.RotaryDesc(total=total, q_heads=H, kv_heads=KV, head_dim=D, rotary_dim=R, layout=hawq.ROTARY_HALVES if layout == "halves" else hawq.ROTARY_PAIRS,
                           dtype=hawq.F16 if dtype == "f16" else hawq.BF16, scale=scale, **kw)
    hawq.hawq_rotary(desc, x[0], x[1], torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(turns).cuda(), y[0][0], y[1][0])
    torch.cuda.synchronize()
    for (o, whole, v, h), w, b in zip(y, want, bounds):
        got = o.double().cpu().numpy()
        assert (np.abs(got - w) <= b).all(), (total, H, KV, D, R, float((np.abs(got - w) - b).max()))
        if in_place:
            assert int(torch.isnan(whole).sum()) == whole.numel() - total * h * D
        else:
            assert bool((whole[..., D:] == 7.0).all())


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("D,R", [(64, 64), (80, 80), (80, 32), (128, 128), (128, 64), (96, 96), (256, 256), (256, 16), (20, 20), (7, 4), (2, 2), (100, 36), (24, 8), (72, 24), (33, 16)])
def test_heads(layout, D, R):
    for i, dtype in enumerate(("f16", "bf16")):
        _run(5 + 60 * i, 6, 2, D, R, layout, dtype, seed=D + R + i)


@pytest.mark.parametrize("total", [1, 2, 3, 17, 64, 257, 2049, 5000])
def test_tokens(total):
    _run(total, 8, 1, 64, 64, "halves", "f16", seed=total)
    _run(total, 3, 3, 80, 32, "pairs", "bf16", scale=1.2, seed=total)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("pad,at,heads_first", [(0, 0, False), (8, 0, True), (16, 8, False), (2, 0, False), (4, 4, True), (1, 0, False), (0, 1, False), (3, 5, True), (0, 2, False)])
def test_strides_alignment_and_place(pad, at, heads_first, in_place):
    for layout in ("halves", "pairs"):
        _run(9, 4, 2, 64, 64, layout, "bf16", pad=pad, at=at, heads_first=heads_first, in_place=in_place, seed=pad)
        _run(6, 4, 2, 48, 32, layout, "f16", pad=pad, at=at, heads_first=heads_first, in_place=in_place, seed=pad)


def test_far_and_negative_positions():
    """The largest positions there are: 2^31 turns' product still has 24 bits behind the point."""
    for layout in ("halves", "pairs"):
        _run(7, 2, 1, 64, 64, layout, "f16", positions=[0, 1, -1, 1 << 20, -(1 << 24), (1 << 31) - 1, -(1 << 31)], seed=1)
        _run(6, 2, 1, 40, 20, layout, "bf16", positions=[131071, 1000003, 7, 99999999, 0, 5], scale=0.5, seed=2)


def test_one_kind_of_heads_and_many_heads():
    _run(4, 3, 0, 64, 64, "halves", "f16")
    _run(4, 0, 2, 64, 32, "pairs", "f16")
    _run(2, 700, 300, 32, 32, "halves", "bf16")
    _run(3, 65535, 1, 2, 2, "pairs", "bf16")


def test_no_query_is_read_for_a_broadcast_axis_twice():
    """One key row for all tokens (a stride of 0), each token's own result."""
    import torch
    import paper_2011_10680_amd as hawq
    r = np.random.default_rng(1)
    row = torch.from_numpy(r.normal(size=(1, 2, 64)).astype(np.float32)).half().cuda()
    y = torch.empty((50, 2, 64), dtype=torch.float16, device="cuda")
    turns, pos = _turns(64), np.arange(50)
    d = hawq.RotaryDesc(total=50, q_heads=2, kv_heads=0, head_dim=64, rotary_dim=64, layout=hawq.ROTARY_HALVES, dtype=hawq.F16, scale=1.0, q_token=0, q_head=64, yq_token=128,
                        yq_head=64)
    hawq.hawq_rotary(d, row, None, torch.arange(50, dtype=torch.int32, device="cuda"), torch.from_numpy(turns).cuda(), y, None)
    w, size = ref.rotary(np.repeat(row.double().cpu().numpy(), 50, axis=0), pos, turns, "halves", 1.0)
    assert (np.abs(y.double().cpu().numpy() - w) <= ref.rotary_bound(w, size, pos, turns, "f16")).all()


def test_values_that_are_not_numbers_stay_in_their_pair():
    import torch
    import paper_2011_10680_amd as hawq
    for layout, pair in ((hawq.ROTARY_HALVES, (3, 35)), (hawq.ROTARY_PAIRS, (2, 3))):
        x = torch.ones((2, 1, 80), dtype=torch.bfloat16, device="cuda")
        x[0, 0, 3] = float("inf")
        x[1, 0, 70] = float("nan")
        y = torch.empty_like(x)
        d = hawq.RotaryDesc(total=2, q_heads=1, kv_heads=0, head_dim=80, rotary_dim=64, layout=layout, dtype=hawq.BF16, scale=1.0, q_token=80, q_head=80, yq_token=80, yq_head=80)
        hawq.hawq_rotary(d, x, None, torch.tensor([5, 9], dtype=torch.int32, device="cuda"), torch.from_numpy(_turns(64)).cuda(), y, None)
        bad = (~torch.isfinite(y)).nonzero().tolist()
        assert bad == [[0, 0, pair[0]], [0, 0, pair[1]], [1, 0, 70]]
