"""sd_rope against the oracle (extended-precision angles).

Tolerance, per element y of a pair (x1, x2): y is rounded once to its type
(2^-8 |y| for bf16, 2^-24 |y| for fp32) after float32 arithmetic on exactly
reduced angles: the angle's fraction rounded to 24 bits (at most 1.6 units of
2^-24 in sine or cosine), sincospi within 2 units, two products and a sum
within 1 each, so that 8 * 2^-24 (|x1| + |x2|) bounds the rest."""

import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu


def tolerance(x, P, ref, dtype):
    a = np.abs(x)
    other = np.zeros_like(a)
    other[..., :P] = other[..., P:2 * P] = a[..., :P] + a[..., P:2 * P]
    return (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(ref) + 8 * 2.0 ** -24 * other


def values(shape, dtype, seed=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    t = torch.randn(shape, generator=g)
    return t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def positions(axes, T, far, seed=0):
    import torch
    g = torch.Generator().manual_seed(seed + 100)
    return torch.randint(-9, far, (axes, T), generator=g, dtype=torch.int32)


CASES = [  # T, H, D, sections, per_axis, far
    (1, 1, 2, [1], False, 100), (1, 32, 128, [64], False, 131072), (8, 32, 128, [16, 24, 24], False, 6528),
    (129, 5, 80, [20, 20], True, 200), (67, 3, 72, [12, 12, 12], True, 64), (33, 16, 64, [16, 16], False, 999),
    (50, 7, 128, [8, 12, 12], False, 1 << 20), (40, 2, 256, [32, 32, 32, 32], True, 5000),
    (9, 3, 10, [3], False, 77), (5, 2, 7, [1, 2], True, 50), (700, 11, 96, [4, 5, 6], False, 31),
    (3, 300, 64, [32], False, 10), (2, 1, 254, [127], False, 4096)]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope(case, dtype, inverse):
    import paper_2505_12728_amd as sd
    T, H, D, secs, per_axis, far = case
    x, pos = values((T, H, D), dtype), positions(len(secs), T, far)
    y = sd.sd_rope(x.cuda(), pos.cuda(), 1e4, sections=secs, per_axis=per_axis, inverse=inverse)
    ref = oracle.rope_axes(x.float().numpy(), pos.numpy(), secs, 1e4, per_axis, inverse)
    assert y.dtype == x.dtype
    err = np.abs(y.float().cpu().numpy() - ref)
    assert np.all(err <= tolerance(x.float().numpy(), sum(secs), ref, dtype)), err.max()
    rest = y[..., 2 * sum(secs):].cpu()
    assert rest.equal(x[..., 2 * sum(secs):])


@pytest.mark.parametrize("offset,gap", [(0, 0), (0, 8), (8, 24), (4, 12), (1, 3), (0, 7)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rope_strided_rows_and_in_place(offset, gap, dtype):
    # rows that start and end anywhere of a fused buffer; what lies between stays
    import torch
    import paper_2505_12728_amd as sd
    T, H, D, secs = 37, 6, 64, [8, 12, 12]
    buf = values((T, offset + H * D + gap), dtype, 3)
    pos = positions(3, T, 4000)
    x = buf[:, offset:offset + H * D].view(T, H, D)
    ref = oracle.rope_axes(x.float().numpy(), pos.numpy(), secs, 1e6)
    dev = buf.cuda()
    view = dev[:, offset:offset + H * D].view(T, H, D)
    dense = sd.sd_rope(view, pos.cuda(), 1e6, sections=secs)
    other = torch.zeros(T, H * D + 2 * gap, dtype=x.dtype, device="cuda")
    spread = sd.sd_rope(view, pos.cuda(), 1e6, sections=secs, out=other[:, gap:gap + H * D].view(T, H, D))
    assert sd.sd_rope(view, pos.cuda(), 1e6, sections=secs, out=view) is view
    tol = tolerance(x.float().numpy(), 32, ref, dtype)
    assert np.all(np.abs(dense.float().cpu().numpy() - ref) <= tol)
    assert view.equal(dense) and spread.equal(dense)
    after = dev.cpu()
    assert after[:, :offset].equal(buf[:, :offset]) and after[:, offset + H * D:].equal(buf[:, offset + H * D:])
    assert not other[:, :gap].any() and not other[:, gap + H * D:].any()


def test_rope_far_positions():
    # the largest positions: their float64 turn count holds 2^-53 of itself,
    # three roundings of it (frequency, its 1 / 2 pi, the product)
    import torch
    import paper_2505_12728_amd as sd
    pos = torch.tensor([[2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 123456789, 0]], dtype=torch.int32)
    x = values((5, 2, 128), "f32", 5)
    y = sd.sd_rope(x.cuda(), pos.cuda(), 1e6, sections=[64]).cpu().numpy()
    xn = x.numpy()
    ref = oracle.rope_axes(xn, pos.numpy(), [64], 1e6)
    # exp's argument is at most log(1e6) = 13.8, itself rounded: 16 units of 2^-53 more
    far = np.abs(pos.numpy().astype(np.float64))[0][:, None, None] * 20 * 2.0 ** -53
    pair = np.abs(xn[..., :64]) + np.abs(xn[..., 64:])
    tol = tolerance(xn, 64, ref, "f32") + far * np.concatenate([pair, pair], -1)
    assert np.all(np.abs(y - ref) <= tol)


def test_rope_gradient():
    # against the formula's and against differences of the operator itself
    import torch
    import paper_2505_12728_amd as sd
    T, H, D, secs = 6, 2, 16, [3, 4]
    x, dy, pos = values((T, H, D), "f32", 7), values((T, H, D), "f32", 8), positions(2, T, 30)
    f = lambda t: sd.sd_rope(t, pos.cuda(), 1e3, sections=secs, per_axis=True)   # noqa: E731
    dx = sd.sd_rope(dy.cuda(), pos.cuda(), 1e3, sections=secs, per_axis=True, inverse=True).cpu().double()
    xd = x.cuda()
    for i in range(0, x.numel(), 5):
        e = torch.zeros(x.numel())
        e[i] = 0.5
        e = e.view_as(x).cuda()
        # linear in x: a difference over a whole unit has no truncation error,
        # only the float32 roundings of its two values
        num = ((f(xd + e) - f(xd - e)).cpu().double() * dy.double()).sum()
        assert abs(num - dx.flatten()[i]) <= 64 * 2.0 ** -24 * (dy.abs().max() * (x.abs().max() + 1)), i


def test_rope_nothing_and_many_rows():
    import torch
    import paper_2505_12728_amd as sd
    x = values((0, 4, 64), "bf16").cuda()
    assert sd.sd_rope(x, torch.zeros(1, 0, dtype=torch.int32, device="cuda"), 1e4).shape == (0, 4, 64)
    # more rows than the grid holds at once, each its own position
    T = 50000
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    x = torch.ones(T, 1, 4, device="cuda")
    y = sd.sd_rope(x, pos, 100.0).cpu().numpy()
    ref = oracle.rope_axes(np.ones((T, 1, 4)), np.arange(T)[None], [2], 100.0)
    assert np.all(np.abs(y - ref) <= tolerance(np.ones((T, 1, 4)), 2, ref, "f32"))


def test_rope_past_32_bit_offsets():
    # rows 2^20 elements apart: the last one starts 2^32 elements on
    import torch
    import paper_2505_12728_amd as sd
    T = 4097
    buf = torch.empty((T - 1) * (1 << 20) + 128, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (T, 1, 128), (1 << 20, 128, 1))
    v = values((T, 1, 128), "bf16", 9)
    x.copy_(v)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    y = sd.sd_rope(x, pos, 1e4)
    assert y.equal(sd.sd_rope(v.cuda(), pos, 1e4))
    sd.sd_rope(x, pos, 1e4, out=x)
    assert x.equal(y)
    del buf, x
    torch.cuda.empty_cache()


def test_rope_graph_and_stream():
    import torch
    import paper_2505_12728_amd as sd
    pos = positions(3, 9, 100).cuda()
    x = values((9, 4, 128), "bf16", 1).cuda()
    want = sd.sd_rope(x, pos, 1e4, sections=[16, 24, 24])
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sd.sd_rope(x, pos, 1e4, sections=[16, 24, 24], out=out, stream=side)
    side.synchronize()
    assert out.equal(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.sd_rope(x, pos, 1e4, sections=[16, 24, 24], out=out)
    for i in range(3):
        x.copy_(values((9, 4, 128), "bf16", 20 + i))
        pos.add_(5)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert out.equal(sd.sd_rope(x, pos, 1e4, sections=[16, 24, 24]))


def test_rope_binding_refuses():
    import torch
    import paper_2505_12728_amd as sd
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="GPU"):
        sd.sd_rope(x.cpu(), pos, 1e4, sections=[16, 16])
    with pytest.raises(ValueError, match="pos"):
        sd.sd_rope(x, pos[:, :3].contiguous(), 1e4, sections=[16, 16])
    with pytest.raises(ValueError, match="sections"):
        sd.sd_rope(x, pos, 1e4, sections=[16, 8, 8])
    with pytest.raises(TypeError):
        sd.sd_rope(x, pos.long(), 1e4, sections=[16, 16])
    with pytest.raises(TypeError):
        sd.sd_rope(x, pos, 1e4, sections=[16, 16], out=torch.zeros(4, 2, 64, device="cuda"))
    with pytest.raises(TypeError, match="unsupported"):
        sd.sd_rope(x.half(), pos, 1e4, sections=[16, 16])
    with pytest.raises(ValueError, match="shape"):
        sd.sd_rope(x, pos, 1e4, sections=[16, 16], out=x[:3])
    with pytest.raises(ValueError, match="dense rows"):
        sd.sd_rope(x.transpose(0, 1), pos[:, :2].contiguous(), 1e4, sections=[16, 16])
    with pytest.raises(ValueError, match="dense rows"):
        sd.sd_rope(x[..., ::2], pos, 1e4, sections=[8, 8])
    with pytest.raises(ValueError, match="dense rows"):
        sd.sd_rope(x[:1].expand(4, 2, 64), pos, 1e4, sections=[16, 16])
    with pytest.raises(sd.SDError):                     # two axes and no sections
        sd.sd_rope(x, pos, 1e4)
    with pytest.raises(sd.SDError):                     # out one row on in x's own memory
        big = torch.zeros(5, 2, 64, dtype=torch.bfloat16, device="cuda")
        sd.sd_rope(big[:4], pos, 1e4, sections=[16, 16], out=big[1:])
