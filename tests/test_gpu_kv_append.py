"""sd_kv_append against the oracle; tolerances as in test_gpu_rope.py.  Values,
unrotated keys and every cache place that no row takes are exact."""

import numpy as np
import pytest

import oracle
from tests.test_gpu_rope import tolerance, values

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]


def torch_type(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def make(lens, n, Hq, Hkv, D, src, dtype, paged, pad=0, front=0, seed=0, spare=3):
    """Rows of a fused projection, poisoned caches and their lengths."""
    import torch
    B = len(lens)
    T = front + sum(n) + pad
    start = front + np.concatenate([[0], np.cumsum(n)])
    qkv = values((T, (Hq + 2 * Hkv) * D), src, seed)
    d = dict(T=T, q=qkv[:, :Hq * D].view(T, Hq, D), k=qkv[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D),
             v=qkv[:, (Hq + Hkv) * D:].view(T, Hkv, D), start=start.astype(np.int32), qkv=qkv,
             kv_len=np.array(lens, np.int32), table=None, Hq=Hq, Hkv=Hkv, D=D)
    if paged:
        pages = [-(-max(x, 1) // 16) for x in lens]
        g = np.random.default_rng(seed)
        perm = g.permutation(sum(pages) + spare).astype(np.int32)
        d["table"] = np.zeros((B, max(pages) + 1), np.int32)
        at = 0
        for b in range(B):
            d["table"][b, :pages[b]] = perm[at:at + pages[b]]
            at += pages[b]
        shape = (sum(pages) + spare, Hkv, 16, D)
    else:
        shape = (B, max(max(lens), 1) + 2, Hkv, D)
    d["k_cache"], d["v_cache"] = (torch.full(shape, p, dtype=torch_type(dtype)) for p in (512.0, -256.0))
    return d


def check(d, dtype, sections, theta, pos=None, per_axis=False, uniform=False, queries=True):
    import torch
    import paper_2505_12728_amd as sd
    dev = lambda a: None if a is None else torch.as_tensor(a).cuda()      # noqa: E731
    T, Hq, Hkv, D = d["T"], d["Hq"], d["Hkv"], d["D"]
    qkv = d["qkv"].cuda()
    q = qkv[:, :Hq * D].view(T, Hq, D) if queries else None
    k = qkv[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D)
    v = qkv[:, (Hq + Hkv) * D:].view(T, Hkv, D)
    kc, vc = d["k_cache"].cuda(), d["v_cache"].cuda()
    q_out = torch.full((T, Hq, D), 77.0, dtype=kc.dtype, device="cuda") if queries else None
    got = sd.sd_kv_append(q, k, v, kc, vc, dev(d["kv_len"]), theta, pos=dev(pos), sections=sections,
                          per_axis=per_axis, row_start=None if uniform else dev(d["start"]),
                          page_table=dev(d["table"]), q_out=q_out)
    assert got is q_out
    secs = [] if theta is None else (sections or [D // 2])
    ref = [oracle.kv_append(*[d[n].float().numpy() for n in ("q", "k", "v", "k_cache", "v_cache")], d["kv_len"],
                            d["start"], secs, theta, pos=pos, per_axis=per_axis, page_table=d["table"])]
    qo, rk, rv = ref[0]
    assert np.array_equal(vc.float().cpu().numpy(), np.asarray(torch.tensor(rv).to(vc.dtype).float())), "values"
    if not secs:
        assert np.array_equal(kc.float().cpu().numpy(), np.asarray(torch.tensor(rk).to(kc.dtype).float()))
    # a key's two sources are bounded by its row's largest values
    P = sum(secs)
    big = np.abs(d["k"].float().numpy())
    bound = 2 * big.max() if big.size else 0.0
    unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    err = np.abs(kc.float().cpu().numpy() - rk)
    assert np.all(err <= unit * np.abs(rk) + 8 * 2.0 ** -24 * bound), ("keys", err.max())
    fresh = rk != 512.0
    assert np.all(kc.float().cpu().numpy()[~fresh] == 512.0)
    if queries:
        mine = q_out.float().cpu().numpy()
        none = np.isnan(qo)
        assert np.all(mine[none] == 77.0)
        tol = tolerance(d["q"].float().numpy(), P, np.where(none, 0, qo), dtype)
        assert np.all((np.abs(mine - qo) <= tol)[~none])
    return kc, vc


@pytest.mark.parametrize("src,dtype", TYPES)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("lens,n,Hq,Hkv,D", [
    ([1], [1], 1, 1, 64), ([6, 700, 33], [6, 6, 6], 32, 8, 128), ([16, 17, 15, 300], [16, 17, 0, 100], 28, 4, 128),
    ([40, 0, 3], [40, 0, 1], 4, 1, 64), ([1000], [1000], 2, 2, 80), ([37, 64], [21, 33], 3, 3, 10),
    ([50, 20], [7, 9], 0, 2, 256)])
def test_append(src, dtype, paged, lens, n, Hq, Hkv, D):
    d = make(lens, n, Hq, Hkv, D, src, dtype, paged, pad=2, front=1)
    check(d, dtype, None, 1e4, queries=Hq > 0)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("r,B", [(1, 5), (6, 16), (100, 3)])
def test_append_fixed_block(paged, r, B):
    lens = [r + (37 * b) % 200 for b in range(B)]
    d = make(lens, [r] * B, 8, 2, 128, "f32", "bf16", paged)
    check(d, "bf16", None, 1e4, uniform=True)


@pytest.mark.parametrize("sections,per_axis,D", [([16, 24, 24], False, 128), ([12, 12, 12], True, 72),
                                                 ([4, 4], True, 64), ([3, 5, 7, 1], False, 40)])
def test_append_positions_of_several_axes(sections, per_axis, D):
    lens, n = [300, 90, 18], [250, 90, 1]
    d = make(lens, n, 4, 2, D, "bf16", "bf16", True, pad=1)
    g = np.random.default_rng(5)
    pos = g.integers(-3, 7000, (len(sections), d["T"])).astype(np.int32)
    check(d, "bf16", sections, 1e6, pos=pos, per_axis=per_axis)


@pytest.mark.parametrize("src,dtype", TYPES)
def test_append_without_rotation(src, dtype):
    d = make([50, 60], [33, 20], 4, 2, 64, src, dtype, True)
    check(d, dtype, None, None)


def test_append_rows_that_do_not_fit_are_left_out():
    # lengths past the capacity and before position 0, page ids out of range:
    # those rows reach no cache, their queries are still rotated
    d = make([40, 40, 40], [40, 40, 40], 2, 1, 64, "f32", "f32", False)
    d["kv_len"] = np.array([46, 30, 40], np.int32)          # capacity 42: rows 36.. of 0; rows ..9 of 1
    check(d, "f32", None, 1e4)
    d = make([40, 40], [40, 30], 2, 1, 64, "bf16", "bf16", True)
    d["table"][0, 1] = -1
    d["table"][1, 2] = d["k_cache"].shape[0]
    check(d, "bf16", None, 1e4)


def test_append_many_sequences():
    # several steps of the search for a row's sequence, most sequences empty
    g = np.random.default_rng(3)
    for B in (64, 65, 1000, 5000):
        n = np.where(g.random(B) < 0.3, g.integers(0, 4, B), 0)
        n[g.integers(0, B)] += 2
        lens = n + g.integers(0, 9, B)
        d = make(lens.tolist(), n.tolist(), 1, 1, 16, "f32", "f32", False, pad=1)
        check(d, "f32", None, 1e4)


def test_append_unaligned_views():
    # caches and rows that start anywhere their type allows
    import torch
    import paper_2505_12728_amd as sd
    T, Hq, Hkv, D = 19, 3, 2, 64
    for shift in (1, 2, 4):
        buf = values((T, (Hq + 2 * Hkv) * D + 5), "bf16", shift).cuda()
        rows = lambda a, h: buf[:, shift + a * D:shift + (a + h) * D].view(T, h, D)      # noqa: E731
        q, k, v = rows(0, Hq), rows(Hq, Hkv), rows(Hq + Hkv, Hkv)
        store = torch.zeros(2, 30 * Hkv * D + 8, dtype=torch.bfloat16, device="cuda")
        kc, vc = (store[i, shift:shift + 30 * Hkv * D].view(1, 30, Hkv, D) for i in range(2))
        kl = torch.tensor([25], dtype=torch.int32, device="cuda")
        qo = sd.sd_kv_append(q, k, v, kc, vc, kl, 1e4)
        kc2, vc2 = torch.zeros_like(kc), torch.zeros_like(vc)
        qo2 = sd.sd_kv_append(q.contiguous(), k.contiguous(), v.contiguous(), kc2, vc2, kl, 1e4)
        assert qo.equal(qo2) and kc.equal(kc2) and vc.equal(vc2)
        assert vc[0, 6:25].equal(v) and not vc[0, :6].any() and not vc[0, 25:].any()


def test_append_queries_in_place():
    import torch
    import paper_2505_12728_amd as sd
    T, Hq, Hkv, D = 12, 4, 2, 128
    q, k, v = (values((T, h, D), "bf16", h).cuda() for h in (Hq, Hkv, Hkv))
    kc, vc = (torch.zeros(2, 8, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kl = torch.tensor([6, 7], dtype=torch.int32, device="cuda")
    want = sd.sd_kv_append(q, k, v, kc, vc, kl, 1e4)
    assert sd.sd_kv_append(q, k, v, kc, vc, kl, 1e4, q_out=q) is q
    assert q.equal(want)


def test_append_past_32_bit_offsets():
    # the last page of a pool of 2^32 elements and more
    import torch
    import paper_2505_12728_amd as sd
    P, Hkv, D = (1 << 32) // (16 * 128) + 2, 1, 128
    kc, vc = (torch.empty(P, Hkv, 16, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kc[-1] = vc[-1] = 0
    k, v = values((3, 1, D), "bf16", 1).cuda(), values((3, 1, D), "bf16", 2).cuda()
    kl = torch.tensor([19], dtype=torch.int32, device="cuda")
    table = torch.tensor([[0, P - 1]], dtype=torch.int32, device="cuda")
    sd.sd_kv_append(None, k, v, kc, vc, kl, 1e4, page_table=table)
    pos = torch.tensor([16, 17, 18], dtype=torch.int32, device="cuda")
    assert vc[-1, 0, :3].equal(v[:, 0]) and not vc[-1, 0, 3:].any()
    assert kc[-1, 0, :3].equal(sd.sd_rope(k, pos, 1e4)[:, 0])
    del kc, vc
    torch.cuda.empty_cache()


def test_append_graph_replays():
    # one captured call serves every step: lengths, pages and rows are read on the device
    import torch
    import paper_2505_12728_amd as sd
    B, r, Hq, Hkv, D = 3, 4, 4, 2, 128
    d = make([30, 17, 45], [r] * B, Hq, Hkv, D, "bf16", "bf16", True, spare=8)
    qkv, table = d["qkv"].cuda(), torch.from_numpy(d["table"]).cuda()
    part = lambda a, h: qkv[:, a * D:(a + h) * D].view(B * r, h, D)      # noqa: E731
    q, k, v = part(0, Hq), part(Hq, Hkv), part(Hq + Hkv, Hkv)
    kc, vc = d["k_cache"].cuda(), d["v_cache"].cuda()
    kl = torch.tensor([10, 4, 41], dtype=torch.int32, device="cuda")
    out = torch.empty(B * r, Hq, D, dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    sd.sd_kv_append(q, k, v, kc, vc, kl, 1e4, page_table=table, q_out=out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sd.sd_kv_append(q, k, v, kc, vc, kl, 1e4, page_table=table, q_out=out)
    for i in range(3):
        qkv.copy_(values(tuple(qkv.shape), "bf16", 50 + i))
        kl.add_(1)
        k2, v2 = kc.clone(), vc.clone()
        graph.replay()
        torch.cuda.synchronize()
        want = sd.sd_kv_append(q, k, v, k2, v2, kl, 1e4, page_table=table)
        assert out.equal(want) and kc.equal(k2) and vc.equal(v2)


def test_append_binding_refuses():
    import torch
    import paper_2505_12728_amd as sd
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")      # noqa: E731
    q, k, v, kc, vc = z(6, 4, 64), z(6, 2, 64), z(6, 2, 64), z(2, 9, 2, 64), z(2, 9, 2, 64)
    kl = z(2, t=torch.int32)
    with pytest.raises(ValueError, match="same shape"):
        sd.sd_kv_append(q, k, v[:5], kc, vc, kl, 1e4)
    with pytest.raises(ValueError, match="contiguous caches"):
        sd.sd_kv_append(q, k, v, kc[:1], vc[:1], kl, 1e4)
    with pytest.raises(ValueError, match="paged caches"):
        sd.sd_kv_append(q, k, v, kc, vc, kl, 1e4, page_table=z(2, 1, t=torch.int32))
    pool = z(4, 2, 16, 64)
    with pytest.raises(ValueError, match="num_pages"):
        sd.sd_kv_append(q, k, v, pool, pool.clone(), kl, 1e4, page_table=z(2, 1, t=torch.int32), num_pages=5)
    with pytest.raises(ValueError, match="T / B"):
        sd.sd_kv_append(q[:5], k[:5], v[:5], kc, vc, kl, 1e4)
    with pytest.raises(ValueError, match="row_start"):
        sd.sd_kv_append(q, k, v, kc, vc, kl, 1e4, row_start=z(2, t=torch.int32))
    with pytest.raises(TypeError):
        sd.sd_kv_append(q, k, v, kc, vc.float(), kl, 1e4)
    with pytest.raises(TypeError):
        sd.sd_kv_append(q.float(), k, v, kc, vc, kl, 1e4)
    with pytest.raises(sd.SDError):                      # bf16 rows into an fp32 cache
        sd.sd_kv_append(q, k, v, kc.float(), vc.float(), kl, 1e4)
    with pytest.raises(ValueError, match="q_out"):
        sd.sd_kv_append(None, k, v, kc, vc, kl, 1e4, q_out=q)
    with pytest.raises(ValueError, match="contiguous"):
        sd.sd_kv_append(q, k, v, kc, vc, kl, 1e4, q_out=z(6, 8, 64)[:, ::2])
