"""sd_verify_shared against the oracle.

Tolerances, with A = the same average of |V| (the oracle's spread) and n the
scale in units of 1 / sqrt(D) (inputs N(0, 1)):
  scores     D = 128 fp32 products of sum |q k| scale <= 8 n, summed one after
             the other: 128 * 2^-24 * 8 n = 2^-14 n of each weight, in sum and
             normaliser
  weights    all of their bits in three bf16 terms; single bf16 values 2^-8
  sums       up to 2^9 steps of 32 keys, 2^-24 of A each: 2^-15
so that 2^-12 max(1, n) A bounds an fp32 output, and 2^-8 (A + |out|) more a
bf16 one.  fp32 inputs run in float64; their partials and the merge's weights
(a log-sum-exp of up to 2^5 in fp32) hold 2^-19 A."""

import math

import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu


def inputs(lens, plens, sizes, k, Hq, Hkv, D, dtype="bf16", paged=False, seed=0, lead=0, left=0):
    """Groups of `sizes` sequences behind `lead` sequences of none, `left`
    more at the end.  What lies past the lengths is poisoned."""
    import torch
    g = torch.Generator().manual_seed(seed)
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    B, G = len(lens), len(plens)
    assert lead + sum(sizes) + left == B
    rnd = lambda *s: torch.randn(s, generator=g).to(tt)                   # noqa: E731
    d = dict(q=rnd(B, k, Hq, D), kv_len=np.array(lens, np.int32), prefix_len=np.array(plens, np.int32),
             group_start=(lead + np.concatenate([[0], np.cumsum(sizes)])).astype(np.int32), page_table=None,
             prefix_table=None)
    if paged:
        need = [-(-n // 16) for n in list(plens) + list(lens)]
        P = sum(need) + 2
        perm = np.random.default_rng(seed).permutation(P)
        at, tables = 0, []
        for n in need:
            tables.append(perm[at:at + n])
            at += n
        for c in ("k_cache", "v_cache"):
            d[c] = rnd(P, Hkv, 16, D)
        for name, rows, ls in (("prefix_table", tables[:G], plens), ("page_table", tables[G:], lens)):
            d[name] = np.zeros((len(rows), max(1, max(len(r) for r in rows))), np.int32)
            for i, r in enumerate(rows):
                d[name][i, :len(r)] = r
                if ls[i] % 16:
                    for c in ("k_cache", "v_cache"):
                        d[c][r[-1], :, ls[i] % 16:] = 8192.0
        d["k_prefix"] = d["v_prefix"] = None
    else:
        for c, rows, ls in (("cache", B, lens), ("prefix", G, plens)):
            for kv in "kv":
                t = d[f"{kv}_{c}"] = rnd(rows, max(1, max(ls)) + 3, Hkv, D)
                for i, n in enumerate(ls):
                    t[i, n:] = 8192.0
    return d


def call(d, **kw):
    import torch
    import paper_2505_12728_amd as sd
    dev = lambda a: None if a is None else torch.as_tensor(a).cuda()      # noqa: E731
    args = {n: dev(d[n]) for n in ("q", "k_cache", "v_cache", "kv_len", "prefix_len", "k_prefix", "v_prefix",
                                   "prefix_table", "group_start", "page_table")}
    args.update(kw)
    return sd.sd_verify_shared(**args)


def roomy(d, keys=1 << 18):
    """The prefixes in caches of `keys` keys, what lies behind them not a number:
    with many rows the capacity decides on tiles of 256 rows."""
    import torch
    if d["prefix_table"] is not None:
        t = torch.full((len(d["prefix_len"]), keys // 16), -1, dtype=torch.int32, device="cuda")
        t[:, :d["prefix_table"].shape[1]] = torch.as_tensor(d["prefix_table"]).cuda()
        return dict(prefix_table=t)
    big = {}
    for n in ("k_prefix", "v_prefix"):
        G, L, Hkv, D = d[n].shape
        big[n] = torch.full((G, keys, Hkv, D), math.nan, dtype=d[n].dtype, device="cuda")
        big[n][:, :L] = d[n].cuda()
    return big


def reference(d, scale):
    f = lambda t: None if t is None else t.double().numpy()               # noqa: E731
    kp = d["k_prefix"] if d["k_prefix"] is not None else d["k_cache"]
    vp = d["v_prefix"] if d["v_prefix"] is not None else d["v_cache"]
    return oracle.verify_shared(f(d["q"]), f(d["k_cache"]), f(d["v_cache"]), d["kv_len"], f(kp), f(vp), d["prefix_len"],
                                d["group_start"], scale, page_table=d["page_table"], prefix_table=d["prefix_table"])


def check(d, out, lse, ref, dtype, units=1.0):
    ro, rl, A = ref
    out = out.float().cpu().numpy().astype(np.float64) if dtype != "f32" else out.cpu().numpy().astype(np.float64)
    lse = lse.cpu().numpy()
    n = max(1.0, units)
    tol = 2.0 ** -19 * A if dtype == "f32" else 2.0 ** -12 * n * A
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (A + np.abs(ro))
    assert np.all(np.isfinite(out))
    err = np.abs(out - ro) - tol
    assert np.all(err <= 1e-30), (np.unravel_index(err.argmax(), err.shape), err.max())
    none = np.isinf(rl)
    assert np.array_equal(none, np.isinf(lse)) and np.all(lse[none] < 0) and not out[none].any()
    bound = 1e-5 if dtype == "f32" else 2.0 ** -12 * n
    assert np.all(np.abs(lse[~none] - rl[~none]) <= bound)


CASES = [  # own lengths, prefix lengths, group sizes, k, Hq, Hkv, D, paged, lead, left
    ([1], [1], [1], 1, 1, 1, 64, False, 0, 0),
    ([4, 30], [100], [2], 4, 8, 2, 128, False, 0, 0),
    ([6, 70, 33, 32, 31], [640], [5], 6, 32, 8, 128, True, 0, 0),
    ([1, 2, 3, 4], [1136], [4], 1, 32, 32, 128, False, 0, 0),
    # groups of different sizes, one empty, prefixes of no key and of one; sequences of no group
    ([9, 8, 50, 12, 300, 8, 17], [65, 0, 33, 1], [2, 1, 0, 2], 8, 8, 2, 64, True, 1, 1),
    ([9, 8, 50, 12, 300, 8, 17], [65, 0, 33, 1], [2, 1, 0, 2], 8, 8, 2, 64, False, 1, 1),
    # own caches shorter than the block, and empty: rows that see the prefix only, or nothing
    ([0, 2, 5, 3], [40, 0], [2, 2], 5, 4, 4, 128, False, 0, 0),
    ([0, 2, 5, 3], [40, 0], [2, 2], 5, 4, 4, 128, True, 0, 0),
    ([0, 0, 0], [0], [3], 2, 4, 1, 64, False, 0, 0),
    # the three row tiles and their edges: 64, 65, 128, 129, 256, 257 and more rows a group
    ([20] * 8, [333], [8], 8, 2, 2, 128, False, 0, 0),
    ([20] * 13, [333], [13], 5, 1, 1, 128, False, 0, 0),
    ([16] * 8, [257], [8], 16, 1, 1, 64, True, 0, 0),
    ([30] * 43, [129], [43], 3, 2, 2, 128, False, 0, 0),
    ([33] * 16, [1025], [16], 16, 2, 2, 128, True, 0, 0),
    ([40] * 37, [700], [37], 7, 8, 4, 128, False, 0, 0),
    ([64, 5] * 20, [500, 300], [31, 9], 4, 28, 4, 128, True, 0, 0),
    # 256 rows of one sequence; many units
    ([100, 16], [90], [2], 16, 16, 1, 128, False, 0, 0),
    ([7] * 200, [20] * 70, [3] * 66 + [0] * 3 + [2], 2, 2, 1, 64, False, 0, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"B{len(c[0])}G{len(c[1])}k{c[3]}h{c[4]}x{c[5]}d{c[6]}p{c[7]:d}")
@pytest.mark.parametrize("kind", ["hilo", "bf16", "f32"])
def test_shared(case, kind):
    import torch
    lens, plens, sizes, k, Hq, Hkv, D, paged, lead, left = case
    if kind == "f32" and k * Hq // Hkv > 64:
        pytest.skip("fp32 takes up to 64 rows per KV head")
    d = inputs(lens, plens, sizes, k, Hq, Hkv, D, "f32" if kind == "f32" else "bf16", paged, len(lens), lead, left)
    out, lse = call(d, out_dtype=torch.bfloat16 if kind == "bf16" else torch.float32)
    assert out.dtype == (torch.bfloat16 if kind == "bf16" else torch.float32)
    check(d, out, lse, reference(d, 1 / math.sqrt(D)), kind)


@pytest.mark.parametrize("case", [
    ([20] * 32, [333], [32], 8, 1, 1, 128, False, 0, 0),
    ([64, 5] * 20, [500, 300], [31, 9], 4, 28, 4, 128, True, 0, 0),
    ([33] * 16, [1025], [16], 16, 2, 2, 128, True, 0, 0),
    ([40] * 37, [700], [37], 7, 8, 4, 64, False, 0, 0),
    ([0, 3, 70, 9] * 12, [65, 0, 900], [30, 0, 18], 5, 16, 1, 128, False, 0, 0),
    ([100, 16, 8], [90], [3], 16, 16, 1, 64, True, 0, 0),
], ids=lambda c: f"B{len(c[0])}G{len(c[1])}k{c[3]}h{c[4]}x{c[5]}d{c[6]}p{c[7]:d}")
@pytest.mark.parametrize("kind", ["hilo", "bf16"])
def test_shared_roomy_caches(case, kind):
    import torch
    lens, plens, sizes, k, Hq, Hkv, D, paged, lead, left = case
    d = inputs(lens, plens, sizes, k, Hq, Hkv, D, "bf16", paged, len(lens), lead, left)
    out, lse = call(d, out_dtype=torch.bfloat16 if kind == "bf16" else torch.float32, **roomy(d))
    check(d, out, lse, reference(d, 1 / math.sqrt(D)), kind)


@pytest.mark.parametrize("units", [-1.0, 0.0, 6.0])
@pytest.mark.parametrize("kind", ["hilo", "bf16"])
def test_shared_scales(units, kind):
    import torch
    d = inputs([40, 13, 22], [900], [3], 4, 16, 2, 128, paged=True, seed=3)
    scale = units / math.sqrt(128)
    out, lse = call(d, scale=scale, out_dtype=torch.bfloat16 if kind == "bf16" else torch.float32)
    check(d, out, lse, reference(d, scale), kind, abs(units))


@pytest.mark.parametrize("rows", [64, 128, 256])
def test_shared_rising_scores(rows):
    # every tile raises the maximum by more than the headroom: keys grow along
    # the prefix, so that each rescale of (O, l) matters
    import torch
    B = rows // 8
    d = inputs([8] * B, [400], [B], 8, 1, 1, 64, seed=5)
    d["q"].fill_(0.25)
    ramp = torch.linspace(0, 12, 400)[:, None, None]
    d["k_prefix"][0, :400] = (ramp + 0.01 * d["k_prefix"][0, :400].float()).to(torch.bfloat16)
    # scores reach 16 * 12 = 192 from 64 products of one sign: their float32
    # sum is off by at most 64 * 2^-24 * 192, within the bound for n = 8
    ref = reference(d, 1.0)
    out, lse = call(d, scale=1.0)
    check(d, out, lse, ref, "hilo", 8.0)
    out, lse = call(d, scale=1.0, out_dtype=torch.bfloat16, **roomy(d))
    check(d, out, lse, ref, "bf16", 8.0)


@pytest.mark.parametrize("k,lens", [(4, [4, 5, 70]), (16, [16, 65, 79, 130]), (2, [1, 2, 66])])
@pytest.mark.parametrize("rows,prefix", [(64, 0), (256, 8000)])
def test_shared_masked_keys_weigh_nothing(k, lens, rows, prefix):
    # the last key, visible to the last block row only, has a score of 512 where
    # the others have about 0: no other row may know of it, neither where its
    # tile is a segment's first nor behind one, nor where the block crosses tiles
    import torch
    lens = lens * (rows // (k * len(lens)) + 1)
    d = inputs(lens, [max(prefix, 1)], [len(lens)], k, 1, 1, 64, seed=6)
    d["prefix_len"][0] = prefix
    d["q"].fill_(1.0)
    d["k_prefix"] = (d["k_prefix"].float() / 64).to(torch.bfloat16)
    for b, n in enumerate(lens):
        d["k_cache"][b, :n] = (d["k_cache"][b, :n].float() / 64).to(torch.bfloat16)
        d["k_cache"][b, n - 1] = 8.0
    ref = reference(d, 1.0)
    for kind in ("hilo", "bf16"):
        out, lse = call(d, scale=1.0, out_dtype=torch.bfloat16 if kind == "bf16" else torch.float32, **roomy(d))
        # 512 log2(e) is held to about 2^-14 in the last row's lse
        check(d, out, lse, ref, kind)


@pytest.mark.parametrize("kind", ["hilo", "bf16", "f32"])
def test_shared_nonfinite_keys_reach_the_rows_that_see_them(kind):
    # the last key of each sequence, and of one the last two: the block rows
    # before them as without them
    import torch
    d = inputs([9, 64, 70, 131], [200], [4], 5, 4, 2, 128, "f32" if kind == "f32" else "bf16", seed=7)
    out_dtype = torch.bfloat16 if kind == "bf16" else torch.float32
    ref = reference(d, 1 / math.sqrt(128))
    want, want_lse = call(d, out_dtype=out_dtype)
    for b, (n, bad) in enumerate(zip([9, 64, 70, 131], (math.nan, math.inf, -math.inf, math.nan))):
        d["k_cache"][b, n - 1] = bad
    d["k_cache"][2, 68] = math.inf
    out, lse = call(d, out_dtype=out_dtype)
    for b, rows in enumerate((4, 4, 3, 4)):
        out[b, rows:], lse[b, rows:] = want[b, rows:], want_lse[b, rows:]
    check(d, out, lse, ref, kind)


@pytest.mark.parametrize("kind", ["hilo", "bf16", "f32"])
@pytest.mark.parametrize("B", [3, 300])
def test_shared_nan_rows_stay_nan(kind, B):
    # a query that is not a number, and a row whose only own key is none: those
    # rows alone, in out and lse
    import torch
    d = inputs([40] * B, [90], [B], 2, 4, 2, 64, "f32" if kind == "f32" else "bf16", seed=8)
    out_dtype = torch.bfloat16 if kind == "bf16" else torch.float32
    ref = reference(d, 1 / 8)
    want, want_lse = call(d, out_dtype=out_dtype)
    d["q"][1, 0, 3, 5] = math.nan
    d["k_cache"][2, 39, 1] = math.nan              # the last block row of heads 2 and 3
    out, lse = call(d, out_dtype=out_dtype)
    for at in ((1, 0, slice(3, 4)), (2, 1, slice(2, 4))):
        assert bool(torch.isnan(out[at]).all()) and bool(torch.isnan(lse[at]).all())
        out[at], lse[at] = want[at], want_lse[at]
    check(d, out, lse, ref, kind)


def test_shared_most_sequences():
    # the largest batch, each sequence with a prefix of its own: two keys a row
    import torch
    import paper_2505_12728_amd as sd
    B, D = 1 << 16, 64
    g = torch.Generator(device="cuda").manual_seed(18)
    rnd = lambda: torch.randn(B, 1, 1, D, generator=g, device="cuda").to(torch.bfloat16)     # noqa: E731
    q, k, v, kp, vp = (rnd() for _ in range(5))
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    out, lse = sd.sd_verify_shared(q, k, v, one, one, k_prefix=kp, v_prefix=vp)
    s = torch.stack([(q.double() * x.double()).sum(-1) / 8 for x in (k, kp)])
    w = torch.softmax(s, 0)[..., None]
    want = w[0] * v.double() + w[1] * vp.double()
    A = w[0] * v.double().abs() + w[1] * vp.double().abs()
    assert bool(((out - want).abs() <= 2.0 ** -12 * A).all())
    assert bool(((lse - torch.logsumexp(s, 0)).abs() <= 2.0 ** -12).all())


def test_shared_two_calls_at_once():
    # two streams, two workspaces, the same caches: each as it is alone
    import torch
    import paper_2505_12728_amd as sd
    d = inputs([40] * 16, [9000], [16], 8, 8, 2, 128, paged=True, seed=17)
    dev = {n: torch.as_tensor(d[n]).cuda() for n in d if d[n] is not None}
    other = dict(dev, q=dev["q"].flip(0).contiguous(), kv_len=(dev["kv_len"] - 7))
    want = [sd.sd_verify_shared(**a) for a in (dev, other)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = [sd.sd_verify_shared(**a, stream=s) for _ in range(4) for a, s in zip((dev, other), streams)]
        torch.cuda.synchronize()
        for i, (out, lse) in enumerate(got):
            assert torch.equal(out, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])


def test_shared_equals_verify_where_nothing_is_shared():
    import torch
    import paper_2505_12728_amd as sd
    d = inputs([300, 45, 8], [1], [3], 8, 8, 2, 128, seed=9)
    d["prefix_len"][0] = 0
    out, lse = call(d)
    ro, rl = sd.sd_verify_attention(*(d[n].cuda() for n in ("q", "k_cache", "v_cache")),
                                    torch.from_numpy(d["kv_len"]).cuda())
    A = reference(d, 1 / math.sqrt(128))[2]
    assert np.all(np.abs((out - ro).cpu().numpy()) <= 2.0 ** -11 * A)
    assert torch.allclose(lse, rl, atol=2.0 ** -11)


def test_shared_one_prefix_given_twice_is_one_group():
    # the same pages under two groups, and as one group: the same rows
    import torch
    d = inputs([30, 31, 32, 33], [500], [4], 4, 8, 2, 128, paged=True, seed=11)
    one, l1 = call(d)
    d["prefix_len"] = np.array([500, 500], np.int32)
    d["prefix_table"] = np.repeat(d["prefix_table"], 2, 0)
    d["group_start"] = np.array([0, 1, 4], np.int32)
    two, l2 = call(d)
    A = torch.from_numpy(reference(d, 1 / math.sqrt(128))[2]).cuda()
    assert bool(((one - two).abs() <= 2.0 ** -11 * A).all()) and torch.allclose(l1, l2, atol=2.0 ** -11)


def test_shared_equal_groups_without_bounds():
    import torch
    d = inputs([20, 21, 22, 23, 24, 25], [70, 80, 90], [2, 2, 2], 3, 4, 2, 64, seed=12)
    out, lse = call(d)
    d["group_start"] = None
    again, lse2 = call(d)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_shared_decreasing_bounds_stay_in_range():
    # a broken precondition: no fault, finite results, and sequences keep at
    # most one prefix (bounds are raised to the largest one before them)
    import torch
    d = inputs([20] * 6, [70, 80, 90], [2, 2, 2], 3, 4, 2, 64, seed=13)
    d["group_start"] = np.array([4, -7, 1000, 2], np.int32)
    out, _ = call(d)
    d["group_start"] = np.array([4, 4, 6, 6], np.int32)
    want, _ = call(d)
    assert torch.equal(out, want)
    # lengths and page ids out of range are clamped
    d = inputs([20] * 6, [70, 80, 90], [2, 2, 2], 3, 4, 2, 64, paged=True, seed=13)
    d["prefix_len"][:] = [-5, 100000, 90]
    d["kv_len"][0] = 99999
    d["prefix_table"][2, 0], d["page_table"][3, 0] = -4, 1 << 30
    out, _ = call(d)
    assert bool(torch.isfinite(out).all())


def test_shared_outputs_stream_graph_and_workspace():
    # given outputs and workspace, a stream of its own, lengths that change
    # between the replays of one captured call
    import torch
    import paper_2505_12728_amd as sd
    d = inputs([40, 13, 22], [900], [3], 4, 16, 2, 128, seed=14)
    dev = {n: torch.as_tensor(d[n]).cuda() for n in d if d[n] is not None}
    ws = torch.empty(sd.sd_verify_shared_workspace_size(3, 4, 16, 2, 128, 1, dev["k_prefix"].shape[1],
                                                        dev["k_cache"].shape[1], 1), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty(3, 4, 16, 128, device="cuda"), torch.empty(3, 4, 16, device="cuda")
    want, want_lse = sd.sd_verify_shared(**dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, none = sd.sd_verify_shared(**dev, lse=False, stream=side)
    side.synchronize()
    assert none is None and torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.sd_verify_shared(**dev, out=out, lse=lse, workspace=ws)
    for i in range(4):
        dev["prefix_len"].fill_((900, 33, 0, 517)[i])
        dev["kv_len"].copy_(torch.tensor([(40, 13, 22), (4, 0, 9), (1, 40, 3), (39, 38, 37)][i], dtype=torch.int32))
        out.fill_(7)
        ws.random_()                              # the workspace needs no initialisation
        graph.replay()
        torch.cuda.synchronize()
        want, want_lse = sd.sd_verify_shared(**dev)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_shared_runs_are_equal():
    import torch
    d = inputs([40] * 16, [3000], [16], 8, 8, 2, 128, paged=True, seed=15)
    out, lse = call(d)
    for _ in range(5):
        again, l2 = call(d)
        assert torch.equal(out, again) and torch.equal(lse, l2)


def test_shared_past_32_bit_offsets():
    # prefix pages at both ends of a pool of more than 2^32 elements
    import torch
    import paper_2505_12728_amd as sd
    Hkv, D = 8, 128
    P = (1 << 32) // (Hkv * 16 * D) + 3
    d = inputs([5, 16], [64], [2], 4, 8, Hkv, D, paged=True, seed=16)
    big = {}
    where = torch.tensor([0, P - 1, 1, P - 2, P - 3, 2])         # 4 prefix pages, 2 own ones
    for c in ("k_cache", "v_cache"):
        big[c] = torch.empty(P, Hkv, 16, D, dtype=torch.bfloat16, device="cuda")
        src = torch.from_numpy(np.concatenate([d["prefix_table"][0], d["page_table"][:, 0]])).long()
        big[c][where.cuda()] = d[c][src].cuda()
    table = where[:4][None].to(torch.int32).cuda()
    own = where[4:, None].to(torch.int32).contiguous().cuda()
    out, lse = call(d, **big, prefix_table=table, page_table=own)
    want, want_lse = call(d)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    del big
    torch.cuda.empty_cache()


def test_append_then_shared_attention():
    # as a server uses them: one video prompt goes into pages once, three
    # questions behind it into pages of their own, then their drafted blocks are
    # appended and verified; against the oracle's rotation and attention
    import torch
    import paper_2505_12728_amd as sd
    g = torch.Generator().manual_seed(21)
    Hq, Hkv, D, k, secs, theta = 8, 2, 128, 4, [16, 24, 24], 1e6
    n, asked = 150, [20, 7, 33]                                   # prompt; question lengths
    pages = [-(-n // 16)] + [-(-(a + k) // 16) for a in asked]
    perm = torch.randperm(sum(pages), generator=g).to(torch.int32)
    rows = torch.split(perm, pages)
    table = lambda rs: torch.nn.utils.rnn.pad_sequence(rs, batch_first=True).cuda()      # noqa: E731
    ptable, otable = table(rows[:1]), table(rows[1:])
    kc, vc = (torch.zeros(sum(pages), Hkv, 16, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    host = []

    def append(counts, lens, tab, pos):
        T = sum(counts)
        qkv = torch.randn(T, (Hq + 2 * Hkv) * D, generator=g)     # the projection's fp32 rows
        host.append((qkv, pos))
        dev = qkv.cuda()
        start = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda")
        return sd.sd_kv_append(dev[:, :Hq * D].view(T, Hq, D), dev[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D),
                               dev[:, (Hq + Hkv) * D:].view(T, Hkv, D), kc, vc,
                               torch.tensor(lens, dtype=torch.int32, device="cuda"), theta, pos=pos.cuda(),
                               sections=secs, row_start=start, page_table=tab)

    grid = torch.stack([torch.arange(n) // 30, torch.arange(n) // 6 % 5, torch.arange(n) % 6]).to(torch.int32)
    append([n], [n], ptable, grid)
    text = [torch.arange(a) + 40 for a in asked]
    append(asked, asked, otable, torch.cat(text).expand(3, -1).contiguous().to(torch.int32))
    blocks = [torch.arange(k) + 40 + a for a in asked]
    q = append([k] * 3, [a + k for a in asked], otable, torch.cat(blocks).expand(3, -1).contiguous().to(torch.int32))
    out, lse = sd.sd_verify_shared(q.view(3, k, Hq, D), kc, vc, torch.tensor([a + k for a in asked], dtype=torch.int32,
                                                                            device="cuda"),
                                   torch.tensor([n], dtype=torch.int32, device="cuda"), prefix_table=ptable,
                                   page_table=otable)
    bf = lambda x: torch.from_numpy(x).to(torch.bfloat16).double().numpy()               # noqa: E731
    parts = []
    for qkv, pos in host:
        x = qkv.view(len(qkv), -1, D).double().numpy()
        turned = oracle.rope_axes(x[:, :Hq + Hkv], pos.numpy(), secs, theta)
        parts.append((turned[:, :Hq], turned[:, Hq:], x[:, Hq + Hkv:]))
    own_k, own_v = np.zeros((2, 3, max(asked) + k, Hkv, D))
    at = 0
    for b, a in enumerate(asked):
        for c, i in ((own_k, 1), (own_v, 2)):
            c[b, :a] = parts[1][i][at:at + a]
            c[b, a:a + k] = parts[2][i][b * k:(b + 1) * k]
        at += a
    ref = oracle.verify_shared(bf(parts[2][0]).reshape(3, k, Hq, D), bf(own_k), bf(own_v), [a + k for a in asked],
                               bf(parts[0][1])[None], bf(parts[0][2])[None], [n], [0, 3], 1 / math.sqrt(D))
    # both sides round queries, keys and values to bf16 from values within 2^-20
    # of each other: a few land on the other side of a rounding border (2^-7 of
    # the element), one element in 2^-20 / 2^-8 = 2^-12.  A score's 128 products
    # then move by at most a few times 2^-7 |q k| scale = 2^-10
    ro, rl, A = ref
    assert np.all(np.abs(out.cpu().numpy() - ro) <= 2.0 ** -7 * A + 2.0 ** -7 * np.abs(ro))
    assert np.all(np.abs(lse.cpu().numpy() - rl) <= 2.0 ** -8)


def test_shared_binding_refuses():
    import torch
    import paper_2505_12728_amd as sd
    d = inputs([20, 21], [70], [2], 3, 4, 2, 64, seed=20)
    dev = {n: torch.as_tensor(d[n]).cuda() for n in d if d[n] is not None}

    def bad(error, match, **kw):
        with pytest.raises(error, match=match):
            sd.sd_verify_shared(**dict(dev, **kw))
    bad(ValueError, "come together", v_prefix=None)
    bad(ValueError, "both tables", k_prefix=None, v_prefix=None)
    bad(ValueError, "one entry per sequence", kv_len=dev["kv_len"][:1])
    bad(ValueError, "group_start", group_start=dev["group_start"][:1])
    bad(ValueError, "contiguous k_prefix", k_prefix=dev["k_cache"], v_prefix=dev["v_cache"])
    bad(ValueError, "same KV heads", k_prefix=dev["k_prefix"][:, :, :1].contiguous(),
        v_prefix=dev["v_prefix"][:, :, :1].contiguous())
    bad(TypeError, "out_dtype", out_dtype=torch.float16)
    bad(TypeError, "k_prefix", k_prefix=dev["k_prefix"].float(), v_prefix=dev["v_prefix"].float())
    bad(TypeError, "prefix_len", prefix_len=dev["prefix_len"].long())
    bad(ValueError, "shape", out=torch.empty(2, 3, 4, 63, device="cuda"))
    bad(ValueError, "shape", lse=torch.empty(2, 3, 3, device="cuda"))
    bad(ValueError, "GPU", kv_len=dev["kv_len"].cpu())
    bad(ValueError, "paged k_cache", page_table=torch.zeros(2, 2, dtype=torch.int32, device="cuda"))
    bad(sd.SDError, "WORKSPACE", workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    bad(sd.SDError, "INVALID", scale=float("nan"))
    f = {n: t.float() if t.dtype == torch.bfloat16 else t for n, t in dev.items()}
    with pytest.raises(sd.SDError, match="UNSUPPORTED"):
        sd.sd_verify_shared(**f, out_dtype=torch.bfloat16)
