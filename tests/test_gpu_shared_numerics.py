"""sd_verify_shared where its arithmetic can lose bits or rows: bf16 outputs that
cancel, maxima far above the keys before them, scores of -inf, log-sum-exps of
thousands joined from many partials, infinite values, merge waves of several rows.

Lists are long enough that a work-group's segment spans several 64-key tiles
(20000 keys of 8 pairs or more are at least nine tiles for each of 256 of them)."""

import math

import numpy as np
import pytest

from tests.test_gpu_verify_shared import call, check, inputs, reference, roomy

pytestmark = pytest.mark.gpu


def out_type(kind):
    import torch
    return torch.bfloat16 if kind == "bf16" else torch.float32


# ------------------------------------------------ bf16 outputs that cancel

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("wide", [False, True])
def test_shared_bf16_outputs_are_off_by_their_own_rounding(D, wide):
    # few keys of values that cancel: out is far below A, the mean of |V|, and
    # its own rounding (half a step, 2^-8 of it at most) far below what weights
    # of eight bits would leave, 2^-9 A.  The rest as for fp32 outputs: 2^-12 A,
    # of which weights of 16 bits take 2^-16
    d = inputs([4, 5, 6, 7, 9] * 4, [3], [20], 4, 16, 1, D, seed=31)
    for n in ("v_cache", "v_prefix"):
        sign = d[n].float().sign()
        d[n] = (sign * (1 + d[n].float().abs() / 64)).to(d[n].dtype)
    ro, rl, A = reference(d, 1 / math.sqrt(D))
    out, lse = call(d, out_dtype=out_type("bf16"), **(roomy(d) if wide else {}))
    err = np.abs(out.double().cpu().numpy() - ro) - 2.0 ** -8 * np.abs(ro) - 2.0 ** -12 * A
    assert np.all(err <= 0), err.max()
    assert np.all(np.abs(lse.cpu().numpy() - rl) <= 2.0 ** -12)


# --------------------------------------------- maxima far above those before

def long_groups(rows, seed, keys=20000, Hkv=4, D=64, dtype="bf16"):
    """One group of `rows` rows a KV head over one long prefix; q[.., 0] is 1."""
    d = inputs([8] * (rows // 8), [keys], [rows // 8], 8, Hkv, Hkv, D, dtype, seed=seed)
    d["q"][..., 0] = 1.0
    for n in ("k_cache", "k_prefix"):
        d[n][..., 0] = 0.0
    return d


def every_other_tile(d, channel, value):
    n = int(d["prefix_len"][0])
    low = np.nonzero(np.arange(n) // 64 % 2 == 0)[0]
    d["k_prefix"][0, low, :, channel] = value


@pytest.mark.parametrize("low", [50.0, 5e4, 1e6, 1e8])
@pytest.mark.parametrize("rows", [64, 256])
def test_shared_tiles_far_below_the_maximum(low, rows):
    # every other tile of 64 keys lies lower by `low`: segments that begin in
    # one raise their maximum by that much, and the tiles above it keep their bits
    d = long_groups(rows, seed=32)
    every_other_tile(d, 0, -8 * low)
    ref = reference(d, 1 / 8)
    for kind in ("hilo", "bf16"):
        out, lse = call(d, out_dtype=out_type(kind), **(roomy(d) if kind == "bf16" else {}))
        check(d, out, lse, ref, kind)


# ------------------------------------------------------- scores of -inf

@pytest.mark.parametrize("how", ["overflow", "key"])
@pytest.mark.parametrize("rows", [64, 256])
@pytest.mark.parametrize("level", [-300.0, 300.0])
def test_shared_tiles_of_minus_infinity(how, rows, level):
    # every other tile's scores are -inf (a product past fp32's range, or a key of
    # -inf): weight 0, and the tiles behind one are as they are alone, wherever
    # their own scores lie
    d = long_groups(rows, seed=33)
    d["q"][..., 0] = 1e20 if how == "overflow" else 1.0
    d["q"][..., 1] = 1.0
    for n in ("k_cache", "k_prefix"):
        d[n][..., 1] = 8 * level
    every_other_tile(d, 0, -1e20 if how == "overflow" else -math.inf)
    ref = reference(d, 1 / 8)
    # the products' sum passes 300 sqrt(D): bound of the scores as for a scale of
    # 300 / 8 units
    for kind in ("hilo", "bf16"):
        out, lse = call(d, out_dtype=out_type(kind), **(roomy(d) if kind == "bf16" else {}))
        check(d, out, lse, ref, kind, 300 / 8)


@pytest.mark.parametrize("rows", [64, 256])
@pytest.mark.parametrize("scale", [64.0, -64.0])
def test_shared_tiles_below_the_range_once_scaled(rows, scale):
    # every other tile's products are finite, -3e37, and pass fp32's range with the
    # scale alone: weight 0 as well
    d = long_groups(rows, seed=40)
    d["q"] = d["q"] / 512
    d["q"][..., 0] = 1e19 * np.sign(scale)
    d["q"][..., 1] = np.sign(scale)
    for n in ("k_cache", "k_prefix"):
        d[n][..., 1] = -300 / 64
    every_other_tile(d, 0, -3e18)
    ref = reference(d, scale)
    for kind in ("hilo", "bf16"):
        out, lse = call(d, scale=scale, out_dtype=out_type(kind), **(roomy(d) if kind == "bf16" else {}))
        check(d, out, lse, ref, kind, 300 / 8)


@pytest.mark.parametrize("kind", ["hilo", "bf16", "f32"])
def test_shared_only_minus_infinity_is_no_key(kind):
    # rows all of whose scores are -inf see nothing: out 0 and lse -inf
    d = inputs([40, 300], [200], [2], 4, 4, 2, 64, "f32" if kind == "f32" else "bf16", seed=34)
    d["q"][..., 0] = 1.0
    for n in ("k_cache", "k_prefix"):
        d[n][..., 0] = -math.inf
    out, lse = call(d, out_dtype=out_type(kind))
    assert not out.any() and bool((lse == -math.inf).all())


# ------------------------------------------ large log-sum-exps in many partials

def high_scores(rows, level, dtype, seed, keys=20000, Hkv=4):
    """Scores of `level` plus multiples of 2^-6 that float32 sums exactly; values
    of 1 in the first half of the prefix and of -1 behind it."""
    import torch
    d = inputs([8] * (rows // 8), [keys], [rows // 8], 8, Hkv, Hkv, 64, dtype, seed=seed)
    g = torch.Generator().manual_seed(seed)
    d["q"].zero_()
    d["q"][..., 0] = d["q"][..., 1] = 1.0
    for n in ("k_cache", "k_prefix"):
        d[n].zero_()
        d[n][..., 0] = 8.0 * level
        d[n][..., 1] = torch.randint(-64, 64, d[n].shape[:-1], generator=g).to(d[n].dtype) / 8
    d["v_prefix"][0, :keys // 2] = 1.0
    d["v_prefix"][0, keys // 2:] = -1.0
    return d


@pytest.mark.parametrize("rows", [64, 256])
def test_shared_partials_of_high_scores(rows):
    # scores near 30208, their log-sum-exp in fp32 would be off by 2^-10: as a
    # weight between partials that is 2^-10 of what they differ by, 2 A.  Here
    # the weights are off by the exponents' rounding alone.  A segment adds at most
    # 40 tiles, each key's weight through 4 sums a tile (half of them behind it) and
    # then the merge's 64 candidates, 2^-24 each, and a weight is off by 2^-22:
    # under 2^-16 A in all
    d = high_scores(rows, 30208.0, "bf16", 35)
    ro, rl, A = reference(d, 1 / 8)
    out, lse = call(d, out_dtype=out_type("hilo"))
    err = np.abs(out.cpu().numpy() - ro)
    assert np.all(err <= 2.0 ** -16 * A), (err / A).max()
    # lse passes five roundings of its own size (maximum, its sum with the
    # logarithm, log2 e twice, the scale)
    assert np.all(np.abs(lse.cpu().numpy() - rl) <= 5 * 2.0 ** -24 * np.abs(rl))
    out, lse = call(d, out_dtype=out_type("bf16"), **roomy(d))
    err = np.abs(out.double().cpu().numpy() - ro) - 2.0 ** -8 * np.abs(ro)
    assert np.all(err <= 2.0 ** -15 * A), (err / A).max()


@pytest.mark.parametrize("level", [0.0, 300.0, 30208.0])
def test_shared_f32_is_float64_until_its_outputs(level):
    # (the scale 1 / 8 is exact in float32) sums of 10^4 keys in float64, 2^-36 A; 64
    # additions to each score, 2^-53 of it each, here and in the reference, and
    # that twice, in the weights and in their sum: 2^-45 of the level; then one
    # rounding of the output
    d = high_scores(16, level, "f32", 36, keys=9000, Hkv=2)
    import torch
    g = torch.Generator().manual_seed(36)
    d["q"][..., 2:] = torch.randn(d["q"][..., 2:].shape, generator=g)
    for n in ("k_cache", "k_prefix"):
        d[n][..., 2:] = torch.randn(d[n][..., 2:].shape, generator=g) / 4
    ro, rl, A = reference(d, 1 / 8)
    out, lse = call(d)
    err = np.abs(out.cpu().numpy() - ro) - 2.0 ** -24 * np.abs(ro)
    off = 2.0 ** -36 + 2.0 ** -45 * level
    assert np.all(err <= off * A), (err / A).max()
    assert np.all(np.abs(lse.cpu().numpy() - rl) <= 2.0 ** -24 * np.abs(rl) + off)


# ------------------------------------------------------ infinite values

@pytest.mark.parametrize("keys", [200, 9000])
def test_shared_f32_infinite_values_stay_infinite(keys):
    # a value of +inf that a row sees makes that channel +inf, not NaN, and no
    # other channel or row knows of it
    d = inputs([9, 64, 70, 131], [keys], [4], 5, 4, 2, 128, "f32", seed=37)
    d["v_prefix"][0, keys - 1, 1, 7] = math.inf          # every row of heads 2 and 3
    for b, n in enumerate((9, 64, 70, 131)):
        d["v_cache"][b, n - 1, 0, 3] = -math.inf          # the last block row of heads 0 and 1
    with np.errstate(invalid="ignore"):
        ref = reference(d, 1 / math.sqrt(128))
    assert not np.isnan(ref[0]).any()
    out, lse = call(d)
    out = out.cpu().numpy()
    bad = np.isinf(ref[0])
    assert bad[:, :, 2:, 7].all() and bad[:, 4, :2, 3].all() and bad.sum() == 4 * 5 * 2 + 4 * 2
    assert np.array_equal(out[bad], ref[0][bad].astype(np.float32))
    assert np.all(np.abs(out[~bad] - ref[0][~bad]) <= 2.0 ** -19 * ref[2][~bad])
    assert np.all(np.abs(lse.cpu().numpy() - ref[1]) <= 1e-5)


# -------------------------------------- forms of the kernels that no other test runs

@pytest.mark.parametrize("kind", ["hilo", "bf16", "f32"])
@pytest.mark.parametrize("B,k,Hq,Hkv", [(60, 7, 45, 5), (90, 7, 45, 5), (50, 7, 56, 8)])
def test_shared_merge_waves_of_several_rows(kind, B, k, Hq, Hkv):
    # 16384 rows and more: a merge wave takes two or three of them, of 315 or 392
    # rows a sequence, so that last shares are short and some waves have none
    lens = [k + (11 * b) % 90 for b in range(B)]
    sizes = [B // 2, 0, B // 3]
    d = inputs(lens, [150, 9, 65], sizes, k, Hq, Hkv, 64, "f32" if kind == "f32" else "bf16", seed=38, lead=1,
               left=B - sum(sizes) - 1)
    out, lse = call(d, out_dtype=out_type(kind))
    check(d, out, lse, reference(d, 1 / 8), kind)


@pytest.mark.parametrize("kind", ["hilo", "bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_shared_rows_that_see_a_nonfinite_key(kind, bad):
    # the last key of a sequence, in one channel: the last block row alone.  Its
    # scores are NaN or +inf, which leave no softmax, or -inf, a key of no weight
    d = inputs([9, 64, 70, 131], [200], [4], 5, 4, 2, 128, "f32" if kind == "f32" else "bf16", seed=39)
    for b, n in enumerate((9, 64, 70, 131)):
        d["k_cache"][b, n - 1, :, 11] = bad
    d["q"][:, :, 0, 11], d["q"][:, :, 1:, 11] = 1.0, -1.0
    with np.errstate(invalid="ignore"):
        ro, rl, A = reference(d, 1 / math.sqrt(128))
    none = np.isnan(rl)
    assert none[:, 4].sum() == {math.inf: 4, -math.inf: 12}.get(bad, 16) and not none[:, :4].any()
    out, lse = call(d, out_dtype=out_type(kind))
    assert np.array_equal(np.isnan(out.float().cpu().numpy()).all(-1), none)
    assert np.array_equal(np.isnan(lse.cpu().numpy()), none)
    out[torch_mask(none)], lse[torch_mask(none)] = 0.0, 0.0
    ro[none], rl[none], A[none] = 0.0, 0.0, 0.0
    check(d, out, lse, (ro, rl, A), kind)


def torch_mask(x):
    import torch
    return torch.from_numpy(x).cuda()
