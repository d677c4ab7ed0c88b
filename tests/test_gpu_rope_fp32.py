"""sd_rope, sd_kv_append: fp32 sines and cosines, and what the binding refuses
besides."""

import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("far,T", [(100, 300), (100000, 3000)])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("append", [False, True])
def test_fp32_turns_are_rounded_once(far, T, inverse, append):
    # pairs (1, 0) become (cos, sin) and no product rounds: half a step of the
    # type, and what float64 leaves of the angle (20 * 2^-53 of the position, see
    # test_gpu_rope.py; 2^-50 from its reduction and its functions)
    import torch
    import paper_2505_12728_amd as sd
    if append and inverse:
        pytest.skip("the append turns forward only")
    g = torch.Generator().manual_seed(41)
    pos = torch.randint(-far, far, (2, T), generator=g, dtype=torch.int32)
    x = torch.zeros(T, 2, 128)
    x[..., :64] = 1.0
    secs = [24, 40]
    if append:
        kc, vc = torch.zeros(1, T, 2, 128, device="cuda"), torch.zeros(1, T, 2, 128, device="cuda")
        y = sd.sd_kv_append(x.cuda(), x.cuda(), x.cuda(), kc, vc, torch.tensor([T], dtype=torch.int32, device="cuda"),
                            1e6, pos=pos.cuda(), sections=secs)
        assert kc[0].equal(y)
    else:
        y = sd.sd_rope(x.cuda(), pos.cuda(), 1e6, sections=secs, inverse=inverse)
    ref = oracle.rope_axes(x.numpy(), pos.numpy(), secs, 1e6, inverse=inverse)
    err = np.abs(y.cpu().numpy() - ref) - 2.0 ** -24 * np.abs(ref)
    assert np.all(err <= 20 * 2.0 ** -53 * far + 2.0 ** -50), err.max()


def test_rope_needs_positions():
    import torch
    import paper_2505_12728_amd as sd
    with pytest.raises(ValueError, match="pos"):
        sd.sd_rope(torch.zeros(3, 2, 64, device="cuda"), None, 1e4)
