"""Which tile sd_verify_shared takes (CPU: the plan alone, 256 compute units).

The workspace tells: partials [(prefix pairs + work-groups) rows per tile + (own
pairs + work-groups) own rows, D + 2], of 4 bytes (8 for fp32 inputs)."""

import pytest

import paper_2505_12728_amd as sd


def partial_bytes(tile, wgs, B, k, Hq, Hkv, D, G, size):
    kg = k * Hq // Hkv
    prefix_pairs = Hkv * (B * kg // tile + G)
    own_pairs = B * Hkv * -(-kg // tile)
    own_rows = min(-(-kg // 16) * 16, tile)
    return ((prefix_pairs + wgs) * tile + (own_pairs + wgs) * own_rows) * (D + 2) * size


# B, k, Hq, Hkv, D, G, own capacity: the calls of test_shared_roomy_caches and of
# test_gpu_shared_numerics.py in prefix caches of 2^18 keys
ROOMY = [(32, 8, 1, 1, 128, 1, 23), (40, 4, 28, 4, 128, 2, 64), (16, 16, 2, 2, 128, 1, 48), (37, 7, 8, 4, 64, 1, 43),
         (48, 5, 16, 1, 128, 3, 73), (3, 16, 16, 1, 64, 1, 112), (20, 4, 16, 1, 64, 1, 12), (20, 4, 16, 1, 128, 1, 12),
         (32, 8, 4, 4, 64, 1, 11)]


@pytest.fixture(autouse=True)
def no_device():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the plan follows the device's compute units")


@pytest.mark.parametrize("case", ROOMY, ids=str)
def test_bf16_outputs_over_long_caches_take_tiles_of_256_rows(case):
    B, k, Hq, Hkv, D, G, cap = case
    got = sd.sd_verify_shared_workspace_size(B, k, Hq, Hkv, D, G, 1 << 18, cap, sd.SD_BF16)
    assert got == partial_bytes(256, 256, B, k, Hq, Hkv, D, G, 4)
    assert got > partial_bytes(128, 256, B, k, Hq, Hkv, D, G, 4)


@pytest.mark.parametrize("case", [(16, 6, 32, 8, 128, 1, 16016, 704), (4, 1, 32, 32, 128, 1, 1136, 64),
                                  (24, 8, 28, 4, 128, 3, 6528, 528), (8, 8, 8, 4, 64, 1, 20000, 11)], ids=str)
def test_few_rows_or_keys_take_tiles_of_128_rows(case):
    B, k, Hq, Hkv, D, G, pcap, cap = case
    got = sd.sd_verify_shared_workspace_size(B, k, Hq, Hkv, D, G, pcap, cap, sd.SD_BF16)
    assert got == partial_bytes(128, 256, B, k, Hq, Hkv, D, G, 4)


def test_fp32_takes_tiles_of_16_rows_and_partials_of_float64():
    got = sd.sd_verify_shared_workspace_size(5, 4, 4, 1, 64, 2, 6080, 6000, sd.SD_F32)
    assert got == partial_bytes(16, 512, 5, 4, 4, 1, 64, 2, 8)
