"""The 8-bit cache at the top of its range, on the GPU: finite inputs up to the largest bf16, K rotated beyond it, in fresh blocks and
in blocks that hold rows; and attention over such values, which must not reach the queries that they are hidden from."""
import numpy as np
import pytest
import torch

from oracle import lowbit
from paper_2405_05329_amd import kvra, synth
from test_gpu_lowbit import attn_bound, bytes_dev, check_append, f64, random_cache, run_append, run_attn, workspace

pytestmark = pytest.mark.gpu
BASE = synth.ROPE_BASE
# the largest bf16; 248, 244, 240, 232 and 224 * 2^120; the largest that the scale 119 holds (448 * 2^119) and the one above it
TOP = np.array([0x7F7F, 0x7F78, 0x7F74, 0x7F70, 0x7F68, 0x7F60, 0x7F61], dtype=np.uint16)


@pytest.mark.parametrize("H,Hkv,d,prefix,c,base", [
    (2, 2, 64, 0, 70, 0.0), (2, 2, 64, 30, 100, BASE), (4, 2, 128, 63, 2, BASE), (8, 8, 128, 0, 1030, BASE), (3, 3, 128, 40, 1, 0.0),
])
def test_append_of_the_largest_values(H, Hkv, d, prefix, c, base):
    """Bit for bit the oracle's, and every value that a code stands for is finite in bf16."""
    rng = np.random.default_rng(21)
    _, k, v = synth.make_qkv(3, 74, c, H, Hkv, d)
    k, v = k.copy(), v.copy()
    for t in (k, v):
        few = rng.random(t.shape) < 0.05
        t[few] = rng.choice(TOP, int(few.sum())) | (rng.integers(0, 2, int(few.sum())) << 15).astype(np.uint16)
    k[c - 1, 0] = 0x7F7F                        # both halves of every pair: the rotation goes up to sqrt(2) times that
    k[c // 2, Hkv - 1] = 0xFF7F
    cap = prefix + c + 5
    kc, ks = random_cache(1, prefix, cap, Hkv, d)
    vc, vs = random_cache(2, prefix, cap, Hkv, d, std=2.0 ** 118)
    got = run_append(k, v, None, kc, vc, ks, vs, prefix, c, cap, H, Hkv, d, base)
    check_append(got, k, v, kc, vc, ks, vs, prefix, base)
    for cache, scale in ((got[0], got[2]), (got[1], got[3])):
        values = lowbit.cache_values(cache, scale)[prefix:prefix + c]
        assert np.abs(values).max() == 240 * 2.0 ** 120


def test_what_is_not_finite_stays_nan_beside_them():
    c, Hkv, d = 10, 2, 64
    k = np.full((c, Hkv, d), 0x7F7F, np.uint16)
    v = k.copy()
    k[3, 0, 5], k[4, 1, 6], v[5, 0, 7], v[6, 1, 8] = 0x7F80, 0xFFC0, 0xFF80, 0x7FC1
    kc, vc = np.zeros((c, Hkv, d), np.uint8), np.zeros((c, Hkv, d), np.uint8)
    ks, vs = np.zeros((1, Hkv), np.uint8), np.zeros((1, Hkv), np.uint8)
    got = run_append(k, v, None, kc, vc, ks, vs, 0, c, c, Hkv, Hkv, d, 0.0)
    for cache, bits in ((got[0], k), (got[1], v)):
        nan = (bits & 0x7FFF) >= 0x7F80
        assert np.array_equal((cache & 0x7F) == 0x7F, nan) and np.all(cache[~nan] == 0x77)
    assert np.all(got[2] == 247) and np.all(got[3] == 247)


@pytest.mark.parametrize("H,Hkv,d,prefix,c,tiled", [
    (8, 2, 128, 1699, 300, False), (4, 2, 64, 100, 200, False),       # slices
    (71, 1, 64, 4096, 600, True), (32, 32, 128, 3000, 777, True),     # tiled: the cache unpacked; converted tile by tile
])
def test_attention_beside_the_largest_values(H, Hkv, d, prefix, c, tiled):
    """All scores equal (q = 0), so that every weight is exactly 1 and the one large value of a component fits an fp32 sum (3.19e38 and
    small ones).  Rows that do not see it are as near the oracle as ever, those that do have it in their mean."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    assert (kvra.kvra_chunk_attn_q8_row_splits(prefix, c, H, Hkv, d, cus) == 0) == tiled
    n = prefix + c
    _, k, v = synth.make_qkv(5, 75, n, H, Hkv, d)
    v = v.copy()
    places = [(prefix + c // 3, 0, 1, 0x7F7F), (n - 1, Hkv - 1, 2, 0xFF7F), (prefix + c // 2, Hkv // 2, d - 1, 0x7F78)]
    for row, head, col, bits in places:
        v[row, head, col] = bits
    empty = [np.zeros((n, Hkv, d), np.uint8), np.zeros((n, Hkv, d), np.uint8), np.zeros(((n + 63) // 64, Hkv), np.uint8), np.zeros(((n + 63) // 64, Hkv), np.uint8)]
    kc, vc, ks, vs, _ = run_append(k, v, None, *empty, 0, n, n, H, Hkv, d, 0.0)
    q = np.zeros((c, H, d), np.uint16)
    got = f64(run_attn(q, [bytes_dev(t) for t in (kc, vc, ks, vs)], prefix, c, H, Hkv, d, 0.1, workspace()))
    want, bound = attn_bound(f64(q), lowbit.cache_values(kc, ks), lowbit.cache_values(vc, vs), prefix, 0.1)
    assert np.isfinite(got).all(), np.argwhere(~np.isfinite(got))[:3]
    err = np.abs(got - want)
    assert np.all(err <= bound), (float((err / bound).max()), np.argwhere(err > bound)[:3])
    for row, head, col, _ in places:
        seen = np.abs(got[row - prefix:, head * (H // Hkv), col])
        assert np.all(seen > 1e30) and np.all(np.abs(got[:row - prefix, head * (H // Hkv), col]) < 1e30)
