"""The tiled attention kernel that makes the 8-bit cache's values on the way into its rings, at head_dim 64: the launches that get it have
many heads, or caches too long to unpack.  (tests/test_lowbit_launches.py asserts which way each shape goes.)"""
import numpy as np
import pytest
import torch

import test_gpu_lowbit as base
import test_gpu_lowbit_range as top

pytestmark = pytest.mark.gpu

# (H, Hkv, d, prefix, c): whole units of a short cache; groups of 8; cut units, 224 rows to a tile; cut units of a long cache in groups of 4
SHORT = [(128, 128, 64, 116, 262), (1024, 128, 64, 435, 34), (128, 128, 64, 747, 257)]
CUT = [(48, 48, 64, 12000, 400), (192, 48, 64, 20252, 77)]


@pytest.mark.parametrize("H,Hkv,d,prefix,c", SHORT + CUT)
def test_is_the_bf16_kernels(H, Hkv, d, prefix, c):
    base.test_attention_of_many_rows_is_the_bf16_kernels(H, Hkv, d, prefix, c)


@pytest.mark.parametrize("H,Hkv,d,prefix,c", SHORT[:1] + CUT[:1])
def test_in_a_graph(H, Hkv, d, prefix, c):
    base.test_attention_in_a_graph(H, Hkv, d, prefix, c)


@pytest.mark.parametrize("H,Hkv,d,prefix,c", SHORT[:2])
def test_beside_the_largest_values(H, Hkv, d, prefix, c):
    top.test_attention_beside_the_largest_values(H, Hkv, d, prefix, c, True)


@pytest.mark.parametrize("H,Hkv,d,prefix,c", SHORT + CUT[:1])
def test_nan_reaches_those_that_see_it(H, Hkv, d, prefix, c):
    """A NaN in each of many rows at once, each in a head of its own: in K it makes what sees the row NaN, in V the component that holds it;
    what does not see it is as it was up to rounding, other heads bit for bit."""
    n, G = prefix + c, H // Hkv
    q = base.synth.normal_bf16(9, 65, 0, (c, H, d))
    kc, ks = base.random_cache(7, n, n, Hkv, d)
    vc, vs = base.random_cache(8, n, n, Hkv, d)
    call = lambda k, v: base.run_attn(q, [base.bytes_dev(t) for t in (k, v, ks, vs)], prefix, c, H, Hkv, d, 0.125, base.workspace())
    clean = call(kc, vc)
    # A wave that meets a NaN may take another exponent reference: its other rows then round otherwise, each result within its bound of
    # the same exact value, that for scale * Q as rounded.  That one's scores are off by 2^-8 of their terms (at most 11 here) at most, which
    # moves the bound's weights by a factor within exp(2 * 11 * 2^-8) = 1.09.
    apart = 2 * 1.1 * base.attn_bound(base.f64(q), base.lowbit.cache_values(kc, ks), base.lowbit.cache_values(vc, vs), prefix, 0.125)[1]
    # rows of the chunk's first and last keys, around the borders of blocks and tiles, and in the prefix
    rows = sorted({r for r in (0, prefix - 1, prefix, prefix + 1, prefix + c // 3, n - 2, n - 1, *(b + o for b in range(prefix // 64 * 64, n, 64) for o in (-1, 0, 31, 32)))
                   if 0 <= r < n})
    for which in range(2):
        k, v = kc.copy(), vc.copy()
        hit = {}
        for i, row in enumerate(rows):
            head = (5 * i + 3) % Hkv
            if head not in hit:
                hit[head] = row
                (k, v)[which][row, head, row % d] = (0x7F, 0xFF)[which]
        assert len(hit) >= min(len(rows), Hkv // 2)
        got = call(k, v)
        others = [h for h in range(H) if h // G not in hit]
        assert np.array_equal(got[:, others], clean[:, others])
        for head, row in hit.items():
            mine, r = slice(head * G, head * G + G), max(row - prefix, 0)
            seen = base.f64(got[r:, mine])
            assert np.isnan(seen if which == 0 else seen[..., row % d]).all(), (head, row)
            a, b = base.f64(got[:r, mine]), base.f64(clean[:r, mine])
            assert np.all(np.abs(a - b) <= apart[:r, mine]), (head, row)
