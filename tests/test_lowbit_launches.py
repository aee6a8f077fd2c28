"""What the calls over the 8-bit cache and the 4-bit weights enqueue, read off a stand-in for the HIP runtime (lowbit_launches.py): no GPU."""
import random

import pytest

from lowbit_launches import MIB, append, attn, linear, names, pack, record
from paper_2405_05329_amd import kvra
from test_gpu_lowbit import TILED
from test_gpu_lowbit_converting import CUT, SHORT
from test_gpu_lowbit_linear import KERNELS
from test_gpu_lowbit_long import SLICES, TILES


def _shapes(count):
    """Caches from a few rows to several times what the smallest workspace holds, one token to thousands."""
    rng = random.Random(8)
    out = []
    while len(out) < count:
        d, Hkv = rng.choice([64, 128]), rng.choice([1, 2, 3, 5, 8, 16, 32])
        n, c = int(2.0 ** rng.uniform(4, 19)), int(2.0 ** rng.uniform(0, 12))
        if c <= n and n * Hkv * d < 1 << 29:
            out.append((Hkv * rng.choice([1, 2, 4, 8, 32]), Hkv, d, n - c, c))
    return out


def test_slices_or_tiles_is_the_querys_answer_with_any_workspace():
    """Slices and tiles round differently; spare room in the workspace may only choose between the two tiled ways."""
    shapes, sizes = _shapes(400), (128 * MIB, 300 * MIB, 1 << 40)
    results = iter(record([attn(*s, size) for s in shapes for size in sizes]))
    met = set()
    for H, Hkv, d, prefix, c in shapes:
        splits = kvra.kvra_chunk_attn_q8_row_splits(prefix, c, H, Hkv, d, 256)
        for size in sizes:
            r = next(results)
            kernels = names(r)
            if splits > 0:
                rows = 16 if c * (H // Hkv) <= 16 else 32
                assert kernels == [f"attn_rows_q8_kernel<{d}, {rows // 16}>"], (H, Hkv, d, prefix, c, size)
                assert r["launches"][0]["grid"] == [Hkv, splits, -(-c * (H // Hkv) // rows)]
            else:
                assert kernels in ([f"chunk_attn_q8_kernel<{d}>"], [f"unpack_q8_kernel<{d}>", f"chunk_attn_kernel<{d}>"]), (H, Hkv, d, prefix, c, size)
            met.add((d, kernels[0].split("<")[0]))
    assert len(met) == 6, met


def test_nothing_is_allocated():
    calls = [attn(*s) for s in _shapes(60)] + [append(32, 8, 128, 100, 1), append(32, 8, 128, 0, 5000), pack(704, 1088)]
    calls += [linear(m, n, k, form) for m, n, k in ((1, 4096, 4096), (77, 4096, 4096), (777, 4096, 11008), (4096, 4096, 4096))
              for form in ("plain", "residual", "swiglu")]
    for call, r in zip(calls, record(calls)):
        assert r["rc"] == kvra.KVRA_OK and r["launches"] and r["mallocs"] == 0, call


@pytest.mark.parametrize("m,n,k", KERNELS)
def test_the_gpu_tests_of_the_4_bit_linear_layer_meet_every_kernel(m, n, k):
    """Each shape gets the kernel that tests/test_gpu_lowbit_linear.py has it for."""
    for form, dual, short in (("plain", "false", KERNELS[m, n, k][0]), ("swiglu", "true", KERNELS[m, n, k][1])):
        kind, args = short[:-1].split("<")
        want = f"linear_w4_{kind}_kernel<{dual}, {args}{', 8' if kind == 'rows' else ''}>"
        result, = record([linear(m, n, k, form)])
        assert names(result) == [want], (form, names(result))


@pytest.mark.parametrize("H,Hkv,d,prefix,c", TILES)
def test_the_gpu_tests_of_long_caches_meet_the_kernels_they_are_for(H, Hkv, d, prefix, c):
    """More than 64 steps to a piece of the tiled kernel, converting or over the unpacked cache."""
    result, = record([attn(H, Hkv, d, prefix, c)])
    assert (names(result)[0] == f"unpack_q8_kernel<{d}>") == TILES[H, Hkv, d, prefix, c]
    pieces = kvra.kvra_chunk_attn_pieces(prefix, c, H, Hkv, d, 256)
    assert max(p["jt1"] - p["jt0"] for p in pieces) > 64


def test_the_tiled_gpu_tests_meet_both_ways():
    shapes = TILED + SHORT + CUT
    for r, s in zip(record([attn(*s) for s in SHORT + CUT]), SHORT + CUT):
        assert names(r) == [f"chunk_attn_q8_kernel<{s[2]}>"], s
    for s in CUT:
        assert kvra.kvra_chunk_attn_plan(s[3], s[4], s[0], s[1], s[2], 256)["partial_pieces"] > 0
    ways = {d: {names(r)[0] for r in record([attn(*s) for s in shapes if s[2] == d])} for d in (64, 128)}
    assert ways == {d: {f"unpack_q8_kernel<{d}>", f"chunk_attn_q8_kernel<{d}>"} for d in (64, 128)}


def test_the_long_slices_have_more_than_64_tiles_a_wave():
    for H, Hkv, d, prefix, c in SLICES:
        splits = kvra.kvra_chunk_attn_q8_row_splits(prefix, c, H, Hkv, d, 256)
        assert splits > 0 and (prefix + c) // 64 > 64 * 8 * splits, (H, Hkv, d)
