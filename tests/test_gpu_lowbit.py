"""The 8-bit cache and the 4-bit weights on the GPU against the fp64 oracle.

Tolerances, from the roundings the calls are allowed (u = 2^-8 is a bf16 rounding's largest relative error):
  append, pack   none: what is stored is the oracle's, bit for bit (K is rotated in fp64; an angle off by 1e-12 moves one value
                 in 10^10 across a rounding border).  Q: one unit in the last place of bf16 at most, as kvra_append_kv's.
  attention      weights rounded to bf16 for the product with V: u * sum w |v|; the result: u * |out|; fp32 scores off by
                 e = (d + 8) 2^-24 * sum |terms| change every weight by a factor within 1 +- 2 e; fp32 sums of the weights and of
                 the products over n keys: (n / 64 + 80) 2^-23 (the lanes' sums of a tile, then one addition per tile and merge)
  linear         the result: u * |out|; fp32 accumulation in any order: (k / 32 + 48) 2^-24 * sum |terms| (a product of 32, the
                 chain of them, the waves' sums); the SwiGLU's exponential and quotient: 2^-20 of it
"""
import numpy as np
import pytest
import torch

from oracle import kvra_oracle as orc
from oracle import lowbit
from paper_2405_05329_amd import kvra, synth
from gpu_pipeline import to_bits, to_dev

pytestmark = pytest.mark.gpu
U = 2.0 ** -8
BASE = synth.ROPE_BASE


def f64(bits):
    return orc.bf16_bits_to_f64(bits)


def bytes_dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def workspace():
    """Scratch full of NaN, counters zero."""
    w = torch.full((kvra.kvra_chunk_attn_q8_workspace_bytes(),), 0xFF, dtype=torch.uint8, device="cuda")
    w[:16384] = 0
    return w


def random_cache(seed, rows, capacity, Hkv, d, std=1.0, spread=0):
    """(codes, scales) of a cache whose first `rows` rows came in at once; the others, and scales of blocks that hold none, are
    bytes that mean NaN.  spread: the blocks' magnitudes differ by up to 2^spread."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, Hkv, d)) * std
    if spread:
        x *= np.repeat(2.0 ** rng.integers(-spread, spread + 1, ((rows + 63) // 64, Hkv)), 64, axis=0)[:rows, :, None]
    cache = np.full((capacity, Hkv, d), 0x7F, np.uint8)
    scale = np.full(((capacity + 63) // 64, Hkv), 0xFF, np.uint8)
    if rows:
        lowbit.append_rows(cache, scale, x, 0)
    return cache, scale


# ---- append ------------------------------------------------------------------------------------------------------------
def run_append(k, v, q, kc, vc, ks, vs, prefix, c, cap, H, Hkv, d, base, in_place=False):
    dev = [bytes_dev(t) for t in (kc, vc, ks, vs)]
    qd = to_dev(q) if q is not None else None
    qo = qd if in_place or q is None else torch.full_like(qd, 7.0)
    kvra.kvra_append_kv_q8(to_dev(k), to_dev(v), qd, qo, *dev, prefix, c, cap, H, Hkv, d, base)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in dev] + [None if qo is None else to_bits(qo)]


def check_append(got, k, v, kc, vc, ks, vs, prefix, base):
    want = [t.copy() for t in (kc, vc, ks, vs)]
    lowbit.append_rows(want[0], want[2], lowbit.rotate(f64(k), prefix, base), prefix)
    lowbit.append_rows(want[1], want[3], f64(v), prefix)
    for name, g, w in zip(("k", "v", "k_scale", "v_scale"), got, want):
        assert np.array_equal(g, w), (name, int((g != w).sum()), np.argwhere(g != w)[:3])


@pytest.mark.parametrize("H,Hkv,d,prefix,c,base", [
    (2, 2, 64, 0, 1, BASE), (4, 2, 64, 63, 1, BASE), (4, 2, 64, 63, 2, BASE), (3, 3, 128, 64, 64, BASE), (3, 3, 128, 1, 63, BASE),
    (5, 1, 128, 40, 200, BASE), (71, 1, 64, 129, 77, BASE), (32, 32, 128, 15001, 1, BASE), (32, 8, 128, 20000, 333, BASE),
    (2, 2, 64, 70, 100, 0.0), (8, 8, 128, 0, 1030, 500000.0), (32, 32, 128, 100, 2500, BASE),      # several heads per workgroup
    (2, 1, 64, 3, 9000, BASE), (2, 2, 128, 16000000, 5, BASE), (2, 2, 64, 5000, 70, 0.125),       # far positions; angles beyond 2^26
])
def test_append(H, Hkv, d, prefix, c, base):
    if prefix > 100000:                # the cache of a far position is not made on the host
        return far_append(H, Hkv, d, prefix, c, base)
    cap = prefix + c + 5
    q, k, v = synth.make_qkv(3, 71, c, H, Hkv, d)
    kc, ks = random_cache(1, prefix, cap, Hkv, d)
    vc, vs = random_cache(2, prefix, cap, Hkv, d)
    got = run_append(k, v, q, kc, vc, ks, vs, prefix, c, cap, H, Hkv, d, base)
    check_append(got, k, v, kc, vc, ks, vs, prefix, base)
    # Q: the bits kvra_append_kv leaves
    qd, cache = to_dev(q), torch.zeros((cap, Hkv, d), dtype=torch.bfloat16, device="cuda")
    kvra.kvra_append_kv(to_dev(k), to_dev(v), qd, cache, torch.zeros_like(cache), prefix, c, cap, H, Hkv, d, base)
    assert np.array_equal(got[4], to_bits(qd))


def far_append(H, Hkv, d, prefix, c, base):
    """Rows near 2^24: the cache lives on the GPU alone, what lies around the written rows has to stay."""
    q, k, v = synth.make_qkv(3, 72, c, H, Hkv, d)
    cap = prefix + c + 3
    caches = [torch.full((cap, Hkv, d), 0x55, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full(((cap + 63) // 64, Hkv), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
    kvra.kvra_append_kv_q8(to_dev(k), to_dev(v), None, None, *caches, *scales, prefix, c, cap, H, Hkv, d, base)
    first = prefix // 64 * 64
    for cache, scale, new in zip(caches, scales, (lowbit.rotate(f64(k), prefix, base), f64(v))):
        # (positions from `first` on: a block-aligned piece behaves like a cache of its own)
        want, ws = np.full((cap - first, Hkv, d), 0x55, np.uint8), np.full(((cap - first + 63) // 64, Hkv), 127, np.uint8)
        lowbit.append_rows(want, ws, new, prefix - first)
        assert np.array_equal(cache[first:].cpu().numpy(), want) and np.array_equal(scale[first // 64:].cpu().numpy(), ws)
        assert bool((cache[:first] == 0x55).all()) and bool((scale[:first // 64] == 127).all())


def test_a_scale_grows_shrinks_not_and_rows_behind_stay():
    """Token by token into one block, magnitudes up and down by powers of two and borders of the scale; in place for Q."""
    H, Hkv, d, cap = 2, 2, 64, 75
    rng = np.random.default_rng(11)
    kc, vc = np.full((cap, Hkv, d), 0x7F, np.uint8), np.full((cap, Hkv, d), 0x81, np.uint8)
    ks, vs = np.full((2, Hkv), 0xFF, np.uint8), np.full((2, Hkv), 3, np.uint8)
    at = 0
    for c, gain in ((1, 1.0), (2, 2.0 ** -20), (5, 300.0), (1, 0.0), (3, 2.0 ** 40), (20, 1.0), (40, 2.0 ** -60)):
        x = orc.f64_to_bf16_bits(rng.standard_normal((c, Hkv, d)) * gain)
        y = orc.f64_to_bf16_bits(rng.choice([448.0, -449.0, 447.0, 1.75, 0.0], (c, Hkv, d)) * gain)
        q = synth.normal_bf16(4, c, 0, (c, H, d))
        got = run_append(x, y, q, kc, vc, ks, vs, at, c, cap, H, Hkv, d, BASE, in_place=True)
        check_append(got, x, y, kc, vc, ks, vs, at, BASE)
        kc, vc, ks, vs = got[:4]
        at += c


def test_append_non_finite_and_tiny():
    c, Hkv, d = 66, 3, 64
    _, k, v = synth.make_qkv(3, 73, c, Hkv, Hkv, d)
    k, v = k.copy(), v.copy()
    v[5, 0, 3], v[6, 1, 4], v[65, 2, 63] = 0x7F80, 0xFFC0, 0xFF80
    k[7, 1, 9] = 0x7FC0
    k[8, 0], v[8, 0] = 0x0001, 0x0080          # subnormal and smallest normal bf16
    v[:64, 2] = 0x7F80                         # nothing finite: the smallest scale
    f = lambda bits: (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    kc, vc = np.zeros((c, Hkv, d), np.uint8), np.zeros((c, Hkv, d), np.uint8)
    ks, vs = np.zeros((2, Hkv), np.uint8), np.zeros((2, Hkv), np.uint8)
    got = run_append(k, v, None, kc, vc, ks, vs, 0, c, c, Hkv, Hkv, d, 0.0)
    lowbit.append_rows(kc, ks, f(k), 0)
    lowbit.append_rows(vc, vs, f(v), 0)
    assert np.array_equal(got[2], ks) and np.array_equal(got[3], vs) and got[3][0, 2] == 27
    for g, w in ((got[0], kc), (got[1], vc)):
        nan = (w & 0x7F) == 0x7F
        assert np.array_equal((g & 0x7F) == 0x7F, nan) and np.array_equal(g[~nan], w[~nan])


# ---- attention ---------------------------------------------------------------------------------------------------------
def attn_bound(q, K, V, prefix, scale):
    out, mass, reach = lowbit.attention(q, K, V, prefix, scale)
    n, d = K.shape[0], K.shape[2]
    return out, U * (mass + np.abs(out)) * (1 + U) + mass * (2 * (d + 8) * 2.0 ** -24 * reach + (n / 64 + 80) * 2.0 ** -23) + 1e-30


def run_attn(q, caches, prefix, c, H, Hkv, d, scale, ws, stream=None):
    buf = torch.full((c + 4, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
    kvra.kvra_chunk_attn_q8(to_dev(q), *caches, prefix, c, H, Hkv, d, scale, buf[2:2 + c], ws, ws.numel(), stream)
    torch.cuda.synchronize()
    got = to_bits(buf)
    assert np.all(f64(got[:2]) == 7.0) and np.all(f64(got[2 + c:]) == 7.0), "wrote outside the output"
    return got[2:2 + c]


SHAPES = [
    (2, 2, 64, 0, 1), (2, 2, 64, 63, 1), (3, 3, 128, 0, 31), (3, 3, 128, 31, 33), (5, 1, 128, 64, 32),
    (8, 8, 64, 447, 65), (8, 8, 128, 448, 64), (8, 2, 128, 449, 63), (16, 4, 64, 511, 129), (71, 1, 64, 300, 30),
    (8, 2, 128, 1699, 300), (4, 2, 64, 2500, 179), (32, 32, 128, 5824, 77), (32, 32, 128, 8000, 1), (16, 16, 64, 4097, 3),
    (7, 1, 64, 23000, 2), (8, 1, 128, 19999, 4), (16, 1, 128, 4500, 1), (17, 1, 64, 40, 1), (33, 1, 128, 64, 1), (1, 1, 64, 0, 4200),
    (8, 8, 128, 600, 700), (4, 1, 128, 0, 1030), (71, 1, 64, 1000, 130), (2, 2, 64, 33000, 1), (3, 1, 128, 70000, 1),
]


@pytest.mark.parametrize("H,Hkv,d,prefix,c", SHAPES)
def test_attention(H, Hkv, d, prefix, c):
    """Rows of the cache behind the valid ones hold NaN; a second launch gives the same bits; the counters are zero again."""
    n = prefix + c
    q = synth.normal_bf16(7, 61, 0, (c, H, d))
    kc, ks = random_cache(3, n, n + 70, Hkv, d)
    vc, vs = random_cache(4, n, n + 70, Hkv, d, spread=4)
    scale, ws = synth.default_scale(d), workspace()
    caches = [bytes_dev(t) for t in (kc, vc, ks, vs)]
    got = run_attn(q, caches, prefix, c, H, Hkv, d, scale, ws)
    assert np.array_equal(got, run_attn(q, caches, prefix, c, H, Hkv, d, scale, ws))
    assert bool((ws[:16384] == 0).all())
    want, bound = attn_bound(f64(q), lowbit.cache_values(kc, ks)[:n], lowbit.cache_values(vc, vs)[:n], prefix, scale)
    err = np.abs(f64(got) - want)
    assert np.all(err <= bound), (float((err / bound).max()), np.argwhere(err > bound)[:3])


# launches of the kernel with 256 rows a workgroup: whole and cut units, gangs, one and several rounds, row tiles that are not full,
# more than 64 tile steps, tiles past the end, groups of heads
# (over the cache: 16 and 32 heads of their own and (8, 8, 128, 20000, 700), but for (32, 32, 128, 0, 4200); the others unpack it)
TILED = [
    (16, 16, 128, 20000, 600), (32, 32, 64, 9000, 900),
    (32, 32, 128, 100, 1100), (32, 8, 128, 1000, 1090), (32, 32, 128, 3000, 777), (32, 1, 128, 700, 1301), (16, 16, 128, 12000, 500), (8, 8, 128, 20000, 700),
    (32, 32, 128, 0, 4200), (71, 1, 64, 4096, 600), (71, 1, 64, 100, 1500), (8, 8, 64, 20000, 1500), (8, 8, 64, 0, 6000), (16, 8, 64, 3000, 3000),
]


@pytest.mark.parametrize("H,Hkv,d,prefix,c", TILED)
def test_attention_of_many_rows_is_the_bf16_kernels(H, Hkv, d, prefix, c):
    """Bit for bit what kvra_chunk_attn gives on the values that the cache stands for; and near the oracle on some rows."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    assert kvra.kvra_chunk_attn_q8_row_splits(prefix, c, H, Hkv, d, cus) == 0 == kvra.kvra_chunk_attn_row_splits(prefix, c, H, Hkv, d, cus), "not the kernel this shape is here for"
    n = prefix + c
    rng = np.random.default_rng(17)
    q = to_dev(synth.normal_bf16(7, 64, 0, (c, H, d)))
    codes = rng.integers(0, 256, (2, n, Hkv, d), dtype=np.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x33
    codes &= 0xBF                                     # (magnitudes up to 3.75, many subnormal)
    scales = rng.integers(124, 130, (2, (n + 63) // 64, Hkv)).astype(np.uint8)
    scales[0] = 126
    values = [lowbit.cache_values(codes[i], scales[i]) for i in range(2)]
    caches = [bytes_dev(t) for t in (codes[0], codes[1], scales[0], scales[1])]
    scale, ws = synth.default_scale(d), workspace()
    outs = []
    for _ in range(2):
        out = torch.full((c + 2, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
        kvra.kvra_chunk_attn_q8(q, *caches, prefix, c, H, Hkv, d, scale, out[1:-1], ws, ws.numel())
        outs.append(out)
    wide = torch.empty_like(out)
    wide[0], wide[-1] = 7.0, 7.0
    kvra.kvra_chunk_attn(q, to_dev(orc.f64_to_bf16_bits(values[0])), to_dev(orc.f64_to_bf16_bits(values[1])), prefix, c, H, Hkv, d, scale, wide[1:-1])
    torch.cuda.synchronize()
    assert bool((ws[:16384] == 0).all())
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))
    assert torch.equal(outs[0].view(torch.int16), wide.view(torch.int16))
    got = f64(to_bits(outs[0]))[1:-1]
    rows = sorted({0, 1, c // 2, c - 1})
    full = np.zeros((n, H, d))
    full[prefix:] = f64(to_bits(q))
    want = orc.attention_rows(full, values[0], values[1], [prefix + r for r in rows], scale)
    assert np.abs(got[rows] - want).max() <= 2e-2 * max(1.0, np.abs(want).max())


@pytest.mark.parametrize("d,H,Hkv,prefix,c", [(64, 4, 2, 100, 90), (128, 4, 2, 700, 33), (128, 2, 2, 0, 600), (64, 9, 1, 30, 300)])
@pytest.mark.parametrize("kind", ["sharp", "far below", "far above", "uneven blocks", "flat"])
def test_attention_score_ranges(d, H, Hkv, prefix, c, kind):
    """Scores with a standard deviation of 16, all around -+1e6, keys whose blocks differ by 2^16, and all equal."""
    n = prefix + c
    q = synth.normal_bf16(8, 62, 0, (c, H, d), std=16.0 if kind == "sharp" else 1.0)
    kc, ks = random_cache(5, n, n, Hkv, d, std=0.0 if kind == "flat" else 1.0, spread=8 if kind == "uneven blocks" else 0)
    vc, vs = random_cache(6, n, n, Hkv, d)
    if kind.startswith("far"):
        q = q.copy()
        q[..., 0] = synth.f32_to_bf16_bits(np.float32(3e6 if kind == "far above" else -3e6))
        ks = np.full_like(ks, ks.max())
        kc[..., 0] = lowbit.nearest(np.array(256.0), lowbit.E4M3)      # the same component in every key
    scale = synth.default_scale(d)
    got = run_attn(q, [bytes_dev(t) for t in (kc, vc, ks, vs)], prefix, c, H, Hkv, d, scale, workspace())
    want, bound = attn_bound(f64(q), lowbit.cache_values(kc, ks), lowbit.cache_values(vc, vs), prefix, scale)
    err = np.abs(f64(got) - want)
    assert np.isfinite(f64(got)).all() and np.all(err <= bound), float((err / bound).max())


@pytest.mark.parametrize("H,Hkv,d,prefix,c", [(4, 2, 64, 100, 200), (4, 2, 128, 40, 300), (2, 2, 128, 1000, 70), (71, 1, 64, 64, 66), (4, 2, 128, 200, 1),
                                              (8, 8, 128, 0, 1500), (16, 1, 64, 0, 900), (32, 32, 128, 100, 1100), (71, 1, 64, 4096, 600), (32, 32, 128, 3000, 777), (32, 32, 64, 9000, 900)])
def test_attention_nan_reaches_those_that_see_it(H, Hkv, d, prefix, c):
    """NaN in K and in V, in rows of the chunk and of the prefix.  Heads that do not read it keep their bits.  A wave that meets a NaN
    may take its rows' exponents relative to another reference: the rows before it then round otherwise, each result within its bound of
    the same exact value, so that two of them are at most twice the bound apart."""
    n, G = prefix + c, H // Hkv
    q = synth.normal_bf16(9, 63, 0, (c, H, d))
    kc, ks = random_cache(7, n, n, Hkv, d)
    vc, vs = random_cache(8, n, n, Hkv, d)
    call = lambda k, v: run_attn(q, [bytes_dev(t) for t in (k, v, ks, vs)], prefix, c, H, Hkv, d, 0.125, workspace())
    clean = call(kc, vc)
    apart = 2 * attn_bound(f64(q), lowbit.cache_values(kc, ks), lowbit.cache_values(vc, vs), prefix, 0.125)[1]
    for row in sorted({prefix // 2, prefix, prefix + c // 3, prefix + c // 2 + 1, n - 1} - {n}):
        head, col = row % Hkv, row % d
        r = max(row - prefix, 0)
        for which in range(2):
            k, v = kc.copy(), vc.copy()
            (k, v)[which][row, head, col] = (0x7F, 0xFF)[which]
            got = call(k, v)
            mine = slice(head * G, head * G + G)
            others = np.delete(np.arange(H), np.arange(H)[mine])
            assert np.array_equal(got[:, others], clean[:, others])
            assert np.all(np.abs(f64(got[:r]) - f64(clean[:r])) <= apart[:r])
            seen = f64(got[r:, mine])
            assert np.isnan(seen).all() if which == 0 else np.isnan(seen[..., col]).all()


@pytest.mark.parametrize("H,Hkv,d,prefix,c", [(32, 8, 128, 15296, 1088), (8, 8, 64, 40000, 900)])
def test_attention_with_a_larger_workspace(H, Hkv, d, prefix, c):
    """Room to unpack a longer cache: another kernel, the same bits."""
    n = prefix + c
    q = to_dev(synth.normal_bf16(9, 64, 0, (c, H, d)))
    caches = [bytes_dev(t) for pair in (random_cache(7, n, n, Hkv, d), random_cache(8, n, n, Hkv, d)) for t in pair]
    caches = [caches[0], caches[2], caches[1], caches[3]]
    size, outs = kvra.kvra_chunk_attn_q8_workspace_bytes(), []
    assert kvra.kvra_chunk_attn_q8_row_splits(prefix, c, H, Hkv, d, torch.cuda.get_device_properties(0).multi_processor_count) == 0
    for more in (0, 1 << 28):
        ws = torch.zeros(size + more + 4096, dtype=torch.uint8, device="cuda")
        ws[size + more:] = 0xA5
        outs.append(torch.full_like(q, 7.0))
        kvra.kvra_chunk_attn_q8(q, *caches, prefix, c, H, Hkv, d, 0.09, outs[-1], ws, size + more)
        assert bool((ws[size + more:] == 0xA5).all()) and not bool(ws[:16384].any())
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))


@pytest.mark.parametrize("c,tiled", [(1, False), (70, False), (700, True)])
def test_a_cache_beyond_4_gib(c, tiled):
    """One key of each head, behind the first 2^32 bytes, whose score exceeds all others by 90 or more (n e^-90 < 2^-100: what is left of the
    others is below bf16's half step of the result): the result is its row of V.  The rows of the chunk come in by an append there."""
    H, d, prefix = 32, 128, 1_100_000
    n, dev = prefix + c, "cuda"
    kc, vc = (torch.zeros((n, H, d), dtype=torch.uint8, device=dev) for _ in range(2))
    ks, vs = (torch.full(((n + 63) // 64, H), 127, dtype=torch.uint8, device=dev) for _ in range(2))
    assert (prefix - 40) * H * d > 1 << 32
    assert (kvra.kvra_chunk_attn_q8_row_splits(prefix, c, H, H, d, torch.cuda.get_device_properties(0).multi_processor_count) == 0) == tiled
    k = torch.zeros((c, H, d), dtype=torch.bfloat16, device=dev)
    v = torch.full((c, H, d), -2.0, dtype=torch.bfloat16, device=dev)
    k[..., 1] = 1.0
    kvra.kvra_append_kv_q8(k, v, None, None, kc, vc, ks, vs, prefix, c, n, H, H, d, 0.0)
    torch.cuda.synchronize()
    # 1 and -2 as the appended rows' codes stand for them, scales of their blocks included
    first = prefix // 64
    factor = torch.exp2(torch.stack([ks, vs])[:, first:].double() - 127).repeat_interleave(64, dim=1)[:, prefix - 64 * first:n - 64 * first]
    assert bool((kc[prefix:, :, 1].view(torch.float8_e4m3fn).double() * factor[0] == 1.0).all())
    assert bool((vc[prefix:].view(torch.float8_e4m3fn).double() * factor[1][..., None] == -2.0).all())
    assert not bool(kc[:prefix].any()) and not bool(vc[:prefix].any())
    key = prefix - 40 - torch.arange(H, device=dev) * 13                  # its own block for many a head, all ahead of the chunk
    heads = torch.arange(H, device=dev)
    kc[key, heads, 0] = torch.full((H,), 64.0, device=dev).to(torch.float8_e4m3fn).view(torch.uint8)
    row = torch.arange(d, device=dev)[None] % 7 + heads[:, None] % 5 + 1.0     # 1 .. 11: exact in e4m3
    vc[key, heads] = row.to(torch.float8_e4m3fn).view(torch.uint8)
    ks[key // 64, heads] = 127
    vs[key // 64, heads] = 127
    q = torch.zeros((c, H, d), dtype=torch.bfloat16, device=dev)
    q[..., 0] = 16.0
    out, ws = torch.empty_like(q), workspace()
    kvra.kvra_chunk_attn_q8(q, kc, vc, ks, vs, prefix, c, H, H, d, 0.09, out, ws, ws.numel())
    assert bool((out.float() == row[None]).all())


@pytest.mark.parametrize("H,Hkv,d,prefix,c", [(71, 1, 64, 4096, 600), (32, 32, 128, 3000, 777), (8, 8, 128, 9000, 1), (8, 2, 128, 1699, 300)])
def test_attention_in_a_graph(H, Hkv, d, prefix, c):
    """Each of the ways a call can go (unpacked, tiled, slices shared by workgroups, slices), captured; replays with other queries and
    caches in the same tensors, with eager calls over the same workspace between them."""
    n, ws = prefix + c, workspace()
    q = torch.empty((c, H, d), dtype=torch.bfloat16, device="cuda")
    caches = [bytes_dev(np.zeros((n, Hkv, d), np.uint8)) for _ in range(2)] + [bytes_dev(np.zeros(((n + 63) // 64, Hkv), np.uint8)) for _ in range(2)]

    def fill(i):
        q.copy_(to_dev(synth.normal_bf16(9, 70 + i, 0, (c, H, d))))
        for j in range(2):
            codes, scales = random_cache(40 + 2 * i + j, n, n, Hkv, d)
            caches[j].copy_(bytes_dev(codes))
            caches[2 + j].copy_(bytes_dev(scales))

    def call(out, stream=None):
        kvra.kvra_chunk_attn_q8(q, *caches, prefix, c, H, Hkv, d, 0.1, out, ws, ws.numel(), stream)

    fill(0)
    out, eager = torch.empty_like(q), torch.empty_like(q)
    call(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, torch.cuda.current_stream())
    for i in range(4):
        fill(i)
        torch.cuda.synchronize()
        out.fill_(7.0)
        graph.replay()
        call(eager, torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16))
    assert not bool(ws[:16384].any())


def test_attention_on_two_streams_with_a_workspace_each():
    H, Hkv, d, prefix, c = 8, 8, 128, 9000, 1
    jobs = []
    for i in range(2):
        kc, ks = random_cache(20 + i, prefix + c, prefix + c, Hkv, d)
        vc, vs = random_cache(30 + i, prefix + c, prefix + c, Hkv, d)
        jobs.append((to_dev(synth.normal_bf16(10, i, 0, (c, H, d))), [bytes_dev(t) for t in (kc, vc, ks, vs)], workspace(), torch.cuda.Stream()))
    call = lambda q, caches, ws, out, s: kvra.kvra_chunk_attn_q8(q, *caches, prefix, c, H, Hkv, d, 0.09, out, ws, ws.numel(), s)
    alone = [torch.empty_like(j[0]) for j in jobs]
    for (q, caches, ws, s), out in zip(jobs, alone):
        call(q, caches, ws, out, None)
    torch.cuda.synchronize()
    both = [[torch.empty_like(j[0]) for _ in range(20)] for j in jobs]
    for r in range(20):
        for (q, caches, ws, s), outs in zip(jobs, both):
            call(q, caches, ws, outs[r], s)
    torch.cuda.synchronize()
    for a, outs in zip(alone, both):
        assert all(torch.equal(a.view(torch.int16), o.view(torch.int16)) for o in outs)


# ---- weights -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,k", [(32, 64), (64, 192), (704, 1088), (1024, 4096)])
def test_pack_and_unpack(n, k):
    w = synth.normal_bf16(12, n, 0, (n, k), std=0.02).copy()
    w[0, :32], w[1, :8] = 0, synth.f32_to_bf16_bits(np.array([6, 5, 0.25, 0.75, 1.25, -1.75, 2.5, -3.5], np.float32))   # all zeros; ties
    w[1, 8:32] = 0
    w[2, :32] = synth.f32_to_bf16_bits(np.float32(6.03125) * np.ones(32, np.float32))       # just past a scale's border
    w[3, :32], w[4, :32] = 0x0001, 0x7F7F                                                 # the smallest and the largest bf16
    w[5, 40], w[6, 33] = 0x7F80, 0xFFC1
    x = (w.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    codes, scales = torch.full((n, k // 2), 0x99, dtype=torch.uint8, device="cuda"), torch.zeros((n, k // 32), dtype=torch.uint8, device="cuda")
    kvra.kvra_pack_w4(to_dev(w), codes, scales, n, k)
    wc, ws = lowbit.pack(x)
    bad = np.repeat(ws == 255, 16, axis=1)
    assert np.array_equal(scales.cpu().numpy(), ws) and np.array_equal(codes.cpu().numpy()[~bad], wc[~bad])
    back = torch.zeros((n, k), dtype=torch.bfloat16, device="cuda")
    kvra.kvra_unpack_w4(codes, scales, back, n, k)
    got = (to_bits(back).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    assert np.array_equal(got, lowbit.unpack(wc, ws), equal_nan=True)


def weights(seed, n, k):
    return lowbit.pack(f64(synth.normal_bf16(13, seed, 0, (n, k), std=0.02)))


@pytest.mark.parametrize("form", ["plain", "residual", "in place", "swiglu"])
@pytest.mark.parametrize("m,n,k", [
    (1, 32, 64), (1, 96, 192), (2, 160, 128), (15, 64, 320), (16, 256, 1088), (17, 96, 64), (33, 352, 704), (64, 128, 256), (65, 64, 448),
    (100, 1056, 576), (129, 512, 1024), (257, 320, 192), (1, 4096, 4096), (5, 1024, 11008), (300, 1024, 2048), (1, 12288, 4096),
    (300, 4096, 1088), (390, 4064, 512), (1100, 4128, 576), (1090, 4096, 1024), (2050, 2080, 704),   # 256 rows a workgroup, k shared or not, half stages
])
def test_linear(form, m, n, k):
    x = synth.normal_bf16(14, m, 0, (m, k))
    w, s = weights(1, n, k)
    w2, s2 = weights(2, n, k) if form == "swiglu" else (None, None)
    r = synth.normal_bf16(14, m, 1, (m, n)) if form in ("residual", "in place") else None
    out = torch.full((m + 2, n), 7.0, dtype=torch.bfloat16, device="cuda")
    rd = None
    if r is not None:
        rd = to_dev(r)
        if form == "in place":
            out[1:-1] = rd
            rd = out[1:-1]
    d = lambda t: None if t is None else bytes_dev(t)
    kvra.kvra_linear_w4(to_dev(x), d(w), d(s), d(w2), d(s2), rd, out[1:-1], m, n, k)
    torch.cuda.synchronize()
    got = f64(to_bits(out))
    assert np.all(got[0] == 7.0) and np.all(got[-1] == 7.0)
    want, terms = lowbit.linear(f64(x), w, s, w2, s2, None if r is None else f64(r))
    bound = U * np.abs(want) * (1 + U) + (k / 32 + 48) * 2.0 ** -24 * terms + 2.0 ** -20 * np.abs(want) + 1e-30
    err = np.abs(got[1:-1] - want)
    assert np.all(err <= bound), (float((err / bound).max()), np.argwhere(err > bound)[:3])


def test_linear_of_more_tokens_than_a_grid_holds():
    # 65535 tiles of 64 tokens and 70 more: the same 65 tokens over and over give the same 65 results
    n, k, m = 32, 64, 65535 * 64 + 70
    base = synth.normal_bf16(14, 65, 2, (65, k))
    w, s = weights(3, n, k)
    x = to_dev(base).repeat(m // 65 + 1, 1)[:m].contiguous()
    r = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    r[:, 0] = (torch.arange(m, device="cuda") % 128).to(torch.bfloat16)          # (residual rows of their own: exact in bf16)
    out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    kvra.kvra_linear_w4(x, bytes_dev(w), bytes_dev(s), None, None, None, out, m, n, k)
    want, terms = lowbit.linear(f64(base), w, s, None, None, None)
    bound = U * np.abs(want) * (1 + U) + (k / 32 + 48) * 2.0 ** -24 * terms + 2.0 ** -20 * np.abs(want) + 1e-30
    assert np.all(np.abs(f64(to_bits(out[:65])) - want) <= bound)
    assert torch.equal(out, out[:65].repeat(m // 65 + 1, 1)[:m])
    with_residual = torch.empty_like(out)
    kvra.kvra_linear_w4(x, bytes_dev(w), bytes_dev(s), None, None, r, with_residual, m, n, k)
    assert torch.equal(with_residual[:, 1:], out[:, 1:])
    col = torch.from_numpy(want[:, 0]).cuda().repeat(m // 65 + 1)[:m] + r[:, 0].double()
    slack = 2.0 ** -8 * (1 + 2.0 ** -8) * col.abs() + 1e-5 * (1 + float(terms[:, 0].max()))     # half a step of bf16; fp32 sums of 65 terms
    assert bool(((with_residual[:, 0].double() - col).abs() <= slack).all())


@pytest.mark.parametrize("m,n,k", [(1, 32, 64), (3, 64, 1088), (17, 32, 320), (70, 512, 576)])
def test_linear_looks_at_nothing_behind_the_last_token(m, n, k):
    x = synth.normal_bf16(14, m, 3, (m, k))
    w, s = weights(4, n, k)
    behind = torch.full((m + 40, k), float("nan"), dtype=torch.bfloat16, device="cuda")
    behind[:m] = to_dev(x)
    a, b = torch.empty(m, n, dtype=torch.bfloat16, device="cuda"), torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    kvra.kvra_linear_w4(behind[:m], bytes_dev(w), bytes_dev(s), None, None, None, a, m, n, k)
    kvra.kvra_linear_w4(to_dev(x), bytes_dev(w), bytes_dev(s), None, None, None, b, m, n, k)
    assert not bool(torch.isnan(a).any()) and torch.equal(a, b)


def test_linear_groups_of_any_magnitude_and_nan():
    """Scales from 2^-60 to 2^60 along a row; a NaN group reaches its column of the result and no other."""
    m, n, k = 3, 64, 256
    x = synth.normal_bf16(15, 1, 0, (m, k))
    w, s = weights(3, n, k)
    s = np.random.default_rng(9).integers(127 - 60, 127 + 61, s.shape).astype(np.uint8)
    out = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    kvra.kvra_linear_w4(to_dev(x), bytes_dev(w), bytes_dev(s), None, None, None, out, m, n, k)
    want, terms = lowbit.linear(f64(x), w, s)
    assert np.all(np.abs(f64(to_bits(out)) - want) <= U * np.abs(want) * (1 + U) + (k / 32 + 48) * 2.0 ** -24 * terms)
    s[40, 3] = 255
    kvra.kvra_linear_w4(to_dev(x), bytes_dev(w), bytes_dev(s), None, None, None, out, m, n, k)
    assert np.array_equal(np.isnan(f64(to_bits(out))), np.tile(np.arange(n) == 40, (m, 1)))


# ---- together ----------------------------------------------------------------------------------------------------------
class Layer:
    """A LLaMA-style decoder layer from the low-bit calls, as a program writes it, and the same from the oracle's functions."""

    def __init__(self, hidden, ffn, H, Hkv, d, capacity):
        self.shape = hidden, ffn, H, Hkv, d
        self.capacity = capacity
        bits = synth.make_layer_weights(1, 81, hidden, ffn, H, Hkv, d, 0.05)
        self.gains = [bits["norm1"], bits["norm2"]]
        self.w, self.dev = {}, {}
        for name in ("wqkv", "wo", "w_gate", "w_up", "w_down"):
            n, k = bits[name].shape
            codes, scales = torch.empty((n, k // 2), dtype=torch.uint8, device="cuda"), torch.empty((n, k // 32), dtype=torch.uint8, device="cuda")
            kvra.kvra_pack_w4(to_dev(bits[name]), codes, scales, n, k)
            self.dev[name] = codes, scales
            self.w[name] = lowbit.pack(f64(bits[name]))
            assert np.array_equal(codes.cpu().numpy(), self.w[name][0]) and np.array_equal(scales.cpu().numpy(), self.w[name][1])
        self.norms = [to_dev(g) for g in self.gains]
        z = lambda: torch.full((capacity, Hkv, d), 0x7F, dtype=torch.uint8, device="cuda")
        zs = lambda: torch.full(((capacity + 63) // 64, Hkv), 0xFF, dtype=torch.uint8, device="cuda")
        self.cache = z(), z(), zs(), zs()
        self.ws = workspace()

    def buffers(self, c):
        hidden, ffn, H, Hkv, d = self.shape
        b = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
        return dict(h=b(c, hidden), qkv=b(c, (H + 2 * Hkv) * d), q=b(c, H, d), k=b(c, Hkv, d), v=b(c, Hkv, d), qr=b(c, H, d), a=b(c, H, d),
                    x2=b(c, hidden), act=b(c, ffn), y=b(c, hidden))

    def step(self, x, prefix, c, b, stream=None):
        hidden, ffn, H, Hkv, d = self.shape
        kvra.kvra_rms_norm(x, self.norms[0], b["h"], c, hidden, 1e-6, stream)
        rows = [H * d, Hkv * d, Hkv * d]
        at = 0
        for name, n in zip(("q", "k", "v"), rows):             # three rows' ranges of one packed weight
            w, s = (t[at:at + n] for t in self.dev["wqkv"])
            kvra.kvra_linear_w4(b["h"], w, s, None, None, None, b[name], c, n, hidden, stream)
            at += n
        kvra.kvra_append_kv_q8(b["k"], b["v"], b["q"], b["qr"], *self.cache, prefix, c, self.capacity, H, Hkv, d, BASE, stream)
        kvra.kvra_chunk_attn_q8(b["qr"], *self.cache, prefix, c, H, Hkv, d, synth.default_scale(d), b["a"], self.ws, self.ws.numel(), stream)
        kvra.kvra_linear_w4(b["a"], *self.dev["wo"], None, None, x, b["x2"], c, hidden, H * d, stream)
        kvra.kvra_rms_norm(b["x2"], self.norms[1], b["h"], c, hidden, 1e-6, stream)
        kvra.kvra_linear_w4(b["h"], *self.dev["w_gate"], *self.dev["w_up"], None, b["act"], c, ffn, hidden, stream)
        kvra.kvra_linear_w4(b["act"], *self.dev["w_down"], None, None, b["x2"], b["y"], c, hidden, ffn, stream)
        return b["y"]

    def check(self, x, b, prefix, c):
        """Every stage against the oracle on the GPU's own input of that stage, within that stage's bound."""
        hidden, ffn, H, Hkv, d = self.shape
        g = {name: f64(to_bits(t)) for name, t in b.items() if name not in ("qkv",)}
        x = f64(to_bits(x))
        def lin(name, src, res=None, second=None):
            return lowbit.linear(src, *self.w[name], *(self.w[second] if second else ()), **({} if res is None else {"residual": res}))
        def within(got, want, terms, k):
            bound = U * np.abs(want) * (1 + U) + (k / 32 + 48) * 2.0 ** -24 * terms + 2.0 ** -20 * np.abs(want) + 1e-30
            assert np.all(np.abs(got - want) <= bound), float((np.abs(got - want) / bound).max())
        # (h holds the second norm's result)
        h1 = orc.rms_norm(x, f64(self.gains[0]), 1e-6)
        qkv = np.concatenate([g[name].reshape(c, -1) for name in ("q", "k", "v")], axis=1)
        want, terms = lin("wqkv", h1)
        assert np.all(np.abs(qkv - want) <= 2 * U * terms)               # (the norm's result was rounded on the way)
        codes = [t.cpu().numpy() for t in self.cache]
        n = prefix + c
        attn, bound = attn_bound(g["qr"], lowbit.cache_values(codes[0], codes[2])[:n], lowbit.cache_values(codes[1], codes[3])[:n], prefix, synth.default_scale(d))
        assert np.all(np.abs(g["a"] - attn) <= bound)
        within(g["x2"], *lin("wo", g["a"].reshape(c, -1), x), H * d)
        assert np.all(np.abs(g["h"] - orc.rms_norm(g["x2"], f64(self.gains[1]), 1e-6)) <= U * np.abs(g["h"]) * 1.01 + 1e-4)
        within(g["act"], *lin("w_gate", g["h"], second="w_up"), hidden)
        within(g["y"], *lin("w_down", g["act"], g["x2"]), ffn)


@pytest.mark.parametrize("hidden,ffn,H,Hkv,d", [(256, 704, 4, 2, 64), (512, 1344, 4, 4, 128)])
def test_a_prompt_and_the_tokens_behind_it(hidden, ffn, H, Hkv, d):
    layer = Layer(hidden, ffn, H, Hkv, d, 400)
    want = [np.full((400, Hkv, d), 0x7F, np.uint8), np.full((400, Hkv, d), 0x7F, np.uint8), np.full((7, Hkv), 0xFF, np.uint8), np.full((7, Hkv), 0xFF, np.uint8)]
    at = 0
    for i, c in enumerate((187, 113, 1, 1, 20, 1)):
        x = to_dev(synth.normal_bf16(16, i, 0, (c, hidden)))
        b = layer.buffers(c)
        layer.step(x, at, c, b)
        torch.cuda.synchronize()
        layer.check(x, b, at, c)
        lowbit.append_rows(want[0], want[2], lowbit.rotate(f64(to_bits(b["k"])), at, BASE), at)
        lowbit.append_rows(want[1], want[3], f64(to_bits(b["v"])), at)
        at += c
    for got, w in zip(layer.cache, want):
        assert np.array_equal(got.cpu().numpy(), w)


def test_a_captured_step():
    """A token's step in a graph, replayed on changing inputs with eager work in between: the same bits as eager calls."""
    hidden, ffn, H, Hkv, d = 256, 704, 4, 2, 64
    prefix, layer = 700, Layer(256, 704, 4, 2, 64, 800)
    x0, b0 = to_dev(synth.normal_bf16(17, 0, 0, (prefix, hidden))), layer.buffers(prefix)
    layer.step(x0, 0, prefix, b0)
    x, b, e = torch.empty((1, hidden), dtype=torch.bfloat16, device="cuda"), layer.buffers(1), layer.buffers(1)
    saved = [t.clone() for t in layer.cache]
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        layer.step(x, prefix, 1, b, torch.cuda.current_stream())
    for i in range(5):
        x.copy_(to_dev(synth.normal_bf16(18, i, 0, (1, hidden), std=1.0 + i)))
        for t, s in zip(layer.cache, saved):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        after = [t.clone() for t in layer.cache]
        for t, s in zip(layer.cache, saved):
            t.copy_(s)
        layer.step(x, prefix, 1, e)
        torch.cuda.synchronize()
        assert torch.equal(b["y"].view(torch.int16), e["y"].view(torch.int16))
        assert all(torch.equal(s, t) for s, t in zip(after, layer.cache))
