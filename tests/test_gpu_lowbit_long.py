"""Attention over long 8-bit caches whose every block and head has scales of its own: a kernel loads the scales of 64 key tiles at a
time, and one that went on with those of the tiles before, or took another block's or head's, would be far off."""
import pytest
import torch

from paper_2405_05329_amd import kvra, synth
from gpu_pipeline import to_dev
from test_gpu_lowbit import U, workspace

pytestmark = pytest.mark.gpu

# (H, Hkv, d, prefix, c): more than 64 tiles to a wave of the kernel for few rows, slices of 16 and of 32 rows, shared by workgroups or not
SLICES = [(256, 256, 64, 40000, 1), (64, 64, 128, 140000, 1), (1024, 64, 64, 150000, 2), (128, 128, 64, 70000, 3)]
# more than 64 tile steps to a piece of the tiled kernel, and whether the cache is unpacked first
TILES = {(16, 16, 128, 20000, 600): False, (64, 64, 64, 16324, 262): False, (32, 1, 128, 20000, 1301): True, (71, 1, 64, 20000, 600): True}


def random_bytes(g, shape):
    """Codes of every magnitude up to 1.875 (bit 6 is cleared, which leaves no NaN), on the GPU."""
    return torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8) & 0xBF


def long_scales(g, tiles, Hkv, splits):
    """Scales of K and of V, larger from a wave's 64th tile on than ahead of it, so that those tiles decide the result; and for every tile
    the one whose scales a kernel would use that did not load them again."""
    t = torch.arange(tiles, device=g.device)
    first = torch.zeros_like(t)                         # of the workgroup's share; a wave has every eighth from there
    for s in range(splits):
        first[tiles * s // splits:] = tiles * s // splits
    late = (t - first >= 512)[:, None]
    some = lambda lo, hi: torch.randint(lo, hi, (tiles, Hkv), generator=g, device=g.device, dtype=torch.uint8)
    return torch.where(late, some(126, 129), some(124, 127)), torch.where(late, some(128, 132), some(123, 127)), torch.where(late[:, 0], t - 512, t)


def exact(q, kc, vc, ks, vs, prefix, scale, head, G):
    """(result, bound) of one kv head's query rows in 64 bits on the GPU (elementwise products and sums); scales as given."""
    n, d = kc.shape[0], kc.shape[2]
    factor = lambda s: torch.exp2(s[:, head].double() - 127).repeat_interleave(64)[:n, None]
    value = lambda t: t[:, head].contiguous().view(torch.float8_e4m3fn).double()
    K, V = value(kc) * factor(ks), value(vc) * factor(vs)
    out, bound = [], []
    for r in range(q.shape[0]):
        seen = prefix + r + 1
        for h in range(head * G, head * G + G):
            x = q[r, h].double()
            s = scale * (K[:seen] * x).sum(1)
            reach = scale * (K[:seen].abs() * x.abs()).sum(1).max()
            w = torch.exp(s - s.max())
            w = (w / w.sum())[:, None]
            o, mass = (w * V[:seen]).sum(0), (w * V[:seen].abs()).sum(0)
            out.append(o)
            bound.append(U * (mass + o.abs()) * (1 + U) + mass * (2 * (d + 8) * 2.0 ** -24 * reach + (n / 64 + 80) * 2.0 ** -23) + 1e-30)
    return torch.stack(out), torch.stack(bound)


@pytest.mark.parametrize("H,Hkv,d,prefix,c", SLICES)
def test_slices_take_each_tiles_own_scales(H, Hkv, d, prefix, c):
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    splits = kvra.kvra_chunk_attn_q8_row_splits(prefix, c, H, Hkv, d, cus)
    n, G = prefix + c, H // Hkv
    tiles = (n + 63) // 64
    assert splits > 0 and tiles > 64 * 8 * splits, "not a shape for this test"
    g = torch.Generator(device="cuda")
    g.manual_seed(41)
    kc, vc = random_bytes(g, (n, Hkv, d)), random_bytes(g, (n, Hkv, d)) & 0x7F      # (V of one sign, so that sums do not cancel)
    ks, vs, stale = long_scales(g, tiles, Hkv, splits)
    q = to_dev(synth.normal_bf16(41, 1, 0, (c, H, d)))
    out, ws, scale = torch.full_like(q, 7.0), workspace(), synth.default_scale(d)
    kvra.kvra_chunk_attn_q8(q, kc, vc, ks, vs, prefix, c, H, Hkv, d, scale, out, ws, ws.numel())
    torch.cuda.synchronize()
    for head in sorted({0, Hkv // 3, Hkv - 1}):
        got = out[:, head * G:head * G + G].reshape(c * G, d).double()
        want, bound = exact(q, kc, vc, ks, vs, prefix, scale, head, G)
        assert bool(((got - want).abs() <= bound).all()), (head, float(((got - want).abs() / bound).max()))
        # the oracle with the mistake: from a wave's 64th tile on, the scales of the tile 64 of its own earlier
        for wrong in (exact(q, kc, vc, ks[stale], vs, prefix, scale, head, G)[0], exact(q, kc, vc, ks, vs[stale], prefix, scale, head, G)[0]):
            assert bool(((wrong - want).abs() > 8 * bound).any(1).all()), "the test would not see the mistake"


@pytest.mark.parametrize("H,Hkv,d,prefix,c", TILES)
def test_tiles_take_each_tiles_own_scales(H, Hkv, d, prefix, c):
    """Bit for bit what kvra_chunk_attn gives on the values that the cache stands for, K's scales as different as V's."""
    n = prefix + c
    g = torch.Generator(device="cuda")
    g.manual_seed(43)
    codes = [random_bytes(g, (n, Hkv, d)) for _ in range(2)]
    scales = [torch.randint(lo, hi, ((n + 63) // 64, Hkv), generator=g, device="cuda", dtype=torch.uint8) for lo, hi in ((124, 128), (123, 132))]
    values = []
    for code, s in zip(codes, scales):
        v = code.view(torch.float8_e4m3fn).float() * torch.exp2(s.float() - 127).repeat_interleave(64, dim=0)[:n, :, None]
        values.append(v.to(torch.bfloat16))
        assert torch.equal(values[-1].float(), v)                # (exact)
    q = to_dev(synth.normal_bf16(43, 1, 0, (c, H, d)))
    out, want, ws, scale = torch.full_like(q, 7.0), torch.full_like(q, 5.0), workspace(), synth.default_scale(d)
    kvra.kvra_chunk_attn_q8(q, *codes, *scales, prefix, c, H, Hkv, d, scale, out, ws, ws.numel())
    kvra.kvra_chunk_attn(q, *values, prefix, c, H, Hkv, d, scale, want)
    torch.cuda.synchronize()
    assert not bool(torch.isnan(out).any()) and torch.equal(out.view(torch.int16), want.view(torch.int16))
