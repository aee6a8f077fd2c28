"""The 4-bit linear layer where its kernels differ from one another, and at the edges of what the call allows.  KERNELS says which kernel a
shape is here for; tests/test_lowbit_launches.py asserts that it gets it."""
import numpy as np
import pytest
import torch

from oracle import lowbit
from paper_2405_05329_amd import kvra, synth
from gpu_pipeline import to_dev
from test_gpu_lowbit import bytes_dev, f64, weights

pytestmark = pytest.mark.gpu

# (m, n, k): its kernel, plain and SwiGLU.  k = 64 mod 128 and not; the tile kernel with and without k shared by two groups of waves
KERNELS = {
    (1, 96, 192): ("rows<1, 1, 1>", "rows<2, 1, 1>"), (3, 64, 1024): ("rows<1, 1, 1>", "rows<2, 1, 1>"),
    (13, 64, 1088): ("rows<1, 1, 4>", "rows<2, 1, 4>"), (16, 128, 512): ("rows<1, 1, 4>", "rows<2, 1, 4>"),
    (29, 64, 320): ("rows<2, 2, 8>", "rows<2, 2, 8>"), (32, 96, 256): ("rows<2, 2, 8>", "rows<2, 2, 8>"),
    (50, 64, 576): ("rows<2, 4, 16>", "rows<2, 4, 16>"), (70, 512, 640): ("rows<2, 4, 16>", "rows<2, 4, 16>"),
    (300, 4096, 1088): ("tile<2>", "tile<2>"), (390, 4064, 512): ("tile<2>", "tile<2>"),
    (1100, 4128, 576): ("tile<1>", "tile<1>"), (1090, 4096, 1024): ("tile<1>", "tile<1>"),
}


def run(x, ws, ss, m, n, k):
    out = torch.full((m + 2, n), 7.0, dtype=torch.bfloat16, device="cuda")
    kvra.kvra_linear_w4(x, ws[0], ss[0], *((ws[1], ss[1]) if len(ws) > 1 else (None, None)), None, out[1:-1], m, n, k)
    torch.cuda.synchronize()
    assert bool((out[0] == 7.0).all()) and bool((out[-1] == 7.0).all())
    return out[1:-1]


@pytest.mark.parametrize("swiglu", [False, True])
@pytest.mark.parametrize("m,n,k", KERNELS)
def test_scales_at_any_two_byte_address(m, n, k, swiglu):
    """The same bits whether the scale tensors lie at 0 or at 2 modulo 4 bytes, one of them or both."""
    x = to_dev(synth.normal_bf16(14, m, 5, (m, k)))
    pairs = [weights(6 + i, n, k) for i in range(1 + swiglu)]
    ws = [bytes_dev(w) for w, _ in pairs]
    rng = np.random.default_rng(31)
    scales = [rng.integers(110, 120, s.shape).astype(np.uint8) for _, s in pairs]      # (neighbours differ)

    def placed(s, at):
        room = torch.full((s.size + 64,), 0xFF, dtype=torch.uint8, device="cuda")
        room[at:at + s.size] = bytes_dev(s).flatten()
        view = room[at:at + s.size]
        assert view.data_ptr() % 16 == at
        return view

    want = run(x, ws, [placed(s, 0) for s in scales], m, n, k)
    assert not bool(torch.isnan(want).any())
    for ats in ((2, 2), (2, 0), (0, 6), (14, 8)):
        got = run(x, ws, [placed(s, at) for s, at in zip(scales, ats)], m, n, k)
        assert torch.equal(got.view(torch.int16), want.view(torch.int16)), ats
    exact = lowbit.linear(_f64(x[:2]), *_interleaved(pairs, scales))
    bound = 2.0 ** -8 * np.abs(exact[0]) * (1 + 2.0 ** -8) + (k / 32 + 48) * 2.0 ** -24 * exact[1] + 2.0 ** -20 * np.abs(exact[0]) + 1e-30
    assert np.all(np.abs(_f64(want[:2]) - exact[0]) <= bound)


def _f64(t):
    return t.double().cpu().numpy()


def _interleaved(pairs, scales):
    return [t for (w, _), s in zip(pairs, scales) for t in (w, s)]


def clean(m, n, k, swiglu, seed=6):
    """Tokens, codes and scales (host), and the result on them."""
    x = to_dev(synth.normal_bf16(14, m, 5, (m, k)))
    pairs = [weights(seed + i, n, k) for i in range(1 + swiglu)]
    ws, ss = [bytes_dev(w) for w, _ in pairs], [s.copy() for _, s in pairs]
    want = run(x, ws, [bytes_dev(s) for s in ss], m, n, k)
    assert not bool(torch.isnan(want).any())
    return x, pairs, ws, ss, want


@pytest.mark.parametrize("swiglu", [False, True])
@pytest.mark.parametrize("m,n,k", KERNELS)
def test_a_token_of_nan_stays_its_own(m, n, k, swiglu):
    """Tokens of NaN among the others and behind the last: the others keep their bits (a row that ends inside a stage is followed by
    the next token)."""
    x, _, ws, ss, want = clean(m, n, k, swiglu)
    scales = [bytes_dev(s) for s in ss]
    behind = torch.full((m + 70, k), float("nan"), dtype=torch.bfloat16, device="cuda")
    behind[:m] = x
    assert torch.equal(run(behind[:m], ws, scales, m, n, k), want)
    bad = torch.arange(m, device="cuda") % 5 == 4
    behind[:m][bad] = float("nan")
    got = run(behind[:m], ws, scales, m, n, k)
    assert bool(torch.isnan(got[bad]).all()) and torch.equal(got[~bad], want[~bad])


@pytest.mark.parametrize("swiglu", [False, True])
@pytest.mark.parametrize("m,n,k", KERNELS)
def test_a_group_of_nan_stays_in_its_column(m, n, k, swiglu):
    """In a row's last group, with the next row's data behind it, and in a next row's first group, with a row's end ahead of it."""
    x, _, ws, ss, want = clean(m, n, k, swiglu)
    columns = {0: -1, 2: 0, 5: -1, 17: k // 64, n // 2: -1, n // 2 + 3: 0, n - 1: -1, n - 3: 0}
    hit = torch.zeros(n, dtype=torch.bool, device="cuda")
    for i, (row, group) in enumerate(columns.items()):
        ss[i % len(ss)][row, group] = 255
        hit[row] = True
    got = run(x, ws, [bytes_dev(s) for s in ss], m, n, k)
    assert bool(torch.isnan(got[:, hit]).all()) and torch.equal(got[:, ~hit], want[:, ~hit])


@pytest.mark.parametrize("m,n,k", KERNELS)
def test_groups_of_any_magnitude(m, n, k):
    """Scales from 2^-60 to 2^60 along every row: a scale used one group, one stage or one row off would show."""
    x = synth.normal_bf16(14, m, 5, (m, k))
    w, _ = weights(6, n, k)
    s = np.random.default_rng(32).integers(127 - 60, 127 + 61, (n, k // 32)).astype(np.uint8)
    rows = [r for r in sorted({0, 1, 15, 16, 63, 64, 127, 128, 1023, 1024, m // 2, m - 1}) if r < m]
    got = _f64(run(to_dev(x), [bytes_dev(w)], [bytes_dev(s)], m, n, k))[rows]
    want, terms = lowbit.linear(f64(x[rows]), w, s)
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8) + (k / 32 + 48) * 2.0 ** -24 * terms)
