"""The 64-bit statement of the paged cache against closed forms, other statements of the same, and finite differences."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO


def test_codes_are_those_of_the_format():
    x = PO.decode_e4m3(np.arange(256))
    assert x[0] == 0 and x[1] == 2.0 ** -9 and x[8] == 2.0 ** -6 and x[126] == 448 and x[0x38] == 1.0 and x[0xb8] == -1.0
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(x, t, equal_nan=True)


def test_encoding_is_to_nearest_even():
    finite = [c for c in range(127)]
    values = [Fraction(float(v)) for v in PO.decode_e4m3(np.array(finite))]
    tries = []
    for a, b in zip(values, values[1:]):
        mid = (a + b) / 2
        tries += [a, mid, mid - Fraction(1, 1 << 40), mid + Fraction(1, 1 << 40)]
    for x in tries + [values[-1]]:
        best = min(range(127), key=lambda c: (abs(values[c] - x), c % 2))
        assert PO.encode_e4m3(float(x)) == best
        assert PO.encode_e4m3(-float(x)) == best + 128
    assert PO.encode_e4m3(np.nan) & 127 == 127 and PO.encode_e4m3(np.inf) & 127 == 127


@pytest.mark.parametrize("most,scale", [(448.0, 1.0), (448.1, 2.0), (224.0, 0.5), (1.75, 2.0 ** -8), (1.76, 2.0 ** -7),
                                        (0.0, 2.0 ** -100), (2.0 ** -120, 2.0 ** -100)])
def test_scales(most, scale):
    assert PO.scale_for(most) == scale


@pytest.mark.parametrize("pairs", (0, 1))
def test_a_rotation_is_a_product_of_complex_numbers(pairs):
    r = np.random.RandomState(0)
    x, pos = r.standard_normal((5, 2, 48)).astype(np.float32), r.randint(-50, 50, (3, 5))
    freq, axis = r.uniform(0.01, 1, 16), r.randint(0, 3, 16)
    y = PO.turn(x, pos, freq, axis, pairs)
    for t in range(5):
        for i in range(16):
            a, b = (i, i + 16) if pairs == 0 else (2 * i, 2 * i + 1)
            z = (x[t, :, a] + 1j * x[t, :, b].astype(np.float64)) * np.exp(1j * pos[axis[i], t] * freq[i])
            assert np.allclose(y[t, :, a] + 1j * y[t, :, b], z, atol=1e-6)
    assert np.array_equal(y[..., 32:], x[..., 32:])
    back = PO.turn(y, pos, freq, axis, pairs, backward=True)
    assert np.allclose(back, x, atol=1e-6)


@pytest.mark.parametrize("pairs", (0, 1))
def test_the_gradient_of_a_rotation_against_differences(pairs):
    """L = sum w * turn(x): the gradient is turn(w) backward; central differences of the linear map are exact but for rounding."""
    r = np.random.RandomState(1)
    x, w = r.standard_normal((3, 1, 32)).astype(np.float32), r.standard_normal((3, 1, 32)).astype(np.float32)
    pos, freq, axis = r.randint(0, 9, (2, 3)), r.uniform(0.1, 1, 16), np.arange(16) % 2
    g = PO.turn(w, pos, freq, axis, pairs, backward=True)
    for t in range(3):
        for c in range(32):
            e = np.zeros_like(x)
            e[t, 0, c] = 1.0
            diff = (w.astype(np.float64) * (PO.turn(x + e, pos, freq, axis, pairs).astype(np.float64)
                                            - PO.turn(x - e, pos, freq, axis, pairs))).sum() / 2
            assert abs(diff - g[t, 0, c]) < 1e-5


def test_appending_piece_by_piece_stays_within_the_last_step():
    """Whatever the pieces: no element is off by more than half a step of its code plus half the last subnormal step for
    every growth (the steps double at least, so their halves add up to less than one)."""
    r = np.random.RandomState(2)
    page, d = 32, 32
    x = (r.standard_normal((page, 1, d)) * np.exp2(r.uniform(-3, 3, (page, 1, 1)))).astype(np.float32)
    table = [[0]]
    for pieces in ([32], [1] * 32, [5, 20, 7]):
        codes, scale = np.zeros((1, 1, page, d), np.uint8), np.ones((1, 1))
        at = 0
        for n in pieces:
            PO.append(codes, scale, x[at:at + n], table, [at + n], [0, n])
            at += n
        got = PO.decode_e4m3(codes[0, 0]) * scale[0, 0]
        step = np.maximum(2.0 ** -9 * scale[0, 0], np.exp2(np.floor(np.log2(np.abs(x[:, 0])))) / 8)
        assert (np.abs(got - x[:, 0]) <= step).all()
        assert scale[0, 0] == PO.scale_for(np.abs(x).max())


def test_attention_is_the_library_s_on_the_decoded_cache():
    r = np.random.RandomState(3)
    page, d, n, m = 16, 32, 37, 5
    kc, vc = (r.randint(0, 127, (4, 2, page, d)).astype(np.uint8) for _ in range(2))
    ks, vs = (np.exp2(r.randint(-10, -6, (4, 2))).astype(np.float64) for _ in range(2))
    table, q = [[2, 0, 3]], r.standard_normal((m, 6, d))
    out, lse, _, _, _ = PO.attend(q, kc, vc, ks, vs, table, [n], [0, m])
    k = (PO.decode_e4m3(kc) * ks[..., None, None])[[2, 0, 3]].transpose(1, 0, 2, 3).reshape(2, -1, d)[:, :n]
    v = (PO.decode_e4m3(vc) * vs[..., None, None])[[2, 0, 3]].transpose(1, 0, 2, 3).reshape(2, -1, d)[:, :n]
    mask = torch.ones(m, n, dtype=torch.bool).tril(n - m)
    want = torch.nn.functional.scaled_dot_product_attention(
        torch.from_numpy(q).permute(1, 0, 2), torch.from_numpy(k).repeat_interleave(3, 0),
        torch.from_numpy(v).repeat_interleave(3, 0), attn_mask=mask)
    assert np.allclose(out, want.permute(1, 0, 2).numpy(), rtol=1e-12, atol=1e-12)
    s = q[0, 4] @ k[1, :n - m + 1].T / math.sqrt(d)
    assert abs(lse[0, 4] - np.log(np.exp(s).sum())) < 1e-12
    # pages that are not there, and rows before the first token
    out, lse, _, _, _ = PO.attend(q, kc, vc, ks, vs, [[2, -1, 9]], [3], [0, m])
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.isfinite(lse[2:]).all()
