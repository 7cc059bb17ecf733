"""Pins of the plain forms of the operators over resident units (CPU)."""
import numpy as np
import torch

from oracle import model as M


def test_e4m3_values_are_the_type():
    codes = np.arange(256, dtype=np.uint8)
    t = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, M.E4M3_VALUES, equal_nan=True)
    assert np.nanmax(M.E4M3_VALUES) == 448


def test_16_bit_conversions():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(10_000) * 10.0 ** rng.integers(-10, 5, 10_000),
                        [0.0, -0.0, np.inf, -np.inf, 65504.0, 65520.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -9]])
    for kind, dt in ((M.BF16, torch.bfloat16), (M.F16, torch.float16)):
        t = torch.from_numpy(x.astype(np.float32)).to(dt)
        assert np.array_equal(M.to_bits(x, kind), t.view(torch.int16).numpy().view(np.uint16))
        assert np.array_equal(M.from_bits(M.to_bits(x, kind), kind), t.double().numpy())


def test_half_step_covers_nearest_values():
    q = np.linspace(-448, 448, 100_001)
    finite = M.E4M3_VALUES[np.isfinite(M.E4M3_VALUES)]
    order = np.sort(np.unique(finite))
    i = np.clip(np.searchsorted(order, q), 1, len(order) - 1)
    err = np.minimum(np.abs(order[i] - q), np.abs(order[i - 1] - q))
    assert (err <= M.e4m3_half_step(q)).all()
    assert (err > 0.9 * M.e4m3_half_step(q)).any()


def test_attention_against_torch_and_merged():
    """The softmax form against torch's in 64 bits, and against two halves of the
    keys joined by their log-sums."""
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal(s) for s in ((3, 2, 2, 16), (11, 2, 16), (11, 2, 16)))
    seen = np.arange(11) <= np.array([4, 9, 10])[:, None]
    out, lse, mag, _, _ = M.attention(q, k, v, seen, 0.25)
    t = torch.from_numpy(np.einsum("rhgd,thd->rhgt", q, k) * 0.25)
    t = t.masked_fill(~torch.from_numpy(seen)[:, None, None], -np.inf)
    ref = torch.matmul(torch.softmax(t, -1).permute(1, 0, 2, 3).reshape(2, 6, 11),
                       torch.from_numpy(v).permute(1, 0, 2)).reshape(2, 3, 2, 16).permute(1, 0, 2, 3)
    assert np.allclose(out, ref.numpy(), rtol=0, atol=1e-14) and (mag >= np.abs(out) - 1e-14).all()
    a, b = (M.attention(q, k[s], v[s], seen[:, s], 0.25) for s in (slice(0, 4), slice(4, 11)))
    total = np.logaddexp(a[1], b[1])
    joined = a[0] * np.exp(a[1] - total)[..., None] + b[0] * np.exp(b[1] - total)[..., None]
    assert np.allclose(joined, out, atol=1e-14) and np.allclose(total, lse, atol=1e-14)


def test_attention_of_nothing():
    q = np.ones((2, 1, 1, 16))
    v = np.full((3, 1, 16), np.nan)
    out, lse, *_ = M.attention(q, v, v, np.zeros((2, 3), bool), 1.0)
    assert (out == 0).all() and np.isneginf(lse).all()
    out, lse, *_ = M.attention(q, v[:0], v[:0], np.zeros((2, 0), bool), 1.0)
    assert (out == 0).all() and np.isneginf(lse).all()


def test_attention_of_a_nan_is_nan_where_it_is_seen():
    q, k = np.ones((2, 1, 1, 16)), np.ones((3, 1, 16))
    v = k.copy()
    k[2] = v[2] = np.nan
    seen = np.array([[True, True, False], [True, True, True]])
    out, lse, *_ = M.attention(q, np.where(seen.all(0)[:, None, None], k, k), v, seen, 1.0)
    assert np.isnan(out[1]).all() and np.isnan(lse[1]).all() and np.isfinite(lse[0]).all()


def test_positions():
    r, t = M.positions([0, 2, 2, 5], [7, 3, 1])
    assert r.tolist() == [0, 0, 2, 2, 2] and t.tolist() == [5, 6, -2, -1, 0]


def test_e4m3_encode_is_nearest_even():
    rng = np.random.default_rng(2)
    q = np.concatenate([rng.uniform(-500, 500, 20_000), rng.standard_normal(20_000) * 2.0 ** -7,
                        (M.E4M3_VALUES[:126] + M.E4M3_VALUES[1:127]) / 2, [0.0, -0.0, np.nan, 448, -448]])
    q = q.astype(np.float32)
    t = torch.from_numpy(q).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    ours = M.e4m3_encode(q)
    nan = np.isnan(q)
    assert np.array_equal(ours[~nan], t[~nan]) and (ours[nan] & 127 == 127).all()


def test_stored_keeps_16_bit_rows_and_rounds_to_e4m3():
    x = np.random.default_rng(3).standard_normal((5, 2, 32))
    assert M.stored(x, M.BF16) is x
    y = M.stored(x, M.E4M3)
    assert (np.abs(y - x) <= M.e4m3_half_step(x / M.e4m3_scale(x)[..., None]) * M.e4m3_scale(x)[..., None]
            * (1 + 2.0 ** -20)).all()
