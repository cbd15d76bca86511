"""Pins of the 8-bit cache's oracle: e4m3 against torch's type, block order, the
rounding of codes, blocks without a scale, attention's mask."""
import numpy as np
import pytest

from oracle import kvq as ok
from oracle.verify import round_to_bf16

torch = pytest.importorskip("torch")


def test_e4m3_numbers_and_rounding_are_torch_s():
    codes = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(ok.e4m3_values(), codes.view(torch.float8_e4m3fn).double().numpy())
    rng = np.random.default_rng(0)
    y = np.concatenate([rng.uniform(-448, 448, 4000), rng.normal(0, 0.05, 4000), ok.e4m3_values()[:0x7f],
                        # ties between neighbours, the smallest ones too
                        (ok.e4m3_values()[:0x7e] + ok.e4m3_values()[1:0x7f]) / 2]).astype(np.float32)
    np.testing.assert_array_equal(ok.e4m3_code(y), torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("hd", [64, 128])
def test_block_order_is_a_permutation(hd):
    for at in (ok.k_byte(hd), ok.v_byte(hd)):
        assert sorted(at.reshape(-1)) == list(range(32 * hd))
    # 16 bytes of K are 2 x 8 dims of one slot, of V 2 x 8 slots
    slot = np.empty(32 * hd, int)
    slot[ok.k_byte(hd).reshape(-1)] = np.repeat(np.arange(32), hd)
    assert all(len(set(slot[i:i + 16])) == 1 for i in range(0, 32 * hd, 16))
    slot[ok.v_byte(hd).reshape(-1)] = np.repeat(np.arange(32), hd)
    assert all(list(slot[i:i + 8]) == list(range(slot[i], slot[i] + 8)) for i in range(0, 32 * hd, 8))


@pytest.mark.parametrize("fmt", ["i8", "f8"])
def test_codes_are_within_half_a_step(fmt):
    x = round_to_bf16(np.random.default_rng(1).normal(0, 1.4, (32, 128)))
    x[3, 5], x[0, 0] = 0.0, 41.0
    codes, scale = ok.quantise(x, fmt)
    back = ok.numbers(codes, fmt) * np.float64(scale)
    assert np.abs(ok.numbers(codes, fmt)).max() == ok.TOP[fmt]
    # scale, factor and product carry 3 half steps of fp32 on top of the code's half step
    eps = 3 * 2.0 ** -24 * np.abs(x)
    if fmt == "i8":
        assert (np.abs(back - x) <= scale / 2 * (1 + 2.0 ** -20) + eps).all()
    else:
        half = np.maximum(np.abs(x) * 2.0 ** -4, scale * 2.0 ** -10)
        assert (np.abs(back - x) <= half * (1 + 2.0 ** -20) + eps).all()


@pytest.mark.parametrize("fmt", ["i8", "f8"])
def test_blocks_without_a_scale(fmt):
    x = np.full((32, 64), 1.0)
    for bad in (np.inf, -np.inf, np.nan):
        y = x.copy()
        y[7, 9] = bad
        codes, scale = ok.quantise(y, fmt)
        assert np.isnan(scale) and not codes.any()
    for small in (0.0, -0.0, 2.0 ** -101):
        codes, scale = ok.quantise(x * small, fmt)
        assert scale == 0 and not codes.any()
    codes, scale = ok.quantise(x * 2.0 ** -100, fmt)
    assert scale > 0 and np.isfinite(scale)


def test_codes_do_not_depend_on_how_rows_came():
    rows = round_to_bf16(np.random.default_rng(2).normal(size=(101, 64)))
    whole, parts = ok.Cache(64, "i8"), ok.Cache(64, "i8")
    whole.append(rows)
    for at in (0, 1, 30, 31, 33, 100, 101):
        parts.append(rows[len(parts):at])
    assert len(whole) == len(parts) == 101 and len(whole.blocks) == 3
    np.testing.assert_array_equal(whole.rows(), parts.rows())


def test_attention_masks():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(3, 64)), rng.normal(size=(5, 64)), rng.normal(size=(5, 64))
    sees = np.array([[1, 0, 0, 0, 0], [0] * 5, [1, 1, 0, 1, 0]], bool)
    k[4], v[2] = np.inf, np.nan
    o = ok.attention(q, k, v, sees)
    np.testing.assert_array_equal(o[0], v[0])
    np.testing.assert_array_equal(o[1], 0)
    assert np.isfinite(o[2]).all()
