"""Attention over the 8-bit cache where rows that are seen hold infinities: a key whose score
is -inf has no weight and takes nothing else with it, one whose score is +inf, or a
value that is infinite or NaN, shows in every row that sees it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from tests.test_gpu_kvq import Pair, _attend, _check_attention, _rows  # noqa: E402


FORMS = [("i8", 64), ("f8", 64), ("i8", 128), ("f8", 128)]


# (the last two: 32 rows a workgroup)
@pytest.mark.parametrize("fmt,hd,len0,n,group", [(*f, *c) for c in ((0, 6, 1), (40, 40, 1), (300, 9, 3)) for f in FORMS] + [
    ("i8", 128, 300, 40, 1024), ("f8", 64, 300, 40, 1024)])
def test_an_infinite_key(fmt, hd, len0, n, group):
    """Queries of few bits and of many; in every third row the key's score is +inf."""
    rng = np.random.default_rng(len0 + n)
    p = Pair(1, 1, hd, 32 * (len0 // 32 + 4), fmt)
    p.preset(rng, len0)
    new = {w: _rows(rng, (1, 1, n, hd)) for w in "kv"}
    new["k"][0, 0, 2, 3], new["k"][0, 0, n - 1, hd - 1] = np.inf, -np.inf
    q = rng.normal(0, 1.4, (n, group, hd))
    q[::2] = np.round(q[::2] * 2) / 2                  # exact in the first of three parts
    q[:, :, 3], q[:, :, hd - 1] = -1.5, 0.75
    q[1::3, :, 3] = 2.0
    with np.errstate(invalid="ignore"):
        got, _ = _check_attention(p, rng, n, group, "chain", new=new, q=q.astype(np.float32).astype(np.float64))
    seen = np.arange(n) >= 2
    plus = np.arange(n) % 3 == 1
    assert np.isfinite(got[~(seen & plus)]).all() and np.isnan(got[seen & plus]).all()


@pytest.mark.parametrize("fmt,hd,len0", [("i8", 64, 0), ("f8", 128, 50), ("i8", 128, 900)])
def test_an_infinite_value_of_next_to_no_weight(fmt, hd, len0):
    """A key so far below the others that its weight is no fp32 number: its infinity and NaN
    show all the same, in the rows that see it and in their dims alone."""
    rng = np.random.default_rng(hd)
    n = 12
    p = Pair(1, 2, hd, 32 * (len0 // 32 + 4), fmt)
    p.preset(rng, len0)
    new = {w: _rows(rng, (1, 2, n, hd), 1.0) for w in "kv"}
    new["k"][0, :, 4] = -400 / np.sqrt(hd)             # about 400 nats below
    new["v"][0, 0, 4, 7], new["v"][0, 1, 4, 9] = np.inf, np.nan
    q = (1 + rng.normal(0, 0.05, (n, 2, hd))).astype(np.float32).astype(np.float64)
    with np.errstate(invalid="ignore"):
        got, _ = _check_attention(p, rng, n, 1, "chain", new=new, q=q)
    want = np.ones((n, 2, hd), bool)
    want[4:, 0, 7] = want[4:, 1, 9] = False
    np.testing.assert_array_equal(np.isfinite(got), want)


@pytest.mark.parametrize("fmt,hd", FORMS)
def test_a_row_of_nothing_but_minus_infinity(fmt, hd):
    """Zeros, as for a row that sees nothing; the rows that see more are not touched by it."""
    rng = np.random.default_rng(3)
    n = 5
    p = Pair(1, 2, hd, 128, fmt)
    new = {w: _rows(rng, (1, 2, n, hd), 1.0) for w in "kv"}
    new["k"][0, :, 0, 1] = -np.inf
    p.put(new, 0)
    q = np.abs(rng.normal(0, 1, (n, 2, hd)))
    got = _attend(p, q, n, 2, None)
    assert not got[0].any()
    want = _attend(p, q, n, 2, np.array([(2 << i) - 2 for i in range(n)], np.uint64))   # without key 0
    np.testing.assert_array_equal(got, want)
