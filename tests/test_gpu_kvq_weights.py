"""Attention over the 8-bit cache where blocks of very different value scales meet: every
weight keeps the bits of an fp32 number, whatever the scale of its block, of the
blocks before it, and of the row's largest weight.

Errors are held against sum(w |v|), the magnitude of what a row really adds up, and not
against the largest value that it could see.
"""
import numpy as np
import pytest

from oracle import kvq as ok
from oracle import verify as ov

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2412_18934_amd import dv  # noqa: E402
from tests.test_gpu_kvq import Pair, _attend, _kv, _rows  # noqa: E402


def _parts(q, k, v):
    """One head without a mask: the exact output, sum(w |v|), and the relative bound of a
    weight's error; u = 2^-24, a half step of fp32.  A score moves by 4 u max|q| sum|k| /
    sqrt(hd) (its query is cut to 2^-22 of the row's largest number) and by (3 hd / 4 + 16)
    u sum|q k| / sqrt(hd) (products added in fp32, at least 4 at a time, and a few roundings
    of scale, factor and reference); exp2 and V's scales are 16 u; adding up is (keys + 16) u.
    Twice, for numerator and denominator."""
    u, hd, keys = 2.0 ** -24, q.shape[1], len(k)
    z = q @ k.T / np.sqrt(hd)
    w = np.exp(z - z.max(axis=1, keepdims=True))
    w /= w.sum(axis=1, keepdims=True)
    mag = (np.abs(q) @ np.abs(k).T).max(axis=1) / np.sqrt(hd)
    cut = 4 * u * np.abs(q).max(axis=1) * np.abs(k).sum(axis=1).max() / np.sqrt(hd)
    rel = 2 * (cut + (3 * hd / 4 + 16) * u * mag + 16 * u + (keys + 16) * u)
    return w @ v, w @ np.abs(v), rel


def _check(fmt, hd, length, n, rows, q):
    """Heads hold the same q, rows {k, v} [1][heads][length + n][hd], the last n new."""
    heads = rows["k"].shape[1]
    p = Pair(1, heads, hd, 32 * ((length + n) // 32 + 2), fmt)
    rows = {w: ov.round_to_bf16(x) for w, x in rows.items()}
    kv = _kv(p, 32 * ((length + n) // 32 + 2), rows)
    dv.dv_kvq_store(p.g.c, kv.c, length)
    p.append({w: rows[w][:, :, :length] for w in "kv"})
    p.put({w: rows[w][:, :, length:] for w in "kv"}, length % 32)
    got = _attend(p, q, n, heads, np.full(n, 2 ** n - 1, np.uint64))
    for h in range(heads):
        k, v = (np.concatenate([p.o[w][0][h].rows(), rows[w][0, h, length:]]) for w in "kv")
        want, mag, rel = _parts(q[:, h], k, v)
        err = np.abs(got[:, h] - want) / mag
        print("[kvq] %s hd %d: error %.2g of sum(w |v|), bound %.2g" % (fmt, hd, err.max(), rel.min()), flush=True)
        assert (err <= rel[:, None]).all(), "head %d: %g over %g" % (h, err.max(), rel.min())


def _along(rng, n, heads, hd, size):
    """Queries that all but point along the ones' direction."""
    return (size + rng.normal(0, 0.05 * size, (n, heads, hd))).astype(np.float32).astype(np.float64)


@pytest.mark.parametrize("fmt,hd", [("i8", 64), ("f8", 64), ("i8", 128), ("f8", 128)])
@pytest.mark.parametrize("power", [16, 36, 90])
def test_large_values_that_hardly_count(fmt, hd, power):
    """Blocks 0 to 7: values 2^power times the others', scores so low that they are
    nothing.  The same waves go on with blocks 8 to 15 and the tail."""
    rng = np.random.default_rng(power)
    n, length = 5, 517
    rows = {w: _rows(rng, (1, 2, length + n, hd), 1.0) for w in "kv"}
    low = (30 + 0.7 * power) / np.sqrt(hd)             # nats below the others, by sqrt(hd) dims
    rows["k"] = 0.1 * rows["k"]
    rows["k"][:, :, :256] -= low
    rows["v"][:, :, :256] *= 2.0 ** power
    _check(fmt, hd, length, n, rows, _along(rng, n, 2, hd, 1.0))


@pytest.mark.parametrize("fmt,hd", [("i8", 128), ("f8", 64)])
@pytest.mark.parametrize("down", [16, 24, 40])
def test_a_key_that_takes_the_weight_and_has_no_value(fmt, hd, down):
    """A first key of value 0, all others 2^-down of its weight, and between them a block
    of values 2^10 times the others'."""
    rng = np.random.default_rng(down)
    n, length = 3, 700
    rows = {w: _rows(rng, (1, 2, length + n, hd), 1.0) for w in "kv"}
    rows["k"] = 0.1 * rows["k"]
    rows["k"][:, :, 0] = down * np.log(2) / np.sqrt(hd)
    rows["v"][:, :, 0] = 0
    rows["k"][:, :, 64:96] -= 12 / np.sqrt(hd)
    rows["v"][:, :, 64:96] *= 2.0 ** 10
    _check(fmt, hd, length, n, rows, _along(rng, n, 2, hd, 1.0))
