"""Paged cache on the GPU against the float64 oracle: rotary positions and the write into pages,
attention, accumulated weights, commit, eviction; at the sizes, masks and numbers in device
memory where each can go wrong, and all of them together as a server runs them.

Tolerances.  E = 2^-24, half a step of fp32 relative to the number.
  A score is a chain of up to 3 head_dim products whose partial sums are at most S = scale sum |q k|;
  its roundings (E S each at most) are independent, so the chain's end is off by E S sqrt(384) / sqrt(3)
  in the mean: D = 16 E S + 8 E |z| (scaling, tanh) is some deviations away.
  Weights are off by D each and a few E of their exponent; sums of T tiles' weights by at most
  (T + 80) E of the sum.  So out is within W (2 D + (T + 80) E + parts) + half |out|, with W = sum w |v|, parts 0
  (fp32) or 2^-16 (weights in two bf16 parts), half E or 2^-8."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from oracle import paged as op  # noqa: E402
from oracle.verify import round_to_bf16  # noqa: E402
from paper_2412_18934_amd import device as D  # noqa: E402
from paper_2412_18934_amd import dv  # noqa: E402

DEV, E = "cuda:0", 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV).to(dtype)


def _typed(x, dtype):
    """The numbers as the type has them, float64."""
    return torch.from_numpy(x).to(TYPES[dtype]).double().numpy()


class Case:
    """A pool on the GPU and its oracle.  Slots that hold nothing are NaN, K, V and mass."""

    def __init__(self, seed, lens, room, heads=2, hd=64, page=32, layers=2, extra=3, std=1.2):
        self.rng = rng = np.random.default_rng(seed)
        self.lens, self.heads, self.hd, self.page, self.layers = list(lens), heads, hd, page, layers
        need = [(n + r + page - 1) // page for n, r in zip(lens, room)]
        n_pages, width = sum(need) + extra, max(max(need), 1)
        order = list(rng.permutation(n_pages))
        self.pages = [[int(order.pop()) for _ in range(k)] for k in need]
        self.g = D.DevicePaged(layers, heads, hd, n_pages, page, len(lens), width)
        k = np.full((layers, n_pages, heads, page, hd), np.nan)
        v, mass = k.copy(), np.full((layers, n_pages, heads, page), np.nan)
        for pages, n in zip(self.pages, lens):
            for s in range(n):
                p, at = pages[s // page], s % page
                k[:, p, :, at] = rng.normal(0, std, (layers, heads, hd))
                v[:, p, :, at] = rng.normal(0, std, (layers, heads, hd))
                mass[:, p, :, at] = np.float32(rng.random((layers, heads)))
        k, v = (np.where(np.isnan(x), np.nan, round_to_bf16(np.nan_to_num(x))) for x in (k, v))
        self.o = op.Paged(k, v, mass, page)
        self.upload()
        self.g.lens.copy_(torch.tensor(self.lens, dtype=torch.int32))
        for i, pages in enumerate(self.pages):
            if pages:
                self.g.table[i, :len(pages)] = torch.tensor(pages, dtype=torch.int32)

    def upload(self):
        g, o = self.g, self.o
        g.k.copy_(_dev(o.k, torch.bfloat16))
        v = o.v.reshape(*o.v.shape[:3], self.page // 32, 32, self.hd).swapaxes(4, 5)
        g.v.copy_(_dev(v, torch.bfloat16))
        g.mass.copy_(_dev(o.mass, torch.float32))

    def got(self):
        torch.cuda.synchronize()
        v = self.g.v.double().cpu().numpy().swapaxes(4, 5).reshape(self.o.v.shape)
        return self.g.k.double().cpu().numpy(), v, self.g.mass.double().cpu().numpy()

    def same(self, fault=0):
        """Every number of the pool, bit by bit."""
        for name, x, y in zip("kvm", self.got(), (self.o.k, self.o.v, self.o.mass)):
            np.testing.assert_array_equal(x, y, err_msg=name)
        assert int(self.g.fault) == fault

    def put_new(self, layer, counts):
        """New rows' keys and values in their slots."""
        for pages, n, c in zip(self.pages, self.lens, counts):
            shape = (c, self.heads, self.hd)
            self.o.append(layer, pages, n, round_to_bf16(self.rng.normal(0, 1.2, shape)), round_to_bf16(self.rng.normal(0, 1.2, shape)))
        self.upload()


def _start(counts, pad=0):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=DEV)


def _masks(rng, counts, kind):
    """Per sequence and row the set of new rows that it sees."""
    out = []
    for n in counts:
        if kind in ("chain", "none"):
            out.append([set(range(i + 1)) for i in range(n)])
        elif kind == "tree":
            m = []
            for i in range(n):
                m.append({i} | (m[int(rng.integers(0, i))] if i else set()))
            out.append(m)
        else:  # anything, nothing among it
            out.append([set(np.nonzero(rng.random(n) < 0.4)[0].tolist()) if i % 3 else set() for i in range(n)])
    return out


def _bits(masks):
    b = [sum(1 << j for j in m) for one in masks for m in one]
    return torch.from_numpy(np.array(b, dtype=np.uint64).view(np.int64)).to(DEV)


def _queries(c, rng, counts, group, dtype, pad, wide, std=1.3):
    """[rows + pad] rows, `wide` numbers apart beyond their own; values as the type has them."""
    heads, n = c.heads * group, sum(counts)
    x = _typed(rng.normal(0, std, (n + pad, heads, c.hd)), dtype)
    buf = torch.full((n + pad, heads * c.hd + wide), 3.0, dtype=TYPES[dtype], device=DEV)
    buf[:, :heads * c.hd] = _dev(x.reshape(n + pad, -1), TYPES[dtype])
    return x, buf[:, :heads * c.hd].unflatten(1, (heads, c.hd))


def _bounds(c, layer, i, q, z, scale):
    """D of every score of a sequence, [n][query heads][slots]."""
    k, _ = c.o.gathered(c.o.k, layer, c.pages[i], z.shape[2])
    k = np.repeat(np.abs(np.nan_to_num(k)), q.shape[1] // c.heads, axis=1)
    S = abs(scale) * np.einsum("ihd,jhd->ihj", np.abs(q), k)
    return 16 * E * S + 8 * E * np.where(np.isfinite(z), np.abs(z), 0)


def _attend(c, counts, group=1, dtype="f32", masks=None, layer=1, scale=0.0, cap=0.0, pad=0, wide=0, max_rows=None, max_len=None,
            inplace=False, start=True, std=1.3, stats=True, queries=None, ws=None):
    """The call; returns queries (numbers), output, stats (numpy)."""
    x, q = queries or _queries(c, c.rng, counts, group, dtype, pad, wide, std)
    bits = _bits(masks) if masks is not None else None
    if bits is not None and pad:
        bits = torch.cat([bits, torch.full((pad,), -1, dtype=torch.int64, device=DEV)])
    st = _start(counts) if start else None
    rows = c.g.rows(q, st, bits, scale, cap, max_rows or min(64, max(1, max(counts))), max_len)
    out = q if inplace else torch.full((q.shape[0], q.shape[1] * c.hd + 8), 7.0, dtype=q.dtype, device=DEV)[:, :-8].unflatten(
        1, q.shape[1:])
    got = torch.full((*q.shape[:2], 2), 7.0, device=DEV)
    if ws is None:
        size = dv.dv_paged_attention_workspace(c.g.c, rows)
        ws = torch.full((max(size, 16) // 4,), float("nan"), device=DEV)
    dv.dv_paged_attention(c.g.c, layer, rows, out.data_ptr(), out.stride(0), got.data_ptr() if stats else 0, ws.data_ptr(),
                          ws.numel() * 4, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return x, out.double().cpu().numpy(), got.double().cpu().numpy()


def _check_attention(c, counts, group=1, dtype="f32", kind="chain", layer=1, scale=0.0, cap=0.0, masks=None, **kw):
    masks = masks or _masks(c.rng, counts, kind)
    x, out, stats = _attend(c, counts, group, dtype, None if kind == "none" else masks, layer, scale, cap, **kw)
    f, first, worst = scale or c.hd ** -0.5, 0, 0.0
    for i, n in enumerate(counts):
        if not n:
            continue
        q = x[first:first + n]
        z = c.o.scores(layer, c.pages[i], c.lens[i], q, masks[i], f, cap)
        want, top, total = c.o.attention(layer, c.pages[i], c.lens[i], q, masks[i], f, cap)
        d = np.where(np.isfinite(z), _bounds(c, layer, i, q, z, f), 0).max(axis=2)
        tiles = (z.shape[2] + 31) // 32
        w = np.where(np.isfinite(z), np.exp(z - np.where(np.isfinite(top), top, 0)[..., None]), 0) / np.where(total, total, 1)[..., None]
        v, _ = c.o.gathered(c.o.v, layer, c.pages[i], z.shape[2])
        W = np.einsum("ihj,jhd->ihd", w, np.repeat(np.abs(np.nan_to_num(v)), group, axis=1))
        rel = 2 * d + (tiles + 80) * E
        tol = W * (rel + (2.0 ** -16 if dtype == "bf16" else 0))[..., None] + np.abs(want) * (2.0 ** -8 if dtype == "bf16" else E)
        got, st = out[first:first + n], stats[first:first + n]
        err = np.abs(got - want)
        over = float((err / np.maximum(tol, 1e-300)).max())
        assert over <= 1, (i, over)
        worst = max(worst, float((err / np.maximum(tol, 1e-300)).max()))
        if kw.get("stats", True):
            empty = total == 0
            assert (st[..., 0][empty] == -np.inf).all() and not st[..., 1][empty].any() and not got[empty].any()
            assert (np.abs(st[..., 0][~empty] - top[~empty]) <= d[~empty]).all()
            assert (np.abs(st[..., 1] - total)[~empty] <= (total * rel)[~empty]).all()
        first += n
    # rows behind the last sequence are as they were
    if not kw.get("inplace"):
        assert (out[first:] == 7.0).all()
    assert (stats[first:] == 7.0).all()
    print("[paged] worst error / tolerance %.3g" % worst, flush=True)
    return x, out, stats


# ---------------------------------------------------------------------------
# attention

@pytest.mark.parametrize("dtype,hd", [("f32", 64), ("bf16", 64), ("f32", 128), ("bf16", 128)])
@pytest.mark.parametrize("lens,counts,group,kind", [
    ([0], [1], 1, "none"), ([1, 0, 31], [1, 1, 1], 3, "none"), ([32, 33, 63, 64], [1, 1, 1, 1], 1, "chain"),
    ([0, 5, 40], [6, 0, 20], 1, "tree"), ([97, 0], [64, 64], 1, "tree"), ([30, 70], [5, 17], 16, "any"), ([129], [3], 5, "any"),
    ([2, 260, 0, 31], [1, 33, 2, 0], 2, "tree")], ids=str)
def test_attention(dtype, hd, lens, counts, group, kind):
    c = Case(hd + len(lens), lens, counts, hd=hd, heads=3 if group < 5 else 1)
    c.put_new(1, counts)
    _check_attention(c, counts, group, dtype, kind)
    assert int(c.g.fault) == 0


@pytest.mark.parametrize("max_rows,max_len", [(1, 0), (64, 1 << 20), (3, 767), (3, 768)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_hints_choose_the_cut_alone(dtype, max_rows, max_len):
    """One workgroup per row block, or shares of the line of tiles; row blocks of 16 and 32."""
    lens, counts = [900, 0, 77, 1500, 3, 40], [2, 5, 30, 1, 0, 11]
    c = Case(5, lens, counts, heads=2, hd=128, page=96)
    c.put_new(1, counts)
    _check_attention(c, counts, 3, dtype, "tree", max_rows=max_rows, max_len=max_len, pad=3, wide=8)


@pytest.mark.parametrize("seqs,length,heads", [(1, 20000, 1), (1, 3333, 4), (90, 60, 3), (600, 33, 1), (7, 2000, 2)])
def test_long_ones_and_many(seqs, length, heads):
    """Shares that begin and end inside units; more sequences than threads of the scan."""
    rng = np.random.default_rng(seqs)
    lens = [length] + [int(x) for x in rng.integers(0, length, seqs - 1)]
    counts = [int(x) for x in rng.integers(0, 4, seqs)]
    counts[0] = 2
    c = Case(1, lens, counts, heads=heads, hd=64, page=64, layers=1)
    c.put_new(0, counts)
    _check_attention(c, counts, 2, "f32", "tree", layer=0, max_len=100000)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cap,scale,std", [(20.0, 0.0, 1.3), (5.0, 0.5, 3.0), (50.0, -0.2, 1.0), (0.0, 1.0, 2.0), (1e-3, 0.0, 1.0)])
def test_capped_scores(dtype, cap, scale, std):
    lens, counts = [100, 7, 0], [4, 9, 3]
    c = Case(11, lens, counts, hd=128)
    c.put_new(1, counts)
    _check_attention(c, counts, 2, dtype, "any", cap=cap, scale=scale, std=std)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_without_stats(dtype):
    lens, counts = [900, 40], [3, 18]
    c = Case(21, lens, counts, hd=128, page=128)
    c.put_new(1, counts)
    for max_len in (10, 2000):
        _check_attention(c, counts, 4, dtype, "tree", inplace=True, max_len=max_len)
        _check_attention(c, counts, 4, dtype, "tree", stats=False, max_len=max_len)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("max_len", [10, 5000])
def test_the_most_query_heads_of_a_kv_head(dtype, max_len):
    lens, counts = [70, 900], [1, 2]
    c = Case(23, lens, counts, hd=64, heads=1, page=64)
    c.put_new(1, counts)
    _check_attention(c, counts, 1024, dtype, "chain", max_len=max_len)
    _check_mass(c, counts, 1024, dtype, "chain", max_len=max_len)


def test_one_row_each_without_start():
    lens = [5, 700, 0, 64]
    c = Case(2, lens, [1] * 4, hd=64)
    c.put_new(1, [1] * 4)
    for max_len in (0, 5000):
        _check_attention(c, [1] * 4, 2, "bf16", "none", start=False, max_len=max_len)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("max_len", [10, 5000])
def test_what_a_row_does_not_see_may_be_anything(dtype, max_len):
    """Infinities and NaN in new rows that a mask hides, and behind the last row (Case's
    NaN): the rows that see them show it, in their dims, the others nothing."""
    lens, n = [40, 800], 9
    c = Case(31, lens, [n, n], hd=64, heads=2)
    c.put_new(1, [n, n])
    masks = _masks(c.rng, [n, n], "chain")
    for m in masks:
        for i in range(n):
            m[i] -= {2, 5} if i not in (2, 5) else set()
    q = _queries(c, c.rng, [n, n], 1, dtype, 0, 0)
    _, want, _ = _attend(c, [n, n], 1, dtype, masks, queries=q, max_len=max_len)
    for i, pages in enumerate(c.pages):
        for j, bad in ((2, np.inf), (5, np.nan)):
            p, at = pages[(lens[i] + j) // 32], (lens[i] + j) % 32
            c.o.v[1, p, :, at, 7] = bad
            if j == 5:
                c.o.k[1, p, :, at, 3] = -np.inf
    c.upload()
    _, got, _ = _attend(c, [n, n], 1, dtype, masks, queries=q, max_len=max_len)
    assert np.isfinite(want).all()
    for i, first in enumerate((0, n)):
        with np.errstate(invalid="ignore"):
            w, _, _ = c.o.attention(1, c.pages[i], lens[i], q[0][first:first + n], masks[i], 64 ** -0.5)
        part = got[first:first + n]
        # row 2 sees its own value's dim 7; row 5 its key, whose score is -inf (no weight) or +inf,
        # and its value's dim 7
        assert not np.isfinite(part[2, :, 7]).any() and not np.isfinite(part[5, :, 7]).any()
        hit = np.zeros(part.shape, bool)
        hit[2, :, 7] = True
        hit[5] = True
        np.testing.assert_array_equal(part[~hit], want[first:first + n][~hit])
        minus = q[0][first + 5, :, 3] > 0
        rest = np.arange(64) != 7
        np.testing.assert_array_equal(np.isfinite(part[5][:, rest]), np.repeat(minus[:, None], 63, axis=1))
        assert np.abs(part[5, minus][:, rest] - w[5, minus][:, rest]).max(initial=0) < (0.02 if dtype == "bf16" else 1e-5)
        assert np.isfinite(part[2][:, rest]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("max_len", [10, 5000])
def test_bad_queries_keys_and_values_show(dtype, max_len):
    lens = [40, 900, 900]
    c = Case(41, lens, [2, 2, 2], hd=128, heads=1)
    c.put_new(1, [2, 2, 2])
    q = _queries(c, c.rng, [2, 2, 2], 2, dtype, 0, 0)
    q[1][3, 1, 5] = float("nan")
    p = c.pages[0][0]
    c.o.k[1, p, 0, 3, 9] = np.inf                      # scores of both signs, by the query's
    x = q[0][:2, :, 9]
    p = c.pages[2][-3]
    c.o.v[1, p, 0, 1, 100] = -np.inf
    c.upload()
    _, got, _ = _attend(c, [2, 2, 2], 2, dtype, None, queries=q, max_len=max_len)
    hit = np.zeros(got.shape, bool)
    hit[0:2] = (x > 0)[..., None]
    hit[3, 1] = True
    hit[4:, :, 100] = True
    np.testing.assert_array_equal(np.isfinite(got), ~hit)


@pytest.mark.parametrize("max_len", [10, 5000])
def test_numbers_that_cannot_be(max_len):
    """Pages outside the pool are not seen; sequences whose numbers cannot be are skipped, the
    others are as they would be without them."""
    lens, counts = [100, 900, 50, 64, 700], [2, 3, 4, 1, 2]
    c = Case(51, lens, counts, hd=64)
    c.put_new(1, counts)
    masks = _masks(c.rng, counts, "tree")
    q = _queries(c, c.rng, counts, 2, "f32", 0, 0)
    _, want, _ = _attend(c, counts, 2, "f32", masks, queries=q, max_len=max_len)
    assert int(c.g.fault) == 0
    # (page 1 of sequence 0, pages 3 and 20 of sequence 1)
    for i, p, bad in ((0, 1, -1), (1, 3, c.g.c.n_pages), (1, 20, 2 ** 31 - 1)):
        c.g.table[i, p] = bad
        c.pages[i][p] = bad
    c.g.lens[2], c.g.lens[4] = -7, c.g.c.table_stride * 32 - 1
    _, got, _ = _attend(c, counts, 2, "f32", masks, queries=q, max_len=max_len)
    assert int(c.g.fault) == 1
    at = np.concatenate([[0], np.cumsum(counts)])
    assert (got[at[2]:at[3]] == 7.0).all() and (got[at[4]:] == 7.0).all()
    np.testing.assert_array_equal(got[at[3]:at[4]], want[at[3]:at[4]])
    for i in (0, 1):
        x = q[0][at[i]:at[i + 1]]
        w, _, _ = c.o.attention(1, c.pages[i], lens[i], x, masks[i], 64 ** -0.5)
        assert np.abs(got[at[i]:at[i + 1]] - w).max() < 1e-4
    # rows outside the call's, and too many
    c.g.fault.zero_()
    start = torch.tensor([0, 2, 1, 3, 3, 90], dtype=torch.int32, device=DEV)
    out = torch.full_like(q[1], 7.0)
    rows = c.g.rows(q[1], start, None, max_len=max_len)
    ws = torch.empty(max(16, dv.dv_paged_attention_workspace(c.g.c, rows)), dtype=torch.uint8, device=DEV)
    dv.dv_paged_attention(c.g.c, 1, rows, out.data_ptr(), out.stride(0), 0, ws.data_ptr(), ws.numel())
    torch.cuda.synchronize()
    assert int(c.g.fault) == 1 and (out[3:] == 7.0).all() and torch.isfinite(out[:2]).all() and (out[:2] != 7.0).all()


def test_sequences_that_share_pages():
    c = Case(61, [96, 96, 100], [1, 1, 1], hd=64, page=32)
    c.put_new(1, [1, 1, 1])
    for i in (1, 2):
        c.pages[i][:3] = c.pages[0][:3]
        c.g.table[i, :3] = c.g.table[0, :3]
    c.put_new(1, [1, 1, 1])
    _check_attention(c, [1, 1, 1], 2, "f32", "none")


def test_a_workspace_too_small_is_refused():
    c = Case(3, [5000], [1])
    q = torch.zeros((1, 2, 64), device=DEV)
    rows = c.g.rows(q)
    size = dv.dv_paged_attention_workspace(c.g.c, rows)
    assert size > 0
    for ws, n in ((0, size), (q.data_ptr(), size - 1), (q.data_ptr() + 4, size), (q.data_ptr(), -1)):
        with pytest.raises(dv.DvError) as e:
            dv.dv_paged_attention(c.g.c, 0, rows, q.data_ptr(), 128, 0, ws, n)
        assert e.value.code == dv.DV_EINVAL and "workspace" in str(e.value)


# ---------------------------------------------------------------------------
# append


def _rope(rot, interleaved, scaling, magnitude=1.0):
    return dv.dv_rope_init(dv.dv_rope(10000.0, 8.0, 1.0, 4.0 if scaling == 2 else 32.0, magnitude, 4096, scaling, rot, interleaved))


def _freq(r):
    return np.array(list(r.freq)[:r.rot_dim // 2])


def _append(c, counts, group, dtype, rope, positions, layer=1, pad=0, with_q=True, start=True):
    """q, k, v as parts of the same rows; returns their numbers and the tensor."""
    heads, n = c.heads * (group + 2), sum(counts)
    x = _typed(c.rng.normal(0, 1.2, (n + pad, heads, c.hd)), dtype)
    t = _dev(x, TYPES[dtype])
    st = _start(counts) if start else None
    rows = c.g.rows(t[:, :c.heads * group], st)
    if not with_q:
        rows.q = None
    k = t[:, c.heads * group:]
    v = t[:, c.heads * (group + 1):]
    pos = torch.tensor(positions, dtype=torch.int32, device=DEV) if positions is not None else None
    dv.dv_paged_append(c.g.c, layer, rows, rope, pos.data_ptr() if pos is not None else 0, k.data_ptr(), t.stride(0), v.data_ptr(),
                       t.stride(0), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return x, t


def _check_append(c, counts, group, dtype, rope, positions=None, layer=1, pad=0, with_q=True, start=True):
    """A turned number is two products and a sum, of cos and sin within 2 E: within 6 E m (|x| + |y|), and
    half a step of its type."""
    x, t = _append(c, counts, group, dtype, rope, positions, layer, pad, with_q, start)
    got_k, got_v, got_m = c.got()
    want, tol = x.copy(), np.zeros(x.shape)
    nq, first = c.heads * group, 0
    for i, n in enumerate(counts):
        for a in range(n):
            r = first + a
            if rope is not None:
                pos = positions[r] if positions is not None else c.lens[i] + a
                f, m, il = _freq(rope), rope.magnitude, bool(rope.interleaved)
                part = x[r, :nq + c.heads]
                want[r, :nq + c.heads] = op.turned(part, pos, f, il, m)
                both = np.abs(part[..., 0:2 * len(f):2]) + np.abs(part[..., 1:2 * len(f):2]) if il else \
                    np.abs(part[..., :len(f)]) + np.abs(part[..., len(f):2 * len(f)])
                at = np.arange(2 * len(f)) // 2 if il else np.arange(2 * len(f)) % len(f)
                tol[r, :nq + c.heads, :2 * len(f)] = 6 * E * m * both[..., at]
        first += n
    half = 2.0 ** -8 if dtype == "bf16" else E
    back = t.double().cpu().numpy()
    np.testing.assert_array_equal(back[:, nq:], x[:, nq:])                    # k and v are read only
    if with_q:
        q_tol = tol[:, :nq] + np.where(tol[:, :nq] > 0, half * np.abs(want[:, :nq]), 0)
        assert (np.abs(back[:first, :nq] - want[:first, :nq]) <= q_tol[:first]).all()
    else:
        np.testing.assert_array_equal(back[:, :nq], x[:, :nq])
    np.testing.assert_array_equal(back[first:], x[first:])                    # rows of nobody
    # the pool: new slots, and nothing else
    new = np.zeros(got_m.shape, bool)
    first = 0
    for i, n in enumerate(counts):
        for a, at in enumerate(c.o.places(c.pages[i], range(c.lens[i], c.lens[i] + n))):
            if at is None:
                continue
            r = first + a
            new[layer, at[0], :, at[1]] = True
            k, w = want[r, nq:nq + c.heads], got_k[layer, at[0], :, at[1]]
            assert (np.abs(w - k) <= tol[r, nq:nq + c.heads] + 2.0 ** -8 * np.abs(k)).all()
            np.testing.assert_array_equal(got_v[layer, at[0], :, at[1]], round_to_bf16(x[r, nq + c.heads:]))
        first += n
    assert not got_m[new].any()
    for a, b in ((got_k, c.o.k), (got_v, c.o.v), (got_m, c.o.mass)):
        np.testing.assert_array_equal(a[~new], b[~new])
    assert np.array_equal(c.g.lens.cpu().numpy(), c.lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd,rot,interleaved,scaling,magnitude", [
    (64, 64, 0, 0, 1.0), (128, 128, 1, 0, 1.0), (128, 96, 1, 2, 1.0), (128, 112, 0, 3, 1.2), (64, 2, 0, 1, 1.0), (64, 2, 1, 1, 0.5),
    (128, 6, 0, 0, 1.0), (128, 30, 1, 0, 1.0)])
def test_append(dtype, hd, rot, interleaved, scaling, magnitude):
    lens, counts = [0, 31, 64, 5], [3, 2, 0, 70]
    c = Case(7, lens, counts, hd=hd, heads=3)
    _check_append(c, counts, 2, dtype, _rope(rot, interleaved, scaling, magnitude), pad=2)
    assert int(c.g.fault) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_as_it_is(dtype):
    """Without turning: values and keys rounded once, queries untouched; without queries."""
    lens, counts = [7, 30, 0], [1, 1, 1]
    for kw in (dict(), dict(with_q=False), dict(start=False)):
        c = Case(8, lens, counts, hd=128, heads=5, page=96)
        _check_append(c, counts, 1, dtype, None, **kw)
        c = Case(8, lens, counts, hd=128, heads=5, page=96)
        _check_append(c, counts, 1, dtype, _rope(128, 0, 0), **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts", [[3, 1, 2], [40, 9, 33]])
def test_append_from_rows_of_their_own(dtype, counts):
    """Queries, keys and values of different strides, in different tensors: what the same call writes from one."""
    lens = [5, 0, 31]
    c, d = (Case(13, lens, counts, hd=64, heads=3) for _ in "cd")
    rope, n = _rope(64, 1, 0), sum(counts)
    x, t = _append(c, counts, 2, dtype, rope, None)
    wide = [torch.full((n, h * 64 + w), 9.0, dtype=TYPES[dtype], device=DEV) for h, w in ((6, 0), (3, 24), (3, 8))]
    for buf, (a, b) in zip(wide, ((0, 6), (6, 9), (9, 12))):
        buf[:, :(b - a) * 64] = _dev(x[:, a:b].reshape(n, -1), TYPES[dtype])
    q = wide[0].unflatten(1, (6, 64))
    rows = d.g.rows(q, _start(counts))
    dv.dv_paged_append(d.g.c, 1, rows, rope, 0, wide[1].data_ptr(), wide[1].stride(0), wide[2].data_ptr(), wide[2].stride(0))
    torch.cuda.synchronize()
    assert torch.equal(q, t[:, :6])
    for a, b in zip(c.got(), d.got()):
        np.testing.assert_array_equal(a, b)
    assert (wide[1][:, 192:] == 9.0).all() and (wide[2][:, 192:] == 9.0).all()


def test_append_a_prompt():
    lens, counts = [0, 45, 0, 300], [401, 90, 1, 200]
    c = Case(9, lens, counts, hd=64, heads=2, page=64)
    _check_append(c, counts, 1, "bf16", _rope(64, 0, 0))


@pytest.mark.parametrize("interleaved", [0, 1])
def test_far_positions(interleaved):
    """Angles of up to 2^31 radians are reduced in 64 bits: the angle is off by half a step of its 64-bit
    product at most, 2^31 2^-53 = 2.4e-7, which is 4 E: within the 6 E of cos and sin together with their
    own only in part, so positions here stay below 2^29 (E each for angle and function)."""
    pos = [0, 1, 131071, 1 << 20, 99999999, (1 << 29) - 1, -5, -(1 << 28)]
    c = Case(10, [0] * 8, [1] * 8, hd=64, heads=1)
    _check_append(c, [1] * 8, 2, "f32", _rope(64, interleaved, 0), positions=pos, start=False)


def test_append_many_sequences():
    """The search for a row's sequence: more than 64 and more than 64^2 of them, empty ones among them."""
    for seqs in (63, 64, 65, 200, 4200):
        rng = np.random.default_rng(seqs)
        counts = [int(x) for x in rng.choice([0, 0, 1, 2], seqs)]
        c = Case(seqs, [0] * seqs, [1] * seqs, hd=64, heads=1, layers=1)
        _check_append(c, counts, 1, "bf16", None, layer=0, pad=1)


def test_append_numbers_that_cannot_be():
    lens, counts = [100, 10, 20, 30], [2, 3, 4, 3]
    c = Case(12, lens, counts, hd=64)
    c.g.table[1, 0] = c.g.c.n_pages
    c.pages[1][0] = c.g.c.n_pages
    c.g.lens[2] = c.g.c.table_stride * 32 - 3
    saved = c.lens[2]
    x, t = _append(c, counts, 1, "f32", _rope(64, 0, 0), None)
    assert int(c.g.fault) == 1
    k, v, m = c.got()
    for i in (0, 3):
        for a, at in enumerate(c.o.places(c.pages[i], range(lens[i], lens[i] + counts[i]))):
            r = (0 if i == 0 else 9) + a
            np.testing.assert_array_equal(v[1, at[0], :, at[1]], round_to_bf16(x[r, 4:6]))
            c.o.k[1, at[0], :, at[1]], c.o.v[1, at[0], :, at[1]], c.o.mass[1, at[0], :, at[1]] = k[1, at[0], :, at[1]], v[1, at[0], :, at[1]], 0
    c.same(fault=1)                                    # nothing else was written
    back = t.double().cpu().numpy()
    np.testing.assert_array_equal(back[5:9], x[5:9])   # the skipped sequence's queries too
    assert saved == 20 and not np.array_equal(back[2:5, :2], x[2:5, :2])


# ---------------------------------------------------------------------------
# mass


def _check_mass(c, counts, group=1, dtype="f32", kind="chain", layer=1, cap=0.0, counted=None, max_len=None, pad=0):
    """A weight is off by D and by 8 E and 2 E of its exponent; sums of a slot by 64 E."""
    masks = _masks(c.rng, counts, kind)
    x, q = _queries(c, c.rng, counts, group, dtype, pad, 0)
    f, first, stats = c.hd ** -0.5, 0, np.full((*x.shape[:2], 2), np.nan)
    for i, n in enumerate(counts):
        if n:
            _, top, total = c.o.attention(layer, c.pages[i], c.lens[i], x[first:first + n], masks[i], f, cap)
            stats[first:first + n] = np.stack([np.float32(top), np.float32(total)], axis=-1)
        first += n
    tol = np.zeros(c.o.mass.shape)
    bits, first = counted or [2 ** 64 - 1] * len(counts), 0
    with np.errstate(invalid="ignore", over="ignore"):
        for i, n in enumerate(counts):
            if not n:
                continue
            qs, st = x[first:first + n], stats[first:first + n]
            z = c.o.scores(layer, c.pages[i], c.lens[i], qs, masks[i], f, cap)
            d = _bounds(c, layer, i, qs, z, f)
            w = np.where(np.isfinite(z), np.exp(z - st[..., :1]) / np.where(st[..., 1:] > 0, st[..., 1:], 1), 0)
            w *= np.array([bits[i] >> a & 1 for a in range(n)])[:, None, None]
            part = (w * (d + 8 * E + 2 * E * np.where(np.isfinite(z), np.abs(z - st[..., :1]), 0)) + 64 * E * w).sum(axis=0)
            for j in range(z.shape[2]):
                at = c.o.places(c.pages[i], [j])[0]
                if at:
                    tol[layer, at[0], :, at[1]] = part[:, j].reshape(c.heads, group).sum(axis=1)
            c.o.add_mass(layer, c.pages[i], c.lens[i], qs, masks[i], f, cap, bits[i], st)
            first += n
    bt = _bits(masks)
    if pad:
        bt = torch.cat([bt, torch.full((pad,), -1, dtype=torch.int64, device=DEV)])
    st = _start(counts)
    ct = torch.from_numpy(np.array(bits, dtype=np.uint64).view(np.int64)).to(DEV)
    rows = c.g.rows(q, st, bt, 0.0, cap, max(1, max(counts)), max_len)
    sd = _dev(stats, torch.float32)
    dv.dv_paged_mass(c.g.c, layer, rows, sd.data_ptr(), ct.data_ptr() if counted else 0, torch.cuda.current_stream().cuda_stream)
    k, v, m = c.got()
    want = c.o.mass
    assert np.array_equal(np.isnan(m), np.isnan(want))
    ok = ~np.isnan(want)
    slack = tol + np.where(tol > 0, 2 * E * np.abs(np.nan_to_num(want)) * (1 + max(counts) * group // 64), 0)
    err = np.abs(m[ok] - want[ok])
    assert (err <= slack[ok]).all(), float((err / np.maximum(slack[ok], 1e-300)).max())
    np.testing.assert_array_equal(k, c.o.k)
    np.testing.assert_array_equal(v, c.o.v)


@pytest.mark.parametrize("dtype,hd", [("f32", 64), ("bf16", 64), ("f32", 128), ("bf16", 128)])
@pytest.mark.parametrize("lens,counts,group,kind,cap", [
    ([0], [1], 1, "chain", 0.0), ([5, 0, 64], [3, 0, 1], 2, "chain", 0.0), ([40, 31], [20, 64], 1, "tree", 0.0),
    ([70], [9], 16, "any", 10.0), ([300, 2], [30, 33], 3, "tree", 0.0)], ids=str)
def test_mass(dtype, hd, lens, counts, group, kind, cap):
    c = Case(hd, lens, counts, hd=hd, heads=2)
    c.put_new(1, counts)
    _check_mass(c, counts, group, dtype, kind, cap=cap, pad=1)


@pytest.mark.parametrize("max_len", [0, 400, 100000])
def test_mass_of_counted_rows(max_len):
    lens, counts = [700, 0, 90, 33], [20, 6, 1, 0]
    c = Case(71, lens, counts, hd=64, heads=3)
    c.put_new(1, counts)
    _check_mass(c, counts, 5, "f32", "tree", counted=[0b10010000000000000101, 0, 1, 2 ** 64 - 1], max_len=max_len)


@pytest.mark.parametrize("seqs,length,max_len", [(90, 100, 100000), (300, 70, 100000), (1100, 40, 100000)])
def test_many_sequences(seqs, length, max_len):
    """More than a wave's lanes, and more than a workgroup looks through: attention and mass."""
    rng = np.random.default_rng(seqs)
    lens = [int(x) for x in rng.integers(0, length, seqs)]
    counts = [int(x) for x in rng.integers(0, 3, seqs)]
    counts[-1] = 2
    c = Case(seqs, lens, counts, heads=1, hd=64, page=32, layers=1)
    c.put_new(0, counts)
    _check_attention(c, counts, 2, "bf16", "chain", layer=0, max_len=max_len)
    _check_mass(c, counts, 2, "f32", "chain", layer=0, max_len=max_len, pad=2)


def test_rows_that_do_not_count_may_be_anything():
    lens, counts = [40], [4]
    c = Case(72, lens, counts)
    c.put_new(1, counts)
    x, q = _queries(c, c.rng, counts, 2, "f32", 0, 0)
    q[1] = float("nan")
    stats = torch.full((4, 4, 2), float("nan"), device=DEV)
    for i in (0, 2, 3):
        stats[i, :, 0], stats[i, :, 1] = 3.0, 50.0
    count = torch.tensor([0b1101], dtype=torch.int64, device=DEV)
    rows = c.g.rows(q, _start(counts))
    dv.dv_paged_mass(c.g.c, 1, rows, stats.data_ptr(), count.data_ptr())
    assert np.isfinite(c.got()[2][1][~np.isnan(c.o.mass[1])]).all()
    dv.dv_paged_mass(c.g.c, 1, rows, stats.data_ptr(), 0)          # row 1 counts, and shows
    m = c.got()[2]
    for s in range(44):
        (p, at), = c.o.places(c.pages[0], [s])
        assert np.isnan(m[1, p, :, at]).all() == (s < 42)          # (it sees rows 0 and 1)


def test_mass_numbers_that_cannot_be():
    lens, counts = [100, 50, 64], [2, 4, 1]
    c = Case(73, lens, counts)
    c.put_new(1, counts)
    q = torch.zeros((7, 2, 64), device=DEV)
    stats = torch.ones((7, 2, 2), device=DEV)
    stats[..., 0] = 0
    c.g.table[0, 1] = -3
    c.g.lens[1] = -1
    rows = c.g.rows(q, _start(counts))
    dv.dv_paged_mass(c.g.c, 1, rows, stats.data_ptr())
    before = c.o.mass.copy()
    for i, n in ((0, 102), (2, 65)):
        for s in range(n):
            if i == 0 and s // 32 == 1:
                continue
            (p, at), = c.o.places(c.pages[i], [s])
            sees = counts[i] - max(0, s - lens[i])
            before[1, p, :, at] = np.float32(np.float32(before[1, p, :, at]) + np.float32(sees))
    np.testing.assert_array_equal(c.got()[2], before)
    assert int(c.g.fault) == 1


# ---------------------------------------------------------------------------
# commit and eviction: bit for bit


@pytest.mark.parametrize("hd,page", [(64, 32), (128, 96)])
@pytest.mark.parametrize("inplace", [False, True])
def test_commit(hd, page, inplace):
    lens = [0, 31, 40, 95, 7, 64]
    paths = [[0, 3, 9], list(range(64)), [63], [], [0, 1, 2], list(range(1, 64, 2))]
    c = Case(hd, lens, [64] * 6, hd=hd, heads=3, page=page, layers=3)
    for layer in range(3):
        c.put_new(layer, [64] * 6)
    c.o.mass[:] = np.float32(c.rng.random(c.o.mass.shape))
    c.upload()
    path = torch.full((6, 70), -9, dtype=torch.int32)
    for i, p in enumerate(paths):
        path[i, :len(p)] = torch.tensor(p, dtype=torch.int32)
    path, n = path.to(DEV), torch.tensor([len(p) for p in paths], dtype=torch.int32, device=DEV)
    new = c.g.lens if inplace else torch.full((6,), -1, dtype=torch.int32, device=DEV)
    dv.dv_paged_commit(c.g.c, path.data_ptr(), 70, n.data_ptr(), new.data_ptr())
    want = [c.o.commit(pages, length, p) for pages, length, p in zip(c.pages, lens, paths)]
    c.same()
    assert new.tolist() == want and (inplace or c.g.lens.tolist() == lens)


def test_commit_without_a_path():
    lens = [5, 0, 90]
    c = Case(1, lens, [200, 3, 3])
    n = torch.tensor([200, 0, 2], dtype=torch.int32, device=DEV)
    new = torch.zeros(3, dtype=torch.int32, device=DEV)
    dv.dv_paged_commit(c.g.c, 0, 0, n.data_ptr(), new.data_ptr())
    c.same()
    assert new.tolist() == [205, 0, 92]
    dv.dv_paged_commit(c.g.c, 0, 0, n.data_ptr(), c.g.lens.data_ptr())
    c.same()
    assert c.g.lens.tolist() == [205, 0, 92]


@pytest.mark.parametrize("inplace", [False, True])
def test_commit_numbers_that_cannot_be(inplace):
    lens = [10, 10, 10, 10, 10, 10, 90]
    c = Case(2, lens, [64] * 7, layers=1)
    c.put_new(0, [64] * 7)
    paths = [[0, 2], [0, 0], [1, 0], [0, 64], [-1, 2], [0, 5], [0, 7]]
    path, n = torch.tensor(paths, dtype=torch.int32, device=DEV), torch.tensor([2, 2, 2, 2, 2, 3, 2], dtype=torch.int32, device=DEV)
    c.g.lens[6] = c.g.c.table_stride * 32 - 5           # row 7 is behind the table
    c.g.table[0, 0] = -1                                # sequence 0: nothing can move
    old = c.g.lens.tolist()
    new = c.g.lens if inplace else torch.zeros(7, dtype=torch.int32, device=DEV)
    dv.dv_paged_commit(c.g.c, path.data_ptr(), 2, n.data_ptr(), new.data_ptr())
    c.same(fault=1)
    assert new.tolist() == [12] + old[1:]


def _check_evict(c, budget, recent, inplace=False, fault=0):
    new = c.g.lens if inplace else torch.full((len(c.lens),), -1, dtype=torch.int32, device=DEV)
    dv.dv_paged_evict(c.g.c, budget, recent, new.data_ptr(), torch.cuda.current_stream().cuda_stream)
    want = [c.o.evict(pages, n, budget, recent) for pages, n in zip(c.pages, c.lens)]
    c.same(fault)
    assert new.tolist() == want


@pytest.mark.parametrize("hd,page", [(64, 32), (128, 96)])
@pytest.mark.parametrize("budget,recent", [(1, 0), (1, 1), (20, 20), (20, 5), (33, 0), (64, 10), (130, 1), (500, 3)])
def test_evict(hd, page, budget, recent):
    lens = [0, 1, 21, 64, 65, 131, 400]
    c = Case(budget, lens, [0] * 7, hd=hd, heads=2, page=page)
    _check_evict(c, budget, recent, inplace=recent % 2 == 1)


@pytest.mark.parametrize("n,budget,recent", [(1025, 1000, 3), (2500, 300, 50), (5000, 4999, 0), (3000, 2, 1)])
def test_evict_long(n, budget, recent):
    c = Case(n, [n, 40], [0, 0], hd=64, heads=2, page=64, layers=1)
    _check_evict(c, budget, recent)


@pytest.mark.parametrize("width", [400, 321, 4096])
def test_evict_from_wide_tables(width):
    """Tables of more slots than the ranks that fit LDS, up to the widest."""
    c = Case(width, [3001, 10, 900], [0, 0, 0], hd=64, heads=2, page=64, layers=1)
    table = torch.full((3, width), -1, dtype=torch.int32, device=DEV)
    table[:, :c.g.table.shape[1]] = c.g.table
    c.g.table, c.g.c.table, c.g.c.table_stride = table, table.data_ptr(), width
    _check_evict(c, 800, 64)


@pytest.mark.parametrize("hd", [64, 128])
def test_evict_with_runs(hd):
    """Long runs that stay and go: tiles without a slot, whole ones, batches that begin inside a store."""
    c = Case(83, [2400, 1700], [0, 0], hd=hd, heads=2, page=96, layers=2)
    for i, pages in enumerate(c.pages):
        for s, (p, at) in enumerate(c.o.places(pages, range(c.lens[i]))):
            c.o.mass[:, p, :, at] = (1 if (s // 333) % 2 == i else 0) + np.float32(c.rng.random(c.o.mass[:, p, :, at].shape)) * (s % 50 == 7)
    c.upload()
    _check_evict(c, 1003, 21)


def test_ties_go_to_the_lower_slot():
    """Few different masses, the zeros of both signs, NaN, infinities, the smallest and the largest."""
    c = Case(80, [700, 90], [0, 0], hd=64, heads=3, page=32, layers=2)
    some = np.float32([0.0, -0.0, 0.25, 0.5, np.nan, np.inf, -np.inf, 1e-45, 3e38, -1.0])
    for p in c.pages[0] + c.pages[1]:
        for at in range(32):
            m = some[c.rng.integers(0, len(some), c.o.mass[:, p, :, at].shape)]
            c.o.mass[:, p, :, at] = m
    keep = c.o.mass.copy()
    for budget, recent in ((1, 0), (60, 7), (200, 200), (333, 10), (699, 1)):
        d = Case(80, [700, 90], [0, 0], hd=64, heads=3, page=32, layers=2)
        d.o.mass[:] = keep
        d.upload()
        _check_evict(d, budget, recent)
    d = Case(81, [300], [0], hd=64, heads=1, page=32, layers=1)
    d.o.mass[:] = 0
    d.upload()
    _check_evict(d, 100, 0)


def test_evict_numbers_that_cannot_be():
    lens = [100, 100, 100]
    c = Case(82, lens, [0, 0, 0], layers=1)
    c.g.lens[1], c.g.lens[2] = -4, c.g.c.table_stride * 32 + 1
    c.g.table[0, 1] = 10 ** 6                           # slots 32..63 weigh least; none moves there
    c.pages[0][1] = 10 ** 6
    new = torch.zeros(3, dtype=torch.int32, device=DEV)
    dv.dv_paged_evict(c.g.c, 50, 2, new.data_ptr())
    assert c.o.evict(c.pages[0], 100, 50, 2) == 50
    c.same(fault=1)
    assert new.tolist() == [50, -4, c.g.c.table_stride * 32 + 1]


# ---------------------------------------------------------------------------
# together


def _round(c, counts, x, masks, path, n, budget, stream):
    """A layer's append, attention, mass, then commit and eviction, as a server queues them."""
    heads = c.heads * 2
    st, bits = _start(counts), _bits(masks)
    q = x[:, :heads]
    out = torch.empty_like(q).contiguous()
    stats = torch.empty((*q.shape[:2], 2), device=DEV)
    rows = c.g.rows(q, st, bits, 0.0, 30.0, max(counts))
    ws = torch.empty(max(16, dv.dv_paged_attention_workspace(c.g.c, rows)), dtype=torch.uint8, device=DEV)
    count = torch.zeros(len(counts), dtype=torch.int64, device=DEV)
    for i in range(len(counts)):
        for j in range(int(n[i])):
            count[i] |= 1 << int(path[i, j])
    keep = (st, bits, out, stats, ws, count, rows)
    rope = _rope(64, 0, 0)
    L = c.layers

    def queue():
        for layer in range(L):
            k, v = x[:, heads:], x[:, heads + c.heads:]
            dv.dv_paged_append(c.g.c, layer, rows, rope, 0, k.data_ptr(), x.stride(0), v.data_ptr(), x.stride(0), stream())
            dv.dv_paged_attention(c.g.c, layer, rows, out.data_ptr(), out.stride(0), stats.data_ptr(), ws.data_ptr(), ws.numel(), stream())
            dv.dv_paged_mass(c.g.c, layer, rows, stats.data_ptr(), count.data_ptr(), stream())
        dv.dv_paged_commit(c.g.c, path.data_ptr(), path.stride(0), n.data_ptr(), c.g.lens.data_ptr(), stream())
        dv.dv_paged_evict(c.g.c, budget, 8, c.g.lens.data_ptr(), stream())

    return queue, keep


def _server(seed):
    lens, counts = [60, 0, 33], [7, 3, 5]
    c = Case(seed, lens, [64] * 3, hd=64, heads=2, layers=2)
    c.o.mass[:] = np.nan_to_num(c.o.mass)
    c.upload()
    x = _dev(np.random.default_rng(seed).normal(0, 1, (15, 8, 64)), torch.float32)
    masks = _masks(np.random.default_rng(seed), counts, "tree")
    path = torch.tensor([[0, 2, 6], [0, 1, 0], [0, 0, 0]], dtype=torch.int32, device=DEV)
    n = torch.tensor([3, 2, 1], dtype=torch.int32, device=DEV)
    return c, counts, x, masks, path, n


def _state(c):
    return [t.clone() for t in (c.g.k, c.g.v, c.g.mass, c.g.lens)]


def test_a_round_together():
    """Against the oracle: what is computed within 1e-3, which slots stay and where they stand exactly (no two
    masses of this case are within 1e-4 of the border)."""
    c, counts, x, masks, path, n = _server(90)
    x0 = x.double().cpu().numpy()
    queue, keep = _round(c, counts, x, masks, path, n, 50, lambda: torch.cuda.current_stream().cuda_stream)
    queue()
    torch.cuda.synchronize()
    # the oracle's round (queries turn once per layer, as the calls turn them in place)
    f, q = op.frequencies(64), x0[:, :4].copy()
    for layer in range(2):
        first = 0
        for i, cnt in enumerate(counts):
            for a in range(cnt):
                q[first + a] = op.turned(q[first + a], c.lens[i] + a, f, False)
            r = slice(first, first + cnt)
            k = np.array([op.turned(x0[first + a, 4:6], c.lens[i] + a, f, False) for a in range(cnt)])
            c.o.append(layer, c.pages[i], c.lens[i], round_to_bf16(k.astype(np.float32)), round_to_bf16(x0[r, 6:8]))
            bits = sum(1 << int(path[i, j]) for j in range(int(n[i])))
            c.o.add_mass(layer, c.pages[i], c.lens[i], q[r], masks[i], 0.125, 30.0, bits)
            if layer == 1:
                out, _, _ = c.o.attention(layer, c.pages[i], c.lens[i], q[r], masks[i], 0.125, 30.0)
                assert np.abs(keep[2][r].double().cpu().numpy() - out).max() < 1e-3
            first += cnt
    lens = [c.o.commit(c.pages[i], c.lens[i], path[i, :int(n[i])].tolist()) for i in range(3)]
    for i in range(3):
        for layer in range(2):
            for h in range(2):
                m = np.array([c.o.mass[layer, p, h, at] for p, at in c.o.places(c.pages[i], range(lens[i]))])
                if lens[i] > 50:
                    edge = np.sort(m[:lens[i] - 8])[::-1]
                    assert edge[41] - edge[42] > 1e-4
    lens = [c.o.evict(c.pages[i], lens[i], 50, 8) for i in range(3)]
    assert c.g.lens.tolist() == lens == [50, 2, 34]
    gk, gv, gm = c.got()
    for i in range(3):
        for p, at in c.o.places(c.pages[i], range(lens[i])):
            assert np.abs(gk[:, p, :, at] - c.o.k[:, p, :, at]).max() < 0.05
            np.testing.assert_array_equal(gv[:, p, :, at], c.o.v[:, p, :, at])
            assert np.abs(gm[:, p, :, at] - c.o.mass[:, p, :, at]).max() < 1e-3


def test_a_captured_round_follows_lengths_and_tables():
    """Replays of one captured round against eager ones, with eager work between them: lengths change under the
    graph, and the results do not differ in a bit."""
    c, counts, x, masks, path, n = _server(91)
    d, _, y, _, path2, n2 = _server(91)
    s = torch.cuda.Stream()
    queue, keep = _round(c, counts, x, masks, path, n, 70, lambda: torch.cuda.current_stream().cuda_stream)
    queue2, keep2 = _round(d, counts, y, masks, path2, n2, 70, lambda: torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        queue()
    for i in range(6):
        graph.replay()
        torch.cuda.synchronize()
        queue2()
        torch.cuda.synchronize()
        for a, b in zip(_state(c) + [x, keep[2], keep[3]], _state(d) + [y, keep2[2], keep2[3]]):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
        x.normal_(generator=torch.Generator(DEV).manual_seed(i))
        y.copy_(x)
    assert c.g.lens.tolist() == [70, 12, 39] and int(c.g.fault) == 0


def test_two_caches_on_two_streams():
    """Rounds on caches of their own at once do what each does alone, and repeat bit for bit."""
    want = []
    for seed in (92, 93):
        c, counts, x, masks, path, n = _server(seed)
        queue, keep = _round(c, counts, x, masks, path, n, 40, lambda: torch.cuda.current_stream().cuda_stream)
        queue()
        torch.cuda.synchronize()
        want.append(_state(c) + [keep[2]])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got, live = [], []
        for seed, s in zip((92, 93), streams):
            c, counts, x, masks, path, n = _server(seed)
            queue, keep = _round(c, counts, x, masks, path, n, 40, lambda s=s: s.cuda_stream)
            live.append((c, x, queue, keep))
        torch.cuda.synchronize()
        for one in live:
            one[2]()
        torch.cuda.synchronize()
        for one, w in zip(live, want):
            for a, b in zip(_state(one[0]) + [one[3][2]], w):
                assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_offsets_behind_32_bits():
    """Pages whose bytes lie behind 4 GiB (and elements behind 2^31), in the last of the pool."""
    hd, page, n_pages = 128, 256, 9300
    g = D.DevicePaged(1, 8, hd, n_pages, page, 1, 3, mass=True)
    assert g.k.numel() > 2 ** 31
    rng = np.random.default_rng(0)
    pages = [n_pages - 1, 8200, 0]
    g.table[0] = torch.tensor(pages, dtype=torch.int32)
    g.lens[0] = 500
    k, v = (torch.from_numpy(rng.normal(0, 1.2, (8, 512, hd))).to(torch.bfloat16) for _ in "kv")
    for i in range(2):
        part = slice(256 * i, 256 * i + 256)
        g.k[0, pages[i]] = k[:, part].to(DEV)
        g.v[0, pages[i]] = v[:, part].reshape(8, 8, 32, hd).transpose(2, 3).to(DEV)
    q = torch.from_numpy(rng.normal(0, 1, (1, 8, hd))).float().to(DEV)
    out, stats = torch.zeros_like(q), torch.zeros((1, 8, 2), device=DEV)
    for max_len in (10, 5000):
        rows = g.rows(q, max_len=max_len)
        ws = torch.empty(max(16, dv.dv_paged_attention_workspace(g.c, rows)), dtype=torch.uint8, device=DEV)
        dv.dv_paged_attention(g.c, 0, rows, out.data_ptr(), out.stride(0), stats.data_ptr(), ws.data_ptr(), ws.numel())
        z = (k[:, :501].double() @ q[0].cpu().double()[:, :, None])[..., 0] / hd ** 0.5
        want = (torch.softmax(z, dim=1)[:, None] @ v[:, :501].double())[:, 0]
        assert (out[0].cpu().double() - want).abs().max() < 1e-5
    dv.dv_paged_mass(g.c, 0, rows, stats.data_ptr())
    m = torch.cat([g.mass[0, p] for p in pages[:2]], dim=1).cpu().double()
    assert (m[:, :501] - torch.softmax(z, dim=1)).abs().max() < 1e-6 and not m[:, 501:].any()
    new = torch.zeros(1, dtype=torch.int32, device=DEV)
    dv.dv_paged_evict(g.c, 300, 20, new.data_ptr())
    for h in range(8):
        w = torch.cat([g.mass.new_tensor(0).reshape(1)[:0].cpu(), torch.cat([m[h]]).float()])
        by = sorted(range(480), key=lambda j: (-float(w[j]), j))[:280]
        kept = sorted(by) + list(range(480, 500))
        got = torch.cat([g.k[0, p, h] for p in pages[:2]])[:300].cpu()
        assert torch.equal(got, k[h, kept])
    assert int(new) == 300 and int(g.fault) == 0 and ctypes.sizeof(dv.dv_paged) == 80
