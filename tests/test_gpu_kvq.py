"""8-bit KV cache on the GPU against its 64-bit oracle (oracle/kvq.py): codes, scales,
tail and read-back bit for bit, attention within its rounding, and the handle's
prompts, steps and commits over such a cache against the model's oracle.

Buffers that a call may not use are filled with what would show: NaN, sentinel bytes.
"""
import ctypes

import numpy as np
import pytest

import synth
from oracle import kvq as ok
from oracle import verify as ov
from tests.helpers import GpuCase, compare_step, small_cfg

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2412_18934_amd import device as D  # noqa: E402
from paper_2412_18934_amd import dv  # noqa: E402

DEV = "cuda:0"


def _bf16(x):
    """bf16 tensor of floats that bf16 holds."""
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).to(torch.bfloat16)


def _rows(rng, shape, std=1.4):
    return ov.round_to_bf16(rng.normal(0, std, shape))


class Pair:
    """A cache on the GPU and its oracle, per (K or V, layer, head)."""

    def __init__(self, nl, nh, hd, cap, fmt):
        self.nl, self.nh, self.hd, self.cap, self.fmt = nl, nh, hd, cap, fmt
        self.g = D.DeviceKVQ(nl, nh, hd, cap, fmt)
        self.g.k.fill_(0x55)
        self.g.v.fill_(0x55)
        for t in (self.g.scale, self.g.k_tail, self.g.v_tail):
            t.fill_(float("nan"))
        self.o = {w: [[ok.Cache(hd, fmt) for _ in range(nh)] for _ in range(nl)] for w in "kv"}

    def slots(self, which):
        """The tail in slot order, [nl][nh][96][hd] floats."""
        t = (self.g.k_tail if which == "k" else self.g.v_tail.transpose(3, 4).reshape(self.nl, self.nh, 96, self.hd))
        return t.double().cpu().numpy()

    def put(self, rows, at):
        """rows {k, v} [nl][nh][n][hd] into tail slots from `at` on."""
        n = rows["k"].shape[2]
        s = torch.arange(at, at + n, device=DEV)
        for l in range(self.nl):
            self.g.k_tail[l][:, s] = _bf16(rows["k"][l]).to(DEV)
            self.g.v_tail[l][:, s // 32, :, s % 32] = _bf16(rows["v"][l]).to(DEV).transpose(0, 1)

    def append(self, rows):
        for w in "kv":
            for l in range(self.nl):
                for h in range(self.nh):
                    self.o[w][l][h].append(rows[w][l, h])

    def preset(self, rng, n):
        """n committed rows, written as the operators are defined to leave them."""
        rows = {w: _rows(rng, (self.nl, self.nh, n, self.hd)) for w in "kv"}
        self.append(rows)
        r, b = n % 32, n // 32
        for w in "kv":
            at = (ok.k_byte if w == "k" else ok.v_byte)(self.hd)
            codes = np.full((self.nl, self.nh, self.cap // 32, 32 * self.hd), 0x55, np.uint8)
            scale = np.full((self.nl, self.nh, self.cap // 32), np.nan, np.float32)
            for l in range(self.nl):
                for h in range(self.nh):
                    for i, (c, s) in enumerate(self.o[w][l][h].blocks):
                        codes[l, h, i][at] = c
                        scale[l, h, i] = s
            (self.g.k if w == "k" else self.g.v).copy_(torch.from_numpy(codes.view(np.int8)))
            self.g.scale[..., 0 if w == "k" else 1] = torch.from_numpy(scale).to(DEV)
        if r:
            self.put({w: rows[w][:, :, 32 * b:] for w in "kv"}, 0)
        self.g.c.len = n
        return rows

    def check(self):
        """Every block, scale and committed tail row; nothing behind the last block."""
        torch.cuda.synchronize()
        n = len(self.o["k"][0][0])
        assert self.g.len == n
        scale = self.g.scale.cpu().numpy()
        for i, w in enumerate("kv"):
            at = (ok.k_byte if w == "k" else ok.v_byte)(self.hd)
            codes = (self.g.k if w == "k" else self.g.v).cpu().numpy().view(np.uint8)
            tail = self.slots(w)
            for l in range(self.nl):
                for h in range(self.nh):
                    o = self.o[w][l][h]
                    for b, (c, s) in enumerate(o.blocks):
                        np.testing.assert_array_equal(codes[l, h, b][at], c, err_msg="%s %d %d %d" % (w, l, h, b))
                        np.testing.assert_array_equal(scale[l, h, b, i], s)
                    np.testing.assert_array_equal(tail[l, h, :n % 32], o.tail)
            assert (codes[:, :, n // 32:] == 0x55).all() and np.isnan(scale[:, :, n // 32:]).all()


def _kv(pair, cap, rows=None, at=0, fill=float("nan")):
    kv = D.DeviceKV(pair.nl, pair.nh, pair.hd, cap, "bf16", fill=fill)
    if rows is not None:
        n = rows["k"].shape[2]
        s = torch.arange(at, at + n, device=DEV)
        for l in range(pair.nl):
            kv.k[l][:, s] = _bf16(rows["k"][l]).to(DEV)
            kv.v[l][:, s // 32, :, s % 32] = _bf16(rows["v"][l]).to(DEV).transpose(0, 1)
        kv.c.len = at + n
    return kv


# ---------------------------------------------------------------------------
# store, load, advance: bit for bit

LENS = [(0, 1), (0, 31), (0, 32), (0, 33), (5, 20), (31, 1), (31, 70), (64, 100), (95, 2), (96, 31), (7, 25), (1, 62)]


@pytest.mark.parametrize("fmt,hd", [("i8", 64), ("f8", 64), ("i8", 128), ("f8", 128)])
@pytest.mark.parametrize("len0,n", LENS)
def test_store(fmt, hd, len0, n):
    rng = np.random.default_rng(len0 * 100 + n)
    p = Pair(2, 3, hd, 192, fmt)
    p.preset(rng, len0)
    before = {w: p.slots(w) for w in "kv"}
    rows = {w: _rows(rng, (2, 3, n, hd)) * rng.choice([1, 30], (2, 3, 1, hd)) for w in "kv"}
    rows = {w: ov.round_to_bf16(x) for w, x in rows.items()}
    kv = _kv(p, 224, rows, len0)                      # (another capacity, NaN in all other slots)
    dv.dv_kvq_store(p.g.c, kv.c, n)
    p.append(rows)
    p.check()
    end = (len0 + n) % 32
    for w in "kv":                                    # tail slots behind the rows stay as they were
        np.testing.assert_array_equal(p.slots(w)[:, :, max(end, len0 % 32):], before[w][:, :, max(end, len0 % 32):])


@pytest.mark.parametrize("fmt", ["i8", "f8"])
def test_store_of_unusual_blocks(fmt):
    """Zeros, tiny and huge numbers, ties, infinities, NaN, one per head."""
    rng = np.random.default_rng(9)
    p = Pair(1, 10, 64, 64, fmt)
    x = _rows(rng, (1, 10, 32, 64))
    x[0, 0] = 0
    x[0, 1] = np.where(rng.random((32, 64)) < 0.5, -0.0, 2.0 ** -133)
    x[0, 2] = x[0, 2] * 2.0 ** -99
    x[0, 3] = ov.round_to_bf16(np.clip(x[0, 3] * 1e38, -3.3e38, 3.3e38))
    x[0, 4, 3, 7] = np.inf
    x[0, 5, 31, 63] = np.nan
    x[0, 6] = 0
    x[0, 6, 11, 30] = -5.0
    top = ok.TOP[fmt]                                 # codes 0, 1/2, 1, 3/2, .. : ties
    x[0, 7] = ov.round_to_bf16((np.arange(2048).reshape(32, 64) % (2 * top)) / 2)
    x[0, 7, 0, 0] = top
    x[0, 8] = x[0, 8] * 2.0 ** -110
    x[0, 9, 17] *= 2.0 ** -126                        # subnormal among others
    x = ov.round_to_bf16(x)
    rows = {"k": x, "v": x[:, ::-1].copy()}
    kv = _kv(p, 64, rows)
    dv.dv_kvq_store(p.g.c, kv.c, 32)
    p.append(rows)
    p.check()
    back = _kv(p, 64)
    dv.dv_kvq_load(p.g.c, back.c)
    torch.cuda.synchronize()
    got = back.k.double().cpu().numpy()[0, :, :32]
    assert np.isnan(got[4]).all() and np.isnan(got[5]).all() and not got[0].any() and np.isfinite(got[[1, 2, 3, 6, 7, 8, 9]]).all()


@pytest.mark.parametrize("fmt,hd", [("i8", 64), ("f8", 64), ("i8", 128), ("f8", 128)])
@pytest.mark.parametrize("n", [0, 1, 31, 32, 45, 96, 127])
def test_load(fmt, hd, n):
    p = Pair(2, 3, hd, 160, fmt)
    p.preset(np.random.default_rng(n), n)
    kv = _kv(p, 128, fill=-77.0)
    dv.dv_kvq_load(p.g.c, kv.c)
    torch.cuda.synchronize()
    assert kv.len == n
    for w in "kv":
        for l in range(2):
            got = (kv.k[l] if w == "k" else kv._v_slots(l)).double().cpu().numpy()
            for h in range(3):
                o = p.o[w][l][h]
                if n:
                    # fp32 product, then bf16
                    want = ov.round_to_bf16(np.concatenate([o.rows()[:32 * len(o.blocks)].astype(np.float32)
                                                            .astype(np.float64), o.tail]))
                    np.testing.assert_array_equal(got[h, :n], want)
            assert (got[:, n:] == -77.0).all()


PATHS = [(0, [0]), (0, [5]), (30, [0, 1]), (31, [0]), (31, [63]), (13, [0, 2, 3, 9]), (0, list(range(32))),
         (0, list(range(0, 64, 2))), (20, [0, 1, 2, 7, 8, 11, 12, 13, 14, 20, 40, 63]), (31, list(range(64))),
         (31, list(range(30, 63))), (1, list(range(1, 64))), (63, [0, 63]), (40, [0, 1, 2, 3, 4])]


@pytest.mark.parametrize("fmt,hd", [("i8", 64), ("f8", 64), ("i8", 128), ("f8", 128)])
@pytest.mark.parametrize("len0,path", PATHS, ids=["%d+%d" % (a, len(b)) for a, b in PATHS])
def test_advance(fmt, hd, len0, path):
    rng = np.random.default_rng(len0 + len(path))
    p = Pair(2, 3, hd, 192, fmt)
    p.preset(rng, len0)
    new = {w: _rows(rng, (2, 3, 64, hd)) for w in "kv"}
    p.put(new, len0 % 32)
    before = {w: p.slots(w) for w in "kv"}
    dv.dv_kvq_advance(p.g.c, path)
    p.append({w: new[w][:, :, path] for w in "kv"})
    p.check()
    for w in "kv":
        end = len0 % 32 + len(path)
        end = end if end < 32 else end % 32
        np.testing.assert_array_equal(p.slots(w)[:, :, end:], before[w][:, :, end:])


def test_codes_do_not_depend_on_how_rows_came():
    """A prompt at once, in pieces, and as accepted paths: the same cache, byte for
    byte."""
    rng = np.random.default_rng(4)
    rows = {w: _rows(rng, (2, 2, 150, 64)) for w in "kv"}
    caches = []
    for how in range(3):
        p = Pair(2, 2, 64, 160, "i8")
        kv = _kv(p, 160, rows)
        while p.g.len < 150:
            n = 150 if how == 0 else min(150 - p.g.len, int(rng.integers(1, 50)))
            if how < 2:
                dv.dv_kvq_store(p.g.c, kv.c, n)
            else:
                p.put({w: rows[w][:, :, p.g.len:p.g.len + n] for w in "kv"}, p.g.len % 32)
                dv.dv_kvq_advance(p.g.c, list(range(n)))
        caches.append(p)
    torch.cuda.synchronize()
    a = caches[0]
    for b in caches[1:]:
        assert torch.equal(a.g.k, b.g.k) and torch.equal(a.g.v, b.g.v)
        np.testing.assert_array_equal(a.g.scale.cpu().numpy(), b.g.scale.cpu().numpy())
        for w in "kv":
            np.testing.assert_array_equal(a.slots(w)[:, :, :22], b.slots(w)[:, :, :22])


# ---------------------------------------------------------------------------
# attention

def _sees(rng, n, kind):
    """Mask bits and bool [n][n]."""
    if kind == "chain":
        return None, np.tril(np.ones((n, n), bool))
    if kind == "tree":
        par = [-1] + [int(rng.integers(0, i)) for i in range(1, n)]
        m = dv.dv_tree_prepare(par, 0)[2]
    else:   # any bits, some rows none at all; bits past n are ignored
        m = rng.integers(0, 2 ** 63, n).astype(np.uint64)
        m[::3] = 0
    return m, np.array([[int(m[i]) >> j & 1 for j in range(n)] for i in range(n)], bool)


def _tolerance(q, k, v, sees):
    """Bound of one head's error, [n], worst cases added up; u = 2^-24, a half step of fp32.
    A score: its query is cut to 2^-22 of the row's largest number (int8: an integer of
    at most 2^22 rounded; e4m3: two truncated fp16 of a row scaled to at most 2^11), which
    moves it by 4 u max|q| sum|k| / sqrt(hd); at most 3 hd products are added in fp32, by at
    least 4 at a time, and scale, factor and reference round a few times: (3 hd / 4 + 16) u
    times the sum of |q k| / sqrt(hd).  exp2 adds 2 u, a weight in two truncated fp16 is
    cut by 4 u of it, or by 2^-24 / 2^11 of the largest, and V's scales round 4 times: 12 u
    relative and 2^-35 of the largest weight per key.  The sums over keys: (keys + 16) u of
    their absolute terms.  Numerator and denominator each."""
    u, (n, hd) = 2.0 ** -24, q.shape
    tol = np.zeros(n)
    for i in range(n):
        at = np.flatnonzero(sees[i])
        if len(at):
            mag = (np.abs(k[at]) @ np.abs(q[i])).max() / np.sqrt(hd)
            cut = 4 * u * np.abs(q[i]).max() * np.abs(k[at]).sum(axis=1).max() / np.sqrt(hd)
            rel = cut + (3 * hd / 4 + 16) * u * mag + 12 * u + len(at) * 2.0 ** -35 + (len(at) + 16) * u
            tol[i] = 2 * rel * np.abs(v[at]).max()
    return tol


def _attend(p, q, n, n_heads, mask, layer=0, pad_q=0, pad_o=0, stream=0, ws=None):
    """q float64 [n][n_heads][hd] -> out float64; strides with padding."""
    hd = p.hd
    qd = torch.full((n, n_heads * hd + pad_q), float("nan"), device=DEV)
    qd[:, :n_heads * hd] = torch.from_numpy(q.reshape(n, -1)).float().to(DEV)
    out = torch.full((n, n_heads * hd + pad_o), -123.0, device=DEV)
    need = dv.dv_kvq_attention_workspace(p.g.c, n, n_heads)
    ws = torch.full((need // 4 + 8,), float("nan"), device=DEV)
    torch.cuda.synchronize()
    dv.dv_kvq_attention(p.g.c, layer, qd.data_ptr(), qd.stride(0), n, n_heads, mask, out.data_ptr(), out.stride(0),
                        ws.data_ptr() if need else 0, need, stream)
    torch.cuda.synchronize()
    assert torch.isnan(ws[need // 4:]).all()          # nothing past the workspace
    assert (out[:, n_heads * hd:] == -123.0).all()
    return out[:, :n_heads * hd].double().cpu().numpy().reshape(n, n_heads, hd)


def _check_attention(p, rng, n, group, kind, layer=0, new=None, q=None, **kw):
    """Puts n new rows (and NaN behind them), attends, compares with the oracle."""
    nl, nh, hd = p.nl, p.nh, p.hd
    r = p.g.len % 32
    new = new or {w: _rows(rng, (nl, nh, n, hd)) for w in "kv"}
    p.put(new, r)
    if r + n < 96:
        p.put({w: np.full((nl, nh, 96 - r - n, hd), np.nan) for w in "kv"}, r + n)
    q = rng.normal(0, 1.4, (n, nh * group, hd)).astype(np.float32).astype(np.float64) if q is None else q
    mask, sees = _sees(rng, n, kind)
    got = _attend(p, q, n, nh * group, mask, layer, **kw)
    every = np.concatenate([np.ones((n, p.g.len), bool), sees], axis=1)
    worst = 0.0
    for h in range(nh * group):
        k = np.concatenate([p.o["k"][layer][h // group].rows(), new["k"][layer, h // group]])
        v = np.concatenate([p.o["v"][layer][h // group].rows(), new["v"][layer, h // group]])
        want = ok.attention(q[:, h], k, v, every)
        fine = np.isfinite(want)
        assert (np.isfinite(got[:, h]) == fine).all(), "head %d" % h
        clean_k, clean_v = np.nan_to_num(k, posinf=0, neginf=0), np.nan_to_num(v, posinf=0, neginf=0)
        tol = np.broadcast_to(_tolerance(q[:, h], clean_k, clean_v, every)[:, None], want.shape)
        err = np.abs(np.where(fine, got[:, h] - want, 0))
        assert (err <= tol).all(), "head %d: %g over %g" % (h, err.max(), tol[np.unravel_index(err.argmax(), err.shape)])
        worst = max(worst, err.max())
    return got, worst


@pytest.mark.parametrize("fmt,hd", [("i8", 64), ("f8", 64), ("i8", 128), ("f8", 128)])
@pytest.mark.parametrize("len0,n,heads,group,kind", [
    (0, 1, 1, 1, "chain"), (0, 64, 2, 1, "tree"), (0, 5, 3, 1, "any"), (1, 1, 2, 1, "chain"), (31, 1, 2, 1, "tree"),
    (31, 64, 2, 1, "tree"), (32, 2, 3, 1, "chain"), (45, 16, 2, 1, "tree"), (64, 17, 1, 1, "any"), (127, 33, 2, 1, "tree"),
    (300, 8, 2, 4, "tree"), (97, 1, 2, 7, "chain"), (160, 11, 1, 3, "any"), (259, 64, 1, 2, "tree"), (70, 21, 2, 8, "tree"),
    (1537, 3, 3, 1, "tree"), (2048, 40, 1, 1, "tree")])
def test_attention(fmt, hd, len0, n, heads, group, kind):
    rng = np.random.default_rng(len0 + 7 * n + group)
    p = Pair(1, heads, hd, 32 * (len0 // 32 + 4), fmt)
    p.preset(rng, len0)
    got, worst = _check_attention(p, rng, n, group, kind)
    print("[kvq] %s hd %d len %d n %d x %d: worst error %.2g" % (fmt, hd, len0, n, group, worst), flush=True)
    if len0 == 0 and kind == "any":
        assert not got[::3].any()                     # rows that see nothing


@pytest.mark.parametrize("fmt,hd", [("i8", 128), ("f8", 64)])
@pytest.mark.parametrize("len0,n,heads", [(991, 64, 2), (1012, 60, 2), (1037, 2, 64), (1311, 50, 20)])
def test_tail_tiles_of_different_shares(fmt, hd, len0, n, heads):
    """Tail tiles 30..32 and 31..33, in groups of eight that go to different workgroups,
    and tails that follow a workgroup's first tiles."""
    rng = np.random.default_rng(len0)
    p = Pair(1, heads, hd, 32 * (len0 // 32 + 4), fmt)
    p.preset(rng, len0)
    _check_attention(p, rng, n, 1, "tree")


@pytest.mark.parametrize("fmt,hd,len0", [("i8", 64, 45), ("f8", 128, 300)])
def test_the_most_query_heads_of_a_kv_head(fmt, hd, len0):
    """65536 rows, 16 and 32 to a workgroup."""
    rng = np.random.default_rng(len0)
    p = Pair(1, 1, hd, 448, fmt)
    p.preset(rng, len0)
    _check_attention(p, rng, 64, 1024, "tree")


@pytest.mark.parametrize("fmt,hd", [("i8", 64), ("f8", 64), ("i8", 128), ("f8", 128)])
def test_attention_of_many_rows_over_a_long_cache(fmt, hd):
    """32 rows a workgroup (more than 12 tiles a wave), random codes."""
    rng = np.random.default_rng(18)
    heads, n, length = 16, 61, 14005
    g = D.DeviceKVQ(1, heads, hd, 14112, fmt)
    for t in (g.k, g.v):
        codes = rng.integers(-127, 128, t.shape, dtype=np.int8) if fmt == "i8" else ok.e4m3_code(
            rng.normal(0, 100, t.shape).clip(-448, 448)).view(np.int8)
        t.copy_(torch.from_numpy(codes))
    g.scale.copy_(torch.from_numpy(np.exp(rng.normal(-4 if fmt == "i8" else -5, 0.7, g.scale.shape))))
    g.k_tail.normal_()
    g.v_tail.normal_()
    g.c.len = length
    q = rng.normal(0, 1.4, (n, heads, hd)).astype(np.float32)
    mask, sees = _sees(rng, n, "tree")
    qd = torch.from_numpy(q).to(DEV)
    ws = torch.full((dv.dv_kvq_attention_workspace(g.c, n, heads) // 4,), float("nan"), device=DEV)
    dv.dv_kvq_attention(g.c, 0, qd.data_ptr(), heads * hd, n, heads, mask, qd.data_ptr(), heads * hd, ws.data_ptr(), ws.nbytes)
    torch.cuda.synchronize()
    got = qd.double().cpu().numpy()                   # (out may be q)
    k, v = _oracle_kv(g, 1, heads)[0]
    every = np.concatenate([np.ones((n, length), bool), sees], axis=1)
    r = length % 32
    for h in (0, 7, 15):
        kh = np.concatenate([k[h], g.k_tail[0, h, r:r + n].double().cpu().numpy()])
        vt = g.v_tail[0, h].transpose(1, 2).reshape(96, hd)
        vh = np.concatenate([v[h], vt[r:r + n].double().cpu().numpy()])
        qh = q[:, h].astype(np.float64)
        want = ok.attention(qh, kh, vh, every)
        err, tol = np.abs(got[:, h] - want), _tolerance(qh, kh, vh, every)[:, None]
        assert (err <= tol).all(), "head %d: %g" % (h, err.max())
        print("[kvq] %s hd %d head %d: worst error %.2g" % (fmt, hd, h, err.max()), flush=True)


@pytest.mark.parametrize("fmt", ["i8", "f8"])
def test_attention_strides_and_layers(fmt):
    rng = np.random.default_rng(11)
    p = Pair(3, 2, 128, 160, fmt)
    p.preset(rng, 75)
    for layer in range(3):
        _check_attention(p, rng, 9, 2, "tree", layer=layer, pad_q=12, pad_o=4)


def test_attention_long_and_one_row():
    rng = np.random.default_rng(12)
    p = Pair(1, 1, 128, 20032, "i8")
    p.preset(rng, 19999)
    _check_attention(p, rng, 1, 1, "chain")


def test_hidden_rows_may_hold_anything():
    """Infinite and NaN keys and values of new rows count only for the rows that see
    them."""
    rng = np.random.default_rng(13)
    for fmt, len0 in (("i8", 50), ("f8", 0)):
        p = Pair(1, 2, 64, 192, fmt)
        p.preset(rng, len0)
        n = 40
        new = {w: _rows(rng, (1, 2, n, 64)) for w in "kv"}
        new["v"][0, :, 7, 5], new["v"][0, :, 8], new["v"][0, 1, 39, 63] = np.inf, np.nan, -np.inf
        new["k"][0, :, 20, 3] = np.nan
        with np.errstate(invalid="ignore"):
            got, _ = _check_attention(p, rng, n, 1, "tree", new=new)
        assert np.isfinite(got).any() and not np.isfinite(got).all()


def test_a_block_without_a_scale_gives_nan():
    rng = np.random.default_rng(14)
    p = Pair(1, 2, 64, 192, "i8")
    rows = {w: _rows(rng, (1, 2, 100, 64)) for w in "kv"}
    rows["v"][0, 1, 40, 3] = np.inf
    kv = _kv(p, 192, rows)
    dv.dv_kvq_store(p.g.c, kv.c, 100)
    p.append(rows)
    p.put({w: _rows(rng, (1, 2, 3, 64)) for w in "kv"}, 4)
    got = _attend(p, rng.normal(size=(3, 2, 64)), 3, 2, None)
    assert np.isfinite(got[:, 0]).all() and np.isnan(got[:, 1]).all()


def test_large_scores():
    """Peaked and shifted scores: one key takes all, and none overflows."""
    rng = np.random.default_rng(15)
    p = Pair(1, 2, 64, 128, "f8")
    p.preset(rng, 90)
    for size in (1e-30, 60.0, 3000.0):
        _check_attention(p, rng, 6, 1, "tree", q=rng.normal(0, size, (6, 2, 64)).astype(np.float32).astype(np.float64))


def test_values_of_any_size():
    """Tiny and huge values side by side: nothing overflows on the way."""
    rng = np.random.default_rng(19)
    for fmt in ("i8", "f8"):
        for old, new in ((2.0 ** -97, 300.0), (2.0 ** -97, 2.0 ** 118), (2.0 ** 110, 2.0 ** -60), (2.0 ** 118, 2.0 ** 118), (0.0, 1.0)):
            p = Pair(1, 2, 64, 192, fmt)
            rows = {"k": _rows(rng, (1, 2, 70, 64)), "v": ov.round_to_bf16(rng.normal(0, 1, (1, 2, 70, 64)) * old)}
            kv = _kv(p, 192, rows)
            dv.dv_kvq_store(p.g.c, kv.c, 70)
            p.append(rows)
            fresh = {"k": _rows(rng, (1, 2, 5, 64)), "v": ov.round_to_bf16(rng.normal(0, 1, (1, 2, 5, 64)) * new)}
            got, _ = _check_attention(p, rng, 5, 1, "tree", new=fresh)
            assert np.isfinite(got).all()


def test_offsets_past_32_bits():
    """The last layer and head of a cache whose codes and tail lie beyond 4 GiB."""
    nl, nh, hd, cap, n = 9, 64, 128, 65536, 3
    need = 2 * nl * nh * cap * hd
    if torch.cuda.mem_get_info()[0] < 2 * need:
        pytest.skip("needs %d GiB" % (2 * need >> 30))
    big, small = D.DeviceKVQ(1, 1, 64, 32, "i8"), D.DeviceKVQ(1, nh, hd, cap, "i8")
    big.k = torch.empty((nl, nh, cap // 32, 32 * hd), dtype=torch.int8, device=DEV)
    big.v = torch.empty_like(big.k)
    big.scale = torch.empty((nl, nh, cap // 32, 2), device=DEV)
    big.k_tail = torch.empty((nl, nh, 96, hd), dtype=torch.bfloat16, device=DEV)
    big.v_tail = torch.empty((nl, nh, 3, hd, 32), dtype=torch.bfloat16, device=DEV)
    assert big.k.nbytes > 1 << 32
    g = torch.Generator(device=DEV).manual_seed(1)
    for t in (small.k, small.v):
        t.random_(-127, 128, generator=g)
    small.scale.uniform_(0.01, 0.02, generator=g)
    small.k_tail.normal_(generator=g)
    small.v_tail.normal_(generator=g)
    for name in ("k", "v", "scale", "k_tail", "v_tail"):
        getattr(big, name)[nl - 1].copy_(getattr(small, name)[0])
    big.c = dv.dv_kvq(big.k.data_ptr(), big.v.data_ptr(), big.scale.data_ptr(), big.k_tail.data_ptr(), big.v_tail.data_ptr(),
                      nl, nh, hd, dv.DV_I8, cap, cap - 20)
    small.c.len = cap - 20
    q = torch.randn((n, nh * hd), device=DEV)
    outs = []
    for c, layer in ((big, nl - 1), (small, 0)):
        out = torch.empty_like(q)
        ws = torch.empty(dv.dv_kvq_attention_workspace(c.c, n, nh), dtype=torch.uint8, device=DEV)
        dv.dv_kvq_attention(c.c, layer, q.data_ptr(), nh * hd, n, nh, None, out.data_ptr(), nh * hd, ws.data_ptr(),
                            ws.numel())
        outs.append(out)
    torch.cuda.synchronize()
    assert torch.equal(*outs) and torch.isfinite(outs[0]).all()


def test_moves_past_32_bits():
    """Store, advance and read-back of the last layer where codes, rows and their products
    lie beyond 4 GiB: as a cache of that layer alone."""
    nl, nh, hd, cap = 9, 64, 128, 65536
    need = 6 * nl * nh * cap * hd
    if torch.cuda.mem_get_info()[0] < 2 * need:
        pytest.skip("needs %d GiB" % (2 * need >> 30))
    g = torch.Generator(device=DEV).manual_seed(2)
    done = []
    for layers in (1, nl):
        c = D.DeviceKVQ(1, 1, 64, 32, "f8")
        for name, shape, dt in (("k", (cap // 32, 32 * hd), torch.int8), ("v", (cap // 32, 32 * hd), torch.int8),
                                ("scale", (cap // 32, 2), torch.float32), ("k_tail", (96, hd), torch.bfloat16),
                                ("v_tail", (3, hd, 32), torch.bfloat16)):
            t = torch.empty((layers, nh) + shape, dtype=dt, device=DEV)
            if dt == torch.int8:
                t[-1].fill_(0x31)
            else:
                t[-1].normal_(generator=g.manual_seed(len(name)))
            setattr(c, name, t)
        c.c = dv.dv_kvq(c.k.data_ptr(), c.v.data_ptr(), c.scale.data_ptr(), c.k_tail.data_ptr(), c.v_tail.data_ptr(),
                        layers, nh, hd, dv.DV_F8, cap, cap - 150)
        k = torch.empty((layers, nh, cap, hd), dtype=torch.bfloat16, device=DEV)
        v = torch.empty((layers, nh, cap // 32, hd, 32), dtype=torch.bfloat16, device=DEV)
        for t, seed in ((k, 5), (v, 6)):
            t[-1].normal_(generator=g.manual_seed(seed))
        kv = dv.dv_kv(k.data_ptr(), v.data_ptr(), cap, cap)
        dv.dv_kvq_store(c.c, kv, 101)
        dv.dv_kvq_advance(c.c, list(range(3, 23)) + [40])
        codes = [getattr(c, name)[-1].clone() for name in ("k", "v", "scale", "k_tail", "v_tail")]
        dv.dv_kvq_load(c.c, kv)
        torch.cuda.synchronize()
        assert c.len == kv.len == cap - 28
        done.append(codes + [k[-1].clone(), v[-1].clone()])
        del c, k, v, t
        torch.cuda.empty_cache()
    assert (nl - 1) * nh * cap * hd >= 1 << 32       # (the last layer's first code)
    for a, b in zip(*done):
        assert torch.equal(a.view(torch.int8), b.view(torch.int8))


def test_streams_and_graphs():
    """On a stream of the caller's, and captured: every replay as the eager call, with
    other inputs in the same buffers and eager work in between."""
    rng = np.random.default_rng(16)
    p = Pair(1, 4, 128, 1024, "i8")
    rows = {w: _rows(rng, (1, 4, 700, 128)) for w in "kv"}
    kv = _kv(p, 1024, rows)
    n, nh = 5, 8
    q = torch.randn((n, nh * 128), device=DEV)
    need = dv.dv_kvq_attention_workspace(p.g.c, n, nh)
    outs, wss = [torch.zeros_like(q) for _ in range(2)], [torch.empty(need, dtype=torch.uint8, device=DEV) for _ in range(2)]
    s = torch.cuda.Stream()

    def call(i, stream):
        p.g.c.len = 0
        dv.dv_kvq_store(p.g.c, kv.c, 690, stream)
        dv.dv_kvq_advance(p.g.c, [1, 3, 4], stream)
        dv.dv_kvq_attention(p.g.c, 0, q.data_ptr(), nh * 128, n, nh, None, outs[i].data_ptr(), nh * 128, wss[i].data_ptr(),
                            need, stream)

    p.put({w: _rows(rng, (1, 4, 20, 128)) for w in "kv"}, 0)
    p.g.k_tail.nan_to_num_()
    p.g.v_tail.nan_to_num_()
    k_tail, v_tail = p.g.k_tail.clone(), p.g.v_tail.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(0, torch.cuda.current_stream().cuda_stream)
    for i in range(4):
        for t, u in ((p.g.k_tail, k_tail), (p.g.v_tail, v_tail)):
            t.copy_(u)
        q.normal_()
        kv.k[:, :, :700].normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        codes = p.g.k.clone()
        for t, u in ((p.g.k_tail, k_tail), (p.g.v_tail, v_tail)):
            t.copy_(u)
        torch.cuda.synchronize()
        call(1, s.cuda_stream if i % 2 else 0)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(codes, p.g.k) and torch.isfinite(outs[0]).all()


def test_results_repeat_bit_for_bit():
    rng = np.random.default_rng(17)
    p = Pair(1, 3, 128, 4096, "f8")
    p.preset(rng, 1800)
    p.put({w: _rows(rng, (1, 3, 6, 128)) for w in "kv"}, 1800 % 32)
    q = rng.normal(size=(6, 3, 128))
    first = _attend(p, q, 6, 3, None)
    for _ in range(3):
        np.testing.assert_array_equal(_attend(p, q, 6, 3, None), first)


# ---------------------------------------------------------------------------
# the handle's path

def _oracle_kv(g, n_layers, n_heads):
    """The cache as attention sees it, float64, from the GPU's bytes."""
    torch.cuda.synchronize()
    hd, b, r = g.c.head_dim, g.len // 32, g.len % 32
    fmt = "i8" if g.c.format == dv.DV_I8 else "f8"
    scale = g.scale.double().cpu().numpy()
    out = []
    for l in range(n_layers):
        kv = []
        for i, (codes, at) in enumerate(((g.k, ok.k_byte(hd)), (g.v, ok.v_byte(hd)))):
            x = ok.numbers(codes[l, :, :b].cpu().numpy().reshape(n_heads, b, -1)[..., at], fmt) * scale[l, :, :b, i, None, None]
            tail = g.k_tail[l] if i == 0 else g.v_tail[l].transpose(2, 3).reshape(n_heads, 96, hd)
            kv.append(np.concatenate([x.reshape(n_heads, b * 32, hd), tail[:, :r].double().cpu().numpy()], axis=1))
        out.append(tuple(kv))
    return out


@pytest.mark.parametrize("weights,fmt,d,heads,max_tree", [("bf16", "i8", 256, 4, 64), ("bf16", "f8", 512, 4, 16),
                                                         ("i8", "f8", 256, 4, 16), ("i8", "i8", 512, 4, 64)])
def test_prompt_steps_and_commits(weights, fmt, d, heads, max_tree):
    """A prompt, then rounds of step and commit, against the oracle's step on the cache's
    own bytes: the bar of the bf16 cache's steps (2e-2) on the logits."""
    cfg = small_cfg(n_layers=2, d_model=d, n_heads=heads, head_dim=d // heads, d_ffn=2 * d, vocab=512, weight_dtype=weights,
                    init_std=0.05)
    case = GpuCase(cfg, seed=21, capacity=512, max_tree=max_tree)
    try:
        om = case.w.oracle()
        rng = np.random.default_rng(22)
        g = D.DeviceKVQ(2, heads, d // heads, 512, fmt)
        for t in (g.scale, g.k_tail, g.v_tail):
            t.fill_(float("nan"))
        prompt = rng.integers(0, 512, 150)
        # the plain cache's prompt holds the same rows before they are quantised
        kv = case.new_kv()
        root_plain = dv.dv_prefill(case.h, prompt, kv.c)
        root = dv.dv_prefill_kvq(case.h, prompt, g.c)
        assert g.len == 150
        q = D.DeviceKVQ(2, heads, d // heads, 512, fmt)
        dv.dv_kvq_store(q.c, kv.c, 150)
        torch.cuda.synchronize()
        # (one chunk: its own keys enter as bf16, so the same kernels ran on the same numbers)
        assert root == root_plain and torch.equal(q.k[:, :, :4], g.k[:, :, :4]) and torch.equal(q.v[:, :, :4], g.v[:, :, :4])
        for i in range(6):
            n = int(rng.integers(1, max_tree + 1))
            toks, par = synth.random_tree(int(rng.integers(1 << 30)), n, 8, 512)
            toks[0] = root
            kv_o = _oracle_kv(g, 2, heads)
            logits = torch.full((n, 512), float("nan"), device=DEV)
            acc = dv.dv_verify_step_kvq(case.h, toks, par, g.c, logits.data_ptr())
            torch.cuda.synchronize()
            ref = ov.verify_step(om, kv_o, toks, par)
            ref["tokens"], ref["parents"] = np.asarray(toks), np.asarray(par)
            err, near = compare_step(acc, logits.cpu().numpy(), ref, 2e-2)
            print("[kvq] %s/%s round %d: len %d n %d, logits off by %.2g" % (weights, fmt, i, g.len, n, err), flush=True)
            # commit a path of our own through the tree, the deepest node's
            node = int(np.argmax(ov.tree_info(par).depth))
            path = [int(x) for x in ov.tree_info(par).ancestors[node]]
            acc.accept_len = len(path)
            for j, x in enumerate(path):
                acc.path[j] = x
            len0 = g.len
            new = {w: t.clone() for w, t in (("k", g.k_tail), ("v", g.v_tail))}
            dv.dv_kvq_commit(case.h, g.c, acc)
            torch.cuda.synchronize()
            assert g.len == len0 + len(path)
            if g.len // 32 == len0 // 32:             # rows moved up, nothing quantised
                src = torch.tensor(path, device=DEV) + len0 % 32
                dst = torch.arange(len0 % 32, g.len % 32, device=DEV)
                assert torch.equal(g.k_tail[:, :, dst], new["k"][:, :, src])
            root = acc.bonus_token
    finally:
        case.close()


def test_step_is_the_plain_step_while_all_rows_are_in_the_tail():
    """Up to 31 committed rows nothing is quantised: both caches hold the same numbers,
    and the logits differ by the attention kernels' rounding alone."""
    cfg = small_cfg(n_layers=2, d_model=256, n_heads=4, head_dim=64, d_ffn=512, vocab=512, weight_dtype="bf16", init_std=0.05)
    case = GpuCase(cfg, seed=23, capacity=128)
    try:
        kv, g = case.new_kv(), D.DeviceKVQ(2, 4, 64, 128, "i8")
        prompt = np.arange(20) * 7 % 512
        assert dv.dv_prefill(case.h, prompt, kv.c) == dv.dv_prefill_kvq(case.h, prompt, g.c)
        toks, par = synth.random_tree(3, 40, 8, 512)
        a, la = case.step(kv, toks, par)
        lb = torch.empty((40, 512), device=DEV)
        b = dv.dv_verify_step_kvq(case.h, toks, par, g.c, lb.data_ptr())
        torch.cuda.synchronize()
        # bf16 keys and values of layer 2 may round the other way (half a step, 2^-8), as
        # between any two orders of summation; the steps' own bar is 2e-2
        assert np.abs(la - lb.cpu().numpy()).max() <= 2e-2
    finally:
        case.close()


def test_a_prompt_of_two_chunks_and_a_turn_behind_it():
    """The second chunk and the next prompt read the cache back; against the oracle's
    prompt behind the cache's own bytes."""
    cfg = small_cfg(n_layers=2, d_model=256, n_heads=4, head_dim=64, d_ffn=512, vocab=512, weight_dtype="bf16", init_std=0.05)
    case = GpuCase(cfg, seed=24, capacity=1408, max_tree=16)
    try:
        g = D.DeviceKVQ(2, 4, 64, 1408, "i8")
        om = case.w.oracle()
        rng = np.random.default_rng(25)
        dv.dv_prefill_kvq(case.h, rng.integers(0, 512, 1100), g.c)
        assert g.len == 1100
        kv_o = _oracle_kv(g, 2, 4)
        turn = rng.integers(0, 512, 41)
        nxt = dv.dv_prefill_kvq(case.h, turn, g.c)
        assert g.len == 1141
        ref = ov.verify_step(om, kv_o, turn, np.arange(-1, 40))["logits"][-1]
        top = int(np.argmax(ref))
        # read back, rows are scale x code rounded to bf16: half a step, 2^-9 of a number
        assert nxt == top or ref[nxt] >= ref[top] - 4e-2
        got = _oracle_kv(g, 2, 4)
        np.testing.assert_array_equal(got[0][0][:, :1088], kv_o[0][0][:, :1088])   # whole blocks stay
    finally:
        case.close()


def test_sampled_step_over_the_8_bit_cache():
    """The rule on the step's own logits, as for the plain cache."""
    cfg = small_cfg(n_layers=1, d_model=256, n_heads=4, head_dim=64, d_ffn=512, vocab=512, weight_dtype="bf16", init_std=0.05)
    case = GpuCase(cfg, seed=26, capacity=128)
    try:
        g = D.DeviceKVQ(1, 4, 64, 128, "f8")
        dv.dv_prefill_kvq(case.h, np.arange(45), g.c)
        toks, par = synth.random_tree(5, 12, 5, 512)
        q = torch.from_numpy(synth.draft_rows(6, 12, 512)).to(DEV)
        ua, ub = synth.sampling_uniforms(7, 12)
        logits = torch.empty((12, 512), device=DEV)
        acc = dv.dv_verify_step_kvq_sampled(case.h, toks, par, g.c, q.data_ptr(), 0.8, ua, ub, logits.data_ptr())
        rule = dv.dv_accept_sampled(case.h, logits.data_ptr(), toks, par, q.data_ptr(), 0.8, ua, ub)
        assert acc.path_list == rule.path_list and acc.bonus_token == rule.bonus_token and acc.base_len == 45
        dv.dv_kvq_commit(case.h, g.c, acc)
        assert g.len == 45 + acc.accept_len
    finally:
        case.close()
