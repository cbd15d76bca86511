"""Paged cache, host side: arguments that are refused before anything is looked up on the
device, frequencies, how the work is cut, and what the kernels make of the numbers in device
memory (their index functions compiled for the host): lengths, tables, paths that cannot be."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import paged as op
from paper_2412_18934_amd import dv
from tests.test_engine_cpu import CSRC, ROOT

A = 1 << 20  # an aligned address that is never used


def cache(**kw):
    f = dict(k=A, v=A, mass=A, table=A, lens=A, fault=A, n_layers=2, n_heads=4, head_dim=64, n_pages=9, page=64, n_seqs=3,
             table_stride=5)
    f.update(kw)
    return dv.dv_paged(*[f[name] for name, _ in dv.dv_paged._fields_])


def rows(**kw):
    f = dict(q=A, q_stride=512, start=A, mask=A, scale=0.0, cap=0.0, dtype=dv.DV_F32, n_heads=8, n_rows=7, max_rows=4, max_len=300)
    f.update(kw)
    return dv.dv_paged_rows(*[f[name] for name, _ in dv.dv_paged_rows._fields_])


def rope(**kw):
    f = dict(base=10000.0, factor=8.0, low=1.0, high=4.0, magnitude=1.0, original_ctx=4096, scaling=0, rot_dim=64, interleaved=0)
    f.update(kw)
    return dv.dv_rope(*f.values())


CALLS = dict(
    append=lambda c, r: dv.dv_paged_append(c, 1, r, dv.dv_rope_init(rope()), A, A, 256, A, 256),
    workspace=lambda c, r: dv.dv_paged_attention_workspace(c, r),
    attention=lambda c, r: dv.dv_paged_attention(c, 1, r, A, 512, A, A, 1 << 50),
    mass=lambda c, r: dv.dv_paged_mass(c, 1, r, A, A),
    commit=lambda c, r: dv.dv_paged_commit(c, A, 8, A, A),
    evict=lambda c, r: dv.dv_paged_evict(c, 100, 10, A))


def refused(call, *words):
    with pytest.raises(dv.DvError) as e:
        call()
    assert e.value.code == dv.DV_EINVAL and dv.dv_last_error(None)
    for w in words:
        assert w in str(e.value)


@pytest.mark.parametrize("name", ["dv_paged", "dv_paged_rows", "dv_rope"])
def test_the_structs_follow_the_header(name):
    from tests.test_abi_cpu import _header_fields
    assert [f[0] for f in getattr(dv, name)._fields_] == _header_fields(name)


@pytest.mark.parametrize("bad", [
    dict(k=None), dict(v=None), dict(table=None), dict(lens=None), dict(k=A + 8), dict(v=A + 2), dict(mass=A + 4), dict(table=A + 2),
    dict(lens=A + 1), dict(fault=A + 2), dict(n_layers=0), dict(n_heads=0), dict(n_heads=65536), dict(head_dim=96),
    dict(head_dim=256), dict(n_pages=0), dict(page=0), dict(page=16), dict(page=48), dict(page=-32), dict(n_seqs=0),
    dict(n_seqs=65537), dict(table_stride=0), dict(table_stride=(1 << 30) // 64 + 1), dict(n_pages=1 << 25, page=64),
    dict(n_layers=1 << 20)], ids=str)
@pytest.mark.parametrize("call", CALLS)
def test_bad_caches_are_refused_by_every_call(call, bad):
    refused(lambda: CALLS[call](cache(**bad), rows()))


@pytest.mark.parametrize("bad", [
    dict(dtype=dv.DV_I8), dict(dtype=-1), dict(n_rows=0), dict(n_rows=-3), dict(n_rows=(1 << 22) + 1), dict(start=None),
    dict(start=A + 2), dict(n_heads=0), dict(n_heads=6), dict(n_heads=4 * 1025, q_stride=1 << 20), dict(n_heads=65540), dict(q=A + 8),
    dict(q_stride=511), dict(q_stride=508), dict(q_stride=514), dict(q_stride=-512), dict(q_stride=1 << 41),
    dict(dtype=dv.DV_BF16, q_stride=516)], ids=str)
@pytest.mark.parametrize("call", ["append", "workspace", "attention", "mass"])
def test_bad_rows_are_refused(call, bad):
    refused(lambda: CALLS[call](cache(), rows(**bad)))


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(mask=A + 4), dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("inf")),
    dict(cap=float("nan")), dict(max_rows=0), dict(max_rows=65), dict(max_len=-1), dict(max_len=(1 << 30) + 1)], ids=str)
@pytest.mark.parametrize("call", ["workspace", "attention", "mass"])
def test_bad_scores_are_refused(call, bad):
    refused(lambda: CALLS[call](cache(), rows(**bad)))


def test_null_structs_are_refused():
    L = dv.lib()
    assert L.dv_paged_attention(None, 0, rows(), A, 512, None, None, 0, None) == dv.DV_EINVAL
    assert L.dv_paged_attention(cache(), 0, None, A, 512, None, None, 0, None) == dv.DV_EINVAL
    assert L.dv_paged_append(cache(), 0, None, None, None, A, 256, A, 256, None) == dv.DV_EINVAL
    assert L.dv_paged_mass(cache(), 0, None, A, None, None) == dv.DV_EINVAL
    assert L.dv_paged_commit(None, None, 0, A, A, None) == dv.DV_EINVAL
    assert L.dv_paged_evict(None, 1, 0, A, None) == dv.DV_EINVAL
    assert L.dv_rope_init(None) == dv.DV_EINVAL


@pytest.mark.parametrize("layer", [-1, 2])
def test_layers_outside_are_refused(layer):
    refused(lambda: dv.dv_paged_append(cache(), layer, rows(), None, 0, A, 256, A, 256), "layer")
    refused(lambda: dv.dv_paged_attention(cache(), layer, rows(), A, 512, A, A, 1 << 50), "layer")
    refused(lambda: dv.dv_paged_mass(cache(), layer, rows(), A), "layer")


@pytest.mark.parametrize("k,ks,v,vs,pos", [(0, 256, A, 256, A), (A, 256, 0, 256, A), (A + 8, 256, A, 256, A), (A, 256, A + 4, 256, A),
                                           (A, 255, A, 256, A), (A, 256, A, 252, A), (A, 258, A, 256, A), (A, 256, A, 256, A + 2)])
def test_append_refusals(k, ks, v, vs, pos):
    refused(lambda: dv.dv_paged_append(cache(), 0, rows(), None, pos, k, ks, v, vs))


def test_append_needs_a_fitting_rope():
    r = dv.dv_rope_init(rope(rot_dim=128))
    refused(lambda: dv.dv_paged_append(cache(), 0, rows(), r, A, A, 256, A, 256), "rot_dim")
    for bad in (dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=-2), dict(magnitude=0.0), dict(magnitude=float("nan"))):
        refused(lambda: dv.dv_paged_append(cache(), 0, rows(), rope(**bad), A, A, 256, A, 256))


@pytest.mark.parametrize("out,stride,stats,ws,size", [(0, 512, A, A, 1 << 50), (A + 4, 512, A, A, 1 << 50), (A, 500, A, A, 1 << 50),
                                                      (A, 513, A, A, 1 << 50), (A, 512, A + 4, A, 1 << 50), (A, 1024, A, A, 1 << 50)])
def test_attention_refusals(out, stride, stats, ws, size):
    """(the last: in place of the queries with another stride)"""
    refused(lambda: dv.dv_paged_attention(cache(), 0, rows(), out, stride, stats, ws, size))


def test_mass_and_eviction_refusals():
    refused(lambda: dv.dv_paged_mass(cache(mass=None), 0, rows(), A), "mass")
    refused(lambda: dv.dv_paged_mass(cache(), 0, rows(), 0))
    refused(lambda: dv.dv_paged_mass(cache(), 0, rows(), A + 4))
    refused(lambda: dv.dv_paged_mass(cache(), 0, rows(), A, A + 4))
    refused(lambda: dv.dv_paged_evict(cache(mass=None), 5, 1, A), "mass")
    for budget, recent in ((0, 0), (-1, 0), (5, 6), (5, -1)):
        refused(lambda: dv.dv_paged_evict(cache(), budget, recent, A))
    refused(lambda: dv.dv_paged_evict(cache(), 5, 1, 0))
    refused(lambda: dv.dv_paged_evict(cache(), 5, 1, A + 2))
    refused(lambda: dv.dv_paged_evict(cache(table_stride=4097), 5, 1, A), "262144")


def test_commit_refusals():
    for path, stride, n, lens in ((A, 8, 0, A), (A, 8, A, 0), (A + 2, 8, A, A), (A, 8, A + 1, A), (A, 8, A, A + 2), (A, 0, A, A),
                                  (A, -1, A, A), (A, 1 << 41, A, A)):
        refused(lambda: dv.dv_paged_commit(cache(), path, stride, n, lens))


@pytest.mark.parametrize("bad", [
    dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=130), dict(rot_dim=-2), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")),
    dict(magnitude=0.0), dict(magnitude=-1.0), dict(magnitude=1e300), dict(scaling=-1), dict(scaling=4), dict(scaling=1, factor=0.5),
    dict(scaling=1, factor=float("nan")), dict(scaling=1, factor=float("inf")), dict(scaling=2, low=0.0), dict(scaling=2, low=4.0),
    dict(scaling=3, high=float("inf")), dict(scaling=3, original_ctx=0), dict(scaling=2, factor=0.0)], ids=str)
def test_rope_refusals(bad):
    refused(lambda: dv.dv_rope_init(rope(**bad)))


@pytest.mark.parametrize("kw", [dict(), dict(rot_dim=2), dict(rot_dim=128, base=500000.0), dict(scaling=1, factor=3.0),
                                dict(scaling=2), dict(scaling=3, high=32.0, rot_dim=96), dict(scaling=2, factor=1.0)], ids=str)
def test_rope_frequencies(kw):
    r = rope(**kw)
    r.freq[r.rot_dim // 2 if r.rot_dim < 128 else 0] = 7.5
    dv.dv_rope_init(r)
    want = op.frequencies(r.rot_dim, r.base, r.scaling, r.factor, r.low, r.high, r.original_ctx)
    # pow, log and a blend of two: a few steps of 2^-53, of the exponent's too (ln 10^4.. times 2^-53)
    np.testing.assert_allclose(list(r.freq)[:r.rot_dim // 2], want, rtol=64 * 2.0 ** -53)
    if r.rot_dim < 128:
        assert r.freq[r.rot_dim // 2] == 7.5          # nothing is written behind them


# ---------------------------------------------------------------------------
# the kernels' index functions, on the host

STUB = r"""
#include "dv_paged_index.h"
extern "C" {
static PagedView view(int n_seqs, int width, int page, int n_pages, int H, const int32_t *table, const int32_t *lens)
{
    PagedView c{};
    c.table = table, c.lens = lens, c.n_pages = n_pages, c.page = page, c.H = H, c.n_seqs = n_seqs, c.width = width;
    return c;
}
int t_seq(int width, int page, const int32_t *lens, const int32_t *start, int n_rows, int s, int most, int *out)
{
    bool bad = false;
    const Seq q = seq_of(view(1, width, page, 1, 1, nullptr, lens), start, n_rows, s, most, bad);
    out[0] = q.first, out[1] = q.n, out[2] = q.len;
    return bad;
}
uint32_t t_row(int width, int page, int n_pages, int H, const int32_t *table, int s, int h, int slot, int *bad)
{
    bool b = false;
    const uint32_t r = row_of(view(1, width, page, n_pages, H, table, nullptr), s, h, slot, b);
    *bad = b;
    return r;
}
int t_size(int64_t units, int64_t tiles, int most, int least) { return piece_size(units, tiles, most, least); }
int t_pieces(int tiles, int size) { return pieces_of(tiles, size); }
int t_start(int tiles, int pieces, int i) { return piece_start(tiles, pieces, i); }
int t_commit(int width, int page, int len, const int32_t *path, int64_t stride, int n, const int32_t *at)
{
    const int32_t lens[1] = {len}, ns[1] = {n};
    PagedMoveArgs a{};
    a.c = view(1, width, page, 1, 1, nullptr, lens), a.path = path, a.path_len = ns, a.path_stride = stride;
    if (!commit_fits(a, 0)) return 0;
    for (int i = 0; path && i < n; ++i)
        if (!path_ok(a, 0, i, n)) return 0;
    return 1;
}
uint32_t t_rank(float m) { return rank_of(m); }
void t_cut(int seqs, int heads, int group, int n_rows, int rows, int len, int cu, int64_t *out)
{
    const PagedCut c = paged_cut(seqs, heads, group, n_rows, rows, len, cu);
    out[0] = c.rt, out[1] = c.blocks, out[2] = c.groups, out[3] = c.whole, out[4] = (int64_t)paged_attention_bytes(c, seqs, 128);
    out[5] = c.grid, out[6] = paged_mass_cut(seqs, heads, len, cu).grid;
}
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged")
    stub, out = str(d / "stub.cpp"), str(d / "libpaged.so")
    with open(stub, "w") as f:
        f.write(STUB)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover",
                    "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", CSRC, stub,
                    "-o", out], check=True)
    L = ctypes.CDLL(out)
    i64 = ctypes.c_int64
    L.t_size.argtypes = [i64, i64, ctypes.c_int, ctypes.c_int]
    L.t_row.restype = L.t_rank.restype = ctypes.c_uint32
    L.t_rank.argtypes = [ctypes.c_float]
    L.t_commit.argtypes = [ctypes.c_int] * 3 + [ctypes.c_void_p, i64, ctypes.c_int, ctypes.c_void_p]
    return L


def _ints(*x):
    return (ctypes.c_int32 * len(x))(*x)


BIG = 2 ** 31 - 1


@pytest.mark.parametrize("length,start,n_rows,ok", [
    (0, (0, 1), 1, True), (10, (2, 66), 70, True), (10, (3, 3), 7, True), (-5, (3, 3), 7, True), (63, (0, 64), 64, True),
    (96, (0, 64), 64, True), (97, (0, 64), 64, False), (160, (0, 1), 1, False), (-1, (0, 1), 1, False), (BIG, (0, 64), 64, False),
    (0, (0, 65), 70, False), (0, (1, 0), 4, False), (0, (-1, 2), 4, False), (0, (0, 5), 4, False), (0, (BIG, -BIG), 4, False),
    (0, (-BIG, BIG), 4, False), (-2 ** 31, (0, 3), 4, False), (0, (-2, -1), 4, False)])
def test_sequences_that_cannot_be_are_skipped(lib, length, start, n_rows, ok):
    out = (ctypes.c_int * 3)()
    bad = lib.t_seq(5, 32, _ints(length), _ints(*start), n_rows, 0, 64, out)
    assert bad == (not ok)
    assert out[1] == (start[1] - start[0] if ok else 0)
    if out[1]:
        assert 0 <= out[0] and out[0] + out[1] <= n_rows and 0 <= out[2] and out[2] + out[1] <= 5 * 32


def test_pages_outside_the_pool_are_no_rows(lib):
    table, bad = _ints(3, -1, 8, 9, BIG, -2 ** 31), ctypes.c_int()
    for slot in range(6 * 96):
        for h in (0, 4):
            r = lib.t_row(6, 96, 9, 5, table, 0, h, slot, ctypes.byref(bad))
            p = table[slot // 96]
            if 0 <= p < 9:
                assert not bad.value and r == (p * 5 + h) * 96 + slot % 96 < 9 * 5 * 96
            else:
                assert bad.value and r == 2 ** 32 - 1
    # the last row of the largest pool, behind 2^31
    r = lib.t_row(1, 1 << 20, 4095, 1, _ints(4094), 0, 0, (1 << 20) - 1, ctypes.byref(bad))
    assert r == 4095 * 2 ** 20 - 1


@pytest.mark.parametrize("most", [1, 5, 256, 1000, 1 << 20])
def test_pieces_fit_and_cover_their_unit(lib, most):
    """No more pieces than room for their sums, whatever the lengths; each unit's are whole, even and not empty."""
    rng = np.random.default_rng(most)
    for trial in range(200):
        seqs = int(rng.integers(1, 40))
        units = rng.integers(0, 50, seqs) * (rng.random(seqs) < 0.9)
        tiles = np.maximum(1, (2.0 ** rng.uniform(0, rng.choice([3, 10, 25]), seqs)).astype(np.int64))
        size = lib.t_size(int(units.sum()), int((units * tiles).sum()), most, 4)
        n = [lib.t_pieces(int(t), size) for t in tiles]
        total = sum(int(u) * p for u, p in zip(units, n))
        assert total <= max(most, int(units.sum()))
        if units.sum() >= most:
            assert set(n) == {1}
        for t, p in zip(tiles.tolist(), n):
            at = [lib.t_start(t, p, i) for i in {0, 1, p // 2, p - 1, p} if i <= p]
            assert lib.t_start(t, p, 0) == 0 and lib.t_start(t, p, p) == t and 1 <= p <= t and len(at)
            for i in (0, p // 2, p - 1):
                assert 0 < lib.t_start(t, p, i + 1) - lib.t_start(t, p, i) <= max(size, 1)


@pytest.mark.parametrize("length,path,n,ok", [
    (10, (0, 2, 5), 3, True), (10, (0, 2, 5), 0, True), (10, (63,), 1, True), (100, (63,), 1, False), (96, (63,), 1, True),
    (10, (0, 0), 2, False), (10, (2, 1), 2, False), (10, (-1, 1), 2, False), (10, (0, 64), 2, False), (10, (0, 1), -1, False),
    (10, (0, 1), 3, False), (-1, (0,), 1, False), (BIG, (0,), 1, False), (160, (), 0, True), (160, (0,), 1, False)])
def test_paths_that_cannot_be_are_skipped(lib, length, path, n, ok):
    """(n above the stride too: what lies behind the row is another's)"""
    p = _ints(*path, 0)
    assert lib.t_commit(5, 32, length, p, max(len(path), 1), n, None) == ok


@pytest.mark.parametrize("length,n,ok", [(0, 160, True), (1, 160, False), (100, BIG, False), (10, -1, False), (-1, 5, False)])
def test_lengths_without_a_path(lib, length, n, ok):
    assert lib.t_commit(5, 32, length, None, 0, n, None) == ok


def test_ranks_order_masses(lib):
    x = [-np.inf, -3e38, -1.0, -1e-45, 0.0, 1e-45, 1e-38, 0.5, 1.0, 3e38, np.inf]
    r = [lib.t_rank(v) for v in x]
    assert r == sorted(set(r)) and r[0] > 0 and lib.t_rank(-0.0) == lib.t_rank(0.0)
    assert lib.t_rank(float("nan")) == lib.t_rank(-float("nan")) == 2 ** 32 - 1 > r[-1]


@pytest.mark.parametrize("cu", [256, 64])
def test_every_row_block_has_a_workgroup(lib, cu):
    """Also where the sequences have more rows than max_rows says."""
    out, rng = (ctypes.c_int64 * 7)(), np.random.default_rng(0)
    for seqs in (1, 3, 48, 6000):
        for heads in (1, 8, 40):
            for group in (1, 4, 1024):
                for n in (1, 16, 64):
                    for length in (0, 1, 500, 1500, 4100, 1 << 30):
                        rows = rng.integers(0, 65, seqs)
                        rows[0] = max(rows[0], 1)
                        lib.t_cut(seqs, heads, group, int(rows.sum()), n, length, cu, out)
                        rt, blocks, groups, whole, size, grid, mass = out
                        assert 16 * rt * blocks >= n * group > 16 * rt * (blocks - 1)
                        assert whole == (groups == 0) == (size == 0)
                        units = heads * int((-(-rows * group // (16 * rt))).sum())
                        assert grid >= max(units, groups) and mass >= seqs * heads
                        assert whole or 2 * cu <= groups < 18 * cu and size == groups * 16 * rt * 130 * 4 + 8 * seqs
