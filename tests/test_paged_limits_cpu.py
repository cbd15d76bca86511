"""Paged cache, host side: the largest numbers that the calls take, and what lies just behind them."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2412_18934_amd import device, dv
from tests.test_engine_cpu import CSRC, ROOT
from tests.test_paged_cpu import A, CALLS, cache, lib, refused, rope, rows  # noqa: F401 (lib: a fixture)


@pytest.mark.parametrize("units,most,tiles", [(768, 774, 1 << 25), (1, 2, 1 << 25), (1000, 1001, 1 << 25), (896, 897, 9586981)])
def test_pieces_of_the_longest_sequences(lib, units, most, tiles):  # noqa: F811
    """Hardly more pieces than units, each of up to 2^25 tiles (2^30 slots): a piece's size is a number of more than
    32 bits there, of which the low ones alone would be 0, or little."""
    size = lib.t_size(units, units * tiles, most, 4)
    assert size >= 4
    n = lib.t_pieces(tiles, size)
    assert 1 <= n and units * n <= most
    assert lib.t_start(tiles, n, 0) == 0 and lib.t_start(tiles, n, n) == tiles


def test_pieces_fit_where_sizes_are_large(lib):  # noqa: F811
    rng = np.random.default_rng(1)
    for _ in range(2000):
        units = int(rng.integers(1, 4000))
        most = units + int(2.0 ** rng.uniform(0, 11))
        tiles = int(2.0 ** rng.uniform(18, 25))
        size = lib.t_size(units, units * tiles, most, 4)
        assert size >= 4 and units * lib.t_pieces(tiles, size) <= most


# What is refused last shows that all before it was taken: nothing here is launched.
LAST = dict(
    append=lambda c: refused(lambda: dv.dv_paged_append(c, 0, rows(n_heads=c.n_heads, q_stride=1 << 24), rope(magnitude=-1.0), 0,
                                                        A, 1 << 24, A, 1 << 24), "magnitude"),
    attention=lambda c: refused(lambda: dv.dv_paged_attention(c, 0, rows(n_heads=c.n_heads, q_stride=1 << 24), 0, 1 << 24), "outputs"),
    mass=lambda c: refused(lambda: dv.dv_paged_mass(c, 0, rows(n_heads=c.n_heads, q_stride=1 << 24), 0), "stats"),
    commit=lambda c: refused(lambda: dv.dv_paged_commit(c, A, 0, A, A), "path stride"),
    evict=lambda c: refused(lambda: dv.dv_paged_evict(c, 0, 0, A), "budget"))


@pytest.mark.parametrize("call", LAST)
@pytest.mark.parametrize("kw", [dict(n_layers=32, n_heads=8, n_seqs=65536, table_stride=1), dict(n_layers=65535, n_heads=1, n_seqs=65536),
                                dict(n_layers=65535, n_heads=63, n_seqs=65536), dict(n_layers=80, n_heads=65535, n_seqs=64)], ids=str)
def test_many_layers_of_many_sequences_are_taken(call, kw):
    """n_layers up to 65535, n_heads n_seqs below 2^22, as the header says; not their product."""
    LAST[call](cache(**kw))


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw", [dict(n_layers=65536), dict(n_heads=64, n_seqs=65536), dict(n_heads=65535, n_seqs=65)], ids=str)
def test_more_are_refused(call, kw):
    refused(lambda: CALLS[call](cache(**kw), rows(n_heads=kw.get("n_heads", 4), q_stride=1 << 24)))


@pytest.mark.parametrize("n_rows,heads,ok", [(1 << 22, 64, True), (4096, 65535, True), (1 << 22, 65, False), (4097, 65535, False)])
def test_the_most_rows_of_an_append(n_rows, heads, ok):
    """n_rows n_heads up to 2^28."""
    c, r = cache(n_heads=heads), rows(n_rows=n_rows, n_heads=heads, q_stride=1 << 24)
    words = "magnitude" if ok else "too many"
    refused(lambda: dv.dv_paged_append(c, 0, r, rope(magnitude=-1.0), 0, A, 1 << 24, A, 1 << 24), words)


def test_attention_needs_no_more_workgroups_than_a_grid_has(lib):  # noqa: F811
    """Whatever the sequences, heads and rows: grids of 2^24 workgroups of 256 at most, 65535 in the other dimension."""
    out = (ctypes.c_int64 * 7)()
    for cu in (1, 64, 256, 512):
        for seqs in (1, 2, 1000, 1024, 1025, 65536):
            for heads in (1, 7, 63, 4096, 65535):
                if seqs * heads >= 1 << 22:
                    continue
                for group in (1, 2, 15, 16, 17, 1024):
                    for n in (1, 2, 16, 63, 64):
                        for length in (0, 2000, 1 << 30):
                            lib.t_cut(seqs, heads, group, min(seqs * 64, 1 << 22), n, length, cu, out)
                            rt, blocks, groups, whole, size, grid, mass = out
                            assert blocks <= 65535 and mass < 1 << 24
                            assert whole or (grid + 1 < 1 << 24 and seqs * heads < 1 << 24)


@pytest.mark.parametrize("change", [
    dict(q=torch.float16), dict(q=torch.float64), dict(q=torch.int32), dict(start=torch.int64), dict(start=torch.uint8), dict(mask=torch.int32),
    dict(mask=torch.float64), dict(mask=torch.bool)], ids=str)
def test_rows_of_other_types_are_refused(change):
    """By the class that makes the struct of tensors: their addresses alone would be read as the types that the call knows."""
    g = device.DevicePaged(1, 2, 64, 3, 32, 2, 1, device="cpu")
    t = dict(q=torch.zeros((3, 4, 64)), start=torch.zeros(3, dtype=torch.int32), mask=torch.zeros(3, dtype=torch.int64))
    for dtype in (torch.float32, torch.bfloat16):
        assert g.rows(**dict(t, q=t["q"].to(dtype))).dtype == (dv.DV_F32 if dtype == torch.float32 else dv.DV_BF16)
    g.rows(**dict(t, mask=t["mask"].to(torch.uint64)))
    g.rows(t["q"][:2])
    with pytest.raises(TypeError):
        g.rows(**dict(t, **{name: t[name].to(dtype) for name, dtype in change.items()}))


@pytest.mark.parametrize("change", [
    lambda t: dict(q=t["q"][0]), lambda t: dict(q=t["q"][:, :, :32]), lambda t: dict(q=torch.zeros((3, 64, 4)).transpose(1, 2)),
    lambda t: dict(q=torch.zeros((3, 8, 64))[:, ::2]), lambda t: dict(start=t["start"][:2]), lambda t: dict(start=None),
    lambda t: dict(start=torch.zeros(6, dtype=torch.int32)[::2]), lambda t: dict(mask=t["mask"][:2]),
    lambda t: dict(mask=torch.zeros(6, dtype=torch.int64)[::2]), lambda t: dict(q=t["q"].to("meta"))])
def test_rows_of_other_shapes_are_refused(change):
    """Heads and dims stand behind one another; start and mask have an entry for each sequence and row."""
    g = device.DevicePaged(1, 2, 64, 3, 32, 2, 1, device="cpu")
    t = dict(q=torch.zeros((3, 4, 64)), start=torch.zeros(3, dtype=torch.int32), mask=torch.zeros(3, dtype=torch.int64))
    wide = g.rows(**dict(t, q=torch.zeros((3, 9, 64))[:, 2:6]))
    assert (wide.q_stride, wide.n_heads, wide.n_rows) == (9 * 64, 4, 3)
    assert g.rows(**dict(t, q=torch.zeros((3, 2, 64)).expand(3, 2, 64)[:, :1])).n_heads == 1
    with pytest.raises(ValueError):
        g.rows(**dict(t, **change(t)))


STUB = r"""
#include "dv_paged_index.h"
extern "C" int t_from(const int32_t *start, int n_seqs, int s, int row) { return seq_from(start, n_seqs, s, row); }
"""


@pytest.fixture(scope="module")
def search(tmp_path_factory):
    d = tmp_path_factory.mktemp("search")
    stub, out = str(d / "stub.cpp"), str(d / "libsearch.so")
    with open(stub, "w") as f:
        f.write(STUB)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover",
                    "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", CSRC, stub,
                    "-o", out], check=True)
    return ctypes.CDLL(out).t_from


@pytest.mark.parametrize("seqs", [1, 2, 3, 63, 64, 65, 1000, 65536])
def test_the_sequence_of_a_row(search, seqs):
    """Runs of empty sequences of all lengths, rows before the first and behind the last; whatever sequence the search begins at."""
    rng = np.random.default_rng(seqs)
    for empty in (0.0, 0.5, 0.99, 1.0):
        counts = np.where(rng.random(seqs) < empty, 0, rng.integers(0, 9, seqs))
        start = np.concatenate([[2], 2 + np.cumsum(counts)]).astype(np.int32)
        p = start.ctypes.data_as(ctypes.c_void_p)
        rows_ = np.unique(np.concatenate([rng.integers(0, start[-1] + 2, 50), start[rng.integers(0, seqs + 1, 20)], [0, start[-1], start[-1] + 1]]))
        for row in rows_.tolist():
            want = int((start[1:] <= row).sum())
            for s in {0, want, max(want - 1, 0), int(rng.integers(0, want + 1))}:
                assert search(p, seqs, s, row) == want


def test_starts_that_decrease_lead_nowhere_else(search):
    rng = np.random.default_rng(5)
    for _ in range(300):
        seqs = int(rng.integers(1, 200))
        start = rng.integers(-2 ** 31, 2 ** 31 - 1, seqs + 1).astype(np.int32)
        s = int(rng.integers(0, seqs + 1))
        assert s <= search(start.ctypes.data_as(ctypes.c_void_p), seqs, s, int(rng.integers(0, 1 << 22))) <= seqs


@pytest.mark.parametrize("low,high", [(1e-320, 1.0), (5e-324, 1e-300), (1e-300, 1e300), (1e-310, 1e308), (1.0, 1.0 + 2.0 ** -52),
                                      (np.nextafter(2.0, 0), 2.0), (np.nextafter(2.0, 0) * 2.0 ** 9, 2.0 ** 10)], ids=str)
@pytest.mark.parametrize("scaling", [dv.DV_ROPE_TURNS, dv.DV_ROPE_LOG_TURNS])
def test_frequencies_between_bounds_of_all_sizes(low, high, scaling):
    """Every pair's is between f / factor and f, whose turns are past the bounds at one of them; also between bounds that a
    quotient cannot hold, or the logarithm not tell apart."""
    r = rope(scaling=scaling, low=float(low), high=float(high), original_ctx=2 ** 30)
    f = np.array([r.base ** (-2 * i / 64) for i in range(32)])
    dv.dv_rope_init(r)
    got, t = np.array(list(r.freq)[:32]), 2 ** 30 * f / (2 * math.pi)
    assert np.isfinite(got).all()
    assert (got >= f / 8 * (1 - 1e-14)).all() and (got <= f * (1 + 1e-14)).all()
    np.testing.assert_allclose(got[t >= high], f[t >= high], rtol=1e-14)
    np.testing.assert_allclose(got[t <= low], f[t <= low] / 8, rtol=1e-14)
