"""8-bit cache, host side: arguments that are refused (before anything is looked up
on the device), how attention's keys are cut, and the order of a handle's calls over
such a cache, with the host engine compiled against a logging stand-in for the HIP
runtime and the launchers."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2412_18934_amd import dv
from tests.test_engine_cpu import CSRC, HERE, ROOT, STREAM, Engine

A = 1 << 20  # an aligned address that is never used


def cache(**kw):
    f = dict(k=A, v=A, scale=A, k_tail=A, v_tail=A, n_layers=2, n_heads=4, head_dim=64, format=dv.DV_I8, capacity=256, len=40)
    f.update(kw)
    return dv.dv_kvq(*[f[name] for name, _ in dv.dv_kvq._fields_])


def test_the_struct_follows_the_header():
    from tests.test_abi_cpu import _header_fields
    assert [f[0] for f in dv.dv_kvq._fields_] == _header_fields("dv_kvq")


BAD = [dict(k=None), dict(v=None), dict(scale=None), dict(k_tail=None), dict(v_tail=None), dict(k=A + 8), dict(v=A + 1),
       dict(scale=A + 4), dict(k_tail=A + 2), dict(v_tail=A + 8), dict(n_layers=0), dict(n_heads=0), dict(n_heads=65536),
       dict(head_dim=96), dict(format=dv.DV_BF16), dict(format=4), dict(capacity=0), dict(capacity=100), dict(capacity=-32),
       dict(len=-1), dict(len=257), dict(n_layers=1 << 20, n_heads=1 << 10),
       dict(n_layers=1 << 12, n_heads=1 << 9, capacity=1 << 12)]


@pytest.mark.parametrize("bad", BAD, ids=[",".join("%s=%s" % p for p in b.items()) for b in BAD])
def test_bad_caches_are_refused_by_every_call(bad):
    c, kv = cache(**bad), dv.dv_kv(A, A, 256, 200)
    calls = [lambda: dv.dv_kvq_store(c, kv, 3), lambda: dv.dv_kvq_load(c, kv), lambda: dv.dv_kvq_advance(c, [0, 2]),
             lambda: dv.dv_kvq_attention_workspace(c, 4, 4),
             lambda: dv.dv_kvq_attention(c, 0, A, 256, 4, 4, None, A, 256, A, 1 << 40)]
    for call in calls:
        with pytest.raises(dv.DvError) as e:
            call()
        assert e.value.code == dv.DV_EINVAL and dv.dv_last_error(None)
    assert c.len == bad.get("len", 40) and kv.len == 200


@pytest.mark.parametrize("kv,n,code", [
    (dv.dv_kv(0, A, 256, 200), 3, dv.DV_EINVAL), (dv.dv_kv(A, A + 4, 256, 200), 3, dv.DV_EINVAL),
    (dv.dv_kv(A, A, 250, 200), 3, dv.DV_EINVAL), (dv.dv_kv(A, A, 256, 300), 3, dv.DV_EINVAL),
    (dv.dv_kv(A, A, 256, 200), 0, dv.DV_EINVAL), (dv.dv_kv(A, A, 256, 200), -1, dv.DV_EINVAL),
    (dv.dv_kv(A, A, 256, 42), 3, dv.DV_EINVAL),                       # not that many rows there
    (dv.dv_kv(A, A, 256, 200), 2 ** 31 - 1, dv.DV_EINVAL),
    (dv.dv_kv(A, A, 512, 400), 217, dv.DV_ECAPACITY)])
def test_store_refusals(kv, n, code):
    c = cache()
    with pytest.raises(dv.DvError) as e:
        dv.dv_kvq_store(c, kv, n)
    assert e.value.code == code and c.len == 40


def test_load_refusals():
    for kv, code in ((dv.dv_kv(A, 0, 256, 0), dv.DV_EINVAL), (dv.dv_kv(A + 2, A, 256, 0), dv.DV_EINVAL),
                     (dv.dv_kv(A, A, 48, 0), dv.DV_EINVAL), (dv.dv_kv(A, A, 32, 7), dv.DV_ECAPACITY)):
        with pytest.raises(dv.DvError) as e:
            dv.dv_kvq_load(cache(), kv)
        assert e.value.code == code
    assert kv.len == 7
    assert dv.lib().dv_kvq_load(cache(), None, None) == dv.DV_EINVAL


@pytest.mark.parametrize("path", [[], [1, 1], [2, 1], [-1], [0, 64], list(range(65))])
def test_advance_refusals(path):
    c = cache()
    with pytest.raises(dv.DvError) as e:
        dv.dv_kvq_advance(c, path)
    assert e.value.code == dv.DV_EINVAL and c.len == 40
    assert dv.lib().dv_kvq_advance(c, None, 3, None) == dv.DV_EINVAL
    c = cache(len=250)
    with pytest.raises(dv.DvError) as e:
        dv.dv_kvq_advance(c, list(range(7)))
    assert e.value.code == dv.DV_ECAPACITY and c.len == 250


@pytest.mark.parametrize("kw,code", [
    (dict(layer=-1), -1), (dict(layer=2), -1), (dict(q=0), -1), (dict(out=0), -1), (dict(n=0), -1), (dict(n=65), -1),
    (dict(n_heads=0), -1), (dict(n_heads=6), -1), (dict(n_heads=65540), -1), (dict(q=A + 4), -1), (dict(out=A + 8), -1),
    (dict(q_stride=255), -1), (dict(q_stride=258), -1), (dict(out_stride=-256), -1), (dict(out_stride=1 << 50), -1),
    (dict(n_heads=8), -1), (dict(n_heads=4100, q_stride=4100 * 64, out_stride=4100 * 64), -1), (dict(len=250, n=7), dv.DV_ECAPACITY)])
def test_attention_refusals(kw, code):
    a = dict(layer=1, q=A, q_stride=256, n=4, n_heads=4, out=A, out_stride=256, len=40)
    a.update(kw)
    with pytest.raises(dv.DvError) as e:
        dv.dv_kvq_attention(cache(len=a["len"]), a["layer"], a["q"], a["q_stride"], a["n"], a["n_heads"], None, a["out"],
                            a["out_stride"], A, 1 << 40)
    assert e.value.code == code
    if "n" in kw or "n_heads" in kw and kw["n_heads"] != 8:
        if code == dv.DV_EINVAL:
            with pytest.raises(dv.DvError):
                dv.dv_kvq_attention_workspace(cache(), a["n"], a["n_heads"])


def test_attention_in_place_needs_one_stride():
    with pytest.raises(dv.DvError) as e:
        dv.dv_kvq_attention(cache(), 1, A, 512, 4, 4, None, A, 256, A, 1 << 40)
    assert e.value.code == dv.DV_EINVAL and "stride" in str(e.value)


def test_handle_calls_refuse_a_null_handle():
    acc = dv.dv_accept()
    for call in (lambda: dv.dv_verify_step_kvq(None, [0], [-1], cache()), lambda: dv.dv_prefill_kvq(None, [0], cache()),
                 lambda: dv.dv_verify_step_kvq_sampled(None, [0], [-1], cache(), A, 1.0, [0.5], [0.5]),
                 lambda: dv.dv_kvq_commit(None, cache(), acc)):
        with pytest.raises(dv.DvError) as e:
            call()
        assert e.value.code == dv.DV_EINVAL


# ---------------------------------------------------------------------------
# the cut, and the handle's calls

STUB = r"""
#include <cstdio>
#include <string>
#include "dv_kvq.h"
static std::string g_said;
static hipError_t say(const char *what, hipStream_t s, int a, int b, int c)
{
    char t[96];
    std::snprintf(t, sizeof t, "%s %zx %d %d %d\n", what, (size_t)s, a, b, c);
    g_said += t;
    return hipSuccess;
}
hipError_t launch_kvq_store(const KvqLayers &c, const KvqRows &r, int n, hipStream_t s) { return say("store", s, c.len, n, r.cap); }
hipError_t launch_kvq_load(const KvqLayers &c, const KvqRows &r, hipStream_t s) { return say("load", s, c.len, c.L, r.cap); }
hipError_t launch_kvq_advance(const KvqLayers &c, const int32_t *path, int n, hipStream_t s) { return say("advance", s, c.len, n, path[n - 1]); }
hipError_t launch_kvq_attention(const KvqAttnArgs &a, int, int, const KvqCut &, hipStream_t s) { return say("attend", s, a.blocks, a.r, a.n); }
extern "C" const char *kvq_said() { return g_said.c_str(); }
extern "C" void kvq_hush() { g_said.clear(); }
extern "C" void kvq_cut_of(int heads, int rows, int tiles, int n_cu, int *out)
{
    const KvqCut c = kvq_cut(heads, rows, tiles, n_cu);
    out[0] = c.rt, out[1] = c.z, out[2] = c.n_split, out[3] = kvq_max_split(heads, rows, n_cu);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("kvq")
    stub, out = str(d / "kvqstub.cpp"), str(d / "libkvq.so")
    with open(stub, "w") as f:
        f.write(STUB)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__",
                    "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    os.path.join(CSRC, "dv_engine.cpp"), os.path.join(CSRC, "dv_kvq.cpp"),
                    os.path.join(HERE, "hipstub.cpp"), stub, "-o", out], check=True)
    L = ctypes.CDLL(out)
    L.stub_log.restype = L.kvq_said.restype = L.dv_last_error.restype = ctypes.c_char_p
    L.stub_reset.argtypes = [ctypes.c_size_t]
    L.stub_live.restype = ctypes.c_size_t
    L.dv_last_error.argtypes = [ctypes.c_void_p]
    return L


@pytest.mark.parametrize("n_cu", [256, 64])
def test_every_row_and_every_share_has_work(lib, n_cu):
    out = (ctypes.c_int * 4)()
    for heads in (1, 3, 8, 40, 300):
        for rows in (1, 16, 17, 33, 64, 65, 512):
            for tiles in (1, 2, 3, 5, 8, 24, 25, 32, 35, 257, 4100):
                lib.kvq_cut_of(heads, rows, tiles, n_cu, out)
                rt, z, n_split, most = out
                assert 16 * rt * z >= rows > 16 * rt * (z - 1)
                assert 1 <= n_split <= min(most, (tiles + 7) // 8)    # dealt in groups of 8 tiles


class KvqEngine(Engine):
    def __init__(self, lib, dtype, **kw):
        super().__init__(lib, dtype, **kw)
        self.c = cache(n_layers=2, n_heads=4, head_dim=64, capacity=4096, len=0)

    def said(self):
        rows = [r.split() for r in self.lib.kvq_said().decode().splitlines()]
        self.lib.kvq_hush()
        assert all(int(r[1], 16) == STREAM for r in rows)
        return [(r[0], *map(int, r[2:])) for r in rows]

    def prefill_kvq(self, n, fail_at=2 ** 64 - 1):
        self.lib.kvq_hush()
        self.lib.stub_reset(fail_at)
        toks = np.zeros(n, np.int32)
        return self.lib.dv_prefill_kvq(self.h, dv._ptr(toks), n, ctypes.byref(self.c), None)


@pytest.fixture(params=[dv.DV_BF16, dv.DV_I8], ids=["bf16", "i8"])
def engine(request, lib):
    e = KvqEngine(lib, request.param)
    yield e
    e.close()
    assert lib.stub_live() == 0


def test_a_prompt_reads_back_extends_and_stores_every_layer(engine):
    assert engine.prefill_kvq(1100) == 0 and engine.c.len == 1100
    assert engine.said() == 2 * [("load", 0, 1, 1120), ("store", 0, 1024, 1120)] + 2 * [
        ("load", 1024, 1, 1120), ("store", 1024, 76, 1120)]
    # in the order read back, QKV, attention, store
    names = [w for w, _, _ in engine.log()]
    assert names.count("causal") == 4 and names.count("attention") == 0
    # the rows are kept for the next prompt that fits
    live = engine.lib.stub_live()
    engine.c.len = 37
    assert engine.prefill_kvq(300) == 0 and engine.c.len == 337 and engine.lib.stub_live() == live
    assert engine.said() == 2 * [("load", 37, 1, 352), ("store", 37, 300, 352)]


def test_short_prompts_and_those_without_room_run_as_chains(engine):
    engine.c.len = 30
    assert engine.prefill_kvq(5) == 0 and engine.c.len == 35
    assert engine.said() == [("attend", 0, 30, 5)] * 2 + [("advance", 30, 5, 4)]
    live = engine.lib.stub_live()
    assert engine.prefill_kvq(300, fail_at=1 << 16) == 0 and engine.c.len == 335
    said = engine.said()
    assert [s for s in said if s[0] not in ("attend", "advance")] == []
    assert [s[1:3] for s in said if s[0] == "advance"][:2] == [(35, 8), (43, 8)]
    assert engine.lib.stub_live() == live
    # room for the pass but not for the rows: chains too (the pass's workspace is kept)
    engine.c.len = 0
    assert engine.prefill_kvq(300) == 0
    engine.lib.kvq_hush()
    engine.c.len = 3000
    assert engine.prefill_kvq(300, fail_at=1 << 16) == 0 and engine.c.len == 3300
    assert {s[0] for s in engine.said()} == {"attend", "advance"}


def test_step_and_commit(engine):
    lib, c = engine.lib, engine.c
    c.len = 61
    lib.kvq_hush()
    t, p = np.zeros(4, np.int32), np.array([-1, 0, 0, 2], np.int32)
    acc, kv = dv.dv_accept(), dv.dv_kv(A, A, 4096, 61)
    assert lib.dv_verify_step_kvq(engine.h, dv._ptr(t), dv._ptr(p), 4, ctypes.byref(c), None, ctypes.byref(acc)) == 0
    assert engine.said() == [("attend", 1, 29, 4)] * 2 and c.len == 61 and acc.base_len == 61
    acc.accept_len = 3
    acc.path[0], acc.path[1], acc.path[2] = 0, 2, 3
    # not the other kind's commit, not another cache's
    assert lib.dv_kv_commit(engine.h, ctypes.byref(kv), ctypes.byref(acc)) == dv.DV_ESTATE
    other = cache(capacity=4096, len=61, k=2 * A)
    assert lib.dv_kvq_commit(engine.h, ctypes.byref(other), ctypes.byref(acc)) == dv.DV_ESTATE
    acc.path[1] = 1
    assert lib.dv_kvq_commit(engine.h, ctypes.byref(c), ctypes.byref(acc)) == dv.DV_EINVAL and c.len == 61
    acc.path[1] = 2
    assert lib.dv_kvq_commit(engine.h, ctypes.byref(c), None) == dv.DV_EINVAL
    assert lib.dv_kvq_commit(engine.h, ctypes.byref(c), ctypes.byref(acc)) == 0
    assert c.len == 64 and engine.said() == [("advance", 61, 3, 3)]
    assert lib.dv_kvq_commit(engine.h, ctypes.byref(c), ctypes.byref(acc)) == dv.DV_ESTATE
    # a plain step is not committed as one of this kind
    assert lib.dv_verify_step(engine.h, dv._ptr(t), dv._ptr(p), 4, ctypes.byref(kv), None, ctypes.byref(acc)) == 0
    acc.accept_len, acc.path[0] = 1, 0
    c.len = 61
    assert lib.dv_kvq_commit(engine.h, ctypes.byref(c), ctypes.byref(acc)) == dv.DV_ESTATE


def test_handle_refusals(lib):
    t, p, acc = np.zeros(4, np.int32), np.array([-1, 0, 1, 2], np.int32), dv.dv_accept()
    e = KvqEngine(lib, dv.DV_BF16)
    try:
        def step(c, n=4):
            return lib.dv_verify_step_kvq(e.h, dv._ptr(t), dv._ptr(p), n, ctypes.byref(c), None, ctypes.byref(acc))
        for bad in BAD[:20]:
            assert step(cache(**{**dict(capacity=256), **bad})) == dv.DV_EINVAL
            assert lib.dv_prefill_kvq(e.h, dv._ptr(t), 4, ctypes.byref(cache(**bad)), None) == dv.DV_EINVAL
        for other in (dict(n_layers=3), dict(n_heads=8), dict(head_dim=128)):
            assert step(cache(**other)) == dv.DV_EINVAL and b"not this model" in lib.dv_last_error(e.h)
        assert step(cache(capacity=64, len=61)) == dv.DV_ECAPACITY
        assert lib.dv_prefill_kvq(e.h, dv._ptr(t), 4, ctypes.byref(cache(capacity=64, len=61)), None) == dv.DV_ECAPACITY
        assert step(cache(), 0) == dv.DV_EINVAL
        t[2] = 5000
        assert step(cache()) == dv.DV_EINVAL
        t[2] = 0
        assert step(cache()) == 0
    finally:
        e.close()
    e = KvqEngine(lib, dv.DV_F32)
    try:
        assert lib.dv_verify_step_kvq(e.h, dv._ptr(t), dv._ptr(p), 4, ctypes.byref(cache()), None, ctypes.byref(acc)) == dv.DV_EINVAL
        assert lib.dv_prefill_kvq(e.h, dv._ptr(t), 4, ctypes.byref(cache()), None) == dv.DV_EINVAL
    finally:
        e.close()


def test_a_growing_conversation_seldom_allocates(engine):
    """The layer of bf16 rows is made for twice the prompt, as far as the cache goes: turns
    behind it fit, and it grows a few times at most, not with every turn."""
    def rows_made(n, fail_at=2 ** 64 - 1):
        assert engine.prefill_kvq(n, fail_at) == 0
        return [size for what, _, size in engine.log() if what == "malloc"]

    slot = 2 * 4 * 64 * 2                              # K and V of 4 heads of 64
    assert rows_made(300)[-1] == 640 * slot
    for _ in range(3):
        assert rows_made(100) == []                    # 600 slots
    assert rows_made(100) == [1408 * slot]
    made = 0
    while engine.c.len < 4000:
        made += len(rows_made(100))
    assert made <= 2 and engine.c.len == 4000
    # no room for twice: as much as the prompt needs, and nothing of the failure is left
    engine.c.len = 0
    other = KvqEngine(engine.lib, dv.DV_BF16)
    try:
        assert other.prefill_kvq(200) == 0             # (the pass's own workspace is there from here on)
        other.c.len = 1200
        assert other.prefill_kvq(200, fail_at=2000 * slot) == 0
        assert [size for what, _, size in other.log() if what == "malloc"][-2:] == [2816 * slot, 1408 * slot]
        assert other.log()[-1][0] == "sync" and "causal" in [what for what, _, _ in other.log()]
    finally:
        other.close()


def test_a_commit_takes_the_step_s_own_cache(engine):
    """Caches may share blocks and differ in their tails, where a step's rows are; nor may
    the shape that the rows were written with change."""
    lib, c = engine.lib, engine.c
    c.len = 61
    t, p, acc = np.zeros(4, np.int32), np.array([-1, 0, 0, 2], np.int32), dv.dv_accept()
    assert lib.dv_verify_step_kvq(engine.h, dv._ptr(t), dv._ptr(p), 4, ctypes.byref(c), None, ctypes.byref(acc)) == 0
    acc.accept_len, acc.path[0], acc.path[1] = 2, 0, 2
    lib.kvq_hush()
    for other in (dict(k_tail=2 * A), dict(v_tail=2 * A), dict(scale=2 * A), dict(capacity=2048), dict(format=dv.DV_F8)):
        o = cache(**{**dict(capacity=4096, len=61), **other})
        assert lib.dv_kvq_commit(engine.h, ctypes.byref(o), ctypes.byref(acc)) == dv.DV_ESTATE and o.len == 61
    assert engine.said() == []
    # another struct of the same cache is the same cache
    o = cache(capacity=4096, len=61)
    assert lib.dv_kvq_commit(engine.h, ctypes.byref(o), ctypes.byref(acc)) == 0 and o.len == 63
    assert engine.said() == [("advance", 61, 2, 2)]
