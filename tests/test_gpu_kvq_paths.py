"""The handle's paths over the 8-bit cache where they take other kernels than on short
caches: steps whose keys are cut into shares (their partial sums lie in the handle's
workspace and the combining launch writes the O projection's operand), 32 rows to a
workgroup, and prompts of several chunks, row by row.  And calls on different caches at
once, from different threads and streams."""
import threading

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
from tests.test_gpu_kvq import _oracle_kv  # noqa: E402

DEV = "cuda:0"


def _filled(rng, n_layers, heads, hd, cap, fmt, length):
    """A cache of random codes; a block's largest number is about 4."""
    g = D.DeviceKVQ(n_layers, heads, hd, cap, fmt)
    for t in (g.k, g.v):
        z = rng.normal(0, (127 if fmt == "i8" else 448) / 4, t.shape)
        codes = np.rint(z.clip(-127, 127)).astype(np.int8) if fmt == "i8" else ok.e4m3_code(z.clip(-448, 448)).view(np.int8)
        t.copy_(torch.from_numpy(codes))
    g.scale.copy_(torch.from_numpy(np.exp(rng.normal(0, 0.2, g.scale.shape)) * 4 / ok.TOP[fmt]))
    for t in (g.k_tail, g.v_tail):
        t.copy_(torch.from_numpy(rng.normal(0, 1, t.shape)))
    # rows behind the committed ones hold anything
    r = length % 32
    g.k_tail[:, :, r:] = float("nan")
    s = torch.arange(r, 96, device=DEV)
    g.v_tail[:, :, s // 32, :, s % 32] = float("nan")
    g.c.len = length
    return g


def _step(case, om, g, rng, n, heads, vocab):
    """One step against the oracle's on the cache's own bytes, the bf16 cache's bar."""
    toks, par = synth.random_tree(int(rng.integers(1 << 30)), n, 8, vocab)
    kv_o = _oracle_kv(g, case.cfg.n_layers, heads)
    logits = torch.full((n, vocab), float("nan"), device=DEV)
    acc = dv.dv_verify_step_kvq(case.h, toks, par, g.c, logits.data_ptr())
    torch.cuda.synchronize()
    ref = ov.verify_step(om, kv_o, toks, par)
    ref["tokens"], ref["parents"] = np.asarray(toks), np.asarray(par)
    err, _ = compare_step(acc, logits.cpu().numpy(), ref, 2e-2)
    return toks, par, kv_o, ref, err


@pytest.mark.parametrize("weights,fmt,d,heads", [("bf16", "i8", 256, 4), ("i8", "f8", 512, 4), ("bf16", "f8", 256, 4)])
def test_steps_over_several_shares(weights, fmt, d, heads):
    """More than 24 tiles; trees of the half layout, with padding rows and with all 64, and
    a wide one after a narrow one (whose padding must be zeros again)."""
    cfg = small_cfg(n_layers=2, d_model=d, n_heads=heads, head_dim=d // heads, d_ffn=2 * d, vocab=512, weight_dtype=weights,
                    init_std=0.05)
    case = GpuCase(cfg, seed=31, capacity=2048)
    try:
        om, rng = case.w.oracle(), np.random.default_rng(32)
        for length in (1037, 1951):
            g = _filled(rng, 2, heads, d // heads, 2048, fmt, length)
            for n in (1, 5, 8, 9, 17, 33, 64, 48, 3):
                toks, par, kv_o, ref, err = _step(case, om, g, rng, n, heads, 512)
                print("[kvq] %s/%s len %d n %d: logits off by %.2g" % (weights, fmt, length, n, err), flush=True)
            # the bar sees the cache: with its last 64 slots at 0 the logits are elsewhere
            rest = (np.arange(length) < length - 64)[None, :, None]
            gone = [(np.where(rest, k, 0), np.where(rest, v, 0)) for k, v in kv_o]
            assert np.abs(ov.verify_step(om, gone, toks, par)["logits"] - ref["logits"]).max() > 4e-2
    finally:
        case.close()


@pytest.mark.parametrize("fmt", ["i8", "f8"])
def test_a_wide_step_over_a_long_cache(fmt):
    """32 rows a workgroup, several shares, two row groups."""
    heads, hd, cap, length = 32, 64, 6400, 6301
    cfg = small_cfg(n_layers=1, d_model=heads * hd, n_heads=heads, head_dim=hd, d_ffn=512, vocab=256, weight_dtype="bf16",
                    init_std=0.02)
    case = GpuCase(cfg, seed=33, capacity=cap)
    try:
        om, rng = case.w.oracle(), np.random.default_rng(34)
        g = _filled(rng, 1, heads, hd, cap, fmt, length)
        for n in (64, 50):
            err = _step(case, om, g, rng, n, heads, 256)[-1]
            print("[kvq] %s 32 heads, len %d n %d: logits off by %.2g" % (fmt, length, n, err), flush=True)
    finally:
        case.close()


def _same(a, b):
    """Two caches of the same len: every code and scale of whole blocks, every committed tail row."""
    assert a.len == b.len
    blocks, r = a.len // 32, a.len % 32
    for x, y in ((a.k, b.k), (a.v, b.v), (a.scale, b.scale)):
        assert torch.equal(x[:, :, :blocks], y[:, :, :blocks])
    assert torch.equal(a.k_tail[:, :, :r], b.k_tail[:, :, :r])
    assert torch.equal(a.v_tail[:, :, 0, :, :r], b.v_tail[:, :, 0, :, :r])


@pytest.mark.parametrize("weights,fmt,d,heads,max_tree", [("bf16", "i8", 256, 4, 16), ("bf16", "f8", 512, 4, 64),
                                                         ("i8", "i8", 512, 4, 8)])
def test_prompts_are_read_back_plain_prompt_and_store(weights, fmt, d, heads, max_tree):
    """dv_prefill_kvq's own words, chunk by chunk, by the calls that it is made of: read
    the cache back, run the plain prompt behind it, append the new rows.  The same
    kernels on the same numbers: codes, scales, tails and the next token are equal."""
    hd, cap = d // heads, 2304
    cfg = small_cfg(n_layers=3, d_model=d, n_heads=heads, head_dim=hd, d_ffn=2 * d, vocab=512, weight_dtype=weights, init_std=0.05)
    case = GpuCase(cfg, seed=35, capacity=cap, max_tree=max_tree)
    try:
        rng = np.random.default_rng(36)
        a, b = D.DeviceKVQ(3, heads, hd, cap, fmt), D.DeviceKVQ(3, heads, hd, cap, fmt)
        for g in (a, b):
            for t in (g.scale, g.k_tail, g.v_tail):
                t.fill_(float("nan"))
        for n in (1100, 70, 97, 900):                 # (int8: each more than four chains, all on the causal pass)
            prompt = rng.integers(0, 512, n)
            nxt = dv.dv_prefill_kvq(case.h, prompt, a.c)
            for at in range(0, n, 1024):
                part = prompt[at:at + 1024]
                kv = case.new_kv(fill=float("nan"))
                dv.dv_kvq_load(b.c, kv.c)
                plain = dv.dv_prefill(case.h, part, kv.c)
                dv.dv_kvq_store(b.c, kv.c, len(part))
            torch.cuda.synchronize()
            assert nxt == plain
            _same(a, b)
    finally:
        case.close()


def test_different_caches_at_once():
    """Two threads with a cache, a stream and a workspace each: what either gives alone."""
    heads, hd, cap, n = 8, 128, 2048, 6
    rng = np.random.default_rng(37)
    q = torch.randn((n, 2 * heads * hd), device=DEV)
    rows = [(torch.randn((2, heads, cap, hd), device=DEV).bfloat16(), torch.randn((2, heads, cap // 32, hd, 32), device=DEV).bfloat16())
            for _ in range(2)]
    plans = [[int(x) for x in rng.integers(1, 150, 12)] for _ in range(2)]

    def run(i, out):
        g = D.DeviceKVQ(2, heads, hd, cap, "i8" if i == 0 else "f8")
        kv = dv.dv_kv(rows[i][0].data_ptr(), rows[i][1].data_ptr(), cap, cap)
        need = dv.dv_kvq_attention_workspace(g.c, n, 2 * heads)
        ws, stream = torch.empty(need, dtype=torch.uint8, device=DEV), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            s = stream.cuda_stream
            for more in plans[i]:
                dv.dv_kvq_store(g.c, kv, more, s)
                t = torch.empty_like(q)
                dv.dv_kvq_advance(g.c, [0, 2, 3], s)  # (the tail's rows, whatever they are: zeros at first)
                g.set_new(1, rows[i][0][1, :, :n].transpose(0, 1), rows[i][0][1, :, n:2 * n].transpose(0, 1))
                dv.dv_kvq_attention(g.c, 1, q.data_ptr(), q.stride(0), n, 2 * heads, None, t.data_ptr(), t.stride(0),
                                    ws.data_ptr(), need, s)
                out.append(t)
            out += [g.k, g.v, g.scale]
        stream.synchronize()

    alone = [[], []]
    for i in range(2):
        run(i, alone[i])
    for _ in range(3):
        both, errors = [[], []], []

        def guarded(i):
            try:
                run(i, both[i])
            except Exception as e:                    # noqa: BLE001 (reported below)
                errors.append(e)

        threads = [threading.Thread(target=guarded, args=(i,)) for i in range(2)]
        for t in threads:
            t.start()
        for t in threads:
            t.join(60)
        torch.cuda.synchronize()
        assert not errors, errors
        for i in range(2):
            assert len(both[i]) == len(alone[i])
            for x, y in zip(alone[i], both[i]):
                assert torch.equal(x.view(torch.int8), y.view(torch.int8))
                assert x.dtype != torch.float32 or x is alone[i][-1] or torch.isfinite(x).all()
