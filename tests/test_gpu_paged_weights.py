"""The weights with which bf16 rows read the pages keep 24 bits: values chosen so that they cancel to
nothing leave what the weights lost.

E = 2^-24.  Queries are 1 in one dim and 0 in the others, keys multiples of 1/8 there: scores are exact, multiples
of 1/64 within [-2, 2], and so are their differences x.  A weight exp(x) is off by 1.5 E |x| (the constant and the
product of its exponent) <= 6 E and 2 E of the function, a factor between tiles, waves or pieces by as much again;
its three parts are all of it.  The products are exact, their sums off by at most 4 numbers' roundings of 2 E W in
each of two products that count, W = sum w |v|, and by E W in two combinations.  In all (8 + 8 + 16 + 2) E W, and half a
step of the output, 2^-8 of it.  Weights of 16 bits are off by up to 128 E each."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from oracle.verify import round_to_bf16  # noqa: E402
from paper_2412_18934_amd import device as D  # noqa: E402
from paper_2412_18934_amd import dv  # noqa: E402

DEV, E = "cuda:0", 2.0 ** -24


def _bf(x):
    return round_to_bf16(np.float32(x)).astype(np.float64)


@pytest.mark.parametrize("max_len", [10, 5000])
@pytest.mark.parametrize("group", [1, 32])
@pytest.mark.parametrize("hd", [64, 128])
def test_values_that_cancel(hd, group, max_len):
    seqs, heads, page, length = 48, 4, 64, 300
    rng = np.random.default_rng(hd + group)
    g = D.DevicePaged(1, heads, hd, seqs * 5, page, seqs, 5)
    g.table.copy_(torch.arange(seqs * 5, dtype=torch.int32).reshape(seqs, 5))
    g.lens.fill_(length)
    k, v = rng.normal(0, 1, (seqs, heads, 5 * page, hd)), np.zeros((seqs, heads, 5 * page, hd))
    k[..., 0] = -1e30                                  # no weight
    want, W = np.zeros((seqs, heads, hd)), np.zeros((seqs, heads, hd))
    for s in range(seqs):
        for h in range(heads):
            at = rng.choice(length, 4, replace=False)
            k[s, h, at, 0] = rng.integers(-128, 129, 4) / 8
            z = k[s, h, at, 0] / 8
            w = np.exp(z - z.max())
            w /= w.sum()
            x = np.zeros((4, hd))
            x[0] = _bf(rng.normal(0, 1, hd))
            for j in (1, 2, 3):
                x[j] = -_bf(w[:j] @ x[:j] / w[j])
            v[s, h, at] = x
            want[s, h], W[s, h] = w @ x, w @ np.abs(x)
    k = torch.from_numpy(k).to(torch.bfloat16).reshape(seqs, heads, 5, page, hd).transpose(1, 2).reshape(-1, heads, page, hd)
    v = torch.from_numpy(v).to(torch.bfloat16).reshape(seqs, heads, 5, page // 32, 32, hd).transpose(1, 2)
    g.k[0].copy_(k)
    g.v[0].copy_(v.reshape(-1, heads, page // 32, 32, hd).transpose(3, 4))
    q = torch.zeros((seqs, heads * group, hd), dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 1
    out = torch.empty_like(q)
    # (the row's own slot: the last, of no weight)
    rows = g.rows(q, scale=0.125, max_len=max_len)
    ws = torch.empty(max(16, dv.dv_paged_attention_workspace(g.c, rows)), dtype=torch.uint8, device=DEV)
    dv.dv_paged_attention(g.c, 0, rows, out.data_ptr(), out.stride(0), 0, ws.data_ptr(), ws.numel(),
                          torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy().reshape(seqs, heads, group, hd)
    err = np.abs(got - want[:, :, None])
    over = err / (34 * E * W + 2.0 ** -8 * np.abs(want))[:, :, None]
    print("[paged] worst error / tolerance %.3g" % over.max(), flush=True)
    assert over.max() <= 1 and int(g.fault) == 0
