"""A bf16 dv_kv in pages: the rows that a prompt left in the single-sequence cache, taken into pages by plain copies, are
the paged cache's rows, and go back the same way.  Tolerances are those of test_gpu_paged."""
import numpy as np
import pytest

import synth
from oracle import verify as ov
from tests.helpers import GpuCase, small_cfg

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2412_18934_amd import dv  # noqa: E402
from tests.test_gpu_paged import Case, _check_attention, _check_mass  # noqa: E402

CAPACITY, LENGTH = 384, 300


@pytest.fixture(scope="module")
def prompt_kv():
    case = GpuCase(small_cfg(n_layers=2, d_model=256, n_heads=2, head_dim=128, d_ffn=512, vocab=2048, weight_dtype="bf16",
                             init_std=0.09), seed=301, capacity=CAPACITY)
    kv = case.new_kv()
    dv.dv_prefill(case.h, synth.prompt(302, LENGTH, case.cfg.vocab), kv.c)
    torch.cuda.synchronize()
    yield case, kv
    case.close()


@pytest.mark.parametrize("page", [32, 96, 128, 384])
def test_a_prompt_in_pages(prompt_kv, page):
    case, kv = prompt_kv
    c = Case(page, [LENGTH, 40], [CAPACITY - LENGTH, 4], heads=2, hd=128, page=page, layers=2)
    tiles = page // 32
    for i, p in enumerate(c.pages[0]):
        c.g.k[:, p] = kv.k[:, :, i * page:(i + 1) * page]
        c.g.v[:, p] = kv.v[:, :, i * tiles:(i + 1) * tiles]
        for layer in range(2):
            k, v = (ov.bf16_to_f64(x) for x in kv.layer_host(layer, CAPACITY))
            c.o.k[layer, p], c.o.v[layer, p] = k[:, i * page:(i + 1) * page], v[:, i * page:(i + 1) * page]
    c.same()
    assert np.abs(c.o.k[:, c.pages[0][0]]).max() > 0.1
    back = case.new_kv(fill=float("nan"))
    for i, p in enumerate(c.pages[0]):
        back.k[:, :, i * page:(i + 1) * page] = c.g.k[:, p]
        back.v[:, :, i * tiles:(i + 1) * tiles] = c.g.v[:, p]
    assert torch.equal(back.k, kv.k) and torch.equal(back.v, kv.v)
    c.put_new(1, [5, 4])
    _check_attention(c, [5, 4], 1, "bf16", "tree")
    _check_attention(c, [5, 4], 2, "f32", "tree", max_len=5000)
    _check_mass(c, [5, 4], 2, "f32", "tree")
