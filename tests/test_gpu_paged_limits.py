"""Paged cache on the GPU with as many sequences and layers as its calls take, most of them empty.  Tolerances are
those of test_gpu_paged."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2412_18934_amd import dv  # noqa: E402
from tests.test_gpu_paged import DEV, Case, _check_append, _check_attention, _check_evict, _check_mass  # noqa: E402

SEQS, SOME = 65536, (0, 1, 40000, 65535)


def _case(seed, length, room, layers):
    lens, counts = [0] * SEQS, [0] * SEQS
    for i, s in enumerate(SOME):
        lens[s], counts[s] = length + i, room
    return Case(seed, lens, counts, heads=2, hd=64, page=32, layers=layers), lens, counts


def test_rows_of_many_sequences_in_many_layers():
    """More heads in all layers than a grid dimension's workgroups."""
    c, lens, counts = _case(1, 40, 2, 40)
    assert c.layers * c.heads * SEQS > 1 << 22
    _check_append(c, counts, 1, "bf16", None, layer=39, pad=1)
    c, lens, counts = _case(2, 40, 2, 40)
    c.put_new(39, counts)
    _check_attention(c, counts, 2, "f32", "tree", layer=39, pad=1)
    _check_mass(c, counts, 2, "f32", "tree", layer=39, pad=1)
    assert int(c.g.fault) == 0


@pytest.mark.parametrize("inplace", [False, True])
def test_commit_and_eviction_of_many_sequences_in_many_layers(inplace):
    c, lens, counts = _case(3, 40, 9, 40)
    for layer in (0, 39):
        c.put_new(layer, counts)
    c.o.mass[:] = np.float32(c.rng.random(c.o.mass.shape))
    c.upload()
    path, n = torch.zeros((SEQS, 3), dtype=torch.int32), torch.zeros(SEQS, dtype=torch.int32)
    for s in SOME:
        path[s], n[s] = torch.tensor([1, 4, 8]), 3
    path, n = path.to(DEV), n.to(DEV)
    new = c.g.lens if inplace else torch.full((SEQS,), -1, dtype=torch.int32, device=DEV)
    dv.dv_paged_commit(c.g.c, path.data_ptr(), 3, n.data_ptr(), new.data_ptr())
    for s in SOME:
        c.lens[s] = c.o.commit(c.pages[s], lens[s], [1, 4, 8])
    c.same()
    assert new.tolist() == c.lens
    c.g.lens.copy_(new)
    _check_evict(c, 20, 5, inplace=inplace)
