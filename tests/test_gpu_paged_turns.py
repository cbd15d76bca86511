"""Turns of a part of the head where rows are few, and new rows' positions after an eviction.  Tolerances are those of
test_gpu_paged."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from tests.test_gpu_paged import Case, _check_append, _check_attention, _check_evict, _check_mass, _rope  # noqa: E402


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd,rot,interleaved,scaling,magnitude", [
    (64, 62, 0, 0, 1.0), (64, 6, 0, 0, 1.0), (64, 2, 0, 1, 1.0), (64, 2, 1, 1, 0.5), (64, 48, 0, 2, 1.0), (128, 96, 1, 2, 1.0),
    (128, 112, 0, 3, 1.2), (128, 30, 1, 0, 1.0), (128, 30, 0, 0, 1.0), (128, 100, 0, 0, 1.0), (128, 16, 0, 0, 1.0)])
@pytest.mark.parametrize("lens,counts", [([0, 31, 64, 5], [3, 2, 0, 1]), ([7, 40], [1, 1])], ids=["rows", "single"])
def test_few_rows_turned_in_part(dtype, hd, rot, interleaved, scaling, magnitude, lens, counts):
    """Halves that do not begin at a multiple of 8 among them."""
    c = Case(7, lens, counts, hd=hd, heads=3)
    _check_append(c, counts, 2, dtype, _rope(rot, interleaved, scaling, magnitude), pad=0 if max(counts) == 1 else 2,
                  start=max(counts) > 1)
    assert int(c.g.fault) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_behind_an_eviction_have_positions(dtype):
    """A sequence that was cut down: kept keys stay turned as they were, new rows are turned by the positions given
    with them and stand in the slots behind what stayed; attention is over both."""
    lens, counts, budget = [150, 60], [3, 2], 100
    c = Case(17, lens, counts, hd=64, heads=2)
    _check_evict(c, budget, 20, inplace=True)
    c.lens = [budget, 60]
    positions = [150, 151, 152, 60, 61]
    _check_append(c, counts, 2, dtype, _rope(64, 0, 0), positions=positions)
    k, v, m = c.got()
    new = np.zeros(m.shape, bool)
    for i, n in enumerate(counts):
        for p, at in c.o.places(c.pages[i], range(c.lens[i], c.lens[i] + n)):
            new[1, p, :, at] = True
    c.o.k[new], c.o.v[new], c.o.mass[new] = k[new], v[new], 0
    c.same()
    _check_attention(c, counts, 2, dtype, "tree")
    _check_mass(c, counts, 2, dtype, "tree")
