"""Paged attention and mass with caps at the ends of their range: caps that never bind, and caps of next to nothing.
Tolerances are those of test_gpu_paged."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from tests.test_gpu_paged import Case, _check_attention, _check_mass, _queries  # noqa: E402


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cap,scale,std", [(3e38, 0.0, 1.3), (3e38, 1e-4, 500.0), (3e38, 1e-20, 3e18), (3e38, 1e-37, 3e35), (1e30, 1e-12, 3e9), (1e10, 0.0, 1.0), (1e-38, 0.0, 1.0),
                                           (1e-40, 0.5, 1.0)])
def test_caps_at_the_ends(dtype, cap, scale, std):
    """scale / cap is no number of 32 bits there: less than the smallest, or larger than all."""
    lens, counts = [100, 7, 0], [4, 9, 3]
    cap = float(np.float32(cap))
    c = Case(11, lens, counts, hd=128)
    c.put_new(1, counts)
    _check_attention(c, counts, 2, dtype, "any", cap=cap, scale=float(np.float32(scale)), std=std)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cap", [3e38, 1e-40])
def test_mass_at_the_ends(dtype, cap):
    lens, counts = [100, 7], [4, 9]
    c = Case(12, lens, counts, hd=128)
    c.put_new(1, counts)
    _check_mass(c, counts, 2, dtype, "tree", cap=float(np.float32(cap)))


@pytest.mark.parametrize("cap", [1e-40, 1e-44])
def test_queries_of_nothing_under_a_cap_of_next_to_nothing(cap):
    """Scores of 0 stay 0."""
    lens, counts = [100, 7], [4, 9]
    c = Case(13, lens, counts, hd=64)
    c.put_new(1, counts)
    x, q = _queries(c, c.rng, counts, 1, "f32", 0, 0)
    x[:], q[:] = 0, 0
    _check_attention(c, counts, 1, "f32", "tree", cap=float(np.float32(cap)), queries=(x, q))
