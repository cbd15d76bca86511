"""Paged cache on the GPU with as many sequences and layers as its calls take, most of them empty.  Tolerances are
those of test_gpu_paged."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2412_18934_amd import device as D  # noqa: E402
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


def test_empty_sequences_between_two_rows():
    """Prompts of the first and of the last of 65536 sequences, whose rows meet inside a workgroup's: what the same call
    writes for sequences 0 and 1, in about its time (walked one by one the empty sequences cost 4.8 ms)."""
    page, n = 8192, (262144 + 16, 262144 + 16)
    g = D.DevicePaged(1, 1, 64, 66, page, SEQS, 33)
    x = torch.randn((sum(n), 3, 64), generator=torch.Generator(DEV).manual_seed(0), device=DEV).to(torch.bfloat16)
    q = x[:, :1]

    def call(last):
        g.k.zero_(), g.v.zero_()
        g.table.fill_(-1)
        g.table[0] = torch.arange(33, dtype=torch.int32)
        g.table[last] = torch.arange(33, 66, dtype=torch.int32)
        start = torch.full((SEQS + 1,), n[0], dtype=torch.int32, device=DEV)
        start[0] = 0
        start[last + 1:] = sum(n)
        rows = g.rows(q, start)
        rows.q = None
        times = []
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            dv.dv_paged_append(g.c, 0, rows, None, 0, x[:, 1:].data_ptr(), x.stride(0), x[:, 2:].data_ptr(), x.stride(0),
                               torch.cuda.current_stream().cuda_stream)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return g.k.clone(), g.v.clone(), min(times)

    (k, v, t), (k1, v1, t1) = call(SEQS - 1), call(1)
    print("[paged] %.3f ms, without the empty ones between %.3f" % (t, t1), flush=True)
    assert torch.equal(k, k1) and torch.equal(v, v1) and int(g.fault) == 0
    assert torch.equal(k[0, :33, 0].reshape(-1, 64)[:n[0]], x[:n[0], 1]) and torch.equal(k[0, 33:, 0].reshape(-1, 64)[:n[1]], x[n[0]:, 1])
    slots = v[0, :, 0].transpose(2, 3).reshape(66, page, 64)
    assert torch.equal(slots[:33].reshape(-1, 64)[:n[0]], x[:n[0], 2]) and torch.equal(slots[33:].reshape(-1, 64)[:n[1]], x[n[0]:, 2])
    assert t < 5 * t1
