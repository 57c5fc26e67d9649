"""The forms in which layers of 8-bit integer weights are launched, each at a size that takes it."""
import numpy as np
import pytest

from paper_1908_04172_amd import workloads as wl

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def he():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1908_04172_amd import he as he_mod
    he_mod.lib()
    return he_mod


def test_as_many_workgroups_as_a_grid_holds(he):
    """Outputs without terms, each between two that have some, are groups of 2^14 workgroups here: 1023 of them fit the 2^32 threads
    of a grid, and 1024 are refused before anything is enqueued."""
    N = 1 << 15
    q = wl.modulus_chain([60] + [50] * 15, N)                       # 8 MiB a ciphertext
    ctx = he.Context(15, q)
    x = wl.uniform_residues_torch((1, 2), q, N, 3, "cuda")

    def layer(empty):
        n_out = 2 * empty - 1
        off = (np.arange(n_out + 1) // 2).astype(np.uint32)   # outputs 1, 3, 5, ... have the one term
        zeros = np.zeros(off[-1], np.uint32)
        return ctx.i8_layer(1, n_out, 1, off, zeros, zeros, np.ones(1, np.int8))

    out = torch.full((2047, 2, 16, N), -7, dtype=torch.int64, device="cuda")
    with pytest.raises(he.HeError) as e:
        ctx.ct_i8_mac(layer(1024), x, out=out)
    assert e.value.status == -4
    torch.cuda.synchronize()
    assert all(bool((out[k:k + 128] == -7).all()) for k in range(0, 2047, 128))
    ctx.ct_i8_mac(layer(1023), x, out=out[:2045])
    for k in range(0, 2045, 128):
        part = out[k:min(k + 128, 2045)]
        assert not bool(part[0::2].any()) and bool((part[1::2] == x).all())
    assert bool((out[2045:] == -7).all())
