"""What of the int8 layers runs on the host: the refusals of he_i8_layer_create, in the order of the other plans', and the arithmetic of an
output (the functions that the kernels use) against Python integers, up to the longest sums and at the ends of every range."""
import ctypes

import numpy as np
import pytest

from paper_1908_04172_amd import he
from paper_1908_04172_amd import workloads as wl


@pytest.fixture(scope="module")
def ctx():
    return he.Context(10, wl.modulus_chain([30, 30], 1 << 10), device=None)


def status(ctx, n_in=2, n_out=1, n_pt=2, off=(0, 2), ct=(0, 1), pt=(0, 1), w=(1, -1), scale=None):
    arr = [np.asarray(a, np.uint32) for a in (off, ct, pt)]
    weights = None if w is None else np.asarray(w, np.int8)
    channel = None if scale is None else np.asarray(scale, np.float64)
    h = ctypes.c_void_p(1)
    rc = he.lib().he_i8_layer_create(ctx._h if ctx else None, n_in, n_out, n_pt, *(a.ctypes.data for a in arr),
                                     None if weights is None else weights.ctypes.data, None if channel is None else channel.ctypes.data,
                                     1.0, ctypes.byref(h))
    assert h.value is None                                          # no layer from a refused call
    return rc


def test_refusals_of_the_arrays(ctx):
    assert status(ctx) == -5                                        # all is well but for the device
    assert status(None) == -1
    assert status(ctx, w=None) == -1
    assert status(ctx, off=(1, 2)) == -4
    assert status(ctx, n_out=2, off=(0, 2, 1)) == -4
    assert status(ctx, ct=(0, 2)) == -4
    assert status(ctx, pt=(2, 0)) == -4
    assert status(ctx, scale=[float("nan")]) == -1
    assert status(ctx, scale=[float("inf")]) == -1
    assert he.lib().he_i8_layer_create(ctx._h, 1, 1, 1, None, None, None, None, None, 1.0, None) == -1


def test_an_output_takes_131071_terms_and_no_more(ctx):
    for terms, want in ((131071, -5), (131072, -4)):
        z = np.zeros(terms, np.uint32)
        assert status(ctx, off=(0, terms), ct=z, pt=z) == want


def test_refusals_without_a_layer(ctx):
    assert he.lib().he_i8_layer_destroy(None) == -1
    b = ctypes.c_size_t()
    assert he.lib().he_i8_workspace_bytes(None, 1, 0, ctypes.byref(b)) == -1
    assert he.lib().he_ct_i8_mac(ctx._h, None, 1, None, None, None, None, 0, None, 0, None) == -1
    assert he.lib().he_ct_i8_mac32(None, None, 1, None, None, None, None, 0, None, 0, None) == -1


WIDTHS = [14, 16, 17, 20, 24, 25, 29, 30, 31, 32, 33, 39, 40, 41, 47, 48, 49, 50, 55, 56, 57, 58, 59, 60, 61, 62]


@pytest.mark.parametrize("bits", WIDTHS)
def test_an_output_equals_python_integers(bits):
    q = wl.ntt_primes(bits, 1 << 10, 1)[0]
    rng = np.random.default_rng(bits)
    edge = [0, 1, q - 1, q // 2, (1 << (bits - 1)) - 1]
    for case in range(60):
        n = int(rng.choice([0, 1, 2, 31, 200]))
        x = rng.integers(0, q, n, dtype=np.uint64)
        if case % 3 == 0 and n:
            x[:] = edge[case // 3 % 5]
        w = rng.integers(-128, 128, n)
        if case % 4 == 0:
            w[:] = [-128, 127][case // 4 % 2]
        s, tok, b = (int(rng.choice(edge + [int(rng.integers(0, q))] * 5)) for _ in range(3))
        total = sum(int(a) * int(c) for a, c in zip(x, w))
        assert he.host_i8_mac(x, w, q, s, tok, b) == (tok * s * total + b) % q
        if q < 1 << 30:
            assert he.host_i8_mac(x, w, q, s, tok, b, packed=True) == (tok * s * total + b) % q


@pytest.mark.parametrize("bits", [14, 30, 40, 50, 59, 60, 61, 62])
def test_the_longest_sums_of_one_output(bits):
    q, n = wl.ntt_primes(bits, 1 << 10, 1)[0], 131071
    for x in (0, q - 1, (1 << (bits - 1)) - 1):
        for w in (-128, 127):
            for s in (1, q - 1, q // 3):
                want = (q - 2) * (s * n * x * w) % q
                assert he.host_i8_mac(np.full(n, x, np.uint64), np.full(n, w), q, s, q - 2) == want
                if q < 1 << 30:
                    assert he.host_i8_mac(np.full(n, x, np.uint64), np.full(n, w), q, s, q - 2, packed=True) == want


def test_kernels_stay_within_their_registers():
    """What does not fit is fetched back in the middle of a loop; a few values around it are no harm."""
    from test_kernel_registers import kernels, matching
    built = kernels()
    for pattern, registers, spilled in ((r"i8_split_kernel", 256, 0), (r"i8_whole_kernel", 256, 8), (r"sample_kernel", 128, 64)):
        for name, k in matching(built, pattern).items():
            assert k[".vgpr_count"] <= registers and k[".vgpr_spill_count"] <= spilled, (name, k[".vgpr_count"], k[".vgpr_spill_count"])
